"""kvprm_rotary on the GPU against the fp64 oracle.

Tolerance per value of a pair (a, b): the cosine and sine are off by at most pi 2^-24 from rounding
the rest of the angle (half a turn at most) to fp32, 2 units in the last place of the fp32 functions (2 *
2^-24 at most) and 2^-24 from the magnitude; each product and the sum round once more: 9.2 * 2^-24 (|a| +
|b|) m in all, 10 taken. Positions to 2^31 in 64 bits add 2 pi 2^31 * 0.16 * 2^-52 = 5 * 2^-23 at most: 20
there. A bf16 result adds half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

from oracle import growing_cache as gc

from gpu_common import kv

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16}
TRAINED = 4096.0


def _say(*a):
    print("case:", *a, flush=True)


def _near(got, x, want, m, dtype, units):
    """x: the rotated input pairs' |a| + |b| are bounded by the head's two largest values."""
    size = np.abs(x).max(axis=-1, keepdims=True) * 2
    tol = units * 2.0 ** -24 * m * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    err = np.abs(got - want)
    assert np.all(err <= tol), float(np.max(err - tol))


def _run(x, pos, rope, dtype, transpose=False, heads=None, out=None, stride=None):
    """One tensor [rows][heads][d] through the call, contiguous."""
    m = kv()
    rows, h, d = x.shape
    dst = torch.full_like(x, float("nan")) if out is None else out
    m.kvprm_rotary(rope, dtype, rows, pos.data_ptr(),
                   m.make_rope_heads([(x.data_ptr(), dst.data_ptr(), h, h * d, h * d)]), transpose,
                   torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return dst


def _inputs(rows, heads, d, dtype, far, seed=0):
    gen = torch.Generator().manual_seed(seed + 7 * rows + d)
    x = torch.randn((rows, heads, d), generator=gen).to(T[dtype])
    pos = torch.randint(-far, far, (rows,), generator=gen, dtype=torch.int32)
    return x, pos


CASES = [(layout, scaling, dtype, d, rot, rows)
         for layout in ("half", "interleaved") for dtype in ("f32", "bf16")
         for scaling, d, rot, rows in (("none", 128, 128, 17), ("linear", 64, 32, 1), ("base", 128, 128, 5),
                                       ("parts", 256, 256, 3), ("ramp", 128, 64, 65), ("none", 80, 40, 9),
                                       ("base", 6, 2, 33), ("none", 256, 2, 2))]


@pytest.mark.parametrize("layout,scaling,dtype,d,rot,rows", CASES)
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary(layout, scaling, dtype, d, rot, rows, transpose):
    _say(layout, scaling, dtype, d, rot, rows, transpose)
    m = 1.0 if scaling in ("none", "linear") else 1.375
    x, pos = _inputs(rows, 3, d, dtype, 100000)
    rope = kv().make_rope(d, rot, layout, 1e6, scaling, 4.0, TRAINED, 1.0, 32.0, m)
    got = _run(x.cuda(), pos.cuda(), rope, dtype, transpose).cpu().double().numpy()
    f = gc.frequencies(rot, 1e6, scaling, 4.0, TRAINED)
    want = gc.rotary(x.double().numpy(), pos.numpy(), f, layout, m, transpose)
    assert np.array_equal(got[..., rot:], x.double().numpy()[..., rot:])
    _near(got[..., :rot], x.double().numpy()[..., :rot], want[..., :rot], m, dtype, 10)


@pytest.mark.parametrize("rows,heads,dtype", [(5000, 5, "bf16"), (3001, 36, "f32"), (70000, 1, "bf16")])
def test_rotary_many_rows(rows, heads, dtype):
    """Several rows to a block, the last block short."""
    _say(rows, heads, dtype)
    x, pos = _inputs(rows, heads, 64, dtype, 1 << 20)
    got = _run(x.cuda(), pos.cuda(), kv().make_rope(64), dtype).cpu().double().numpy()
    want = gc.rotary(x.double().numpy(), pos.numpy(), gc.frequencies(64, 1e6))
    _near(got, x.double().numpy(), want, 1, dtype, 10)


def test_rotary_farthest_positions():
    _say("positions to 2^31")
    x, _ = _inputs(4, 2, 128, "f32", 10)
    pos = torch.tensor([2**31 - 1, -2**31, 2**30 + 1, 0], dtype=torch.int32)
    got = _run(x.cuda(), pos.cuda(), kv().make_rope(128, theta=1e4), "f32").cpu().double().numpy()
    want = gc.rotary(x.double().numpy(), pos.numpy(), gc.frequencies(128, 1e4))
    _near(got, x.double().numpy(), want, 1, "f32", 20)
    assert np.array_equal(got[3], x[3].double().numpy())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shift,extra", [(0, 8), (1, 0), (3, 5)])
def test_rotary_of_a_fused_buffer(dtype, layout, shift, extra):
    """Queries and keys inside one buffer of odd strides and alignments, out of it and in place; the
    buffer's other columns, and rows past the last, keep their bytes."""
    _say(dtype, layout, shift, extra)
    m, d, hq, hk, rows = kv(), 64, 5, 2, 37
    width = (hq + 2 * hk) * d + extra
    gen = torch.Generator().manual_seed(shift + extra)
    host = torch.randn(shift + (rows + 1) * width, generator=gen).to(T[dtype])
    pos = torch.randint(0, 5000, (rows,), generator=gen, dtype=torch.int32)
    view = host[shift:shift + rows * width].view(rows, width)[:, :(hq + hk) * d].reshape(rows, hq + hk, d).double().numpy()
    want = gc.rotary(view, pos.numpy(), gc.frequencies(d, 1e6), layout)
    rope, dev, p = m.make_rope(d, layout=layout), host.cuda(), pos.cuda()
    e, st = host.element_size(), torch.cuda.current_stream().cuda_stream
    q = torch.full((rows + 1, hq, d), 7.0, dtype=T[dtype], device="cuda")
    k = torch.full((rows + 1, hk, d), 7.0, dtype=T[dtype], device="cuda")
    at = dev.data_ptr() + shift * e
    m.kvprm_rotary(rope, dtype, rows, p.data_ptr(), m.make_rope_heads(
        [(at, q.data_ptr(), hq, width, hq * d), (at + hq * d * e, k.data_ptr(), hk, width, hk * d)]), stream=st)
    torch.cuda.synchronize()
    assert torch.equal(dev.cpu(), host)
    for t, h0 in ((q, 0), (k, hq)):
        _near(t[:rows].cpu().double().numpy(), view[:, h0:h0 + t.shape[1]], want[:, h0:h0 + t.shape[1]], 1, dtype, 10)
        assert torch.all(t[rows] == 7.0)
    m.kvprm_rotary(rope, dtype, rows, p.data_ptr(), m.make_rope_heads(
        [(at, at, hq, width, width), (at + hq * d * e, at + hq * d * e, hk, width, width)]), stream=st)
    torch.cuda.synchronize()
    after = dev.cpu()
    body = after[shift:shift + rows * width].view(rows, width)
    assert torch.equal(body[:, :hq * d].reshape(rows, hq, d), q[:rows].cpu())
    assert torch.equal(body[:, hq * d:(hq + hk) * d].reshape(rows, hk, d), k[:rows].cpu())
    body[:, :(hq + hk) * d] = host[shift:shift + rows * width].view(rows, width)[:, :(hq + hk) * d]
    assert torch.equal(after, host)  # everything else is as it was


def test_rotary_gradient():
    """transpose is the gradient: <R x, y> = <x, R^T y>, and central differences of <R x, y> (linear in x:
    exact up to fp32 sums, 64 * 2^-23 of the terms' size)."""
    _say("gradient")
    rope = kv().make_rope(64, 48, "interleaved", 1e4, "parts", 2.0, TRAINED, magnitude=1.25)
    x, pos = _inputs(8, 2, 64, "f32", 9000)
    y = torch.randn(x.shape, generator=torch.Generator().manual_seed(3))
    dx, dp = x.cuda(), pos.cuda()
    fwd = _run(dx, dp, rope, "f32").cpu().double()
    back = _run(y.cuda(), dp, rope, "f32", transpose=True).cpu().double()
    tol = 64 * 2.0 ** -23 * float((fwd.abs() * y.abs()).sum())
    assert abs(float((fwd * y).sum() - (x.double() * back).sum())) <= tol
    for r, h, i in ((0, 0, 0), (3, 1, 47), (7, 0, 63)):
        out = []
        for s in (1.0, -1.0):
            z = x.clone()
            z[r, h, i] += s
            out.append(float((_run(z.cuda(), dp, rope, "f32").cpu().double() * y).sum()))
        assert abs((out[0] - out[1]) / 2 - float(back[r, h, i])) <= tol


def test_rotary_in_a_graph():
    """Replays follow the positions and inputs that are on the device, and equal the eager call."""
    _say("graph")
    m = kv()
    x, pos = _inputs(33, 4, 128, "bf16", 9000)
    rope, dx, dp = m.make_rope(128), x.cuda(), pos.cuda()
    out = torch.zeros_like(dx)
    _run(dx, dp, rope, "bf16", out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.kvprm_rotary(rope, "bf16", 33, dp.data_ptr(),
                       m.make_rope_heads([(dx.data_ptr(), out.data_ptr(), 4, 512, 512)]),
                       stream=torch.cuda.current_stream().cuda_stream)
    for seed in (1, 2, 3):
        y, p2 = _inputs(33, 4, 128, "bf16", 70000, seed)
        dx.copy_(y)
        dp.copy_(p2)
        want = _run(dx, dp, rope, "bf16")
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    del g
