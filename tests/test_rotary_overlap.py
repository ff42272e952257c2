"""Which rows of kvprm_rotary's tensors may share memory: what the documentation rules out is refused before anything
is enqueued (CPU), what it allows gives the result of separate buffers (GPU)."""
import pytest
import torch

import paper_2607_09153_amd as kv

A, B, C = 0x10000, 0x80000, 0x100000
E, W = 2, 2 * 64  # bytes and values of a row of two heads


def _call(parts, rows=4, pos=0x200000):
    kv.kvprm_rotary(kv.make_rope(64), "bf16", rows, pos, kv.make_rope_heads(parts))


@pytest.mark.parametrize("kw", [
    dict(parts=[(A, B, 2, W, W), (B, C, 2, W, W)]),                          # the first's result is the second's input
    dict(parts=[(A, B, 2, W, W), (C, A, 2, W, W)]),                          # the second's result is the first's input
    dict(parts=[(A, B, 2, W, W), (C, B, 2, W, W)]),                          # one place for both results
    dict(parts=[(A, A, 2, W, W), (A, A, 2, W, W)]),                          # both in place
    dict(parts=[(A, B, 2, W, W), (B + 3 * W * E, C, 2, W, W)]),              # the last row alone
    dict(parts=[(A, B, 2, W, 4 * W), (B + W, C, 1, 4 * W, W)]),              # columns by half
    dict(parts=[(A, B + 3 * W * E + 2, 2, W, 4 * W), (B, C, 2, 4 * W, W)]),  # a row's end in the next one's columns
    dict(parts=[(A, B, 2, W, 4 * W), (B + 2 * W * E, C, 2, 2 * W, W)]),      # unequal strides, between each other
    dict(parts=[(A, B, 2, W, W)], pos=0x200002),                             # positions at an odd address
    dict(parts=[(A, A + 2, 2, W, W)], rows=1),
])
def test_rotary_refuses_overlaps(kw):
    with pytest.raises(kv.KvprmError) as e:
        _call(**kw)
    assert e.value.status == kv.KVPRM_E_INVALID, kv.kvprm_last_error()


def _rotate(rope, rows, pos, parts):
    kv.kvprm_rotary(rope, "bf16", rows, pos.data_ptr(), kv.make_rope_heads(parts),
                    stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 7])
def test_rotary_beside_each_other(rows):
    """Queries and keys rotated into columns of the buffer that holds them, one input for both tensors, one row in
    place whose strides differ."""
    print("case:", rows, flush=True)
    d, hq, hk = 64, 4, 2
    width = 2 * (hq + hk) * d
    gen = torch.Generator().manual_seed(rows)
    x = torch.randn((rows, width), generator=gen).bfloat16().cuda()
    pos = torch.randint(0, 9000, (rows,), generator=gen, dtype=torch.int32).cuda()
    rope, keep, at = kv.make_rope(d), x.clone(), x.data_ptr()
    q = torch.empty((rows, hq * d), dtype=x.dtype, device="cuda")
    k = torch.empty((rows, hk * d), dtype=x.dtype, device="cuda")
    _rotate(rope, rows, pos, [(at, q.data_ptr(), hq, width, hq * d), (at + hq * d * E, k.data_ptr(), hk, width, hk * d)])
    half = (hq + hk) * d
    _rotate(rope, rows, pos, [(at, at + half * E, hq, width, width),
                              (at + hq * d * E, at + (half + hq * d) * E, hk, width, width)])
    assert torch.equal(x[:, :half], keep[:, :half])
    assert torch.equal(x[:, half:half + hq * d], q) and torch.equal(x[:, half + hq * d:], k)
    y = [torch.empty((rows, hk * d), dtype=x.dtype, device="cuda") for _ in (0, 1)]
    _rotate(rope, rows, pos, [(at + hq * d * E, t.data_ptr(), hk, width, hk * d) for t in y])
    assert torch.equal(y[0], k) and torch.equal(y[1], k)
    if rows == 1:
        _rotate(rope, 1, pos, [(at, at, hq, width, hq * d), (at + hq * d * E, at + hq * d * E, hk, hk * d, width)])
        assert torch.equal(x[:, :hq * d], q) and torch.equal(x[:, hq * d:half], k)
