"""kvprm_attention and the scoring calls over 4-bit caches.

Tolerance of an attention output against the fp64 oracle: with |q|, |k| entries near N(0, 1) and d <= 128, a score's
fp32 sum is off by at most d 2^-24 sum|q k| / sqrt(d) ~ 5.5e-5 if every rounding went one way, and by the root of d
of them, 5e-6, as they fall; the query's and the weights' terms keep 20 bits or more (2^-20 of each); weights follow
their score (e^x) and the sums add 2^-24 each. An output is a mean of values with these weights: within
2 * 1e-5 max|v|. Scores are compared with those over a bf16 cache that holds the same values."""
import numpy as np
import pytest
import torch

from oracle import fp4
from oracle import growing_cache as gc
from oracle import kvprm_oracle as ko

from fp4_common import Cache
from gpu_common import kv

pytestmark = pytest.mark.gpu
LAYER = 1


def _say(*a):
    print("case:", *a, flush=True)


def _inputs(c, seed):
    rng = np.random.default_rng(seed)
    nq, nkv, d = c.shape
    return [rng.normal(size=(len(c.lengths), h, d)).astype(np.float32) for h in (nq, nkv, nkv)]


def _run(c, x, batch=None, stream=None):
    m = c.m
    batch = batch or c.batch
    n = m.kvprm_workspace_size(c.h, batch)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # (fp32 NaN)
    q, k, v = (torch.from_numpy(t).cuda() for t in x)
    o = torch.full(q.shape, 7.0, device="cuda")
    st = stream or torch.cuda.current_stream()
    st.wait_stream(torch.cuda.current_stream())
    m.kvprm_attention(c.h, c.cache, batch, LAYER, q.data_ptr(), k.data_ptr(), v.data_ptr(), ws.data_ptr(), n, o.data_ptr(),
                      st.cuda_stream)
    torch.cuda.synchronize()
    return o.cpu().numpy()


def _check(c, x, got):
    nq, nkv, d = c.shape
    for b in range(len(c.lengths)):
        ck, cv = (c.cached(p, LAYER, b) for p in (0, 1))
        for h in range(nq):
            j = h // (nq // nkv)
            K, V = np.concatenate([ck[:, j], x[1][b, j][None]]), np.concatenate([cv[:, j], x[2][b, j][None]])
            want = ko.attention(x[0][b, h].astype(np.float64), K, V)
            off = np.abs(got[b, h] - want).max()
            assert off <= 2e-5 * np.abs(V).max(), (b, h, off)


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (16, 8, 128), (28, 4, 128), (32, 2, 128), (5, 1, 64), (3, 3, 128),
                                      (16, 1, 64), (22, 2, 128)])
def test_lengths(nq, nkv, d):
    _say("lengths", nq, nkv, d)
    c = Cache(nq, nkv, d, [0, 1, 15, 16, 17, 31, 32, 33, 100, 511, 512, 513], seed=d + nq)
    x = _inputs(c, 3)
    _check(c, x, _run(c, x))


@pytest.mark.parametrize("d,lengths", [(128, [1103]), (64, [5000]), (128, [3000, 1, 0, 2048, 700]), (64, [2000] * 6),
                                       (128, [40 + 97 * i for i in range(40)])])
def test_long(d, lengths):
    """Chunked caches, with and without host lengths."""
    _say("long", d, lengths[:4])
    c = Cache(8, 2, d, lengths, seed=len(lengths))
    x = _inputs(c, 4)
    _check(c, x, _run(c, x))
    _check(c, x, _run(c, x, c.m.make_batch(len(lengths), c.dtab.data_ptr(), c.width, c.dlen.data_ptr())))


def test_values_of_many_sizes():
    """Scales from 2^-40 to 2^40 among the values (keys near 1); large scores."""
    _say("sizes")
    c = Cache(4, 2, 128, [800, 33], seed=8)
    rng = np.random.default_rng(1)
    c.scale[1] = np.where(c.scale[1] == 255, 255, c.scale[1] + rng.integers(-40, 40, size=c.scale[1].shape)).astype(np.uint8)
    c.upload()
    x = _inputs(c, 5)
    _check(c, x, _run(c, x))
    c = Cache(4, 2, 64, [800, 33], seed=9)
    x = _inputs(c, 6)
    x[0] *= 40  # scores of some hundreds: the largest alone counts, and its error grows with the score
    nq, nkv, d = c.shape
    got = _run(c, x)
    for b in range(2):
        ck, cv = (c.cached(p, LAYER, b) for p in (0, 1))
        for h in range(nq):
            K, V = (np.concatenate([t[:, h // 2], s[b, h // 2][None]]) for t, s in ((ck, x[1]), (cv, x[2])))
            want = ko.attention(x[0][b, h].astype(np.float64), K, V)
            assert np.abs(got[b, h] - want).max() <= 40 * 2e-5 * np.abs(V).max()


def test_nan_tokens():
    """A stored NaN reaches the candidate that attends to it, in the heads and dims it belongs to, and nobody else."""
    _say("nan")
    c = Cache(4, 2, 128, [200, 200, 20], seed=10)
    page, slot = c.table[0, 150 // 16], 150 % 16
    c.scale[1][LAYER, page, 1, slot, 2] = 255  # a value: dims 64 .. 95 of kv-head 1
    c.scale[0][LAYER, c.table[2, 0], 0, 3, 0] = 255  # a key of kv-head 0
    c.upload()
    x = _inputs(c, 7)
    got = _run(c, x)
    want = np.zeros(got.shape, bool)
    want[0, 2:, 64:96] = True
    want[2, :2] = True
    assert np.array_equal(np.isnan(got), want)
    c.lengths = c.lengths[1:2]
    _check_rows = got[1:2]
    c.table = c.table[1:2]
    _check(c, [t[1:2] for t in x], _check_rows)


def test_shared_prefix_hint():
    """Candidates that share pages, with the hint and without."""
    _say("prefix")
    for g, kvh in ((7, 2), (2, 4)):
        c = Cache(g * kvh, kvh, 128, [700, 640, 900, 33, 320, 400], seed=11)
        for b in (1, 2):
            c.table[b, :40] = c.table[0, :40]
        c.table[5, :20] = c.table[4, :20]
        c.upload()
        x = _inputs(c, 8)
        _check(c, x, _run(c, x))
        hint = c.m.make_batch(6, c.dtab.data_ptr(), c.width, c.dlen.data_ptr(), c.lengths, [0, 3, 4, 6], [640, 0, 320])
        _check(c, x, _run(c, x, hint))


def test_streams_and_graph():
    _say("graph")
    c = Cache(8, 2, 128, [600, 90], seed=12)
    x = _inputs(c, 9)
    want = _run(c, x)
    assert np.array_equal(want, _run(c, x, stream=torch.cuda.Stream()))
    m = c.m
    n = m.kvprm_workspace_size(c.h, c.batch)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    q, k, v = (torch.zeros(t.shape, device="cuda") for t in x)
    o = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.kvprm_attention(c.h, c.cache, c.batch, LAYER, q.data_ptr(), k.data_ptr(), v.data_ptr(), ws.data_ptr(), n,
                          o.data_ptr(), torch.cuda.current_stream().cuda_stream)
    for s in range(3):
        x = _inputs(c, 30 + s)
        for t, a in zip((q, k, v), x):
            t.copy_(torch.from_numpy(a))
        graph.replay()
        torch.cuda.synchronize()
        got = o.cpu().numpy()
        assert np.array_equal(got, _run(c, x))
    _check(c, x, got)


def _bf16_twin(dw, w):
    """A 4-bit cache and a bf16 one with its values, for the workload `w` (bf16) on the device."""
    s = w.shape
    rng = np.random.default_rng(5)
    pools4, pools16 = [], []
    for part in (0, 1):
        code, scale = fp4.encode(rng.normal(size=(s.num_layers * w.num_pages, s.num_kv_heads, 16, s.head_dim)))
        pools4.append(torch.from_numpy(fp4.store(code, scale, part)).cuda())
        words = gc.to_bf16(fp4.decode(code, scale).astype(np.float32))
        pools16.append(torch.from_numpy(gc.store(words, part).view(np.uint8)).cuda())
    return [kv().make_cache(p[0].data_ptr(), p[1].data_ptr(), w.num_pages) for p in (pools4, pools16)], pools4 + pools16


@pytest.mark.parametrize("d", [64, 128])
def test_scores(d):
    """kvprm_score, _score_ex (depth 2), _score_lora and _score_static over the 4-bit cache and over its values in bf16."""
    import synth
    from synth.device import DeviceWorkload

    _say("scores", d)
    m = kv()
    shape = synth.ModelShape(3, 256, 4, 2, d, 512)
    w = synth.make_workload("custom", shape=shape, lengths=[700, 0, 17, 300, 33], seed=21)
    dw = DeviceWorkload(w)
    dw.add_lora(32)
    caches, keep = _bf16_twin(dw, w)
    got = []
    for cdt, cache in zip(("fp4", "bf16"), caches):
        desc = dw.desc(m)
        desc.kv_dtype = m.DTYPE_CODE[cdt]
        h = m.kvprm_create(desc)
        st = torch.cuda.current_stream().cuda_stream
        batch, wts, out = dw.batch(m), dw.readout(m), []
        try:
            for call in ("score", "depth", "lora", "static"):
                score, z = (torch.full((w.batch,), float("nan"), device="cuda") for _ in (0, 1))
                opt = m.make_options(dw.lora(m) if call == "lora" else None, 2 if call == "depth" else 1)
                n = m.kvprm_workspace_size_ex(h, batch, opt)
                ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
                if call == "static":
                    m.kvprm_score_static(h, cache, batch, wts, score.data_ptr(), z.data_ptr(), st)
                elif call == "score":
                    m.kvprm_score(h, cache, batch, wts, ws.data_ptr(), n, score.data_ptr(), z.data_ptr(), st)
                else:
                    m.kvprm_score_ex(h, cache, batch, wts, opt, ws.data_ptr(), n, score.data_ptr(), z.data_ptr(), st)
                torch.cuda.synchronize()
                out += [score.cpu().numpy(), z.cpu().numpy()]
        finally:
            m.kvprm_destroy(h)
        got.append(np.stack(out))
    assert np.all(np.isfinite(got[0]))
    # (both are within 1e-5 of the fp64 oracle by the parity tests' bound on P, 1e-4 on z)
    assert np.abs(got[0] - got[1])[0::2].max() <= 2e-5 and np.abs(got[0] - got[1])[1::2].max() <= 2e-4
    del keep
