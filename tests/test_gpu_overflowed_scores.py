"""kvprm_attention where the first cached keys are so large that their scores pass fp32's range downwards: weights of 0,
as in the fp64 oracle, and the later tokens and the own key make the result.

Tolerance: the keys that count are near N(0, 1) and the queries 0.3 to 0.4, so that scores are below 10 and those of
the other tests' bound (2e-5 max|v|, test_gpu_fp4_attention.py); two bf16 terms of a weight (bf16 and fp8 caches) add
2^-16 max|v|."""
import numpy as np
import pytest
import torch

from oracle import growing_cache as gc
from oracle import kvprm_oracle as ko

import fp4_common
from test_gpu_fp4_tree import Draft
from test_gpu_tree import LAYER, Case

pytestmark = pytest.mark.gpu
LENGTHS = [0, 1, 16, 17, 32, 33, 48, 100, 400, 400, 3000]
LARGE = [0, 1, 16, 16, 32, 32, 40, 32, 400, 96, 700]  # the first of these many tokens
SHARED = [400, 400, 400, 500]  # a prefix of 320 tokens in one table


def _fill(cdt, nq, nkv, d, lengths, large, seed, shared=0):
    """A cache whose first `large` tokens of each candidate have keys of about -2^127 in every dim."""
    c = fp4_common.Cache(nq, nkv, d, lengths, seed=seed) if cdt == "fp4" else Case(cdt, "f32" if cdt == "f32" else "bf16", nq, nkv,
                                                                                    d, lengths, [1] * len(lengths), seed=seed)
    for b in range(1, len(lengths) if shared else 0):
        c.table[b, :shared // 16] = c.table[0, :shared // 16]
    for b, n in enumerate(large):
        for t in range(n):
            page, slot = c.table[b, t // 16], t % 16
            if cdt == "fp4":
                c.code[0][:, page, :, slot], c.scale[0][:, page, :, slot] = 15, 252  # -6 * 2^125
            elif cdt == "f32":
                c.tok[0][:, page, :, slot] = np.float32(-2.5e38).view(np.uint32)
            elif cdt == "bf16":
                c.tok[0][:, page, :, slot] = gc.to_bf16(np.float32(-2.5e38))
            else:  # a scale belongs to a page: the page's other tokens are as small as it is large
                c.tok[0][:, page, :, slot] = gc.to_e4m3(np.array(-448.0))
                c.scale[0][:, page] = np.float32(5e35)
                if slot == 0:
                    rest = c.tok[0][:, page, :, 1:]
                    c.tok[0][:, page, :, 1:] = np.where(rest == 0x7F, rest, 0)
    c.upload()
    return c


def _check(c, cdt, lengths, x, got, what, size=1.0):
    """size: that of the queries beside N(0, 1), with which the scores' error grows."""
    nq, nkv, d = c.shape
    assert np.all(np.isfinite(got)), (what, np.argwhere(~np.isfinite(got))[:4])
    for b, n in enumerate(lengths):
        ck, cv = ((c.cached(p, LAYER, b) if cdt == "fp4" else gc.cached(c.tok[p][LAYER], c.scale[p][LAYER], cdt, c.table[b], n))
                  for p in (0, 1))
        for h in range(nq):
            j = h // (nq // nkv)
            K, V = np.concatenate([ck[:, j], x[1][b, j][None]]), np.concatenate([cv[:, j], x[2][b, j][None]])
            want = ko.attention(x[0][b, h].astype(np.float64), K, V)
            off = np.abs(got[b, h] - want).max()
            assert off <= (2e-5 * size + 2.0 ** -16) * np.abs(V).max(), (what, b, h, off)


def _inputs(c, n, seed):
    rng = np.random.default_rng(seed)
    nq, nkv, d = c.shape
    return [t.astype(np.float32) for t in (rng.uniform(0.3, 0.4, size=(n, nq, d)), rng.normal(size=(n, nkv, d)),
                                           rng.normal(size=(n, nkv, d)))]


def _run(c, x, batch):
    m = c.m
    n = m.kvprm_workspace_size(c.h, batch)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    q, k, v = (torch.from_numpy(t).cuda() for t in x)
    o = torch.full(q.shape, 7.0, device="cuda")
    m.kvprm_attention(c.h, c.cache, batch, LAYER, q.data_ptr(), k.data_ptr(), v.data_ptr(), ws.data_ptr(), n, o.data_ptr(),
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return o.cpu().numpy()


@pytest.mark.parametrize("cdt", ["fp4", "f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_private_pages(cdt, d):
    """The whole batch in chunks, and its shorter candidates in one launch."""
    print("case:", cdt, d, flush=True)
    for lengths, large in ((LENGTHS, LARGE), (LENGTHS[:8], LARGE[:8])):
        c = _fill(cdt, 4, 2, d, lengths, large, d)
        x = _inputs(c, len(lengths), d)
        batch = c.m.make_batch(len(lengths), c.dtab.data_ptr(), c.width, c.dlen.data_ptr(), lengths)
        _check(c, cdt, lengths, x, _run(c, x, batch), len(lengths))


@pytest.mark.parametrize("cdt", ["fp4", "bf16", "fp8"])
@pytest.mark.parametrize("large", [32, 320])
def test_shared_prefix(cdt, large):
    print("case: prefix", cdt, large, flush=True)
    c = _fill(cdt, 4, 2, 128, SHARED, [large] * 4, 3, shared=320)
    x = _inputs(c, 4, 5)
    hint = c.m.make_batch(4, c.dtab.data_ptr(), c.width, c.dlen.data_ptr(), SHARED, [0, 4], [320])
    _check(c, cdt, SHARED, x, _run(c, x, hint), "hint")


@pytest.mark.parametrize("lo,hi", [(100, 100), (11, 11), (50, 150), (0, 1000), (1e4, 1e6)])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_far_past_the_range(d, lo, hi):
    """4-bit caches: a query is summed in terms, whose parts of such a score pass the range with either sign."""
    print("case: far", d, lo, hi, flush=True)
    for lengths, large in ((LENGTHS, LARGE), (LENGTHS[:8], LARGE[:8])):
        c = _fill("fp4", 4, 2, d, lengths, large, d)
        x = _inputs(c, len(lengths), d)
        x[0] = np.random.default_rng(7).uniform(lo, hi, size=x[0].shape).astype(np.float32)
        batch = c.m.make_batch(len(lengths), c.dtab.data_ptr(), c.width, c.dlen.data_ptr(), lengths)
        _check(c, "fp4", lengths, x, _run(c, x, batch), len(lengths), size=hi)
    c = _fill("fp4", 4, 2, d, SHARED, [32] * 4, 3, shared=320)
    x = _inputs(c, 4, 5)
    x[0] = np.random.default_rng(8).uniform(lo, hi, size=x[0].shape).astype(np.float32)
    hint = c.m.make_batch(4, c.dtab.data_ptr(), c.width, c.dlen.data_ptr(), SHARED, [0, 4], [320])
    _check(c, "fp4", SHARED, x, _run(c, x, hint), "hint", size=hi)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lo,hi", [(0.3, 0.4), (100, 100), (50, 150), (0, 1000)])
@pytest.mark.parametrize("counts", [3, 60])
@pytest.mark.parametrize("d", [64, 128])
def test_drafts(d, counts, lo, hi, dtype):
    """Drafted tokens over such 4-bit caches (within the bound of test_gpu_fp4_tree.py, times the queries' size)."""
    print("case: drafts", d, counts, lo, hi, dtype, flush=True)
    nq, nkv, lengths, large = 4, 2, LENGTHS[1:9], LARGE[1:9]
    c = _fill("fp4", nq, nkv, d, lengths, large, d)
    dr = Draft(c, dtype, [counts] * len(lengths), "chain", seed=d)
    q = np.random.default_rng(counts).uniform(lo, hi, size=(dr.rows, nq * d)).astype(np.float32)
    dr.x[:dr.rows, :nq * d] = torch.from_numpy(q).to(dr.x.dtype)
    dr.dx = dr.x.cuda()
    got = dr.run()[:dr.rows, :nq * d].double().numpy()
    assert np.all(np.isfinite(got)), np.argwhere(~np.isfinite(got))[:4]
    for b, n in enumerate(lengths):
        rows = slice(b * counts, (b + 1) * counts)
        x = dr.x[rows, :(nq + 2 * nkv) * d].double().numpy().reshape(counts, nq + 2 * nkv, d)
        ck, cv = (c.cached(p, LAYER, b) for p in (0, 1))
        want = gc.tree_attention(x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], ck, cv, dr.sees[b]).reshape(counts, nq * d)
        big = max(np.abs(cv).max(), np.abs(x[:, nq + nkv:]).max())
        tol = 2e-5 * max(hi, 1) * big + ((2.0 ** -16) * big + 2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
        assert np.all(np.abs(got[rows] - want) <= tol), (b, np.abs(got[rows] - want).max(), big)
