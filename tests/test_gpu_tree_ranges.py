"""kvprm_attention_tree where values span many powers of two and where a chunk is longer than the page ids a
block holds at a time. The tolerance is that of test_gpu_tree.py with max|v| of each candidate: a scale per page
is exact in the weights or in the exponent of the sums, and what far smaller pages lose is below 2^-40 of it."""
import numpy as np
import pytest

from oracle import growing_cache as gc

from test_gpu_tree import LAYER, Case, _say

pytestmark = pytest.mark.gpu


def _check(c):
    got, want = c.run(), c.want()
    nq, nkv, d = c.shape
    for b, (n, t) in enumerate(zip(c.lengths, c.counts)):
        rows = slice(c.start[b], c.start[b] + t)
        v = c.qkv[rows, (nq + nkv) * d:(nq + 2 * nkv) * d].double().numpy()
        cv = gc.cached(c.tok[1][LAYER], c.scale[1][LAYER], c.cdt, c.table[b], n)
        size = max([float(np.abs(x).max()) for x in (v, cv) if x.size] + [0.0])
        y = got[rows, :nq * d].double().numpy()
        tol = 2e-5 * size if c.dtype == "f32" else (2.0 ** -11 + 2e-5) * size + 2.0 ** -8 * np.abs(want[rows])
        err = np.abs(y - want[rows])
        assert np.all(err <= tol), (b, size, float(err.max()))


@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (4, 1, 128)])
@pytest.mark.parametrize("n,dtype", [(5, "bf16"), (40, "bf16"), (100, "bf16"), (7, "f32")])
def test_tree_fp8_value_scales(nq, nkv, d, n, dtype):
    """Pages of zeros hold the smallest scale, 2^-100: between pages of ordinary ones, alone, below larger ones;
    scales of 0; drafted values far above and below the cached ones, and tiny ones behind a page pair of
    zeros."""
    _say("value scales", nq, nkv, d, n, dtype)
    lengths = [700, 300, 900, 40, 0, 33]
    c = Case("fp8", dtype, nq, nkv, d, lengths, [n] * 6, seed=n + d)
    rng = np.random.default_rng(n)
    sets = [(2.0 ** -100, 1.25 * 2.0 ** -7, 0.0), (1.25 * 2.0 ** -100, 2.0 ** -97), (2.0 ** 10, 1.1 * 2.0 ** -20, 2.0 ** -60),
            (0.0,), (1.0,), (2.0 ** -100,)]
    c.scale[1][:] = 1.0
    for b, values in enumerate(sets):
        for page in c.table[b][c.table[b] >= 0]:
            c.scale[1][:, page] = rng.choice(values, size=c.scale[1][:, page].shape)
    vs = slice((nq + nkv) * d, (nq + 2 * nkv) * d)
    for b, f in enumerate((1.0, 2.0 ** -95, 2.0 ** -60, 2.0 ** 40, 2.0 ** -90, 2.0 ** 100)):
        rows = slice(c.start[b], c.start[b] + n)
        c.qkv[rows, vs] *= f
        if b == 4:
            c.qkv[c.start[b]:c.start[b] + min(n, 33), vs] = 0
    c.upload()
    _check(c)


@pytest.mark.parametrize("cdt,dtype,n", [("bf16", "bf16", 20), ("fp8", "bf16", 20), ("f32", "f32", 3), ("bf16", "bf16", 3),
                                         ("fp8", "f32", 3)])
def test_tree_long_chunk(cdt, dtype, n):
    """So many candidates that each cache is one chunk, one of them of more than 256 pages."""
    _say("long chunk", cdt, dtype, n)
    lengths = [9 + 4096 + 500] + [i % 37 for i in range(63)]
    c = Case(cdt, dtype, 16, 8, 64, lengths, [n] + [1 + i % n for i in range(63)], seed=n)
    if cdt == "fp8":  # later pages hold far larger values than the first, the last ones far smaller
        for i, page in enumerate(c.table[0][c.table[0] >= 0]):
            c.scale[1][:, page] = 2.0 ** (-100 if i < 256 or i > 280 else -7)
        c.upload()
    _check(c)


@pytest.mark.parametrize("cdt,dtype,nq,nkv,d", [("bf16", "bf16", 32, 2, 128), ("fp8", "bf16", 32, 2, 64), ("f32", "f32", 13, 1, 64),
                                                ("fp8", "f32", 16, 1, 128), ("bf16", "bf16", 11, 1, 64)])
def test_tree_most_columns(cdt, dtype, nq, nkv, d):
    """256 drafted tokens of 11 to 16 query heads per kv-head: up to 4096 columns."""
    _say("most columns", cdt, dtype, nq, nkv, d)
    _check(Case(cdt, dtype, nq, nkv, d, [40, 500, 0], [256, 255, 1], seed=nq))
