"""kvprm_attention_tree where a row's own keys and values bound its result, whatever the others hold.

Tolerance of a row: the weights p of what it attends to are rounded to 16 bits (two bf16 terms) or, over fp8 caches
with more than 32 columns, 11 (fp16), and are off by 2e-5 through the scores (test_gpu_tree.py), so that o = sum p v /
sum p is off by at most (2^-16 or 2^-11, and 2e-5) sum p |v| / sum p; the bf16 result adds its own half step, 2^-8 |o|."""
import numpy as np
import pytest

from oracle import growing_cache as gc

from test_gpu_tree import LAYER, Case, _say
from test_gpu_tree_full import _sizes

pytestmark = pytest.mark.gpu


def _set_bits(c):
    """The case's mask words from its `sees`, and everything back on the device."""
    c.bits[:] = 0
    for b, s in enumerate(c.sees):
        for j in range(len(s)):
            c.bits[c.start[b]:c.start[b] + len(s), j // 32] |= s[:, j].astype(np.uint32) << np.uint32(j % 32)
    c.upload()


def _check_rows(c, eps, got=None, scores=1.0):
    """eps: the weights' rounding; scores: the size of the scores, with which their error grows."""
    got, want = c.run() if got is None else got, c.want()
    nq, nkv, d = c.shape
    y = got[:c.rows, :nq * d].double().numpy()
    assert np.array_equal(np.isnan(y), np.isnan(want))
    assert np.array_equal(np.isinf(y), np.isinf(want)) and np.array_equal(y[np.isinf(want)], want[np.isinf(want)])
    for b, (n, t) in enumerate(zip(c.lengths, c.counts)):
        if t == 0:
            continue
        rows = slice(c.start[b], c.start[b] + t)
        x = c.qkv[rows].double().numpy()
        q, k, v = (x[:, i * d:j * d].reshape(t, j - i, d) for i, j in ((0, nq), (nq, nq + nkv), (nq + nkv, nq + 2 * nkv)))
        ck, cv = (gc.cached(c.tok[p][LAYER], c.scale[p][LAYER], c.cdt, c.table[b], n) for p in (0, 1))
        v, cv = (np.where(np.isfinite(z), np.abs(z), 0) for z in (v, cv))
        size = gc.tree_attention(q, k, v, ck, cv, c.sees[b]).reshape(t, nq * d)
        w, fine = want[rows], np.isfinite(want[rows])
        tol = (eps + 2e-5 * scores) * size + (2.0 ** -8 * np.abs(w) if c.dtype == "bf16" else 0)
        off = np.argwhere(fine & ~(np.abs(np.where(fine, y[rows] - w, 0)) <= tol))
        assert not len(off), (b, off[:3], y[rows][tuple(off[0])], w[tuple(off[0])], tol[tuple(off[0])])


@pytest.mark.parametrize("cdt,eps", [("fp8", 2.0 ** -11), ("bf16", 2.0 ** -16)])
@pytest.mark.parametrize("d", [64, 128])
def test_tree_large_values_where_masked(cdt, eps, d):
    """Drafted values of 2^100 and 2^110 that other tokens do not attend to, among values near 1 that they do: in the
    same 32 tokens, and in earlier ones."""
    _say("large values where masked", cdt, d)
    nq, nkv = 8, 2
    c = Case(cdt, "bf16", nq, nkv, d, *_sizes(60), seed=d)
    vs = slice((nq + nkv) * d, (nq + 2 * nkv) * d)
    for b, n in enumerate(c.counts):
        for t, f in ((1, 2.0 ** 100), (n - 2, 2.0 ** 110)):
            if n >= 8:
                c.qkv[c.start[b] + t, vs] *= f
                c.sees[b][:, t] = np.arange(n) == t
    _set_bits(c)
    _check_rows(c, eps)


@pytest.mark.parametrize("d", [64, 128])
def test_tree_small_pages_beside_large_ones(d):
    """Pages of values near 2^-60 beside one of values near 1 whose tokens have weights below 2^-200."""
    _say("small pages", d)
    nq, nkv = 8, 2
    c = Case("fp8", "bf16", nq, nkv, d, *_sizes(60), seed=d + 1, masked="chain")
    c.qkv[:, :nq * d] = c.qkv[:, :nq * d].abs()
    c.qkv[:, (nq + nkv) * d:] *= 2.0 ** -60
    c.scale[1][:] *= 2.0 ** -60
    for b, n in enumerate(c.lengths):
        if n >= 32:
            page = c.table[b, (n // 16) // 2]
            c.scale[1][:, page] *= 2.0 ** 60
            c.tok[0][:, page] = gc.to_e4m3(np.array(-256.0))
            c.scale[0][:, page] = 0.125
    c.upload()
    _check_rows(c, 2.0 ** -11)


@pytest.mark.parametrize("cdt,eps", [("bf16", 2.0 ** -16), ("fp8", 2.0 ** -11)])
@pytest.mark.parametrize("d", [64, 128])
def test_tree_values_near_the_largest(cdt, eps, d):
    """Cached and drafted values of 2^119 and more."""
    _say("values near the largest", cdt, d)
    nq, nkv = 8, 2
    c = Case(cdt, "bf16", nq, nkv, d, *_sizes(60), seed=d + 2)
    c.qkv[:, (nq + nkv) * d:(nq + 2 * nkv) * d] *= 2.0 ** 119
    if cdt == "fp8":
        c.scale[1][:] *= 2.0 ** 119
    else:
        x = (c.tok[1].astype(np.uint32) << 16).view(np.float32) * np.float32(2.0 ** 119)
        c.tok[1] = gc.to_bf16(x)
    c.upload()
    _check_rows(c, eps)


@pytest.mark.parametrize("dtype,counts", [("bf16", None), ("bf16", 5), ("f32", 9), ("bf16", 40)])
@pytest.mark.parametrize("cdt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_tree_cached_infinities(cdt, dtype, counts, d):
    """Infinities and NaN among the cached values reach every token as the definition says; those of drafted values
    meet them. Several chunks, the cache's last page among those that hold them; slots past the length hold NaN."""
    _say("cached infinities", cdt, dtype, counts, d)
    nq, nkv = 8, 2
    sizes = _sizes(60) if counts is None else ([2000, 33, 7, 300], [counts, 2, 8, counts])
    c = Case(cdt, dtype, nq, nkv, d, *sizes, seed=d + 3)
    word = {"bf16": (0x7F80, 0xFF80, 0x7FC0), "f32": (0x7F800000, 0xFF800000, 0x7FC00000)}[cdt]
    rng = np.random.default_rng(d)
    for b, n in enumerate(c.lengths):
        for i in range(6 if n >= 5 and b % 3 != 1 else 0):
            t = n - 1 if i == 0 else int(rng.integers(0, n))
            # one sign to a dim, most of the time; a NaN now and then
            dims = rng.integers(0, d, size=4)
            kind = 2 if rng.random() < 0.1 else None
            for m in dims:
                c.tok[1][:, c.table[b, t // 16], :, t % 16, m] = word[int(m) % 2 if kind is None else kind]
        if b % 4 == 0 and c.counts[b] >= 2:
            c.qkv[c.start[b], (nq + nkv) * d + 5:(nq + nkv) * d + d] = float("inf")
    c.upload()
    want = c.want()
    assert np.isinf(want).any() and np.isnan(want).any() and np.isfinite(want).any()
    assert (want == np.inf).any() and (want == -np.inf).any()
    _check_rows(c, 2.0 ** -16)


@pytest.mark.parametrize("counts", [None, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_tree_scores_of_minus_infinity(counts, d):
    """The first cached keys, 40 of them, and every second drafted one give scores of minus infinity: weights of 0."""
    _say("scores of minus infinity", counts, d)
    nq, nkv = 8, 2
    sizes = _sizes(60) if counts is None else ([700, 100, 0], [counts] * 3)
    c = Case("bf16", "bf16", nq, nkv, d, *sizes, seed=d + 4, masked="chain")
    c.qkv[:, :nq * d] = c.qkv[:, :nq * d].abs() + 0.125
    c.qkv[1::2, nq * d:(nq + nkv) * d] = -float("inf")
    for b, n in enumerate(c.lengths):
        c.qkv[c.start[b]:c.start[b] + 1, nq * d:(nq + nkv) * d] = 0.5  # (the first drafted key is finite)
        for t in range(min(n, 40)):
            c.tok[0][:, c.table[b, t // 16], :, t % 16] = 0xFF80
    c.upload()
    assert np.isfinite(c.want()).all()
    _check_rows(c, 2.0 ** -16)


@pytest.mark.parametrize("cdt,n", [("bf16", 16), ("bf16", 64), ("fp8", 64), ("f32", 16)])
def test_tree_padded_rows(cdt, n):
    """Arrays with rows to spare: the same bits as without them."""
    _say("padded rows", cdt, n)
    c = Case(cdt, "f32" if cdt == "f32" else "bf16", 16, 8, 128, [300] * 24, [n] * 24, seed=n, masked="chain",
             spare_rows=6000)
    c.o = c.o.new_full((c.rows + 6000, c.o.shape[1]), 7.0)
    got = c.run(tree=c.tree(num_rows=c.rows))
    c.o.fill_(7.0)
    padded = c.run(tree=c.tree(num_rows=c.rows + 6000))
    assert bool((got == padded).all())


@pytest.mark.parametrize("cdt,dtype,eps", [("bf16", "bf16", 2.0 ** -16), ("bf16", "f32", 2.0 ** -16), ("f32", "bf16", 2.0 ** -16),
                                           ("f32", "f32", 2.0 ** -16), ("fp8", "bf16", 2.0 ** -11)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("masked", ["tree", "any"])
def test_tree_weights(cdt, dtype, eps, d, masked):
    """The weights' bits on a batch that fills the chip."""
    _say("weights", cdt, dtype, d, masked)
    _check_rows(Case(cdt, dtype, 8, 2, d, *_sizes(60), seed=d + 5, masked=masked), eps)


@pytest.mark.parametrize("cdt,dtype", [("bf16", "bf16"), ("fp8", "bf16"), ("fp8", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [3, 8])
def test_tree_weights_of_few_columns(cdt, dtype, d, n):
    """Up to 32 columns: 16 bits whatever the cache."""
    _say("weights of few columns", cdt, dtype, d, n)
    _check_rows(Case(cdt, dtype, 8, 2, d, [700, 0, 33, 5000], [n, n, 1, n], seed=d + n), 2.0 ** -16)


@pytest.mark.parametrize("cdt,dtype,eps", [("bf16", "bf16", 2.0 ** -16), ("fp8", "bf16", 2.0 ** -11), ("f32", "f32", 2.0 ** -16)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts", [None, 3])
def test_tree_rising_scores(cdt, dtype, eps, d, counts):
    """Scores that rise along the cache to several hundred, the largest among the last drafted keys: the running
    maximum moves again and again."""
    if cdt == "fp8" and counts:
        eps = 2.0 ** -16
    _say("rising scores", cdt, dtype, d, counts)
    nq, nkv = 8, 2
    sizes = _sizes(60) if counts is None else ([700, 0, 3000], [counts] * 3)
    c = Case(cdt, dtype, nq, nkv, d, *sizes, seed=d + 6, masked="chain")
    c.qkv[:, :nq * d] = c.qkv[:, :nq * d] + 3.0
    rng = np.random.default_rng(d)
    for b, n in enumerate(c.lengths):
        for p in range(-(-n // 16)):
            t = np.minimum(np.arange(16 * p, 16 * p + 16), n)
            x = (t[:, None] / max(n, 1) * 9 + rng.normal(size=(16, d)) * 0.1).astype(np.float32)
            page = c.table[b, p]
            if cdt == "fp8":
                c.scale[0][:, page] = 0.03125
                x = gc.to_e4m3(x.astype(np.float64) * 32)
            else:
                x = gc.to_bf16(x) if cdt == "bf16" else x.view(np.uint32)
            c.tok[0][:, page, :, :min(16, n - 16 * p)] = x[:min(16, n - 16 * p)]
        m = c.counts[b]
        for t in range(m):
            c.qkv[c.start[b] + t, nq * d:(nq + nkv) * d] += 9 + t / 8
    c.upload()
    _check_rows(c, eps, scores=60)
