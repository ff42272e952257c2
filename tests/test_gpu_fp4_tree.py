"""kvprm_attention_tree over 4-bit caches against the fp64 oracle.

Tolerance: as over bf16 caches (the stored values are bf16 values): scores within 1e-5 as their roundings fall, weights
in two bf16 terms (2^-16, bf16 rows) or three (fp32 rows), an output is a mean of values with these weights: within
2 * 1e-5 max|v| (fp32 rows) or (2^-16 + 2 * 1e-5) max|v| and the result's own half step 2^-8 |o| (bf16 rows)."""
import numpy as np
import pytest
import torch

from oracle import growing_cache as gc

from fp4_common import T, Cache

pytestmark = pytest.mark.gpu
LAYER = 1


def _say(*a):
    print("case:", *a, flush=True)


def _mask(rng, n, kind):
    sees = np.tril(np.ones((n, n), bool))
    if kind == "tree":
        for t in range(n):
            p = int(rng.integers(-1, t)) if t else -1
            sees[t] = sees[p] if p >= 0 else False
            sees[t, t] = True
    if kind == "any":
        sees = rng.random((n, n)) < 0.3
        sees[::3] = False
    return sees


class Draft:
    def __init__(self, c, dtype, counts, kind, seed=0, spare=2):
        rng = np.random.default_rng(seed)
        nq, nkv, d = c.shape
        self.c, self.dtype, self.counts, self.kind = c, dtype, counts, kind
        n = self.rows = sum(counts)
        self.start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        x = rng.normal(size=(n + spare, (nq + 2 * nkv) * d + 8)).astype(np.float32)
        x[n:] = np.nan
        self.x = torch.from_numpy(x).to(T[dtype])
        self.sees = [_mask(rng, k, kind) for k in counts]
        self.words = (max(counts + [1]) + 31) // 32
        bits = np.zeros((n + spare, self.words), dtype=np.uint32)
        for b, k in enumerate(counts):
            for j in range(32 * self.words):  # bits past the candidate's tokens are set
                on = self.sees[b][:, j] if j < k else np.ones(k, bool)
                bits[self.start[b]:self.start[b] + k, j // 32] |= on.astype(np.uint32) << np.uint32(j % 32)
        self.dx, self.dbits = self.x.cuda(), torch.from_numpy(bits.view(np.int32)).cuda()
        self.dstart = torch.from_numpy(self.start).cuda()
        self.o = torch.full((n + spare, nq * d + 8), 7.0, dtype=T[dtype], device="cuda")

    def run(self, host=True, stream=None):
        c, m = self.c, self.c.m
        nq, nkv, d = c.shape
        e, w, at = self.dx.element_size(), self.dx.shape[1], self.dx.data_ptr()
        t = m.make_tree(at, at + nq * d * e, at + (nq + nkv) * d * e, self.o.data_ptr(), self.dtype, w, w, w, nq * d + 8,
                        self.rows + 2, self.dstart.data_ptr(), max(self.counts + [1]),
                        0 if self.kind == "chain" else self.dbits.data_ptr(), self.words)
        batch = c.batch if host else m.make_batch(len(c.lengths), c.dtab.data_ptr(), c.width, c.dlen.data_ptr())
        n = m.kvprm_workspace_size_tree(c.h, batch, t)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        st = stream or torch.cuda.current_stream()
        st.wait_stream(torch.cuda.current_stream())
        m.kvprm_attention_tree(c.h, c.cache, batch, LAYER, t, ws.data_ptr(), n, st.cuda_stream)
        torch.cuda.synchronize()
        return self.o.cpu()

    def check(self, got):
        c = self.c
        nq, nkv, d = c.shape
        assert torch.all(got[:, nq * d:] == 7.0) and torch.all(got[self.rows:] == 7.0)
        for b, (L, k) in enumerate(zip(c.lengths, self.counts)):
            x = self.x[self.start[b]:self.start[b] + k].double().numpy()
            ck, cv = (c.cached(p, LAYER, b) for p in (0, 1))
            v = x[:, (nq + nkv) * d:(nq + 2 * nkv) * d].reshape(k, nkv, d)
            want = gc.tree_attention(x[:, :nq * d].reshape(k, nq, d), x[:, nq * d:(nq + nkv) * d].reshape(k, nkv, d), v, ck,
                                     cv, self.sees[b]).reshape(k, nq * d)
            y = got[self.start[b]:self.start[b] + k, :nq * d].double().numpy()
            big = max([np.abs(t).max() for t in (cv, v) if t.size] + [0.0])
            tol = 2e-5 * big if self.dtype == "f32" else (2.0 ** -16 + 2e-5) * big + 2.0 ** -8 * np.abs(want)
            assert np.all(np.abs(y - want) <= tol), (b, np.abs(y - want).max(), big)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,d", [(4, 2, 64), (14, 2, 128), (16, 1, 128), (6, 3, 64)])
@pytest.mark.parametrize("kind", ["tree", "chain", "any"])
def test_drafts(dtype, nq, nkv, d, kind):
    """Few columns and many, ragged drafts, empty caches and drafts, chunks."""
    _say("drafts", dtype, nq, nkv, d, kind)
    c = Cache(nq, nkv, d, [0, 1, 16, 33, 100, 257, 40], seed=d)
    dr = Draft(c, dtype, [5, 1, 3, 40, 0, 17, 2], kind, seed=nq)
    dr.check(dr.run())
    dr.check(dr.run(host=False))


@pytest.mark.parametrize("nq,nkv,d,lengths,counts", [
    (8, 4, 128, [1103], [16]), (28, 4, 128, [2500, 900], [64, 33]), (16, 4, 64, [3000, 5, 700], [48, 48, 1]),
    (16, 8, 128, [1500] * 12, [64] * 12), (8, 2, 64, [900] * 24, [96] * 24), (4, 4, 128, [300], [256])])
def test_long(nq, nkv, d, lengths, counts):
    """Batches that fill the chip and that do not: every kernel form."""
    _say("long", nq, nkv, d, lengths[:3])
    c = Cache(nq, nkv, d, lengths, seed=nq)
    for dtype in ("bf16", "f32"):
        dr = Draft(c, dtype, counts, "tree", seed=2)
        dr.check(dr.run())


def test_nan_tokens_and_masked_drafts():
    """A stored NaN reaches every draft of its candidate; infinities and NaN among drafted rows reach those that see
    them."""
    _say("nan")
    for counts in ([4, 4], [60, 60]):
        c = Cache(4, 2, 128, [90, 200], seed=4)
        c.scale[1][LAYER, c.table[0, 3], 1, 5, 2] = 255  # a value: dims 64 .. 95 of kv-head 1
        c.upload()
        dr = Draft(c, "bf16", counts, "chain", seed=5)
        nq, nkv, d = c.shape
        got = dr.run()[:dr.rows, :nq * d].reshape(-1, nq, d).isnan().numpy()
        want = np.zeros(got.shape, bool)
        want[:counts[0], 2:, 64:96] = True
        assert np.array_equal(got, want)


def test_streams_and_repeats():
    _say("streams")
    c = Cache(16, 4, 128, [2000, 700, 30], seed=6)
    for counts in ([5, 3, 6], [64, 50, 64]):
        dr = Draft(c, "bf16", counts, "tree", seed=7)
        first = dr.run().clone()
        dr.check(first)
        for _ in range(3):
            assert torch.equal(first, dr.run(stream=torch.cuda.Stream()))
