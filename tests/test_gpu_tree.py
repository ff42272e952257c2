"""kvprm_attention_tree on the GPU against the fp64 oracle.

Tolerance: with |q|, |k| entries near N(0, 1) and d <= 128, a score's fp32 sum of d products is off by at
most d 2^-24 sum|q k| / sqrt(d) ~ 128 * 2^-24 * 0.64 sqrt(128) = 5.5e-5 if every rounding went one way, and
by the root of d of them, 5e-6, as they fall; the weights follow it (e^x), the hardware exp2 adds 2^-22, the
weights' rounding half a step of fp16, 2^-11 (bf16 rows; 2^-16, two bf16 terms, up to 32 columns), or 2^-24 (fp32
rows, three terms), the sums' roundings 2^-24 each. An output is a mean of values of size max|v| with these
weights, so its error is within 2 * 1e-5 max|v| (fp32 rows), or (2^-11 + 2 * 1e-5) max|v| and the result's own
half step 2^-8 |o| (bf16 rows)."""
import math

import numpy as np
import pytest
import torch

from oracle import growing_cache as gc

from gpu_common import kv

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16}
LAYERS, LAYER = 2, 1


def _say(*a):
    print("case:", *a, flush=True)


class Case:
    """Caches, drafts and masks of a batch. Slots past a length, pages of nobody and rows of nobody hold
    NaN."""

    def __init__(self, cdt, dtype, nq, nkv, d, lengths, counts, seed=0, masked="tree", spare_rows=2):
        rng = np.random.default_rng(seed)
        self.m, self.cdt, self.dtype, self.shape = kv(), cdt, dtype, (nq, nkv, d)
        self.lengths, self.counts = list(lengths), list(counts)
        want = [-(-n // 16) for n in lengths]
        self.pages, self.width = sum(want) + 3, max(want + [1]) + 1
        ids = rng.permutation(self.pages)
        self.table = np.full((len(lengths), self.width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(want):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.tok, self.scale = [], []
        for _ in (0, 1):
            x = rng.normal(size=(LAYERS, self.pages, nkv, 16, d)).astype(np.float32)
            s = np.exp2(rng.integers(-8, -6, size=x.shape[:3])) * 1.25
            if cdt == "fp8":
                w = gc.to_e4m3(np.clip(x / s[..., None, None], -448, 448).astype(np.float64))
            else:
                w = gc.to_bf16(x) if cdt == "bf16" else x.view(np.uint32)
            nan = {"f32": np.uint32(0x7FC00000), "bf16": np.uint16(0x7FC0), "fp8": np.uint8(0x7F)}[cdt]
            mine = np.zeros((self.pages, 16), dtype=bool)
            for b, n in enumerate(lengths):
                for p in range(want[b]):
                    mine[self.table[b, p], :min(16, n - 16 * p)] = True
            w[np.broadcast_to(~mine[None, :, None, :, None], w.shape)] = nan
            self.tok.append(w)
            self.scale.append(s.astype(np.float32))
        n = self.rows = sum(counts)
        self.start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        pad = 8
        w = (nq + 2 * nkv) * d + pad
        x = rng.normal(size=(n + spare_rows, w)).astype(np.float32)
        x[n:] = np.nan
        x[:, w - pad:] = np.nan
        self.qkv = torch.from_numpy(x).to(T[dtype])
        self.sees = [self._mask(rng, c, masked) for c in counts]
        self.masked = masked
        self.words = (max(counts + [1]) + 31) // 32 + 1
        bits = np.zeros((n + spare_rows, self.words), dtype=np.uint32)
        bits[n:] = 0xFFFFFFFF
        for b, c in enumerate(counts):
            for j in range(32 * self.words):  # bits past the candidate's tokens are set
                on = self.sees[b][:, j] if j < c else np.ones(c, bool)
                bits[self.start[b]:self.start[b] + c, j // 32] |= on.astype(np.uint32) << np.uint32(j % 32)
        self.bits = bits
        self.upload()
        self.h = self.m.kvprm_create(self.m.make_desc(LAYERS, 64 * nq, nq, nkv, d, 64,
                                                      weight_dtype="f32" if cdt == "f32" else "bf16",
                                                      kv_dtype=cdt))

    @staticmethod
    def _mask(rng, n, kind):
        sees = np.tril(np.ones((n, n), bool))
        if kind == "tree":
            for t in range(n):
                sees[t] = False
                p = int(rng.integers(-1, t)) if t else -1
                if p >= 0:
                    sees[t] = sees[p]
                sees[t, t] = True
        if kind == "any":
            sees = rng.random((n, n)) < 0.3
            sees[::3] = False
        if kind == "none":
            sees[:] = False
        return sees

    def upload(self):
        self.pool = [torch.from_numpy(np.stack([gc.store(t[l], part) for l in range(LAYERS)])
                                      .view(np.uint8)).cuda() for part, t in enumerate(self.tok)]
        self.sc = [torch.from_numpy(s).cuda() for s in self.scale]
        self.dtab, self.dstart = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.start).cuda()
        self.dlen = torch.tensor(self.lengths, dtype=torch.int32).cuda()
        self.dqkv, self.dbits = self.qkv.cuda(), torch.from_numpy(self.bits.view(np.int32)).cuda()
        nq, nkv, d = self.shape
        self.o = torch.full((self.rows + 2, nq * d + 8), 7.0, dtype=T[self.dtype], device="cuda")
        self.cache = self.m.make_cache(self.pool[0].data_ptr(), self.pool[1].data_ptr(), self.pages,
                                       *([s.data_ptr() for s in self.sc] if self.cdt == "fp8" else (0, 0)))

    def batch(self, host=True):
        return self.m.make_batch(len(self.lengths), self.dtab.data_ptr(), self.width, self.dlen.data_ptr(),
                                 self.lengths if host else None)

    def tree(self, max_rows=None, num_rows=None):
        nq, nkv, d = self.shape
        e, w, at = self.dqkv.element_size(), self.dqkv.shape[1], self.dqkv.data_ptr()
        chain = self.masked == "chain"
        return self.m.make_tree(at, at + nq * d * e, at + (nq + nkv) * d * e, self.o.data_ptr(), self.dtype, w, w, w,
                                nq * d + 8, self.rows + 2 if num_rows is None else num_rows,
                                self.dstart.data_ptr(), max(self.counts + [1]) if max_rows is None else max_rows,
                                0 if chain else self.dbits.data_ptr(), 0 if chain else self.words)

    def run(self, host=True, stream=None, tree=None):
        b, t = self.batch(host), tree or self.tree()
        n = self.m.kvprm_workspace_size_tree(self.h, b, t)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # (fp32 NaN)
        st = stream or torch.cuda.current_stream()
        st.wait_stream(torch.cuda.current_stream())
        self.m.kvprm_attention_tree(self.h, self.cache, b, LAYER, t, ws.data_ptr(), n, st.cuda_stream)
        torch.cuda.synchronize()
        return self.o.cpu()

    def want(self):
        nq, nkv, d = self.shape
        out = []
        for b, (n, c) in enumerate(zip(self.lengths, self.counts)):
            x = self.qkv[self.start[b]:self.start[b] + c].double().numpy()
            ck, cv = (gc.cached(self.tok[p][LAYER], self.scale[p][LAYER], self.cdt, self.table[b], n) for p in (0, 1))
            out.append(gc.tree_attention(x[:, :nq * d].reshape(c, nq, d), x[:, nq * d:(nq + nkv) * d].reshape(c, nkv, d),
                                         x[:, (nq + nkv) * d:(nq + 2 * nkv) * d].reshape(c, nkv, d), ck, cv,
                                         self.sees[b]).reshape(c, nq * d))
        return np.concatenate(out)

    def check(self, got=None, big=None):
        got, want = self.run() if got is None else got, self.want()
        nq, nkv, d = self.shape
        assert torch.all(got[:, nq * d:] == 7.0) and torch.all(got[self.rows:] == 7.0)
        y = got[:self.rows, :nq * d].double().numpy()
        assert np.array_equal(np.isfinite(y), np.isfinite(want))
        assert np.array_equal(np.isnan(y), np.isnan(want))
        fine = np.isfinite(want)
        size = 5.0 if big is None else big  # max|v| of N(0, 1) values
        tol = 2e-5 * size if self.dtype == "f32" else (2.0 ** -11 + 2e-5) * size + 2.0 ** -8 * np.abs(want[fine])
        err = np.abs(y[fine] - want[fine])
        assert np.all(err <= tol), (float(err.max()), float(np.max(err - tol)))

    def __del__(self):
        self.m.kvprm_destroy(self.h)


@pytest.mark.parametrize("cdt,dtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"),
                                       ("fp8", "bf16"), ("fp8", "f32")])
@pytest.mark.parametrize("nq,nkv,d", [(2, 2, 64), (4, 2, 128), (7, 1, 128), (16, 1, 64)])
@pytest.mark.parametrize("masked", ["tree", "any"])
def test_tree(cdt, dtype, nq, nkv, d, masked):
    _say("tree", cdt, dtype, nq, nkv, d, masked)
    lengths = [0, 1, 15, 16, 17, 32, 33, 129, 700]
    counts = [1, 3, 5, 1, 17, 0, 9, 40, 33]
    Case(cdt, dtype, nq, nkv, d, lengths, counts, seed=nq + d, masked=masked).check()


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("n", [1, 2, 4, 8, 16, 23, 31, 64, 100, 256])
def test_tree_sizes(cdt, n):
    """Every number of column tiles, drafts of one size, caches of one and several chunks."""
    _say("sizes", cdt, n)
    Case(cdt, "bf16", 4, 2, 64, [40, 0, 1500], [n, n, max(1, n - 1)], seed=n).check()


@pytest.mark.parametrize("cdt,dtype", [("f32", "f32"), ("bf16", "bf16"), ("fp8", "bf16"), ("fp8", "f32")])
def test_tree_chain(cdt, dtype):
    _say("chain", cdt, dtype)
    Case(cdt, dtype, 6, 2, 128, [100, 0, 17], [8, 40, 1], masked="chain").check()


@pytest.mark.parametrize("cdt,dtype,n", [("bf16", "bf16", 3), ("fp8", "bf16", 30), ("bf16", "f32", 9), ("f32", "f32", 2),
                                         ("bf16", "bf16", 50)])
def test_tree_many_chunks(cdt, dtype, n):
    """Long caches, chunks with and without host lengths (another chunk length: other sums, same
    values), and the same bits when the call is repeated."""
    _say("many chunks", cdt, dtype, n)
    c = Case(cdt, dtype, 4, 1, 128, [9001, 5, 4096], [n, 1, n], seed=n)
    got = c.run()
    c.check(got)
    assert torch.equal(got, c.run())
    c.check(c.run(host=False))


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_rows_that_see_nothing(cdt, dtype):
    """No cache and no bits: zeros. A cache and no bits: the cache alone."""
    _say("nothing", cdt, dtype)
    c = Case(cdt, dtype, 4, 2, 64, [0, 33, 0], [5, 20, 40], masked="none")
    got = c.run()
    c.check(got)
    assert torch.all(got[:5, :256] == 0) and torch.all(got[25:65, :256] == 0)


@pytest.mark.parametrize("cdt,dtype", [("f32", "f32"), ("bf16", "bf16"), ("fp8", "f32")])
def test_tree_infinities_and_nan_where_masked(cdt, dtype):
    """Drafted keys and values that hold infinities and NaN reach the tokens that attend to them and no
    other one."""
    _say("inf and nan", cdt, dtype)
    nq, nkv, d = 4, 2, 64
    c = Case(cdt, dtype, nq, nkv, d, [50, 0], [40, 20], seed=3)
    for b, t, what, value in ((0, 7, "v", math.inf), (0, 20, "v", -math.inf), (0, 39, "v", math.nan),
                              (0, 12, "k", math.nan), (1, 3, "v", math.nan), (1, 19, "v", math.inf)):
        at = (nq + (nkv if what == "v" else 0)) * d
        c.qkv[c.start[b] + t, at + 3:at + 70:5] = value
        # (of each, the later half of the tokens does not see it)
        c.sees[b][len(c.sees[b]) // 2:, t] = False
    c.bits[:] = 0
    for b, s in enumerate(c.sees):
        for j in range(len(s)):
            c.bits[c.start[b]:c.start[b] + len(s), j // 32] |= s[:, j].astype(np.uint32) << np.uint32(j % 32)
    c.upload()
    got = c.run()
    want = c.want()
    assert np.isnan(want).any() and np.isinf(want).any()
    assert np.isfinite(want[20:40]).all() and np.isfinite(want[50:60]).all()
    # (a weight of exactly the sort that underflows would turn infinity into NaN on both sides alike;
    # scores here lie within 30 of each other)
    c.check(got)


@pytest.mark.parametrize("cdt,dtype", [("bf16", "f32"), ("fp8", "bf16"), ("f32", "f32")])
def test_tree_large_scores(cdt, dtype):
    """Scores of several hundred: the softmax is nearly one-hot, nothing overflows. A score s is off by
    about 2^-24 |s| sqrt(d) / 2 here, so tolerances are 60 times those of scores near one."""
    _say("large scores", cdt, dtype)
    c = Case(cdt, dtype, 4, 2, 64, [300, 0], [20, 10], seed=4)
    c.qkv[:, :256] *= 60
    c.upload()
    c.check(big=5.0 * 60)


def test_tree_drops_rows():
    """Rows past max_rows and num_rows are left alone; the others are as in the whole call. (Fewer rows can
    mean another kernel, whose sums have another order: each result is within the tolerance of 64 bits,
    so their difference is within two of them.)"""
    _say("drops rows")
    c = Case("bf16", "bf16", 4, 2, 64, [40, 100], [12, 30], seed=5, masked="chain")
    full = c.run()
    c.check(full)

    def same(x, y):
        x, y = x[:, :256].double(), y[:, :256].double()
        return bool(torch.all((x - y).abs() <= 2 * (5 * (2.0 ** -11 + 2e-5) + 2.0 ** -8 * y.abs())))

    c.o.fill_(7.0)
    got = c.run(tree=c.tree(max_rows=10))
    assert same(got[:10], full[:10]) and torch.all(got[10:12] == 7.0)
    assert same(got[12:22], full[12:22]) and torch.all(got[22:] == 7.0)
    c.o.fill_(7.0)
    got = c.run(tree=c.tree(num_rows=20))
    assert same(got[:20], full[:20]) and torch.all(got[20:] == 7.0)


def test_tree_without_pages():
    """Every cache empty: drafted tokens alone."""
    _say("no pages")
    Case("fp8", "bf16", 28, 4, 128, [0, 0], [5, 70], seed=6).check()


def test_tree_two_streams():
    """Two calls at once on streams of their own, each with its workspace."""
    _say("two streams")
    cs = [Case("bf16", "bf16", 8, 2, 128, [3000, 77], [20, 5], seed=s) for s in (7, 8)]
    want = [c.run() for c in cs]
    for c in cs:
        c.o.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    keep = []
    for c, st in zip(cs, streams):
        b, t = c.batch(), c.tree()
        n = c.m.kvprm_workspace_size_tree(c.h, b, t)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        keep.append((b, t, ws))
    torch.cuda.synchronize()
    for _ in range(4):
        for c, st, (b, t, ws) in zip(cs, streams, keep):
            c.m.kvprm_attention_tree(c.h, c.cache, b, LAYER, t, ws.data_ptr(), ws.numel(), st.cuda_stream)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        assert torch.equal(c.o.cpu(), w)


def test_tree_in_a_graph():
    """One captured call without host lengths: replays follow the lengths, drafts and masks on the
    device, with eager work between them, and equal the eager call bit for bit."""
    _say("graph")
    c = Case("bf16", "bf16", 8, 2, 128, [3000, 77, 500], [20, 5, 9], seed=9)
    b, t = c.batch(host=False), c.tree()
    n = c.m.kvprm_workspace_size_tree(c.h, b, t)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def call():
        c.m.kvprm_attention_tree(c.h, c.cache, b, LAYER, t, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    junk = torch.randn(1 << 20, device="cuda")
    for lengths in ([3000, 77, 500], [1, 0, 16], [2999, 64, 33]):
        c.dlen.copy_(torch.tensor(lengths, dtype=torch.int32))
        c.dqkv.mul_(-0.5)
        c.dbits[:c.rows] ^= 0b101
        got = []
        for run in (call, g.replay, g.replay):
            c.o.fill_(7.0)
            junk.mul_(1.0001).add_(0.5)
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            got.append(c.o.clone())
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
        assert torch.all(torch.isfinite(got[0]))
    del g


def test_one_drafted_token_is_the_attention_step():
    """A draft of one token that sees itself is kvprm_attention with its own key (fp32 rows; both are
    within 1e-5 max|v| of 64 bits)."""
    _say("against kvprm_attention")
    c = Case("bf16", "f32", 8, 2, 128, [1000, 0, 17], [1, 1, 1], seed=10)
    got = c.run()[:3, :1024].reshape(3, 8, 128)
    b = c.batch()
    x = c.dqkv[:3]
    q, k, v = (x[:, i:j].contiguous() for i, j in ((0, 1024), (1024, 1280), (1280, 1536)))
    n = c.m.kvprm_workspace_size(c.h, b)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    o = torch.empty((3, 8, 128), device="cuda")
    c.m.kvprm_attention(c.h, c.cache, b, LAYER, q.data_ptr(), k.data_ptr(), v.data_ptr(), ws.data_ptr(), n,
                        o.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert float((o.cpu() - got).abs().max()) <= 2 * 5.0 * 1e-5
