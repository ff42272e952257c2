"""kvprm_write_kv and kvprm_read_kv on the GPU, bit for bit against the oracle: stored words, scales and
everything that the calls leave alone. (Scales are powers of two, so that every value has one right
code; code times scale is one fp32 product, which the oracle rounds the same way.)"""
import numpy as np
import pytest
import torch

from oracle import growing_cache as gc

from gpu_common import kv

pytestmark = pytest.mark.gpu
NKV, LAYERS, LAYER = 3, 2, 1
T = {"f32": torch.float32, "bf16": torch.bfloat16}


def _say(*a):
    print("case:", *a, flush=True)


class Cache:
    """A pool of random valid values, its token-major copy on the host, and the handle."""

    def __init__(self, dtype, d, lengths, rows, seed=0, spare=3, bad_table=False):
        rng = np.random.default_rng(seed)
        self.m, self.dtype, self.d, self.lengths = kv(), dtype, d, list(lengths)
        want = [-(-(n + r) // 16) for n, r in zip(lengths, rows)]
        self.pages, width = sum(want) + spare, max(want + [1]) + 1
        ids = rng.permutation(self.pages)
        self.table = np.full((len(lengths), width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(want):
            self.table[b, :n] = ids[at:at + n]
            at += n
        shape = (LAYERS, self.pages, NKV, 16, d)
        self.tok, self.scale = [], []
        for _ in (0, 1):
            x = rng.normal(size=shape).astype(np.float32)
            if dtype == "f32":
                self.tok.append(x.view(np.uint32))
            elif dtype == "bf16":
                self.tok.append(gc.to_bf16(x))
            else:
                self.tok.append(gc.to_e4m3(np.clip(x * 100.0, -448, 448).astype(np.float64)))
            # scales of several kinds: powers of two and not
            s = np.exp2(rng.integers(-9, -5, size=shape[:3])) * rng.choice([1.0, 1.0, 1.3, 1.99], size=shape[:3])
            self.scale.append(s.astype(np.float32))
        self.upload()
        self.h = self.m.kvprm_create(self.m.make_desc(LAYERS, 64 * NKV, NKV, NKV, d, 64,
                                                      weight_dtype="f32" if dtype == "f32" else "bf16",
                                                      kv_dtype=dtype))

    def upload(self):
        self.pool = [torch.from_numpy(np.stack([gc.store(t[l], part) for l in range(LAYERS)])
                                      .view(np.uint8)).cuda() for part, t in enumerate(self.tok)]
        self.sc = [torch.from_numpy(s.copy()).cuda() for s in self.scale]
        self.dtab = torch.from_numpy(self.table).cuda()
        self.dlen = torch.tensor(self.lengths, dtype=torch.int32).cuda()
        fp8 = self.dtype == "fp8"
        self.cache = self.m.make_cache(self.pool[0].data_ptr(), self.pool[1].data_ptr(), self.pages,
                                       *([s.data_ptr() for s in self.sc] if fp8 else (0, 0)))
        self.batch = self.m.make_batch(len(self.lengths), self.dtab.data_ptr(), self.table.shape[1],
                                       self.dlen.data_ptr(), self.lengths)

    def check(self):
        """The device's pools and scales are the host's."""
        for part in (0, 1):
            words = self.pool[part].cpu().numpy().view(gc.WORD[self.dtype])
            for l in range(LAYERS):
                got, want = gc.load(words[l], part), self.tok[part][l]
                if self.dtype == "fp8":  # NaN has two codes
                    got, want = (np.where((t & 0x7F) == 0x7F, 0x7F, t) for t in (got, want))
                if self.dtype == "bf16":
                    got, want = (np.where((t & 0x7FFF) > 0x7F80, 0x7FC0, t) for t in (got, want))
                assert np.array_equal(got, want), (part, l, np.argwhere(got != want)[:4])
            assert np.array_equal(self.sc[part].cpu().numpy(), self.scale[part]), part

    def __del__(self):
        self.m.kvprm_destroy(self.h)


def _rows(n, d, dtype, seed, sizes=(0.01, 1.0, 30.0)):
    rng = np.random.default_rng(seed)
    size = rng.choice(sizes, size=(n, 1, 1))
    return [torch.from_numpy((rng.normal(size=(n, NKV, d)) * size).astype(np.float32)).to(T[dtype])
            for _ in (0, 1)]


def _write(c, rows, dtype, counts, index=None, max_rows=None, start=None, stream=None):
    """The call with rows inside wider buffers, and the same on the host."""
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32) if start is None else start
    width = [NKV * c.d + 16, 2 * NKV * c.d]
    dev = []
    for t, w in zip(rows, width):
        buf = torch.full((max(1, len(t)), w), float("nan"), dtype=t.dtype)
        buf[:len(t), :NKV * c.d] = t.reshape(len(t), -1)
        dev.append(buf.cuda())
    ds = torch.from_numpy(start).cuda()
    di = None if index is None else torch.tensor(list(index) + [0], dtype=torch.int32).cuda()
    most = max(list(counts) + [1]) if max_rows is None else max_rows
    r = c.m.make_kv_rows(dev[0].data_ptr(), dev[1].data_ptr(), dtype, *width, len(rows[0]), ds.data_ptr(), most,
                         0 if di is None else di.data_ptr())
    st = stream or torch.cuda.current_stream()
    c.m.kvprm_write_kv(c.h, c.cache, c.batch, LAYER, r, st.cuda_stream)
    torch.cuda.synchronize()
    for part in (0, 1):
        gc.write(c.tok[part][LAYER], c.scale[part][LAYER] if c.dtype == "fp8" else None, c.dtype, c.table,
                 c.lengths, start, rows[part].float().numpy(), index, most)


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write(cdt, d, dtype):
    _say("write", cdt, d, dtype)
    lengths = [0, 0, 1, 15, 16, 17, 31, 300, 5, 47]
    counts = [1, 40, 1, 1, 1, 3, 33, 0, 16, 129]
    c = Cache(cdt, d, lengths, counts, seed=d)
    _write(c, _rows(sum(counts), d, dtype, 5), dtype, counts)
    c.check()


@pytest.mark.parametrize("cdt", ["bf16", "fp8"])
def test_write_token_by_token(cdt):
    """The same tokens one call each: scales only grow, older codes follow them."""
    _say("token by token", cdt)
    c = Cache(cdt, 128, [3, 0], [40, 40], seed=9)
    for step in range(20):
        _write(c, _rows(2, 128, "bf16", 100 + step, sizes=(0.1, 1.0, 4.0, 20.0)), "bf16", [1, 1])
        c.lengths = [n + 1 for n in c.lengths]
        c.dlen.add_(1)
        c.batch = c.m.make_batch(2, c.dtab.data_ptr(), c.table.shape[1], c.dlen.data_ptr(), c.lengths)
    c.check()


@pytest.mark.parametrize("cdt", ["f32", "fp8"])
def test_write_picked_rows(cdt):
    """Rows by index, in any order, one of them twice; rows outside the array are dropped."""
    _say("index", cdt)
    c = Cache(cdt, 64, [7, 30, 0], [5, 4, 3], seed=2)
    _write(c, _rows(20, 64, "f32", 3), "f32", [5, 4, 3], index=[19, 0, 4, 4, 7, 12, -1, 20, 3, 1, 2, 1 << 30])
    c.check()


@pytest.mark.parametrize("cdt", ["bf16", "fp8"])
def test_write_drops_what_has_no_place(cdt):
    """Rows past the page table, past max_rows, past num_rows, on page ids outside the pool, of empty
    candidates and of a start that runs past the rows."""
    _say("drops", cdt)
    c = Cache(cdt, 64, [10, 20, 3, 0], [10, 20, 10, 0], seed=4)
    c.table[1, 1], c.table[2, 0] = c.pages, -7
    c.upload()
    _write(c, _rows(200, 64, "bf16", 6), "bf16", [100, 20, 10, 0])
    c.check()
    _write(c, _rows(9, 64, "bf16", 7), "bf16", [6, 6, 6, 6], max_rows=4)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write_fp8_extremes(dtype):
    """Zero rows, the smallest and largest magnitudes, infinities and NaN, a page of nothing else."""
    _say("extremes", dtype)
    counts = [1, 1, 1, 4, 2, 16, 1, 3]
    rows = _rows(sum(counts), 64, dtype, 8)
    for t in rows:
        t[0] = 0
        t[1] = 1e-38
        t[2] = 3.0e38
        t[3, :, 5] = float("inf")
        t[4, 0, 0], t[4, 1, 1] = float("nan"), -float("inf")
        t[7] = float("nan")
        t[8] = float("-inf")
        t[9:25] = 0
        t[9, 1, 3] = 448.0
        t[10, 1, 3] = -449.0
        t[25] = -0.0
    c = Cache("fp8", 64, [0, 16, 32, 14, 48, 0, 5, 1], counts, seed=1)
    _write(c, rows, dtype, counts)
    c.check()


def test_write_on_another_stream_and_in_a_graph():
    """A captured append of one token: every replay follows the device's lengths and rows."""
    _say("graph")
    c = Cache("fp8", 128, [14, 31, 0], [8, 8, 8], seed=11)
    side = torch.cuda.Stream()
    _write(c, _rows(3, 128, "bf16", 1), "bf16", [1, 1, 1], stream=side)
    c.check()
    rows = torch.zeros((2, 3, NKV * 128), dtype=torch.bfloat16, device="cuda")
    start = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    c.batch = c.m.make_batch(3, c.dtab.data_ptr(), c.table.shape[1], c.dlen.data_ptr())
    r = c.m.make_kv_rows(rows[0].data_ptr(), rows[1].data_ptr(), "bf16", NKV * 128, NKV * 128, 3, start.data_ptr(), 1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.m.kvprm_write_kv(c.h, c.cache, c.batch, LAYER, r, torch.cuda.current_stream().cuda_stream)
    for step in range(5):
        c.lengths = [n + 1 for n in c.lengths]
        c.dlen.add_(1)
        new = _rows(3, 128, "bf16", 50 + step)
        rows.copy_(torch.stack(new).reshape(2, 3, -1))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for part in (0, 1):
            gc.write(c.tok[part][LAYER], c.scale[part][LAYER], "fp8", c.table, c.lengths, [0, 1, 2, 3],
                     new[part].float().numpy())
        c.check()
    del g


def _read(c, dtype, counts, first=None, parts=(0, 1), num_rows=None, max_rows=None):
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n, width = int(start[-1]), NKV * c.d + 8
    out = [torch.full((n + 2, width), 7.0, dtype=T[dtype], device="cuda") for _ in (0, 1)]
    ds = torch.from_numpy(start).cuda()
    df = None if first is None else torch.tensor(first, dtype=torch.int32).cuda()
    ptr = [out[p].data_ptr() if p in parts else 0 for p in (0, 1)]
    r = c.m.make_kv_rows(*ptr, dtype, width, width, n if num_rows is None else num_rows, ds.data_ptr(),
                         max(counts + [1]) if max_rows is None else max_rows)
    c.m.kvprm_read_kv(c.h, c.cache, c.batch, LAYER, r, 0 if df is None else df.data_ptr(),
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for part in (0, 1):
        want = torch.full((n + 2, width), 7.0, dtype=T[dtype])
        for b, L in enumerate(c.lengths):
            p0 = first[b] if first is not None else 0
            v = gc.cached(c.tok[part][LAYER], c.scale[part][LAYER], c.dtype, c.table[b], L)
            for i in range(min(counts[b], counts[b] if max_rows is None else max_rows)):
                row = start[b] + i
                if part in parts and 0 <= p0 + i < L and (num_rows is None or row < num_rows):
                    # one fp32 product, then the rows' rounding
                    x = torch.from_numpy(v[p0 + i].astype(np.float32)).to(T[dtype])
                    want[row, :NKV * c.d] = x.reshape(-1)
        assert torch.equal(out[part].cpu(), want), part


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read(cdt, d, dtype):
    _say("read", cdt, d, dtype)
    lengths = [0, 1, 15, 16, 17, 300, 40]
    c = Cache(cdt, d, lengths, [0] * 7, seed=d + 1)
    _read(c, dtype, lengths)
    _read(c, dtype, [0, 1, 3, 5, 17, 100, 7], first=[0, 0, 12, 11, 0, 199, 33])


def test_read_leaves_other_rows():
    """Positions outside the cache, rows past num_rows and max_rows, one part alone."""
    _say("read outside")
    c = Cache("fp8", 64, [20, 33, 0, 16], [0] * 4, seed=3)
    _read(c, "bf16", [30, 10, 4, 8], first=[-5, 30, 0, 20])
    _read(c, "f32", [20, 33, 0, 16], num_rows=40)
    _read(c, "f32", [20, 33, 0, 16], max_rows=17)
    _read(c, "bf16", [20, 33, 0, 16], parts=(1,))
    _read(c, "bf16", [20, 33, 0, 16], parts=(0,))
    c.table[1, 1], c.table[3, 0] = c.pages, -7
    c.dtab.copy_(torch.from_numpy(c.table))
    want = c.table.copy()
    out = torch.full((69, NKV * 64), 7.0, device="cuda")
    start = torch.tensor([0, 20, 53, 53, 69], dtype=torch.int32, device="cuda")
    r = c.m.make_kv_rows(out.data_ptr(), 0, "f32", NKV * 64, NKV * 64, 69, start.data_ptr(), 33)
    c.m.kvprm_read_kv(c.h, c.cache, c.batch, LAYER, r, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(c.dtab.cpu().numpy(), want)
    lost = (out == 7.0).all(dim=1).cpu().numpy()
    assert np.array_equal(np.flatnonzero(lost), np.concatenate([np.arange(36, 52), np.arange(53, 69)]))


def test_read_far_outside():
    """More rows than the page table has slots, most of them at positions below 0 or past the cache."""
    _say("read far outside")
    c = Cache("bf16", 64, [20, 33, 0, 16], [0] * 4, seed=11)
    _read(c, "bf16", [300, 200, 90, 400], first=[-250, -190, -50, -399])
    _read(c, "bf16", [300, 2, 90, 4], first=[-2 ** 31, 2 ** 31 - 1, 2 ** 31 - 16, 15])


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8"])
def test_write_then_read(cdt):
    """What fp32 rows become in the cache comes back within half a step of its type (fp8: of the
    tile's scale too)."""
    _say("round trip", cdt)
    counts = [70, 1, 16]
    c = Cache(cdt, 128, [0, 0, 0], counts, seed=6)
    rows = _rows(87, 128, "f32", 2, sizes=(1.0,))
    _write(c, rows, "f32", counts)
    c.lengths = counts
    c.upload()
    c.check()
    _read(c, "f32", counts)
    half = {"f32": 0.0, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}[cdt]
    for part in (0, 1):
        for b, n in enumerate(counts):
            v = gc.cached(c.tok[part][LAYER], c.scale[part][LAYER], cdt, c.table[b], n)
            x = rows[part][sum(counts[:b]):sum(counts[:b + 1])].double().numpy()
            # (below e4m3's normal range, 2^-6 of the scale, half a step is 2^-10 of it)
            assert np.all(np.abs(v - x) <= half * np.abs(x) + (0 if cdt != "fp8" else 2.0 ** -10 * c.scale[part].max()))


def test_write_debug_refusals(monkeypatch):
    """KVPRM_DEBUG=1: what would be dropped, and a page that would get rows twice, is refused on the host;
    nothing is written. A good call passes."""
    _say("debug")
    monkeypatch.setenv("KVPRM_DEBUG", "1")
    counts = [6, 20]

    def call(table=None, lengths=None, start=None):
        c = Cache("fp8", 64, [10, 20], counts, seed=8)
        if table is not None:
            c.table[table[0], table[1]] = table[2] if len(table) == 3 else c.table[table[3], table[4]]
            c.upload()
        if lengths is not None:
            c.dlen.copy_(torch.tensor(lengths, dtype=torch.int32))
        before = [t.clone() for t in c.pool + c.sc]
        rows = [t.cuda() for t in _rows(26, 64, "bf16", 9)]
        ds = torch.tensor([0, 6, 26] if start is None else start, dtype=torch.int32).cuda()
        r = c.m.make_kv_rows(rows[0].data_ptr(), rows[1].data_ptr(), "bf16", NKV * 64, NKV * 64, 26, ds.data_ptr(), 20)
        refused = None
        try:
            c.m.kvprm_write_kv(c.h, c.cache, c.batch, LAYER, r, torch.cuda.current_stream().cuda_stream)
        except RuntimeError as e:
            refused = str(e)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(before, c.pool + c.sc)) == (refused is not None)
        return refused

    assert call() is None
    for bad in (dict(table=(0, 0, -1)), dict(table=(1, 2, 1 << 20)), dict(table=(1, 1, None, 0, 0)),
                dict(table=(1, 2, None, 1, 1)), dict(lengths=[10, 60]), dict(lengths=[-1, 20]), dict(start=[0, 6, 27]),
                dict(start=[-1, 6, 26]), dict(start=[0, 6, 5])):
        assert "kvprm_write_kv" in call(**bad)
