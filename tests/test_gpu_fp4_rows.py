"""kvprm_write_kv and kvprm_read_kv on 4-bit caches, byte for byte against the oracle (scales are powers of two, so
that every value has one right code), and everything that the calls leave alone."""
import numpy as np
import pytest
import torch

from oracle import fp4

from fp4_common import T, Cache

pytestmark = pytest.mark.gpu
NKV, LAYER = 3, 1


def _say(*a):
    print("case:", *a, flush=True)


def _cache(d, lengths, counts=None, **o):
    return Cache(NKV, NKV, d, lengths, counts, **o)


def _rows(n, d, dtype, seed, sizes=(0.01, 1.0, 30.0)):
    rng = np.random.default_rng(seed)
    size = rng.choice(sizes, size=(n, 1, 1))
    return [torch.from_numpy((rng.normal(size=(n, NKV, d)) * size).astype(np.float32)).to(T[dtype]) for _ in (0, 1)]


def _write(c, rows, dtype, counts, index=None, max_rows=None, start=None, stream=None):
    """The call with rows inside wider buffers, and the same on the host."""
    d = c.shape[2]
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32) if start is None else start
    width = [NKV * d + 16, 2 * NKV * d]
    dev = []
    for t, w in zip(rows, width):
        buf = torch.full((max(1, len(t)), w), float("nan"), dtype=t.dtype)
        buf[:len(t), :NKV * d] = t.reshape(len(t), -1)
        dev.append(buf.cuda())
    ds = torch.from_numpy(start).cuda()
    di = None if index is None else torch.tensor(list(index) + [0], dtype=torch.int32).cuda()
    most = max(list(counts) + [1]) if max_rows is None else max_rows
    r = c.m.make_kv_rows(dev[0].data_ptr(), dev[1].data_ptr(), dtype, *width, len(rows[0]), ds.data_ptr(), most,
                         0 if di is None else di.data_ptr())
    st = stream or torch.cuda.current_stream()
    st.wait_stream(torch.cuda.current_stream())
    c.m.kvprm_write_kv(c.h, c.cache, c.batch, LAYER, r, st.cuda_stream)
    torch.cuda.synchronize()
    for part in (0, 1):
        fp4.write(c.code[part][LAYER], c.scale[part][LAYER], c.table, c.lengths, start, rows[part].double().numpy(), index,
                  most)


LENGTHS, COUNTS = [0, 0, 1, 15, 16, 17, 31, 300, 5, 47], [1, 40, 1, 1, 1, 3, 33, 0, 16, 129]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write(d, dtype):
    _say("write", d, dtype)
    c = _cache(d, LENGTHS, COUNTS, seed=d)
    _write(c, _rows(sum(COUNTS), d, dtype, 5), dtype, COUNTS)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write_ties_specials_and_sizes(dtype):
    """Ties between codes, signed zeros, the ends of the scales' range, infinities and NaN (their 32 dims alone)."""
    _say("specials", dtype)
    d, rng = 128, np.random.default_rng(1)
    n = 48
    rows = []
    for _ in (0, 1):
        x = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -5.0, 0.0, -0.0], size=(n, NKV, d))
        x[:, :, ::32] = 6.0
        x[:8] *= 2.0 ** rng.integers(-120, 120, size=(8, 1, 1))
        x[8] = 0.0
        x[9] = -0.0
        x[10] = 2.0 ** -126
        x[11, :, 5] = 3.3e38
        x[12, :, 40] = np.inf
        x[13, 1, 100] = -np.inf
        x[14, 2, 64] = np.nan
        x[15, :, 31], x[15, :, 32] = np.nan, np.inf
        x[16, 0], x[16, 1], x[16, 2] = 7.0, 7.03125, 1.75
        rows.append(torch.from_numpy(x.astype(np.float32)).to(T[dtype]))
    c = _cache(d, [3, 16], [20, 28])
    _write(c, rows, dtype, [20, 28])
    c.check()


def test_write_by_index_and_dropped_rows():
    """Rows picked by index (one twice), numbers outside the rows, a table's bad ids, rows past the table."""
    _say("index")
    d, rng = 64, np.random.default_rng(2)
    c = _cache(d, [10, 30, 0], [40, 20, 16])
    c.table[1, 2] = c.pages + 5
    c.table[2, 0] = -7
    c.upload()
    index = list(rng.integers(0, 50, size=40)) + [3] * 10 + [-1, 50, 1 << 30, 4, 5, 6, 7, 8, 9, 10] + list(range(16))
    _write(c, _rows(50, d, "bf16", 3), "bf16", [40, 20, 16], index=index)
    c.check()
    c = _cache(d, [40], [8])  # one spare entry, of id -1, then the table's end
    _write(c, _rows(60, d, "f32", 4), "f32", [60])
    c.check()
    c = _cache(d, [5, 6], [30, 30])  # at most max_rows
    _write(c, _rows(60, d, "f32", 4), "f32", [30, 30], max_rows=11)
    c.check()


def test_tokens_one_at_a_time_are_the_same_bytes():
    """A token's bytes depend on it alone: a page filled one by one is the page filled at once."""
    _say("one by one")
    d = 128
    rows = _rows(34, d, "bf16", 7)
    a, b = (_cache(d, [3], [34], seed=9) for _ in (0, 1))
    _write(a, rows, "bf16", [34])
    for t in range(34):
        _write(b, [r[t:t + 1] for r in rows], "bf16", [1])
        b.lengths = [4 + t]
        b.dlen += 1
        b.batch = b.m.make_batch(1, b.dtab.data_ptr(), b.width, b.dlen.data_ptr(), b.lengths)
    b.check()
    for p in (0, 1):
        assert torch.equal(a.pool[p], b.pool[p])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read(d, dtype):
    _say("read", d, dtype)
    lengths = [0, 1, 16, 33, 300, 47, 20]
    c = _cache(d, lengths, seed=3, sizes=(1e-3, 1.0, 1e6))
    first = [0, 0, 5, 30, 100, -4, 25]
    counts = [4, 1, 20, 3, 150, 30, 6]  # rows past the tokens, before the first
    start = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    n, w = int(start[-1]) + 2, NKV * d + 8
    for parts in ((0, 1), (0,), (1,)):
        out = [torch.full((n, w), 7.0, dtype=T[dtype], device="cuda") for _ in (0, 1)]
        ds, df = torch.from_numpy(start).cuda(), torch.tensor(first, dtype=torch.int32).cuda()
        r = c.m.make_kv_rows(*[out[p].data_ptr() if p in parts else 0 for p in (0, 1)], dtype, w, w, n, ds.data_ptr(),
                             max(counts))
        c.m.kvprm_read_kv(c.h, c.cache, c.batch, LAYER, r, df.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for p in (0, 1):
            want = np.full((n, w), 7.0)
            for b, L in enumerate(lengths):
                held = c.cached(p, LAYER, b)
                for i in range(counts[b] if p in parts else 0):
                    if 0 <= first[b] + i < L:
                        want[start[b] + i, :NKV * d] = held[first[b] + i].reshape(-1)
            assert np.array_equal(out[p].cpu().double().numpy(), want), p


def test_read_every_code_and_scale():
    """Every code under every scale that has finite values comes back exactly in fp32; 255 is NaN."""
    _say("all codes")
    c = _cache(64, [16 * 17], [0])
    used = c.table[0, :17]
    for p in (0, 1):
        c.code[p][LAYER][used] = np.arange(64) % 16
        for i, page in enumerate(used):
            for s in range(16):
                e = 16 * i + s
                c.scale[p][LAYER][page, :, s] = e if e <= 252 else 255
    c.upload()
    out = [torch.zeros((272, NKV * 64), device="cuda") for _ in (0, 1)]
    ds = torch.tensor([0, 272], dtype=torch.int32).cuda()
    r = c.m.make_kv_rows(out[0].data_ptr(), out[1].data_ptr(), "f32", NKV * 64, NKV * 64, 272, ds.data_ptr(), 272)
    c.m.kvprm_read_kv(c.h, c.cache, c.batch, LAYER, r, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for p in (0, 1):
        assert np.array_equal(out[p].cpu().double().numpy(), c.cached(p, LAYER, 0).reshape(272, -1), equal_nan=True)


def test_streams_and_graph():
    """On a side stream; captured once and replayed on new rows and lengths."""
    _say("graph")
    d = 128
    c = _cache(d, [7, 30], [64, 64])
    side = torch.cuda.Stream()
    _write(c, _rows(20, d, "bf16", 1), "bf16", [8, 12], stream=side)
    c.check()
    counts, start = [3, 9], np.array([0, 3, 12], dtype=np.int32)
    k, v = (torch.zeros((12, NKV * d), dtype=torch.bfloat16, device="cuda") for _ in (0, 1))
    ds = torch.from_numpy(start).cuda()
    r = c.m.make_kv_rows(k.data_ptr(), v.data_ptr(), "bf16", NKV * d, NKV * d, 12, ds.data_ptr(), 9)
    batch = c.m.make_batch(2, c.dtab.data_ptr(), c.width, c.dlen.data_ptr())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.m.kvprm_write_kv(c.h, c.cache, batch, LAYER, r, torch.cuda.current_stream().cuda_stream)
    for step in range(3):
        rows = _rows(12, d, "bf16", 20 + step)
        k.copy_(rows[0].reshape(12, -1)), v.copy_(rows[1].reshape(12, -1))
        c.lengths = [16 * step + 7, 10 * step + 30]
        c.dlen.copy_(torch.tensor(c.lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for p in (0, 1):
            fp4.write(c.code[p][LAYER], c.scale[p][LAYER], c.table, c.lengths, start, rows[p].double().numpy(), None, 9)
        c.check()
