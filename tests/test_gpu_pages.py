"""kvprm_fork_pages and kvprm_compact_pages on the GPU against the oracle: tables, holders, results and every byte of
the pools."""
import numpy as np
import pytest
import torch

from oracle import cache_pages as cp

from gpu_common import kv

pytestmark = pytest.mark.gpu
LAYERS, NKV, D = 3, 2, 64
TILE = {"f32": 4 * 16 * D, "bf16": 2 * 16 * D, "fp8": 16 * D, "fp4": 17 * D // 2}


def _say(*a):
    print("case:", *a, flush=True)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Pool:
    def __init__(self, cdt, pages, seed=0, layers=LAYERS):
        self.m, self.cdt, self.pages = kv(), cdt, pages
        self.rng = np.random.default_rng(seed)
        shape = (layers, pages, NKV)
        self.host = [self.rng.integers(0, 256, size=(*shape, TILE[cdt]), dtype=np.uint8) for _ in (0, 1)]
        if cdt == "fp8":
            self.host += [self.rng.random(size=shape, dtype=np.float32) for _ in (0, 1)]
        self.dev = [torch.from_numpy(t).cuda() for t in self.host]
        self.h = self.m.kvprm_create(self.m.make_desc(layers, 64 * NKV, NKV, NKV, D, 64,
                                                      weight_dtype="f32" if cdt == "f32" else "bf16", kv_dtype=cdt))
        self.cache = self.m.make_cache(self.dev[0].data_ptr(), self.dev[1].data_ptr(), pages,
                                       *[t.data_ptr() for t in self.dev[2:]])
        n = self.m.kvprm_workspace_size_pages(self.h, pages)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")

    def __del__(self):
        self.m.kvprm_destroy(self.h)

    def page_rows(self, rows, width, lengths=None, fill=None):
        """Rows on the device; entries past a row's own hold anything."""
        t = self.rng.integers(-3, self.pages + 9, size=(max(1, len(rows)), width)).astype(np.int32)
        for i, row in enumerate(rows):
            t[i, :len(row)] = row
        keep = [torch.from_numpy(t).cuda(), _ints(lengths or [0] * max(1, len(rows))), _ints([len(r) for r in rows] or [0])]
        if fill is not None:
            for k in keep:
                k.fill_(fill)
        p = self.m.make_page_rows(len(rows), width, *[k.data_ptr() for k in keep])
        p._keep = keep
        return p

    def copied(self, copies):
        for t in self.host:
            was = t.copy()
            for src, to in copies:
                t[:, to] = was[:, src]

    def same(self):
        for t, d in zip(self.host, self.dev):
            assert np.array_equal(d.cpu().numpy(), t)

    def fork(self, rows, lengths, parent, room, refs, width, to_width, stream=None):
        """The call, checked against the oracle; returns the oracle's answer."""
        m = self.m
        src, dst = self.page_rows(rows, width, lengths), self.page_rows([[]] * len(parent), to_width, fill=-9)
        dp, dr = _ints(parent or [0]), None if room is None else _ints(room or [0])
        refs_d, new, res = _ints(refs), _ints([-9] * self.pages), _ints([-9] * 4)
        st = stream or torch.cuda.current_stream()
        st.wait_stream(torch.cuda.current_stream())
        m.kvprm_fork_pages(self.h, self.cache, src, dst, dp.data_ptr(), 0 if dr is None else dr.data_ptr(), refs_d.data_ptr(),
                           new.data_ptr(), res.data_ptr(), self.ws.data_ptr(), self.ws.numel(), st.cuda_stream)
        torch.cuda.synchronize()
        room = room if room is not None else [0] * len(parent)
        status, out, lens, after, copies, need, have = cp.fork(rows, lengths, parent, room, refs, to_width)
        table, dl, dh = (k.cpu().tolist() for k in dst._keep)
        assert refs_d.cpu().tolist() == refs
        if status:
            assert res.cpu().tolist() == [status, need, have, 0]
            assert set(sum(table, []) + dl + dh + new.cpu().tolist()) == {-9}
        else:
            assert res.cpu().tolist() == [0, need, have, after.count(0)]
            if parent:
                assert table == [r + [-1] * (to_width - len(r)) for r in out]
                assert dl == lens and dh == [len(r) for r in out]
            assert new.cpu().tolist() == after
            self.copied(copies)
        self.same()
        return status, out, lens, after


def _case(rng, pages, n, prefix, most, spare=True):
    ids = [int(p) for p in rng.permutation(pages)]
    rows, lengths, at = [], [], prefix
    for _ in range(n):
        k = int(rng.integers(0, most + 1))
        rows.append(ids[:prefix] + ids[at:at + k])
        at += k
        h = len(rows[-1])
        lengths.append(int(rng.integers(0 if spare else max(0, 16 * h - 15), 16 * h + 1)))
    refs = [0] * pages
    for row in rows:
        for p in row:
            refs[p] += 1
    return rows, lengths, refs


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8", "fp4"])
@pytest.mark.parametrize("seed", range(4))
def test_fork(cdt, seed):
    _say("fork", cdt, seed)
    pool = Pool(cdt, 150 + seed, seed)
    rng = np.random.default_rng(seed)
    rows, lengths, refs = _case(rng, pool.pages, 5, 7, 9)
    parent = [int(p) for p in rng.integers(-1, 5, size=6)]
    room = None if seed == 3 else [int(r) for r in rng.choice([0, 1, 16, 40], size=6)]
    assert pool.fork(rows, lengths, parent, room, refs, 17, 21)[0] == 0


def test_fork_edges():
    """No rows, no children, new sequences alone, one parent for all, lengths at page ends, a page held outside."""
    _say("edges")
    pool = Pool("bf16", 64)
    free = [0] * 64
    _, rows, lens, refs = pool.fork([], [], [-1] * 3, [40, 0, 16], free, 1, 5)
    assert [len(r) for r in rows] == [3, 0, 1]
    lens = [33, 0, 16]
    _, rows, lens, refs = pool.fork(rows, lens, [0] * 5 + [2, 2, 1], [15] * 8, refs, 5, 4)
    assert lens == [33] * 5 + [16, 16, 0]
    # a page with a holder that is no row: even the first child gets a copy
    refs[rows[0][2]] += 1
    _, rows, lens, refs = pool.fork(rows, lens, [0, 3], None, refs, 4, 3)
    assert sum(refs) == 7
    _, _, _, refs = pool.fork(rows, lens, [], None, refs, 3, 1)
    assert sum(refs) == 1


def test_fork_that_cannot_be():
    """Nothing but the result is written: too few pages, a bad parent, room, length, held, entry, width or count."""
    _say("cannot")
    pool = Pool("fp8", 20)
    rows, lengths, refs = [[3, 5], [3, 9, 11]], [20, 48], [0] * 20
    for row in rows:
        for p in row:
            refs[p] += 1
    for change in (dict(room=[400, 0]), dict(parent=[0, 2]), dict(room=[0, -1]), dict(lengths=[33, 48]),
                   dict(lengths=[-1, 48]), dict(to_width=2), dict(rows=[[3, 20], [3, 9, 11]]), dict(rows=[[-1, 5], [3, 9, 11]]),
                   dict(refs=[0] * 20), dict(refs=[r - (p == 3) for p, r in enumerate(refs)])):
        a = {**dict(rows=rows, lengths=lengths, parent=[0, 1], room=[0, 0], refs=refs, width=4, to_width=40), **change}
        assert pool.fork(**a)[0] != 0
    src, dst = pool.page_rows(rows, 4, lengths), pool.page_rows([[]] * 2, 4, fill=-9)
    for held in (-1, 5):  # outside 0 .. 4
        src._keep[2][1] = held
        new, res, par = _ints([-9] * 20), _ints([-9] * 4), _ints([0, 0])
        rd = _ints(refs)
        pool.m.kvprm_fork_pages(pool.h, pool.cache, src, dst, par.data_ptr(), 0, rd.data_ptr(), new.data_ptr(), res.data_ptr(),
                                pool.ws.data_ptr(), pool.ws.numel(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert res.cpu().tolist() == [2, 0, 0, 0] and set(new.cpu().tolist()) == {-9}
    pool.same()


@pytest.mark.parametrize("pages,n,most", [(4096, 30, 60), (4097, 40, 100), (16384, 64, 200), (16385, 64, 200),
                                          (20000, 64, 200), (70000, 256, 150)])
def test_large_pools(pages, n, most):
    """Pools of several scan blocks, up to 256 rows; a long prefix."""
    _say("large", pages)
    pool = Pool("fp4", pages, layers=1)
    rng = np.random.default_rng(n)
    rows, lengths, refs = _case(rng, pages, n, 37, most, spare=False)
    parent = [int(p) for p in rng.integers(-1, n // 2, size=n)]
    room = [int(r) for r in rng.integers(0, 100, size=n)]
    status, rows, lengths, refs = pool.fork(rows, lengths, parent, room, refs, most + 40, most + 60)
    assert status == 0
    _compact(pool, rows, refs, most + 60)


def _compact(pool, rows, refs, width, stream=None):
    m = pool.m
    src = pool.page_rows(rows, width)
    table = torch.full((max(1, len(rows)), width), -9, dtype=torch.int32, device="cuda")
    rd, new, moved, res = _ints(refs), _ints([-9] * pool.pages), _ints([-9] * pool.pages), _ints([-9] * 4)
    st = stream or torch.cuda.current_stream()
    st.wait_stream(torch.cuda.current_stream())
    m.kvprm_compact_pages(pool.h, pool.cache, src, table.data_ptr(), rd.data_ptr(), new.data_ptr(), moved.data_ptr(),
                          res.data_ptr(), pool.ws.data_ptr(), pool.ws.numel(), st.cuda_stream)
    torch.cuda.synchronize()
    status, out, after, to, copies = cp.compact(rows, refs)
    if status:
        assert res.cpu().tolist() == [2, 0, 0, 0]
        assert set(table.cpu().reshape(-1).tolist() + new.cpu().tolist() + moved.cpu().tolist()) == {-9}
    else:
        live = sum(r > 0 for r in refs)
        assert res.cpu().tolist() == [0, live, len(copies), pool.pages - live]
        assert new.cpu().tolist() == after and moved.cpu().tolist() == to
        if rows:
            assert table.cpu().tolist() == [r + [-1] * (width - len(r)) for r in out]
        pool.copied(copies)
    pool.same()
    return status


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8", "fp4"])
@pytest.mark.parametrize("pages", [1, 63, 64, 65, 130, 333])
def test_compact(cdt, pages):
    _say("compact", cdt, pages)
    pool = Pool(cdt, pages, pages)
    rng = np.random.default_rng(pages)
    rows, _, refs = _case(rng, pages, 6, min(3, pages // 8), max(0, (pages - 8) // 8))
    for p in rng.integers(0, pages, size=max(1, pages // 9)):  # pages that other tables hold
        refs[int(p)] += 2
    assert _compact(pool, rows, refs, 60) == 0


def test_compact_edges():
    """Nothing held, everything held, already dense, the last page alone; entries and counts that cannot be."""
    _say("compact edges")
    pool = Pool("bf16", 40)
    assert _compact(pool, [], [0] * 40, 1) == 0
    assert _compact(pool, [list(range(40))], [1] * 40, 40) == 0
    assert _compact(pool, [[0, 1], [2, 0]], [2, 1, 1] + [0] * 37, 3) == 0
    assert _compact(pool, [[39]], [0] * 39 + [1], 3) == 0
    for rows, refs in (([[5]], [1] * 5 + [0] + [1] * 34), ([[40]], [1] * 40), ([[-1]], [1] * 40), ([[3]], [1] * 39 + [-1])):
        assert _compact(pool, rows, refs, 3) == 2


def test_streams_and_graph():
    """On a side stream; both calls captured in one graph and replayed on new tables."""
    _say("graph")
    pool = Pool("fp8", 90, 5)
    rng = np.random.default_rng(3)
    rows, lengths, refs = _case(rng, 90, 4, 5, 6)
    pool.fork(rows, lengths, [0, 1, 1, 3], [9] * 4, refs, 11, 12, stream=torch.cuda.Stream())
    _compact(pool, rows, refs, 11, stream=torch.cuda.Stream())
    m, n, width = pool.m, 4, 12
    src, mid = pool.page_rows([[]] * n, 11, fill=0), pool.page_rows([[]] * n, width, fill=0)
    table = torch.zeros((n, width), dtype=torch.int32, device="cuda")
    par, room = _ints([0] * n), _ints([0] * n)
    r0, r1, r2, moved, res, res2 = (_ints([0] * k) for k in (90, 90, 90, 90, 4, 4))
    ws = [torch.empty_like(pool.ws) for _ in (0, 1)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st = torch.cuda.current_stream().cuda_stream
        m.kvprm_fork_pages(pool.h, pool.cache, src, mid, par.data_ptr(), room.data_ptr(), r0.data_ptr(), r1.data_ptr(),
                           res.data_ptr(), ws[0].data_ptr(), ws[0].numel(), st)
        m.kvprm_compact_pages(pool.h, pool.cache, mid, table.data_ptr(), r1.data_ptr(), r2.data_ptr(), moved.data_ptr(),
                              res2.data_ptr(), ws[1].data_ptr(), ws[1].numel(), st)
    for step in range(3):
        rows, lengths, refs = _case(rng, 90, n, 4, 6)
        parent, extra = [int(p) for p in rng.integers(0, n, size=n)], [int(x) for x in rng.integers(0, 20, size=n)]
        fresh = pool.page_rows(rows, 11, lengths)
        for a, b in zip(src._keep, fresh._keep):
            a.copy_(b)
        par.copy_(_ints(parent)), room.copy_(_ints(extra)), r0.copy_(_ints(refs))
        graph.replay()
        torch.cuda.synchronize()
        status, out, lens, after, copies, need, have = cp.fork(rows, lengths, parent, extra, refs, width)
        pool.copied(copies)
        status, out, after, to, copies = cp.compact(out, after)
        pool.copied(copies)
        assert table.cpu().tolist() == [r + [-1] * (width - len(r)) for r in out]
        assert r2.cpu().tolist() == after and moved.cpu().tolist() == to
        pool.same()


@pytest.mark.parametrize("cdt,layers", [("fp8", 3), ("bf16", 5), ("fp4", 1)])
@pytest.mark.parametrize("children", [65, 128, 256])
def test_many_copies_in_one_launch(cdt, layers, children):
    """More children than a wave has lanes, in a pool that one launch serves. Most of them copy a partly filled page:
    every block takes its share of all copies' bytes, so that the blocks have to list the copies in one order."""
    _say("copies", cdt, children)
    pool = Pool(cdt, 6 * children + 200, children, layers=layers)
    rng = np.random.default_rng(children)
    rows, lengths, refs = _case(rng, pool.pages, 20, 3, 5)
    lengths = [min(n + (n % 16 == 0), 16 * len(r)) for n, r in zip(lengths, rows)]
    parent = [int(p) for p in rng.integers(0, 20, size=children)]
    room = [int(r) for r in rng.choice([0, 1, 16, 40], size=children)]
    status, _, lens, _ = pool.fork(rows, lengths, parent, room, refs, 9, 12)
    assert status == 0 and sum(n % 16 > 0 for n in lens) > children // 2


@pytest.mark.parametrize("pages,n,width", [(900, 140, 1000), (1200, 256, 514)])
def test_wide_tables_of_small_pools(pages, n, width):
    """Tables of more entries than the one-launch calls take, over pools that they would take."""
    _say("wide", pages, n, width)
    pool = Pool("fp8", pages, n, layers=2)
    rng = np.random.default_rng(n)
    rows, lengths, refs = _case(rng, pages, n, 30, 2, spare=False)
    parent = [int(p) for p in rng.integers(-1, n // 2, size=n)]
    status, rows, lengths, refs = pool.fork(rows, lengths, parent, None, refs, width, width)
    assert status == 0
    assert _compact(pool, rows, refs, width) == 0
