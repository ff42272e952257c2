"""Offsets past 32 bits: calls on pages that lie more than 4 GiB into their pool give the bits that they give on the same
pages at the front of a small one, and the page calls copy there byte for byte."""
import numpy as np
import pytest
import torch

from fp4_common import Cache
from gpu_common import kv
from test_gpu_fp4_attention import _inputs
from test_gpu_fp4_attention import _run as _attend
from test_gpu_fp4_tree import Draft

pytestmark = pytest.mark.gpu
PAGES = 500_000  # of 8 kv-heads of 128 dims: 4.35 GB


def _say(*a):
    print("case:", *a, flush=True)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Far:
    """A cache's pages at the end of a large pool."""

    def __init__(self, c):
        nq, nkv, d = c.shape
        self.m, self.shape, self.lengths, self.rows = c.m, c.shape, c.lengths, c.pages
        self.width, self.dlen, self.small = c.width, c.dlen, c
        self.pool = [torch.empty((1, PAGES, nkv, 17 * d // 2), dtype=torch.uint8, device="cuda") for _ in (0, 1)]
        for far, near in zip(self.pool, c.pool):
            far[:, PAGES - c.pages:] = near.view(1, c.pages, nkv, -1)
        self.dtab = torch.where(c.dtab >= 0, c.dtab + (PAGES - c.pages), c.dtab)
        self.h = c.m.kvprm_create(c.m.make_desc(1, 64 * nq, nq, nkv, d, 64, kv_dtype="fp4"))
        self.cache = c.m.make_cache(self.pool[0].data_ptr(), self.pool[1].data_ptr(), PAGES)
        self.batch = c.m.make_batch(len(c.lengths), self.dtab.data_ptr(), self.width, self.dlen.data_ptr(), c.lengths)

    def same(self):
        for far, near in zip(self.pool, self.small.pool):
            assert torch.equal(far[:, PAGES - self.rows:].reshape(-1), near.reshape(-1))

    def __del__(self):
        self.m.kvprm_destroy(self.h)


@pytest.mark.parametrize("lengths,counts", [([30, 500, 1], [3, 1, 2]), ([4000, 900], [64, 40])])
def test_far_pages(lengths, counts, monkeypatch):
    _say("far", lengths)
    monkeypatch.setattr("test_gpu_fp4_attention.LAYER", 0)
    monkeypatch.setattr("test_gpu_fp4_tree.LAYER", 0)
    near = Cache(16, 8, 128, lengths, rows=[70] * len(lengths), layers=1)
    far = Far(near)
    x = _inputs(near, 3)
    assert np.array_equal(_attend(near, x), _attend(far, x))
    for dtype in ("bf16", "f32"):
        got = []
        for c in (near, far):
            got.append(Draft(c, dtype, counts, "tree", seed=1).run())
        assert torch.equal(got[0][:sum(counts)], got[1][:sum(counts)])
    n, start = sum(counts), _ints([0] + list(np.cumsum(counts)))
    rows = torch.randn((2, n, 1024), device="cuda").to(torch.bfloat16)
    back = []
    for c in (near, far):
        m, out = c.m, torch.zeros_like(rows)
        for call, t in ((m.kvprm_write_kv, rows), (m.kvprm_read_kv, out)):
            r = m.make_kv_rows(t[0].data_ptr(), t[1].data_ptr(), "bf16", 1024, 1024, n, start.data_ptr(), max(counts))
            call(c.h, c.cache, c.batch, 0, r, stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        back.append(out)
    assert torch.equal(back[0], back[1]) and bool(back[0].any())
    far.same()


@pytest.mark.parametrize("cdt,layers,pages", [("fp4", 1, PAGES), ("bf16", 9, 16_000)])
def test_far_copies(cdt, layers, pages):
    """Copies from and to pages past 4 GiB (several launches, and one)."""
    _say("copies", cdt, pages)
    m, nkv, d = kv(), 8, 128
    tile = 17 * d // 2 if cdt == "fp4" else 32 * d
    h = m.kvprm_create(m.make_desc(layers, 1024, 16, nkv, d, 64, kv_dtype=cdt))
    try:
        pool = [torch.empty((layers, pages, nkv, tile), dtype=torch.uint8, device="cuda") for _ in (0, 1)]
        g = torch.Generator(device="cuda").manual_seed(1)
        for t in pool:
            t[:, pages - 8:] = torch.randint(0, 256, (layers, 8, nkv, tile), dtype=torch.uint8, device="cuda", generator=g)
        was = [t[:, pages - 8:].clone() for t in pool]
        cache = m.make_cache(pool[0].data_ptr(), pool[1].data_ptr(), pages)
        ws = torch.empty(m.kvprm_workspace_size_pages(h, pages), dtype=torch.uint8, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        # two rows of the last pages, the first of 20 tokens; pages below are held elsewhere
        refs = torch.ones(pages, dtype=torch.int32, device="cuda")
        refs[pages - 8:] = _ints([0, 1, 0, 1, 1, 0, 0, 0])
        src = [_ints([[pages - 7, pages - 5], [pages - 4, -1]]), _ints([20, 16]), _ints([2, 1])]
        dst = [torch.zeros((3, 3), dtype=torch.int32, device="cuda"), _ints([0] * 3), _ints([0] * 3)]
        new, res, parent = torch.empty_like(refs), _ints([0] * 4), _ints([0, 0, 0])
        m.kvprm_fork_pages(h, cache, m.make_page_rows(2, 2, *[t.data_ptr() for t in src]),
                           m.make_page_rows(3, 3, *[t.data_ptr() for t in dst]), parent.data_ptr(), 0, refs.data_ptr(),
                           new.data_ptr(), res.data_ptr(), ws.data_ptr(), ws.numel(), st)
        torch.cuda.synchronize()
        assert res.cpu().tolist() == [0, 2, 6, 4]
        assert dst[0].cpu().tolist() == [[pages - 7, pages - 5, -1], [pages - 7, pages - 8, -1], [pages - 7, pages - 6, -1]]
        assert new[pages - 8:].cpu().tolist() == [1, 3, 1, 1, 0, 0, 0, 0] and bool((new[:pages - 8] == 1).all())
        for t, w in zip(pool, was):
            w[:, 0], w[:, 2] = w[:, 3].clone(), w[:, 3].clone()
            assert torch.equal(t[:, pages - 8:], w)
        # pages 5 and 9 become free: the last live ones move there
        refs = new.clone()
        refs[5] = refs[9] = 0
        table, after, moved = torch.zeros_like(dst[0]), torch.empty_like(refs), torch.empty_like(refs)
        m.kvprm_compact_pages(h, cache, m.make_page_rows(3, 3, *[t.data_ptr() for t in dst]), table.data_ptr(), refs.data_ptr(),
                              after.data_ptr(), moved.data_ptr(), res.data_ptr(), ws.data_ptr(), ws.numel(), st)
        torch.cuda.synchronize()
        assert res.cpu().tolist() == [0, pages - 6, 2, 6]
        assert table.cpu().tolist() == [[pages - 7, 9, -1], [pages - 7, pages - 8, -1], [pages - 7, 5, -1]]
        assert moved[pages - 8:].cpu().tolist() == [pages - 8, pages - 7, 5, 9, -1, -1, -1, -1]
        assert after[pages - 8:].cpu().tolist() == [1, 3] + [0] * 6 and bool((after[:pages - 8] == 1).all())
        for t, w in zip(pool, was):
            assert torch.equal(t[:, 5], w[:, 2]) and torch.equal(t[:, 9], w[:, 3]) and torch.equal(t[:, pages - 8:], w)
    finally:
        m.kvprm_destroy(h)
