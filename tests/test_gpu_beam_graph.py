"""A beam's step captured into a graph: fork, rows appended, drafted tokens' attention, compaction, the verify token's
attention, all from tables and lengths that the step itself leaves on the device. Every replay, between eager
steps of the same buffers, is the eager step bit for bit."""
import numpy as np
import pytest
import torch

from gpu_common import kv

pytestmark = pytest.mark.gpu
NQ, NKV, D, PAGES, WIDTH, LAYERS, N, ADD = 14, 2, 128, 80, 12, 2, 5, 19


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Step:
    """A step's buffers and its calls."""

    def __init__(self, cdt):
        self.m = m = kv()
        self.cdt = cdt
        self.h = m.kvprm_create(m.make_desc(LAYERS, 64 * NQ, NQ, NKV, D, 64, kv_dtype=cdt))
        tile = 17 * D // 2 if cdt == "fp4" else 32 * D
        self.pool = [torch.zeros((LAYERS, PAGES, NKV, tile), dtype=torch.uint8, device="cuda") for _ in (0, 1)]
        self.cache = m.make_cache(self.pool[0].data_ptr(), self.pool[1].data_ptr(), PAGES)
        ints = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.old = [ints(N, WIDTH), ints(N), ints(N)]
        self.new = [ints(N, WIDTH), ints(N), ints(N)]
        self.table, self.parent, self.room = ints(N, WIDTH), ints(N), ints(N)
        self.refs = [ints(PAGES) for _ in range(3)]
        self.moved, self.res = ints(PAGES), [ints(4), ints(4)]
        self.start = _ints([ADD * i for i in range(N + 1)])
        self.rows = torch.zeros((2, N * ADD, NKV * D), dtype=torch.bfloat16, device="cuda")
        self.draft = torch.zeros((N * ADD, (NQ + 2 * NKV) * D), dtype=torch.bfloat16, device="cuda")
        self.tree_o = torch.zeros((N * ADD, NQ * D), dtype=torch.bfloat16, device="cuda")
        self.x = [torch.zeros((N, k, D), device="cuda") for k in (NQ, NKV, NKV)]
        self.o = torch.zeros((N, NQ, D), device="cuda")
        self.mid = m.make_batch(N, self.new[0].data_ptr(), WIDTH, self.new[1].data_ptr())
        self.end = m.make_batch(N, self.table.data_ptr(), WIDTH, self.new[1].data_ptr())
        w = (NQ + 2 * NKV) * D
        at = self.draft.data_ptr()
        self.tree = m.make_tree(at, at + 2 * NQ * D, at + 2 * (NQ + NKV) * D, self.tree_o.data_ptr(), "bf16", w, w, w, NQ * D,
                                N * ADD, self.start.data_ptr(), ADD, 0, 0)
        sizes = (m.kvprm_workspace_size_pages(self.h, PAGES), m.kvprm_workspace_size_tree(self.h, self.mid, self.tree),
                 m.kvprm_workspace_size(self.h, self.end))
        self.ws = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in sizes]

    def __del__(self):
        self.m.kvprm_destroy(self.h)

    def page_rows(self, t):
        return self.m.make_page_rows(N, WIDTH, *[x.data_ptr() for x in t])

    def fill(self, seed):
        rng = np.random.default_rng(seed)
        ids = rng.permutation(PAGES)[:32]
        held = rng.integers(2, 6, size=N)
        table, refs, at = np.full((N, WIDTH), -1), np.zeros(PAGES), 2
        for i, n in enumerate(held):  # two pages that all share
            table[i, :2], table[i, 2:n] = ids[:2], ids[at:at + n - 2]
            at += n - 2
            np.add.at(refs, table[i, :n], 1)
        lengths = [int(rng.integers(32, 16 * n + 1)) for n in held]
        for t, v in zip(self.old, (table, lengths, held)):
            t.copy_(torch.tensor(np.asarray(v), dtype=torch.int32))
        self.parent.copy_(torch.tensor(rng.integers(0, N, size=N), dtype=torch.int32))
        self.room.fill_(ADD)
        self.refs[0].copy_(torch.tensor(refs, dtype=torch.int32))
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.rows, self.draft, *self.x):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))

    def run(self):
        m, st = self.m, torch.cuda.current_stream().cuda_stream
        m.kvprm_fork_pages(self.h, self.cache, self.page_rows(self.old), self.page_rows(self.new), self.parent.data_ptr(),
                           self.room.data_ptr(), self.refs[0].data_ptr(), self.refs[1].data_ptr(), self.res[0].data_ptr(),
                           self.ws[0].data_ptr(), self.ws[0].numel(), st)
        m.kvprm_attention_tree(self.h, self.cache, self.mid, 1, self.tree, self.ws[1].data_ptr(), self.ws[1].numel(), st)
        for layer in range(LAYERS):
            r = m.make_kv_rows(self.rows[0].data_ptr(), self.rows[1].data_ptr(), "bf16", NKV * D, NKV * D, N * ADD,
                               self.start.data_ptr(), ADD)
            m.kvprm_write_kv(self.h, self.cache, self.mid, layer, r, st)
        self.new[1].add_(ADD)
        m.kvprm_compact_pages(self.h, self.cache, self.page_rows(self.new), self.table.data_ptr(), self.refs[1].data_ptr(),
                              self.refs[2].data_ptr(), self.moved.data_ptr(), self.res[1].data_ptr(), self.ws[0].data_ptr(),
                              self.ws[0].numel(), st)
        q, k, v = self.x
        m.kvprm_attention(self.h, self.cache, self.end, 1, q.data_ptr(), k.data_ptr(), v.data_ptr(), self.ws[2].data_ptr(),
                          self.ws[2].numel(), self.o.data_ptr(), st)

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (*self.pool, *self.new, self.table, *self.refs[1:], self.moved, *self.res, self.tree_o, self.o)]


@pytest.mark.parametrize("cdt", ["fp4", "bf16"])
def test_beam_step_in_a_graph(cdt):
    print("case: beam graph", cdt, flush=True)
    s = Step(cdt)
    s.fill(0)
    s.run()
    torch.cuda.synchronize()
    pool = [t.clone() for t in s.pool]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for seed in range(1, 5):
        got = []
        for go in (s.run, graph.replay):
            for t, p in zip(s.pool, pool):
                t.copy_(p)
            s.fill(seed)
            go()
            got.append(s.state())
        for a, b in zip(*got):
            assert torch.equal(a, b)
        assert s.res[0][0].item() == 0 and s.res[1][0].item() == 0
        assert bool(torch.isfinite(s.o).all()) and bool(s.o.any()) and bool(s.tree_o.any())
        for t, p in zip(pool, s.pool):  # the next step's cache is this one's
            t.copy_(p)
