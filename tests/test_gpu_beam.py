"""The page calls, the row calls and attention as a beam search uses them together, with tables and lengths on the
device throughout: prompts get pages, are written, the beam forks, its children append tokens of their own, some end,
the pool is compacted. Every text's attention is checked against the tokens that were written for it.

Tolerance: rows are values that the cache holds exactly (decoded 4-bit values; bf16), so that the attention's own
bound is left, 2 * 1e-5 max|v| (4 bits) or, with weights in two bf16 terms, (2^-16 + 2 * 1e-5) max|v|."""
import numpy as np
import pytest
import torch

from oracle import fp4
from oracle import kvprm_oracle as ko

from gpu_common import kv

pytestmark = pytest.mark.gpu
NQ, NKV, D, PAGES, WIDTH, LAYERS = 8, 2, 128, 96, 16, 2


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Beam:
    def __init__(self, cdt):
        self.m, self.cdt, self.rng = kv(), cdt, np.random.default_rng(7)
        self.h = self.m.kvprm_create(self.m.make_desc(LAYERS, 1024, NQ, NKV, D, 64, kv_dtype=cdt))
        tile = 17 * D // 2 if cdt == "fp4" else 32 * D
        self.pool = [torch.full((LAYERS, PAGES, NKV, tile), 0xFF, dtype=torch.uint8, device="cuda") for _ in (0, 1)]
        self.cache = self.m.make_cache(self.pool[0].data_ptr(), self.pool[1].data_ptr(), PAGES)
        self.ws = torch.empty(self.m.kvprm_workspace_size_pages(self.h, PAGES), dtype=torch.uint8, device="cuda")
        self.refs = _ints([0] * PAGES)
        self.set(*self.blank(0))
        self.texts = []  # per row, layer and part: its tokens [n][NKV][D]

    def blank(self, n):
        return [torch.zeros((max(n, 1), WIDTH), dtype=torch.int32, device="cuda"), _ints([0] * max(n, 1)),
                _ints([0] * max(n, 1)), n]

    def set(self, table, lengths, held, n):
        self.table, self.lengths, self.held, self.n = table, lengths, held, n

    def rows(self, t):
        return self.m.make_page_rows(t[3], WIDTH, *[x.data_ptr() for x in t[:3]])

    def fork(self, parent, room):
        to, new, res, par, more = self.blank(len(parent)), torch.empty_like(self.refs), _ints([0] * 4), _ints(parent), _ints(room)
        self.m.kvprm_fork_pages(self.h, self.cache, self.rows([self.table, self.lengths, self.held, self.n]), self.rows(to),
                                par.data_ptr(), more.data_ptr(), self.refs.data_ptr(), new.data_ptr(), res.data_ptr(),
                                self.ws.data_ptr(), self.ws.numel(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert res[0].item() == 0
        self.refs = new
        self.set(*to)
        self.texts = [[[t.copy() for t in layer] for layer in self.texts[p]] if p >= 0 else
                      [[np.zeros((0, NKV, D)) for _ in (0, 1)] for _ in range(LAYERS)] for p in parent]

    def compact(self):
        table, new, moved, res = torch.empty_like(self.table), torch.empty_like(self.refs), torch.empty_like(self.refs), _ints([0] * 4)
        self.m.kvprm_compact_pages(self.h, self.cache, self.rows([self.table, self.lengths, self.held, self.n]),
                                   table.data_ptr(), self.refs.data_ptr(), new.data_ptr(), moved.data_ptr(), res.data_ptr(),
                                   self.ws.data_ptr(), self.ws.numel(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        status, live, moves, _ = res.cpu().tolist()
        assert status == 0
        self.table, self.refs = table, new
        for t in self.pool:  # what lies past the live pages is nobody's
            t[:, live:] = 0xFF
        return moves

    def batch(self):
        return self.m.make_batch(self.n, self.table.data_ptr(), WIDTH, self.lengths.data_ptr())

    def append(self, counts):
        n, start = sum(counts), _ints([0] + list(np.cumsum(counts)))
        at = np.concatenate([[0], np.cumsum(counts)])
        for layer in range(LAYERS):
            x = [self.rng.normal(size=(n, NKV, D)) for _ in (0, 1)]
            x = [fp4.decode(*fp4.encode(t)) if self.cdt == "fp4" else
                 torch.from_numpy(t).to(torch.bfloat16).double().numpy() for t in x]
            dev = [torch.from_numpy(t).to(torch.bfloat16).cuda() for t in x]
            r = self.m.make_kv_rows(dev[0].data_ptr(), dev[1].data_ptr(), "bf16", NKV * D, NKV * D, n, start.data_ptr(),
                                    max(counts))
            self.m.kvprm_write_kv(self.h, self.cache, self.batch(), layer, r, torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            for i in range(self.n):
                for p in (0, 1):
                    self.texts[i][layer][p] = np.concatenate([self.texts[i][layer][p], x[p][at[i]:at[i + 1]]])
        self.lengths = self.lengths + _ints(counts)

    def attend(self, layer):
        rng = np.random.default_rng(layer + 40)
        q, k, v = (rng.normal(size=(self.n, h, D)).astype(np.float32) for h in (NQ, NKV, NKV))
        dq, dk, dv = (torch.from_numpy(t).cuda() for t in (q, k, v))
        o, b = torch.zeros_like(dq), self.batch()
        n = self.m.kvprm_workspace_size(self.h, b)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        self.m.kvprm_attention(self.h, self.cache, b, layer, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), n,
                               o.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        got = o.cpu().numpy()
        for i in range(self.n):
            for h in range(NQ):
                K, V = (np.concatenate([self.texts[i][layer][p][:, h // 4], t[i, h // 4][None]]) for p, t in ((0, k), (1, v)))
                want = ko.attention(q[i, h].astype(np.float64), K, V)
                tol = (2e-5 if self.cdt == "fp4" else 2e-5 + 2.0 ** -16) * np.abs(V).max()
                assert np.abs(got[i, h] - want).max() <= tol, (layer, i, h)
        return got


@pytest.mark.parametrize("cdt", ["fp4", "bf16"])
def test_beam(cdt):
    print("case: beam", cdt, flush=True)
    b = Beam(cdt)
    try:
        b.fork([-1, -1, -1], [70, 33, 16])
        b.append([70, 33, 16])
        for parent, counts in (([0, 0, 0, 1, 2, 2], [5, 1, 0, 15, 16, 17]), ([5, 0, 0, 3, 5, 5], [3, 11, 7, 1, 2, 20]),
                               ([1, 1, 4], [1, 9, 16])):
            b.fork(parent, counts)
            b.append(counts)
            before = [b.attend(layer) for layer in range(LAYERS)]
            b.compact()
            for layer in range(LAYERS):
                assert np.array_equal(before[layer], b.attend(layer))
        b.fork([], [])
        assert not b.refs.any()
    finally:
        b.m.kvprm_destroy(b.h)
