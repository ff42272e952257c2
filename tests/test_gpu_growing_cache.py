"""The calls of a growing cache as a generator uses them together: rotate the drafted tokens' queries
and keys, attend to the cache and the tree, append the accepted path, score over the grown cache,
read it back. Two rounds, fp8 and bf16 caches, against the fp64 oracle.

Tolerances: bf16 rows as in test_gpu_tree; the oracle's inputs of each step are the rows that the step
before left on the device, so that errors do not add up over the steps."""
import numpy as np
import pytest
import torch

from oracle import growing_cache as gc
from oracle import kvprm_oracle as ko

from gpu_common import kv

pytestmark = pytest.mark.gpu
NQ, NKV, D, PAGES, WIDTH = 8, 2, 128, 64, 20


@pytest.mark.parametrize("cdt", ["bf16", "fp8"])
def test_draft_verify_append_read(cdt):
    print("case: together", cdt, flush=True)
    m, rng = kv(), np.random.default_rng(12)
    bf, st = torch.bfloat16, torch.cuda.current_stream().cuda_stream
    h = m.kvprm_create(m.make_desc(1, 1024, NQ, NKV, D, 64, kv_dtype=cdt))
    rope = m.make_rope(D)
    table = rng.permutation(PAGES)[:3 * WIDTH].reshape(3, WIDTH).astype(np.int32)
    dtab = torch.from_numpy(table).cuda()
    eb = 1 if cdt == "fp8" else 2
    pools = [torch.zeros((PAGES, NKV, 16, D * eb), dtype=torch.uint8, device="cuda") for _ in (0, 1)]
    scales = [torch.zeros((PAGES, NKV), device="cuda") for _ in (0, 1)]
    cache = m.make_cache(pools[0].data_ptr(), pools[1].data_ptr(), PAGES,
                         *([s.data_ptr() for s in scales] if cdt == "fp8" else (0, 0)))
    lengths = [0, 0, 0]

    def batch():
        dlen = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        b = m.make_batch(3, dtab.data_ptr(), WIDTH, dlen.data_ptr(), lengths)
        b._dlen = dlen
        return b

    def rows(counts):
        n = sum(counts)
        return torch.from_numpy(rng.normal(size=(n, (NQ + 2 * NKV) * D)).astype(np.float32)).to(bf).cuda()

    def rotate(x, pos):
        q = torch.empty((len(x), NQ * D), dtype=bf, device="cuda")
        k = torch.empty((len(x), NKV * D), dtype=bf, device="cuda")
        p = torch.tensor(pos, dtype=torch.int32, device="cuda")
        w = x.shape[1]
        m.kvprm_rotary(rope, "bf16", len(x), p.data_ptr(), m.make_rope_heads(
            [(x.data_ptr(), q.data_ptr(), NQ, w, NQ * D), (x.data_ptr() + 2 * NQ * D, k.data_ptr(), NKV, w, NKV * D)]),
            stream=st)
        return q, k

    def append(k, x, counts, index=None):
        start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        di = None if index is None else torch.tensor(index, dtype=torch.int32, device="cuda")
        r = m.make_kv_rows(k.data_ptr(), x.data_ptr() + 2 * (NQ + NKV) * D, "bf16", NKV * D, x.shape[1], len(x),
                           start.data_ptr(), max(counts), 0 if di is None else di.data_ptr())
        m.kvprm_write_kv(h, cache, batch(), 0, r, st)
        torch.cuda.synchronize()
        for i, c in enumerate(counts):
            lengths[i] += c

    def read():
        """Every cached token through the call, [sequence] -> (k, v) in float64."""
        start = np.concatenate([[0], np.cumsum(lengths)])
        ds = torch.tensor(start, dtype=torch.int32, device="cuda")
        out = [torch.zeros((sum(lengths), NKV * D), device="cuda") for _ in (0, 1)]
        r = m.make_kv_rows(out[0].data_ptr(), out[1].data_ptr(), "f32", NKV * D, NKV * D, sum(lengths), ds.data_ptr(),
                           max(lengths))
        m.kvprm_read_kv(h, cache, batch(), 0, r, 0, st)
        torch.cuda.synchronize()
        return [[t[start[b]:start[b + 1]].cpu().double().numpy().reshape(-1, NKV, D) for t in out] for b in range(3)]

    try:
        prompt = [37, 200, 16]
        x = rows(prompt)
        q, k = rotate(x, [t for n in prompt for t in range(n)])
        append(k, x, prompt)
        for step in range(2):
            # drafted trees: token 0 and 1 continue the cache, 2 and 3 continue 0, 4 continues 2
            parent, depth, counts = [-1, -1, 0, 0, 2], [0, 0, 1, 1, 2], [5, 5, 5]
            sees = np.eye(5, dtype=bool)
            for t, p in enumerate(parent):
                if p >= 0:
                    sees[t] |= sees[p]
            bits = (sees * (1 << np.arange(5))).sum(axis=1).astype(np.int32)
            x = rows(counts)
            q, k = rotate(x, [lengths[b] + e for b in range(3) for e in depth])
            mask = torch.from_numpy(np.tile(bits, 3)).cuda()
            start = torch.tensor([0, 5, 10, 15], dtype=torch.int32, device="cuda")
            o = torch.empty((15, NQ * D), dtype=bf, device="cuda")
            w = x.shape[1]
            tree = m.make_tree(q.data_ptr(), k.data_ptr(), x.data_ptr() + 2 * (NQ + NKV) * D, o.data_ptr(), "bf16", NQ * D,
                               NKV * D, w, NQ * D, 15, start.data_ptr(), 5, mask.data_ptr(), 1)
            b = batch()
            n = m.kvprm_workspace_size_tree(h, b, tree)
            ws = torch.empty(n, dtype=torch.uint8, device="cuda")
            m.kvprm_attention_tree(h, cache, b, 0, tree, ws.data_ptr(), n, st)
            torch.cuda.synchronize()
            before = read()
            f = gc.frequencies(D, 1e6)
            for s in range(3):
                xs = x[5 * s:5 * s + 5].cpu().double().numpy()
                pos = [lengths[s] + e for e in depth]
                wq = gc.rotary(xs[:, :NQ * D].reshape(5, NQ, D), pos, f)
                gq = q[5 * s:5 * s + 5].cpu().double().numpy().reshape(5, NQ, D)
                gk = k[5 * s:5 * s + 5].cpu().double().numpy().reshape(5, NKV, D)
                assert np.all(np.abs(gq - wq) <= 2.0 ** -8 * np.abs(wq) + 1e-5)
                want = gc.tree_attention(gq, gk, xs[:, (NQ + NKV) * D:].reshape(5, NKV, D), *before[s], sees)
                got = o[5 * s:5 * s + 5].cpu().double().numpy().reshape(5, NQ, D)
                assert np.all(np.abs(got - want) <= 2 * (2.0 ** -16 + 1e-5) * 5 + 2.0 ** -8 * np.abs(want))
            # accepted: the paths 0-2-4, 1 and 0-3
            paths = [[0, 2, 4], [1], [0, 3]]
            append(k, x, [len(p) for p in paths], [5 * s + t for s, p in enumerate(paths) for t in p])
            after = read()
            for s, p in enumerate(paths):
                for part in (0, 1):
                    src = (k if part == 0 else x[:, (NQ + NKV) * D:])[[5 * s + t for t in p]].cpu().double().numpy()
                    new = after[s][part][-len(p):].reshape(len(p), -1)
                    half = 2.0 ** -4 if cdt == "fp8" else 0.0
                    # (below e4m3's normal range: 2^-10 of a scale of at most 2^-6)
                    assert np.all(np.abs(new - src) <= half * np.abs(src) + half * 2.0 ** -12)
                    old, was = after[s][part][:-len(p)], before[s][part]
                    # (a grown scale rounds values below its normal range again)
                    assert np.all(np.abs(old - was) <= (2.0 ** -16 if cdt == "fp8" else 0.0))
        # the scoring step's attention over the cache that was written
        q1, k1, v1 = (torch.from_numpy(rng.normal(size=(3, n, D)).astype(np.float32)).cuda() for n in (NQ, NKV, NKV))
        b = batch()
        n = m.kvprm_workspace_size(h, b)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        o1 = torch.empty_like(q1)
        m.kvprm_attention(h, cache, b, 0, q1.data_ptr(), k1.data_ptr(), v1.data_ptr(), ws.data_ptr(), n, o1.data_ptr(), st)
        torch.cuda.synchronize()
        held = read()
        for s in range(3):
            for i in range(NQ):
                K, V = (np.concatenate([held[s][p][:, i // 4], t[s, i // 4].cpu().double().numpy()[None]])
                        for p, t in ((0, k1), (1, v1)))
                want = ko.attention(q1[s, i].cpu().double().numpy(), K, V)
                assert np.all(np.abs(o1[s, i].cpu().numpy() - want) <= 1e-4)
    finally:
        m.kvprm_destroy(h)
