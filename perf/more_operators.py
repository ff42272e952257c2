"""Two groups of operators of a serving cache as cases to measure: a cache held in 4 bits (its rows
quantised and read back, attention of a verify token and of drafted tokens over it), and its pages
(a beam's rows forked with copy-on-write, the pool compacted).

A case is a dict of plain values. ``prepare`` makes what a program holds before the call, ``run``
makes one pass, ``exact`` computes the same outputs in float64. With ``own`` false, ``run`` is the
plain form: elementary torch operations in 32 bits, rounded once at the end. With ``own`` true it
makes the calls of the library.

The 4-bit format: e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one power of two
for 32 dims of a token as an 8-bit exponent (biased by 127), the smallest s with 7 s >= |x| (2^-100
to 2^125), codes to the nearest value, ties to the even code. Model shapes are those of the benchmark
and the tests. Lengths, row counts and who is whose child belong to the case (the same for every
seed), so that its work is known; everything else comes from the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16
GROUP = 32  # dims that share a scale of the 4-bit cache
# query heads, kv-heads, head dim
SHAPES = {
    "tiny": (4, 2, 64),      # the parity shape
    "g4": (16, 4, 64),       # head dim 64
    "b06": (16, 8, 128),     # the shape of the depth-k readout experiment
    "g16": (32, 2, 128),     # 16 query heads per kv-head
    "b7": (28, 4, 128),      # the 7B shape of the benchmark
    "large": (64, 8, 128),   # the large shape of the benchmark
}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "fp8": 1}
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _attn(name, shape, batch, lo, hi):
    return {"name": name, "op": "attn", "shape": shape, "batch": batch, "lo": lo, "hi": hi}


def _tree(name, shape, dtype, batch, lo, hi, nlo, nhi, chain=False):
    return {"name": name, "op": "tree", "shape": shape, "dtype": dtype, "batch": batch, "lo": lo, "hi": hi,
            "nlo": nlo, "nhi": nhi, "chain": chain}


def _write(name, shape, dtype, batch, lo, hi, nlo, nhi, pick=0):
    return {"name": name, "op": "write", "shape": shape, "dtype": dtype, "batch": batch, "lo": lo, "hi": hi,
            "nlo": nlo, "nhi": nhi, "pick": pick}


def _fork(name, shape, kvdt, layers, rows, prefix, lo, hi, children, room, fresh=0):
    return {"name": name, "op": "fork", "shape": shape, "kvdt": kvdt, "layers": layers, "rows": rows,
            "prefix": prefix, "lo": lo, "hi": hi, "children": children, "room": room, "fresh": fresh}


def _compact(name, shape, kvdt, layers, rows, prefix, lo, hi, loose):
    return {"name": name, "op": "compact", "shape": shape, "kvdt": kvdt, "layers": layers, "rows": rows,
            "prefix": prefix, "lo": lo, "hi": hi, "loose": loose}


def listed():
    return [
        # the verify token of one trajectory of a small policy: latency
        _attn("attn_one_b06", "b06", 1, 1103, 1103),
        # ragged batch, head dim 64, down to a single cached token
        _attn("attn_ragged_g4", "g4", 24, 1, 9000),
        # long ragged trajectories: the benchmark's batch over a cache of 4 bits
        _attn("attn_long_b7", "b7", 8, 16384, 32768),
        # one trajectory, a tree of 16 drafted tokens: latency
        _tree("tree_one_b06", "b06", "bf16", 1, 1103, 1103, 16, 16),
        # long ragged trajectories, 64 drafted tokens each: products, not memory
        _tree("tree_long_b7", "b7", "bf16", 8, 16384, 32768, 64, 64),
        # one new token of 16 sequences: latency
        _write("write_step_large", "large", "bf16", 16, 8192, 16384, 1, 1),
        # long ragged prompts quantised as they are written, and what the cache holds of them
        _write("write_prompts_b7", "b7", "bf16", 8, 0, 300, 16384, 32768),
        # four candidates of an fp32 model, two of them dropped: latency
        _fork("fork_few_tiny", "tiny", "f32", 2, 4, 64, 1, 200, 4, 16),
        # a beam of 64 over one prompt after pruning, room for the next step
        _fork("fork_beam_b7", "b7", "bf16", 28, 64, 4096, 150, 450, 64, 64),
        # sequences that leave an fp8 server's batch and new ones that join it
        _fork("fork_server_fp8", "large", "fp8", 16, 16, 0, 300, 2000, 16, 300, 8),
        # a small pool with holes: latency
        _compact("compact_few_tiny", "tiny", "f32", 2, 4, 64, 1, 300, 200),
        # a pool that a beam's end has left a third empty, made dense so that its end can go
        _compact("compact_pool_b7", "b7", "bf16", 28, 32, 0, 300, 1200, 150),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _fit(case):
    """The case with fewer sequences where it would cost more than the largest listed one of its operator."""
    most = {k: max(work(c)[k] for c in listed() if c["op"] == case["op"]) for k in ("bytes", "flops")}
    pools = max(_pool_bytes(c) for c in listed())
    size = "rows" if "rows" in case else "batch"
    while case[size] > 1 and (any(work(case)[k] > most[k] for k in most) or _pool_bytes(case) > pools):
        case[size] //= 2
    while "layers" in case and case["layers"] > 1 and (work(case)["bytes"] > most["bytes"] or
                                                       _pool_bytes(case) > pools):
        case["layers"] //= 2
    return case


def draw(rng):
    op = rng.choice(["attn", "attn", "tree", "tree", "write", "fork", "compact"])
    shape = rng.choice(["tiny", "g4", "b06", "g16", "b7", "large"])
    if op in ("fork", "compact"):
        rows, hi = _log(rng, 1, 64), _log(rng, 1, 4000)
        lo, prefix = rng.randint(1, hi), rng.choice([0, PAGE * _log(rng, 1, 256)])
        common = ("", shape, rng.choice(["f32", "bf16", "fp8"]), _log(rng, 1, 28), rows, prefix, lo, hi)
        if op == "fork":
            return _fit(_fork(*common, _log(rng, 1, 64), rng.choice([0, _log(rng, 1, 500)]), rng.choice([0, rng.randint(1, 8)])))
        return _fit(_compact(*common, rng.randint(101, 400)))
    batch, hi = _log(rng, 1, 32), _log(rng, 1, 32768)
    lo = rng.randint(0, hi)
    if op == "attn":
        return _fit(_attn("", shape, batch, lo, hi))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "write":
        nhi = _log(rng, 1, 16384)
        return _fit(_write("", shape, dtype, batch, lo // 4, hi // 4, rng.randint(1, nhi), nhi,
                           pick=rng.choice([0, 64]) if nhi <= 64 else 0))
    nhi = _log(rng, 1, 256)
    return _fit(_tree("", shape, dtype, batch, lo, hi, rng.randint(1, nhi), nhi, rng.random() < 0.2))


# ------------------------------------------------------------------------------ inputs


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _own_rng(case):
    """A random.Random that depends on the case alone (not on its name or a seed)."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _counts(case):
    """Cached lengths and new rows of every sequence."""
    rng = _own_rng(case)
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    return lens, [rng.randint(case["nlo"], case["nhi"]) for _ in lens] if "nlo" in case else [0] * len(lens)


def _rows_held(case):
    """For the cases of pages: each row's tokens and held pages; of a fork, the children's parents as well."""
    rng = _own_rng(case)
    lens = [case["prefix"] + rng.randint(case["lo"], case["hi"]) for _ in range(case["rows"])]
    held = [_pages(n + rng.choice([0, 0, rng.randint(1, 40)])) for n in lens]
    if case["op"] != "fork":
        return lens, held, []
    kept = rng.sample(range(case["rows"]), (case["rows"] + 1) // 2)  # the rows that have children
    parent = [rng.choice(kept) for _ in range(case["children"])]
    for i in rng.sample(range(case["children"]), min(case["fresh"], case["children"])):
        parent[i] = -1  # a new sequence
    return lens, held, parent


def _pool_pages(case):
    lens, held, _ = _rows_held(case)
    live = case["prefix"] // PAGE + sum(h - case["prefix"] // PAGE for h in held)
    if case["op"] == "compact":
        return max(live, live * case["loose"] // 100)
    return (live + case["children"] * (1 + _pages(case["room"]))) * 5 // 4


def _page_bytes(case):
    """Keys and values of one page and layer, with their scales."""
    _, nkv, d = SHAPES[case["shape"]]
    return 2 * nkv * (PAGE * d * SIZE[case["kvdt"]] + (4 if case["kvdt"] == "fp8" else 0))


def _pool_bytes(case):
    return _pool_pages(case) * case["layers"] * _page_bytes(case) if "layers" in case else 0


def _copies(case):
    """Pages that a fork copies: partly filled ones of children that are not their parent's first."""
    lens, _, parent = _rows_held(case)
    return sum(p >= 0 and lens[p] % PAGE != 0 and p in parent[:i] for i, p in enumerate(parent))


def _gen(seed, what, device="cuda"):
    return torch.Generator(device=device).manual_seed((seed * 1_000_003 + what) & 0x7FFFFFFFFFFF)


def _normal(shape, std, seed, what, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, what), device="cuda").mul_(std).to(dtype)


def _table(case, seed, lens, rows):
    """Page ids of every sequence, room for its new rows included, scattered over a pool."""
    want = [_pages(n + (r if case["op"] == "write" else 0)) for n, r in zip(lens, rows)]
    pool = max(1, sum(want) * 5 // 4)
    ids = torch.randperm(pool, generator=_gen(seed, 1, "cpu")).tolist()
    at, width, table = 0, max(1, max(want)), []
    for n in want:
        table.append(ids[at:at + n] + [-1] * (width - n))
        at += n
    return table, pool


def _power(k):
    """2^k in fp32, k whole, -126 to 127."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _quantised(x):
    """Values [..., d] in 32 bits -> 4-bit codes [..., d] and scale bytes [..., d / 32]."""
    g = x.unflatten(-1, (-1, GROUP))
    m, e = torch.frexp(g.abs().amax(dim=-1))
    k = (e - 3 + (m > 0.875).int()).clamp(-100, 125)
    y = g * _power(-k[..., None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    return (code + 8 * torch.signbit(y)).flatten(-2).to(torch.uint8), (k + 127).to(torch.uint8)


def _values(code, scale):
    """The reverse, in 32 bits."""
    lut = torch.tensor(VALUES + [-v for v in VALUES], device=code.device)
    v = torch.index_select(lut, 0, code.reshape(-1).int()).reshape(code.shape).unflatten(-1, (-1, GROUP))
    return (v * _power(scale.int() - 127)[..., None]).flatten(-2)


# Views of a pool [pages][kv-heads][8.5 d bytes]: the code bytes and the scale bytes of keys by (group, slot),
# of values by (slot / 4, slot % 4) and so on. A byte of keys holds two neighbouring dims of a slot, one of
# values dims m and m + 16 of a slot.


def _key_views(pool, d):
    n = pool.shape[:2]
    return pool[..., :8 * d].unflatten(-1, (d // GROUP, PAGE, 16)), pool[..., 8 * d:].reshape(*n, d // GROUP, PAGE)


def _value_views(pool, d):
    return (pool[..., :8 * d].unflatten(-1, (4, 16, d // GROUP, 4)),
            pool[..., 8 * d:].unflatten(-1, (4, d // GROUP, 4)))


def _put(pool, part, d, page, slot, code, scale):
    """Codes [n][kv-heads][d] and scales [n][kv-heads][d / 32] of n tokens into their pages."""
    n, nkv = code.shape[:2]
    if part == 0:
        cells, scales = _key_views(pool, d)
        pair = code.reshape(n, nkv, d // GROUP, 16, 2)
        cells[page, :, :, slot] = pair[..., 0] + 16 * pair[..., 1]
        scales[page, :, :, slot] = scale
    else:
        cells, scales = _value_views(pool, d)
        half = code.reshape(n, nkv, d // GROUP, 2, 16)
        cells[page, :, slot // 4, :, :, slot % 4] = (half[..., 0, :] + 16 * half[..., 1, :]).transpose(2, 3)
        scales[page, :, slot // 4, :, slot % 4] = scale


def _get(pool, part, d, page, slot):
    """Codes and scales of tokens, as _put takes them."""
    nkv = pool.shape[1]
    if part == 0:
        cells, scales = _key_views(pool, d)
        b = cells[page, :, :, slot]
        return torch.stack([b & 15, b >> 4], dim=-1).reshape(-1, nkv, d), scales[page, :, :, slot]
    cells, scales = _value_views(pool, d)
    b = cells[page, :, slot // 4, :, :, slot % 4].transpose(2, 3)
    return torch.stack([b & 15, b >> 4], dim=3).reshape(-1, nkv, d), scales[page, :, slot // 4, :, slot % 4]


def _four_bit_pool(shape, pool, seed, part):
    """Pages of keys or values near N(0, 1): some dims of the keys are several times larger, as a rotary
    model's are."""
    _, nkv, d = SHAPES[shape]
    out = torch.empty((pool, nkv, 17 * d // 2), dtype=torch.uint8, device="cuda")
    gen = _gen(seed, 20 + part)
    wide = torch.ones(d, device="cuda")
    if part == 0:
        wide[torch.randperm(d, generator=gen, device="cuda")[:d // 16]] = 4.0
    step = max(1, (1 << 25) // (nkv * PAGE * d))
    slots = torch.arange(PAGE, device="cuda")
    for at in range(0, pool, step):
        n = min(step, pool - at)
        x = torch.randn((n * PAGE, nkv, d), generator=gen, device="cuda") * wide
        code, scale = _quantised(x)
        _put(out[at:at + n], part, d, torch.arange(n, device="cuda").repeat_interleave(PAGE), slots.repeat(n),
             code, scale)
    return out


def _ancestors(seed, rows):
    """One random tree per sequence: for each drafted token the bits of the tokens it attends to
    (itself and its ancestors), as 32-bit words."""
    words = (max(rows) + 31) // 32
    out = np.zeros((sum(rows), words), dtype=np.uint32)
    rng, at = random.Random(seed), 0
    for n in rows:
        bits = []
        for t in range(n):
            parent = t - 1 - int(rng.expovariate(0.5))
            bits.append((bits[parent] if parent >= 0 else 0) | 1 << t)
        raw = b"".join(v.to_bytes(4 * words, "little") for v in bits)
        out[at:at + n] = np.frombuffer(raw, dtype="<u4").reshape(n, words)
        at += n
    return torch.from_numpy(out.view(np.int32))


class _State:
    handle = None

    def __del__(self):
        if self.handle is not None:
            import paper_2607_09153_amd as kv
            kv.kvprm_destroy(self.handle)


def _ints(v, *shape):
    t = torch.tensor(v, dtype=torch.int32, device="cuda")
    return t.reshape(shape) if shape else t


def _prepare_pages(s, case, seed):
    """A pool whose pages rows hold (a shared prefix first), the rows' table, and every page's holders."""
    _, nkv, d = SHAPES[case["shape"]]
    s.lens, s.held, s.parent = _rows_held(case)
    s.pool = _pool_pages(case)
    # which pages are held decides how many a compaction moves: that belongs to the case
    ids = list(range(s.pool))
    (_own_rng(case) if case["op"] == "compact" else random.Random(seed)).shuffle(ids)
    pre = case["prefix"] // PAGE
    at, width, table = pre, max(1, max(s.held)), []
    for h in s.held:
        table.append(ids[:pre] + ids[at:at + h - pre] + [-1] * (width - h))
        at += h - pre
    refs = [0] * s.pool
    for row, h in zip(table, s.held):
        for p in row[:h]:
            refs[p] += 1
    s.width = width
    s.table, s.refs = _ints(table, len(table), width), _ints(refs)
    s.lengths, s.holds = _ints(s.lens), _ints(s.held)
    shape = (case["layers"], s.pool, nkv, PAGE * d)
    s.pools, s.scales = [], []
    for part in (0, 1):
        s.pools.append(torch.empty(shape, dtype=TORCH[case["kvdt"]], device="cuda"))
        for layer in range(case["layers"]):
            s.pools[-1][layer] = _normal(shape[1:], 1.0, seed, 100 + 2 * layer + part)
        if case["kvdt"] == "fp8":
            s.scales.append(torch.exp2(_normal(shape[:3], 1.0, seed, 50 + part).round()))
    s.new_refs, s.result = torch.zeros_like(s.refs), _ints([0] * 4)
    if case["op"] == "fork":
        n = case["children"]
        s.parents = _ints(s.parent)
        s.room = _ints([case["room"]] * n)
        s.new_width = max(_pages((s.lens[p] if p >= 0 else 0) + case["room"]) for p in s.parent) or 1
        s.new_table = torch.zeros((n, s.new_width), dtype=torch.int32, device="cuda")
        s.new_lengths, s.new_holds = _ints([0] * n), _ints([0] * n)
    else:
        s.new_table = torch.zeros_like(s.table)
        s.moved = torch.zeros_like(s.refs)


def prepare(case, seed):
    s = _State()
    s.case, s.op = case, case["op"]
    nq, nkv, d = SHAPES[case["shape"]]
    if s.op in ("fork", "compact"):
        _prepare_pages(s, case, seed)
        if own:
            _bind_pages(s)
        return s
    lens, rows = _counts(case)
    table, s.pool = _table(case, seed, lens, rows)
    s.counts, s.n = (lens, rows), sum(rows)
    s.table, s.lens = _ints(table, len(lens), -1), _ints(lens)
    s.start = _ints([0] + [int(x) for x in np.cumsum(rows)])
    s.pools = [_four_bit_pool(case["shape"], s.pool, seed, part) for part in (0, 1)]
    s.index = None
    if s.op == "attn":
        # the rotated query, key and value of each verify token, as the projection leaves them
        B = len(lens)
        s.q = _normal((B, nq, d), 1.0, seed, 3)
        s.k, s.v = (_normal((B, nkv, d), 1.0, seed, w) for w in (4, 5))
        s.o = torch.zeros((B, nq, d), device="cuda")
    elif s.op == "tree":
        # q, k, v inside the fused projection's output
        dt = TORCH[case["dtype"]]
        s.qkv = _normal((s.n, (nq + 2 * nkv) * d), 1.0, seed, 8, dt)
        s.mask = None if case["chain"] else _ancestors(seed, rows).cuda()
        s.o = torch.zeros((s.n, nq, d), dtype=dt, device="cuda")
    else:
        dt, have = TORCH[case["dtype"]], s.n
        if case["pick"]:  # each sequence's rows out of its draft of `pick`, in ascending order
            rng = random.Random(seed)
            have = case["pick"] * len(lens)
            s.index = _ints([b * case["pick"] + t for b, r in enumerate(rows)
                             for t in sorted(rng.sample(range(case["pick"]), r))])
        # keys as the rotary step left them, values inside the fused projection's output
        size = torch.exp(_normal((have, 1), 0.5, seed, 5))
        s.k = (_normal((have, nkv * d), 1.0, seed, 6) * size).to(dt)
        s.v = torch.cat([torch.zeros((have, (nq + nkv) * d), dtype=dt, device="cuda"),
                         (_normal((have, nkv * d), 1.0, seed, 7) * size).to(dt)], dim=1)
        s.out = [torch.zeros((s.n, nkv, d), dtype=dt, device="cuda") for _ in (0, 1)]
        s.after = s.lens + (s.start[1:] - s.start[:-1])  # lengths once the rows are in
    if own:
        _bind(s)
    return s


# ------------------------------------------------------------------------------ the library


def _bind(s):
    """What a program keeps beside its tensors: the handle, the descriptors, the workspace."""
    import paper_2607_09153_amd as kv
    c = s.case
    nq, nkv, d = SHAPES[c["shape"]]
    lens, rows = s.counts
    s.kv = kv
    s.handle = kv.kvprm_create(kv.make_desc(1, 64 * nq, nq, nkv, d, 64, 1.0e6, 1e-6, "bf16", "fp4"))
    s.cache = kv.make_cache(s.pools[0].data_ptr(), s.pools[1].data_ptr(), s.pool)
    s.batch = kv.make_batch(len(lens), s.table.data_ptr(), s.table.shape[1], s.lens.data_ptr(), lens)
    most = max(rows)
    if s.op == "attn":
        need = kv.kvprm_workspace_size(s.handle, s.batch)
    elif s.op == "tree":
        base, e, width = s.qkv.data_ptr(), s.qkv.element_size(), s.qkv.shape[1]
        s.tree = kv.make_tree(base, base + nq * d * e, base + (nq + nkv) * d * e, s.o.data_ptr(), c["dtype"],
                              width, width, width, nq * d, s.n, s.start.data_ptr(), most,
                              s.mask.data_ptr() if s.mask is not None else 0,
                              s.mask.shape[1] if s.mask is not None else 0)
        need = kv.kvprm_workspace_size_tree(s.handle, s.batch, s.tree)
    else:
        s.rows = kv.make_kv_rows(s.k.data_ptr(), s.v.data_ptr() + (nq + nkv) * d * s.v.element_size(),
                                 c["dtype"], nkv * d, s.v.shape[1], s.k.shape[0], s.start.data_ptr(), most,
                                 s.index.data_ptr() if s.index is not None else 0)
        s.back = kv.make_kv_rows(s.out[0].data_ptr(), s.out[1].data_ptr(), c["dtype"], nkv * d, nkv * d, s.n,
                                 s.start.data_ptr(), most)
        s.later = kv.make_batch(len(lens), s.table.data_ptr(), s.table.shape[1], s.after.data_ptr(),
                                [n + r for n, r in zip(lens, rows)])
        return
    s.ws = torch.empty(need, dtype=torch.uint8, device="cuda")


def _bind_pages(s):
    import paper_2607_09153_amd as kv
    c = s.case
    nq, nkv, d = SHAPES[c["shape"]]
    s.kv = kv
    s.handle = kv.kvprm_create(kv.make_desc(c["layers"], 64 * nq, nq, nkv, d, 64, 1.0e6, 1e-6,
                                            "f32" if c["kvdt"] == "f32" else "bf16", c["kvdt"]))
    s.cache = kv.make_cache(s.pools[0].data_ptr(), s.pools[1].data_ptr(), s.pool,
                            *[t.data_ptr() for t in s.scales])
    s.rows = kv.make_page_rows(len(s.lens), s.width, s.table.data_ptr(), s.lengths.data_ptr(), s.holds.data_ptr())
    if s.op == "fork":
        s.to = kv.make_page_rows(c["children"], s.new_width, s.new_table.data_ptr(), s.new_lengths.data_ptr(),
                                 s.new_holds.data_ptr())
    s.ws = torch.empty(kv.kvprm_workspace_size_pages(s.handle, s.pool), dtype=torch.uint8, device="cuda")


def _run_own(s):
    kv, st = s.kv, torch.cuda.current_stream().cuda_stream
    if s.op == "attn":
        kv.kvprm_attention(s.handle, s.cache, s.batch, 0, s.q.data_ptr(), s.k.data_ptr(), s.v.data_ptr(),
                           s.ws.data_ptr(), s.ws.numel(), s.o.data_ptr(), st)
        return s.o
    if s.op == "tree":
        kv.kvprm_attention_tree(s.handle, s.cache, s.batch, 0, s.tree, s.ws.data_ptr(), s.ws.numel(), st)
        return s.o
    if s.op == "write":
        kv.kvprm_write_kv(s.handle, s.cache, s.batch, 0, s.rows, st)
        kv.kvprm_read_kv(s.handle, s.cache, s.later, 0, s.back, s.lens.data_ptr(), st)
        return s.out
    if s.op == "fork":
        kv.kvprm_fork_pages(s.handle, s.cache, s.rows, s.to, s.parents.data_ptr(), s.room.data_ptr(),
                            s.refs.data_ptr(), s.new_refs.data_ptr(), s.result.data_ptr(), s.ws.data_ptr(),
                            s.ws.numel(), st)
        return [s.new_table, s.new_lengths, s.new_holds, s.new_refs, s.result] + s.pools + s.scales
    kv.kvprm_compact_pages(s.handle, s.cache, s.rows, s.new_table.data_ptr(), s.refs.data_ptr(),
                           s.new_refs.data_ptr(), s.moved.data_ptr(), s.result.data_ptr(), s.ws.data_ptr(),
                           s.ws.numel(), st)
    return [s.new_table, s.new_refs, s.moved, s.result] + s.pools + s.scales


# ------------------------------------------------------------------------------ the plain form


def _cached(s, part, count):
    """Keys or values at positions 0 .. count - 1 of every sequence, [B][count][kv-heads][d], in 32 bits
    (positions past a sequence's length repeat its first)."""
    nkv, d = SHAPES[s.case["shape"]][1:]
    B = s.lens.shape[0]
    pos = torch.arange(count, device="cuda").expand(B, count)
    pos = torch.where(pos < s.lens[:, None], pos, 0)
    page = torch.gather(s.table.long(), 1, pos // PAGE).clamp(min=0)
    return _values(*_get(s.pools[part], part, d, page.reshape(-1), (pos % PAGE).reshape(-1))).reshape(B, count, nkv, d)


def _softmax_sum(q, key, val, ok):
    """softmax(q key^T / sqrt(d)) val where ok; rows that attend to nothing are 0. Batches of matrices."""
    sc = torch.bmm(q, key.transpose(1, 2).contiguous()).mul_(q.shape[-1] ** -0.5).masked_fill_(~ok, -math.inf)
    top = sc.amax(dim=2, keepdim=True)
    p = sc.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = p.sum(dim=2, keepdim=True)
    return torch.bmm(p, val) / torch.where(total > 0, total, 1)


def _plain_attn(s):
    nq, nkv, d = SHAPES[s.case["shape"]]
    B, Lm = len(s.counts[0]), max(s.counts[0])
    ok = torch.arange(Lm + 1, device="cuda") < s.lens[:, None]
    ok[:, Lm] = True  # the verify token itself
    key, val = (torch.cat([_cached(s, part, Lm), own_row[:, None]], dim=1).transpose(1, 2)
                .reshape(B * nkv, Lm + 1, d) for part, own_row in ((0, s.k), (1, s.v)))
    ok = ok[:, None, None].expand(B, nkv, nq // nkv, Lm + 1).reshape(B * nkv, nq // nkv, Lm + 1)
    return _softmax_sum(s.q.reshape(B * nkv, nq // nkv, d), key, val, ok).reshape(B, nq, d)


def _row_places(s):
    """Sequence of every row, and its place among that sequence's rows."""
    r = torch.arange(s.n, device="cuda")
    b = torch.searchsorted(s.start[1:].contiguous(), r, right=True)
    return b, r - s.start[b]


def _plain_tree(s):
    nq, nkv, d = SHAPES[s.case["shape"]]
    lens, rows = s.counts
    B, T, Lm, g = len(lens), max(rows), max(lens), nq // nkv
    q, k, v = s.qkv.split([nq * d, nkv * d, nkv * d], dim=1)
    t = torch.arange(T, device="cuda")
    count = (s.start[1:] - s.start[:-1])[:, None]
    row = (s.start[:-1].long()[:, None] + t).clamp(max=s.n - 1)
    q = q.reshape(-1, nkv, g, d)[row].permute(0, 2, 1, 3, 4).reshape(B * nkv, T * g, d).float()
    seen = (torch.arange(Lm, device="cuda") < s.lens[:, None])[:, None, :].expand(B, T, Lm)
    if s.mask is None:
        bits = (t[None, :] <= t[:, None])[None].expand(B, T, T)
    else:
        bits = (s.mask[row][..., t // 32] >> (t % 32)) & 1 != 0
    ok = torch.cat([seen, bits & (t < count)[:, None, :]], dim=2)
    ok = ok[:, None, :, None].expand(B, nkv, T, g, Lm + T).reshape(B * nkv, T * g, Lm + T)
    key, val = (torch.cat([_cached(s, part, Lm), x.reshape(-1, nkv, d)[row].float()], dim=1)
                .transpose(1, 2).reshape(B * nkv, Lm + T, d) for part, x in ((0, k), (1, v)))
    o = _softmax_sum(q, key, val, ok).reshape(B, nkv, T, g, d).permute(0, 2, 1, 3, 4).reshape(B, T, nq, d)
    return o[_row_places(s)].to(s.o.dtype)


def _plain_write(s):
    nq, nkv, d = SHAPES[s.case["shape"]]
    b, i = _row_places(s)
    pos = s.lens[b].long() + i
    page, slot = s.table[b, pos // PAGE].long(), pos % PAGE
    out = []
    for part, src in ((0, s.k), (1, s.v[:, (nq + nkv) * d:])):
        x = src.reshape(-1, nkv, d)
        x = (x if s.index is None else x[s.index.long()]).float()
        _put(s.pools[part], part, d, page, slot, *_quantised(x))
        out.append(_values(*_get(s.pools[part], part, d, page, slot)).to(src.dtype))
    return out


def _free_ids(free, most):
    """Ids of the first `most` free pages in ascending order."""
    rank = torch.cumsum(free, 0) - 1
    ids = torch.zeros(most + 1, dtype=torch.long, device="cuda")
    at = torch.where(free & (rank < most), rank, most)
    return ids.scatter_(0, at, torch.arange(free.shape[0], device="cuda"))[:most]


def _count(ids, ok, like):
    """How often each page stands among the entries that are ok."""
    return torch.zeros_like(like).index_add_(0, torch.where(ok, ids, 0).reshape(-1).long(),
                                             ok.reshape(-1).to(like.dtype))


def _plain_fork(s):
    c, W = s.case, s.new_width
    n, par = c["children"], s.parents.long()
    got = par >= 0
    src = par.clamp(min=0)
    length = torch.where(got, s.lengths[src], 0)
    full, part = length // PAGE, length % PAGE != 0
    held = (length + s.room + PAGE - 1) // PAGE
    col = torch.arange(W, device="cuda")
    old = s.table.gather(1, col.clamp(max=s.width - 1).expand(len(s.lens), W))[src]
    last = old.gather(1, full.long()[:, None].clamp(max=W - 1))[:, 0].clamp(min=0).long()
    first = ~((par[None, :] == par[:, None]).tril(-1).any(dim=1))
    keep = got & part & first & (s.refs[last] == 1)
    copy = got & part & ~keep
    shared = col < (full + keep.int())[:, None]
    refs = s.refs - _count(s.table, torch.arange(s.width, device="cuda") < s.holds[:, None], s.refs)
    refs += _count(old, shared, s.refs)
    free = (refs == 0) & (_count(last, copy, s.refs) == 0)
    # fresh pages in the order of the children's entries, the lowest free ids first
    want = (col < held[:, None]) & ~shared
    rank = (torch.cumsum(want.reshape(-1), 0) - 1).reshape(n, W)
    most = n * W
    ids = _free_ids(free, most)
    table = torch.where(shared, old, torch.where(want, ids[rank.clamp(min=0)].int(), -1))
    refs += _count(table, want, s.refs)
    fresh = table.gather(1, full.long()[:, None].clamp(max=W - 1))[:, 0].long()
    to, come = fresh[copy], last[copy]
    for t in s.pools + s.scales:
        b = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
        b[:, to] = b[:, come]
    need = want.sum()
    result = torch.stack([torch.zeros_like(need), need, free.sum(), (refs == 0).sum()]).int()
    return [table, length.int(), held.int(), refs, result] + s.pools + s.scales


def _plain_compact(s):
    live = s.refs > 0
    count = live.sum()
    ids = torch.arange(s.pool, device="cuda")
    high, low = live & (ids >= count), ~live & (ids < count)
    rank = torch.cumsum(high, 0) - 1
    to = torch.where(high, _free_ids(low, s.pool)[rank.clamp(min=0)], ids)
    refs = torch.zeros_like(s.refs).index_add_(0, to, torch.where(live, s.refs, 0))
    moved = torch.where(live, to, -1).int()
    own_entry = torch.arange(s.width, device="cuda") < s.holds[:, None]
    table = torch.where(own_entry, moved[s.table.clamp(min=0).long()], -1)
    goes, come = to[high], ids[high]
    for t in s.pools + s.scales:
        b = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
        b[:, goes] = b[:, come]
    result = torch.stack([torch.zeros_like(count), count, high.sum(), s.pool - count]).int()
    return [table, refs, moved, result] + s.pools + s.scales


def run(s):
    if own:
        return _run_own(s)
    return {"attn": _plain_attn, "tree": _plain_tree, "write": _plain_write, "fork": _plain_fork,
            "compact": _plain_compact}[s.op](s)


# ------------------------------------------------------------------------------ the measure


def work(case):
    nq, nkv, d = SHAPES[case["shape"]]
    if case["op"] in ("fork", "compact"):
        lens, held, parent = _rows_held(case)
        pool, tables = _pool_pages(case), 4 * (sum(held) + 2 * len(held))
        if case["op"] == "fork":
            pages = _copies(case)
            tables += 4 * sum(_pages((lens[p] if p >= 0 else 0) + case["room"]) + 4 for p in parent)
        else:
            ids = list(range(pool))
            _own_rng(case).shuffle(ids)
            live = case["prefix"] // PAGE + sum(h - case["prefix"] // PAGE for h in held)
            pages = sum(p >= live for p in ids[:live])
            tables = 2 * tables + 4 * pool
        return {"bytes": 2 * pages * case["layers"] * _page_bytes(case) + tables + 8 * pool, "flops": 0}
    lens, rows = _counts(case)
    code = 17 / 32  # bytes of a value and its share of the scale
    if case["op"] == "write":  # rows read, codes written and read, rows written
        n = 2 * sum(rows) * nkv * d
        return {"bytes": 2 * n * (SIZE[case["dtype"]] + code), "flops": n}
    cache = 2 * sum(lens) * nkv * d * code
    if case["op"] == "attn":
        return {"bytes": cache + len(lens) * (2 * nq + 2 * nkv) * d * 4, "flops": 4 * (sum(lens) + len(lens)) * nq * d}
    seen = sum(r * (n + (r + 1) / 2) for n, r in zip(lens, rows))
    return {"bytes": cache + sum(rows) * (2 * nq + 2 * nkv) * d * SIZE[case["dtype"]], "flops": 4 * seen * nq * d}


# ------------------------------------------------------------------------------ in 64 bits


def _two(k):
    """2^k in float64, k whole."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_cached(s, part, b, first, last):
    """Cached vectors [kv-heads][tokens][d] of sequence b in float64, byte by byte from the format."""
    d = SHAPES[s.case["shape"]][2]
    slot = torch.arange(PAGE, device="cuda")[:, None]
    m = torch.arange(d, device="cuda")[None]
    if part == 0:
        byte, high, scale = (m // 32 * 16 + slot) * 16 + m % 32 // 2, m % 2, 8 * d + m // 32 * 16 + slot
    else:
        in_cell = m // 32 * 4 + slot % 4
        byte, high, scale = (slot // 4 * 16 + m % 16) * (d // 8) + in_cell, m // 16 % 2, 8 * d + slot // 4 * (d // 8) + in_cell
    n = _pages(last)
    tiles = s.pools[part][s.table[b, :n].long()].transpose(0, 1)
    nibble = tiles[..., byte].int() >> (4 * high) & 15
    e, frac = (nibble >> 1 & 3).double(), (nibble & 1).double()
    v = torch.where(e == 0, frac / 2, (1 + frac / 2) * _two(e - 1)) * (1 - 2 * (nibble >> 3).double())
    v = v * _two(tiles[..., scale].int() - 127)
    return v.reshape(v.shape[0], n * PAGE, d)[:, first:last]


def _exact_heads(q, k, v, mask=None):
    """q [g][r][d] over k, v [n][d]; mask [r][n]: what a row may attend to."""
    g, r, d = q.shape
    z = torch.mm(q.reshape(-1, d), k.t().contiguous()).reshape(g, r, -1) / math.sqrt(d)
    if mask is not None:
        z.masked_fill_(~mask, -math.inf)
    return torch.mm(torch.softmax(z, dim=2).reshape(g * r, -1), v).reshape(g, r, d)


def _exact_attn(case, seed):
    s = prepare(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    out = torch.empty((len(s.counts[0]), nq, d), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s.counts[0]):
        K, V = (torch.cat([_exact_cached(s, p, b, 0, n), x[b].double()[:, None]], dim=1) if n else x[b].double()[:, None]
                for p, x in ((0, s.k), (1, s.v)))
        for j in range(nkv):
            q = s.q[b].double().reshape(nkv, nq // nkv, 1, d)[j]
            out[b].reshape(nkv, nq // nkv, 1, d)[j] = _exact_heads(q, K[j], V[j])
    return out


def _exact_tree(case, seed):
    s = prepare(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    out, at = [], 0
    for b, (n, r) in enumerate(zip(*s.counts)):
        x = s.qkv[at:at + r].double()
        q = x[:, :nq * d].reshape(r, nkv, nq // nkv, d).permute(1, 2, 0, 3)
        own_k, own_v = (y.reshape(r, nkv, d).transpose(0, 1) for y in x[:, nq * d:].split(nkv * d, dim=1))
        sees = torch.ones((r, r), dtype=torch.bool, device="cuda").tril() if s.mask is None else torch.stack(
            [(s.mask[at:at + r, j // 32] >> (j % 32)) & 1 == 1 for j in range(r)], dim=1)
        mask = torch.cat([torch.ones((r, n), dtype=torch.bool, device="cuda"), sees], dim=1)
        K, V = (torch.cat([_exact_cached(s, p, b, 0, n), y], dim=1) if n else y for p, y in ((0, own_k), (1, own_v)))
        out.append(torch.cat([_exact_heads(q[j], K[j], V[j], mask) for j in range(nkv)]).transpose(0, 1))
        at += r
    return torch.cat(out)


def _exact_write(case, seed):
    s = prepare(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    index = s.index.long() if s.index is not None else torch.arange(s.n, device="cuda")
    out = []
    for src in (s.k, s.v[:, (nq + nkv) * d:]):
        done = []
        for at in range(0, s.n, 16384):
            x = src[index[at:at + 16384]].double().reshape(-1, nkv, d // 32, 32)
            top = x.abs().amax(dim=3, keepdim=True)
            k = torch.floor(torch.log2(top / 7)).clamp(-100, 125)  # or the next, if that is too small
            unit = _two(torch.where(7 * _two(k) >= top, k, k + 1).clamp(max=125))
            y = x / unit
            step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
            y = (torch.round(y / step) * step).clamp(-6, 6)
            done.append((y * unit).reshape(-1, nkv, d))
        out.append(torch.cat(done))
    return out


def _exact_moved(s, src, dst):
    """The pools and scales with pages src copied to dst, as values in 64 bits."""
    out = []
    for t in s.pools + s.scales:
        v = t.double()
        if src:
            v[:, torch.tensor(dst, device="cuda")] = v[:, torch.tensor(src, device="cuda")]
        out.append(v)
    return out


def _exact_fork(case, seed):
    s = prepare(case, seed)
    table, refs = s.table.tolist(), s.refs.tolist()
    holders = list(refs)
    for row, h in zip(table, s.held):
        for p in row[:h]:
            refs[p] -= 1
    rows, copies, had = [], [], set()
    for i, p in enumerate(s.parent):
        n = s.lens[p] if p >= 0 else 0
        row = table[p][:n // PAGE] if p >= 0 else []
        row = list(row)
        if n % PAGE:
            page = table[p][n // PAGE]
            if p not in had and holders[page] == 1:
                row.append(page)
            else:
                copies.append((page, i, n // PAGE))
            had.add(p)
        for page in row:
            refs[page] += 1
        rows.append((row, n, _pages(n + case["room"])))
    sources = {c[0] for c in copies}
    free = [p for p in range(s.pool) if refs[p] == 0 and p not in sources]
    used = 0
    out = []
    for row, n, want in rows:
        more = free[used:used + want - len(row)]
        used += len(more)
        for p in more:
            refs[p] += 1
        out.append(row + more + [-1] * (s.new_width - want))
    moved = _exact_moved(s, [c[0] for c in copies], [out[i][at] for _, i, at in copies])
    return [_ints(out, len(out), s.new_width), _ints([r[1] for r in rows]), _ints([r[2] for r in rows]), _ints(refs),
            _ints([0, used, len(free), refs.count(0)])] + moved


def _exact_compact(case, seed):
    s = prepare(case, seed)
    table, refs = s.table.tolist(), s.refs.tolist()
    live = [p for p in range(s.pool) if refs[p] > 0]
    holes = iter([p for p in range(len(live)) if refs[p] == 0])
    goes = {p: p if p < len(live) else next(holes) for p in live}
    new = [0] * s.pool
    for p, q in goes.items():
        new[q] = refs[p]
    out = [[goes[p] for p in row[:h]] + [-1] * (s.width - h) for row, h in zip(table, s.held)]
    far = [p for p in live if goes[p] != p]
    return [_ints(out, len(out), s.width), _ints(new), _ints([goes.get(p, -1) for p in range(s.pool)]),
            _ints([0, len(live), len(far), s.pool - len(live)])] + _exact_moved(s, far, [goes[p] for p in far])


def exact(case, seed):
    return {"attn": _exact_attn, "tree": _exact_tree, "write": _exact_write, "fork": _exact_fork,
            "compact": _exact_compact}[case["op"]](case, seed)
