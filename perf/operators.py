"""The operators around a cache that grows while a tree of drafted tokens is verified, as cases to
measure: rotary positions, writing rows of keys and values into the paged cache (quantising them
where the cache is fp8), reading them back, and attention of a drafted tree over the cache.

A case is a dict of plain values. ``prepare`` makes what a program holds before the call, ``run``
makes one pass, ``exact`` computes the same outputs in float64. With ``own`` false, ``run`` is the
plain form: elementary torch operations in 32 bits (64 for the angles of far positions), rounded
once at the end. With ``own`` true it makes the calls of the library.

Model shapes are those of the benchmark and the tests. The lengths and row counts of a case belong to
the case (the same for every seed), so that its work is known; everything else comes from the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 16
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
THETA = 1.0e6
TRAINED = 32768.0  # positions the rotary frequencies were trained on, where they are scaled
MIN_EXP = -100     # exponent of the smallest scale of an fp8 tile


def _rotary(name, rows, heads_q, heads_k, d, rot, layout, scaling, dtype, far, grad=False):
    return {"name": name, "op": "rotary", "rows": rows, "hq": heads_q, "hk": heads_k, "d": d, "rot": rot,
            "layout": layout, "scaling": scaling, "dtype": dtype, "far": far, "grad": grad}


def _write(name, shape, kvdt, dtype, batch, lo, hi, nlo, nhi, pick=0):
    return {"name": name, "op": "write", "shape": shape, "kvdt": kvdt, "dtype": dtype, "batch": batch,
            "lo": lo, "hi": hi, "nlo": nlo, "nhi": nhi, "pick": pick}


def _read(name, shape, kvdt, dtype, batch, lo, hi, tail=0):
    return {"name": name, "op": "read", "shape": shape, "kvdt": kvdt, "dtype": dtype, "batch": batch,
            "lo": lo, "hi": hi, "tail": tail}


def _tree(name, shape, kvdt, dtype, batch, lo, hi, nlo, nhi, chain=False):
    return {"name": name, "op": "tree", "shape": shape, "kvdt": kvdt, "dtype": dtype, "batch": batch,
            "lo": lo, "hi": hi, "nlo": nlo, "nhi": nhi, "chain": chain}


def listed():
    return [
        # queries and keys of one decoding step of 16 sequences: latency
        _rotary("rotary_step_b7", 16, 28, 4, 128, 128, "half", "none", "bf16", 32768),
        # a prompt of 8192 tokens past the trained length, frequencies scaled by parts
        _rotary("rotary_prompt_b06", 8192, 16, 8, 128, 128, "half", "parts", "bf16", 131072),
        # the gradient's way back: fp32, adjacent pairs, half of each head rotated
        _rotary("rotary_grad_f32", 4093, 32, 4, 64, 32, "interleaved", "linear", "f32", 32768, grad=True),
        # one new token of 16 sequences into an fp8 cache, pages partly filled: latency
        _write("write_step_fp8", "large", "fp8", "bf16", 16, 8192, 16384, 1, 1),
        # long ragged prompts quantised as they are written
        _write("write_prompts_fp8", "b7", "fp8", "bf16", 8, 0, 300, 16384, 32768),
        # the accepted path of each drafted tree appended, its rows picked out of the draft
        _write("write_accepted_bf16", "b06", "bf16", "f32", 32, 100, 5000, 1, 9, pick=64),
        # ragged fp8 caches read back for another engine
        _read("read_all_fp8", "large", "fp8", "bf16", 16, 8192, 16384),
        # the last tokens of a few bf16 caches, for a comparison in fp32
        _read("read_tail_f32", "g4", "bf16", "f32", 5, 700, 3000, tail=100),
        # one trajectory of a small policy, a tree of 16 drafted tokens: latency
        _tree("tree_one_b06", "b06", "bf16", "bf16", 1, 1103, 1103, 16, 16),
        # an fp32 model, chains of 8
        _tree("tree_tiny_f32", "tiny", "f32", "f32", 4, 512, 512, 8, 8, chain=True),
        # ragged fp8 caches and trees of every size up to 48, head dim 64
        _tree("tree_ragged_fp8", "g4", "fp8", "bf16", 24, 1, 9000, 1, 48),
        # long ragged trajectories, 64 drafted tokens each: products, not memory
        _tree("tree_long_b7", "b7", "bf16", "bf16", 8, 16384, 32768, 64, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _fit(case):
    """The case with fewer sequences (rows) where it would cost more than the largest listed one."""
    largest = [work(c) for c in listed() if c["op"] == case["op"]]
    size = "rows" if case["op"] == "rotary" else "batch"
    # (the matrix cores' fp32 rate is a sixteenth of the bf16 one)
    slow = 16 if case.get("kvdt") == "f32" else 1
    while case[size] > 1 and any(work(case)[k] * (slow if k == "flops" else 1) > max(w[k] for w in largest)
                                 for k in ("bytes", "flops")):
        case[size] //= 2
    return case


def draw(rng):
    op = rng.choice(["rotary", "write", "read", "tree", "tree"])
    shape = rng.choice(["tiny", "g4", "b06", "g16", "b7", "large"])
    if op == "rotary":
        d = rng.choice([64, 80, 96, 128, 128, 256])
        rot = rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)])
        return _fit(_rotary("", _log(rng, 1, 8192), rng.randint(1, 32), rng.randint(0, 8), d, rot,
                            rng.choice(["half", "interleaved"]),
                            rng.choice(["none", "linear", "base", "parts", "ramp"]),
                            rng.choice(["bf16", "f32"]), _log(rng, 64, 1 << 20), rng.random() < 0.3))
    kvdt, dtype = rng.choice([("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("fp8", "bf16"),
                              ("fp8", "f32"), ("bf16", "bf16"), ("fp8", "bf16")])
    batch, hi = _log(rng, 1, 32), _log(rng, 1, 32768)
    lo = rng.randint(0, hi)
    if op == "write":
        nhi = _log(rng, 1, 16384)
        return _fit(_write("", shape, kvdt, dtype, batch, lo // 4, hi // 4, rng.randint(1, nhi), nhi,
                           pick=rng.choice([0, 64]) if nhi <= 64 else 0))
    if op == "read":
        return _fit(_read("", shape, kvdt, dtype, batch, lo + 1, hi + 1, tail=rng.choice([0, 0, _log(rng, 1, 4096)])))
    nhi = _log(rng, 1, 256)
    return _fit(_tree("", shape, kvdt, dtype, batch, lo, hi, rng.randint(1, nhi), nhi, rng.random() < 0.2))


# ------------------------------------------------------------------------------ inputs


def _counts(case):
    """Cached lengths and rows of every sequence."""
    rng = random.Random("%d %d %d" % (case["batch"], case["lo"], case["hi"]))
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    if case["op"] == "read":
        return lens, [min(n, case["tail"]) if case["tail"] else n for n in lens]
    return lens, [rng.randint(case["nlo"], case["nhi"]) for _ in lens]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _normal(shape, std, seed, what, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed((seed * 1_000_003 + what) & 0x7FFFFFFFFFFF)
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def _positions(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, case["far"], (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)


def _rope_args(case):
    """theta, factor, low, high, magnitude of a case's scaling. The last three: turns over the
    trained length below which a pair is interpolated and above which it is left, and the factor
    on the rotated values that goes with it."""
    s = case["scaling"]
    return (THETA, 1.0 if s == "none" else 4.0, 1.0, 32.0,
            0.1 * math.log(4.0) + 1.0 if s in ("parts", "ramp") else 1.0)


def _table(case, seed, lens, rows):
    """Page ids of every sequence, room for its new rows included, scattered over a pool."""
    want = [_pages(n + (r if case["op"] == "write" else 0)) for n, r in zip(lens, rows)]
    pool = max(1, sum(want) * 5 // 4)
    ids = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).tolist()
    at, width, table = 0, max(1, max(want)), []
    for n in want:
        table.append(ids[at:at + n] + [-1] * (width - n))
        at += n
    return table, pool


def _tiles(case, seed, pool, part):
    """Token-major cache tiles [pages][kv-heads][16][head dim] and, for fp8, the tiles' scales
    (powers of two: keys and values near N(0, 1))."""
    _, nkv, d = SHAPES[case["shape"]]
    if case["kvdt"] != "fp8":
        return _normal((pool, nkv, PAGE, d), 1.0, seed, 10 + part, TORCH[case["kvdt"]]), None
    gen = torch.Generator(device="cuda").manual_seed(seed * 2 + part)
    scale = torch.exp2(torch.randint(-8, -5, (pool, nkv), generator=gen, device="cuda").float())
    z = _normal((pool, nkv, PAGE, d), 1.0, seed, 10 + part)
    return (z / scale[:, :, None, None]).clamp_(-448, 448).to(torch.float8_e4m3fn), scale


def _bytes(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def _to_stored(t, part):
    """Token-major tiles in the stored K or V order (a tile's values keep the shape [16][d])."""
    eb, (pool, nkv, _, d) = t.element_size(), t.shape
    x, r = 16 // eb, 4 // eb
    b = _bytes(t)
    if part == 0:
        out = b.reshape(pool, nkv, PAGE, d // x, x).transpose(2, 3)
    else:
        out = b.reshape(pool, nkv, 4, 4, d // (16 * r), r, 16).permute(0, 1, 4, 2, 6, 5, 3)
    return out.reshape(t.shape).view(t.dtype)


def _to_tokens(t, part):
    """Stored tiles in token-major order."""
    eb, (pool, nkv, _, d) = t.element_size(), t.shape
    x, r = 16 // eb, 4 // eb
    b = _bytes(t)
    if part == 0:
        out = b.reshape(pool, nkv, d // x, PAGE, x).transpose(2, 3)
    else:
        out = b.reshape(pool, nkv, d // (16 * r), 4, 16, r, 4).permute(0, 1, 3, 6, 2, 5, 4)
    return out.reshape(t.shape).view(t.dtype)


def _ancestors(case, seed, rows):
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
        if bits:
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


def prepare(case, seed):
    s = _State()
    s.case, s.op = case, case["op"]
    if s.op == "rotary":
        rows, hq, hk, d = case["rows"], case["hq"], case["hk"], case["d"]
        # the query and key part of a fused projection's output, whose rows hold the values too
        s.src = _normal((rows, (hq + 2 * hk) * d), 1.0, seed, 1, TORCH[case["dtype"]])
        s.pos = _positions(case, seed)
        s.dst = [torch.empty((rows, h, d), dtype=s.src.dtype, device="cuda") for h in (hq, hk) if h]
        if own:
            _bind_rotary(s)
        return s
    nq, nkv, d = SHAPES[case["shape"]]
    lens, rows = _counts(case)
    table, s.pool = _table(case, seed, lens, rows)
    s.counts = (lens, rows)
    s.table = torch.tensor(table, dtype=torch.int32, device="cuda").reshape(len(lens), -1)
    s.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s.start = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
    n, dt = sum(rows), TORCH[case["dtype"]]
    s.n = n
    s.pools, s.scales = [], []
    for part in (0, 1):
        t, scale = _tiles(case, seed, s.pool, part)
        s.pools.append(_to_stored(t, part))
        s.scales.append(scale)
    s.index = None
    if s.op == "read":
        s.first = s.lens - (s.start[1:] - s.start[:-1])
        s.out = [torch.zeros((n, nkv, d), dtype=dt, device="cuda") for _ in (0, 1)]
    elif s.op == "write":
        have = n
        if case["pick"]:  # each sequence's rows out of its draft of `pick`, in ascending order
            rng = random.Random(seed)
            have = case["pick"] * len(lens)
            s.index = torch.tensor([b * case["pick"] + t for b, r in enumerate(rows)
                                    for t in sorted(rng.sample(range(case["pick"]), r))],
                                   dtype=torch.int32, device="cuda")
        # keys as the rotary step left them, values inside the fused projection's output; rows
        # differ in size, so that some need a larger scale than their page has
        size = torch.exp(_normal((have, 1), 0.5, seed, 5))
        s.k = (_normal((have, nkv * d), 1.0, seed, 6) * size).to(dt)
        s.v = torch.cat([torch.zeros((have, (nq + nkv) * d), dtype=dt, device="cuda"),
                         (_normal((have, nkv * d), 1.0, seed, 7) * size).to(dt)], dim=1)
    else:
        # q, k, v inside the fused projection's output
        s.qkv = _normal((n, (nq + 2 * nkv) * d), 1.0, seed, 8, dt)
        s.mask = None if case["chain"] else _ancestors(case, seed, rows).cuda()
        s.o = torch.zeros((n, nq, d), dtype=dt, device="cuda")
    if own:
        _bind(s)
    return s


# ------------------------------------------------------------------------------ the library


def _bind_rotary(s):
    import paper_2607_09153_amd as kv
    c = s.case
    theta, factor, low, high, magnitude = _rope_args(c)
    s.kv = kv
    s.rope = kv.make_rope(c["d"], c["rot"], c["layout"], theta, c["scaling"], factor, TRAINED, low, high,
                          magnitude)
    width, at, parts = s.src.shape[1], 0, []
    for t in s.dst:
        h = t.shape[1]
        parts.append((s.src.data_ptr() + at * s.src.element_size(), t.data_ptr(), h, width, h * c["d"]))
        at += h * c["d"]
    s.parts = kv.make_rope_heads(parts)


def _bind(s):
    """What a program keeps beside its tensors: the handle, the descriptors, the workspace."""
    import paper_2607_09153_amd as kv
    c = s.case
    nq, nkv, d = SHAPES[c["shape"]]
    wdt = "f32" if c["kvdt"] == "f32" else "bf16"
    lens, rows = s.counts
    s.kv = kv
    s.handle = kv.kvprm_create(kv.make_desc(1, 64 * nq, nq, nkv, d, 64, THETA, 1e-6, wdt, c["kvdt"]))
    sc = [t.data_ptr() if t is not None else 0 for t in s.scales]
    s.cache = kv.make_cache(s.pools[0].data_ptr(), s.pools[1].data_ptr(), s.pool, *sc)
    s.batch = kv.make_batch(len(lens), s.table.data_ptr(), s.table.shape[1], s.lens.data_ptr(), lens)
    most = max(rows)
    if s.op == "read":
        s.rows = kv.make_kv_rows(s.out[0].data_ptr(), s.out[1].data_ptr(), c["dtype"], nkv * d, nkv * d,
                                 s.n, s.start.data_ptr(), most)
    elif s.op == "write":
        s.rows = kv.make_kv_rows(s.k.data_ptr(), s.v.data_ptr() + (nq + nkv) * d * s.v.element_size(),
                                 c["dtype"], nkv * d, s.v.shape[1], s.k.shape[0], s.start.data_ptr(), most,
                                 s.index.data_ptr() if s.index is not None else 0)
    else:
        base, e, width = s.qkv.data_ptr(), s.qkv.element_size(), s.qkv.shape[1]
        s.tree = kv.make_tree(base, base + nq * d * e, base + (nq + nkv) * d * e, s.o.data_ptr(), c["dtype"],
                              width, width, width, nq * d, s.n, s.start.data_ptr(), most,
                              s.mask.data_ptr() if s.mask is not None else 0,
                              s.mask.shape[1] if s.mask is not None else 0)
        s.ws = torch.empty(kv.kvprm_workspace_size_tree(s.handle, s.batch, s.tree), dtype=torch.uint8,
                           device="cuda")


def _run_own(s):
    kv, st = s.kv, torch.cuda.current_stream().cuda_stream
    if s.op == "rotary":
        kv.kvprm_rotary(s.rope, s.case["dtype"], s.case["rows"], s.pos.data_ptr(), s.parts, s.case["grad"], st)
        return s.dst
    if s.op == "write":
        kv.kvprm_write_kv(s.handle, s.cache, s.batch, 0, s.rows, st)
        return [t for t in s.pools + s.scales if t is not None]
    if s.op == "read":
        kv.kvprm_read_kv(s.handle, s.cache, s.batch, 0, s.rows, s.first.data_ptr(), st)
        return s.out
    kv.kvprm_attention_tree(s.handle, s.cache, s.batch, 0, s.tree, s.ws.data_ptr(), s.ws.numel(), st)
    return s.o


# ------------------------------------------------------------------------------ the plain form


def _turns(case):
    """Angle per position of every pair, in float64."""
    theta, factor, low, high, _ = _rope_args(case)
    n, s = case["rot"], case["scaling"]
    i = torch.arange(n // 2, dtype=torch.float64, device="cuda")
    if s == "base":
        theta = theta * factor ** (n / max(1, n - 2))
    f = theta ** (-2.0 * i / n)
    if s == "linear":
        return f / factor
    if s == "parts":
        keep = ((TRAINED * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep
    if s == "ramp":
        at = lambda turns: n * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
        a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), n - 1)
        keep = 1 - ((i - a) / max(b - a, 0.001)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep
    return f


def _plain_rotary(s):
    c = s.case
    n, hq, hk, d, half = c["rot"], c["hq"], c["hk"], c["d"], c["rot"] // 2
    angle = s.pos.double()[:, None] * _turns(c)
    mag = _rope_args(c)[4]
    cos = (angle.cos() * mag).float()[:, None]
    sin = (angle.sin() * (-mag if c["grad"] else mag)).float()[:, None]
    x = s.src[:, :(hq + hk) * d].reshape(-1, hq + hk, d)
    r = x[..., :n].float()
    if c["layout"] == "half":
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    y = torch.cat([r.to(x.dtype), x[..., n:]], dim=-1)
    return [y[:, :hq], y[:, hq:]][:len(s.dst)]


def _row_places(s):
    """Sequence of every row, and its place among that sequence's rows."""
    r = torch.arange(s.n, device="cuda")
    b = torch.searchsorted(s.start[1:].contiguous(), r, right=True)
    return b, r - s.start[b]


def _gather(s, part, seq, pos):
    """Cached vectors [..., kv-heads, d] at positions `pos` of sequences `seq`, in 32 bits."""
    pool, scale = s.pools[part], s.scales[part]
    eb, (_, nkv, _, d) = pool.element_size(), pool.shape
    x, r = 16 // eb, 4 // eb
    page, slot = s.table[seq, pos // PAGE].clamp(min=0).long(), pos % PAGE
    b = _bytes(pool)
    if part == 0:
        t = b.reshape(-1, nkv, d // x, PAGE, x).permute(0, 3, 1, 2, 4)[page, slot]
    else:
        t = b.reshape(-1, nkv, d // (16 * r), 4, 16, r, 4).permute(0, 3, 6, 1, 2, 5, 4)[page, slot // 4, slot % 4]
    t = t.reshape(*page.shape, nkv, d).view(pool.dtype).float()
    return t if scale is None else t * scale[page][..., None]


def _plain_read(s):
    b, i = _row_places(s)
    pos = s.first[b].long() + i
    return [_gather(s, part, b, pos).to(s.out[0].dtype) for part in (0, 1)]


def _power(amax):
    """The smallest power of two (2^MIN_EXP at least) whose 448-fold reaches amax."""
    m, e = torch.frexp(amax)
    return torch.exp2((e - 9 + (m > 0.875).int()).clamp(min=MIN_EXP).double()).float()


def _plain_write(s):
    """The pages that get rows, each with its 16 slots: new rows and old ones side by side."""
    nq, nkv, d = SHAPES[s.case["shape"]]
    most = sum(_pages(n + r) - n // PAGE for n, r in zip(*s.counts) if r)
    L, count = s.lens.long(), (s.start[1:] - s.start[:-1]).long()
    pages = torch.where(count > 0, (L + count + PAGE - 1) // PAGE - L // PAGE, 0)
    b = torch.repeat_interleave(torch.arange(len(L), device=L.device), pages, output_size=most)
    page = L[b] // PAGE + torch.arange(most, device=L.device) - (torch.cumsum(pages, 0) - pages)[b]
    ids = s.table[b, page].long()
    pos = page[:, None] * PAGE + torch.arange(PAGE, device=L.device)
    new = (pos >= L[b, None]) & (pos < (L + count)[b, None])
    old = pos < L[b, None]
    row = torch.where(new, s.start[b].long()[:, None] + pos - L[b, None], 0)
    if s.index is not None and s.n:
        row = s.index[row].long()
    new, old = new[:, None, :, None], old[:, None, :, None]
    for part in (0, 1) if most else ():
        src = s.k if part == 0 else s.v[:, (nq + nkv) * d:]
        x = src.reshape(-1, nkv, d)[row].transpose(1, 2).float()
        pool, scales = s.pools[part], s.scales[part]
        have = _to_tokens(pool[ids], part)
        if scales is None:
            tile = torch.where(new, x.to(pool.dtype), have)
        else:
            before = scales[ids]
            m, e = torch.frexp(before)  # a scale that is no power of two grows to the next
            up = torch.exp2((e - (m == 0.5).int()).double()).float()
            up = torch.where(old.any(dim=2)[..., 0], up, 0)
            scale = torch.maximum(_power(torch.where(new, x.abs(), 0).amax(dim=(2, 3))), up)
            kept = (have.float() * (before / scale)[..., None, None]).to(pool.dtype)
            kept = torch.where((scale == before)[..., None, None] | ~old, _bytes(have), _bytes(kept))
            tile = torch.where(new, _bytes((x / scale[..., None, None]).to(pool.dtype)), kept).view(pool.dtype)
            scales[ids] = scale
        _bytes(pool)[ids] = _bytes(_to_stored(tile, part))
    return [t for t in s.pools + s.scales if t is not None]


def _plain_tree(s):
    nq, nkv, d = SHAPES[s.case["shape"]]
    lens, rows = s.counts
    B, T, Lm, g = len(lens), max(rows), max(lens), nq // nkv
    q, k, v = s.qkv.split([nq * d, nkv * d, nkv * d], dim=1)
    b = torch.arange(B, device="cuda")[:, None]
    t = torch.arange(T, device="cuda")
    count = (s.start[1:] - s.start[:-1])[:, None]
    row = (s.start[:-1].long()[:, None] + t).clamp(max=s.n - 1)
    have = t < count
    q = q.reshape(-1, nkv, g, d)[row].permute(0, 2, 1, 3, 4).reshape(B * nkv, T * g, d).float()
    pos = torch.arange(Lm, device="cuda")
    seen = (pos < s.lens[:, None])[:, None, :].expand(B, T, Lm)
    at = torch.where(pos < s.lens[:, None], pos, 0)
    if s.mask is None:
        bits = (t[None, :] <= t[:, None])[None].expand(B, T, T)
    else:
        bits = (s.mask[row][..., t // 32] >> (t % 32)) & 1 != 0
    ok = torch.cat([seen, bits & have[:, None, :]], dim=2)
    ok = ok[:, None, :, None].expand(B, nkv, T, g, Lm + T).reshape(B * nkv, T * g, Lm + T)
    key, val = (torch.cat([_gather(s, part, b, at), x.reshape(-1, nkv, d)[row].float()], dim=1)
                .transpose(1, 2).reshape(B * nkv, Lm + T, d) for part, x in ((0, k), (1, v)))
    sc = torch.bmm(q, key.transpose(1, 2).contiguous()).mul_(d ** -0.5).masked_fill_(~ok, -math.inf)
    top = sc.amax(dim=2, keepdim=True)
    p = sc.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = p.sum(dim=2, keepdim=True)
    o = torch.bmm(p, val) / torch.where(total > 0, total, 1)
    o = o.reshape(B, nkv, T, g, d).permute(0, 2, 1, 3, 4).reshape(B, T, nq, d)
    seq, i = _row_places(s)
    return o[seq, i].to(s.o.dtype)


def run(s):
    if own:
        return _run_own(s)
    return {"rotary": _plain_rotary, "write": _plain_write, "read": _plain_read, "tree": _plain_tree}[s.op](s)


# ------------------------------------------------------------------------------ the measure


def work(case):
    e = {"f32": 4, "bf16": 2, "fp8": 1}
    eb = e[case["dtype"]]
    if case["op"] == "rotary":
        n = case["rows"] * (case["hq"] + case["hk"])
        return {"bytes": 2 * n * case["d"] * eb + 4 * case["rows"], "flops": 3 * n * case["rot"]}
    nq, nkv, d = SHAPES[case["shape"]]
    lens, rows = _counts(case)
    kb = e[case["kvdt"]]
    if case["op"] == "tree":
        cache = 2 * sum(lens) * nkv * d * kb
        if case["kvdt"] == "fp8":
            cache += 2 * sum(_pages(n) for n in lens) * nkv * 4
        seen = sum(r * (n + (r + 1) / 2) for n, r in zip(lens, rows))
        return {"bytes": cache + sum(rows) * (2 * nq + 2 * nkv) * d * eb, "flops": 4 * seen * nq * d}
    both = 2 * sum(rows) * nkv * d
    if case["kvdt"] == "fp8":  # (each tile's scale, read or written)
        pages = sum(_pages(n + r) - n // PAGE for n, r in zip(lens, rows)) if case["op"] == "write" else \
            sum(_pages(n) - (n - r) // PAGE for n, r in zip(lens, rows))
        return {"bytes": both * (eb + kb) + 2 * 4 * nkv * pages, "flops": both}
    return {"bytes": both * (eb + kb), "flops": 0}


# ------------------------------------------------------------------------------ in 64 bits


def _exact_rotary(case, seed):
    s = prepare(case, seed)
    theta, factor, low, high, mag = _rope_args(case)
    n, half, kind = case["rot"], case["rot"] // 2, case["scaling"]
    speed = []
    for i in range(half):
        base = theta * factor ** (n / (n - 2)) if kind == "base" and n > 2 else theta
        if kind == "base" and n == 2:
            base = theta * factor ** 2
        f = base ** (-2 * i / n)
        if kind == "linear":
            f /= factor
        elif kind == "parts":
            turns = TRAINED * f / (2 * math.pi)
            g = 0.0 if turns < low else 1.0 if turns > high else (turns - low) / (high - low)
            f *= g + (1 - g) / factor
        elif kind == "ramp":
            first = math.floor(n * math.log(TRAINED / (high * 2 * math.pi)) / (2 * math.log(theta)))
            last = math.ceil(n * math.log(TRAINED / (low * 2 * math.pi)) / (2 * math.log(theta)))
            first, last = max(first, 0), min(last, n - 1)
            g = 1 - min(1.0, max(0.0, (i - first) / max(last - first, 0.001)))
            f *= g + (1 - g) / factor
        speed.append(f)
    angle = torch.outer(s.pos.double(), torch.tensor(speed, dtype=torch.float64, device="cuda"))
    turn = torch.polar(torch.full_like(angle, mag), -angle if case["grad"] else angle)
    out, at = [], 0
    for t in s.dst:
        x = s.src[:, at:at + t.shape[1] * case["d"]].reshape(t.shape).double()
        at += t.shape[1] * case["d"]
        y = x.clone()
        lo, hi = (slice(0, half), slice(half, n)) if case["layout"] == "half" else \
            (slice(0, n, 2), slice(1, n, 2))
        z = torch.complex(x[..., lo].contiguous(), x[..., hi].contiguous()) * turn[:, None]
        y[..., lo], y[..., hi] = z.real, z.imag
        out.append(y)
    return out


def _e4m3(x):
    """float64 values rounded to the nearest e4m3 value (ties to even), |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -9))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_write(case, seed):
    s = prepare(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    lens, rows = s.counts
    start, table = s.start.tolist(), s.table.tolist()
    index = s.index.tolist() if s.index is not None else list(range(s.n))
    out, scales = [], []
    for part in (0, 1):
        src = (s.k if part == 0 else s.v[:, (nq + nkv) * d:]).reshape(-1, nkv, d)
        tiles = _to_tokens(s.pools[part], part).double()
        if case["kvdt"] != "fp8":
            for b, (n, r) in enumerate(zip(lens, rows)):
                if r:
                    pos = torch.arange(n, n + r, device="cuda")
                    page = torch.tensor(table[b], device="cuda")[pos // PAGE]
                    pick = torch.tensor(index[start[b]:start[b + 1]], device="cuda")
                    tiles[page, :, pos % PAGE] = src[pick].double()
            out.append(_stored64(tiles, part, {"f32": 4, "bf16": 2}[case["kvdt"]]))
            continue
        scale = s.scales[part].double()
        for b, (n, r) in enumerate(zip(lens, rows)):
            if not r:
                continue
            p0, p1 = n // PAGE, _pages(n + r)
            ids = torch.tensor(table[b][p0:p1], device="cuda")
            x = torch.zeros(((p1 - p0) * PAGE, nkv, d), dtype=torch.float64, device="cuda")
            pick = torch.tensor(index[start[b]:start[b + 1]], device="cuda")
            x[n - p0 * PAGE:n - p0 * PAGE + r] = src[pick].double()
            x = x.reshape(p1 - p0, PAGE, nkv, d).transpose(1, 2)
            k = torch.ceil(torch.log2(x.abs().amax(dim=(2, 3)) / 448)).clamp(min=MIN_EXP)
            if n % PAGE:
                k[0] = torch.maximum(k[0], torch.ceil(torch.log2(scale[ids[0]])))
            unit = torch.exp2(k)
            was = tiles[ids]
            now = _e4m3(x / unit[..., None, None])
            if n % PAGE:
                keep = n % PAGE
                now[0, :, :keep] = _e4m3(was[0, :, :keep] * (scale[ids[0]] / unit[0])[:, None, None])
            end = (n + r) - (p1 - 1) * PAGE
            now[-1, :, end:] = was[-1, :, end:]
            tiles[ids], scale[ids] = now, unit
        out.append(_stored64(tiles, part, 1))
        scales.append(scale)
    return out + scales


def _stored64(t, part, eb):
    """_to_stored for values held in 64 bits, of a pool of eb-byte elements."""
    pool, nkv, _, d = t.shape
    if part == 0:
        return t.reshape(pool, nkv, PAGE, d * eb // 16, 16 // eb).transpose(2, 3).reshape(t.shape)
    return t.reshape(pool, nkv, 4, 4, d * eb // 64, 4 // eb, 16).permute(0, 1, 4, 2, 6, 5, 3).reshape(t.shape)


def _exact_cached(s, part, b, first, last):
    """Cached vectors [kv-heads][tokens][d] of sequence b in float64."""
    n = _pages(last)
    ids = s.table[b, :n].long()
    t = _to_tokens(s.pools[part][ids], part).double()
    if s.scales[part] is not None:
        t = t * s.scales[part][ids].double()[..., None, None]
    return t.transpose(0, 1).reshape(t.shape[1], n * PAGE, -1)[:, first:last]


def _exact_read(case, seed):
    s = prepare(case, seed)
    out = [[], []]
    for b, (n, r) in enumerate(zip(*s.counts)):
        for part in (0, 1):
            if r:
                out[part].append(_exact_cached(s, part, b, n - r, n).transpose(0, 1))
    return [torch.cat(o) if o else torch.zeros(t.shape, dtype=torch.float64, device="cuda")
            for o, t in zip(out, s.out)]


def _exact_tree(case, seed):
    s = prepare(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    out, at = [], 0
    for b, (n, r) in enumerate(zip(*s.counts)):
        x = s.qkv[at:at + r].double()
        q = x[:, :nq * d].reshape(r, nkv, nq // nkv, d).permute(1, 2, 0, 3)
        k = x[:, nq * d:(nq + nkv) * d].reshape(r, nkv, d).transpose(0, 1)
        v = x[:, (nq + nkv) * d:].reshape(r, nkv, d).transpose(0, 1)
        sees = torch.ones((r, r), dtype=torch.bool, device="cuda").tril() if s.mask is None else torch.stack(
            [(s.mask[at:at + r, j // 32] >> (j % 32)) & 1 == 1 for j in range(r)], dim=1)
        heads = []
        for j in range(nkv):
            K = torch.cat([_exact_cached(s, 0, b, 0, n)[j], k[j]]) if n else k[j]
            V = torch.cat([_exact_cached(s, 1, b, 0, n)[j], v[j]]) if n else v[j]
            z = torch.mm(q[j].reshape(-1, d), K.t().contiguous()).reshape(-1, r, n + r) / math.sqrt(d)
            z[:, :, n:].masked_fill_(~sees, -math.inf)
            p = torch.softmax(z, dim=2)
            heads.append(torch.mm(p.reshape(-1, n + r), V).reshape(-1, r, d))
        out.append(torch.cat(heads).transpose(0, 1))
        at += r
    return torch.cat(out)


def exact(case, seed):
    return {"rotary": _exact_rotary, "write": _exact_write, "read": _exact_read,
            "tree": _exact_tree}[case["op"]](case, seed)
