"""kvprm_attention_tree on batches that fill the chip, where drafts of many columns take another kernel than in
small ones: every length around a page pair, drafts of 0 to 64 tokens, all kinds of masks, infinities and NaN,
fp8 scales. Tolerances as in test_gpu_tree.py and test_gpu_tree_ranges.py."""
import math

import numpy as np
import pytest
import torch

from test_gpu_tree import Case, _say
from test_gpu_tree_ranges import _check

pytestmark = pytest.mark.gpu
LENGTHS = [0, 1, 15, 16, 17, 31, 32, 33, 129, 700]
COUNTS = [40, 3, 64, 33, 17, 0, 32, 1, 50, 20, 31, 34, 7]


def _sizes(n):
    return [LENGTHS[i % len(LENGTHS)] for i in range(n)], [COUNTS[i % len(COUNTS)] for i in range(n)]


@pytest.mark.parametrize("cdt", ["bf16", "fp8"])
@pytest.mark.parametrize("nq,nkv,d", [(8, 4, 64), (14, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("masked", ["tree", "any", "chain", "none"])
def test_tree_full(cdt, nq, nkv, d, masked):
    _say("full", cdt, nq, nkv, d, masked)
    Case(cdt, "bf16", nq, nkv, d, *_sizes(60), seed=nq, masked=masked).check()


@pytest.mark.parametrize("cdt", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_tree_full_infinities_and_nan_where_masked(cdt, d):
    """Every second candidate has drafted keys and values that hold infinities and NaN, which the later half of its
    tokens does not see."""
    _say("full, inf and nan", cdt, d)
    nq, nkv = 8, 2
    c = Case(cdt, "bf16", nq, nkv, d, *_sizes(60), seed=d)
    rng = np.random.default_rng(1)
    for b in range(0, 60, 2):
        n = c.counts[b]
        for what, value in (("v", math.inf), ("v", -math.inf), ("v", math.nan), ("k", math.nan)):
            if n < 8:
                continue
            t = int(rng.integers(0, n))
            at = (nq + (nkv if what == "v" else 0)) * d
            c.qkv[c.start[b] + t, at + 3:at + d + 6:5] = value
            c.sees[b][n // 2:, t] = False
    c.bits[:] = 0
    for b, s in enumerate(c.sees):
        for j in range(len(s)):
            c.bits[c.start[b]:c.start[b] + len(s), j // 32] |= s[:, j].astype(np.uint32) << np.uint32(j % 32)
    c.upload()
    want = c.want()
    assert np.isnan(want).any() and np.isinf(want).any() and np.isfinite(want).all(axis=1).sum() > len(want) // 4
    c.check(c.run())


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 64), (8, 2, 128)])
def test_tree_full_fp8_value_scales(nq, nkv, d):
    """As test_tree_fp8_value_scales, each kind of candidate five times."""
    _say("full, value scales", nq, nkv, d)
    n = 40
    lengths = [700, 300, 900, 40, 0, 33] * 5
    c = Case("fp8", "bf16", nq, nkv, d, lengths, [n] * 30, seed=d)
    rng = np.random.default_rng(d)
    sets = [(2.0 ** -100, 1.25 * 2.0 ** -7, 0.0), (1.25 * 2.0 ** -100, 2.0 ** -97), (2.0 ** 10, 1.1 * 2.0 ** -20, 2.0 ** -60),
            (0.0,), (1.0,), (2.0 ** -100,)]
    c.scale[1][:] = 1.0
    vs = slice((nq + nkv) * d, (nq + 2 * nkv) * d)
    for b in range(30):
        for page in c.table[b][c.table[b] >= 0]:
            c.scale[1][:, page] = rng.choice(sets[b % 6], size=c.scale[1][:, page].shape)
        c.qkv[c.start[b]:c.start[b] + n, vs] *= (1.0, 2.0 ** -95, 2.0 ** -60, 2.0 ** 40, 2.0 ** -90, 2.0 ** 100)[b % 6]
        if b % 6 == 4:
            c.qkv[c.start[b]:c.start[b] + 33, vs] = 0
    c.upload()
    _check(c)


def test_tree_full_repeats_and_replays():
    """The same bits from a second call and from a captured one."""
    _say("full, repeated")
    c = Case("fp8", "bf16", 8, 2, 64, *_sizes(60), seed=2)
    b, t = c.batch(host=False), c.tree()
    n = c.m.kvprm_workspace_size_tree(c.h, b, t)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def call():
        c.m.kvprm_attention_tree(c.h, c.cache, b, 1, t, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)

    call()
    torch.cuda.synchronize()
    first = c.o.clone()
    c.check(first.cpu())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for run in (call, g.replay, g.replay):
        c.o.fill_(7.0)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        assert torch.equal(c.o, first)
    del g
