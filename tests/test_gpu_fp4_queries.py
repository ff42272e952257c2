"""kvprm_attention over 4-bit caches with queries whose dims differ in size: one dim of every 32 is 30 to 1000 times the
others, and its keys are as many times smaller, so that scores stay near those of alike dims.

Tolerance of an output against the fp64 oracle. Each query value is held to 2^-29 of the largest of its 32 dims (3 or
4 times the outlier's factor R, at most 4000): 7.5e-6, and the other keys are near N(0, 1), so that a score (a sum over d dims
divided by sqrt(d)) is off by about 7.5e-6 if they fell one way in half of their range, by 4e-6 of rms. Its fp32 sum is
off by 5e-6 as roundings fall (the outlier's own products, R q / R k, are as large as the others). Weights follow
their score, and an output is a mean of values with these weights: within 2 * 1e-5 max|v|, as for alike dims. With
2^-21 in place of 2^-29 the scores were off by up to 7e-4 (2e-5 at R = 30)."""
import numpy as np
import pytest
import torch

from oracle import fp4
from oracle import kvprm_oracle as ko

from fp4_common import Cache

pytestmark = pytest.mark.gpu
LAYER = 1


def _uneven(c, ratio, seed):
    """Inputs and a cache with an outlier dim in every 32, in other places for every kv-head."""
    rng = np.random.default_rng(seed)
    nq, nkv, d = c.shape
    factor = np.ones((nkv, d))
    for j in range(nkv):
        factor[j, 32 * np.arange(d // 32) + rng.integers(0, 32, size=d // 32)] = ratio
    keys = rng.normal(size=(c.layers, c.pages, nkv, 16, d)) / factor[:, None, :]
    code, scale = fp4.encode(keys)
    scale[c.scale[0] == 255] = 255
    c.code[0], c.scale[0] = code, scale
    c.upload()
    q = rng.normal(size=(len(c.lengths), nq, d)) * np.repeat(factor, nq // nkv, axis=0)
    k = rng.normal(size=(len(c.lengths), nkv, d)) / factor
    return [t.astype(np.float32) for t in (q, k, rng.normal(size=k.shape))]


def _run(c, x, batch):
    m = c.m
    n = m.kvprm_workspace_size(c.h, batch)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    q, k, v = (torch.from_numpy(t).cuda() for t in x)
    o = torch.full(q.shape, 7.0, device="cuda")
    m.kvprm_attention(c.h, c.cache, batch, LAYER, q.data_ptr(), k.data_ptr(), v.data_ptr(), ws.data_ptr(), n, o.data_ptr(),
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return o.cpu().numpy()


def _check(c, x, got, what):
    nq, nkv, _ = c.shape
    assert np.all(np.isfinite(got)), what
    worst = 0.0
    for b in range(len(c.lengths)):
        ck, cv = (c.cached(p, LAYER, b) for p in (0, 1))
        for h in range(nq):
            j = h // (nq // nkv)
            K, V = np.concatenate([ck[:, j], x[1][b, j][None]]), np.concatenate([cv[:, j], x[2][b, j][None]])
            want = ko.attention(x[0][b, h].astype(np.float64), K, V)
            worst = max(worst, np.abs(got[b, h] - want).max() / np.abs(V).max())
    print("off by", what, worst, flush=True)
    assert worst <= 2e-5, what


@pytest.mark.parametrize("ratio", [30, 100, 1000])
@pytest.mark.parametrize("nq,nkv,d", [(28, 4, 128), (8, 8, 128), (16, 4, 64), (16, 1, 128)])
def test_private_pages(nq, nkv, d, ratio):
    """Caches of one launch, and ones in chunks."""
    print("case:", nq, nkv, d, ratio, flush=True)
    for lengths in ([0, 1, 2, 5, 15, 17, 33, 100, 400], [1, 3, 17, 2500, 4000]):
        c = Cache(nq, nkv, d, lengths, seed=ratio + d)
        x = _uneven(c, ratio, nq)
        _check(c, x, _run(c, x, c.batch), lengths)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ratio", [1, 100, 1000])
def test_shared_prefix(d, ratio):
    """A group's prefix and the members' own pages meet in one softmax; with the hint and without."""
    print("case: prefix", d, ratio, flush=True)
    c = Cache(14, 2, d, [700, 640, 900, 33, 320, 400, 325], seed=ratio)
    x = _uneven(c, ratio, d)
    for b in (1, 2):
        c.table[b, :40] = c.table[0, :40]
    for b in (5, 6):
        c.table[b, :20] = c.table[4, :20]
    c.upload()
    _check(c, x, _run(c, x, c.batch), "no hint")
    hint = c.m.make_batch(7, c.dtab.data_ptr(), c.width, c.dlen.data_ptr(), c.lengths, [0, 3, 4, 7], [640, 0, 320])
    _check(c, x, _run(c, x, hint), "hint")
