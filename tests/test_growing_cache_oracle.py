"""The fp64 oracle of the growing cache against closed forms and torch's conversions (CPU)."""
import numpy as np
import pytest
import torch

from oracle import growing_cache as gc
from oracle import kvprm_oracle as ko


def test_e4m3_rounding_is_torch_s():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=20000) * np.exp2(rng.integers(-14, 8, 20000)),
                        ko.e4m3fn_to_f64(np.arange(0x7F))]).astype(np.float32)
    # the midpoints between neighbours too (ties)
    v = ko.e4m3fn_to_f64(np.arange(0x7F))
    x = np.clip(np.concatenate([x, ((v[1:] + v[:-1]) / 2).astype(np.float32)]), -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(gc.to_e4m3(x.astype(np.float64)), want)
    assert gc.to_e4m3(np.array([np.inf, -np.inf, np.nan])).tolist() == [0x7F] * 3


def test_bf16_rounding_is_torch_s():
    x = np.random.default_rng(2).normal(size=5000).astype(np.float32)
    want = torch.from_numpy(x).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    assert np.array_equal(gc.to_bf16(x), want)


def test_power_of_two():
    assert [gc.power(x) for x in (1.0, 1.5, 2.0, 0.5, 0.51)] == [1.0, 2.0, 2.0, 0.5, 1.0]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("part", [0, 1])
def test_store_and_load_are_inverse(dtype, part):
    tok = np.random.default_rng(3).integers(0, 256, size=(2, 3, 16, 64)).astype(gc.WORD[dtype])
    st = gc.store(tok, part)
    assert np.array_equal(gc.load(st, part), tok)
    dec = ko.v_tile_to_tokens if part else ko.k_tile_to_tokens
    assert np.array_equal(dec(st[1, 2].reshape(-1), 16, 64, tok.itemsize), tok[1, 2])


def test_rotary_is_the_decoder_s():
    """The unscaled half layout is the rotary embedding of the scoring oracle; frequencies scaled by 1
    are the unscaled ones; the interleaved layout is the half one on reordered dims."""
    rng = np.random.default_rng(4)
    x, pos = rng.normal(size=(3, 2, 64)), [0, 7, 30000]
    f = gc.frequencies(64, 1e6)
    want = np.stack([ko.rope(x[r], pos[r], 1e6) for r in range(3)])
    assert np.allclose(gc.rotary(x, pos, f), want, atol=1e-12)
    for kind in ("linear", "base", "parts", "ramp"):
        assert np.allclose(gc.frequencies(64, 1e6, kind, 1.0, 4096.0), f, rtol=1e-15)
    perm = np.concatenate([np.arange(0, 64, 2), np.arange(1, 64, 2)])
    assert np.allclose(gc.rotary(x, pos, f, "interleaved")[..., perm], gc.rotary(x[..., perm], pos, f), atol=1e-12)


def test_rotary_scaled_frequencies():
    """Fast pairs keep their frequency, slow ones are divided by the factor, in both ramps; the base
    change leaves the first pair and divides the last by the factor."""
    n, s = 128, 8.0
    f = gc.frequencies(n, 1e4)
    for kind in ("parts", "ramp"):
        r = gc.frequencies(n, 1e4, kind, s, 4096.0) / f
        assert r[0] == 1 and np.isclose(r[-1], 1 / s) and np.all(np.diff(r) <= 1e-12)
    r = gc.frequencies(n, 1e4, "base", s) / f
    assert r[0] == 1 and np.isclose(r[-1], 1 / s)


def test_rotary_transpose_is_the_gradient():
    rng = np.random.default_rng(5)
    x, y, pos = rng.normal(size=(4, 3, 16)), rng.normal(size=(4, 3, 16)), [0, 1, 5, 1000]
    f = gc.frequencies(8, 100.0)
    for layout in ("half", "interleaved"):
        fwd = gc.rotary(x, pos, f, layout, 1.25)
        back = gc.rotary(y, pos, f, layout, 1.25, transpose=True)
        assert np.isclose(np.sum(fwd * y), np.sum(x * back), rtol=1e-13)


def test_tree_attention_chain_is_causal_attention():
    """A chain over a cache is causal attention over the whole sequence (torch, float64); a token that
    attends to nothing gets zeros; one that attends to itself alone gets its value."""
    rng = np.random.default_rng(6)
    T, L, nq, nkv, d = 5, 9, 4, 2, 16
    q, k, v = rng.normal(size=(T, nq, d)), rng.normal(size=(T, nkv, d)), rng.normal(size=(T, nkv, d))
    ck, cv = rng.normal(size=(L, nkv, d)), rng.normal(size=(L, nkv, d))
    o = gc.tree_attention(q, k, v, ck, cv, np.tril(np.ones((T, T), bool)))
    K, V = np.concatenate([ck, k]).repeat(2, axis=1), np.concatenate([cv, v]).repeat(2, axis=1)
    tq, tk, tv = (torch.from_numpy(a).transpose(0, 1)[None].contiguous() for a in (q, K, V))
    mask = torch.ones(T, L + T, dtype=torch.bool).tril(L)
    want = torch.nn.functional.scaled_dot_product_attention(tq, tk, tv, attn_mask=mask)[0].transpose(0, 1)
    assert np.allclose(o, want.numpy(), atol=1e-12)
    none = np.zeros((T, T), bool)
    assert np.all(gc.tree_attention(q, k, v, ck[:0], cv[:0], none) == 0)
    one = gc.tree_attention(q, k, v, ck[:0], cv[:0], np.eye(T, dtype=bool))
    assert np.allclose(one, v.repeat(2, axis=1), atol=1e-14)
