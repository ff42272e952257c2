"""Workspace of kvprm_attention_tree (CPU): the size asked for never falls when a batch, its page table, its rows or the
rows of a candidate grow, and holds what every smaller call takes (kvprm::tree_ws_need, called in the library)."""
import ctypes
import itertools
import random

import pytest

import paper_2607_09153_amd as kv

from test_chunk_rule import KVDT, Dims

FAKE = 0x10000
SHAPES = [(28, 4, 128), (16, 8, 128), (4, 2, 64), (32, 2, 128), (64, 8, 128), (16, 4, 64)]

_need = kv.lib._ZN5kvprm12tree_ws_needERKNS_4DimsERK11kvprm_batchRK10kvprm_tree
_need.restype = ctypes.c_size_t
_need.argtypes = [ctypes.POINTER(Dims), ctypes.POINTER(kv.Batch), ctypes.POINTER(kv.Tree)]


def _call(shape, dtype, B, pages, rows, most):
    nq, nkv, d = shape
    t = kv.make_tree(FAKE, FAKE, FAKE, FAKE, dtype, nq * d, nkv * d, nkv * d, nq * d, rows, FAKE, most)
    return kv.make_batch(B, FAKE, pages, FAKE), t


def _forms():
    return [("f32", "f32"), ("bf16", "bf16"), ("fp8", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("kvdt,dtype", _forms())
@pytest.mark.parametrize("shape", SHAPES)
def test_tree_workspace_never_falls(shape, kvdt, dtype):
    nq, nkv, d = shape
    h = kv.kvprm_create(kv.make_desc(1, 64 * nq, nq, nkv, d, 64, weight_dtype="f32" if kvdt == "f32" else "bf16",
                                     kv_dtype=kvdt))
    axes = [(1, 2, 7, 8, 24, 64), (1, 2, 5, 70, 300, 2048), (1, 5, 16, 64, 100, 2000, 16384), (1, 3, 8, 17, 48, 64, 256)]
    try:
        size = {at: kv.kvprm_workspace_size_tree(h, *_call(shape, dtype, *(a[i] for a, i in zip(axes, at))))
                for at in itertools.product(*(range(len(a)) for a in axes))}
    finally:
        kv.kvprm_destroy(h)
    for at, n in size.items():
        for i in range(4):
            if at[i]:
                less = tuple(x - (k == i) for k, x in enumerate(at))
                assert n >= size[less], (at, less)


@pytest.mark.parametrize("kvdt,dtype", _forms())
@pytest.mark.parametrize("shape", SHAPES)
def test_tree_workspace_holds_smaller_calls(shape, kvdt, dtype):
    nq, nkv, d = shape
    rng = random.Random(nq + d)
    dims = Dims(1, 64, nq, nkv, d, 64, nq // nkv, 1.0, 0.0, 0 if kvdt == "f32" else 1, KVDT[kvdt])
    h = kv.kvprm_create(kv.make_desc(1, 64 * nq, nq, nkv, d, 64, weight_dtype="f32" if kvdt == "f32" else "bf16",
                                     kv_dtype=kvdt))
    try:
        for _ in range(300):
            big = [rng.randint(1, 64), rng.randint(1, 4000), rng.randint(1, 5000), rng.randint(1, 256)]
            n = kv.kvprm_workspace_size_tree(h, *_call(shape, dtype, *big))
            for small in [big] + [[rng.choice([1, x, rng.randint(1, x)]) for x in big] for _ in range(10)]:
                b, t = _call(shape, dtype, *small)
                assert _need(ctypes.byref(dims), ctypes.byref(b), ctypes.byref(t)) <= n, (big, small)
    finally:
        kv.kvprm_destroy(h)
