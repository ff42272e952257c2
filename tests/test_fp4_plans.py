"""Workspaces and chunks of calls over 4-bit caches (CPU): sizes never fall when a call grows and hold what every smaller
call takes; chunks (kvprm::chunk_pages4, called in the library) are even, fit a wave's page ids and the candidates'
slots, and those of unknown lengths are no longer than a full table's long ones."""
import ctypes
import itertools
import random

import pytest

import paper_2607_09153_amd as kv

from test_chunk_rule import Dims, _long
from test_tree_workspace import FAKE, SHAPES, _call, _need

_chunk = kv.lib._ZN5kvprm12chunk_pages4ERKNS_4DimsEiPKiS4_b
_chunk.argtypes = [ctypes.POINTER(Dims), ctypes.c_int, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int),
                   ctypes.c_bool]


def _dims(shape):
    nq, nkv, d = shape
    return Dims(1, 64, nq, nkv, d, 64, nq // nkv, 1.0, 0.0, 1, 3)


@pytest.fixture(params=SHAPES, ids=str)
def shape_and_handle(request):
    nq, nkv, d = request.param
    h = kv.kvprm_create(kv.make_desc(1, 64 * nq, nq, nkv, d, 64, kv_dtype="fp4"))
    yield request.param, h
    kv.kvprm_destroy(h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_workspace(shape_and_handle, dtype):
    shape, h = shape_and_handle
    axes = [(1, 2, 8, 24, 64), (1, 2, 70, 300, 2048), (1, 16, 100, 2000, 16384), (1, 8, 17, 48, 256)]
    size = {at: kv.kvprm_workspace_size_tree(h, *_call(shape, dtype, *(a[i] for a, i in zip(axes, at))))
            for at in itertools.product(*(range(len(a)) for a in axes))}
    for at, n in size.items():
        for i in range(4):
            if at[i]:
                assert n >= size[tuple(x - (k == i) for k, x in enumerate(at))], (at, i)
    rng = random.Random(sum(shape))
    for _ in range(200):
        big = [rng.randint(1, 64), rng.randint(1, 4000), rng.randint(1, 5000), rng.randint(1, 256)]
        small = [rng.randint(1, x) for x in big]
        b, t = _call(shape, dtype, *small)
        assert _need(_dims(shape), b, t) <= kv.kvprm_workspace_size_tree(h, *_call(shape, dtype, *big)), (big, small)


def test_attention_workspace_never_falls(shape_and_handle):
    _, h = shape_and_handle
    pages = (1, 2, 36, 37, 60, 64, 128, 129, 500, 2047, 2048, 16352)
    size = [[kv.kvprm_workspace_size(h, kv.make_batch(n, FAKE, p, FAKE)) for p in pages] for n in (1, 2, 7, 8, 33, 64)]
    for rows in (size, list(zip(*size))):
        for row in rows:
            assert list(row) == sorted(row)


@pytest.mark.parametrize("shape", SHAPES)
def test_chunks(shape):
    rng = random.Random(sum(shape))
    seen = set()
    for _ in range(2000):
        n, most = rng.choice([1, 2, 8, 24, 64]), rng.choice([1, 4, 40, 300, 2048, 16352])
        pages = [rng.randint(0, most) for _ in range(n)]
        slots = [max(-(-most // 16) + 1, 129)] * n
        ints = ctypes.c_int * n
        c = _chunk(_dims(shape), n, ints(*pages), ints(*slots), True)
        assert c % 2 == 0 and 4 <= c <= 64
        assert all(-(-p // c) <= s for p, s in zip(pages, slots))
        seen.add(c)
        full = [most] * n
        u = _chunk(_dims(shape), n, ints(*full), ints(*slots), False)
        assert u % 2 == 0 and 4 <= u <= 1 << _long(sum(full)) and -(-most // u) <= slots[0]
    assert len(seen) > 8
