"""Refusals of kvprm_rotary, kvprm_write_kv, kvprm_read_kv and kvprm_attention_tree: every bad
argument is turned down with its status before anything is enqueued (CPU; the pointers are never
dereferenced)."""
import math

import pytest

import paper_2607_09153_amd as kv

FAKE = 0x10000


def _refused(status, call):
    with pytest.raises(kv.KvprmError) as e:
        call()
    assert e.value.status == status, kv.kvprm_last_error()
    assert kv.kvprm_last_error()


# ------------------------------------------------------------------------------ rotary


def _rotary(rope=None, dtype="bf16", rows=4, pos=FAKE, parts=None):
    kv.kvprm_rotary(rope or kv.make_rope(64), dtype, rows, pos,
                    kv.make_rope_heads(parts or [(FAKE, 2 * FAKE, 2, 128, 128)]))


@pytest.mark.parametrize("rope", [
    dict(head_dim=0), dict(head_dim=63), dict(head_dim=258), dict(head_dim=64, rotary_dim=66),
    dict(head_dim=64, rotary_dim=0), dict(head_dim=64, rotary_dim=31), dict(head_dim=64, theta=1.0),
    dict(head_dim=64, theta=math.nan), dict(head_dim=64, magnitude=math.inf),
    dict(head_dim=64, scaling="linear", factor=0.5), dict(head_dim=64, scaling="base", factor=math.nan),
    dict(head_dim=64, scaling="parts", factor=2.0),
    dict(head_dim=64, scaling="ramp", factor=2.0, trained_len=4096.0, low=2.0, high=1.0),
    dict(head_dim=64, scaling="parts", factor=2.0, trained_len=4096.0, low=0.0, high=1.0),
])
def test_rotary_refuses_embeddings(rope):
    _refused(kv.KVPRM_E_INVALID, lambda: _rotary(kv.make_rope(**rope)))


@pytest.mark.parametrize("kw,status", [
    (dict(dtype="fp8"), kv.KVPRM_E_INVALID),
    (dict(rows=-1), kv.KVPRM_E_INVALID),
    (dict(rows=1 << 31), kv.KVPRM_E_UNSUPPORTED),
    (dict(pos=0), kv.KVPRM_E_INVALID),
    (dict(parts=[(0, FAKE, 2, 128, 128)]), kv.KVPRM_E_INVALID),
    (dict(parts=[(FAKE, 0, 2, 128, 128)]), kv.KVPRM_E_INVALID),
    (dict(parts=[(FAKE + 1, 2 * FAKE, 2, 128, 128)]), kv.KVPRM_E_INVALID),
    (dict(parts=[(FAKE, 2 * FAKE, 0, 128, 128)]), kv.KVPRM_E_INVALID),
    (dict(parts=[(FAKE, 2 * FAKE, 2, 127, 128)]), kv.KVPRM_E_INVALID),
    (dict(parts=[(FAKE, 2 * FAKE, 2, 128, 100)]), kv.KVPRM_E_INVALID),
    (dict(parts=[(FAKE, 2 * FAKE, 1025, 1 << 20, 1 << 20)], rows=1), kv.KVPRM_E_UNSUPPORTED),
    (dict(parts=[(FAKE, FAKE + 128, 2, 128, 128)]), kv.KVPRM_E_INVALID),   # rows written are rows read
    (dict(parts=[(FAKE, FAKE, 2, 128, 256)]), kv.KVPRM_E_INVALID),         # in place, another stride
    (dict(parts=[(FAKE, FAKE + 384, 2, 256, 256)]), kv.KVPRM_E_INVALID),   # columns overlap by half
    (dict(parts=[(FAKE, 2 * FAKE, 2, 128, 128)] * 3), kv.KVPRM_E_INVALID),
])
def test_rotary_refuses_tensors(kw, status):
    _refused(status, lambda: _rotary(**kw))


def test_rotary_of_no_rows_is_nothing():
    _rotary(rows=0, pos=0, parts=[(0, 0, 2, 128, 128)])


# ------------------------------------------------------------------------------ rows and trees


@pytest.fixture
def handle():
    h = kv.kvprm_create(kv.make_desc(2, 256, 4, 2, 64, 1024))
    yield h
    kv.kvprm_destroy(h)


def _batch(**o):
    a = dict(batch=2, page_table_ptr=FAKE, max_pages=4, lengths_ptr=FAKE, lengths_host=[10, 64])
    a.update(o)
    return kv.make_batch(**a)


def _rows(**o):
    a = dict(k_ptr=FAKE, v_ptr=FAKE, dtype="bf16", k_stride=128, v_stride=128, num_rows=8, start_ptr=FAKE,
             max_rows=4)
    a.update(o)
    return kv.make_kv_rows(**a)


@pytest.mark.parametrize("rows,status", [
    (dict(k_ptr=0), kv.KVPRM_E_INVALID), (dict(v_ptr=0), kv.KVPRM_E_INVALID),
    (dict(start_ptr=0), kv.KVPRM_E_INVALID), (dict(dtype="fp8"), kv.KVPRM_E_INVALID),
    (dict(k_stride=120), kv.KVPRM_E_INVALID), (dict(v_stride=132), kv.KVPRM_E_INVALID),
    (dict(k_ptr=FAKE + 8), kv.KVPRM_E_INVALID), (dict(num_rows=-1), kv.KVPRM_E_INVALID),
    (dict(max_rows=-1), kv.KVPRM_E_INVALID), (dict(num_rows=1 << 31), kv.KVPRM_E_UNSUPPORTED),
])
def test_write_refuses_rows(handle, rows, status):
    cache = kv.make_cache(FAKE, FAKE, 4)
    _refused(status, lambda: kv.kvprm_write_kv(handle, cache, _batch(), 0, _rows(**rows)))


@pytest.mark.parametrize("call", ["write", "read"])
def test_rows_refuse_batches_caches_and_layers(handle, call):
    def f(h=handle, cache=None, batch=None, layer=0, rows=None):
        cache = cache or kv.make_cache(FAKE, FAKE, 4)
        getattr(kv, f"kvprm_{call}_kv")(h, cache, batch or _batch(), layer, rows or _rows())

    for kw in (dict(h=None), dict(layer=2), dict(layer=-1), dict(cache=kv.make_cache(0, FAKE, 4)),
               dict(cache=kv.make_cache(FAKE, FAKE, 0)), dict(batch=_batch(max_pages=0)),
               dict(batch=_batch(lengths_host=[10, 65])), dict(batch=_batch(page_table_ptr=0))):
        _refused(kv.KVPRM_E_INVALID, lambda: f(**kw))
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: f(batch=_batch(batch=65, lengths_host=None)))
    f(batch=_batch(batch=0))
    f(rows=_rows(num_rows=0))
    f(rows=_rows(max_rows=0, k_ptr=0))


def test_read_refuses_rows(handle):
    cache = kv.make_cache(FAKE, FAKE, 4)
    for rows in (dict(k_ptr=0, v_ptr=0), dict(index_ptr=FAKE), dict(k_stride=64), dict(v_ptr=FAKE + 2)):
        _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_read_kv(handle, cache, _batch(), 0, _rows(**rows)))


def test_fp8_rows_need_scales():
    h = kv.kvprm_create(kv.make_desc(2, 256, 4, 2, 64, 1024, kv_dtype="fp8"))
    try:
        cache = kv.make_cache(FAKE, FAKE, 4, FAKE, 0)
        _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_write_kv(h, cache, _batch(), 0, _rows()))
    finally:
        kv.kvprm_destroy(h)


def _tree(**o):
    a = dict(q_ptr=FAKE, k_ptr=FAKE, v_ptr=FAKE, o_ptr=FAKE, dtype="bf16", q_stride=256, k_stride=128,
             v_stride=128, o_stride=256, num_rows=8, start_ptr=FAKE, max_rows=4)
    a.update(o)
    return kv.make_tree(**a)


@pytest.mark.parametrize("tree,status", [
    (dict(q_ptr=0), kv.KVPRM_E_INVALID), (dict(k_ptr=0), kv.KVPRM_E_INVALID),
    (dict(v_ptr=0), kv.KVPRM_E_INVALID), (dict(o_ptr=0), kv.KVPRM_E_INVALID),
    (dict(start_ptr=0), kv.KVPRM_E_INVALID), (dict(dtype="fp8"), kv.KVPRM_E_INVALID),
    (dict(q_stride=248), kv.KVPRM_E_INVALID), (dict(k_stride=124), kv.KVPRM_E_INVALID),
    (dict(v_stride=132), kv.KVPRM_E_INVALID), (dict(o_stride=128), kv.KVPRM_E_INVALID),
    (dict(q_ptr=FAKE + 4), kv.KVPRM_E_INVALID), (dict(num_rows=-1), kv.KVPRM_E_INVALID),
    (dict(max_rows=0), kv.KVPRM_E_INVALID), (dict(max_rows=257), kv.KVPRM_E_UNSUPPORTED),
    (dict(max_rows=33, mask_ptr=FAKE, mask_words=1), kv.KVPRM_E_INVALID),
])
def test_tree_refuses(handle, tree, status):
    cache = kv.make_cache(FAKE, FAKE, 4)
    _refused(status, lambda: kv.kvprm_attention_tree(handle, cache, _batch(), 0, _tree(**tree), FAKE, 1 << 40))


def test_tree_refuses_calls(handle):
    def f(h=handle, cache=None, batch=None, layer=0, ws=FAKE, n=1 << 40):
        kv.kvprm_attention_tree(h, cache or kv.make_cache(FAKE, FAKE, 4), batch or _batch(), layer, _tree(), ws, n)

    for kw in (dict(h=None), dict(layer=2), dict(layer=-1), dict(cache=kv.make_cache(FAKE, 0, 4)),
               dict(batch=_batch(max_pages=0)), dict(batch=_batch(lengths_ptr=0))):
        _refused(kv.KVPRM_E_INVALID, lambda: f(**kw))
    for kw in (dict(ws=0), dict(n=0), dict(ws=FAKE + 128)):
        _refused(kv.KVPRM_E_WORKSPACE, lambda: f(**kw))
    f(batch=_batch(batch=0))


def test_tree_workspace_size(handle):
    """The size needs no lengths, and holds for every call of at most its rows and pages."""
    f = lambda b, t: kv.kvprm_workspace_size_tree(handle, b, t)  # noqa: E731
    assert f(_batch(batch=0), _tree()) == 0
    assert f(_batch(), _tree()) == f(_batch(lengths_host=None), _tree()) > 0
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: f(_batch(), _tree(max_rows=300)))
    _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_workspace_size_tree(None, _batch(), _tree()))
