"""Refusals of the 4-bit cache type and of the calls on pages, before anything is enqueued (CPU; the
pointers are never dereferenced)."""
import pytest

import paper_2607_09153_amd as kv

FAKE = 0x1000000


def _refused(status, call):
    with pytest.raises(kv.KvprmError) as e:
        call()
    assert e.value.status == status, kv.kvprm_last_error()
    assert kv.kvprm_last_error()


def _handle(cdt="fp4", **o):
    return kv.kvprm_create(kv.make_desc(**{**dict(num_layers=2, hidden=256, num_q_heads=4, num_kv_heads=2, head_dim=64,
                                                  ffn_dim=1024, kv_dtype=cdt), **o}))


@pytest.fixture
def handle():
    h = _handle()
    yield h
    kv.kvprm_destroy(h)


def _batch(n=2):
    return kv.make_batch(n, FAKE, 4, FAKE, [10, 64][:n])


def test_create_takes_bf16_weights():
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: _handle(weight_dtype="f32"))
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: _handle(num_q_heads=16, num_kv_heads=16))
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: _handle(head_dim=96))
    d = kv.make_desc(2, 256, 4, 2, 64, 1024)
    d.kv_dtype = 4
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: kv.kvprm_create(d))


def test_no_gradients_and_no_packing(handle):
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: kv.kvprm_workspace_size_grad(handle, _batch()))
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: kv.kvprm_pack_kv(FAKE, 2 * FAKE, 4, 64, "fp4", kv.KVPRM_KEYS))


def test_pools_are_aligned(handle):
    rows = kv.make_kv_rows(FAKE, FAKE, "bf16", 128, 128, 8, FAKE, 4)
    for k, v in ((FAKE + 8, FAKE), (FAKE, FAKE + 4), (0, FAKE), (FAKE, 0)):
        cache = kv.make_cache(k, v, 4)
        _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_write_kv(handle, cache, _batch(), 0, rows))
        _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_read_kv(handle, cache, _batch(), 0, rows))
        _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_attention(handle, cache, _batch(), 0, FAKE, FAKE, FAKE, FAKE, 1 << 30, FAKE))
    cache = kv.make_cache(FAKE, FAKE, 4)
    for dtype in ("fp8", "fp4"):
        bad = kv.make_kv_rows(FAKE, FAKE, dtype, 128, 128, 8, FAKE, 4)
        _refused(kv.KVPRM_E_INVALID, lambda: kv.kvprm_write_kv(handle, cache, _batch(), 0, bad))


# ------------------------------------------------------------------------------ pages

POOL = 100


def _place():
    """Distinct addresses for the arrays of a call."""
    return {n: FAKE * (i + 2) for i, n in enumerate(("ft", "fl", "fh", "tt", "tl", "th", "parent", "room", "refs", "new",
                                                     "result", "moved", "ws"))}


def _fork(h, ws_bytes=1 << 30, cache=None, rows=3, pages=8, children=4, to_pages=9, **at):
    a = {**_place(), **at}
    kv.kvprm_fork_pages(h, cache or kv.make_cache(FAKE, FAKE, POOL, FAKE, FAKE),
                        kv.make_page_rows(rows, pages, a["ft"], a["fl"], a["fh"]),
                        kv.make_page_rows(children, to_pages, a["tt"], a["tl"], a["th"]), a["parent"], a["room"],
                        a["refs"], a["new"], a["result"], a["ws"], ws_bytes)


def _compact(h, ws_bytes=1 << 30, cache=None, rows=3, pages=8, **at):
    a = {**_place(), **at}
    kv.kvprm_compact_pages(h, cache or kv.make_cache(FAKE, FAKE, POOL, FAKE, FAKE),
                           kv.make_page_rows(rows, pages, a["ft"], 0, a["fh"]), a["tt"], a["refs"], a["new"], a["moved"],
                           a["result"], a["ws"], ws_bytes)


@pytest.mark.parametrize("call", [_fork, _compact])
def test_pages_refuse(call):
    with_handle = lambda cdt: _handle(cdt, weight_dtype="f32" if cdt == "f32" else "bf16")  # noqa: E731
    for cdt in ("f32", "bf16", "fp8", "fp4"):
        h = with_handle(cdt)
        p = _place()
        try:
            for kw in (dict(rows=-1), dict(pages=0), dict(ft=0), dict(fh=0), dict(refs=0), dict(new=0), dict(result=0),
                       dict(tt=0), dict(cache=kv.make_cache(FAKE + 8, FAKE, POOL, FAKE, FAKE)),
                       dict(cache=kv.make_cache(FAKE, FAKE, 0, FAKE, FAKE)), dict(refs=p["refs"] + 2),
                       dict(new=p["refs"]), dict(new=p["refs"] + 4 * POOL - 4), dict(tt=p["ft"] + 4),
                       dict(result=p["fh"] + 8), dict(ws=p["refs"] - 256)):
                _refused(kv.KVPRM_E_INVALID, lambda: call(h, **kw))
            for kw in (dict(rows=257), dict(pages=(1 << 20) + 1),
                       dict(cache=kv.make_cache(FAKE, FAKE, (1 << 22) + 1, FAKE, FAKE))):
                _refused(kv.KVPRM_E_UNSUPPORTED, lambda: call(h, **kw))
            need = kv.kvprm_workspace_size_pages(h, POOL)
            for kw in (dict(ws=0), dict(ws_bytes=need - 1), dict(ws=p["ws"] + 128)):
                _refused(kv.KVPRM_E_WORKSPACE, lambda: call(h, **kw))
        finally:
            kv.kvprm_destroy(h)
    _refused(kv.KVPRM_E_INVALID, lambda: call(None))


def test_fork_refuses(handle):
    p = _place()
    for kw in (dict(children=-1), dict(to_pages=0), dict(parent=0), dict(tl=0), dict(th=0), dict(fl=0),
               dict(tt=p["tl"] - 4), dict(th=p["parent"]), dict(tl=p["room"] + 12), dict(result=p["new"] + 4 * POOL - 4)):
        _refused(kv.KVPRM_E_INVALID, lambda: _fork(handle, **kw))
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: _fork(handle, children=257))


def test_compact_refuses(handle):
    _refused(kv.KVPRM_E_INVALID, lambda: _compact(handle, moved=0))
    _refused(kv.KVPRM_E_INVALID, lambda: _compact(handle, moved=_place()["new"] + 8))


def test_pages_workspace_size(handle):
    f = kv.kvprm_workspace_size_pages
    sizes = [f(handle, n) for n in (1, 2, 63, 64, 65, 4096, 4097, 100000, 1 << 22)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    _refused(kv.KVPRM_E_INVALID, lambda: f(handle, 0))
    _refused(kv.KVPRM_E_INVALID, lambda: f(None, 4))
    _refused(kv.KVPRM_E_UNSUPPORTED, lambda: f(handle, (1 << 22) + 1))


@pytest.mark.parametrize("cdt", ["f32", "bf16", "fp8", "fp4"])
@pytest.mark.parametrize("call", [_fork, _compact])
def test_pages_refuse_arrays_in_the_pools(call, cdt):
    """The pools and their fp8 scales are written: no array or workspace lies in them, nor one over another."""
    h = _handle(cdt, weight_dtype="f32" if cdt == "f32" else "bf16")
    tile = {"f32": 64 * 64, "bf16": 32 * 64, "fp8": 16 * 64, "fp4": 17 * 32}[cdt]
    tiles = 2 * POOL * 2  # layers, pages, kv-heads
    k, v, ks, vs = (n * FAKE for n in (0x100, 0x200, 0x300, 0x400))
    end = k + tiles * tile  # the first byte past the keys
    names = ["ft", "fh", "refs", "new", "result", "tt"] + (["fl", "tl", "th", "parent", "room"] if call is _fork else ["moved"])
    places = [k, v + 256, end - 4] + ([ks, vs + 4 * tiles - 4] if cdt == "fp8" else [])
    cache = kv.make_cache(k, v, POOL, ks, vs)
    try:
        for at in places:
            for name in names:
                _refused(kv.KVPRM_E_INVALID, lambda: call(h, cache=cache, **{name: at}))
        need = kv.kvprm_workspace_size_pages(h, POOL)
        for at in (k, v + 256, k - need // 256 * 256 + 256) + ((ks, vs) if cdt == "fp8" else ()):
            _refused(kv.KVPRM_E_INVALID, lambda: call(h, cache=cache, ws=at))
        others = [(k, k, ks, vs), (k, end - 16, ks, vs), (end - 16, k, ks, vs)]
        others += [(k, v, ks, ks), (k, v, end - 4, vs), (k, v, ks, ks + 4 * tiles - 4)] if cdt == "fp8" else []
        for pools in others:
            _refused(kv.KVPRM_E_INVALID, lambda: call(h, cache=kv.make_cache(*pools[:2], POOL, *pools[2:])))
    finally:
        kv.kvprm_destroy(h)
