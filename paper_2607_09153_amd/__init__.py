"""Python binding of libkvprm (KV-PRM verify-token scoring on MI355X).

Argument marshalling only: every step of the scoring pass runs in the HIP kernels of
``libkvprm.so``; this module maps the C structures of ``include/kvprm.h`` onto ctypes and
raises on a non-OK status. Device memory and streams are the caller's (torch tensors and
streams are the usual source; pass their ``data_ptr()`` and ``cuda_stream``).
There is no fallback: if the library is not built, importing the binding raises.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvprm.so")

KVPRM_OK, KVPRM_E_INVALID, KVPRM_E_UNSUPPORTED, KVPRM_E_WORKSPACE, KVPRM_E_HIP, KVPRM_E_INTERNAL = range(6)
KVPRM_F32, KVPRM_BF16, KVPRM_FP8_E4M3, KVPRM_FP4_E2M1 = 0, 1, 2, 3
DTYPE_CODE = {"f32": KVPRM_F32, "bf16": KVPRM_BF16, "fp8": KVPRM_FP8_E4M3, "fp4": KVPRM_FP4_E2M1}

EXPORTED = ["kvprm_create", "kvprm_destroy", "kvprm_workspace_size", "kvprm_score",
            "kvprm_attention", "kvprm_attention_partials", "kvprm_pack_weight",
            "kvprm_workspace_size_lora", "kvprm_score_lora", "kvprm_workspace_size_ex",
            "kvprm_score_ex", "kvprm_workspace_size_grad", "kvprm_score_grad", "kvprm_steer",
            "kvprm_stream_read", "kvprm_score_static", "kvprm_pack_kv", "kvprm_rotary",
            "kvprm_write_kv", "kvprm_read_kv", "kvprm_workspace_size_tree",
            "kvprm_attention_tree", "kvprm_workspace_size_pages", "kvprm_fork_pages",
            "kvprm_compact_pages", "kvprm_last_error"]
KVPRM_KEYS, KVPRM_VALUES = 0, 1
STATIC_WORKSPACE_BYTES = 64 << 20  # KVPRM_STATIC_WORKSPACE_BYTES
ROPE_LAYOUT = {"half": 0, "interleaved": 1}
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "parts": 3, "ramp": 4}
LORA_PROJECTIONS = ("q", "k", "v", "o", "gate", "up", "down")


class ModelDesc(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float),
                ("weight_dtype", ctypes.c_int), ("kv_dtype", ctypes.c_int),
                ("page_size", ctypes.c_int32)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class ReadoutWeights(ctypes.Structure):
    _fields_ = [("layers", ctypes.POINTER(LayerWeights)), ("verify_embed", ctypes.c_void_p),
                ("final_norm", ctypes.c_void_p), ("reward_w", ctypes.c_void_p),
                ("reward_b", ctypes.c_float)]


class LoraFactors(ctypes.Structure):
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p)]


class LayerLora(ctypes.Structure):
    _fields_ = [(n, LoraFactors) for n in LORA_PROJECTIONS]


class Lora(ctypes.Structure):
    _fields_ = [("layers", ctypes.POINTER(LayerLora)), ("rank", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class ScoreOptions(ctypes.Structure):
    _fields_ = [("lora", ctypes.POINTER(Lora)), ("depth", ctypes.c_int32)]


class KVCache(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_pages", ctypes.c_int32)]


class Batch(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("page_table", ctypes.c_void_p),
                ("max_pages", ctypes.c_int32), ("lengths", ctypes.c_void_p),
                ("lengths_host", ctypes.POINTER(ctypes.c_int32)),
                ("num_groups", ctypes.c_int32),
                ("group_start_host", ctypes.POINTER(ctypes.c_int32)),
                ("group_prefix_len_host", ctypes.POINTER(ctypes.c_int32))]


class Rope(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("layout", ctypes.c_int), ("scaling", ctypes.c_int), ("theta", ctypes.c_double),
                ("factor", ctypes.c_double), ("trained_len", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double),
                ("magnitude", ctypes.c_double)]


class RopeHeads(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("heads", ctypes.c_int32),
                ("src_stride", ctypes.c_int64), ("dst_stride", ctypes.c_int64)]


class KVRows(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("num_rows", ctypes.c_int64), ("start", ctypes.c_void_p),
                ("index", ctypes.c_void_p), ("max_rows", ctypes.c_int32)]


class Tree(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("o", ctypes.c_void_p), ("dtype", ctypes.c_int), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("o_stride", ctypes.c_int64), ("num_rows", ctypes.c_int64),
                ("start", ctypes.c_void_p), ("max_rows", ctypes.c_int32),
                ("mask", ctypes.c_void_p), ("mask_words", ctypes.c_int32)]


class PageRows(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("page_table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("held", ctypes.c_void_p)]


class KvprmError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"kvprm status {status}: {msg}")
        self.status = status


def _preload_hip_runtime():
    """One HIP runtime per process: when torch is installed, load the runtime it ships with
    before this library, so that the library binds to that copy (torch's streams and memory
    are then valid here) rather than starting a second runtime beside torch's."""
    spec = importlib.util.find_spec("torch")
    for d in (spec.submodule_search_locations or []) if spec else []:
        rt = os.path.join(d, "lib", "libamdhip64.so")
        if os.path.exists(rt):
            ctypes.CDLL(rt, mode=ctypes.RTLD_GLOBAL)
            return


def _load():
    _preload_hip_runtime()
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built (run __graft_entry__.build()); "
                          "the scoring pass has no non-GPU implementation")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.kvprm_create.argtypes = [ctypes.POINTER(ModelDesc), ctypes.POINTER(vp)]
    lib.kvprm_destroy.argtypes = [vp]
    lib.kvprm_workspace_size.argtypes = [vp, ctypes.POINTER(Batch), ctypes.POINTER(sz)]
    lib.kvprm_score.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                ctypes.POINTER(ReadoutWeights), vp, sz, vp, vp, vp]
    lib.kvprm_attention.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                    ctypes.c_int32, vp, vp, vp, vp, sz, vp, vp]
    lib.kvprm_attention_partials.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                             ctypes.c_int32, vp, vp, sz, vp]
    lib.kvprm_score_static.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                       ctypes.POINTER(ReadoutWeights), vp, vp, vp]
    lib.kvprm_pack_weight.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int64, vp]
    lib.kvprm_pack_kv.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int32, ctypes.c_int,
                                  ctypes.c_int, vp]
    lib.kvprm_stream_read.argtypes = [vp, sz, vp, vp]
    lib.kvprm_workspace_size_lora.argtypes = [vp, ctypes.POINTER(Batch), ctypes.c_int32,
                                              ctypes.POINTER(sz)]
    lib.kvprm_score_lora.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                     ctypes.POINTER(ReadoutWeights), ctypes.POINTER(Lora), vp, sz,
                                     vp, vp, vp]
    lib.kvprm_workspace_size_ex.argtypes = [vp, ctypes.POINTER(Batch), ctypes.POINTER(ScoreOptions),
                                            ctypes.POINTER(sz)]
    lib.kvprm_score_ex.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                   ctypes.POINTER(ReadoutWeights), ctypes.POINTER(ScoreOptions),
                                   vp, sz, vp, vp, vp]
    lib.kvprm_workspace_size_grad.argtypes = [vp, ctypes.POINTER(Batch), ctypes.POINTER(sz)]
    lib.kvprm_score_grad.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                     ctypes.POINTER(ReadoutWeights), vp, sz, vp, vp, vp, vp]
    lib.kvprm_steer.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                ctypes.POINTER(ReadoutWeights), ctypes.c_float, ctypes.c_int32, vp,
                                sz, vp, vp, vp]
    lib.kvprm_rotary.argtypes = [ctypes.POINTER(Rope), ctypes.c_int, ctypes.c_int64, vp,
                                 ctypes.POINTER(RopeHeads), ctypes.c_int32, ctypes.c_int32, vp]
    lib.kvprm_write_kv.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                   ctypes.c_int32, ctypes.POINTER(KVRows), vp]
    lib.kvprm_read_kv.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                  ctypes.c_int32, ctypes.POINTER(KVRows), vp, vp]
    lib.kvprm_workspace_size_tree.argtypes = [vp, ctypes.POINTER(Batch), ctypes.POINTER(Tree),
                                              ctypes.POINTER(sz)]
    lib.kvprm_attention_tree.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(Batch),
                                         ctypes.c_int32, ctypes.POINTER(Tree), vp, sz, vp]
    lib.kvprm_workspace_size_pages.argtypes = [vp, ctypes.c_int32, ctypes.POINTER(sz)]
    lib.kvprm_fork_pages.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(PageRows),
                                     ctypes.POINTER(PageRows), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.kvprm_compact_pages.argtypes = [vp, ctypes.POINTER(KVCache), ctypes.POINTER(PageRows), vp, vp,
                                        vp, vp, vp, vp, sz, vp]
    for f in ("kvprm_create", "kvprm_destroy", "kvprm_workspace_size", "kvprm_score",
              "kvprm_attention", "kvprm_attention_partials", "kvprm_pack_weight",
              "kvprm_workspace_size_lora", "kvprm_score_lora", "kvprm_workspace_size_ex",
              "kvprm_score_ex", "kvprm_workspace_size_grad", "kvprm_score_grad", "kvprm_steer",
              "kvprm_stream_read", "kvprm_score_static", "kvprm_pack_kv", "kvprm_rotary",
              "kvprm_write_kv", "kvprm_read_kv", "kvprm_workspace_size_tree",
              "kvprm_attention_tree", "kvprm_workspace_size_pages", "kvprm_fork_pages",
              "kvprm_compact_pages"):
        getattr(lib, f).restype = ctypes.c_int
    lib.kvprm_last_error.argtypes = []
    lib.kvprm_last_error.restype = ctypes.c_char_p
    return lib


lib = _load()


def _check(st: int):
    if st != KVPRM_OK:
        raise KvprmError(st, lib.kvprm_last_error().decode())


def kvprm_last_error() -> str:
    return lib.kvprm_last_error().decode()


def make_desc(num_layers, hidden, num_q_heads, num_kv_heads, head_dim, ffn_dim,
              rope_theta=1.0e6, rms_eps=1.0e-6, weight_dtype="bf16", kv_dtype="bf16",
              page_size=16) -> ModelDesc:
    return ModelDesc(num_layers, hidden, num_q_heads, num_kv_heads, head_dim, ffn_dim,
                     rope_theta, rms_eps, DTYPE_CODE[weight_dtype], DTYPE_CODE[kv_dtype],
                     page_size)


def kvprm_create(desc: ModelDesc) -> int:
    h = ctypes.c_void_p()
    _check(lib.kvprm_create(ctypes.byref(desc), ctypes.byref(h)))
    return h.value


def kvprm_destroy(handle: int) -> None:
    _check(lib.kvprm_destroy(handle))


def make_batch(batch: int, page_table_ptr: int, max_pages: int, lengths_ptr: int,
               lengths_host: Optional[Sequence[int]] = None,
               group_start: Optional[Sequence[int]] = None,
               group_prefix_len: Optional[Sequence[int]] = None) -> Batch:
    """Batch descriptor; host arrays are copied into ctypes buffers kept alive on the struct."""
    b = Batch()
    b.batch, b.page_table, b.max_pages, b.lengths = batch, page_table_ptr, max_pages, lengths_ptr
    keep = []
    if lengths_host is not None:
        arr = (ctypes.c_int32 * len(lengths_host))(*lengths_host)
        keep.append(arr)
        b.lengths_host = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32))
    if group_start:
        gs = (ctypes.c_int32 * len(group_start))(*group_start)
        gp = (ctypes.c_int32 * len(group_prefix_len))(*group_prefix_len)
        keep += [gs, gp]
        b.num_groups = len(group_prefix_len)
        b.group_start_host = ctypes.cast(gs, ctypes.POINTER(ctypes.c_int32))
        b.group_prefix_len_host = ctypes.cast(gp, ctypes.POINTER(ctypes.c_int32))
    b._keep = keep
    return b


def make_cache(k_ptr: int, v_ptr: int, num_pages: int, k_scale_ptr: int = 0,
               v_scale_ptr: int = 0) -> KVCache:
    return KVCache(k_ptr, v_ptr, k_scale_ptr or None, v_scale_ptr or None, num_pages)


def make_readout(layers: Sequence[dict], verify_embed: int, final_norm: int, reward_w: int,
                 reward_b: float = 0.0) -> ReadoutWeights:
    """layers: per layer a dict of device pointers with the LayerWeights field names."""
    arr = (LayerWeights * len(layers))()
    for i, d in enumerate(layers):
        for name, _ in LayerWeights._fields_:
            setattr(arr[i], name, d[name])
    r = ReadoutWeights(ctypes.cast(arr, ctypes.POINTER(LayerWeights)), verify_embed, final_norm,
                       reward_w, reward_b)
    r._keep = arr
    return r


def make_lora(layers: Sequence[dict], rank: int, scale: float) -> Lora:
    """layers: per layer a dict projection -> (a_ptr, b_ptr) of device pointers; projections
    missing from the dict have no adapter."""
    arr = (LayerLora * len(layers))()
    for i, d in enumerate(layers):
        for p in LORA_PROJECTIONS:
            a, b = d.get(p, (None, None))
            setattr(arr[i], p, LoraFactors(a or None, b or None))
    r = Lora(ctypes.cast(arr, ctypes.POINTER(LayerLora)), rank, scale)
    r._keep = arr
    return r


def kvprm_workspace_size_lora(handle: int, batch: Batch, rank: int) -> int:
    n = ctypes.c_size_t()
    _check(lib.kvprm_workspace_size_lora(handle, ctypes.byref(batch), rank, ctypes.byref(n)))
    return n.value


def kvprm_score_lora(handle: int, cache: KVCache, batch: Batch, base: ReadoutWeights,
                     lora: Lora, workspace_ptr: int, ws_bytes: int, scores_ptr: int,
                     logits_ptr: int = 0, stream: int = 0) -> None:
    _check(lib.kvprm_score_lora(handle, ctypes.byref(cache), ctypes.byref(batch),
                                ctypes.byref(base), ctypes.byref(lora), workspace_ptr, ws_bytes,
                                scores_ptr, logits_ptr or None, stream or None))


def make_options(lora: Optional[Lora] = None, depth: int = 1) -> ScoreOptions:
    o = ScoreOptions(ctypes.pointer(lora) if lora is not None else None, depth)
    o._keep = lora
    return o


def kvprm_workspace_size_ex(handle: int, batch: Batch, options: Optional[ScoreOptions]) -> int:
    n = ctypes.c_size_t()
    _check(lib.kvprm_workspace_size_ex(handle, ctypes.byref(batch),
                                       ctypes.byref(options) if options is not None else None,
                                       ctypes.byref(n)))
    return n.value


def kvprm_score_ex(handle: int, cache: KVCache, batch: Batch, weights: ReadoutWeights,
                   options: Optional[ScoreOptions], workspace_ptr: int, ws_bytes: int,
                   scores_ptr: int, logits_ptr: int = 0, stream: int = 0) -> None:
    _check(lib.kvprm_score_ex(handle, ctypes.byref(cache), ctypes.byref(batch),
                              ctypes.byref(weights),
                              ctypes.byref(options) if options is not None else None,
                              workspace_ptr, ws_bytes, scores_ptr, logits_ptr or None,
                              stream or None))


def kvprm_workspace_size_grad(handle: int, batch: Batch) -> int:
    n = ctypes.c_size_t()
    _check(lib.kvprm_workspace_size_grad(handle, ctypes.byref(batch), ctypes.byref(n)))
    return n.value


def kvprm_score_grad(handle: int, cache: KVCache, batch: Batch, weights: ReadoutWeights,
                     workspace_ptr: int, ws_bytes: int, scores_ptr: int, grad_k_ptr: int,
                     grad_v_ptr: int, stream: int = 0) -> None:
    _check(lib.kvprm_score_grad(handle, ctypes.byref(cache), ctypes.byref(batch),
                                ctypes.byref(weights), workspace_ptr, ws_bytes, scores_ptr,
                                grad_k_ptr, grad_v_ptr, stream or None))


def kvprm_steer(handle: int, cache: KVCache, batch: Batch, weights: ReadoutWeights, eta: float,
                steps: int, workspace_ptr: int, ws_bytes: int, scores_before_ptr: int,
                scores_after_ptr: int, stream: int = 0) -> None:
    _check(lib.kvprm_steer(handle, ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(weights),
                           eta, steps, workspace_ptr, ws_bytes, scores_before_ptr,
                           scores_after_ptr, stream or None))


def kvprm_workspace_size(handle: int, batch: Batch) -> int:
    n = ctypes.c_size_t()
    _check(lib.kvprm_workspace_size(handle, ctypes.byref(batch), ctypes.byref(n)))
    return n.value


def kvprm_score(handle: int, cache: KVCache, batch: Batch, weights: ReadoutWeights,
                workspace_ptr: int, ws_bytes: int, scores_ptr: int, logits_ptr: int = 0,
                stream: int = 0) -> None:
    _check(lib.kvprm_score(handle, ctypes.byref(cache), ctypes.byref(batch), ctypes.byref(weights),
                           workspace_ptr, ws_bytes, scores_ptr, logits_ptr or None, stream or None))


def kvprm_score_static(handle: int, cache: KVCache, batch: Batch, weights: ReadoutWeights,
                       scores_ptr: int, logits_ptr: int = 0, stream: int = 0) -> None:
    _check(lib.kvprm_score_static(handle, ctypes.byref(cache), ctypes.byref(batch),
                                  ctypes.byref(weights), scores_ptr, logits_ptr or None,
                                  stream or None))


def kvprm_stream_read(buf_ptr: int, nbytes: int, sink_ptr: int, stream: int = 0) -> None:
    _check(lib.kvprm_stream_read(buf_ptr, nbytes, sink_ptr, stream or None))


def kvprm_pack_weight(src_ptr: int, dst_ptr: int, rows: int, K: int, stream: int = 0) -> None:
    _check(lib.kvprm_pack_weight(src_ptr, dst_ptr, rows, K, stream or None))


def kvprm_pack_kv(src_ptr: int, dst_ptr: int, num_tiles: int, head_dim: int, dtype: str,
                  part: int, stream: int = 0) -> None:
    """Token-major cache tiles -> the stored K (part = KVPRM_KEYS) or V tile layout."""
    _check(lib.kvprm_pack_kv(src_ptr or None, dst_ptr or None, num_tiles, head_dim,
                             DTYPE_CODE[dtype], part, stream or None))


def kvprm_attention_partials(handle: int, cache: KVCache, batch: Batch, layer: int, q_ptr: int,
                             workspace_ptr: int, ws_bytes: int, stream: int = 0) -> None:
    _check(lib.kvprm_attention_partials(handle, ctypes.byref(cache), ctypes.byref(batch), layer,
                                        q_ptr, workspace_ptr, ws_bytes, stream or None))


def kvprm_attention(handle: int, cache: KVCache, batch: Batch, layer: int, q_ptr: int,
                    k_self_ptr: int, v_self_ptr: int, workspace_ptr: int, ws_bytes: int,
                    o_ptr: int, stream: int = 0) -> None:
    _check(lib.kvprm_attention(handle, ctypes.byref(cache), ctypes.byref(batch), layer, q_ptr,
                               k_self_ptr, v_self_ptr, workspace_ptr, ws_bytes, o_ptr,
                               stream or None))


def make_rope(head_dim: int, rotary_dim: Optional[int] = None, layout: str = "half",
              theta: float = 1.0e6, scaling: str = "none", factor: float = 1.0,
              trained_len: float = 0.0, low: float = 1.0, high: float = 32.0,
              magnitude: float = 1.0) -> Rope:
    """Rotary embedding: the first rotary_dim (default: all) dims of each head; layout "half" or
    "interleaved"; scaling "none", "linear", "base", "parts" or "ramp" (kvprm_rope_scaling)."""
    return Rope(head_dim, head_dim if rotary_dim is None else rotary_dim, ROPE_LAYOUT[layout],
                ROPE_SCALING[scaling], theta, factor, trained_len, low, high, magnitude)


def make_rope_heads(tensors: Sequence[tuple]):
    """tensors: one or two of (src_ptr, dst_ptr, heads, src_stride, dst_stride)."""
    return (RopeHeads * len(tensors))(*[RopeHeads(s or None, d or None, *rest)
                                        for s, d, *rest in tensors])


def kvprm_rotary(rope: Rope, dtype: str, rows: int, positions_ptr: int, tensors,
                 transpose: bool = False, stream: int = 0) -> None:
    """tensors: of make_rope_heads."""
    _check(lib.kvprm_rotary(ctypes.byref(rope), DTYPE_CODE[dtype], rows, positions_ptr or None,
                            tensors, len(tensors), int(transpose), stream or None))


def make_kv_rows(k_ptr: int, v_ptr: int, dtype: str, k_stride: int, v_stride: int, num_rows: int,
                 start_ptr: int, max_rows: int, index_ptr: int = 0) -> KVRows:
    return KVRows(k_ptr or None, v_ptr or None, DTYPE_CODE[dtype], k_stride, v_stride, num_rows,
                  start_ptr or None, index_ptr or None, max_rows)


def kvprm_write_kv(handle: int, cache: KVCache, batch: Batch, layer: int, rows: KVRows,
                   stream: int = 0) -> None:
    _check(lib.kvprm_write_kv(handle, ctypes.byref(cache), ctypes.byref(batch), layer,
                              ctypes.byref(rows), stream or None))


def kvprm_read_kv(handle: int, cache: KVCache, batch: Batch, layer: int, rows: KVRows,
                  first_ptr: int = 0, stream: int = 0) -> None:
    _check(lib.kvprm_read_kv(handle, ctypes.byref(cache), ctypes.byref(batch), layer,
                             ctypes.byref(rows), first_ptr or None, stream or None))


def make_tree(q_ptr: int, k_ptr: int, v_ptr: int, o_ptr: int, dtype: str, q_stride: int,
              k_stride: int, v_stride: int, o_stride: int, num_rows: int, start_ptr: int,
              max_rows: int, mask_ptr: int = 0, mask_words: int = 0) -> Tree:
    return Tree(q_ptr or None, k_ptr or None, v_ptr or None, o_ptr or None, DTYPE_CODE[dtype],
                q_stride, k_stride, v_stride, o_stride, num_rows, start_ptr or None, max_rows,
                mask_ptr or None, mask_words)


def kvprm_workspace_size_tree(handle: int, batch: Batch, tree: Tree) -> int:
    n = ctypes.c_size_t()
    _check(lib.kvprm_workspace_size_tree(handle, ctypes.byref(batch), ctypes.byref(tree),
                                         ctypes.byref(n)))
    return n.value


def kvprm_attention_tree(handle: int, cache: KVCache, batch: Batch, layer: int, tree: Tree,
                         workspace_ptr: int, ws_bytes: int, stream: int = 0) -> None:
    _check(lib.kvprm_attention_tree(handle, ctypes.byref(cache), ctypes.byref(batch), layer,
                                    ctypes.byref(tree), workspace_ptr, ws_bytes, stream or None))


def make_page_rows(rows: int, max_pages: int, page_table_ptr: int, lengths_ptr: int, held_ptr: int) -> PageRows:
    return PageRows(rows, max_pages, page_table_ptr or None, lengths_ptr or None, held_ptr or None)


def kvprm_workspace_size_pages(handle: int, num_pages: int) -> int:
    n = ctypes.c_size_t()
    _check(lib.kvprm_workspace_size_pages(handle, num_pages, ctypes.byref(n)))
    return n.value


def kvprm_fork_pages(handle: int, cache: KVCache, from_rows: PageRows, to_rows: PageRows, parent_ptr: int,
                     room_ptr: int, refs_ptr: int, new_refs_ptr: int, result_ptr: int, workspace_ptr: int,
                     ws_bytes: int, stream: int = 0) -> None:
    """room_ptr 0: no pages beyond the tokens'."""
    _check(lib.kvprm_fork_pages(handle, ctypes.byref(cache), ctypes.byref(from_rows), ctypes.byref(to_rows),
                                parent_ptr or None, room_ptr or None, refs_ptr or None, new_refs_ptr or None,
                                result_ptr or None, workspace_ptr, ws_bytes, stream or None))


def kvprm_compact_pages(handle: int, cache: KVCache, rows: PageRows, new_table_ptr: int, refs_ptr: int,
                        new_refs_ptr: int, moved_ptr: int, result_ptr: int, workspace_ptr: int, ws_bytes: int,
                        stream: int = 0) -> None:
    _check(lib.kvprm_compact_pages(handle, ctypes.byref(cache), ctypes.byref(rows), new_table_ptr or None,
                                   refs_ptr or None, new_refs_ptr or None, moved_ptr or None, result_ptr or None,
                                   workspace_ptr, ws_bytes, stream or None))
