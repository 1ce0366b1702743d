"""Python binding of libhb.so (include/hb.h): argument marshalling only.

Every step of the layer runs in the library's HIP kernels; PyTorch supplies
device memory and streams. Names and arguments follow the C ABI.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Iterable, List, Optional, Sequence, Tuple

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhb.so")

HB_OK, HB_ERR_INVALID, HB_ERR_RANGE, HB_ERR_OOM, HB_ERR_HIP, HB_ERR_UNSUPPORTED = range(6)
HB_OUT_F32, HB_OUT_BF16 = 0, 1
(HB_K_RMSNORM_ATTN, HB_K_GEMM_QKV, HB_K_ATTENTION, HB_K_ATTN_MERGE, HB_K_GEMM_O,
 HB_K_RMSNORM_FFN, HB_K_GEMM_GATE_UP, HB_K_GEMM_DOWN, HB_K_COUNT) = range(9)
HB_STAGE_Q, HB_STAGE_ATTN, HB_STAGE_H2, HB_STAGE_MLP = range(4)
HB_GEMM_QKV, HB_GEMM_O, HB_GEMM_GATE_UP, HB_GEMM_DOWN, HB_GEMM_COUNT = range(5)
GEMM_NAMES = ("gemm_qkv", "gemm_o", "gemm_gate_up", "gemm_down")

EXPORTED = ("hb_create_layer", "hb_destroy_layer", "hb_append_kv", "hb_run_iteration", "hb_validate_batch",
            "hb_profile", "hb_profile_batches", "hb_latency_features", "hb_fit_latency_model", "hb_predict_latency", "hb_select_chunk",
            "hb_create_model", "hb_destroy_model", "hb_model_layer", "hb_run_model",
            "hb_set_kernel_timing", "hb_kernel_times", "hb_kernel_name", "hb_layer_stage", "hb_last_error",
            "hb_gemm_tile_count", "hb_plan_gemms", "hb_layer_gemm_plans", "hb_run_iteration_noalloc",
            "hb_measure_device_rates", "hb_set_attention_window", "hb_window_dead_blocks", "hb_create_attention",
            "hb_destroy_attention", "hb_plan_attention", "hb_run_attention", "hb_copy_blocks", "hb_copy_model_blocks",
            "hb_plan_compaction", "hb_plan_shared_attention", "hb_rope_frequencies", "hb_set_attention_rope",
            "hb_run_append", "hb_create_sampler", "hb_destroy_sampler", "hb_sample")
HB_LAT_FEATURES = 5
HB_ROPE_HALF, HB_ROPE_INTERLEAVED = 0, 1
HB_ROPE_UNSCALED, HB_ROPE_LINEAR, HB_ROPE_BY_PARTS = range(3)


class hb_layer_config(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("ffn_dim", C.c_int32), ("kv_block_size", C.c_int32),
                ("rope_theta", C.c_float), ("rms_eps", C.c_float),
                ("max_batch_tokens", C.c_int32), ("max_requests", C.c_int32)]


class hb_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_qkv", "w_o", "w_gate_up", "w_down", "g_attn", "g_ffn")]


class hb_kv_pool(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("num_blocks", C.c_int32)]


class hb_request(C.Structure):
    _fields_ = [("chunk_len", C.c_int32), ("context_len", C.c_int32),
                ("block_table", C.POINTER(C.c_int32)), ("n_blocks", C.c_int32)]


class hb_batch_desc(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("requests", C.POINTER(hb_request)),
                ("x_in", C.c_void_p), ("x_out", C.c_void_p), ("out_dtype", C.c_int32)]


class hb_prefix_group(C.Structure):
    _fields_ = [("first", C.c_int32), ("count", C.c_int32), ("prefix_len", C.c_int32)]


class hb_rope_scaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("original_context", C.c_int32), ("factor", C.c_double), ("low", C.c_double),
                ("high", C.c_double)]


class hb_sample_desc(C.Structure):
    _fields_ = ([("n_rows", C.c_int32), ("logits_dtype", C.c_int32), ("logits", C.c_void_p), ("row_stride", C.c_int64)]
                + [(n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p", "u", "tokens", "probs")])


class hb_device_rates(C.Structure):
    _fields_ = [("random_4kb_read_bytes_per_s", C.c_double), ("stream_read_bytes_per_s", C.c_double),
                ("mfma_bf16_flop_per_s", C.c_double)]


class hb_decode_mix(C.Structure):
    _fields_ = [("n_decode", C.c_int32), ("decode_contexts", C.POINTER(C.c_int32)), ("chunk_context", C.c_int32)]


class hb_profile_cell(C.Structure):
    _fields_ = [(n, C.c_float) for n in ("median_ms", "p10_ms", "p90_ms", "tokens_per_s", "hbm_frac", "mfma_frac")]


class hb_latency_model(C.Structure):
    _fields_ = [("coef", C.c_double * HB_LAT_FEATURES), ("fit_rel_rms", C.c_double), ("fit_max_under", C.c_double),
                ("n_cells", C.c_int32)]


class hb_model_desc(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("vocab", C.c_int32), ("layers", C.POINTER(hb_layer_weights)),
                ("pools", C.POINTER(hb_kv_pool)), ("embed", C.c_void_p), ("g_final", C.c_void_p),
                ("lm_head", C.c_void_p)]


class hb_model_batch(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("requests", C.POINTER(hb_request)), ("token_ids", C.c_void_p),
                ("logits", C.c_void_p), ("next_tokens", C.c_void_p), ("hidden_states", C.c_void_p)]


class HBError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"hb status {status}: {message}")
        self.status = status


_lib: Optional[C.CDLL] = None


def load() -> C.CDLL:
    """Load libhb.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_22562_amd.build`")
    # torch first: libhb then binds to the HIP runtime torch already loaded,
    # so torch's streams and allocations are valid handles for the library.
    import torch  # noqa: F401
    lib = C.CDLL(LIB_PATH)
    st = C.c_int
    lib.hb_create_layer.argtypes = [C.POINTER(hb_layer_config), C.POINTER(hb_layer_weights), C.POINTER(hb_kv_pool),
                                    C.c_void_p, C.POINTER(C.c_void_p)]
    lib.hb_create_layer.restype = st
    lib.hb_destroy_layer.argtypes = [C.c_void_p]
    lib.hb_destroy_layer.restype = None
    lib.hb_append_kv.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                 C.c_void_p]
    lib.hb_append_kv.restype = st
    lib.hb_run_iteration.argtypes = [C.c_void_p, C.POINTER(hb_batch_desc)]
    lib.hb_run_iteration.restype = st
    lib.hb_run_iteration_noalloc.argtypes = [C.c_void_p, C.POINTER(hb_batch_desc)]
    lib.hb_run_iteration_noalloc.restype = st
    lib.hb_validate_batch.argtypes = [C.POINTER(hb_layer_config), C.c_int32, C.POINTER(hb_batch_desc)]
    lib.hb_validate_batch.restype = st
    lib.hb_profile.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_int32, C.POINTER(hb_decode_mix), C.c_int32,
                               C.c_int32, C.c_int32, C.c_uint64, C.POINTER(hb_profile_cell)]
    lib.hb_profile.restype = st
    lib.hb_profile_batches.argtypes = [C.c_void_p, C.POINTER(hb_batch_desc), C.c_int32, C.c_int32, C.c_int32,
                                       C.POINTER(hb_profile_cell)]
    lib.hb_profile_batches.restype = st
    lib.hb_latency_features.argtypes = [C.POINTER(hb_layer_config), C.POINTER(hb_request), C.c_int32,
                                        C.POINTER(C.c_double)]
    lib.hb_latency_features.restype = st
    lib.hb_fit_latency_model.argtypes = [C.POINTER(hb_layer_config), C.POINTER(C.c_int32), C.c_int32,
                                         C.POINTER(hb_decode_mix), C.c_int32, C.POINTER(hb_profile_cell),
                                         C.POINTER(hb_latency_model)]
    lib.hb_fit_latency_model.restype = st
    lib.hb_predict_latency.argtypes = [C.POINTER(hb_latency_model), C.POINTER(hb_layer_config), C.POINTER(hb_request),
                                       C.c_int32, C.POINTER(C.c_double)]
    lib.hb_predict_latency.restype = st
    lib.hb_select_chunk.argtypes = [C.POINTER(hb_latency_model), C.POINTER(hb_layer_config), C.POINTER(C.c_int32),
                                    C.POINTER(C.c_double), C.c_int32, C.c_double, C.c_int32, C.c_int32, C.c_int32,
                                    C.c_double, C.POINTER(C.c_int32), C.POINTER(C.c_double)]
    lib.hb_select_chunk.restype = st
    lib.hb_create_model.argtypes = [C.POINTER(hb_layer_config), C.POINTER(hb_model_desc), C.c_void_p,
                                    C.POINTER(C.c_void_p)]
    lib.hb_create_model.restype = st
    lib.hb_destroy_model.argtypes = [C.c_void_p]
    lib.hb_destroy_model.restype = None
    lib.hb_model_layer.argtypes = [C.c_void_p, C.c_int32]
    lib.hb_model_layer.restype = C.c_void_p
    lib.hb_run_model.argtypes = [C.c_void_p, C.POINTER(hb_model_batch)]
    lib.hb_run_model.restype = st
    lib.hb_set_kernel_timing.argtypes = [C.c_void_p, C.c_uint32]
    lib.hb_set_kernel_timing.restype = st
    lib.hb_kernel_times.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64), C.c_int32]
    lib.hb_kernel_times.restype = st
    lib.hb_kernel_name.argtypes = [C.c_int32]
    lib.hb_kernel_name.restype = C.c_char_p
    lib.hb_layer_stage.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_void_p), C.POINTER(C.c_int64)]
    lib.hb_layer_stage.restype = st
    lib.hb_last_error.argtypes = []
    lib.hb_last_error.restype = C.c_char_p
    lib.hb_gemm_tile_count.argtypes = []
    lib.hb_gemm_tile_count.restype = C.c_int32
    lib.hb_plan_gemms.argtypes = [C.POINTER(hb_layer_config), C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                  C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.hb_plan_gemms.restype = st
    lib.hb_layer_gemm_plans.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.hb_layer_gemm_plans.restype = st
    lib.hb_measure_device_rates.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.POINTER(hb_device_rates)]
    lib.hb_measure_device_rates.restype = st
    i32p = C.POINTER(C.c_int32)
    lib.hb_set_attention_window.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
    lib.hb_set_attention_window.restype = st
    lib.hb_window_dead_blocks.argtypes = [C.c_int32, C.c_int32, C.c_int32, i32p, i32p]
    lib.hb_window_dead_blocks.restype = st
    lib.hb_create_attention.argtypes = [C.POINTER(hb_layer_config), C.c_int32, C.c_void_p, C.POINTER(C.c_void_p)]
    lib.hb_create_attention.restype = st
    lib.hb_destroy_attention.argtypes = [C.c_void_p]
    lib.hb_destroy_attention.restype = None
    lib.hb_plan_attention.argtypes = [C.c_void_p, C.c_int32, C.POINTER(hb_request), C.c_int32, C.c_int32]
    lib.hb_plan_attention.restype = st
    lib.hb_run_attention.argtypes = [C.c_void_p, C.POINTER(hb_kv_pool), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64]
    lib.hb_run_attention.restype = st
    lib.hb_plan_shared_attention.argtypes = [C.c_void_p, C.c_int32, C.POINTER(hb_request), C.c_int32, C.c_void_p]
    lib.hb_plan_shared_attention.restype = st
    lib.hb_rope_frequencies.argtypes = [C.c_int32, C.c_double, C.POINTER(hb_rope_scaling), C.c_void_p]
    lib.hb_rope_frequencies.restype = st
    lib.hb_set_attention_rope.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_double]
    lib.hb_set_attention_rope.restype = st
    lib.hb_run_append.argtypes = [C.c_void_p, C.POINTER(hb_kv_pool), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                  C.c_void_p, C.c_int64, C.c_void_p, C.c_int64]
    lib.hb_run_append.restype = st
    lib.hb_create_sampler.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_void_p)]
    lib.hb_create_sampler.restype = st
    lib.hb_destroy_sampler.argtypes = [C.c_void_p]
    lib.hb_destroy_sampler.restype = None
    lib.hb_sample.argtypes = [C.c_void_p, C.POINTER(hb_sample_desc)]
    lib.hb_sample.restype = st
    for f in (lib.hb_copy_blocks, lib.hb_copy_model_blocks):
        f.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32]
        f.restype = st
    lib.hb_plan_compaction.argtypes = [C.c_int32, C.POINTER(C.c_void_p), i32p, C.c_int32, C.c_void_p, C.c_void_p,
                                       i32p, i32p]
    lib.hb_plan_compaction.restype = st
    _lib = lib
    return lib


def hb_last_error() -> str:
    return load().hb_last_error().decode()


def _check(status: int) -> None:
    if status != HB_OK:
        raise HBError(status, hb_last_error())


def make_config(shape, max_batch_tokens: int, max_requests: int) -> hb_layer_config:
    """hb_layer_config from any object with the layer-shape attributes."""
    return hb_layer_config(shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn_dim,
                           getattr(shape, "kv_block", 16), float(shape.rope_theta), float(shape.rms_eps),
                           int(max_batch_tokens), int(max_requests))


class Layer:
    """Owns an hb_layer handle (unless borrowed from a model) and keeps the
    tensors it points at alive."""

    borrowed = False

    def __init__(self, handle: C.c_void_p, cfg: hb_layer_config, keep: list):
        self.handle = handle
        self.cfg = cfg
        self._keep = keep

    def __del__(self):
        try:
            if not self.borrowed:
                hb_destroy_layer(self)
        except Exception:
            pass


class Model:
    """Owns an hb_model handle and keeps the tensors it points at alive."""

    def __init__(self, handle: C.c_void_p, cfg: hb_layer_config, n_layers: int, vocab: int, keep: list):
        self.handle = handle
        self.cfg = cfg
        self.n_layers = n_layers
        self.vocab = vocab
        self._keep = keep

    def layer(self, index: int) -> "Layer":
        """Borrowed handle of layer `index` (the model destroys it)."""
        h = load().hb_model_layer(self.handle, int(index))
        if not h:
            raise IndexError(index)
        lay = Layer(C.c_void_p(h), self.cfg, [self])
        lay.borrowed = True
        return lay

    def __del__(self):
        try:
            hb_destroy_model(self)
        except Exception:
            pass


def hb_create_model(cfg: hb_layer_config, layer_weights: Sequence[Dict[str, "torch.Tensor"]], pools,
                    num_blocks: int, embed, g_final, lm_head, stream: Optional[int] = None) -> Model:
    """pools: [(k_pool, v_pool)] per layer."""
    n = len(layer_weights)
    wa = (hb_layer_weights * n)()
    pa = (hb_kv_pool * n)()
    for i, (w, (kp, vp)) in enumerate(zip(layer_weights, pools)):
        wa[i] = hb_layer_weights(*(_ptr(w[k]) for k in ("w_qkv", "w_o", "w_gate_up", "w_down", "g_attn", "g_ffn")))
        pa[i] = hb_kv_pool(_ptr(kp), _ptr(vp), int(num_blocks))
    vocab = int(embed.shape[0])
    d = hb_model_desc(n, vocab, wa, pa, C.c_void_p(_ptr(embed)), C.c_void_p(_ptr(g_final)), C.c_void_p(_ptr(lm_head)))
    if stream is None:
        import torch
        stream = torch.cuda.current_stream().cuda_stream
    h = C.c_void_p()
    _check(load().hb_create_model(C.byref(cfg), C.byref(d), C.c_void_p(stream), C.byref(h)))
    return Model(h, cfg, n, vocab, [layer_weights, pools, embed, g_final, lm_head])


def hb_destroy_model(model: Model) -> None:
    if model.handle is not None and model.handle.value:
        load().hb_destroy_model(model.handle)
        model.handle = None


def hb_run_model(model: Model, requests: Sequence[Tuple[int, int, Iterable[int]]], token_ids, next_tokens,
                 logits=None, hidden_states=None) -> None:
    """token_ids: device int32 [T]; next_tokens: device int32 [n_requests];
    logits: device fp32 [n_requests][vocab] or None; hidden_states: device
    bf16 [n_layers][T][H] (every layer's output) or None."""
    d, keep = _desc(requests, 0, 0, HB_OUT_BF16)
    b = hb_model_batch(len(requests), d.requests, C.c_void_p(_ptr(token_ids)), C.c_void_p(_ptr(logits)),
                       C.c_void_p(_ptr(next_tokens)), C.c_void_p(_ptr(hidden_states)))
    _check(load().hb_run_model(model.handle, C.byref(b)))


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def hb_create_layer(cfg: hb_layer_config, weights: Dict[str, "torch.Tensor"], k_pool, v_pool,
                    num_blocks: int, stream: Optional[int] = None) -> Layer:
    lib = load()
    w = hb_layer_weights(*(_ptr(weights[n]) for n in ("w_qkv", "w_o", "w_gate_up", "w_down", "g_attn", "g_ffn")))
    pool = hb_kv_pool(_ptr(k_pool), _ptr(v_pool), int(num_blocks))
    if stream is None:
        import torch
        stream = torch.cuda.current_stream().cuda_stream
    h = C.c_void_p()
    _check(lib.hb_create_layer(C.byref(cfg), C.byref(w), C.byref(pool), C.c_void_p(stream), C.byref(h)))
    return Layer(h, cfg, [weights, k_pool, v_pool])


def hb_destroy_layer(layer: Layer) -> None:
    if layer.handle is not None and layer.handle.value:
        load().hb_destroy_layer(layer.handle)
        layer.handle = None


_INT32 = np.dtype(np.int32)


def _i32(a) -> np.ndarray:
    """The values of `a` as int32, or a ValueError: NumPy checks Python integers by itself, but keeps the low 32 bits
    of an array's wider ones."""
    if getattr(a, "dtype", _INT32) is _INT32:
        try:
            return np.ascontiguousarray(a, dtype=np.int32)
        except OverflowError as e:
            raise ValueError(str(e)) from None
    a = np.asarray(a)
    with np.errstate(invalid="ignore"):
        b = np.ascontiguousarray(a, dtype=np.int32)
    if (a != b).any():
        raise ValueError(f"values of {a.dtype} that are no 32-bit integers")
    return b


def _int32(v) -> int:
    """An argument of the C interface: ctypes would keep its low 32 bits without a word."""
    v = int(v)
    if not -(1 << 31) <= v < 1 << 31:
        raise ValueError(f"{v} does not fit 32 bits")
    return v


def _ids(a) -> np.ndarray:
    """Block ids as a new or the caller's int32 array."""
    if getattr(a, "dtype", _INT32) is not _INT32:
        a = np.asarray(a)
        if a.size and a.dtype.kind not in "iu":
            raise ValueError(f"block ids are 32-bit integers, not {a.dtype}")
    return _i32(a)


def hb_append_kv(layer: Layer, block_table, context_len: int, k, v) -> None:
    bt = _i32(block_table)
    n = 0 if k is None else int(k.shape[0])
    _check(load().hb_append_kv(layer.handle, bt.ctypes.data_as(C.POINTER(C.c_int32)), len(bt), _int32(context_len), _int32(n),
                               C.c_void_p(_ptr(k)), C.c_void_p(_ptr(v))))


# hb_request as a NumPy record: the request array is filled with array
# operations instead of one ctypes object per request
_REQ_DTYPE = np.dtype({"names": ["chunk_len", "context_len", "block_table", "n_blocks"],
                       "formats": [np.int32, np.int32, np.uintp, np.int32],
                       "offsets": [hb_request.chunk_len.offset, hb_request.context_len.offset,
                                   hb_request.block_table.offset, hb_request.n_blocks.offset],
                       "itemsize": C.sizeof(hb_request)})


def _desc(requests: Sequence[Tuple[int, int, Iterable[int]]], x_in_ptr: int, x_out_ptr: int, out_dtype: int):
    n = len(requests)
    tables = [bt if getattr(bt, "dtype", None) is _INT32 else _i32(bt) for (_, _, bt) in requests]
    flat = np.concatenate(tables) if n else np.zeros(1, np.int32)
    lens = np.fromiter((len(bt) for bt in tables), dtype=np.int64, count=n)
    rec = np.zeros(max(1, n), dtype=_REQ_DTYPE)
    if n:
        cx = _i32([(r[0], r[1]) for r in requests]).reshape(n, 2)
        rec["chunk_len"][:n] = cx[:, 0]
        rec["context_len"][:n] = cx[:, 1]
        starts = np.concatenate([[0], np.cumsum(lens)[:-1]])
        rec["block_table"][:n] = flat.ctypes.data + 4 * starts
        rec["n_blocks"][:n] = lens
    arr = rec.ctypes.data_as(C.POINTER(hb_request))
    d = hb_batch_desc(n, arr, C.c_void_p(x_in_ptr), C.c_void_p(x_out_ptr), int(out_dtype))
    return d, (flat, rec, arr)


def hb_run_iteration(layer: Layer, requests: Sequence[Tuple[int, int, Iterable[int]]], x_in, x_out,
                     out_dtype: Optional[int] = None) -> None:
    """requests: (chunk_len, context_len, block_table) per request, in row order."""
    if out_dtype is None:
        import torch
        out_dtype = HB_OUT_F32 if x_out.dtype == torch.float32 else HB_OUT_BF16
    d, keep = _desc(requests, _ptr(x_in), _ptr(x_out), out_dtype)
    _check(load().hb_run_iteration(layer.handle, C.byref(d)))


def hb_run_iteration_noalloc(layer: Layer, requests: Sequence[Tuple[int, int, Iterable[int]]], x_in, x_out,
                             out_dtype: Optional[int] = None) -> None:
    """As hb_run_iteration, through the allocation-free entry point."""
    if out_dtype is None:
        import torch
        out_dtype = HB_OUT_F32 if x_out.dtype == torch.float32 else HB_OUT_BF16
    d, keep = _desc(requests, _ptr(x_in), _ptr(x_out), out_dtype)
    _check(load().hb_run_iteration_noalloc(layer.handle, C.byref(d)))


def hb_set_attention_window(layer: Layer, window: int, sinks: int = 0) -> None:
    """Sliding window of the layer's later iterations (0: every earlier key)."""
    _check(load().hb_set_attention_window(layer.handle, _int32(window), _int32(sinks)))


def hb_window_dead_blocks(context_len: int, window: int, sinks: int = 0) -> Tuple[int, int]:
    """(first, count): the block-table entries that no row at a position >= context_len sees."""
    first, count = C.c_int32(), C.c_int32()
    _check(load().hb_window_dead_blocks(_int32(context_len), _int32(window), _int32(sinks), C.byref(first), C.byref(count)))
    return first.value, count.value


class Attention:
    """Owns an hb_attention handle; n_tokens: rows of the current plan."""

    def __init__(self, handle: C.c_void_p, cfg: hb_layer_config, num_blocks: int, device: int):
        self.handle = handle
        self.device = device
        self.cfg = cfg
        self.num_blocks = num_blocks
        self.row = cfg.n_q_heads * cfg.head_dim             # values of a row of q
        self.kv_row = cfg.n_kv_heads * cfg.head_dim         # values of a row of k or v
        self.block_values = cfg.n_kv_heads * 16 * cfg.head_dim  # values of a block of one pool
        self.n_tokens = 0
        self.pool = hb_kv_pool(0, 0, num_blocks)            # of the call at hand

    def __del__(self):
        try:
            hb_destroy_attention(self)
        except Exception:
            pass


def hb_create_attention(cfg: hb_layer_config, num_blocks: int, stream: Optional[int] = None) -> Attention:
    import torch
    global _bf16
    _bf16 = torch.bfloat16
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    h = C.c_void_p()
    _check(load().hb_create_attention(C.byref(cfg), _int32(num_blocks), C.c_void_p(stream), C.byref(h)))
    return Attention(h, cfg, int(num_blocks), torch.cuda.current_device())


def hb_destroy_attention(attention: Attention) -> None:
    if attention.handle is not None and attention.handle.value:
        load().hb_destroy_attention(attention.handle)
        attention.handle = None


def hb_plan_attention(attention: Attention, requests: Sequence[Tuple[int, int, Iterable[int]]], window: int = 0,
                      sinks: int = 0) -> None:
    """requests: (chunk_len, context_len, block_table) per request, in row order."""
    d, keep = _desc(requests, 0, 0, HB_OUT_BF16)
    _check(load().hb_plan_attention(attention.handle, d.n_requests, d.requests, _int32(window), _int32(sinks)))
    attention.n_tokens = sum(int(r[0]) for r in requests)


def hb_plan_shared_attention(attention: Attention, requests: Sequence[Tuple[int, int, Iterable[int]]],
                             groups: Sequence[Tuple[int, int, int]]) -> None:
    """requests as for hb_plan_attention; groups: (first request, number of requests, prefix_len in tokens)."""
    d, keep = _desc(requests, 0, 0, HB_OUT_BF16)
    g = np.asarray(groups if len(groups) else np.zeros((0, 3), np.int32))
    if g.ndim != 2 or g.shape[1] != 3 or g.dtype.kind not in "iu":
        raise ValueError(f"groups: (first, count, prefix_len) each, not {g.dtype} {g.shape}")
    g = _i32(g)
    _check(load().hb_plan_shared_attention(attention.handle, d.n_requests, d.requests, len(g), g.ctypes.data))
    attention.n_tokens = sum(int(r[0]) for r in requests)


def hb_rope_frequencies(rotary_dim: int, theta: float, factor: Optional[float] = None, low: Optional[float] = None,
                        high: Optional[float] = None, original_context: int = 0) -> np.ndarray:
    """The rotary_dim / 2 frequencies: unscaled, divided by factor, or (low and high given) scaled by parts."""
    if (low is None) != (high is None) or (low is not None and factor is None):
        raise ValueError("scaling by parts: factor, low, high and original_context")
    kind = HB_ROPE_UNSCALED if factor is None else HB_ROPE_LINEAR if low is None else HB_ROPE_BY_PARTS
    s = hb_rope_scaling(kind, _int32(original_context), factor or 0.0, low or 0.0, high or 0.0)
    f = np.zeros(max(1, _int32(rotary_dim) // 2))
    _check(load().hb_rope_frequencies(_int32(rotary_dim), theta, C.byref(s), f.ctypes.data))
    return f[:rotary_dim // 2]


def hb_set_attention_rope(attention: Attention, inv_freq, layout: int = HB_ROPE_HALF, magnitude: float = 1.0) -> None:
    """Rotation of later hb_run_append calls: the first 2 len(inv_freq) dimensions of a head. The latest one
    counts, for a plan that stands too; plans made before the first one cannot append."""
    f = np.ascontiguousarray(inv_freq, dtype=np.float64).reshape(-1)
    _check(load().hb_set_attention_rope(attention.handle, 2 * len(f), _int32(layout), f.ctypes.data, magnitude))


_bf16 = None  # torch.bfloat16, once torch is there


def _rows(name: str, t, n: int, row: int, device: int) -> int:
    """Row stride of n rows of `row` contiguous bf16 values ([n][heads][head_dim] or [n][heads * head_dim])."""
    if t.dtype is not _bf16 or t.get_device() != device:
        raise ValueError(f"{name}: a bf16 tensor on GPU {device}, not {t.dtype} on {t.device}")
    if t.numel() != n * row or t.dim() < 2 or t.size(0) != n:
        raise ValueError(f"{name}: {n} rows of {row} values, not {tuple(t.shape)}")
    if t.is_contiguous():
        return row
    shape, stride = t.shape, t.stride()
    run = 1
    for size, step in zip(shape[:0:-1], stride[:0:-1]):
        if size != 1 and step != run:
            raise ValueError(f"{name}: the values of a row must be contiguous, strides {stride}")
        run *= size
    return stride[0] if n > 1 else row


def _pools(attention: Attention, k_pool, v_pool) -> hb_kv_pool:
    # (written for few calls of few attributes: beside a small launch they are most of the time)
    blocks, device = attention.num_blocks, attention.device
    for p in (k_pool, v_pool):
        if p.dtype is not _bf16 or p.get_device() != device or not p.is_contiguous():
            raise ValueError(f"{'k_pool' if p is k_pool else 'v_pool'}: a contiguous bf16 tensor on GPU {device}")
        have = p.numel()
        if have < blocks * attention.block_values or have % attention.block_values:
            raise ValueError(f"{'k_pool' if p is k_pool else 'v_pool'}: at least {blocks} blocks of "
                             f"{attention.block_values} values, not {tuple(p.shape)}")
    pool = attention.pool
    pool.k_pool, pool.v_pool = k_pool.data_ptr(), v_pool.data_ptr()
    return pool


def hb_run_append(attention: Attention, q, k, v, k_pool, v_pool, q_out) -> None:
    """q, k, v, q_out: bf16 [T][heads][head_dim] (or [T][heads * head_dim]), rows any multiple of 8 elements apart;
    q_out may be q."""
    pool = _pools(attention, k_pool, v_pool)
    n, row, kv_row, device = attention.n_tokens, attention.row, attention.kv_row, attention.device
    status = load().hb_run_append(attention.handle, pool, q.data_ptr(), _rows("q", q, n, row, device),
                                  k.data_ptr(), _rows("k", k, n, kv_row, device),
                                  v.data_ptr(), _rows("v", v, n, kv_row, device),
                                  q_out.data_ptr(), _rows("q_out", q_out, n, row, device))
    if status:
        _check(status)


def hb_run_attention(attention: Attention, q, k_pool, v_pool, out) -> None:
    """q, out: bf16 [T][n_q_heads][head_dim] (or [T][n_q_heads * head_dim]), rows any multiple of 8 elements apart."""
    pool = _pools(attention, k_pool, v_pool)
    n, row, device = attention.n_tokens, attention.row, attention.device
    status = load().hb_run_attention(attention.handle, pool, q.data_ptr(), _rows("q", q, n, row, device),
                                     out.data_ptr(), _rows("out", out, n, row, device))
    if status:
        _check(status)


def _block_pairs(src, dst):
    s, d = _ids(src), _ids(dst)
    if s.ndim != 1 or s.shape != d.shape:
        raise ValueError(f"src and dst: one list of block ids each, of equal length, not {s.shape} and {d.shape}")
    return s, d


def hb_copy_blocks(layer: Layer, src, dst) -> None:
    """Block dst[i] of the layer's pool takes the contents of block src[i]."""
    s, d = _block_pairs(src, dst)
    _check(load().hb_copy_blocks(layer.handle, s.tobytes(), d.tobytes(), len(s)))


def hb_copy_model_blocks(model: Model, src, dst) -> None:
    """hb_copy_blocks in the pools of every layer."""
    s, d = _block_pairs(src, dst)
    _check(load().hb_copy_model_blocks(model.handle, s.tobytes(), d.tobytes(), len(s)))


def hb_plan_compaction(num_blocks: int, tables: Sequence[Iterable[int]]):
    """(tables, src, dst, n_used): the tables over blocks [0, n_used), and the moves that make them true."""
    num_blocks = _int32(num_blocks)
    ts = [_ids(t).reshape(-1).copy() for t in tables]
    ptrs = (C.c_void_p * max(1, len(ts)))(*[t.ctypes.data for t in ts])
    lens = _i32([len(t) for t in ts] or [0])
    src, dst = (np.zeros(max(1, num_blocks // 2), np.int32) for _ in range(2))
    moves, used = C.c_int32(), C.c_int32()
    _check(load().hb_plan_compaction(num_blocks, ptrs, lens.ctypes.data_as(C.POINTER(C.c_int32)), len(ts),
                                     src.ctypes.data, dst.ctypes.data, C.byref(moves), C.byref(used)))
    return ts, src[:moves.value], dst[:moves.value], used.value


def hb_validate_batch(cfg: hb_layer_config, num_blocks: int, requests, x_in_ptr: int, x_out_ptr: int,
                      out_dtype: int = HB_OUT_F32) -> int:
    """Host-only check; returns the status code (no exception)."""
    d, keep = _desc(requests, x_in_ptr, x_out_ptr, out_dtype)
    return load().hb_validate_batch(C.byref(cfg), int(num_blocks), C.byref(d))


def hb_profile(layer: Layer, chunk_sizes: Sequence[int], mixes: Sequence[Tuple[Sequence[int], int]],
               warmup: int = 10, iters: int = 100, seed: int = 0) -> np.ndarray:
    """mixes: (decode_contexts, chunk_context) per row. Returns a structured array [n_mix][n_chunk]."""
    cs = _i32(chunk_sizes)
    ctxs = [_i32(m[0]) for m in mixes]
    marr = (hb_decode_mix * len(mixes))()
    for i, (c, (_, cc)) in enumerate(zip(ctxs, mixes)):
        marr[i] = hb_decode_mix(len(c), c.ctypes.data_as(C.POINTER(C.c_int32)), int(cc))
    out = (hb_profile_cell * (len(mixes) * len(cs)))()
    _check(load().hb_profile(layer.handle, cs.ctypes.data_as(C.POINTER(C.c_int32)), len(cs), marr, len(mixes),
                             int(warmup), int(iters), C.c_uint64(seed), out))
    names = [f[0] for f in hb_profile_cell._fields_]
    res = np.zeros((len(mixes), len(cs)), dtype=[(n, np.float64) for n in names])
    for i in range(len(mixes)):
        for j in range(len(cs)):
            cell = out[i * len(cs) + j]
            res[i, j] = tuple(getattr(cell, n) for n in names)
    return res


def hb_profile_batches(layer: Layer, batches, warmup: int = 3, iters: int = 15) -> np.ndarray:
    """batches: (requests, x_in, x_out) each, requests as for hb_run_iteration.
    Returns a structured array [n_batches] of profile cells."""
    descs = (hb_batch_desc * max(1, len(batches)))()
    keep = []
    for i, (reqs, x_in, x_out) in enumerate(batches):
        import torch
        out_dtype = HB_OUT_F32 if x_out.dtype == torch.float32 else HB_OUT_BF16
        d, k = _desc(reqs, _ptr(x_in), _ptr(x_out), out_dtype)
        descs[i] = d
        keep.append(k)
    out = (hb_profile_cell * max(1, len(batches)))()
    _check(load().hb_profile_batches(layer.handle, descs, len(batches), int(warmup), int(iters), out))
    names = [f[0] for f in hb_profile_cell._fields_]
    res = np.zeros(len(batches), dtype=[(n, np.float64) for n in names])
    for i in range(len(batches)):
        res[i] = tuple(getattr(out[i], n) for n in names)
    return res


def _requests_only(requests: Sequence[Tuple[int, int]]):
    """hb_request array of (chunk_len, context_len) pairs without block tables."""
    arr = (hb_request * max(1, len(requests)))()
    for i, r in enumerate(requests):
        arr[i] = hb_request(_int32(r[0]), _int32(r[1]), None, 0)
    return arr


def _mix_array(mixes: Sequence[Tuple[Sequence[int], int]]):
    ctxs = [_i32(m[0]) for m in mixes]
    marr = (hb_decode_mix * len(mixes))()
    for i, (c, (_, cc)) in enumerate(zip(ctxs, mixes)):
        marr[i] = hb_decode_mix(len(c), c.ctypes.data_as(C.POINTER(C.c_int32)), int(cc))
    return marr, ctxs


def hb_latency_features(cfg: hb_layer_config, requests: Sequence[Tuple[int, int]]) -> np.ndarray:
    """requests: (chunk_len, context_len) per request."""
    f = (C.c_double * HB_LAT_FEATURES)()
    _check(load().hb_latency_features(C.byref(cfg), _requests_only(requests), len(requests), f))
    return np.array(f[:], dtype=np.float64)


def hb_fit_latency_model(cfg: hb_layer_config, chunk_sizes: Sequence[int],
                         mixes: Sequence[Tuple[Sequence[int], int]], median_ms) -> hb_latency_model:
    """median_ms[n_mix][n_chunk]: the cells' medians (hb_profile's "median_ms")."""
    cs = _i32(chunk_sizes)
    marr, keep = _mix_array(mixes)
    med = np.asarray(median_ms, dtype=np.float64).reshape(len(mixes), len(cs))
    cells = (hb_profile_cell * med.size)()
    for i in range(len(mixes)):
        for j in range(len(cs)):
            cells[i * len(cs) + j].median_ms = float(med[i, j])
    model = hb_latency_model()
    _check(load().hb_fit_latency_model(C.byref(cfg), cs.ctypes.data_as(C.POINTER(C.c_int32)), len(cs), marr,
                                       len(mixes), cells, C.byref(model)))
    return model


def hb_predict_latency(model: hb_latency_model, cfg: hb_layer_config, requests: Sequence[Tuple[int, int]]) -> float:
    ms = C.c_double()
    _check(load().hb_predict_latency(C.byref(model), C.byref(cfg), _requests_only(requests), len(requests),
                                     C.byref(ms)))
    return ms.value


def hb_select_chunk(model: hb_latency_model, cfg: hb_layer_config, decode_contexts: Sequence[int],
                    decode_deadlines_ms: Sequence[float], now_ms: float, chunk_context: int, max_chunk: int,
                    granularity: int, margin: float = 0.0) -> Tuple[int, float]:
    ctx = _i32(decode_contexts)
    dl = np.ascontiguousarray(decode_deadlines_ms, dtype=np.float64)
    chunk, ms = C.c_int32(), C.c_double()
    _check(load().hb_select_chunk(C.byref(model), C.byref(cfg), ctx.ctypes.data_as(C.POINTER(C.c_int32)),
                                  dl.ctypes.data_as(C.POINTER(C.c_double)), len(ctx), float(now_ms),
                                  int(chunk_context), int(max_chunk), int(granularity), float(margin),
                                  C.byref(chunk), C.byref(ms)))
    return chunk.value, ms.value


class Sampler:
    """Owns an hb_sampler handle."""

    def __init__(self, handle: C.c_void_p, max_rows: int, vocab: int, device: int):
        import torch
        self.handle = handle
        self.max_rows = max_rows
        self.vocab = vocab
        self.device = device
        self.dtypes = {torch.float32: HB_OUT_F32, torch.bfloat16: HB_OUT_BF16}
        self.f32, self.i32 = torch.float32, torch.int32

    def __del__(self):
        try:
            hb_destroy_sampler(self)
        except Exception:
            pass


def hb_create_sampler(max_rows: int, vocab: int, stream: Optional[int] = None) -> Sampler:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    h = C.c_void_p()
    _check(load().hb_create_sampler(_int32(max_rows), _int32(vocab), C.c_void_p(stream), C.byref(h)))
    return Sampler(h, int(max_rows), int(vocab), torch.cuda.current_device())


def hb_destroy_sampler(sampler: Sampler) -> None:
    if sampler.handle is not None and sampler.handle.value:
        load().hb_destroy_sampler(sampler.handle)
        sampler.handle = None


def hb_sample(sampler: Sampler, logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None,
              probs=None) -> None:
    """logits: fp32 or bf16 [n][vocab], rows any distance apart; the others [n], top_k and tokens int32, the rest fp32."""
    dtype = sampler.dtypes.get(logits.dtype)
    if dtype is None or logits.get_device() != sampler.device:
        raise ValueError(f"logits: an fp32 or bf16 tensor on GPU {sampler.device}, not {logits.dtype} on {logits.device}")
    if logits.dim() != 2 or logits.size(1) != sampler.vocab or (logits.size(1) > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits: rows of {sampler.vocab} contiguous values, not {tuple(logits.shape)}, strides {logits.stride()}")
    n = logits.size(0)

    def row(name, t, want):
        if t is None:
            return 0
        if t.dtype is not want or t.get_device() != sampler.device or t.dim() != 1 or t.size(0) != n or not t.is_contiguous():
            raise ValueError(f"{name}: {n} contiguous values of {want} on GPU {sampler.device}, not {tuple(t.shape)} "
                             f"of {t.dtype} on {t.device}")
        return t.data_ptr()

    f32, i32 = sampler.f32, sampler.i32
    d = hb_sample_desc(n, dtype, logits.data_ptr(), logits.stride(0) if n > 1 else sampler.vocab,
                       row("temperature", temperature, f32), row("top_k", top_k, i32), row("top_p", top_p, f32),
                       row("min_p", min_p, f32), row("u", u, f32), row("tokens", tokens, i32), row("probs", probs, f32))
    status = load().hb_sample(sampler.handle, C.byref(d))
    if status:
        _check(status)


def hb_set_kernel_timing(layer: Layer, kernels) -> None:
    """kernels: True (all), False (none) or an iterable of kernel names."""
    if kernels is True:
        mask = (1 << HB_K_COUNT) - 1
    elif kernels is False or kernels is None:
        mask = 0
    else:
        names = [hb_kernel_name(k) for k in range(HB_K_COUNT)]
        mask = 0
        for n in kernels:
            mask |= 1 << names.index(n)
    _check(load().hb_set_kernel_timing(layer.handle, mask))


def hb_kernel_times(layer: Layer, reset: bool = False) -> Dict[str, Tuple[float, int]]:
    ms = (C.c_double * HB_K_COUNT)()
    n = (C.c_int64 * HB_K_COUNT)()
    _check(load().hb_kernel_times(layer.handle, ms, n, 1 if reset else 0))
    return {hb_kernel_name(k): (ms[k], n[k]) for k in range(HB_K_COUNT)}


def hb_kernel_name(k: int) -> str:
    return load().hb_kernel_name(int(k)).decode()


def hb_gemm_tile_count() -> int:
    return int(load().hb_gemm_tile_count())


def hb_plan_gemms(cfg: hb_layer_config, n_tokens: int, cu_count: int, force_tile: int = -1,
                  force_ksplit: int = 0) -> List[Tuple[int, int]]:
    """(tile, ksplit) of the QKV, O, gate/up and down GEMMs for a batch of n_tokens."""
    t, k = (C.c_int32 * HB_GEMM_COUNT)(), (C.c_int32 * HB_GEMM_COUNT)()
    _check(load().hb_plan_gemms(C.byref(cfg), int(n_tokens), int(cu_count), int(force_tile), int(force_ksplit), t, k))
    return [(t[i], k[i]) for i in range(HB_GEMM_COUNT)]


def hb_layer_gemm_plans(layer: Layer) -> List[Tuple[int, int]]:
    """(tile, ksplit) of each GEMM of the layer's most recent iteration."""
    t, k = (C.c_int32 * HB_GEMM_COUNT)(), (C.c_int32 * HB_GEMM_COUNT)()
    _check(load().hb_layer_gemm_plans(layer.handle, t, k))
    return [(t[i], k[i]) for i in range(HB_GEMM_COUNT)]


def hb_layer_stage(layer: Layer, stage: int) -> Tuple[int, int]:
    p = C.c_void_p()
    s = C.c_int64()
    _check(load().hb_layer_stage(layer.handle, int(stage), C.byref(p), C.byref(s)))
    return int(p.value or 0), int(s.value)


def hb_measure_device_rates(buf, stream=None) -> Dict[str, float]:
    """Sustained random-4-KB read, streaming read and bf16 MFMA rates of the
    current device; buf: a device tensor of at least 1 GiB (scratch)."""
    r = hb_device_rates()
    s = 0 if stream is None else int(stream.cuda_stream)
    _check(load().hb_measure_device_rates(C.c_void_p(buf.data_ptr()), int(buf.numel() * buf.element_size()),
                                          C.c_void_p(s), C.byref(r)))
    return {f[0]: float(getattr(r, f[0])) for f in hb_device_rates._fields_}
