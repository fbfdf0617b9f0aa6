"""ctypes binding of libspts.so (the C boundary declared in include/spts.h).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
PyTorch is used for device memory and streams.  There is no CPU fallback: importing this
module without the built library raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SPTS_LIBRARY") or os.path.join(_PKG, "libspts.so")     # SPTS_LIBRARY: another build of the library

SPTS_BF16, SPTS_FP32 = 0, 1
FORCE_LAST = 1
OPT_REFERENCE_KERNELS = 2
OPT_PAP_WINDOW = 8
OPT_FFN_SCORE_PAP_ONLY = 16
OPT_DEBUG_CHECKS = 32
W4_NORM, W4_FP32_OUT, W4_MAX_N = 1, 2, 32
PAGED_MAX_SEQ, PAGED_MAX_ROWS, PAGE_SIZES = 1024, 1 << 25, (16, 32, 64, 128, 256)
LOGPROBS_MAX_TOP = 32

STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "SHAPE", 3: "WORKSPACE", 4: "CUDA", 5: "TIMEOUT",
                6: "NONFINITE", 7: "UNSUPPORTED", 8: "INDEX"}


class SptsError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: SPTS_ERR_{STATUS_NAMES.get(code, code)}")
        self.code = code


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn_dim",
                                          "ltp_dlow", "ltp_rank", "n_layers", "vocab")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float), ("dtype", C.c_int32)]


WEIGHT_NAMES = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "ug", "vg", "uu", "vu", "vd", "ud")


class LayerWeightsC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_NAMES] + [("prepared", C.c_void_p)]


class KvLayerC(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pos", C.c_void_p), ("len", C.c_int32),
                ("capacity", C.c_int32)]


class LayerPlanC(C.Structure):
    _fields_ = [("m_attn", C.c_int32), ("m_ffn", C.c_int32), ("prune_to", C.c_int32)]


class MsdpStageC(C.Structure):
    _fields_ = [("last_layer", C.c_int32), ("m_attn_fixed", C.c_int32), ("m_ffn_fixed", C.c_int32),
                ("n_next", C.c_int32)]


class W4C(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("params", C.c_void_p), ("out_features", C.c_int32), ("in_features", C.c_int32),
                ("group", C.c_int32)]


class Kv4CacheC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_params", "v_params", "pos", "len")] + \
               [(n, C.c_int32) for n in ("n_seq", "capacity", "group")]


class LayerWeights4C(C.Structure):
    _fields_ = [(n, W4C) for n in ("wqkv", "wo", "w_gate", "w_up", "w_down")]


class ModelWeights4C(C.Structure):
    _fields_ = [("layers", C.POINTER(LayerWeights4C)), ("lm_head", W4C), ("embed", C.c_void_p)]


class PagedKvC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "pos", "weight", "table", "len")] + \
               [(n, C.c_int32) for n in ("n_pages", "page_size", "max_pages", "n_seq")]


LOGITS_RULES = ("history", "history_start", "generated_start", "repetition", "presence", "frequency", "bias_token",
                "bias_value", "bias_start", "mask")


class LogitsRulesC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LOGITS_RULES] + \
               [("ld_mask", C.c_int64), ("n_history", C.c_int32), ("n_bias", C.c_int32)]


class ModelWeightsC(C.Structure):
    _fields_ = [("layers", C.POINTER(LayerWeightsC)), ("lm_head", C.c_void_p), ("embed", C.c_void_p)]


EXPORTS = ("spts_workspace_bytes", "spts_create", "spts_destroy", "spts_set_option",
           "spts_last_device_status", "spts_launch_count", "spts_fold_norm_gain", "spts_pap_score",
           "spts_ltp_score", "spts_topk_select", "spts_layer_prefill_skip", "spts_msdp_compact",
           "spts_first_token", "spts_prefill", "spts_decode_step", "spts_profile_begin", "spts_profile_end",
           "spts_topk_select_static", "spts_proxy_scratch_bytes", "spts_proxy_build",
           "spts_layer_prefill_skip_batch", "spts_msdp_plan", "spts_check_guards", "spts_selftest_wait_timeout",
           "spts_debug_check_index_list", "spts_reduced_attention", "spts_prepared_bytes", "spts_prepare_layer",
           "spts_w4_quantize", "spts_w4_gemv", "spts_kv4_append", "spts_kv4_attention", "spts_process_logits",
           "spts_decode_step4", "spts_paged_append", "spts_paged_attention", "spts_paged_weights", "spts_paged_evict",
           "spts_token_logprobs")

OP_NAMES = {1: "prep", 2: "kproj_pap", 3: "pap_softmax", 4: "topk", 5: "kv_gather", 6: "qv_proj", 7: "attention",
            8: "o_proj", 9: "ltp", 10: "gate_up", 11: "down", 12: "compact", 13: "head", 14: "decode"}
OP_COUNT = 16


def load_library() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2601_13155_b200.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, u32 = C.c_void_p, C.c_int, C.c_uint32
    lib.spts_workspace_bytes.restype = C.c_size_t
    lib.spts_workspace_bytes.argtypes = [C.POINTER(ModelDesc), i32]
    lib.spts_create.argtypes = [C.POINTER(ModelDesc), i32, vp, C.c_size_t, vp, C.POINTER(vp)]
    lib.spts_destroy.argtypes = [vp]
    lib.spts_destroy.restype = None
    lib.spts_set_option.argtypes = [vp, u32, i32]
    lib.spts_last_device_status.argtypes = [vp]
    lib.spts_launch_count.argtypes = [vp]
    lib.spts_launch_count.restype = C.c_int64
    lib.spts_fold_norm_gain.argtypes = [vp, vp, vp, i32, i32]
    lib.spts_pap_score.argtypes = [vp, C.POINTER(LayerWeightsC), vp, vp, i32, vp, vp]
    lib.spts_ltp_score.argtypes = [vp, C.POINTER(LayerWeightsC), vp, vp, i32, vp, vp]
    lib.spts_topk_select.argtypes = [vp, vp, i32, i32, u32, vp]
    lib.spts_topk_select_static.argtypes = [vp, i32, i32, u32, vp, vp]
    lib.spts_proxy_scratch_bytes.restype = C.c_size_t
    lib.spts_proxy_scratch_bytes.argtypes = [C.POINTER(ModelDesc), i32]
    lib.spts_proxy_build.argtypes = [vp, C.POINTER(LayerWeightsC), vp, i32, C.c_double, vp, C.c_size_t, vp, vp,
                                     vp, vp, vp, vp, vp, vp, vp]
    lib.spts_layer_prefill_skip.argtypes = [vp, C.POINTER(LayerWeightsC), vp, vp, i32, i32, i32, u32,
                                            C.POINTER(KvLayerC), vp, vp, vp]
    lib.spts_layer_prefill_skip_batch.argtypes = [vp, C.POINTER(LayerWeightsC), vp, vp, i32, C.POINTER(C.c_int32),
                                                  C.POINTER(C.c_int32), C.POINTER(C.c_int32), u32,
                                                  C.POINTER(KvLayerC), vp, vp, vp]
    lib.spts_msdp_compact.argtypes = [vp, vp, vp, vp, vp, i32, i32, u32, vp, vp, vp, vp]
    lib.spts_msdp_plan.argtypes = [i32, i32, i32, C.POINTER(MsdpStageC), i32, C.POINTER(LayerPlanC),
                                   C.POINTER(C.c_int32), C.POINTER(C.c_int64)]
    lib.spts_check_guards.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.spts_selftest_wait_timeout.argtypes = [vp, u32]
    lib.spts_debug_check_index_list.argtypes = [vp, vp, i32, i32]
    lib.spts_reduced_attention.argtypes = [vp, vp, vp, vp, i32, vp]
    lib.spts_prepared_bytes.restype = C.c_size_t
    lib.spts_prepared_bytes.argtypes = [C.POINTER(ModelDesc)]
    lib.spts_prepare_layer.argtypes = [vp, C.POINTER(LayerWeightsC), vp, C.c_size_t]
    lib.spts_first_token.argtypes = [vp, vp, vp, vp, vp]
    lib.spts_prefill.argtypes = [vp, C.POINTER(ModelWeightsC), C.POINTER(LayerPlanC), vp, vp, vp, vp, vp, vp,
                                 i32, u32, C.POINTER(KvLayerC), C.POINTER(C.c_int32), C.POINTER(C.c_int32), vp]
    lib.spts_decode_step.argtypes = [vp, C.POINTER(ModelWeightsC), C.POINTER(KvLayerC), vp, C.c_int32,
                                     C.c_int32, vp, vp, vp]
    lib.spts_profile_begin.argtypes = [vp, i32]
    lib.spts_profile_end.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(C.c_int64), C.POINTER(C.c_double),
                                     C.POINTER(C.c_double)]
    i64 = C.c_int64
    lib.spts_w4_quantize.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    lib.spts_w4_gemv.argtypes = [vp, C.POINTER(W4C), C.POINTER(W4C), vp, i64, i32, vp, i64, u32, vp, i64]
    lib.spts_kv4_append.argtypes = [vp, C.POINTER(Kv4CacheC), vp, i64, vp, i64, vp, vp, vp, i32, vp, vp]
    lib.spts_kv4_attention.argtypes = [vp, C.POINTER(Kv4CacheC), vp, i64, vp, i64]
    lib.spts_decode_step4.argtypes = [vp, C.POINTER(ModelWeights4C), C.POINTER(Kv4CacheC), vp, vp, vp, C.POINTER(LogitsRulesC),
                                      vp, vp, vp]
    lib.spts_process_logits.argtypes = [vp, vp, i64, i32, i32, C.POINTER(LogitsRulesC), vp, i64, vp]
    paged = C.POINTER(PagedKvC)
    lib.spts_paged_append.argtypes = [vp, paged, vp, i64, vp, i64, vp, vp, vp, i32]
    lib.spts_paged_attention.argtypes = [vp, paged, vp, i64, vp, i32, vp, i64, vp]
    lib.spts_paged_weights.argtypes = [vp, paged, vp, i64, vp, i32, vp, C.c_float]
    lib.spts_paged_evict.argtypes = [vp, paged, vp, i32, i32]
    lib.spts_token_logprobs.argtypes = [vp, vp, i64, i32, i32, vp, i32, vp, vp, vp, vp, vp]
    for n in EXPORTS:
        if n not in ("spts_workspace_bytes", "spts_destroy", "spts_launch_count", "spts_proxy_scratch_bytes",
                     "spts_prepared_bytes"):
            getattr(lib, n).restype = C.c_int
    return lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return C.c_void_p(t.data_ptr())


def torch_dtype(dtype: str):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def to_device(a: np.ndarray, dtype: str, device="cuda:0") -> torch.Tensor:
    """Uploads a float32 array (already rounded to the storage type) as a device tensor."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)
    return t.to(torch_dtype(dtype)).contiguous()


TOPK_STATIC_MAX_N = 8388608
_static_lib = None


def topk_select_static(scores: torch.Tensor, k: int, flags: int = 0, idx_out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """spts_topk_select_static: top-k without a context or a workspace, for callers that cannot allocate
    device memory (the scratch is a fixed array inside the library).  The index buffer is the caller's:
    pass `idx_out` [k] int32 to keep this call itself free of allocations."""
    global _static_lib
    if _static_lib is None:
        _static_lib = load_library()
    N = scores.shape[0]
    if idx_out is None:
        idx_out = torch.empty(max(k, 1), dtype=torch.int32, device=scores.device)
    st = stream if stream is not None else torch.cuda.current_stream(scores.device)
    with torch.cuda.device(scores.device):
        code = _static_lib.spts_topk_select_static(_ptr(scores), N, k, flags, _ptr(idx_out), C.c_void_p(st.cuda_stream))
    if code != 0:
        raise SptsError(code, "spts_topk_select_static")
    return idx_out


class LayerWeights:
    """Device copies of one layer's matrices plus the C struct that points at them."""

    def __init__(self, arrays: Dict[str, np.ndarray], dtype: str, device="cuda:0"):
        self.t = {n: to_device(arrays[n], dtype, device) for n in WEIGHT_NAMES}
        self.c = LayerWeightsC(**{n: self.t[n].data_ptr() for n in WEIGHT_NAMES})
        self.prepared = None

    @classmethod
    def from_tensors(cls, tensors: Dict[str, torch.Tensor]) -> "LayerWeights":
        """Wraps device tensors that already hold the matrices in the storage type (no copy)."""
        w = cls.__new__(cls)
        w.t = tensors
        w.c = LayerWeightsC(**{n: tensors[n].data_ptr() for n in WEIGHT_NAMES})
        w.prepared = None
        return w


class KvCache:
    """Per-layer caches [capacity, Hkv, d] (K after RoPE), original positions and lengths."""

    def __init__(self, shape, n_layers: int, capacity, device="cuda:0"):
        caps = list(capacity) if hasattr(capacity, "__len__") else [capacity] * n_layers
        dt = torch_dtype(shape.dtype)
        self.k = [torch.zeros(c, shape.n_kv_heads, shape.head_dim, dtype=dt, device=device) for c in caps]
        self.v = [torch.zeros(c, shape.n_kv_heads, shape.head_dim, dtype=dt, device=device) for c in caps]
        self.pos = [torch.zeros(c, dtype=torch.int32, device=device) for c in caps]
        self.c = (KvLayerC * n_layers)()
        for l in range(n_layers):
            self.c[l] = KvLayerC(self.k[l].data_ptr(), self.v[l].data_ptr(), self.pos[l].data_ptr(), 0, caps[l])

    def length(self, l: int) -> int:
        return int(self.c[l].len)

    def reset(self):
        for e in self.c:
            e.len = 0


def _rows(t: torch.Tensor, width: int, dtype, what: str, dev: int):
    """Address and row stride of a [n, ...] tensor whose rows of `width` elements are contiguous (a view into wider
    rows is fine)."""
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{what}: a tensor of {dtype} on cuda:{dev} is needed, got {t.dtype} on {t.device}")
    shape = t.shape
    if len(shape) == 2 and shape[1] == width and t.stride(1) == 1:
        return t.data_ptr(), (t.stride(0) if shape[0] > 1 else width)
    if len(shape) == 3 and shape[1] * shape[2] == width and t.is_contiguous():
        return t.data_ptr(), width
    if len(shape) < 2 or math.prod(shape[1:]) != width:
        raise ValueError(f"{what}: rows of {width} elements are needed, got {tuple(shape)}")
    inner = 1
    for size, stride in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != inner:
            raise ValueError(f"{what}: the elements of a row must be contiguous")
        inner *= size
    return t.data_ptr(), (t.stride(0) if shape[0] > 1 else width)


def _vec(t: Optional[torch.Tensor], n: Optional[int], dtype, what: str, dev: Optional[int] = None):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous() or t.dtype is not dtype or (n is not None and t.numel() != n):
        raise ValueError(f"{what}: a contiguous CUDA tensor of {dtype}" + (f" with {n} elements" if n is not None else "") + " is needed")
    if dev is not None and t.get_device() != dev:
        raise ValueError(f"{what}: on {t.device}, cuda:{dev} is needed")
    return t.data_ptr()


class W4Weight:
    """A weight matrix [out, in] in 4 bits: codes uint8 [out, in / 2], params bf16 [out, in / group, 2] = (scale, mid)."""

    def __init__(self, codes: torch.Tensor, params: torch.Tensor):
        if codes.dim() != 2 or params.dim() != 3 or params.shape[0] != codes.shape[0] or params.shape[2] != 2 or params.shape[1] < 1:
            raise ValueError(f"codes [out, in / 2] and params [out, in / group, 2] are needed, got {tuple(codes.shape)}, {tuple(params.shape)}")
        _vec(codes, None, torch.uint8, "codes")
        _vec(params, None, torch.bfloat16, "params", codes.get_device())
        self.codes, self.params = codes, params
        self.out_features, self.in_features = codes.shape[0], 2 * codes.shape[1]
        if self.in_features % params.shape[1] != 0:
            raise ValueError("params do not divide the rows into equal groups")
        self.group = self.in_features // params.shape[1]
        self.device_index = codes.get_device()
        self.c = W4C(codes.data_ptr(), params.data_ptr(), self.out_features, self.in_features, self.group)


class Kv4Cache:
    """One layer's 4-bit cache of n_seq sequences (layouts in include/spts.h).  `length` is a device int32 [n_seq]; the
    capacity is rounded up to a multiple of 32.  Existing buffers can be handed in."""

    def __init__(self, shape, n_seq: int, capacity: int, group: int = 64, device="cuda:0", k_codes=None, v_codes=None,
                 k_params=None, v_params=None, length=None, pos=None, positions: bool = False):
        cap = (capacity + 31) // 32 * 32
        hkv, d = shape.n_kv_heads, shape.head_dim
        if group not in (32, 64, 128) or group > d:
            raise ValueError(f"groups of 32, 64 or 128 within {d} dims, got {group}")

        def buf(t, size, dtype, what):
            if t is None:
                return torch.zeros(size, dtype=dtype, device=device)
            _vec(t, None, dtype, what)
            if tuple(t.shape) != size:
                raise ValueError(f"{what}: {size} is needed, got {tuple(t.shape)}")
            return t
        self.k_codes = buf(k_codes, (n_seq, hkv, cap, d // 2), torch.uint8, "k_codes")
        self.v_codes = buf(v_codes, (n_seq, hkv, cap, d // 2), torch.uint8, "v_codes")
        self.k_params = buf(k_params, (n_seq, hkv, cap, d // group, 2), torch.bfloat16, "k_params")
        self.v_params = buf(v_params, (n_seq, hkv, cap, d // group, 2), torch.bfloat16, "v_params")
        self.length = buf(length, (n_seq,), torch.int32, "length")
        self.pos = buf(pos, (n_seq, cap), torch.int32, "pos") if pos is not None or positions else None
        for t in (self.v_codes, self.k_params, self.v_params, self.length) + ((self.pos,) if self.pos is not None else ()):
            if t.device != self.k_codes.device:
                raise ValueError("the buffers of a cache are on one device")
        self.n_seq, self.capacity, self.group = n_seq, cap, group
        self.heads, self.device_index = (hkv, d), self.k_codes.get_device()
        self.c = Kv4CacheC(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_params.data_ptr(),
                           self.v_params.data_ptr(), self.pos.data_ptr() if self.pos is not None else None,
                           self.length.data_ptr(), n_seq, cap, group)


class PagedKv:
    """One layer's paged cache in the storage type (spts_paged_kv): row j of sequence b lies in page table[b, j // page_size].
    `table` is device int32 [n_seq, max_pages], `length` device int32 [n_seq].  Existing buffers can be handed in; k and v are made with
    n_pages pages where they are not, positions and weights where they are asked for."""

    def __init__(self, shape, table: torch.Tensor, page_size: int = 64, n_pages: Optional[int] = None, length=None, k=None, v=None, pos=None,
                 weight=None, positions: bool = False, weights: bool = False):
        if page_size not in PAGE_SIZES:
            raise ValueError(f"pages of {PAGE_SIZES} rows, got {page_size}")
        _vec(table, None, torch.int32, "table")
        if table.dim() != 2 or table.shape[0] > PAGED_MAX_SEQ or not 1 <= table.shape[1] <= PAGED_MAX_ROWS // page_size:
            raise ValueError(f"table: [up to {PAGED_MAX_SEQ}, 1 to {PAGED_MAX_ROWS // page_size}] is needed, got {tuple(table.shape)}")
        device, dev = table.device, table.get_device()
        n_seq, max_pages = table.shape
        hkv, d = shape.n_kv_heads, shape.head_dim
        if k is not None:
            n_pages = k.shape[0]
        if not n_pages or n_pages < 1:
            raise ValueError("n_pages is needed where k is not given")

        def buf(t, size, dtype, what):
            if t is None:
                return torch.zeros(size, dtype=dtype, device=device)
            _vec(t, None, dtype, what, dev)
            if tuple(t.shape) != size:
                raise ValueError(f"{what}: {size} is needed, got {tuple(t.shape)}")
            return t
        dt = torch_dtype(shape.dtype)
        self.k = buf(k, (n_pages, page_size, hkv, d), dt, "k")
        self.v = buf(v, (n_pages, page_size, hkv, d), dt, "v")
        self.length = buf(length, (n_seq,), torch.int32, "length")
        self.pos = buf(pos, (n_pages, page_size), torch.int32, "pos") if pos is not None or positions else None
        self.weight = buf(weight, (n_pages, page_size), torch.float32, "weight") if weight is not None or weights else None
        self.table, self.n_seq, self.n_pages, self.page_size, self.max_pages = table, n_seq, n_pages, page_size, max_pages
        self.heads, self.dtype, self.device_index = (hkv, d), dt, dev
        ptr = lambda t: t.data_ptr() if t is not None else None
        self.c = PagedKvC(ptr(self.k), ptr(self.v), ptr(self.pos), ptr(self.weight), ptr(table), ptr(self.length), n_pages, page_size,
                          max_pages, n_seq)


class LogitsRules:
    """The device lists of spts_logits_rules; every one is optional."""

    def __init__(self, history=None, history_start=None, generated_start=None, repetition=None, presence=None, frequency=None,
                 bias_token=None, bias_value=None, bias_start=None, mask=None):
        i32, f32 = torch.int32, torch.float32
        given = dict(history=(history, i32), history_start=(history_start, i32), generated_start=(generated_start, i32),
                     repetition=(repetition, f32), presence=(presence, f32), frequency=(frequency, f32),
                     bias_token=(bias_token, i32), bias_value=(bias_value, f32), bias_start=(bias_start, i32))
        self.t = {}
        for name, (t, dtype) in given.items():
            _vec(t, None, dtype, name)
            self.t[name] = t
        if mask is not None and (mask.dim() != 2 or mask.dtype != i32 or not mask.is_cuda or mask.stride(1) != 1):
            raise ValueError("mask: a CUDA int32 tensor [n, words] is needed")
        if (history is None) != (history_start is None) or len({t is None for t in (bias_token, bias_value, bias_start)}) > 1:
            raise ValueError("a history needs its history_start; biases need bias_token, bias_value and bias_start")
        if bias_token is not None and bias_token.numel() != bias_value.numel():
            raise ValueError("as many bias tokens as values are needed")
        self.t["mask"] = mask
        self.c = LogitsRulesC(*[self.t[n].data_ptr() if self.t[n] is not None else None for n in LOGITS_RULES],
                              mask.stride(0) if mask is not None else 0, history.numel() if history is not None else 0,
                              bias_token.numel() if bias_token is not None else 0)

        self.sizes = [(name, t.numel(), 1 if name.endswith("_start") and name != "generated_start" else 0) for name, t in self.t.items()
                      if t is not None and name in ("history_start", "generated_start", "repetition", "presence", "frequency", "bias_start")]
        self.devices = {t.get_device() for t in self.t.values() if t is not None}

    def check(self, n: int, vocab: int, dev: int):
        for name, size, more in self.sizes:
            if size != n + more:
                raise ValueError(f"{name}: {n + more} entries are needed for {n} rows, got {size}")
        m = self.t["mask"]
        if m is not None and (m.shape[0] != n or m.shape[1] < (vocab + 31) // 32):
            raise ValueError(f"mask: [{n}, {(vocab + 31) // 32}] words are needed, got {tuple(m.shape)}")
        if self.devices - {dev}:
            raise ValueError(f"the rules' tensors are on cuda:{self.devices}, the context is on cuda:{dev}")


class Spts:
    """One library context bound to a device and a stream.  Calls run on that stream: a caller whose tensors are made or read on
    another one orders the two (wait_stream)."""

    def __init__(self, shape, max_seq: int, device="cuda:0", stream: Optional[torch.cuda.Stream] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("the SPTS library needs a CUDA device (no CPU fallback)")
        self.lib = load_library()
        self.shape = shape
        self.device = torch.device(device)
        self.dtype = torch_dtype(shape.dtype)
        self.desc = ModelDesc(shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn_dim,
                              shape.ltp_dlow, shape.ltp_rank, shape.n_layers, shape.vocab, shape.rms_eps,
                              shape.rope_theta, SPTS_BF16 if shape.dtype == "bf16" else SPTS_FP32)
        torch.cuda.set_device(self.device)
        self.dev = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        nbytes = self.lib.spts_workspace_bytes(C.byref(self.desc), max_seq)
        if nbytes == 0:
            raise SptsError(2, "spts_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.max_seq = max_seq
        h = C.c_void_p()
        self._check(self.lib.spts_create(C.byref(self.desc), max_seq, _ptr(self.workspace), nbytes,
                                         C.c_void_p(self.stream.cuda_stream), C.byref(h)), "spts_create")
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.spts_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, code: int, where: str):
        if code != 0:
            raise SptsError(code, where)

    # ------------------------------------------------------------------ options / status
    def set_reference_kernels(self, on: bool):
        self._check(self.lib.spts_set_option(self.h, OPT_REFERENCE_KERNELS, 1 if on else 0), "spts_set_option")

    def set_pap_window(self, window: int):
        self._check(self.lib.spts_set_option(self.h, OPT_PAP_WINDOW, int(window)), "spts_set_option")

    def set_ffn_score_pap_only(self, on: bool):
        """T_f = TopK(S_mha, m_ffn): the FFN criterion without the proxy network (Table 4's baseline row)."""
        self._check(self.lib.spts_set_option(self.h, OPT_FFN_SCORE_PAP_ONLY, 1 if on else 0), "spts_set_option")

    def set_debug_checks(self, on: bool):
        """Every selected index list is checked on the device (range, strictly ascending); SPTS_ERR_INDEX otherwise."""
        self._check(self.lib.spts_set_option(self.h, OPT_DEBUG_CHECKS, 1 if on else 0), "spts_set_option")

    def check_guards(self) -> int:
        """Number of guard bands between the workspace slices that no longer hold their pattern (0 = intact)."""
        n = C.c_int32(-1)
        self._check(self.lib.spts_check_guards(self.h, C.byref(n)), "spts_check_guards")
        return int(n.value)

    def debug_check_index_list(self, idx, N: int):
        self._check(self.lib.spts_debug_check_index_list(self.h, _ptr(idx), idx.shape[0], N), "spts_debug_check_index_list")

    def selftest_wait_timeout(self, limit_us: int = 1000):
        self._check(self.lib.spts_selftest_wait_timeout(self.h, int(limit_us)), "spts_selftest_wait_timeout")

    def device_status(self) -> int:
        return int(self.lib.spts_last_device_status(self.h))

    def launch_count(self) -> int:
        return int(self.lib.spts_launch_count(self.h))

    def fold_norm_gain(self, W: torch.Tensor, g: torch.Tensor):
        self._check(self.lib.spts_fold_norm_gain(self.h, _ptr(W), _ptr(g), W.shape[0], W.shape[1]),
                    "spts_fold_norm_gain")

    def profile_begin(self, op: int = -1):
        self._check(self.lib.spts_profile_begin(self.h, op), "spts_profile_begin")

    def profile_end(self):
        """Returns {op name: {"ms", "calls", "flops", "bytes"}} for the operations timed since profile_begin."""
        ms = (C.c_float * OP_COUNT)()
        calls = (C.c_int64 * OP_COUNT)()
        fl = (C.c_double * OP_COUNT)()
        by = (C.c_double * OP_COUNT)()
        self._check(self.lib.spts_profile_end(self.h, ms, calls, fl, by), "spts_profile_end")
        return {OP_NAMES[i]: {"ms": float(ms[i]), "calls": int(calls[i]), "flops": float(fl[i]), "bytes": float(by[i])}
                for i in OP_NAMES if calls[i] > 0}

    # ------------------------------------------------------------------ the six calls
    def pap_score(self, w: LayerWeights, X, pos, K_out=None, S_out=None):
        N = X.shape[0]
        if S_out is None:
            S_out = torch.empty(N, dtype=torch.float32, device=self.device)
        self._check(self.lib.spts_pap_score(self.h, C.byref(w.c), _ptr(X), _ptr(pos), N, _ptr(K_out), _ptr(S_out)),
                    "spts_pap_score")
        return S_out

    def ltp_score(self, w: LayerWeights, X, S_mha, C_out=None, S_out=None):
        N = X.shape[0]
        if S_out is None:
            S_out = torch.empty(N, dtype=torch.float32, device=self.device)
        self._check(self.lib.spts_ltp_score(self.h, C.byref(w.c), _ptr(X), _ptr(S_mha), N, _ptr(C_out), _ptr(S_out)),
                    "spts_ltp_score")
        return S_out

    def topk_select(self, scores, k: int, flags: int = 0, idx_out=None):
        N = scores.shape[0]
        if idx_out is None:
            idx_out = torch.empty(max(k, 1), dtype=torch.int32, device=self.device)
        self._check(self.lib.spts_topk_select(self.h, _ptr(scores), N, k, flags, _ptr(idx_out)), "spts_topk_select")
        return idx_out

    def layer_prefill_skip(self, w: LayerWeights, X, pos, m_attn: int, m_ffn: int, cache: KvCache, layer: int = 0,
                           flags: int = FORCE_LAST, S_out=None, idx_attn_out=None, idx_ffn_out=None):
        N = X.shape[0]
        self._check(self.lib.spts_layer_prefill_skip(self.h, C.byref(w.c), _ptr(X), _ptr(pos), N, m_attn, m_ffn,
                                                     flags, C.byref(cache.c[layer]), _ptr(S_out),
                                                     _ptr(idx_attn_out), _ptr(idx_ffn_out)),
                    "spts_layer_prefill_skip")

    def prepare_layer(self, w: "LayerWeights"):
        """spts_prepare_layer: repacks the layer's proxy factors once into a buffer the weights object then owns;
        later calls with `w` skip the per-call repacking.  Redo after changing ug / uu / vg / vu / ud."""
        nbytes = self.lib.spts_prepared_bytes(C.byref(self.desc))
        buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        w.c.prepared = None
        self._check(self.lib.spts_prepare_layer(self.h, C.byref(w.c), _ptr(buf), nbytes), "spts_prepare_layer")
        w.prepared = buf
        w.c.prepared = buf.data_ptr()
        return w

    def reduced_attention(self, Q, K, V, O_out=None):
        """spts_reduced_attention: causal GQA attention among the m rows of Q [m,H,d], K, V [m,Hkv,d] -> [m, H*d]."""
        m = Q.shape[0]
        if O_out is None:
            O_out = torch.empty(m, self.shape.n_q_heads * self.shape.head_dim, dtype=self.dtype, device=self.device)
        self._check(self.lib.spts_reduced_attention(self.h, _ptr(Q), _ptr(K), _ptr(V), m, _ptr(O_out)),
                    "spts_reduced_attention")
        return O_out

    def layer_prefill_skip_batch(self, w: LayerWeights, X, pos, seq_start, m_attn, m_ffn, caches: KvCache,
                                 flags: int = FORCE_LAST, S_out=None, idx_attn_out=None, idx_ffn_out=None):
        """Several prompts packed into X; `caches` holds one entry per sequence (a KvCache built with
        n_layers = number of sequences); seq_start, m_attn, m_ffn are host integer lists."""
        n_seq = len(m_attn)
        arr = lambda v: (C.c_int32 * len(v))(*[int(x) for x in v])
        self._check(self.lib.spts_layer_prefill_skip_batch(self.h, C.byref(w.c), _ptr(X), _ptr(pos), n_seq,
                                                           arr(seq_start), arr(m_attn), arr(m_ffn), flags, caches.c,
                                                           _ptr(S_out), _ptr(idx_attn_out), _ptr(idx_ffn_out)),
                    "spts_layer_prefill_skip_batch")

    def msdp_compact(self, X_in, pos_in, orig_in, S_mha, n_next: int, X_out, pos_out, orig_out, idx_out=None,
                     flags: int = FORCE_LAST):
        N = X_in.shape[0]
        self._check(self.lib.spts_msdp_compact(self.h, _ptr(X_in), _ptr(pos_in), _ptr(orig_in), _ptr(S_mha), N,
                                               n_next, flags, _ptr(X_out), _ptr(pos_out), _ptr(orig_out),
                                               _ptr(idx_out)), "spts_msdp_compact")

    def proxy_build(self, w: LayerWeights, calib, rho: float = 0.2, want_sigma: bool = False):
        """spts_proxy_build: returns {"importance", "channels", "ug", "vg", "uu", "vu", "vd", "ud"[, "sigma"]} as
        device tensors (the factors in the storage type and the layouts LayerWeights uses)."""
        s = self.shape
        n_cal = calib.shape[0]
        nbytes = self.lib.spts_proxy_scratch_bytes(C.byref(self.desc), n_cal)
        if nbytes == 0:
            raise SptsError(2, "spts_proxy_scratch_bytes")
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        dt, dv = self.dtype, self.device
        out = {"importance": torch.empty(s.ffn_dim, dtype=torch.float32, device=dv),
               "channels": torch.empty(s.ltp_dlow, dtype=torch.int32, device=dv),
               "ug": torch.empty(s.ltp_rank, s.hidden, dtype=dt, device=dv),
               "vg": torch.empty(s.ltp_dlow, s.ltp_rank, dtype=dt, device=dv),
               "uu": torch.empty(s.ltp_rank, s.hidden, dtype=dt, device=dv),
               "vu": torch.empty(s.ltp_dlow, s.ltp_rank, dtype=dt, device=dv),
               "vd": torch.empty(s.ltp_rank, s.ltp_dlow, dtype=dt, device=dv),
               "ud": torch.empty(s.hidden, s.ltp_rank, dtype=dt, device=dv)}
        if want_sigma:
            out["sigma"] = torch.empty(3, s.ltp_dlow, dtype=torch.float32, device=dv)
        self._check(self.lib.spts_proxy_build(self.h, C.byref(w.c), _ptr(calib), n_cal, float(rho), _ptr(scratch), nbytes,
                                              _ptr(out["importance"]), _ptr(out["channels"]), _ptr(out["ug"]),
                                              _ptr(out["vg"]), _ptr(out["uu"]), _ptr(out["vu"]), _ptr(out["vd"]),
                                              _ptr(out["ud"]), _ptr(out.get("sigma"))), "spts_proxy_build")
        self.stream.synchronize()                                  # scratch is released on return
        return out

    def first_token(self, x_row, lm_head, logits_out=None, token_out=None):
        self._check(self.lib.spts_first_token(self.h, _ptr(x_row), _ptr(lm_head), _ptr(logits_out), _ptr(token_out)),
                    "spts_first_token")

    def prefill(self, model: "Model", plan: Sequence[Sequence[int]], X, pos, orig, X_alt, pos_alt, orig_alt,
                cache: KvCache, token_out=None, flags: int = FORCE_LAST, n_tokens: Optional[int] = None):
        """Algorithm 1 over all layers.  Returns (n_final, result_is_in_alt)."""
        L = self.shape.n_layers
        cplan = (LayerPlanC * L)(*[LayerPlanC(int(a), int(b), int(c or 0)) for a, b, c in plan])
        nf, ia = C.c_int32(0), C.c_int32(0)
        N = X.shape[0] if n_tokens is None else n_tokens
        self._check(self.lib.spts_prefill(self.h, C.byref(model.c), cplan, _ptr(X), _ptr(pos), _ptr(orig),
                                          _ptr(X_alt), _ptr(pos_alt), _ptr(orig_alt), N, flags, cache.c,
                                          C.byref(nf), C.byref(ia), _ptr(token_out)), "spts_prefill")
        return nf.value, bool(ia.value)

    def decode_step(self, model: "Model", cache: KvCache, pos: int, x_in=None, token_in: int = 0, x_out=None,
                    logits_out=None, token_out=None):
        self._check(self.lib.spts_decode_step(self.h, C.byref(model.c), cache.c, _ptr(x_in), token_in, pos,
                                              _ptr(x_out), _ptr(logits_out), _ptr(token_out)), "spts_decode_step")

    # ------------------------------------------------------------------ generation with 4-bit weights and caches
    def w4_quantize(self, W: torch.Tensor, group: int = 128) -> W4Weight:
        """spts_w4_quantize: the 4-bit form of W [out, in] (storage type)."""
        out, k = W.shape
        if group not in (32, 64, 128) or k % group:
            raise ValueError(f"groups of 32, 64 or 128 that divide {k} are needed, got {group}")
        codes = torch.empty(out, k // 2, dtype=torch.uint8, device=self.device)
        params = torch.empty(out, k // group, 2, dtype=torch.bfloat16, device=self.device)
        self._check(self.lib.spts_w4_quantize(self.h, _vec(W, out * k, self.dtype, "W", self.dev), out, k, group, _ptr(codes),
                                              _ptr(params)), "spts_w4_quantize")
        return W4Weight(codes, params)

    def w4_gemv(self, w: W4Weight, X: torch.Tensor, w2: Optional[W4Weight] = None, norm: bool = False, residual=None,
                fp32_out: bool = False, out=None):
        """spts_w4_gemv: X [n, in] W^T for up to 32 tokens; w2: silu(X W^T) * (X W2^T); residual is added."""
        n, width, dev = X.shape[0], w.out_features, self.dev
        odt = torch.float32 if fp32_out else self.dtype
        if out is None:
            out = torch.empty((n, width), dtype=odt, device=self.device)
        if w.device_index != dev or (w2 is not None and w2.device_index != dev):
            raise ValueError(f"the weights are not on cuda:{dev}")
        xp, ldx = _rows(X, w.in_features, self.dtype, "X", dev)
        yp, ldy = _rows(out, width, odt, "out", dev)
        rp, ldr = (None, 0) if residual is None else _rows(residual, width, self.dtype, "residual", dev)
        if out.shape[0] != n or (residual is not None and residual.shape[0] != n):
            raise ValueError("X, residual and out have the same number of rows")
        code = self.lib.spts_w4_gemv(self.h, w.c, w2.c if w2 is not None else None, xp, ldx, n, rp, ldr,
                                     (W4_NORM if norm else 0) | (W4_FP32_OUT if fp32_out else 0), yp, ldy)
        if code:
            raise SptsError(code, "spts_w4_gemv")
        return out

    def _kv4_shape(self, cache: Kv4Cache):
        if cache.heads != (self.shape.n_kv_heads, self.shape.head_dim):
            raise ValueError("the cache was made for other heads than this context's")
        if cache.device_index != self.dev:
            raise ValueError(f"the cache is not on cuda:{self.dev}")

    def kv4_append(self, cache: Kv4Cache, K: torch.Tensor, V: torch.Tensor, pos=None, row_start=None, at=None, K_out=None,
                   V_out=None):
        """spts_kv4_append: rows of K, V [n, Hkv, d] (K after RoPE) into the cache; row_start [n_seq + 1] and at [n_seq]
        are device int32.  K_out, V_out: the values that the cache then stands for."""
        n, w, dev = K.shape[0], self.shape.n_kv_heads * self.shape.head_dim, self.dev
        self._kv4_shape(cache)
        if V.shape[0] != n:
            raise ValueError("as many rows of V as of K are needed")
        kp, ldk = _rows(K, w, self.dtype, "K", dev)
        vp, ldv = _rows(V, w, self.dtype, "V", dev)
        i32 = torch.int32
        code = self.lib.spts_kv4_append(self.h, cache.c, kp, ldk, vp, ldv, _vec(pos, n, i32, "pos", dev),
                                        _vec(row_start, cache.n_seq + 1, i32, "row_start", dev), _vec(at, cache.n_seq, i32, "at", dev),
                                        n, _vec(K_out, n * w, self.dtype, "K_out", dev), _vec(V_out, n * w, self.dtype, "V_out", dev))
        if code:
            raise SptsError(code, "spts_kv4_append")

    def kv4_attention(self, cache: Kv4Cache, Q: torch.Tensor, O_out=None):
        """spts_kv4_attention: one query per sequence, Q [n_seq, H, d] (or [n_seq, H * d]) -> [n_seq, H * d]."""
        n, w = cache.n_seq, self.shape.n_q_heads * self.shape.head_dim
        self._kv4_shape(cache)
        if O_out is None:
            O_out = torch.empty((n, w), dtype=self.dtype, device=self.device)
        if Q.shape[0] != n or O_out.shape[0] != n:
            raise ValueError(f"one query per sequence of the cache: {n} rows are needed")
        qp, ldq = _rows(Q, w, self.dtype, "Q", self.dev)
        op, ldo = _rows(O_out, w, self.dtype, "O_out", self.dev)
        code = self.lib.spts_kv4_attention(self.h, cache.c, qp, ldq, op, ldo)
        if code:
            raise SptsError(code, "spts_kv4_attention")
        return O_out

    def process_logits(self, logits: torch.Tensor, rules: LogitsRules, out=None, token_out=None, want_logits: bool = True):
        """spts_process_logits: (logits under the rules, token).  out may be the logits themselves; with
        want_logits=False only the token is computed."""
        n, v = logits.shape
        rules.check(n, v, self.dev)
        if out is None and want_logits:
            out = torch.empty((n, v), dtype=torch.float32, device=self.device)
        if token_out is None:
            token_out = torch.empty(n, dtype=torch.int32, device=self.device)
        lp, ld = _rows(logits, v, torch.float32, "logits", self.dev)
        op, ldo = (None, 0) if out is None else _rows(out, v, torch.float32, "out", self.dev)
        if out is not None and out.shape[0] != n:
            raise ValueError("as many rows of out as of logits are needed")
        code = self.lib.spts_process_logits(self.h, lp, ld, n, v, rules.c, op, ldo, _vec(token_out, n, torch.int32, "token_out", self.dev))
        if code:
            raise SptsError(code, "spts_process_logits")
        return out, token_out

    def quantize_layer4(self, tensors: Dict[str, torch.Tensor], group: int = 128) -> Dict[str, W4Weight]:
        """The 4-bit form of one layer's matrices (wq, wk, wv, wo, w_gate, w_up, w_down in the storage type)."""
        # the stacked matrix is made here, so only here can its making be ordered before the kernels that read it
        self.stream.wait_stream(torch.cuda.current_stream(self.device))
        with torch.cuda.stream(self.stream):
            qkv = torch.cat([tensors["wq"], tensors["wk"], tensors["wv"]], 0).contiguous()
            out = {"wqkv": self.w4_quantize(qkv, group)}
            for name in ("wo", "w_gate", "w_up", "w_down"):
                out[name] = self.w4_quantize(tensors[name], group)
        self.stream.synchronize()                                  # qkv is released on return, and the codes are for any stream
        return out

    def decode_step4(self, model: "Model4", caches: "Kv4Caches", pos, x_in=None, token_in=None, rules: Optional[LogitsRules] = None,
                     x_out=None, logits_out=None, token_out=None):
        """spts_decode_step4: one token for every sequence of the caches; pos, token_in, token_out are device int32 [n_seq]."""
        n, s, dev, i32 = caches.n_seq, self.shape, self.dev, torch.int32
        if len(model.layers) != s.n_layers or len(caches.layers) != s.n_layers:
            raise ValueError(f"{s.n_layers} layers of weights and caches are needed")
        for cache in caches.layers:
            self._kv4_shape(cache)
        if model.devices - {dev}:
            raise ValueError(f"the weights are on cuda:{model.devices}, the context is on cuda:{dev}")
        table = model.embed
        if x_in is None and table is not None and (table.dtype is not self.dtype or table.get_device() != dev or table.shape[0] < s.vocab or
                                                   table.shape[1] != s.hidden):
            raise ValueError(f"embed: a {self.dtype} table [{s.vocab}, {s.hidden}] on cuda:{dev} is needed, got {table.dtype} "
                             f"{tuple(table.shape)} on {table.device}")
        if rules is not None:
            rules.check(n, s.vocab, dev)
        code = self.lib.spts_decode_step4(self.h, model.c, caches.c, _vec(x_in, n * s.hidden, self.dtype, "x_in", dev),
                                          _vec(token_in, n, i32, "token_in", dev), _vec(pos, n, i32, "pos", dev),
                                          rules.c if rules is not None else None, _vec(x_out, n * s.hidden, self.dtype, "x_out", dev),
                                          _vec(logits_out, n * s.vocab, torch.float32, "logits_out", dev),
                                          _vec(token_out, n, i32, "token_out", dev))
        if code:
            raise SptsError(code, "spts_decode_step4")


    # ------------------------------------------------------------------ serving over a paged cache
    def _paged_shape(self, cache: PagedKv):
        if cache.heads != (self.shape.n_kv_heads, self.shape.head_dim) or cache.dtype is not self.dtype:
            raise ValueError("the cache was made for other heads or another storage type than this context's")
        if cache.device_index != self.dev:
            raise ValueError(f"the cache is not on cuda:{self.dev}")

    def paged_append(self, cache: PagedKv, K: torch.Tensor, V: torch.Tensor, pos=None, row_start=None, at=None):
        """spts_paged_append: rows of K, V [n, Hkv, d] (K after RoPE) become rows of the cache; row_start [n_seq + 1] and at [n_seq]
        are device int32."""
        n, w, dev, i32 = K.shape[0], self.shape.n_kv_heads * self.shape.head_dim, self.dev, torch.int32
        self._paged_shape(cache)
        if V.shape[0] != n:
            raise ValueError("as many rows of V as of K are needed")
        kp, ldk = _rows(K, w, self.dtype, "K", dev)
        vp, ldv = _rows(V, w, self.dtype, "V", dev)
        code = self.lib.spts_paged_append(self.h, cache.c, kp, ldk, vp, ldv, _vec(pos, n, i32, "pos", dev),
                                          _vec(row_start, cache.n_seq + 1, i32, "row_start", dev), _vec(at, cache.n_seq, i32, "at", dev), n)
        if code:
            raise SptsError(code, "spts_paged_append")

    def paged_attention(self, cache: PagedKv, Q: torch.Tensor, row_start=None, O_out=None, lse_out=None, want_lse: bool = False):
        """spts_paged_attention: Q [n, H, d] (or [n, H * d]), the last rows of their sequences -> O [n, H * d]; with want_lse or lse_out
        (O, lse [n, H])."""
        n, heads, dev = Q.shape[0], self.shape.n_q_heads, self.dev
        w = heads * self.shape.head_dim
        self._paged_shape(cache)
        qp, ldq = _rows(Q, w, self.dtype, "Q", dev)
        if O_out is None:
            O_out = Q.new_empty((n, w))
        elif O_out.shape[0] != n:
            raise ValueError("as many rows of O_out as of Q are needed")
        if lse_out is None and want_lse:
            lse_out = Q.new_empty((n, heads), dtype=torch.float32)
        op, ldo = _rows(O_out, w, self.dtype, "O_out", dev)
        code = self.lib.spts_paged_attention(self.h, cache.c, qp, ldq, _vec(row_start, cache.n_seq + 1, torch.int32, "row_start", dev), n, op,
                                             ldo, _vec(lse_out, n * heads, torch.float32, "lse_out", dev))
        if code:
            raise SptsError(code, "spts_paged_attention")
        return O_out if lse_out is None else (O_out, lse_out)

    def paged_weights(self, cache: PagedKv, Q: torch.Tensor, lse: torch.Tensor, row_start=None, decay: float = 1.0):
        """spts_paged_weights: cache.weight = decay * cache.weight + the weight that the rows get from these queries."""
        n, dev = Q.shape[0], self.dev
        self._paged_shape(cache)
        if cache.weight is None:
            raise ValueError("the cache was made without weights")
        qp, ldq = _rows(Q, self.shape.n_q_heads * self.shape.head_dim, self.dtype, "Q", dev)
        code = self.lib.spts_paged_weights(self.h, cache.c, qp, ldq, _vec(row_start, cache.n_seq + 1, torch.int32, "row_start", dev), n,
                                           _vec(lse, n * self.shape.n_q_heads, torch.float32, "lse", dev), float(decay))
        if code:
            raise SptsError(code, "spts_paged_weights")

    def paged_evict(self, cache: PagedKv, keep: torch.Tensor, n_sink: int = 0, n_recent: int = 0):
        """spts_paged_evict: every sequence down to keep[b] rows (device int32 [n_seq])."""
        self._paged_shape(cache)
        if cache.weight is None or (cache.pos is None and (n_sink or n_recent)):
            raise ValueError("the cache was made without weights, or without the positions that n_sink and n_recent go by")
        code = self.lib.spts_paged_evict(self.h, cache.c, _vec(keep, cache.n_seq, torch.int32, "keep", self.dev), int(n_sink), int(n_recent))
        if code:
            raise SptsError(code, "spts_paged_evict")

    def token_logprobs(self, logits: torch.Tensor, targets: Optional[torch.Tensor] = None, n_top: int = 0, entropy: bool = True):
        """spts_token_logprobs: a dict of logprob and rank [n] (with targets, device int32), entropy [n], top_logprob and top_token
        [n, n_top] (n_top > 0)."""
        n, v = logits.shape
        if not 0 <= n_top <= LOGPROBS_MAX_TOP:
            raise ValueError(f"up to {LOGPROBS_MAX_TOP} alternatives, got {n_top}")
        lp, ld = _rows(logits, v, torch.float32, "logits", self.dev)
        tp = _vec(targets, n, torch.int32, "targets", self.dev)
        new, i32, out = logits.new_empty, torch.int32, {}
        logprob = rank = ent = top = token = None
        if targets is not None:
            out["logprob"], out["rank"] = logprob, rank = new(n), new(n, dtype=i32)
            logprob, rank = logprob.data_ptr(), rank.data_ptr()
        if entropy:
            out["entropy"] = ent = new(n)
            ent = ent.data_ptr()
        if n_top:
            out["top_logprob"], out["top_token"] = top, token = new((n, n_top)), new((n, n_top), dtype=i32)
            top, token = top.data_ptr(), token.data_ptr()
        code = self.lib.spts_token_logprobs(self.h, lp, ld, n, v, tp, n_top, logprob, rank, ent, top, token)
        if code:
            raise SptsError(code, "spts_token_logprobs")
        return out


class Kv4Caches:
    """The 4-bit caches of all layers, n_seq sequences each."""

    def __init__(self, shape, n_layers: int, n_seq: int, capacity: int, group: int = 64, device="cuda:0", positions: bool = True):
        self.layers = [Kv4Cache(shape, n_seq, capacity, group, device, positions=positions) for _ in range(n_layers)]
        self.n_seq = n_seq
        self.c = (Kv4CacheC * n_layers)(*[cache.c for cache in self.layers])


class Model4:
    """All layers' weights in 4 bits (dicts as Spts.quantize_layer4 gives them), the LM head and the embedding table."""

    def __init__(self, layers: List[Dict[str, W4Weight]], lm_head: Optional[W4Weight] = None, embed: Optional[torch.Tensor] = None):
        self.layers, self.lm_head, self.embed = layers, lm_head, embed
        if embed is not None:
            _vec(embed, None, embed.dtype, "embed")
            if embed.dim() != 2:
                raise ValueError(f"embed: a table [vocab, hidden] is needed, got {tuple(embed.shape)}")
        names = [n for n, _ in LayerWeights4C._fields_]
        self.devices = {w[n].device_index for w in layers for n in names} | ({lm_head.device_index} if lm_head is not None else set())
        self._arr = (LayerWeights4C * len(layers))(*[LayerWeights4C(*[w[n].c for n in names]) for w in layers])
        self.c = ModelWeights4C(self._arr, lm_head.c if lm_head is not None else W4C(), embed.data_ptr() if embed is not None else None)


class Model:
    """All layers' weights plus the LM head / embedding table."""

    def __init__(self, layers: List[LayerWeights], lm_head: Optional[torch.Tensor] = None,
                 embed: Optional[torch.Tensor] = None):
        self.layers = layers
        self.lm_head, self.embed = lm_head, embed
        self._arr = (LayerWeightsC * len(layers))(*[l.c for l in layers])
        self.c = ModelWeightsC(self._arr, lm_head.data_ptr() if lm_head is not None else None,
                               embed.data_ptr() if embed is not None else None)
