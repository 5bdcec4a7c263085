"""Thin Python binding of libmoe355 (include/moe.h): argument marshalling only.

Every step of the layer runs in the library's HIP kernels; torch is used for device
memory (tensors own the buffers) and for the current stream.  If the library has not been
built the import of this module's functions raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe355.so")

MOE_OK = 0
MOE_ERR_INVALID_ARG = -1
MOE_ERR_UNSUPPORTED = -2
MOE_ERR_WORKSPACE = -3
MOE_ERR_HIP = -4
MOE_DTYPE_F32 = 0
MOE_DTYPE_BF16 = 1
MOE_STATIC_EINSUM = 0
MOE_STATIC_INDEXED = 1
MOE_CAPACITY_PAPER = 0
MOE_CAPACITY_SHARE = 1
MOE_SCORE_SOFTMAX = 0
MOE_SCORE_SIGMOID = 1
MOE_ACT_RELU = 0
MOE_ACT_SILU = 1

EXPORTS = [
    "moe_create", "moe_destroy", "moe_last_error", "moe_workspace_bytes", "moe_static_workspace_bytes",
    "moe_capacity", "moe_gate_topk", "moe_route_counts", "moe_dispatch", "moe_expert_ffn", "moe_combine",
    "moe_layer_forward", "moe_layer_forward_static", "moe_profile_begin", "moe_profile_end", "moe_profile_name",
    "moe_cache_policy_create", "moe_cache_policy_destroy", "moe_cache_policy_reset", "moe_cache_policy_step",
    "moe_cache_policy_stats", "moe_expert_cache_bytes", "moe_expert_cache_create", "moe_expert_cache_destroy",
    "moe_expert_cache_reset", "moe_expert_cache_stats", "moe_layer_forward_buffered",
    "moe_placement_greedy", "moe_placement_anticorrelation", "moe_placement_loads",
    "moe_quantize_e4m3", "moe_expert_ffn_w8", "moe_layer_forward_w8",
    "moe_mxfp4_scale_bytes", "moe_quantize_mxfp4", "moe_expert_ffn_w4", "moe_layer_forward_w4",
    "moe_expert_cache_bytes_q", "moe_expert_cache_create_q", "moe_layer_forward_noalloc",
    "moe_attn_create", "moe_attn_destroy", "moe_attn_workspace_bytes", "moe_kv_append", "moe_attn_forward",
    "moe_sample", "moe_sample_workspace_bytes",
    "moe_select_experts", "moe_b128_scale_cols", "moe_quantize_b128", "moe_gemm_b128", "moe_b128_workspace_bytes", "moe_expert_ffn_b128",
    "moe_layer_forward_b128",
]
MOE_NOALLOC_SCRATCH_BYTES = 8 * 1024 * 1024


class MoeConfig(ctypes.Structure):
    _fields_ = [("T_max", ctypes.c_int32), ("D", ctypes.c_int32), ("F", ctypes.c_int32), ("E", ctypes.c_int32),
                ("k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("renormalize", ctypes.c_int32)]


class MoeRouting(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("topk_idx", ctypes.c_void_p), ("topk_w", ctypes.c_void_p),
                ("counts", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("dst_row", ctypes.c_void_p),
                ("src_tok", ctypes.c_void_p)]


class MoeKvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class MoeAttnConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B_max", "T_max", "n_heads", "n_kv_heads", "head_dim", "page_size", "num_pages",
                                              "max_pages", "dtype", "rot_dim", "rot_interleaved")]


class MoeSelectConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("E", "k", "score", "n_groups", "groups_kept", "group_top", "renormalize")] + [("scale", ctypes.c_float)]


class MoeError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("libmoe355 error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libmoe355.so (built by paper_2303_06182_amd.build); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libmoe355.so is not built (run `python -m paper_2303_06182_amd.build`); "
                           "there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.moe_create.argtypes = [ctypes.POINTER(MoeConfig), ctypes.POINTER(vp)]
    lib.moe_create.restype = ctypes.c_int
    lib.moe_destroy.argtypes = [vp]
    lib.moe_destroy.restype = ctypes.c_int
    lib.moe_last_error.argtypes = []
    lib.moe_last_error.restype = ctypes.c_char_p
    lib.moe_workspace_bytes.argtypes = [vp]
    lib.moe_workspace_bytes.restype = i64
    lib.moe_static_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.moe_static_workspace_bytes.restype = i64
    lib.moe_capacity.argtypes = [i32, i32, i32, ctypes.c_double, i32]
    lib.moe_capacity.restype = i32
    lib.moe_gate_topk.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, i64, vp]
    lib.moe_gate_topk.restype = ctypes.c_int
    lib.moe_route_counts.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, i64, vp]
    lib.moe_route_counts.restype = ctypes.c_int
    lib.moe_dispatch.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.moe_dispatch.restype = ctypes.c_int
    lib.moe_expert_ffn.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i64, vp]
    lib.moe_expert_ffn.restype = ctypes.c_int
    lib.moe_combine.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.moe_combine.restype = ctypes.c_int
    lib.moe_layer_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, ctypes.POINTER(MoeRouting), vp, i64, vp]
    lib.moe_layer_forward.restype = ctypes.c_int
    lib.moe_layer_forward_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, ctypes.POINTER(MoeRouting), vp]
    lib.moe_layer_forward_noalloc.restype = ctypes.c_int
    lib.moe_layer_forward_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, vp, vp,
                                             ctypes.POINTER(MoeRouting), vp, i64, vp]
    lib.moe_layer_forward_static.restype = ctypes.c_int
    lib.moe_profile_begin.argtypes = [vp]
    lib.moe_profile_begin.restype = ctypes.c_int
    lib.moe_profile_end.argtypes = [vp, ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(i32)]
    lib.moe_profile_end.restype = ctypes.c_int
    lib.moe_profile_name.argtypes = [vp, i32]
    lib.moe_profile_name.restype = ctypes.c_char_p
    pi32, pi64 = ctypes.POINTER(i32), ctypes.POINTER(i64)
    lib.moe_cache_policy_create.argtypes = [i32, i32, ctypes.POINTER(vp)]
    lib.moe_cache_policy_create.restype = ctypes.c_int
    lib.moe_cache_policy_destroy.argtypes = [vp]
    lib.moe_cache_policy_destroy.restype = ctypes.c_int
    lib.moe_cache_policy_reset.argtypes = [vp]
    lib.moe_cache_policy_reset.restype = ctypes.c_int
    lib.moe_cache_policy_step.argtypes = [vp, pi32, pi32, pi32, pi32, i32, pi32, pi32]
    lib.moe_cache_policy_step.restype = ctypes.c_int
    lib.moe_cache_policy_stats.argtypes = [vp, pi64, pi64, pi32]
    lib.moe_cache_policy_stats.restype = ctypes.c_int
    lib.moe_expert_cache_bytes.argtypes = [vp, i32]
    lib.moe_expert_cache_bytes.restype = i64
    lib.moe_expert_cache_create.argtypes = [vp, i32, vp, vp, vp, i64, ctypes.POINTER(vp)]
    lib.moe_expert_cache_create.restype = ctypes.c_int
    lib.moe_expert_cache_destroy.argtypes = [vp]
    lib.moe_expert_cache_destroy.restype = ctypes.c_int
    lib.moe_expert_cache_reset.argtypes = [vp]
    lib.moe_expert_cache_reset.restype = ctypes.c_int
    lib.moe_expert_cache_stats.argtypes = [vp, pi64, pi64, pi64, pi64]
    lib.moe_expert_cache_stats.restype = ctypes.c_int
    lib.moe_layer_forward_buffered.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, ctypes.POINTER(MoeRouting), vp,
                                               i64, vp]
    lib.moe_layer_forward_buffered.restype = ctypes.c_int
    pf, pd = ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_double)
    lib.moe_placement_greedy.argtypes = [pf, i32, i32, i32, pi32]
    lib.moe_placement_greedy.restype = ctypes.c_int
    lib.moe_placement_anticorrelation.argtypes = [pf, i32, i32, i32, ctypes.c_double, pi32]
    lib.moe_placement_anticorrelation.restype = ctypes.c_int
    lib.moe_placement_loads.argtypes = [pf, i32, i32, pi32, i32, pd, pd]
    lib.moe_placement_loads.restype = ctypes.c_int
    lib.moe_quantize_e4m3.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
    lib.moe_quantize_e4m3.restype = ctypes.c_int
    lib.moe_expert_ffn_w8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i64, vp]
    lib.moe_expert_ffn_w8.restype = ctypes.c_int
    lib.moe_layer_forward_w8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, ctypes.POINTER(MoeRouting),
                                         vp, i64, vp]
    lib.moe_layer_forward_w8.restype = ctypes.c_int
    lib.moe_mxfp4_scale_bytes.argtypes = [i32, i32]
    lib.moe_mxfp4_scale_bytes.restype = i64
    lib.moe_quantize_mxfp4.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
    lib.moe_quantize_mxfp4.restype = ctypes.c_int
    lib.moe_expert_ffn_w4.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i64, vp]
    lib.moe_expert_ffn_w4.restype = ctypes.c_int
    lib.moe_layer_forward_w4.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, ctypes.POINTER(MoeRouting),
                                         vp, i64, vp]
    lib.moe_layer_forward_w4.restype = ctypes.c_int
    lib.moe_expert_cache_bytes_q.argtypes = [vp, i32, i32]
    lib.moe_expert_cache_bytes_q.restype = i64
    lib.moe_expert_cache_create_q.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, i64, ctypes.POINTER(vp)]
    lib.moe_expert_cache_create_q.restype = ctypes.c_int
    lib.moe_attn_create.argtypes = [ctypes.POINTER(MoeAttnConfig), ctypes.POINTER(vp)]
    lib.moe_attn_create.restype = ctypes.c_int
    lib.moe_attn_destroy.argtypes = [vp]
    lib.moe_attn_destroy.restype = ctypes.c_int
    lib.moe_attn_workspace_bytes.argtypes = [vp]
    lib.moe_attn_workspace_bytes.restype = i64
    lib.moe_kv_append.argtypes = [vp, ctypes.POINTER(MoeKvCache), vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, i32, i32, i32, vp, vp]
    lib.moe_kv_append.restype = ctypes.c_int
    lib.moe_attn_forward.argtypes = [vp, ctypes.POINTER(MoeKvCache), vp, i64, vp, vp, vp, i32, i32, i32, i32, ctypes.c_float, i32, i32,
                                     vp, vp, vp, i64, vp]
    lib.moe_attn_forward.restype = ctypes.c_int
    lib.moe_sample_workspace_bytes.argtypes = [i32, i32]
    lib.moe_sample_workspace_bytes.restype = i64
    lib.moe_sample.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.moe_sample.restype = ctypes.c_int
    lib.moe_select_experts.argtypes = [ctypes.POINTER(MoeSelectConfig), vp, i32, i64, vp, i32, vp, vp, vp]
    lib.moe_select_experts.restype = ctypes.c_int
    lib.moe_b128_scale_cols.argtypes = [i32]
    lib.moe_b128_scale_cols.restype = i64
    lib.moe_quantize_b128.argtypes = [vp, i32, i64, i32, i32, i32, i32, vp, vp, vp]
    lib.moe_quantize_b128.restype = ctypes.c_int
    lib.moe_gemm_b128.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, vp, i32, vp]
    lib.moe_gemm_b128.restype = ctypes.c_int
    lib.moe_b128_workspace_bytes.argtypes = [vp]
    lib.moe_b128_workspace_bytes.restype = i64
    lib.moe_expert_ffn_b128.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, i64, vp]
    lib.moe_expert_ffn_b128.restype = ctypes.c_int
    lib.moe_layer_forward_b128.argtypes = [vp, vp, vp, vp, ctypes.POINTER(MoeSelectConfig), vp, vp, vp, vp, vp, i32, i32, vp,
                                           ctypes.POINTER(MoeRouting), vp, i64, vp]
    lib.moe_layer_forward_b128.restype = ctypes.c_int
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != MOE_OK:
        raise MoeError(rc, load_library().moe_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _addr(t: Optional[torch.Tensor]) -> Optional[int]:
    """_ptr for calls of a few microseconds: the address alone, which an argument declared as a pointer takes."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _stream_on(index: int) -> int:
    """The current stream of a device, without making a stream object."""
    return torch._C._cuda_getCurrentRawStream(index)


def _gpu(device) -> torch.device:
    """The GPU that a handle is for, by its number; without one the current GPU."""
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError("device must be a GPU, not %s" % device)
    return device if device.index is not None else torch.device("cuda", torch.cuda.current_device())


def _output(t: torch.Tensor, shape: tuple, dtype: torch.dtype, index: int, name: str) -> torch.Tensor:
    """An output that the caller has allocated, as it has to be."""
    if tuple(t.shape) != shape or t.dtype != dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be %s of %s, contiguous, on cuda:%d" % (name, list(shape), dtype, index))
    return t


def moe_capacity(T: int, E: int, k: int, cf: float, convention: int = MOE_CAPACITY_SHARE) -> int:
    c = load_library().moe_capacity(T, E, k, cf, convention)
    if c < 0:
        _check(c)
    return c


class MoeLayer:
    """A handle (moe_create) plus a workspace tensor.  Methods mirror the C entry points and
    only marshal arguments; outputs are allocated by the caller or, for convenience, here
    (torch.empty) before the call."""

    def __init__(self, T_max: int, D: int, F: int, E: int, k: int = 2, dtype: str = "bf16",
                 renormalize: bool = True, device: str = "cuda:0", alloc_workspace: bool = True):
        self.lib = load_library()
        self.cfg = MoeConfig(T_max, D, F, E, k, MOE_DTYPE_BF16 if dtype == "bf16" else MOE_DTYPE_F32,
                             int(renormalize))
        self.T_max, self.D, self.F, self.E, self.k = T_max, D, F, E, k
        self.dtype = dtype
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device = _gpu(device)
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.moe_create(ctypes.byref(self.cfg), ctypes.byref(h)))
        self.h = h
        self.workspace_bytes = int(self.lib.moe_workspace_bytes(self.h))
        self.workspace = None
        self.workspace_b128 = None
        if alloc_workspace:
            self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)

    def __del__(self):
        try:
            if getattr(self, "h", None):
                self.lib.moe_destroy(self.h)
                self.h = None
        except Exception:
            pass

    # -- helpers ---------------------------------------------------------------------------
    def _ws(self):
        if self.workspace is None:
            return None, 0
        return _ptr(self.workspace), self.workspace.numel()

    def _new(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def empty_routing(self, T: int) -> dict:
        return dict(logits=self._new((T, self.E), torch.float32), topk_idx=self._new((T, self.k), torch.int32),
                    topk_w=self._new((T, self.k), torch.float32), counts=self._new((self.E,), torch.int32),
                    offsets=self._new((self.E + 1,), torch.int32), dst_row=self._new((T, self.k), torch.int32),
                    src_tok=self._new((T * self.k,), torch.int32))

    @staticmethod
    def _routing_struct(r: Optional[dict]):
        if r is None:
            return None
        s = MoeRouting()
        for name in ("logits", "topk_idx", "topk_w", "counts", "offsets", "dst_row", "src_tok"):
            t = r.get(name)
            setattr(s, name, None if t is None else t.data_ptr())
        return ctypes.byref(s)

    # -- the entry points ------------------------------------------------------------------
    def moe_gate_topk(self, x, wg, gate_bias=None, logits_out=None, topk_idx=None, topk_w=None):
        T = x.shape[0]
        if logits_out is None:
            logits_out = self._new((T, self.E), torch.float32)
        if topk_idx is None:
            topk_idx = self._new((T, self.k), torch.int32)
        if topk_w is None:
            topk_w = self._new((T, self.k), torch.float32)
        ws, wsb = self._ws()
        _check(self.lib.moe_gate_topk(self.h, _ptr(x), _ptr(wg), _ptr(gate_bias), T, _ptr(logits_out),
                                      _ptr(topk_idx), _ptr(topk_w), ws, wsb, _stream()))
        return logits_out, topk_idx, topk_w

    def moe_route_counts(self, topk_idx):
        T = topk_idx.shape[0]
        counts = self._new((self.E,), torch.int32)
        offsets = self._new((self.E + 1,), torch.int32)
        dst_row = self._new((T, self.k), torch.int32)
        src_tok = self._new((T * self.k,), torch.int32)
        ws, wsb = self._ws()
        _check(self.lib.moe_route_counts(self.h, _ptr(topk_idx), T, _ptr(counts), _ptr(offsets), _ptr(dst_row),
                                         _ptr(src_tok), ws, wsb, _stream()))
        return counts, offsets, dst_row, src_tok

    def moe_dispatch(self, x, dst_row):
        T = x.shape[0]
        xp = self._new((T * self.k, self.D), self.torch_dtype)
        _check(self.lib.moe_dispatch(self.h, _ptr(x), _ptr(dst_row), T, _ptr(xp), _stream()))
        return xp

    def moe_expert_ffn(self, xp, offsets, w1, w2, b1=None, b2=None):
        n_rows = xp.shape[0]
        yp = self._new((n_rows, self.D), self.torch_dtype)
        ws, wsb = self._ws()
        _check(self.lib.moe_expert_ffn(self.h, _ptr(xp), _ptr(offsets), _ptr(w1), _ptr(w2), _ptr(b1), _ptr(b2),
                                       n_rows, _ptr(yp), ws, wsb, _stream()))
        return yp

    def moe_combine(self, yp, dst_row, topk_w):
        T = dst_row.shape[0]
        y = self._new((T, self.D), self.torch_dtype)
        _check(self.lib.moe_combine(self.h, _ptr(yp), _ptr(dst_row), _ptr(topk_w), T, _ptr(y), _stream()))
        return y

    def moe_layer_forward(self, x, wg, w1, w2, gate_bias=None, b1=None, b2=None, y=None, routing_out=None):
        T = x.shape[0]
        if y is None:
            y = self._new((T, self.D), self.torch_dtype)
        ws, wsb = self._ws()
        _check(self.lib.moe_layer_forward(self.h, _ptr(x), _ptr(wg), _ptr(gate_bias), _ptr(w1), _ptr(w2), _ptr(b1),
                                          _ptr(b2), T, _ptr(y), self._routing_struct(routing_out), ws, wsb,
                                          _stream()))
        return y

    def moe_layer_forward_noalloc(self, x, wg, w1, w2, y, gate_bias=None, b1=None, b2=None, routing_out=None):
        """moe_layer_forward on the library's own scratch array: no workspace, and nothing is allocated
        here either (the caller brings y and the routing arrays)."""
        _check(self.lib.moe_layer_forward_noalloc(self.h, _ptr(x), _ptr(wg), _ptr(gate_bias), _ptr(w1), _ptr(w2),
                                                  _ptr(b1), _ptr(b2), x.shape[0], _ptr(y),
                                                  self._routing_struct(routing_out), _stream()))
        return y

    def moe_quantize_e4m3(self, w):
        """w [E, rows, cols] -> (q uint8 [E, rows * cols] in the library's blocked layout, scale [E] fp32)."""
        E, rows, cols = w.shape
        q = self._new((E, rows * cols), torch.uint8)
        scale = self._new((E,), torch.float32)
        _check(self.lib.moe_quantize_e4m3(self.h, _ptr(w), E, rows, cols, _ptr(q), _ptr(scale), _stream()))
        return q, scale

    def moe_expert_ffn_w8(self, xp, offsets, w1_q, w2_q, w1_scale, w2_scale, b1=None, b2=None):
        n_rows = xp.shape[0]
        yp = self._new((n_rows, self.D), self.torch_dtype)
        ws, wsb = self._ws()
        _check(self.lib.moe_expert_ffn_w8(self.h, _ptr(xp), _ptr(offsets), _ptr(w1_q), _ptr(w2_q), _ptr(w1_scale),
                                          _ptr(w2_scale), _ptr(b1), _ptr(b2), n_rows, _ptr(yp), ws, wsb, _stream()))
        return yp

    def moe_layer_forward_w8(self, x, wg, w1_q, w2_q, w1_scale, w2_scale, gate_bias=None, b1=None, b2=None, y=None,
                             routing_out=None):
        T = x.shape[0]
        if y is None:
            y = self._new((T, self.D), self.torch_dtype)
        ws, wsb = self._ws()
        _check(self.lib.moe_layer_forward_w8(self.h, _ptr(x), _ptr(wg), _ptr(gate_bias), _ptr(w1_q), _ptr(w2_q),
                                             _ptr(w1_scale), _ptr(w2_scale), _ptr(b1), _ptr(b2), T, _ptr(y),
                                             self._routing_struct(routing_out), ws, wsb, _stream()))
        return y

    def moe_quantize_mxfp4(self, w):
        """w [E, rows, cols] -> (q uint8 [E, rows * cols / 2], scale bytes uint8 [E, moe_mxfp4_scale_bytes]),
        both in the library's blocked layouts."""
        E, rows, cols = w.shape
        nb = int(self.lib.moe_mxfp4_scale_bytes(rows, cols))
        if nb < 0:
            _check(nb)
        q = self._new((E, rows * cols // 2), torch.uint8)
        scale = torch.full((E, nb), 127, dtype=torch.uint8, device=self.device)
        _check(self.lib.moe_quantize_mxfp4(self.h, _ptr(w), E, rows, cols, _ptr(q), _ptr(scale), _stream()))
        return q, scale

    def moe_expert_ffn_w4(self, xp, offsets, w1_q, w2_q, w1_scale, w2_scale, b1=None, b2=None):
        n_rows = xp.shape[0]
        yp = self._new((n_rows, self.D), self.torch_dtype)
        ws, wsb = self._ws()
        _check(self.lib.moe_expert_ffn_w4(self.h, _ptr(xp), _ptr(offsets), _ptr(w1_q), _ptr(w2_q), _ptr(w1_scale),
                                          _ptr(w2_scale), _ptr(b1), _ptr(b2), n_rows, _ptr(yp), ws, wsb, _stream()))
        return yp

    def moe_layer_forward_w4(self, x, wg, w1_q, w2_q, w1_scale, w2_scale, gate_bias=None, b1=None, b2=None, y=None,
                             routing_out=None):
        T = x.shape[0]
        if y is None:
            y = self._new((T, self.D), self.torch_dtype)
        ws, wsb = self._ws()
        _check(self.lib.moe_layer_forward_w4(self.h, _ptr(x), _ptr(wg), _ptr(gate_bias), _ptr(w1_q), _ptr(w2_q),
                                             _ptr(w1_scale), _ptr(w2_scale), _ptr(b1), _ptr(b2), T, _ptr(y),
                                             self._routing_struct(routing_out), ws, wsb, _stream()))
        return y

    # -- experts in e4m3 with a scale per block of 128 -------------------------------------------
    def b128_workspace(self) -> torch.Tensor:
        """The workspace of the two calls below, allocated on first use (before a capture, so that no graph owns it)."""
        if self.workspace_b128 is None:
            n = int(self.lib.moe_b128_workspace_bytes(self.h))
            if n < 0:
                _check(n)
            self.workspace_b128 = torch.empty(n, dtype=torch.uint8, device=self.device)
        return self.workspace_b128

    def _b128_weights(self, w1_q, w2_q, w1_scale, w2_scale, activation: str) -> int:
        act = _choice("activation", activation, {"relu": MOE_ACT_RELU, "silu": MOE_ACT_SILU})
        E, D, F = self.E, self.D, self.F
        halves = (2,) if act == MOE_ACT_SILU else ()
        _b128_operand(w1_q, w1_scale, (E, *halves, F, D), (E, *halves), 128, self.device.index, "w1")
        _b128_operand(w2_q, w2_scale, (E, D, F), (E,), 128, self.device.index, "w2")
        return act

    def _rows_of(self, t, shape, dtype, name: str):
        if t is not None and (tuple(t.shape) != shape or t.dtype != dtype or t.get_device() != self.device.index):
            raise ValueError("%s must be %s of %s on %s" % (name, list(shape), dtype, self.device))
        return _addr(t)

    def moe_expert_ffn_b128(self, x, offsets, w1_q, w2_q, w1_scale, w2_scale, activation: str = "silu", src_tok=None, yp=None):
        """x [x_rows, D]; w1_q [E, 2, F, D] (silu: gate, up) or [E, F, D] (relu), w2_q [E, D, F] and their scales from moe_quantize_b128 ->
        yp, a row for each of src_tok (None: of x)."""
        x_rows = x.shape[0]
        n_rows = x_rows if src_tok is None else src_tok.shape[0]
        _fit_32_bits(x_rows, n_rows)
        act = self._b128_weights(w1_q, w2_q, w1_scale, w2_scale, activation)
        if yp is None:
            yp = self._new((n_rows, self.D), self.torch_dtype)
        else:
            _output(yp, (n_rows, self.D), self.torch_dtype, self.device.index, "yp")
        ws = self.b128_workspace()
        _check(self.lib.moe_expert_ffn_b128(self.h, self._rows_of(x, (x_rows, self.D), self.torch_dtype, "x"), x_rows,
                                            self._rows_of(src_tok, (n_rows,), torch.int32, "src_tok"),
                                            self._rows_of(offsets, (self.E + 1,), torch.int32, "offsets"), _addr(w1_q), _addr(w2_q), _addr(w1_scale),
                                            _addr(w2_scale), act, n_rows, _addr(yp), ws.data_ptr(), ws.numel(), _stream_on(self.device.index)))
        return yp

    def moe_layer_forward_b128(self, x, wg, w1_q, w2_q, w1_scale, w2_scale, activation: str = "silu", score: str = "sigmoid", select_bias=None,
                               n_groups: int = 1, groups_kept: int = 1, group_top: int = 2, renormalize: bool = True, scale: float = 1.0,
                               gate_bias=None, y=None, routing_out=None):
        """The layer with experts chosen as moe_select_experts does, and moe_expert_ffn_b128."""
        T = x.shape[0]
        _fit_32_bits(T)
        act = self._b128_weights(w1_q, w2_q, w1_scale, w2_scale, activation)
        cfg = _select_config(self.E, self.k, score, n_groups, groups_kept, group_top, renormalize, scale)
        if y is None:
            y = self._new((T, self.D), self.torch_dtype)
        else:
            _output(y, (T, self.D), self.torch_dtype, self.device.index, "y")
        ws = self.b128_workspace()
        _check(self.lib.moe_layer_forward_b128(self.h, self._rows_of(x, (T, self.D), self.torch_dtype, "x"),
                                               self._rows_of(wg, (self.E, self.D), self.torch_dtype, "wg"),
                                               self._rows_of(gate_bias, (self.E,), torch.float32, "gate_bias"), ctypes.byref(cfg),
                                               self._rows_of(select_bias, (self.E,), torch.float32, "select_bias"), _addr(w1_q), _addr(w2_q),
                                               _addr(w1_scale), _addr(w2_scale), act, T, _addr(y), self._routing_struct(routing_out), ws.data_ptr(),
                                               ws.numel(), _stream_on(self.device.index)))
        return y

    def moe_profile_begin(self) -> None:
        _check(self.lib.moe_profile_begin(self.h))

    def moe_profile_end(self):
        """-> list of (kernel name, milliseconds) in launch order.  Waits for the device."""
        ms = (ctypes.c_float * 64)()
        n = ctypes.c_int32(0)
        _check(self.lib.moe_profile_end(self.h, ms, 64, ctypes.byref(n)))
        return [(self.lib.moe_profile_name(self.h, i).decode(), float(ms[i])) for i in range(n.value)]

    def moe_static_workspace_bytes(self, T: int, capacity: int, mode: int) -> int:
        n = int(self.lib.moe_static_workspace_bytes(self.h, T, capacity, mode))
        if n < 0:
            _check(n)
        return n

    def moe_layer_forward_static(self, x, wg, w1, w2, capacity: int, mode: int = MOE_STATIC_INDEXED,
                                 gate_bias=None, b1=None, b2=None, y=None, routing_out=None, workspace=None):
        T = x.shape[0]
        if y is None:
            y = self._new((T, self.D), self.torch_dtype)
        dropped = torch.zeros(4, dtype=torch.int32, device=self.device)
        if workspace is None:
            workspace = torch.empty(self.moe_static_workspace_bytes(T, capacity, mode), dtype=torch.uint8,
                                    device=self.device)
        _check(self.lib.moe_layer_forward_static(self.h, _ptr(x), _ptr(wg), _ptr(gate_bias), _ptr(w1), _ptr(w2),
                                                 _ptr(b1), _ptr(b2), T, capacity, mode, _ptr(y), _ptr(dropped),
                                                 self._routing_struct(routing_out), _ptr(workspace),
                                                 workspace.numel(), _stream()))
        return y, dropped[:1]


class CachePolicy:
    """moe_cache_policy_*: the cache management of Expert Buffering alone (host logic, no GPU)."""

    def __init__(self, E: int, slots: int):
        self.lib = load_library()
        self.E, self.slots = E, slots
        self.p = ctypes.c_void_p()
        _check(self.lib.moe_cache_policy_create(E, slots, ctypes.byref(self.p)))

    def __del__(self):
        if getattr(self, "p", None) is not None and self.p:
            self.lib.moe_cache_policy_destroy(self.p)
            self.p = None

    def reset(self) -> None:
        _check(self.lib.moe_cache_policy_reset(self.p))

    def step(self, counts):
        """counts: E host integers -> (slot_of, stage_of, loads, n_stages); loads = list of
        (expert, slot, victim, stage)."""
        E = self.E
        c = (ctypes.c_int32 * E)(*[int(v) for v in counts])
        slot_of, stage_of = (ctypes.c_int32 * E)(), (ctypes.c_int32 * E)()
        loads = (ctypes.c_int32 * (4 * E))()
        n_loads, n_stages = ctypes.c_int32(0), ctypes.c_int32(0)
        _check(self.lib.moe_cache_policy_step(self.p, c, slot_of, stage_of, loads, E, ctypes.byref(n_loads),
                                              ctypes.byref(n_stages)))
        ll = [tuple(loads[4 * i + j] for j in range(4)) for i in range(n_loads.value)]
        return list(slot_of), list(stage_of), ll, n_stages.value

    def stats(self):
        """-> (hits, misses, expert held by every slot)."""
        h, m = ctypes.c_int64(0), ctypes.c_int64(0)
        se = (ctypes.c_int32 * self.slots)()
        _check(self.lib.moe_cache_policy_stats(self.p, ctypes.byref(h), ctypes.byref(m), se))
        return h.value, m.value, list(se)


class ExpertCache:
    """moe_expert_cache_*: `slots` device slots in front of expert parameters kept in pinned host
    memory (host_w1 [E,F,D], host_w2 [E,D,F], torch CPU tensors with pin_memory)."""

    def __init__(self, layer: "MoeLayer", slots: int, host_w1: torch.Tensor, host_w2: torch.Tensor, wbits: int = 0,
                 w1_scale: Optional[torch.Tensor] = None, w2_scale: Optional[torch.Tensor] = None):
        """wbits = 8 / 4: host_w1 / host_w2 hold the quantised bytes (moe_quantize_e4m3 / moe_quantize_mxfp4,
        copied to pinned host memory), w1_scale / w2_scale their scales, which stay on the device."""
        self.lib = layer.lib
        self.layer = layer
        self.slots = slots
        if host_w1.device.type != "cpu" or host_w2.device.type != "cpu":
            raise ValueError("host_w1 / host_w2 must be CPU tensors (pinned)")
        self.host_w1, self.host_w2 = host_w1, host_w2  # kept alive
        self.w1_scale, self.w2_scale = w1_scale, w2_scale
        nbytes = int(self.lib.moe_expert_cache_bytes_q(layer.h, slots, wbits))
        if nbytes < 0:
            _check(nbytes)
        self.device_mem = torch.empty(nbytes, dtype=torch.uint8, device=layer.device)
        self.c = ctypes.c_void_p()
        _check(self.lib.moe_expert_cache_create_q(layer.h, slots, wbits, host_w1.data_ptr(), host_w2.data_ptr(),
                                                  _ptr(w1_scale), _ptr(w2_scale), _ptr(self.device_mem), nbytes,
                                                  ctypes.byref(self.c)))

    def __del__(self):
        if getattr(self, "c", None) is not None and self.c:
            self.lib.moe_expert_cache_destroy(self.c)
            self.c = None

    def reset(self) -> None:
        _check(self.lib.moe_expert_cache_reset(self.c))

    def stats(self):
        """-> dict(hits, misses, bytes_copied, stages)."""
        v = [ctypes.c_int64(0) for _ in range(4)]
        _check(self.lib.moe_expert_cache_stats(self.c, *[ctypes.byref(x) for x in v]))
        return dict(hits=v[0].value, misses=v[1].value, bytes_copied=v[2].value, stages=v[3].value)

    def moe_layer_forward_buffered(self, x, wg, gate_bias=None, b1=None, b2=None, y=None, routing_out=None):
        L = self.layer
        T = x.shape[0]
        if y is None:
            y = L._new((T, L.D), L.torch_dtype)
        ws, wsb = L._ws()
        _check(self.lib.moe_layer_forward_buffered(L.h, self.c, _ptr(x), _ptr(wg), _ptr(gate_bias), _ptr(b1),
                                                   _ptr(b2), T, _ptr(y), L._routing_struct(routing_out), ws, wsb,
                                                   _stream()))
        return y


def _activation_array(A):
    E = len(A)
    B = len(A[0]) if E else 0
    flat = (ctypes.c_float * (E * B))(*[float(v) for row in A for v in row])
    return flat, E, B


def moe_placement_greedy(A, n_devices: int):
    """A: E rows of B activation fractions (host) -> device of every expert (Sec. 7.1)."""
    flat, E, B = _activation_array(A)
    out = (ctypes.c_int32 * max(E, 1))()
    _check(load_library().moe_placement_greedy(flat, E, B, n_devices, out))
    return list(out)[:E]


def moe_placement_anticorrelation(A, n_devices: int, corr_weight: float = 0.5):
    flat, E, B = _activation_array(A)
    out = (ctypes.c_int32 * max(E, 1))()
    _check(load_library().moe_placement_anticorrelation(flat, E, B, n_devices, corr_weight, out))
    return list(out)[:E]


def moe_placement_loads(A, device_of, n_devices: int):
    """-> (Max Load, Avg Max Load) of a placement on activation data A (Sec. 7.1)."""
    flat, E, B = _activation_array(A)
    d = (ctypes.c_int32 * max(E, 1))(*[int(v) for v in device_of])
    mx, av = ctypes.c_double(0), ctypes.c_double(0)
    _check(load_library().moe_placement_loads(flat, E, B, d, n_devices, ctypes.byref(mx), ctypes.byref(av)))
    return mx.value, av.value


class KvCache:
    """One layer's paged cache (moe_kv_cache_t): k and v [num_pages, n_kv_heads, page_size, head_dim] in torch.float8_e4m3fn (or
    uint8), k_scale and v_scale [num_pages, n_kv_heads] fp32, on the device.  PagedAttention.new_cache allocates one."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        for name, t in (("k", k), ("v", v)):
            if t.dim() != 4 or t.element_size() != 1:
                raise ValueError("%s must be [num_pages, n_kv_heads, page_size, head_dim] of one byte each" % name)
        if k.shape != v.shape or tuple(k_scale.shape) != tuple(k.shape[:2]) or tuple(v_scale.shape) != tuple(k.shape[:2]):
            raise ValueError("k and v must have the same shape, the scales their first two dimensions")
        if k_scale.dtype != torch.float32 or v_scale.dtype != torch.float32:
            raise ValueError("scales must be float32")
        self.index = k.get_device()
        if any(t.get_device() != self.index for t in (v, k_scale, v_scale)):
            raise ValueError("k, v and their scales must be on one device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.shape = tuple(k.shape)
        self.struct = MoeKvCache(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale))
        self.ref = ctypes.byref(self.struct)


class PagedAttention:
    """A handle (moe_attn_create) plus a workspace tensor, for every layer of one geometry.  Methods mirror the C entry
    points; q, k and v may be views of one projection's output (a token's heads together, any stride from token to token)."""

    def __init__(self, B_max: int, T_max: int, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int, num_pages: int, max_pages: int,
                 dtype: str = "bf16", rot_dim: int = 0, interleaved: bool = False, device: str = "cuda:0"):
        self.lib = load_library()
        self.cfg = MoeAttnConfig(B_max, T_max, n_heads, n_kv_heads, head_dim, page_size, num_pages, max_pages,
                                 MOE_DTYPE_BF16 if dtype == "bf16" else MOE_DTYPE_F32, rot_dim, int(interleaved))
        self.cache_shape = (num_pages, n_kv_heads, page_size, head_dim)
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.device = _gpu(device)
        self.index = self.device.index
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(self.lib.moe_attn_create(ctypes.byref(self.cfg), ctypes.byref(h)))
        self.h = h
        self.workspace = torch.empty(int(self.lib.moe_attn_workspace_bytes(h)), dtype=torch.uint8, device=self.device)

    def __del__(self):
        try:
            if getattr(self, "h", None):
                self.lib.moe_attn_destroy(self.h)
                self.h = None
        except Exception:
            pass

    def new_cache(self) -> KvCache:
        shape = self.cache_shape
        k, v = (torch.empty(shape, dtype=torch.uint8, device=self.device).view(torch.float8_e4m3fn) for _ in range(2))
        ks, vs = (torch.empty(shape[:2], dtype=torch.float32, device=self.device) for _ in range(2))
        return KvCache(k, v, ks, vs)

    def _rows(self, t: Optional[torch.Tensor], heads: int, name: str):
        """(address, elements from token to token) of [T, heads, head_dim]."""
        if t is None:
            return None, 0
        dim, shape, strides = self.cfg.head_dim, t.shape, t.stride()
        if len(shape) != 3 or shape[1] != heads or shape[2] != dim or t.dtype != self.torch_dtype:
            raise ValueError("%s must be [T, %d, %d] of %s" % (name, heads, dim, self.torch_dtype))
        if shape[0] and (strides[2] != 1 or (heads > 1 and strides[1] != dim)):
            raise ValueError("%s: the heads of a token must lie together" % name)
        if t.get_device() != self.index:
            raise ValueError("%s must be on %s" % (name, self.device))
        return t.data_ptr(), strides[0] if shape[0] > 1 else heads * dim

    def _batch(self, cache: KvCache, q_offsets, kv_len, page_table):
        if cache.shape != self.cache_shape:
            raise ValueError("the cache has shape %s, the handle another geometry" % (cache.shape,))
        B = kv_len.shape[0]
        if q_offsets.shape[0] != B + 1 or page_table.shape != (B, self.cfg.max_pages):
            raise ValueError("q_offsets must be [B + 1], kv_len [B] and page_table [B, max_pages]")
        if q_offsets.dtype != torch.int32 or kv_len.dtype != torch.int32 or page_table.dtype != torch.int32:
            raise ValueError("q_offsets, kv_len and page_table must be int32")
        i = self.index
        if q_offsets.get_device() != i or kv_len.get_device() != i or page_table.get_device() != i or cache.index != i:
            raise ValueError("the cache, q_offsets, kv_len and page_table must be on %s" % self.device)
        return B

    def moe_kv_append(self, cache: KvCache, q, k, v, inv_freq, q_offsets, kv_len, page_table, max_q: int, q_out=None):
        """Rotates q (None: only keys and values) and k, and appends k and v to the cache; returns the rotated queries."""
        B, T, c = self._batch(cache, q_offsets, kv_len, page_table), k.shape[0], self.cfg
        if v.shape[0] != T or (q is not None and q.shape[0] != T):
            raise ValueError("q, k and v must have the same number of tokens")
        if inv_freq is not None and (inv_freq.dtype != torch.float64 or inv_freq.numel() != c.rot_dim // 2):
            raise ValueError("inv_freq must be [rot_dim / 2] float64")
        if inv_freq is not None and inv_freq.get_device() != self.index:
            raise ValueError("inv_freq must be on %s" % self.device)
        if q_out is not None:
            _output(q_out, (T, c.n_heads, c.head_dim), self.torch_dtype, self.index, "q_out")
        elif q is not None:
            q_out = torch.empty((T, c.n_heads, c.head_dim), dtype=self.torch_dtype, device=self.device)
        (qp, qs), (kp, ks), (vp, vs) = self._rows(q, c.n_heads, "q"), self._rows(k, c.n_kv_heads, "k"), self._rows(v, c.n_kv_heads, "v")
        _check(self.lib.moe_kv_append(self.h, cache.ref, qp, qs, kp, ks, vp, vs, _addr(inv_freq), _addr(q_offsets), _addr(kv_len),
                                      _addr(page_table), B, T, max_q, _addr(q_out), _stream_on(self.index)))
        return q_out

    def moe_attn_forward(self, cache: KvCache, q, q_offsets, kv_len, page_table, max_q: int, max_kv: int, scale: Optional[float] = None,
                         causal: bool = True, window: int = 0, out=None, lse=None, want_lse: bool = True):
        """-> (out [T, n_heads, head_dim], lse [T, n_heads] fp32 or None).  scale: 1 / sqrt(head_dim) where not given."""
        B, T, c = self._batch(cache, q_offsets, kv_len, page_table), q.shape[0], self.cfg
        if out is None:
            out = torch.empty((T, c.n_heads, c.head_dim), dtype=self.torch_dtype, device=self.device)
        else:
            _output(out, (T, c.n_heads, c.head_dim), self.torch_dtype, self.index, "out")
        if lse is not None:
            _output(lse, (T, c.n_heads), torch.float32, self.index, "lse")
        elif want_lse:
            lse = torch.empty((T, c.n_heads), dtype=torch.float32, device=self.device)
        qp, qs = self._rows(q, c.n_heads, "q")
        _check(self.lib.moe_attn_forward(self.h, cache.ref, qp, qs, _addr(q_offsets), _addr(kv_len), _addr(page_table), B, T, max_q,
                                         max_kv, c.head_dim ** -0.5 if scale is None else scale, int(causal), window, _addr(out), _addr(lse),
                                         self.workspace.data_ptr(), self.workspace.numel(), _stream_on(self.index)))
        return out, lse


def moe_sample_workspace_bytes(B: int, V: int) -> int:
    n = int(load_library().moe_sample_workspace_bytes(B, V))
    if n < 0:
        _check(n)
    return n


def moe_sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, token=None, logprob=None, workspace=None):
    """logits [B, V] (float32 or bfloat16, rows at any stride), u [B] in [0, 1), every row's settings or None
    -> (token [B] int32, logprob [B] fp32)."""
    lib = load_library()
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [B, V] of float32 or bfloat16 with dense rows")
    B, V = logits.shape
    index = logits.get_device()
    if index < 0 or index != torch.cuda.current_device():
        raise ValueError("logits are on %s, which is not the current GPU" % logits.device)
    for t, dtype in ((u, torch.float32), (temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32)):
        if t is not None and (t.dtype != dtype or t.numel() != B or t.get_device() != index):
            raise ValueError("u, temperature, top_p and min_p must be [B] float32, top_k [B] int32, on %s" % logits.device)
    new = lambda dtype: torch.empty((B,), dtype=dtype, device=logits.device)  # noqa: E731
    token = new(torch.int32) if token is None else _output(token, (B,), torch.int32, index, "token")
    logprob = new(torch.float32) if logprob is None else _output(logprob, (B,), torch.float32, index, "logprob")
    if workspace is None:
        workspace = torch.empty(moe_sample_workspace_bytes(B, V), dtype=torch.uint8, device=logits.device)
    elif workspace.dtype != torch.uint8 or workspace.get_device() != index:
        raise ValueError("workspace must be uint8 on %s" % logits.device)
    _check(lib.moe_sample(logits.data_ptr(), MOE_DTYPE_BF16 if logits.dtype == torch.bfloat16 else MOE_DTYPE_F32,
                          logits.stride(0) if B > 1 else V, B, V, _addr(u), _addr(temperature), _addr(top_k), _addr(top_p), _addr(min_p), _addr(token),
                          _addr(logprob), _addr(workspace), workspace.numel(), _stream_on(index)))
    return token, logprob


def _choice(name: str, value: str, choices: dict) -> int:
    if value not in choices:
        raise ValueError("%s must be one of %s, not %r" % (name, sorted(choices), value))
    return choices[value]


def _current_gpu(t: torch.Tensor, name: str) -> int:
    index = t.get_device()
    if index < 0 or index != torch.cuda.current_device():
        raise ValueError("%s is on %s, which is not the current GPU" % (name, t.device))
    return index


def _fit_32_bits(*sizes: int) -> None:
    """The library takes sizes in 32 bits; ctypes would pass the low ones of a larger one on."""
    if max(sizes) > 0x7fffffff:
        raise ValueError("sizes must fit 32 bits, not %d" % max(sizes))


def _select_config(E: int, k: int, score: str, n_groups: int, groups_kept: int, group_top: int, renormalize: bool, scale: float) -> MoeSelectConfig:
    _fit_32_bits(*map(abs, (E, k, n_groups, groups_kept, group_top, int(renormalize))))
    return MoeSelectConfig(E, k, _choice("score", score, {"softmax": MOE_SCORE_SOFTMAX, "sigmoid": MOE_SCORE_SIGMOID}), n_groups, groups_kept, group_top,
                           int(renormalize), scale)


def moe_select_experts(logits, k: int, bias=None, score: str = "sigmoid", n_groups: int = 1, groups_kept: int = 1, group_top: int = 2,
                       renormalize: bool = True, scale: float = 1.0, topk_idx=None, topk_w=None):
    """logits [T, E] (float32 or bfloat16, rows at any stride), bias [E] fp32 or None -> (topk_idx [T, k] int32, topk_w [T, k] fp32)."""
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [T, E] of float32 or bfloat16 with dense rows")
    T, E = logits.shape
    _fit_32_bits(T)
    cfg = _select_config(E, k, score, n_groups, groups_kept, group_top, renormalize, scale)
    index = _current_gpu(logits, "logits")
    if bias is not None and (tuple(bias.shape) != (E,) or bias.dtype != torch.float32 or bias.get_device() != index):
        raise ValueError("bias must be [%d] of float32 on %s" % (E, logits.device))
    new = lambda dtype: torch.empty((T, max(k, 0)), dtype=dtype, device=logits.device)  # noqa: E731
    topk_idx = new(torch.int32) if topk_idx is None else _output(topk_idx, (T, k), torch.int32, index, "topk_idx")
    topk_w = new(torch.float32) if topk_w is None else _output(topk_w, (T, k), torch.float32, index, "topk_w")
    _check(load_library().moe_select_experts(ctypes.byref(cfg), logits.data_ptr(), MOE_DTYPE_BF16 if logits.dtype == torch.bfloat16 else MOE_DTYPE_F32,
                                             logits.stride(0) if T > 1 else E, _addr(bias), T, topk_idx.data_ptr(), topk_w.data_ptr(), _stream_on(index)))
    return topk_idx, topk_w


def b128_scale_cols(cols: int) -> int:
    """Scale bytes of a row of `cols` elements: one for each block of 128, in groups of four."""
    n = int(load_library().moe_b128_scale_cols(cols))
    if n < 0:
        _check(n)
    return n


def _b128_operand(q, scale, shape: tuple, scale_rows: tuple, block_rows: int, index: int, name: str) -> None:
    """q of `shape` and its scales; scale_rows: the dimensions in front of a matrix's rows, of the scales."""
    scales = scale_rows + (-(-shape[-2] // block_rows), -(-shape[-1] // 512) * 4)
    if tuple(q.shape) != shape or q.dtype not in (torch.float8_e4m3fn, torch.uint8) or not q.is_contiguous() or q.get_device() != index:
        raise ValueError("%s_q must be %s of float8_e4m3fn or its bytes, contiguous, on cuda:%d" % (name, list(shape), index))
    if tuple(scale.shape) != scales or scale.dtype != torch.uint8 or not scale.is_contiguous() or scale.get_device() != index:
        raise ValueError("%s_scale must be %s of uint8, contiguous, on cuda:%d" % (name, list(scales), index))


def moe_quantize_b128(x, block_rows: int = 1, q=None, scale=None):
    """x [rows, cols] or [..., rows, cols] (float32 or bfloat16; rows at one stride throughout) -> (q of the same shape, torch.float8_e4m3fn, scale
    bytes [..., rows or blocks of 128 rows, b128_scale_cols(cols)])."""
    if x.dim() < 2 or x.dtype not in (torch.float32, torch.bfloat16) or (x.shape[-1] > 1 and x.stride(-1) != 1):
        raise ValueError("x must be [..., rows, cols] of float32 or bfloat16 with dense rows")
    lead, (rows, cols) = tuple(x.shape[:-2]), x.shape[-2:]
    matrices = 1
    for n in lead:
        matrices *= n
    _fit_32_bits(matrices, rows, cols)
    index = _current_gpu(x, "x")
    # all rows, of all matrices, at one stride
    outer = [(n, s) for n, s in zip(x.shape[:-1], x.stride()[:-1]) if n > 1] if x.numel() else []
    stride = outer[-1][1] if outer else cols
    step = stride
    for n, s in reversed(outer):
        if s != step:
            raise ValueError("the rows of x must lie at one stride")
        step *= n
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    scales = lead + (-(-rows // block_rows), b128_scale_cols(cols))
    q = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device) if q is None else _output(q, tuple(x.shape), torch.float8_e4m3fn, index, "q")
    scale = torch.empty(scales, dtype=torch.uint8, device=x.device) if scale is None else _output(scale, scales, torch.uint8, index, "scale")
    _check(load_library().moe_quantize_b128(x.data_ptr(), MOE_DTYPE_BF16 if x.dtype == torch.bfloat16 else MOE_DTYPE_F32, stride, matrices, rows, cols,
                                            block_rows, q.data_ptr(), scale.data_ptr(), _stream_on(index)))
    return q, scale


def moe_gemm_b128(a_q, a_scale, w_q, w_scale, offsets=None, a_rows=None, out_dtype=torch.bfloat16, out=None):
    """a_q [a_count, K] and w_q [E, N, K] (or [N, K]) with their scales from moe_quantize_b128 -> [rows, N]; a_rows: which row of a_q each row is
    (None: all, in order); offsets [E + 1] int32: where every expert's rows begin (None: one expert)."""
    if a_q.dim() != 2 or w_q.dim() not in (2, 3):
        raise ValueError("a_q must be [rows, K], w_q [E, N, K]")
    (count, K), N = a_q.shape, w_q.shape[-2]
    E = w_q.shape[0] if w_q.dim() == 3 else 1
    rows = count if a_rows is None else a_rows.shape[0]
    _fit_32_bits(count, rows, E, N, K)
    index = _current_gpu(a_q, "a_q")
    _b128_operand(a_q, a_scale, (count, K), (), 1, index, "a")
    _b128_operand(w_q, w_scale, (*w_q.shape[:-1], K), tuple(w_q.shape[:-2]), 128, index, "w")
    for name, t, shape in (("a_rows", a_rows, (rows,)), ("offsets", offsets, (E + 1,))):
        if t is not None and (tuple(t.shape) != shape or t.dtype != torch.int32 or t.get_device() != index):
            raise ValueError("%s must be %s of int32 on cuda:%d" % (name, list(shape), index))
    if out is not None:
        out_dtype = out.dtype
    if out_dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("out_dtype must be bfloat16 or float32")
    out = torch.empty((rows, N), dtype=out_dtype, device=a_q.device) if out is None else _output(out, (rows, N), out_dtype, index, "out")
    _check(load_library().moe_gemm_b128(a_q.data_ptr(), a_scale.data_ptr(), count, _addr(a_rows), w_q.data_ptr(), w_scale.data_ptr(), _addr(offsets), E, rows, N,
                                        K, out.data_ptr(), MOE_DTYPE_BF16 if out_dtype == torch.bfloat16 else MOE_DTYPE_F32, _stream_on(index)))
    return out
