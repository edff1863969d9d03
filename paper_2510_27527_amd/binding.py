"""ctypes binding of libtjnvfp4.so: argument marshalling only.

Every step of the path (maxima, quantizers, re-quantizers, matrix products) runs in the
library's HIP kernels; this module turns torch CUDA tensors into raw device pointers and
the current torch stream into a hipStream_t.  There is no CPU fallback: if the library is
missing the import fails.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtjnvfp4.so")

ROUND_RTN, ROUND_SR = 0, 1
SCALE_DEFAULT, SCALE_NE, SCALE_UP = 0, 1, 2
OUTER_TENSOR, OUTER_BLOCK128 = 0, 1
SRC_BF16, SRC_NVFP4, SRC_F32, SRC_CKPT8 = 0, 1, 2, 3
OUT_BF16, OUT_F32 = 0, 1
OP_QUANTIZE, OP_GEMM, OP_LINEAR_FWD, OP_LINEAR_BWD_DX, OP_LINEAR_BWD_DW, OP_LINEAR_BWD = 0, 1, 2, 3, 4, 5
NORM_LAYER, NORM_RMS = 0, 1
ACT_SWIGLU, ACT_GELU = 0, 1
ROPE_HALF, ROPE_PAIRS = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_PARTS = 0, 1, 2, 3
KV_BF16, KV_8 = 0, 1
CKPT_GROUP = 128               # elements of a row that share a power of two in an 8-bit checkpoint

EXPORTS = ["nvfp4_quantize", "nvfp4_quantize_dual", "nvfp4_gemm_nt", "nvfp4_gemm_nt_static", "nvfp4_linear_fwd", "nvfp4_linear_bwd_dx", "nvfp4_linear_bwd_dw", "nvfp4_linear_bwd", "nvfp4_osci_update", "nvfp4_osci_suppress", "nvfp4_osci_select", "nvfp4_osci_update_sparse", "nvfp4_osci_suppress_sparse", "nvfp4_osci_select_workspace_bytes", "nvfp4_outctl_fwd", "nvfp4_outctl_bwd", "nvfp4_outctl_workspace_bytes", "nvfp4_outctl_dw_plan", "nvfp4_backward_plan", "nvfp4_backward_product_plan",
           "nvfp4_norm_fwd", "nvfp4_norm_bwd", "nvfp4_norm_workspace_bytes", "nvfp4_act_fwd", "nvfp4_act_bwd", "nvfp4_ckpt8_save", "nvfp4_ckpt8_load", "nvfp4_gemv",
           "nvfp4_rope_frequencies", "nvfp4_rope", "nvfp4_kv_append", "nvfp4_kv_load", "nvfp4_attn", "nvfp4_attn_workspace_bytes", "nvfp4_sample", "nvfp4_sample_workspace_bytes",
           "nvfp4_workspace_bytes", "nvfp4_gemm_plan", "nvfp4_gemm_plan_kernel", "nvfp4_amax_bf16", "nvfp4_stream_key", "nvfp4_strerror", "nvfp4_version"]


class NVFP4Error(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (%d)" % (where, lib().nvfp4_strerror(code).decode(), code))


class CTensor(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("gscale", C.c_void_p), ("amax_deq", C.c_void_p),
                ("rows", C.c_int64), ("K", C.c_int64), ("outer_mode", C.c_int32), ("reserved", C.c_int32)]


class CQcfg(C.Structure):
    _fields_ = [("rounding", C.c_int32), ("scale_round", C.c_int32), ("outer_mode", C.c_int32),
                ("tensor_id", C.c_uint32), ("seed", C.c_uint64), ("amax_in", C.c_void_p), ("rht", C.c_int32),
                ("rht_id", C.c_uint32)]


class CCkpt8(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("exps", C.c_void_p), ("rows", C.c_int64), ("K", C.c_int64)]


# nvfp4_rotation, nvfp4_kvcache and nvfp4_kvbatch as bytes: 0.3 us of the host each, where a ctypes structure takes 1.0 to make.
_ROTATION, _KVCACHE, _KVBATCH = struct.Struct("Pqif"), struct.Struct("PPPPqqqqii"), struct.Struct("PPPPqqq")


class CProductPlan(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("tile_m", "tile_n", "split", "split_waves", "blocked", "together")]


@dataclass(frozen=True)
class ProductPlan:
    """How one product of a backward call is computed: workgroup tile, pieces of the reduction, whether the waves split it, whether the operands
    are blocked along it, whether the call's products share a launch."""
    tile: tuple
    split: int
    split_waves: bool
    blocked: bool
    together: bool


_lib = None


def lib():
    """Load the library (raises OSError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError("libtjnvfp4.so is not built: run `python -m paper_2510_27527_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i64, i32, u64, u32, sz = C.c_void_p, C.c_int64, C.c_int, C.c_uint64, C.c_uint32, C.c_size_t
        L.nvfp4_quantize.restype = i32
        L.nvfp4_quantize.argtypes = [vp, i32, i64, i64, i32, C.POINTER(CQcfg), C.POINTER(CTensor), vp, sz, vp]
        L.nvfp4_quantize_dual.restype = i32
        L.nvfp4_quantize_dual.argtypes = [vp, i64, i64, C.POINTER(CQcfg), u32, C.POINTER(CTensor), C.POINTER(CTensor), vp, sz,
                                          vp]
        L.nvfp4_gemm_nt.restype = i32
        L.nvfp4_gemm_nt.argtypes = [C.POINTER(CTensor), C.POINTER(CTensor), vp, i32, vp, sz, vp]
        L.nvfp4_gemm_nt_static.restype = i32
        L.nvfp4_gemm_nt_static.argtypes = [C.POINTER(CTensor), C.POINTER(CTensor), vp, i32, vp]
        L.nvfp4_linear_fwd.restype = i32
        L.nvfp4_linear_fwd.argtypes = [vp, vp, i64, i64, i64, vp, i32, C.POINTER(CTensor), C.POINTER(CTensor),
                                       i32, vp, sz, vp]
        L.nvfp4_linear_bwd_dx.restype = i32
        L.nvfp4_linear_bwd_dx.argtypes = [vp, C.POINTER(CTensor), i64, i64, i64, vp, i32, u64, u32, i32, vp, sz, vp]
        L.nvfp4_linear_bwd_dw.restype = i32
        L.nvfp4_linear_bwd_dw.argtypes = [vp, C.POINTER(CTensor), i64, i64, i64, vp, i32, u64, u32, i32, vp, sz, vp]
        L.nvfp4_linear_bwd.restype = i32
        L.nvfp4_linear_bwd.argtypes = [vp, C.POINTER(CTensor), C.POINTER(CTensor), i64, i64, i64, vp, vp, i32, u64, u32,
                                       i32, vp, sz, vp]
        L.nvfp4_outctl_fwd.restype = i32
        L.nvfp4_outctl_fwd.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp, i32, C.POINTER(CTensor), C.POINTER(CTensor), i32, vp,
                                       sz, vp]
        L.nvfp4_outctl_bwd.restype = i32
        L.nvfp4_outctl_bwd.argtypes = [vp, C.POINTER(CTensor), C.POINTER(CTensor), vp, vp, i64, i64, i64, i64, vp, vp, vp, vp, i32,
                                       u64, u32, i32, vp, sz, vp]
        L.nvfp4_outctl_workspace_bytes.restype = sz
        L.nvfp4_outctl_workspace_bytes.argtypes = [i32, i64, i64, i64, i64, i32, i32]
        L.nvfp4_osci_update.restype = i32
        L.nvfp4_osci_update.argtypes = [vp, vp, vp, vp, i64, i64, i32, vp]
        L.nvfp4_osci_suppress.restype = i32
        L.nvfp4_osci_suppress.argtypes = [vp, vp, vp, C.c_float, i64, i64, vp, vp]
        L.nvfp4_osci_select_workspace_bytes.restype = C.c_size_t
        L.nvfp4_osci_select_workspace_bytes.argtypes = [i64, i64]
        L.nvfp4_osci_select.restype = i32
        L.nvfp4_osci_select.argtypes = [vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        L.nvfp4_osci_update_sparse.restype = i32
        L.nvfp4_osci_update_sparse.argtypes = [vp, i64, i64, vp, i64, vp, vp, vp, vp, vp]
        L.nvfp4_osci_suppress_sparse.restype = i32
        L.nvfp4_osci_suppress_sparse.argtypes = [vp, i64, i64, vp, i64, vp, vp, C.c_float, vp, vp]
        L.nvfp4_norm_fwd.restype = i32
        L.nvfp4_norm_fwd.argtypes = [vp, i32, i64, i64, i64, vp, vp, C.c_float, i32, vp, i32, i64, vp, vp, vp]
        L.nvfp4_norm_bwd.restype = i32
        L.nvfp4_norm_bwd.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, i64, i64, i32, vp, i32, i64, vp, vp, vp, sz, vp]
        L.nvfp4_norm_workspace_bytes.restype = sz
        L.nvfp4_norm_workspace_bytes.argtypes = [i64, i64]
        L.nvfp4_act_fwd.restype = i32
        L.nvfp4_act_fwd.argtypes = [vp, i32, i64, i64, i64, i32, vp, i32, i64, vp, vp]
        L.nvfp4_act_bwd.restype = i32
        L.nvfp4_act_bwd.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, i32, vp, i32, i64, vp]
        L.nvfp4_ckpt8_save.restype = i32
        L.nvfp4_ckpt8_save.argtypes = [vp, i32, i64, i64, i64, vp, vp]
        L.nvfp4_ckpt8_load.restype = i32
        L.nvfp4_ckpt8_load.argtypes = [vp, vp, i32, i64, vp]
        L.nvfp4_gemv.restype = i32
        L.nvfp4_gemv.argtypes = [vp, i64, i64, vp, vp, i32, i64, vp]
        dbl = C.c_double
        L.nvfp4_rope_frequencies.restype = i32
        L.nvfp4_rope_frequencies.argtypes = [i64, dbl, i32, dbl, dbl, dbl, dbl, vp]
        L.nvfp4_rope.restype = i32
        L.nvfp4_rope.argtypes = [vp, i32, i64, vp, i64, i64, i64, vp, i32, vp, i32, i64, vp]
        L.nvfp4_kv_append.restype = i32
        L.nvfp4_kv_append.argtypes = [vp, i64, i64, vp, i64, vp, i64, i32, i64, vp, vp, vp, vp, i32, i64, vp]
        L.nvfp4_kv_load.restype = i32
        L.nvfp4_kv_load.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, vp]
        L.nvfp4_attn.restype = i32
        L.nvfp4_attn.argtypes = [vp, i64, i64, i64, vp, vp, C.c_float, vp, i64, vp, sz, vp]
        L.nvfp4_attn_workspace_bytes.restype = sz
        L.nvfp4_attn_workspace_bytes.argtypes = [i64] * 8
        L.nvfp4_sample.restype = i32
        L.nvfp4_sample.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.nvfp4_sample_workspace_bytes.restype = sz
        L.nvfp4_sample_workspace_bytes.argtypes = [i64, i64]
        L.nvfp4_workspace_bytes.restype = sz
        L.nvfp4_workspace_bytes.argtypes = [i32, i64, i64, i64, i32]
        L.nvfp4_gemm_plan.restype = i32
        L.nvfp4_gemm_plan.argtypes = [i64, i64, i64, i32, C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_int)]
        L.nvfp4_gemm_plan_kernel.restype = i32
        L.nvfp4_gemm_plan_kernel.argtypes = [i64, i64, i64, i32, C.POINTER(C.c_int)]
        L.nvfp4_backward_plan.restype = i32
        L.nvfp4_backward_plan.argtypes = [i64, i64, i64, i64, i32, C.POINTER(C.c_int), C.POINTER(C.c_int)]
        L.nvfp4_backward_product_plan.restype = i32
        L.nvfp4_backward_product_plan.argtypes = [i32, i64, i64, i64, i64, i32, i32, C.POINTER(CProductPlan)]
        L.nvfp4_outctl_dw_plan.restype = i32
        L.nvfp4_outctl_dw_plan.argtypes = [i64, i64, i64, i64, i32, C.POINTER(C.c_int), C.POINTER(C.c_int)]
        L.nvfp4_amax_bf16.restype = i32
        L.nvfp4_amax_bf16.argtypes = [vp, i64, vp, vp, sz, vp]
        L.nvfp4_stream_key.restype = u64
        L.nvfp4_stream_key.argtypes = [u64, u32]
        L.nvfp4_strerror.restype = C.c_char_p
        L.nvfp4_strerror.argtypes = [i32]
        L.nvfp4_version.restype = C.c_char_p
        L.nvfp4_version.argtypes = []
        _lib = L
    return _lib


def _check(rc: int, where: str):
    if rc != 0:
        raise NVFP4Error(rc, where)


# The current device and its current stream without a Stream object (0.2 us a call instead of 2.8).  torch does not document these two: where
# it does not have them, the documented calls.
try:
    _current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
except AttributeError:
    def _current_device() -> int:
        return torch.cuda.current_device()

    def _raw_stream(device: int) -> int:
        return torch.cuda.current_stream(device).cuda_stream


def _stream() -> int:
    """The current stream of the current device."""
    return _raw_stream(_current_device())


_EMPTY = {}


def _ptr(t: Optional[torch.Tensor]):
    """Device address of a tensor.  An empty tensor has no storage; the library still wants a non-NULL, 16-byte
    aligned pointer for it (it never dereferences it), so it gets the address of a small per-device placeholder."""
    if t is None:
        return None
    p = t.data_ptr()               # 0 for an empty tensor
    if p == 0 and t.is_cuda:
        key = t.device.index
        if key not in _EMPTY:
            _EMPTY[key] = torch.zeros(64, dtype=torch.uint8, device=t.device)
        return _EMPTY[key].data_ptr()
    return p


@dataclass
class NVFP4Tensor:
    """Device buffers of one quantized operand [rows, K] (K contiguous, grouped axis)."""
    codes: torch.Tensor      # uint8 [rows, K/2]
    scales: torch.Tensor     # uint8 [rows, K/16]
    gscale: torch.Tensor     # float32 [1] or [rows, K/128]
    amax_deq: Optional[torch.Tensor]   # float32 [1] or None
    rows: int
    K: int
    outer: int

    def c_struct(self) -> CTensor:
        return CTensor(_ptr(self.codes), _ptr(self.scales), _ptr(self.gscale), _ptr(self.amax_deq),
                       self.rows, self.K, self.outer, 0)


def alloc_nvfp4(rows: int, K: int, outer: int = OUTER_TENSOR, device="cuda", with_amax: bool = True) -> NVFP4Tensor:
    codes = torch.empty((rows, K // 2), dtype=torch.uint8, device=device)
    scales = torch.empty((rows, K // 16), dtype=torch.uint8, device=device)
    gshape = (1,) if outer == OUTER_TENSOR else (rows, max(K // 128, 1))
    gscale = torch.empty(gshape, dtype=torch.float32, device=device)
    amax = torch.zeros((1,), dtype=torch.float32, device=device) if with_amax else None
    return NVFP4Tensor(codes, scales, gscale, amax, rows, K, outer)


def workspace_bytes(op: int, N: int, D: int, Cc: int, outer: int = OUTER_TENSOR) -> int:
    return int(lib().nvfp4_workspace_bytes(op, N, D, Cc, outer))


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty((max(int(nbytes), 16),), dtype=torch.uint8, device=device)


def gemm_plan(M: int, N: int, K: int, outer: int = OUTER_TENSOR):
    """(tile rows, tile columns, K splits) nvfp4_gemm_nt will use for this shape and outer mode."""
    a, b, c = C.c_int(), C.c_int(), C.c_int()
    _check(lib().nvfp4_gemm_plan(M, N, K, outer, C.byref(a), C.byref(b), C.byref(c)), "nvfp4_gemm_plan")
    return a.value, b.value, c.value


def gemm_splits_waves(M: int, N: int, K: int, outer: int = OUTER_TENSOR) -> bool:
    """Whether the planned launch runs the kernel whose waves split the reduction."""
    a = C.c_int(0)
    _check(lib().nvfp4_gemm_plan_kernel(M, N, K, outer, C.byref(a)), "nvfp4_gemm_plan_kernel")
    return bool(a.value)


def backward_plan(N: int, D_lo: int, D_hp: int, Cc: int, outer: int = OUTER_TENSOR):
    """The workgroup tile of a backward call's products where they share a launch, (0, 0) where they do not."""
    a, b = C.c_int(0), C.c_int(0)
    _check(lib().nvfp4_backward_plan(N, D_lo, D_hp, Cc, outer, C.byref(a), C.byref(b)), "nvfp4_backward_plan")
    return a.value, b.value


def backward_product_plan(op: int, N: int, D_lo: int, D_hp: int, Cc: int, outer: int, product: int) -> ProductPlan:
    """Product 0 (dX), 1 (dW) or 2 (dX of the outlier channels) of a backward call: op OP_LINEAR_BWD_DX, _DW or _BWD."""
    p = CProductPlan()
    _check(lib().nvfp4_backward_product_plan(op, N, D_lo, D_hp, Cc, outer, product, C.byref(p)), "nvfp4_backward_product_plan")
    return ProductPlan((p.tile_m, p.tile_n), p.split, bool(p.split_waves), bool(p.blocked), bool(p.together))


def outctl_dw_plan(N: int, D_lo: int, D_hp: int, Cc: int, outer: int = OUTER_TENSOR):
    """(splits, 32-token stages per split) of the outlier channels' weight gradient in nvfp4_outctl_bwd."""
    a, b = C.c_int(), C.c_int()
    _check(lib().nvfp4_outctl_dw_plan(N, D_lo, D_hp, Cc, outer, C.byref(a), C.byref(b)), "nvfp4_outctl_dw_plan")
    return a.value, b.value


def stream_key(seed: int, tensor_id: int) -> int:
    return int(lib().nvfp4_stream_key(seed, tensor_id))


def amax_bf16(src: torch.Tensor, ws: torch.Tensor) -> torch.Tensor:
    out = torch.empty((1,), dtype=torch.float32, device=src.device)
    _check(lib().nvfp4_amax_bf16(_ptr(src), src.numel(), _ptr(out), _ptr(ws), ws.numel(), _stream()), "nvfp4_amax_bf16")
    return out


def quantize(src, axis: int, rounding: int, out: Optional[NVFP4Tensor] = None, *, scale_round: int = SCALE_DEFAULT,
             outer: int = OUTER_TENSOR, seed: int = 0, tensor_id: int = 0, amax_in: Optional[torch.Tensor] = None,
             ws: Optional[torch.Tensor] = None, rht_id: Optional[int] = None) -> NVFP4Tensor:
    """nvfp4_quantize: src is a bf16 [R, C] tensor or an NVFP4Tensor."""
    if isinstance(src, NVFP4Tensor):
        kind, R, Cc = SRC_NVFP4, src.rows, src.K
        cs = src.c_struct()
        src_arg = C.cast(C.pointer(cs), C.c_void_p)
        dev = src.codes.device
    else:
        assert src.dtype == torch.bfloat16 and src.dim() == 2 and src.is_contiguous()
        kind, (R, Cc) = SRC_BF16, src.shape
        src_arg = _ptr(src)
        dev = src.device
    rows, K = (R, Cc) if axis == 0 else (Cc, R)
    if out is None:
        out = alloc_nvfp4(rows, K, outer, dev)
    if ws is None:
        ws = alloc_workspace(workspace_bytes(OP_QUANTIZE, R, Cc, 0, outer), dev)
    cfg = CQcfg(rounding, scale_round, outer, tensor_id, seed, _ptr(amax_in), 0 if rht_id is None else 1, rht_id or 0)
    co = out.c_struct()
    rc = lib().nvfp4_quantize(src_arg, kind, R, Cc, axis, C.byref(cfg), C.byref(co), _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_quantize")
    out.rows, out.K, out.outer = co.rows, co.K, co.outer_mode
    return out


def quantize_dual(src: torch.Tensor, rounding: int, out_row: Optional[NVFP4Tensor] = None,
                  out_col: Optional[NVFP4Tensor] = None, *, scale_round: int = SCALE_DEFAULT, seed: int = 0,
                  tensor_id_row: int = 0, tensor_id_col: int = 0, amax_in: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None):
    """nvfp4_quantize_dual: row-wise [R, C] and column-wise [C, R] operands of a bf16 [R, C] tensor from one read."""
    assert src.dtype == torch.bfloat16 and src.dim() == 2 and src.is_contiguous()
    R, Cc = src.shape
    dev = src.device
    if out_row is None:
        out_row = alloc_nvfp4(R, Cc, OUTER_TENSOR, dev)
    if out_col is None:
        out_col = alloc_nvfp4(Cc, R, OUTER_TENSOR, dev)
    if ws is None:
        ws = alloc_workspace(workspace_bytes(OP_QUANTIZE, R, Cc, 0, OUTER_TENSOR), dev)
    cfg = CQcfg(rounding, scale_round, OUTER_TENSOR, tensor_id_row, seed, _ptr(amax_in), 0, 0)
    cr, cc = out_row.c_struct(), out_col.c_struct()
    rc = lib().nvfp4_quantize_dual(_ptr(src), R, Cc, C.byref(cfg), tensor_id_col, C.byref(cr), C.byref(cc), _ptr(ws),
                                   ws.numel(), _stream())
    _check(rc, "nvfp4_quantize_dual")
    out_row.rows, out_row.K, out_row.outer = cr.rows, cr.K, cr.outer_mode
    out_col.rows, out_col.K, out_col.outer = cc.rows, cc.K, cc.outer_mode
    return out_row, out_col


def _check_bf16(t: torch.Tensor, what: str):
    assert t.dtype == torch.bfloat16 and t.dim() == 2 and t.is_contiguous() and t.is_cuda, what + ": bf16, 2-D, contiguous, on the GPU"


def _check_out(t: torch.Tensor, shape, out_dtype: int, what: str):
    want = torch.bfloat16 if out_dtype == OUT_BF16 else torch.float32
    assert t.dtype == want and tuple(t.shape) == tuple(shape) and t.is_contiguous() and t.is_cuda, what


def _out_tensor(M, N, out_dtype, device):
    return torch.empty((M, N), dtype=torch.bfloat16 if out_dtype == OUT_BF16 else torch.float32, device=device)


def gemm_nt(A: NVFP4Tensor, B: NVFP4Tensor, out_dtype: int = OUT_BF16, out: Optional[torch.Tensor] = None,
            ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    dev = A.codes.device
    if out is None:
        out = _out_tensor(A.rows, B.rows, out_dtype, dev)
    if ws is None:
        ws = alloc_workspace(workspace_bytes(OP_GEMM, A.rows, A.K, B.rows, A.outer), dev)
    ca, cb = A.c_struct(), B.c_struct()
    rc = lib().nvfp4_gemm_nt(C.byref(ca), C.byref(cb), _ptr(out), out_dtype, _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_gemm_nt")
    return out


STATIC_SCRATCH_BYTES = 64 << 20
ERR_SCRATCH = -8


def gemm_nt_static(A: NVFP4Tensor, B: NVFP4Tensor, out: torch.Tensor, out_dtype: int = OUT_BF16) -> torch.Tensor:
    """nvfp4_gemm_nt_static: the product with the library's static scratch array; `out` is the caller's."""
    _check_out(out, (A.rows, B.rows), out_dtype, "out")
    ca, cb = A.c_struct(), B.c_struct()
    rc = lib().nvfp4_gemm_nt_static(C.byref(ca), C.byref(cb), _ptr(out), out_dtype, _stream())
    _check(rc, "nvfp4_gemm_nt_static")
    return out


def linear_fwd(X: torch.Tensor, W: torch.Tensor, out_dtype: int = OUT_BF16, *, Y: Optional[torch.Tensor] = None,
               Xq: Optional[NVFP4Tensor] = None, Wq: Optional[NVFP4Tensor] = None,
               ws: Optional[torch.Tensor] = None, outer: int = OUTER_TENSOR):
    _check_bf16(X, "X")
    _check_bf16(W, "W")
    N, D = X.shape
    Cc, D2 = W.shape
    assert D == D2
    dev = X.device
    Y = _out_tensor(N, Cc, out_dtype, dev) if Y is None else Y
    _check_out(Y, (N, Cc), out_dtype, "Y")
    Xq = alloc_nvfp4(N, D, outer, dev) if Xq is None else Xq
    Wq = alloc_nvfp4(Cc, D, outer, dev) if Wq is None else Wq
    ws = alloc_workspace(workspace_bytes(OP_LINEAR_FWD, N, D, Cc, outer), dev) if ws is None else ws
    cx, cw = Xq.c_struct(), Wq.c_struct()
    rc = lib().nvfp4_linear_fwd(_ptr(X), _ptr(W), N, D, Cc, _ptr(Y), out_dtype, C.byref(cx), C.byref(cw), outer,
                                _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_linear_fwd")
    Xq.rows, Xq.K, Xq.outer = cx.rows, cx.K, cx.outer_mode
    Wq.rows, Wq.K, Wq.outer = cw.rows, cw.K, cw.outer_mode
    return Y, Xq, Wq


def linear_bwd_dx(dY: torch.Tensor, Wq: NVFP4Tensor, seed: int, layer_id: int, out_dtype: int = OUT_BF16, *,
                  dX: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, rht: bool = False) -> torch.Tensor:
    _check_bf16(dY, "dY")
    N, Cc = dY.shape
    D = Wq.K
    dev = dY.device
    dX = _out_tensor(N, D, out_dtype, dev) if dX is None else dX
    _check_out(dX, (N, D), out_dtype, "dX")
    ws = alloc_workspace(workspace_bytes(OP_LINEAR_BWD_DX, N, D, Cc, Wq.outer), dev) if ws is None else ws
    cw = Wq.c_struct()
    rc = lib().nvfp4_linear_bwd_dx(_ptr(dY), C.byref(cw), N, D, Cc, _ptr(dX), out_dtype, seed, layer_id, int(rht),
                                   _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_linear_bwd_dx")
    return dX


def linear_bwd_dw(dY: torch.Tensor, Xq: NVFP4Tensor, seed: int, layer_id: int, out_dtype: int = OUT_BF16, *,
                  dW: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, rht: bool = False) -> torch.Tensor:
    _check_bf16(dY, "dY")
    N, Cc = dY.shape
    D = Xq.K
    dev = dY.device
    dW = _out_tensor(Cc, D, out_dtype, dev) if dW is None else dW
    _check_out(dW, (Cc, D), out_dtype, "dW")
    ws = alloc_workspace(workspace_bytes(OP_LINEAR_BWD_DW, N, D, Cc, Xq.outer), dev) if ws is None else ws
    cx = Xq.c_struct()
    rc = lib().nvfp4_linear_bwd_dw(_ptr(dY), C.byref(cx), N, D, Cc, _ptr(dW), out_dtype, seed, layer_id, int(rht),
                                   _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_linear_bwd_dw")
    return dW


def linear_bwd(dY: torch.Tensor, Xq: NVFP4Tensor, Wq: NVFP4Tensor, seed: int, layer_id: int, out_dtype: int = OUT_BF16, *,
               dX: Optional[torch.Tensor] = None, dW: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
               rht: bool = False):
    """nvfp4_linear_bwd: both gradients, dY read once for its maximum and once for both quantizations."""
    _check_bf16(dY, "dY")
    N, Cc = dY.shape
    D = Xq.K
    dev = dY.device
    dX = _out_tensor(N, D, out_dtype, dev) if dX is None else dX
    dW = _out_tensor(Cc, D, out_dtype, dev) if dW is None else dW
    _check_out(dX, (N, D), out_dtype, "dX")
    _check_out(dW, (Cc, D), out_dtype, "dW")
    ws = alloc_workspace(workspace_bytes(OP_LINEAR_BWD, N, D, Cc, Xq.outer), dev) if ws is None else ws
    cx, cw = Xq.c_struct(), Wq.c_struct()
    rc = lib().nvfp4_linear_bwd(_ptr(dY), C.byref(cx), C.byref(cw), N, D, Cc, _ptr(dX), _ptr(dW), out_dtype, seed,
                                layer_id, int(rht), _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_linear_bwd")
    return dX, dW


def _check_f32(t: torch.Tensor, shape, what: str):
    assert t.dtype == torch.float32 and tuple(t.shape) == tuple(shape) and t.is_contiguous() and t.is_cuda, what


def osci_update(W: torch.Tensor, W_prev: torch.Tensor, dist_m: torch.Tensor, dist_q: torch.Tensor, t0: int):
    """nvfp4_osci_update: one step of the oscillation statistics of a float32 [C, D] weight, in place."""
    Cc, D = W.shape
    for t, n in ((W, "W"), (W_prev, "W_prev"), (dist_m, "dist_m"), (dist_q, "dist_q")):
        _check_f32(t, (Cc, D), n)
    _check(lib().nvfp4_osci_update(_ptr(W), _ptr(W_prev), _ptr(dist_m), _ptr(dist_q), Cc, D, t0, _stream()), "nvfp4_osci_update")


def osci_suppress(W: torch.Tensor, dist_m: torch.Tensor, dist_q: torch.Tensor, tau: float,
                  n_reset: Optional[torch.Tensor] = None):
    """nvfp4_osci_suppress: reset the oscillating elements of W in place; n_reset (int64 [1], optional) accumulates
    their number."""
    Cc, D = W.shape
    for t, n in ((W, "W"), (dist_m, "dist_m"), (dist_q, "dist_q")):
        _check_f32(t, (Cc, D), n)
    if n_reset is not None:
        assert n_reset.dtype == torch.int64 and n_reset.numel() == 1 and n_reset.is_cuda
    _check(lib().nvfp4_osci_suppress(_ptr(W), _ptr(dist_m), _ptr(dist_q), tau, Cc, D, _ptr(n_reset), _stream()),
           "nvfp4_osci_suppress")


def _check_subset(k: int, idx, *states):
    assert idx.dtype == torch.int32 and idx.numel() == k and idx.is_contiguous() and idx.is_cuda, "idx"
    for t in states:
        assert t.dtype == torch.float32 and t.numel() == k and t.is_contiguous() and t.is_cuda, "subset state"


def osci_select(W: torch.Tensor, k: int):
    """nvfp4_osci_select (Appendix Alg. 3, first step of a period): returns (idx, W_prev_s, Q_prev_s, dist_m_s, dist_q_s)
    of the k weights with the largest sensitivity scores; idx holds 32-bit flat indices (int32 storage, read as unsigned)."""
    Cc, D = W.shape
    _check_f32(W, (Cc, D), "W")
    idx = torch.empty(k, dtype=torch.int32, device=W.device)
    st = [torch.empty(k, dtype=torch.float32, device=W.device) for _ in range(4)]
    nbytes = lib().nvfp4_osci_select_workspace_bytes(Cc, D)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=W.device)
    _check(lib().nvfp4_osci_select(_ptr(W), Cc, D, k, _ptr(idx), *[_ptr(t) for t in st], _ptr(ws), ws.numel(), _stream()),
           "nvfp4_osci_select")
    return (idx, *st)


def osci_update_sparse(W, idx, W_prev_s, Q_prev_s, dist_m_s, dist_q_s):
    """nvfp4_osci_update_sparse: a later step of the period, in place on the four subset states."""
    Cc, D = W.shape
    _check_f32(W, (Cc, D), "W")
    _check_subset(idx.numel(), idx, W_prev_s, Q_prev_s, dist_m_s, dist_q_s)
    _check(lib().nvfp4_osci_update_sparse(_ptr(W), Cc, D, _ptr(idx), idx.numel(), _ptr(W_prev_s), _ptr(Q_prev_s), _ptr(dist_m_s),
                                          _ptr(dist_q_s), _stream()), "nvfp4_osci_update_sparse")


def osci_suppress_sparse(W, idx, dist_m_s, dist_q_s, tau: float, n_reset: Optional[torch.Tensor] = None):
    """nvfp4_osci_suppress_sparse: reset the oscillating tracked elements of W in place."""
    Cc, D = W.shape
    _check_f32(W, (Cc, D), "W")
    _check_subset(idx.numel(), idx, dist_m_s, dist_q_s)
    if n_reset is not None:
        assert n_reset.dtype == torch.int64 and n_reset.numel() == 1 and n_reset.is_cuda
    _check(lib().nvfp4_osci_suppress_sparse(_ptr(W), Cc, D, _ptr(idx), idx.numel(), _ptr(dist_m_s), _ptr(dist_q_s), tau,
                                            _ptr(n_reset), _stream()), "nvfp4_osci_suppress_sparse")


def outctl_fwd(X_lo, W_lo, X_hp, W_hp, out_dtype: int = OUT_BF16, *, outer: int = OUTER_TENSOR, Y=None, Xq=None, Wq=None, ws=None):
    """nvfp4_outctl_fwd: Y = Q1(X_lo) Q2(W_lo)^T + X_hp W_hp^T (Sec. 4.2); returns (Y, Xq, Wq) of the ordinary channels."""
    for t, n in ((X_lo, "X_lo"), (W_lo, "W_lo"), (X_hp, "X_hp"), (W_hp, "W_hp")):
        _check_bf16(t, n)
    N, D_lo = X_lo.shape
    Cc, D_hp = W_hp.shape
    assert W_lo.shape == (Cc, D_lo) and X_hp.shape == (N, D_hp)
    dev = X_lo.device
    Y = _out_tensor(N, Cc, out_dtype, dev) if Y is None else Y
    _check_out(Y, (N, Cc), out_dtype, "Y")
    Xq = alloc_nvfp4(N, D_lo, outer, dev) if Xq is None else Xq
    Wq = alloc_nvfp4(Cc, D_lo, outer, dev) if Wq is None else Wq
    if ws is None:
        ws = alloc_workspace(lib().nvfp4_outctl_workspace_bytes(0, N, D_lo, D_hp, Cc, outer, out_dtype), dev)
    cx, cw = Xq.c_struct(), Wq.c_struct()
    rc = lib().nvfp4_outctl_fwd(_ptr(X_lo), _ptr(W_lo), _ptr(X_hp), _ptr(W_hp), N, D_lo, D_hp, Cc, _ptr(Y), out_dtype,
                                C.byref(cx), C.byref(cw), outer, _ptr(ws), ws.numel(), _stream())
    _check(rc, "nvfp4_outctl_fwd")
    Xq.rows, Xq.K, Xq.outer = cx.rows, cx.K, cx.outer_mode
    Wq.rows, Wq.K, Wq.outer = cw.rows, cw.K, cw.outer_mode
    return Y, Xq, Wq


def outctl_bwd(dY, Xq: NVFP4Tensor, Wq: NVFP4Tensor, X_hp, W_hp, seed: int, layer_id: int, out_dtype: int = OUT_BF16, *,
               rht: bool = False, ws=None, outs=None):
    """nvfp4_outctl_bwd: returns (dX_lo, dX_hp, dW_lo, dW_hp) (written into `outs` when given)."""
    for t, n in ((dY, "dY"), (X_hp, "X_hp"), (W_hp, "W_hp")):
        _check_bf16(t, n)
    N, Cc = dY.shape
    D_lo, D_hp = Xq.K, X_hp.shape[1]
    dev = dY.device
    shapes = [(N, D_lo), (N, D_hp), (Cc, D_lo), (Cc, D_hp)]
    if outs is None:
        outs = [_out_tensor(a, b, out_dtype, dev) for a, b in shapes]
    for t, sh in zip(outs, shapes):
        _check_out(t, sh, out_dtype, "gradient output")
    if ws is None:
        ws = alloc_workspace(lib().nvfp4_outctl_workspace_bytes(1, N, D_lo, D_hp, Cc, Xq.outer, out_dtype), dev)
    cx, cw = Xq.c_struct(), Wq.c_struct()
    rc = lib().nvfp4_outctl_bwd(_ptr(dY), C.byref(cx), C.byref(cw), _ptr(X_hp), _ptr(W_hp), N, D_lo, D_hp, Cc, _ptr(outs[0]),
                                _ptr(outs[1]), _ptr(outs[2]), _ptr(outs[3]), out_dtype, seed, layer_id, int(rht), _ptr(ws),
                                ws.numel(), _stream())
    _check(rc, "nvfp4_outctl_bwd")
    return tuple(outs)


# ---- operators around the linears: norms, nonlinearities, 8-bit checkpoints, the linear of single tokens ----
#
# They are enqueued on the current device's current stream, and every tensor has to be on that device (`dev` below): a kernel of
# another device might not reach it.

@dataclass
class Ckpt8:
    """Device buffers of an 8-bit checkpoint of a [rows, K] array."""
    codes: torch.Tensor      # uint8 [rows, K]: E4M3 codes
    exps: torch.Tensor       # uint8 [rows, ceil(K / 128)]: 127 + e, the values being code * 2^e
    rows: int
    K: int

    def c_struct(self) -> CCkpt8:
        return CCkpt8(_ptr(self.codes), _ptr(self.exps), self.rows, self.K)


def alloc_ckpt8(rows: int, K: int, device="cuda") -> Ckpt8:
    return Ckpt8(torch.empty((rows, K), dtype=torch.uint8, device=device),
                 torch.empty((rows, -(-K // CKPT_GROUP)), dtype=torch.uint8, device=device), rows, K)


def alloc_act_ckpt8(N: int, F: int, act: int, device="cuda") -> Ckpt8:
    """The checkpoint of a nonlinearity's input: the gates and the up values of a token are rows of their own (SwiGLU)."""
    return alloc_ckpt8(2 * N if act == ACT_SWIGLU else N, F, device)


def alloc_stats(N: int, device="cuda") -> torch.Tensor:
    """The statistics of a norm's rows (mean, 1 / deviation) that its backward pass reads."""
    return torch.empty((N, 2), dtype=torch.float32, device=device)


_BF16, _F32, _U8, _I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32
_KINDS = {torch.bfloat16: SRC_BF16, torch.float32: SRC_F32}


def _rows(t: torch.Tensor, what: str, dev: int):
    """(kind, row stride, rows, elements of a row) of a bf16 or float32 matrix whose rows are contiguous; the rows may be any distance apart."""
    kind = _KINDS.get(t.dtype)
    shape = t.shape
    assert kind is not None and len(shape) == 2 and t.get_device() == dev, what + ": bf16 or float32, 2-D, on the current device"
    rows, n = shape
    s0, s1 = t.stride()
    assert s1 == 1 or n <= 1, what + ": rows of contiguous elements"
    return kind, s0 if rows > 1 else n, rows, n


def _out_rows(t: Optional[torch.Tensor], rows: int, n: int, out_dtype: int, like: torch.Tensor, what: str, dev: int):
    """The output matrix, allocated on like's device where none is given, and its row stride."""
    if t is None:
        dtype = torch.bfloat16 if out_dtype == OUT_BF16 else torch.float32
        if dtype == like.dtype:              # 0.3 us of the host's less
            return like.new_empty((rows, n)), n
        return torch.empty((rows, n), dtype=dtype, device=like.device), n
    kind, ld, r, c = _rows(t, what, dev)
    assert r == rows and c == n and kind == (SRC_BF16 if out_dtype == OUT_BF16 else SRC_F32), what
    return t, ld


def _param(t: Optional[torch.Tensor], D: int, what: str, dev: int):
    assert t is None or (t.dtype == torch.float32 and t.dim() == 1 and t.numel() == D and t.is_contiguous() and t.get_device() == dev), what + ": float32 [D], on the current device"
    return _ptr(t)


def _check_ckpt(c: Ckpt8, rows: int, K: int, dev: int):
    assert c.rows == rows and c.K == K, "checkpoint of another shape"
    for t, shape in ((c.codes, (rows, K)), (c.exps, (rows, -(-K // CKPT_GROUP)))):
        assert t.dtype == torch.uint8 and tuple(t.shape) == shape and t.is_contiguous() and t.get_device() == dev, "checkpoint buffers, on the current device"


def _check_stats(t: torch.Tensor, N: int, dev: int):
    assert t.dtype == torch.float32 and tuple(t.shape) == (N, 2) and t.is_contiguous() and t.get_device() == dev, "stats: float32 [N, 2], on the current device"


def norm_fwd(X: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, *, eps: float = 1e-5,
             norm: int = NORM_LAYER, out_dtype: int = OUT_BF16, Y: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
             ckpt: Optional[Ckpt8] = None) -> torch.Tensor:
    """nvfp4_norm_fwd: layer norm (NORM_LAYER) or RMS norm (NORM_RMS) of every row of X.  For training pass stats (alloc_stats) and, to keep
    the input in 8 bits, ckpt (alloc_ckpt8); both are filled."""
    dev = _current_device()
    kind, ldx, N, D = _rows(X, "X", dev)
    Y, ldy = _out_rows(Y, N, D, out_dtype, X, "Y", dev)
    cs = None
    if ckpt is not None:
        _check_ckpt(ckpt, N, D, dev)
        cs = C.byref(ckpt.c_struct())
    if stats is not None:
        _check_stats(stats, N, dev)
    _check(lib().nvfp4_norm_fwd(_ptr(X), kind, ldx, N, D, _param(gamma, D, "gamma", dev), _param(beta, D, "beta", dev), eps, norm, _ptr(Y), out_dtype,
                                ldy, _ptr(stats), cs, _raw_stream(dev)), "nvfp4_norm_fwd")
    return Y


def norm_bwd(dY: torch.Tensor, X, stats: torch.Tensor, gamma: Optional[torch.Tensor] = None, *, norm: int = NORM_LAYER,
             out_dtype: int = OUT_BF16, dX: Optional[torch.Tensor] = None, dgamma: Optional[torch.Tensor] = None,
             dbeta: Optional[torch.Tensor] = None, params: bool = True, ws: Optional[torch.Tensor] = None):
    """nvfp4_norm_bwd: (dX, dgamma, dbeta); X is the forward call's input or its Ckpt8.  params=False: dX alone; RMS norm has no dbeta
    unless one is passed."""
    dev = _current_device()
    dkind, lddy, N, D = _rows(dY, "dY", dev)
    if isinstance(X, Ckpt8):
        _check_ckpt(X, N, D, dev)
        kind, ldx, src = SRC_CKPT8, 0, C.byref(X.c_struct())
    else:
        kind, ldx, *shape = _rows(X, "X", dev)
        assert shape == [N, D], "X: the shape of dY"
        src = _ptr(X)
    _check_stats(stats, N, dev)
    dX, lddx = _out_rows(dX, N, D, out_dtype, dY, "dX", dev)
    if params:
        dgamma = stats.new_empty(D) if dgamma is None else dgamma
        if dbeta is None and norm == NORM_LAYER:
            dbeta = stats.new_empty(D)
        if ws is None:
            ws = alloc_workspace(lib().nvfp4_norm_workspace_bytes(N, D), dY.device)
        else:
            assert ws.get_device() == dev, "ws: on the current device"
    else:
        dgamma = dbeta = None
    _check(lib().nvfp4_norm_bwd(_ptr(dY), dkind, lddy, src, kind, ldx, _ptr(stats), _param(gamma, D, "gamma", dev), N, D, norm, _ptr(dX), out_dtype,
                                lddx, _param(dgamma, D, "dgamma", dev), _param(dbeta, D, "dbeta", dev), _ptr(ws), 0 if ws is None else ws.numel(),
                                _raw_stream(dev)), "nvfp4_norm_bwd")
    return dX, dgamma, dbeta


def act_fwd(H: torch.Tensor, act: int = ACT_SWIGLU, out_dtype: int = OUT_BF16, *, A: Optional[torch.Tensor] = None,
            ckpt: Optional[Ckpt8] = None) -> torch.Tensor:
    """nvfp4_act_fwd: SwiGLU of H [N, 2F] (gates, then up values) or GELU (tanh form) of H [N, F]; ckpt (alloc_act_ckpt8) receives H in 8 bits."""
    dev = _current_device()
    kind, ldh, N, F = _rows(H, "H", dev)
    if act == ACT_SWIGLU:
        assert F % 2 == 0, "H: gates and up values"
        F //= 2
    A, lda = _out_rows(A, N, F, out_dtype, H, "A", dev)
    cs = None
    if ckpt is not None:
        _check_ckpt(ckpt, 2 * N if act == ACT_SWIGLU else N, F, dev)
        cs = C.byref(ckpt.c_struct())
    _check(lib().nvfp4_act_fwd(_ptr(H), kind, ldh, N, F, act, _ptr(A), out_dtype, lda, cs, _raw_stream(dev)), "nvfp4_act_fwd")
    return A


def act_bwd(dA: torch.Tensor, H, act: int = ACT_SWIGLU, out_dtype: int = OUT_BF16, *, dH: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nvfp4_act_bwd: dH from dA and the forward call's input or its Ckpt8."""
    dev = _current_device()
    dkind, ldda, N, F = _rows(dA, "dA", dev)
    parts = 2 if act == ACT_SWIGLU else 1
    if isinstance(H, Ckpt8):
        _check_ckpt(H, parts * N, F, dev)
        kind, ldh, src = SRC_CKPT8, 0, C.byref(H.c_struct())
    else:
        kind, ldh, *shape = _rows(H, "H", dev)
        assert shape == [N, parts * F], "H"
        src = _ptr(H)
    dH, lddh = _out_rows(dH, N, parts * F, out_dtype, dA, "dH", dev)
    _check(lib().nvfp4_act_bwd(_ptr(dA), dkind, ldda, src, kind, ldh, N, F, act, _ptr(dH), out_dtype, lddh, _raw_stream(dev)), "nvfp4_act_bwd")
    return dH


def ckpt8_save(X: torch.Tensor, out: Optional[Ckpt8] = None) -> Ckpt8:
    """nvfp4_ckpt8_save: an activation [N, D] in 8 bits."""
    dev = _current_device()
    kind, ldx, N, D = _rows(X, "X", dev)
    out = alloc_ckpt8(N, D, X.device) if out is None else out
    _check_ckpt(out, N, D, dev)
    _check(lib().nvfp4_ckpt8_save(_ptr(X), kind, ldx, N, D, C.byref(out.c_struct()), _raw_stream(dev)), "nvfp4_ckpt8_save")
    return out


def ckpt8_load(src: Ckpt8, out_dtype: int = OUT_BF16, *, Y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nvfp4_ckpt8_load: the activation that a checkpoint holds."""
    dev = _current_device()
    _check_ckpt(src, src.rows, src.K, dev)
    Y, ldy = _out_rows(Y, src.rows, src.K, out_dtype, src.codes, "Y", dev)
    _check(lib().nvfp4_ckpt8_load(C.byref(src.c_struct()), _ptr(Y), out_dtype, ldy, _raw_stream(dev)), "nvfp4_ckpt8_load")
    return Y


def gemv(X: torch.Tensor, W: NVFP4Tensor, out_dtype: int = OUT_BF16, *, Y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nvfp4_gemv: Y = X W^T for the bf16 activations of a few tokens on packed weights (linear_fwd's Wq)."""
    dev = _current_device()
    kind, ldx, M, K = _rows(X, "X", dev)
    assert kind == SRC_BF16 and K == W.K, "X: bf16 [M, W.K]"
    assert W.codes.get_device() == W.scales.get_device() == W.gscale.get_device() == dev, "W: on the current device"
    Y, ldy = _out_rows(Y, M, W.rows, out_dtype, X, "Y", dev)
    _check(lib().nvfp4_gemv(_ptr(X), ldx, M, C.byref(W.c_struct()), _ptr(Y), out_dtype, ldy, _raw_stream(dev)), "nvfp4_gemv")
    return Y


# ---- operators on sequences of tokens: rotary positions, the paged cache of keys and values, attention over it, sampling ----
#
# As above: on the current device's current stream, every tensor on that device.

def rope_frequencies(R: int, base: float = 10000.0, *, scaling: int = ROPE_PLAIN, factor: float = 1.0, trained: float = 0.0, low: float = 1.0, high: float = 32.0,
                     device="cuda") -> torch.Tensor:
    """nvfp4_rope_frequencies: float32 [R / 2], scaled for contexts `factor` times as long as the trained ones."""
    f = torch.empty(max(R, 0) // 2, dtype=torch.float32)
    _check(lib().nvfp4_rope_frequencies(R, base, scaling, factor, trained, low, high, f.data_ptr()), "nvfp4_rope_frequencies")
    return f.to(device)


@dataclass
class Rope:
    """Rotary positions of a head's first 2 * freqs.numel() elements."""
    freqs: torch.Tensor      # float32 [R / 2]
    form: int = ROPE_HALF
    scale: float = 1.0       # of cosine and sine

    def packed(self, dev: int) -> bytes:
        f = self.freqs
        assert f.dtype == _F32 and f.dim() == 1 and f.is_contiguous() and f.get_device() == dev, "freqs: float32 [R / 2], on the current device"
        return _ROTATION.pack(f.data_ptr() or _ptr(f) or 0, 2 * f.numel(), self.form, self.scale)


@dataclass
class KVCache:
    """Pages of keys and values: [pages, heads, tokens of a page, D], bf16, or E4M3 codes (uint8) with exponents [.., ceil(D / 128)]."""
    k: torch.Tensor
    v: torch.Tensor
    k_exps: Optional[torch.Tensor] = None
    v_exps: Optional[torch.Tensor] = None

    def packed(self, dev: int) -> bytes:
        k, v, ke, ve = self.k, self.v, self.k_exps, self.v_exps
        shape, dtype = k.shape, k.dtype
        assert len(shape) == 4 and v.shape == shape and v.dtype == dtype and (dtype == _BF16 or dtype == _U8), "cache: bf16 or uint8 [pages, heads, page, D], keys and values alike"
        assert k.is_contiguous() and v.is_contiguous() and k.get_device() == dev == v.get_device(), "cache: contiguous, on the current device"
        pages, heads, page, D = shape
        if dtype == _BF16:
            assert ke is None and ve is None, "exponents: of an 8-bit cache alone"
            return _KVCACHE.pack(k.data_ptr() or _ptr(k) or 0, v.data_ptr() or _ptr(v) or 0, 0, 0, pages, heads, page, D, KV_BF16, 0)
        for e in (ke, ve):
            assert e is not None and e.dtype == _U8 and e.shape == (pages, heads, page, -(-D // CKPT_GROUP)) and e.is_contiguous() and e.get_device() == dev, "exponents of an 8-bit cache, on the current device"
        return _KVCACHE.pack(*(t.data_ptr() or _ptr(t) or 0 for t in (k, v, ke, ve)), pages, heads, page, D, KV_8, 0)


def alloc_kv_cache(pages: int, heads: int, page: int, D: int, kind: int = KV_BF16, device="cuda") -> KVCache:
    if kind == KV_BF16:
        return KVCache(*(torch.empty((pages, heads, page, D), dtype=torch.bfloat16, device=device) for _ in range(2)))
    u8 = lambda n: [torch.empty((pages, heads, page, n), dtype=torch.uint8, device=device) for _ in range(2)]
    return KVCache(*u8(D), *u8(-(-D // CKPT_GROUP)))


@dataclass
class KVBatch:
    """A batch of sequences (nvfp4_kvbatch): int32 tensors on the device."""
    table: torch.Tensor                           # [B, width]: pages of the sequences' own tokens
    lens: torch.Tensor                            # [B]: own tokens, the call's among them
    starts: Optional[torch.Tensor] = None         # [B + 1]: rows of the call; None: one each
    prefix_table: Optional[torch.Tensor] = None   # pages of the tokens that all sequences share
    prefix: int = 0                               # how many those are

    def packed(self, dev: int, page: int) -> bytes:
        table, lens, starts, prefix_table, prefix = self.table, self.lens, self.starts, self.prefix_table, self.prefix
        shape = table.shape
        assert len(shape) == 2 and table.dtype == _I32 and table.is_contiguous() and table.get_device() == dev, "table: int32 [B, width], contiguous, on the current device"
        B, width = shape
        _check_ints(lens, B, "lens", dev)
        if starts is not None:
            _check_ints(starts, B + 1, "starts", dev)
            starts = starts.data_ptr()
        if prefix > 0:
            assert prefix_table is not None, "prefix_table: pages of the whole prefix"
            _check_ints(prefix_table, prefix_table.numel(), "prefix_table", dev)
            assert prefix_table.numel() * page >= prefix, "prefix_table: pages of the whole prefix"
            prefix_table = prefix_table.data_ptr()
        else:
            prefix_table = 0
        return _KVBATCH.pack(table.data_ptr() or _ptr(table) or 0, lens.data_ptr() or _ptr(lens) or 0, starts or 0, prefix_table, B, width, prefix)


def _check_ints(t: torch.Tensor, n: int, what: str, dev: int):
    assert t.dtype == _I32 and t.shape == (n,) and t.is_contiguous() and t.get_device() == dev, what + ": int32 [%d], on the current device" % n


def _scratch(nbytes: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    """A workspace in elements of another tensor's type, 1 us of the host's less than one of bytes."""
    return like.new_empty(-(-nbytes // like.element_size())) if nbytes else None


def rope(X: torch.Tensor, pos: torch.Tensor, rotation: Rope, heads: int, out_dtype: int = OUT_BF16, *, inverse: bool = False,
         Y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nvfp4_rope: the heads of every row of X [N, heads * D] turned by pos (int32 [N]); inverse: the gradient's way back.  Y may be X."""
    dev = _current_device()
    kind, ldx, N, width = _rows(X, "X", dev)
    assert heads > 0 and width % heads == 0, "X: rows of whole heads"
    _check_ints(pos, N, "pos", dev)
    Y, ldy = _out_rows(Y, N, width, out_dtype, X, "Y", dev)
    _check(lib().nvfp4_rope(_ptr(X), kind, ldx, _ptr(pos), N, heads, width // heads, rotation.packed(dev), int(inverse), _ptr(Y), out_dtype, ldy,
                            _raw_stream(dev)), "nvfp4_rope")
    return Y


def kv_append(K: torch.Tensor, V: torch.Tensor, cache: KVCache, batch: KVBatch, rotation: Optional[Rope] = None, *, Q: Optional[torch.Tensor] = None,
              out_dtype: int = OUT_BF16, Qo: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """nvfp4_kv_append: keys (turned at their positions) and values [N, heads * D] of the batch's rows into the cache; Q [N, any heads * D] turned in the same way is returned."""
    dev = _current_device()
    cc = cache.packed(dev)
    _, heads, page, D = cache.k.shape
    kind, ldk, N, width = _rows(K, "K", dev)
    vkind, ldv, *shape = _rows(V, "V", dev)
    assert width == heads * D and shape == [N, width] and vkind == kind, "K, V: one type, [N, heads * D] of the cache"
    ldq = Hq = ldo = 0
    if Q is not None:
        qkind, ldq, rows, qwidth = _rows(Q, "Q", dev)
        assert rows == N and qwidth % D == 0 and qkind == kind, "Q: the type and rows of K, whole heads"
        Hq = qwidth // D
        Qo, ldo = _out_rows(Qo, N, qwidth, out_dtype, Q, "Qo", dev)
    else:
        assert Qo is None, "Qo: the output of Q"
    _check(lib().nvfp4_kv_append(_ptr(Q), ldq, Hq, _ptr(K), ldk, _ptr(V), ldv, kind, N, cc, batch.packed(dev, page),
                                 None if rotation is None else rotation.packed(dev), _ptr(Qo), out_dtype, ldo, _raw_stream(dev)), "nvfp4_kv_append")
    return Qo


def kv_load(cache: KVCache, batch: KVBatch, N: int, out_dtype: int = OUT_BF16, *, K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None):
    """nvfp4_kv_load: (K, V) [N, heads * D] of the batch's N rows as the cache holds them."""
    dev = _current_device()
    cc = cache.packed(dev)
    _, heads, page, D = cache.k.shape
    K, ldk = _out_rows(K, N, heads * D, out_dtype, cache.k, "K", dev)
    V, ldv = _out_rows(V, N, heads * D, out_dtype, cache.k, "V", dev)
    _check(lib().nvfp4_kv_load(cc, batch.packed(dev, page), N, _ptr(K), ldk, _ptr(V), ldv, out_dtype, _raw_stream(dev)), "nvfp4_kv_load")
    return K, V


def attn_workspace_bytes(N: int, Hq: int, cache: KVCache, batch: KVBatch) -> int:
    pages, heads, page, D = cache.k.shape
    return int(lib().nvfp4_attn_workspace_bytes(N, Hq, heads, D, page, *batch.table.shape, batch.prefix))


def attn(Q: torch.Tensor, cache: KVCache, batch: KVBatch, heads: int, *, scale: Optional[float] = None, Out: Optional[torch.Tensor] = None,
         ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nvfp4_attn: the batch's rows Q [N, heads * D] (bf16) over the cache; scale: 1 / sqrt(D) unless given.  Rows that belong to no sequence are not written."""
    dev = _current_device()
    cc = cache.packed(dev)
    _, kv_heads, page, D = cache.k.shape
    kind, ldq, N, width = _rows(Q, "Q", dev)
    assert kind == SRC_BF16 and width == heads * D, "Q: bf16 [N, heads * D]"
    cb = batch.packed(dev, page)
    Out, ldo = _out_rows(Out, N, width, OUT_BF16, Q, "Out", dev)
    L = lib()
    if ws is None:
        B, table_width = batch.table.shape
        ws = _scratch(L.nvfp4_attn_workspace_bytes(N, heads, kv_heads, D, page, B, table_width, batch.prefix), Q)
    else:
        assert ws.get_device() == dev, "ws: on the current device"
    _check(L.nvfp4_attn(_ptr(Q), ldq, N, heads, cc, cb, D ** -0.5 if scale is None else scale, _ptr(Out), ldo, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                        _raw_stream(dev)), "nvfp4_attn")
    return Out


def sample(logits: torch.Tensor, u: torch.Tensor, *, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, tokens: Optional[torch.Tensor] = None,
           ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nvfp4_sample: a token (int64 [N]) per row of logits [N, V] from u (float32 [N], 0 <= u < 1); the other parameters are [N], float32 (top_k: int32)."""
    dev = _current_device()
    kind, ld, N, V = _rows(logits, "logits", dev)
    for t, what, dtype in ((u, "u", _F32), (temperature, "temperature", _F32), (top_k, "top_k", _I32), (top_p, "top_p", _F32), (min_p, "min_p", _F32), (tokens, "tokens", torch.int64)):
        assert t is None or (t.dtype == dtype and t.shape == (N,) and t.is_contiguous() and t.get_device() == dev), what + ": %s [N], on the current device" % dtype
    if tokens is None:
        tokens = torch.empty(N, dtype=torch.int64, device=logits.device)
    if ws is None:
        ws = _scratch(lib().nvfp4_sample_workspace_bytes(N, V), logits)
    else:
        assert ws.get_device() == dev, "ws: on the current device"
    _check(lib().nvfp4_sample(_ptr(logits), kind, ld, N, V, _ptr(u), _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), _ptr(tokens), _ptr(ws),
                              0 if ws is None else ws.numel() * ws.element_size(), _raw_stream(dev)), "nvfp4_sample")
    return tokens
