"""Thin ctypes binding of libchorus.so (C ABI in include/chorus.h).

Argument marshalling only: torch tensors are used for device memory and the
current HIP stream; every step of the mask builder, the plan, the FP8
quantiser and the attention runs in the library's HIP kernels.  There is no
fallback: if the library is missing or a call fails, a RuntimeError is raised.

Function names follow the C entry points without their ``chorus_`` prefix.
"""

from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libchorus.so")

F16, BF16, FP8_E4M3 = 0, 1, 2
BLOCK = 64
_STATUS = {0: "CHORUS_OK", 1: "CHORUS_ERR_INVALID_ARG", 2: "CHORUS_ERR_UNSUPPORTED",
           3: "CHORUS_ERR_CAPACITY", 4: "CHORUS_ERR_HIP", 5: "CHORUS_ERR_WORKSPACE"}


class Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("S", ctypes.c_int32), ("H", ctypes.c_int32),
                ("D", ctypes.c_int32)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64),
                ("stride_s", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class Mask(ctypes.Structure):
    _fields_ = [("mask_batch", ctypes.c_int32), ("H", ctypes.c_int32),
                ("n_blocks", ctypes.c_int32), ("block", ctypes.c_int32),
                ("row_ptr", ctypes.c_void_p), ("col_idx", ctypes.c_void_p)]


class Schedule(ctypes.Structure):
    _fields_ = [("order", ctypes.c_void_p), ("n_units", ctypes.c_int32)]


class KeyScale(ctypes.Structure):
    _fields_ = [("n_first", ctypes.c_int32), ("beta", ctypes.c_float)]


class Rotary(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32), ("pairs", ctypes.c_int32 * 4), ("adjacent", ctypes.c_int32),
                ("freqs", ctypes.c_double * 64)]


class PackedShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "total_q", "total_k", "prefix", "q_heads", "kv_heads", "D",
                                              "causal", "max_q")]


def _key_scale(key_scale):
    """(n_first, beta) -> pointer to a chorus_key_scale, None -> NULL."""
    if key_scale is None:
        return None
    n_first, beta = key_scale
    return ctypes.byref(KeyScale(int(n_first), float(beta)))


EXPORTS = [
    "chorus_build_block_mask_workspace_size", "chorus_build_block_mask", "chorus_build_block_mask_fp8",
    "chorus_build_block_mask_noalloc", "chorus_build_block_mask_from_sums",
    "chorus_plan_workspace_size", "chorus_plan_block_mask", "chorus_validate_block_mask",
    "chorus_quantize_fp8_blockwise", "chorus_quantize_fp8_blockwise_sums", "chorus_attn_workspace_size",
    "chorus_block_sparse_attn_fwd", "chorus_block_sparse_attn_fwd_f16",
    "chorus_block_sparse_attn_fwd_bf16", "chorus_block_sparse_attn_fwd_fp8",
    "chorus_attn_block_mass", "chorus_select_block_mask_workspace_size", "chorus_select_block_mask",
    "chorus_mask_coverage",
    "chorus_visit_map_bytes", "chorus_visit_reset", "chorus_visit_update",
    "chorus_visit_refresh_workspace_size", "chorus_visit_refresh",
    "chorus_qk_norm_rope", "chorus_packed_plan_bytes", "chorus_plan_packed_attn",
    "chorus_packed_attn_workspace_size", "chorus_packed_attn_fwd",
    "chorus_status_string", "chorus_last_error", "chorus_version",
]

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libchorus.so (once) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run `python -m paper_2606_25040_amd.build` "
                           "(or __graft_entry__.build())")
    L = ctypes.CDLL(path)
    P, VP, I32, I64, F32, F64, SZ = (ctypes.POINTER, ctypes.c_void_p, ctypes.c_int32,
                                    ctypes.c_int64, ctypes.c_float, ctypes.c_double, ctypes.c_size_t)
    sig = {
        "chorus_build_block_mask_workspace_size": (SZ, [P(Shape)]),
        "chorus_build_block_mask": (I32, [I32, P(Shape), P(Tensor), P(Tensor), F64, F64, F64, I32,
                                          P(KeyScale), VP, VP, I64, VP, VP, SZ, VP]),
        "chorus_build_block_mask_fp8": (I32, [P(Shape), P(Tensor), VP, P(Tensor), VP, F64, F64, F64, I32,
                                              P(KeyScale), VP, VP, I64, VP, VP, SZ, VP]),
        "chorus_build_block_mask_noalloc": (I32, [I32, P(Shape), P(Tensor), P(Tensor), F64, F64, F64, I32,
                                                  P(KeyScale), VP, VP, I64, VP, VP]),
        "chorus_build_block_mask_from_sums": (I32, [P(Shape), VP, VP, F64, F64, F64, I32, VP, VP, I64, VP,
                                                    VP, SZ, VP]),
        "chorus_plan_workspace_size": (SZ, [P(Shape), P(Mask)]),
        "chorus_plan_block_mask": (I32, [P(Shape), P(Mask), VP, VP, SZ, VP]),
        "chorus_validate_block_mask": (I32, [P(Mask), I64, VP, VP]),
        "chorus_quantize_fp8_blockwise": (I32, [I32, P(Shape), P(Tensor), P(Tensor), VP, VP]),
        "chorus_quantize_fp8_blockwise_sums": (I32, [I32, P(Shape), P(Tensor), P(Tensor), VP, P(KeyScale), VP,
                                                     VP]),
        "chorus_attn_workspace_size": (SZ, [I32, P(Shape), P(Mask)]),
        "chorus_block_sparse_attn_fwd": (I32, [I32, P(Shape), P(Tensor), P(Tensor), P(Tensor), VP,
                                               VP, VP, P(Mask), P(Schedule), F32, P(KeyScale),
                                               P(Tensor), VP, VP, SZ, VP]),
        "chorus_block_sparse_attn_fwd_f16": (I32, [P(Shape), P(Tensor), P(Tensor), P(Tensor),
                                                   P(Mask), P(Schedule), F32, P(KeyScale),
                                                   P(Tensor), VP, VP, SZ, VP]),
        "chorus_block_sparse_attn_fwd_bf16": (I32, [P(Shape), P(Tensor), P(Tensor), P(Tensor),
                                                    P(Mask), P(Schedule), F32, P(KeyScale),
                                                    P(Tensor), VP, VP, SZ, VP]),
        "chorus_block_sparse_attn_fwd_fp8": (I32, [P(Shape), P(Tensor), P(Tensor), P(Tensor), VP,
                                                   VP, VP, P(Mask), P(Schedule), F32, P(KeyScale),
                                                   P(Tensor), VP, VP, SZ, VP]),
        "chorus_attn_block_mass": (I32, [I32, P(Shape), P(Tensor), P(Tensor), VP, F32, I32,
                                         P(KeyScale), VP, VP]),
        "chorus_select_block_mask_workspace_size": (SZ, [P(Shape)]),
        "chorus_select_block_mask": (I32, [P(Shape), VP, I32, F64, F64, VP, VP, I64, VP, SZ, VP]),
        "chorus_mask_coverage": (I32, [P(Shape), P(Mask), VP, VP, VP]),
        "chorus_visit_map_bytes": (SZ, [P(Mask)]),
        "chorus_visit_reset": (I32, [P(Mask), VP, VP]),
        "chorus_visit_update": (I32, [P(Mask), VP, VP]),
        "chorus_visit_refresh_workspace_size": (SZ, [P(Mask)]),
        "chorus_visit_refresh": (I32, [P(Mask), VP, VP, VP, I64, VP, SZ, VP]),
        "chorus_qk_norm_rope": (I32, [I32, P(Shape), I32, P(Tensor), P(Tensor), I32, VP, VP, F32, P(Rotary), VP, I64,
                                      I64, P(Tensor), P(Tensor), VP]),
        "chorus_packed_plan_bytes": (SZ, [P(PackedShape)]),
        "chorus_plan_packed_attn": (I32, [P(PackedShape), VP, VP, VP, VP, SZ, VP]),
        "chorus_packed_attn_workspace_size": (SZ, [P(PackedShape)]),
        "chorus_packed_attn_fwd": (I32, [I32, P(PackedShape), P(Tensor), P(Tensor), P(Tensor), P(Tensor), P(Tensor),
                                         F32, VP, SZ, P(Tensor), VP, VP, SZ, VP]),
        "chorus_status_string": (ctypes.c_char_p, [I32]),
        "chorus_last_error": (ctypes.c_char_p, []),
        "chorus_version": (I32, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(status: int, what: str) -> None:
    if status != 0:
        L = load_library()
        raise RuntimeError(f"{what} failed: {_STATUS.get(status, status)}: "
                           f"{L.chorus_last_error().decode()}")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return F16
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.uint8:
        return FP8_E4M3
    raise TypeError(f"unsupported dtype {t.dtype}")


def _tensor(t: torch.Tensor) -> Tensor:
    if t.dim() != 4:
        raise ValueError("expected a [B, S, H, D] tensor")
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if t.stride(3) != 1:
        raise ValueError("head dim must be contiguous")
    return Tensor(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def _shape(t: torch.Tensor) -> Shape:
    B, S, H, D = t.shape
    return Shape(B, S, H, D)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None else t.data_ptr()


def _workspace(nbytes: int, device) -> torch.Tensor | None:
    if nbytes == 0:
        return None
    return torch.empty(nbytes + 256, dtype=torch.uint8, device=device)


def _aligned(ws: torch.Tensor | None) -> int | None:
    if ws is None:
        return None
    p = ws.data_ptr()
    return (p + 255) // 256 * 256


@dataclass
class BlockMask:
    """CSR block mask on device (rows (b_m * H + h) * n_blocks + i, ascending ids)."""
    row_ptr: torch.Tensor      # int32 [mask_batch * H * n_blocks + 1]
    col_idx: torch.Tensor      # int32 [capacity]
    mask_batch: int
    H: int
    n_blocks: int
    block: int = BLOCK
    block_scores: torch.Tensor | None = None

    @property
    def rows(self) -> int:
        return self.mask_batch * self.H * self.n_blocks

    @property
    def n_kv(self) -> int:
        """Columns: kv blocks of ``block`` tokens per row."""
        return (self.n_blocks * BLOCK + self.block - 1) // self.block

    @property
    def nnz(self) -> int:
        return int(self.row_ptr[-1].item())

    @property
    def density(self) -> float:
        return self.nnz / float(self.rows * self.n_kv)

    def as_c(self) -> Mask:
        return Mask(self.mask_batch, self.H, self.n_blocks, self.block, self.row_ptr.data_ptr(),
                    self.col_idx.data_ptr())

    def to_host(self):
        """(row_ptr, col_idx[:nnz]) as int64 numpy arrays."""
        rp = self.row_ptr.cpu().numpy().astype("int64")
        return rp, self.col_idx[: int(rp[-1])].cpu().numpy().astype("int64")

    @staticmethod
    def from_host(row_ptr, col_idx, mask_batch: int, H: int, n_blocks: int, device="cuda",
                  block: int = BLOCK):
        rp = torch.as_tensor(row_ptr, dtype=torch.int32).to(device)
        ci = torch.as_tensor(col_idx, dtype=torch.int32)
        if ci.numel() == 0:
            ci = torch.zeros(1, dtype=torch.int32)
        return BlockMask(rp, ci.to(device), mask_batch, H, n_blocks, block)


def build_block_mask(q: torch.Tensor, k: torch.Tensor, top_p: float, min_top_k: float,
                     sm_scale: float | None = None, return_scores: bool = False,
                     out: BlockMask | None = None, workspace: torch.Tensor | None = None,
                     key_scale=None, scales=None, kv_block: int = BLOCK) -> BlockMask:
    """chorus_build_block_mask: one mask per request of ``q, k [B, S, H, D]``;
    ``key_scale = (n_first, beta)`` pools the first-frame-enhanced keys.  For
    fp8 codes (uint8) pass ``scales = (q_scale, k_scale)`` from the quantiser
    (chorus_build_block_mask_fp8).  ``kv_block`` = 64 or 128 tokens per kv
    block (the mask's columns)."""
    L = load_library()
    if q.shape != k.shape or q.dtype != k.dtype:
        raise ValueError("q and k must share shape and dtype")
    fp8 = q.dtype == torch.uint8
    if fp8 != (scales is not None):
        raise ValueError("scales are given exactly for fp8 codes")
    B, S, H, D = q.shape
    n = (S + BLOCK - 1) // BLOCK
    nk = (S + kv_block - 1) // kv_block
    rows = B * H * n
    shape = _shape(q)
    sm = 1.0 / math.sqrt(D) if sm_scale is None else float(sm_scale)
    if out is None:
        out = BlockMask(torch.empty(rows + 1, dtype=torch.int32, device=q.device),
                        torch.empty(rows * nk, dtype=torch.int32, device=q.device), B, H, n, kv_block)
    out.block = kv_block
    if return_scores and (out.block_scores is None or out.block_scores.shape != (rows, nk)):
        out.block_scores = torch.empty((rows, nk), dtype=torch.float32, device=q.device)
    need = L.chorus_build_block_mask_workspace_size(ctypes.byref(shape))
    if workspace is None or workspace.numel() < need + 256:
        workspace = _workspace(need, q.device)
    tail = (sm, float(top_p), float(min_top_k), int(kv_block), _key_scale(key_scale), out.row_ptr.data_ptr(),
            out.col_idx.data_ptr(), out.col_idx.numel(),
            _ptr(out.block_scores if return_scores else None), _aligned(workspace), need, _stream())
    if fp8:
        st = L.chorus_build_block_mask_fp8(ctypes.byref(shape), ctypes.byref(_tensor(q)),
                                           scales[0].data_ptr(), ctypes.byref(_tensor(k)),
                                           scales[1].data_ptr(), *tail)
        _check(st, "chorus_build_block_mask_fp8")
    else:
        st = L.chorus_build_block_mask(_dtype_code(q), ctypes.byref(shape), ctypes.byref(_tensor(q)),
                                       ctypes.byref(_tensor(k)), *tail)
        _check(st, "chorus_build_block_mask")
    return out


def build_block_mask_noalloc(q: torch.Tensor, k: torch.Tensor, top_p: float, min_top_k: float, out: BlockMask,
                             sm_scale: float | None = None, key_scale=None, kv_block: int = BLOCK,
                             block_scores: torch.Tensor | None = None) -> BlockMask:
    """chorus_build_block_mask_noalloc: the builder on f16 / bf16 ``q, k`` with
    the library's own fixed scratch; the caller passes the output mask
    buffers (``out``, and ``block_scores`` [rows, n_kv] fp32 to receive the
    scores) so that nothing is allocated."""
    L = load_library()
    if q.shape != k.shape or q.dtype != k.dtype:
        raise ValueError("q and k must share shape and dtype")
    B, S, H, D = q.shape
    sm = 1.0 / math.sqrt(D) if sm_scale is None else float(sm_scale)
    out.block = kv_block
    out.block_scores = block_scores
    st = L.chorus_build_block_mask_noalloc(_dtype_code(q), ctypes.byref(_shape(q)), ctypes.byref(_tensor(q)),
                                           ctypes.byref(_tensor(k)), sm, float(top_p), float(min_top_k),
                                           int(kv_block), _key_scale(key_scale), out.row_ptr.data_ptr(),
                                           out.col_idx.data_ptr(), out.col_idx.numel(), _ptr(block_scores),
                                           _stream())
    _check(st, "chorus_build_block_mask_noalloc")
    return out


def plan_block_mask(mask: BlockMask, B: int, S: int, out: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None) -> torch.Tensor:
    """chorus_plan_block_mask: (request, head) unit order for applying ``mask``
    to B requests (int32 [B * H])."""
    L = load_library()
    shape = Shape(B, S, mask.H, 128)
    cm = mask.as_c()
    order = out if out is not None else torch.empty(B * mask.H, dtype=torch.int32,
                                                    device=mask.row_ptr.device)
    need = L.chorus_plan_workspace_size(ctypes.byref(shape), ctypes.byref(cm))
    ws = workspace if workspace is not None and workspace.numel() >= need + 256 else \
        _workspace(need, mask.row_ptr.device)
    st = L.chorus_plan_block_mask(ctypes.byref(shape), ctypes.byref(cm), order.data_ptr(),
                                  _aligned(ws), need, _stream())
    _check(st, "chorus_plan_block_mask")
    return order


def validate_block_mask(mask: BlockMask) -> int:
    """chorus_validate_block_mask; synchronises and returns the flag word (0 = valid)."""
    L = load_library()
    flags = torch.empty(1, dtype=torch.int32, device=mask.row_ptr.device)
    cm = mask.as_c()
    st = L.chorus_validate_block_mask(ctypes.byref(cm), mask.col_idx.numel(), flags.data_ptr(),
                                      _stream())
    _check(st, "chorus_validate_block_mask")
    return int(flags.item())


def quantize_fp8_blockwise(x: torch.Tensor, codes: torch.Tensor | None = None,
                           scales: torch.Tensor | None = None):
    """chorus_quantize_fp8_blockwise: returns (codes uint8 [B,S,H,D], scales fp32 [B,H,n])."""
    L = load_library()
    B, S, H, D = x.shape
    n = (S + BLOCK - 1) // BLOCK
    if codes is None:
        codes = torch.empty((B, S, H, D), dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty((B, H, n), dtype=torch.float32, device=x.device)
    st = L.chorus_quantize_fp8_blockwise(_dtype_code(x), ctypes.byref(_shape(x)),
                                         ctypes.byref(_tensor(x)), ctypes.byref(_tensor(codes)),
                                         scales.data_ptr(), _stream())
    _check(st, "chorus_quantize_fp8_blockwise")
    return codes, scales


def quantize_fp8_blockwise_sums(x: torch.Tensor, codes: torch.Tensor | None = None,
                                scales: torch.Tensor | None = None, block_sums: torch.Tensor | None = None,
                                key_scale=None):
    """chorus_quantize_fp8_blockwise_sums: returns (codes, scales, block_sums float64 [B, H, n, 128]),
    the sums over each 64-token block's valid tokens (first-frame tokens times
    beta when ``key_scale = (n_first, beta)``)."""
    L = load_library()
    B, S, H, D = x.shape
    n = (S + BLOCK - 1) // BLOCK
    if codes is None:
        codes = torch.empty((B, S, H, D), dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty((B, H, n), dtype=torch.float32, device=x.device)
    if block_sums is None:
        block_sums = torch.empty((B, H, n, D), dtype=torch.float64, device=x.device)
    elif block_sums.shape != (B, H, n, D) or block_sums.dtype != torch.float64 or not block_sums.is_contiguous():
        raise ValueError(f"block_sums must be a contiguous float64 [{B}, {H}, {n}, {D}] tensor")
    st = L.chorus_quantize_fp8_blockwise_sums(_dtype_code(x), ctypes.byref(_shape(x)),
                                              ctypes.byref(_tensor(x)), ctypes.byref(_tensor(codes)),
                                              scales.data_ptr(), _key_scale(key_scale),
                                              block_sums.data_ptr(), _stream())
    _check(st, "chorus_quantize_fp8_blockwise_sums")
    return codes, scales, block_sums


def build_block_mask_from_sums(q_sums: torch.Tensor, k_sums: torch.Tensor, S: int, top_p: float,
                               min_top_k: float, sm_scale: float | None = None, return_scores: bool = False,
                               out: BlockMask | None = None, workspace: torch.Tensor | None = None,
                               kv_block: int = BLOCK) -> BlockMask:
    """chorus_build_block_mask_from_sums: the mask of sequence length ``S``
    from the quantiser's float64 block sums ``[B, H, n, 128]`` of Q and K."""
    L = load_library()
    if q_sums.shape != k_sums.shape or q_sums.dim() != 4:
        raise ValueError("q_sums and k_sums must share one [B, H, n, D] shape")
    for t in (q_sums, k_sums):
        if t.dtype != torch.float64 or not t.is_contiguous():
            raise ValueError("block sums must be contiguous float64")
    B, H, n, D = q_sums.shape
    if n != (S + BLOCK - 1) // BLOCK:
        raise ValueError(f"block sums hold {n} blocks, S = {S} needs {(S + BLOCK - 1) // BLOCK}")
    nk = (S + kv_block - 1) // kv_block
    rows = B * H * n
    shape = Shape(B, S, H, D)
    sm = 1.0 / math.sqrt(D) if sm_scale is None else float(sm_scale)
    dev = q_sums.device
    if out is None:
        out = BlockMask(torch.empty(rows + 1, dtype=torch.int32, device=dev),
                        torch.empty(rows * nk, dtype=torch.int32, device=dev), B, H, n, kv_block)
    out.block = kv_block
    if return_scores and (out.block_scores is None or out.block_scores.shape != (rows, nk)):
        out.block_scores = torch.empty((rows, nk), dtype=torch.float32, device=dev)
    need = L.chorus_build_block_mask_workspace_size(ctypes.byref(shape))
    if workspace is None or workspace.numel() < need + 256:
        workspace = _workspace(need, dev)
    st = L.chorus_build_block_mask_from_sums(ctypes.byref(shape), q_sums.data_ptr(), k_sums.data_ptr(), sm,
                                             float(top_p), float(min_top_k), int(kv_block), out.row_ptr.data_ptr(),
                                             out.col_idx.data_ptr(), out.col_idx.numel(),
                                             _ptr(out.block_scores if return_scores else None),
                                             _aligned(workspace), need, _stream())
    _check(st, "chorus_build_block_mask_from_sums")
    return out


def block_sparse_attn_fwd(q, k, v, mask: BlockMask | None, sm_scale: float | None = None,
                          scales=None, out: torch.Tensor | None = None, return_lse: bool = False,
                          schedule: torch.Tensor | None = None, key_scale=None):
    """chorus_block_sparse_attn_fwd (dtype taken from q: f16, bf16 or uint8 fp8 codes).

    ``scales`` = (q_scale, k_scale, v_scale) for fp8 codes; ``mask=None`` runs
    every block pair (dense attention); ``key_scale = (n_first, beta)`` applies
    the first-frame key enhancement.  Returns ``out`` (and ``lse [B, H, S]``
    fp32 when ``return_lse``).
    """
    L = load_library()
    dt = _dtype_code(q)
    if k.shape != q.shape or v.shape != q.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k and v must share shape and dtype")
    B, S, H, D = q.shape
    sm = 1.0 / math.sqrt(D) if sm_scale is None else float(sm_scale)
    odt = torch.bfloat16 if dt == FP8_E4M3 else q.dtype
    if out is None:
        out = torch.empty((B, S, H, D), dtype=odt, device=q.device)
    elif out.shape != q.shape or out.dtype != odt:
        raise ValueError(f"out must be a {odt} tensor of q's shape")
    lse = torch.empty((B, H, S), dtype=torch.float32, device=q.device) if return_lse else None
    qs = ks = vs = None
    if dt == FP8_E4M3:
        if scales is None:
            raise ValueError("fp8 attention needs (q_scale, k_scale, v_scale)")
        qs, ks, vs = (s.data_ptr() for s in scales)
    shape = _shape(q)
    cm = ctypes.byref(mask.as_c()) if mask is not None else None
    sched = None
    if schedule is not None:
        sched = ctypes.byref(Schedule(schedule.data_ptr(), schedule.numel()))
    need = L.chorus_attn_workspace_size(dt, ctypes.byref(shape), cm)
    ws = _workspace(need, q.device)
    st = L.chorus_block_sparse_attn_fwd(dt, ctypes.byref(shape), ctypes.byref(_tensor(q)),
                                        ctypes.byref(_tensor(k)), ctypes.byref(_tensor(v)), qs, ks,
                                        vs, cm, sched, sm, _key_scale(key_scale),
                                        ctypes.byref(_tensor(out)),
                                        _ptr(lse), _aligned(ws), need, _stream())
    _check(st, "chorus_block_sparse_attn_fwd")
    return (out, lse) if return_lse else out


def block_sparse_attn_fwd_f16(q, k, v, mask, **kw):
    assert q.dtype == torch.float16
    return block_sparse_attn_fwd(q, k, v, mask, **kw)


def block_sparse_attn_fwd_bf16(q, k, v, mask, **kw):
    assert q.dtype == torch.bfloat16
    return block_sparse_attn_fwd(q, k, v, mask, **kw)


def block_sparse_attn_fwd_fp8(q, k, v, q_scale, k_scale, v_scale, mask, **kw):
    assert q.dtype == torch.uint8
    return block_sparse_attn_fwd(q, k, v, mask, scales=(q_scale, k_scale, v_scale), **kw)


def attn_block_mass(q: torch.Tensor, k: torch.Tensor, lse: torch.Tensor, sm_scale: float | None = None,
                    out: torch.Tensor | None = None, key_scale=None, kv_block: int = BLOCK) -> torch.Tensor:
    """chorus_attn_block_mass: true block attention mass [B, H, n, n_kv]
    (fp32) of ``q, k [B, S, H, D]`` given the dense attention's ``lse [B, H, S]``
    (computed with the same ``key_scale``); kv blocks of ``kv_block`` tokens."""
    L = load_library()
    if q.shape != k.shape or q.dtype != k.dtype:
        raise ValueError("q and k must share shape and dtype")
    B, S, H, D = q.shape
    n = (S + 63) // 64
    if lse.shape != (B, H, S) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [B, H, S] tensor")
    sm = (1.0 / math.sqrt(D)) if sm_scale is None else sm_scale
    nk = (S + kv_block - 1) // kv_block
    mass = out if out is not None else torch.empty((B, H, n, nk), dtype=torch.float32, device=q.device)
    if mass.shape != (B, H, n, nk) or mass.dtype != torch.float32 or not mass.is_contiguous():
        raise ValueError("out must be a contiguous float32 [B, H, n, n_kv] tensor")
    st = L.chorus_attn_block_mass(_dtype_code(q), ctypes.byref(_shape(q)), ctypes.byref(_tensor(q)),
                                  ctypes.byref(_tensor(k)), lse.data_ptr(), sm, int(kv_block),
                                  _key_scale(key_scale),
                                  mass.data_ptr(), _stream())
    _check(st, "chorus_attn_block_mass")
    return mass


def select_block_mask(mass: torch.Tensor, S: int, top_p: float, min_top_k: float,
                      out: BlockMask | None = None, workspace: torch.Tensor | None = None,
                      kv_block: int = BLOCK) -> BlockMask:
    """chorus_select_block_mask: CSR mask (mask_batch = B) cut from block
    masses ``mass [B, H, n, n_kv]`` of a sequence of S tokens."""
    L = load_library()
    B, H, n, nk = mass.shape
    if (n != (S + 63) // 64 or nk != (S + kv_block - 1) // kv_block or mass.dtype != torch.float32
            or not mass.is_contiguous()):
        raise ValueError("mass must be a contiguous float32 [B, H, ceil(S / 64), ceil(S / kv_block)] tensor")
    shape = Shape(B, S, H, 128)
    rows = B * H * n
    m = out if out is not None else BlockMask(
        torch.empty(rows + 1, dtype=torch.int32, device=mass.device),
        torch.empty(rows * nk, dtype=torch.int32, device=mass.device), B, H, n, kv_block)
    m.block = kv_block
    need = L.chorus_select_block_mask_workspace_size(ctypes.byref(shape))
    ws = workspace if workspace is not None and workspace.numel() >= need + 256 else \
        _workspace(need, mass.device)
    st = L.chorus_select_block_mask(ctypes.byref(shape), mass.data_ptr(), int(kv_block), top_p, min_top_k,
                                    m.row_ptr.data_ptr(), m.col_idx.data_ptr(), m.col_idx.numel(),
                                    _aligned(ws), need, _stream())
    _check(st, "chorus_select_block_mask")
    return m


def mask_coverage(mask: BlockMask, mass: torch.Tensor, S: int) -> torch.Tensor:
    """chorus_mask_coverage: coverage [B, H] (float64) of ``mask`` on the
    requests whose block masses are ``mass [B, H, n, n]``."""
    L = load_library()
    B, H, n, _ = mass.shape
    if mass.dtype != torch.float32 or not mass.is_contiguous():
        raise ValueError("mass must be a contiguous float32 tensor")
    cov = torch.empty((B, H), dtype=torch.float64, device=mass.device)
    cm = mask.as_c()
    st = L.chorus_mask_coverage(ctypes.byref(Shape(B, S, H, 128)), ctypes.byref(cm), mass.data_ptr(),
                                cov.data_ptr(), _stream())
    _check(st, "chorus_mask_coverage")
    return cov


class VisitMap:
    """Device visited bitmap of a layer group (chorus_visit_*), sized for
    masks with the given mask_batch / H / n_blocks."""

    def __init__(self, mask_batch: int, H: int, n_blocks: int, device="cuda", block: int = BLOCK):
        L = load_library()
        desc = Mask(mask_batch, H, n_blocks, block, None, None)
        nbytes = L.chorus_visit_map_bytes(ctypes.byref(desc))
        if nbytes == 0:
            raise ValueError("invalid mask description for a visited map")
        self.mask_batch, self.H, self.n_blocks, self.block = mask_batch, H, n_blocks, block
        self.n_kv = (n_blocks * BLOCK + block - 1) // block
        self.words = (self.n_kv + 31) // 32
        self.bits = torch.empty(nbytes // 4, dtype=torch.int32, device=device)

    def _check_mask(self, mask: BlockMask):
        if (mask.mask_batch, mask.H, mask.n_blocks, mask.block) != (self.mask_batch, self.H, self.n_blocks,
                                                                    self.block):
            raise ValueError("mask dimensions differ from the visited map's")

    def reset(self, like: BlockMask):
        self._check_mask(like)
        st = load_library().chorus_visit_reset(ctypes.byref(like.as_c()), self.bits.data_ptr(), _stream())
        _check(st, "chorus_visit_reset")

    def update(self, mask: BlockMask):
        self._check_mask(mask)
        st = load_library().chorus_visit_update(ctypes.byref(mask.as_c()), self.bits.data_ptr(), _stream())
        _check(st, "chorus_visit_update")

    def refresh(self, mask: BlockMask, out: BlockMask | None = None,
                workspace: torch.Tensor | None = None) -> BlockMask:
        """The group's last-layer mask: mask | (pairs not visited)."""
        self._check_mask(mask)
        L = load_library()
        rows = mask.rows
        m = out if out is not None else BlockMask(
            torch.empty(rows + 1, dtype=torch.int32, device=self.bits.device),
            torch.empty(rows * mask.n_kv, dtype=torch.int32, device=self.bits.device), mask.mask_batch, mask.H,
            mask.n_blocks, mask.block)
        cm = mask.as_c()
        need = L.chorus_visit_refresh_workspace_size(ctypes.byref(cm))
        ws = workspace if workspace is not None and workspace.numel() >= need + 256 else \
            _workspace(need, self.bits.device)
        st = L.chorus_visit_refresh(ctypes.byref(cm), self.bits.data_ptr(), m.row_ptr.data_ptr(),
                                    m.col_idx.data_ptr(), m.col_idx.numel(), _aligned(ws), need, _stream())
        _check(st, "chorus_visit_refresh")
        return m

    def to_host(self):
        """Boolean [rows, n_blocks] numpy view of the map."""
        import numpy as np
        w = self.bits.cpu().numpy().view(np.uint32).reshape(-1, self.words)
        bits = ((w[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1).astype(bool)
        return bits.reshape(w.shape[0], -1)[:, : self.n_kv]


def _current(*tensors) -> int:
    """Every given tensor lives on the current device; returns that device's current stream, which the call is put on."""
    here = None
    for t in tensors:
        if t is None:
            continue
        on = t.get_device()
        if on < 0:
            raise ValueError("expected a device tensor")
        if here is None:
            here = torch.cuda.current_device()
        if on != here:
            raise ValueError(f"tensor on {t.device}, but the current device is cuda:{here}")
    return torch._C._cuda_getCurrentRawStream(here)


def _heads(t: torch.Tensor):
    """Pointer to a chorus_tensor of a [B, S, H, 128] tensor."""
    sb, ss, sh, sd = t.stride()
    if sd != 1:
        raise ValueError("head dim must be contiguous")
    return ctypes.byref(Tensor(t.data_ptr(), sb, ss, sh))


def _writable(t: torch.Tensor, name: str) -> None:
    """Rows of an output do not share memory: each stride reaches past what the smaller ones span."""
    if t.is_contiguous():
        return
    reach = 1
    for stride, size in sorted((s, n) for n, s in zip(t.shape, t.stride()) if n > 1):
        if stride < reach:
            raise ValueError(f"{name} has rows that share memory")
        reach = stride * (size - 1) + reach


class RotaryAxes:
    """A rotation of 64 pairs per head dealt to position axes: ``pairs[a]`` pairs to axis a, in order; pair p turns
    by position * ``freqs[p]`` radians.  ``freqs=None``: each axis has the ladder theta^(-i / pairs[a]), i = 0 ..
    pairs[a] - 1.  ``adjacent`` pairs are the values (2p, 2p + 1) of a head, others (p, p + 64)."""

    def __init__(self, pairs, freqs=None, adjacent: bool = True, theta: float = 10000.0):
        pairs = [int(n) for n in pairs]
        if not 1 <= len(pairs) <= 4 or any(n < 0 for n in pairs) or sum(pairs) != 64:
            raise ValueError("pairs must hold 1 to 4 counts >= 0 that add up to 64")
        if freqs is None:
            freqs = [float(theta) ** (-i / n) for n in pairs for i in range(n)]
        freqs = [float(f) for f in freqs]
        if len(freqs) != 64 or not all(math.isfinite(f) for f in freqs):
            raise ValueError("freqs must hold 64 finite values")
        self.pairs, self.freqs, self.adjacent = tuple(pairs), tuple(freqs), bool(adjacent)
        self.c = Rotary(len(pairs), (ctypes.c_int32 * 4)(*pairs), int(self.adjacent), (ctypes.c_double * 64)(*freqs))


_NORMS = {None: 0, "head": 1, "token": 2}


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor | None = None, rotary: RotaryAxes | None = None,
                 positions: torch.Tensor | None = None, norm: str | None = None, q_weight: torch.Tensor | None = None,
                 k_weight: torch.Tensor | None = None, eps: float = 1e-6, q_out: torch.Tensor | None = None,
                 k_out: torch.Tensor | None = None):
    """chorus_qk_norm_rope: norm and rotation of ``q [B, S, H, 128]`` and ``k [B, S, Hk, 128]`` (f16 or bf16) in one
    pass; returns (q_out, k_out), or q_out alone without ``k``.

    ``norm``: "head" (fp32 weights [128]), "token" (over a token's heads, weights [heads, 128]) or None.
    ``positions``: int32 [axes, S] (shared by the requests) or [axes, B, S].  ``q_out`` / ``k_out`` may be the
    inputs themselves."""
    L = load_library()
    if norm not in _NORMS:
        raise ValueError("norm must be None, 'head' or 'token'")
    stream = _current(q, k, positions, q_weight, k_weight, q_out, k_out)
    dt = _dtype_code(q)
    if q.dim() != 4:
        raise ValueError("expected a [B, S, H, D] tensor")
    B, S, H, D = q.shape
    Hk = 0
    if k is not None:
        if k.dim() != 4 or k.dtype != q.dtype or (k.shape[0], k.shape[1], k.shape[3]) != (B, S, D):
            raise ValueError("k must share q's dtype, requests, tokens and head dim")
        Hk = k.shape[2]
    elif k_out is not None:
        raise ValueError("k_out without k")
    for w, heads in ((q_weight, H), (k_weight, Hk)):
        if w is not None and (norm is None or w.dtype != torch.float32 or not w.is_contiguous()
                              or w.numel() != (D if norm == "head" else heads * D)):
            raise ValueError("a weight must be a contiguous float32 tensor, [128] for norm='head', [heads, 128] for 'token'")
    if (rotary is None) != (positions is None):
        raise ValueError("rotary and positions go together")
    axis_stride = batch_stride = 0
    if rotary is not None:
        dims, strides = positions.shape, positions.stride()
        if positions.dtype != torch.int32 or dims not in ((len(rotary.pairs), S), (len(rotary.pairs), B, S)) \
                or (strides[-1] != 1 and S > 1):
            raise ValueError("positions must be int32 [axes, S] or [axes, B, S] with contiguous tokens")
        axis_stride = strides[0]
        batch_stride = strides[1] if len(dims) == 3 else 0
    if q_out is None:
        q_out = torch.empty((B, S, H, D), dtype=q.dtype, device=q.device)
    elif q_out.shape != q.shape or q_out.dtype != q.dtype:
        raise ValueError("q_out must have q's shape and dtype")
    else:
        _writable(q_out, "q_out")
    if k is not None and k_out is None:
        k_out = torch.empty((B, S, Hk, D), dtype=k.dtype, device=k.device)
    elif k is not None and (k_out.shape != k.shape or k_out.dtype != k.dtype):
        raise ValueError("k_out must have k's shape and dtype")
    elif k is not None:
        _writable(k_out, "k_out")
    st = L.chorus_qk_norm_rope(dt, ctypes.byref(Shape(B, S, H, D)), Hk, _heads(q), None if k is None else _heads(k),
                               _NORMS[norm], _ptr(q_weight), _ptr(k_weight), float(eps),
                               None if rotary is None else ctypes.byref(rotary.c), _ptr(positions), axis_stride,
                               batch_stride, _heads(q_out), None if k is None else _heads(k_out), stream)
    _check(st, "chorus_qk_norm_rope")
    return q_out if k is None else (q_out, k_out)


@dataclass
class PackedPlan:
    """Work plan of a batch of packed sequences (chorus_plan_packed_attn), for every layer of a step."""
    data: torch.Tensor       # uint8; the plan starts at its first 256-byte boundary
    shape: PackedShape
    plan_bytes: int = 0      # chorus_packed_plan_bytes(shape)

    def __post_init__(self):
        L, s = load_library(), self.shape
        self.workspace_bytes = L.chorus_packed_attn_workspace_size(ctypes.byref(s))
        self.plan_bytes = self.plan_bytes or L.chorus_packed_plan_bytes(ctypes.byref(s))
        if self.data.numel() * self.data.element_size() < self.plan_bytes + _aligned(self.data) - self.data.data_ptr():
            raise ValueError(f"data is shorter than the {self.plan_bytes} bytes of a plan of this shape")
        self.q_dims, self.k_dims = (s.total_q, s.q_heads, s.D), (s.total_k, s.kv_heads, s.D)
        self.prefix_dims = (s.prefix, s.kv_heads, s.D)

    def flags(self) -> int:
        """Synchronises; 0, or 1 (q_offsets) | 2 (k_offsets, k_lens) where offsets or lengths had to be clamped."""
        at = _aligned(self.data) - self.data.data_ptr()
        return int(self.data[at:at + 64].view(torch.int32)[2].item())


def plan_packed_attn(q_offsets: torch.Tensor, k_offsets: torch.Tensor, total_q: int, total_k: int, q_heads: int,
                     kv_heads: int, causal: bool = True, k_lens: torch.Tensor | None = None, prefix: int = 0,
                     max_q: int = 0, out: PackedPlan | None = None) -> PackedPlan:
    """chorus_plan_packed_attn: the plan for N sequences with query rows ``q_offsets[i] : q_offsets[i + 1]`` of
    ``total_q`` and key rows from ``k_offsets[i]`` of ``total_k``, ``k_lens[i]`` of them (without ``k_lens`` up to
    ``k_offsets[i + 1]``).  ``q_offsets``: int32 [N + 1] on the device; ``k_offsets`` likewise, or [N] with
    ``k_lens`` [N].  ``prefix``: rows of a prefix that every sequence sees.  ``max_q``: the longest sequence's
    queries, if known.  ``out``: a plan of the same shape to write again."""
    L = load_library()
    stream = _current(q_offsets, k_offsets, k_lens, None if out is None else out.data)
    N = q_offsets.numel() - 1
    for t, name in ((q_offsets, "q_offsets"), (k_offsets, "k_offsets"), (k_lens, "k_lens")):
        if t is not None and (t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous int32 vector")
    if N < 1 or k_offsets.numel() < (N if k_lens is not None else N + 1) or (k_lens is not None and k_lens.numel() != N):
        raise ValueError("q_offsets holds N + 1 entries, k_offsets N + 1 (N with k_lens), k_lens N")
    shape = PackedShape(N, int(total_q), int(total_k), int(prefix), int(q_heads), int(kv_heads), 128, int(bool(causal)),
                        int(max_q))
    if out is None:
        need = L.chorus_packed_plan_bytes(ctypes.byref(shape))
        out = PackedPlan(torch.empty(need + 256, dtype=torch.uint8, device=q_offsets.device), shape, need)
    elif bytes(out.shape) != bytes(shape):
        raise ValueError("out is a plan of another shape")
    st = L.chorus_plan_packed_attn(ctypes.byref(shape), q_offsets.data_ptr(), k_offsets.data_ptr(), _ptr(k_lens),
                                   _aligned(out.data), out.plan_bytes, stream)
    _check(st, "chorus_plan_packed_attn")
    return out


def _rows(t: torch.Tensor, dims, dtype, name: str):
    """Pointer to a chorus_tensor of a [rows, heads, 128] tensor."""
    if t.shape != dims or t.dtype != dtype:
        raise ValueError(f"{name} must be a {dtype} {list(dims)} tensor")
    ss, sh, sd = t.stride()
    if sd != 1:
        raise ValueError("head dim must be contiguous")
    return ctypes.byref(Tensor(t.data_ptr(), 0, ss, sh))


def packed_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, plan: PackedPlan, sm_scale: float | None = None,
                    prefix_k: torch.Tensor | None = None, prefix_v: torch.Tensor | None = None,
                    out: torch.Tensor | None = None, return_lse: bool = False):
    """chorus_packed_attn_fwd: attention of ``q [total_q, q_heads, 128]`` to ``k, v [total_k, kv_heads, 128]`` (and
    ``prefix_k, prefix_v [prefix, kv_heads, 128]``) by ``plan``; f16 or bf16.  Returns ``out`` (and ``lse [q_heads,
    total_q]`` fp32 when ``return_lse``); rows of no sequence are not written."""
    L = load_library()
    stream = _current(q, k, v, prefix_k, prefix_v, out, plan.data)
    s, dtype = plan.shape, q.dtype
    dt = _dtype_code(q)
    if (prefix_k is None) != (s.prefix == 0) or (prefix_v is None) != (s.prefix == 0):
        raise ValueError(f"the plan's prefix has {s.prefix} rows")
    cq = _rows(q, plan.q_dims, dtype, "q")
    ck, cv = _rows(k, plan.k_dims, dtype, "k"), _rows(v, plan.k_dims, dtype, "v")
    cpk = cpv = None
    if prefix_k is not None:
        cpk = _rows(prefix_k, plan.prefix_dims, dtype, "prefix_k")
        cpv = _rows(prefix_v, plan.prefix_dims, dtype, "prefix_v")
    if out is None:
        out = torch.empty(plan.q_dims, dtype=dtype, device=q.device)
    else:
        _writable(out, "out")
    co = _rows(out, plan.q_dims, dtype, "out")
    lse = torch.empty((s.q_heads, s.total_q), dtype=torch.float32, device=q.device) if return_lse else None
    sm = 128 ** -0.5 if sm_scale is None else float(sm_scale)
    ws = _workspace(plan.workspace_bytes, q.device)
    st = L.chorus_packed_attn_fwd(dt, ctypes.byref(s), cq, ck, cv, cpk, cpv, sm, _aligned(plan.data), plan.plan_bytes, co,
                                  _ptr(lse), _aligned(ws), plan.workspace_bytes, stream)
    _check(st, "chorus_packed_attn_fwd")
    return (out, lse) if return_lse else out
