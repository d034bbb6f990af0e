"""Python binding of ``liblora_mi355x.so`` (the C ABI in include/lora_mi355x.h).

Argument marshalling only: every step of the LoRA forward and backward runs in
the library's HIP kernels on the caller's stream.  PyTorch provides device
memory and the current HIP stream.  If the library has not been built the
binding raises -- there is no fallback path.
"""
from __future__ import annotations

import bisect
import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "liblora_mi355x.so")

LORA_OK, LORA_EINVAL, LORA_EUNSUPPORTED, LORA_EWORKSPACE, LORA_EHIP = range(5)
LORA_BF16, LORA_F32 = 0, 1
LORA_OP_FWD, LORA_OP_BWD, LORA_OP_FROZEN_DX = 0, 1, 2

_lib = None


class _Node(ctypes.Structure):
    """lora_node_t of the C ABI."""
    _fields_ = [("W", ctypes.c_void_p), ("A", ctypes.c_void_p), ("B", ctypes.c_void_p),
                ("dA", ctypes.c_void_p), ("dB", ctypes.c_void_p), ("d_in", ctypes.c_int64),
                ("d_out", ctypes.c_int64), ("r", ctypes.c_int64), ("scale", ctypes.c_float)]


class _Plan(ctypes.Structure):
    """lora_plan_t of the C ABI."""
    _fields_ = [(n, ctypes.c_int) for n in ("fwd_tile_m", "fwd_tile_n", "fwd_fused", "fwd_u_parts",
                                             "bwd_tile_m", "bwd_tile_n", "bwd_fused", "bwd_du_parts",
                                             "bwd_side_parts")]


class _FewTokenPlan(ctypes.Structure):
    """lora_few_token_plan_t of the C ABI."""
    _fields_ = [(n, ctypes.c_int) for n in ("fwd_taken", "fwd_tiles_m", "fwd_tiles_n", "fwd_parts",
                                            "bwd_taken", "bwd_tiles_m", "bwd_tiles_n", "bwd_parts")]
    _fields_ += [(n, ctypes.c_size_t) for n in ("fwd_bytes", "bwd_bytes", "fwd_tiled_bytes", "bwd_tiled_bytes")]


class _X8Plan(ctypes.Structure):
    """lora_x8_plan_t of the C ABI."""
    _fields_ = [(n, ctypes.c_int) for n in ("few_tokens", "few_parts", "fused", "du_parts", "u_parts", "token_ranges")]


class _Grad(ctypes.Structure):
    """lora_grad_t of the C ABI."""
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dt", ctypes.c_int), ("out_dt", ctypes.c_int)]


class _GradList(ctypes.Structure):
    """lora_grad_list_t of the C ABI."""
    _fields_ = [("mem", ctypes.c_void_p), ("elems", ctypes.c_int64), ("nchunk", ctypes.c_int32),
                ("chunk", ctypes.c_int32), ("has_out", ctypes.c_int32)]


class _Act8(ctypes.Structure):
    """lora_act8_t of the C ABI."""
    _fields_ = [("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class _BlockNorm(ctypes.Structure):
    """block_norm_t of the C ABI."""
    _fields_ = [("T", ctypes.c_int64), ("D", ctypes.c_int64), ("dt", ctypes.c_int), ("res_dt", ctypes.c_int),
                ("post_norm", ctypes.c_int), ("gate_mode", ctypes.c_int), ("gain_offset", ctypes.c_double),
                ("res_scale", ctypes.c_double), ("w_post", ctypes.c_void_p), ("w_pre", ctypes.c_void_p),
                ("gate", ctypes.c_void_p)]


class LoraError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status} ({detail})")
        self.status = status


def lib() -> ctypes.CDLL:
    """Load the HIP library (once).  Raises if it is missing: build it with
    ``python -m paper_2606_19528_amd.build``."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"HIP library not built: {LIB_PATH} is missing "
                           "(run python -m paper_2606_19528_amd.build)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, f32, sz, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t, ctypes.c_int
    L.lora_linear_workspace_bytes.argtypes = [i32, i64, i64, i64, i64, i32]
    L.lora_linear_workspace_bytes.restype = sz
    L.lora_linear_fwd.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, f32, i32, vp, sz, vp]
    L.lora_linear_fwd.restype = i32
    L.lora_linear_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, f32, i32,
                                  vp, sz, vp]
    L.lora_linear_bwd.restype = i32
    L.lora_linear_bwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, f32, i32,
                                          vp]
    L.lora_linear_bwd_noalloc.restype = i32
    L.frozen_linear_bwd_dx.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, sz, vp]
    L.frozen_linear_bwd_dx.restype = i32
    L.lora_linear_fwd_q.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp, vp, i64, i64, i64, i64,
                                    f32, vp, sz, vp]
    L.lora_linear_fwd_q.restype = i32
    L.lora_linear_bwd_q.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp, i64, i64,
                                    i64, i64, f32, vp, sz, vp]
    L.lora_linear_bwd_q.restype = i32
    L.frozen_linear_bwd_dx_q.argtypes = [vp, vp, vp, vp, i32, i64, vp, i64, i64, i64, vp, sz, vp]
    L.frozen_linear_bwd_dx_q.restype = i32
    L.lm_head_workspace_bytes.argtypes = [i32, i64, i64, i64, i64, i64]
    L.lm_head_workspace_bytes.restype = sz
    L.lm_head_build_vocab.argtypes = [vp, i64, i64, i64, vp, i64, vp, i64, vp, vp,
                                      ctypes.POINTER(i64), vp, sz, vp]
    L.lm_head_build_vocab.restype = i32
    L.lm_head_reduced_ce.argtypes = [vp, vp, i64, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, f32,
                                     vp, sz, vp]
    L.lm_head_reduced_ce.restype = i32
    NP = ctypes.POINTER(_Node)
    L.lora_ckpt_workspace_bytes.argtypes = [NP, i32, i64]
    L.lora_ckpt_workspace_bytes.restype = sz
    L.lora_ckpt_host_bytes.argtypes = [NP, i32, i64]
    L.lora_ckpt_host_bytes.restype = sz
    L.lora_ckpt_forward.argtypes = [NP, i32, i64, vp, vp, vp, sz, vp, sz, vp, vp]
    L.lora_ckpt_forward.restype = i32
    L.lora_ckpt_backward.argtypes = [NP, i32, i64, vp, vp, vp, sz, vp, sz, vp, vp]
    L.lora_ckpt_backward.restype = i32
    L.topk_table_workspace_bytes.argtypes = [i64, i64, i64]
    L.topk_table_workspace_bytes.restype = sz
    L.frozen_linear_split_bytes.argtypes = [i64, i64, i64, ctypes.c_int]
    L.frozen_linear_split_bytes.restype = sz
    L.topk_table_workspace_bytes_paired.argtypes = [i64, i64, i64]
    L.topk_table_workspace_bytes_paired.restype = sz
    L.topk_table_build.argtypes = [vp, i64, i64, i64, vp, vp, vp, sz, vp]
    L.topk_table_build.restype = i32
    L.embed_fwd.argtypes = [vp, vp, vp, i64, i64, i64, f32, i32, vp]
    L.embed_fwd.restype = i32
    L.embed_bwd_workspace_bytes.argtypes = [i64, i64, i64]
    L.embed_bwd_workspace_bytes.restype = sz
    L.embed_bwd.argtypes = [vp, vp, vp, i64, i64, i64, f32, i32, i32, vp, sz, vp]
    L.embed_bwd.restype = i32
    L.embed_bwd_rows.argtypes = [vp, vp, vp, vp, i64, i64, i64, f32, i32, vp, sz, vp]
    L.embed_bwd_rows.restype = i32
    L.token_loss_workspace_bytes.argtypes = [i32, i64, i64, i64, i64, i32]
    L.token_loss_workspace_bytes.restype = sz
    L.token_logp.argtypes = [vp, i64, vp, vp, vp, i64, i64, i32, vp, sz, vp]
    L.token_logp.restype = i32
    L.policy_loss.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, f32, f32, f32, i32, vp, sz, vp]
    L.policy_loss.restype = i32
    L.preference_loss.argtypes = [vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, vp, i64, i64, f32, f32, i32, vp, sz, vp]
    L.preference_loss.restype = i32
    GP, LP = ctypes.POINTER(_Grad), ctypes.POINTER(_GradList)
    L.grad_list_bytes.argtypes = [GP, i64]
    L.grad_list_bytes.restype = sz
    L.grad_list_init.argtypes = [LP, GP, i64, vp, sz, vp]
    L.grad_list_init.restype = i32
    L.grad_norm.argtypes = [LP, vp, vp]
    L.grad_norm.restype = i32
    L.grad_clip.argtypes = [LP, f32, vp, vp]
    L.grad_clip.restype = i32
    L.act8_quantize.argtypes = [vp, vp, vp, i64, i64, i32, vp]
    L.act8_quantize.restype = i32
    L.act8_dequantize.argtypes = [vp, vp, vp, i64, i64, i32, vp]
    L.act8_dequantize.restype = i32
    L.lora_linear_x8_workspace_bytes.argtypes = [i64, i64, i64, i64]
    L.lora_linear_x8_workspace_bytes.restype = sz
    L.lora_linear_bwd_x8.argtypes = [vp] * 10 + [i64, i64, i64, i64, f32, vp, sz, vp]
    L.lora_linear_bwd_x8.restype = i32
    L.lora_linear_bwd_q_x8.argtypes = [vp] * 5 + [i32, i64] + [vp] * 7 + [i64, i64, i64, i64, f32, vp, sz, vp]
    L.lora_linear_bwd_q_x8.restype = i32
    for name in ("lora_ckpt_workspace_bytes_x8", "lora_ckpt_host_bytes_x8"):
        getattr(L, name).argtypes = [NP, i32, i64]
        getattr(L, name).restype = sz
    for name in ("lora_ckpt_forward_x8", "lora_ckpt_backward_x8"):
        getattr(L, name).argtypes = [NP, i32, i64, vp, vp, vp, sz, vp, sz, vp, vp]
        getattr(L, name).restype = i32
    BP, AP = ctypes.POINTER(_BlockNorm), ctypes.POINTER(_Act8)
    L.block_norm_fwd.argtypes = [BP, vp, vp, vp, vp, vp, vp, AP, AP, AP, ctypes.c_double, vp]
    L.block_norm_fwd.restype = i32
    L.block_norm_workspace_bytes.argtypes = [i64, i64]
    L.block_norm_workspace_bytes.restype = sz
    L.block_norm_bwd.argtypes = [BP, vp, vp, vp, AP, vp, AP] + [vp] * 8 + [sz, vp]
    L.block_norm_bwd.restype = i32
    L.lora_status_str.argtypes = [i32]
    L.lora_status_str.restype = ctypes.c_char_p
    L.lora_last_error.argtypes = []
    L.lora_last_error.restype = ctypes.c_char_p
    L.lora_profiler_enable.argtypes = [i32]
    L.lora_profiler_enable.restype = i32
    L.lora_profiler_reset.argtypes = []
    L.lora_profiler_reset.restype = i32
    L.lora_profiler_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
    L.lora_profiler_read.restype = i32
    L.lora_kernel_name.argtypes = [i32]
    L.lora_kernel_name.restype = ctypes.c_char_p
    L.lora_kernel_count.argtypes = []
    L.lora_kernel_count.restype = i32
    L.lora_linear_plan.argtypes = [i64, i64, i64, i64, i32, ctypes.POINTER(_Plan)]
    L.lora_linear_plan.restype = i32
    L.lora_few_token_plan.argtypes = [i64, i64, i64, i64, i32, ctypes.POINTER(_FewTokenPlan)]
    L.lora_few_token_plan.restype = i32
    L.lora_linear_x8_plan.argtypes = [i64, i64, i64, i64, i32, i32, ctypes.POINTER(_X8Plan)]
    L.lora_linear_x8_plan.restype = i32
    L.lora_debug_host_mapped.argtypes = [vp, sz]
    L.lora_debug_host_mapped.restype = i32
    L.lora_handover_giveups.argtypes = [ctypes.POINTER(ctypes.c_uint64), i32]
    L.lora_handover_giveups.restype = i32
    L.lora_debug_set_handover.argtypes = [i32]
    L.lora_debug_set_handover.restype = i32
    _lib = L
    return L


def _check(status: int, where: str):
    if status != LORA_OK:
        detail = lib().lora_last_error().decode()
        raise LoraError(status, where, detail)


def _dtype_code(t) -> int:
    import torch

    if t.dtype == torch.bfloat16:
        return LORA_BF16
    if t.dtype == torch.float32:
        return LORA_F32
    raise TypeError(f"unsupported dtype {t.dtype} (bf16 or fp32)")


def _ptr(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous (row-major, no padding)")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    import torch

    if stream is None:
        # (the current stream's handle; building torch's Stream object for it takes 3 us, so that
        # is left to a torch without this function, which is not public)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return ctypes.c_void_p(raw(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ws(ws, nbytes: int, like, stream=None):
    """The caller's workspace, or a temporary one.  A temporary is allocated on
    the stream the call is enqueued on, so the caching allocator does not hand
    its block to another tensor while that stream's kernels still use it."""
    import torch

    if nbytes == 0:
        return None, 0
    if ws is None:
        if stream is None:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
        else:
            with torch.cuda.stream(stream):
                ws = torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    return ws, ws.numel() * ws.element_size()


def _ws_optional(nbytes: int, like, stream=None):
    """A temporary workspace that speeds a call up but is not needed by it:
    None where the device has no room.  (A caller that wants neither the
    allocation nor its failure passes a workspace of its own.)"""
    import torch

    try:
        return _ws(None, nbytes, like, stream)[0]
    except torch.cuda.OutOfMemoryError:
        return None


def lora_linear_workspace_bytes(op: int, T: int, d_in: int, d_out: int, r: int, dt: int) -> int:
    n = lib().lora_linear_workspace_bytes(op, T, d_in, d_out, r, dt)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "lora_linear_workspace_bytes", lib().lora_last_error().decode())
    return int(n)


def lora_linear_fwd(x, W, A, B, y, u_save=None, scale: float = 1.0, ws=None, stream=None):
    """y = x W^T + scale (x A^T) B^T; u_save (fp32 [T, r]) receives x A^T."""
    T, d_in = x.shape
    d_out = W.shape[0]
    r = 0 if A is None else A.shape[0]
    dt = _dtype_code(x)
    ws, ws_bytes = _ws(ws, lora_linear_workspace_bytes(LORA_OP_FWD, T, d_in, d_out, r, dt), x, stream)
    st = lib().lora_linear_fwd(_ptr(x), _ptr(W), _ptr(A), _ptr(B), _ptr(y), _ptr(u_save), T, d_in,
                               d_out, r, float(scale), dt, _ptr(ws), ws_bytes, _stream(stream))
    _check(st, "lora_linear_fwd")
    return y


def lora_linear_bwd(x, W, A, B, u_saved, dy, dx, dA, dB, scale: float = 1.0, ws=None, stream=None):
    """dx = dy W + du A, dA = du^T x, dB = scale dy^T u with du = scale dy B."""
    T, d_out = dy.shape
    d_in = W.shape[1]
    r = 0 if A is None else A.shape[0]
    dt = _dtype_code(dy)
    ws, ws_bytes = _ws(ws, lora_linear_workspace_bytes(LORA_OP_BWD, T, d_in, d_out, r, dt), dy, stream)
    st = lib().lora_linear_bwd(_ptr(x), _ptr(W), _ptr(A), _ptr(B), _ptr(u_saved), _ptr(dy),
                               _ptr(dx), _ptr(dA), _ptr(dB), T, d_in, d_out, r, float(scale), dt,
                               _ptr(ws), ws_bytes, _stream(stream))
    _check(st, "lora_linear_bwd")
    return dx, dA, dB


def lora_linear_bwd_noalloc(x, W, A, B, u_saved, dy, dx, dA, dB, scale: float = 1.0, stream=None):
    """lora_linear_bwd with the library's static device scratch as workspace
    (no allocation by the library or by this wrapper)."""
    T, d_out = dy.shape
    d_in = W.shape[1]
    r = 0 if A is None else A.shape[0]
    dt = _dtype_code(dy)
    st = lib().lora_linear_bwd_noalloc(_ptr(x), _ptr(W), _ptr(A), _ptr(B), _ptr(u_saved), _ptr(dy),
                                       _ptr(dx), _ptr(dA), _ptr(dB), T, d_in, d_out, r, float(scale), dt,
                                       _stream(stream))
    _check(st, "lora_linear_bwd_noalloc")
    return dx, dA, dB


def _split_ws(T, d_in, d_out, dt, like, stream):
    n = lib().frozen_linear_split_bytes(T, d_in, d_out, dt)
    return None if n == 0 or n == ctypes.c_size_t(-1).value else _ws_optional(int(n), like, stream)


def frozen_linear_bwd_dx(dy, W, dx, ws=None, stream=None):
    """Rank-0 frozen linear input gradient dx = dy W.

    Without `ws`, a long reduction is split over a temporary workspace of up to 64
    MiB (frozen_linear_split_bytes), or, where the device has no room for it, runs
    unsplit, with sums in another order.  A `ws` of the caller's fixes which: one of
    that size splits, a smaller one (an empty tensor too) does not."""
    T, d_out = dy.shape
    d_in = W.shape[1]
    dt = _dtype_code(dy)
    if ws is None:
        ws = _split_ws(T, d_in, d_out, dt, dy, stream)
    st = lib().frozen_linear_bwd_dx(_ptr(dy), _ptr(W), _ptr(dx), T, d_in, d_out, dt, _ptr(ws),
                                    0 if ws is None else ws.numel() * ws.element_size(),
                                    _stream(stream))
    _check(st, "frozen_linear_bwd_dx")
    return dx


# --- quantized frozen base (codes + per-group scale / offset) ----------------------
def _qw(Wq):
    """(codes, scale, offset, bits, group, d_out, d_in) of a quantized weight given
    as a dict with keys codes (uint8 [d_out, d_in*bits/8]), scale and offset
    (fp32 [d_in/group, d_out], group-major) and bits."""
    codes, sc, off, bits = Wq["codes"], Wq["scale"], Wq["offset"], int(Wq["bits"])
    d_out = codes.shape[0]
    d_in = codes.shape[1] * 8 // bits
    group = d_in // sc.shape[0]
    return codes, sc, off, bits, group, d_out, d_in


def lora_linear_fwd_q(x, Wq, A, B, y, u_save=None, scale: float = 1.0, ws=None, stream=None):
    """lora_linear_fwd with the frozen W quantized (dict, see _qw)."""
    codes, sc, off, bits, group, d_out, d_in = _qw(Wq)
    T = x.shape[0]
    r = 0 if A is None else A.shape[0]
    ws, ws_bytes = _ws(ws, lora_linear_workspace_bytes(LORA_OP_FWD, T, d_in, d_out, r, LORA_BF16), x, stream)
    st = lib().lora_linear_fwd_q(_ptr(x), _ptr(codes), _ptr(sc), _ptr(off), bits, group, _ptr(A),
                                 _ptr(B), _ptr(y), _ptr(u_save), T, d_in, d_out, r, float(scale),
                                 _ptr(ws), ws_bytes, _stream(stream))
    _check(st, "lora_linear_fwd_q")
    return y


def lora_linear_bwd_q(x, Wq, A, B, u_saved, dy, dx, dA, dB, scale: float = 1.0, ws=None,
                      stream=None):
    """lora_linear_bwd with the frozen W quantized (dict, see _qw)."""
    codes, sc, off, bits, group, d_out, d_in = _qw(Wq)
    T = dy.shape[0]
    r = 0 if A is None else A.shape[0]
    ws, ws_bytes = _ws(ws, lora_linear_workspace_bytes(LORA_OP_BWD, T, d_in, d_out, r, LORA_BF16), dy, stream)
    st = lib().lora_linear_bwd_q(_ptr(x), _ptr(codes), _ptr(sc), _ptr(off), bits, group, _ptr(A),
                                 _ptr(B), _ptr(u_saved), _ptr(dy), _ptr(dx), _ptr(dA), _ptr(dB), T,
                                 d_in, d_out, r, float(scale), _ptr(ws), ws_bytes, _stream(stream))
    _check(st, "lora_linear_bwd_q")
    return dx, dA, dB


def frozen_linear_bwd_dx_q(dy, Wq, dx, ws=None, stream=None):
    """frozen_linear_bwd_dx with W quantized (dict, see _qw)."""
    codes, sc, off, bits, group, d_out, d_in = _qw(Wq)
    T = dy.shape[0]
    if ws is None:
        ws = _split_ws(T, d_in, d_out, LORA_BF16, dy, stream)
    st = lib().frozen_linear_bwd_dx_q(_ptr(dy), _ptr(codes), _ptr(sc), _ptr(off), bits, group,
                                      _ptr(dx), T, d_in, d_out, _ptr(ws),
                                      0 if ws is None else ws.numel() * ws.element_size(),
                                      _stream(stream))
    _check(st, "frozen_linear_bwd_dx_q")
    return dx


# --- frozen LM head: reduced-vocabulary cross entropy with logits masking -----------
LM_HEAD_OP_VOCAB, LM_HEAD_OP_LOSS, LM_HEAD_OP_LOSS_DH = 0, 1, 2


def lm_head_workspace_bytes(op: int, T: int, V: int, D: int, nrows: int, nJ: int = 1) -> int:
    n = lib().lm_head_workspace_bytes(op, T, V, D, nrows, nJ)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "lm_head_workspace_bytes", "sizes rejected")
    return int(n)


def lm_head_build_vocab(table, k: int, targets, rows, ws=None, stream=None):
    """(J [nJ] int32, tpos [nrows] int32) on the device; waits for the stream."""
    import torch

    V, ldtab = table.shape
    T = targets.shape[0]
    nrows = rows.shape[0]
    J = torch.empty(V, dtype=torch.int32, device=table.device)
    tpos = torch.empty(nrows, dtype=torch.int32, device=table.device)
    ws, ws_bytes = _ws(ws, lm_head_workspace_bytes(LM_HEAD_OP_VOCAB, T, V, 8, nrows), table, stream)
    nJ = ctypes.c_int64(0)
    st = lib().lm_head_build_vocab(_ptr(table), V, ldtab, k, _ptr(targets), T, _ptr(rows), nrows,
                                   _ptr(J), _ptr(tpos), ctypes.byref(nJ), _ptr(ws), ws_bytes,
                                   _stream(stream))
    _check(st, "lm_head_build_vocab")
    return J[: nJ.value], tpos


def lm_head_reduced_ce(h, W, rows, J, tpos, loss_rows, loss_total=None, dh=None,
                       dscale: float = 1.0, ws=None, stream=None):
    """Per-position losses (and their sum, and dh) of the reduced-vocabulary
    cross entropy over the trainable positions `rows`."""
    T, D = h.shape
    V = W.shape[0]
    nrows, nJ = rows.shape[0], J.shape[0]
    op = LM_HEAD_OP_LOSS if dh is None else LM_HEAD_OP_LOSS_DH
    ws, ws_bytes = _ws(ws, lm_head_workspace_bytes(op, T, V, D, nrows, nJ), h, stream)
    st = lib().lm_head_reduced_ce(_ptr(h), _ptr(W), T, V, D, _ptr(rows), nrows, _ptr(J), nJ,
                                  _ptr(tpos), _ptr(loss_rows), _ptr(loss_total), _ptr(dh),
                                  float(dscale), _ptr(ws), ws_bytes, _stream(stream))
    _check(st, "lm_head_reduced_ce")
    return loss_rows


# --- top-k similarity table ---------------------------------------------------------
def topk_table_build(W, k: int, table=None, values=None, ws=None, stream=None):
    """table [V, k] int32 (and optionally values [V, k] fp32) of each token's k
    most cosine-similar tokens.

    Without `ws`, a temporary workspace of topk_table_workspace_bytes_paired (7.4 GB
    at V = 128256, k = 1000) is taken where the device has room, else the smaller
    one of topk_table_workspace_bytes; a `ws` of the caller's fixes which.  Table and
    values are the same bitwise."""
    import torch

    V, D = W.shape
    if table is None:
        table = torch.empty(V, k, dtype=torch.int32, device=W.device)
    n = lib().topk_table_workspace_bytes(V, D, k)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "topk_table_workspace_bytes", "sizes rejected")
    if ws is None:
        ws = _ws_optional(int(lib().topk_table_workspace_bytes_paired(V, D, k)), W, stream)
    ws, ws_bytes = _ws(ws, int(n), W, stream)
    st = lib().topk_table_build(_ptr(W), V, D, k, _ptr(table), _ptr(values), _ptr(ws), ws_bytes,
                                _stream(stream))
    _check(st, "topk_table_build")
    return table


# --- checkpointed step over a chain of LoRA linears ---------------------------------
def _nodes(nodes):
    arr = (_Node * len(nodes))()
    for i, nd in enumerate(nodes):
        W, A, B = nd["W"], nd.get("A"), nd.get("B")
        r = 0 if A is None else A.shape[0]
        arr[i] = _Node(W.data_ptr(), None if A is None else A.data_ptr(),
                       None if B is None else B.data_ptr(),
                       None if nd.get("dA") is None else nd["dA"].data_ptr(),
                       None if nd.get("dB") is None else nd["dB"].data_ptr(),
                       W.shape[1], W.shape[0], r, float(nd.get("scale", 1.0)))
    return arr


def lora_ckpt_sizes(nodes, T: int):
    """(device workspace bytes, pinned host stash bytes) of a checkpointed step."""
    arr = _nodes(nodes)
    w = lib().lora_ckpt_workspace_bytes(arr, len(nodes), T)
    h = lib().lora_ckpt_host_bytes(arr, len(nodes), T)
    if w == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "lora_ckpt_workspace_bytes", "chain rejected")
    return int(w), int(h)


def lora_ckpt_forward(nodes, x0, out, host_stash, ws, compute_stream=None, copy_stream=None):
    """Checkpointed forward: out = x_n; every node input goes to host_stash
    (pinned) on copy_stream.  nodes: dicts W, A, B, dA, dB, scale."""
    arr = _nodes(nodes)
    T = x0.shape[0]
    st = lib().lora_ckpt_forward(arr, len(nodes), T, _ptr(x0), _ptr(out), _ptr(host_stash),
                                 host_stash.numel() * host_stash.element_size(), _ptr(ws),
                                 ws.numel() * ws.element_size(), _stream(compute_stream),
                                 _stream(copy_stream))
    _check(st, "lora_ckpt_forward")
    return out


def lora_ckpt_backward(nodes, g_n, dx0, host_stash, ws, compute_stream=None, copy_stream=None):
    """Checkpointed backward from g_n = dL/dx_n: fills every node's dA, dB and dx0."""
    arr = _nodes(nodes)
    T = g_n.shape[0]
    st = lib().lora_ckpt_backward(arr, len(nodes), T, _ptr(g_n), _ptr(dx0), _ptr(host_stash),
                                  host_stash.numel() * host_stash.element_size(), _ptr(ws),
                                  ws.numel() * ws.element_size(), _stream(compute_stream),
                                  _stream(copy_stream))
    _check(st, "lora_ckpt_backward")
    return dx0


def lora_ckpt_sizes_x8(nodes, T: int):
    """lora_ckpt_sizes of a step with its stash in 8 bits."""
    arr = _nodes(nodes)
    w = lib().lora_ckpt_workspace_bytes_x8(arr, len(nodes), T)
    h = lib().lora_ckpt_host_bytes_x8(arr, len(nodes), T)
    if w == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "lora_ckpt_workspace_bytes_x8", "chain rejected")
    return int(w), int(h)


def lora_ckpt_forward_x8(nodes, x0, out, host_stash, ws, compute_stream=None, copy_stream=None):
    """lora_ckpt_forward with every node input quantized to 8 bits before it leaves for the host."""
    arr = _nodes(nodes)
    T = x0.shape[0]
    st = lib().lora_ckpt_forward_x8(arr, len(nodes), T, _ptr(x0), _ptr(out), _ptr(host_stash),
                                    host_stash.numel() * host_stash.element_size(), _ptr(ws),
                                    ws.numel() * ws.element_size(), _stream(compute_stream),
                                    _stream(copy_stream))
    _check(st, "lora_ckpt_forward_x8")
    return out


def lora_ckpt_backward_x8(nodes, g_n, dx0, host_stash, ws, compute_stream=None, copy_stream=None):
    """lora_ckpt_backward from a stash of lora_ckpt_forward_x8."""
    arr = _nodes(nodes)
    T = g_n.shape[0]
    st = lib().lora_ckpt_backward_x8(arr, len(nodes), T, _ptr(g_n), _ptr(dx0), _ptr(host_stash),
                                     host_stash.numel() * host_stash.element_size(), _ptr(ws),
                                     ws.numel() * ws.element_size(), _stream(compute_stream),
                                     _stream(copy_stream))
    _check(st, "lora_ckpt_backward_x8")
    return dx0


# --- embedding, losses over the targets, clipping ------------------------------------
def _arg(t, name: str, dtype, shape):
    """Address of a tensor argument; refuses one of another type, shape, layout or
    place than the call takes."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous (row-major, no padding)")
    return t.data_ptr()


def _opt(t, name: str, dtype, shape):
    return None if t is None else _arg(t, name, dtype, shape)


def _ws_for(ws, query, like, stream):
    """(address, bytes) of the caller's workspace, or of a temporary one of the size
    that `query` reports, and the tensor itself."""
    if ws is None:
        ws, nbytes = _ws(None, query(), like, stream)
        return (None, 0, None) if ws is None else (ws.data_ptr(), nbytes, ws)
    return _ptr(ws), ws.numel() * ws.element_size(), ws


def embed_fwd(table, ids, out, scale: float = 1.0, stream=None):
    """out[t] = scale table[ids[t]]; an id outside the table gives zeros."""
    import torch

    (V, D), T = table.shape, ids.shape[0]
    dt, ty = _dtype_code(table), table.dtype
    st = lib().embed_fwd(_arg(table, "table", ty, (V, D)), _arg(ids, "ids", torch.int32, (T,)), _arg(out, "out", ty, (T, D)),
                         T, V, D, scale, dt, _stream(stream))
    _check(st, "embed_fwd")
    return out


def embed_bwd_workspace_bytes(T: int, V: int, D: int) -> int:
    n = lib().embed_bwd_workspace_bytes(T, V, D)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "embed_bwd_workspace_bytes", lib().lora_last_error().decode())
    return int(n)


def embed_bwd(ids, dout, dtable, scale: float = 1.0, accumulate: bool = False, ws=None, stream=None):
    """dtable[v] = scale times the sum of dout over the positions of token v
    (added to dtable with `accumulate`)."""
    import torch

    (T, D), V = dout.shape, dtable.shape[0]
    dt = _dtype_code(dout)
    args = (_arg(ids, "ids", torch.int32, (T,)), _arg(dout, "dout", dout.dtype, (T, D)),
            _arg(dtable, "dtable", torch.float32, (V, D)))
    wp, wn, ws = _ws_for(ws, lambda: embed_bwd_workspace_bytes(T, V, D), dout, stream)
    st = lib().embed_bwd(*args, T, V, D, scale, 1 if accumulate else 0, dt, wp, wn, _stream(stream))
    _check(st, "embed_bwd")
    return dtable


def embed_bwd_rows(ids, dout, V: int, tokens, rows, scale: float = 1.0, ws=None, stream=None):
    """embed_bwd without the rows of absent tokens: tokens [min(T, V)] receives the
    distinct ids in ascending order and then -1, rows their gradients and then zeros."""
    import torch

    T, D = dout.shape
    dt, n = _dtype_code(dout), min(T, V)
    args = (_arg(ids, "ids", torch.int32, (T,)), _arg(dout, "dout", dout.dtype, (T, D)),
            _arg(tokens, "tokens", torch.int32, (n,)), _arg(rows, "rows", torch.float32, (n, D)))
    wp, wn, ws = _ws_for(ws, lambda: embed_bwd_workspace_bytes(T, V, D), dout, stream)
    st = lib().embed_bwd_rows(*args, T, V, D, scale, dt, wp, wn, _stream(stream))
    _check(st, "embed_bwd_rows")
    return tokens, rows


TOKEN_LOSS_OP_LOGP, TOKEN_LOSS_OP_POLICY, TOKEN_LOSS_OP_PREFERENCE = 0, 1, 2


def token_loss_workspace_bytes(op: int, T: int, V: int, ldz: int, npairs: int = 0, dt: int = LORA_BF16) -> int:
    n = lib().token_loss_workspace_bytes(op, T, V, ldz, npairs, dt)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "token_loss_workspace_bytes", lib().lora_last_error().decode())
    return int(n)


def token_logp(logits, targets, logp, weights=None, vocab=None, ws=None, stream=None):
    """logp[t] = log softmax(logits[t, :vocab])[targets[t]]; 0 where weights[t] is 0."""
    import torch

    T, ldz = logits.shape
    V, dt, f32 = ldz if vocab is None else vocab, _dtype_code(logits), torch.float32
    args = (_arg(logits, "logits", logits.dtype, (T, ldz)), ldz, _arg(targets, "targets", torch.int32, (T,)),
            _opt(weights, "weights", f32, (T,)), _arg(logp, "logp", f32, (T,)))
    wp, wn, ws = _ws_for(ws, lambda: token_loss_workspace_bytes(TOKEN_LOSS_OP_LOGP, T, V, ldz, 0, dt), logits, stream)
    st = lib().token_logp(*args, T, V, dt, wp, wn, _stream(stream))
    _check(st, "token_logp")
    return logp


def policy_loss(logits, targets, weights, advantages, old_logp, ref_logp, loss, logp, dlogits=None, clip_lo: float = 0.2,
                clip_hi: float = 0.2, kl_coef: float = 0.0, vocab=None, ws=None, stream=None):
    """Clipped policy loss with a KL term (see the header): fills loss [1], logp [T]
    and, when given, dlogits (which may be logits)."""
    import torch

    T, ldz = logits.shape
    V, dt, f32 = ldz if vocab is None else vocab, _dtype_code(logits), torch.float32
    args = (_arg(logits, "logits", logits.dtype, (T, ldz)), ldz, _arg(targets, "targets", torch.int32, (T,)),
            _opt(weights, "weights", f32, (T,)), _arg(advantages, "advantages", f32, (T,)), _arg(old_logp, "old_logp", f32, (T,)),
            _opt(ref_logp, "ref_logp", f32, (T,)), _arg(loss, "loss", f32, (1,)), _arg(logp, "logp", f32, (T,)),
            _opt(dlogits, "dlogits", logits.dtype, (T, ldz)))
    wp, wn, ws = _ws_for(ws, lambda: token_loss_workspace_bytes(TOKEN_LOSS_OP_POLICY, T, V, ldz, 0, dt), logits, stream)
    st = lib().policy_loss(*args, T, V, clip_lo, clip_hi, kl_coef, dt, wp, wn, _stream(stream))
    _check(st, "policy_loss")
    return loss


def preference_loss(logits, targets, weights, ref_logp, seq, loss, margins, logp, dlogits=None, beta: float = 0.1,
                    label_smoothing: float = 0.0, vocab=None, ws=None, stream=None):
    """Preference loss of the pairs of sequences that seq [2 pairs + 1] delimits (see
    the header): fills loss [1], margins [pairs], logp [T] and, when given, dlogits."""
    import torch

    (T, ldz), npairs = logits.shape, margins.shape[0]
    V, dt, f32 = ldz if vocab is None else vocab, _dtype_code(logits), torch.float32
    args = (_arg(logits, "logits", logits.dtype, (T, ldz)), ldz, _arg(targets, "targets", torch.int32, (T,)),
            _opt(weights, "weights", f32, (T,)), _opt(ref_logp, "ref_logp", f32, (T,)),
            _arg(seq, "seq", torch.int32, (2 * npairs + 1,)), npairs, _arg(loss, "loss", f32, (1,)),
            _arg(margins, "margins", f32, (npairs,)), _arg(logp, "logp", f32, (T,)),
            _opt(dlogits, "dlogits", logits.dtype, (T, ldz)))
    wp, wn, ws = _ws_for(ws, lambda: token_loss_workspace_bytes(TOKEN_LOSS_OP_PREFERENCE, T, V, ldz, npairs, dt), logits, stream)
    st = lib().preference_loss(*args, T, V, beta, label_smoothing, dt, wp, wn, _stream(stream))
    _check(st, "preference_loss")
    return loss


class GradList:
    """Gradients laid out for grad_norm and grad_clip (grad_list).  Holds the
    tensors, so that their memory stays theirs."""

    def __init__(self, grads, out=None, stream=None):
        import torch

        grads = list(grads)
        out = grads if out is None else list(out)
        if len(out) != len(grads):
            raise ValueError("as many outputs as gradients are required")
        arr = (_Grad * max(len(grads), 1))()
        ranges = []
        for i, (g, o) in enumerate(zip(grads, out)):
            n = g.numel()
            if o.numel() != n:
                raise ValueError("an output has another size than its gradient")
            dg, do = _dtype_code(g), _dtype_code(o)
            pg, po = _arg(g, "a gradient", g.dtype, g.shape), _arg(o, "an output", o.dtype, o.shape)
            arr[i] = _Grad(pg, po, n, dg, do)
            if n:
                ranges.append((pg, pg + n * (2 if dg == LORA_BF16 else 4)))
                if po != pg:
                    ranges.append((po, po + n * (2 if do == LORA_BF16 else 4)))
        n = lib().grad_list_bytes(arr, len(grads))
        if n == ctypes.c_size_t(-1).value:
            raise LoraError(LORA_EINVAL, "grad_list_bytes", lib().lora_last_error().decode())
        self.mem, nbytes = _ws(None, int(n), grads[0], stream)
        self.list = _GradList()
        self.ref = ctypes.byref(self.list)
        self.tensors = (grads, out)
        # Where the listed tensors lie, as disjoint ranges in ascending order (_list_args).
        self.starts, self.ends = [], []
        end = -1
        for lo, hi in sorted(ranges):
            if lo > end:
                self.starts.append(lo)
                self.ends.append(hi)
                end = hi
            elif hi > end:
                self.ends[-1] = end = hi
        st = _stream(stream)
        self.stream = st.value
        _check(lib().grad_list_init(self.ref, arr, len(grads), _ptr(self.mem), nbytes, st), "grad_list_init")


def _list_args(grads: GradList, norm, n: int, stream, where: str):
    """(list, address of norm [n], stream) for a call on a list."""
    import torch

    at = _arg(norm, "norm", torch.float32, (n,))
    # A norm in a listed tensor would be written while others read there.  (The C entry points
    # cannot refuse it: the list's addresses are in device memory.)
    i = bisect.bisect_right(grads.ends, at)  # the first range that ends behind `at`
    if i < len(grads.starts) and grads.starts[i] < at + 4 * n:
        raise LoraError(LORA_EINVAL, where, "norm overlaps a listed gradient or output")
    st = _stream(stream)
    if st.value != grads.stream:
        # The list's memory was allocated on the stream that laid it out: the allocator keeps
        # it until this one, too, is done with it.
        grads.mem.record_stream(torch.cuda.current_stream() if stream is None else stream)
    return grads.ref, at, st


def grad_list(grads, out=None, stream=None) -> GradList:
    """Lays out a step's gradients (bf16 or fp32 tensors) once for grad_norm and
    grad_clip; `out` receives the clipped gradients (default: in place)."""
    return GradList(grads, out, stream)


def grad_norm(grads: GradList, norm, stream=None):
    """norm [1] = global norm of the listed gradients."""
    ref, at, st = _list_args(grads, norm, 1, stream, "grad_norm")
    _check(lib().grad_norm(ref, at, st), "grad_norm")
    return norm


def grad_clip(grads: GradList, max_norm: float, norm, stream=None):
    """Scales the listed gradients so that their global norm is at most max_norm;
    norm [2] receives the norm before and the factor."""
    ref, at, st = _list_args(grads, norm, 2, stream, "grad_clip")
    _check(lib().grad_clip(ref, max_norm, at, st), "grad_clip")
    return norm


# --- activations in 8 bits, and the backward from them --------------------------------
ACT8_GROUP = 128


_names = None


def _torch_names():
    """torch and its types, looked up once: an import statement in each of a call's helpers takes
    longer than the call's launch where the sizes are small."""
    global _names
    if _names is None:
        import torch

        _names = (torch, torch.bfloat16, torch.float32, torch.int8, {torch.bfloat16: LORA_BF16, torch.float32: LORA_F32},
                  getattr(torch._C, "_cuda_getCurrentRawStream", None))
    return _names


def _stream_on(stream, dev: int):
    """_stream, for a caller that knows the current device."""
    if stream is None:
        raw = _torch_names()[5]
        if raw is not None:
            return raw(dev)
    return _stream(stream)


def _code(dtype) -> int:
    code = _torch_names()[4].get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype} (bf16 or fp32)")
    return code


def _dev_arg(t, name: str, dtype, shape, dev: int):
    """_arg of a tensor that has to be on device `dev`, the current one."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the current GPU")
    raise ValueError("tensors must be contiguous (row-major, no padding)")


def _dev_opt(t, name: str, dtype, shape, dev: int):
    return None if t is None else _dev_arg(t, name, dtype, shape, dev)


def _x8_args(x8, name: str, T: int, D: int, dev: int):
    """Addresses of (codes, scale) of an activation [T, D] in 8 bits."""
    codes, scale = x8
    _, _, f32, i8, _, _ = _torch_names()
    return (_dev_arg(codes, name + "'s codes", i8, (T, D), dev),
            _dev_arg(scale, name + "'s scale", f32, (T, -(-D // ACT8_GROUP)), dev))


def act8_empty(T: int, D: int, device="cuda"):
    """(codes int8 [T, D], scale fp32 [T, ceil(D / 128)]) for an activation [T, D] in 8 bits."""
    import torch

    return (torch.empty(T, D, dtype=torch.int8, device=device),
            torch.empty(T, -(-D // ACT8_GROUP), dtype=torch.float32, device=device))


def act8_quantize(x, x8, stream=None):
    """x8 = (codes, scale) of x [T, D]: of each 128 columns of a row the largest magnitude over
    127, and the nearest multiples of it."""
    shape, dt, dev = x.shape, x.dtype, _torch_names()[0].cuda.current_device()
    T, D = shape
    code = _code(dt)
    st = lib().act8_quantize(_dev_arg(x, "x", dt, shape, dev), *_x8_args(x8, "x8", T, D, dev), T, D, code, _stream_on(stream, dev))
    if st:
        _check(st, "act8_quantize")
    return x8


def act8_dequantize(x8, x, stream=None):
    """x [T, D] = scale times codes, rounded to x's type."""
    shape, dt, dev = x.shape, x.dtype, _torch_names()[0].cuda.current_device()
    T, D = shape
    code = _code(dt)
    st = lib().act8_dequantize(*_x8_args(x8, "x8", T, D, dev), _dev_arg(x, "x", dt, shape, dev), T, D, code, _stream_on(stream, dev))
    if st:
        _check(st, "act8_dequantize")
    return x


def lora_linear_x8_workspace_bytes(T: int, d_in: int, d_out: int, r: int) -> int:
    n = lib().lora_linear_x8_workspace_bytes(T, d_in, d_out, r)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "lora_linear_x8_workspace_bytes", lib().lora_last_error().decode())
    return int(n)


def _bwd_x8_args(x8, A, B, u_saved, dy, dx, dA, dB, T, d_in, d_out, dev):
    _, bf, f32, _, _, _ = _torch_names()
    r = 0 if A is None else A.shape[0]
    # (at rank 0 x, A and B do not enter)
    head = _x8_args(x8, "x8", T, d_in, dev) if r else (None, None)
    AB = (_dev_arg(A, "A", bf, (r, d_in), dev), _dev_arg(B, "B", bf, (d_out, r), dev)) if r else (None, None)
    grads = (_dev_arg(dA, "dA", f32, (r, d_in), dev), _dev_arg(dB, "dB", f32, (d_out, r), dev)) if r else (None, None)
    return r, head, (*AB, _dev_opt(u_saved, "u_saved", f32, (T, r), dev) if r else None, _dev_arg(dy, "dy", bf, (T, d_out), dev),
                     _dev_opt(dx, "dx", bf, (T, d_in), dev), *grads)


def lora_linear_bwd_x8(x8, W, A, B, u_saved, dy, dx, dA, dB, scale: float = 1.0, ws=None, stream=None):
    """lora_linear_bwd from an x kept in 8 bits (act8_quantize); u_saved None recomputes u from it."""
    (T, d_out), d_in, dev = dy.shape, W.shape[1], _torch_names()[0].cuda.current_device()
    r, head, rest = _bwd_x8_args(x8, A, B, u_saved, dy, dx, dA, dB, T, d_in, d_out, dev)
    wp, wn, ws = _ws_for(ws, lambda: lora_linear_x8_workspace_bytes(T, d_in, d_out, r), dy, stream)
    st = lib().lora_linear_bwd_x8(*head, _dev_arg(W, "W", _torch_names()[1], (d_out, d_in), dev), *rest, T, d_in, d_out, r, scale, wp,
                                  wn, _stream_on(stream, dev))
    _check(st, "lora_linear_bwd_x8")
    return dx, dA, dB


def lora_linear_bwd_q_x8(x8, Wq, A, B, u_saved, dy, dx, dA, dB, scale: float = 1.0, ws=None, stream=None):
    """lora_linear_bwd_x8 with the frozen W quantized (dict, see _qw)."""
    import torch

    codes, sc, off, bits, group, d_out, d_in = _qw(Wq)
    T, dev = dy.shape[0], torch.cuda.current_device()
    r, head, rest = _bwd_x8_args(x8, A, B, u_saved, dy, dx, dA, dB, T, d_in, d_out, dev)
    weight = (_dev_arg(codes, "codes", torch.uint8, (d_out, codes.shape[1]), dev),
              _dev_arg(sc, "scale", torch.float32, (sc.shape[0], d_out), dev),
              _dev_arg(off, "offset", torch.float32, (sc.shape[0], d_out), dev))
    wp, wn, ws = _ws_for(ws, lambda: lora_linear_x8_workspace_bytes(T, d_in, d_out, r), dy, stream)
    st = lib().lora_linear_bwd_q_x8(*head, *weight, bits, group, *rest, T, d_in, d_out, r, scale, wp, wn, _stream_on(stream, dev))
    _check(st, "lora_linear_bwd_q_x8")
    return dx, dA, dB


# --- norms, gate and residual sum between two blocks ----------------------------------
BLOCK_GATE_NONE, BLOCK_GATE_CHANNEL, BLOCK_GATE_TOKEN, BLOCK_GATE_FULL = range(4)


def _gate_mode(gate, T: int, D: int) -> int:
    if gate is None:
        return BLOCK_GATE_NONE
    for mode, shape in ((BLOCK_GATE_CHANNEL, (D,)), (BLOCK_GATE_TOKEN, (T, 1)), (BLOCK_GATE_FULL, (T, D))):
        if gate.shape == shape:
            return mode
    raise ValueError(f"gate has shape {tuple(gate.shape)}, expected ({D},), ({T}, 1) or ({T}, {D})")


def _block(T, D, dtype, res_dtype, post_norm, w_post, w_pre, gate, gain_offset, res_scale, dev):
    if post_norm is None:
        post_norm = w_post is not None
    mode = _gate_mode(gate, T, D)
    return _BlockNorm(T, D, _code(dtype), _code(res_dtype), 1 if post_norm else 0, mode, gain_offset, res_scale,
                      _dev_opt(w_post, "w_post", dtype, (D,), dev), _dev_opt(w_pre, "w_pre", dtype, (D,), dev),
                      None if gate is None else _dev_arg(gate, "gate", dtype, gate.shape, dev))


def _act8(x8, name, T, D, dev):
    return None if x8 is None else ctypes.byref(_Act8(*_x8_args(x8, name, T, D, dev)))


def block_norm_fwd(h, y=None, h_out=None, n=None, w_pre=None, w_post=None, gate=None, post_norm=None, rstd_pre=None,
                   rstd_post=None, y8=None, h8=None, n8=None, eps: float = 1e-6, gain_offset: float = 0.0,
                   res_scale: float = 1.0, stream=None):
    """h_out = h + res_scale gate norm(y) and n = norm(h_out) (see the header): the norm behind a block
    (`post_norm`, by default where w_post is given), its gate ([D], [T, 1] or [T, D]) and residual
    sum, and the norm before the next.  rstd_pre, rstd_post [T] are kept for the backward pass;
    y8, h8, n8 receive copies in 8 bits.  Without y the norm alone."""
    shape, rt = h.shape, h.dtype
    torch, _, f32, _, _, _ = _torch_names()
    (T, D), dev = shape, torch.cuda.current_device()
    dt = (y if y is not None else n if n is not None else w_pre if w_pre is not None else h).dtype
    b = _block(T, D, dt, rt, post_norm, w_post, w_pre, gate, gain_offset, res_scale, dev)
    st = lib().block_norm_fwd(ctypes.byref(b), _dev_arg(h, "h", rt, shape, dev), _dev_opt(y, "y", dt, shape, dev),
                              _dev_opt(h_out, "h_out", rt, shape, dev), _dev_opt(n, "n", dt, shape, dev),
                              _dev_opt(rstd_post, "rstd_post", f32, (T,), dev), _dev_opt(rstd_pre, "rstd_pre", f32, (T,), dev),
                              _act8(y8, "y8", T, D, dev), _act8(h8, "h8", T, D, dev), _act8(n8, "n8", T, D, dev), eps,
                              _stream_on(stream, dev))
    if st:
        _check(st, "block_norm_fwd")
    return h_out, n


def block_norm_workspace_bytes(T: int, D: int) -> int:
    n = lib().block_norm_workspace_bytes(T, D)
    if n == ctypes.c_size_t(-1).value:
        raise LoraError(LORA_EINVAL, "block_norm_workspace_bytes", lib().lora_last_error().decode())
    return int(n)


def block_norm_bwd(dn, dh_out, h, y=None, dh=None, dy=None, w_pre=None, w_post=None, gate=None, post_norm=None,
                   rstd_pre=None, rstd_post=None, dw_pre=None, dw_post=None, dgate=None, gain_offset: float = 0.0,
                   res_scale: float = 1.0, ws=None, stream=None):
    """Gradients of block_norm_fwd (see the header): dh of its h (may be dh_out) and, where given, dy,
    dw_pre, dw_post [D] fp32 and dgate.  h is the forward's h_out, y its y, each a
    tensor or a pair (codes, scale) in 8 bits."""
    shape, rt = dh.shape, dh.dtype
    torch, _, f32, _, _, _ = _torch_names()
    (T, D), dev = shape, torch.cuda.current_device()
    whole_h, whole_y = not isinstance(h, (tuple, list)), not isinstance(y, (tuple, list))
    dt = next((t for t in (dn, dy, w_pre, gate, w_post, y if whole_y else None) if t is not None), dh).dtype
    b = _block(T, D, dt, rt, post_norm, w_post, w_pre, gate, gain_offset, res_scale, dev)
    wp, wn = None, 0
    if ws is not None or dw_pre is not None or dw_post is not None or (dgate is not None and b.gate_mode == BLOCK_GATE_CHANNEL):
        wp, wn, ws = _ws_for(ws, lambda: block_norm_workspace_bytes(T, D), dh, stream)
    dgate_at = None
    if dgate is not None:
        if gate is None:
            raise ValueError("dgate needs a gate")
        dgate_at = _dev_arg(dgate, "dgate", dt if b.gate_mode == BLOCK_GATE_FULL else f32, gate.shape, dev)
    st = lib().block_norm_bwd(ctypes.byref(b), _dev_opt(dn, "dn", dt, shape, dev), _dev_opt(dh_out, "dh_out", rt, shape, dev),
                              _dev_opt(h, "h", rt, shape, dev) if whole_h else None, None if whole_h else _act8(h, "h", T, D, dev),
                              _dev_opt(y, "y", dt, shape, dev) if whole_y else None, None if whole_y else _act8(y, "y", T, D, dev),
                              _dev_opt(rstd_post, "rstd_post", f32, (T,), dev), _dev_opt(rstd_pre, "rstd_pre", f32, (T,), dev),
                              _dev_arg(dh, "dh", rt, shape, dev), _dev_opt(dy, "dy", dt, shape, dev),
                              _dev_opt(dw_pre, "dw_pre", f32, (D,), dev), _dev_opt(dw_post, "dw_post", f32, (D,), dev), dgate_at,
                              wp, wn, _stream_on(stream, dev))
    _check(st, "block_norm_bwd")
    return dh, dy


# --- kernel timing hook (benchmarks) -----------------------------------------------
def kernel_names() -> list:
    L = lib()
    return [L.lora_kernel_name(i).decode() for i in range(L.lora_kernel_count())]


def profiler_enable(on: bool = True):
    _check(lib().lora_profiler_enable(1 if on else 0), "lora_profiler_enable")


def profiler_reset():
    _check(lib().lora_profiler_reset(), "lora_profiler_reset")


def profiler_read(name: str):
    """(total milliseconds, launches) recorded for the kernel `name`."""
    idx = kernel_names().index(name)
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(lib().lora_profiler_read(idx, ctypes.byref(ms), ctypes.byref(n)), "lora_profiler_read")
    return ms.value, n.value


# --- plan and hand-over diagnostics -------------------------------------------------
def lora_linear_plan(T: int, d_in: int, d_out: int, r: int, dt: int = LORA_BF16) -> dict:
    """Kernel configuration of lora_linear_fwd / lora_linear_bwd for these sizes:
    GEMM output tiles, whether the rank-r pass is fused, number of partial sums."""
    p = _Plan()
    _check(lib().lora_linear_plan(T, d_in, d_out, r, dt, ctypes.byref(p)), "lora_linear_plan")
    return {n: getattr(p, n) for n, _ in _Plan._fields_}


def lora_few_token_plan(T: int, d_in: int, d_out: int, r: int, dt: int = LORA_BF16) -> dict:
    """Whether the few-token kernel takes the forward and the backward of these sizes,
    its tiles and parts, and the workspaces that it and the tiled kernels want."""
    p = _FewTokenPlan()
    _check(lib().lora_few_token_plan(T, d_in, d_out, r, dt, ctypes.byref(p)), "lora_few_token_plan")
    return {n: getattr(p, n) for n, _ in _FewTokenPlan._fields_}


def lora_linear_x8_plan(T: int, d_in: int, d_out: int, r: int, quantized: bool = False, want_dx: bool = True) -> dict:
    """How lora_linear_bwd_x8 (lora_linear_bwd_q_x8 where `quantized`) runs these sizes: the kernel that dx comes from,
    partial sums of du and u, ranges of tokens of dA and dB."""
    p = _X8Plan()
    _check(lib().lora_linear_x8_plan(T, d_in, d_out, r, int(quantized), int(want_dx), ctypes.byref(p)), "lora_linear_x8_plan")
    return {n: getattr(p, n) for n, _ in _X8Plan._fields_}


def handover_giveups(reset: bool = False) -> int:
    """Hand-over waits that gave up on the current device (synchronises it)."""
    n = ctypes.c_uint64(0)
    _check(lib().lora_handover_giveups(ctypes.byref(n), 1 if reset else 0), "lora_handover_giveups")
    return n.value


def debug_set_handover(hold: int = 0):
    """Test hook: 1 makes every tile's hand-over wait give up (results invalid)."""
    _check(lib().lora_debug_set_handover(hold), "lora_debug_set_handover")
