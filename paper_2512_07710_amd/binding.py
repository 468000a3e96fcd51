"""ctypes binding of libmoe355.so: argument marshalling only.

Every function here has the name of the C entry point it calls (see
include/moe355.h); tensors are torch CUDA tensors used purely as device
memory.  There is no CPU fallback: if the shared library is missing or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe355.so")
_lib: Optional[ctypes.CDLL] = None

EXPORTS = ("moe_create", "moe_destroy", "moe_strerror", "moe_route", "moe_route_replay", "moe_route_replay_noalloc",
           "moe_route_replay_ids", "moe_route_quantize", "moe_route_replay_quantize",
           "moe_check_ids", "moe_quantize_fp8", "moe_quantize_weights_fp8", "moe_linear_fp8", "moe_expert_ffn_fp8",
           "moe_expert_ffn_fp8_gather", "moe_combine", "moe_balance_lengths", "moe_debug_copy_hidden",
           "moe_reserve_gradients", "moe_add_rmsnorm", "moe_add_rmsnorm_backward", "moe_dispatch", "moe_dispatch_backward",
           "moe_combine_backward", "moe_policy_loss", "moe_linear_fp8_dgrad", "moe_linear_fp8_wgrad",
           "moe_embed", "moe_embed_backward", "moe_token_logp", "moe_token_logp_backward", "moe_grad_norm", "moe_clip_grads",
           "moe_probe_copy", "moe_probe_fp8_mfma", "moe_profile_enable", "moe_profile_read", "moe_version")


class MoEError(RuntimeError):
    pass


_shapes = {}                       # (T, d, E, k) of the contexts made here, for the checks of the calls that go by them


class _Dims(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("E", ctypes.c_int32),
                ("k", ctypes.c_int32), ("F", ctypes.c_int32)]


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libmoe355.so (built by paper_2512_07710_amd.build); raises if it is not there."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise MoEError(f"{p} not found: build it with `python -m paper_2512_07710_amd.build` "
                       "(there is no fallback implementation)")
    lib = ctypes.CDLL(p)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.moe_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_Dims), vp]
    lib.moe_destroy.argtypes = [vp]
    lib.moe_strerror.argtypes = [ctypes.c_int]
    lib.moe_strerror.restype = ctypes.c_char_p
    lib.moe_version.restype = ctypes.c_char_p
    lib.moe_route.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.moe_route_replay.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.moe_route_quantize.argtypes = [vp, vp, vp, vp, i32] + [vp] * 7
    lib.moe_route_replay_quantize.argtypes = [vp] * 11
    lib.moe_route_replay_ids.argtypes = [vp] * 9
    lib.moe_route_replay_noalloc.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.moe_check_ids.argtypes = [vp]
    lib.moe_quantize_weights_fp8.argtypes = [vp, vp, i64, i32, vp, vp]
    lib.moe_linear_fp8.argtypes = [vp, vp, vp, i32, i32, vp, vp, i32, vp]
    lib.moe_quantize_fp8.argtypes = [vp, vp, i64, i32, i32, vp, i32, vp, vp]
    lib.moe_expert_ffn_fp8.argtypes = [vp] * 11
    lib.moe_expert_ffn_fp8_gather.argtypes = [vp] * 12
    lib.moe_combine.argtypes = [vp] * 6
    lib.moe_balance_lengths.argtypes = [vp, i64, i32, i32, vp, vp, vp, vp]
    lib.moe_debug_copy_hidden.argtypes = [vp, vp, vp]
    f32 = ctypes.c_float
    lib.moe_reserve_gradients.argtypes = [vp]
    lib.moe_add_rmsnorm.argtypes = [vp, vp, vp, vp, i64, i32, i64, i64, i32, f32] + [vp] * 5
    lib.moe_add_rmsnorm_backward.argtypes = [vp] * 6 + [i64, i32, i32, vp, vp]
    lib.moe_dispatch.argtypes = [vp, vp, vp, i32, vp]
    lib.moe_dispatch_backward.argtypes = [vp, vp, vp, vp, i32, vp]
    lib.moe_combine_backward.argtypes = [vp] * 6 + [i32, vp, vp, vp]
    lib.moe_policy_loss.argtypes = [vp, vp, i64, i32, i64, i32] + [vp] * 6 + [f32] * 5 + [vp] * 5 + [i64, i32]
    lib.moe_linear_fp8_dgrad.argtypes = [vp, vp, i64, i32, vp, vp, i32, vp, i32, vp]
    lib.moe_linear_fp8_wgrad.argtypes = [vp, vp, i64, i32, vp, vp, i32, vp, i32, i32, i32, vp]
    lib.moe_embed.argtypes = [vp, vp, i64, vp, i32, i32, i64, i32, f32, vp, i64, i32]
    lib.moe_embed_backward.argtypes = [vp, vp, vp, i64, i32, i32, i64, i32, f32, i32, vp, i64, i32]
    lib.moe_token_logp.argtypes = [vp, vp, i64, i32, i64, i32, vp, i32, f32, vp, vp, i32, vp, vp, vp]
    lib.moe_token_logp_backward.argtypes = [vp, vp, i64, i32, i64, i32, vp, i32, f32, vp, vp, vp, vp, vp, i64, i32]
    lib.moe_grad_norm.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.moe_clip_grads.argtypes = [vp, vp, vp, vp, i32, vp, f32, vp]
    lib.moe_probe_copy.argtypes = [vp, vp, vp, i64]
    lib.moe_probe_fp8_mfma.argtypes = [vp, i32, i32, i32, vp]
    lib.moe_profile_enable.argtypes = [vp, i32]
    lib.moe_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    for name in EXPORTS:
        if name not in ("moe_strerror", "moe_version"):
            getattr(lib, name).restype = ctypes.c_int
    if path is None:
        _lib = lib
    return lib


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise MoEError(f"{what} failed: {load_library().moe_strerror(rc).decode()} ({rc})")


def _ptr(t: Optional[torch.Tensor], dtype=None) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise MoEError("expected a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise MoEError(f"expected dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def moe_create(T: int, d: int, E: int, k: int, F: int, stream: Optional[torch.cuda.Stream] = None) -> int:
    """Returns an opaque context handle bound to `stream` (default: torch's current stream)."""
    lib = load_library()
    s = stream if stream is not None else torch.cuda.current_stream()
    dims = _Dims(T, d, E, k, F)
    h = ctypes.c_void_p()
    _check(lib.moe_create(ctypes.byref(h), ctypes.byref(dims), ctypes.c_void_p(s.cuda_stream)), "moe_create")
    _shapes[h.value] = (T, d, E, k)
    return h.value


def moe_destroy(ctx: int) -> None:
    _shapes.pop(ctx, None)
    _check(load_library().moe_destroy(ctx), "moe_destroy")


def moe_version() -> str:
    return load_library().moe_version().decode()


def moe_route(ctx, x, W_router, sel_bias, k, topk_idx, topk_w, offsets, perm, inv_perm) -> None:
    _check(load_library().moe_route(ctx, _ptr(x, torch.bfloat16), _ptr(W_router, torch.float32),
                                    _ptr(sel_bias, torch.float32), k, _ptr(topk_idx, torch.int32),
                                    _ptr(topk_w, torch.float32), _ptr(offsets, torch.int32),
                                    _ptr(perm, torch.int32), _ptr(inv_perm, torch.int32)), "moe_route")


def moe_route_replay(ctx, x, logged_idx, logged_w, topk_idx, topk_w, offsets, perm, inv_perm) -> None:
    _check(load_library().moe_route_replay(ctx, _ptr(x), _ptr(logged_idx, torch.int32),
                                           _ptr(logged_w, torch.float32), _ptr(topk_idx, torch.int32),
                                           _ptr(topk_w, torch.float32), _ptr(offsets, torch.int32),
                                           _ptr(perm, torch.int32), _ptr(inv_perm, torch.int32)),
           "moe_route_replay")


def moe_route_quantize(ctx, x, W_router, sel_bias, k, topk_idx, topk_w, offsets, perm, inv_perm, xq_tok, xs_tok) -> None:
    i32, f32 = torch.int32, torch.float32
    _check(load_library().moe_route_quantize(ctx, _ptr(x, torch.bfloat16), _ptr(W_router, f32), _ptr(sel_bias, f32), k,
                                             _ptr(topk_idx, i32), _ptr(topk_w, f32), _ptr(offsets, i32), _ptr(perm, i32),
                                             _ptr(inv_perm, i32), _ptr(xq_tok, torch.uint8), _ptr(xs_tok, f32)),
           "moe_route_quantize")


def moe_route_replay_quantize(ctx, x, logged_idx, logged_w, topk_idx, topk_w, offsets, perm, inv_perm, xq_tok, xs_tok) -> None:
    i32, f32 = torch.int32, torch.float32
    _check(load_library().moe_route_replay_quantize(ctx, _ptr(x, torch.bfloat16), _ptr(logged_idx, i32), _ptr(logged_w, f32),
                                                    _ptr(topk_idx, i32), _ptr(topk_w, f32), _ptr(offsets, i32),
                                                    _ptr(perm, i32), _ptr(inv_perm, i32), _ptr(xq_tok, torch.uint8),
                                                    _ptr(xs_tok, f32)), "moe_route_replay_quantize")


def moe_route_replay_noalloc(stream, T, E, k, logged_idx, logged_w, topk_idx, topk_w, offsets, perm, inv_perm,
                             id_flags=None) -> None:
    """`stream`: a torch.cuda.Stream or None for torch's current stream."""
    s = stream if stream is not None else torch.cuda.current_stream()
    i32 = torch.int32
    _check(load_library().moe_route_replay_noalloc(ctypes.c_void_p(s.cuda_stream), T, E, k, _ptr(logged_idx, i32),
                                                   _ptr(logged_w, torch.float32), _ptr(topk_idx, i32),
                                                   _ptr(topk_w, torch.float32), _ptr(offsets, i32), _ptr(perm, i32),
                                                   _ptr(inv_perm, i32), _ptr(id_flags, i32)),
           "moe_route_replay_noalloc")


def moe_check_ids(ctx) -> int:
    """Returns the raw status (0 or MOE_EBADIDS) after synchronising the context's stream."""
    return load_library().moe_check_ids(ctx)


def moe_route_replay_ids(ctx, x, W_router, logged_idx, topk_idx, topk_w, offsets, perm, inv_perm) -> None:
    i32 = torch.int32
    _check(load_library().moe_route_replay_ids(ctx, _ptr(x, torch.bfloat16), _ptr(W_router, torch.float32),
                                               _ptr(logged_idx, i32), _ptr(topk_idx, i32),
                                               _ptr(topk_w, torch.float32), _ptr(offsets, i32), _ptr(perm, i32),
                                               _ptr(inv_perm, i32)), "moe_route_replay_ids")


def moe_quantize_weights_fp8(ctx, w, rows, cols, q, scales) -> None:
    _check(load_library().moe_quantize_weights_fp8(ctx, _ptr(w, torch.bfloat16), rows, cols, _ptr(q, torch.uint8),
                                                   _ptr(scales, torch.float32)), "moe_quantize_weights_fp8")


def moe_linear_fp8(ctx, xq, xs, rows, K, Wq, ws, NOUT, y) -> None:
    u8, f32 = torch.uint8, torch.float32
    _check(load_library().moe_linear_fp8(ctx, _ptr(xq, u8), _ptr(xs, f32), rows, K, _ptr(Wq, u8), _ptr(ws, f32),
                                         NOUT, _ptr(y, f32)), "moe_linear_fp8")


def moe_quantize_fp8(ctx, x, rows_in, cols, block, dst_rows, fanout, q, scales) -> None:
    _check(load_library().moe_quantize_fp8(ctx, _ptr(x, torch.bfloat16), rows_in, cols, block,
                                           _ptr(dst_rows, torch.int32), fanout, _ptr(q, torch.uint8),
                                           _ptr(scales, torch.float32)), "moe_quantize_fp8")


def moe_expert_ffn_fp8(ctx, xq_perm, xs_perm, offsets, W1, W3, W2, s1, s3, s2, y_perm) -> None:
    u8, f32 = torch.uint8, torch.float32
    _check(load_library().moe_expert_ffn_fp8(ctx, _ptr(xq_perm, u8), _ptr(xs_perm, f32),
                                             _ptr(offsets, torch.int32), _ptr(W1, u8), _ptr(W3, u8),
                                             _ptr(W2, u8), _ptr(s1, f32), _ptr(s3, f32), _ptr(s2, f32),
                                             _ptr(y_perm, f32)), "moe_expert_ffn_fp8")


def moe_expert_ffn_fp8_gather(ctx, xq_tok, xs_tok, perm, offsets, W1, W3, W2, s1, s3, s2, y_perm) -> None:
    u8, f32 = torch.uint8, torch.float32
    _check(load_library().moe_expert_ffn_fp8_gather(ctx, _ptr(xq_tok, u8), _ptr(xs_tok, f32),
                                                    _ptr(perm, torch.int32),
                                                    _ptr(offsets, torch.int32), _ptr(W1, u8), _ptr(W3, u8),
                                                    _ptr(W2, u8), _ptr(s1, f32), _ptr(s3, f32), _ptr(s2, f32),
                                                    _ptr(y_perm, f32)), "moe_expert_ffn_fp8_gather")


def moe_combine(ctx, y_perm, inv_perm, topk_w, y, y_f32=None) -> None:
    _check(load_library().moe_combine(ctx, _ptr(y_perm, torch.float32), _ptr(inv_perm, torch.int32),
                                      _ptr(topk_w, torch.float32), _ptr(y, torch.bfloat16),
                                      _ptr(y_f32, torch.float32)), "moe_combine")


# ---- the training side: sizes are taken from the tensors, and every tensor's type and shape is checked.  Short calls are bound by the
# time on the host, and half of that is spent here: types as names of the module, shapes as ready tuples, no helper around the call
_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_TYPES = {_BF16: 0, _F32: 1}


def _type(t: torch.Tensor) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise MoEError(f"expected bfloat16 or float32, got {t.dtype}")
    return code


def _of(t: Optional[torch.Tensor], dtype, shape: tuple) -> Optional[int]:
    """Address of a contiguous tensor of this type and shape; None for None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous() or not t.is_cuda:
        raise MoEError(f"expected a contiguous CUDA tensor {shape} of {dtype}, got {tuple(t.shape)} of {t.dtype}, strides {t.stride()}, on {t.device}")
    return t.data_ptr()


def _flat(t: torch.Tensor, n: int) -> int:
    """Address of a contiguous int32 tensor of n elements, of any shape."""
    if t.numel() != n or t.dtype is not _I32 or not t.is_contiguous() or not t.is_cuda:
        raise MoEError(f"expected a contiguous CUDA tensor of {n} elements of {_I32}, got {tuple(t.shape)} of {t.dtype}, strides {t.stride()}, on {t.device}")
    return t.data_ptr()


def _rows_of(t: Optional[torch.Tensor], dtype, shape: tuple):
    """(address, row stride) of a 2-D tensor of this type and shape whose rows are contiguous."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda or (t.stride(1) != 1 and shape[1] > 1):
        raise MoEError(f"expected a CUDA tensor {shape} of {dtype} with contiguous rows, got {tuple(t.shape)} of {t.dtype}, "
                       f"strides {t.stride()}, on {t.device}")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else max(shape[1], 1)


def _two(t: torch.Tensor) -> tuple:
    shape = t.shape
    if len(shape) != 2:
        raise MoEError("expected a 2-D tensor")
    return shape


def moe_reserve_gradients(ctx) -> None:
    """Allocates what the gradient calls need beside their arguments (64 MiB, once per context)."""
    _check(load_library().moe_reserve_gradients(ctx), "moe_reserve_gradients")


def moe_add_rmsnorm(ctx, x, residual, gain, eps, sum=None, y=None, q=None, scales=None, rstd=None) -> None:
    """x, residual [rows, cols] (bf16 or f32, rows may be strided); every output given is written."""
    lib = _lib or load_library()
    shape = rows, cols = _two(x)
    code, t = _type(x), x.dtype
    px, ld_x = _rows_of(x, t, shape)
    pr, ld_r = _rows_of(residual, t, shape)
    rc = lib.moe_add_rmsnorm(ctx, px, pr, _of(gain, _F32, (cols,)), rows, cols, ld_x, ld_r, code, eps, _of(sum, t, shape), _of(y, t, shape),
                             _of(q, _U8, shape), _of(scales, _F32, (cols // 128, rows)), _of(rstd, _F32, (rows,)))
    if rc:
        _check(rc, "moe_add_rmsnorm")


def moe_add_rmsnorm_backward(ctx, dy, h, rstd, gain, dh, dx, dgain) -> None:
    lib = _lib or load_library()
    shape = rows, cols = _two(dy)
    code, t = _type(dy), dy.dtype
    rc = lib.moe_add_rmsnorm_backward(ctx, _of(dy, t, shape), _of(h, t, shape), _of(rstd, _F32, (rows,)), _of(gain, _F32, (cols,)),
                                      _of(dh, t, shape), rows, cols, code, _of(dx, t, shape), _of(dgain, _F32, (cols,)))
    if rc:
        _check(rc, "moe_add_rmsnorm_backward")


def _shape_of(ctx):
    shape = _shapes.get(ctx)
    if shape is None:
        raise MoEError("not a context")
    return shape


def moe_dispatch(ctx, x, inv_perm, x_perm) -> None:
    lib = _lib or load_library()
    T, d, _, k = _shape_of(ctx)
    code, t = _type(x), x.dtype
    rc = lib.moe_dispatch(ctx, _of(x, t, (T, d)), _flat(inv_perm, T * k), code, _of(x_perm, t, (T * k, d)))
    if rc:
        _check(rc, "moe_dispatch")


def moe_dispatch_backward(ctx, dx_perm, inv_perm, dx_add, dx) -> None:
    lib = _lib or load_library()
    T, d, _, k = _shape_of(ctx)
    code, t = _type(dx_perm), dx_perm.dtype
    rc = lib.moe_dispatch_backward(ctx, _of(dx_perm, t, (T * k, d)), _flat(inv_perm, T * k), _of(dx_add, t, (T, d)), code, _of(dx, t, (T, d)))
    if rc:
        _check(rc, "moe_dispatch_backward")


def moe_combine_backward(ctx, dy, y_perm, inv_perm, topk_w, topk_idx, dy_perm, dw, dlogits) -> None:
    """topk_idx and dlogits: both given or both None."""
    lib = _lib or load_library()
    T, d, E, k = _shape_of(ctx)
    code, t, rows, slots = _type(dy), dy.dtype, (T * k, d), (T, k)
    rc = lib.moe_combine_backward(ctx, _of(dy, t, (T, d)), _of(y_perm, _F32, rows), _flat(inv_perm, T * k), _of(topk_w, _F32, slots),
                                  _of(topk_idx, _I32, slots), code, _of(dy_perm, t, rows), _of(dw, _F32, slots), _of(dlogits, _F32, (T, E)))
    if rc:
        _check(rc, "moe_combine_backward")


def moe_policy_loss(ctx, logits, target, old_logp, ref_logp, advantage, weight, logp, entropy, row_loss, loss, dlogits=None, *,
                    clip_rows=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, temperature=1.0) -> None:
    """logits [rows, V] (bf16 or f32, rows may be strided); dlogits None: forward only; it may be logits itself."""
    lib = _lib or load_library()
    shape = rows, V = _two(logits)
    row = (rows,)
    code = gcode = _type(logits)
    pz, ld = _rows_of(logits, logits.dtype, shape)
    pg, ld_g = None, 0
    if dlogits is not None:
        gcode = _type(dlogits)
        pg, ld_g = _rows_of(dlogits, dlogits.dtype, shape)
    rc = lib.moe_policy_loss(ctx, pz, ld, code, rows, V, _of(target, _I32, row), _of(old_logp, _F32, row), _of(ref_logp, _F32, row),
                             _of(advantage, _F32, row), _of(weight, _F32, row), _of(clip_rows, _F32, row), clip_low, clip_high, kl_coef,
                             entropy_coef, temperature, _of(logp, _F32, row), _of(entropy, _F32, row), _of(row_loss, _F32, row),
                             _of(loss, _F32, (1,)), pg, ld_g, gcode)
    if rc:
        _check(rc, "moe_policy_loss")


def _experts(offsets, matrices: torch.Tensor):
    """(E, NOUT, K, shape prefix) of a linear's matrices: dense without offsets, one per expert with them."""
    shape = matrices.shape
    if offsets is None:
        if len(shape) != 2:
            raise MoEError("a dense linear has one matrix")
        return 1, shape[0], shape[1], ()
    if len(shape) != 3:
        raise MoEError("a grouped linear has a matrix per expert")
    return shape[0], shape[1], shape[2], (shape[0],)


def moe_linear_fp8_dgrad(ctx, dy, Wq, ws, offsets, dx) -> None:
    """dy [rows, NOUT] bf16; Wq [NOUT, K] (offsets None) or [E, NOUT, K]; dx [rows, K] bf16."""
    lib = _lib or load_library()
    E, NOUT, K, pre = _experts(offsets, Wq)
    rows = dy.shape[0]
    rc = lib.moe_linear_fp8_dgrad(ctx, _of(dy, _BF16, (rows, NOUT)), rows, NOUT, _of(Wq, _U8, pre + (NOUT, K)),
                                  _of(ws, _F32, pre + (NOUT // 128, K // 128)), K, _of(offsets, _I32, (E + 1,)), E, _of(dx, _BF16, (rows, K)))
    if rc:
        _check(rc, "moe_linear_fp8_dgrad")


def moe_linear_fp8_wgrad(ctx, dy, xq, xs, offsets, dW, accumulate=False) -> None:
    """dy [rows, NOUT] bf16; xq [rows, K] u8 and xs [K/128, rows] as the forward pass read them; dW [NOUT, K] or [E, NOUT, K], bf16 or f32."""
    lib = _lib or load_library()
    E, NOUT, K, pre = _experts(offsets, dW)
    rows = dy.shape[0]
    rc = lib.moe_linear_fp8_wgrad(ctx, _of(dy, _BF16, (rows, NOUT)), rows, NOUT, _of(xq, _U8, (rows, K)), _of(xs, _F32, (K // 128, rows)), K,
                                  _of(offsets, _I32, (E + 1,)), E, 1 if accumulate else 0, _type(dW), _of(dW, dW.dtype, pre + (NOUT, K)))
    if rc:
        _check(rc, "moe_linear_fp8_wgrad")


# ---- the two ends of a policy step
def moe_embed(ctx, ids, table, scale, y) -> None:
    """ids int32 of any shape, T in all; table [V, d]; y [T, d] (bf16 or f32 each, rows may be strided)."""
    lib = _lib or load_library()
    V, d = _two(table)
    T = ids.numel()
    code, out = _type(table), _type(y)
    pt, ld = _rows_of(table, table.dtype, (V, d))
    py, ld_y = _rows_of(y, y.dtype, (T, d))
    rc = lib.moe_embed(ctx, _flat(ids, T), T, pt, V, d, ld, code, scale, py, ld_y, out)
    if rc:
        _check(rc, "moe_embed")


def moe_embed_backward(ctx, dy, ids, scale, dtable, accumulate=False) -> None:
    """dy [T, d]; ids int32 of any shape, T in all; dtable [V, d] (bf16 or f32 each, rows may be strided)."""
    lib = _lib or load_library()
    V, d = _two(dtable)
    T = ids.numel()
    code, out = _type(dy), _type(dtable)
    py, ld = _rows_of(dy, dy.dtype, (T, d))
    pg, ld_g = _rows_of(dtable, dtable.dtype, (V, d))
    rc = lib.moe_embed_backward(ctx, py, _flat(ids, T), T, V, d, ld, code, scale, 1 if accumulate else 0, pg, ld_g, out)
    if rc:
        _check(rc, "moe_embed_backward")


def _given(ids: Optional[torch.Tensor], rows: int):
    """(m, shape) of the given tokens: [rows], [rows, m] or None."""
    if ids is None:
        return 0, (rows, 0)
    shape = ids.shape
    return (1 if len(shape) == 1 else shape[1] if len(shape) == 2 else -1), shape


def moe_token_logp(ctx, logits, ids, logp, entropy=None, top_idx=None, top_logp=None, stats=None, *, temperature=1.0) -> None:
    """logits [rows, V] (bf16 or f32, rows may be strided); ids, logp [rows] or [rows, m], or None; top_idx, top_logp [rows, n], or None; every output
    given is written."""
    lib = _lib or load_library()
    shape = rows, V = _two(logits)
    code = _type(logits)
    pz, ld = _rows_of(logits, logits.dtype, shape)
    m, given = _given(ids, rows)
    n = 0 if top_idx is None else _two(top_idx)[1]
    rc = lib.moe_token_logp(ctx, pz, ld, code, rows, V, _of(ids, _I32, (rows, *given[1:])), m, temperature, _of(logp, _F32, given),
                            _of(entropy, _F32, (rows,)), n, _of(top_idx, _I32, (rows, n)), _of(top_logp, _F32, (rows, n)), _of(stats, _F32, (rows, 2)))
    if rc:
        _check(rc, "moe_token_logp")


def moe_token_logp_backward(ctx, logits, ids, dlogp, dentropy, stats, entropy, dlogits, *, temperature=1.0) -> None:
    """ids, dlogp [rows] or [rows, m], or None; dentropy None: entropy is not read; dlogits [rows, V] may be logits itself."""
    lib = _lib or load_library()
    shape = rows, V = _two(logits)
    code, gcode = _type(logits), _type(dlogits)
    pz, ld = _rows_of(logits, logits.dtype, shape)
    pg, ld_g = _rows_of(dlogits, dlogits.dtype, shape)
    m, given = _given(ids, rows)
    row = (rows,)
    rc = lib.moe_token_logp_backward(ctx, pz, ld, code, rows, V, _of(ids, _I32, (rows, *given[1:])), m, temperature, _of(dlogp, _F32, given),
                                     _of(dentropy, _F32, row), _of(stats, _F32, (rows, 2)), _of(entropy, _F32, row), pg, ld_g, gcode)
    if rc:
        _check(rc, "moe_token_logp_backward")


class GradList:
    """Gradients (bf16 or f32, contiguous, apart from each other) as the list that moe_grad_norm and moe_clip_grads take: their addresses, counts and types,
    read once, which takes about a microsecond a tensor.  It keeps the tensors; one that is given other memory later (set_, resize_) needs a new list."""

    def __init__(self, tensors):
        self.tensors = tensors = list(tensors)
        self.n = n = len(tensors)
        for t in tensors:
            if not t.is_cuda or not t.is_contiguous():
                raise MoEError(f"expected contiguous CUDA tensors, got {tuple(t.shape)} of {t.dtype}, strides {t.stride()}, on {t.device}")
            if t.device != tensors[0].device:
                raise MoEError("expected tensors on one device")
        self.shapes = [(t.dtype, t.numel()) for t in tensors]
        ends = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors if t.numel())
        if any(a[1] > b[0] for a, b in zip(ends, ends[1:])):
            raise MoEError("two of the tensors share memory")
        self.addresses = (ctypes.c_void_p * n)(*[t.data_ptr() for t in tensors])
        self.counts = (ctypes.c_int64 * n)(*[t.numel() for t in tensors])
        self.types = (ctypes.c_int32 * n)(*[_type(t) for t in tensors])


def _list(grads) -> GradList:
    return grads if isinstance(grads, GradList) else GradList(grads)


def moe_grad_norm(ctx, grads, sum_sq, norm=None) -> None:
    """grads: a GradList, or tensors to make one of; sum_sq [1] f64, norm [1] f32."""
    lib = _lib or load_library()
    g = _list(grads)
    rc = lib.moe_grad_norm(ctx, g.addresses, g.counts, g.types, g.n, _of(sum_sq, torch.float64, (1,)), _of(norm, _F32, (1,)))
    if rc:
        _check(rc, "moe_grad_norm")


def moe_clip_grads(ctx, grads, sum_sq, max_norm, outs=None) -> None:
    """grads, outs: GradLists, or tensors to make them of, of the same types and sizes; outs None: in place.  An output has its gradient's place or memory of
    its own."""
    lib = _lib or load_library()
    g = _list(grads)
    o = None if outs is None else _list(outs)
    if o is not None and o is not g and o.shapes != g.shapes:
        raise MoEError("outs must have the types and sizes of grads")
    rc = lib.moe_clip_grads(ctx, g.addresses, g.counts, g.types, g.n, _of(sum_sq, torch.float64, (1,)), max_norm, None if o is None else o.addresses)
    if rc:
        _check(rc, "moe_clip_grads")


def moe_balance_lengths(pred_len, n_groups: int, equal_count: bool = True):
    """Host-side length-based load balancing: pred_len is a CPU int64 tensor [n]; returns CPU tensors
    (group_of int32 [n], order int64 [n], bounds int64 [n_groups+1], totals int64 [n_groups])."""
    if pred_len.is_cuda or pred_len.dtype != torch.int64 or not pred_len.is_contiguous() or pred_len.dim() != 1:
        raise MoEError("expected a contiguous 1-D CPU int64 tensor")
    if n_groups < 1:
        raise MoEError("n_groups must be at least 1")
    n = pred_len.numel()
    group_of = torch.empty(n, dtype=torch.int32)
    order = torch.empty(n, dtype=torch.int64)
    bounds = torch.empty(n_groups + 1, dtype=torch.int64)
    totals = torch.empty(n_groups, dtype=torch.int64)
    _check(load_library().moe_balance_lengths(pred_len.data_ptr(), n, n_groups, 1 if equal_count else 0,
                                              group_of.data_ptr(), order.data_ptr(), bounds.data_ptr(),
                                              totals.data_ptr()), "moe_balance_lengths")
    return group_of, order, bounds, totals


def moe_debug_copy_hidden(ctx, hq_out, hs_out) -> None:
    _check(load_library().moe_debug_copy_hidden(ctx, _ptr(hq_out, torch.uint8), _ptr(hs_out, torch.float32)),
           "moe_debug_copy_hidden")


def moe_probe_copy(ctx, src, dst, nbytes: int) -> None:
    _check(load_library().moe_probe_copy(ctx, _ptr(src), _ptr(dst), nbytes), "moe_probe_copy")


def moe_probe_fp8_mfma(ctx, blocks: int, steps: int, scaled: bool, sink) -> None:
    _check(load_library().moe_probe_fp8_mfma(ctx, blocks, steps, 1 if scaled else 0, _ptr(sink, torch.float32)),
           "moe_probe_fp8_mfma")


def moe_profile_enable(ctx, on: bool) -> None:
    _check(load_library().moe_profile_enable(ctx, 1 if on else 0), "moe_profile_enable")


def moe_profile_read(ctx):
    """(mean ms of the gate/up GEMM, mean ms of the down GEMM, recorded calls); synchronises."""
    ms = (ctypes.c_float * 2)()
    n = ctypes.c_int32()
    _check(load_library().moe_profile_read(ctx, ms, ctypes.byref(n)), "moe_profile_read")
    return float(ms[0]), float(ms[1]), int(n.value)
