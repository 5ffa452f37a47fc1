"""ctypes binding of the norm and scoring operators (include/aj_score.h): checks of the tensors and argument marshalling.

Tensors are torch tensors on the handle's device (strides and extents are read from them); optional ones may be None.
"""
from __future__ import annotations

import ctypes
import struct

from . import binding
from .binding import AJ_BF16, AJ_ERR_INVALID_ARG, AJ_F32, AJ_OK, AjError

AJ_E4M3 = 2
AJ_SCORE_FLAG_FORCE_SIMT = 1
AJ_SCORE_MAX_TOP, AJ_SCORE_MAX_TOKENS = 32, 1024

EXPORTS = ("aj_add_norm", "aj_add_norm_call", "aj_score_create", "aj_score_destroy", "aj_score_tokens", "aj_score_call", "aj_score_last_status", "aj_score_last_launch_count",
           "aj_score_last_path")

_vp, _ci, _cf, _cl, _cu = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong, ctypes.c_uint
_ARGS = {
    "aj_add_norm": [_ci, _vp, _cl, _vp, _cl, _vp, _cf, _cl, _ci, _ci, _vp, _cl, _vp, _cl, _vp, _cl, _vp, _vp],
    "aj_add_norm_call": [ctypes.c_char_p],
    "aj_score_call": [_vp, ctypes.c_char_p],
    "aj_score_create": [ctypes.POINTER(_vp), _ci, _ci, _ci, _ci, _ci, _ci, _cu],
    "aj_score_destroy": [_vp],
    "aj_score_tokens": [_vp, _vp, _cl, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _cf, _vp, _vp, _vp, _vp, _vp, _vp],
    "aj_score_last_status": [_vp],
    "aj_score_last_launch_count": [_vp],
    "aj_score_last_path": [_vp],
}
# aj_norm_args and aj_score_args: eight bytes a field; a pointer that is not given is 0
_NORM_ARGS, _SCORE_ARGS = struct.Struct("6qd11q"), struct.Struct("9qd6q")
_fns = _types = _f32 = _i32 = _f8 = _add_norm = None


def _lib():
    global _fns, _types, _f32, _i32, _f8, _add_norm
    if _fns is None:
        import torch

        lib = binding.lib()
        fns = {}
        for name, args in _ARGS.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ctypes.c_char_p if name == "aj_score_last_path" else _ci
            fns[name] = fn
        _types = {torch.bfloat16: AJ_BF16, torch.float32: AJ_F32, torch.float8_e4m3fn: AJ_E4M3}
        _f32, _i32, _f8, _add_norm = torch.float32, torch.int32, torch.float8_e4m3fn, fns["aj_add_norm_call"]
        _fns = fns
    return _fns


def add_norm(x, weight, eps: float = 1e-5, out=None, residual=None, residual_out=None, out8=None, scale8=None, stream: int = 0,
             check: bool = True) -> int:
    """aj_add_norm: s = x + residual, out = s * rsqrt(mean(s^2) + eps) * weight, in the storage type and / or in 8 bits.

    x, residual, residual_out, out [rows, d] (rows may be strided) bf16 or f32, weight [d] f32, out8 [rows, d] float8_e4m3fn with
    scale8 [rows] f32: a row's values are out8 * scale8.  residual_out may be x or residual, out may be x or residual."""
    fn = _add_norm or _lib()["aj_add_norm_call"]
    st = AJ_ERR_INVALID_ARG
    dt, shape, dev = x.dtype, x.shape, x.get_device()
    if len(shape) == 2 and dt in _types and dev >= 0 and weight.dtype is _f32 and weight.numel() == shape[1] and weight.is_contiguous() and weight.get_device() == dev:
        xs = x.stride()
        thin = shape[1] == 1  # rows of one element: any stride along them
        ok = xs[1] == 1 or thin
        r = ro = o = o8 = s8 = rs = ros = os = o8s = 0
        if residual is not None:
            ok = ok and residual.dtype is dt and residual.shape == shape and residual.get_device() == dev
            if ok:
                r, (rs, e) = residual.data_ptr(), residual.stride()
                ok = e == 1 or thin
        if residual_out is not None:
            ok = ok and residual_out.dtype is dt and residual_out.shape == shape and residual_out.get_device() == dev
            if ok:
                ro, (ros, e) = residual_out.data_ptr(), residual_out.stride()
                ok = e == 1 or thin
        if out is not None:
            ok = ok and out.dtype is dt and out.shape == shape and out.get_device() == dev
            if ok:
                o, (os, e) = out.data_ptr(), out.stride()
                ok = e == 1 or thin
        if out8 is not None:
            ok = ok and out8.dtype is _f8 and out8.shape == shape and out8.get_device() == dev
            if ok:
                o8, (o8s, e) = out8.data_ptr(), out8.stride()
                ok = e == 1 or thin
        if scale8 is not None:
            s8 = scale8.data_ptr()
            ok = ok and scale8.dtype is _f32 and scale8.numel() == shape[0] and scale8.is_contiguous() and scale8.get_device() == dev
        if ok:
            st = fn(_NORM_ARGS.pack(dev, x.data_ptr(), xs[0], r, rs, weight.data_ptr(), eps, shape[0], shape[1], _types[dt], ro, ros, o, os, o8, o8s, s8, stream or 0))
    if check and st != AJ_OK:
        raise AjError(st, "aj_add_norm")
    return st


class ScoreHandle:
    """aj_score_create / aj_score_destroy as an object; score() mirrors aj_score_tokens.

    d, V: width and entries of the LM head; dtype: storage of the hidden states and the head (AJ_BF16, AJ_F32, AJ_E4M3)."""

    def __init__(self, device: int, max_rows: int, d: int, V: int, dtype: int = AJ_BF16, max_top: int = 20, flags: int = 0):
        import torch

        self._h = _vp()
        f = _lib()
        st = f["aj_score_create"](ctypes.byref(self._h), device, max_rows, d, V, dtype, max_top, flags)
        if st != AJ_OK:
            self._h = _vp()
            raise AjError(st, "aj_score_create")
        self._score, self._device, self._d, self._V = f["aj_score_call"], device, d, V
        self._dtype = {AJ_BF16: torch.bfloat16, AJ_F32: torch.float32, AJ_E4M3: torch.float8_e4m3fn}[dtype]

    def score(self, h, W, tokens=None, logprob=None, lse=None, entropy=None, top_id=None, top_logprob=None, inv_temperature: float = 1.0,
              h_scale=None, w_scale=None, stream: int = 0, check: bool = True) -> int:
        """aj_score_tokens: log probabilities of given tokens, entropy and the most likely entries of each row of h.

        h [rows, d] (rows may be strided), W [V, d]; tokens [rows, n_tok] int32 with logprob [rows, n_tok]; lse, entropy [rows];
        top_id [rows, n_top] int32 with top_logprob [rows, n_top]; h_scale [rows], w_scale [V] for AJ_E4M3."""
        st, dev, dt, i32, d, V = AJ_ERR_INVALID_ARG, self._device, self._dtype, _i32, self._d, self._V
        hshape = h.shape
        if len(hshape) == 2 and hshape[1] == d and h.dtype is dt and h.get_device() == dev and W.dtype is dt and W.is_contiguous() and W.get_device() == dev and W.shape == (V, d):
            rows, (hs, e) = hshape[0], h.stride()
            ok = e == 1 or d == 1
            n_tok = n_top = 0
            p_tok = p_lp = p_lse = p_ent = p_top = p_tlp = p_hs = p_ws = 0
            if tokens is not None:
                p_tok, n_tok = tokens.data_ptr(), tokens.numel() // rows if rows else 0
                ok = ok and tokens.dtype is i32 and tokens.is_contiguous() and tokens.get_device() == dev and tokens.shape[0] == rows and tokens.dim() == 2
            if logprob is not None:
                p_lp = logprob.data_ptr()
                ok = ok and tokens is not None and logprob.dtype is _f32 and logprob.is_contiguous() and logprob.get_device() == dev and logprob.shape == tokens.shape
            if lse is not None:
                p_lse = lse.data_ptr()
                ok = ok and lse.dtype is _f32 and lse.is_contiguous() and lse.get_device() == dev and lse.numel() == rows
            if entropy is not None:
                p_ent = entropy.data_ptr()
                ok = ok and entropy.dtype is _f32 and entropy.is_contiguous() and entropy.get_device() == dev and entropy.numel() == rows
            if top_id is not None:
                p_top, n_top = top_id.data_ptr(), top_id.numel() // rows if rows else 0
                ok = ok and top_id.dtype is i32 and top_id.is_contiguous() and top_id.get_device() == dev and top_id.shape[0] == rows and top_id.dim() == 2
            if top_logprob is not None:
                p_tlp = top_logprob.data_ptr()
                ok = (ok and top_id is not None and top_logprob.dtype is _f32 and top_logprob.is_contiguous() and top_logprob.get_device() == dev
                      and top_logprob.shape == top_id.shape)
            if h_scale is not None:
                p_hs = h_scale.data_ptr()
                ok = ok and h_scale.dtype is _f32 and h_scale.is_contiguous() and h_scale.get_device() == dev and h_scale.numel() == rows
            if w_scale is not None:
                p_ws = w_scale.data_ptr()
                ok = ok and w_scale.dtype is _f32 and w_scale.is_contiguous() and w_scale.get_device() == dev and w_scale.numel() == V
            if ok:
                st = self._score(self._h, _SCORE_ARGS.pack(h.data_ptr(), hs, p_hs, W.data_ptr(), p_ws, p_tok, n_tok, rows, n_top, inv_temperature, p_lp, p_lse,
                                                           p_ent, p_top, p_tlp, stream or 0))
        if check and st != AJ_OK:
            raise AjError(st, "aj_score_tokens")
        return st

    def last_status(self) -> int:
        return _lib()["aj_score_last_status"](self._h)

    def last_launch_count(self) -> int:
        return _lib()["aj_score_last_launch_count"](self._h)

    def last_path(self) -> str:
        return _lib()["aj_score_last_path"](self._h).decode()

    def destroy(self) -> None:
        if self._h:
            _lib()["aj_score_destroy"](self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
