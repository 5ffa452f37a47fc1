"""ctypes binding of the norm and scoring operators (include/aj_score.h): checks of the tensors and argument marshalling.

Tensors are torch tensors on the handle's device (strides and extents are read from them); optional ones may be None.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import AJ_BF16, AJ_ERR_INVALID_ARG, AJ_F32, AJ_OK, AjError

AJ_E4M3 = 2
AJ_SCORE_FLAG_FORCE_SIMT = 1
AJ_SCORE_MAX_TOP, AJ_SCORE_MAX_TOKENS = 32, 1024

EXPORTS = ("aj_add_norm", "aj_score_create", "aj_score_destroy", "aj_score_tokens", "aj_score_last_status", "aj_score_last_launch_count",
           "aj_score_last_path")

_vp, _ci, _cf, _cl, _cu = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong, ctypes.c_uint
_ARGS = {
    "aj_add_norm": [_ci, _vp, _cl, _vp, _cl, _vp, _cf, _cl, _ci, _ci, _vp, _cl, _vp, _cl, _vp, _cl, _vp, _vp],
    "aj_score_create": [ctypes.POINTER(_vp), _ci, _ci, _ci, _ci, _ci, _ci, _cu],
    "aj_score_destroy": [_vp],
    "aj_score_tokens": [_vp, _vp, _cl, _vp, _vp, _vp, _vp, _ci, _ci, _ci, _cf, _vp, _vp, _vp, _vp, _vp, _vp],
    "aj_score_last_status": [_vp],
    "aj_score_last_launch_count": [_vp],
    "aj_score_last_path": [_vp],
}
_fns = None
_types = None


def _lib():
    global _fns, _types
    if _fns is None:
        import torch

        lib = binding.lib()
        fns = {}
        for name, args in _ARGS.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ctypes.c_char_p if name == "aj_score_last_path" else _ci
            fns[name] = fn
        _types = {torch.bfloat16: AJ_BF16, torch.float32: AJ_F32, torch.float8_e4m3fn: AJ_E4M3}
        _fns = fns
    return _fns


def add_norm(x, weight, eps: float = 1e-5, out=None, residual=None, residual_out=None, out8=None, scale8=None, stream: int = 0,
             check: bool = True) -> int:
    """aj_add_norm: s = x + residual, out = s * rsqrt(mean(s^2) + eps) * weight, in the storage type and / or in 8 bits.

    x, residual, residual_out, out [rows, d] (rows may be strided) bf16 or f32, weight [d] f32, out8 [rows, d] float8_e4m3fn with
    scale8 [rows] f32: a row's values are out8 * scale8.  residual_out may be x or residual, out may be x or residual."""
    f = _fns or _lib()
    dt = x.dtype
    if x.dim() != 2:
        if check:
            raise AjError(AJ_ERR_INVALID_ARG, "aj_add_norm")
        return AJ_ERR_INVALID_ARG
    rows, d = shape = x.shape
    dev = x.get_device()
    xs = x.stride()
    ok = (dt in _types and dev >= 0 and (xs[1] == 1 or d == 1) and weight.numel() == d and weight.dtype.itemsize == 4 and weight.is_floating_point()
          and weight.is_contiguous() and weight.get_device() == dev)
    args = []
    for t, want in ((residual, dt), (residual_out, dt), (out, dt), (out8, None)):
        if t is None:
            args.append((None, 0))
            continue
        ts = t.stride()
        ok = (ok and t.shape == shape and (t.dtype is dt if want is not None else _types.get(t.dtype) == AJ_E4M3) and t.get_device() == dev
              and (ts[1] == 1 or d == 1))
        args.append((t.data_ptr(), ts[0]))
    if scale8 is not None:
        ok = ok and scale8.numel() == rows and _types.get(scale8.dtype) == AJ_F32 and scale8.is_contiguous() and scale8.get_device() == dev
    if not ok:
        st = AJ_ERR_INVALID_ARG
    else:
        (r, rs), (ro, ros), (o, os), (o8, o8s) = args
        st = f["aj_add_norm"](dev, x.data_ptr(), xs[0], r, rs, weight.data_ptr(), eps, rows, d, _types[dt], ro, ros, o, os, o8, o8s,
                              None if scale8 is None else scale8.data_ptr(), stream or None)
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
        self._score, self._device, self._d, self._V = f["aj_score_tokens"], device, d, V
        self._dtype = {AJ_BF16: torch.bfloat16, AJ_F32: torch.float32, AJ_E4M3: torch.float8_e4m3fn}[dtype]
        self._i32, self._f32 = torch.int32, torch.float32

    def score(self, h, W, tokens=None, logprob=None, lse=None, entropy=None, top_id=None, top_logprob=None, inv_temperature: float = 1.0,
              h_scale=None, w_scale=None, stream: int = 0, check: bool = True) -> int:
        """aj_score_tokens: log probabilities of given tokens, entropy and the most likely entries of each row of h.

        h [rows, d] (rows may be strided), W [V, d]; tokens [rows, n_tok] int32 with logprob [rows, n_tok]; lse, entropy [rows];
        top_id [rows, n_top] int32 with top_logprob [rows, n_top]; h_scale [rows], w_scale [V] for AJ_E4M3."""
        dev, f32, i32 = self._device, self._f32, self._i32
        hs = h.stride()
        rows = h.shape[0] if h.dim() == 2 else -1
        n_tok = tokens.shape[1] if tokens is not None and tokens.dim() == 2 else 0
        n_top = top_id.shape[1] if top_id is not None and top_id.dim() == 2 else 0

        def fits(t, dtype, *shape):
            return t is None or t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev

        if (rows < 0 or h.shape[1] != self._d or h.dtype is not self._dtype or h.get_device() != dev or hs[1] != 1 and self._d > 1
                or W is None or not fits(W, self._dtype, self._V, self._d) or not fits(tokens, i32, rows, n_tok) or not fits(logprob, f32, rows, n_tok)
                or not fits(lse, f32, rows) or not fits(entropy, f32, rows) or not fits(top_id, i32, rows, n_top)
                or not fits(top_logprob, f32, rows, n_top) or not fits(h_scale, f32, rows) or not fits(w_scale, f32, self._V)):
            st = AJ_ERR_INVALID_ARG
        else:
            p = [None if t is None else t.data_ptr() for t in (h_scale, w_scale, tokens, logprob, lse, entropy, top_id, top_logprob)]
            st = self._score(self._h, h.data_ptr(), hs[0], p[0], W.data_ptr(), p[1], p[2], n_tok, rows, n_top, inv_temperature, p[3], p[4], p[5],
                             p[6], p[7], stream or None)
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
