"""ctypes binding of the key-value cache operators (include/aj_kv.h): argument marshalling only.

Tensors are torch tensors on the handle's device (strides and extents are read from them); optional ones may be None.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import AJ_BF16, AJ_ERR_INVALID_ARG, AJ_OK, AjError

AJ_KV_FLAG_FORCE_SIMT = 1

EXPORTS = ("aj_kv_create", "aj_kv_destroy", "aj_kv_append", "aj_kv_attend", "aj_kv_weigh", "aj_kv_evict", "aj_kv_last_status",
           "aj_kv_last_launch_count", "aj_kv_last_path")

_vp, _ci, _cf, _cl, _cu = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong, ctypes.c_uint
_ARGS = {
    "aj_kv_create": [ctypes.POINTER(_vp), _ci, _ci, _ci, _ci, _ci, _ci, _ci, _ci, _cu],
    "aj_kv_destroy": [_vp],
    "aj_kv_append": [_vp, _vp, _cl, _vp, _cl, _vp, _cl, _vp, _vp, _cf, _vp, _ci, _ci, _ci, _vp, _vp, _vp, _ci, _vp, _ci, _vp, _vp, _ci,
                     _ci, _vp, _cl, _vp, _vp, _vp],
    "aj_kv_attend": [_vp, _vp, _cl, _vp, _vp, _ci, _vp, _ci, _vp, _vp, _ci, _ci, _cf, _ci, _ci, _vp, _cl, _vp, _vp],
    "aj_kv_weigh": [_vp, _vp, _cl, _vp, _vp, _ci, _vp, _ci, _vp, _vp, _vp, _ci, _ci, _cf, _ci, _ci, _vp, _vp, _vp],
    "aj_kv_evict": [_vp, _vp, _vp, _ci, _vp, _ci, _vp, _ci, _ci, _ci, _ci, _vp, _vp, _vp, _vp, _vp, _vp],
    "aj_kv_last_status": [_vp],
    "aj_kv_last_launch_count": [_vp],
    "aj_kv_last_path": [_vp],
}
_fns = None


def _lib():
    global _fns
    if _fns is None:
        lib = binding.lib()
        fns = {}
        for name, args in _ARGS.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, ctypes.c_char_p if name == "aj_kv_last_path" else _ci
            fns[name] = fn
        _fns = fns
    return _fns


def _p(t):
    return None if t is None else t.data_ptr()


class KvHandle:
    """aj_kv_create / aj_kv_destroy as an object; the methods mirror the C entry points.

    The cache's tensors are passed with each call: k_pages, v_pages [n_pages, Hkv, page_size, D], block_table
    [B, width] int32, seq_lens [B] int32 (the new tokens of the call counted in).  `q_start` [B + 1] int32 makes the
    new tokens ragged (at most n_q per sequence); without it there are n_q of each.  Rows of q, k, v and out are
    2-D tensors [rows, heads * D] whose rows may be strided."""

    def __init__(self, device: int, max_B: int, max_q: int, Hq: int, Hkv: int, D: int, page_size: int, dtype: int = AJ_BF16, flags: int = 0):
        self._h = _vp()
        f = _lib()
        st = f["aj_kv_create"](ctypes.byref(self._h), device, max_B, max_q, Hq, Hkv, D, page_size, dtype, flags)
        if st != AJ_OK:
            self._h = _vp()
            raise AjError(st, "aj_kv_create")
        self._append, self._attend, self._weigh, self._evict = (f["aj_kv_" + n] for n in ("append", "attend", "weigh", "evict"))

    def append(self, q, k, v, k_pages, v_pages, block_table, seq_lens, q_out, B: int, n_q: int, cos_sin=None, q_start=None, positions=None,
               q_norm=None, k_norm=None, eps: float = 1e-6, rot_dim=None, interleaved: bool = False, slot_pos=None, weight=None,
               stream: int = 0, check: bool = True) -> int:
        """aj_kv_append: per-head norms and position rotation of q and k, and the write of k and v into their slots.

        cos_sin [n_pos, rot_dim] f32 holds rot_dim / 2 cosines, then as many sines, of each position."""
        n_pos, width = cos_sin.shape if cos_sin is not None else (0, 0)
        if cos_sin is not None and rot_dim not in (None, width, 0):  # the library takes rot_dim for the length of the table's rows
            if check:
                raise AjError(AJ_ERR_INVALID_ARG, "aj_kv_append")
            return AJ_ERR_INVALID_ARG
        st = self._append(self._h, q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), _p(q_norm), _p(k_norm),
                          eps, _p(cos_sin), n_pos, width if rot_dim is None else rot_dim, interleaved, _p(positions), k_pages.data_ptr(),
                          v_pages.data_ptr(), k_pages.shape[0], block_table.data_ptr(), block_table.shape[1], seq_lens.data_ptr(), _p(q_start),
                          B, n_q, q_out.data_ptr(), q_out.stride(0), _p(slot_pos), _p(weight), stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_append")
        return st

    def attend(self, q, k_pages, v_pages, block_table, seq_lens, out, B: int, n_q: int, scale: float, q_start=None, window: int = 0,
               sinks: int = 0, lse=None, stream: int = 0, check: bool = True) -> int:
        """aj_kv_attend: out = softmax(scale * q K^T) V of the new tokens over the slots each of them sees."""
        st = self._attend(self._h, q.data_ptr(), q.stride(0), k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0], block_table.data_ptr(),
                          block_table.shape[1], seq_lens.data_ptr(), _p(q_start), B, n_q, scale, window, sinks, out.data_ptr(), out.stride(0),
                          _p(lse), stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_attend")
        return st

    def weigh(self, q, lse, k_pages, block_table, seq_lens, weight, weight_out, B: int, n_q: int, scale: float, q_start=None, n_rows=None,
              window: int = 0, sinks: int = 0, stream: int = 0, check: bool = True) -> int:
        """aj_kv_weigh: add to each slot's accumulated weight the attention it gets from the counted new tokens."""
        st = self._weigh(self._h, q.data_ptr(), q.stride(0), lse.data_ptr(), k_pages.data_ptr(), k_pages.shape[0], block_table.data_ptr(),
                         block_table.shape[1], seq_lens.data_ptr(), _p(q_start), _p(n_rows), B, n_q, scale, window, sinks, weight.data_ptr(),
                         weight_out.data_ptr(), stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_weigh")
        return st

    def evict(self, k_pages, v_pages, block_table, seq_lens, weight, slot_pos, lens_out, weight_out, slot_pos_out, B: int, keep: int,
              sinks: int = 0, recent: int = 0, stream: int = 0, check: bool = True) -> int:
        """aj_kv_evict: cut every longer (sequence, key head) to its `keep` most attended slots."""
        st = self._evict(self._h, k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0], block_table.data_ptr(), block_table.shape[1],
                         seq_lens.data_ptr(), B, keep, sinks, recent, weight.data_ptr(), slot_pos.data_ptr(), lens_out.data_ptr(),
                         weight_out.data_ptr(), slot_pos_out.data_ptr(), stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_evict")
        return st

    def last_status(self) -> int:
        return _lib()["aj_kv_last_status"](self._h)

    def last_launch_count(self) -> int:
        return _lib()["aj_kv_last_launch_count"](self._h)

    def last_path(self) -> str:
        return _lib()["aj_kv_last_path"](self._h).decode()

    def destroy(self) -> None:
        if self._h:
            _lib()["aj_kv_destroy"](self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
