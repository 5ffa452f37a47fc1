"""ctypes binding of the key-value cache operators (include/aj_kv.h): checks of the tensors and argument marshalling.

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
    2-D tensors [rows, heads * D] whose rows may be strided.

    Every call looks at its tensors' types and at the layout of pages and state, and refuses others with
    AJ_ERR_INVALID_ARG.  With `strict` it also looks at their devices, extents and the rest of their layout, which costs a
    call 6 to 8 us of the host's time: for a program that is being written.  What only the device knows is taken on trust: how
    many rows a q_start speaks of, what the tables hold."""

    def __init__(self, device: int, max_B: int, max_q: int, Hq: int, Hkv: int, D: int, page_size: int, dtype: int = AJ_BF16, flags: int = 0,
                 strict: bool = False):
        self._h = _vp()
        f = _lib()
        st = f["aj_kv_create"](ctypes.byref(self._h), device, max_B, max_q, Hq, Hkv, D, page_size, dtype, flags)
        if st != AJ_OK:
            self._h = _vp()
            raise AjError(st, "aj_kv_create")
        self._append, self._attend, self._weigh, self._evict = (f["aj_kv_" + n] for n in ("append", "attend", "weigh", "evict"))
        self._take(device, max_B, max_q, Hq, Hkv, D, page_size, dtype, strict)

    def _take(self, device, max_B, max_q, Hq, Hkv, D, page_size, dtype, strict):
        import torch

        self._device, self._max_B, self._max_q, self._Hq, self._Hkv, self._D, self._page = device, max_B, max_q, Hq, Hkv, D, page_size
        self._dtype, self._i32, self._f32, self._strict = torch.bfloat16 if dtype == AJ_BF16 else torch.float32, torch.int32, torch.float32, strict

    # ---- strict checks.  A batch or number of new tokens above the handle's is refused by the call itself.

    def _fits(self, B, n_q, pages, table, rows=(), q_start=None, per_row=(), per_seq=(), per_slot=(), tables=()):
        """Do all tensors lie on the device, whole, with the extents of a call?  rows: (tensor, heads); per_row, tables: (tensor, elements)."""
        B, n = min(B, self._max_B), min(n_q, self._max_q)
        n_rows = B * n if q_start is None else 0  # ragged: the device knows
        shape = (self._Hkv, self._page, self._D)
        if table.dim() != 2 or table.shape[0] < B or any(p.dim() != 4 or tuple(p.shape[1:]) != shape or p.shape[0] != pages[0].shape[0] for p in pages):
            return False
        slots = B * self._Hkv * table.shape[1] * self._page
        flat = [(x, 0) for x in (*pages, table)] + [(x, B) for x in per_seq] + [(x, slots) for x in per_slot] + [(x, n_rows * e) for x, e in per_row]
        flat += [*tables, (q_start, B + 1)]
        whole = [(x, n_rows * h * self._D) for x, h in rows]
        return (all(x is None or x.get_device() == self._device and x.is_contiguous() and x.numel() >= m for x, m in flat)
                and all(x.get_device() == self._device and x.numel() >= m and (x.dim() == 2 or x.dim() == 3 and x.stride(1) == self._D) for x, m in whole))

    def append(self, q, k, v, k_pages, v_pages, block_table, seq_lens, q_out, B: int, n_q: int, cos_sin=None, q_start=None, positions=None,
               q_norm=None, k_norm=None, eps: float = 1e-6, rot_dim=None, interleaved: bool = False, slot_pos=None, weight=None,
               stream: int = 0, check: bool = True) -> int:
        """aj_kv_append: per-head norms and position rotation of q and k, and the write of k and v into their slots.

        cos_sin [n_pos, rot_dim] f32 holds rot_dim / 2 cosines, then as many sines, of each position."""
        dt, f32, i32 = self._dtype, self._f32, self._i32
        qs, ks, vs, os = q.stride(), k.stride(), v.stride(), q_out.stride()
        n_pos, width = cos_sin.shape if cos_sin is not None else (0, 0)
        if rot_dim is None:
            rot_dim = width
        if (q.dtype is not dt or k.dtype is not dt or v.dtype is not dt or q_out.dtype is not dt or k_pages.dtype is not dt or v_pages.dtype is not dt
                or block_table.dtype is not i32 or seq_lens.dtype is not i32 or qs[-1] != 1 or ks[-1] != 1 or vs[-1] != 1 or os[-1] != 1
                or not k_pages.is_contiguous() or not v_pages.is_contiguous()
                or cos_sin is not None and (cos_sin.dtype is not f32 or rot_dim != width and rot_dim != 0)
                or q_norm is not None and q_norm.dtype is not f32 or k_norm is not None and k_norm.dtype is not f32
                or q_start is not None and q_start.dtype is not i32 or positions is not None and positions.dtype is not i32
                or slot_pos is not None and (slot_pos.dtype is not i32 or not slot_pos.is_contiguous())
                or weight is not None and (weight.dtype is not f32 or not weight.is_contiguous())
                or self._strict and not self._fits(B, n_q, (k_pages, v_pages), block_table, ((q, self._Hq), (k, self._Hkv), (v, self._Hkv), (q_out, self._Hq)),
                                                   q_start, ((positions, 1),), (seq_lens,), (slot_pos, weight),
                                                   ((cos_sin, 0), (q_norm, self._D), (k_norm, self._D)))):
            st = AJ_ERR_INVALID_ARG
        else:
            st = self._append(self._h, q.data_ptr(), qs[0], k.data_ptr(), ks[0], v.data_ptr(), vs[0], None if q_norm is None else q_norm.data_ptr(),
                              None if k_norm is None else k_norm.data_ptr(), eps, None if cos_sin is None else cos_sin.data_ptr(), n_pos, rot_dim,
                              interleaved, None if positions is None else positions.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0],
                              block_table.data_ptr(), block_table.shape[1], seq_lens.data_ptr(), None if q_start is None else q_start.data_ptr(), B, n_q,
                              q_out.data_ptr(), os[0], None if slot_pos is None else slot_pos.data_ptr(), None if weight is None else weight.data_ptr(),
                              stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_append")
        return st

    def attend(self, q, k_pages, v_pages, block_table, seq_lens, out, B: int, n_q: int, scale: float, q_start=None, window: int = 0,
               sinks: int = 0, lse=None, stream: int = 0, check: bool = True) -> int:
        """aj_kv_attend: out = softmax(scale * q K^T) V of the new tokens over the slots each of them sees."""
        dt, i32 = self._dtype, self._i32
        qs, os = q.stride(), out.stride()
        if (q.dtype is not dt or out.dtype is not dt or k_pages.dtype is not dt or v_pages.dtype is not dt or block_table.dtype is not i32
                or seq_lens.dtype is not i32 or qs[-1] != 1 or os[-1] != 1 or not k_pages.is_contiguous() or not v_pages.is_contiguous()
                or lse is not None and (lse.dtype is not self._f32 or not lse.is_contiguous()) or q_start is not None and q_start.dtype is not i32
                or self._strict and not self._fits(B, n_q, (k_pages, v_pages), block_table, ((q, self._Hq), (out, self._Hq)), q_start, ((lse, self._Hq),),
                                                   (seq_lens,))):
            st = AJ_ERR_INVALID_ARG
        else:
            st = self._attend(self._h, q.data_ptr(), qs[0], k_pages.data_ptr(), v_pages.data_ptr(), k_pages.shape[0], block_table.data_ptr(),
                              block_table.shape[1], seq_lens.data_ptr(), None if q_start is None else q_start.data_ptr(), B, n_q, scale, window, sinks,
                              out.data_ptr(), os[0], None if lse is None else lse.data_ptr(), stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_attend")
        return st

    def weigh(self, q, lse, k_pages, block_table, seq_lens, weight, weight_out, B: int, n_q: int, scale: float, q_start=None, n_rows=None,
              window: int = 0, sinks: int = 0, stream: int = 0, check: bool = True) -> int:
        """aj_kv_weigh: add to each slot's accumulated weight the attention it gets from the counted new tokens."""
        dt, f32, i32 = self._dtype, self._f32, self._i32
        qs = q.stride()
        if (q.dtype is not dt or k_pages.dtype is not dt or lse.dtype is not f32 or weight.dtype is not f32 or weight_out.dtype is not f32
                or block_table.dtype is not i32 or seq_lens.dtype is not i32 or qs[-1] != 1 or not k_pages.is_contiguous() or not lse.is_contiguous()
                or not weight.is_contiguous() or not weight_out.is_contiguous() or q_start is not None and q_start.dtype is not i32
                or n_rows is not None and n_rows.dtype is not i32
                or self._strict and not self._fits(B, n_q, (k_pages,), block_table, ((q, self._Hq),), q_start, ((lse, self._Hq),), (seq_lens, n_rows),
                                                   (weight, weight_out))):
            st = AJ_ERR_INVALID_ARG
        else:
            st = self._weigh(self._h, q.data_ptr(), qs[0], lse.data_ptr(), k_pages.data_ptr(), k_pages.shape[0], block_table.data_ptr(),
                             block_table.shape[1], seq_lens.data_ptr(), None if q_start is None else q_start.data_ptr(),
                             None if n_rows is None else n_rows.data_ptr(), B, n_q, scale, window, sinks, weight.data_ptr(), weight_out.data_ptr(),
                             stream or None)
        if check and st != AJ_OK:
            raise AjError(st, "aj_kv_weigh")
        return st

    def evict(self, k_pages, v_pages, block_table, seq_lens, weight, slot_pos, lens_out, weight_out, slot_pos_out, B: int, keep: int,
              sinks: int = 0, recent: int = 0, stream: int = 0, check: bool = True) -> int:
        """aj_kv_evict: cut every longer (sequence, key head) to its `keep` most attended slots."""
        dt, f32, i32 = self._dtype, self._f32, self._i32
        if (k_pages.dtype is not dt or v_pages.dtype is not dt or block_table.dtype is not i32 or seq_lens.dtype is not i32 or lens_out.dtype is not i32
                or weight.dtype is not f32 or weight_out.dtype is not f32 or slot_pos.dtype is not i32 or slot_pos_out.dtype is not i32
                or not k_pages.is_contiguous() or not v_pages.is_contiguous() or not weight.is_contiguous() or not weight_out.is_contiguous()
                or not slot_pos.is_contiguous() or not slot_pos_out.is_contiguous()
                or self._strict and not self._fits(B, 1, (k_pages, v_pages), block_table, per_seq=(seq_lens, lens_out),
                                                   per_slot=(weight, slot_pos, weight_out, slot_pos_out))):
            st = AJ_ERR_INVALID_ARG
        else:
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
