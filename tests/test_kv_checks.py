"""The binding of the key-value cache operators refuses tensors that the library would read as something else or past their end.
No device: a handle of CPU tensors whose calls are recorded instead of made."""
import pytest
import torch

import paper_2504_20039_b200 as aj

B, N, HQ, HKV, D, PAGE, WIDTH, POOL = 3, 2, 8, 2, 64, 16, 5, 11
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Recorder:
    def __init__(self, dtype=aj.AJ_BF16, device=-1, strict=True):
        from paper_2504_20039_b200.kv import KvHandle

        self.calls = []
        h = self.h = object.__new__(KvHandle)
        h._h = None
        for name in ("_append", "_attend", "_weigh", "_evict"):
            setattr(h, name, lambda *a, name=name: self.calls.append((name, a)) or aj.AJ_OK)
        h._take(device, B, N, HQ, HKV, D, PAGE, dtype, strict)  # -1: what get_device says of a CPU tensor


def arguments(op, dt=BF):
    z = torch.zeros
    pages = dict(k_pages=z(POOL, HKV, PAGE, D, dtype=dt), v_pages=z(POOL, HKV, PAGE, D, dtype=dt))
    cache = dict(block_table=z(B, WIDTH, dtype=I32), seq_lens=z(B, dtype=I32))
    state = lambda dtype: z(B, HKV, WIDTH * PAGE, dtype=dtype)  # noqa: E731
    qkv = z(B * N, (HQ + 2 * HKV) * D, dtype=dt)
    q, k, v = qkv.split([HQ * D, HKV * D, HKV * D], 1)
    if op == "append":
        return dict(q=q, k=k, v=v, **pages, **cache, q_out=z(B * N, HQ * D, dtype=dt), B=B, n_q=N, cos_sin=z(40, 32), q_norm=z(D), k_norm=z(D),
                    positions=z(B * N, dtype=I32), slot_pos=state(I32), weight=state(F32))
    if op == "attend":
        return dict(q=q, **pages, **cache, out=z(B * N, HQ * D, dtype=dt), B=B, n_q=N, scale=0.1, lse=z(B * N, HQ))
    if op == "weigh":
        return dict(q=q, lse=z(B * N, HQ), k_pages=pages["k_pages"], **cache, weight=state(F32), weight_out=state(F32), B=B, n_q=N, scale=0.1, n_rows=z(B, dtype=I32))
    return dict(**pages, **cache, weight=state(F32), slot_pos=state(I32), lens_out=z(B, dtype=I32), weight_out=state(F32), slot_pos_out=state(I32), B=B, keep=7)


ROWS = ("q", "k", "v", "q_out", "out")


def spoiled(name, t):
    """The same tensor in forms that a call must not take."""
    other = {BF: torch.float16, F32: torch.float64, I32: torch.int64}[t.dtype]
    yield "type", t.to(other)
    if t.is_cuda:
        yield "device", t.cpu()
    if name == "cos_sin":
        yield "layout", t.t().contiguous().t()
        return
    yield "extent", t[:-1] if name != "k_pages" else t[:, :, :-1].contiguous()
    if name in ROWS:
        yield "layout", t.t().contiguous().t()
    elif t.dim() > 1:
        yield "layout", t.transpose(0, 1).contiguous().transpose(0, 1)
    else:
        yield "layout", torch.zeros(2 * t.numel(), dtype=t.dtype, device=t.device)[::2]


STATE = ("k_pages", "v_pages", "lse", "weight", "weight_out", "slot_pos", "slot_pos_out")


@pytest.mark.parametrize("op", ["append", "attend", "weigh", "evict"])
@pytest.mark.parametrize("strict", [False, True])
@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_every_tensor_is_looked_at(op, strict, device):
    """Types always, the layout of rows, pages and state always; everything else on a strict handle."""
    r = Recorder(device=-1 if device == "cpu" else 0, strict=strict)
    good = {n: x.to(device) if isinstance(x, torch.Tensor) else x for n, x in arguments(op).items()}
    call = getattr(r.h, op)
    assert call(**good) == aj.AJ_OK and len(r.calls) == 1
    names = [n for n, x in good.items() if isinstance(x, torch.Tensor)]
    for n in names:
        for what, bad in spoiled(n, good[n]):
            if not strict and what != "type" and not (what == "layout" and n in ROWS + STATE):
                continue
            with pytest.raises(aj.AjError) as e:
                call(**{**good, n: bad})
            assert e.value.status == aj.AJ_ERR_INVALID_ARG, (n, what)
            assert call(**{**good, n: bad}, check=False) == aj.AJ_ERR_INVALID_ARG
            assert len(r.calls) == 1, (n, what)


def test_what_stays_allowed():
    r = Recorder()
    good = arguments("attend")
    wide = torch.zeros(B * N + 4, HQ * D + 24, dtype=BF)
    r.h.attend(**{**good, "q": wide[:, : HQ * D], "out": wide[2:, : HQ * D]})                          # strided rows, more of them
    r.h.attend(**{**good, "q": torch.zeros(B * N, HQ, D, dtype=BF)})                                  # heads as a dimension
    r.h.attend(**{**good, "q": wide[:1, : HQ * D], "out": wide[:1, : HQ * D], "lse": None, "q_start": torch.zeros(B + 1, dtype=I32)})  # ragged: any number
    r.h.attend(**{**good, "B": B + 1})                                                               # the library's own refusal
    r.h.attend(**{**good, "n_q": N + 1})
    a = arguments("append")
    r.h.append(**{**a, "cos_sin": None, "q_norm": None, "k_norm": None, "positions": None, "slot_pos": None, "weight": None})
    r.h.append(**{**a, "rot_dim": 0})
    r.h.append(**{**a, "rot_dim": 32})
    e = arguments("evict")
    r.h.evict(**{**e, "lens_out": e["seq_lens"], "weight_out": e["weight"], "slot_pos_out": e["slot_pos"]})
    assert len(r.calls) == 9
    f = Recorder(aj.AJ_F32)
    f.h.attend(**arguments("attend", F32))
    assert len(f.calls) == 1


def test_ragged_begins():
    r = Recorder()
    good = arguments("attend")
    for bad in (torch.zeros(B, dtype=I32), torch.zeros(B + 1, dtype=torch.int64)):
        with pytest.raises(aj.AjError):
            r.h.attend(**{**good, "q_start": bad})
    assert not r.calls
