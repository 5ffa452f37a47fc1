"""The key-value cache operators on the GPU where their kernels' inner steps meet rare values."""
import pytest

from kv_testlib import Setup

pytestmark = pytest.mark.gpu


def attend(s, h, window=0, sinks=0, stream=0, times=1):
    """(out, lse) of a call, compared bit by bit over `times` runs."""
    import torch

    first = None
    for _ in range(times):
        out = s.guard(torch.full((max(1, s.T), s.Hq * s.D), 7.0, dtype=s.dt), "out")
        lse = s.guard(torch.full((max(1, s.T), s.Hq), 7.0), "lse")
        torch.cuda.synchronize()
        h.attend(s.q, s.k, s.v, s.block_table, s.seq_lens, out, s.B, s.max_n, s.scale, q_start=s.q_start, window=window, sinks=sinks, lse=lse, stream=stream)
        torch.cuda.synchronize()
        assert h.last_status() == 0
        if first is None:
            first = out, lse
        else:
            assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    s.check_guards()
    return first[0][: s.T], first[1][: s.T]


def set_slots(s, pages, b, values):
    """Write rows [L, D] (the same for every key head) into the slots of sequence b."""
    L = s.lens[b]
    for j in range(0, L, s.page):
        n = min(s.page, L - j)
        pages[int(s.table[b, j // s.page]), :, :n] = values[j : j + n].to(pages)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,path", [(1, "few"), (4, "few"), (17, "umma"), (33, "umma"), (65, "umma")])
@pytest.mark.parametrize("window", [0, 1500])
def test_attend_scores_that_rise_with_every_half_tile(n, path, D, window):
    """A third of the rows meet scores that rise by more than the running reference tolerates (30 in units of log2) every 64 slots,
    so that the output is rescaled at nearly every half tile, behind the product before it; a third meet falling
    scores, a third flat ones.  17 x 4 rows: streams that share them; 33 x 4 and 65 x 4: streams of their own."""
    import torch

    s = Setup(n + D, [2300, 2049, 700, 2304, 1999, 2111, 1024, 65], [n] * 8, 32, 8, D, 32, ragged=False)
    g = torch.Generator().manual_seed(1)
    u = torch.randint(0, 2, (D,), generator=g) * 2.0 - 1.0
    step = 0.25 if D == 128 else 0.5
    for b, L in enumerate(s.lens):
        rise = step * (torch.arange(L) // 64)[:, None]
        set_slots(s, s.k, b, rise * u + 0.02 * torch.randn(L, D, generator=g))
    slope = torch.tensor([8.0, -8.0, 0.0])[torch.arange(s.T * s.Hq) % 3].view(s.T, s.Hq, 1)
    s.q.copy_((slope * u + 0.1 * torch.randn(s.T, s.Hq, D, generator=g)).view(s.T, s.Hq * D))
    h = s.handle()
    out, lse = attend(s, h, window, 4 if window else 0, times=6)
    assert h.last_path() == path
    s.check_attend(out, lse, window, 4 if window else 0, rounded_weights=True)


@pytest.mark.parametrize("n", [1, 17])
def test_a_fresh_handle_is_ready_for_any_stream(n):
    """Creation leaves nothing of its own behind work that is queued on the default stream: a handle made there serves a stream that does
    not wait for it, wherever its memory was before.  (An item that spans CTAs is stored by the part that arrives last, by a count
    from zero; an eviction writes its lengths likewise.)"""
    import ctypes

    import torch

    s = Setup(3, [5000, 3000], [n, n], 8, 2, 128, 16, ragged=False)
    warm = s.handle()
    out, lse = attend(s, warm)  # kernels are loaded
    w, p = torch.rand(2, 2, s.cap, device="cuda"), torch.arange(s.cap, device="cuda", dtype=torch.int32).repeat(2, 2, 1)
    rows = [torch.zeros_like(x) for x in (s.seq_lens, w, p)]
    warm.evict(s.k, s.v, s.block_table, s.seq_lens, w, p, *rows, 2, 6000)
    assert rows[0].tolist() == s.lens

    # small pieces of device memory full of ones, every other one given back
    rt = ctypes.CDLL("libcudart.so.12")
    held = []
    for _ in range(1024):
        x = ctypes.c_void_p()
        assert rt.cudaMalloc(ctypes.byref(x), 2048) == 0 and rt.cudaMemset(x, 0xFF, 2048) == 0
        held.append(x)
    torch.cuda.synchronize()
    for x in held[::2]:
        assert rt.cudaFree(x) == 0
    side = torch.cuda.Stream()
    o, ls, lens = torch.full_like(out, 7.0), torch.full_like(lse, 7.0), torch.full_like(s.seq_lens, -3)
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)
    busy = torch.cuda.Event()
    busy.record()
    h = s.handle()
    h.attend(s.q, s.k, s.v, s.block_table, s.seq_lens, o, 2, n, s.scale, lse=ls, stream=side.cuda_stream)
    h.evict(s.k, s.v, s.block_table, s.seq_lens, w, p, lens, rows[1], rows[2], 2, 6000, stream=side.cuda_stream)
    side.synchronize()
    queued = not busy.query()
    torch.cuda.synchronize()
    for x in held[1::2]:
        assert rt.cudaFree(x) == 0
    assert torch.equal(o, out) and torch.equal(ls, lse) and lens.tolist() == s.lens
    assert queued, "the side stream did not run beside the default stream: nothing was tested"


PATHS = [("bf16", 1, 0, "few"), ("bf16", 4, 0, "few"), ("bf16", 17, 0, "umma"), ("bf16", 33, 0, "umma"), ("bf16", 70, 0, "umma"), ("bf16", 4, 1, "simt"), ("f32", 1, 0, "simt"),
         ("f32", 9, 0, "simt")]


@pytest.mark.parametrize("dtype,n,flags,path", PATHS)
@pytest.mark.parametrize("what", ["nan_key", "inf_score", "nan_query", "nan_everywhere", "minus_inf_scores"])
@pytest.mark.parametrize("window", [0, 150])
def test_attend_scores_that_are_no_numbers(dtype, n, flags, path, what, window):
    """A NaN or +infinite score of a slot that a row sees makes the row NaN, lse too, wherever the slot lies in a tile; rows that do not see the
    slot keep their bits.  Scores of -infinity weigh nothing."""
    import torch

    B = 8
    s = Setup(n, [700 + 37 * b for b in range(B)], [n] * B, 8, 2, 128, 32, dtype, ragged=False)
    h = s.handle(flags)
    sinks = 4 if window else 0
    base, base_lse = attend(s, h, window, sinks)
    s.check_attend(base, base_lse, window, sinks, rounded_weights=path != "simt")
    hit = torch.zeros(s.T, s.Hq, dtype=torch.bool)
    if what in ("nan_key", "inf_score", "minus_inf_scores"):
        if what != "nan_key":
            s.q.view(s.T, s.Hq, 128)[:, :, 5] = 1.0
            base, base_lse = attend(s, h, window, sinks)
        value = {"nan_key": float("nan"), "inf_score": float("inf"), "minus_inf_scores": -float("inf")}[what]
        for b in range(B):  # every place in a group of eight, of either half of a tile, seen by some of the new tokens at least
            L = s.lens[b]
            slots = [L - n - 8 - (L - n) % 8 + b] + ([L - 1 - b % n] if n > 1 else [])
            for j in slots:
                s.k[int(s.table[b, j // 32]), 1, j % 32, 5] = value
                seen = s.visible(b, window, sinks)[:, j]
                hit[b * n : (b + 1) * n, 4:] |= seen[:, None]
    elif what == "nan_query":
        for b in range(B):
            t, i = b * n + b % n, b % 8
            s.q[t, i * 128 + 7 * b] = float("nan")
            hit[t, i] = True
    else:
        for b in range(B):
            p = torch.from_numpy(s.table[b, : -(-s.lens[b] // 32)])
            s.k[p, 1] = float("nan")
        hit[:, 4:] = True
    out, lse = attend(s, h, window, sinks)
    assert h.last_path() == path
    out, base = out.view(s.T, s.Hq, 128).cpu(), base.view(s.T, s.Hq, 128).cpu()
    lse, base_lse = lse.cpu(), base_lse.cpu()
    assert hit.any()
    if what == "minus_inf_scores":
        s.check_attend(out.reshape(s.T, -1), lse, window, sinks, rounded_weights=path != "simt")
    else:
        assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(out[~hit], base[~hit]) and torch.equal(lse[~hit], base_lse[~hit])


@pytest.mark.parametrize("dtype,n,flags,path", PATHS)
def test_attend_rows_whose_every_score_is_minus_infinity(dtype, n, flags, path):
    """Nothing is left of a row whose every visible score is -infinity: zeros and lse = -inf, as for a row that sees nothing."""
    import torch

    s = Setup(n, [300, 100], [n] * 2, 8, 2, 128, 32, dtype, ragged=False)
    s.k[..., 5] = torch.where(torch.isnan(s.k[..., 5]), s.k[..., 5], -float("inf"))
    s.q.view(s.T, s.Hq, 128)[:, :, 5] = 1.0
    h = s.handle(flags)
    out, lse = attend(s, h)
    assert h.last_path() == path
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("dtype,n,flags,path", [("bf16", 1, 0, "mma"), ("bf16", 4, 0, "mma"), ("bf16", 17, 0, "umma"), ("bf16", 33, 0, "umma"), ("bf16", 70, 0, "umma"),
                                                ("bf16", 9, 1, "simt"), ("f32", 9, 0, "simt")])
@pytest.mark.parametrize("what", ["nan_lse", "nan_query", "nan_key"])
@pytest.mark.parametrize("window", [0, 150])
def test_weigh_keeps_a_nan_to_the_slots_that_see_it(dtype, n, flags, path, what, window):
    """A NaN in a row's lse or query reaches the slots that the row sees and no others, a NaN key its own slot if a counted row sees it;
    every other weight keeps its bits."""
    import torch

    s = Setup(n, [300 + 61 * b for b in range(4)], [n] * 4, 8, 2, 128, 32, dtype, ragged=False)
    h = s.handle(flags)
    sinks = 4 if window else 0
    lse = attend(s, h, window, sinks)[1].clone()
    before = torch.rand(s.B, s.Hkv, s.cap, device="cuda")
    rows = torch.tensor([n, max(1, n // 2), n, n], dtype=torch.int32, device="cuda")

    def weigh():
        out = s.guard(torch.full((s.B, s.Hkv, s.cap), -3.0), "weight_out")
        h.weigh(s.q, lse, s.k, s.block_table, s.seq_lens, before, out, s.B, n, s.scale, n_rows=rows, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert h.last_status() == 0 and h.last_path() == path
        return out.cpu()

    base = weigh()
    assert not torch.isnan(base).any()
    hit = torch.zeros(s.B, s.Hkv, s.cap, dtype=torch.bool)
    for b, L in enumerate(s.lens):
        m = int(rows[b])
        seen = s.visible(b, window, sinks)[:m]
        if what == "nan_key":
            for j in (5, L // 2, L - n + n // 3, L - 1):
                s.k[int(s.table[b, j // 32]), 1, j % 32, 9] = float("nan")
                hit[b, 1, j] = seen[:, j].any()
        else:
            t, i = (0 if b % 2 else m // 2), 1 + 2 * b  # a row that counts
            if what == "nan_lse":
                lse[b * n + t, i] = float("nan")
            else:
                s.q[b * n + t, i * 128 + 3] = float("nan")
            hit[b, i // 4, :L] |= seen[t]
            if m < n:  # and one that does not
                if what == "nan_lse":
                    lse[b * n + n - 1, i] = float("nan")
                else:
                    s.q[b * n + n - 1, i * 128 + 3] = float("nan")
    got = weigh()
    s.check_guards()
    assert hit.any() and torch.isnan(got[hit]).all()
    assert torch.equal(got[~hit], base[~hit])


@pytest.mark.parametrize("dtype,n,flags,path", PATHS)
@pytest.mark.parametrize("window,sinks", [(2**31 - 1, 0), (2**31 - 1, 2**31 - 1), (7, 2**31 - 1), (1000, 2**30)])
def test_windows_and_sinks_as_large_as_an_int(dtype, n, flags, path, window, sinks):
    """A window or sinks of no limit, with sequences that have fewer slots than new tokens: the bits of the call without a window."""
    import torch

    s = Setup(n, [3, 500, 1, 0, n + 2, 5, 77, 300], [n] * 8, 8, 2, 128, 32, dtype, ragged=False)
    h = s.handle(flags)
    base, base_lse = attend(s, h)
    s.check_attend(base, base_lse, 0, 0, rounded_weights=path != "simt")
    out, lse = attend(s, h, window, sinks)
    assert h.last_path() == path
    s.check_attend(out, lse, 0, 0, rounded_weights=path != "simt")
    if window >= s.cap:
        assert torch.equal(out, base) and torch.equal(lse, base_lse)
    before = torch.rand(s.B, s.Hkv, s.cap, device="cuda")
    weights = [s.guard(torch.full((s.B, s.Hkv, s.cap), -3.0), "weight_out") for _ in range(2)]
    for w, (win, snk) in zip(weights, [(0, 0), (window, sinks)]):
        h.weigh(s.q, base_lse, s.k, s.block_table, s.seq_lens, before, w, s.B, n, s.scale, window=win, sinks=snk)
    torch.cuda.synchronize()
    s.check_guards()
    assert torch.equal(weights[0], weights[1])
