"""The key-value cache operators on the GPU against their definitions in 64 bits: sizes, masks and layouts where
they can go wrong, and calls that have to be refused."""
import numpy as np
import pytest

from kv_testlib import NEG, Setup

pytestmark = pytest.mark.gpu

# name, lens, nq, Hq, Hkv, D, page, dtype, window, sinks
ATTEND = [
    ("one_token_bf16", [37], [1], 8, 2, 128, 16, "bf16", 0, 0),
    ("one_token_first", [1], [1], 8, 2, 64, 16, "bf16", 0, 0),
    ("empty_and_full", [0, 1, 16, 17, 300], [1, 1, 1, 1, 1], 8, 8, 128, 16, "bf16", 0, 0),
    ("ragged_with_none", [50, 0, 200, 129, 7], [1, 0, 3, 0, 2], 6, 2, 64, 32, "bf16", 0, 0),
    ("more_new_than_cached", [3, 40], [5, 5], 4, 2, 64, 16, "bf16", 0, 0),
    ("one_token_group_16", [513, 64], [1, 1], 16, 1, 128, 64, "bf16", 0, 0),
    ("two_tokens_group_8", [700, 128, 2], [2, 2, 2], 16, 2, 128, 32, "bf16", 0, 0),
    ("group_7", [333, 65], [2, 1], 14, 2, 64, 16, "bf16", 0, 0),
    ("long_one_token", [5000], [1], 4, 1, 128, 128, "bf16", 0, 0),
    ("window_one_token", [1000, 90, 4], [1, 1, 1], 8, 2, 128, 16, "bf16", 100, 4),
    ("window_of_one", [200, 3], [1, 2], 8, 2, 64, 16, "bf16", 1, 0),
    ("window_longer_than_cache", [200, 77], [1, 1], 8, 2, 64, 32, "bf16", 4096, 9),
    ("sinks_meet_window", [300, 130], [1, 1], 8, 2, 128, 32, "bf16", 200, 101),
    ("verify_17", [400, 17, 1037], [17, 17, 17], 8, 2, 128, 16, "bf16", 0, 0),
    ("verify_33_group_4", [300, 33, 161], [33, 33, 33], 8, 2, 128, 32, "bf16", 0, 0),
    ("verify_65_group_8", [65, 600], [65, 65], 16, 2, 128, 64, "bf16", 0, 0),
    ("verify_17_head_64", [513, 128], [17, 17], 8, 2, 64, 64, "bf16", 0, 0),
    ("verify_window", [513, 40, 2000], [17, 17, 17], 8, 2, 64, 16, "bf16", 64, 5),
    ("verify_long", [9000], [9], 8, 2, 128, 32, "bf16", 0, 0),
    ("prompt_causal", [300, 129], [300, 129], 4, 1, 128, 64, "bf16", 0, 0),
    ("prompt_ragged", [515, 0, 1, 128, 257], [515, 0, 1, 128, 257], 4, 2, 64, 32, "bf16", 0, 0),
    ("prompt_window", [700, 333], [700, 333], 4, 2, 128, 16, "bf16", 100, 4),
    ("prompt_window_head_64", [1025], [1025], 6, 2, 64, 128, "bf16", 256, 17),
    ("prompt_after_cache", [900, 300], [200, 37], 4, 2, 64, 64, "bf16", 0, 0),
    ("prompt_group_1", [260], [260], 2, 2, 128, 16, "bf16", 0, 0),
    ("f32_one_token", [37, 1037], [1, 1], 8, 2, 64, 16, "f32", 0, 0),
    ("f32_verify", [150, 20], [9, 9], 8, 2, 128, 32, "f32", 0, 0),
    ("f32_prompt_window", [150, 3, 0], [150, 3, 0], 4, 4, 64, 16, "f32", 32, 4),
    ("f32_group_8_long", [3000], [1], 8, 1, 128, 64, "f32", 0, 0),
    ("head_80", [130, 20], [3, 3], 6, 3, 80, 16, "bf16", 0, 0),
    ("head_8_f32", [70], [5], 2, 2, 8, 16, "f32", 0, 0),
    ("head_256", [90, 333], [2, 2], 4, 2, 256, 32, "bf16", 50, 3),
    ("head_96_f32", [200], [1], 4, 2, 96, 32, "f32", 0, 0),
]


def _attend(s, h, window, sinks, stream=0, pad=0, lse=True):
    import torch

    out = s.guard(torch.full((max(1, s.T), s.Hq * s.D + pad), 7.0, dtype=s.dt), "out")
    ls = s.guard(torch.full((max(1, s.T), s.Hq), 7.0), "lse") if lse else None
    h.attend(s.q, s.k, s.v, s.block_table, s.seq_lens, out[:, : s.Hq * s.D], s.B, s.max_n, s.scale, q_start=s.q_start, window=window, sinks=sinks,
             lse=ls, stream=stream)
    torch.cuda.synchronize()
    assert h.last_status() == 0
    s.check_guards()
    if pad:
        assert (out[:, s.Hq * s.D :] == 7.0).all()
    return out[: s.T, : s.Hq * s.D], None if ls is None else ls[: s.T]


@pytest.mark.parametrize("case", ATTEND, ids=[c[0] for c in ATTEND])
@pytest.mark.parametrize("simt", [False, True], ids=["default", "simt"])
def test_attend(case, simt):
    _, lens, nq, Hq, Hkv, D, page, dtype, window, sinks = case
    if simt and (dtype == "f32" or D not in (64, 128)):
        pytest.skip("the default path already is the CUDA-core kernel")
    s = Setup(len(case[0]) * 1000 + sum(lens), lens, nq, Hq, Hkv, D, page, dtype)
    h = s.handle(flags=1 if simt else 0)
    out, lse = _attend(s, h, window, sinks)
    s.check_attend(out, lse, window, sinks, rounded_weights=h.last_path() != "simt")
    again, lse2 = _attend(s, h, window, sinks)
    assert (again == out).all() and ((lse2 == lse) | (lse != lse)).all()  # two runs give the same bits


@pytest.mark.parametrize("n", [1, 17, 130])
def test_attend_strided_rows_side_stream_and_no_lse(n):
    import torch

    s = Setup(5, [200, 300], [n, n], 8, 2, 128, 16, ragged=False, pad=24)
    h = s.handle()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        out, _ = _attend(s, h, 0, 0, stream=st.cuda_stream, pad=40, lse=False)
    s.check_attend(out, None, 0, 0, rounded_weights=True)


@pytest.mark.parametrize("n,D", [(1, 128), (17, 64), (17, 128)])
def test_attend_large_scores_and_equal_keys(n, D):
    """Scores of several hundred (one key takes all the weight), and all keys equal (the mean of V)."""
    import torch

    s = Setup(9, [260, 131], [n, n], 8, 2, D, 16, ragged=False, q_scale=100.0)
    h = s.handle()
    out, lse = _attend(s, h, 0, 0)
    s.check_attend(out, lse, 0, 0, rounded_weights=True)
    good = ~torch.isnan(s.k)
    s.k[good] = 0.5
    out, lse = _attend(s, h, 0, 0)
    s.check_attend(out, lse, 0, 0, rounded_weights=True)


@pytest.mark.parametrize("D,page", [(128, 32), (64, 16)])
def test_attend_many_tiles_per_cta(D, page):
    """Windows whose two streams share the rows, over enough tiles that the ring of loads wraps several times in a
    CTA, with cold and warm caches (loads then land out of order): the same bits every time, and the right ones."""
    import torch

    s = Setup(4, [4096, 3000, 4095, 2049, 700, 4096, 1, 4096], [17] * 8, 32, 8, D, page, ragged=False)
    h = s.handle()
    out, lse = _attend(s, h, 0, 0)
    flush = torch.empty(64 * 1024 * 1024, device="cuda")
    for _ in range(30):
        flush.zero_()
        again, lse2 = _attend(s, h, 0, 0)
        assert torch.equal(again, out) and torch.equal(lse2, lse)
    s.check_attend(out, lse, 0, 0, rounded_weights=True)


@pytest.mark.parametrize("n", [1, 17])
def test_attend_joins_many_calls_on_one_handle(n):
    """Calls of different shape back to back: the counters and partial results of one leave nothing for the next."""
    big = Setup(1, [4000, 10, 900], [n] * 3, 8, 2, 128, 16, ragged=False)
    h = big.handle()
    small = Setup(2, [100], [1], 8, 2, 128, 16, ragged=False)
    for s in (big, small, big, small, small, big):
        out, lse = _attend(s, h, 0, 0)
        s.check_attend(out, lse, 0, 0, rounded_weights=True)


@pytest.mark.parametrize("n,D,window", [(17, 128, 0), (33, 128, 0), (65, 128, 0), (65, 64, 0), (17, 64, 2500), (65, 128, 4000)])
def test_attend_joins_many_parts(n, D, window):
    """One key head and a long cache: an item spans many CTAs, in streams that share the rows (17 x 4) and in streams of
    their own (33 x 4, 65 x 4).  Whichever CTA arrives last, the parts are joined in one order: the same bits every time."""
    import torch

    s = Setup(n + D, [5000, n, 0, 2063], [n] * 4, 4, 1, D, 64, ragged=False)
    h = s.handle()
    out, lse = _attend(s, h, window, 4 if window else 0)
    assert h.last_path() == "umma" and h.last_launch_count() == 1
    for _ in range(20):
        again, lse2 = _attend(s, h, window, 4 if window else 0)
        assert torch.equal(again, out) and torch.equal(lse2, lse)
    s.check_attend(out, lse, window, 4 if window else 0, rounded_weights=True)


WEIGH = [
    # name, lens, nq, counted rows, Hq, Hkv, D, page, dtype, window, sinks
    ("one_token", [37, 300, 0], [1, 1, 1], None, 8, 2, 128, 16, "bf16", 0, 0),
    ("one_token_head_64", [1000, 129], [1, 1], None, 4, 4, 64, 32, "bf16", 0, 0),
    ("verify", [400, 33, 129], [33, 33, 33], [1, 33, 17], 8, 2, 128, 32, "bf16", 0, 0),
    ("none_counted", [100, 60], [5, 5], [0, 9], 8, 2, 64, 16, "bf16", 0, 0),
    ("window", [500, 40], [9, 9], [9, 4], 16, 2, 128, 16, "bf16", 64, 4),
    ("group_7", [130, 260], [20, 20], [20, 3], 14, 2, 64, 64, "bf16", 0, 0),
    ("prompt", [300, 0, 77], [300, 0, 77], None, 4, 2, 128, 64, "bf16", 0, 0),
    ("more_new_than_cached", [3], [5], None, 4, 2, 64, 16, "bf16", 0, 0),
    ("many_rows", [700], [130], [129], 16, 2, 128, 16, "bf16", 0, 0),
    ("f32", [150, 20], [9, 9], [3, 9], 8, 2, 128, 32, "f32", 0, 0),
    ("f32_head_96", [70], [2], None, 4, 2, 96, 16, "f32", 0, 0),
]


@pytest.mark.parametrize("case", WEIGH, ids=[c[0] for c in WEIGH])
@pytest.mark.parametrize("inplace", [False, True])
def test_weigh(case, inplace):
    import torch

    _, lens, nq, rows, Hq, Hkv, D, page, dtype, window, sinks = case
    s = Setup(sum(lens) + 3, lens, nq, Hq, Hkv, D, page, dtype)
    ref_out, ref_lse, _, mag = s.attend_reference(window, sinks)
    lse = s.guard(ref_lse.float(), "lse")
    weight = s.guard(torch.rand(s.B, Hkv, s.cap), "weight")
    before = weight.cpu().double()
    out = weight if inplace else s.guard(torch.full((s.B, Hkv, s.cap), -3.0), "weight_out")
    n_rows = None if rows is None else s.guard(torch.tensor(rows, dtype=torch.int32), "n_rows")
    h = s.handle()
    h.weigh(s.q, lse, s.k, s.block_table, s.seq_lens, weight, out, s.B, s.max_n, s.scale, q_start=s.q_start, n_rows=n_rows, window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert h.last_status() == 0
    s.check_guards()
    got = out.cpu().double()
    lse64 = lse.cpu().double()
    for b in range(s.B):
        L, m = s.lens[b], s.nq[b] if rows is None else min(s.nq[b], rows[b])
        seen = s.visible(b, window, sinks)[:m] if L else None
        for hh in range(Hkv):
            want, tol = before[b, hh].clone(), 2.0**-22 * (1 + before[b, hh])
            for i in range(hh * s.G, (hh + 1) * s.G) if L and m else []:
                r = slice(int(s.start[b]), int(s.start[b]) + m)
                z = s.q.cpu()[r].double().view(m, Hq, D)[:, i] @ s.rows_of(s.k, b, hh).T * s.scale - lse64[r, i][:, None]
                z = torch.where(seen & (lse64[r, i] > NEG)[:, None], z, torch.tensor(NEG, dtype=torch.float64))
                p = z.exp()
                want[:L] += p.sum(0)
                # a score's error, the 32-bit product of lse and log2 e, and the sum over the rows
                tol[:L] += (p * (s.score_error(mag[r, i]) + 2.0**-22 * (2 + lse64[r, i].clamp_min(-1e3).abs()))[:, None] * 2).sum(0) + 2.0**-20 * p.sum(0)
            err = (got[b, hh, :L] - want[:L]).abs()
            assert (err <= tol[:L]).all(), float((err / tol[:L]).max())
    past = torch.arange(s.cap)[None, None] >= torch.tensor(s.lens)[:, None, None]
    keep = before if inplace else torch.full_like(before, -3.0)
    assert (got == keep)[past.expand_as(got)].all()


EVICT = [
    # name, lens, Hkv, D, page, keep, sinks, recent, dtype, weights
    ("one_over", [65], 2, 64, 16, 64, 4, 16, "bf16", "random"),
    ("batch", [200, 64, 10, 0, 131], 2, 128, 16, 64, 4, 16, "bf16", "random"),
    ("keep_one", [40, 1], 3, 64, 16, 1, 0, 0, "bf16", "random"),
    ("only_protected", [300], 2, 64, 32, 20, 4, 16, "bf16", "random"),
    ("all_equal", [500, 77], 2, 64, 32, 70, 0, 8, "bf16", "equal"),
    ("few_values", [2000, 333], 4, 64, 64, 256, 4, 32, "bf16", "few"),
    ("special_values", [400], 2, 64, 16, 150, 0, 0, "bf16", "special"),
    ("long", [9001], 1, 64, 128, 3000, 4, 128, "bf16", "random"),
    ("past_the_keys_that_fit", [50000], 1, 8, 128, 20001, 4, 128, "f32", "random"),
    ("many_items", [90 + i for i in range(40)], 8, 64, 16, 100, 4, 16, "bf16", "random"),
    ("head_80_f32", [130], 2, 80, 16, 33, 2, 3, "f32", "few"),
]


@pytest.mark.parametrize("case", EVICT, ids=[c[0] for c in EVICT])
@pytest.mark.parametrize("inplace", [False, True])
def test_evict(case, inplace):
    import torch

    _, lens, Hkv, D, page, keep, sinks, recent, dtype, kind = case
    s = Setup(sum(lens), lens, [1] * len(lens), Hkv, Hkv, D, page, dtype)
    rng = np.random.default_rng(7)
    w = rng.random((s.B, Hkv, s.cap)).astype(np.float32)
    if kind == "equal":
        w[:] = 0.25
    elif kind == "few":
        w = np.floor(w * 5).astype(np.float32) - 2.0
    elif kind == "special":
        pick = rng.integers(0, 8, w.shape)
        for i, x in enumerate([np.inf, -np.inf, np.nan, 0.0, -0.0, 1e-45, -1e-45]):
            w[pick == i] = x
    pos = np.stack([[rng.permutation(2 * s.cap)[: s.cap] for _ in range(Hkv)] for _ in range(s.B)]).astype(np.int32)
    weight, slot_pos = s.guard(torch.from_numpy(w.copy()), "weight"), s.guard(torch.from_numpy(pos.copy()), "slot_pos")
    k0, v0 = s.k.clone(), s.v.clone()
    if inplace:
        w_out, p_out, l_out = weight, slot_pos, s.seq_lens
    else:
        w_out, p_out = s.guard(torch.full((s.B, Hkv, s.cap), -3.0), "weight_out"), s.guard(torch.full((s.B, Hkv, s.cap), -3, dtype=torch.int32), "pos_out")
        l_out = s.guard(torch.full((s.B,), -3, dtype=torch.int32), "lens_out")
    h = s.handle()
    h.evict(s.k, s.v, s.block_table, s.seq_lens, weight, slot_pos, l_out, w_out, p_out, s.B, keep, sinks, recent)
    torch.cuda.synchronize()
    s.check_guards()
    got_w, got_p, got_l = w_out.cpu().numpy(), p_out.cpu().numpy(), l_out.cpu().numpy()
    base_w, base_p = (w, pos) if inplace else (np.full_like(w, -3.0), np.full_like(pos, -3))
    want_k, want_v = k0.clone(), v0.clone()
    for b, L in enumerate(lens):
        assert got_l[b] == min(L, keep)
        for hh in range(Hkv):
            ww, pp = w[b, hh], pos[b, hh]
            want_w, want_p = base_w[b, hh].copy(), base_p[b, hh].copy()
            n = min(L, keep)
            take = list(range(n))
            if L > keep:
                newest = pp[:L].max()

                def rank(j):
                    fixed = pp[j] < sinks or pp[j] > newest - recent
                    x = ww[j]
                    return (0 if fixed else 1, 1 if np.isnan(x) else 0, 0.0 if np.isnan(x) or fixed else -x, j)

                stay = set(sorted(range(L), key=rank)[:keep])
                holes = [j for j in range(keep) if j not in stay]
                movers = [j for j in range(keep, L) if j in stay]
                assert len(holes) == len(movers)
                for d, f in zip(holes, movers):
                    take[d] = f
                    at = lambda j: (int(s.table[b, j // page]), hh, j % page)  # noqa: E731, B023
                    want_k[at(d)], want_v[at(d)] = k0[at(f)], v0[at(f)]
            want_w[:n], want_p[:n] = ww[take], pp[take]
            np.testing.assert_array_equal(got_w[b, hh], want_w)
            np.testing.assert_array_equal(got_p[b, hh], want_p)
    assert torch.equal(torch.nan_to_num(s.k.float(), nan=99.0), torch.nan_to_num(want_k.float(), nan=99.0))
    assert torch.equal(torch.nan_to_num(s.v.float(), nan=99.0), torch.nan_to_num(want_v.float(), nan=99.0))


APPEND = [
    # name, lens, nq, Hq, Hkv, D, page, dtype, rot, interleaved, norm, positions
    ("one", [37], [1], 8, 2, 128, 16, "bf16", 128, False, True, False),
    ("one_head_64", [1, 16, 17], [1, 1, 1], 8, 2, 64, 16, "bf16", 64, False, False, False),
    ("window", [50, 33, 200], [33, 33, 33], 8, 2, 128, 32, "bf16", 128, False, True, True),
    ("pairs", [40, 77], [9, 9], 8, 2, 128, 16, "bf16", 128, True, True, False),
    ("pairs_half", [40, 77], [9, 9], 4, 2, 64, 16, "bf16", 32, True, False, False),
    ("half_rotated", [20, 19], [5, 5], 4, 2, 128, 16, "bf16", 64, False, True, False),
    ("half_rotated_64", [20, 19], [5, 5], 4, 2, 64, 16, "bf16", 32, False, True, False),
    ("odd_rotation", [20], [5], 4, 2, 64, 16, "bf16", 22, False, True, False),
    ("no_rotation", [20], [5], 4, 2, 64, 16, "bf16", 0, False, True, False),
    ("ragged_prompts", [300, 0, 1, 77], [300, 0, 1, 77], 14, 2, 128, 64, "bf16", 128, False, False, True),
    ("more_new_than_cached", [3], [5], 4, 2, 64, 16, "bf16", 64, False, False, True),
    ("f32", [37, 20], [3, 3], 8, 2, 128, 16, "f32", 128, False, True, False),
    ("f32_head_64_pairs", [37, 20], [3, 3], 6, 2, 64, 16, "f32", 64, True, False, True),
    ("f32_half", [37, 20], [3, 3], 6, 2, 64, 16, "f32", 32, False, True, True),
    ("head_80", [37], [3], 4, 1, 80, 16, "bf16", 80, False, True, False),
    ("head_256", [37], [3], 4, 1, 256, 16, "f32", 256, False, True, False),
]


@pytest.mark.parametrize("case", APPEND, ids=[c[0] for c in APPEND])
@pytest.mark.parametrize("fused_rows", [False, True])
def test_append(case, fused_rows):
    import torch

    _, lens, nq, Hq, Hkv, D, page, dtype, rot, pairs, norm, with_pos = case
    s = Setup(sum(lens) + D, lens, nq, Hq, Hkv, D, page, dtype)
    g = torch.Generator().manual_seed(3)
    T = s.T
    x = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g).to(s.dt)
    parts = [x[:, : Hq * D], x[:, Hq * D : (Hq + Hkv) * D], x[:, (Hq + Hkv) * D :]]
    if fused_rows:  # slices of one projection's output
        whole = s.guard(x, "qkv")
        q, k, v = whole[:, : Hq * D], whole[:, Hq * D : (Hq + Hkv) * D], whole[:, (Hq + Hkv) * D :]
    else:
        q, k, v = (s.guard(p.contiguous(), n) for p, n in zip(parts, "qkv"))
    n_pos = 400
    ang = torch.rand(n_pos, max(1, rot // 2), generator=g, dtype=torch.float64) * 6.28
    cs = s.guard(torch.cat([ang.cos(), ang.sin()], 1).float(), "cos_sin") if rot else None
    qw, kw = (s.guard(1 + 0.2 * torch.randn(D, generator=g), n) if norm else None for n in ("q_norm", "k_norm"))
    positions = s.guard(torch.randint(0, n_pos, (T,), generator=g, dtype=torch.int32), "positions") if with_pos else None
    q_out = q if fused_rows else s.guard(torch.full((T, Hq * D), 7.0, dtype=s.dt), "q_out")
    slot_pos = s.guard(torch.full((s.B, Hkv, s.cap), -9, dtype=torch.int32), "slot_pos")
    weight = s.guard(torch.full((s.B, Hkv, s.cap), 5.0), "weight")
    k0, v0 = s.k.cpu().clone(), s.v.cpu().clone()
    h = s.handle()
    h.append(q, k, v, s.k, s.v, s.block_table, s.seq_lens, q_out, s.B, s.max_n, cs, q_start=s.q_start, positions=positions, q_norm=qw, k_norm=kw,
             eps=1e-5, rot_dim=rot, interleaved=pairs, slot_pos=slot_pos, weight=weight)
    torch.cuda.synchronize()
    s.check_guards()

    def turned(row, H, w, p):
        y = row.double().view(H, D)
        if w is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-5) * w.cpu().double()
        z, m = y.clone(), y.abs().clone()
        for i in range(rot // 2):
            a, b2 = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
            c, sn = float(cs[p, i]), float(cs[p, rot // 2 + i])
            z[:, a], z[:, b2] = y[:, a] * c - y[:, b2] * sn, y[:, b2] * c + y[:, a] * sn
            m[:, a] = m[:, b2] = y[:, a].abs() + y[:, b2].abs()
        return z, m

    unit = 2.0**-8 if s.dt == torch.bfloat16 else 2.0**-23

    def close(got, want, mag):
        # one rounding on the store; a few 32-bit operations and the square root before it
        assert ((got.double() - want).abs() <= unit * want.abs() + 2.0**-20 * mag).all()

    want_k, got_k, got_v = k0.clone(), s.k.cpu(), s.v.cpu()
    want_pos, want_w = np.full((s.B, Hkv, s.cap), -9), np.full((s.B, Hkv, s.cap), 5.0)
    for b in range(s.B):
        for t in range(nq[b]):
            r, slot = int(s.start[b]) + t, lens[b] - nq[b] + t
            p = int(positions[r]) if with_pos else slot
            p = min(max(p, 0), n_pos - 1) if rot else p
            z, m = turned(parts[0][r], Hq, qw, p)
            close(q_out[r].cpu().view(Hq, D), z, m)
            if slot < 0:
                continue
            at = (int(s.table[b, slot // page]), slice(None), slot % page)
            z, m = turned(parts[1][r], Hkv, kw, p)
            close(got_k[at], z, m)
            want_k[at] = got_k[at]
            assert torch.equal(got_v[at], parts[2][r].view(Hkv, D))
            v0[at] = got_v[at]
            want_pos[b, :, slot] = int(positions[r]) if with_pos else slot
            want_w[b, :, slot] = 0.0
    same = lambda a, b: torch.equal(torch.nan_to_num(a.float(), nan=99.0), torch.nan_to_num(b.float(), nan=99.0))  # noqa: E731
    assert same(got_k, want_k) and same(got_v, v0)  # nothing else in the pages changed
    np.testing.assert_array_equal(slot_pos.cpu().numpy(), want_pos)
    np.testing.assert_array_equal(weight.cpu().numpy(), want_w)


def test_refusals():
    import torch

    import paper_2504_20039_b200 as aj

    s = Setup(1, [40, 50], [2, 2], 8, 2, 64, 16, ragged=False)
    h = s.handle()
    out = torch.zeros(4, 8 * 64, dtype=torch.bfloat16, device="cuda")

    def status(fn):
        with pytest.raises(aj.AjError) as e:
            fn()
        return e.value.status

    def attend(**kw):
        a = dict(q=s.q, k_pages=s.k, v_pages=s.v, block_table=s.block_table, seq_lens=s.seq_lens, out=out, B=2, n_q=2, scale=0.125)
        a.update(kw)
        h.attend(**a)

    attend()
    assert status(lambda: attend(B=0)) == aj.AJ_ERR_INVALID_ARG
    assert status(lambda: attend(n_q=0)) == aj.AJ_ERR_INVALID_ARG
    assert status(lambda: attend(B=3)) == aj.AJ_ERR_WORKSPACE
    assert status(lambda: attend(n_q=3)) == aj.AJ_ERR_WORKSPACE
    assert status(lambda: attend(scale=0.0)) == aj.AJ_ERR_INVALID_ARG
    assert status(lambda: attend(scale=float("nan"))) == aj.AJ_ERR_INVALID_ARG
    assert status(lambda: attend(window=-1)) == aj.AJ_ERR_INVALID_ARG
    assert status(lambda: attend(sinks=-1)) == aj.AJ_ERR_INVALID_ARG
    assert status(lambda: attend(q=s.q[:, : 4 * 64].contiguous())) == aj.AJ_ERR_INVALID_ARG  # rows shorter than the heads
    odd = torch.zeros(4, 8 * 64 + 1, dtype=torch.bfloat16, device="cuda")
    assert status(lambda: attend(q=odd[:, : 8 * 64])) == aj.AJ_ERR_UNSUPPORTED  # rows off 16 bytes
    assert status(lambda: attend(out=odd[:, 1:])) == aj.AJ_ERR_UNSUPPORTED
    w = torch.zeros(2, 2, s.cap, device="cuda")
    p = torch.zeros(2, 2, s.cap, dtype=torch.int32, device="cuda")
    for keep, sinks, recent in [(0, 0, 0), (10, -1, 0), (10, 0, -1), (10, 6, 5)]:
        assert status(lambda: h.evict(s.k, s.v, s.block_table, s.seq_lens, w, p, s.seq_lens, w, p, 2, keep, sinks, recent)) == aj.AJ_ERR_INVALID_ARG  # noqa: B023
    cs = torch.zeros(64, 64, device="cuda")
    kk = s.q[:, : 2 * 64]
    for kw in (dict(rot_dim=7), dict(rot_dim=66), dict(rot_dim=-2), dict(cos_sin=None, rot_dim=64), dict(eps=float("nan")), dict(eps=-1.0)):
        a = dict(cos_sin=cs, rot_dim=64)
        a.update(kw)
        assert status(lambda: h.append(s.q, kk, kk, s.k, s.v, s.block_table, s.seq_lens, out, 2, 2, **a)) == aj.AJ_ERR_INVALID_ARG  # noqa: B023
    assert status(lambda: h.weigh(s.q, w, s.k, s.block_table, s.seq_lens, w, w, 2, 2, -1.0)) == aj.AJ_ERR_INVALID_ARG
    torch.cuda.synchronize()
    s.check_guards()
