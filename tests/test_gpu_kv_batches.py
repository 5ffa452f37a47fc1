"""The key-value cache operators on the GPU over batches large enough that each CTA of a kernel walks over several sequences and
key heads: ring of loads, prefix sums over the batch, lists of moves, wide groups of query heads, and every slot counted once."""
import numpy as np
import pytest

from kv_testlib import NEG, Setup
from test_gpu_kv_edges import attend, set_slots

pytestmark = pytest.mark.gpu

RAGGED = [4096, 0, 1, 3001, 2049, 16, 17, 64, 129, 4095, 700, 2500, 63, 65, 1999, 3333, 5, 128, 1025, 2]


def weigh_and_check(s, h, n_rows=None, window=0, sinks=0, times=1):
    """One call of weigh, equal bits over `times` runs, against the definition in 64 bits."""
    import torch

    _, ref_lse, _, mag = s.attend_reference(window, sinks)
    lse = s.guard(ref_lse.float(), "lse")
    weight = s.guard(torch.rand(s.B, s.Hkv, s.cap), "weight")
    rows = None if n_rows is None else s.guard(torch.tensor(n_rows, dtype=torch.int32), "n_rows")
    first = None
    for _ in range(times):
        out = s.guard(torch.full((s.B, s.Hkv, s.cap), -3.0), "weight_out")
        h.weigh(s.q, lse, s.k, s.block_table, s.seq_lens, weight, out, s.B, s.max_n, s.scale, q_start=s.q_start, n_rows=rows, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert h.last_status() == 0
        first = out if first is None else first
        assert torch.equal(out, first)
    s.check_guards()
    got, before, lse64, q = first.cpu().double(), weight.cpu().double(), lse.cpu().double(), s.q.cpu().double()
    for b in range(s.B):
        L, m = s.lens[b], s.nq[b] if n_rows is None else min(s.nq[b], max(0, n_rows[b]))
        assert (got[b, :, L:] == -3.0).all()
        if not L:
            continue
        r = slice(int(s.start[b]), int(s.start[b]) + m)
        seen = s.visible(b, window, sinks)[:m]
        for hh in range(s.Hkv):
            heads = slice(hh * s.G, (hh + 1) * s.G)
            z = q[r].view(m, s.Hq, s.D)[:, heads] @ s.rows_of(s.k, b, hh).T * s.scale - lse64[r, heads, None]
            p = torch.where((seen[:, None] & (lse64[r, heads, None] > NEG)), z, torch.tensor(NEG, dtype=torch.float64)).exp()
            # a score's error, the 32-bit product of lse and log2 e, and the sum over the rows
            err = (p * (s.score_error(mag[r, heads]) + 2.0**-22 * (2 + lse64[r, heads].clamp_min(-1e3).abs()))[..., None] * 2).sum((0, 1)) + 2.0**-20 * p.sum((0, 1))
            tol = 2.0**-22 * (1 + before[b, hh, :L]) + err
            assert ((got[b, hh, :L] - before[b, hh, :L] - p.sum((0, 1))).abs() <= tol).all()


@pytest.mark.parametrize("D,page", [(128, 16), (64, 64)])
@pytest.mark.parametrize("n,window,sinks", [(1, 0, 0), (4, 0, 0), (1, 1000, 4), (2, 70, 100)])
def test_decode_over_many_blocks(n, window, sinks, D, page):
    """Some 5,000 blocks of 64 slots for 296 CTAs: the ring is refilled, CTAs go on from item to item and sequence to sequence, and hold the
    end of one item and the beginning of another."""
    s = Setup(n + D, RAGGED, [n] * len(RAGGED), 32, 8, D, page, ragged=False)
    h = s.handle()
    out, lse = attend(s, h, window, sinks, times=5)
    assert h.last_path() == "few"
    s.check_attend(out, lse, window, sinks, rounded_weights=True)


@pytest.mark.parametrize("n,D,window", [(17, 128, 0), (33, 64, 0), (33, 128, 900), (50, 128, 0)])
def test_windows_over_many_tiles(n, D, window):
    s = Setup(n + D, RAGGED, [n] * len(RAGGED), 32, 8, D, 32, ragged=False)
    h = s.handle()
    out, lse = attend(s, h, window, 4 if window else 0, times=5)
    assert h.last_path() == "umma"
    s.check_attend(out, lse, window, 4 if window else 0, rounded_weights=True)


@pytest.mark.parametrize("n,D,path,window", [(1, 128, "mma", 0), (4, 64, "mma", 900), (17, 128, "umma", 0), (33, 64, "umma", 900), (70, 64, "umma", 0)])
def test_weigh_over_many_blocks(n, D, path, window):
    """Several blocks and several (sequence, key head) pairs for each CTA of both tensor-core kernels."""
    s = Setup(n + D, RAGGED, [n] * len(RAGGED), 16, 8, D, 16, ragged=False)
    h = s.handle()
    weigh_and_check(s, h, [(7 * b) % (n + 2) for b in range(s.B)], window, 4 if window else 0, times=5)
    assert h.last_path() == path


@pytest.mark.parametrize("B", [33, 129, 385, 4096])
@pytest.mark.parametrize("n,path", [(1, "few"), (9, "umma")])
def test_many_sequences(B, n, path):
    """Prefix sums over more sequences than a warp has lanes and a CTA has threads, up to the most that a handle allows; lengths of zero and
    one among them."""
    rng = np.random.default_rng(B + n)
    lens = rng.integers(0, 40, B)
    lens[:: B // 8] = rng.integers(300, 900, len(lens[:: B // 8]))
    s = Setup(B, lens.tolist(), [n] * B, 2, 1, 64, 16, ragged=False)
    h = s.handle()
    out, lse = attend(s, h, times=2)
    assert h.last_path() == path
    s.check_attend(out, lse, 0, 0, rounded_weights=True)
    weigh_and_check(s, h, rng.integers(0, n + 1, B).tolist())


@pytest.mark.parametrize("G", [9, 16, 17, 20, 32, 64, 100, 128])
@pytest.mark.parametrize("n,D", [(2, 128), (5, 64), (9, 128)])
def test_wide_groups_of_query_heads(G, n, D):
    """More than eight query heads per key head: row tiles of few tokens, queries in boxes of one token where a tile has fewer than eight."""
    s = Setup(G + n, [300, 2, 129, 1500], [n] * 4, 2 * G, 2, D, 32, ragged=False)
    h = s.handle()
    for window, sinks in [(0, 0), (100, 3)]:
        out, lse = attend(s, h, window, sinks, times=2)
        assert h.last_path() == "umma"
        s.check_attend(out, lse, window, sinks, rounded_weights=True)
        weigh_and_check(s, h, [n, 1, n, 2], window, sinks)
        assert h.last_path() == "umma"


@pytest.mark.parametrize("dtype,n,path", [("bf16", 1, "few"), ("bf16", 4, "few"), ("bf16", 17, "umma"), ("bf16", 33, "umma"), ("bf16", 70, "umma"), ("f32", 1, "simt"),
                                          ("f32", 17, "simt")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 1100])
def test_every_slot_counts_once(dtype, n, path, D, window):
    """All keys alike, and the value of slot j one in column j % D: an output is the share of a row's visible slots that lie in its column.
    Times the number of visible slots it is a whole number, at most 64, and the rounding of the store (2^-8) takes it a quarter
    away at most: the nearest whole number has to be the count itself.  A lost or doubled slot also moves lse by 1 in 4000."""
    import torch

    s = Setup(n, [4096, 1, 3000, 100, 4095, 2050, 64, 2176], [n] * 8, 8, 2, D, 32, dtype, ragged=False, q_scale=0.1)
    for b, L in enumerate(s.lens):
        set_slots(s, s.k, b, torch.full((L, D), 0.5))
        set_slots(s, s.v, b, torch.nn.functional.one_hot(torch.arange(L) % D, D).float())
    h = s.handle()
    out, lse = attend(s, h, window, 4 if window else 0)
    assert h.last_path() == path
    ref, ref_lse, _, mag = s.attend_reference(window, 4 if window else 0)
    seen = torch.cat([s.visible(b, window, 4 if window else 0).sum(1) for b in range(s.B)])[:, None, None]
    assert torch.equal((out.cpu().double().view(s.T, s.Hq, D) * seen).round(), (ref * seen).round())
    fin = ~torch.isinf(ref_lse)
    assert torch.equal(torch.isinf(lse.cpu()), ~fin)
    assert ((lse.cpu().double() - ref_lse).abs()[fin] <= (2 * s.score_error(mag) + 2.0**-18 + 2.0**-21 * ref_lse.abs())[fin]).all()


@pytest.mark.parametrize("lens,Hkv,keep", [([40000, 39990, 33000, 20001, 36000], 16, 20000), ([300000], 1, 100000), ([300000, 150001], 1, 150000)])
@pytest.mark.parametrize("inplace", [False, True])
def test_evict_where_keys_and_moves_do_not_fit(lens, Hkv, keep, inplace):
    """More slots for a CTA than keys fit its shared memory (the weights are read again for every digit) and more moves than its list holds
    (several passes): 80 pairs, for which no clusters are formed, and one and two pairs in clusters of eight."""
    import torch

    D, page, sinks, recent = 8, 128, 4, 128
    s = Setup(len(lens), lens, [1] * len(lens), Hkv, Hkv, D, page, "f32")
    rng = np.random.default_rng(7)
    w = np.round(rng.random((s.B, Hkv, s.cap)) * 2000).astype(np.float32)  # ties among them
    pos = np.stack([[rng.permutation(2 * s.cap)[: s.cap] for _ in range(Hkv)] for _ in range(s.B)]).astype(np.int32)
    weight, slot_pos = s.guard(torch.from_numpy(w.copy()), "weight"), s.guard(torch.from_numpy(pos.copy()), "slot_pos")
    k0, v0 = s.k.cpu().clone(), s.v.cpu().clone()
    if inplace:
        w_out, p_out, l_out = weight, slot_pos, s.seq_lens
    else:
        w_out, p_out = s.guard(torch.full((s.B, Hkv, s.cap), -3.0), "weight_out"), s.guard(torch.full((s.B, Hkv, s.cap), -3, dtype=torch.int32), "pos_out")
        l_out = s.guard(torch.full((s.B,), -3, dtype=torch.int32), "lens_out")
    h = s.handle()
    h.evict(s.k, s.v, s.block_table, s.seq_lens, weight, slot_pos, l_out, w_out, p_out, s.B, keep, sinks, recent)
    torch.cuda.synchronize()
    s.check_guards()
    assert l_out.tolist() == [min(L, keep) for L in lens]
    got_w, got_p = w_out.cpu().numpy(), p_out.cpu().numpy()
    for b, L in enumerate(lens):
        n, slot = min(L, keep), np.arange(L)
        for hh in range(Hkv):
            ww, pp = w[b, hh, :L], pos[b, hh, :L]
            fixed = (pp < sinks) | (pp > int(pp.max()) - recent)
            stay = np.zeros(L, bool)
            stay[np.lexsort((slot, -ww.astype(np.float64), ~fixed))[:keep]] = True
            take = slot[:n].copy()
            dst, src = take[~stay[:n]], slot[stay & (slot >= keep)]
            take[dst] = src
            np.testing.assert_array_equal(got_w[b, hh, :n], ww[take])
            np.testing.assert_array_equal(got_p[b, hh, :n], pp[take])
            if not inplace:
                assert (got_w[b, hh, n:] == -3.0).all() and (got_p[b, hh, n:] == -3).all()
            to, fro = (s.table[b, dst // page], dst % page), (s.table[b, src // page], src % page)
            k0[to[0], hh, to[1]], v0[to[0], hh, to[1]] = k0[fro[0], hh, fro[1]], v0[fro[0], hh, fro[1]]
    for got, want in ((s.k.cpu(), k0), (s.v.cpu(), v0)):
        assert torch.equal(torch.nan_to_num(got, nan=99.0), torch.nan_to_num(want, nan=99.0))


@pytest.mark.parametrize("n,D", [(3, 128), (9, 64)])
def test_more_query_heads_than_a_row_tile(n, D):
    """200 query heads on one key head: attention goes to the CUDA cores, weights stay on the tensor cores."""
    s = Setup(n, [300, 2, 129], [n] * 3, 200, 1, D, 32, ragged=False)
    h = s.handle()
    out, lse = attend(s, h, 100, 3)
    assert h.last_path() == "simt"
    s.check_attend(out, lse, 100, 3, rounded_weights=False)
    weigh_and_check(s, h, [n, 1, 2], 100, 3)
    assert h.last_path() == "umma"


@pytest.mark.parametrize("n,D,paths", [(1, 128, ("few", "mma")), (17, 128, ("simt", "mma")), (33, 64, ("simt", "mma"))])
@pytest.mark.parametrize("window", [0, 150])
def test_pages_off_128_bytes(n, D, paths, window):
    """Pages that start on 16 bytes but not on 128, as a slice of a larger tensor may."""
    import torch

    s = Setup(n, [700, 64, 333, 1], [n] * 4, 8, 2, D, 16, ragged=False)
    for name in ("k", "v"):
        t = getattr(s, name)
        room = s.guard(torch.zeros(t.numel() + 8, dtype=t.dtype), name + "_off")
        moved = room[8:].view(t.shape)
        moved.copy_(t)
        assert moved.data_ptr() % 128 == 16
        setattr(s, name, moved)
    h = s.handle()
    out, lse = attend(s, h, window, 4 if window else 0, times=2)
    assert h.last_path() == paths[0]
    s.check_attend(out, lse, window, 4 if window else 0, rounded_weights=paths[0] != "simt")
    weigh_and_check(s, h, None, window, 4 if window else 0)
    assert h.last_path() == paths[1]


@pytest.mark.parametrize("n", [1, 17, 130])
@pytest.mark.parametrize("off", [8, 64])
def test_query_rows_off_128_bytes(n, off):
    """Query rows that do not start on 128 bytes are copied by a warp; on 128 bytes they come by TMA: the same bits."""
    import torch

    s = Setup(n, [700, 333], [n] * 2, 8, 2, 128, 16, ragged=False)
    h = s.handle()
    out, lse = attend(s, h)
    room = torch.zeros(s.T, s.Hq * s.D + 128, dtype=s.dt, device="cuda")
    rows = room[:, off : off + s.Hq * s.D]
    rows.copy_(s.q)
    s.q = rows
    again, lse2 = attend(s, h)
    assert torch.equal(again, out) and torch.equal(lse2, lse)
