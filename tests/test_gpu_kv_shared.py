"""aj_kv_attend_shared against the definition of attention in 64 bits, over caches whose first pages belong to all sequences."""
import numpy as np
import pytest
import torch

import paper_2504_20039_b200 as aj
from kv_testlib import Setup

pytestmark = pytest.mark.gpu
SIMT, SHARED = aj.AJ_KV_FLAG_FORCE_SIMT, aj.AJ_KV_FLAG_FORCE_SHARED


def shared_setup(seed, shared, own, nq, Hq, Hkv, D, page, alone=(), **kw):
    """own: slots behind the prefix (new tokens among them); sequences in `alone` have own slots only."""
    lens = [n if b in alone else shared + n for b, n in enumerate(own)]
    s = Setup(seed, lens, nq, Hq, Hkv, D, page, **kw)
    first = -(-shared // page)
    lead = next(b for b in range(s.B) if b not in alone)
    # a page that holds the end of the prefix and tokens of one sequence is that sequence's own: it holds the same prefix slots
    whole = shared // page
    for b in range(s.B):
        if b in alone or b == lead:
            continue
        s.table[b, :whole] = s.table[lead, :whole]
        if first > whole:
            r = shared - whole * page
            for t in (s.k, s.v):
                t[int(s.table[b, whole]), :, :r] = t[int(s.table[lead, whole]), :, :r]
    s.block_table.copy_(torch.tensor(np.minimum(s.table, 2**31 - 1), dtype=torch.int32))
    s.shared = shared
    s.prefix = s.guard(torch.tensor(s.table[lead, :first], dtype=torch.int32), "shared_table")
    return s


def run(s, rows=None, flags=SHARED, with_lse=True, handle=None, stream=0):
    h = handle or s.handle(flags)
    h.reserve_shared(rows or max(1, s.T))
    out = s.guard(torch.full((max(1, s.T), s.Hq * s.D), 99.0, dtype=s.dt), "out")[: s.T]
    lse = s.guard(torch.full((s.T, s.Hq), 99.0), "lse") if with_lse else None
    h.attend_shared(s.q, s.k, s.v, s.prefix, s.shared, s.block_table, s.seq_lens, out, s.B, s.max_n, s.scale, q_start=s.q_start, lse=lse, stream=stream)
    torch.cuda.synchronize()
    assert h.last_status() == aj.AJ_OK
    s.check_guards()
    s.path, s.launches = h.last_path(), h.last_launch_count()
    if not handle:
        h.destroy()
    return out, lse


def check(s, out, lse, rounded=True):
    s.check_attend(out, lse, 0, 0, rounded_weights=rounded)


@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 8, 2, 16), (64, 6, 2, 32), (128, 16, 1, 64), (64, 2, 2, 128)])
@pytest.mark.parametrize("shared,own", [(128, [1, 1]), (256, [1, 200, 7, 129]), (384, [64, 65, 66, 500, 1, 128, 127]), (1000, [3, 40, 41])])
def test_single_tokens(D, Hq, Hkv, page, shared, own):
    s = shared_setup(shared + D, shared, own, [1] * len(own), Hq, Hkv, D, page, ragged=False)
    check(s, *run(s))
    assert s.path == "shared_few"


@pytest.mark.parametrize("D,Hq,Hkv,page", [(128, 8, 2, 16), (64, 6, 2, 32), (128, 16, 1, 64)])
@pytest.mark.parametrize("shared,n,own", [(128, 33, [33, 33]), (512, 9, [9, 300, 10]), (300, 65, [65, 66, 300, 129, 70]), (2048, 17, [20, 30, 17])])
def test_windows(D, Hq, Hkv, page, shared, n, own):
    s = shared_setup(shared + n, shared, own, [n] * len(own), Hq, Hkv, D, page, ragged=False)
    check(s, *run(s, with_lse=n != 9))


@pytest.mark.parametrize("G,Hkv,D", [(4, 2, 128), (1, 3, 64), (32, 1, 128), (128, 1, 64), (5, 2, 64)])
def test_ragged_batches_with_sequences_of_their_own(G, Hkv, D):
    """Prompts of any length behind the prefix, none among them, one that is shorter than the prefix, one without new tokens, an empty one."""
    own = [100, 37, 5, 0, 260, 1, 0]
    nq = [100, 30, 5, 0, 200, 1, 0]
    for alone in ((), (1,), (0, 4, 6), (1, 2, 3, 4, 5, 6)):
        s = shared_setup(9 + G, 256, own, nq, G * Hkv, Hkv, D, 32, alone=alone)
        check(s, *run(s))


def test_a_shorter_sequence_under_the_same_table():
    """A sequence whose new tokens lie inside the prefix keeps its causal mask."""
    s = shared_setup(4, 512, [20, 20, 20], [17, 17, 17], 8, 2, 128, 16, ragged=False)
    s.lens[1] = 300
    s.seq_lens[1] = 300
    check(s, *run(s))
    s.lens[2] = s.lens[2] - 5  # three of its tokens are missing from the prefix's end on
    s.lens[2] = 512 + 16
    s.seq_lens[2] = 512 + 16
    check(s, *run(s))


def test_many_sequences():
    rng = np.random.default_rng(0)
    own = rng.integers(1, 90, 150).tolist()
    s = shared_setup(1, 640, own, [1] * 150, 4, 1, 64, 16, ragged=False)
    check(s, *run(s))
    nq = [int(rng.integers(0, n + 1)) for n in own]
    s = shared_setup(2, 640, own, nq, 4, 1, 64, 16)
    check(s, *run(s))


def test_less_room_than_rows():
    """Sequences of a ragged call whose tokens lie past the reserved rows are attended alone."""
    own = nq = [50, 60, 3, 70]
    s = shared_setup(3, 256, own, nq, 8, 2, 128, 16)
    for rows in (1, 50, 109, 110, 112, 113, 183):
        check(s, *run(s, rows=rows))


def test_first_row_of_a_ragged_call():
    """q_start may begin behind rows that are no business of the call."""
    s = shared_setup(5, 256, [40, 30], [33, 30], 8, 2, 128, 16)
    n = 7
    q = torch.full((s.T + n, s.Hq * s.D), float("nan"), dtype=s.dt, device="cuda")
    q[n:] = s.q
    out = torch.full_like(q, 5.0)
    lse = torch.full((s.T + n, s.Hq), 5.0, device="cuda")
    h = s.handle(SHARED)
    for rows in (40, s.T):
        h.reserve_shared(rows)
        h.attend_shared(q, s.k, s.v, s.prefix, s.shared, s.block_table, s.seq_lens, out, s.B, s.max_n, s.scale, q_start=s.q_start + n, lse=lse)
        torch.cuda.synchronize()
        check(s, out[n:], lse[n:])
        assert (out[:n] == 5).all() and (lse[:n] == 5).all()


def test_calls_that_share_nothing():
    """f32, other head sizes, the comparison switch, one sequence, a prefix below a tile: the plain kernels, nothing reserved."""
    for kw, flags in (({"dtype": "f32"}, 0), ({"D": 80}, 0), ({}, SIMT | SHARED), ({"shared": 100}, 0), ({"shared": 0}, 0), ({"one": True}, 0)):
        shared, D = kw.get("shared", 256), kw.get("D", 64)
        own = [20] if kw.get("one") else [20, 30, 40]
        s = shared_setup(6, shared, own, [9] * len(own), 4, 2, D, 16, ragged=False, dtype=kw.get("dtype", "bf16"))
        h = s.handle(flags)
        out, lse = torch.zeros(s.T, s.Hq * D, dtype=s.dt, device="cuda"), torch.zeros(s.T, s.Hq, device="cuda")
        h.attend_shared(s.q, s.k, s.v, s.prefix if shared else None, shared, s.block_table, s.seq_lens, out, s.B, s.max_n, s.scale, lse=lse)
        torch.cuda.synchronize()
        check(s, out, lse)
        assert h.last_launch_count() == 1


def test_queries_off_128_bytes_and_outputs_in_strides():
    s = shared_setup(7, 384, [40, 33, 100], [33] * 3, 8, 2, 128, 16, ragged=False, pad=8)
    h = s.handle(SHARED)
    h.reserve_shared(s.T)
    wide = torch.full((s.T, s.Hq * s.D + 24), 3.0, dtype=s.dt, device="cuda")
    h.attend_shared(s.q, s.k, s.v, s.prefix, s.shared, s.block_table, s.seq_lens, wide[:, : s.Hq * s.D], s.B, s.max_n, s.scale)
    torch.cuda.synchronize()
    check(s, wide[:, : s.Hq * s.D], None)
    assert (wide[:, s.Hq * s.D :] == 3).all()


@pytest.mark.parametrize("n", [1, 17])
def test_scores_that_are_no_numbers(n):
    """A NaN or +infinite score makes its row NaN whichever part it lies in; the other rows keep their numbers."""
    s = shared_setup(8, 256, [30, 40], [n, n], 4, 1, 128, 16, ragged=False)
    want, want_lse = run(s)
    for page, slot, rows in ((int(s.table[0, 3]), 5, range(2 * n)), (int(s.table[1, 16]), 2, range(n, 2 * n))):
        keep = s.k[page, 0, slot].clone()
        for bad in (float("nan"), float("inf")):
            s.k[page, 0, slot] = bad if bad != bad else 0.0
            if bad == bad:
                s.k[page, 0, slot, 0] = bad
                s.q[:, :: s.D] = s.q[:, :: s.D].abs() + 1  # (the product is +infinite)
            out, lse = run(s)
            hit = torch.zeros(2 * n, dtype=torch.bool)
            hit[list(rows)] = True
            assert lse[hit].isnan().all() and out[hit].isnan().all()
            assert not lse[~hit].isnan().any()
        s.k[page, 0, slot] = keep


def test_large_and_small_scores():
    """The maximum lies in the prefix for some rows and behind it for others, far apart."""
    s = shared_setup(12, 256, [60, 60, 60], [20] * 3, 8, 2, 64, 16, ragged=False, q_scale=12.0)
    check(s, *run(s))
    lead = s.table[0, :16]
    s.k[torch.tensor(lead)] *= 1.0 / 64
    check(s, *run(s))


def test_same_bits_every_time():
    s = shared_setup(10, 1280, [200, 77, 300, 64], [33] * 4, 32, 8, 128, 16, ragged=False)
    h = s.handle(SHARED)
    a, al = run(s, handle=h)
    for _ in range(5):
        b, bl = run(s, handle=h)
        assert torch.equal(a, b) and torch.equal(al, bl)


def test_one_handle_for_changing_calls():
    h = aj.KvHandle(0, 6, 40, 8, 2, 128, 16, flags=SHARED)
    for seed, (shared, own, n) in enumerate([(512, [40, 50, 60, 70, 41, 40], 40), (128, [1, 2], 1), (256, [4, 4, 4], 4), (100, [9, 9], 9), (1280, [33] * 5, 33)]):
        s = shared_setup(seed, shared, own, [n] * len(own), 8, 2, 128, 16, ragged=False)
        check(s, *run(s, handle=h))
        out = torch.zeros(s.T, s.Hq * s.D, dtype=s.dt, device="cuda")
        h.attend(s.q, s.k, s.v, s.block_table, s.seq_lens, out, s.B, n, s.scale)
        torch.cuda.synchronize()
        check(s, out, None)


@pytest.mark.parametrize("n", [1, 17])
def test_another_stream_and_a_graph(n):
    s = shared_setup(11, 384, [50, 60, 70], [n] * 3, 8, 2, 128, 16, ragged=False)
    h = s.handle(SHARED)
    h.reserve_shared(s.T)
    out, lse = torch.zeros(s.T, s.Hq * s.D, dtype=s.dt, device="cuda"), torch.zeros(s.T, s.Hq, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        h.attend_shared(s.q, s.k, s.v, s.prefix, s.shared, s.block_table, s.seq_lens, out, s.B, n, s.scale, lse=lse,
                        stream=torch.cuda.current_stream().cuda_stream)
    for seed in (0, 1):
        s.q.copy_(torch.randn(s.q.shape, generator=torch.Generator().manual_seed(seed)) * 2)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        check(s, out, lse)


def test_refusals():
    s = shared_setup(13, 256, [20, 30], [9, 9], 8, 2, 128, 16, ragged=False)
    h = s.handle(SHARED)
    out = torch.zeros(s.T, s.Hq * s.D, dtype=s.dt, device="cuda")

    def status(**kw):
        a = dict(shared_table=s.prefix, shared=256, B=2, n_q=9, scale=s.scale) | kw
        return h.attend_shared(s.q, s.k, s.v, a["shared_table"], a["shared"], s.block_table, s.seq_lens, out, a["B"], a["n_q"], a["scale"], check=False)

    assert status() == aj.AJ_ERR_WORKSPACE  # nothing reserved
    h.reserve_shared(17)
    assert status() == aj.AJ_ERR_WORKSPACE
    h.reserve_shared(18)
    assert status() == aj.AJ_OK
    h.reserve_shared(0)
    assert status() == aj.AJ_ERR_WORKSPACE
    h.reserve_shared(30)
    assert status(shared=-1) == status(shared=s.width * 16 + 1) == status(shared_table=None) == status(scale=0.0) == status(B=0) == aj.AJ_ERR_INVALID_ARG
    assert status(shared_table=s.prefix[:10]) == status(shared_table=s.prefix.long()) == aj.AJ_ERR_INVALID_ARG
    assert status(B=3) == status(n_q=10) == aj.AJ_ERR_WORKSPACE
    assert h.reserve_shared(-1, check=False) == h.reserve_shared(2**30, check=False) == aj.AJ_ERR_INVALID_ARG
    torch.cuda.synchronize()
