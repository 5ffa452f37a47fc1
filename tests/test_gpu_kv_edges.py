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
