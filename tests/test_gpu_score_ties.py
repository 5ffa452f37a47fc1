"""aj_score_tokens where many entries have the same logit: which of them come first, and what such rows cost."""
import pytest
import torch

import paper_2504_20039_b200 as aj
from score_testlib import Head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 140])
@pytest.mark.parametrize("V,n_top", [(700, 32), (5000, 1), (5000, 9), (5000, 16), (5000, 17), (9000, 32)])
def test_entries_above_many_equal_ones(V, n_top, rows, dtype):
    """A few different entries first, then hundreds of equal ones in any places, the lowest of which fill the rest."""
    t = Head(V + n_top, rows, 64, V, dtype)
    g = torch.Generator().manual_seed(1)
    t.h[:], t.W[:] = 0.0, 0.0
    t.h[:, 0] = 1.0
    t.h[1] = -0.0  # a row of zeros: every entry equal
    some = torch.randperm(V, generator=g)[: V // 2]
    t.W[some, 0] = 2.0
    for above in (0, 1, n_top // 2, n_top - 1):
        t.W[some[:above], 0] = 2.0 + torch.arange(1, above + 1).to(t.W.dtype) / 8
        t.check(t.run(n_top=n_top))


def elapsed(call):
    for _ in range(3):
        call()
    best = 1e9
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(4):
            call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("rows,V,n_top", [(64, 128256, 20), (256, 32000, 32), (256, 32000, 8)])
def test_rows_of_zeros_cost_little_more(rows, V, n_top):
    """A padded batch has them.  (Two to three times an ordinary row's time; counting through all equal entries took 15 to 60 times.)"""
    d = 256
    h = aj.ScoreHandle(0, rows, d, V, max_top=n_top)
    W, x = torch.randn(V, d, device="cuda").mul(0.02).bfloat16(), torch.randn(rows, d, device="cuda").bfloat16()
    ids, zeros = torch.zeros(rows, n_top, device="cuda", dtype=torch.int32), torch.zeros_like(x)
    ordinary, equal = elapsed(lambda: h.score(x, W, top_id=ids)), elapsed(lambda: h.score(zeros, W, top_id=ids))
    assert torch.equal(ids.cpu(), torch.arange(n_top, dtype=torch.int32).expand(rows, n_top))
    assert equal < 6 * ordinary, (equal, ordinary)
