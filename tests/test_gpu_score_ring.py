"""aj_score_tokens where the ring of stages comes round to its last one several times, with few rows staged per k-block: narrow tiles of a
small head or of one whose tiles take turns on an SM, widths of an even and an odd number of k-blocks."""
import pytest

from score_testlib import Head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("V,d", [(3000, 2048), (4096, 4096), (4736, 2112), (50257, 2048)])
def test_the_ring_goes_round(V, d, dtype):
    for rows in (1, 9, 25, 31, 32, 33, 96):
        t = Head(rows + V, rows, d, V, dtype)
        t.check(t.run(n_top=6, n_tok=1))
        assert t.path == "umma_one_sm"
