"""aj_score_tokens on the CUDA cores with 9 to 32 rows, whose tiles of rows are 16 and 32 high, and around them."""
import pytest

import paper_2504_20039_b200 as aj
from score_testlib import Head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("d,V", [(16, 5), (40, 130), (256, 1000), (264, 3001)])
def test_every_height_of_a_row_tile(d, V, dtype):
    if dtype == "e4m3" and d % 16:
        d += 8
    for rows in (7, 8, 9, 12, 15, 16, 17, 24, 31, 32, 33):
        t = Head(rows + V, rows, d, V, dtype, pad=3 * (rows % 2))
        t.check(t.run(n_top=min(V, 6), flags=aj.AJ_SCORE_FLAG_FORCE_SIMT))
        assert t.path == "simt"
