"""aj_kv_attend_shared where the shared slots end inside a tile: only a sequence with all of them before its new tokens shares any."""
import pytest

from test_gpu_kv_shared import check, run, shared_setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 17])
@pytest.mark.parametrize("shared", [200, 255, 300])
def test_a_sequence_of_its_own_as_long_as_the_whole_tiles(shared, n):
    """Other tokens under another table, with as many slots as the shared tiles but fewer than `shared` before the new tokens."""
    whole = shared // 128 * 128
    for before in (whole, whole + 1, (whole + shared) // 2, shared - 1):
        s = shared_setup(shared + n, shared, [n + 20, before + n, n, n + 90], [n] * 4, 8, 2, 128, 16, alone=(1,), ragged=False)
        assert s.lens[1] - n == before
        check(s, *run(s))
        s = shared_setup(shared + n, shared, [n + 20, before + n, n, n + 90], [n, n, 0, n], 8, 2, 64, 16, alone=(1,))
        check(s, *run(s))


@pytest.mark.parametrize("n", [1, 17])
def test_the_first_length_that_shares(n):
    """New tokens right behind the last shared slot, one token short of it, and beginning inside the shared tiles, under one table."""
    s = shared_setup(7 + n, 300, [n + 20, n + 1, n, n + 90, n], [n] * 5, 8, 2, 128, 16, ragged=False)
    for b, length in ((2, 299 + n), (4, 255 + n)):
        s.lens[b] = length
        s.seq_lens[b] = length
    check(s, *run(s))
