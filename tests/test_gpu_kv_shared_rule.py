"""aj_kv_attend_shared attends the shared slots together where that measured clearly faster than one by one, and only there."""
import pytest
import torch

import paper_2504_20039_b200 as aj

pytestmark = pytest.mark.gpu

# query heads, key heads, head size, sequences, new tokens of each, shared slots; us together and one by one (own slots 250 to 300 each)
MEASURED = [
    (32, 8, 128, 64, 1, 2048, 32.4, 80.2), (32, 8, 128, 64, 1, 512, 28.7, 34.5), (32, 8, 128, 2, 1, 32768, 61.1, 48.1), (32, 8, 128, 32, 5, 1024, 40.3, 48.5),
    (32, 8, 128, 32, 9, 2048, 51.5, 70.3), (32, 8, 128, 32, 33, 1504, 86.4, 73.7), (32, 8, 128, 16, 33, 8192, 108.2, 134.1), (32, 8, 128, 16, 128, 1024, 110.3, 58.4),
    (32, 8, 64, 16, 1, 4096, 22.4, 34.0), (32, 8, 64, 2, 1, 32768, 52.6, 33.8), (32, 8, 64, 16, 33, 4096, 63.1, 72.6), (32, 8, 64, 32, 33, 512, 52.9, 41.0),
    (64, 8, 128, 32, 33, 1504, 147.1, 117.8), (64, 8, 128, 32, 33, 2048, 166.2, 141.7), (64, 8, 128, 16, 33, 8192, 188.2, 219.1), (64, 8, 64, 16, 1, 4096, 23.6, 34.1),
    (64, 8, 64, 32, 33, 512, 93.9, 64.2), (16, 16, 64, 16, 1, 4096, 22.5, 56.7), (16, 16, 64, 32, 33, 2048, 66.9, 114.7), (16, 16, 64, 2, 1, 32768, 99.0, 58.0),
    (8, 1, 128, 64, 1, 2048, 30.3, 21.1), (8, 1, 128, 128, 2, 4096, 32.1, 54.3), (14, 2, 64, 64, 1, 2048, 26.6, 21.8), (14, 2, 64, 128, 2, 4096, 34.0, 71.6),
]


@pytest.mark.parametrize("Hq,Hkv,D,B,n,shared,together,one_by_one", MEASURED)
def test_the_faster_way(Hq, Hkv, D, B, n, shared, together, one_by_one):
    assert abs(together - one_by_one) > 0.1 * min(together, one_by_one)
    page, own = 32, 64 * (-(-n // 64) + 1)
    first, each = -(-shared // page), own // page
    table = torch.cat([torch.arange(first).expand(B, first), first + torch.arange(B * each).view(B, each)], 1).int().cuda()
    k, v = (torch.randn(first + B * each, Hkv, page, D, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(B * n, Hq * D, device="cuda").bfloat16()
    lens, out = torch.full((B,), first * page + n, dtype=torch.int32, device="cuda"), torch.empty_like(q)
    h = aj.KvHandle(0, B, n, Hq, Hkv, D, page)
    h.reserve_shared(B * n)
    h.attend_shared(q, k, v, table[0, :first].contiguous(), shared, table, lens, out, B, n, D**-0.5)
    torch.cuda.synchronize()
    assert h.last_path().startswith("shared") == (together < one_by_one)
