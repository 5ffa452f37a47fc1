"""ScoreHandle refuses tensors that do not fit, before anything reaches the library (a handle without a device, fake tensors)."""
import struct

import pytest
import torch


class Fake:
    """A tensor that claims to lie on a device."""

    def __init__(self, *shape, dtype=torch.float32, device=0, stride=None, contiguous=True):
        self.shape, self.dtype, self._device, self._c = torch.Size(shape), dtype, device, contiguous
        s, n = [], 1
        for x in reversed(shape):
            s.insert(0, n)
            n *= x
        self._s = tuple(stride or s)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self._s

    def get_device(self):
        return self._device

    def is_contiguous(self):
        return self._c

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def handle():
    import paper_2504_20039_b200 as aj

    h = aj.ScoreHandle.__new__(aj.ScoreHandle)
    h._h, h._device, h._d, h._V = None, 0, 64, 1000
    h._dtype = torch.bfloat16
    from paper_2504_20039_b200 import score

    score._lib()
    h.calls = []
    h._score = lambda *a: h.calls.append(a) or 0
    return h


def test_what_is_passed_on(handle):
    B, i32 = torch.bfloat16, torch.int32
    ok = dict(h=Fake(6, 64, dtype=B), W=Fake(1000, 64, dtype=B), tokens=Fake(6, 2, dtype=i32), logprob=Fake(6, 2), lse=Fake(6), entropy=Fake(6),
              top_id=Fake(6, 5, dtype=i32), top_logprob=Fake(6, 5))
    assert handle.score(**ok) == 0
    fields = lambda: struct.unpack("9qd6q", handle.calls[-1][1])  # noqa: E731
    assert fields() == (1 << 20, 64, 0, 1 << 20, 0, 1 << 20, 2, 6, 5, 1.0, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 0)
    assert handle.score(**(ok | {"h": Fake(6, 64, dtype=B, stride=(80, 1)), "lse": None, "stream": 77})) == 0
    assert fields()[1] == 80 and fields()[11] == 0 and fields()[15] == 77
    n = len(handle.calls)
    bad = [{"h": Fake(6, 63, dtype=B)}, {"h": Fake(6, 64)}, {"h": Fake(6, 64, dtype=B, device=1)}, {"h": Fake(6, 64, dtype=B, stride=(64, 2))}, {"h": Fake(64, dtype=B)},
           {"W": Fake(999, 64, dtype=B)}, {"W": Fake(1000, 64, dtype=B, contiguous=False)}, {"W": Fake(1000, 64)}, {"tokens": Fake(6, 2, dtype=torch.int64)},
           {"tokens": Fake(6, dtype=i32)}, {"tokens": Fake(5, 2, dtype=i32)}, {"logprob": Fake(6, 3)}, {"logprob": Fake(6, 2, dtype=B)}, {"lse": Fake(5)},
           {"entropy": Fake(6, dtype=torch.float64)}, {"top_id": Fake(6, 5)}, {"top_id": Fake(6, 5, dtype=i32, contiguous=False)}, {"top_logprob": Fake(6, 4)},
           {"h_scale": Fake(5)}, {"w_scale": Fake(6)}, {"lse": Fake(6, device=1)}]
    for b in bad:
        assert handle.score(**(ok | b), check=False) == 1, b
    assert len(handle.calls) == n
