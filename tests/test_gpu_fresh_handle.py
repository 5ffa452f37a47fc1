"""A verification handle that has just been made serves any stream."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu


def test_a_fresh_handle_does_not_lean_on_the_default_stream():
    """Creation leaves nothing of its own behind work that is queued on the default stream: the keys of a fresh handle are zero for a
    stream that does not wait for it, whatever their memory held before (a key there would win against every logit)."""
    import torch

    import paper_2504_20039_b200 as aj

    B, K, d, dd, V = 4, 7, 128, 64, 1000
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    ht, hd, W = r(B, K + 1, d), r(B, K + 1, dd), r(V, d)
    w = torch.randn(d + dd, generator=g).cuda()
    tok = torch.randint(0, V, (B, K), generator=g, dtype=torch.int32).cuda()

    def outputs():
        return [torch.full(s, -7, dtype=torch.int32, device="cuda") for s in ((B,), (B,), (B, K + 1))]

    def cycle(h, o, stream):
        h.verify(ht, hd, W, tok, w, 0.0, 0.5, B, K, o[0], o[1], o[2], stream=stream)

    warm = aj.Handle(0, B, K, d, dd, V)
    want, got = outputs(), outputs()
    cycle(warm, want, 0)
    torch.cuda.synchronize()
    assert torch.equal(want[2].long(), (ht.float() @ W.float().T).argmax(-1))

    # small pieces of device memory full of ones, every other one given back
    rt = ctypes.CDLL("libcudart.so.12")
    held = []
    for i in range(2048):
        x, n = ctypes.c_void_p(), 256 if i % 4 < 2 else 512
        assert rt.cudaMalloc(ctypes.byref(x), n) == 0 and rt.cudaMemset(x, 0xFF, n) == 0
        held.append(x)
    torch.cuda.synchronize()
    for x in held[::2]:
        assert rt.cudaFree(x) == 0
    side = torch.cuda.Stream()
    torch.cuda._sleep(400_000_000)
    busy = torch.cuda.Event()
    busy.record()
    h = aj.Handle(0, B, K, d, dd, V)
    cycle(h, got, side.cuda_stream)
    side.synchronize()
    queued = not busy.query()
    torch.cuda.synchronize()
    for x in held[1::2]:
        assert rt.cudaFree(x) == 0
    assert h.last_status() == aj.AJ_OK
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert queued, "the side stream did not run beside the default stream: nothing was tested"
