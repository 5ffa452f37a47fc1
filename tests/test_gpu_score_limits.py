"""The largest widths, heads and numbers of alternatives of aj_score_tokens, a captured call of several groups of rows, and outputs of
aj_add_norm whose rows lie in strides of their own."""
import pytest
import torch

import paper_2504_20039_b200 as aj
from aj_testlib import Guarded
from score_testlib import Head, norm_reference
from test_gpu_norm import check, check8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [3, 130])
def test_the_widest_states(rows, dtype):
    """d = 65536, values on a grid so coarse that every sum is exact: halves and whole numbers of two bits."""
    d, V = 65536, 700
    t = Head(1, rows, 64, V, dtype)
    g = torch.Generator().manual_seed(rows)
    t.d, t.h, t.W = d, torch.randint(-2, 3, (rows, d), generator=g).to(t.h.dtype), (torch.randint(-1, 2, (V, d), generator=g) / 64).to(t.W.dtype)
    t.check(t.run(n_top=32))
    assert t.path.startswith("umma")


@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("e4m3", 16), ("f32", 4)])
@pytest.mark.parametrize("rows", [1, 130])
def test_the_largest_head(rows, dtype, d):
    V = 2**21
    t = Head(2, rows, d, V, dtype)
    t.tokens[0, 0], t.tokens[0, 1] = V - 1, 0
    for n_top in (1, 16, 32):
        t.check(t.run(n_top=n_top))
    with pytest.raises(aj.AjError):
        aj.ScoreHandle(0, 1, d, V + 1, t.aj_dtype)


def test_a_captured_call_of_several_groups():
    rows, d, V = 5200, 64, 600
    h = aj.ScoreHandle(0, rows, d, V, max_top=3)
    t = Head(3, rows, d, V)
    x, W, tok = t.h.cuda(), t.W.cuda(), t.tokens[:, :1].contiguous().cuda()
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    got = {"logprob": f(rows, 1), "lse": f(rows), "entropy": f(rows), "top_id": f(rows, 3).int(), "top_logprob": f(rows, 3)}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        h.score(x, W, tok, stream=torch.cuda.current_stream().cuda_stream, **got)
    assert h.last_launch_count() == 6
    for seed in (4, 5):
        other = Head(seed, rows, d, V)
        x.copy_(other.h)
        W.copy_(other.W)
        tok.copy_(other.tokens[:, :1])
        g.replay()
        torch.cuda.synchronize()
        other.check(got)
    assert h.last_status() == aj.AJ_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,pads", [(4096, (8, 16, 24, 32, 8)), (4096, (0, 0, 0, 0, 4)), (4096, (0, 0, 1, 0, 0)), (300, (1, 2, 3, 4, 5)), (8192, (0, 8, 0, 8, 3)), (64, (4, 4, 4, 4, 8))])
def test_norm_outputs_in_strides(d, pads, dtype):
    dt, rows = torch.bfloat16 if dtype == "bf16" else torch.float32, 41
    g = torch.Generator().manual_seed(d)
    x, r, w = torch.randn(rows, d, generator=g).to(dt), torch.randn(rows, d, generator=g).to(dt), 1 + 0.2 * torch.randn(d, generator=g)
    wide = [Guarded(torch.full((rows, d + p), 9.0).to(torch.uint8 if i == 4 else dt), str(i)) for i, p in enumerate(pads)]
    a, b, r_out, out, out8 = (t.t[:, :d] for t in wide)
    a.copy_(x)
    b.copy_(r)
    out8, sc = out8.view(torch.float8_e4m3fn), torch.zeros(rows, device="cuda")
    aj.add_norm(a, w.cuda(), 1e-5, out=out, residual=b, residual_out=r_out, out8=out8, scale8=sc)
    torch.cuda.synchronize()
    s, y = norm_reference(x, r, w, 1e-5)
    check(out, y, dt, d)
    check8(out8, sc, y)
    assert ((r_out.double().cpu() - s).abs() <= s.abs() * ((2.0**-8 if dtype == "bf16" else 2.0**-24) + 2.0**-24)).all()
    for t, p in zip(wide, pads):
        t.check()
        assert (t.t[:, d:] == 9).all()
