"""aj_add_norm against its definition in 64 bits."""
import pytest
import torch

from aj_testlib import Guarded
from score_testlib import norm_reference

pytestmark = pytest.mark.gpu
U = 2.0**-24


def inputs(seed, rows, d, dt, pads=(0, 0, 0, 0)):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, d + pads[0], generator=g) * torch.where(torch.rand(rows, 1, generator=g) < 0.3, 100.0, 1.0)
    r = torch.randn(rows, d + pads[1], generator=g) * 3
    w = 1 + 0.2 * torch.randn(d, generator=g)
    return x.to(dt), r.to(dt), w


def check(got, ref, dt, d):
    # the sum: one rounding; the square sum: 32 products a thread and trees, at most 64 roundings, halved by the root; division, root
    # and two products: 8 more
    err = (got.double().cpu() - ref).abs()
    tol = ref.abs() * ((2.0**-8 if dt is torch.bfloat16 else U) + 48 * U) + 1e-37
    assert (err <= tol).all(), float((err / tol).max())


def check8(out8, scale8, ref):
    top = ref.abs().amax(-1)
    assert ((scale8.double().cpu() - top / 448).abs() <= top / 448 * 64 * U).all()
    v = torch.where(top[:, None] > 0, ref / top[:, None].clamp_min(1e-300) * 448, torch.zeros_like(ref))
    # half a step: 2^-4 of the value, 2^-10 below the smallest normal one (2^-6)
    tol = (v.abs() * 2.0**-4).clamp_min(2.0**-10) + v.abs() * 128 * U
    assert ((out8.float().double().cpu() - v).abs() <= tol).all()
    assert (out8.float().abs().amax(-1).cpu()[top > 0] == 448).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (1, 8), (130, 64), (5, 250), (33, 256), (9, 264), (7, 1000), (17, 2048), (4, 2050), (3, 4096), (2112, 4096),
                                    (5, 5000), (300, 8192), (2, 8200), (2, 16384), (3, 20001), (2, 32768)])
def test_sizes(rows, d, dtype):
    import paper_2504_20039_b200 as aj

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, r, w = inputs(rows * 31 + d, rows, d, dt)
    s, y = norm_reference(x, r, w, 1e-5)
    gs = [Guarded(t, n) for t, n in ((x, "x"), (r, "r"), (w, "w"), (torch.zeros_like(x), "r_out"), (torch.zeros_like(x), "out"),
                                     (torch.zeros(rows, d, dtype=torch.uint8), "out8"), (torch.zeros(rows), "scale8"))]
    gx, gr, gw, r_out, out, out8, scale8 = (g.t for g in gs)
    out8 = out8.view(torch.float8_e4m3fn)
    aj.add_norm(gx, gw, 1e-5, out=out, residual=gr, residual_out=r_out, out8=out8, scale8=scale8)
    torch.cuda.synchronize()
    for g in gs:
        g.check()
    assert ((r_out.double().cpu() - s).abs() <= s.abs() * (2.0**-8 if dtype == "bf16" else U) + (s.abs() * U)).all()
    check(out, y, dt, d)
    check8(out8, scale8, y)
    # each output alone gives the same bits
    only = torch.zeros_like(out)
    aj.add_norm(gx, gw, 1e-5, out=only, residual=gr)
    only8, only_s = torch.zeros_like(out8), torch.zeros_like(scale8)
    aj.add_norm(gx, gw, 1e-5, residual=gr, out8=only8, scale8=only_s)
    assert torch.equal(only, out) and torch.equal(only8.view(torch.uint8), out8.view(torch.uint8)) and torch.equal(only_s, scale8)


@pytest.mark.parametrize("d", [64, 4096, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_residual_strided_and_in_place(d, dtype):
    import paper_2504_20039_b200 as aj

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for pad in (8, 3):  # rows on 16 bytes, and off them
        x, r, w = inputs(d + pad, 37, d, dt, (pad, pad, 0, 0))
        gx, gr = Guarded(x, "x"), Guarded(r, "r")
        a, b = gx.t[:, :d], gr.t[:, :d]
        s, y = norm_reference(x[:, :d], r[:, :d], w, 1e-6)
        _, y0 = norm_reference(x[:, :d], None, w, 1e-6)
        out = torch.zeros(37, d, dtype=dt, device="cuda")
        aj.add_norm(a, w.cuda(), 1e-6, out=out)
        check(out, y0, dt, d)
        assert torch.equal(a.cpu(), x[:, :d])
        aj.add_norm(a, w.cuda(), 1e-6, out=a, residual=b, residual_out=b)  # both in place
        check(a, y, dt, d)
        assert ((b.double().cpu() - s).abs() <= s.abs() * ((2.0**-8 if dtype == "bf16" else U) + U)).all()
        if pad:
            assert torch.equal(gx.t[:, d:].cpu(), x[:, d:]) and torch.equal(gr.t[:, d:].cpu(), r[:, d:])
        gx.check()
        gr.check()


def test_rows_without_numbers():
    import paper_2504_20039_b200 as aj

    d = 4096
    x = torch.randn(6, d)
    x[1] = 0.0
    x[2, 100] = float("nan")
    x[3, 5] = float("inf")
    x[4] = 1e-30  # eps decides
    out, out8, sc = torch.zeros(6, d, device="cuda"), torch.zeros(6, d, device="cuda").to(torch.float8_e4m3fn), torch.zeros(6, device="cuda")
    w = torch.ones(d)
    aj.add_norm(x.cuda(), w.cuda(), 1e-5, out=out, out8=out8, scale8=sc)
    _, y = norm_reference(x, None, w, 1e-5)
    for i in (0, 4, 5):
        check(out[i : i + 1], y[i : i + 1], torch.float32, d)
    check8(out8[[0, 4, 5]], sc[[0, 4, 5]], y[[0, 4, 5]])
    assert not out[1].any() and sc[1] == 0 and not out8[1].float().any()
    assert out[2].isnan().all() and sc[2].isnan()
    assert out[3, 5].isnan() and sc[3].isnan()


def test_another_stream_and_a_graph():
    import paper_2504_20039_b200 as aj

    x, r, w = (t.cuda() for t in inputs(3, 64, 4096, torch.bfloat16))
    out, out8, sc = torch.zeros_like(x), torch.zeros(64, 4096, device="cuda").to(torch.float8_e4m3fn), torch.zeros(64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        aj.add_norm(x, w, out=out, residual=r, out8=out8, scale8=sc, stream=torch.cuda.current_stream().cuda_stream)
    for seed in (4, 5):
        x2, r2, _ = inputs(seed, 64, 4096, torch.bfloat16)
        x.copy_(x2)
        r.copy_(r2)
        g.replay()
        torch.cuda.synchronize()
        _, y = norm_reference(x2, r2, w.cpu(), 1e-5)
        check(out, y, torch.bfloat16, 4096)
        check8(out8, sc, y)
