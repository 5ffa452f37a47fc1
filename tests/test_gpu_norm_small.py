"""aj_add_norm to 8 bits where a row's values, or its scale, lie near the end of f32's range."""
import pytest
import torch

from score_testlib import norm_reference

pytestmark = pytest.mark.gpu
U = 2.0**-24


def check8_against_its_scale(out8, scale8, ref):
    """scale8 = max |y| / 448 and out8 = y / scale8, each as exact as f32 is there."""
    scale8, got = scale8.double().cpu(), out8.float().double().cpu()
    top = ref.abs().amax(-1)
    tiny = 2.0**-150  # half of f32's last step below 2^-126
    # y: 64 roundings, and two products below 2^-126, the first times a weight of at most 1.2; the scale's own rounding
    assert ((scale8 - top / 448).abs() <= top / 448 * 64 * U + 2.2 * tiny / 448 + tiny).all()
    some = scale8 > 0
    assert not got[~some].any()
    v = (ref[some] / scale8[some, None]).clamp(-448, 448)
    # half a step of e4m3: 2^-4 of the value, 2^-10 below the smallest normal one
    tol = (v.abs() * 2.0**-4).clamp_min(2.0**-10) + v.abs() * 128 * U + 2.2 * tiny / scale8[some, None]
    assert ((got[some] - v).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 300, 4096, 9000])
def test_small_rows_to_8_bits(d, dtype):
    """Rows of 1e-44 to 1 under eps = 1e-5, zeros among their values."""
    import paper_2504_20039_b200 as aj

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(d)
    size = torch.cat([torch.logspace(-44, 0, 89), torch.logspace(-39.2, -38.2, 41)])  # (the second half: largest values around 448 / FLT_MAX)
    x = (torch.randn(len(size), d, generator=g).clamp(-2, 2) * size[:, None]).to(dt)
    x[:, ::5] = 0.0
    w = 1 + 0.2 * torch.rand(d, generator=g)
    out8, sc = torch.zeros(len(size), d, device="cuda").to(torch.float8_e4m3fn), torch.full((len(size),), 9.0, device="cuda")
    aj.add_norm(x.cuda(), w.cuda(), 1e-5, out8=out8, scale8=sc)
    check8_against_its_scale(out8, sc, norm_reference(x, None, w, 1e-5)[1])


@pytest.mark.parametrize("w_size", [1e-35, 1e-36, 1e-37, 1e-39, 1e-42, 1e-43, 1e-45])
def test_small_weights_to_8_bits(w_size):
    import paper_2504_20039_b200 as aj

    g = torch.Generator().manual_seed(1)
    x = torch.randn(20, 512, generator=g)
    x[:, ::5] = 0.0
    w = torch.rand(512, generator=g) * w_size
    out8, sc = torch.zeros(20, 512, device="cuda").to(torch.float8_e4m3fn), torch.full((20,), 9.0, device="cuda")
    aj.add_norm(x.cuda(), w.cuda(), 1e-5, out8=out8, scale8=sc)
    check8_against_its_scale(out8, sc, norm_reference(x, None, w, 1e-5)[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 300, 4096])
def test_rows_of_zeros_under_any_eps(d, dtype):
    """Zeros and scale 0, with eps = 0 too; the rows beside them keep their numbers."""
    import paper_2504_20039_b200 as aj

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn(5, d, generator=torch.Generator().manual_seed(d)).to(dt)
    x[1], x[3] = 0.0, -0.0
    w = torch.ones(d)
    for eps in (0.0, 1e-30, 1e-5):
        out, out8, sc = torch.full((5, d), 7.0, dtype=dt, device="cuda"), torch.ones(5, d, device="cuda").to(torch.float8_e4m3fn), torch.full((5,), 9.0, device="cuda")
        aj.add_norm(x.cuda(), w.cuda(), eps, out=out, out8=out8, scale8=sc)
        for i in (1, 3):
            assert not out[i].any() and not out[i].isnan().any() and sc[i] == 0 and not out8[i].float().any() and not out8[i].float().isnan().any()
        y = norm_reference(x[::2], None, w, eps)[1]
        check8_against_its_scale(out8[::2], sc[::2], y)
        # 64 roundings and the last one
        assert ((out[::2].double().cpu() - y).abs() <= y.abs() * ((2.0**-8 if dtype == "bf16" else U) + 64 * U)).all()
