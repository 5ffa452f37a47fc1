"""aj_score_tokens against its definition in 64 bits."""
import pytest
import torch

from score_testlib import Head, tied_order

pytestmark = pytest.mark.gpu


def paths(dtype):
    import paper_2504_20039_b200 as aj

    return [0] if dtype == "f32" else [0, aj.AJ_SCORE_FLAG_FORCE_SIMT]


@pytest.mark.parametrize("dtype", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("rows,d,V,n_top", [(1, 64, 1, 1), (1, 8, 3, 3), (5, 256, 1000, 5), (2, 64, 255, 20), (17, 512, 257, 1), (17, 256, 5000, 32), (3, 64, 8000, 32), (200, 64, 7900, 32), (140, 64, 300000, 32), (33, 72, 3001, 8),
                                            (64, 320, 2048, 5), (96, 128, 4099, 20), (128, 256, 777, 3), (129, 192, 2500, 5), (256, 512, 6001, 8),
                                            (257, 264, 1111, 5), (300, 1024, 20000, 20), (513, 128, 515, 0), (777, 448, 3333, 4)])
def test_sizes(rows, d, V, n_top, dtype):
    if dtype == "e4m3" and d % 16:
        d += 8
    for flags in paths(dtype):
        t = Head(rows + d + V, rows, d, V, dtype)
        inv_t = 1.0 if rows % 2 else 1 / 0.7
        got = t.run(n_top=n_top, n_tok=min(3, rows % 4), inv_t=inv_t, flags=flags)
        t.check(got, inv_t)


@pytest.mark.parametrize("dtype,rows,d,V", [("bf16", 17, 4096, 128256), ("bf16", 264, 2048, 50000), ("e4m3", 17, 4096, 128256), ("e4m3", 300, 4096, 32000),
                                            ("bf16", 128, 8192, 32000), ("f32", 3, 4096, 32000)])
def test_full_heads(dtype, rows, d, V):
    t = Head(11, rows, d, V, dtype, lean=14.0)
    t.check(t.run(n_top=20, inv_t=1 / 0.6), 1 / 0.6)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_values_off_the_grid(dtype):
    """Plain Gaussian values: a logit is off by the roundings of its products' sum."""
    for rows, d, V in ((9, 1024, 3000), (200, 2048, 3000)):
        t = Head(5, rows, d, V, dtype)
        g = torch.Generator().manual_seed(1)
        h, W = torch.randn(rows, d, generator=g), torch.randn(V, d, generator=g) * 0.03
        if dtype == "e4m3":
            t.h_scale, t.w_scale = h.abs().amax(-1) / 448, W.abs().amax(-1) / 448
            h, W = h / t.h_scale[:, None], W / t.w_scale[:, None]
        t.h, t.W = h.to(t.h.dtype), W.to(t.W.dtype)
        mag = (t.h.cuda().double().abs() @ t.W.cuda().double().abs().T)
        if dtype == "e4m3":
            mag = mag * t.h_scale.cuda().double()[:, None] * t.w_scale.cuda().double()
        t.check(t.run(n_top=6), logit_error=mag.amax(-1) * (d + 4) * 2.0**-24)


def test_more_rows_than_a_group():
    t = Head(3, 5200, 64, 600, "bf16")
    got = t.run(n_top=3)
    t.check(got)


def test_fewer_rows_than_the_handle_and_changing_calls():
    import paper_2504_20039_b200 as aj

    V, d = 3000, 256
    h = aj.ScoreHandle(0, 400, d, V, max_top=20)
    for seed, (rows, n_top, n_tok) in enumerate([(400, 20, 3), (1, 5, 1), (130, 0, 2), (20, 1, 0), (399, 7, 3), (5, 20, 1)]):
        t = Head(seed, rows, d, V, pad=8 * (seed % 2))
        t.check(t.run(n_top=n_top, n_tok=n_tok, handle=h, lse=seed % 2 == 0, entropy=seed % 3 == 0, top_lp=seed != 4))
    h.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
def test_rows_off_16_bytes(dtype):
    t = Head(8, 40, 256, 2000, dtype, pad=3)
    t.check(t.run())
    assert t.path == "simt"


@pytest.mark.parametrize("rows", [4, 140])
def test_equal_logits(rows):
    """Copies of an entry far apart, a head of copies, and logits that are zeros of either sign: the lowest entries come first."""
    t = Head(2, rows, 128, 5000)
    t.W[[7, 900, 901, 4999, 2600]] = t.W[3].clone()
    t.check(t.run(n_top=10))
    t.W[:] = t.W[0].clone()
    got = t.run(n_top=20)
    assert torch.equal(got["top_id"].cpu(), torch.arange(20, dtype=torch.int32).expand(rows, 20))
    assert torch.allclose(got["entropy"].cpu(), torch.full((rows,), 8.517193191), atol=2e-5, rtol=0)
    t.h[:] = 0.0
    t.h[1] = -0.0
    t.check(t.run(n_top=20))


@pytest.mark.parametrize("rows", [3, 140])
@pytest.mark.parametrize("order", ["rising", "falling", "one far above", "all but one far below"])
def test_orders_of_logits(rows, order):
    """Sorted logits, where every tile beats the ones before it or none does, and rows with almost all weight on one entry."""
    V, d = 6000, 64
    t = Head(4, rows, d, V)
    t.h[:] = 0.0
    t.h[:, 0] = 1.0
    t.h[:, 1] = 4.0
    x = torch.arange(V)
    if order == "falling":
        x = V - 1 - x
    t.W[:] = 0.0
    t.W[:, 0], t.W[:, 1] = (x % 64).float() / 64, (x // 64).float() / 4
    if order == "one far above":
        t.W[:, 1] = 0.0
        t.W[4321, 1] = 30.0
    if order == "all but one far below":
        t.W[:, 1] = -100.0
        t.W[77, 1] = 0.0
    got = t.run(n_top=12)
    t.check(got)


def test_tokens_outside_and_rows_without_numbers():
    for rows in (6, 150):
        t = Head(6, rows, 128, 3000)
        good = tied_order(t.logits())[:, :4]
        t.tokens[0, 0], t.tokens[1, 0], t.tokens[2, 1] = -1, 3000, 2**31 - 1
        t.h[3, 5] = float("nan")
        t.h[4, 7] = float("inf")
        got = t.run(n_top=4)
        lp = got["logprob"].cpu()
        assert lp[0, 0].isnan() and lp[1, 0].isnan() and lp[2, 1].isnan() and not lp[0, 1:].isnan().any() and not lp[1, 1:].isnan().any()
        for r in (3, 4):
            assert lp[r].isnan().all() and got["lse"][r].isnan() and got["entropy"][r].isnan() and got["top_logprob"][r].isnan().all()
        ids = got["top_id"]
        assert (ids >= 0).all() and (ids < 3000).all()
        keep = [i for i in range(rows) if i not in (3, 4)]
        assert torch.equal(ids.long()[keep], good[keep])
        # a NaN in an entry reaches every row
        t = Head(6, rows, 128, 3000)
        t.W[2900, 3] = float("nan")
        got = t.run(n_top=4)
        assert got["lse"].isnan().all() and got["top_logprob"].isnan().all() and (got["top_id"] >= 0).all() and (got["top_id"] < 3000).all()


def test_scales_of_any_sign_and_size():
    t = Head(9, 30, 256, 2000, "e4m3")
    t.w_scale[::3] *= -1
    t.w_scale[5] = 0.0
    t.h_scale[2] = 0.0
    t.h_scale[3] *= -4
    t.check(t.run(n_top=8))


def test_same_bits_every_time():
    for rows in (20, 300):
        t = Head(7, rows, 512, 9000)
        a, b = t.run(n_top=9), t.run(n_top=9)
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_a_row_does_not_depend_on_its_neighbours():
    t = Head(7, 256, 512, 9000)
    a = t.run(n_top=9)
    t.rows, t.h, t.tokens = 20, t.h[:20], t.tokens[:20]
    b = t.run(n_top=9)
    assert torch.equal(a["top_id"][:20], b["top_id"])


def test_no_rows():
    import paper_2504_20039_b200 as aj

    h = aj.ScoreHandle(0, 4, 64, 100, max_top=2)
    e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    assert h.score(e(0, 64, dt=torch.bfloat16), e(100, 64, dt=torch.bfloat16), e(0, 1, dt=torch.int32), e(0, 1)) == aj.AJ_OK
    assert h.last_launch_count() == 0


@pytest.mark.parametrize("rows", [17, 200])
def test_another_stream_and_a_graph(rows):
    import paper_2504_20039_b200 as aj

    t = Head(1, rows, 256, 5000)
    h = aj.ScoreHandle(0, rows, 256, 5000, max_top=5)
    W, x, tok = t.W.cuda(), t.h.cuda(), t.tokens[:, :1].contiguous().cuda()
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    got = {"logprob": f(rows, 1), "lse": f(rows), "entropy": f(rows), "top_id": f(rows, 5).int(), "top_logprob": f(rows, 5)}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        h.score(x, W, tok, stream=torch.cuda.current_stream().cuda_stream, **got)
    for seed in (2, 3, 4):
        other = Head(seed, rows, 256, 5000)
        x.copy_(other.h)
        W.copy_(other.W)
        tok.copy_(other.tokens[:, :1])
        g.replay()
        torch.cuda.synchronize()
        other.check(got)
    assert h.last_status() == aj.AJ_OK
