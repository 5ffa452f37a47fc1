"""Calls of the norm, the scores and the shared attention that the documentation allows and the other tests do not make: two handles
at once, a captured pair on one workspace, extreme temperatures, many tokens, offsets past 32 bits, no rows."""
import math

import pytest
import torch

import paper_2504_20039_b200 as aj
from score_testlib import Head, norm_reference
from test_gpu_kv_shared import SHARED, check, shared_setup

pytestmark = pytest.mark.gpu


def outputs(rows, n_tok, n_top):
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    return {"logprob": f(rows, n_tok), "lse": f(rows), "entropy": f(rows), "top_id": f(rows, n_top).int(), "top_logprob": f(rows, n_top)}


def test_two_handles_on_two_streams():
    """Their launches overlap; each has its own workspace."""
    work = []
    for seed, rows in ((1, 20), (2, 300)):
        t = Head(seed, rows, 512, 9000)
        work.append((t, aj.ScoreHandle(0, rows, 512, 9000, max_top=5), t.h.cuda(), t.W.cuda(), t.tokens[:, :2].contiguous().cuda(), outputs(rows, 2, 5), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for t, h, x, W, tok, got, s in work:
            h.score(x, W, tok, stream=s.cuda_stream, **got)
    torch.cuda.synchronize()
    for t, h, x, W, tok, got, s in work:
        assert h.last_status() == aj.AJ_OK
        t.check(got)


def test_two_shared_handles_on_two_streams():
    work = []
    for seed, n in ((1, 1), (2, 17)):
        s = shared_setup(seed, 384, [50, 60, 70, 40], [n] * 4, 8, 2, 128, 16, ragged=False)
        h = s.handle(SHARED)
        h.reserve_shared(s.T)
        work.append((s, h, torch.zeros(s.T, s.Hq * s.D, dtype=s.dt, device="cuda"), torch.zeros(s.T, s.Hq, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, h, out, lse, st in work:
            h.attend_shared(s.q, s.k, s.v, s.prefix, s.shared, s.block_table, s.seq_lens, out, s.B, s.max_n, s.scale, lse=lse, stream=st.cuda_stream)
    torch.cuda.synchronize()
    for s, h, out, lse, st in work:
        assert h.last_status() == aj.AJ_OK
        check(s, out, lse)


def test_two_captured_calls_share_a_workspace():
    """Two graphs of one handle, of different sizes, replayed in turn on one stream."""
    h = aj.ScoreHandle(0, 400, 256, 5000, max_top=20)
    side = torch.cuda.Stream()
    graphs = []
    for seed, (rows, n_top) in enumerate(((400, 5), (17, 20), (130, 1))):
        t = Head(seed, rows, 256, 5000)
        x, W, tok, got = t.h.cuda(), t.W.cuda(), t.tokens[:, :1].contiguous().cuda(), outputs(rows, 1, n_top)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            h.score(x, W, tok, stream=torch.cuda.current_stream().cuda_stream, **got)
        graphs.append((t, g, got, x, W, tok))
    for _ in range(3):
        for _, g, got, *_ in graphs:
            for k in got:
                got[k].zero_()
            g.replay()
    torch.cuda.synchronize()
    for t, _, got, *_ in graphs:
        t.check(got)

    s1, s2 = (shared_setup(seed, 384, [50, 60, 70], [n] * 3, 8, 2, 128, 16, ragged=False) for seed, n in ((3, 1), (4, 17)))
    h = aj.KvHandle(0, 3, 17, 8, 2, 128, 16, flags=SHARED)
    h.reserve_shared(51)
    graphs = []
    for s in (s1, s2):
        out, lse = torch.zeros(s.T, s.Hq * s.D, dtype=s.dt, device="cuda"), torch.zeros(s.T, s.Hq, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            h.attend_shared(s.q, s.k, s.v, s.prefix, s.shared, s.block_table, s.seq_lens, out, s.B, s.max_n, s.scale, lse=lse,
                            stream=torch.cuda.current_stream().cuda_stream)
        graphs.append((s, g, out, lse))
    for _ in range(3):
        for s, g, out, lse in graphs:
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            check(s, out, lse)


@pytest.mark.parametrize("rows", [6, 140])
def test_extreme_temperatures(rows):
    t = Head(3, rows, 128, 4000)
    x = t.logits()
    got = t.run(n_top=3, inv_t=1e-9)  # nothing is left of the logits
    assert torch.allclose(got["entropy"], torch.full_like(got["entropy"], math.log(4000)), atol=1e-5, rtol=0)
    assert torch.equal(got["top_id"].long(), x.sort(dim=-1, descending=True, stable=True).indices[:, :3])
    got = t.run(n_top=3, inv_t=1e6)  # one entry has all the weight, or those that share the largest logit
    top = x.amax(-1)
    ties = (x == top[:, None]).sum(-1).double()
    assert ((got["entropy"].double() - ties.log()).abs() <= 1e-6).all()
    assert ((got["top_logprob"][:, 0].double() + ties.log()).abs() <= 1e-6).all()
    ref = (x.gather(1, got["top_id"].long()) - top[:, None]) * 1e6 - ties.log()[:, None]
    assert ((got["top_logprob"].double() - ref).abs() <= ref.abs() * 2.0**-21 + 1e-6).all()


@pytest.mark.parametrize("rows,n_tok", [(5, 300), (5, 1024), (150, 9), (150, 8)])
def test_many_tokens_per_row(rows, n_tok):
    t = Head(5, rows, 128, 3000)
    t.tokens = torch.randint(3000, (rows, n_tok), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    t.tokens[:, -1] = t.tokens[:, 0]  # the same token twice
    t.check(t.run(n_top=4, n_tok=n_tok))


def test_refusals_of_a_handle():
    h = aj.ScoreHandle(0, 10, 64, 100, max_top=5)
    x, W = torch.zeros(11, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(100, 64, dtype=torch.bfloat16, device="cuda")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    assert h.score(x, W, check=False) == aj.AJ_ERR_WORKSPACE
    assert h.score(x[:10], W, top_id=i(10, 6), check=False) == aj.AJ_ERR_WORKSPACE
    for kw in ({"inv_temperature": 0.0}, {"inv_temperature": -1.0}, {"inv_temperature": float("nan")}, {"inv_temperature": float("inf")}, {"tokens": i(10, 2)},
               {"logprob": f(10, 2)}, {"top_logprob": f(10, 2)}, {"h_scale": f(10), "w_scale": f(100)}, {"tokens": i(10, 1025), "logprob": f(10, 1025)}):
        assert h.score(x[:10], W, check=False, **kw) == aj.AJ_ERR_INVALID_ARG, kw
    with pytest.raises(aj.AjError):
        h.score(x[:10].float(), W)
    assert h.score(x[:10], W, lse=f(10)) == aj.AJ_OK
    e = aj.ScoreHandle(0, 10, 64, 100, aj.AJ_E4M3, max_top=5)
    x8, W8 = x[:10].to(torch.float8_e4m3fn), W.to(torch.float8_e4m3fn)
    assert e.score(x8, W8, check=False) == e.score(x8, W8, h_scale=f(10), check=False) == e.score(x8, W8, w_scale=f(100), check=False) == aj.AJ_ERR_INVALID_ARG
    assert e.score(x8, W8, h_scale=f(10), w_scale=f(100)) == aj.AJ_OK
    torch.cuda.synchronize()


def test_norm_of_no_rows_and_of_one_place_twice():
    x, w = torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(64, device="cuda")
    assert aj.add_norm(x, w, out=torch.empty_like(x)) == aj.AJ_OK
    y = torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")
    assert aj.add_norm(y, w, out=y, residual=y.clone(), residual_out=y, check=False) == aj.AJ_ERR_INVALID_ARG
    assert aj.add_norm(y, w, check=False) == aj.AJ_ERR_INVALID_ARG
    for bad in ({"out": y[None]}, {"out": y[0]}, {"out": y.t().contiguous().t()}, {"out": y.cpu()}, {"out": y.float()}, {"out": y, "residual": y[:2]}, {"out8": y}):
        assert aj.add_norm(y, w, check=False, **bad) == aj.AJ_ERR_INVALID_ARG, bad


def test_norm_offsets_past_32_bits():
    rows, d = 270000, 8192  # 2.2e9 elements
    x = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    w = torch.ones(d, device="cuda")
    out8, sc = torch.zeros(rows, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), torch.zeros(rows, device="cuda")
    at = torch.tensor([0, 131071, 262143, 262144, 262145, rows - 1], device="cuda")
    before = x[at].cpu()
    aj.add_norm(x, w, 1e-5, out=x, out8=out8, scale8=sc)  # in place
    torch.cuda.synchronize()
    _, y = norm_reference(before, None, w.cpu(), 1e-5)
    assert ((x[at].cpu().double() - y).abs() <= y.abs() * (2.0**-8 + 2.0**-18)).all()
    back = out8.view(torch.uint8)[at].view(torch.float8_e4m3fn).float().cpu().double() * sc[at].cpu().double()[:, None]
    assert ((back - y).abs() <= y.abs() * (2.0**-4 + 2.0**-16) + sc[at].cpu().double()[:, None] * 2.0**-10).all()


def test_a_head_whose_offsets_pass_32_bits():
    V, d = 600000, 4096  # 2.5e9 elements
    g = torch.Generator(device="cuda").manual_seed(2)
    W = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    for v in range(0, V, 50000):
        W[v : v + 50000] = torch.randn(50000, d, generator=g, device="cuda").mul_(41).round_().clamp_(-127, 127).mul_(2.0**-11).bfloat16()
    for rows in (3, 140):
        x = torch.randn(rows, d, generator=g, device="cuda").mul_(16).round_().clamp_(-127, 127).div_(16).bfloat16()
        logits = torch.cat([x.double() @ W[v : v + 20000].double().T for v in range(0, V, 20000)], 1)
        tok = torch.randint(V - 1000, V, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
        h = aj.ScoreHandle(0, rows, d, V, max_top=7)
        got = outputs(rows, 1, 7)
        h.score(x, W, tok, **got)
        torch.cuda.synchronize()
        assert torch.equal(got["top_id"].long(), logits.sort(dim=-1, descending=True, stable=True).indices[:, :7])
        lse = logits.logsumexp(-1)
        assert ((got["lse"].double() - lse).abs() <= 2e-5).all()
        assert ((got["logprob"].double() - logits.gather(1, tok.long()) + lse[:, None]).abs() <= 2e-5).all()
        h.destroy()
