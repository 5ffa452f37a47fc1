"""Verification windows of many questions behind the same few-shot examples, verified and scored, with a toy model of one layer.

    python examples/few_shot_scoring.py

The examples enter the paged cache once; every question's block table begins with their pages.  Then, for a window of K + 1
rows per question: aj_kv_append writes the window's keys and values, aj_kv_attend_shared attends to the examples for all
questions together, aj_add_norm adds the residual and makes the final hidden states (in bf16, and in 8 bits with
scales), aj_verify says how many draft tokens stand, and aj_score_tokens gives the draft tokens' log probabilities, each row's
entropy and its best alternatives, through the bf16 head and through one in 8 bits.  Weights are random.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_20039_b200 as aj  # noqa: E402


def run(B=12, K=8, examples=600, questions=(40, 7, 120, 1), V=3000, Hq=16, Hkv=4, D=128, page=16, top=5, seed=0, flags=0):
    """One window per question; questions' lengths repeat over the batch.  Returns what was read and what came out."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).bfloat16()  # noqa: E731
    dev, d = torch.cuda.current_device(), Hq * D
    emb, qkv_w, out_w, lm = w(V, d) * 30, w((Hq + 2 * Hkv) * D, d), w(d, Hq * D), w(V, d) * 4
    norm_w = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    scale8 = lm.float().abs().amax(-1) / 448  # the head in 8 bits
    lm8 = (lm.float() / scale8[:, None]).to(torch.float8_e4m3fn)
    n = torch.tensor([questions[b % len(questions)] for b in range(B)])

    # pages: the examples' first, then each question's own.  (The examples fill whole pages; a question begins in a new one.)
    first = examples // page
    shared = first * page
    own = -(-(int(n.max()) + K + 1) // page)
    perm = torch.randperm(first + B * own, generator=g, device="cuda").int()
    table = torch.cat([perm[:first].expand(B, first), perm[first:].view(B, own)], 1).contiguous()
    k_pages, v_pages = (torch.zeros(first + B * own, Hkv, page, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ang = torch.arange(shared + own * page, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
    cos_sin = torch.cat([ang.cos(), ang.sin()], 1).float().contiguous()
    h = aj.KvHandle(dev, B, max(shared, int(n.max()), K + 1), Hq, Hkv, D, page, flags=flags, strict=True)
    h.reserve_shared(B * (K + 1))
    stream = torch.cuda.current_stream().cuda_stream

    def append(ids, tab, lens, rows, start=None):
        qkv = emb[ids] @ qkv_w.T
        q, k, v = qkv.split([Hq * D, Hkv * D, Hkv * D], 1)
        rotated = torch.empty_like(q)
        h.append(q, k, v, k_pages, v_pages, tab, lens, rotated, tab.shape[0], rows, cos_sin, q_start=start, stream=stream)
        return rotated

    draw = lambda *s: torch.randint(V, s, generator=g, device="cuda")  # noqa: E731
    shots, texts = draw(shared), [draw(int(m)) for m in n]
    append(shots, table[:1].contiguous(), torch.tensor([shared], dtype=torch.int32, device="cuda"), shared)
    lens = (shared + n).int().cuda()
    start = torch.cat([torch.zeros(1), n.cumsum(0)]).int().cuda()
    append(torch.cat(texts), table, lens, int(n.max()), start)

    # the window: the question's last token was cached with it, the draft's K tokens and one more row come now
    window = draw(B, K + 1)
    lens += K + 1
    q = append(window.reshape(-1), table, lens, K + 1)
    o = torch.empty_like(q)
    h.attend_shared(q, k_pages, v_pages, table[0, :first].contiguous(), shared, table, lens, o, B, K + 1, D**-0.5, stream=stream)
    x = emb[window.reshape(-1)]
    hidden, hidden8, hscale = torch.empty_like(x), torch.empty(x.shape, device="cuda", dtype=torch.float8_e4m3fn), torch.empty(len(x), device="cuda")
    residual = torch.empty_like(x)
    aj.add_norm(o @ out_w.T, norm_w, 1e-5, out=hidden, residual=x, residual_out=residual, out8=hidden8, scale8=hscale, stream=stream)

    drafted = window[:, 1:].int().contiguous()
    verify = aj.Handle(dev, B, K, d, 0, V)
    accept, nxt, target = (torch.zeros(s, device="cuda", dtype=torch.int32) for s in ((B,), (B,), (B, K + 1)))
    verify.verify(hidden.view(B, K + 1, d), None, lm, drafted, torch.zeros(d, device="cuda"), 0.0, 0.0, B, K, accept, nxt, target_tok=target, stream=stream)
    # row i predicts draft token i + 1; the last row has none
    asked = torch.cat([drafted, torch.full((B, 1), -1, device="cuda", dtype=torch.int32)], 1).view(-1, 1)
    scores = {}
    for name, dtype, states, head, kw in (("bf16", aj.AJ_BF16, hidden, lm, {}), ("e4m3", aj.AJ_E4M3, hidden8, lm8, {"h_scale": hscale, "w_scale": scale8})):
        s = aj.ScoreHandle(dev, len(x), d, V, dtype, max_top=top)
        f = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
        got = {"logprob": f(len(x), 1), "lse": f(len(x)), "entropy": f(len(x)), "top_id": torch.empty(len(x), top, device="cuda", dtype=torch.int32),
               "top_logprob": f(len(x), top)}
        s.score(states, head, asked, stream=stream, **got, **kw)
        scores[name] = got
    torch.cuda.synchronize()
    assert h.last_status() == 0
    return dict(emb=emb, qkv_w=qkv_w, out_w=out_w, lm=lm, lm8=lm8, scale8=scale8, norm_w=norm_w, cos_sin=cos_sin, shots=shots, texts=texts, window=window,
                hidden=hidden, residual=residual, hidden8=hidden8, hscale=hscale, accept=accept, target=target, drafted=drafted, asked=asked, scores=scores,
                path=h.last_path(), Hq=Hq, Hkv=Hkv, D=D)


if __name__ == "__main__":
    r = run()
    s = r["scores"]["bf16"]
    print("accepted", r["accept"].tolist())
    print("log probabilities of the first window's draft tokens", [round(x, 2) for x in s["logprob"][: r["drafted"].shape[1], 0].tolist()])
    print("entropies", [round(x, 2) for x in s["entropy"][: r["drafted"].shape[1]].tolist()])
