"""A speculative-decoding loop on the framework's operators, with toy models of one attention layer each.

    python examples/speculative_cycle.py [cycles]

Prompts of different length enter two paged caches (aj_kv_append, aj_kv_attend, ragged).  Then, cycle by cycle: the draft
model takes K + 1 single-token steps; the target model runs the window of K + 1 rows against its cache; aj_verify
says how many draft tokens stand; the attention weight of the rows that stand is accumulated (aj_kv_weigh); the
rejected rows are taken back by lowering the lengths; and a cache that has outgrown its budget is cut to its most
attended slots (aj_kv_evict).  Weights are random, so the text is noise; the calls, shapes and bookkeeping are real.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_20039_b200 as aj  # noqa: E402


class ToyModel:
    """Embedding, one attention layer with a residual, and an LM head, with its own paged cache."""

    def __init__(self, V, Hq, Hkv, D, B, max_q, max_tokens, page, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).bfloat16()  # noqa: E731
        self.d, self.Hq, self.Hkv, self.D, self.B = Hq * D, Hq, Hkv, D, B
        self.emb, self.qkv, self.out, self.lm = w(V, self.d), w((Hq + 2 * Hkv) * D, self.d), w(self.d, Hq * D), w(V, self.d)
        width = -(-max_tokens // page)
        pages = (B * width, Hkv, page, D)
        self.k, self.v = (torch.zeros(pages, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        self.table = torch.randperm(B * width, generator=g, device="cuda").int().view(B, width)
        self.lens = torch.zeros(B, device="cuda", dtype=torch.int32)   # slots in use
        self.seen = torch.zeros(B, device="cuda", dtype=torch.int32)   # tokens seen: positions go on after an eviction
        self.weight = torch.zeros(B, Hkv, width * page, device="cuda")
        self.slot_pos = torch.zeros(B, Hkv, width * page, device="cuda", dtype=torch.int32)
        ang = torch.arange(4 * max_tokens, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
        self.cos_sin = torch.cat([ang.cos(), ang.sin()], 1).float().contiguous()
        self.q_norm, self.k_norm = torch.ones(D, device="cuda"), torch.ones(D, device="cuda")
        self.h = aj.KvHandle(torch.cuda.current_device(), B, max_q, Hq, Hkv, D, page, strict=True)

    def forward(self, tokens, row_seq, positions, n_q, q_start=None):
        """Hidden states [rows, d] of new tokens; leaves the queries and lse of the call for `weigh`."""
        stream = torch.cuda.current_stream().cuda_stream
        x = self.emb[tokens]
        qkv = x @ self.qkv.T
        a, b = self.Hq * self.D, (self.Hq + self.Hkv) * self.D
        q, k, v = qkv[:, :a], qkv[:, a:b], qkv[:, b:]
        self.lens += torch.bincount(row_seq, minlength=self.B).int()
        self.q, self.lse = torch.empty_like(q), torch.empty(len(x), self.Hq, device="cuda")
        o = torch.empty_like(self.q)
        self.h.append(q, k, v, self.k, self.v, self.table, self.lens, self.q, self.B, n_q, self.cos_sin, q_start=q_start, positions=positions,
                      q_norm=self.q_norm, k_norm=self.k_norm, slot_pos=self.slot_pos, weight=self.weight, stream=stream)
        self.h.attend(self.q, self.k, self.v, self.table, self.lens, o, self.B, n_q, self.D**-0.5, q_start=q_start, lse=self.lse, stream=stream)
        return x + o @ self.out.T

    def count(self, n_q, n_rows, q_start=None):
        """Accumulate the attention weight of the rows that stand."""
        self.h.weigh(self.q, self.lse, self.k, self.table, self.lens, self.weight, self.weight, self.B, n_q, self.D**-0.5, q_start=q_start,
                     n_rows=n_rows, stream=torch.cuda.current_stream().cuda_stream)

    def cut(self, keep, sinks=4, recent=16):
        self.h.evict(self.k, self.v, self.table, self.lens, self.weight, self.slot_pos, self.lens, self.weight, self.slot_pos, self.B, keep,
                     sinks, recent, stream=torch.cuda.current_stream().cuda_stream)


def run(cycles=8, B=4, K=8, prompt=(70, 33, 128, 5), keep=0, V=1000, tau=0.5, seed=0, log=None):
    """Returns (tokens of each sequence, accepted lengths [cycles, B], target model, hidden states of the last window)."""
    g = torch.Generator().manual_seed(seed)
    room = max(prompt) + cycles * (K + 1) + 16
    target = ToyModel(V, 16, 4, 128, B, max(max(prompt), K + 1), room, 16, seed + 1)
    draft = ToyModel(V, 16, 4, 64, B, max(max(prompt), 1), room, 16, seed + 2)
    verify = aj.Handle(torch.cuda.current_device(), B, K, target.d, draft.d, V)
    judge_w = 0.02 * torch.randn(draft.d + target.d, generator=g).cuda()
    accept, nxt = (torch.zeros(B, device="cuda", dtype=torch.int32) for _ in range(2))

    texts = [torch.randint(0, V, (n,), generator=g).tolist() for n in prompt]
    lens = torch.tensor(prompt)
    start = torch.cat([torch.zeros(1), lens.cumsum(0)]).int().cuda()
    row_seq = torch.repeat_interleave(torch.arange(B), lens).cuda()
    pos = torch.cat([torch.arange(n) for n in prompt]).int().cuda()
    tokens = torch.tensor(sum(texts, [])).cuda()
    for m in (target, draft):  # the prompts, but for each one's last token, which begins the first window
        m.forward(tokens, row_seq, pos, max(prompt), start)
        m.count(max(prompt), (lens - 1).int().cuda(), start)
        m.lens -= 1
        m.seen += lens.int().cuda() - 1
    last = torch.tensor([t[-1] for t in texts]).cuda()
    history = []
    one = torch.arange(B, device="cuda")
    for _ in range(cycles):
        tok, h_draft, window = last, [], [last]
        for i in range(K + 1):  # the draft's own steps; the last one only encodes its last token for the classifier
            h_draft.append(draft.forward(tok, one, draft.seen + i, 1))
            draft.count(1, None)
            if i < K:
                tok = (h_draft[-1] @ draft.lm.T).argmax(-1)
                window.append(tok)
        win = torch.stack(window, 1)
        at = (target.seen[:, None] + torch.arange(K + 1, device="cuda")).int().reshape(-1)
        h_target = target.forward(win.reshape(-1), one.repeat_interleave(K + 1), at, K + 1)
        drafted = win[:, 1:].int().contiguous()
        verify.verify(h_target.view(B, K + 1, -1), torch.stack(h_draft, 1).contiguous(), target.lm, drafted, judge_w, 0.0, tau, B, K, accept, nxt,
                      stream=torch.cuda.current_stream().cuda_stream)
        target.count(K + 1, accept + 1)
        for m in (target, draft):  # the rows behind the stop are taken back
            m.lens -= K - accept
            m.seen += accept + 1
            if keep:
                m.cut(keep)
        last = nxt.long()
        history.append(accept.cpu().clone())
        for b in range(B):
            n = int(accept[b])
            texts[b] += drafted[b, :n].tolist() + [int(nxt[b])]
        if log:
            log("accepted %s of %d, cache %s" % (history[-1].tolist(), K, target.lens.tolist()))
    torch.cuda.synchronize()
    assert target.h.last_status() == 0 and draft.h.last_status() == 0
    return texts, torch.stack(history), target, h_target.view(B, K + 1, -1)


if __name__ == "__main__":
    run(int(sys.argv[1]) if len(sys.argv) > 1 else 8, keep=96, log=print)
