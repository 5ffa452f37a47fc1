"""Seeded inputs for the norm and scoring tests, and the operators from their definitions in 64 bits."""
from __future__ import annotations

import math

import torch

from aj_testlib import Guarded

LOG2E = 1.4426950408889634


def tied_order(logits):
    """Entries of each row by falling logit, the lowest entry first among equals (a zero's sign does not count)."""
    return (logits + 0.0).sort(dim=-1, descending=True, stable=True).indices


class Head:
    """Hidden states and an LM head whose logits are the same number in whatever order the products are added: values on a
    grid of 7 or 8 bits, scales that are powers of two.  With `lean` a state leans towards an entry."""

    def __init__(self, seed, rows, d, V, dtype="bf16", lean=8.0, pad=0):
        import paper_2504_20039_b200 as aj

        g = torch.Generator().manual_seed(seed)
        self.rows, self.d, self.V, self.dtype = rows, d, V, dtype
        self.aj_dtype = {"bf16": aj.AJ_BF16, "f32": aj.AJ_F32, "e4m3": aj.AJ_E4M3}[dtype]
        dt = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[dtype]
        n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        at = torch.randint(V, (rows,), generator=g)
        lean = lean * torch.rand(rows, 1, generator=g)
        self.h_scale = self.w_scale = None
        if dtype == "e4m3":
            W = (40 * n(V, d)).round().clamp(-240, 240).to(dt)
            self.w_scale = 2.0 ** -torch.randint(11, 13, (V,), generator=g).float()
            self.h_scale = 2.0 ** -torch.randint(7, 9, (rows,), generator=g).float() * math.sqrt(4096 / 2.0 ** round(math.log2(d)))
            self.h_scale = 2.0 ** self.h_scale.log2().round()
            h = (100 * n(rows, d) + W[at].float() * lean * 2.0**18 / (1600 * d)).round().clamp(-448, 448).to(dt)
        else:
            W = (41 * n(V, d)).round().clamp(-127, 127).mul(2.0**-11).to(dt)
            h = (n(rows, d) + W[at].float() * lean / (0.0004 * d)).mul(16).round().clamp(-127, 127).div(16).to(dt)
        self.tokens = torch.stack([at, torch.randint(V, (rows,), generator=g), torch.randint(V, (rows,), generator=g)], 1).to(torch.int32)
        self.W, self.h = W, h
        self.pad = pad
        self.guards = []

    def guard(self, t, name):
        self.guards.append(Guarded(t, name))
        return self.guards[-1].t

    def check_guards(self):
        for x in self.guards:
            x.check()

    def logits(self):
        x = self.h.cuda().double() @ self.W.cuda().double().T
        if self.dtype == "e4m3":
            x = x * self.h_scale.cuda().double()[:, None] * self.w_scale.cuda().double()
        return x

    def run(self, n_top=5, n_tok=3, inv_t=1.0, flags=0, max_rows=None, handle=None, stream=0, lse=True, entropy=True, top_lp=True):
        import paper_2504_20039_b200 as aj

        rows = self.rows
        wide = torch.zeros(max(1, rows), self.d + self.pad, dtype=torch.float32).to(self.h.dtype)
        wide[:rows, : self.d] = self.h
        h = self.guard(wide, "h")[:rows, : self.d]
        W = self.guard(self.W, "W")
        f = lambda name, *s: self.guard(torch.full(s, -77.0), name)  # noqa: E731
        sc = {} if self.h_scale is None else {"h_scale": self.guard(self.h_scale, "h_scale"), "w_scale": self.guard(self.w_scale, "w_scale")}
        own = handle is None
        if own:
            handle = aj.ScoreHandle(0, max_rows or max(1, rows), self.d, self.V, self.aj_dtype, max_top=n_top, flags=flags)
        got = {"logprob": f("logprob", rows, n_tok) if n_tok else None, "lse": f("lse", rows) if lse else None,
               "entropy": f("entropy", rows) if entropy else None,
               "top_id": self.guard(torch.full((rows, n_top), -7, dtype=torch.int32), "top_id") if n_top else None,
               "top_logprob": f("top_logprob", rows, n_top) if n_top and top_lp else None}
        tokens = self.guard(self.tokens[:, :n_tok].contiguous(), "tokens") if n_tok else None
        handle.score(h, W, tokens, inv_temperature=inv_t, stream=stream, **got, **sc)
        torch.cuda.synchronize()
        assert handle.last_status() == aj.AJ_OK
        self.path, self.launches = handle.last_path(), handle.last_launch_count()
        if own:
            handle.destroy()
        self.check_guards()
        return got

    def check(self, got, inv_t=1.0, logit_error=0.0):
        """logit_error [rows]: how far a logit may be off (0 on the grid)."""
        x = self.logits()
        z = x * inv_t
        M = z.amax(-1)
        p = torch.softmax(z, -1)
        lse = torch.logsumexp(z, -1)
        far = M[:, None] - z
        Ed, Ed2 = (p * far).sum(-1), (p * far * far).sum(-1)
        # exponent arguments (z - M) log2 e: two roundings; the exponential 2^-22; sums over at most 64 terms in a chain, 128
        # threads' worth of partial sums and tiles in trees and short chains, so at most 160 roundings; the logarithm and what is added to it
        u = 2.0**-24
        rel = 4 * u + 160 * u
        e_s = rel + 3 * u * Ed * LOG2E + 2 * logit_error * inv_t
        tol = e_s + 4 * u * (lse.abs() + M.abs() + (lse - M).abs())

        def close(name, a, ref, tol):
            if a is None:
                return
            err = (a.double() - ref).abs()
            assert (err <= tol).all(), f"{name}: worst {float((err / tol).max()):.3g} of the tolerance, off by {float(err.max()):.3g}"

        close("lse", got["lse"], lse, tol)
        ent = lse - (p * z).sum(-1)
        close("entropy", got["entropy"], ent, tol + 4 * u * ent + Ed * rel + 4 * u * Ed + 3 * u * LOG2E * Ed2 + 2 * logit_error * inv_t * (1 + Ed))
        if got["logprob"] is not None:
            n = got["logprob"].shape[1]
            ref = z.gather(1, self.tokens[:, :n].long().cuda()) - lse[:, None]
            close("logprob", got["logprob"], ref, tol[:, None] + 4 * u * ref.abs())
        if got["top_id"] is not None:
            n = got["top_id"].shape[1]
            if torch.as_tensor(logit_error).sum() == 0:
                order = tied_order(x)[:, :n]
                assert torch.equal(got["top_id"].long(), order)
            else:  # the same values within the error, in falling order, no entry twice
                order = got["top_id"].long()
                best = x.sort(dim=-1, descending=True).values[:, :n]
                assert ((x.gather(1, order) - best).abs() <= 2 * logit_error[:, None]).all()
                assert all(len(set(r.tolist())) == n for r in order)
            if got["top_logprob"] is not None:
                ref = z.gather(1, order) - lse[:, None]
                close("top_logprob", got["top_logprob"], ref, tol[:, None] + 4 * u * ref.abs())


def norm_reference(x, r, w, eps):
    s = x.double() if r is None else x.double() + r.double()
    return s, s / (s.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
