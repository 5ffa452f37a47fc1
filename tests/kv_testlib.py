"""Seeded caches for the key-value cache tests, and the operators from their definitions in 64 bits (plain loops over
sequences and heads; nothing here is shared with the library)."""
from __future__ import annotations

import math

import numpy as np
import torch

from aj_testlib import Guarded

NEG = float("-inf")


class Setup:
    """A paged cache with shuffled pages whose unused slots and pages hold NaN, and new tokens for it.

    lens / nq: slots in use (new tokens included) and new tokens of each sequence; ragged: pass q_start."""

    def __init__(self, seed, lens, nq, Hq, Hkv, D, page, dtype="bf16", ragged=True, spare_width=1, q_scale=2.0, pad=0):
        import paper_2504_20039_b200 as aj

        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.nq, self.Hq, self.Hkv, self.D, self.page = list(lens), list(nq), Hq, Hkv, D, page
        self.G, self.B = Hq // Hkv, len(lens)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.aj_dtype = aj.AJ_BF16 if dtype == "bf16" else aj.AJ_F32
        need = [-(-L // page) for L in self.lens]
        self.width = max(1, max(need)) + spare_width
        self.cap = self.width * page
        self.n_pages = sum(need) + 3
        perm = rng.permutation(self.n_pages)
        self.table = np.full((self.B, self.width), 0x7FFFFFF0, np.int64)  # entries past a sequence are junk
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at : at + n]
            at += n
        k = torch.full((self.n_pages, Hkv, page, D), float("nan"))
        v = torch.full((self.n_pages, Hkv, page, D), float("nan"))
        for b, L in enumerate(self.lens):
            for j in range(need[b]):
                n = min(page, L - j * page)
                k[self.table[b, j], :, :n] = torch.randn(Hkv, n, D, generator=g)
                v[self.table[b, j], :, :n] = torch.randn(Hkv, n, D, generator=g)
        self.T = sum(self.nq)
        self.start = np.concatenate([[0], np.cumsum(self.nq)])
        self.max_n = max(1, max(self.nq))
        self.ragged = ragged
        assert ragged or all(n == self.max_n for n in self.nq)
        self.pad = pad  # elements between the rows of q
        q = torch.randn(max(1, self.T), Hq * D + pad, generator=g) * q_scale
        dev = lambda t, name: Guarded(t.cuda(), name)  # noqa: E731
        self.guards = [dev(k.to(self.dt), "k_pages"), dev(v.to(self.dt), "v_pages"), dev(q.to(self.dt), "q"),
                       dev(torch.tensor(np.minimum(self.table, 2**31 - 1), dtype=torch.int32), "block_table"),
                       dev(torch.tensor(self.lens, dtype=torch.int32), "seq_lens"), dev(torch.tensor(self.start, dtype=torch.int32), "q_start")]
        self.k, self.v, self.q_all, self.block_table, self.seq_lens, q_start = (x.t for x in self.guards)
        self.q = self.q_all[: self.T, : Hq * D] if self.T else self.q_all[:1, : Hq * D]
        self.q_start = q_start if ragged else None
        self.scale = 1.0 / math.sqrt(D)

    def guard(self, t, name):
        self.guards.append(Guarded(t.cuda(), name))
        return self.guards[-1].t

    def check_guards(self):
        for x in self.guards:
            x.check()

    def handle(self, flags=0):
        import paper_2504_20039_b200 as aj

        return aj.KvHandle(0, self.B, self.max_n, self.Hq, self.Hkv, self.D, self.page, self.aj_dtype, flags)

    def rows_of(self, pages, b, h, L=None):
        """[L, D] rows of one sequence's key head, 64 bits, on the CPU."""
        L = self.lens[b] if L is None else L
        p = self.table[b, : -(-L // self.page)]
        return pages.cpu()[p, h].reshape(-1, self.D)[:L].double()

    def visible(self, b, window, sinks):
        """[nq, L] truth values."""
        L, n = self.lens[b], self.nq[b]
        p, j = np.arange(L - n, L)[:, None], np.arange(L)[None]
        ok = j <= p
        if window:
            ok &= (j > p - window) | (j < sinks)
        return torch.from_numpy(ok)

    def attend_reference(self, window=0, sinks=0):
        """(out, lse, sum of p |v|, largest scale * sum |q k|) in 64 bits."""
        out = torch.zeros(self.T, self.Hq, self.D, dtype=torch.float64)
        absum = torch.zeros_like(out)
        lse = torch.full((self.T, self.Hq), NEG, dtype=torch.float64)
        mag = torch.zeros(self.T, self.Hq, dtype=torch.float64)
        q = self.q.cpu()[: self.T].double().view(self.T, self.Hq, self.D) if self.T else None
        for b in range(self.B):
            if self.nq[b] == 0 or self.lens[b] == 0:
                continue
            r = slice(int(self.start[b]), int(self.start[b + 1]))
            seen = self.visible(b, window, sinks)
            for h in range(self.Hkv):
                K, V = self.rows_of(self.k, b, h), self.rows_of(self.v, b, h)
                for i in range(h * self.G, (h + 1) * self.G):
                    s = torch.where(seen, q[r, i] @ K.T * self.scale, torch.tensor(NEG, dtype=torch.float64))
                    m = s.amax(-1, keepdim=True)
                    e = torch.exp(s - torch.where(m == NEG, torch.zeros_like(m), m))
                    tot = e.sum(-1, keepdim=True)
                    p = torch.where(tot > 0, e / tot.clamp_min(1e-300), torch.zeros_like(e))
                    out[r, i], absum[r, i] = p @ V, p @ V.abs()
                    lse[r, i] = (torch.log(tot) + m)[:, 0]
                    mag[r, i] = (q[r, i].abs() @ K.abs().T * self.scale).amax(-1)
        return out, lse, absum, mag

    def score_error(self, mag):
        """Bound on a score's error: D products and their sum in 32 bits, the scaling, and the exponential's argument."""
        return 2.0**-23 * (self.D + 16) * mag + 2.0**-22 * (1 + mag)

    def check_attend(self, out, lse, window, sinks, rounded_weights):
        ref, ref_lse, absum, mag = self.attend_reference(window, sinks)
        got = out.float().cpu().double().view(self.T, self.Hq, self.D)
        es = self.score_error(mag)[..., None]
        # rounding on the store, weights rounded before they meet V, scores off by es, 32-bit sums
        store = 2.0**-8 * ref.abs() if self.dt == torch.bfloat16 else 2.0**-23 * ref.abs()
        tol = store + absum * ((2.0**-8 if rounded_weights else 0.0) + 4 * es + 2.0**-18) + 1e-30
        bad = ~((got - ref).abs() <= tol)
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outputs off, worst {((got - ref).abs() / tol).max()} of the tolerance"
        if lse is not None:
            got = lse.cpu().double()
            assert torch.equal(torch.isinf(got), torch.isinf(ref_lse))
            fin = ~torch.isinf(ref_lse)
            assert ((got - ref_lse).abs()[fin] <= (2 * es[..., 0] + 2.0**-18 + 2.0**-21 * ref_lse.abs())[fin]).all()
