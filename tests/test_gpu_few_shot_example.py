"""append, attend_shared, add_norm, verify and score together: the example's windows behind shared examples."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("K", [8, 1])
def test_windows_behind_shared_examples(K):
    import torch

    import few_shot_scoring as ex
    import paper_2504_20039_b200 as aj

    r = ex.run(K=K, flags=aj.AJ_KV_FLAG_FORCE_SHARED)
    assert r["path"].startswith("shared")
    Hq, Hkv, D, B = r["Hq"], r["Hkv"], r["D"], len(r["texts"])
    hidden = r["hidden"].view(B, K + 1, -1)
    for b in range(B):
        ids = torch.cat([r["shots"], r["texts"][b], r["window"][b]])
        x = r["emb"][ids]
        qkv = (x @ r["qkv_w"].T).float()
        q, k, v = (y.view(len(ids), -1, D) for y in qkv.split([Hq * D, Hkv * D, Hkv * D], 1))
        cs = r["cos_sin"][: len(ids), None]
        c, s = cs[..., : D // 2], cs[..., D // 2 :]

        def turn(y):
            a, e = y[..., : D // 2], y[..., D // 2 :]
            return torch.cat([a * c - e * s, e * c + a * s], -1).bfloat16().double()

        q, k, v = turn(q)[-(K + 1) :], turn(k).repeat_interleave(Hq // Hkv, 1), v.bfloat16().double().repeat_interleave(Hq // Hkv, 1)
        z = torch.einsum("qhd,khd->hqk", q, k) * D**-0.5
        at = torch.arange(len(ids), device="cuda")
        z.masked_fill_(at > at[-(K + 1) :, None], float("-inf"))
        o = torch.einsum("hqk,khd->qhd", z.softmax(-1), v).reshape(K + 1, -1)
        y = x[-(K + 1) :].double() + o @ r["out_w"].double().T
        want = y / (y.square().mean(-1, keepdim=True) + 1e-5).sqrt() * r["norm_w"].double()
        # bf16 queries, attention weights and outputs, projection and hidden states: a few roundings of 2^-8
        assert (hidden[b].double() - want).norm() <= 0.02 * want.norm()
    # 8 bits: half a step of the largest value's scale at most
    back = r["hidden8"].float() * r["hscale"][:, None]
    assert ((back - r["hidden"].float()).abs() <= back.abs() * (2.0**-4 + 2.0**-7) + r["hscale"][:, None] * 2.0**-9).all()

    # the scores are those of the hidden states that were verified, and the best alternative is the token that the verification took
    for name, h, W in (("bf16", r["hidden"].double(), r["lm"].double()), ("e4m3", back.double(), r["lm8"].double() * r["scale8"].double()[:, None])):
        s, z = r["scores"][name], h @ W.T
        logp = z.log_softmax(-1)
        # a logit: d products and their sum in 32 bits; two scalings
        tol = (h.abs() @ W.abs().T).amax(-1) * (h.shape[1] + 8) * 2.0**-24 * 2 + 1e-4
        asked = r["asked"].view(-1)
        has = asked >= 0
        got = s["logprob"][:, 0]
        assert got[~has].isnan().all()
        ref = logp.gather(1, asked.clamp_min(0).long()[:, None])[:, 0]
        assert ((got.double() - ref).abs() <= tol)[has].all()
        assert ((s["lse"].double() - z.logsumexp(-1)).abs() <= tol).all()
        best = z.sort(dim=-1, descending=True).values[:, : s["top_id"].shape[1]]
        assert ((z.gather(1, s["top_id"].long()) - best).abs() <= 2 * tol[:, None]).all()
        if name == "bf16":
            gap = best[:, 0] - best[:, 1] > 2 * tol
            assert torch.equal(s["top_id"][:, 0][gap], r["target"].view(-1)[gap])
    match = r["drafted"] == r["target"][:, :-1]
    assert torch.equal(r["accept"], match.int().cumprod(1).sum(1).int())
