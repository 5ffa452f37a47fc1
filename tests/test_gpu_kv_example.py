"""The key-value cache operators used together: the example's speculative-decoding loop."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_cycles_match_dense_attention_over_the_text():
    """Without eviction, the target's hidden states of the last window are those of plain attention over each whole text:
    appended, rolled back and overwritten slots left nothing behind."""
    import torch

    import speculative_cycle as ex

    K, cycles, prompt = 8, 5, (70, 33, 128, 5)
    texts, accepted, m, hidden = ex.run(cycles=cycles, K=K, prompt=prompt)
    for b in range(4):
        assert len(texts[b]) == prompt[b] + int(accepted[:, b].sum()) + cycles
        n_last = int(accepted[-1, b]) + 1                      # rows of the last window that stand
        begin = len(texts[b]) - n_last - 1                     # its first token's position
        ids = torch.tensor(texts[b][: begin + n_last], device="cuda")
        assert int(m.lens[b]) == len(ids) and int(m.seen[b]) == len(ids)
        x = m.emb[ids]
        qkv = (x @ m.qkv.T).float()
        q, k, v = (y.view(len(ids), -1, m.D) for y in qkv.split([m.Hq * m.D, m.Hkv * m.D, m.Hkv * m.D], 1))
        cs = m.cos_sin[: len(ids), None]
        c, s = cs[..., : m.D // 2], cs[..., m.D // 2 :]

        def turn(y):
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)
            a, d = y[..., : m.D // 2], y[..., m.D // 2 :]
            return torch.cat([a * c - d * s, d * c + a * s], -1).bfloat16().float()

        q, k = turn(q), turn(k).repeat_interleave(m.Hq // m.Hkv, 1)
        v = v.bfloat16().float().repeat_interleave(m.Hq // m.Hkv, 1)
        z = torch.einsum("qhd,khd->hqk", q, k) * m.D**-0.5
        z.masked_fill_(torch.ones(len(ids), len(ids), device="cuda").triu(1).bool(), float("-inf"))
        o = torch.einsum("hqk,khd->qhd", z.softmax(-1), v).reshape(len(ids), -1)
        want = (x.float() + o @ m.out.float().T)[begin:]
        got = hidden[b, :n_last].float()
        # bf16 attention outputs, weights and hidden states: a few roundings of 2^-8 on each side
        assert (got - want).norm() <= 0.02 * want.norm()


def test_eviction_holds_the_budget():
    import speculative_cycle as ex

    keep = 64
    texts, accepted, m, _ = ex.run(cycles=6, K=4, prompt=(90, 20, 64, 65), keep=keep)
    for b in range(4):
        seen = len(texts[b]) - 1
        assert int(m.seen[b]) == seen
        assert int(m.lens[b]) <= keep and (seen >= keep + 5) <= (int(m.lens[b]) == keep)
        pos = m.slot_pos[b, :, : int(m.lens[b])]
        for h in range(m.Hkv):
            p = sorted(pos[h].tolist())
            assert len(set(p)) == len(p) and p[-1] == seen - 1
            assert p[:4] == [0, 1, 2, 3] and p[-16:] == list(range(seen - 16, seen))  # the first and the newest stay
