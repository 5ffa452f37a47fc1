"""Cases of the key-value cache operators: what a serving program runs around the verify-and-judge cycle.

Four operators on one paged cache [n_pages, Hkv, page, D]: `append` (per-head norms, rotation, write into the pages),
`attend` (new tokens against the cached ones), `weigh` (attention weight a cached token has received) and `evict`
(keep the slots with the most of it).  `run` computes them in plain torch, or with `own` through the framework.
"""
import math

import numpy as np
import torch

own = False

NEG = float("-inf")


def _case(name, op, **kw):
    base = {"name": name, "op": op, "B": 1, "n": 1, "ragged_n": False, "lo": 0, "hi": 1024, "Hq": 32, "Hkv": 8, "D": 128, "page": 16,
            "dtype": "bf16"}
    return {**base, **kw}


def listed():
    return [
        # The draft model's or the target's single token of one user: nothing but latency.
        _case("append 1 token", "append", lo=1037, hi=1037, page=16, norm=True, interleaved=False, rot=128),
        # A batch of prompts entering the cache, 64 query heads, pairs rotated next to one another, no norms.
        _case("append prompts", "append", B=8, n=4096, ragged_n=True, lo=0, hi=4096, Hq=64, page=64, norm=False, interleaved=True, rot=128),
        # One user's draft step in the storage type of the small configuration (f32), head size of the draft model.
        _case("attend 1 token f32", "attend", lo=1037, hi=1037, D=64, dtype="f32", window=0, sinks=0),
        # The ordinary decode step: a batch of users with caches of very different length.
        _case("attend 1 token x64", "attend", B=64, lo=33, hi=8191, window=0, sinks=0),
        # Long caches read through a sliding window with a few first tokens that stay visible.
        _case("attend 1 token window", "attend", B=32, lo=2001, hi=32768, Hq=64, page=64, window=4096, sinks=4),
        # The verification pass: K = 32 draft tokens and the last accepted one, for 64 users.
        _case("attend verify 64x33", "attend", B=64, n=33, lo=129, hi=4100, page=32, window=0, sinks=0),
        # A long prompt of one user.
        _case("attend prompt 8192", "attend", n=8192, lo=8192, hi=8192, page=64, window=0, sinks=0),
        # Prompts of the draft model with a sliding window and sinks.
        _case("attend prompts window", "attend", B=4, n=4096, ragged_n=True, lo=0, hi=4096, D=64, page=32, window=1024, sinks=4),
        # Accumulated weight after a decode step of a batch.
        _case("weigh 1 token x64", "weigh", B=64, lo=100, hi=4096, page=16),
        # Accumulated weight of the accepted rows of verified windows.
        _case("weigh verify 8x33", "weigh", B=8, n=33, lo=1000, hi=8192, page=32),
        # A long prompt's cache cut to its budget.
        _case("evict 16384 to 4096", "evict", lo=16384, hi=16384, page=64, keep=4096, sinks=4, recent=128),
        # A batch that has grown past its budget by up to a window.
        _case("evict x32 to 2048", "evict", B=32, lo=2040, hi=2113, page=16, keep=2048, sinks=4, recent=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weigh", "evict"])
    D = rng.choice([64, 128, 128])
    Hq = rng.choice([32, 32, 64])
    page = rng.choice([16, 32, 64])
    c = {"op": op, "B": 1, "n": 1, "ragged_n": False, "lo": 0, "hi": 1024, "Hq": Hq, "Hkv": 8, "D": D, "page": page, "dtype": "bf16"}
    if op == "append":
        n = _log(rng, 1, 4096)
        B = min(_log(rng, 1, 256), max(1, 16384 // n))
        c.update(B=B, n=n, ragged_n=n > 64, lo=0 if n > 64 else n, hi=n if n > 64 else n + _log(rng, 1, 2048), norm=rng.random() < 0.5,
                 interleaved=rng.random() < 0.3, rot=rng.choice([D, D, D // 2]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    elif op == "attend":
        kind = rng.choice(["one", "window", "prompt"])
        slide = rng.random() < 0.35
        if kind == "one":
            B = _log(rng, 1, 128)
            hi = _log(rng, 64, max(65, min(32768, 400000 // B)))
            c.update(B=B, n=rng.choice([1, 1, 1, 2]), lo=max(2, hi // rng.choice([1, 4, 50])), hi=hi, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        elif kind == "window":
            n = rng.choice([5, 8, 9, 17, 33, 65, _log(rng, 5, 80)])
            B = _log(rng, 1, 64)
            hi = n + _log(rng, 32, max(64, min(16384, 260000 // B)))
            c.update(B=B, n=n, lo=max(n, hi // rng.choice([1, 4, 30])), hi=hi)
        else:
            n = _log(rng, 100, 8192)
            B = min(rng.choice([1, 1, 2, 4, 8]), max(1, (8192 * 8192 * 32) // (n * n * Hq)), max(1, 16384 // n))
            if n * n * Hq * B > 8192 * 8192 * 32:
                c["Hq"] = 32
            c.update(B=B, n=n, ragged_n=B > 1, lo=0 if B > 1 else n, hi=n)
        c.update(window=_log(rng, 16, 4096) if slide else 0, sinks=rng.choice([0, 4, 17]) if slide else 0)
    elif op == "weigh":
        B = _log(rng, 1, 64)
        n = rng.choice([1, 1, 17, 33, _log(rng, 2, 65)])
        hi = n + _log(rng, 64, max(65, min(16384, 260000 // B)))
        c.update(B=B, n=n, lo=max(n, hi // rng.choice([1, 4, 30])), hi=hi)
    else:
        B = _log(rng, 1, 64)
        keep = _log(rng, 200, max(201, min(8192, 65536 // B)))
        hi = keep + rng.choice([1, 17, 64, keep // 2, 3 * keep])
        c.update(B=B, lo=max(1, keep - rng.choice([0, 50])) if hi < 2 * keep else hi, hi=hi, keep=keep, sinks=rng.choice([0, 4]), recent=rng.choice([16, 64, 128]),
                 dtype=rng.choice(["bf16", "bf16", "f32"]))
    return c


# ------------------------------------------------------------------------------------ inputs


def _lengths(c, rng):
    """New tokens and cached tokens (the new ones among them) of each sequence, on the host: the case fixes which
    lengths there are (so every seed has the same work and shapes), the seed which sequence has which."""
    B, n = c["B"], c["n"]
    L = np.random.default_rng([c["lo"], c["hi"], B, n]).integers(c["lo"], c["hi"] + 1, B)
    L[0] = c["hi"]
    L = rng.permutation(L)
    if c["ragged_n"]:
        return L.copy(), L  # prompts: everything that is cached is new
    return np.full(B, n), np.maximum(L, n)


def _host(c, seed):
    rng = np.random.default_rng([int(seed), 77])
    nq, L = _lengths(c, rng)
    width = -(-int(max(L.max(), c["hi"])) // c["page"])
    need = -(-L // c["page"])
    n_pages = int(need.sum()) + 3
    perm = rng.permutation(n_pages)
    table = np.zeros((c["B"], width), np.int32)
    at = 0
    for b in range(c["B"]):
        table[b, : need[b]] = perm[at : at + need[b]]
        at += need[b]
    return nq, L, width, n_pages, table, rng


def prepare(case, seed):
    c = dict(case)
    nq, L, width, n_pages, table, rng = _host(c, seed)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, Hq, Hkv, D, page = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    T = int(nq.sum())
    start = np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)
    s = {"c": c, "nq": nq, "L": L, "T": T, "max_n": int(nq.max()), "cap": width * page,
         "lens": torch.tensor(L, dtype=torch.int32, device=dev), "start": torch.tensor(start, device=dev),
         "table": torch.tensor(table, device=dev), "scale": 1.0 / math.sqrt(D)}
    row_b = np.repeat(np.arange(B), nq)
    row_t = np.arange(T) - start[row_b]
    s["row_b"], s["row_t"] = torch.tensor(row_b, device=dev), torch.tensor(row_t, device=dev)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    if own:
        import paper_2504_20039_b200 as aj

        s["h"] = aj.KvHandle(torch.cuda.current_device(), B, max(1, s["max_n"]), Hq, Hkv, D, page, aj.AJ_BF16 if c["dtype"] == "bf16" else aj.AJ_F32)
    s["k"] = normal(n_pages, Hkv, page, D).to(dt)
    s["v"] = normal(n_pages, Hkv, page, D).to(dt)
    if c["op"] == "append":
        qkv = normal(T, (Hq + 2 * Hkv) * D).to(dt)  # one projection's output, the three parts side by side
        s["q_in"], s["k_in"], s["v_in"] = qkv[:, : Hq * D], qkv[:, Hq * D : (Hq + Hkv) * D], qkv[:, (Hq + Hkv) * D :]
        s["q_out"] = torch.zeros(T, Hq * D, device=dev, dtype=dt)
        rot = c["rot"]
        freq = 500000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        ang = torch.arange(int(L.max()), device=dev, dtype=torch.float64)[:, None] * freq[None]
        s["cos_sin"] = torch.cat([ang.cos(), ang.sin()], 1).float().contiguous()
        if c["norm"]:
            s["qw"], s["kw"] = 1 + 0.1 * normal(D), 1 + 0.1 * normal(D)
    elif c["op"] in ("attend", "weigh"):
        s["q"] = (2 * normal(T, Hq * D)).to(dt)
        s["out"] = torch.zeros(T, Hq * D, device=dev, dtype=dt)
        s["lse"] = torch.zeros(T, Hq, device=dev)
        if c["op"] == "weigh":
            s["rows"] = torch.tensor(rng.integers(1, c["n"] + 1, B), dtype=torch.int32, device=dev)
            s["weight"] = normal(B, Hkv, s["cap"]).abs()
            s["weight_out"] = torch.zeros_like(s["weight"])
            s["lse"] = _attend_plain(s, 0, 0)[1]
    else:
        s["weight"] = normal(B, Hkv, s["cap"]).square()
        key = torch.rand(B, Hkv, s["cap"], generator=g, device=dev)
        valid = torch.arange(s["cap"], device=dev)[None, None] < s["lens"][:, None, None]
        # After an eviction the slots of a head are in no order, and positions that were evicted are missing.
        rank = torch.where(valid, key, 2.0).argsort(-1).argsort(-1)
        s["pos"] = (rank + 37 * (rank >= 4)).to(torch.int32)
        s["lens_out"] = torch.zeros(B, dtype=torch.int32, device=dev)
        s["weight_out"], s["pos_out"] = torch.zeros_like(s["weight"]), torch.zeros_like(s["pos"])
    return s


# ------------------------------------------------------------------------------- plain forms


def _flat_rows(s, slots):
    """Row of the pages, as [n_pages * Hkv * page, D], of slots [B, Hkv, n]."""
    c = s["c"]
    B, Hkv, n = slots.shape
    page = torch.gather(s["table"].long()[:, None].expand(B, Hkv, -1), 2, slots // c["page"])
    head = torch.arange(Hkv, device=slots.device)[None, :, None]
    return (page * Hkv + head) * c["page"] + slots % c["page"]


def _rotate(x, cos, sin, rot, interleaved):
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2 : rot])
    y, z = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _append_plain(s):
    c = s["c"]
    slot = (s["lens"][s["row_b"]] - (s["start"][1:] - s["start"][:-1])[s["row_b"]] + s["row_t"]).long()
    cs = s["cos_sin"][slot][:, None]
    cos, sin = cs[..., : c["rot"] // 2], cs[..., c["rot"] // 2 :]
    q, k = s["q_in"].float().view(-1, c["Hq"], c["D"]), s["k_in"].float().view(-1, c["Hkv"], c["D"])
    if c["norm"]:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + 1e-6) * s["qw"]
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + 1e-6) * s["kw"]
    q, k = _rotate(q, cos, sin, c["rot"], c["interleaved"]), _rotate(k, cos, sin, c["rot"], c["interleaved"])
    at = s["table"].long()[s["row_b"], slot // c["page"]], slice(None), slot % c["page"]
    s["k"][at] = k.to(s["k"].dtype)
    s["v"][at] = s["v_in"].reshape(-1, c["Hkv"], c["D"])
    return q.reshape(-1, c["Hq"] * c["D"]).to(s["q_in"].dtype), s["k"], s["v"]


def _scores(s, window, sinks):
    """Masked, scaled scores [B, Hkv, n * G, cap] in 32 bits, and the rows of the pages that hold the slots."""
    c = s["c"]
    B, n, G, cap = c["B"], s["max_n"], c["Hq"] // c["Hkv"], s["cap"]
    slots = torch.arange(cap, device=s["lens"].device)
    rows = _flat_rows(s, slots[None, None].expand(B, c["Hkv"], cap))
    q = torch.zeros(B, n, c["Hq"], c["D"], device=slots.device)
    q[s["row_b"], s["row_t"]] = s["q"].float().view(-1, c["Hq"], c["D"])
    q = q.view(B, n, c["Hkv"], G, c["D"]).transpose(1, 2).reshape(B, c["Hkv"], n * G, c["D"])
    x = q @ s["k"].view(-1, c["D"])[rows].float().transpose(-1, -2) * s["scale"]
    nq = s["start"][1:] - s["start"][:-1]
    pos = (s["lens"] - nq)[:, None] + torch.arange(n, device=slots.device)[None]  # [B, n]
    seen = slots <= pos[..., None]
    if window:
        seen &= (slots > pos[..., None] - window) | (slots < sinks)
    return x.masked_fill_(~seen.repeat_interleave(G, 1)[:, None], NEG), rows


def _attend_plain(s, window, sinks):
    c = s["c"]
    x, rows = _scores(s, window, sinks)
    B, n, G = c["B"], s["max_n"], c["Hq"] // c["Hkv"]
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ s["v"].view(-1, c["D"])[rows].float()) / total.clamp_min(1e-38)
    lse = (total.log() + m).view(B, c["Hkv"], n, G).transpose(1, 2).reshape(B, n, c["Hq"])
    o = o.view(B, c["Hkv"], n, G, c["D"]).transpose(1, 2).reshape(B, n, c["Hq"] * c["D"])
    return o[s["row_b"], s["row_t"]].to(s["q"].dtype), lse[s["row_b"], s["row_t"]]


def _weigh_plain(s):
    c = s["c"]
    B, n, G = c["B"], s["max_n"], c["Hq"] // c["Hkv"]
    x, _ = _scores(s, 0, 0)
    lse = s["lse"].view(B, n, c["Hkv"], G).transpose(1, 2).reshape(B, c["Hkv"], n * G, 1)
    counted = torch.arange(n, device=x.device)[None] < s["rows"][:, None]
    p = (x - lse).exp() * counted.repeat_interleave(G, 1)[:, None, :, None]
    valid = torch.arange(s["cap"], device=x.device)[None, None] < s["lens"][:, None, None]
    return (s["weight"] + p.sum(2)).masked_fill(~valid, 0)


def _evict_plain(s):
    c = s["c"]
    cap, keep = s["cap"], c["keep"]
    slots = torch.arange(cap, device=s["lens"].device)[None, None]
    valid = slots < s["lens"][:, None, None]
    newest = s["pos"].masked_fill(~valid, -1).amax(-1, keepdim=True)
    fixed = (s["pos"] < c["sinks"]) | (s["pos"] > newest - c["recent"])
    key = s["weight"].masked_fill(fixed, math.inf).masked_fill(~valid, NEG)
    order = key.sort(dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(valid.expand_as(key)).scatter(2, order[..., :keep], True) & valid
    hole, mover = ~kept & valid & (slots < keep), kept & (slots >= keep)
    n = min(keep, cap - keep) if cap > keep else 0
    dst, src = (x.to(torch.int8).sort(dim=-1, descending=True, stable=True).indices[..., :n] for x in (hole, mover))
    moves = slots[..., :n] < mover.sum(-1, keepdim=True)
    to, fro = _flat_rows(s, dst)[moves], _flat_rows(s, src)[moves]
    k, v = s["k"].view(-1, c["D"]), s["v"].view(-1, c["D"])
    k[to], v[to] = k[fro], v[fro]
    lens = s["lens"].clamp_max(keep)
    left = slots < lens[:, None, None]
    take = slots.expand_as(key).scatter(2, dst, torch.where(moves, src, dst))
    return lens, s["weight"].gather(2, take).masked_fill(~left, 0), s["pos"].gather(2, take).masked_fill(~left, 0), s["k"], s["v"]


def run(s):
    c = s["c"]
    if not own:
        if c["op"] == "append":
            return _append_plain(s)
        if c["op"] == "attend":
            return _attend_plain(s, c["window"], c["sinks"])
        return _weigh_plain(s) if c["op"] == "weigh" else _evict_plain(s)
    h, stream = s["h"], torch.cuda.current_stream().cuda_stream
    start = s["start"] if c["ragged_n"] else None
    if c["op"] == "append":
        h.append(s["q_in"], s["k_in"], s["v_in"], s["k"], s["v"], s["table"], s["lens"], s["q_out"], c["B"], s["max_n"], s["cos_sin"],
                 q_start=start, q_norm=s.get("qw"), k_norm=s.get("kw"), eps=1e-6, rot_dim=c["rot"], interleaved=c["interleaved"], stream=stream)
        return s["q_out"], s["k"], s["v"]
    if c["op"] == "attend":
        h.attend(s["q"], s["k"], s["v"], s["table"], s["lens"], s["out"], c["B"], s["max_n"], s["scale"], q_start=start,
                 window=c["window"], sinks=c["sinks"], lse=s["lse"], stream=stream)
        return s["out"], s["lse"]
    if c["op"] == "weigh":
        h.weigh(s["q"], s["lse"], s["k"], s["table"], s["lens"], s["weight"], s["weight_out"], c["B"], s["max_n"], s["scale"],
                n_rows=s["rows"], stream=stream)
        return s["weight_out"]
    h.evict(s["k"], s["v"], s["table"], s["lens"], s["weight"], s["pos"], s["lens_out"], s["weight_out"], s["pos_out"], c["B"], c["keep"],
            c["sinks"], c["recent"], stream=stream)
    return s["lens_out"], s["weight_out"], s["pos_out"], s["k"], s["v"]


# --------------------------------------------------------------------------- work and 64 bits


def work(case):
    """Each visible key and value, each query and each output once; what the mask hides is neither read nor multiplied."""
    c = dict(case)
    e = 2 if c["dtype"] == "bf16" else 4
    D, Hq, Hkv, B = c["D"], c["Hq"], c["Hkv"], c["B"]
    nq, L, _, _, _, rng = _host(c, 1)
    T = int(nq.sum())
    if c["op"] == "append":
        return {"bytes": T * (2 * (Hq + 2 * Hkv) * D * e + 4 * c["rot"]), "flops": T * (Hq + Hkv) * D * (6 if c["norm"] else 3)}
    if c["op"] == "attend":
        w, sinks = c["window"], c["sinks"]
        pairs = keys = 0
        for b in range(B):
            p = np.arange(L[b] - nq[b], L[b])
            first = np.maximum(0, p - w + 1) if w else np.zeros_like(p)
            pairs += int((p + 1 - first + np.minimum(first, sinks)).sum())
            if nq[b]:
                keys += int(L[b] - first[0] + min(first[0], sinks))
        return {"bytes": keys * Hkv * D * e * 2 + 2 * T * Hq * D * e + 4 * T * Hq, "flops": 4 * pairs * Hq * D}
    if c["op"] == "weigh":
        rows = rng.integers(1, c["n"] + 1, B)
        return {"bytes": int(L.sum()) * Hkv * (D * e + 8) + int(rows.sum()) * Hq * (D * e + 4), "flops": 2 * int((L * rows).sum()) * Hq * D}
    cut = L > c["keep"]
    # With weights in no order a kept slot lies past the budget in proportion: (L - keep) * keep / L of them move.
    moved = float((cut * (L - c["keep"]) * c["keep"] / L).sum())
    return {"bytes": int(L.sum()) * Hkv * 8 + int(np.minimum(L, c["keep"]).sum()) * Hkv * 8 + moved * Hkv * 4 * D * e, "flops": 0}


def exact(case, seed):
    """The operators from their definitions in 64 bits, one sequence and head at a time."""
    s = prepare(case, seed)
    c = s["c"]
    B, Hq, Hkv, D, P = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"]
    G, start, table = Hq // Hkv, np.concatenate([[0], np.cumsum(s["nq"])]), s["table"].long()

    def cached(pages, b, h):
        L = int(s["L"][b])
        return pages[table[b, : -(-L // P)], h].reshape(-1, D)[:L].double()

    if c["op"] == "append":
        K, V = s["k"].double(), s["v"].double()
        Q = torch.empty(s["T"], Hq * D, device=K.device, dtype=torch.float64)
        half = c["rot"] // 2
        i = torch.arange(half, device=K.device)
        ia, ib = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        for b in range(B):
            r, L = slice(int(start[b]), int(start[b + 1])), int(s["L"][b])
            at = torch.arange(L - int(s["nq"][b]), L, device=K.device)
            co, si = s["cos_sin"][at, :half].double()[:, None], s["cos_sin"][at, half:].double()[:, None]

            def turned(x, w, H):
                x = x[r].double().reshape(-1, H, D)
                if w is not None:
                    x = x / ((x * x).sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
                y = x.clone()
                y[..., ia], y[..., ib] = x[..., ia] * co - x[..., ib] * si, x[..., ia] * si + x[..., ib] * co
                return y

            Q[r] = turned(s["q_in"], s.get("qw"), Hq).reshape(-1, Hq * D)
            K[table[b, at // P], :, at % P] = turned(s["k_in"], s.get("kw"), Hkv)
            V[table[b, at // P], :, at % P] = s["v_in"][r].double().reshape(-1, Hkv, D)
        return Q, K, V
    if c["op"] == "attend":
        out = torch.empty(s["T"], Hq, D, device=s["q"].device, dtype=torch.float64)
        lse = torch.empty(s["T"], Hq, device=s["q"].device, dtype=torch.float64)
        q = s["q"].view(-1, Hq, D)
        for b in range(B):
            if not s["nq"][b]:
                continue
            L, n = int(s["L"][b]), int(s["nq"][b])
            j = torch.arange(L, device=out.device)[None]
            p = torch.arange(L - n, L, device=out.device)[:, None]
            hidden = j > p
            if c["window"]:
                hidden |= (j <= p - c["window"]) & (j >= c["sinks"])
            r = slice(int(start[b]), int(start[b + 1]))
            for h in range(Hkv):
                K, V = cached(s["k"], b, h), cached(s["v"], b, h)
                for x in range(h * G, (h + 1) * G) if n > 64 else [slice(h * G, (h + 1) * G)]:
                    z = torch.einsum("t...d,jd->t...j", q[r, x].double(), K) * s["scale"]
                    z[hidden if z.dim() == 2 else hidden[:, None].expand_as(z)] = NEG
                    lse[r, x] = torch.logsumexp(z, -1)
                    out[r, x] = torch.softmax(z, -1) @ V
        return out.reshape(s["T"], Hq * D), lse
    if c["op"] == "weigh":
        W = torch.zeros_like(s["weight"], dtype=torch.float64)
        for b in range(B):
            L, m, r0 = int(s["L"][b]), int(s["rows"][b]), int(start[b])
            at = torch.arange(L - int(s["nq"][b]), L, device=W.device)[:m, None, None]
            j = torch.arange(L, device=W.device)[None, None]
            for h in range(Hkv):
                q = s["q"].view(-1, Hq, D)[r0 : r0 + m, h * G : (h + 1) * G].double()
                z = q @ cached(s["k"], b, h).T * s["scale"] - s["lse"][r0 : r0 + m, h * G : (h + 1) * G, None].double()
                W[b, h, :L] = s["weight"][b, h, :L].double() + (z.exp() * (j <= at)).sum((0, 1))
        return W
    # Choosing and moving compute no numbers: the weights and the rows that stay are the inputs' own.
    weight, pos = s["weight"].cpu().numpy(), s["pos"].cpu().numpy()
    W = np.zeros(weight.shape)
    to, fro = [], []
    page = table.cpu().numpy()
    for b in range(B):
        L = int(s["L"][b])
        for h in range(Hkv):
            w, p = weight[b, h, :L], pos[b, h, :L]
            first = (p < c["sinks"]) | (p > p.max() - c["recent"])
            best = np.lexsort((np.arange(L), -w.astype(np.float64), ~first))[: c["keep"]]
            stay = np.zeros(L, bool)
            stay[best] = True
            slot = np.arange(L)
            take = slot[: min(L, c["keep"])].copy()
            src = slot[stay & (slot >= c["keep"])]
            dst = take[~stay[: len(take)]]
            take[dst] = src
            W[b, h, : len(take)] = w[take]
            to.append((page[b, dst // P] * Hkv + h) * P + dst % P)
            fro.append((page[b, src // P] * Hkv + h) * P + src % P)
    to, fro = (torch.tensor(np.concatenate(x), device=s["k"].device) for x in (to, fro))
    K, V = s["k"].double().view(-1, D), s["v"].double().view(-1, D)
    K[to], V[to] = K[fro], V[fro]
    return None, torch.tensor(W), None, K.view(s["k"].shape), V.view(s["v"].shape)
