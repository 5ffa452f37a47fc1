"""Cases of the operators around a verification pass: the norm that makes the hidden states, the scores that are read off
them, and the attention of a batch that shares its beginning.

`norm`: residual addition and root-mean-square norm, output in bf16 and / or in 8 bits (e4m3) with a scale per row.
`score`: through the LM head, log probabilities of given tokens, entropy and the most likely alternatives of each row.
`shared`: attention over a paged cache whose first slots are the same pages for every sequence.
`run` computes them in plain torch, or with `own` through the framework.
"""
import math

import numpy as np
import torch

own = False

NEG = float("-inf")


def _norm(rows, d, **kw):
    return {"op": "norm", "rows": rows, "d": d, "dtype": "bf16", "residual": True, "wide": True, "narrow": False, **kw}


def _score(rows, d, V, **kw):
    return {"op": "score", "rows": rows, "d": d, "V": V, "dtype": "bf16", "n_tok": 1, "n_top": 5, "temperature": 1.0, **kw}


def _shared(B, n, shared, lo, hi, **kw):
    return {"op": "shared", "B": B, "n": n, "ragged_n": False, "shared": shared, "lo": lo, "hi": hi, "Hq": 32, "Hkv": 8, "D": 128,
            "page": 16, **kw}


def listed():
    return [
        # One token of one user between two layers: nothing but latency.
        _norm(1, 4096, name="norm 1 row"),
        # The final norm of 64 verification windows of 33 rows, for a verification in bf16 and a scoring in 8 bits.
        _norm(2112, 4096, narrow=True, name="norm 64x33 rows, both"),
        # Prompts of the large shape on their way into a product in 8 bits.
        _norm(16000, 8192, wide=False, narrow=True, name="norm 16000 rows to 8 bits"),
        # The small configuration: a window of five rows in 32 bits.
        _score(5, 256, 1000, dtype="f32", name="score 5 rows, f32, small head"),
        # One user's window of 16 draft tokens against the full head, with alternatives to show.
        _score(17, 4096, 128256, n_top=8, name="score 17 rows"),
        # Eight windows of 33 rows, four candidates per position (a tree's children), only the best alternative.
        _score(264, 4096, 128256, n_tok=4, n_top=1, name="score 8x33 rows"),
        # 64 windows of 33 rows under a temperature.
        _score(2112, 4096, 128256, n_top=5, temperature=0.7, name="score 64x33 rows"),
        # One user's window against a head in 8 bits.
        _score(17, 4096, 128256, dtype="e4m3", n_top=8, name="score 17 rows, 8 bits"),
        # A prompt's own tokens, as an evaluation scores them, 8 bits.
        _score(4096, 4096, 128256, dtype="e4m3", n_top=0, name="score 4096 rows, 8 bits"),
        # 64 users decode behind the same few-shot examples.
        _shared(64, 1, 2048, 1, 500, name="shared 64x1 behind 2048"),
        # 32 verification windows of 33 rows behind a shorter prefix whose end lies inside a tile.
        _shared(32, 33, 1504, 33, 600, page=32, name="shared 32x33 behind 1504"),
        # Eight questions of different length enter the cache behind a long document.
        _shared(8, 384, 8192, 0, 384, ragged_n=True, page=64, name="shared 8 prompts behind 8192"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "score", "score", "shared", "shared"])
    if op == "norm":
        d = 8 * _log(rng, 32, 1024)
        rows = _log(rng, 1, max(2, min(16000, 16000 * 8192 // d)))
        wide, narrow = rng.choice([(True, False), (True, True), (False, True)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return _norm(max(1, rows // 2) if dtype == "f32" else rows, d, dtype=dtype, residual=rng.random() < 0.8, wide=wide, narrow=narrow)
    if op == "score":
        d = 64 * _log(rng, 4, 128)
        V = rng.choice([128256, 32000 + rng.randrange(1000), _log(rng, 1000, 128256)])
        dtype = rng.choice(["bf16", "bf16", "e4m3"])
        most = min(2112, 2112 * 4096 * 128256 // (d * V))
        return _score(_log(rng, 1, max(2, most)), d, V, dtype=dtype, n_tok=rng.choice([1, 1, 2, 5]), n_top=rng.choice([0, 1, 5, 20]),
                      temperature=rng.choice([1.0, 1.0, 0.6, 1.3]))
    D, Hq, page = rng.choice([64, 128, 128]), rng.choice([32, 32, 64]), rng.choice([16, 32, 64])
    kind = rng.choice(["one", "window", "prompt"])
    if kind == "one":
        B, n = _log(rng, 2, 128), rng.choice([1, 1, 2])
        hi = n + _log(rng, 1, max(2, min(4096, 64000 // B)))
    elif kind == "window":
        n = rng.choice([5, 9, 17, 33, 65])
        B = _log(rng, 2, max(3, 2048 // n))
        hi = n + _log(rng, 1, max(2, min(2048, 64000 // B)))
    else:
        B, n = rng.choice([2, 4, 8]), _log(rng, 50, 384)
        hi = n
    most = 8 * 192 * 32 * 8192 // (B * n * Hq)  # rows x prefix of the largest listed case
    shared = page * _log(rng, 4, max(5, min(8192, most) // page))
    return _shared(B, n, shared, 0 if kind == "prompt" else n, hi, ragged_n=kind == "prompt", Hq=Hq, D=D, page=page)


# ------------------------------------------------------------------------------------ inputs


def _lengths(c, rng):
    """New tokens and own slots (behind the prefix, the new tokens among them) of each sequence: the case fixes which there are,
    the seed which sequence has which."""
    B, n = c["B"], c["n"]
    L = np.random.default_rng([c["lo"], c["hi"], B, n]).integers(c["lo"], c["hi"] + 1, B)
    L[0] = c["hi"]
    L = rng.permutation(L)
    return (L.copy(), L) if c["ragged_n"] else (np.full(B, n), np.maximum(L, n))


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    dt = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[c.get("dtype", "bf16")]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=dev, dtype=torch.float32)

    s = {"c": c}
    if c["op"] == "norm":
        rows, d = c["rows"], c["d"]
        # a few channels are far larger than the others, as in the residual stream of a language model
        loud = torch.where(uniform(d) < 0.004, 30.0, 1.0)
        s["x"] = (normal(rows, d) * loud).to(dt)
        s["r"] = (3 * normal(rows, d) * loud).to(dt) if c["residual"] else None
        s["w"] = 1 + 0.2 * normal(d)
        s["r_out"] = torch.zeros(rows, d, device=dev, dtype=dt) if c["residual"] else None
        s["out"] = torch.zeros(rows, d, device=dev, dtype=dt) if c["wide"] else None
        s["out8"] = torch.zeros(rows, d, device=dev, dtype=torch.float8_e4m3fn) if c["narrow"] else None
        s["scale8"] = torch.zeros(rows, device=dev) if c["narrow"] else None
        return s
    if c["op"] == "score":
        rows, d, V, eight = c["rows"], c["d"], c["V"], c["dtype"] == "e4m3"
        # Weights and states lie on the grid of a checkpoint in 8 bits (scales are powers of two), so that a logit is
        # the same number in whatever order its products are added, and the order of near alternatives is well defined.
        # Each state leans towards a token, some strongly and some not at all.
        lean = torch.randint(V, (rows,), generator=g, device=dev)
        strength = 14 * uniform(rows, 1)
        if eight:
            W = (40 * normal(V, d)).round_().clamp_(-240, 240).to(dt)
            s["w_scale"] = 2.0 ** -torch.randint(11, 13, (V,), generator=g, device=dev).float()
            s["h_scale"] = 2.0 ** -torch.randint(7, 9, (rows,), generator=g, device=dev).float()
            h = 100 * normal(rows, d) + W[lean].float() * (strength * 2.0**18 / (1600 * d))
            s["h"] = h.round_().clamp_(-448, 448).to(dt)
        else:
            W = (41 * normal(V, d)).round_().clamp_(-127, 127).mul_(2.0**-11).to(dt)
            h = normal(rows, d) + W[lean].float() * (strength / (0.0004 * d))
            s["h"] = h.mul_(16).round_().clamp_(-127, 127).mul_(1 / 16).to(dt)
        s["W"] = W
        tokens = torch.randint(V, (rows, c["n_tok"]), generator=g, device=dev)
        tokens[:, 0] = torch.where(uniform(rows) < 0.7, lean, tokens[:, 0])
        s["tokens"] = tokens.to(torch.int32)
        s["logprob"], s["entropy"], s["lse"] = torch.zeros(rows, c["n_tok"], device=dev), torch.zeros(rows, device=dev), torch.zeros(rows, device=dev)
        s["top_id"] = torch.zeros(rows, c["n_top"], device=dev, dtype=torch.int32) if c["n_top"] else None
        s["top_logprob"] = torch.zeros(rows, c["n_top"], device=dev) if c["n_top"] else None
        if own:
            import paper_2504_20039_b200 as aj

            s["handle"] = aj.ScoreHandle(torch.cuda.current_device(), rows, d, V, {"bf16": aj.AJ_BF16, "f32": aj.AJ_F32, "e4m3": aj.AJ_E4M3}[c["dtype"]],
                                         max_top=c["n_top"])
        return s
    rng = np.random.default_rng([int(seed), 78])
    nq, L = _lengths(c, rng)
    B, Hq, Hkv, D, page, S = c["B"], c["Hq"], c["Hkv"], c["D"], c["page"], c["shared"]
    first = S // page  # pages of the prefix
    need = -(-L // page)
    width = first + max(1, -(-int(max(L.max(), c["hi"])) // page))
    n_pages = first + int(need.sum()) + 3
    perm = rng.permutation(n_pages)
    table = np.zeros((B, width), np.int32)
    table[:, :first] = perm[:first]
    at = first
    for b in range(B):
        table[b, first : first + need[b]] = perm[at : at + need[b]]
        at += need[b]
    T = int(nq.sum())
    start = np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)
    row_b = np.repeat(np.arange(B), nq)
    s.update(nq=nq, L=L, T=T, max_n=max(1, int(nq.max())), width=width, start=torch.tensor(start, device=dev), table=torch.tensor(table, device=dev),
             prefix=torch.tensor(table[0, :first].copy(), device=dev), lens=torch.tensor(S + L, dtype=torch.int32, device=dev),
             row_b=torch.tensor(row_b, device=dev), row_t=torch.tensor(np.arange(T) - start[row_b], device=dev), scale=1.0 / math.sqrt(D))
    s["k"], s["v"] = normal(n_pages, Hkv, page, D).to(dt), normal(n_pages, Hkv, page, D).to(dt)
    s["q"] = (2 * normal(T, Hq * D)).to(dt)
    s["out"], s["lse"] = torch.zeros(T, Hq * D, device=dev, dtype=dt), torch.zeros(T, Hq, device=dev)
    if own:
        import paper_2504_20039_b200 as aj

        s["handle"] = aj.KvHandle(torch.cuda.current_device(), B, s["max_n"], Hq, Hkv, D, page)
        s["handle"].reserve_shared(T)
    return s


# ------------------------------------------------------------------------------- plain forms


def _norm_plain(s):
    c = s["c"]
    x = s["x"].float()
    if c["residual"]:
        x = x + s["r"].float()
    got = [x.to(s["x"].dtype)] if c["residual"] else []
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * s["w"]
    if c["wide"]:
        got.append(y.to(s["x"].dtype))
    if c["narrow"]:
        scale = y.abs().amax(-1) / 448
        got += [(y / scale[:, None]).clamp_(-448, 448).to(torch.float8_e4m3fn), scale]
    return got


def _score_plain(s):
    c = s["c"]
    x = s["h"].float() @ s["W"].float().T
    if c["dtype"] == "e4m3":
        x.mul_(s["h_scale"][:, None]).mul_(s["w_scale"])
    got = {}
    if c["n_top"]:
        # one whole number per entry: the logit's order above, the lower index first below
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long().bitwise_left_shift_(32)
        key += torch.arange(c["V"] - 1, -1, -1, device=x.device)
        ids = c["V"] - 1 - (key.topk(c["n_top"]).values & 0xFFFFFFFF)
        got["top_id"] = ids.to(torch.int32)
    z = x.mul_(1 / c["temperature"])
    given = z.gather(1, s["tokens"].long())
    best = z.gather(1, ids) if c["n_top"] else None
    m = z.amax(-1, keepdim=True)
    z = z.sub_(m)
    e = z.exp()
    S = e.sum(-1)
    log_s = S.log()
    got["lse"] = m[:, 0] + log_s
    got["logprob"] = given - got["lse"][:, None]
    got["entropy"] = log_s - e.mul_(z).sum(-1) / S
    if c["n_top"]:
        got["top_logprob"] = best - got["lse"][:, None]
    return got


def _pages(pages, table):
    """Slots in order, [..., Hkv, slots, D] in 32 bits, of the pages that a table [..., n] names."""
    x = pages[table.long()].transpose(-4, -3)
    return x.reshape(*x.shape[:-3], -1, x.shape[-1]).float()


def _shared_plain(s):
    c = s["c"]
    B, n, Hq, Hkv, D, S = c["B"], s["max_n"], c["Hq"], c["Hkv"], c["D"], c["shared"]
    G, first = Hq // Hkv, S // c["page"]
    q = torch.zeros(B, n, Hq, D, device=s["q"].device)
    q[s["row_b"], s["row_t"]] = s["q"].float().view(-1, Hq, D)
    q = q.view(B, n, Hkv, G, D).permute(2, 0, 1, 3, 4) * s["scale"]  # [Hkv, B, n, G, D]
    x1 = q.reshape(Hkv, B * n * G, D) @ _pages(s["k"], s["prefix"]).transpose(-1, -2)
    own_table = s["table"][:, first:]
    K, V = _pages(s["k"], own_table).transpose(0, 1), _pages(s["v"], own_table).transpose(0, 1)  # [Hkv, B, slots, D]
    x2 = q.reshape(Hkv, B, n * G, D) @ K.transpose(-1, -2)
    nq = s["start"][1:] - s["start"][:-1]
    pos = (s["lens"] - S - nq)[:, None] + torch.arange(n, device=q.device)  # [B, n]
    hidden = torch.arange(K.shape[2], device=q.device) > pos[..., None]
    x2 = x2.masked_fill_(hidden.repeat_interleave(G, 1), NEG)
    x1 = x1.view(Hkv, B, n * G, S)
    m = torch.maximum(x1.amax(-1, keepdim=True), x2.amax(-1, keepdim=True))
    x1, x2 = x1.sub_(m).exp_(), x2.sub_(m).exp_()
    total = x1.sum(-1, keepdim=True) + x2.sum(-1, keepdim=True)
    o = (x1.view(Hkv, B * n * G, S) @ _pages(s["v"], s["prefix"])).view(Hkv, B, n * G, D)
    o = (o + x2 @ V) / total
    lse = (total.log() + m).view(Hkv, B, n, G).permute(1, 2, 0, 3).reshape(B, n, Hq)
    o = o.view(Hkv, B, n, G, D).permute(1, 2, 0, 3, 4).reshape(B, n, Hq * D)
    return o[s["row_b"], s["row_t"]].to(s["q"].dtype), lse[s["row_b"], s["row_t"]]


def run(s):
    c = s["c"]
    if not own:
        return _norm_plain(s) if c["op"] == "norm" else _score_plain(s) if c["op"] == "score" else _shared_plain(s)
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "norm":
        import paper_2504_20039_b200 as aj

        aj.add_norm(s["x"], s["w"], 1e-5, out=s["out"], residual=s["r"], residual_out=s["r_out"], out8=s["out8"], scale8=s["scale8"], stream=stream)
        return [t for t in (s["r_out"], s["out"], s["out8"], s["scale8"]) if t is not None]
    if c["op"] == "score":
        s["handle"].score(s["h"], s["W"], s["tokens"], s["logprob"], lse=s["lse"], entropy=s["entropy"], top_id=s["top_id"],
                          top_logprob=s["top_logprob"], inv_temperature=1 / c["temperature"], h_scale=s.get("h_scale"), w_scale=s.get("w_scale"),
                          stream=stream)
        return {k: s[k] for k in ("top_id", "lse", "logprob", "entropy", "top_logprob") if s[k] is not None}
    s["handle"].attend_shared(s["q"], s["k"], s["v"], s["prefix"], c["shared"], s["table"], s["lens"], s["out"], c["B"], s["max_n"], s["scale"],
                              q_start=s["start"] if c["ragged_n"] else None, lse=s["lse"], stream=stream)
    return s["out"], s["lse"]


# --------------------------------------------------------------------------- work and 64 bits


def work(case):
    """Weights, states and visible keys and values once, results once; what the mask hides is neither read nor multiplied."""
    c = dict(case)
    e = {"bf16": 2, "f32": 4, "e4m3": 1}[c.get("dtype", "bf16")]
    if c["op"] == "norm":
        n = c["rows"] * c["d"]
        return {"bytes": n * e * (1 + 2 * c["residual"] + c["wide"]) + (n + 4 * c["rows"]) * c["narrow"] + 4 * c["d"],
                "flops": n * (4 + c["residual"] + 2 * c["narrow"])}
    if c["op"] == "score":
        rows, d, V = c["rows"], c["d"], c["V"]
        scales = 4 * (rows + V) if e == 1 else 0
        return {"bytes": (V + rows) * d * e + scales + rows * (8 * c["n_tok"] + 8 * c["n_top"] + 8), "flops": 2 * rows * d * V}
    nq, L = _lengths(c, np.random.default_rng(1))
    T, D, Hq, Hkv = int(nq.sum()), c["D"], c["Hq"], c["Hkv"]
    pairs = T * c["shared"] + int((nq * L - nq * (nq - 1) // 2).sum())
    return {"bytes": (c["shared"] + int(L.sum())) * Hkv * D * 4 + 4 * T * Hq * D + 4 * T * Hq, "flops": 4 * pairs * Hq * D}


def exact(case, seed):
    """The operators from their definitions in 64 bits."""
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "norm":
        a = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
        y = a / ((a * a).sum(1, keepdim=True) / c["d"] + 1e-5).sqrt() * s["w"].double()
        got = [] if s["r"] is None else [a]
        if c["wide"]:
            got.append(y)
        if c["narrow"]:
            top = y.abs().max(1).values
            got += [y * (448 / top)[:, None], top / 448]
        return got
    if c["op"] == "score":
        rows, V = c["rows"], c["V"]
        logits = torch.empty(rows, V, device=s["h"].device, dtype=torch.float64)
        h = s["h"].double()
        for v in range(0, V, 16384):
            logits[:, v : v + 16384] = torch.mm(h, s["W"][v : v + 16384].double().t())
        if c["dtype"] == "e4m3":
            logits *= s["h_scale"].double()[:, None] * s["w_scale"].double()[None]
        got = {k: [] for k in ("lse", "logprob", "entropy", "top_logprob", "top_id")}
        for r in range(0, rows, 256):
            x = logits[r : r + 256]
            z = x / c["temperature"]
            logp = torch.log_softmax(z, -1)
            got["lse"].append(torch.logsumexp(z, -1))
            got["logprob"].append(logp.gather(1, s["tokens"][r : r + 256].long()))
            got["entropy"].append(-(logp.exp() * logp).sum(-1))
            if c["n_top"]:
                order = x.sort(dim=-1, descending=True, stable=True).indices[:, : c["n_top"]]
                got["top_id"].append(order.to(torch.int32))
                got["top_logprob"].append(logp.gather(1, order))
        return {k: torch.cat(v) for k, v in got.items() if v}
    B, Hq, Hkv, D, S = c["B"], c["Hq"], c["Hkv"], c["D"], c["shared"]
    G, page, start, table = Hq // Hkv, c["page"], s["start"].tolist(), s["table"].long()
    out = torch.empty(s["T"], Hq, D, device=s["q"].device, dtype=torch.float64)
    lse = torch.empty(s["T"], Hq, device=s["q"].device, dtype=torch.float64)
    q = s["q"].view(-1, Hq, D).double()
    for b in range(B):
        n, L = int(s["nq"][b]), S + int(s["L"][b])
        if not n:
            continue
        r = slice(start[b], start[b + 1])
        hidden = torch.arange(L, device=q.device)[None] > torch.arange(L - n, L, device=q.device)[:, None]
        for h in range(Hkv):
            K, V = (t[table[b, : -(-L // page)], h].reshape(-1, D)[:L].double() for t in (s["k"], s["v"]))
            i = slice(h * G, (h + 1) * G)
            z = torch.einsum("tgd,jd->tgj", q[r, i], K) * s["scale"]
            z[hidden[:, None].expand_as(z)] = NEG
            lse[r, i] = torch.logsumexp(z, -1)
            out[r, i] = torch.softmax(z, -1) @ V
    return out.reshape(s["T"], Hq * D), lse
