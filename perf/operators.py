"""Performance cases of decoding on a compacted cache: attention of new tokens over it, with an account of what weight every
cached token gets (``attend``), the same for a batch of sequences that share a long context (``shared``), and eviction by that
account (``evict``).

A case is a dict of plain values.  ``run`` makes one pass: with ``own`` through the library, otherwise in elementary torch operations.
Heads are those of the package's own model pairs: 8 KV heads of 128 with 4 or 5 query heads each, 4 with 7, 8 of 64 with 4.
"""
import math

import torch

own = False
_context = None


def listed():
    return [
        # the smallest call: one sequence, a short cache, one new token; launches and latency
        {"name": "attend_short", "op": "attend", "rows": 4, "group": 4, "T": 1, "N": 512, "D": 128, "dtype": "bf16", "lens": "ragged", "weight": True},
        # one user's decoding step on a layer of a 32k context of which 30 % was kept, room for 410 new tokens
        {"name": "attend_10k", "op": "attend", "rows": 8, "group": 4, "T": 1, "N": 10240, "D": 128, "dtype": "bf16", "lens": "full", "weight": True},
        # 32 sequences side by side, caches of all lengths, one of them empty
        {"name": "attend_batch", "op": "attend", "rows": 256, "group": 4, "T": 1, "N": 8192, "D": 128, "dtype": "bf16", "lens": "ragged", "weight": True},
        # budgets of their own for every head, groups of seven, no account, half precision, an odd capacity
        {"name": "attend_pooled", "op": "attend", "rows": 112, "group": 7, "T": 1, "N": 5003, "D": 128, "dtype": "fp16", "lens": "ragged", "weight": False},
        # five drafted tokens checked at once, heads of 64
        {"name": "attend_draft", "op": "attend", "rows": 64, "group": 4, "T": 5, "N": 4001, "D": 64, "dtype": "bf16", "lens": "ragged", "weight": True},
        # the largest: a further question of 512 tokens read in on a compacted context
        {"name": "attend_chunk", "op": "attend", "rows": 8, "group": 4, "T": 512, "N": 10343, "D": 128, "dtype": "bf16", "lens": "full", "weight": True},
        # a few sequences on a short shared context, heads of 64, one sequence without tokens of its own
        {"name": "shared_1k", "op": "shared", "batch": 3, "heads": 8, "group": 4, "T": 1, "P": 1001, "N": 77, "D": 64, "dtype": "fp16", "lens": "ragged", "weight": False},
        # eight answers drawn from one compacted 32k context
        {"name": "shared_10k", "op": "shared", "batch": 8, "heads": 8, "group": 4, "T": 1, "P": 9830, "N": 512, "D": 128, "dtype": "bf16", "lens": "ragged", "weight": True},
        # a document that 64 users ask about, answers of up to 1000 tokens
        {"name": "shared_32k", "op": "shared", "batch": 64, "heads": 8, "group": 4, "T": 1, "P": 32768, "N": 1000, "D": 128, "dtype": "bf16", "lens": "ragged", "weight": True},
        # one layer of one sequence, 64 tokens over its budget
        {"name": "evict_layer", "op": "evict", "rows": 8, "N": 1088, "budget": 1024, "recent": 128, "D": 128, "dtype": "bf16", "lens": "full"},
        # all layers of one sequence, 256 tokens over the budget
        {"name": "evict_model", "op": "evict", "rows": 256, "N": 4352, "budget": 4096, "recent": 512, "D": 128, "dtype": "bf16", "lens": "full"},
        # long rows of all lengths cut to a third of the longest, some not that long
        {"name": "evict_long", "op": "evict", "rows": 112, "N": 30001, "budget": 9999, "recent": 333, "D": 128, "dtype": "bf16", "lens": "ragged"},
    ]


def draw(rng):
    """One more case: lengths spread over their logarithm, every operator, type and head layout that is listed."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "shared", "evict"])
    case = {"op": op, "D": rng.choice([64, 128, 128]), "dtype": rng.choice(["bf16", "bf16", "fp16"]), "lens": rng.choice(["full", "ragged"])}
    if op == "evict":
        case["rows"] = log_int(1, 300)
        case["N"] = min(log_int(200, 40000), 1600000 // case["rows"])
        case["budget"] = max(1, int(case["N"] * rng.choice([rng.uniform(0.2, 0.6), rng.uniform(0.9, 0.99)])))
        case["recent"] = min(case["budget"], log_int(1, 1024))
        return case
    case["group"] = rng.choice([1, 4, 4, 5, 7, 8])
    case["T"] = rng.choice([1, 1, 1, log_int(2, 8), log_int(16, 400)])
    case["weight"] = rng.random() < 0.6
    if op == "attend":
        case["rows"] = log_int(1, 300)
        most = min(1000000 // case["rows"], 30000000 // (case["rows"] * case["group"] * case["T"]))
        case["N"] = min(log_int(100, 40000), max(most, 100))
    else:
        case["heads"], case["batch"] = rng.choice([1, 4, 8]), log_int(2, 64)
        case["T"] = min(case["T"], 8)
        queries = case["batch"] * case["heads"] * case["group"] * case["T"]
        case["P"] = min(log_int(100, 40000), 60000000 // queries)
        case["N"] = min(log_int(max(16, case["T"]), 2000), 1000000 // (case["batch"] * case["heads"]))
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _lens(case, rows, most, least):
    """Tokens of every row, the same for every seed: full rows, or lengths spread over the whole range, one at either end."""
    if case["lens"] == "full":
        return [most] * rows
    span = [least + int((most - least) * math.modf(0.31 + 0.6180339887 * r)[0]) for r in range(rows)]
    span[0] = most
    if rows > 2:
        span[2] = least
    return span


def _dims(case):
    """(batch, heads): a call of ``attend`` is one sequence after the other, rows of their own."""
    return (case["batch"], case["heads"]) if case["op"] == "shared" else (1, case["rows"])


def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _keys(q, shape, dtype, g):
    """Keys of unit variance; one in 200 leans towards a query of its group: a heavy hitter.  q [rows, queries, D], shape [rows, N, D]."""
    k = _normal(shape, dtype, g)
    rows, N, D = shape
    P = N // 200
    if P:
        pos = torch.randint(N, (rows, 1, 1), generator=g, device="cuda") + 200 * torch.arange(P, device="cuda").view(1, P, 1)
        src = torch.randint(q.shape[1], (rows, P, 1), generator=g, device="cuda")
        k.scatter_(1, (pos % N).expand(-1, -1, D), (0.5 * torch.gather(q, 1, src.expand(-1, -1, D)).float() + _normal((rows, P, D), torch.float32, g)).to(dtype))
    return k


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt, D, N = _dtype(case), case["D"], case["N"]
    s = {"case": dict(case)}
    if case["op"] == "evict":
        R = case["rows"]
        s["k"], s["v"] = _normal((R, N, D), dt, g), _normal((R, N, D), dt, g)
        s["lens_grown"] = torch.tensor(_lens(case, R, N, case["recent"]), dtype=torch.int32, device="cuda")
        # what attention has left on every token: a skewed account; in every fourth row it is coarse, so that many are level
        w = torch.exp(1.5 * torch.randn(R, N, generator=g, device="cuda") - 2.0)
        w[3::4] = torch.round(w[3::4] * 8) / 8
        s["weight_grown"] = w
        s["weight"], s["lens"] = w.clone(), s["lens_grown"].clone()
        s["positions"] = torch.arange(N, dtype=torch.int32, device="cuda").expand(R, N).contiguous()
        return s
    B, H = _dims(case)
    G, T = case["group"], case["T"]
    s["q"] = _normal((B, H, G, T, D), dt, g)
    qr = s["q"].view(B * H, G * T, D)
    s["k"], s["v"] = _keys(qr, (B * H, N, D), dt, g).view(B, H, N, D), _normal((B, H, N, D), dt, g)
    least = 0 if B * H > 2 and T == 1 else min(T, N)
    s["lens"] = torch.tensor(_lens(case, B * H, N, least), dtype=torch.int32, device="cuda").view(B, H)
    s["weight"] = torch.rand(B, H, N, generator=g, device="cuda") if case["weight"] else None
    if case["op"] == "shared":
        P = case["P"]
        qs = s["q"].transpose(0, 1).reshape(H, B * G * T, D)
        s["k_shared"], s["v_shared"] = _keys(qs, (H, P, D), dt, g), _normal((H, P, D), dt, g)
        s["weight_shared"] = torch.rand(H, P, generator=g, device="cuda") if case["weight"] else None
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def _ctx(pk):
    """The library's context, which a program keeps."""
    global _context
    if _context is None:
        _context = pk.proxykv_create(pk.make_config(16, 32, 8, 64, 32, 8, 128))
    return _context


def run(state):
    op = state["case"]["op"]
    return {"attend": _attend, "shared": _shared, "evict": _evict}[op](state)


def _own_visible(s):
    """[B, H, 1, T, N]: own tokens that query t of a row sees; the T new ones are the last of the row."""
    T, N = s["case"]["T"], s["case"]["N"]
    n, t = torch.arange(N, device="cuda"), torch.arange(T, device="cuda")
    return n.view(1, 1, 1, 1, N) < (s["lens"].view(*s["lens"].shape, 1, 1, 1) - T + 1 + t.view(1, 1, 1, T, 1))


def _attend(s):
    c = s["case"]
    if own:
        from paper_2605_16360_amd import binding as pk
        rows = lambda x: None if x is None else x[0]  # noqa: E731
        before = max(c["T"] - c["N"], 0)  # tokens in front of all that the cache has room for: they see nothing, and the call takes no more than it holds
        q = s["q"][0, :, :, before:].contiguous() if before else s["q"][0]
        out = pk.proxykv_attend(_ctx(pk), q, s["k"][0], s["v"][0], lens=None if c["lens"] == "full" else s["lens"][0], weight=rows(s["weight"]))
        if before:
            out = torch.nn.functional.pad(out, (0, 0, before, 0))
        return {"out": out.unsqueeze(0), "weight": s["weight"]}
    B, H, G, T, D = s["q"].shape
    k, v = s["k"].float(), s["v"].float()
    x = torch.matmul(s["q"].float().view(B, H, G * T, D), k.transpose(2, 3)).view(B, H, G, T, -1) * (1.0 / math.sqrt(D))
    x = torch.where(_own_visible(s), x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total == 0, 1.0, total)
    if s["weight"] is not None:
        s["weight"] += p.sum((2, 3))
    out = torch.matmul(p.view(B, H, G * T, -1), v).view(B, H, G, T, D)
    return {"out": out.to(s["q"].dtype), "weight": s["weight"]}


def _shared(s):
    c = s["case"]
    if own:
        from paper_2605_16360_amd import binding as pk
        out = pk.proxykv_attend_shared(_ctx(pk), s["q"], s["k_shared"], s["v_shared"], s["k"], s["v"], lens=None if c["lens"] == "full" else s["lens"],
                                       weight_shared=s["weight_shared"], weight=s["weight"])
        return {"out": out, "weight": s["weight"], "weight_shared": s["weight_shared"]}
    B, H, G, T, D = s["q"].shape
    q = s["q"].float()
    flat = q.transpose(0, 1).reshape(H, B * G * T, D)
    scale = 1.0 / math.sqrt(D)
    xs = (torch.matmul(flat, s["k_shared"].float().transpose(1, 2)) * scale).view(H, B, G, T, -1).transpose(0, 1)
    xo = torch.matmul(q.view(B, H, G * T, D), s["k"].float().transpose(2, 3)).view(B, H, G, T, -1) * scale
    xo = torch.where(_own_visible(s), xo, -math.inf)
    top = torch.maximum(xs.amax(-1, keepdim=True), xo.amax(-1, keepdim=True))
    es, eo = torch.exp(xs - top), torch.exp(xo - top)
    total = es.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    ps, po = es / total, eo / total
    if s["weight"] is not None:
        s["weight_shared"] += ps.sum((0, 2, 3))
        s["weight"] += po.sum((2, 3))
    out = torch.matmul(ps.transpose(0, 1).reshape(H, B * G * T, -1), s["v_shared"].float()).view(H, B, G, T, D).transpose(0, 1)
    out = out + torch.matmul(po.view(B, H, G * T, -1), s["v"].float()).view(B, H, G, T, D)
    return {"out": out.to(s["q"].dtype), "weight": s["weight"], "weight_shared": s["weight_shared"]}


def _evict(s):
    c = s["case"]
    # the tokens decoded since the last eviction have brought the rows to these lengths and their tokens to this account again
    s["weight"].copy_(s["weight_grown"])
    s["lens"].copy_(s["lens_grown"])
    if own:
        from paper_2605_16360_amd import binding as pk
        pk.proxykv_evict(_ctx(pk), s["k"], s["v"], s["weight"], s["lens"], c["budget"], c["recent"], positions=s["positions"])
    else:
        R, N = s["weight"].shape
        n = torch.arange(N, device="cuda")
        cand = (s["lens"] - c["recent"]).view(R, 1)
        keep = c["budget"] - c["recent"]
        key = torch.where(n < cand, s["weight"], -math.inf)  # (weights are finite)
        order = torch.sort(key, dim=1, descending=True, stable=True).indices
        kept = torch.zeros(R, N, dtype=torch.bool, device="cuda").scatter_(1, order[:, :keep], True) & (n < cand)
        over = s["lens"].view(R, 1) > c["budget"]
        hole, filler = ~kept & (n < keep) & over, kept & (n >= keep) & over
        # the j-th token kept beyond the first `keep` slots goes to the j-th slot given up among them
        which = torch.where(filler, n, N).sort(dim=1).values
        source = torch.where(hole, torch.gather(which, 1, (hole.cumsum(1) - 1).clamp_min(0)), n)
        source = torch.where(over & (n >= keep) & (n < c["budget"]), n - keep + cand, source)
        wide = source.unsqueeze(2).expand_as(s["k"])
        s["k"].copy_(torch.gather(s["k"], 1, wide))
        s["v"].copy_(torch.gather(s["v"], 1, wide))
        s["weight"].copy_(torch.gather(s["weight"], 1, source))
        s["positions"].copy_(torch.gather(s["positions"], 1, source))
        s["lens"].clamp_max_(c["budget"])
    return {x: s[x] for x in ("k", "v", "weight", "positions", "lens")}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    D, N = case["D"], case["N"]
    if case["op"] == "evict":
        lens, b, r = _lens(case, case["rows"], N, case["recent"]), case["budget"], case["recent"]
        over = [n for n in lens if n > b]
        moved = sum((b - r) * (n - b) / (n - r) + r for n in over)  # tokens kept behind the first b - r slots, and the recent ones
        return {"bytes": 4 * sum(n - r for n in over) + moved * (8 * D + 16), "flops": 0}
    B, H = _dims(case)
    G, T = case["group"], case["T"]
    tokens = sum(_lens(case, B * H, N, 0 if B * H > 2 and T == 1 else min(T, N)))
    pairs, account, q = tokens * G * T, tokens, B * H * G * T
    if case["op"] == "shared":
        tokens += H * case["P"]
        account += H * case["P"]
        pairs += H * case["P"] * B * G * T
    return {"bytes": 4 * D * tokens + (8 * account if case["weight"] else 0) + 4 * D * q, "flops": 4 * D * pairs}


# ---- the definitions in 64 bits, a row at a time --------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(s, case)
    B, H, G, T, D = s["q"].shape
    out = torch.zeros(B, H, G * T, D, dtype=torch.float64, device="cuda")
    account = None if s["weight"] is None else s["weight"].double()
    account_shared = s["weight_shared"].double() if s.get("weight_shared") is not None else None
    lens = s["lens"].tolist()
    for h in range(H):
        ks, vs = (s["k_shared"][h].double(), s["v_shared"][h].double()) if case["op"] == "shared" else (None, None)
        for b in range(B):
            n = lens[b][h]
            k, v = s["k"][b, h, :n].double(), s["v"][b, h, :n].double()
            if ks is not None:
                k, v = torch.cat([ks, k]), torch.cat([vs, v])
            first = k.shape[0] - n
            q = s["q"][b, h].reshape(G * T, D).double()
            logits = q.mm(k.t()) / D ** 0.5
            last = first + n - T + torch.arange(T, device="cuda").repeat(G)  # the last token that a query sees
            logits.masked_fill_(torch.arange(k.shape[0], device="cuda")[None, :] > last[:, None], -math.inf)
            p = torch.exp(logits - torch.logsumexp(logits, 1, keepdim=True)).nan_to_num(0.0) if k.shape[0] else logits
            out[b, h] = p.mm(v)
            if account is not None:
                account[b, h, :n] += p[:, first:].sum(0)
            if account_shared is not None:
                account_shared[h] += p[:, :first].sum(0)
    r = {"out": out.view(B, H, G, T, D), "weight": account}
    if case["op"] == "shared":
        r["weight_shared"] = account_shared
    return r


def _exact_evict(s, case):
    budget, recent = case["budget"], case["recent"]
    lens, weights = s["lens_grown"].tolist(), s["weight_grown"].cpu().numpy()
    r = {x: s[x].clone() for x in ("k", "v", "weight", "positions", "lens")}
    for i, n in enumerate(lens):
        if n <= budget:
            continue
        cand, keep = n - recent, budget - recent
        best = sorted(range(cand), key=(-weights[i, :cand].astype("float64")).__getitem__)[:keep]  # (a stable sort)
        there, further = set(x for x in best if x < keep), sorted(x for x in best if x >= keep)
        free = [x for x in range(keep) if x not in there]
        to = torch.tensor(free + list(range(keep, budget)), dtype=torch.int64, device="cuda")
        at = torch.tensor(further + list(range(cand, n)), dtype=torch.int64, device="cuda")
        for x in ("k", "v", "weight", "positions"):
            r[x][i, to] = s[x][i, at]
        r["lens"][i] = budget
    return r
