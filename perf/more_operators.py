"""Performance cases of long-lived rollouts: projections in 8-bit integers with a
scale for each token and each channel, the weight that attention gives to each
cached token, and the eviction of the tokens it gives least from a paged cache.

Every case is a dict of plain values; ``prepare`` makes the tensors a program
holds before the call, ``run`` makes one pass -- with ``own`` the framework's
operators, otherwise the same arithmetic in elementary torch operations -- and
``exact`` restates the result in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
F64 = torch.float64


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


# ------------------------------------------------------------------- cases
def _linear(name, dtype, tokens, n, k, epilogue):
    return {"name": name, "op": "linear", "dtype": dtype, "tokens": tokens, "n": n, "k": k, "epilogue": epilogue}


def _quantize(name, dtype, rows, k):
    return {"name": name, "op": "quantize", "dtype": dtype, "rows": rows, "k": k}


def _weigh(name, dtype, heads, kv_heads, head_dim, page, branches, n_q, shared, own_min, own_max, causal):
    return {"name": name, "op": "weigh", "dtype": dtype, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "branches": branches, "n_q": n_q, "shared": shared,
            "own_min": own_min, "own_max": own_max, "causal": causal}


def _evict(name, dtype, layers, kv_heads, head_dim, page, seqs, shared, own_min, own_max, keep, first, last):
    return {"name": name, "op": "evict", "dtype": dtype, "layers": layers, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "seqs": seqs, "shared": shared, "own_min": own_min,
            "own_max": own_max, "keep": keep, "first": first, "last": last}


def listed():
    return [
        # one token of each of 4 branches through the widest query / key / value
        # projection: the weights' bytes are what counts
        _linear("linear_token", "bf16", 4, 15360, 5120, "bias"),
        # 16 branches of 20 tokens, one of them padded by 11, through an output projection with its residual
        _linear("linear_branches", "bf16", 331, 5120, 13824, "resid"),
        # a whole chunk through the widest up-projection: bound by the products
        _linear("linear_chunk", "bf16", 12960, 13824, 5120, "gelu"),
        # 8 tokens' activations: latency
        _quantize("quantize_token", "bf16", 8, 5120),
        # a projection's float32 weights when they are laid out, an odd number of channels
        _quantize("quantize_weights", "f32", 8961, 1536),
        # one new token of each of 4 branches over a short history: the latency of a decode step
        _weigh("weigh_token_small", "bf16", 8, 8, 64, 16, 4, 1, 2016, 1, 40, True),
        # single tokens of 8 branches over a full ring's worth of history, grouped heads: the keys' bytes
        _weigh("weigh_token_long", "bf16", 40, 8, 128, 32, 8, 1, 38880, 1, 1500, True),
        # prompts of an odd length without a common part, three query heads to a key head
        _weigh("weigh_prompt", "bf16", 12, 4, 128, 128, 6, 1031, 0, 1031, 2500, True),
        # a float32 model's chunk of 232 tokens in 4 branches
        _weigh("weigh_f32_chunk", "f32", 4, 4, 16, 16, 4, 232, 464, 232, 232, False),
        # two branches of one frame of every camera over two chunks of history: the largest call
        _weigh("weigh_chunk_large", "bf16", 12, 12, 128, 32, 2, 4320, 25920, 4320, 4320, False),
        # 4 short sequences that have outgrown their bound by a page or two, in a small model: latency
        _evict("evict_small", "bf16", 8, 8, 64, 16, 4, 0, 261, 283, 256, 16, 64),
        # 6 branches of a common history over 30 layers, a third of their tokens dropped
        _evict("evict_large", "bf16", 30, 12, 128, 32, 6, 1024, 2000, 2977, 2003, 64, 512),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _length(rng, lo, hi):
    """A length in [lo, hi]: half of them odd, the others multiples of ten where that is in range."""
    x = _log_int(rng, lo, hi)
    return max(lo, min(hi, x | 1)) if rng.random() < 0.5 else max(lo, x // 10 * 10)


def draw(rng):
    op = rng.choice(["linear"] * 4 + ["quantize"] + ["weigh"] * 4 + ["evict"] * 2)
    f32 = rng.random() < 0.15
    dtype = "f32" if f32 else "bf16"
    page = rng.choice([16, 32, 64, 128])
    head_dim = rng.choice([16, 32, 64, 128]) if f32 else rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 10])
    if op == "linear":
        while True:
            # any number of tokens, from few channels to the widest projections
            c = _linear("", dtype, _length(rng, 1, 12960), 8 * _log_int(rng, 8, 1920), 16 * _log_int(rng, 4, 864),
                        rng.choice(["bias", "gelu", "resid"]))
            if c["tokens"] * c["n"] * c["k"] <= 9.0e11:
                break
    elif op == "quantize":
        c = _quantize("", dtype, _length(rng, 1, 15360), 16 * _log_int(rng, 4, 864))
    elif op == "weigh":
        group = rng.choice([1, 1, 2, 4, 5, 7])
        while True:
            branches = _log_int(rng, 1, 64)
            n_q = 1 if rng.random() < 0.35 else _length(rng, 1, 4320)
            shared = 0 if rng.random() < 0.15 else (_log_int(rng, 1, 38000 // page) | 1) * page
            own_max = _length(rng, n_q, n_q + 4000)
            own_min = rng.randint(n_q, own_max)
            c = _weigh("", dtype, kv_heads * group, kv_heads, head_dim, page, branches, n_q, shared,
                       own_min, own_max, rng.random() < 0.6)
            rows = branches * n_q * kv_heads * group
            if rows * (shared + own_max) <= (2.0e8 if f32 else 3.0e9) and \
                    branches * (shared + own_max) * kv_heads * head_dim <= 1.0e9:
                break
    else:
        layers, seqs = rng.choice([1, 2, 8, 30]), _log_int(rng, 1, 12)
        row = layers * kv_heads * head_dim * (4 if f32 else 2)
        most = max(64, min(20000, int(1.2e9 / (row * (2 * seqs + 2)))))   # tokens of a sequence
        shared = 0 if rng.random() < 0.5 else rng.randint(1, max(1, most // 3 // page)) * page
        own_max = _length(rng, 32, max(33, most - shared))
        own_min = rng.randint(1, own_max)
        total = shared + own_max
        keep = _length(rng, max(1, total // 8), total)
        first = rng.randint(0, keep // 4)
        last = rng.randint(0, keep // 2)
        c = _evict("", dtype, layers, kv_heads, head_dim, page, seqs, shared, own_min, own_max, keep, first, last)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _own_lens(case, n):
    """Tokens past the shared part, per sequence: spread over [own_min, own_max]."""
    lo, hi = case["own_min"], case["own_max"]
    return [hi - (hi - lo) * ((7 * b) % n) // max(n - 1, 1) if n > 1 else hi for b in range(n)]


def _quantized(x):
    """Rows of x as whole numbers in [-127, 127] (float32) and the scale of each row: the
    largest magnitude becomes 127.  Decided in 64 bits where 32 may fall on a border."""
    a = x.abs().amax(dim=1, keepdim=True).float()
    if x.dtype == torch.bfloat16:
        q = torch.round(x.float() * 127.0 / a)             # 127 x is exact, the quotient decided by 32 bits
    else:
        q = torch.round(x.double() * 127.0 / a.double()).float()
    return torch.where(a > 0, q, torch.zeros_like(q)), a / 127.0


def _pages(case, g, n, spare):
    """Tables of n sequences with a common part, scattered over the pool; table, ref and len
    are views of one buffer, so that a program restores a snapshot with one copy."""
    ps, lens = case["page"], _own_lens(case, n)
    n_sh = case["shared"] // ps
    need = [-(-x // ps) for x in lens]
    max_pages = n_sh + max(need)
    n_pages = n_sh + sum(need) + spare
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    flat = torch.zeros(n_pages + n + n * max_pages, dtype=torch.int32, device=DEV)
    ref, ln, table = flat[:n_pages], flat[n_pages:n_pages + n], flat[n_pages + n:].view(n, max_pages)
    table.fill_(-1)
    table[:, :n_sh] = perm[:n_sh]
    at = n_sh
    for b, x in enumerate(need):
        table[b, n_sh:n_sh + x] = perm[at:at + x]
        at += x
    live = table[table >= 0].long()
    ref.index_add_(0, live, torch.ones_like(live, dtype=torch.int32))
    ln.copy_(torch.tensor([case["shared"] + x for x in lens], dtype=torch.int32))
    return {"flat": flat, "ref": ref, "len": ln, "table": table,
            "seqs": torch.arange(n, dtype=torch.int32, device=DEV)}


def prepare(case, seed):
    g = _gen(seed)
    dt = _dt(case)
    s = {"case": dict(case), "handle": None}
    if case["op"] == "linear":
        M, N, K = case["tokens"], case["n"], case["k"]
        s["x"] = (_randn(g, M, K) * torch.exp(0.5 * _randn(g, M, 1))).to(dt)     # tokens of unlike sizes
        s["x"][:, 3] *= 8                                                        # a channel that stands out
        wq, ws = _quantized((K ** -0.5 * _randn(g, N, K)).bfloat16())
        s["wq"], s["ws"] = wq.to(torch.int8), ws.view(-1).contiguous()
        s["bias"] = 0.05 * _randn(g, N)
        if case["epilogue"] == "resid":
            s["resid"], s["gate"] = _randn(g, M, N).to(dt), 1.0 + 0.2 * _randn(g, N)
        return s
    if case["op"] == "quantize":
        s["x"] = (_randn(g, case["rows"], case["k"]) * torch.exp(0.5 * _randn(g, case["rows"], 1))).to(dt)
        return s
    hd, hk, ps = case["head_dim"], case["kv_heads"], case["page"]
    if case["op"] == "weigh":
        B, n, H = case["branches"], case["n_q"], case["heads"]
        s.update(_pages(case, g, B, 3))
        n_pages = s["ref"].numel()
        s["k"] = _randn(g, 1, n_pages, ps, hk * hd).to(dt)
        s["v"] = torch.zeros_like(s["k"])
        s["q"] = (2.0 * _randn(g, B * n, H * hd)).to(dt)                         # peaked scores, as trained heads have
        x = _scores(s)
        s["lse"] = torch.logsumexp(x, dim=-1).permute(0, 2, 1, 3).reshape(B * n, H).contiguous()
        del x
        w = _randn(g, B, s["table"].shape[1] * ps).abs()                         # what earlier steps have added up
        s["weights"] = w.masked_fill_(torch.arange(w.shape[1], device=DEV) >= s["len"][:, None], 0.0)
        return s
    n = case["seqs"]
    n_new = -(-case["keep"] // ps)
    s.update(_pages(case, g, n, n * min(n_new, case["shared"] // ps) + 2))       # room for the shared pages that change
    shape = (case["layers"], s["ref"].numel(), ps, hk * hd)
    s["k"] = torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g)
    s["v"] = torch.empty(shape, dtype=dt, device=DEV).normal_(generator=g)
    # few tokens carry most of the weight, and rounded weights make ties
    w = torch.exp(2.0 * _randn(g, n, s["table"].shape[1] * ps)).mul_(64).round_().div_(64)
    s["weights"] = w.masked_fill_(torch.arange(w.shape[1], device=DEV) >= s["len"][:, None], 0.0)
    s["flat0"], s["weights0"] = s["flat"].clone(), s["weights"].clone()
    return s


# --------------------------------------------------------------- one pass
def _cache(s):
    """The framework's handle on the cache, which a program makes once."""
    if s["handle"] is None:
        from paper_2604_20289_gb300 import xcache as xb
        c = s["case"]
        cache = xb.KVCache(c["dtype"], c["kv_heads"], c["head_dim"], s["k"], s["v"], s["ref"], s["table"], s["len"])
        s["handle"] = xb, cache
    return s["handle"]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"linear": _linear_own, "quantize": _quantize_own, "weigh": _weigh_own, "evict": _evict_own}[op](state)
    return {"linear": _linear_plain, "quantize": _quantize_plain, "weigh": _weigh_plain,
            "evict": _evict_plain}[op](state)


def _linear_own(s):
    from paper_2604_20289_gb300 import xcache as xb
    c = s["case"]
    out = torch.empty(c["tokens"], c["n"], dtype=s["x"].dtype, device=DEV)
    if c["epilogue"] == "resid":
        xb.op_linear_i8(c["dtype"], xb.XC_EPI_RESID_GATE, s["x"], s["wq"], s["ws"], s["bias"], out, gate=s["gate"],
                        resid=s["resid"])
    else:
        xb.op_linear_i8(c["dtype"], xb.XC_EPI_GELU if c["epilogue"] == "gelu" else xb.XC_EPI_BIAS, s["x"], s["wq"],
                        s["ws"], s["bias"], out)
    return out


def _quantize_own(s):
    from paper_2604_20289_gb300 import xcache as xb
    c = s["case"]
    q = torch.empty(c["rows"], c["k"], dtype=torch.int8, device=DEV)
    scale = torch.empty(c["rows"], device=DEV)
    xb.op_quantize_rows(c["dtype"], s["x"], q, scale)
    return {"values": q * scale[:, None], "scale": scale}


def _weigh_own(s):
    xb, cache = _cache(s)
    c = s["case"]
    xb.op_key_weights(cache, 0, s["seqs"], c["n_q"], s["q"], s["lse"], s["weights"], shared_len=c["shared"],
                      causal=c["causal"], decay=0.9)
    return s["weights"]


def _evict_own(s):
    xb, cache = _cache(s)
    c = s["case"]
    s["flat"].copy_(s["flat0"])                                       # back to the snapshot
    s["weights"].copy_(s["weights0"])
    kept = torch.empty(c["seqs"], c["keep"], dtype=torch.int32, device=DEV)
    xb.op_kv_evict(cache, s["seqs"], c["keep"], s["weights"], n_first=c["first"], n_last=c["last"], kept=kept)
    return {"kept": kept, "k": s["k"], "v": s["v"], "ref": s["ref"], "table": s["table"], "len": s["len"],
            "weights": s["weights"]}


def _linear_plain(s):
    c = s["case"]
    q, scale = _quantized(s["x"])
    y = torch.matmul(q, s["wq"].float().t()) * scale * s["ws"] + s["bias"]
    if c["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    elif c["epilogue"] == "resid":
        y = s["resid"].float() + s["gate"] * y
    return y.to(s["x"].dtype)


def _quantize_plain(s):
    q, scale = _quantized(s["x"])
    return {"values": q * scale, "scale": scale.view(-1)}


def _scores(s):
    """Scaled scores [branch, key head, token, query head of it, key], -inf where a token does not see the key."""
    c = s["case"]
    B, n, hk, hd, ps, P = c["branches"], c["n_q"], c["kv_heads"], c["head_dim"], c["page"], c["shared"]
    S = c["own_max"]
    kp = s["k"][0].view(-1, hk, hd)
    lens, tab = s["len"].long(), s["table"].long()
    q = s["q"].float().view(B, n, hk, c["heads"] // hk, hd)
    j = torch.arange(P, device=DEV)
    k1 = kp[tab[0][j // ps] * ps + j % ps].float()                    # shared part, once: [P, hk, hd]
    j = torch.arange(S, device=DEV)
    rows = tab[:, P // ps:].clamp(min=0)[:, j // ps] * ps + j % ps
    there = (j[None] < (lens - P)[:, None])[..., None, None]
    k2 = kp[rows].float().masked_fill(~there, 0.0)                    # own parts: [B, S, hk, hd]
    x = torch.cat([torch.einsum("bnhgd,phd->bhngp", q, k1), torch.einsum("bnhgd,bshd->bhngs", q, k2)], dim=-1)
    x = x.mul_(1.0 / math.sqrt(hd))
    i = torch.arange(n, device=DEV)
    limit = (lens[:, None] - n + i + 1) if c["causal"] else lens[:, None].expand(B, n)
    hidden = torch.arange(P + S, device=DEV) >= limit[..., None]      # [B, n, keys]
    return x.masked_fill_(hidden[:, None, :, None], -math.inf)


def _weigh_plain(s):
    c = s["case"]
    B, n, hk = c["branches"], c["n_q"], c["kv_heads"]
    x = _scores(s)
    lse = s["lse"].view(B, n, hk, -1).permute(0, 2, 1, 3)
    p = x.sub_(lse[..., None]).exp_().sum(dim=3).sum(dim=2).sum(dim=1)
    w = s["weights"][:, :p.shape[1]]
    here = torch.arange(p.shape[1], device=DEV) < s["len"][:, None]
    w.copy_(torch.where(here, 0.9 * w + p, w))
    return s["weights"]


def _evict_plain(s):
    c = s["case"]
    s["flat"].copy_(s["flat0"])
    s["weights"].copy_(s["weights0"])
    ps, keep, hk = c["page"], c["keep"], c["kv_heads"]
    lens, tab, ref = s["len"].long(), s["table"].long(), s["ref"]
    n, S = lens.numel(), c["shared"] + c["own_max"]
    j = torch.arange(S, device=DEV)
    i = torch.arange(keep, device=DEV)
    w = s["weights"][:, :S]
    # what comes first and last stays, then the largest weights, the lowest index where they are equal
    rank = torch.where((j < c["first"]) | (j >= lens[:, None] - c["last"]), math.inf, w)
    rank = rank.masked_fill(j >= lens[:, None], -math.inf)
    idx = torch.sort(torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :keep], dim=1).values
    full = (lens > keep)[:, None]
    kept = torch.where(full, idx, torch.where(i < lens[:, None], i, -torch.ones_like(i)))
    # a page whose rows change, or that ends inside, is replaced where other sequences hold it
    p = torch.arange(-(-keep // ps), device=DEV)
    end = torch.clamp((p + 1) * ps, max=keep) - 1
    changed = ((idx[:, end] != end) | ((p + 1) * ps > keep)) & full
    old = tab[:, :p.numel()]
    copied = changed & (ref[old.clamp(min=0)] > 1)
    fresh = torch.nonzero(ref == 0)[:, 0][:int(copied.sum())]
    new = old.clone()
    new[copied] = fresh
    move = full.expand(n, keep)
    src = (tab.gather(1, idx // ps) * ps + idx % ps)[move]
    dst = (new[:, i // ps] * ps + i % ps)[move]
    k, v = (t.view(t.shape[0], -1, t.shape[3]) for t in (s["k"], s["v"]))
    k[:, dst] = k[:, src]
    v[:, dst] = v[:, src]
    gone = full & (tab >= 0)
    gone[:, :p.numel()] &= copied
    ref.index_add_(0, tab[gone], torch.full_like(tab[gone], -1, dtype=torch.int32))
    ref[fresh] = 1
    tail = torch.full_like(s["table"][:, p.numel():], -1)
    s["table"].copy_(torch.where(full, torch.cat([new.int(), tail], dim=1), s["table"]))
    s["len"].copy_(torch.where(full[:, 0], keep, lens))
    packed = torch.zeros_like(w)
    packed[:, :keep] = w.gather(1, idx)
    w.copy_(torch.where(full, packed, w))
    return {"kept": kept.int(), "k": s["k"], "v": s["v"], "ref": ref, "table": s["table"], "len": s["len"],
            "weights": s["weights"]}


# ------------------------------------------------------- work and 64 bits
def work(case):
    es = _es(case)
    if case["op"] == "linear":
        M, N, K = case["tokens"], case["n"], case["k"]
        outs = 2 if case["epilogue"] == "resid" else 1
        return {"bytes": M * K * es + N * K + 8 * N + outs * M * N * es, "flops": 2 * M * N * K}
    if case["op"] == "quantize":
        return {"bytes": case["rows"] * (case["k"] * (es + 4) + 4), "flops": 3 * case["rows"] * case["k"]}
    hd, hk, ps = case["head_dim"], case["kv_heads"], case["page"]
    row = hk * hd * es
    if case["op"] == "weigh":
        B, n, P, H = case["branches"], case["n_q"], case["shared"], case["heads"]
        lens = _own_lens(case, B)
        if case["causal"]:
            seen = sum(sum(max(0, P + x - n + i + 1) for i in range(n)) for x in lens)
        else:
            seen = sum(n * (P + x) for x in lens)
        return {"bytes": B * n * H * (hd * es + 4) + (P + sum(lens)) * row + 8 * sum(P + x for x in lens),
                "flops": 2 * hd * H * seen}
    lens = [case["shared"] + x for x in _own_lens(case, case["seqs"])]
    keep, first, last = case["keep"], case["first"], case["last"]
    moved = 0.0                                # kept rows behind the first dropped one, which is near `first`
    for x in lens:
        if x > keep:
            moved += keep - first if keep - first - last < x - first - last else 0
    return {"bytes": 2 * moved * 2 * case["layers"] * row + 8 * sum(lens), "flops": 0}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("linear", "quantize"):
        x = s["x"].to(F64)
        top = x.abs().max(dim=1).values[:, None]
        q = torch.where(top > 0, (x * 127 / top).round(), torch.zeros_like(x))
        unit = (top.float() / torch.tensor(127.0, device=DEV)).to(F64)           # the scale is a float32
        if case["op"] == "quantize":
            return {"values": q.mul_(unit), "scale": unit.view(-1)}
        y = q @ s["wq"].to(F64).t()
        del q, x
        y.mul_(unit).mul_(s["ws"].to(F64)).add_(s["bias"].to(F64))
        if case["epilogue"] == "gelu":
            t = y.pow(3).mul_(0.044715).add_(y).mul_(math.sqrt(8.0 / math.pi))   # 0.5 (1 + tanh u) = sigmoid(2 u)
            y.mul_(torch.sigmoid(t))
        elif case["epilogue"] == "resid":
            y.mul_(s["gate"].to(F64)).add_(s["resid"].to(F64))
        return y
    hd, hk, ps = case["head_dim"], case["kv_heads"], case["page"]
    lens = s["len"].tolist()
    if case["op"] == "weigh":
        B, n, H = case["branches"], case["n_q"], case["heads"]
        if 2.0 * B * n * H * hd * (case["shared"] + case["own_max"]) > 4e12:
            return None
        out = s["weights"].to(F64)
        q, lse = s["q"].view(B, n, H, hd), s["lse"].view(B, n, H).to(F64)
        block = max(1, int(4e8 // max(1, H * max(lens))))
        for b in range(B):
            pos = torch.arange(lens[b], device=DEV)
            rows = s["table"][b].long()[pos // ps] * ps + pos % ps
            kk = s["k"].view(-1, hk, hd)[rows].to(F64).transpose(0, 1).repeat_interleave(H // hk, dim=0)
            out[b, :lens[b]] *= 0.9
            for i0 in range(0, n, block):
                tok = torch.arange(i0, min(n, i0 + block), device=DEV)
                z = q[b, tok].to(F64).transpose(0, 1) @ kk.transpose(1, 2)       # [H, tokens, keys]
                z = torch.exp(z / math.sqrt(hd) - lse[b, tok].t()[..., None])
                if case["causal"]:
                    z = z * (pos[None] <= (lens[b] - n + tok)[:, None])
                out[b, :lens[b]] += z.sum(dim=(0, 1))
        return out
    # the same drops one sequence after another on the host's lists
    keep = case["keep"]
    ref, table = s["ref"].tolist(), s["table"].tolist()
    count = list(ref)
    free = [p for p, r in enumerate(ref) if r == 0]
    k, v, w = s["k"].to(F64), s["v"].to(F64), s["weights"].to(F64)
    k0, v0 = s["k"], s["v"]
    for b, length in enumerate(lens):
        if length <= keep:
            continue
        mid = list(range(case["first"], length - case["last"]))
        have = s["weights"][b].tolist()
        mid.sort(key=lambda t: (-have[t], t))
        idx = sorted(list(range(case["first"])) + list(range(length - case["last"], length)) +
                     mid[:keep - case["first"] - case["last"]])
        at = torch.tensor(idx, device=DEV)
        pages = []
        for p in range(-(-keep // ps)):
            stop = min((p + 1) * ps, keep)
            other = idx[stop - 1] != stop - 1 or (p + 1) * ps > keep
            pages.append(free.pop(0) if other and count[table[b][p]] > 1 else table[b][p])
        old = s["table"][b].long()
        to = torch.tensor(pages, device=DEV)
        i = torch.arange(keep, device=DEV)
        k[:, to[i // ps], i % ps] = k0[:, old[at // ps], at % ps].to(F64)
        v[:, to[i // ps], i % ps] = v0[:, old[at // ps], at % ps].to(F64)
        w[b, :keep] = s["weights"][b][at].to(F64)
        w[b, keep:length] = 0.0
    return {"kept": None, "k": k, "v": v, "ref": None, "table": None, "len": None, "weights": w}
