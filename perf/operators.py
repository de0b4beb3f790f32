"""Performance cases of the branched-rollout operators: a paged key / value
cache whose pages several sequences share, the head-wise norm of queries and
keys with the position rotation that fills it, the page operations that fork,
extend, free and compact it, and the attention of a batch of branches over a
shared history.

Every case is a dict of plain values; ``prepare`` makes the tensors a program
holds before the call, ``run`` makes one pass -- with ``own`` the framework's
operators, otherwise the same arithmetic in elementary torch operations in 32
bits -- and ``exact`` restates the result in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


# ------------------------------------------------------------------- cases
def _attend(name, dtype, heads, kv_heads, head_dim, page, branches, n_q, shared, own_min, own_max, causal):
    return {"name": name, "op": "attend", "dtype": dtype, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "branches": branches, "n_q": n_q, "shared": shared,
            "own_min": own_min, "own_max": own_max, "causal": causal}


def _append(name, dtype, heads, kv_heads, head_dim, page, tokens, axes, half_split):
    return {"name": name, "op": "append", "dtype": dtype, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "tokens": tokens, "axes": axes, "half_split": half_split}


def _fork(name, dtype, layers, kv_heads, head_dim, page, n_pages, length, children, n_new):
    return {"name": name, "op": "fork", "dtype": dtype, "layers": layers, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "n_pages": n_pages, "length": length,
            "children": children, "n_new": n_new}


def _compact(name, dtype, layers, kv_heads, head_dim, page, n_pages, seqs, live):
    return {"name": name, "op": "compact", "dtype": dtype, "layers": layers, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "n_pages": n_pages, "seqs": seqs, "live": live}


def listed():
    return [
        # one new token of each of 4 branches over a short common history:
        # the latency of a decode step
        _attend("attend_token_small", "bf16", 8, 8, 64, 16, 4, 1, 2016, 1, 40, True),
        # single tokens of 32 branches over a full ring's worth of history,
        # grouped heads: what the history's keys cost when read once
        _attend("attend_token_long", "bf16", 40, 8, 128, 32, 32, 1, 38880, 1, 1500, True),
        # 16 candidate futures advanced by 20 tokens each over one chunk of history
        _attend("attend_branches", "bf16", 12, 12, 128, 32, 16, 20, 12960, 20, 700, True),
        # prompts without a common part, an odd length and three query heads to a key head
        _attend("attend_prompt", "bf16", 12, 4, 128, 128, 6, 1031, 0, 1031, 2500, True),
        # a float32 model's chunk of 232 tokens in 4 branches
        _attend("attend_f32_chunk", "f32", 4, 4, 16, 16, 4, 232, 464, 232, 232, False),
        # two branches of one frame of every camera over two chunks of history:
        # the largest call, bound by the matrix products
        _attend("attend_chunk_large", "bf16", 12, 12, 128, 32, 2, 4320, 25920, 4320, 4320, False),
        # one new token of each of 8 branches: latency
        _append("append_token", "bf16", 40, 40, 128, 32, 8, 4, False),
        # a prompt of odd length with grouped heads, halves rotated against each other
        _append("append_prompt", "bf16", 40, 8, 64, 16, 4099, 1, True),
        # a whole chunk of the widest model, positions on four axes
        _append("append_chunk", "bf16", 40, 40, 128, 32, 12960, 4, False),
        # 4 children of one sequence, one new token each, freed again: latency
        _fork("fork_small", "bf16", 8, 8, 64, 16, 1024, 8073, 4, 1),
        # 16 children over 30 layers: the copies of the partly filled page
        _fork("fork_large", "bf16", 30, 12, 128, 32, 512, 12977, 16, 16),
        # a pool of 30 layers, 60 % of its pages live and scattered
        _compact("compact_pool", "bf16", 30, 12, 128, 32, 512, 8, 0.6),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _length(rng, lo, hi):
    """A length in [lo, hi]: half of them odd, the others multiples of ten where that is in range."""
    x = _log_int(rng, lo, hi)
    return max(lo, min(hi, x | 1)) if rng.random() < 0.5 else max(lo, x // 10 * 10)


def draw(rng):
    kind = rng.choice(["attend"] * 6 + ["append"] * 3 + ["fork", "compact"])
    f32 = rng.random() < 0.15
    dtype = "f32" if f32 else "bf16"
    page = rng.choice([16, 32, 64, 128])
    head_dim = rng.choice([16, 32, 64, 128]) if f32 else rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 10])
    group = rng.choice([1, 1, 2, 4, 5, 7])
    if kind == "attend":
        while True:
            branches = _log_int(rng, 1, 64)
            n_q = 1 if rng.random() < 0.35 else _length(rng, 1, 4320)
            shared = 0 if rng.random() < 0.15 else (_log_int(rng, 1, 38000 // page) | 1) * page
            own_max = _length(rng, n_q, n_q + 4000)
            own_min = rng.randint(n_q, own_max)
            c = _attend("", dtype, kv_heads * group, kv_heads, head_dim, page, branches, n_q, shared,
                        own_min, own_max, rng.random() < 0.6)
            rows = branches * n_q * kv_heads * group
            most = 2.0e8 if f32 else 3.0e9
            if rows * (shared + own_max) <= most and branches * own_max * kv_heads * head_dim <= 2.0e8:
                break
    elif kind == "append":
        c = _append("", dtype, kv_heads * group, kv_heads, head_dim, page, _length(rng, 1, 12960),
                    rng.choice([1, 4]), rng.random() < 0.5)
    else:
        layers = rng.choice([1, 2, 8, 30])
        row = kv_heads * head_dim * (4 if f32 else 2)
        n_pages = max(48, min(1024, int(1.5e9 / (layers * page * row))))
        if kind == "fork":
            children = _log_int(rng, 1, 16)
            n_new = _log_int(rng, 1, 2 * page)
            room = n_pages - children * (2 + -(-n_new // page))
            c = _fork("", dtype, layers, kv_heads, head_dim, page, n_pages,
                      _length(rng, 1, max(1, room - 1) * page), children, n_new)
        else:
            c = _compact("", dtype, layers, kv_heads, head_dim, page, n_pages, rng.randint(1, 16),
                         round(rng.uniform(0.1, 0.95), 3))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _own_lens(case):
    """Tokens past the shared part, per branch: spread over [own_min, own_max]."""
    B, lo, hi = case["branches"], case["own_min"], case["own_max"]
    return [hi - (hi - lo) * ((7 * b) % B) // max(B - 1, 1) if B > 1 else hi for b in range(B)]


def _axis_pairs(case):
    """Rotation pairs of each position axis: one axis, or camera / frame / h / w
    in the proportions 1 : 3 : 2 : 2 of the head."""
    hd = case["head_dim"]
    return [hd // 2] if case["axes"] == 1 else [hd // 16, 3 * hd // 16, hd // 8, hd // 8]


def _grid(tokens):
    """Positions (camera, frame, h, w) of a chunk of 6 x 3 x 20 x 36 tokens, and their bounds."""
    r = torch.arange(tokens, device=DEV)
    return torch.stack([r // 2160 % 6, r // 720 % 3 + 57, r // 36 % 20, r % 36], dim=1), [6, 64, 20, 36]


def _rotation_table(pairs, n_pos):
    """(cos, sin) of every position and pair of each axis, axis after axis."""
    parts = []
    for n, p in zip(pairs, n_pos):
        f = 10000.0 ** (-torch.arange(n, device=DEV, dtype=torch.float64) / n)
        a = torch.arange(p, device=DEV, dtype=torch.float64)[:, None] * f
        parts.append(torch.stack([a.cos(), a.sin()], dim=-1).reshape(-1, 2))
    return torch.cat(parts).float().contiguous()


def prepare(case, seed):
    g = _gen(seed)
    dt = _dt(case)
    hd, hk, ps = case["head_dim"], case["kv_heads"], case["page"]
    s = {"case": dict(case), "handle": None}
    if case["op"] == "attend":
        B, H = case["branches"], case["heads"]
        own_lens = _own_lens(case)
        n_shared = case["shared"] // ps
        need = [-(-n // ps) for n in own_lens]
        max_pages = n_shared + max(need)
        n_pages = n_shared + sum(need) + 3
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((B, max_pages), -1, dtype=torch.int32, device=DEV)
        table[:, :n_shared] = perm[:n_shared]
        at = n_shared
        for b, n in enumerate(need):
            table[b, n_shared:n_shared + n] = perm[at:at + n]
            at += n
        ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        live = table[table >= 0].long()
        ref.index_add_(0, live, torch.ones_like(live, dtype=torch.int32))
        s["table"], s["ref"] = table, ref
        s["len"] = torch.tensor([case["shared"] + n for n in own_lens], dtype=torch.int32, device=DEV)
        s["seqs"] = torch.arange(B, dtype=torch.int32, device=DEV)
        s["k"] = _randn(g, 1, n_pages, ps, hk * hd).to(dt)
        s["v"] = _randn(g, 1, n_pages, ps, hk * hd).to(dt)
        s["q"] = (2.0 * _randn(g, B * case["n_q"], H * hd)).to(dt)   # peaked scores, as trained heads have
    elif case["op"] == "append":
        T, H = case["tokens"], case["heads"]
        n_pages = -(-T // ps) + 2
        s["q"] = _randn(g, T, H * hd).to(dt)
        s["kv"] = _randn(g, T, 2 * hk * hd).to(dt)                   # one projection's output: strided views
        s["k_new"], s["v_new"] = s["kv"][:, :hk * hd], s["kv"][:, hk * hd:]
        s["gamma_q"] = 1.0 + 0.1 * _randn(g, hd)
        s["gamma_k"] = 1.0 + 0.1 * _randn(g, hd)
        if case["axes"] == 1:
            s["pos"], s["n_pos"] = torch.arange(T, device=DEV)[:, None] + 100, [T + 100]
        else:
            s["pos"], s["n_pos"] = _grid(T)
        s["pos"] = s["pos"].to(torch.int32).contiguous()
        s["pairs"] = _axis_pairs(case)
        s["rotation"] = _rotation_table(s["pairs"], s["n_pos"])
        perm = torch.randperm(n_pages, generator=g, device=DEV)
        r = torch.arange(T, device=DEV) + 5                           # the sequence begins inside a page
        s["slots"] = (perm[r // ps] * ps + r % ps).to(torch.int32)
        if T > 16:
            s["slots"][T // 2] = -1                                   # a padding token keeps no keys
        s["ref"] = torch.ones(n_pages, dtype=torch.int32, device=DEV)
        s["table"] = perm[None].to(torch.int32).contiguous()
        s["len"] = torch.full((1,), T + 5, dtype=torch.int32, device=DEV)
        s["k"] = _randn(g, 1, n_pages, ps, hk * hd).to(dt)
        s["v"] = _randn(g, 1, n_pages, ps, hk * hd).to(dt)
    else:
        n_pages, layers = case["n_pages"], case["layers"]
        s["k"] = torch.empty(layers, n_pages, ps, hk * hd, dtype=dt, device=DEV)
        s["v"] = torch.empty_like(s["k"])
        s["k"].normal_(generator=g)
        s["v"].normal_(generator=g)
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        s["ref"] = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        if case["op"] == "fork":
            n, C = -(-case["length"] // ps), case["children"]
            max_pages = -(-(case["length"] + case["n_new"]) // ps)
            s["table"] = torch.full((C + 1, max_pages), -1, dtype=torch.int32, device=DEV)
            s["table"][0, :n] = perm[:n]
            s["ref"][perm[:n].long()] = 1
            s["len"] = torch.zeros(C + 1, dtype=torch.int32, device=DEV)
            s["len"][0] = case["length"]
            s["src"] = torch.zeros(C, dtype=torch.int32, device=DEV)
            s["dst"] = torch.arange(1, C + 1, dtype=torch.int32, device=DEV)
        else:
            S = case["seqs"]
            per = max(1, int(case["live"] * n_pages) // S)
            rows = perm[:per * S].view(S, per).clone()
            s["table"] = torch.full((S, per + 4), -1, dtype=torch.int32, device=DEV)
            s["table"][:, :per] = rows
            s["table"][:, 0] = rows[0, 0]                             # a page that all of them share
            live = s["table"][s["table"] >= 0].long()
            s["ref"].index_add_(0, live, torch.ones_like(live, dtype=torch.int32))
            s["len"] = torch.full((S,), per * ps - 3, dtype=torch.int32, device=DEV)
            s["table0"], s["ref0"] = s["table"].clone(), s["ref"].clone()
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
        return {"attend": _attend_own, "append": _append_own, "fork": _fork_own, "compact": _compact_own}[op](state)
    return {"attend": _attend_plain, "append": _append_plain, "fork": _fork_plain, "compact": _compact_plain}[op](state)


def _attend_own(s):
    xb, cache = _cache(s)
    c = s["case"]
    o = torch.empty_like(s["q"])
    xb.op_branch_attention(cache, 0, s["seqs"], c["n_q"], s["q"], o, shared_len=c["shared"], causal=c["causal"])
    return o


def _append_own(s):
    xb, cache = _cache(s)
    q = torch.empty_like(s["q"])
    xb.op_qk_norm_rope(cache, 0, s["q"], s["k_new"], s["v_new"], s["gamma_q"], s["gamma_k"], s["pos"], s["pairs"],
                       s["n_pos"], s["rotation"], s["slots"], q, half_split=s["case"]["half_split"])
    return {"q": q, "k": s["k"], "v": s["v"]}


def _fork_own(s):
    xb, cache = _cache(s)
    c = s["case"]
    slots = torch.empty(c["children"], c["n_new"], dtype=torch.int32, device=DEV)
    xb.op_kv_fork(cache, s["src"], s["dst"])
    xb.op_kv_extend(cache, s["dst"], c["n_new"], slots)
    xb.op_kv_free(cache, s["dst"])
    return {"slots": slots, "k": s["k"], "v": s["v"], "ref": s["ref"], "table": s["table"], "len": s["len"]}


def _compact_own(s):
    xb, cache = _cache(s)
    s["table"].copy_(s["table0"])                                     # back to the fragmented snapshot
    s["ref"].copy_(s["ref0"])
    live = torch.empty(1, dtype=torch.int32, device=DEV)
    xb.op_kv_compact(cache, live)
    return {"live": live, "k": s["k"], "v": s["v"], "ref": s["ref"], "table": s["table"]}


def _attend_plain(s):
    c = s["case"]
    B, n, hk, hd, ps, P = c["branches"], c["n_q"], c["kv_heads"], c["head_dim"], c["page"], c["shared"]
    grp = c["heads"] // hk
    S = c["own_max"]
    kp, vp = (t[0].view(-1, hk, hd) for t in (s["k"], s["v"]))
    lens = s["len"].long()[s["seqs"].long()]
    tab = s["table"].long()[s["seqs"].long()]
    q = s["q"].float().view(B, n, hk, grp, hd)
    j = torch.arange(P, device=DEV)
    rows = tab[0][j // ps] * ps + j % ps
    k1, v1 = kp[rows].float(), vp[rows].float()                       # shared part, once: [P, hk, hd]
    j = torch.arange(S, device=DEV)
    rows = tab[:, P // ps:].clamp(min=0)[:, j // ps] * ps + j % ps
    there = (j[None] < (lens - P)[:, None])[..., None, None]
    k2 = kp[rows].float().masked_fill(~there, 0.0)                    # own parts: [B, S, hk, hd]
    v2 = vp[rows].float().masked_fill(~there, 0.0)
    x = torch.cat([torch.einsum("bnhgd,phd->bhngp", q, k1), torch.einsum("bnhgd,bshd->bhngs", q, k2)], dim=-1)
    x = x.mul_(1.0 / math.sqrt(hd))
    i = torch.arange(n, device=DEV)
    limit = (lens[:, None] - n + i + 1) if c["causal"] else lens[:, None].expand(B, n)
    hidden = torch.arange(P + S, device=DEV) >= limit[..., None]      # [B, n, keys]
    x = x.masked_fill_(hidden[:, None, :, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    z = p.sum(dim=-1, keepdim=True)
    o = torch.einsum("bhngp,phd->bhngd", p[..., :P], v1) + torch.einsum("bhngs,bshd->bhngd", p[..., P:], v2)
    o = torch.where(z > 0, o / z, torch.zeros_like(o))
    return o.permute(0, 2, 1, 3, 4).reshape(B * n, -1).to(s["q"].dtype)


def _rotated(s, x, heads, gamma, f):
    """Head-wise RMS norm with gain and the position rotation, in the floating type f."""
    c = s["case"]
    hd = c["head_dim"]
    x = x.to(f).reshape(x.shape[0], heads, hd)
    x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * gamma.to(f)
    pairs = torch.tensor(s["pairs"], device=DEV)
    axis = torch.repeat_interleave(torch.arange(len(s["pairs"]), device=DEV), pairs)
    first = torch.cumsum(pairs, 0) - pairs
    spans = pairs * torch.tensor(s["n_pos"], device=DEV)
    base = torch.cumsum(spans, 0) - spans
    at = base[axis] + s["pos"].long()[:, axis] * pairs[axis] + torch.arange(hd // 2, device=DEV) - first[axis]
    cs = s["rotation"][at].to(f)[:, None]                             # [T, 1, hd / 2, 2]
    if c["half_split"]:
        a, b = x[..., :hd // 2], x[..., hd // 2:]
    else:
        a, b = x[..., 0::2], x[..., 1::2]
    y = (a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0])
    y = torch.cat(y, dim=-1) if c["half_split"] else torch.stack(y, dim=-1)
    return y.reshape(x.shape[0], heads * hd)


def _append_plain(s):
    c = s["case"]
    dt = s["q"].dtype
    q = _rotated(s, s["q"], c["heads"], s["gamma_q"], torch.float32).to(dt)
    k = _rotated(s, s["k_new"], c["kv_heads"], s["gamma_k"], torch.float32).to(dt)
    keep = s["slots"] >= 0
    rows = s["slots"].long()[keep]
    s["k"][0].view(-1, k.shape[1])[rows] = k[keep]
    s["v"][0].view(-1, k.shape[1])[rows] = s["v_new"][keep]
    return {"q": q, "k": s["k"], "v": s["v"]}


def _fork_plain(s):
    c = s["case"]
    ps, C, N = c["page"], c["children"], c["n_new"]
    ref, table, ln = s["ref"], s["table"], s["len"]
    src, dst = s["src"].long(), s["dst"].long()
    # fork: whole pages are shared, a partly filled one is copied
    full, part = c["length"] // ps, c["length"] % ps
    pages = table[0, :full].long()
    ref[pages] += C
    table[dst, :full] = table[src, :full]
    if part:
        fresh = torch.nonzero(ref == 0)[:C, 0]
        ref[fresh] = 1
        table[dst, full] = fresh.to(torch.int32)
        last = table[0, full:full + 1].long()
        s["k"][:, fresh, :part] = s["k"][:, last, :part]
        s["v"][:, fresh, :part] = s["v"][:, last, :part]
    ln[dst] = ln[src]
    # extend every child by N tokens
    have, want = -(-c["length"] // ps), -(-(c["length"] + N) // ps)
    if want > have:
        fresh = torch.nonzero(ref == 0)[:C * (want - have), 0]
        ref[fresh] = 1
        table[dst, have:want] = fresh.to(torch.int32).view(C, want - have)
    at = c["length"] + torch.arange(N, device=DEV)
    slots = (table[dst][:, at // ps] * ps + at % ps).to(torch.int32)
    # free the children
    held = table[dst]
    held = held[held >= 0].long()
    ref.index_add_(0, held, torch.full_like(held, -1, dtype=torch.int32))
    table[dst] = -1
    ln[dst] = 0
    return {"slots": slots, "k": s["k"], "v": s["v"], "ref": ref, "table": table, "len": ln}


def _compact_plain(s):
    s["table"].copy_(s["table0"])
    s["ref"].copy_(s["ref0"])
    ref, table = s["ref"], s["table"]
    used = ref > 0
    live = used.sum()
    ids = torch.arange(ref.numel(), device=DEV)
    hole = ids[~used & (ids < live)]                                  # k-th live page past the end fills the k-th hole
    mover = ids[used & (ids >= live)]
    s["k"][:, hole] = s["k"][:, mover]
    s["v"][:, hole] = s["v"][:, mover]
    new = ids.clone()
    new[mover] = hole
    ref[hole] = ref[mover]
    ref[mover] = 0
    table.copy_(torch.where(table >= 0, new[table.clamp(min=0).long()].to(torch.int32), table))
    return {"live": live.to(torch.int32).view(1), "k": s["k"], "v": s["v"], "ref": ref, "table": table}


# ------------------------------------------------------- work and 64 bits
def work(case):
    es, hd, hk = _es(case), case["head_dim"], case["kv_heads"]
    row = hk * hd * es
    if case["op"] == "attend":
        own_lens, n, P, H = _own_lens(case), case["n_q"], case["shared"], case["heads"]
        if case["causal"]:
            seen = sum(sum(max(0, P + x - n + i + 1) for i in range(n)) for x in own_lens)
        else:
            seen = sum(n * (P + x) for x in own_lens)
        return {"bytes": 2 * case["branches"] * n * H * hd * es + 2 * (P + sum(own_lens)) * row,
                "flops": 4 * hd * H * seen}
    if case["op"] == "append":
        T, H = case["tokens"], case["heads"]
        return {"bytes": 2 * T * (H + 2 * hk) * hd * es, "flops": T * (H + hk) * hd * 8}
    if case["op"] == "fork":
        ps = case["page"]
        copied = 2 * case["layers"] * case["children"] * (case["length"] % ps) * row
        lists = 4 * (2 * case["n_pages"] + 4 * case["children"] * (case["length"] // ps + 1 + case["n_new"]))
        return {"bytes": 2 * copied + lists, "flops": 0}
    n_pages, S = case["n_pages"], case["seqs"]
    used = S * (max(1, int(case["live"] * n_pages) // S) - 1) + 1
    moved = used * (n_pages - used) / n_pages                         # of a random layout
    return {"bytes": 2 * moved * 2 * case["layers"] * case["page"] * row + 12 * n_pages, "flops": 0}


def exact(case, seed):
    s = prepare(case, seed)
    f = torch.float64
    if case["op"] == "attend":
        B, n, H, hk, hd, ps = (case[x] for x in ("branches", "n_q", "heads", "kv_heads", "head_dim", "page"))
        if 4.0 * B * n * H * hd * (case["shared"] + case["own_max"]) > 8e12:
            return None
        out = torch.zeros(B, n, H, hd, dtype=f, device=DEV)
        lens, tab = s["len"].tolist(), s["table"].long()
        q = s["q"].view(B, n, H, hd)
        block = max(1, int(4e8 // max(1, H * max(lens))))
        for b in range(B):
            pos = torch.arange(lens[b], device=DEV)
            at = (tab[b][pos // ps], pos % ps)
            kk = s["k"][0][at].to(f).view(-1, hk, hd).repeat_interleave(H // hk, dim=1).transpose(0, 1)
            vv = s["v"][0][at].to(f).view(-1, hk, hd).repeat_interleave(H // hk, dim=1).transpose(0, 1)
            for i0 in range(0, n, block):
                qq = q[b, i0:i0 + block].to(f).transpose(0, 1)
                w = qq @ kk.transpose(1, 2) / math.sqrt(hd)
                if case["causal"]:
                    row = torch.arange(i0, min(n, i0 + block), device=DEV)
                    w = w.masked_fill(pos[None, None] > (lens[b] - n + row)[None, :, None], -math.inf)
                out[b, i0:i0 + block] = (torch.softmax(w, dim=-1).nan_to_num(0.0) @ vv).transpose(0, 1)
        return out.view(B * n, H * hd)
    if case["op"] == "append":
        hd, H, hk, T = case["head_dim"], case["heads"], case["kv_heads"], case["tokens"]
        pairs, n_pos = s["pairs"], s["n_pos"]
        ang, base = [], 0
        for a in range(len(pairs)):
            span = pairs[a] * n_pos[a]
            cs = s["rotation"][base:base + span].view(n_pos[a], pairs[a], 2)
            ang.append(torch.view_as_complex(cs.to(f).contiguous())[s["pos"][:, a].long()])
            base += span
        turn = torch.cat(ang, dim=1)[:, None]                         # [T, 1, hd / 2] unit complex numbers

        def rotate(x, heads, gamma):
            x = x.to(f).reshape(T, heads, hd)
            x = x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / hd + 1e-6) * gamma.to(f)
            if case["half_split"]:
                z = torch.complex(x[..., :hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * turn
                return torch.cat([z.real, z.imag], -1).reshape(T, heads * hd)
            z = torch.view_as_complex(x.reshape(T, heads, hd // 2, 2).contiguous()) * turn
            return torch.view_as_real(z).reshape(T, heads * hd)

        k, v = s["k"].to(f), s["v"].to(f)
        kn, vn = rotate(s["k_new"], hk, s["gamma_k"]), s["v_new"].to(f)
        flat_k, flat_v = k.view(-1, hk * hd), v.view(-1, hk * hd)
        here = torch.full((flat_k.shape[0],), -1, dtype=torch.long, device=DEV)
        ok = torch.nonzero(s["slots"] >= 0)[:, 0]
        here[s["slots"][ok].long()] = ok
        put = (here >= 0)[:, None]
        flat_k.copy_(torch.where(put, kn[here.clamp(min=0)], flat_k))
        flat_v.copy_(torch.where(put, vn[here.clamp(min=0)], flat_v))
        return {"q": rotate(s["q"], H, s["gamma_q"]), "k": k, "v": v}
    # pages: the same moves one by one on the host's lists
    ref, ps = s["ref"].tolist(), case["page"]
    k, v = s["k"].to(f), s["v"].to(f)
    if case["op"] == "fork":
        part, last = case["length"] % ps, s["table"][0, case["length"] // ps - (case["length"] % ps == 0)].item()
        free = [p for p, r in enumerate(ref) if r == 0]
        if part:
            for page in free[:case["children"]]:
                k[:, page, :part] = k[:, last, :part]
                v[:, page, :part] = v[:, last, :part]
        return {"slots": None, "k": k, "v": v, "ref": None, "table": None, "len": None}
    live = sum(r > 0 for r in ref)
    holes = [p for p in range(live) if ref[p] == 0]
    movers = [p for p in range(live, len(ref)) if ref[p] > 0]
    for a, b in zip(holes, movers):
        k[:, a], v[:, a] = k[:, b], v[:, b]
    return {"live": None, "k": k, "v": v, "ref": None, "table": None}
