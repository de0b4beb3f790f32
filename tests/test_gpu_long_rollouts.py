"""Long branched rollouts: 8-bit projections, attention with its rows' sums, weights of
the cached keys and eviction by them, as BranchedLayers runs them together, against the
same layers in 64 bits (which take the device's choice of tokens, after checking it)."""
import math

import numpy as np
import pytest
import torch

from paper_2604_20289_gb300 import xcache as xb
from tests.test_gpu_branch import DEV, host, ref_rotate, rel_l2, tdt

pytestmark = pytest.mark.gpu


def quantised(x):
    """Rows as 8-bit integers times their scale: nearest integers of 127 x / max |x|, halves to even."""
    a = np.abs(x).max(-1, keepdims=True)
    return np.where(a > 0, np.rint(127.0 * x / np.where(a > 0, a, 1.0)) * a / 127.0, 0.0)


class Plain:
    """The layers on one sequence, in 64 bits, with what its cache keeps."""

    def __init__(self, weights, H, hk, hd, track):
        self.w, self.H, self.hk, self.hd, self.track = weights, H, hk, hd, track
        self.pos = 0
        self.k = [np.zeros((0, hk, hd)) for _ in weights]
        self.v = [np.zeros((0, hk, hd)) for _ in weights]
        self.weight = np.zeros(0)

    def copy(self):
        p = Plain(self.w, self.H, self.hk, self.hd, self.track)
        p.pos, p.k, p.v, p.weight = self.pos, list(self.k), list(self.v), self.weight.copy()
        return p

    def linear(self, x, w, name):
        m = host(w[name + "_w"])
        if w[name + "_w"].dtype is torch.int8:
            x, m = quantised(x), m * host(w[name + "_s"])[:, None]
        return x @ m.T + host(w[name + "_b"])

    def step(self, x, eps=1e-6, theta=1e4):
        n, H, hk, hd = x.shape[0], self.H, self.hk, self.hd
        self.weight = np.concatenate([self.weight * self.track, np.zeros(n)])
        pos = self.pos + np.arange(n)[:, None]
        for i, w in enumerate(self.w):
            h = (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + eps)
            qkv = self.linear(h, w, "qkv")
            q = ref_rotate(qkv[:, :H * hd], H, hd, host(w["gamma_q"]), pos, [hd // 2], theta, False, eps).reshape(n, H, hd)
            k = ref_rotate(qkv[:, H * hd:(H + hk) * hd], hk, hd, host(w["gamma_k"]), pos, [hd // 2], theta, False, eps)
            self.k[i] = np.concatenate([self.k[i], k.reshape(n, hk, hd)])
            self.v[i] = np.concatenate([self.v[i], qkv[:, (H + hk) * hd:].reshape(n, hk, hd)])
            kk, vv = (t[i].repeat(H // hk, axis=1) for t in (self.k, self.v))
            s = np.einsum("ihd,jhd->hij", q, kk) / math.sqrt(hd)
            L = kk.shape[0]
            s[:, np.arange(L)[None] > L - n + np.arange(n)[:, None]] = -np.inf
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            self.weight = self.weight + p.sum((0, 1))
            x = x + self.linear(np.einsum("hij,jhd->ihd", p, vv).reshape(n, H * hd), w, "o")
        self.pos += n
        return x

    def keep(self, kept):
        self.k, self.v = [k[kept] for k in self.k], [v[kept] for v in self.v]
        self.weight = self.weight[kept]


def chosen(weights, length, keep, first, last):
    """The tokens that stay, by the device's own weights."""
    if length <= keep:
        return list(range(length))
    mid = np.arange(first, length - last)
    order = mid[np.lexsort((mid, -weights[mid]))][:keep - first - last]
    return list(range(first)) + sorted(order.tolist()) + list(range(length - last, length))


class Rollout:
    def __init__(self, dtype, int8, H, hk, hd, tol, tol_w, track=0.9, **sizes):
        from paper_2604_20289_gb300 import branches
        self.d, self.dtype, self.tol, self.tol_w = 256, dtype, tol, tol_w
        w = branches.random_layers(2, self.d, H, hk, hd, dtype, seed=4)
        w = branches.quantize_layers(w, dtype) if int8 else w
        sizes = dict(dict(n_pages=60, page_size=16, max_seqs=8, max_len=96, max_pos=300), **sizes)
        self.m = branches.BranchedLayers(w, H, hk, hd, dtype=dtype, track=track, **sizes)
        self.rng = np.random.default_rng(2)
        self.make = lambda: Plain(w, H, hk, hd, track)
        self.plain = {}

    def new(self):
        s = self.m.new()
        self.plain[s] = self.make()
        return s

    def fork(self, s, n):
        kids = self.m.fork(s, n)
        for k in kids:
            self.plain[k] = self.plain[s].copy()
        return kids

    def free(self, seqs):
        self.m.free(seqs)
        for s in seqs:
            del self.plain[s]

    def step(self, seqs, n):
        x = torch.from_numpy(self.rng.standard_normal((len(seqs), n, self.d))).to(DEV).to(tdt(self.dtype))
        y = host(self.m.step(seqs, x))
        for i, s in enumerate(seqs):
            want = self.plain[s].step(host(x[i]))
            assert rel_l2(y[i], want) <= self.tol, rel_l2(y[i], want)
        self.check()

    def check(self):
        m = self.m
        assert xb.op_device_error() == 0
        assert m.cache.len.tolist() == m.length and m._used == int((m.cache.ref > 0).sum())
        got = host(m.key_weights)
        for s in range(len(m.length)):
            L = m.length[s]
            assert not got[s, L:].any()
            if s in self.plain:
                p = self.plain[s]
                assert m.position[s] == p.pos and L == len(p.weight)
                assert L == 0 or rel_l2(got[s, :L], p.weight) <= self.tol_w, rel_l2(got[s, :L], p.weight)

    def evict(self, seqs, keep, first, last):
        m = self.m
        before, lens = m.key_weights.cpu().numpy().copy(), list(m.length)
        kept = m.evict(seqs, keep, first, last)
        after = m.key_weights.cpu().numpy()
        for i, s in enumerate(seqs):
            assert kept[i] == chosen(before[s], lens[s], keep, first, last)
            assert (after[s, :len(kept[i])] == before[s, kept[i]]).all()
            self.plain[s].keep(kept[i])
        self.check()


# Outputs.  fp32: a few 1e-6 a layer.  With 8-bit products a rounding that falls the other way changes
# one of 256 elements of a token by a 127th of its row's largest, some 0.17 % of the token's output: three of them.
# bf16: some ten roundings of 2^-9 a layer; where the projections round to 8 bits, a fifth of the elements may
# fall the other way, 1 % of each of four products' outputs.
# Weights of keys: the error of a score is that of q and k together; 1e-4 of fp32's, 1e-2 with three elements the
# other way, and for bf16 twice the outputs' 2e-2 and sqrt(2) x 4e-2.
CASES = [("f32", False, 4, 2, 32, 2e-5, 1e-4), ("f32", True, 4, 2, 32, 5e-3, 1e-2), ("bf16", False, 8, 4, 64, 2e-2, 4e-2),
         ("bf16", True, 8, 4, 64, 4e-2, 6e-2), ("bf16", True, 4, 1, 128, 4e-2, 6e-2)]


@pytest.mark.parametrize("dtype,int8,H,hk,hd,tol,tol_w", CASES)
def test_operators_together(dtype, int8, H, hk, hd, tol, tol_w):
    r = Rollout(dtype, int8, H, hk, hd, tol, tol_w)
    root = r.new()
    r.step([root], 70)
    kids = r.fork(root, 3)
    r.step(kids, 1)
    r.step(kids, 1)
    r.step(kids, 12)                                      # 84 tokens, 64 in common
    r.evict([kids[1], root, kids[0]], 61, 20, 16)         # 16 in common stay where they are; pages are replaced
    assert r.m.shared_len([kids[0], kids[2]]) >= 16
    r.step(kids, 3)                                       # 64, 64 and 87 tokens
    r.step([root], 34)
    grand = r.fork(kids[0], 2)
    r.step(grand + [kids[0]], 1)
    r.evict(grand, 40, 0, 8)                              # all of a common history
    r.evict([kids[0]], 64, 64, 0)                         # the last token, without looking at the weights
    r.step([kids[0]] + grand, 9)
    r.free([kids[1], kids[2]])
    live = int(r.m.compact())
    assert live == r.m._used
    fresh = r.new()                                       # where an old sequence's weights were
    r.step([fresh, root, grand[1]], 1)
    for _ in range(4):                                    # past max_len positions, in the same memory
        r.evict([grand[0], fresh], 33, 4, 16)
        r.step([grand[0], fresh], 33)
    assert r.m.position[grand[0]] > 96 >= r.m.length[grand[0]]
    r.free(list(r.plain))
    assert int(r.m.cache.ref.sum()) == 0 and r.m._used == 0 and not r.m.key_weights.any()


@pytest.mark.parametrize("keep,first,last", [(16, 0, 0), (32, 32, 0), (33, 0, 33), (47, 5, 10), (1, 0, 0), (64, 16, 16)])
def test_evict_at_page_ends(keep, first, last):
    r = Rollout("f32", False, 4, 2, 32, 2e-5, 1e-4)
    root = r.new()
    r.step([root], 64)
    kids = r.fork(root, 2)                                # no partly filled page
    r.step([kids[0]], 1)
    r.evict(kids + [root], keep, first, last)
    r.step(kids + [root], 2)
    r.evict([root], keep, first, last)
    r.step([root], 1)


def common(m, a, b):
    table, n = m.cache.table.tolist(), 0
    for i in range(min(m.length[a], m.length[b]) // m.cache.page_size):
        if table[a][i] != table[b][i]:
            break
        n += 1
    return n * m.cache.page_size


def test_pages_in_use_and_shared_parts_follow_the_tables():
    """Forks grown, evicted from and freed in any order: what the host counts is what the device holds."""
    from paper_2604_20289_gb300 import branches
    H, hk, hd, d = 2, 1, 16, 32
    m = branches.BranchedLayers(branches.random_layers(1, d, H, hk, hd, "f32"), H, hk, hd, n_pages=50, page_size=16,
                                max_seqs=10, max_len=160, max_pos=100000, dtype="f32", track=1.0)
    rng = np.random.default_rng(3)
    live, refused = [m.new()], 0
    for _ in range(250):
        op = rng.integers(5)
        some = [int(s) for s in rng.permutation(live)[:rng.integers(1, 4)]]
        state = [list(m.length), list(m.position), m._used, m.cache.table.tolist(), m.cache.ref.tolist()]
        try:
            if op == 0 and len(live) < 8:
                live += m.fork(some[0], int(rng.integers(1, 3)))
            elif op == 1 and len(live) > 4:
                m.free(some[:1])
                live.remove(some[0])
            elif op == 2:
                keep = int(rng.integers(1, 100))
                first = int(rng.integers(0, keep + 1))
                m.evict(some, keep, first, int(rng.integers(0, keep - first + 1)))
            elif op > 2:
                n = int(rng.integers(1, 30))
                if all(m.length[s] + n <= 160 for s in some):
                    m.step(some, torch.randn(len(some), n, d, device=DEV))
        except ValueError:
            refused += 1
            assert state == [list(m.length), list(m.position), m._used, m.cache.table.tolist(), m.cache.ref.tolist()]
        assert xb.op_device_error() == 0
        assert m.cache.len.tolist() == m.length and m._used == int((m.cache.ref > 0).sum())
        for a in live:
            for b in live:
                if a != b:
                    assert m.shared_len([a, b]) <= common(m, a, b)
            assert not m.key_weights[a, m.length[a]:].any()
    m.free(live)
    assert m._used == 0 and int(m.cache.ref.sum()) == 0


def test_refusals_change_nothing():
    from paper_2604_20289_gb300 import branches
    H, hk, hd, d = 4, 2, 32, 64
    w = branches.random_layers(1, d, H, hk, hd, "f32")
    size = dict(n_pages=9, page_size=16, max_seqs=4, max_len=64, dtype="f32")
    for bad in (-0.1, 1.5, float("nan")):
        with pytest.raises(ValueError):
            branches.BranchedLayers(w, H, hk, hd, track=bad, **size)
    q = branches.quantize_layers(w, "f32")
    for name, t in (("qkv_s", q[0]["qkv_s"][:-1]), ("o_s", q[0]["o_s"].double()), ("o_w", q[0]["o_w"].to(torch.int16))):
        with pytest.raises(ValueError):
            branches.BranchedLayers([dict(q[0], **{name: t})], H, hk, hd, **size)
    m = branches.BranchedLayers(w, H, hk, hd, max_pos=70, track=1.0, **size)
    root = m.new()
    m.step([root], torch.randn(1, 64, d, device=DEV))
    kids = m.fork(root, 2)                                # 4 pages of 9, all in common

    def state():
        c = m.cache
        return [t.tolist() for t in (c.ref, c.table, c.len, m.key_weights)] + [list(m.length), list(m.position), m._used]

    before = state()
    for args in (([root], 0), ([root], 8, 5, 4), ([root], 8, -1, 4), ([root], 8, 4, -1), ([root, root], 8), ([3], 8), ([9], 8),
                 ([root] + kids, 33)):                    # the last: 3 copies each of 3 pages, 5 free
        with pytest.raises(ValueError):
            m.evict(*args)
        assert state() == before and xb.op_device_error() == 0
    assert m.fork(root, 0) == [] and m.evict([], 8) == [] and m.evict([root], 64) == [list(range(64))] and state() == before
    m.evict([root], 33)
    with pytest.raises(ValueError):
        m.step([root], torch.randn(1, 7, d, device=DEV))  # there is room for the tokens, not for their positions
    m.step([root], torch.randn(1, 6, d, device=DEV))
    n = branches.BranchedLayers(w, H, hk, hd, **size)
    s = n.new()
    n.step([s], torch.randn(1, 20, d, device=DEV))
    with pytest.raises(ValueError):
        n.evict([s], 8, 4, 3)
    assert n.evict([s], 8, 4, 4) == [[0, 1, 2, 3, 16, 17, 18, 19]] and n.length[s] == 8
    assert xb.op_device_error() == 0


def test_layers_of_either_kind():
    """Sizes that only the 8-bit product takes (384 channels) are refused at once where any layer is of the other kind."""
    from paper_2604_20289_gb300 import branches
    H, hk, hd, d = 4, 1, 64, 256
    w = branches.random_layers(2, d, H, hk, hd, "bf16")
    q = branches.quantize_layers(w)
    size = dict(n_pages=8, page_size=16, max_seqs=2, max_len=64)
    for layers in (w, [q[0], w[1]], [w[0], q[1]]):
        with pytest.raises(xb.XCacheError):
            branches.BranchedLayers(layers, H, hk, hd, **size)
    odd = torch.empty(q[0]["o_w"].numel() + 16, dtype=torch.int8, device=DEV)[8:-8].view(q[0]["o_w"].shape)
    with pytest.raises(ValueError):
        branches.BranchedLayers([q[0], dict(q[1], o_w=odd)], H, hk, hd, **size)
    m = branches.BranchedLayers([q[0], dict(q[1], o_w=w[1]["o_w"])], H, hk, hd, **size)      # mixed, where both take it
    y = m.step([m.new()], torch.randn(1, 20, d, device=DEV))
    assert y.isfinite().all() and xb.op_device_error() == 0


def test_steps_and_evictions_on_streams_in_turn():
    a, b = (Rollout("f32", True, 4, 2, 32, 5e-3, 1e-2) for _ in range(2))
    streams = [torch.cuda.Stream() for _ in range(2)]
    sa, sb = a.new(), b.new()
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):           # two rollouts at a time, each in its own order
            a.step([sa], 40)
            a.evict([sa], 50, 3, 10)
        with torch.cuda.stream(streams[(i + 1) % 2]):
            b.step([sb], 23)
            b.evict([sb], 31, 0, 31)


@pytest.mark.parametrize("dtype,n_q,max_pages", [("bf16", 1, 4), ("bf16", 1, 400), ("bf16", 70, 4), ("f32", 3, 4)])
def test_offsets_past_32_bits(dtype, n_q, max_pages):
    """Pages whose element offsets pass 2^31: read for their keys' weights, and moved by an eviction."""
    ps, hk, hd, n_pages = 64, 8, 128, 40000                     # 2.6e9 elements
    if torch.cuda.mem_get_info()[0] < 32 << 30:
        pytest.skip("needs 32 GB")
    cache = xb.KVCache.empty(dtype, 1, n_pages, ps, hk, hd, 3, max_pages)
    pages, L = [n_pages - 1, n_pages - 3], 101                  # few keys, many, long rows by the table's width and n_q
    g = torch.Generator(device=DEV).manual_seed(1)

    def r(*shape):
        return torch.randn(*shape, generator=g, device=DEV).to(tdt(dtype))

    for p in pages:
        cache.k[0, p], cache.v[0, p] = r(ps, hk * hd), r(ps, hk * hd)
        cache.ref[p] = 1
    cache.table[1, :2] = torch.tensor(pages, dtype=torch.int32, device=DEV)
    cache.len[1] = L
    seqs = torch.tensor([1], dtype=torch.int32, device=DEV)
    q, w = r(n_q, 2 * hk * hd), torch.zeros(3, max_pages * ps, device=DEV)
    o, lse = torch.empty_like(q), torch.empty(n_q, 2 * hk, device=DEV)
    xb.op_branch_attention(cache, 0, seqs, n_q, q, o, causal=True, lse=lse)
    xb.op_key_weights(cache, 0, seqs, n_q, q, lse, w, causal=True)
    assert xb.op_device_error() == 0
    k = torch.cat([cache.k[0, p] for p in pages])[:L].double().view(L, hk, hd).repeat_interleave(2, 1)
    s = torch.einsum("ihd,jhd->hij", q.double().view(n_q, 2 * hk, hd), k) / math.sqrt(hd)
    s.masked_fill_(torch.arange(L, device=DEV)[None] > L - n_q + torch.arange(n_q, device=DEV)[:, None], -math.inf)
    want = torch.softmax(s, -1).sum((0, 1)).cpu().numpy()
    assert rel_l2(host(w[1, :L]), want) <= 1e-5 and not w[1, L:].any() and not w[0].any() and not w[2].any()
    before, rows = host(w[1, :L]), [torch.cat([t[0, p] for p in pages]) for t in (cache.k, cache.v)]
    kept = torch.empty(1, 70, dtype=torch.int32, device=DEV)
    xb.op_kv_evict(cache, seqs, 70, w, n_first=3, n_last=20, kept=kept)
    assert xb.op_device_error() == 0 and kept[0].tolist() == chosen(before, L, 70, 3, 20)
    for t, old in zip((cache.k, cache.v), rows):
        assert torch.equal(torch.cat([t[0, p] for p in pages])[:70], old[kept[0].long()])


def test_a_step_with_its_eviction_in_one_graph():
    """Projection, norm and rotation into the cache, attention, weights, output projection and eviction, captured once:
    replays do what the same calls do, bit by bit, while another stream makes calls of its own."""
    H, hk, hd, d, ps, n, B, keep = 8, 4, 64, 256, 16, 5, 3, 40
    dt, rows = torch.bfloat16, (8 + 2 * 4) * 64
    g = torch.Generator(device=DEV).manual_seed(2)

    def r(*shape, std=1.0):
        return std * torch.randn(*shape, generator=g, device=DEV)

    wq, ws, wo, wos = (torch.empty(s, dtype=t, device=DEV) for s, t in
                       (((rows, d), torch.int8), ((rows,), torch.float32), ((d, H * hd), torch.int8), ((d,), torch.float32)))
    xb.op_quantize_rows("bf16", r(rows, d, std=d ** -0.5).to(dt), wq, ws)
    xb.op_quantize_rows("bf16", r(d, H * hd, std=(H * hd) ** -0.5).to(dt), wo, wos)
    bias, bo, gate, gamma = r(rows, std=0.05), r(d, std=0.05), torch.ones(d, device=DEV), torch.ones(hd, device=DEV)
    rotation = torch.empty(2 * (hd // 2) * 64, device=DEV)
    xb.op_rope_table([hd // 2], [64], 1e4, rotation)
    xs = [r(B * n, d).to(dt) for _ in range(12)]

    def state():
        c = xb.KVCache.empty("bf16", 1, 20, ps, hk, hd, 4, 4)
        return dict(c=c, w=torch.zeros(4, 64, device=DEV), x=torch.zeros(B * n, d, dtype=dt, device=DEV), ids=torch.tensor([2, 0, 3], dtype=torch.int32, device=DEV),
                    pos=torch.zeros(B * n, 1, dtype=torch.int32, device=DEV), slots=torch.empty(B, n, dtype=torch.int32, device=DEV),
                    qkv=torch.empty(B * n, rows, dtype=dt, device=DEV), q=torch.empty(B * n, H * hd, dtype=dt, device=DEV),
                    o=torch.empty(B * n, H * hd, dtype=dt, device=DEV), lse=torch.empty(B * n, H, device=DEV),
                    y=torch.empty(B * n, d, dtype=dt, device=DEV), kept=torch.empty(B, keep, dtype=torch.int32, device=DEV))

    def step(s):
        c, q, dq, dk = s["c"], s["qkv"], H * hd, hk * hd
        xb.op_kv_extend(c, s["ids"], n, s["slots"])
        xb.op_linear_i8("bf16", xb.XC_EPI_BIAS, s["x"], wq, ws, bias, q)
        xb.op_qk_norm_rope(c, 0, q[:, :dq], q[:, dq:dq + dk], q[:, dq + dk:], gamma, gamma, s["pos"], [hd // 2], [64], rotation,
                           s["slots"].view(-1), s["q"])
        xb.op_branch_attention(c, 0, s["ids"], n, s["q"], s["o"], causal=True, lse=s["lse"])
        xb.op_key_weights(c, 0, s["ids"], n, s["q"], s["lse"], s["w"], causal=True, decay=0.9)
        xb.op_linear_i8("bf16", xb.XC_EPI_RESID_GATE, s["o"], wo, wos, bo, s["y"], gate=gate, resid=s["x"])
        xb.op_kv_evict(c, s["ids"], keep, s["w"], n_first=2, n_last=8, kept=s["kept"])

    eager, replayed, other = state(), state(), state()
    warm = state()
    step(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i, x in enumerate(xs):
        for s in (eager, replayed):
            s["x"].copy_(x)
            s["pos"].fill_(i)
        step(eager)
        graph.replay()
        with torch.cuda.stream(side):
            step(other)
        for name in ("y", "w", "kept", "lse"):
            assert torch.equal(eager[name].view(torch.uint8), replayed[name].view(torch.uint8)), (i, name)
        assert all(torch.equal(getattr(eager["c"], t), getattr(replayed["c"], t)) for t in ("ref", "table", "len"))
    torch.cuda.synchronize()
    assert eager["c"].len.tolist() == [keep, 0, keep, keep] and xb.op_device_error() == 0
    assert eager["kept"][:, 0].tolist() == [0] * B and int((eager["c"].ref > 0).sum()) == B * 3
