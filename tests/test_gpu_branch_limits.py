"""Branched rollouts where calls meet their limits: a full pool, ids that are
not in use, a bad first sequence, other streams, captured graphs, long rows
and thousands of branches, against the plain restatements of test_gpu_branch.

Tolerances are those of test_gpu_branch: page operations exact; bf16 attention
rel-L2 5e-3, fp32 5e-6; bf16 norm 2.3e-3; two fp32 layers 2e-5.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402
from test_gpu_branch import (DEV, PageModel, check_attention, host, i32, make_cache, plain_layers, rand,  # noqa: E402
                             ref_attention, ref_rotate, rel_l2, tdt)

D, H, HK, HD = 256, 4, 2, 32


class Rollout:
    """BranchedLayers (fp32, two layers) with the tokens of every sequence kept on the host."""

    def __init__(self, n_pages, max_seqs=8, max_len=160):
        from paper_2604_20289_gb300.branches import BranchedLayers, random_layers
        self.weights = random_layers(2, D, H, HK, HD, "f32", seed=4)
        self.m = BranchedLayers(self.weights, H, HK, HD, n_pages=n_pages, page_size=16, max_seqs=max_seqs,
                                max_len=max_len, dtype="f32")
        self.rng = np.random.default_rng(2)
        self.text = {}

    def tokens(self, n_seqs, n):
        return torch.from_numpy(self.rng.standard_normal((n_seqs, n, D))).float().to(DEV)

    def new(self):
        s = self.m.new()
        self.text[s] = np.zeros((0, D))
        return s

    def fork(self, seq, n):
        kids = self.m.fork(seq, n)
        for k in kids:
            self.text[k] = self.text[seq]
        return kids

    def step(self, seqs, n):
        x = self.tokens(len(seqs), n)
        y = self.m.step(seqs, x)
        self.check(seqs, x, y)

    def check(self, seqs, x, y):
        n = x.shape[1]
        for i, s in enumerate(seqs):
            self.text[s] = np.concatenate([self.text[s], host(x[i])])
            err = rel_l2(host(y[i]), plain_layers(self.weights, H, HK, HD, self.text[s])[-n:])
            assert err <= 2e-5, err
        assert xb.op_device_error() == 0

    def state(self):
        c, m = self.m.cache, self.m
        return [t.tolist() for t in (c.ref, c.table, c.len)] + [list(m.length), list(m._free)]


def test_a_full_pool_is_refused_before_anything_changes():
    r = Rollout(n_pages=5)
    m = r.m
    root = r.new()
    r.step([root], 37)                                    # 3 pages of 5
    before = r.state()
    with pytest.raises(ValueError):
        m.fork(root, 3)                                   # 3 copies of the last page
    with pytest.raises(ValueError):
        m.step([root], r.tokens(1, 44))                   # 81 tokens: 6 pages
    assert r.state() == before and xb.op_device_error() == 0
    kids = r.fork(root, 2)                                # the pool is full
    before = r.state()
    with pytest.raises(ValueError):
        m.step(kids, r.tokens(2, 12))                     # 49 tokens each: a fourth page
    with pytest.raises(ValueError):
        m.step([root], r.tokens(1, 12))
    assert r.state() == before and xb.op_device_error() == 0
    r.step(kids, 11)                                      # what still fits
    m.free([root])                                        # its last page only: the others are the children's
    r.step([kids[0]], 1)
    with pytest.raises(ValueError):
        m.step([kids[1]], r.tokens(1, 1))
    m.free([kids[0]])
    r.step([kids[1]], 17)
    m.free([kids[1]])
    assert int(m.cache.ref.sum()) == 0
    other = r.new()
    r.step([other], 80)                                   # the whole pool again


def test_shared_parts_and_pages_in_use_follow_the_tables():
    """Forks of forks, grown and freed in any order: what the host counts is what the device's tables hold."""
    r = Rollout(n_pages=60, max_seqs=10)
    m, rng = r.m, np.random.default_rng(6)
    live = [m.new()]
    for _ in range(80):
        op = rng.integers(4)
        some = [int(s) for s in rng.permutation(live)[:rng.integers(1, 4)]]
        if op == 0 and len(live) < 9:
            live += m.fork(some[0], int(rng.integers(0, 3)))
        elif op == 1 and len(live) > 3:
            m.free(some[:2])
            live = [s for s in live if s not in some[:2]]
        else:
            n = int(rng.integers(1, 21))
            if max(m.length[s] for s in some) + n <= m.max_len:
                try:
                    m.step(some, r.tokens(len(some), n))
                except ValueError:
                    m.free([live.pop()])
        table, ref = m.cache.table.tolist(), m.cache.ref
        pages = 60 - int((ref > 0).sum())                 # what is free: one page more is refused
        if m.length[live[0]] % 16 == 0 and m.length[live[0]] + 16 * pages + 16 <= m.max_len:
            with pytest.raises(ValueError):
                m.step(live[:1], r.tokens(1, 16 * pages + 1))
        for a in live:
            for b in live:
                n = min(m.length[a], m.length[b]) // 16
                same = next((i for i in range(n) if table[a][i] != table[b][i]), n)
                assert m.shared_len([a, b]) == 16 * same
        assert m.cache.len.tolist() == m.length and xb.op_device_error() == 0
    m.free(live)
    assert int(m.cache.ref.sum()) == 0


def test_ids_are_refused_before_anything_changes():
    r = Rollout(n_pages=20)
    m = r.m
    a = r.new()
    r.step([a], 20)
    b = r.fork(a, 1)[0]
    x = r.tokens(2, 1)
    before = r.state()
    for ids in ([a, a], [a, 7], [b, -1], [b, 8]):         # twice, not in use, out of range
        with pytest.raises(ValueError):
            m.step(ids, x)
        with pytest.raises(ValueError):
            m.free(ids)
        assert r.state() == before
    for s in (7, -1, 8):
        with pytest.raises(ValueError):
            m.fork(s, 1)
        with pytest.raises(ValueError):
            m.shared_len([a, s])
    assert m.shared_len([a, b, a]) == 16
    assert r.state() == before and xb.op_device_error() == 0
    m.free(s for s in [b])
    with pytest.raises(ValueError):
        m.free([b])                                       # no longer in use
    ids = [r.new() for _ in range(7)]
    assert len(set(ids + [a])) == 8                       # no id is handed out twice
    with pytest.raises(ValueError):
        m.new()
    r.step([a, ids[3]], 2)


def test_a_refused_call_takes_no_sequences():
    """More children than one fork call of the library takes."""
    r = Rollout(n_pages=40, max_seqs=1500)
    root = r.new()
    r.step([root], 16)
    before = r.state()
    with pytest.raises((ValueError, xb.XCacheError)):
        r.m.fork(root, 1400)
    assert r.state() == before
    kids = r.fork(root, 3)
    r.step(kids, 2)


def test_a_step_without_memory_changes_nothing(monkeypatch):
    """Whichever allocation fails, the object and the device stay as they were, and the step can be made again."""
    r = Rollout(n_pages=40)
    root = r.new()
    r.step([root], 37)
    kids = r.fork(root, 3)
    x = r.tokens(3, 9)
    before = r.state()
    made = {name: getattr(torch, name) for name in ("empty", "empty_like", "tensor")}
    fails = 0
    while True:
        left = [fails]

        def limited(name):
            def make(*args, **kw):
                if left[0] == 0:
                    raise torch.cuda.OutOfMemoryError(name)
                left[0] -= 1
                return made[name](*args, **kw)
            return make

        for name in made:
            monkeypatch.setattr(torch, name, limited(name))
        try:
            y = r.m.step(kids, x)
        except torch.cuda.OutOfMemoryError:
            y = None
        monkeypatch.undo()
        if y is not None:
            break
        assert r.state() == before and xb.op_device_error() == 0
        fails += 1
    assert fails >= 8
    r.check(kids, x, y)


def test_a_step_of_a_host_tensor_is_refused():
    r = Rollout(n_pages=20)
    root = r.new()
    r.step([root], 20)
    before = r.state()
    for x in (r.tokens(1, 2).cpu(), r.tokens(1, 2)[0], r.tokens(2, 2), r.tokens(1, 2)[..., :-1]):
        with pytest.raises(ValueError):
            r.m.step([root], x)
    assert r.state() == before and xb.op_device_error() == 0
    r.step([root], 2)


def test_a_step_that_the_attention_refuses_changes_nothing(monkeypatch):
    r = Rollout(n_pages=20)
    root = r.new()
    r.step([root], 20)
    before = r.state()
    monkeypatch.setattr(xb, "op_branch_attention_workspace_bytes", lambda *a: 0)   # as for too many query rows
    with pytest.raises(xb.XCacheError):
        r.m.step([root], r.tokens(1, 2))
    monkeypatch.undo()
    assert r.state() == before
    r.step([root], 2)


@pytest.mark.parametrize("name", ["qkv_w", "o_w", "qkv_b", "o_b", "gamma_q", "gamma_k"])
def test_weights_of_other_shapes_or_types_are_refused(name):
    from paper_2604_20289_gb300.branches import BranchedLayers, random_layers

    def build(weights, dtype="f32"):
        return BranchedLayers(weights, H, HK, HD, n_pages=8, page_size=16, max_seqs=2, max_len=64, dtype=dtype)

    good = random_layers(2, D, H, HK, HD, "f32", seed=1)
    build(good)
    t = good[1][name]
    for wrong in (t[:-1], t.double(), t.cpu(), torch.cat([t, t]), t.repeat_interleave(2, dim=-1)[..., ::2]):
        with pytest.raises(ValueError):
            build([good[0], {**good[1], name: wrong}])
    with pytest.raises(ValueError):
        build(good, "bf16")                               # fp32 weights of a bf16 stack


@pytest.mark.parametrize("dtype,name", [(xb.XC_F32, "f32"), (xb.XC_BF16, "bf16")])
def test_types_by_their_codes(dtype, name):
    from paper_2604_20289_gb300.branches import BranchedLayers, random_layers
    m = BranchedLayers(random_layers(1, D, H, HK, 64, name), H, HK, 64, n_pages=8, page_size=16, max_seqs=2, max_len=64,
                       dtype=dtype)
    y = m.step([m.new()], torch.ones(1, 3, D, device=DEV))
    assert y.dtype == tdt(name) and bool(torch.isfinite(y).all()) and xb.op_device_error() == 0


@pytest.mark.parametrize("dtype,d,h,hk,hd,page", [
    ("bf16", 128, 4, 4, 64, 16), ("bf16", 256, 3, 1, 64, 16),     # widths that the bf16 linear operator does not take
    ("bf16", 256, 8, 8, 32, 16),                                  # a head size that the bf16 attention does not read
    ("f32", 256, 3, 2, 32, 16), ("f32", 256, 130, 2, 16, 16),     # heads that are not shared evenly, or by too many
    ("f32", 40, 4, 2, 32, 16), ("f32", 256, 4, 2, 48, 16), ("f32", 256, 4, 2, 32, 24)])
def test_sizes_that_a_step_would_refuse_are_refused_at_once(dtype, d, h, hk, hd, page):
    from paper_2604_20289_gb300.branches import BranchedLayers, random_layers
    with pytest.raises(xb.XCacheError):
        BranchedLayers(random_layers(1, d, h, hk, hd, dtype), h, hk, hd, n_pages=8, page_size=page, max_seqs=2,
                       max_len=64, dtype=dtype)
    assert xb.op_device_error() == 0


@pytest.mark.parametrize("eps", [-1e-6, float("nan"), float("inf")])
def test_an_eps_that_the_norm_refuses_is_refused_at_once(eps):
    from paper_2604_20289_gb300.branches import BranchedLayers, random_layers
    weights = random_layers(1, D, H, HK, HD, "f32")
    with pytest.raises(xb.XCacheError):
        BranchedLayers(weights, H, HK, HD, n_pages=8, page_size=16, max_seqs=2, max_len=64, dtype="f32", eps=eps)
    m = BranchedLayers(weights, H, HK, HD, n_pages=8, page_size=16, max_seqs=2, max_len=64, dtype="f32", eps=0.0)
    assert xb.op_device_error() == 0 and int(m.cache.ref.sum()) == 0


@pytest.mark.parametrize("dtype,H,hk,hd,n_q", [("bf16", 8, 1, 64, 1), ("bf16", 8, 1, 128, 1), ("bf16", 4, 4, 64, 9),
                                               ("f32", 8, 1, 32, 1)])
@pytest.mark.parametrize("bad", [-1, 33, 1 << 30])
def test_shared_keys_of_a_bad_first_sequence_are_zeros(dtype, H, hk, hd, n_q, bad):
    """The shared part is read from the first listed sequence's row: an id out of range there is
    flagged, and the other branches see keys and values of zero in its place."""
    lens, shared = [320 + n_q + (7 * b) % 40 for b in range(33)], 320
    cache = make_cache(dtype, hk, hd, 16, lens, shared)
    seqs = [bad] + list(range(1, 33))
    q = rand((33 * n_q, H * hd), dtype, 8, 1.5)
    o = torch.full_like(q, float("nan"))
    good = torch.empty_like(q)
    xb.op_branch_attention(cache, 0, i32(list(range(33))), n_q, q, good, shared_len=shared, causal=True)
    assert xb.op_device_error() == 0
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, o, shared_len=shared, causal=True)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    pages = cache.table[0, :shared // 16].long()
    cache.k[:, pages] = 0
    cache.v[:, pages] = 0
    want = ref_attention(cache, 0, list(range(33)), n_q, q, True)
    got = host(o)
    assert (got[:n_q] == 0).all()
    assert rel_l2(got[n_q:], want[n_q:]) <= (5e-3 if dtype == "bf16" else 5e-6)


def test_integers_in_place_of_float_operands_are_refused():
    """Four-byte integers have the size of a float, not its meaning."""
    cache = make_cache("bf16", 2, 64, 16, [40, 50], 32, dead=0.0)
    x, out = rand((2, 128), "bf16", 4), rand((2, 128), "bf16", 5)
    gamma, table = torch.ones(64, device=DEV), torch.zeros(2 * 32 * 64, device=DEV)
    args = [gamma, gamma, table]
    for i in range(3):
        a = [t.int() if j == i else t for j, t in enumerate(args)]
        with pytest.raises(ValueError):
            xb.op_qk_norm_rope(cache, 0, x, x, x, a[0], a[1], i32([0, 1]), [32], [64], a[2], i32([0, 1]), out)
    with pytest.raises(ValueError):
        xb.op_rope_table([32], [64], 1e4, table.int())
    assert xb.op_device_error() == 0


def test_captured_calls_have_workspaces_of_their_own():
    """A larger call on the capture's stream and replays on another stream leave a graph's results,
    the other calls' results and other memory as they are."""
    small = make_cache("bf16", 2, 64, 16, [700 + 9 * b for b in range(8)], 640, dead=0.0)
    cache = xb.KVCache("bf16", 2, 64, torch.cat([small.k] * 2, 1), torch.cat([small.v] * 2, 1),
                       torch.cat([small.ref, torch.zeros_like(small.ref)]),
                       torch.nn.functional.pad(small.table, (0, 8), value=-1).contiguous(), small.len)
    q, seqs = rand((8, 8 * 64), "bf16", 3), i32(list(range(8)))
    qs, few = rand((8 * 300, 8 * 64), "bf16", 4), i32(list(range(8)))
    o, big = torch.empty_like(q), torch.empty_like(qs)
    want, want_big = torch.empty_like(q), torch.empty_like(qs)
    xb.op_branch_attention(cache, 0, seqs, 1, q, want, shared_len=640, causal=True)
    xb.op_branch_attention(cache, 0, few, 300, qs, want_big, causal=True)
    st, other = torch.cuda.Stream(), torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    slots = torch.empty(8, 1, dtype=torch.int32, device=DEV)
    with torch.cuda.stream(st):
        xb.op_branch_attention(cache, 0, seqs, 1, q, o, shared_len=640, causal=True)
    st.synchronize()
    kept = cache._ws[st.cuda_stream]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        xb.op_kv_extend(cache, seqs, 0, slots[:, :0])      # no work, no page taken
        xb.op_branch_attention(cache, 0, seqs, 1, q, o, shared_len=640, causal=True)
    assert cache._ws[st.cuda_stream] is kept               # the capture has put nothing in its place
    with torch.cuda.stream(st):
        xb.op_branch_attention(cache, 0, few, 300, qs, big, causal=True)
    st.synchronize()
    assert cache._ws[st.cuda_stream][2] > kept[2]
    size = kept[2]
    del kept
    fresh = []
    for s in (st, other, torch.cuda.current_stream()):     # what the allocator hands out now is not the graph's
        with torch.cuda.stream(s):
            fresh += [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    for i in range(20):
        o.fill_(float("nan"))
        big.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            graph.replay()
        with torch.cuda.stream(st):
            xb.op_branch_attention(cache, 0, few, 300, qs, big, causal=True)
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(big, want_big)
    assert all(bool((f == 7).all()) for f in fresh)
    assert xb.op_device_error() == 0


def test_workspaces_of_the_caller():
    cache = xb.KVCache.empty("bf16", 1, 12, 16, 1, 64, 4, 4)
    cache.k.zero_()
    cache.v.zero_()
    need = xb.op_kv_workspace_bytes(cache)
    ws = torch.full((need + 16,), 0x5A, dtype=torch.uint8, device=DEV)
    slots, live = i32([[0] * 20]), i32([0])
    xb.op_kv_extend(cache, i32([0]), 20, slots, workspace=ws[:need])
    xb.op_kv_fork(cache, i32([0]), i32([1]), workspace=ws[:need])
    xb.op_kv_free(cache, i32([0]))
    xb.op_kv_compact(cache, live, workspace=ws[:need])
    assert xb.op_device_error() == 0 and live.item() == 2 and cache.table[1].tolist() == [0, 1, -1, -1]
    assert bool((ws[need:] == 0x5A).all()) and not cache._ws
    q = rand((1, 64), "bf16", 1)
    o = torch.empty_like(q)
    calls = [lambda w: xb.op_kv_extend(cache, i32([1]), 1, i32([[0]]), workspace=w),
             lambda w: xb.op_kv_fork(cache, i32([1]), i32([2]), workspace=w),
             lambda w: xb.op_kv_compact(cache, live, workspace=w),
             lambda w: xb.op_branch_attention(cache, 0, i32([1]), 1, q, o, workspace=w)]
    state = [t.clone() for t in (cache.ref, cache.table, cache.len)]
    for call in calls:
        with pytest.raises(ValueError):
            call(ws.cpu())
        with pytest.raises(ValueError):
            call(ws[:16].expand(1 << 20, 16))              # 16 bytes that look like 16 MB
        with pytest.raises(xb.XCacheError):
            call(ws[:32])
    for a, b in zip(state, (cache.ref, cache.table, cache.len)):
        assert torch.equal(a, b)
    assert xb.op_device_error() == 0


def test_a_handle_does_not_grow_with_the_shapes_it_has_seen():
    cache = xb.KVCache.empty("bf16", 1, 8, 16, 1, 64, 2, 4)
    q, none = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), i32([])
    table, gamma = torch.zeros(64 * 9000, device=DEV), torch.ones(64, device=DEV)
    for n in range(1, 9000):
        xb.op_qk_norm_rope(cache, 0, q, q, q, gamma, gamma, none, [32], [n], table[:64 * n], none, q)
        xb.op_branch_attention(cache, 0, none, n, q, q)
    assert len(cache._axes) <= 4096 and len(cache._attn_bytes) <= 4096
    assert xb.op_device_error() == 0


def test_steps_on_other_streams():
    """Built on one stream, called on others, each behind a delay, with no event of the caller's
    between the calls: the object orders them, and inputs and outputs are of the calling stream."""
    main, a, b = torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()
    r = Rollout(n_pages=40)
    m = r.m
    torch.cuda.synchronize()
    raw = [r.tokens(1, 37), r.tokens(3, 2), r.tokens(3, 5), r.tokens(2, 3)]
    torch.cuda.synchronize()
    got = []

    def step(seqs, i):
        torch.cuda._sleep(20_000_000)                     # some 10 ms: what was not ordered would run before it
        x = raw[i] + 1.0                                  # made on this stream, behind the delay
        y = m.step(seqs, x)
        got.append((seqs, x, y, y + 0.0))                 # read on this stream
        del x
        torch.full((1 << 20,), float("nan"), device=DEV)  # memory that the call has let go of

    with torch.cuda.stream(a):
        root = r.new()
        step([root], 0)
    with torch.cuda.stream(b):
        kids = r.fork(root, 3)
        step(kids, 1)
    torch.full((1 << 20,), float("nan"), device=DEV)      # on the stream that the object was made on
    step(kids, 2)
    with torch.cuda.stream(a):
        m.free([root, kids[2]])
        live = m.compact()
        step(kids[:2], 3)
    torch.cuda.synchronize()
    assert m.cache.len.tolist() == [{k: 47 for k in kids[:2]}.get(s, 0) for s in range(8)]
    assert int(live) == int((m.cache.ref > 0).sum())      # (the last step stays within its pages)
    for i, (seqs, x, y, z) in enumerate(got):
        assert torch.equal(y, z)
        if i == 1:
            for k in kids:
                r.text[k] = r.text[root]
        r.check(seqs, x, y)
    assert main == torch.cuda.current_stream()


@pytest.mark.parametrize("n,sources,pages", [(1, 1, 8400), (16, 1, 600), (16, 3, 530), (64, 4, 150), (1000, 7, 13),
                                             (1024, 1, 12)])
@pytest.mark.parametrize("part", [0, 5])
def test_forks_of_long_rows_and_many_pairs(n, sources, pages, part):
    """Rows longer than what the plan's threads keep in registers, several children per source."""
    ps, max_seqs, n_pages = 16, n + sources, sources * (pages + 1) + n + 9
    cache = xb.KVCache.empty("bf16", 1, n_pages, ps, 1, 16, max_seqs, pages + 1)
    n_rows = n_pages * ps
    cache.k.copy_(rand(tuple(cache.k.shape), "bf16", 1))
    cache.v.copy_(rand(tuple(cache.v.shape), "bf16", 2))
    first = [host(t[0]).reshape(n_rows, -1) for t in (cache.k, cache.v)]
    m = PageModel(n_pages, ps, max_seqs, pages + 1, np.arange(n_rows).reshape(n_pages, ps))
    src = list(range(sources))
    n_new = pages * ps + part
    slots = torch.empty(sources, n_new, dtype=torch.int32, device=DEV)
    xb.op_kv_extend(cache, i32(src), n_new, slots)
    assert slots.tolist() == m.extend(src, n_new)
    rng = np.random.default_rng(7)
    pairs = [(int(rng.integers(sources)), sources + int(d)) for d in rng.permutation(n)]
    a, b = i32([p[0] for p in pairs]), i32([p[1] for p in pairs])
    tail = int(cache.table[pairs[-1][0], pages - 1])
    for wrong in (n_pages, -3):                           # a bad page id in the row's last part: nothing changes
        cache.table[pairs[-1][0], pages - 1] = wrong
        xb.op_kv_fork(cache, a, b)
        assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
        assert cache.ref.tolist() == m.ref and cache.len.tolist() == m.len
    cache.table[pairs[-1][0], pages - 1] = tail
    xb.op_kv_fork(cache, a, b)
    assert m.fork(pairs) and xb.op_device_error() == 0
    m.check(cache, lambda layer, x: first[x])
    xb.op_kv_free(cache, b)
    m.free([p[1] for p in pairs])
    assert cache.ref.tolist() == m.ref and xb.op_device_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_thousands_of_branches(dtype):
    check_attention(dtype, 2, 1, 64, 16, [32 + (7 * b) % 30 for b in range(3000)], 1, 32, True)
    check_attention(dtype, 2, 2, 64, 16, [(11 * b) % 37 for b in range(2500)], 2, 0, True)


def test_a_whole_planning_step_in_one_graph():
    """fork, extend, norm and append, attention, free: captured once, replayed with other inputs and
    a history that grew in between."""
    hk, Hq, hd, ps, eps, n = 2, 4, 64, 16, 1e-6, 3
    cache = xb.KVCache.empty("bf16", 2, 64, ps, hk, hd, 6, 8)
    cache.k.zero_()
    cache.v.zero_()
    table = torch.empty(2 * 32 * 128, device=DEV)
    xb.op_rope_table([32], [128], 1e4, table)
    gq, gk = rand((hd,), "f32", 1), rand((hd,), "f32", 2)
    root, kids = i32([0]), i32([3, 1, 4])
    qkv = torch.empty(n, (Hq + 2 * hk) * hd, dtype=torch.bfloat16, device=DEV)
    pos, slots = i32([[0]] * n), torch.empty(n, 1, dtype=torch.int32, device=DEV)
    q, o = (torch.empty(n, Hq * hd, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    heads = (qkv[:, :Hq * hd], qkv[:, Hq * hd:(Hq + hk) * hd], qkv[:, (Hq + hk) * hd:])

    def grow(m, seed):                                    # m tokens of history, keys and values at random
        s = torch.empty(1, m, dtype=torch.int32, device=DEV)
        xb.op_kv_extend(cache, root, m, s)
        for t, x in ((cache.k, seed), (cache.v, seed + 1)):
            t[1].view(-1, hk * hd)[s.long().view(-1)] = rand((m, hk * hd), "bf16", x)

    def plan():
        xb.op_kv_fork(cache, root.expand(n).contiguous(), kids)
        xb.op_kv_extend(cache, kids, 1, slots)
        xb.op_qk_norm_rope(cache, 1, *heads, gq, gk, pos, [32], [128], table, slots.view(-1), q, eps=eps)
        xb.op_branch_attention(cache, 1, kids, 1, q, o, shared_len=32, causal=True)
        xb.op_kv_free(cache, kids)

    grow(41, 10)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        plan()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        plan()
    for i in range(4):
        length = int(cache.len[0])
        qkv.copy_(rand(tuple(qkv.shape), "bf16", 20 + i))
        pos.fill_(length)
        o.fill_(float("nan"))
        graph.replay()
        assert xb.op_device_error() == 0
        at = slots.view(-1).tolist()
        assert len(set(at)) == n
        ang = np.full((n, 1), length)
        assert rel_l2(host(q), ref_rotate(host(heads[0]), Hq, hd, host(gq), ang, [32], 1e4, False, eps)) <= 2.3e-3
        k, v = (host(t[1]).reshape(-1, hk * hd) for t in (cache.k, cache.v))
        assert rel_l2(k[at], ref_rotate(host(heads[1]), hk, hd, host(gk), ang, [32], 1e4, False, eps)) <= 2.3e-3
        np.testing.assert_array_equal(v[at], host(heads[2]))
        j = np.arange(length)
        rows = cache.table[0].cpu().numpy()[j // ps] * ps + j % ps
        got = host(o).reshape(n, Hq, hd)
        for b in range(n):
            kk = np.concatenate([k[rows], k[at[b]][None]]).reshape(-1, hk, hd)
            vv = np.concatenate([v[rows], v[at[b]][None]]).reshape(-1, hk, hd)
            w = np.einsum("hd,jhd->hj", host(q)[b].reshape(Hq, hd), kk.repeat(Hq // hk, axis=1)) / np.sqrt(hd)
            w = np.exp(w - w.max(1, keepdims=True))
            want = np.einsum("hj,jhd->hd", w / w.sum(1, keepdims=True), vv.repeat(Hq // hk, axis=1))
            assert rel_l2(got[b], want) <= 5e-3
        assert cache.len.tolist() == [length] + [0] * 5
        assert int(cache.ref.sum()) == -(-length // ps)
        grow(6 + i, 50 + 2 * i)
        assert xb.op_device_error() == 0
