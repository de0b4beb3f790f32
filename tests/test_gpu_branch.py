"""Branched rollouts over a paged key / value cache: the page operations, the
head-wise norm with rotation that fills the pages, and the attention of a
batch of branches over a shared history, against plain 64-bit restatements.

Tolerances (derived from the arithmetic):
* page operations: copies and integers, exact.
* norm and rotation, bf16: one rounding to bf16 of an fp32 value, rel-L2 <=
  2^-8 / sqrt(3) = 2.3e-3; fp32: a sum of head_dim squares, a root and a
  rotation, a few 2^-24 each: rel-L2 <= 1e-6.
* attention, bf16: the weights are rounded to bf16 before the product with V
  (independent relative errors of 2^-9 rms / sqrt(3) per weight) and the
  output once: together well under rel-L2 5e-3; single rows, whose few
  elements may cancel, 2e-2.  fp32: scores of size up to ~30 carry 30 * 2^-24
  of relative error into the weights: rel-L2 <= 5e-6.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402

DEV = torch.device("cuda")


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rel_l2(a, b):
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-30))


def tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def rand(shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (std * torch.randn(*shape, generator=g, device=DEV)).to(tdt(dtype))


# --------------------------------------------------------------- attention
def make_cache(dtype, hk, hd, ps, lens, shared, layers=1, seed=3, max_pages=None, dead=float("nan")):
    """A cache with scattered pages; rows no sequence has reached hold ``dead``."""
    rng = np.random.default_rng(seed)
    n_sh = shared // ps
    need = [max(0, -(-l // ps) - n_sh) for l in lens]
    max_pages = max_pages or max(1, n_sh + max(need))
    n_pages = n_sh + sum(need) + 2
    perm = rng.permutation(n_pages)
    table = np.full((len(lens), max_pages), -1, np.int32)
    ref = np.zeros(n_pages, np.int32)
    at = n_sh
    for b, l in enumerate(lens):
        mine = min(n_sh, -(-l // ps))
        table[b, :mine] = perm[:mine]
        table[b, n_sh:n_sh + need[b]] = perm[at:at + need[b]]
        at += need[b]
        ref[table[b][table[b] >= 0]] += 1
    k = rand((layers, n_pages, ps, hk * hd), dtype, seed)
    v = rand((layers, n_pages, ps, hk * hd), dtype, seed + 1)
    reached = np.zeros((n_pages, ps), bool)
    for b, l in enumerate(lens):
        j = np.arange(l)
        reached[table[b, j // ps], j % ps] = True
    gone = torch.from_numpy(~reached).to(DEV)[None, :, :, None]
    k.masked_fill_(gone, dead)
    v.masked_fill_(gone, dead)
    return xb.KVCache(dtype, hk, hd, k, v, i32(ref), i32(table), i32(lens))


def ref_attention(cache, layer, seqs, n_q, q, causal, scale=None):
    hd, hk, ps = cache.head_dim, cache.n_kv_heads, cache.page_size
    k, v = host(cache.k[layer]), host(cache.v[layer])
    table, lens = cache.table.cpu().numpy(), cache.len.cpu().numpy()
    B = len(seqs)
    q = host(q).reshape(B, n_q, -1, hd)
    H = q.shape[2]
    out = np.zeros_like(q)
    for b, s in enumerate(seqs):
        j = np.arange(lens[s])
        kk = k[table[s, j // ps], j % ps].reshape(-1, hk, hd)
        vv = v[table[s, j // ps], j % ps].reshape(-1, hk, hd)
        for i in range(n_q):
            lim = lens[s] - n_q + i + 1 if causal else lens[s]
            if lim <= 0:
                continue
            for h in range(H):
                x = kk[:lim, h // (H // hk)] @ q[b, i, h] * (scale or 1 / math.sqrt(hd))
                p = np.exp(x - x.max())
                out[b, i, h] = p @ vv[:lim, h // (H // hk)] / p.sum()
    return out.reshape(B * n_q, H * hd)


def check_attention(dtype, H, hk, hd, ps, lens, n_q, shared, causal, seqs=None, scale=0.0, seed=3, std=1.5,
                    max_pages=None, poison=True):
    cache = make_cache(dtype, hk, hd, ps, lens, shared, seed=seed, max_pages=max_pages)
    seqs = list(range(len(lens))) if seqs is None else seqs
    q = rand((len(seqs) * n_q, H * hd), dtype, seed + 7, std)
    o = torch.full_like(q, float("nan"))
    need = xb.op_branch_attention_workspace_bytes(cache, len(seqs), n_q, H, shared)
    ws = torch.full((need // 4,), float("nan"), device=DEV) if poison else None   # its contents do not matter
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, o, shared_len=shared, causal=causal, scale=scale, workspace=ws)
    torch.cuda.synchronize()
    assert xb.op_device_error() == 0
    got, want = host(o), ref_attention(cache, 0, seqs, n_q, q, causal, scale or None)
    assert np.isfinite(got).all()
    assert rel_l2(got, want) <= (5e-3 if dtype == "bf16" else 5e-6), rel_l2(got, want)
    rows = got.reshape(-1, hd), want.reshape(-1, hd)
    norm = np.linalg.norm(rows[1], axis=1)
    err = np.linalg.norm(rows[0] - rows[1], axis=1)
    assert (err <= (2e-2 if dtype == "bf16" else 2e-5) * norm).all(), float(np.max(err / np.maximum(norm, 1e-30)))
    return cache, q, o


TOKEN_CASES = [
    # H, hk, hd, page, lens, shared
    (1, 1, 64, 16, [1], 0),
    (4, 4, 64, 16, [33, 16, 17, 20], 16),                # empty and one-key own parts
    (8, 8, 64, 16, [2017, 2030, 2056, 2016], 2016),
    (8, 1, 128, 32, [130, 129, 128, 700, 64], 64),
    (5, 1, 128, 64, [64, 1000, 65], 64),
    (21, 3, 128, 128, [300, 511, 129, 128, 2000, 131, 140], 128),
    (40, 8, 128, 32, [4000 + 37 * b for b in range(32)], 3968),
    (32, 4, 64, 256, [256 + b for b in range(9)], 256),  # pages larger than a key tile
    (12, 12, 128, 16, [0, 5, 0, 129], 0),                # sequences without a key
    (64, 1, 64, 16, [700, 900], 640),
    (128, 1, 128, 16, [200, 220, 240], 192),             # a whole tile per token
    (2, 2, 64, 1024, [3000, 2050], 2048),
    (2, 2, 64, 16, [64 + (37 * b) % 90 for b in range(130)], 64),   # more branches than lengths in shared memory
    (1, 1, 128, 64, [19968 + 5 * b for b in range(3)], 19968),      # one head: a row in as many pieces as CTAs
]


@pytest.mark.parametrize("H,hk,hd,ps,lens,shared", TOKEN_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_single_tokens(H, hk, hd, ps, lens, shared, causal):
    check_attention("bf16", H, hk, hd, ps, lens, 1, shared, causal)


MULTI_CASES = [
    # H, hk, hd, page, lens, n_q, shared
    (4, 4, 64, 16, [200, 33, 100], 20, 0),
    (12, 12, 128, 32, [352, 340, 400, 321], 20, 320),
    (6, 2, 128, 128, [300, 259, 1000], 259, 0),          # prompts; the second is all new
    (6, 2, 64, 32, [300, 259, 1000], 130, 256),          # queries reach into the shared part
    (7, 1, 128, 16, [90, 60, 75], 37, 48),
    (3, 3, 64, 16, [10, 40, 0], 25, 0),                  # causal: rows before the first key are empty
    (8, 8, 64, 64, [64 + 513] * 2, 513, 64),             # two full row tiles and a row
    (4, 4, 128, 64, [1000, 1000], 257, 0),
    (10, 2, 128, 32, [96 + 24] * 16, 24, 96),
    (4, 4, 128, 128, [128 * 5, 128 * 6], 128, 512),
    (100, 1, 64, 16, [70, 90], 5, 64),                   # 100 query heads of one key head
    (2, 2, 128, 16, [100 + (13 * b) % 61 for b in range(70)], 3, 0),
    (1, 1, 64, 32, [160 + b % 30 for b in range(40)], 20, 128),      # packed rows fill several row tiles
    # several whole units per CTA, each begun at another key tile: causal rows meet their first visible key late
    (10, 10, 64, 16, [210 + (31 * b) % 400 for b in range(40)], 40, 0),
    (9, 9, 128, 64, [150 + (53 * b) % 700 for b in range(24)], 130, 0),
]


@pytest.mark.parametrize("H,hk,hd,ps,lens,n_q,shared", MULTI_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_several_tokens(H, hk, hd, ps, lens, n_q, shared, causal):
    check_attention("bf16", H, hk, hd, ps, lens, n_q, shared, causal)


@pytest.mark.parametrize("H,hk,hd,ps,lens,n_q,shared", [
    # long shared parts: prefix units of two row tiles
    (2, 2, 128, 32, [2760, 2700], 128, 2560),
    (4, 2, 64, 16, [2760, 2700, 2690, 2800], 64, 2560),
    (40, 8, 128, 128, [16384 + (61 * b) % 300 for b in range(32)], 1, 16384),
    # packed rows just past whole pairs of row tiles
    (3, 3, 128, 16, [1040 + 40 * b for b in range(5)], 65, 960),
    (8, 1, 64, 32, [320 + 7 * b for b in range(33)], 1, 320),
])
@pytest.mark.parametrize("causal", [True, False])
def test_one_or_two_row_tiles(H, hk, hd, ps, lens, n_q, shared, causal):
    check_attention("bf16", H, hk, hd, ps, lens, n_q, shared, causal)


@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,shared", [
    # entries of few rows, merged by small CTAs: many of them; few with few pieces a row
    ("bf16", 16, 8, 64, 16, [256 + (29 * b) % 90 for b in range(90)], 256),
    ("bf16", 32, 8, 128, 16, [256 + (29 * b) % 90 for b in range(70)], 256),
    ("bf16", 16, 16, 128, 64, [2048 + 17 * b for b in range(4)], 2048),
    ("bf16", 3, 3, 128, 64, [4096 + 17 * b for b in range(4)], 4096),      # many pieces a row
    ("f32", 8, 8, 16, 16, [256 + (29 * b) % 90 for b in range(90)], 256),
    ("f32", 24, 8, 128, 16, [256 + (29 * b) % 90 for b in range(70)], 256),
])
def test_merge_of_short_entries(dtype, H, hk, hd, ps, lens, shared):
    check_attention(dtype, H, hk, hd, ps, lens, 1, shared, True)


F32_CASES = [
    (4, 4, 16, 16, [464 + 232] * 2, 58, 464), (4, 2, 32, 16, [50, 1, 0, 33], 1, 0), (6, 1, 64, 32, [200, 130], 70, 96),
    (8, 8, 128, 64, [64, 65, 400], 3, 64), (64, 1, 16, 16, [40, 50], 2, 32), (3, 3, 64, 16, [10, 40, 0], 25, 0),
]


@pytest.mark.parametrize("H,hk,hd,ps,lens,n_q,shared", F32_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_float32(H, hk, hd, ps, lens, n_q, shared, causal):
    check_attention("f32", H, hk, hd, ps, lens, n_q, shared, causal)


@pytest.mark.parametrize("H,hk,hd,lens,n_q,shared", [
    (8, 8, 16, [1344, 1501], 300, 1024),          # two CTAs an SM, prefix units
    (16, 8, 32, [1040, 903, 700], 211, 0),        # whole and cut units
    (8, 4, 64, [2500, 2307], 257, 2048),
    (8, 8, 128, [1344, 1501], 300, 1024),
])
def test_float32_long_calls(H, hk, hd, lens, n_q, shared):
    check_attention("f32", H, hk, hd, 16, lens, n_q, shared, True)


def test_float32_flags_a_bad_page_and_reads_on():
    cache = make_cache("f32", 2, 32, 16, [100, 90], 0, dead=0.0)
    q = rand((2, 4 * 32), "f32", 4)
    o = torch.empty_like(q)
    cache.table[1, 2] = 1 << 20
    xb.op_branch_attention(cache, 0, i32([0, 1]), 1, q, o)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    assert torch.isfinite(o).all()


def test_more_key_tiles_than_ctas_and_long_tables():
    """Lines of many key tiles per CTA, cut inside units, with a table row longer than its sequence."""
    check_attention("bf16", 2, 2, 128, 16, [9000, 5000, 7001], 300, 0, True, max_pages=1000)
    check_attention("bf16", 4, 2, 64, 16, [20000 + 30 * b for b in range(6)], 2, 20000, True)


def test_peaked_scores_move_the_running_maximum():
    """Scores that grow along the keys by far more than the lazy-rescale step."""
    for dtype, hd in (("bf16", 128), ("bf16", 64), ("f32", 64)):
        cache = make_cache(dtype, 1, hd, 16, [1500, 1400], 1280)
        ramp = torch.linspace(0.0, 4.0, 1500, device=DEV)
        table, lens = cache.table.cpu().numpy(), [1500, 1400]
        for s in range(2):
            j = np.arange(lens[s])
            cache.k[0, table[s, j // 16].tolist(), (j % 16).tolist()] *= ramp[:lens[s], None].to(cache.k.dtype)
        q = rand((2, 2 * hd), dtype, 5, 6.0)
        o = torch.empty_like(q)
        xb.op_branch_attention(cache, 0, i32([0, 1]), 1, q, o, shared_len=1280, causal=True)
        want = ref_attention(cache, 0, [0, 1], 1, q, True)
        assert rel_l2(host(o), want) <= (5e-3 if dtype == "bf16" else 2e-5)


def test_order_of_branches_repeats_and_scale():
    cache, q, o = check_attention("bf16", 8, 2, 64, 16, [90, 120, 77, 64], 3, 64, True, seqs=[3, 1, 1, 0, 2],
                                  scale=0.05)
    again = torch.empty_like(o)
    xb.op_branch_attention(cache, 0, i32([3, 1, 1, 0, 2]), 3, q, again, shared_len=64, causal=True, scale=0.05)
    assert torch.equal(o, again)                          # the same bits on every run


def test_shared_len_does_not_change_what_a_row_sees():
    cache = make_cache("bf16", 4, 128, 32, [400, 416, 333, 321], 320)
    q = rand((4 * 7, 8 * 128), "bf16", 9)
    outs = []
    for shared in (0, 32, 320):
        o = torch.empty_like(q)
        xb.op_branch_attention(cache, 0, i32([0, 1, 2, 3]), 7, q, o, shared_len=shared, causal=True)
        outs.append(host(o))
    want = ref_attention(cache, 0, [0, 1, 2, 3], 7, q, True)
    for o in outs:
        assert rel_l2(o, want) <= 5e-3


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 32)])
def test_strided_rows_and_layers(dtype, hd):
    """q a column block of a wider buffer, o rows apart, layer 1 of 2, on another stream."""
    hk, H, n_q, lens = 2, 4, 5, [70, 99]
    cache = make_cache(dtype, hk, hd, 16, lens, 48, layers=2)
    wide = rand((2 * n_q, 3 * H * hd), dtype, 4)
    q = wide[:, H * hd:2 * H * hd]
    buf = torch.full((2 * n_q, H * hd + 16), 7.0, device=DEV, dtype=tdt(dtype))
    o = buf[:, 8:8 + H * hd]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    xb.op_branch_attention(cache, 1, i32([0, 1]), n_q, q, o, shared_len=48, causal=True, stream=st)
    st.synchronize()
    want = ref_attention(cache, 1, [0, 1], n_q, q.contiguous(), True)
    assert rel_l2(host(o), want) <= (5e-3 if dtype == "bf16" else 5e-6)
    assert (buf[:, :8] == 7.0).all() and (buf[:, 8 + H * hd:] == 7.0).all()
    assert xb.op_device_error() == 0


def test_attention_flags_what_the_host_cannot_see():
    cache = make_cache("bf16", 2, 64, 16, [40, 50], 32, dead=0.0)
    q = rand((2, 128), "bf16", 4)
    o = torch.empty_like(q)
    xb.op_branch_attention(cache, 0, i32([0, 2]), 1, q, o)                     # no such sequence
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    assert (o[1] == 0).all() and torch.isfinite(o[0].float()).all()
    cache.table[1, 3] = 1 << 20                                               # a page id out of range
    xb.op_branch_attention(cache, 0, i32([0, 1]), 1, q, o)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    cache.table[1, 3] = -5
    xb.op_branch_attention(cache, 0, i32([0, 1]), 1, q, o)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    cache.len[1] = 16                                                         # shorter than the shared part
    xb.op_branch_attention(cache, 0, i32([0, 1]), 1, q, o, shared_len=32)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    assert xb.op_device_error() == 0


def test_host_tensors_are_refused():
    """A host address never reaches a kernel: every operand of every call is refused before the launch."""
    cache = make_cache("bf16", 2, 64, 16, [40, 50], 32, dead=0.0)
    q, seqs = rand((2, 128), "bf16", 4), i32([0, 1])
    o = torch.empty_like(q)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    args = [seqs, q, o, ws]
    for i in range(4):
        a = [x.cpu() if j == i else x for j, x in enumerate(args)]
        with pytest.raises(ValueError):
            xb.op_branch_attention(cache, 0, a[0], 1, a[1], a[2], workspace=a[3])
    for call in (lambda: xb.op_kv_fork(cache, seqs.cpu(), seqs), lambda: xb.op_kv_fork(cache, seqs, seqs.cpu()),
                 lambda: xb.op_kv_extend(cache, seqs, 1, i32([0, 0]).cpu()), lambda: xb.op_kv_free(cache, seqs.cpu()),
                 lambda: xb.op_kv_compact(cache, i32([0]).cpu()),
                 lambda: xb.op_rope_table([32], [64], 1e4, torch.empty(2 * 32 * 64))):
        with pytest.raises(ValueError):
            call()
    gamma, table = torch.ones(64, device=DEV), torch.empty(2 * 32 * 64, device=DEV)
    args = [q, q, q, gamma, gamma, seqs, table, seqs, o]
    for i in range(9):
        a = [x.cpu() if j == i else x for j, x in enumerate(args)]
        with pytest.raises(ValueError):
            xb.op_qk_norm_rope(cache, 0, *a[:6], [32], [64], *a[6:])
    assert xb.op_device_error() == 0


def test_one_workspace_for_calls_in_turn():
    """Two shapes through one workspace, back to back and again: nothing is kept between calls."""
    a = make_cache("bf16", 2, 64, 16, [300, 310, 290], 256)
    b = make_cache("bf16", 4, 128, 32, [700, 500], 0, seed=9)
    qa, qb = rand((3, 8 * 64), "bf16", 1), rand((2 * 90, 4 * 128), "bf16", 2)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    outs = []
    for _ in range(3):
        oa, ob = torch.empty_like(qa), torch.empty_like(qb)
        xb.op_branch_attention(a, 0, i32([0, 1, 2]), 1, qa, oa, shared_len=256, causal=True, workspace=ws)
        xb.op_branch_attention(b, 0, i32([0, 1]), 90, qb, ob, causal=True, workspace=ws)
        outs.append((oa, ob))
    for oa, ob in outs[1:]:
        assert torch.equal(oa, outs[0][0]) and torch.equal(ob, outs[0][1])
    assert rel_l2(host(outs[0][0]), ref_attention(a, 0, [0, 1, 2], 1, qa, True)) <= 5e-3
    assert rel_l2(host(outs[0][1]), ref_attention(b, 0, [0, 1], 90, qb, True)) <= 5e-3


def test_replayed_in_a_graph_with_new_lengths():
    """A captured planning step (extend, attend) follows the lengths on the device."""
    cache = make_cache("bf16", 2, 64, 16, [100, 130], 96, max_pages=20, dead=0.0)
    free = xb.KVCache("bf16", 2, 64, torch.cat([cache.k, cache.k], 1), torch.cat([cache.v, cache.v], 1),
                      torch.cat([cache.ref, torch.zeros_like(cache.ref)]), cache.table, cache.len)
    q, seqs, slots = rand((2, 4 * 64), "bf16", 3), i32([0, 1]), torch.empty(2, 1, dtype=torch.int32, device=DEV)
    o = torch.empty_like(q)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):                           # workspaces and one-time set-up before the capture
        xb.op_kv_extend(free, seqs, 1, slots)
        xb.op_branch_attention(free, 0, seqs, 1, q, o, shared_len=96, causal=True)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        xb.op_kv_extend(free, seqs, 1, slots)
        xb.op_branch_attention(free, 0, seqs, 1, q, o, shared_len=96, causal=True)
    for n in range(1, 30, 7):
        while free.len[0].item() < 101 + n:
            graph.replay()
        torch.cuda.synchronize()
        assert free.len.tolist() == [101 + n, 131 + n]
        assert rel_l2(host(o), ref_attention(free, 0, [0, 1], 1, q, True)) <= 5e-3
    assert xb.op_device_error() == 0


# ------------------------------------------------------- norm and rotation
def ref_rotate(x, heads, hd, gamma, pos, pairs, theta, half, eps):
    x = x.reshape(x.shape[0], heads, hd)
    x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gamma
    axis = np.repeat(np.arange(len(pairs)), pairs)
    j = np.concatenate([np.arange(p) for p in pairs])
    ang = pos[:, axis] * theta ** (-j / np.array(pairs)[axis])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = (x[..., :hd // 2], x[..., hd // 2:]) if half else (x[..., 0::2], x[..., 1::2])
    y = np.empty_like(x)
    if half:
        y[..., :hd // 2], y[..., hd // 2:] = a * c - b * s, a * s + b * c
    else:
        y[..., 0::2], y[..., 1::2] = a * c - b * s, a * s + b * c
    return y.reshape(x.shape[0], heads * hd)


NORM_CASES = [
    # dtype, H, hk, hd, T, pairs, n_pos
    ("bf16", 40, 8, 64, 77, [32], [500]), ("bf16", 3, 3, 128, 1, [8, 24, 16, 16], [6, 30, 20, 36]),
    ("bf16", 12, 4, 128, 130, [20, 44], [9, 1000]), ("bf16", 2, 1, 16, 5, [8], [64]), ("bf16", 5, 5, 32, 33, [1, 15], [7, 8]),
    ("f32", 4, 4, 16, 64, [1, 3, 2, 2], [2, 8, 4, 4]), ("f32", 8, 2, 32, 9, [16], [100]), ("f32", 6, 3, 64, 50, [32], [99]),
    ("f32", 7, 1, 128, 21, [30, 34], [3, 70]),
]


@pytest.mark.parametrize("dtype,H,hk,hd,T,pairs,n_pos", NORM_CASES)
@pytest.mark.parametrize("half", [False, True])
def test_norm_rotation_and_page_write(dtype, H, hk, hd, T, pairs, n_pos, half):
    rng = np.random.default_rng(5)
    theta, eps, ps = 10000.0, 1e-5, 16
    n_pages = T // ps + 3
    cache = xb.KVCache.empty(dtype, 2, n_pages, ps, hk, hd, 1, n_pages)
    cache.k.fill_(3.0)
    cache.v.fill_(4.0)
    q = rand((T, H * hd), dtype, 1, 2.0)
    kv = rand((T, 2 * hk * hd), dtype, 2, 0.3)            # fused: strided k and v
    k, v = kv[:, :hk * hd], kv[:, hk * hd:]
    gq, gk = rand((hd,), "f32", 3), rand((hd,), "f32", 4)
    pos = np.stack([rng.integers(0, n, T) for n in n_pos], 1)
    pos[0] = np.array(n_pos) - 1
    slots = rng.permutation(n_pages * ps)[:T].astype(np.int32)
    if T > 3:
        slots[[1, T - 1]] = -1
    table = torch.empty(2 * sum(a * b for a, b in zip(pairs, n_pos)), device=DEV)
    xb.op_rope_table(pairs, n_pos, theta, table)
    wide = torch.full((T, H * hd + 8), 9.0, device=DEV, dtype=tdt(dtype))
    out = wide[:, :H * hd]
    xb.op_qk_norm_rope(cache, 1, q, k, v, gq, gk, i32(pos), pairs, n_pos, table, i32(slots), out, eps=eps,
                       half_split=half)
    assert xb.op_device_error() == 0
    tol = 2.3e-3 if dtype == "bf16" else 1e-6
    assert rel_l2(host(out), ref_rotate(host(q), H, hd, host(gq), pos, pairs, theta, half, eps)) <= tol
    assert (wide[:, H * hd:] == 9.0).all()
    keep = slots >= 0
    want_k = np.full((n_pages * ps, hk * hd), 3.0)
    want_v = np.full((n_pages * ps, hk * hd), 4.0)
    want_k[slots[keep]] = ref_rotate(host(k), hk, hd, host(gk), pos, pairs, theta, half, eps)[keep]
    want_v[slots[keep]] = host(v)[keep]
    got_k, got_v = host(cache.k[1]).reshape(want_k.shape), host(cache.v[1]).reshape(want_v.shape)
    idle = np.ones(n_pages * ps, bool)
    idle[slots[keep]] = False
    assert (got_k[idle] == 3.0).all() and (host(cache.k[0]) == 3.0).all() and (host(cache.v[0]) == 4.0).all()
    assert rel_l2(got_k[~idle], want_k[~idle]) <= tol
    np.testing.assert_array_equal(got_v, want_v)
    # in place gives the same bits
    before = out.clone()
    xb.op_qk_norm_rope(cache, 1, q, k, v, gq, gk, i32(pos), pairs, n_pos, table, i32(slots), q, eps=eps,
                       half_split=half)
    assert torch.equal(q, before)


def test_norm_of_zero_rows_and_bad_positions():
    cache = xb.KVCache.empty("bf16", 1, 2, 16, 1, 64, 1, 2)
    cache.k.zero_()
    cache.v.zero_()
    q, k, v = (torch.zeros(4, 64, device=DEV, dtype=torch.bfloat16) for _ in range(3))
    v += 1
    g = torch.ones(64, device=DEV)
    table = torch.empty(2 * 32 * 10, device=DEV)
    xb.op_rope_table([32], [10], 1e4, table)
    out = torch.full_like(q, 5.0)
    xb.op_qk_norm_rope(cache, 0, q, k, v, g, g, i32([[0], [10], [-1], [9]]), [32], [10], table, i32([0, 1, 2, 32]), out)
    assert xb.op_device_error() == xb.XC_DEV_BAD_POSITION
    assert (out[0] == 0).all() and (out[1:] == 5.0).all()              # bad tokens are skipped whole
    assert (cache.v[0, 0, 0] == 1).all() and (cache.v[0, 0, 1:] == 0).all() and (cache.v[0, 1] == 0).all()


# ------------------------------------------------------------------- pages
class PageModel:
    """The page operations on host lists."""

    def __init__(self, n_pages, ps, max_seqs, max_pages, data):
        self.ps, self.max_pages, self.data = ps, max_pages, data      # data [n_pages, ps]: one value per cache row
        self.ref, self.rows, self.len = [0] * n_pages, [[] for _ in range(max_seqs)], [0] * max_seqs

    def free_ids(self):
        return [p for p, r in enumerate(self.ref) if r == 0]

    def fork(self, pairs):
        ids = self.free_ids()
        if sum(self.len[s] % self.ps != 0 for s, _ in pairs) > len(ids):
            return False
        for s, d in pairs:
            n, part = divmod(self.len[s], self.ps)
            self.rows[d] = self.rows[s][:n]
            for p in self.rows[d]:
                self.ref[p] += 1
            if part:
                p = ids.pop(0)
                self.data[p, :part] = self.data[self.rows[s][n], :part]
                self.ref[p] = 1
                self.rows[d] = self.rows[d] + [p]
            self.len[d] = self.len[s]
        return True

    def extend(self, seqs, n):
        ids = self.free_ids()
        need = [-(-(self.len[s] + n) // self.ps) - len(self.rows[s]) for s in seqs]
        if sum(need) > len(ids) or any(self.len[s] + n > self.max_pages * self.ps for s in seqs):
            return None
        slots = []
        for s, k in zip(seqs, need):
            for _ in range(k):
                self.rows[s].append(ids.pop(0))
                self.ref[self.rows[s][-1]] = 1
            at = range(self.len[s], self.len[s] + n)
            slots.append([self.rows[s][j // self.ps] * self.ps + j % self.ps for j in at])
            self.len[s] += n
        return slots

    def free(self, seqs):
        for s in seqs:
            for p in self.rows[s]:
                self.ref[p] -= 1
            self.rows[s], self.len[s] = [], 0

    def compact(self):
        used = [p for p, r in enumerate(self.ref) if r > 0]
        n = len(used)
        new = dict(zip([p for p in used if p >= n], [p for p in range(n) if self.ref[p] == 0]))
        for a, b in new.items():
            self.data[b] = self.data[a]
            self.ref[b], self.ref[a] = self.ref[a], 0
        self.rows = [[new.get(p, p) for p in r] for r in self.rows]
        return n

    def check(self, cache, rows):
        assert cache.ref.tolist() == self.ref
        assert cache.len.tolist() == self.len
        for s, r in enumerate(self.rows):
            assert cache.table[s].tolist() == r + [-1] * (self.max_pages - len(r))
        got_k, got_v = host(cache.k), host(cache.v)
        for layer in range(got_k.shape[0]):
            np.testing.assert_array_equal(got_k[layer], rows(layer, 0)[self.data])
            np.testing.assert_array_equal(got_v[layer], rows(layer, 1)[self.data])


@pytest.mark.parametrize("dtype,ps,n_pages,max_seqs,max_pages,layers,hk,hd", [
    ("bf16", 16, 40, 6, 12, 2, 1, 16), ("f32", 32, 23, 9, 7, 3, 3, 32), ("bf16", 64, 9000, 1100, 8, 1, 1, 16)])
def test_page_operations_follow_the_model(dtype, ps, n_pages, max_seqs, max_pages, layers, hk, hd):
    rng = np.random.default_rng(11)
    cache = xb.KVCache.empty(dtype, layers, n_pages, ps, hk, hd, max_seqs, max_pages)
    n_rows = n_pages * ps
    cache.k.copy_(rand(tuple(cache.k.shape), dtype, 1))
    cache.v.copy_(rand(tuple(cache.v.shape), dtype, 2))
    first = [[host(t[layer]).reshape(n_rows, -1) for t in (cache.k, cache.v)] for layer in range(layers)]
    m = PageModel(n_pages, ps, max_seqs, max_pages, np.arange(n_rows).reshape(n_pages, ps))
    many = max_seqs > 1000
    for step in range(8 if many else 60):
        empty = [s for s in range(max_seqs) if m.len[s] == 0]
        full = [s for s in range(max_seqs) if m.len[s] > 0]
        op = ["extend", "fork", "free", "compact"][rng.integers(4)] if step > 1 else "extend"
        if op == "extend":
            n_new = int(rng.integers(1, 2 * ps + 2))
            pick = rng.permutation(max_seqs)[:rng.integers(1, (1025 if many else 4))].tolist()
            slots = torch.full((len(pick), n_new), 77, dtype=torch.int32, device=DEV)
            xb.op_kv_extend(cache, i32(pick), n_new, slots)
            want = m.extend(pick, n_new)
            assert xb.op_device_error() == (0 if want is not None else xb.XC_DEV_CACHE_FULL)
            assert slots.tolist() == (want if want is not None else [[-1] * n_new] * len(pick))
        elif op == "fork" and empty and full:
            d = rng.permutation(empty)[:rng.integers(1, 4)].tolist()
            pairs = [(int(rng.choice(full)), x) for x in d]
            xb.op_kv_fork(cache, i32([p[0] for p in pairs]), i32([p[1] for p in pairs]))
            assert xb.op_device_error() == (0 if m.fork(pairs) else xb.XC_DEV_CACHE_FULL)
        elif op == "free" and full:
            pick = rng.permutation(full)[:rng.integers(1, 3)].tolist()
            xb.op_kv_free(cache, i32(pick))
            m.free(pick)
        elif op == "compact":
            live = i32([0])
            xb.op_kv_compact(cache, live)
            assert live.item() == m.compact()
        if not many or step == 7:
            m.check(cache, lambda layer, x: first[layer][x])
    assert xb.op_device_error() == 0


def test_page_calls_change_nothing_on_bad_input():
    cache = xb.KVCache.empty("bf16", 1, 8, 16, 1, 16, 4, 4)
    slots = i32([[0] * 20])
    xb.op_kv_extend(cache, i32([0]), 20, slots)
    assert xb.op_device_error() == 0 and slots[0].tolist() == list(range(20))
    state = [t.clone() for t in (cache.ref, cache.table, cache.len)]

    def same(code):
        assert xb.op_device_error() == code
        for a, b in zip(state, (cache.ref, cache.table, cache.len)):
            assert torch.equal(a, b)

    two = i32([[0] * 8] * 2)
    xb.op_kv_fork(cache, i32([0, 0]), i32([1, 1]))              # a destination twice
    same(xb.XC_DEV_BAD_SEQUENCE)
    xb.op_kv_fork(cache, i32([0]), i32([0]))                    # into itself
    same(xb.XC_DEV_BAD_SEQUENCE)
    xb.op_kv_fork(cache, i32([0, 1]), i32([1, 2]))              # a source that is a destination
    same(xb.XC_DEV_BAD_SEQUENCE)
    xb.op_kv_fork(cache, i32([4]), i32([1]))                    # no such sequence
    same(xb.XC_DEV_BAD_SEQUENCE)
    xb.op_kv_extend(cache, i32([2, 2]), 8, two)                 # a sequence twice
    same(xb.XC_DEV_BAD_SEQUENCE)
    xb.op_kv_extend(cache, i32([-1, 2]), 8, two)
    same(xb.XC_DEV_BAD_SEQUENCE)
    assert (two == -1).all()
    xb.op_kv_extend(cache, i32([0]), 45, i32([[0] * 45]))       # past the table row
    same(xb.XC_DEV_CACHE_FULL)
    xb.op_kv_extend(cache, i32([1, 2]), 49, i32([[0] * 49] * 2))   # 8 pages of 6
    same(xb.XC_DEV_CACHE_FULL)
    cache.ref[1] = 2                                            # a shared last page is never appended to
    xb.op_kv_extend(cache, i32([0]), 1, i32([[0]]))
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    cache.ref[1] = 1
    xb.op_kv_free(cache, i32([0, 0, 3]))                        # listed twice: released once
    assert xb.op_device_error() == 0 and cache.ref.sum().item() == 0 and cache.len.sum().item() == 0
    xb.op_kv_free(cache, i32([9]))
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE


def test_free_skips_a_bad_id_and_empties_the_others():
    cache = xb.KVCache.empty("bf16", 1, 8, 16, 1, 16, 4, 4)
    xb.op_kv_extend(cache, i32([0, 2]), 20, i32([[0] * 20] * 2))
    xb.op_kv_free(cache, i32([9, 0, -1]))
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    assert cache.len.tolist() == [0, 0, 20, 0] and cache.ref.sum().item() == 2


@pytest.mark.parametrize("n,n_new", [(1, 5000), (3, 1700), (700, 17), (1024, 1)])
def test_extend_many_tokens_or_sequences(n, n_new):
    ps, rows = 16, -(-n_new // 16) + 1
    cache = xb.KVCache.empty("bf16", 1, n * rows, ps, 1, 16, n, rows)
    order = np.random.default_rng(3).permutation(n).tolist()
    m = PageModel(n * rows, ps, n, rows, np.zeros((1, 1)))
    for step in (n_new, 3):
        slots = torch.empty(n, step, dtype=torch.int32, device=DEV)
        xb.op_kv_extend(cache, i32(order), step, slots)
        assert xb.op_device_error() == 0
        assert slots.tolist() == m.extend(order, step)
    assert cache.ref.tolist() == m.ref and cache.len.tolist() == m.len


def test_offsets_past_32_bits():
    """A pool whose element offsets pass 2^31: pages at both ends, copied, filled and read."""
    ps, hk, hd, n_pages = 64, 8, 128, 40000                     # 2.6e9 elements, 5.2 GB each
    free = torch.cuda.mem_get_info()[0]
    if free < 16 << 30:
        pytest.skip("needs 16 GB")
    cache = xb.KVCache.empty("bf16", 1, n_pages, ps, hk, hd, 3, 4)
    last = n_pages - 1
    cache.k[0, last] = rand((ps, hk * hd), "bf16", 1)
    cache.v[0, last] = rand((ps, hk * hd), "bf16", 2)
    cache.k[0, 0].zero_()
    cache.v[0, 0].zero_()
    cache.ref[last] = 1
    cache.table[0, 0] = last
    cache.len[0] = 41
    q = rand((1, hk * hd), "bf16", 3)
    o = torch.empty_like(q)
    xb.op_branch_attention(cache, 0, i32([0]), 1, q, o)
    far = host(o)
    kk, vv = host(cache.k[0, last, :41]).reshape(41, hk, hd), host(cache.v[0, last, :41]).reshape(41, hk, hd)
    w = np.einsum("hd,jhd->hj", host(q).reshape(hk, hd), kk) / math.sqrt(hd)
    w = np.exp(w - w.max(1, keepdims=True))
    assert rel_l2(far, (np.einsum("hj,jhd->hd", w, vv) / w.sum(1)[:, None]).reshape(1, -1)) <= 5e-3
    live = i32([0])
    xb.op_kv_compact(cache, live)                               # page 39999 -> page 0
    assert live.item() == 1 and cache.table[0].tolist() == [0, -1, -1, -1]
    assert torch.equal(cache.k[0, 0], cache.k[0, last]) and torch.equal(cache.v[0, 0], cache.v[0, last])
    g = torch.ones(hd, device=DEV)
    table = torch.empty(2 * 64, device=DEV)
    xb.op_rope_table([64], [1], 1e4, table)
    x = rand((1, hk * hd), "bf16", 5)
    xb.op_qk_norm_rope(cache, 0, x, x, x, g, g, i32([[0]]), [64], [1], table, i32([last * ps + 63]), torch.empty_like(x))
    assert torch.equal(cache.v[0, last, 63], x[0])
    assert xb.op_device_error() == 0


# ---------------------------------------------------------------- together
def plain_layers(weights, H, hk, hd, x, eps=1e-6, theta=1e4):
    """The causal layers of one whole sequence x [n, d], in 64 bits."""
    n = x.shape[0]
    for w in weights:
        h = (x - x.mean(1, keepdims=True)) / np.sqrt(x.var(1, keepdims=True) + eps)
        qkv = h @ host(w["qkv_w"]).T + host(w["qkv_b"])
        pos = np.arange(n)[:, None]
        q = ref_rotate(qkv[:, :H * hd], H, hd, host(w["gamma_q"]), pos, [hd // 2], theta, False, eps).reshape(n, H, hd)
        k = ref_rotate(qkv[:, H * hd:(H + hk) * hd], hk, hd, host(w["gamma_k"]), pos, [hd // 2], theta, False,
                       eps).reshape(n, hk, hd).repeat(H // hk, axis=1)
        v = qkv[:, (H + hk) * hd:].reshape(n, hk, hd).repeat(H // hk, axis=1)
        s = np.einsum("ihd,jhd->hij", q, k) / math.sqrt(hd)
        s[:, np.triu(np.ones((n, n), bool), 1)] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        o = np.einsum("hij,jhd->ihd", p / p.sum(-1, keepdims=True), v).reshape(n, H * hd)
        x = x + o @ host(w["o_w"]).T + host(w["o_b"])
    return x


@pytest.mark.parametrize("dtype,H,hk,hd,tol", [("f32", 4, 2, 32, 2e-5), ("bf16", 8, 4, 64, 2e-2)])
def test_branched_layers_match_whole_sequences(dtype, H, hk, hd, tol):
    """History once, forked, branches advanced together, freed, compacted, forked
    again: every output equals the layers run on that branch's whole sequence.
    fp32: a few 1e-6 per layer; bf16: some ten roundings of 2^-9 per layer."""
    from paper_2604_20289_gb300.branches import BranchedLayers, random_layers
    d = 256
    weights = random_layers(2, d, H, hk, hd, dtype, seed=4)
    m = BranchedLayers(weights, H, hk, hd, n_pages=40, page_size=16, max_seqs=8, max_len=160, dtype=dtype)
    rng = np.random.default_rng(2)
    text = {}                                             # tokens of every sequence

    def step(seqs, n):
        x = torch.from_numpy(rng.standard_normal((len(seqs), n, d))).to(DEV).to(tdt(dtype))
        for i, s in enumerate(seqs):
            text[s] = np.concatenate([text[s], host(x[i])])
        y = host(m.step(seqs, x))
        assert xb.op_device_error() == 0
        for i, s in enumerate(seqs):
            want = plain_layers(weights, H, hk, hd, text[s])[-n:]
            assert rel_l2(y[i], want) <= tol, rel_l2(y[i], want)

    root = m.new()
    text[root] = np.zeros((0, d))
    step([root], 37)
    kids = m.fork(root, 3)
    for k in kids:
        text[k] = text[root]
    assert m.shared_len(kids) == 32
    step(kids, 1)
    step(kids, 12)
    step([kids[2], root], 5)
    grand = m.fork(kids[1], 2)
    for k in grand:
        text[k] = text[kids[1]]
    assert m.shared_len(grand) == 48 and m.shared_len([grand[0], root]) == 32
    m.free([kids[0], kids[1]])
    live = int(m.compact())
    assert live == int((m.cache.ref > 0).sum()) and bool((m.cache.ref[:live] > 0).all())
    step(grand + [root, kids[2]], 3)
    step(grand, 17)
    m.free(grand + [root, kids[2]])
    assert int(m.cache.ref.sum()) == 0
    with pytest.raises(ValueError):
        m.fork(root, 9)


def test_example_runs():
    from paper_2604_20289_gb300 import branches
    branches.main()
