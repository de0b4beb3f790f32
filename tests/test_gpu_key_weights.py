"""The log of each row's sum of exponentials that the attention leaves, and the
weight it gave to each cached key, against plain 64-bit restatements.

Tolerances (derived from the arithmetic).  A score in units of log2 e is a sum of
terms of size 20 or so over the head; the tensor core adds it in head_dim / 16 <= 8
steps, each good to 2^-23 of that size (2e-5 in all, absolute), and what follows
rounds values up to 64 a few times at 2^-24 (1e-5).  So a log of a sum is good to
4e-5 (fp32: 1e-5), each weight to 4e-5 of itself, and their sums, of positive terms,
to as much element by element; the errors are independent, so the 2-norm stays below 1e-5.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402
from test_gpu_branch import DEV, MULTI_CASES, TOKEN_CASES, host, i32, make_cache, rand, rel_l2  # noqa: E402


def reference(cache, seqs, n_q, q, causal, scale=None):
    """(lse [T, H], per branch the weight of each key) in 64 bits."""
    hd, hk, ps = cache.head_dim, cache.n_kv_heads, cache.page_size
    k, table, lens = host(cache.k[0]), cache.table.cpu().numpy(), cache.len.cpu().numpy()
    B = len(seqs)
    q = host(q).reshape(B, n_q, -1, hd)
    H = q.shape[2]
    lse, out = np.full((B, n_q, H), -np.inf), []
    for b, s in enumerate(seqs):
        n = int(lens[s])
        j = np.arange(n)
        kk = k[table[s, j // ps], j % ps].reshape(n, hk, hd)
        sees = j[None] < ((n - n_q + np.arange(n_q) + 1) if causal else np.full(n_q, n))[:, None]
        w = np.zeros(n)
        for h in range(H):
            x = np.where(sees, q[b, :, h] @ kk[:, h // (H // hk)].T * (scale or 1 / math.sqrt(hd)), -np.inf)
            for i in range(n_q):
                if sees[i].any():
                    m = x[i].max()
                    lse[b, i, h] = m + math.log(np.exp(x[i] - m).sum())
                    w += np.exp(x[i] - lse[b, i, h])
        out.append(w)
    return lse.reshape(B * n_q, H), out


def check(dtype, H, hk, hd, ps, lens, n_q, shared, causal, seqs=None, scale=0.0, decay=1.0, seed=3, std=1.5, strided=False,
          max_pages=None):
    cache = make_cache(dtype, hk, hd, ps, lens, shared, seed=seed, max_pages=max_pages)
    seqs = list(range(len(lens))) if seqs is None else seqs
    q = rand((len(seqs) * n_q, H * hd + (64 if strided else 0)), dtype, seed + 7, std)[:, :H * hd]
    o = torch.empty(len(seqs) * n_q, H * hd, dtype=q.dtype, device=DEV)
    lse = torch.full((len(seqs) * n_q, H), float("nan"), device=DEV)
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, o, shared_len=shared, causal=causal, scale=scale, lse=lse)
    plain = torch.empty_like(o)
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, plain, shared_len=shared, causal=causal, scale=scale)
    assert torch.equal(o, plain)
    want_lse, want = reference(cache, seqs, n_q, q, causal, scale or None)
    got_lse = host(lse)
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got_lse), empty)
    if not empty.all():
        assert np.abs(got_lse[~empty] - want_lse[~empty]).max() <= (4e-5 if dtype == "bf16" else 1e-5)
    # the row of weights is wider than the table's, and what is past a sequence's end may hold anything
    width = cache.table.shape[1] * ps + 12
    old = rand((len(lens), width), "f32", seed + 9).abs()
    for s, n in enumerate(lens):
        old[s, n:] = float("nan")
        if decay == 0.0:
            old[s] = float("nan")
    w = old.clone()
    need = xb.op_key_weights_workspace_bytes(cache, len(seqs), n_q, H, shared)
    ws = torch.full((need // 4,), float("nan"), device=DEV)
    xb.op_key_weights(cache, 0, i32(seqs), n_q, q, lse, w, shared_len=shared, causal=causal, scale=scale, decay=decay,
                      workspace=ws)
    torch.cuda.synchronize()
    assert xb.op_device_error() == 0
    for s, n in enumerate(lens):
        here = [b for b, x in enumerate(seqs) if x == s]
        if not here:
            assert torch.equal(w[s].isnan(), old[s].isnan()) and torch.equal(w[s].nan_to_num(), old[s].nan_to_num())
            continue
        assert w[s, n:].isnan().all()
        if n == 0:
            continue
        add = want[here[0]]
        base = decay * host(old[s, :n]) if decay else np.zeros(n)
        off = np.abs(host(w[s, :n]) - base - add)
        assert (off <= 4e-5 * add + 2.0 ** -22 * (base + add)).all(), float((off / np.maximum(add, 1e-30)).max())
        assert np.linalg.norm(off) <= 1e-5 * np.linalg.norm(add) + 2.0 ** -23 * np.linalg.norm(base + add)
    again = old.clone()
    xb.op_key_weights(cache, 0, i32(seqs), n_q, q, lse, again, shared_len=shared, causal=causal, scale=scale, decay=decay)
    assert torch.equal(again.view(torch.int32), w.view(torch.int32))          # the same bits every time
    return cache, q, lse, w


@pytest.mark.parametrize("H,hk,hd,ps,lens,shared", TOKEN_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_single_tokens(H, hk, hd, ps, lens, shared, causal):
    check("bf16", H, hk, hd, ps, lens, 1, shared, causal)


@pytest.mark.parametrize("H,hk,hd,ps,lens,n_q,shared", MULTI_CASES)
@pytest.mark.parametrize("causal", [True, False])
def test_several_tokens(H, hk, hd, ps, lens, n_q, shared, causal):
    check("bf16", H, hk, hd, ps, lens, n_q, shared, causal)


@pytest.mark.parametrize("H,hk,hd,ps,lens,n_q,shared", [
    (4, 4, 16, 16, [200, 33, 100], 20, 0), (12, 4, 32, 32, [352, 340, 400, 321], 20, 320), (6, 2, 64, 128, [300, 259, 1000], 259, 0),
    (3, 3, 128, 16, [10, 40, 0], 25, 0), (5, 1, 128, 64, [64, 1000, 65], 1, 64), (64, 1, 16, 16, [70, 90], 5, 64),
    (2, 2, 64, 1024, [3000, 2050], 1, 2048)])
@pytest.mark.parametrize("causal", [True, False])
def test_fp32(H, hk, hd, ps, lens, n_q, shared, causal):
    check("f32", H, hk, hd, ps, lens, n_q, shared, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("shared", [0, 96])
def test_decay_and_scale(dtype, decay, shared):
    check(dtype, 6, 2, 64, 32, [200, 130, 97], 3, shared, True, decay=decay, scale=0.07, strided=True)


@pytest.mark.parametrize("n_q,shared", [(1, 0), (1, 64), (40, 0)])
def test_rows_of_other_branches_do_not_leak(n_q, shared):
    """A branch whose queries are NaN spoils its own weights only."""
    H, hk, hd, ps, lens = 5, 1, 64, 16, [100, 90, 120]
    cache, q, lse, w = check("bf16", H, hk, hd, ps, lens, n_q, shared, True)
    q = q.clone()
    q[n_q:2 * n_q] = float("nan")
    got = torch.zeros_like(w)
    xb.op_key_weights(cache, 0, i32([0, 1, 2]), n_q, q, lse, got, shared_len=shared, causal=True)
    clean = torch.zeros_like(w)
    xb.op_key_weights(cache, 0, i32([0, 1, 2]), n_q, q.nan_to_num(), lse, clean, shared_len=shared, causal=True)
    assert torch.equal(got[[0, 2]], clean[[0, 2]]) and got[1, :lens[1]].isnan().all()


def test_every_row_adds_one():
    lens, n_q, H = [700, 513, 600], 9, 8
    *_, w = check("bf16", H, 4, 64, 16, lens, n_q, 512, True, decay=0.0)
    for s, n in enumerate(lens):
        assert abs(w[s, :n].double().sum().item() - n_q * H) <= 4e-5 * n_q * H


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,shared", [(1, 64), (3, 0), (50, 0)])
def test_sequences_in_another_order_and_left_out(dtype, n_q, shared):
    check(dtype, 4, 2, 64, 16, [100, 222, 70, 190, 130], n_q, shared, True, seqs=[3, 0, 4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,shared", [(1, 64), (1, 0), (40, 0)])
def test_a_sequence_listed_twice_or_out_of_range_is_flagged(dtype, n_q, shared):
    cache, q, lse, w = check(dtype, 4, 2, 64, 16, [100, 122, 70], n_q, shared, True)
    q, lse = torch.cat([q, q[:n_q], q[:n_q]]), torch.cat([lse, lse[:n_q], lse[:n_q]])
    want = torch.zeros_like(w)
    xb.op_key_weights(cache, 0, i32([0, 1, 2]), n_q, q[:3 * n_q], lse[:3 * n_q], want, shared_len=shared, causal=True)
    assert xb.op_device_error() == 0
    for last in (1, -1, 3, 1 << 30):
        got = torch.zeros_like(w)
        xb.op_key_weights(cache, 0, i32([0, 1, 2, 0, last]), n_q, q, lse, got, shared_len=shared, causal=True)
        assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
        assert (got - want).abs().max().item() <= 1e-5 * want.max().item()     # (other cuts, other orders)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bad_page_counts_as_zeros(dtype):
    cache, q, lse, w = check(dtype, 2, 2, 64, 16, [100, 122], 1, 0, True)
    cache.table[1, 3] = 1 << 20
    got = torch.zeros_like(w)
    xb.op_key_weights(cache, 0, i32([0, 1]), 1, q, lse, got, causal=True)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    want = torch.exp(-lse[1]).sum().item()                                     # scores of 0
    assert (got[1, 48:64] - want).abs().max().item() <= 1e-5 * want


def test_a_thousand_branches():
    lens = [64 + (37 * b) % 90 for b in range(1024)]
    check("bf16", 2, 2, 64, 16, lens, 1, 64, True)
    check("bf16", 1, 1, 64, 16, lens, 2, 0, True)


@pytest.mark.parametrize("H,hk,hd,lens,n_q,shared", [
    (128, 128, 128, [200, 150], 1, 64),                # more key heads than rows fit shared memory
    (40, 40, 128, [300, 260, 290], 1, 256), (3, 3, 64, [300, 260, 290], 7, 256), (5, 5, 128, [130] * 9, 12, 64),
    (48, 16, 64, [400, 333], 5, 320), (1, 1, 64, [300 + 3 * b for b in range(70)], 1, 288),
    (2, 2, 128, [300 + b for b in range(66)], 1, 288), (17, 17, 64, [90, 70], 3, 0), (64, 2, 64, [99, 500, 64], 2, 0), (2, 1, 128, [700], 32, 0),
    (2, 1, 128, [700], 33, 0), (6, 6, 128, [1000] * 3, 64, 512), (6, 6, 128, [1000] * 3, 65, 512)])
def test_head_layouts_of_few_rows(H, hk, hd, lens, n_q, shared):
    check("bf16", H, hk, hd, 32, lens, n_q, shared, True)


def wide(hk, hd, ps, shared=0):
    """Pages of a table row that allow for more keys than few rows take into registers (12 MB)."""
    return (13 * 2 ** 20 // (hk * hd * 2) + shared) // ps + 1


@pytest.mark.parametrize("H,hk,hd,ps,lens,n_q,shared", [
    (1, 1, 64, 16, [1], 1, 0), (4, 4, 64, 16, [33, 16, 17, 20], 1, 16), (8, 8, 64, 16, [2017, 2030, 2056, 2016], 1, 2016),
    (8, 1, 128, 32, [130, 129, 128, 700, 64], 1, 64), (5, 1, 128, 64, [64, 1000, 65], 1, 64),
    (21, 3, 128, 128, [300, 511, 129, 128, 2000, 131, 140], 1, 128), (40, 8, 128, 32, [4000 + 37 * b for b in range(32)], 1, 3968),
    (32, 4, 64, 256, [256 + b for b in range(9)], 1, 256), (12, 12, 128, 16, [0, 5, 0, 129], 1, 0), (64, 1, 64, 16, [700, 900], 1, 640),
    (2, 2, 64, 1024, [3000, 2050], 1, 2048), (2, 2, 64, 16, [64 + (37 * b) % 90 for b in range(130)], 1, 64),
    (1, 1, 128, 64, [19968 + 5 * b for b in range(3)], 1, 19968), (3, 3, 64, 16, [10, 40, 0], 25, 0), (12, 12, 128, 32, [352, 340, 400, 321], 20, 320),
    (2, 2, 128, 16, [100 + (13 * b) % 61 for b in range(70)], 3, 0), (1, 1, 64, 32, [160 + b % 30 for b in range(40)], 20, 128),
    (3, 1, 64, 16, [300, 260, 290, 250], 1, 240), (6, 1, 64, 16, [300, 260, 290, 250], 1, 240), (7, 1, 64, 16, [300, 260, 290, 250] * 2, 1, 240),
    (2, 1, 64, 64, [400 + b for b in range(30)], 2, 384), (9, 3, 128, 32, [200, 333, 64], 2, 64), (11, 1, 64, 16, [150, 140], 1, 128),
    (16, 1, 64, 32, [290, 300, 310, 320], 1, 288), (17, 1, 64, 32, [290, 300, 310, 320], 1, 288), (128, 128, 64, 16, [129, 257], 1, 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows_over_many_keys(H, hk, hd, ps, lens, n_q, shared, causal):
    check("bf16", H, hk, hd, ps, lens, n_q, shared, causal, max_pages=wide(hk, hd, ps, shared), decay=0.5)


@pytest.mark.parametrize("decay", [0.0, 1.0])
def test_many_keys_decay_scale_strides_and_order(decay):
    check("bf16", 4, 2, 64, 16, [100, 122, 70], 2, 64, True, seqs=[2, 0], scale=0.3, decay=decay, strided=True, max_pages=wide(2, 64, 16))
    check("bf16", 4, 2, 64, 16, [100, 122, 70], 2, 0, True, seqs=[1, 2], decay=decay, strided=True, max_pages=wide(2, 64, 16))


def test_many_keys_flags():
    cache, q, lse, w = check("bf16", 2, 2, 64, 16, [100, 122, 300], 1, 64, True, max_pages=wide(2, 64, 16))
    want, got = torch.zeros_like(w), torch.zeros_like(w)
    xb.op_key_weights(cache, 0, i32([0, 1, 2]), 1, q, lse, want, shared_len=64, causal=True)
    assert xb.op_device_error() == 0
    for last in (1, -1, 3, 1 << 30):                       # listed twice, out of range
        got.zero_()
        xb.op_key_weights(cache, 0, i32([0, 1, 2, last]), 1, torch.cat([q, q[:1]]), torch.cat([lse, lse[:1]]), got, shared_len=64, causal=True)
        assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
        assert (got - want).abs().max().item() <= 1e-5 * want.max().item()
    cache.table[2, 5] = 1 << 20                            # a bad page counts as zeros
    got.zero_()
    xb.op_key_weights(cache, 0, i32([0, 1, 2]), 1, q, lse, got, shared_len=64, causal=True)
    assert xb.op_device_error() == xb.XC_DEV_BAD_SEQUENCE
    zero = torch.exp(-lse[2]).sum().item()
    assert (got[2, 80:96] - zero).abs().max().item() <= 1e-5 * zero
    assert torch.equal(got[:2], want[:2]) and torch.equal(got[2, :80], want[2, :80]) and torch.equal(got[2, 96:], want[2, 96:])


def test_long_rows_and_many_cuts():
    check("bf16", 1, 1, 128, 64, [19968 + 5 * b for b in range(3)], 1, 19968, True)
    check("bf16", 2, 1, 128, 128, [5000], 1, 0, True)


@pytest.mark.parametrize("many", [False, True])
def test_a_captured_step_follows_the_lengths(many):
    """Attention and weights in one graph: replays see the cache as it is then."""
    H, hk, hd, ps = 4, 2, 64, 16
    lens, longer = [40, 90], [47, 200]
    cache = make_cache("bf16", hk, hd, ps, longer, 0, dead=0.0, max_pages=wide(hk, hd, ps) if many else None)
    q = rand((2, H * hd), "bf16", 5, 1.5)
    o, lse = torch.empty_like(q), torch.empty(2, H, device=DEV)
    w = torch.zeros(2, cache.table.shape[1] * ps, device=DEV)
    cache.len.copy_(i32(lens))
    seqs = i32([0, 1])

    def step():
        xb.op_branch_attention(cache, 0, seqs, 1, q, o, causal=True, lse=lse)
        xb.op_key_weights(cache, 0, seqs, 1, q, lse, w, causal=True, decay=0.0)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for now in (lens, longer):
        cache.len.copy_(i32(now))
        w.zero_()
        g.replay()
        torch.cuda.synchronize()
        for b, want in enumerate(reference(cache, [0, 1], 1, q, True)[1]):
            assert rel_l2(host(w[b, :now[b]]), want) <= 1e-5 and not w[b, now[b]:].any()
    assert xb.op_device_error() == 0


def test_refusals():
    cache = make_cache("bf16", 2, 64, 16, [40, 90], 0)
    q, lse, w = rand((2, 4 * 64), "bf16", 1), torch.zeros(2, 4, device=DEV), torch.zeros(2, cache.table.shape[1] * 16, device=DEV)
    xb.op_key_weights(cache, 0, i32([0, 1]), 1, q, lse, w)
    for bad in (dict(q=q.float()), dict(q=q[:1]), dict(q=q.t().contiguous().t()), dict(lse=lse.double()), dict(lse=lse[:, :3]),
                dict(lse=lse.t().contiguous().t()), dict(w=w[:1]), dict(w=w[:, :-1].contiguous()), dict(w=w.double()),
                dict(w=w.t().contiguous().t()), dict(w=w.cpu()), dict(lse=lse.cpu()), dict(seqs=i32([0, 1]).long())):
        a = dict(q=q, lse=lse, w=w, seqs=i32([0, 1]))
        a.update(bad)
        with pytest.raises(ValueError):
            xb.op_key_weights(cache, 0, a["seqs"], 1, a["q"], a["lse"], a["w"])
    for bad in (dict(decay=-1.0), dict(decay=float("nan")), dict(scale=-1.0), dict(shared_len=8),
                dict(workspace=torch.empty(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(xb.XCacheError):
            xb.op_key_weights(cache, 0, i32([0, 1]), 1, q, lse, w, **bad)
    with pytest.raises(ValueError):
        xb.op_branch_attention(cache, 0, i32([0, 1]), 1, q, torch.empty_like(q), lse=lse.double())
