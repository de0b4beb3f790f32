"""Rows of the branch attention that are not finite: what their log of a sum of
exponentials, their output and the weights of their keys become.

What is expected follows from the definition in 64 bits, rounded to the outputs' type:
* a NaN in a query, or in a key that a row sees, makes the row's lse and output NaN;
* a score of +infinity makes lse +infinity; the output is NaN, as the softmax then is in every term;
* a score of -infinity adds nothing: the row is as if it did not see the key;
* -infinity is the lse of a row that sees no key, and of no other row here.
Rows beside them, of the same unit and of others, keep their bits.  Finite lse are
compared within the bound that holds for them elsewhere (4e-5 bf16, 1e-5 fp32)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402
from test_gpu_branch import DEV, host, i32, make_cache, rand  # noqa: E402

BIG = 2.0 ** 100                                          # its square passes every score of 32 bits
# H, hk, hd, page, lens, n_q, shared: key tiles are 128 keys (bf16) or 64 (fp32), so short sequences are
# units that one CTA runs whole, long ones are cut between CTAs
LAYOUTS = [
    (4, 2, 64, 16, [100, 60, 128, 77], 1, 0),             # whole units, some of whose keys are masked
    (4, 2, 128, 16, [100, 60, 128, 77], 40, 0),
    (2, 1, 64, 64, [5000, 4990], 1, 0),                   # cut
    (2, 1, 128, 64, [5003, 4097], 1, 0),                  # and a last tile of one key, a piece by itself
    (6, 2, 128, 32, [3000, 2900, 3100], 300, 0),          # cut units of many rows
    (12, 12, 64, 32, [700] * 6, 130, 0),                  # whole and cut ones
    (4, 2, 64, 16, [1040, 1030, 1100, 1025], 1, 1024),    # keys in common
    (8, 1, 128, 32, [4000 + 37 * b for b in range(16)], 1, 3968),
    (4, 2, 128, 32, [2100, 2090, 2200], 20, 2048),
    (12, 12, 128, 32, [2000, 1990, 2100], 1, 0),          # single tokens over more than 12 MB of keys
    (24, 12, 128, 32, [2100, 2090, 2200], 2, 1024),
]
F32_LAYOUTS = [(4, 2, 16, 16, [50, 60, 64], 1, 0), (4, 4, 32, 16, [50, 33, 64], 20, 0), (2, 1, 64, 64, [3000, 2945], 1, 0),
               (2, 2, 128, 64, [1500, 1003], 50, 0), (4, 2, 16, 16, [1040, 1030, 1100], 1, 1024), (4, 2, 64, 32, [2100, 2090], 20, 2048)]


def cases():
    return [("bf16", *c) for c in LAYOUTS] + [("f32", *c) for c in F32_LAYOUTS]


def output(cache, seqs, n_q, q, shared, causal):
    o = torch.full_like(q, 3.0)
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, o, shared_len=shared, causal=causal)
    assert xb.op_device_error() == 0
    return o


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,n_q,shared", cases())
def test_output_of_a_nan_query(dtype, H, hk, hd, ps, lens, n_q, shared, causal):
    """Whole units and cut ones, whose pieces may hold masked keys."""
    cache = make_cache(dtype, hk, hd, ps, lens, shared, seed=11)
    q, seqs = rand((len(lens) * n_q, H * hd), dtype, 12, 1.5), list(range(len(lens)))
    o0 = output(cache, seqs, n_q, q, shared, causal)
    t = 2 * n_q - 1                                        # branch 1's last row, one head of it
    q[t, (H - 1) * hd + 3] = float("nan")
    o = output(cache, seqs, n_q, q, shared, causal)
    assert o[t, (H - 1) * hd:].isnan().all()
    hurt = torch.zeros_like(o, dtype=torch.bool)
    hurt[t, (H - 1) * hd:] = True
    assert torch.equal(o[~hurt], o0[~hurt])


@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,n_q,shared", cases())
def test_output_of_a_nan_key(dtype, H, hk, hd, ps, lens, n_q, shared):
    cache = make_cache(dtype, hk, hd, ps, lens, shared, seed=11)
    q, seqs = rand((len(lens) * n_q, H * hd), dtype, 12, 1.5), list(range(len(lens)))
    o0 = output(cache, seqs, n_q, q, shared, False)
    grp, k0 = H // hk, cache.k.clone()
    for j in sorted({shared, (shared + lens[1]) // 2, lens[1] - 1}) + ([0, shared - 1] if shared else []):
        cache.k.copy_(k0)
        cache.k[0, int(cache.table[1, j // ps]), j % ps, (hk - 1) * hd + 5] = float("nan")
        o = output(cache, seqs, n_q, q, shared, False)
        rows = slice(0, len(lens) * n_q) if j < shared else slice(n_q, 2 * n_q)
        hurt = torch.zeros_like(o, dtype=torch.bool)
        hurt[rows, (hk - 1) * grp * hd:] = True
        assert o[hurt].isnan().all()
        assert torch.equal(o[~hurt], o0[~hurt])


# ------------------------------------------------- the log of the sum and the weights
def place(cache, seq, j):
    return int(cache.table[seq, j // cache.page_size]), j % cache.page_size


def attend(cache, seqs, n_q, q, H, shared, causal):
    o, lse = torch.full_like(q, 3.0), torch.full((q.shape[0], H), 5.0, device=DEV)
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, o, shared_len=shared, causal=causal, lse=lse)
    plain = torch.full_like(q, 3.0)
    xb.op_branch_attention(cache, 0, i32(seqs), n_q, q, plain, shared_len=shared, causal=causal)
    bits = torch.int16 if q.dtype is torch.bfloat16 else torch.int32
    assert torch.equal(torch.nan_to_num(o, nan=9.0).view(bits), torch.nan_to_num(plain, nan=9.0).view(bits))
    assert xb.op_device_error() == 0
    return o, lse


def weigh(cache, seqs, n_q, q, lse, shared, causal):
    w = torch.zeros(cache.table.shape[0], cache.table.shape[1] * cache.page_size, device=DEV)
    xb.op_key_weights(cache, 0, i32(seqs), n_q, q, lse, w, shared_len=shared, causal=causal)
    assert xb.op_device_error() == 0
    return w


def setup(dtype, H, hk, hd, ps, lens, n_q, shared):
    """A cache and queries of which the first numbers of a head stay free: 0 in every row."""
    cache = make_cache(dtype, hk, hd, ps, lens, shared, seed=11)
    q = rand((len(lens) * n_q, H * hd), dtype, 12, 1.5)
    q.view(-1, H, hd)[:, :, 0] = 0
    heads = cache.k.view(*cache.k.shape[:3], hk, hd)
    heads[..., 0] = torch.where(heads[..., 0].isnan(), heads[..., 0], torch.zeros_like(heads[..., 0]))
    return cache, q, list(range(len(lens)))


def others_keep_their_bits(o, o0, lse, lse0, hurt, hd):
    """hurt [rows, heads]: who may change."""
    assert torch.equal(lse[~hurt], lse0[~hurt])
    wide = hurt.repeat_interleave(hd, 1)
    assert torch.equal(o[~wide], o0[~wide])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,n_q,shared", cases())
def test_a_nan_query(dtype, H, hk, hd, ps, lens, n_q, shared, causal):
    cache, q, seqs = setup(dtype, H, hk, hd, ps, lens, n_q, shared)
    o0, lse0 = attend(cache, seqs, n_q, q, H, shared, causal)
    w0 = weigh(cache, seqs, n_q, q, lse0, shared, causal)
    t = n_q + n_q // 2                                    # a row of branch 1
    bad = q.clone()
    bad[t, (H - 1) * hd + 3] = float("nan")
    o, lse = attend(cache, seqs, n_q, bad, H, shared, causal)
    hurt = torch.zeros_like(lse, dtype=torch.bool)
    hurt[t, H - 1] = True
    sees = max(lens[1] - (n_q - 1 - n_q // 2 if causal else 0), 0)
    if sees:
        assert lse[t, H - 1].isnan() and o[t, (H - 1) * hd:].isnan().all()
    else:
        assert lse[t, H - 1] == -math.inf and not o[t, (H - 1) * hd:].any()
    others_keep_their_bits(o, o0, lse, lse0, hurt, hd)
    w = weigh(cache, seqs, n_q, bad, lse, shared, causal)
    keep = [s for s in seqs if s != 1]
    assert torch.equal(w[keep], w0[keep]) and w[1, :sees].isnan().all() and torch.equal(w[1, sees:], w0[1, sees:])


@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,n_q,shared", cases())
def test_a_nan_key(dtype, H, hk, hd, ps, lens, n_q, shared):
    """Of a branch's own keys, first, last and in between, and of those in common."""
    cache, q, seqs = setup(dtype, H, hk, hd, ps, lens, n_q, shared)
    o0, lse0 = attend(cache, seqs, n_q, q, H, shared, False)
    w0 = weigh(cache, seqs, n_q, q, lse0, shared, False)
    grp, k0 = H // hk, cache.k.clone()
    for j in sorted({shared, (shared + lens[1]) // 2, lens[1] - 1}) + ([0, shared - 1] if shared else []):
        cache.k.copy_(k0)
        page, slot = place(cache, 1, j)
        cache.k[0, page, slot, (hk - 1) * hd + 5] = float("nan")
        o, lse = attend(cache, seqs, n_q, q, H, shared, False)
        hurt = torch.zeros_like(lse, dtype=torch.bool)
        rows = slice(0, len(lens) * n_q) if j < shared else slice(n_q, 2 * n_q)
        hurt[rows, (hk - 1) * grp:] = True
        assert lse[hurt].isnan().all() and o[hurt.repeat_interleave(hd, 1)].isnan().all()
        others_keep_their_bits(o, o0, lse, lse0, hurt, hd)
        w = weigh(cache, seqs, n_q, q, lse, shared, False)
        for s in seqs:
            if j < shared or s == 1:
                assert w[s, :lens[s]].isnan().all()
            else:
                assert torch.equal(w[s], w0[s])


@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,n_q,shared", cases())
def test_infinite_scores(dtype, H, hk, hd, ps, lens, n_q, shared):
    cache, q, seqs = setup(dtype, H, hk, hd, ps, lens, n_q, shared)
    grp, t = H // hk, n_q + n_q // 2
    q.view(-1, H, hd)[t, H - 1, 0] = BIG                  # the only row with a number there
    o0, lse0 = attend(cache, seqs, n_q, q, H, shared, False)
    w0 = weigh(cache, seqs, n_q, q, lse0, shared, False)
    k0 = cache.k.clone()
    hurt = torch.zeros_like(lse0, dtype=torch.bool)
    hurt[t, H - 1] = True
    for j in sorted({0, lens[1] // 2, lens[1] - 1}):
        page, slot = place(cache, 1, j)
        cache.k.copy_(k0)
        cache.k[0, page, slot, (hk - 1) * hd] = BIG
        o, lse = attend(cache, seqs, n_q, q, H, shared, False)
        assert lse[t, H - 1] == math.inf and o[t, (H - 1) * hd:].isnan().all()
        others_keep_their_bits(o, o0, lse, lse0, hurt, hd)
        w = weigh(cache, seqs, n_q, q, lse, shared, False)
        assert w[1, j].isnan() and w.isnan().sum() == 1   # the row's other keys get nothing of it
        assert all(torch.equal(w[s], w0[s]) for s in seqs if s != 1)
        # -infinity: the key is as good as gone for this row
        cache.k[0, page, slot, (hk - 1) * hd] = -BIG
        o, lse = attend(cache, seqs, n_q, q, H, shared, False)
        others_keep_their_bits(o, o0, lse, lse0, hurt, hd)
        keys = np.arange(lens[1])
        table = cache.table.cpu().numpy()
        k = host(k0[0]).reshape(-1, ps, hk, hd)[table[1, keys // ps], keys % ps, hk - 1]
        s = np.delete(k, j, 0) @ host(q[t, (H - 1) * hd:]) / math.sqrt(hd)
        want = s.max() + math.log(np.exp(s - s.max()).sum())
        assert abs(lse[t, H - 1].item() - want) <= (4e-5 if dtype == "bf16" else 1e-5)
        assert o[t].isfinite().all()
        assert weigh(cache, seqs, n_q, q, lse, shared, False).isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,shared", [(1, 0), (1, 64), (3, 0)])
def test_rows_that_see_no_key_stay_apart(dtype, n_q, shared):
    """-infinity beside NaN: an empty sequence, and one whose queries are NaN."""
    H, hk, hd, lens = 4, 2, 64, [0 if shared == 0 else 64, 90, 70]
    cache, q, seqs = setup(dtype, H, hk, hd, 16, lens, n_q, shared)
    q[n_q:2 * n_q] = float("nan")
    o, lse = attend(cache, seqs, n_q, q, H, shared, True)
    assert lse[n_q:2 * n_q].isnan().all() and o[n_q:2 * n_q].isnan().all()
    assert lse[2 * n_q:].isfinite().all() and o[2 * n_q:].isfinite().all()
    if shared == 0:
        assert (lse[:n_q] == -math.inf).all() and not o[:n_q].any()
    w = weigh(cache, seqs, n_q, q, lse, shared, True)
    assert w[1, :90 - n_q + 1].isnan().all() and w[[0, 2]].isfinite().all()


def test_what_a_layer_does_with_such_a_row():
    """8-bit projections give NaN rows for a token that is not finite; its weights show it, and eviction still runs."""
    from paper_2604_20289_gb300 import branches
    d, H, Hk, hd = 256, 4, 2, 64
    m = branches.BranchedLayers(branches.quantize_layers(branches.random_layers(2, d, H, Hk, hd)), H, Hk, hd, n_pages=64, page_size=16,
                                max_seqs=4, max_len=256, track=0.5)
    a, b = m.new(), m.new()
    g = torch.Generator(device=DEV).manual_seed(3)
    for _ in range(6):
        m.step([a, b], torch.randn(2, 16, d, generator=g, device=DEV))
    x = torch.randn(2, 1, d, generator=g, device=DEV)
    x[0, 0, 7] = float("inf")
    y = m.step([a, b], x)
    assert y[0].isnan().all() and y[1].isfinite().all()
    assert m.key_weights[a, :97].isnan().all() and m.key_weights[b, :97].isfinite().all()
    kept = m.evict([a, b], 40, n_first=4, n_last=4)
    assert kept[0] == list(range(36)) + list(range(93, 97))              # equal weights: the earliest stay
    assert len(kept[1]) == 40 and xb.op_device_error() == 0
