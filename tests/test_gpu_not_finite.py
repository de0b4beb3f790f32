"""Rows of the branch attention that are not finite.

What is expected follows from the definition in 64 bits, rounded to the output's type: a
NaN in a query, or in a key that a row sees, makes the row's output NaN, and rows beside
them, of the same unit and of others, keep their bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402
from test_gpu_branch import i32, make_cache, rand  # noqa: E402

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
]
F32_LAYOUTS = [(4, 2, 16, 16, [50, 60, 64], 1, 0), (4, 4, 32, 16, [50, 33, 64], 20, 0), (2, 1, 64, 64, [3000, 2945], 1, 0),
               (2, 2, 128, 64, [1500, 1003], 50, 0), (4, 2, 16, 16, [1040, 1030, 1100], 1, 1024), (4, 2, 64, 32, [2100, 2090], 20, 2048)]


def cases():
    return [("bf16", *c) for c in LAYOUTS] + [("f32", *c) for c in F32_LAYOUTS]


def attend(cache, seqs, n_q, q, shared, causal):
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
    o0 = attend(cache, seqs, n_q, q, shared, causal)
    t = 2 * n_q - 1                                        # branch 1's last row, one head of it
    q[t, (H - 1) * hd + 3] = float("nan")
    o = attend(cache, seqs, n_q, q, shared, causal)
    assert o[t, (H - 1) * hd:].isnan().all()
    hurt = torch.zeros_like(o, dtype=torch.bool)
    hurt[t, (H - 1) * hd:] = True
    assert torch.equal(o[~hurt], o0[~hurt])


@pytest.mark.parametrize("dtype,H,hk,hd,ps,lens,n_q,shared", cases())
def test_output_of_a_nan_key(dtype, H, hk, hd, ps, lens, n_q, shared):
    cache = make_cache(dtype, hk, hd, ps, lens, shared, seed=11)
    q, seqs = rand((len(lens) * n_q, H * hd), dtype, 12, 1.5), list(range(len(lens)))
    o0 = attend(cache, seqs, n_q, q, shared, False)
    grp, k0 = H // hk, cache.k.clone()
    for j in sorted({shared, (shared + lens[1]) // 2, lens[1] - 1}) + ([0, shared - 1] if shared else []):
        cache.k.copy_(k0)
        cache.k[0, int(cache.table[1, j // ps]), j % ps, (hk - 1) * hd + 5] = float("nan")
        o = attend(cache, seqs, n_q, q, shared, False)
        rows = slice(0, len(lens) * n_q) if j < shared else slice(n_q, 2 * n_q)
        hurt = torch.zeros_like(o, dtype=torch.bool)
        hurt[rows, (hk - 1) * grp * hd:] = True
        assert o[hurt].isnan().all()
        assert torch.equal(o[~hurt], o0[~hurt])
