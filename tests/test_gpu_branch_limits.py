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
