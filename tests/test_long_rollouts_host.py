"""Host-side argument checks of the operators of long rollouts (8-bit products):
every refusal comes before any CUDA call, so no GPU is needed."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2604_20289_gb300", "libxcache.so")
P = 1 << 20          # a 256-byte aligned address that is never read


@pytest.fixture(scope="module")
def xb():
    if not os.path.exists(LIB):
        from paper_2604_20289_gb300 import build
        build.build()
    from paper_2604_20289_gb300 import xcache
    return xcache


@pytest.mark.parametrize("kw,msg", [
    (dict(dtype=2), "dtype"), (dict(dtype=-1), "dtype"), (dict(M=-1), "K a multiple"), (dict(M=1 << 24), "K a multiple"),
    (dict(K=0), "K a multiple"), (dict(K=24), "K a multiple"), (dict(K=-16), "K a multiple"),
    (dict(K=(1 << 17) + 16), "K a multiple"), (dict(x=0), "pointer"), (dict(q=0), "pointer"), (dict(scale=0), "pointer"),
    (dict(x=P + 8), "pointer"), (dict(q=P + 4), "pointer")])
def test_quantise_refusals(xb, kw, msg):
    a = dict(dtype=xb.XC_BF16, M=4, K=64, x=P, q=P, scale=P)
    a.update(kw)
    assert xb.LIB.xc_op_quantize_rows(a["dtype"], a["M"], a["K"], a["x"], a["q"], a["scale"], None) == xb.XC_EINVAL
    assert msg in xb.last_error(None)


@pytest.mark.parametrize("kw,msg", [
    (dict(dtype=2), "dtype"), (dict(epi=3), "epilogue"), (dict(epi=-1), "epilogue"), (dict(epi=16), "epilogue"),
    (dict(M=-1), "K a multiple"), (dict(N=0), "K a multiple"), (dict(K=40), "K a multiple"), (dict(N=1 << 24), "K a multiple"),
    (dict(M=(1 << 24) - 1, N=(1 << 24) - 1, K=1 << 17), "K a multiple"), (dict(A=0), "NULL"), (dict(W=0), "NULL"),
    (dict(ws=0), "NULL"), (dict(bias=0), "NULL"), (dict(out=0), "NULL"), (dict(epi=2), "residual"),
    (dict(epi=2, gate=P), "residual"), (dict(A=P + 8), "aligned"), (dict(W=P + 8), "aligned"), (dict(work=0), "workspace"),
    (dict(work=P + 16), "workspace"), (dict(bytes=100), "workspace")])
def test_product_refusals(xb, kw, msg):
    a = dict(dtype=xb.XC_BF16, epi=0, M=40, N=100, K=64, A=P, W=P, ws=P, bias=P, gate=0, resid=0, out=P, work=P, bytes=1 << 40)
    a.update(kw)
    st = xb.LIB.xc_op_linear_i8(a["dtype"], a["epi"], a["M"], a["N"], a["K"], a["A"], None, a["W"], a["ws"], a["bias"],
                                a["gate"], a["resid"], a["out"], a["work"], a["bytes"], None)
    assert st == xb.XC_EINVAL
    assert msg in xb.last_error(None), xb.last_error(None)


def test_nothing_to_do(xb):
    assert xb.LIB.xc_op_quantize_rows(xb.XC_BF16, 0, 64, None, None, None, None) == xb.XC_OK
    assert xb.LIB.xc_op_linear_i8(xb.XC_F32, 0, 0, 8, 64, *[None] * 8, None, 0, None) == xb.XC_OK
    assert xb.op_linear_i8_workspace_bytes(0, 8, 64) == 0
    assert xb.op_linear_i8_workspace_bytes(4, 8, 64) == 0 and xb.op_linear_i8_workspace_bytes(40, 8, 64) > 0
    assert xb.op_linear_i8_workspace_bytes(4, 8, 40) == 0 and "K a multiple" in xb.last_error(None)


# ------------------------------------------------------------ key weights
def desc(xb, **kw):
    f = dict(dtype=xb.XC_BF16, n_layers=2, n_pages=64, page_size=16, n_kv_heads=2, head_dim=64, max_seqs=4,
             max_pages=16, k=P, v=P, ref=P, table=P, len=P)
    f.update(kw)
    return xb.KVCacheDesc(**f)


@pytest.mark.parametrize("kw,msg", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(n_heads=3), "n_heads"), (dict(n_heads=2 * 129), "n_heads"),
    (dict(n_branches=-1), "n_branches"), (dict(n_branches=1025), "branches"), (dict(shared_len=8), "shared_len"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(decay=-0.5), "decay"), (dict(decay=float("inf")), "decay"),
    (dict(q=0), "rows"), (dict(q=P + 4), "rows"), (dict(q_stride=120), "rows"), (dict(lse=0), "NULL"), (dict(w=0), "NULL"),
    (dict(seqs=0), "NULL"), (dict(w_stride=255), "w_stride"), (dict(ws=0), "workspace"), (dict(ws=P + 8), "workspace"),
    (dict(ws_bytes=10), "workspace")])
def test_key_weight_refusals(xb, kw, msg):
    d = desc(xb)
    a = dict(layer=0, n_branches=2, seqs=P, n_q=1, n_heads=2, q=P, q_stride=128, lse=P, shared_len=0, causal=1, scale=0.0, decay=1.0,
             w=P, w_stride=256, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    st = xb.LIB.xc_op_key_weights(ctypes.addressof(d), a["layer"], a["n_branches"], a["seqs"], a["n_q"], a["n_heads"], a["q"],
                                  a["q_stride"], a["lse"], a["shared_len"], a["causal"], a["scale"], a["decay"], a["w"],
                                  a["w_stride"], a["ws"], a["ws_bytes"], None)
    assert st == xb.XC_EINVAL
    assert msg in xb.last_error(None), xb.last_error(None)


def test_key_weights_of_nothing_and_of_bad_caches(xb):
    d = desc(xb)
    assert xb.LIB.xc_op_key_weights(ctypes.addressof(d), 0, 0, None, 1, 2, None, 0, None, 0, 1, 0.0, 1.0, None, 0, None, 0, None) == 0
    assert xb.LIB.xc_op_key_weights_workspace_bytes(None, 1, 1, 2, 0) == 0
    for kw in (dict(head_dim=32), dict(page_size=24), dict(k=0)):
        bad = desc(xb, **kw)
        st = xb.LIB.xc_op_key_weights(ctypes.addressof(bad), 0, 1, P, 1, 2, P, 128, P, 0, 1, 0.0, 1.0, P, 256, P, 1 << 30, None)
        assert st == xb.XC_EINVAL


# --------------------------------------------------------------- eviction
@pytest.mark.parametrize("kw,msg", [
    (dict(n=-1), "max_seqs"), (dict(n=5), "max_seqs"), (dict(keep=0), "keep"), (dict(keep=257), "keep"), (dict(first=-1), "n_first"),
    (dict(last=-1), "n_first"), (dict(first=30, last=11), "n_first"), (dict(first=1 << 30, last=1 << 30), "n_first"),
    (dict(w=0), "without weights"), (dict(w_stride=255), "w_stride"), (dict(seqs=0), "seqs"), (dict(ws=0), "workspace"),
    (dict(ws=P + 8), "workspace"), (dict(ws_bytes=10), "workspace")])
def test_eviction_refusals(xb, kw, msg):
    d = desc(xb)
    a = dict(n=2, seqs=P, keep=40, first=2, last=3, w=P, w_stride=256, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    st = xb.LIB.xc_op_kv_evict(ctypes.addressof(d), a["n"], a["seqs"], a["keep"], a["first"], a["last"], a["w"], a["w_stride"],
                               None, a["ws"], a["ws_bytes"], None)
    assert st == xb.XC_EINVAL
    assert msg in xb.last_error(None), xb.last_error(None)


def test_eviction_of_nothing_and_from_bad_caches(xb):
    d = desc(xb)
    assert xb.LIB.xc_op_kv_evict(ctypes.addressof(d), 0, None, 40, 0, 0, P, 256, None, None, 0, None) == xb.XC_OK
    assert xb.LIB.xc_op_kv_evict_workspace_bytes(ctypes.addressof(d), 0, 40) == 0
    assert xb.LIB.xc_op_kv_evict_workspace_bytes(None, 1, 40) == 0
    for kw in (dict(page_size=24), dict(k=0), dict(table=0)):
        bad = desc(xb, **kw)
        assert xb.LIB.xc_op_kv_evict(ctypes.addressof(bad), 1, P, 40, 0, 0, P, 256, None, P, 1 << 30, None) == xb.XC_EINVAL
