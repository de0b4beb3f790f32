"""Host-side argument checks of the paged-cache operators: every refusal comes
before any CUDA call, so no GPU is needed."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2604_20289_gb300", "libxcache.so")
P = 1 << 20          # a 16-byte aligned address that is never read


@pytest.fixture(scope="module")
def xb():
    if not os.path.exists(LIB):
        from paper_2604_20289_gb300 import build
        build.build()
    from paper_2604_20289_gb300 import xcache
    return xcache


def desc(xb, **kw):
    f = dict(dtype=xb.XC_BF16, n_layers=2, n_pages=64, page_size=16, n_kv_heads=2, head_dim=64, max_seqs=4,
             max_pages=16, k=P, v=P, ref=P, table=P, len=P)
    f.update(kw)
    return xb.KVCacheDesc(**f)


def addr(d):
    return ctypes.addressof(d) if d is not None else None


BAD_CACHE = [dict(dtype=2), dict(page_size=24), dict(page_size=8), dict(page_size=2048), dict(head_dim=48),
             dict(n_layers=0), dict(n_pages=0), dict(n_kv_heads=0), dict(max_seqs=0), dict(max_pages=0),
             dict(n_pages=1 << 28), dict(max_pages=1 << 27), dict(k=0), dict(v=0), dict(ref=0), dict(table=0),
             dict(len=0), dict(k=P + 2)]


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_bad_caches_are_refused_by_every_call(xb, kw):
    d = addr(desc(xb, **kw))
    keep = desc(xb, **kw)
    d = addr(keep)
    two = (ctypes.c_int * 1)(32)
    calls = [xb.LIB.xc_op_kv_fork(d, 1, P, P, P, 1 << 30, None), xb.LIB.xc_op_kv_extend(d, 1, P, 1, P, P, 1 << 30, None),
             xb.LIB.xc_op_kv_free(d, 1, P, None), xb.LIB.xc_op_kv_compact(d, P, P, 1 << 30, None),
             xb.LIB.xc_op_qk_norm_rope(d, 0, 1, 2, P, 128, P, 128, P, 128, P, P, 1e-6, 1, two, two, P, P, 0, P, P, 128, None),
             xb.LIB.xc_op_branch_attention(d, 0, 1, P, 1, 2, P, 128, 0, 1, 0.0, P, 128, P, 1 << 30, None)]
    assert calls == [xb.XC_EINVAL] * 6
    assert "cache" in xb.last_error(None)


def test_null_cache(xb):
    assert xb.LIB.xc_op_kv_workspace_bytes(None) == 0
    assert xb.LIB.xc_op_branch_attention_workspace_bytes(None, 1, 1, 2, 0) == 0
    assert xb.LIB.xc_op_kv_free(None, 1, P, None) == xb.XC_EINVAL


def attn(xb, d, **kw):
    a = dict(layer=0, n_branches=1, seqs=P, n_q=1, n_heads=2, q=P, q_stride=128, shared_len=0, causal=1, scale=0.0, o=P,
             o_stride=128, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return xb.LIB.xc_op_branch_attention(addr(d), a["layer"], a["n_branches"], a["seqs"], a["n_q"], a["n_heads"], a["q"],
                                         a["q_stride"], a["shared_len"], a["causal"], a["scale"], a["o"], a["o_stride"],
                                         a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,msg", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(n_heads=3), "n_heads"), (dict(n_heads=2 * 129), "n_heads"),
    (dict(n_branches=-1), "n_branches"), (dict(shared_len=8), "shared_len"), (dict(shared_len=-16), "shared_len"),
    (dict(shared_len=16 * 17), "shared_len"), (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(q=0), "rows"), (dict(q=P + 4), "rows"), (dict(q_stride=120), "rows"),
    (dict(o_stride=132), "rows"), (dict(o=0), "rows"), (dict(seqs=0), "seqs"), (dict(ws=0), "workspace"),
    (dict(ws_bytes=100), "workspace"), (dict(ws=P + 8), "workspace"), (dict(n_branches=1 << 15, n_q=1 << 16), "n_branches"),
    (dict(n_branches=1 << 20, n_q=1 << 10), "too many")])
def test_attention_refusals(xb, kw, msg):
    d = desc(xb)
    assert attn(xb, d, **kw) == xb.XC_EINVAL
    assert msg in xb.last_error(None), xb.last_error(None)


def test_attention_head_sizes(xb):
    d = desc(xb, head_dim=32)
    assert attn(xb, d, q_stride=64, o_stride=64) == xb.XC_EINVAL and "head_dim" in xb.last_error(None)
    d = desc(xb, dtype=xb.XC_F32)
    assert attn(xb, d, n_heads=2 * 65, q_stride=1 << 14, o_stride=1 << 14) == xb.XC_EINVAL


def test_nothing_to_do(xb):
    """Empty lists and zero lengths are no work and no error, whatever the other pointers."""
    d = desc(xb)
    assert attn(xb, d, n_branches=0, q=0, o=0, seqs=0, ws=0) == xb.XC_OK
    assert attn(xb, d, n_q=0) == xb.XC_OK
    p = addr(d)
    assert xb.LIB.xc_op_kv_fork(p, 0, None, None, None, 0, None) == xb.XC_OK
    assert xb.LIB.xc_op_kv_extend(p, 0, None, 5, None, None, 0, None) == xb.XC_OK
    assert xb.LIB.xc_op_kv_extend(p, 2, P, 0, None, None, 0, None) == xb.XC_OK
    assert xb.LIB.xc_op_kv_free(p, 0, None, None) == xb.XC_OK


def test_page_call_refusals(xb):
    d = desc(xb)
    p, big = addr(d), 1 << 30
    assert xb.LIB.xc_op_kv_workspace_bytes(p) > 0
    assert xb.LIB.xc_op_kv_fork(p, 5, P, P, P, big, None) == xb.XC_EINVAL          # more pairs than sequences
    assert xb.LIB.xc_op_kv_fork(p, 1, None, P, P, big, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_kv_fork(p, 1, P, P, P, 8, None) == xb.XC_EINVAL
    assert "workspace" in xb.last_error(None)
    wide = desc(xb, max_seqs=2000)
    assert xb.LIB.xc_op_kv_fork(addr(wide), 1025, P, P, P, big, None) == xb.XC_EINVAL and "1024" in xb.last_error(None)
    assert xb.LIB.xc_op_kv_extend(addr(wide), 1025, P, 1, P, P, big, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_kv_extend(p, 1, P, 16 * 16 + 1, P, P, big, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_kv_extend(p, 1, P, -1, P, P, big, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_kv_extend(p, 1, P, 1, None, P, big, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_kv_free(p, 1, None, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_kv_compact(p, None, P, big, None) == xb.XC_EINVAL


def norm(xb, d, pairs=(32,), n_pos=(10,), **kw):
    a = dict(layer=0, T=1, H=2, q=P, ql=128, k=P, kl=128, v=P, vl=128, gq=P, gk=P, eps=1e-6, pos=P, table=P, slots=P,
             out=P, ol=128)
    a.update(kw)
    n = len(pairs)
    return xb.LIB.xc_op_qk_norm_rope(addr(d), a["layer"], a["T"], a["H"], a["q"], a["ql"], a["k"], a["kl"], a["v"],
                                     a["vl"], a["gq"], a["gk"], a["eps"], n, (ctypes.c_int * n)(*pairs),
                                     (ctypes.c_int * n)(*n_pos), a["pos"], a["table"], 0, a["slots"], a["out"], a["ol"],
                                     None)


@pytest.mark.parametrize("kw,msg", [
    (dict(layer=2), "layer"), (dict(T=-1), "token"), (dict(H=3), "n_heads"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(pairs=(31,)), "axis_pairs"), (dict(pairs=(16, 8, 4, 2, 2), n_pos=(1,) * 5), "axes"),
    (dict(pairs=(32, 0), n_pos=(1, 1)), "axis"), (dict(n_pos=(0,)), "axis"), (dict(n_pos=(1 << 28,)), "table"),
    (dict(q=0), "rows"), (dict(kl=100), "rows"), (dict(vl=130), "rows"), (dict(out=P + 8), "rows"), (dict(gq=0), "pointer"),
    (dict(gk=P + 4), "pointer"), (dict(pos=0), "pointer"), (dict(table=P + 4), "pointer"), (dict(slots=0), "pointer")])
def test_norm_refusals(xb, kw, msg):
    assert norm(xb, desc(xb), **kw) == xb.XC_EINVAL
    assert msg in xb.last_error(None), xb.last_error(None)


def test_norm_of_no_tokens(xb):
    assert norm(xb, desc(xb), T=0, q=0, pos=0) == xb.XC_OK


def test_rotation_table_refusals(xb):
    one = (ctypes.c_int * 1)(32)
    assert xb.LIB.xc_op_rope_table(0, one, one, 1e4, P, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_rope_table(1, one, one, 0.0, P, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_rope_table(1, one, one, float("nan"), P, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_rope_table(1, one, one, 1e4, None, None) == xb.XC_EINVAL
    assert xb.LIB.xc_op_rope_table(1, None, one, 1e4, P, None) == xb.XC_EINVAL
