"""Memory of another GPU than the current one is refused before any launch.  No GPU is
needed: the tensors are stand-ins that say where they are, and the library is not called."""
import os

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32, I32, I8 = torch.bfloat16, torch.float32, torch.int32, torch.int8


class Tensor:
    """A contiguous CUDA tensor, as far as the argument checks look."""
    is_cuda = True

    def __init__(self, shape, dtype, device=0):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, device
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.at

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def stride(self, i=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]

    def data_ptr(self):
        return 1 << 20


@pytest.fixture()
def xb(monkeypatch):
    if not os.path.exists(os.path.join(ROOT, "paper_2604_20289_gb300", "libxcache.so")):
        from paper_2604_20289_gb300 import build
        build.build()
    from paper_2604_20289_gb300 import xcache

    class Lib:
        calls = []

        def __getattr__(self, name):
            if name.endswith("bytes"):
                return lambda *a: 64
            return lambda *a: self.calls.append(name) or 0

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(xcache, "LIB", Lib())
    Lib.calls.clear()
    xcache.calls = Lib.calls
    yield xcache
    del xcache.calls


def cache(xb, **at):
    """Pages of two sequences of up to 4 pages of 16 tokens, 2 key heads of 64."""
    at = {**dict(k=0, v=0, ref=0, table=0, len=0), **at}
    k, v = (Tensor((1, 8, 16, 128), BF16, at[n]) for n in "kv")
    return xb.KVCache("bf16", 2, 64, k, v, Tensor((8,), I32, at["ref"]), Tensor((2, 4), I32, at["table"]), Tensor((2,), I32, at["len"]))


def calls(xb):
    """name -> (call, its tensors)"""
    q, o, kv = ((2, 256), BF16), ((2, 256), BF16), ((2, 128), BF16)
    seqs, lse, w, ws = ((2,), I32), ((2, 4), F32), ((2, 64), F32), ((64,), torch.uint8)
    return dict(
        attention=(lambda c, t: xb.op_branch_attention(c, 0, t["seqs"], 1, t["q"], t["o"], lse=t["lse"], workspace=t["ws"], stream=7),
                   dict(seqs=seqs, q=q, o=o, lse=lse, ws=ws)),
        key_weights=(lambda c, t: xb.op_key_weights(c, 0, t["seqs"], 1, t["q"], t["lse"], t["w"], workspace=t["ws"], stream=7),
                     dict(seqs=seqs, q=q, lse=lse, w=w, ws=ws)),
        evict=(lambda c, t: xb.op_kv_evict(c, t["seqs"], 5, t["w"], kept=t["kept"], workspace=t["ws"], stream=7),
               dict(seqs=seqs, w=w, kept=((2, 5), I32), ws=ws)),
        fork=(lambda c, t: xb.op_kv_fork(c, t["src"], t["seqs"], workspace=t["ws"], stream=7), dict(src=seqs, seqs=seqs, ws=ws)),
        extend=(lambda c, t: xb.op_kv_extend(c, t["seqs"], 1, t["slots"], workspace=t["ws"], stream=7),
                dict(seqs=seqs, slots=((2, 1), I32), ws=ws)),
        free=(lambda c, t: xb.op_kv_free(c, t["seqs"], stream=7), dict(seqs=seqs)),
        compact=(lambda c, t: xb.op_kv_compact(c, t["n"], workspace=t["ws"], stream=7), dict(n=((1,), I32), ws=ws)),
        norm=(lambda c, t: xb.op_qk_norm_rope(c, 0, t["q"], t["k"], t["v"], t["gq"], t["gk"], t["pos"], [32], [9], t["table"],
                                              t["slots"], t["o"], stream=7),
              dict(q=q, k=kv, v=kv, gq=((64,), F32), gk=((64,), F32), pos=((2,), I32), table=((576,), F32), slots=((2,), I32), o=o)))


NAMES = ["attention", "key_weights", "evict", "fork", "extend", "free", "compact", "norm"]


@pytest.mark.parametrize("name", NAMES)
def test_calls_on_a_cache(xb, name):
    call, tensors = calls(xb)[name]
    c = cache(xb)
    call(c, {k: Tensor(*v) for k, v in tensors.items()})
    assert len(xb.calls) == 1                              # reached the library
    for other in tensors:
        with pytest.raises(ValueError):
            call(c, {k: Tensor(*v, device=int(k == other)) for k, v in tensors.items()})
    assert len(xb.calls) == 1


@pytest.mark.parametrize("name", NAMES)
def test_a_cache_that_is_not_on_the_current_device(xb, name, monkeypatch):
    call, tensors = calls(xb)[name]
    there = cache(xb, k=1, v=1, ref=1, table=1, len=1)
    with pytest.raises(ValueError):
        call(there, {k: Tensor(*v, device=1) for k, v in tensors.items()})
    assert not xb.calls


@pytest.mark.parametrize("part", ["k", "v", "ref", "table", "len"])
def test_a_cache_on_two_devices(xb, part):
    with pytest.raises(ValueError):
        cache(xb, **{part: 1})


def test_products(xb):
    shapes = dict(A=((40, 64), BF16), Wq=((32, 64), I8), w_scale=((32,), F32), bias=((32,), F32), out=((40, 32), BF16),
                  gate=((32,), F32), resid=((40, 32), BF16), workspace=((64,), torch.uint8))

    def call(**at):
        t = {k: Tensor(*v, device=at.get(k, 0)) for k, v in shapes.items()}
        xb.op_linear_i8("bf16", xb.XC_EPI_RESID_GATE, t.pop("A"), t.pop("Wq"), t.pop("w_scale"), t.pop("bias"), t.pop("out"),
                        stream=7, **t)

    call()
    assert xb.calls == ["xc_op_linear_i8"]
    for other in shapes:
        with pytest.raises(ValueError):
            call(**{other: 1})
    with pytest.raises(ValueError):
        call(**{k: 1 for k in shapes})                     # all of them on a device that is not current
    assert xb.calls == ["xc_op_linear_i8"]
