"""Eviction from the paged cache by the weight of its tokens, against a plain
model on the host.  Copies and whole numbers: everything is compared exactly."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402
from test_gpu_branch import DEV, i32, make_cache  # noqa: E402


def bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32).cpu().numpy().copy()


def picked(w, length, keep, first, last):
    """Tokens that stay, by sorting."""
    if length <= keep:
        return list(range(length))
    key = np.where(np.isnan(w), -np.inf, w + 0.0)
    nan = np.isnan(w)
    mid = sorted(range(first, length - last), key=lambda t: (-key[t], nan[t], t))
    return sorted(list(range(first)) + list(range(length - last, length)) + mid[:keep - first - last])


class Model:
    def __init__(self, cache, w):
        self.c = cache
        self.k, self.v = bits(cache.k), bits(cache.v)
        self.ref, self.table, self.len = (t.cpu().numpy().copy() for t in (cache.ref, cache.table, cache.len))
        self.w = w.cpu().numpy().copy() if w is not None else None
        self.ps = cache.page_size

    def evict(self, seqs, keep, first, last):
        """(kept, whether it went through)"""
        ps = self.ps
        idx = [picked(self.w[s] if self.w is not None else None, self.len[s], keep, first, last)
               if self.w is not None or self.len[s] <= keep
               else list(range(first)) + list(range(self.len[s] - last, self.len[s])) for s in seqs]
        free = [p for p in range(len(self.ref)) if self.ref[p] == 0]
        plan, before = [], self.ref.copy()
        for s, ix in zip(seqs, idx):
            new = []
            if self.len[s] > keep:
                for p in range(-(-keep // ps)):
                    end = min((p + 1) * ps, keep)
                    other = ix[end - 1] != end - 1 or (p + 1) * ps > keep
                    fresh = other and before[self.table[s, p]] > 1
                    if fresh and not free:
                        return np.full((len(seqs), keep), -1), False
                    new.append(free.pop(0) if fresh else self.table[s, p])
            plan.append(new)
        k, v = self.k.copy(), self.v.copy()
        for s, ix, new in zip(seqs, idx, plan):
            if self.len[s] <= keep:
                continue
            old = self.table[s].copy()
            a, i = np.array(ix), np.arange(keep)
            new = np.array(new)
            # rows of pages that stay as they are keep what lies behind the sequence; replaced ones take theirs along
            k[:, new[i // ps], i % ps] = self.k[:, old[a // ps], a % ps]
            v[:, new[i // ps], i % ps] = self.v[:, old[a // ps], a % ps]
            n_old = -(-self.len[s] // ps)
            for p in range(n_old):
                if p >= len(new) or new[p] != old[p]:
                    self.ref[old[p]] -= 1
            for p, n in enumerate(new):
                if n != old[p]:
                    self.ref[n] += 1
            self.table[s, :] = -1
            self.table[s, :len(new)] = new
            if self.w is not None:
                self.w[s, :keep] = self.w[s][a]
                self.w[s, keep:self.len[s]] = 0
            self.len[s] = keep
        self.k, self.v = k, v
        kept = np.full((len(seqs), keep), -1)
        for b, ix in enumerate(idx):
            kept[b, :len(ix)] = ix
        return kept, True


def compare(cache, w, m, replaced_rows_matter=True):
    assert np.array_equal(cache.ref.cpu().numpy(), m.ref)
    assert np.array_equal(cache.table.cpu().numpy(), m.table)
    assert np.array_equal(cache.len.cpu().numpy(), m.len)
    if w is not None:
        assert np.array_equal(bits(w), m.w.view(np.int32))
    assert np.array_equal(bits(cache.k), m.k) and np.array_equal(bits(cache.v), m.v)


def weights(cache, kind="skewed", seed=0, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, width = cache.table.shape[0], cache.table.shape[1] * cache.page_size + extra
    w = torch.randn(n, width, generator=g, device=DEV)
    if kind == "skewed":
        w = torch.exp(2 * w)
    elif kind == "ties":
        w = torch.round(torch.exp(w) * 2)
    elif kind == "equal":
        w = torch.ones_like(w)
    elif kind == "odd":
        r = torch.randint(0, 8, w.shape, generator=g, device=DEV)
        for i, x in enumerate((float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45)):
            w[r == i] = x
    return w


def check(lens, keep, first, last, kind="skewed", dtype="bf16", hk=2, hd=64, ps=16, shared=0, layers=2, seqs=None, w_none=False,
          seed=3, kept=True):
    cache = make_cache(dtype, hk, hd, ps, lens, shared, layers=layers, seed=seed, dead=7.0)
    # room for the shared pages that are replaced
    more = len(lens) * (min(shared, keep) // ps + 1)
    cache = grown(cache, more)
    w = None if w_none else weights(cache, kind, seed, extra=5)
    seqs = list(range(len(lens))) if seqs is None else seqs
    m = Model(cache, w)
    want, ok = m.evict(seqs, keep, first, last)
    assert ok
    out = torch.full((len(seqs), keep), -7, dtype=torch.int32, device=DEV) if kept else None
    xb.op_kv_evict(cache, i32(seqs), keep, w, first, last, kept=out)
    assert xb.op_device_error() == 0
    if kept:
        assert np.array_equal(out.cpu().numpy(), want)
    compare(cache, w, m)
    return cache, w


def grown(cache, more):
    """The cache with `more` free pages behind its own."""
    def wide(t, dim, fill):
        shape = list(t.shape)
        shape[dim] = more
        return torch.cat([t, torch.full(shape, fill, dtype=t.dtype, device=DEV)], dim=dim).contiguous()
    return xb.KVCache(cache.dtype, cache.n_kv_heads, cache.head_dim, wide(cache.k, 1, 5.0), wide(cache.v, 1, 5.0),
                      wide(cache.ref, 0, 0), cache.table, cache.len)


@pytest.mark.parametrize("kind", ["skewed", "ties", "equal", "odd"])
@pytest.mark.parametrize("lens,keep,first,last", [
    ([2], 1, 0, 0), ([2], 1, 1, 0), ([2], 1, 0, 1), ([17, 33, 5, 0, 16], 16, 2, 5), ([100], 99, 0, 0), ([100], 99, 98, 0),
    ([64, 65, 63], 64, 0, 0), ([200, 150, 333], 37, 4, 16), ([200, 150, 333], 48, 0, 48), ([200, 150, 333], 48, 48, 0),
    ([1031, 1063, 1040], 1024, 16, 128), ([700] * 9, 500, 0, 10)])
def test_small(lens, keep, first, last, kind):
    check(lens, keep, first, last, kind)


@pytest.mark.parametrize("dtype,hk,hd,ps,layers", [("bf16", 1, 16, 16, 1), ("f32", 1, 16, 32, 3), ("bf16", 3, 32, 64, 1), ("f32", 5, 128, 128, 2),
                                                   ("bf16", 12, 128, 1024, 2), ("bf16", 33, 64, 16, 1), ("f32", 40, 128, 16, 1)])
def test_layouts(dtype, hk, hd, ps, layers):
    check([1500, 90, 700], 77, 3, 20, dtype=dtype, hk=hk, hd=hd, ps=ps, layers=layers)
    check([1500, 2100, 1200], 1111, 3, 20, dtype=dtype, hk=hk, hd=hd, ps=ps, layers=layers)


@pytest.mark.parametrize("kind", ["skewed", "ties", "equal", "odd"])
@pytest.mark.parametrize("length,keep,first,last", [(9000, 5000, 0, 0), (9000, 100, 10, 30), (40000, 39000, 64, 512), (40000, 1, 0, 0),
                                                   (300000, 150000, 4, 100)])
def test_long(length, keep, first, last, kind):
    check([length, length - 7], keep, first, last, kind, hk=1, hd=16, ps=128, layers=1)


@pytest.mark.parametrize("shared,lens,keep,first,last", [
    (96, [200, 150, 97], 64, 4, 8),                    # every branch gets pages of its own
    (96, [200, 150, 97], 96, 96, 0),                   # the shared part stays as it is, whole pages
    (96, [200, 150, 97], 40, 40, 0),                   # and ends inside a shared page
    (96, [200, 150, 97], 100, 96, 2),                  # the first own page changes
    (96, [200, 150, 97], 97, 90, 2), (512, [600] * 20, 300, 0, 64)])
@pytest.mark.parametrize("seqs", [None, "some"])
def test_shared_pages(shared, lens, keep, first, last, seqs):
    seqs = None if seqs is None else [len(lens) - 1, 0]
    check(lens, keep, first, last, shared=shared, seqs=seqs)


def test_a_page_whose_last_other_holder_is_evicted_in_the_same_call():
    check([200, 200], 64, 4, 8, shared=128, seqs=[1, 0])


@pytest.mark.parametrize("first,last", [(0, 40), (40, 0), (4, 36)])
def test_without_weights(first, last):
    check([200, 30, 90], 40, first, last, w_none=True)
    check([200, 30, 90], 40, first, last, w_none=True, kept=False)


def test_without_kept():
    check([200, 30, 90], 40, 1, 7, kept=False)


def test_a_full_pool_is_enough_for_a_sequence_of_its_own():
    cache = make_cache("bf16", 2, 64, 16, [200, 100], 0, layers=2, dead=7.0)
    full = xb.KVCache("bf16", 2, 64, cache.k, cache.v, cache.ref, cache.table, cache.len)
    cache.ref[cache.ref == 0] = 1                      # pages that others hold
    w = weights(full)
    m = Model(full, w)
    want, ok = m.evict([0, 1], 50, 3, 9)
    kept = torch.empty(2, 50, dtype=torch.int32, device=DEV)
    xb.op_kv_evict(full, i32([0, 1]), 50, w, 3, 9, kept=kept)
    assert ok and xb.op_device_error() == 0 and np.array_equal(kept.cpu().numpy(), want)
    compare(full, w, m)


def refused(cache, w, seqs, keep, first, last, flag):
    m = Model(cache, w)
    kept = torch.full((len(seqs), keep), -7, dtype=torch.int32, device=DEV)
    xb.op_kv_evict(cache, i32(seqs), keep, w, first, last, kept=kept)
    assert xb.op_device_error() == flag
    assert (kept == -1).all()
    compare(cache, w, m)


def test_a_pool_without_room_for_shared_pages_changes_nothing():
    cache = make_cache("bf16", 2, 64, 16, [200, 150], 96, layers=1, dead=7.0)      # two free pages, twelve needed
    refused(cache, weights(cache), [0, 1], 96, 0, 8, xb.XC_DEV_CACHE_FULL)


@pytest.mark.parametrize("seqs", [[0, 0], [0, 1, 0], [-1], [2], [1, 1 << 30], [0, 2]])
def test_bad_lists_change_nothing(seqs):
    cache = make_cache("bf16", 2, 64, 16, [200, 150], 0, layers=1, dead=7.0)
    if len(seqs) > 2:
        cache = make_cache("bf16", 2, 64, 16, [200, 150, 40], 0, layers=1, dead=7.0)
    if 2 in seqs:
        cache.table[1, 3] = 1 << 20                    # a page out of range
        seqs = [1 if s == 2 else s for s in seqs]
    refused(cache, weights(cache), seqs, 40, 4, 8, xb.XC_DEV_BAD_SEQUENCE)


def test_a_bad_length_changes_nothing():
    cache = make_cache("bf16", 2, 64, 16, [200, 150], 0, layers=1, dead=7.0)
    for bad in (-1, cache.table.shape[1] * 16 + 1):
        cache.len[1] = bad
        refused(cache, weights(cache), [0, 1], 40, 4, 8, xb.XC_DEV_BAD_SEQUENCE)


def test_a_thousand_sequences():
    check([30 + (37 * b) % 60 for b in range(1000)], 40, 2, 8, "ties", layers=1)


def test_captured_evictions():
    """A loop of extend and evict in one graph: the sequence stays at its bound."""
    cache = grown(make_cache("bf16", 2, 64, 16, [64], 0, layers=1, max_pages=8, dead=0.0), 8)
    w = torch.zeros(1, 8 * 16, device=DEV)
    w[0, :64] = torch.arange(64, device=DEV) % 7
    seqs, slots = i32([0]), torch.empty(1, 20, dtype=torch.int32, device=DEV)
    kept = torch.empty(1, 64, dtype=torch.int32, device=DEV)

    def step():
        xb.op_kv_extend(cache, seqs, 20, slots)
        xb.op_kv_evict(cache, seqs, 64, w, 4, 16, kept=kept)

    step()
    assert xb.op_device_error() == 0
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(5):
        before = w.cpu().numpy().copy()
        g.replay()
        torch.cuda.synchronize()
        assert kept[0].tolist() == picked(before[0], 84, 64, 4, 16)
        assert cache.len.tolist() == [64] and int((cache.ref > 0).sum()) == 4
    assert xb.op_device_error() == 0


def test_refusals():
    cache = make_cache("bf16", 2, 64, 16, [200, 150], 0)
    w = weights(cache)
    for bad in (dict(weights=w[:1]), dict(weights=w[:, :50]), dict(weights=w.double()), dict(kept=torch.empty(2, 39, dtype=torch.int32, device=DEV)),
                dict(kept=torch.empty(2, 40, device=DEV)), dict(seqs=i32([0, 1]).long())):
        a = dict(seqs=i32([0, 1]), keep=40, weights=w)
        a.update(bad)
        with pytest.raises(ValueError):
            xb.op_kv_evict(cache, **a)
    for bad in (dict(keep=0), dict(keep=-3), dict(keep=cache.table.shape[1] * 16 + 1), dict(n_first=-1), dict(n_last=-1),
                dict(n_first=30, n_last=11), dict(weights=None), dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        a = dict(keep=40, weights=w)
        a.update(bad)
        with pytest.raises(xb.XCacheError):
            xb.op_kv_evict(cache, i32([0, 1]), **a)
