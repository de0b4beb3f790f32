"""Branched rollouts: several candidate futures from one history.

``BranchedLayers`` runs a stack of causal self-attention layers

    x <- x + W_o attn(rope(norm(W_q h)), cache) + b_o,   h = LN(x),

over a paged key / value cache (``xcache.KVCache``) in which the branches of a
rollout share the pages of their common history.  A planner that compares
candidate actions runs the history once, forks it once per candidate without
copying it, advances all candidates together -- the shared keys are read once
for the whole batch -- and drops the ones it does not follow.  All arithmetic
runs in the CUDA library; this module sequences calls and keeps, on the host,
the lengths and which pages sequences have in common, so that a call the pool
has no pages for is refused before anything changes.  Ids and positions are
uploaded from host lists in every call, so these calls cannot be captured into
a graph; the operators they make can.

``python -m paper_2604_20289_gb300.branches`` runs such a planning step on
random weights.
"""
from __future__ import annotations

import operator

import torch

from . import xcache as xb


class BranchedLayers:
    """weights: per layer a dict of CUDA tensors -- ``qkv_w`` [(H + 2 Hk) hd, d] and
    ``o_w`` [d, H hd] (K-major, the storage type), ``qkv_b``, ``o_b`` (float32),
    ``gamma_q``, ``gamma_k`` [hd] (float32).  A call runs on the stream that is
    current when it is made, after the object's earlier calls on whatever stream.
    ``cache`` is for reading: its sequences change through this object alone."""

    def __init__(self, weights, n_heads, n_kv_heads, head_dim, n_pages, page_size=64, max_seqs=64, max_len=4096,
                 dtype="bf16", theta=10000.0, eps=1e-6):
        self.weights, self.dtype, self.eps = weights, dtype, float(eps)
        self.H, self.Hk, self.hd = n_heads, n_kv_heads, head_dim
        self.d = weights[0]["o_w"].shape[0]
        self.max_len = max_len
        self.cache = xb.KVCache.empty(dtype, len(weights), n_pages, page_size, n_kv_heads, head_dim, max_seqs,
                                      -(-max_len // page_size))
        self.pairs, self.n_pos = [head_dim // 2], [max_len]
        self.rotation = torch.empty(2 * self.pairs[0] * max_len, device="cuda")
        xb.op_rope_table(self.pairs, self.n_pos, theta, self.rotation)
        self.zeros = torch.zeros(self.d, device="cuda")
        self.ones = torch.ones(self.d, device="cuda")
        self._check_weights()
        self._check_sizes()
        self._last = torch.cuda.current_stream()          # stream of the last call
        self._streams = {self._last.cuda_stream}          # streams that have used the tensors kept here
        self.length = [0] * max_seqs
        # The pages of a sequence: runs that it has in common with its forks, [pages, sequences that hold the run],
        # then pages of its own.
        self._runs = [[] for _ in range(max_seqs)]
        self._used = 0                                    # pages in use
        self._free = list(range(max_seqs - 1, -1, -1))

    def _check_weights(self):
        rows, dt = (self.H + 2 * self.Hk) * self.hd, self.cache.torch_dtype
        want = dict(qkv_w=((rows, self.d), dt), o_w=((self.d, self.H * self.hd), dt), qkv_b=((rows,), torch.float32),
                    o_b=((self.d,), torch.float32), gamma_q=((self.hd,), torch.float32),
                    gamma_k=((self.hd,), torch.float32))
        for layer, w in enumerate(self.weights):
            for name, (shape, dtype) in want.items():
                t = w[name]
                if t.shape != shape or t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
                    raise ValueError(f"layer {layer}: {name}: contiguous CUDA tensor {list(shape)} of {dtype} expected")

    def _check_sizes(self):
        """What the library refuses of these sizes, it refuses here: one row through the operators of a layer."""
        c, w, dt = self.cache, self.weights[0], self.cache.torch_dtype
        if xb.op_branch_attention_workspace_bytes(c, 1, 1, self.H) == 0:
            raise xb.XCacheError(xb.XC_EINVAL, xb.last_error())
        x, o = (torch.zeros(1, n, dtype=dt, device="cuda") for n in (self.d, self.H * self.hd))
        y, qkv = torch.empty_like(x), torch.empty(1, w["qkv_w"].shape[0], dtype=dt, device="cuda")
        xb.op_ln_mod(self.dtype, x, self.zeros, self.zeros, y, eps=self.eps)
        xb.op_linear(self.dtype, xb.XC_EPI_BIAS, y, w["qkv_w"], w["qkv_b"], qkv)
        dq, dk, none = o.shape[1], self.Hk * self.hd, self._ids([-1])      # slot -1: no keys are kept
        xb.op_qk_norm_rope(c, 0, qkv[:, :dq], qkv[:, dq:dq + dk], qkv[:, dq + dk:], w["gamma_q"], w["gamma_k"],
                           self._ids([0]), self.pairs, self.n_pos, self.rotation, none, o, eps=self.eps)
        xb.op_linear(self.dtype, xb.XC_EPI_RESID_GATE, o, w["o_w"], w["o_b"], y, gate=self.ones, resid=x)

    def _on_current_stream(self):
        """Orders the current stream after the object's earlier calls.  Every method that
        launches work begins with it: its temporaries and its launches are then of one stream."""
        st = torch.cuda.current_stream()
        if st != self._last:
            st.wait_stream(self._last)
            self._last = st
        if st.cuda_stream not in self._streams:           # memory kept here is not reused under work of this stream
            self._streams.add(st.cuda_stream)
            c = self.cache
            for t in (c.k, c.v, c.ref, c.table, c.len, self.rotation, self.zeros, self.ones,
                      *(t for w in self.weights for t in w.values())):
                t.record_stream(st)

    def _ids(self, seqs):
        return torch.tensor(list(seqs), dtype=torch.int32, device="cuda")

    def _take(self, n):
        if n > len(self._free):
            raise ValueError(f"{n} sequences asked for, {len(self._free)} free")
        return [self._free.pop() for _ in range(n)]

    def _n_pages(self, length):
        return -(-length // self.cache.page_size)

    def _own_pages(self, s):
        return self._n_pages(self.length[s]) - sum(pages for pages, _ in self._runs[s])

    def _room(self, pages):
        free = self.cache.ref.numel() - self._used
        if pages > free:
            raise ValueError(f"{pages} pages asked for, {free} free")

    def _in_use(self, seqs, once=True):
        """The sequences as a list of ints, each handed out and (once) listed once."""
        ids = [operator.index(s) for s in seqs]
        idle = set(self._free)
        for s in ids:
            if not 0 <= s < len(self.length) or s in idle:
                raise ValueError(f"sequence {s} is not in use")
        if once and len(set(ids)) != len(ids):
            raise ValueError("a sequence is listed twice")
        return ids

    def new(self) -> int:
        """An empty sequence."""
        return self._take(1)[0]

    def fork(self, seq: int, n: int) -> list:
        """n sequences that continue ``seq``; full pages are shared, not copied."""
        seq, = self._in_use([seq])
        part = self.length[seq] % self.cache.page_size != 0
        self._room(n if part else 0)
        ids = self._take(n)
        self._on_current_stream()
        try:
            xb.op_kv_fork(self.cache, self._ids([seq] * n), self._ids(ids))
        except Exception:                                 # nothing was launched
            self._free += reversed(ids)
            raise
        full = self._own_pages(seq) - part                # pages of its own that it shares from now on
        if ids and full > 0:
            self._runs[seq].append([full, 1])
        for run in self._runs[seq]:
            run[1] += len(ids)
        for i in ids:
            self.length[i], self._runs[i] = self.length[seq], list(self._runs[seq])
        self._used += len(ids) if part else 0
        return ids

    def free(self, seqs):
        seqs = self._in_use(seqs)
        self._on_current_stream()
        xb.op_kv_free(self.cache, self._ids(seqs))
        for s in seqs:
            self._used -= self._own_pages(s)
            for run in self._runs[s]:
                run[1] -= 1
                self._used -= run[0] if run[1] == 0 else 0
            self.length[s], self._runs[s] = 0, []
            self._free.append(s)

    def compact(self) -> torch.Tensor:
        """Moves the pages in use to the front of the pool; returns their count (on the device)."""
        self._on_current_stream()
        live = torch.empty(1, dtype=torch.int32, device="cuda")
        xb.op_kv_compact(self.cache, live)
        return live

    def shared_len(self, seqs) -> int:
        """Tokens whose pages all of these sequences have in common."""
        seqs = self._in_use(seqs, once=False)
        if len(set(seqs)) == 1:
            return self.length[seqs[0]] // self.cache.page_size * self.cache.page_size
        pages = 0
        for runs in zip(*(self._runs[s] for s in seqs)):
            if any(run is not runs[0] for run in runs):
                break
            pages += runs[0][0]
        return pages * self.cache.page_size

    def step(self, seqs, x):
        """Appends x [len(seqs), n, d] to the sequences and returns the layers' output
        of the new tokens (same shape).  Every new token sees its sequence up to itself."""
        seqs = self._in_use(seqs)
        if x.dim() != 3 or x.shape[0] != len(seqs) or x.shape[2] != self.d or not x.is_cuda:
            raise ValueError(f"x: CUDA tensor [{len(seqs)}, n, {self.d}] expected")
        B, n, d = x.shape
        if n == 0 or B == 0:
            return x
        if any(self.length[s] + n > self.max_len for s in seqs):
            raise ValueError(f"sequences hold at most {self.max_len} tokens")
        new_pages = sum(self._n_pages(self.length[s] + n) - self._n_pages(self.length[s]) for s in seqs)
        self._room(new_pages)
        self._on_current_stream()
        c, st, T = self.cache, self._last.cuda_stream, B * n
        dt = c.k.dtype
        dq, dk = self.H * self.hd, self.Hk * self.hd
        # What can fail for want of memory comes before the extension, which the host's lengths follow.  (No page
        # that the new tokens go to is shared, so the shared part is the same before and after.)
        shared = self.shared_len(seqs) if B > 1 else 0
        ids = self._ids(seqs)
        slots = torch.empty(B, n, dtype=torch.int32, device="cuda")
        pos = torch.tensor([[self.length[s] + i] for s in seqs for i in range(n)], dtype=torch.int32, device="cuda")
        x = x.reshape(T, d).to(dt).contiguous()
        h, out = torch.empty_like(x), [torch.empty_like(x) for _ in self.weights[:2]]
        qkv = torch.empty(T, dq + 2 * dk, dtype=dt, device="cuda")
        q = torch.empty(T, dq, dtype=dt, device="cuda")
        o = torch.empty_like(q)
        need = xb.op_branch_attention_workspace_bytes(c, B, n, self.H, shared)
        if need == 0:                                     # more rows than the attention takes
            raise xb.XCacheError(xb.XC_EINVAL, xb.last_error())
        c.workspace(need, st)
        xb.op_kv_extend(c, ids, n, slots, stream=st)
        self._used += new_pages
        for s in seqs:
            self.length[s] += n
        for layer, w in enumerate(self.weights):
            xb.op_ln_mod(self.dtype, x, self.zeros, self.zeros, h, eps=self.eps, stream=st)
            xb.op_linear(self.dtype, xb.XC_EPI_BIAS, h, w["qkv_w"], w["qkv_b"], qkv, stream=st)
            xb.op_qk_norm_rope(c, layer, qkv[:, :dq], qkv[:, dq:dq + dk], qkv[:, dq + dk:], w["gamma_q"], w["gamma_k"],
                               pos, self.pairs, self.n_pos, self.rotation, slots.view(-1), q, eps=self.eps, stream=st)
            xb.op_branch_attention(c, layer, ids, n, q, o, shared_len=shared, causal=True, stream=st)
            y = out[layer % 2]
            xb.op_linear(self.dtype, xb.XC_EPI_RESID_GATE, o, w["o_w"], w["o_b"], y, gate=self.ones, resid=x, stream=st)
            x = y
        return x.view(B, n, d)


def random_layers(n_layers, d, n_heads, n_kv_heads, head_dim, dtype="bf16", seed=0):
    """Random weights of the shapes BranchedLayers takes."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows = (n_heads + 2 * n_kv_heads) * head_dim

    def r(*shape, std=1.0):
        return std * torch.randn(*shape, generator=g, device="cuda")

    return [dict(qkv_w=r(rows, d, std=d ** -0.5).to(dt), qkv_b=r(rows, std=0.05),
                 o_w=r(d, n_heads * head_dim, std=(n_heads * head_dim) ** -0.5).to(dt), o_b=r(d, std=0.05),
                 gamma_q=1.0 + 0.1 * r(head_dim), gamma_k=1.0 + 0.1 * r(head_dim)) for _ in range(n_layers)]


def main():
    d, H, Hk, hd, candidates = 512, 8, 8, 64, 6
    m = BranchedLayers(random_layers(4, d, H, Hk, hd), H, Hk, hd, n_pages=256, page_size=64, max_seqs=16, max_len=8192)
    g = torch.Generator(device="cuda").manual_seed(1)
    history = m.new()
    m.step([history], torch.randn(1, 2016, d, generator=g, device="cuda"))
    kids = m.fork(history, candidates)
    pages = int((m.cache.ref > 0).sum())
    first = torch.randn(candidates, 1, d, generator=g, device="cuda")
    x = first
    for _ in range(8):                                    # one token at a time, all candidates together
        x = m.step(kids, x)
    score = x.float().square().mean(dim=(1, 2))
    best = int(score.argmin())
    m.free([k for i, k in enumerate(kids) if i != best] + [history])
    live = int(m.compact())
    xb.check(xb.XC_OK if xb.op_device_error() == 0 else xb.XC_ECUDA)
    print(f"history 2016 tokens, {candidates} candidates on {pages} pages (shared {m.shared_len(kids[best:best + 1])} "
          f"tokens); kept candidate {best}: {m.length[kids[best]]} tokens on {live} pages")


if __name__ == "__main__":
    main()
