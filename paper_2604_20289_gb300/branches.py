"""Branched rollouts: several candidate futures from one history.

``BranchedLayers`` runs a stack of causal self-attention layers

    x <- x + W_o attn(rope(norm(W_q h)), cache) + b_o,   h = LN(x),

over a paged key / value cache (``xcache.KVCache``) in which the branches of a
rollout share the pages of their common history.  A planner that compares
candidate actions runs the history once, forks it once per candidate without
copying it, advances all candidates together -- the shared keys are read once
for the whole batch -- and drops the ones it does not follow.  A rollout that goes
on for longer than its memory lasts keeps count of the weight that attention gives
to each token (``track``) and drops the tokens that get least of it (``evict``).
The projections' weights are of the storage type or 8-bit integers
(``quantize_layers``).  All arithmetic runs in the CUDA library; this module sequences calls and keeps, on the host,
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
    ``o_w`` [d, H hd] (K-major, the storage type, or int8 with their rows' ``qkv_s``, ``o_s``, float32),
    ``qkv_b``, ``o_b`` (float32), ``gamma_q``, ``gamma_k`` [hd] (float32).  A sequence holds at most
    max_len tokens at a time, at positions below max_pos (max_len).  track: None, or the factor (0 to 1) by
    which a sequence's ``key_weights`` shrink with each of its steps, before that step's
    weights, of all layers, heads and new tokens, are added.  A call runs on the stream that is
    current when it is made, after the object's earlier calls on whatever stream; the device that was
    current when the object was made is current in every call.
    ``cache`` is for reading: its sequences change through this object alone."""

    def __init__(self, weights, n_heads, n_kv_heads, head_dim, n_pages, page_size=64, max_seqs=64, max_len=4096,
                 dtype="bf16", theta=10000.0, eps=1e-6, max_pos=None, track=None):
        self.weights, self.dtype, self.eps = weights, dtype, float(eps)
        self.H, self.Hk, self.hd = n_heads, n_kv_heads, head_dim
        self.d = weights[0]["o_w"].shape[0]
        self.max_len, self.max_pos = max_len, max_len if max_pos is None else max_pos
        if track is not None and not 0.0 <= track <= 1.0:
            raise ValueError("track: None or a factor from 0 to 1 expected")
        self.track = track
        self.cache = xb.KVCache.empty(dtype, len(weights), n_pages, page_size, n_kv_heads, head_dim, max_seqs,
                                      -(-max_len // page_size))
        self.pairs, self.n_pos = [head_dim // 2], [self.max_pos]
        self.rotation = torch.empty(2 * self.pairs[0] * self.max_pos, device="cuda")
        xb.op_rope_table(self.pairs, self.n_pos, theta, self.rotation)
        self.zeros = torch.zeros(self.d, device="cuda")
        self.ones = torch.ones(self.d, device="cuda")
        self.key_weights = None                           # [sequence][token], 0 past a sequence's end
        if track is not None:
            self.key_weights = torch.zeros(max_seqs, self.cache.table.shape[1] * page_size, device="cuda")
        self._check_weights()
        self._check_sizes()
        self._last = torch.cuda.current_stream()          # stream of the last call
        self._streams = {self._last.cuda_stream}          # streams that have used the tensors kept here
        self.length = [0] * max_seqs
        self.position = [0] * max_seqs                    # of the next token: tokens seen so far
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
            here = dict(want)
            for name, n in (("qkv", rows), ("o", self.d)):
                if w[name + "_w"].dtype is torch.int8:
                    here[name + "_w"] = (want[name + "_w"][0], torch.int8)
                    here[name + "_s"] = ((n,), torch.float32)
            for name, (shape, dtype) in here.items():
                t = w[name]
                if t.shape != shape or t.dtype != dtype or t.get_device() != self.cache.device or not t.is_contiguous():
                    raise ValueError(f"layer {layer}: {name}: contiguous CUDA tensor {list(shape)} of {dtype} on the "
                                     "current device expected")
                if dtype is torch.int8 and t.data_ptr() % 16 != 0:
                    raise ValueError(f"layer {layer}: {name}: 16-byte aligned memory expected")

    def _linear(self, epilogue, x, w, name, out, workspace=None, resid=None, stream=None):
        gate = None if resid is None else self.ones
        if w[name + "_w"].dtype is torch.int8:
            xb.op_linear_i8(self.dtype, epilogue, x, w[name + "_w"], w[name + "_s"], w[name + "_b"], out, gate=gate,
                            resid=resid, workspace=workspace, stream=stream)
        else:
            xb.op_linear(self.dtype, epilogue, x, w[name + "_w"], w[name + "_b"], out, gate=gate, resid=resid,
                         stream=stream)

    def _check_sizes(self):
        """What the library refuses of these sizes, it refuses here: one row through the operators of a layer."""
        c, w, dt = self.cache, self.weights[0], self.cache.torch_dtype
        if xb.op_branch_attention_workspace_bytes(c, 1, 1, self.H) == 0 or \
                (self.track is not None and xb.op_key_weights_workspace_bytes(c, 1, 1, self.H) == 0):
            raise xb.XCacheError(xb.XC_EINVAL, xb.last_error())
        x, o = (torch.zeros(1, n, dtype=dt, device="cuda") for n in (self.d, self.H * self.hd))
        y, qkv = torch.empty_like(x), torch.empty(1, w["qkv_w"].shape[0], dtype=dt, device="cuda")
        xb.op_ln_mod(self.dtype, x, self.zeros, self.zeros, y, eps=self.eps)
        for each in {v["qkv_w"].dtype: v for v in self.weights}.values():  # a layer of either kind
            self._linear(xb.XC_EPI_BIAS, y, each, "qkv", qkv)
        dq, dk, none = o.shape[1], self.Hk * self.hd, self._ids([-1])      # slot -1: no keys are kept
        xb.op_qk_norm_rope(c, 0, qkv[:, :dq], qkv[:, dq:dq + dk], qkv[:, dq + dk:], w["gamma_q"], w["gamma_k"],
                           self._ids([0]), self.pairs, self.n_pos, self.rotation, none, o, eps=self.eps)
        for each in {v["o_w"].dtype: v for v in self.weights}.values():
            self._linear(xb.XC_EPI_RESID_GATE, o, each, "o", y, resid=x)

    def _on_current_stream(self):
        """Orders the current stream after the object's earlier calls.  Every method that
        launches work begins with it: its temporaries and its launches are then of one stream."""
        if torch.cuda.current_device() != self.cache.device:
            raise ValueError(f"CUDA device {self.cache.device}, which holds the cache, is not the current one")
        st = torch.cuda.current_stream()
        if st != self._last:
            st.wait_stream(self._last)
            self._last = st
        if st.cuda_stream not in self._streams:           # memory kept here is not reused under work of this stream
            self._streams.add(st.cuda_stream)
            c = self.cache
            for t in (c.k, c.v, c.ref, c.table, c.len, self.rotation, self.zeros, self.ones,
                      *(() if self.key_weights is None else (self.key_weights,)),
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
        self._on_current_stream()
        ids = self._take(n)
        try:
            to = self._ids(ids)
            rows = to.long()
            copies = self.key_weights[seq].repeat(n, 1) if self.key_weights is not None else None
            xb.op_kv_fork(self.cache, self._ids([seq] * n), to)
        except Exception:                                 # nothing was launched
            self._free += reversed(ids)
            raise
        if copies is not None:
            self.key_weights.index_copy_(0, rows, copies)
        full = self._own_pages(seq) - part                # pages of its own that it shares from now on
        if ids and full > 0:
            self._runs[seq].append([full, 1])
        for run in self._runs[seq]:
            run[1] += len(ids)
        for i in ids:
            self.length[i], self.position[i], self._runs[i] = self.length[seq], self.position[seq], list(self._runs[seq])
        self._used += len(ids) if part else 0
        return ids

    def free(self, seqs):
        seqs = self._in_use(seqs)
        self._on_current_stream()
        ids = self._ids(seqs)
        rows = ids.long() if self.key_weights is not None else None
        xb.op_kv_free(self.cache, ids)
        if rows is not None:
            self.key_weights.index_fill_(0, rows, 0.0)
        for s in seqs:
            self._used -= self._own_pages(s)
            for run in self._runs[s]:
                run[1] -= 1
                self._used -= run[0] if run[1] == 0 else 0
            self.length[s], self.position[s], self._runs[s] = 0, 0, []
            self._free.append(s)

    def evict(self, seqs, keep, n_first=0, n_last=0) -> list:
        """Shortens the listed sequences that are longer than keep: their first n_first tokens
        stay, their last n_last and, between them, those of the largest ``key_weights`` (which are not
        looked at where n_first + n_last == keep).  Keys keep the rotation of their positions, and new tokens'
        positions go on as before.  Returns, for each listed sequence, the indexes that stayed; to read them
        the call waits for the device.  A call is refused if the pool might not hold the
        pages that have to be copied because other sequences have them in common: those behind the first
        n_first tokens, at worst."""
        seqs = self._in_use(seqs)
        keep, n_first, n_last = (operator.index(i) for i in (keep, n_first, n_last))
        if keep < 1 or n_first < 0 or n_last < 0 or n_first + n_last > keep:
            raise ValueError("keep >= 1 with n_first + n_last <= keep expected")
        if self.key_weights is None and n_first + n_last != keep:
            raise ValueError("track the keys' weights, or give n_first + n_last == keep")
        long = [s for s in seqs if self.length[s] > keep]
        stay, page = self._n_pages(keep), self.cache.page_size
        need = 0
        for s in long:
            at = 0
            for pages, holders in self._runs[s]:
                need += max(0, min(at + pages, stay) - max(at, n_first // page)) if holders > 1 else 0
                at += pages
        self._room(need)
        if not long:
            return [list(range(self.length[s])) for s in seqs]
        self._on_current_stream()
        kept = torch.empty(len(seqs), keep, dtype=torch.int32, device="cuda")
        xb.op_kv_evict(self.cache, self._ids(seqs), keep, self.key_weights, n_first, n_last, kept=kept)
        kept = kept.tolist()
        if any(kept[i][0] < 0 for i, s in enumerate(seqs) if self.length[s] > 0):
            raise xb.XCacheError(xb.XC_ECUDA, "evict: the device found the cache in another state")
        for i, s in enumerate(seqs):
            if self.length[s] <= keep:
                kept[i] = kept[i][:self.length[s]]
                continue
            same = next((j for j, t in enumerate(kept[i]) if t != j), keep)
            self._leave_runs(s, same // page)             # from the first page whose rows change, its pages are its own
            self.length[s] = keep
        runs = {id(run): run for s in range(len(self.length)) for run in self._runs[s]}
        self._used = sum(pages for pages, _ in runs.values()) + sum(self._own_pages(s) for s in range(len(self.length)))
        return kept

    def _leave_runs(self, s, pages):
        """Sequence s has only its first ``pages`` pages in common with others from now on."""
        at = 0
        for i, run in enumerate(self._runs[s]):
            if at + run[0] > pages:
                break
            at += run[0]
        else:
            return
        if at < pages:                                    # the run is split, for all sequences that hold it
            front, back = [pages - at, run[1]], [run[0] - (pages - at), run[1]]
            for held in self._runs:
                for j, r in enumerate(held):
                    if r is run:
                        held[j:j + 1] = [front, back]
                        break
            i += 1
        for gone in self._runs[s][i:]:
            gone[1] -= 1
        del self._runs[s][i:]

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
        if x.dim() != 3 or x.shape[0] != len(seqs) or x.shape[2] != self.d or x.get_device() != self.cache.device:
            raise ValueError(f"x: CUDA tensor [{len(seqs)}, n, {self.d}] on the cache's device expected")
        B, n, d = x.shape
        if n == 0 or B == 0:
            return x
        if any(self.length[s] + n > self.max_len for s in seqs):
            raise ValueError(f"sequences hold at most {self.max_len} tokens")
        if any(self.position[s] + n > self.max_pos for s in seqs):
            raise ValueError(f"positions go up to {self.max_pos}")
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
        pos = torch.tensor([[self.position[s] + i] for s in seqs for i in range(n)], dtype=torch.int32, device="cuda")
        x = x.reshape(T, d).to(dt).contiguous()
        h, out = torch.empty_like(x), [torch.empty_like(x) for _ in self.weights[:2]]
        qkv = torch.empty(T, dq + 2 * dk, dtype=dt, device="cuda")
        q = torch.empty(T, dq, dtype=dt, device="cuda")
        o = torch.empty_like(q)
        need = xb.op_branch_attention_workspace_bytes(c, B, n, self.H, shared)
        if need == 0:                                     # more rows than the attention takes
            raise xb.XCacheError(xb.XC_EINVAL, xb.last_error())
        lse = None
        if self.track is not None:
            lse = torch.empty(T, self.H, device="cuda")
            weigh = xb.op_key_weights_workspace_bytes(c, B, n, self.H, shared)
            if weigh == 0:
                raise xb.XCacheError(xb.XC_EINVAL, xb.last_error())
            need = max(need, weigh)
        c.workspace(need, st)
        scratch = [xb.op_linear_i8_workspace_bytes(T, *w[name].shape) for w in self.weights for name in ("qkv_w", "o_w")
                   if w[name].dtype is torch.int8]
        scratch = torch.empty(max(scratch), dtype=torch.uint8, device="cuda") if scratch and max(scratch) else None
        xb.op_kv_extend(c, ids, n, slots, stream=st)
        self._used += new_pages
        for s in seqs:
            self.length[s] += n
            self.position[s] += n
        for layer, w in enumerate(self.weights):
            xb.op_ln_mod(self.dtype, x, self.zeros, self.zeros, h, eps=self.eps, stream=st)
            self._linear(xb.XC_EPI_BIAS, h, w, "qkv", qkv, scratch, stream=st)
            xb.op_qk_norm_rope(c, layer, qkv[:, :dq], qkv[:, dq:dq + dk], qkv[:, dq + dk:], w["gamma_q"], w["gamma_k"],
                               pos, self.pairs, self.n_pos, self.rotation, slots.view(-1), q, eps=self.eps, stream=st)
            xb.op_branch_attention(c, layer, ids, n, q, o, shared_len=shared, causal=True, stream=st, lse=lse)
            if lse is not None:
                xb.op_key_weights(c, layer, ids, n, q, lse, self.key_weights, shared_len=shared, causal=True,
                                  decay=self.track if layer == 0 else 1.0, stream=st)
            y = out[layer % 2]
            self._linear(xb.XC_EPI_RESID_GATE, o, w, "o", y, scratch, resid=x, stream=st)
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


def quantize_layers(weights, dtype="bf16"):
    """The layers with ``qkv_w`` and ``o_w`` as 8-bit integers, a scale for each row."""
    layers = []
    for w in weights:
        w = dict(w)
        for name in ("qkv", "o"):
            x = w[name + "_w"]
            q, scale = torch.empty_like(x, dtype=torch.int8), torch.empty(x.shape[0], device=x.device)
            xb.op_quantize_rows(dtype, x, q, scale)
            w[name + "_w"], w[name + "_s"] = q, scale
        layers.append(w)
    return layers


def main():
    d, H, Hk, hd, candidates = 512, 8, 8, 64, 6
    m = BranchedLayers(quantize_layers(random_layers(4, d, H, Hk, hd)), H, Hk, hd, n_pages=256, page_size=64, max_seqs=16,
                       max_len=2304, max_pos=8192, track=0.99)
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
    shared = m.shared_len(kids)
    m.free([k for i, k in enumerate(kids) if i != best] + [history])
    live = int(m.compact())
    kept = m.length[kids[best]]
    for _ in range(4):                                    # on from there, in memory for some 2000 tokens
        m.evict([kids[best]], 2000, n_first=16, n_last=256)
        m.step([kids[best]], torch.randn(1, 240, d, generator=g, device="cuda"))
    xb.check(xb.XC_OK if xb.op_device_error() == 0 else xb.XC_ECUDA)
    print(f"history 2016 tokens, {candidates} candidates on {pages} pages (shared {shared} tokens); kept candidate {best}: "
          f"{kept} tokens on {live} pages; after 4 more chunks {m.length[kids[best]]} of {m.position[kids[best]]} tokens")


if __name__ == "__main__":
    main()
