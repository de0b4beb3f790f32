"""ctypes binding of libxcache.so (include/xcache.h, include/xcache_ops.h).

Argument marshalling only: every step of the chunk step runs in the CUDA
library.  Device buffers are torch CUDA tensors (passed by data_ptr());
streams are torch streams.  Importing this module loads the library and
raises if it is missing -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libxcache.so")

XC_OK, XC_EINVAL, XC_ESTATE, XC_ENOMEM, XC_ECUDA, XC_ENUMERIC, XC_ETIMEOUT = range(7)
XC_F32, XC_BF16 = 0, 1
XC_DEC_FORCED, XC_DEC_COMPUTE, XC_DEC_SKIP = 0, 1, 2
XC_EPI_BIAS, XC_EPI_GELU, XC_EPI_RESID_GATE, XC_EPI_RESID_CACHE = 0, 1, 2, 3
XC_MAX_BLOCKS = 64
XC_MAX_GROUPS = 4
XC_DEV_CACHE_FULL, XC_DEV_BAD_SEQUENCE, XC_DEV_BAD_POSITION = 64, 128, 256
STATUS_NAMES = {0: "XC_OK", 1: "XC_EINVAL", 2: "XC_ESTATE", 3: "XC_ENOMEM", 4: "XC_ECUDA",
                5: "XC_ENUMERIC", 6: "XC_ETIMEOUT"}


class XCacheError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class ModelCfg(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in (
        "n_blocks", "d_model", "n_heads", "head_dim", "d_ffn", "c_latent", "action_dim",
        "n_cams", "frames", "grid_h", "grid_w", "kv_window_chunks", "n_denoise_steps", "dtype",
        "t_freq_dim")] + [("ln_eps", ctypes.c_float), ("rope_theta", ctypes.c_float),
                          ("kv_period", ctypes.c_int), ("n_groups", ctypes.c_int),
                          ("group_cams", ctypes.c_int * XC_MAX_GROUPS),
                          ("group_h", ctypes.c_int * XC_MAX_GROUPS),
                          ("group_w", ctypes.c_int * XC_MAX_GROUPS),
                          ("d_ctx", ctypes.c_int), ("max_ctx", ctypes.c_int)]


WEIGHT_NAMES = ("pe_w", "pe_b", "t_w1", "t_b1", "t_w2", "t_b2", "a_w1", "a_b1", "a_w2", "a_b2",
                "mod_w", "mod_b", "blk_mod", "qkv_w", "qkv_b", "o_w", "o_b", "f1_w", "f1_b",
                "f2_w", "f2_b", "head_w", "head_b", "head_tab", "out_w", "out_b",
                "ca_ln_w", "ca_ln_b", "ca_q_w", "ca_q_b", "ca_kv_w", "ca_kv_b", "ca_o_w", "ca_o_b")


class Weights(ctypes.Structure):
    _fields_ = [(n, ctypes.POINTER(ctypes.c_float)) for n in WEIGHT_NAMES]


class GateParams(ctypes.Structure):
    _fields_ = [("enabled", ctypes.c_int), ("tau_floor", ctypes.c_float), ("margin", ctypes.c_float),
                ("alpha", ctypes.c_float), ("tau_dev", ctypes.c_float), ("eps_dev", ctypes.c_float),
                ("front_anchors", ctypes.c_int), ("back_anchors", ctypes.c_int),
                ("warmup_chunks", ctypes.c_int), ("max_skips", ctypes.c_int),
                ("protect_step0", ctypes.c_int), ("step0_strict_tau", ctypes.c_float),
                ("fp_tokens", ctypes.c_int), ("fp_refresh", ctypes.c_int), ("fp_linear", ctypes.c_int),
                ("chain", ctypes.c_int),
                ("replay_skip", ctypes.POINTER(ctypes.c_uint8)),
                ("replay_table", ctypes.c_void_p)]


class StepStats(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int), ("chunk_index", ctypes.c_int),
                ("decision", ctypes.c_uint8 * XC_MAX_BLOCKS),
                ("s_cos", ctypes.c_float * XC_MAX_BLOCKS),
                ("d_max", ctypes.c_float * XC_MAX_BLOCKS),
                ("tau_cos", ctypes.c_float * XC_MAX_BLOCKS)]


class ProfileRec(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int), ("block", ctypes.c_int), ("pass_seq", ctypes.c_int),
                ("decision", ctypes.c_int), ("chunk", ctypes.c_int), ("n_keys", ctypes.c_int),
                ("ms", ctypes.c_float)]


class KVCacheDesc(ctypes.Structure):
    """xc_kv_cache: one pool of pages and the sequences in it."""
    _fields_ = [(n, ctypes.c_int) for n in ("dtype", "n_layers", "n_pages", "page_size", "n_kv_heads", "head_dim",
                                            "max_seqs", "max_pages")] + \
               [(n, ctypes.c_void_p) for n in ("k", "v", "ref", "table", "len")]


KERNEL_KINDS = ("cond", "embed", "gate", "ln", "qkv", "attn", "oproj", "ffn1", "ffn2", "reuse", "head",
                "xattn", "chain")

_P = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float
_L = ctypes.c_long
SIGNATURES = {
    "xc_gate_params_default": (None, [ctypes.POINTER(GateParams)]),
    "xc_init": (_I, [ctypes.POINTER(ModelCfg), ctypes.POINTER(Weights), _P, ctypes.POINTER(_P)]),
    "xc_chunk_step": (_I, [_P, _P, _P, _F, _I, _I, ctypes.POINTER(GateParams), _P,
                           ctypes.POINTER(StepStats)]),
    "xc_reset": (_I, [_P]),
    "xc_set_context": (_I, [_P, _P, _I]),
    "xc_destroy": (None, [_P]),
    "xc_last_error": (ctypes.c_char_p, [_P]),
    "xc_euler_update": (_I, [_P, _P, _P, _F, _L]),
    "xc_set_block_trace": (_I, [_P, _P]),
    "xc_sync": (_I, [_P]),
    "xc_chunk_index": (_I, [_P]),
    "xc_debug_fail_alloc": (None, [_I]),
    "xc_debug_expire_wait": (_I, [_P]),
    "xc_launch_count": (ctypes.c_longlong, [_P]),
    "xc_profile_start": (_I, [_P, ctypes.c_uint, _I]),
    "xc_profile_stop": (_I, [_P, ctypes.POINTER(ProfileRec), _I, ctypes.POINTER(_I)]),
    "xc_op_linear": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "xc_op_quantize_rows": (_I, [_I, _I, _I, _P, _P, _P, _P]),
    "xc_op_linear_i8_workspace_bytes": (ctypes.c_size_t, [_I, _I, _I]),
    "xc_op_linear_i8": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_qkv_rope": (_I, [_I, _I, _I, _I, _I, _I, _I, _I, _F, _P, _P, _P, _P, _P, _P, _P]),
    "xc_op_attention_workspace_bytes": (ctypes.c_size_t, [_I, _I]),
    "xc_op_attention": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_ln_mod": (_I, [_I, _I, _I, _F, _P, _P, _P, _P, _P]),
    "xc_op_residual_reuse": (_I, [_I, _L, _P, _P, _P, _P]),
    "xc_op_device_error": (_I, []),
    "xc_op_gate_workspace_bytes": (ctypes.c_size_t, [_I, _I, _I, _I]),
    "xc_op_gate": (_I, [_I, _I, _I, _I, _P, _P, _I, _P, _P, _P, _P, _I, _I, _I, ctypes.POINTER(GateParams),
                        _P, _P, _P, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_gate_static": (_I, [_I, _I, _I, _I, _P, _P, _I, _P, _P, _P, _P, _I, _I, _I,
                               ctypes.POINTER(GateParams), _P, _P, _P, _P, _P]),
    "xc_op_kv_workspace_bytes": (ctypes.c_size_t, [_P]),
    "xc_op_kv_fork": (_I, [_P, _I, _P, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_kv_extend": (_I, [_P, _I, _P, _I, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_kv_free": (_I, [_P, _I, _P, _P]),
    "xc_op_kv_compact": (_I, [_P, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_kv_evict_workspace_bytes": (ctypes.c_size_t, [_P, _I, _I]),
    "xc_op_kv_evict": (_I, [_P, _I, _P, _I, _I, _I, _P, _L, _P, _P, ctypes.c_size_t, _P]),
    "xc_op_rope_table": (_I, [_I, _P, _P, ctypes.c_double, _P, _P]),
    "xc_op_qk_norm_rope": (_I, [_P, _I, _I, _I, _P, _L, _P, _L, _P, _L, _P, _P, _F, _I, _P, _P, _P, _P, _I, _P, _P,
                                _L, _P]),
    "xc_op_stream_capturing": (_I, [_P]),
    "xc_op_branch_attention_workspace_bytes": (ctypes.c_size_t, [_P, _I, _I, _I, _I]),
    "xc_op_branch_attention": (_I, [_P, _I, _I, _P, _I, _I, _P, _L, _I, _I, _F, _P, _L, _P, ctypes.c_size_t, _P]),
    "xc_op_key_weights_workspace_bytes": (ctypes.c_size_t, [_P, _I, _I, _I, _I]),
    "xc_op_key_weights": (_I, [_P, _I, _I, _P, _I, _I, _P, _L, _P, _I, _I, _F, _F, _P, _L, _P, ctypes.c_size_t, _P]),
    "xc_op_branch_attention_lse": (_I, [_P, _I, _I, _P, _I, _I, _P, _L, _I, _I, _F, _P, _L, _P, _P, ctypes.c_size_t, _P]),
}


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2604_20289_gb300.build` (no fallback path exists)")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in SIGNATURES.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


LIB = _load()


def last_error(ctx=None) -> str:
    return LIB.xc_last_error(ctx).decode(errors="replace")


def check(status: int, ctx=None):
    if status != XC_OK:
        raise XCacheError(status, last_error(ctx))


def _ptr(t) -> int | None:
    """Device pointer of a torch tensor, host pointer of a numpy array, None."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


_raw_stream = None


def _stream(stream) -> int | None:
    if stream is None:
        global _raw_stream
        if _raw_stream is None:                   # the handle alone: a Stream object costs 3 us a call
            import torch
            torch.cuda.current_stream()           # sets torch's CUDA state up, or says why it cannot
            _raw_stream = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        return _raw_stream[0](_raw_stream[1]())
    return getattr(stream, "cuda_stream", stream)


def dtype_code(dtype) -> int:
    return {"f32": XC_F32, "bf16": XC_BF16, XC_F32: XC_F32, XC_BF16: XC_BF16}[dtype]


def model_cfg(cfg) -> ModelCfg:
    """ModelCfg from any object with the shape attributes (e.g. xc_inputs.ModelCfg);
    optional ``view_groups`` ((cameras, grid_h, grid_w), ...) and ``kv_period``."""
    m = ModelCfg(cfg.n_blocks, cfg.d_model, cfg.n_heads, cfg.head_dim, cfg.d_ffn, cfg.c_latent,
                 cfg.action_dim, cfg.n_cams, cfg.frames, cfg.grid_h, cfg.grid_w, cfg.kv_window,
                 cfg.n_steps, dtype_code(cfg.dtype), cfg.t_freq, cfg.ln_eps, cfg.rope_theta)
    m.kv_period = int(getattr(cfg, "kv_period", 0))
    groups = tuple(getattr(cfg, "view_groups", ()))
    if len(groups) > XC_MAX_GROUPS:
        raise ValueError(f"at most {XC_MAX_GROUPS} view groups")
    m.n_groups = len(groups)
    for i, (c, h, w) in enumerate(groups):
        m.group_cams[i], m.group_h[i], m.group_w[i] = c, h, w
    m.d_ctx = int(getattr(cfg, "d_ctx", 0))
    m.max_ctx = int(getattr(cfg, "max_ctx", 0))
    return m


def gate_params(**kw) -> GateParams:
    """Table 1 defaults, overridden by keyword (replay_skip: sequence of 0/1;
    replay_table: torch CUDA uint8 tensor [n_denoise_steps, n_blocks], kept
    alive by the caller)."""
    p = GateParams()
    LIB.xc_gate_params_default(ctypes.byref(p))
    replay = kw.pop("replay_skip", None)
    table = kw.pop("replay_table", None)
    if table is not None:
        p.replay_table = table.data_ptr()
    for k, v in kw.items():
        if not hasattr(p, k):
            raise KeyError(k)
        setattr(p, k, int(v) if isinstance(getattr(p, k), int) else float(v))
    if replay is not None:
        arr = (ctypes.c_uint8 * len(replay))(*[1 if r else 0 for r in replay])
        p._replay_keepalive = arr
        p.replay_skip = ctypes.cast(arr, ctypes.POINTER(ctypes.c_uint8))
    return p


class XCache:
    """One X-Cache context (xc_init .. xc_destroy) on the current CUDA device."""

    def __init__(self, cfg, weights: dict, stream=None):
        self.cfg = cfg
        self._c_cfg = model_cfg(cfg)
        # numpy arrays (host) or contiguous float32 torch CUDA tensors (device)
        keep = {k: (weights[k] if hasattr(weights[k], "data_ptr") else
                    np.ascontiguousarray(weights[k], dtype=np.float32))
                for k in WEIGHT_NAMES if k in weights}
        w = Weights(*[ctypes.cast(_ptr(keep[k]), ctypes.POINTER(ctypes.c_float)) if k in keep else None
                      for k in WEIGHT_NAMES])
        ctx = ctypes.c_void_p()
        self._stream = _stream(stream)
        check(LIB.xc_init(ctypes.byref(self._c_cfg), ctypes.byref(w), self._stream, ctypes.byref(ctx)))
        self.ctx = ctx

    def close(self):
        if getattr(self, "ctx", None):
            LIB.xc_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def chunk_step(self, latent, action, sigma: float, step: int, is_kv_update: bool = False,
                   gate: GateParams | None = None, v_out=None, want_stats: bool = True):
        """latent / v_out: torch CUDA tensors or numpy float32 host arrays."""
        act = np.ascontiguousarray(action, dtype=np.float32)
        st = StepStats() if want_stats else None
        check(LIB.xc_chunk_step(self.ctx, _ptr(latent), act.ctypes.data, float(sigma), int(step),
                                int(bool(is_kv_update)), ctypes.byref(gate) if gate is not None else None,
                                _ptr(v_out), ctypes.byref(st) if st is not None else None), self.ctx)
        if st is None:
            return None
        B = st.n_blocks
        return dict(chunk=st.chunk_index,
                    decision=np.array(st.decision[:B], dtype=np.int64),
                    s_cos=np.array(st.s_cos[:B], dtype=np.float64),
                    d_max=np.array(st.d_max[:B], dtype=np.float64),
                    tau=np.array(st.tau_cos[:B], dtype=np.float64))

    def reset(self):
        check(LIB.xc_reset(self.ctx), self.ctx)

    def set_context(self, tokens):
        """Condition tokens [n_ctx, d_ctx] (torch CUDA tensor or numpy float32)."""
        if isinstance(tokens, np.ndarray):
            tokens = np.ascontiguousarray(tokens, dtype=np.float32)
        check(LIB.xc_set_context(self.ctx, _ptr(tokens), int(tokens.shape[0])), self.ctx)

    def euler(self, x, v, dsigma: float):
        check(LIB.xc_euler_update(self.ctx, _ptr(x), _ptr(v), float(dsigma), x.numel()), self.ctx)

    def set_trace(self, buf):
        check(LIB.xc_set_block_trace(self.ctx, _ptr(buf)), self.ctx)

    def sync(self):
        check(LIB.xc_sync(self.ctx), self.ctx)

    @property
    def chunk_index(self) -> int:
        return LIB.xc_chunk_index(self.ctx)

    @property
    def launch_count(self) -> int:
        return LIB.xc_launch_count(self.ctx)

    def profile_start(self, kinds=KERNEL_KINDS, capacity: int = 65536):
        mask = 0
        for k in kinds:
            mask |= 1 << KERNEL_KINDS.index(k)
        self._prof_cap = capacity
        check(LIB.xc_profile_start(self.ctx, mask, capacity), self.ctx)

    def profile_stop(self) -> list:
        """Synchronises; returns dicts (kind, block, pass_seq, decision, chunk, n_keys, ms)."""
        cap = getattr(self, "_prof_cap", 65536)
        recs = (ProfileRec * cap)()
        n = ctypes.c_int()
        check(LIB.xc_profile_stop(self.ctx, recs, cap, ctypes.byref(n)), self.ctx)
        return [dict(kind=KERNEL_KINDS[r.kind], block=r.block, pass_seq=r.pass_seq,
                     decision=r.decision, chunk=r.chunk, n_keys=r.n_keys, ms=r.ms)
                for r in recs[:min(n.value, cap)]]


# --------------------------------------------------------------- operators
def op_linear(dtype, epilogue, A, Wt, bias, out, gate=None, resid=None, xin=None, rhat=None,
              stream=None):
    M, K = A.shape
    N = Wt.shape[0]
    check(LIB.xc_op_linear(dtype_code(dtype), epilogue, M, N, K, _ptr(A), _ptr(Wt), _ptr(bias),
                           _ptr(gate), _ptr(resid), _ptr(xin), _ptr(out), _ptr(rhat),
                           _stream(stream)))


_types = None


def _torch_types(dtype):
    """(the activations' torch type, float32, int8)"""
    global _types
    if _types is None:
        import torch
        _types = {XC_F32: (torch.float32, torch.float32, torch.int8), XC_BF16: (torch.bfloat16, torch.float32, torch.int8)}
    return _types[dtype_code(dtype)]


def _on_device(*tensors):
    """Refuses tensors that are not on the current CUDA device."""
    import torch
    dev = torch._C._cuda_getDevice() if tensors[0].is_cuda else -2
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("expected CUDA tensors on the current device")


def op_quantize_rows(dtype, x, q, scale, stream=None):
    """8-bit integers q [M, K] (int8) and scale [M] (float32) of the rows of x [M, K]; all contiguous."""
    dt, f32, i8 = _torch_types(dtype)
    _on_device(x, q, scale)
    if x.dim() != 2 or x.dtype is not dt or q.shape != x.shape or q.dtype is not i8 or \
            scale.shape != x.shape[:1] or scale.dtype is not f32 or \
            not (x.is_contiguous() and q.is_contiguous() and scale.is_contiguous()):
        raise ValueError("x [M, K] of dtype, q [M, K] int8, scale [M] float32, all contiguous")
    M, K = x.shape
    check(LIB.xc_op_quantize_rows(dtype_code(dtype), M, K, x.data_ptr(), q.data_ptr(), scale.data_ptr(), _stream(stream)))


_I8_BYTES = {}                                    # workspace sizes by device and shape


def op_linear_i8_workspace_bytes(M, N, K) -> int:
    """0 where a call of few tokens needs none."""
    return LIB.xc_op_linear_i8_workspace_bytes(M, N, K)


def op_linear_i8(dtype, epilogue, A, Wq, w_scale, bias, out, gate=None, resid=None, a_scale=None, workspace=None,
                 stream=None):
    """out [M, N] = epilogue of A [M, K] by Wq [N, K] (int8) with w_scale [N] and bias [N] (float32).  A is of dtype and
    quantised by the call, or with a_scale [M] (float32) int8.  gate [N] float32 and resid [M, N] of dtype for
    XC_EPI_RESID_GATE.  All contiguous.  workspace: a device tensor of op_linear_i8_workspace_bytes, or None: allocated
    for the call (in a capture: from the graph's memory)."""
    dt, f32, i8 = _torch_types(dtype)
    _on_device(A, Wq, w_scale, bias, out, gate, resid, a_scale)
    (M, K), N = A.shape, Wq.shape[0]
    if A.dtype is not (dt if a_scale is None else i8) or Wq.dtype is not i8 or Wq.shape != (N, K) or \
            out.shape != (M, N) or out.dtype is not dt or w_scale.shape != (N,) or bias.shape != (N,) or \
            w_scale.dtype is not f32 or bias.dtype is not f32 or not (A.is_contiguous() and Wq.is_contiguous() and
            w_scale.is_contiguous() and bias.is_contiguous() and out.is_contiguous()):
        raise ValueError("A [M, K] of dtype (int8 with a_scale), Wq [N, K] int8, w_scale, bias [N] float32, out [M, N] of "
                         "dtype, all contiguous")
    if (gate is not None and (gate.shape != (N,) or gate.dtype is not f32 or not gate.is_contiguous())) or \
            (resid is not None and (resid.shape != (M, N) or resid.dtype is not dt or not resid.is_contiguous())) or \
            (a_scale is not None and (a_scale.shape != (M,) or a_scale.dtype is not f32 or not a_scale.is_contiguous())):
        raise ValueError("gate [N] and a_scale [M] float32, resid [M, N] of dtype, all contiguous")
    cuda = _stream(stream)
    if workspace is None:
        key = A.get_device(), M, N, K
        need = _I8_BYTES.get(key)
        if need is None:
            if len(_I8_BYTES) >= 4096:
                _I8_BYTES.clear()
            need = _I8_BYTES[key] = LIB.xc_op_linear_i8_workspace_bytes(M, N, K)
        buf, ws, nbytes = _scratch(need, stream, cuda, A.device) if need else (None, None, 0)
    else:
        buf, ws, nbytes = _given(workspace)
    st = LIB.xc_op_linear_i8(dtype_code(dtype), epilogue, M, N, K, A.data_ptr(), _ptr(a_scale), Wq.data_ptr(),
                             w_scale.data_ptr(), bias.data_ptr(), _ptr(gate), _ptr(resid), out.data_ptr(), ws, nbytes,
                             cuda)
    if st:
        check(st)


def op_qkv_rope(dtype, n_cams, frames, gh, gw, chunk, head_dim, theta, A, Wt, bias, q, k, v,
                stream=None):
    d = A.shape[1]
    check(LIB.xc_op_qkv_rope(dtype_code(dtype), n_cams, frames, gh, gw, chunk, d, head_dim,
                             float(theta), _ptr(A), _ptr(Wt), _ptr(bias), _ptr(q), _ptr(k), _ptr(v),
                             _stream(stream)))


def op_attention_workspace_bytes(dtype, head_dim):
    return LIB.xc_op_attention_workspace_bytes(dtype_code(dtype), head_dim)


def op_attention(dtype, n_heads, head_dim, q, k, v, o, workspace=None, stream=None):
    """workspace: None (one SM per unit), "auto" (a device buffer of
    op_attention_workspace_bytes is allocated for the call) or a device
    tensor of at least that many bytes."""
    if isinstance(workspace, str) and workspace == "auto":
        import torch
        nb = op_attention_workspace_bytes(dtype, head_dim)
        workspace = torch.empty(max(nb, 1), dtype=torch.uint8, device=q.device) if nb else None
    ws_ptr = _ptr(workspace) if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    check(LIB.xc_op_attention(dtype_code(dtype), q.shape[0], k.shape[0], n_heads, head_dim, _ptr(q),
                              _ptr(k), _ptr(v), _ptr(o), ws_ptr, ws_bytes, _stream(stream)))


def op_ln_mod(dtype, x, shift, scale, out, eps=1e-6, stream=None):
    M, d = x.shape
    check(LIB.xc_op_ln_mod(dtype_code(dtype), M, d, float(eps), _ptr(x), _ptr(shift), _ptr(scale),
                           _ptr(out), _stream(stream)))


def op_residual_reuse(dtype, x, rhat, out, stream=None):
    check(LIB.xc_op_residual_reuse(dtype_code(dtype), x.numel(), _ptr(x), _ptr(rhat), _ptr(out),
                                   _stream(stream)))


def op_device_error() -> int:
    return LIB.xc_op_device_error()


class GateCell(ctypes.Structure):
    """xc_gate_cell: per-(t, b) gate state (32 bytes)."""
    _fields_ = [("ema", ctypes.c_double), ("has_hist", ctypes.c_int), ("stale", ctypes.c_int),
                ("valid", ctypes.c_int), ("active", ctypes.c_int), ("pad", ctypes.c_int * 2)]


def op_gate_workspace_bytes(dtype, n_cams, tokens_per_cam, d) -> int:
    return LIB.xc_op_gate_workspace_bytes(dtype_code(dtype), n_cams, tokens_per_cam, d)


def op_gate(dtype, n_cams, tokens_per_cam, x, fp_rows, phi, phi_act, cell, action, mode, step,
            gate, flag, s_cos, d_max, tau, workspace, stream=None):
    """x, fp_rows [n_cams, kfp] int32, phi, phi_act, cell (uint8 tensor of 32 bytes), flag,
    s_cos, d_max, tau, workspace: torch CUDA tensors; action: numpy float32."""
    act = np.ascontiguousarray(action, dtype=np.float32)
    check(LIB.xc_op_gate(dtype_code(dtype), n_cams, tokens_per_cam, x.shape[1], _ptr(x), _ptr(fp_rows),
            fp_rows.shape[1], _ptr(phi), _ptr(phi_act), _ptr(cell), act.ctypes.data, act.size, mode,
            step, ctypes.byref(gate) if gate is not None else None, _ptr(flag), _ptr(s_cos),
            _ptr(d_max), _ptr(tau), _ptr(workspace), workspace.numel() * workspace.element_size(),
            _stream(stream)))


# --------------------------------- branched rollouts over a paged K/V cache
class KVCache:
    """Handle on a paged key / value cache (xc_kv_cache) over the caller's torch
    CUDA tensors: k, v [n_layers, n_pages, page_size, n_kv_heads * head_dim]
    (float32 or bfloat16), ref [n_pages], table [max_seqs, max_pages] and len
    [max_seqs] int32, all contiguous and on one device, which is the current one in
    every call.  Keeps the tensors, and one workspace per stream that grows to the
    largest call.  ``empty`` allocates them.

    A call that torch captures into a graph (``torch.cuda.graph``) takes a
    workspace of its own from the graph's memory instead: it lives as long as the
    graph, whatever larger calls follow, and replays may overlap other calls'
    workspaces.  Calls in a capture that torch does not run need ``workspace=``."""

    def __init__(self, dtype, n_kv_heads, head_dim, k, v, ref, table, length):
        import torch
        want = torch.float32 if dtype_code(dtype) == XC_F32 else torch.bfloat16
        if k.dim() != 4 or k.shape != v.shape or k.shape[3] != n_kv_heads * head_dim or k.dtype != want or \
                v.dtype != want:
            raise ValueError("k, v: [n_layers, n_pages, page_size, n_kv_heads * head_dim] of the cache's dtype")
        if table.dim() != 2 or ref.shape != k.shape[1:2] or length.shape != table.shape[:1]:
            raise ValueError("ref [n_pages], table [max_seqs, max_pages], len [max_seqs]")
        for t in (ref, table, length):
            if t.dtype != torch.int32:
                raise ValueError("ref, table and len are int32")
        self.device = k.get_device()
        for t in (k, v, ref, table, length):
            if not t.is_contiguous() or not t.is_cuda or t.get_device() != self.device:
                raise ValueError("cache tensors are contiguous CUDA tensors of one device")
        self._current_device = torch._C._cuda_getDevice
        self.k, self.v, self.ref, self.table, self.len = k, v, ref, table, length
        self.dtype, self.n_kv_heads, self.head_dim = dtype, n_kv_heads, head_dim
        self.page_size = k.shape[2]
        self.torch_dtype, self._int32, self._float32 = want, torch.int32, torch.float32
        self.desc = KVCacheDesc(dtype_code(dtype), k.shape[0], k.shape[1], k.shape[2], n_kv_heads, head_dim,
                                table.shape[0], table.shape[1], k.data_ptr(), v.data_ptr(), ref.data_ptr(),
                                table.data_ptr(), length.data_ptr())
        self.ptr = ctypes.addressof(self.desc)
        self._ws = {}                             # stream -> (tensor, pointer, bytes)
        self._attn_bytes, self._axes = {}, {}     # workspace sizes by shape, axis arrays by value
        self._weigh_bytes, self._evict_bytes = {}, {}
        self._page_bytes = LIB.xc_op_kv_workspace_bytes(self.ptr)

    @classmethod
    def empty(cls, dtype, n_layers, n_pages, page_size, n_kv_heads, head_dim, max_seqs, max_pages, device="cuda"):
        import torch
        dt = torch.float32 if dtype_code(dtype) == XC_F32 else torch.bfloat16
        shape = (n_layers, n_pages, page_size, n_kv_heads * head_dim)
        return cls(dtype, n_kv_heads, head_dim, torch.empty(shape, dtype=dt, device=device),
                   torch.empty(shape, dtype=dt, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device),
                   torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(max_seqs, dtype=torch.int32, device=device))

    def note(self, memo: dict, key, value):
        """Keeps value under key in one of the handle's dicts, which hold 4096 shapes at most."""
        if len(memo) >= 4096:
            memo.clear()
        memo[key] = value
        return value

    def workspace(self, nbytes: int, stream: int):
        """(tensor, pointer, bytes) of a device workspace for one call on this stream (cudaStream_t)."""
        capturing = LIB.xc_op_stream_capturing(stream)
        ws = None if capturing else self._ws.get(stream)
        if ws is None or ws[2] < nbytes:
            import torch
            ext = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
            with torch.cuda.stream(ext):       # freed memory is reused in this stream's order
                buf = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=self.k.device)
            ws = buf, buf.data_ptr(), buf.numel()
            if not capturing:                  # a graph's memory is the graph's: never kept, never handed to other calls
                self._ws[stream] = ws
        return ws

    def int32(self, t, n: int) -> int:
        """Device pointer of a contiguous int32 tensor of n elements on the cache's device."""
        if t.dtype is not self._int32 or t.numel() != n or not t.is_contiguous() or t.get_device() != self.device:
            raise ValueError(f"expected a contiguous int32 CUDA tensor of {n} elements on the cache's device")
        return t.data_ptr()

    def stream(self, stream) -> int:
        """cudaStream_t of a call, which runs on the cache's device."""
        if self._current_device() != self.device:
            raise ValueError(f"the cache is on CUDA device {self.device}, which is not the current one")
        return _stream(stream)


def _scratch(nbytes, stream, cuda, device):
    """(tensor, pointer, bytes) of a workspace for one call, from the memory of the stream it runs on."""
    import torch
    if stream is None:
        buf = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(torch.cuda.ExternalStream(cuda) if cuda else torch.cuda.default_stream()):
            buf = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)
    return buf, buf.data_ptr(), buf.numel()


def _given(workspace):
    """(tensor, pointer, bytes) of the caller's own workspace."""
    import torch
    if not workspace.is_cuda or not workspace.is_contiguous() or workspace.get_device() != torch._C._cuda_getDevice():
        raise ValueError("workspace: expected a contiguous CUDA tensor on the current device")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def op_kv_workspace_bytes(cache: KVCache) -> int:
    """Bytes of a workspace for op_kv_fork, op_kv_extend and op_kv_compact, whose ``workspace`` is a device tensor of
    that size, or None for the cache's own."""
    return cache._page_bytes


def op_kv_fork(cache: KVCache, src, dst, stream=None, workspace=None):
    """Sequence dst[i] becomes a copy of src[i] (int32 CUDA tensors)."""
    st = cache.stream(stream)
    n = src.numel()
    buf, ws, nbytes = cache.workspace(cache._page_bytes, st) if workspace is None else _given(workspace)
    check(LIB.xc_op_kv_fork(cache.ptr, n, cache.int32(src, n), cache.int32(dst, n), ws, nbytes, st))


def op_kv_extend(cache: KVCache, seqs, n_new: int, slots, stream=None, workspace=None):
    """Appends n_new tokens to every listed sequence; slots [n, n_new] int32 receives their cache slots."""
    st = cache.stream(stream)
    n = seqs.numel()
    buf, ws, nbytes = cache.workspace(cache._page_bytes, st) if workspace is None else _given(workspace)
    check(LIB.xc_op_kv_extend(cache.ptr, n, cache.int32(seqs, n), n_new, cache.int32(slots, n * n_new), ws, nbytes,
                              st))


def op_kv_free(cache: KVCache, seqs, stream=None):
    n = seqs.numel()
    check(LIB.xc_op_kv_free(cache.ptr, n, cache.int32(seqs, n), cache.stream(stream)))


def op_kv_compact(cache: KVCache, n_live, stream=None, workspace=None):
    """n_live: int32 CUDA tensor of one element, receives the pages in use."""
    st = cache.stream(stream)
    buf, ws, nbytes = cache.workspace(cache._page_bytes, st) if workspace is None else _given(workspace)
    check(LIB.xc_op_kv_compact(cache.ptr, cache.int32(n_live, 1), ws, nbytes, st))


def op_rope_table(axis_pairs, n_pos, theta, out, stream=None):
    """out: contiguous float32 CUDA tensor of 2 * sum(axis_pairs * n_pos) elements."""
    n = len(axis_pairs)
    if len(n_pos) != n or out.numel() != 2 * sum(a * b for a, b in zip(axis_pairs, n_pos)) or \
            not out.is_contiguous() or not out.is_cuda or out.element_size() != 4 or \
            not out.is_floating_point():
        raise ValueError("out: float32, one (cos, sin) pair per position and pair of every axis")
    check(LIB.xc_op_rope_table(n, (_I * n)(*axis_pairs), (_I * n)(*n_pos), float(theta), out.data_ptr(),
                               _stream(stream)))


def op_qk_norm_rope(cache: KVCache, layer, q, k, v, gamma_q, gamma_k, pos, axis_pairs, n_pos, table, slots, q_out,
                    eps=1e-6, half_split=False, stream=None):
    """q, q_out [T, n_heads * head_dim], k, v [T, n_kv_heads * head_dim] (row-strided views allowed), pos [T, axes]
    and slots [T] int32, table from op_rope_table; axis_pairs, n_pos: host sequences."""
    T, dq = q.shape
    hd, dt = cache.head_dim, cache.torch_dtype
    dk = cache.n_kv_heads * hd
    key = (len(axis_pairs), *axis_pairs, *n_pos)
    axes = cache._axes.get(key)
    if axes is None:
        if len(n_pos) != len(axis_pairs):
            raise ValueError("one n_pos per axis")
        axes = cache.note(cache._axes, key, (len(axis_pairs), (_I * len(axis_pairs))(*axis_pairs),
                                             (_I * len(n_pos))(*n_pos), 2 * sum(a * b for a, b in zip(axis_pairs, n_pos))))
    n, c_pairs, c_pos, entries = axes
    if dq % hd or q_out.shape != q.shape or k.shape != (T, dk) or v.shape != (T, dk) or q.dtype is not dt or \
            k.dtype is not dt or v.dtype is not dt or q_out.dtype is not dt:
        raise ValueError("q, q_out [T, n_heads * head_dim], k, v [T, n_kv_heads * head_dim] of the cache's dtype")
    f32 = cache._float32
    if gamma_q.numel() != hd or gamma_k.numel() != hd or table.numel() != entries or gamma_q.dtype is not f32 or \
            gamma_k.dtype is not f32 or table.dtype is not f32 or not gamma_q.is_contiguous() or \
            not gamma_k.is_contiguous() or not table.is_contiguous():
        raise ValueError("float32 gamma_q, gamma_k [head_dim]; table: one (cos, sin) pair per position and pair of every axis")
    (sq, u0), (sk, u1), (sv, u2), (so, u3) = q.stride(), k.stride(), v.stride(), q_out.stride()
    if u0 != 1 or u1 != 1 or u2 != 1 or u3 != 1:
        raise ValueError("rows must have unit column stride")
    dev = cache.device
    if not (q.get_device() == k.get_device() == v.get_device() == q_out.get_device() == gamma_q.get_device() ==
            gamma_k.get_device() == table.get_device() == dev):
        raise ValueError("expected CUDA tensors on the cache's device")
    if T == 1:
        sq, sk, sv, so = dq, dk, dk, dq
    st = LIB.xc_op_qk_norm_rope(cache.ptr, layer, T, dq // hd, q.data_ptr(), sq, k.data_ptr(), sk, v.data_ptr(), sv,
                                gamma_q.data_ptr(), gamma_k.data_ptr(), eps, n, c_pairs, c_pos,
                                cache.int32(pos, T * n), table.data_ptr(), half_split, cache.int32(slots, T),
                                q_out.data_ptr(), so, cache.stream(stream))
    if st:
        check(st)


def op_branch_attention_workspace_bytes(cache: KVCache, n_branches, n_q, n_heads, shared_len=0) -> int:
    return LIB.xc_op_branch_attention_workspace_bytes(cache.ptr, n_branches, n_q, n_heads, shared_len)


def _lse(cache: KVCache, lse, rows, heads) -> int:
    if lse.shape != (rows, heads) or lse.dtype is not cache._float32 or not lse.is_contiguous() or \
            lse.get_device() != cache.device:
        raise ValueError("lse: contiguous float32 tensor [len(seqs) * n_q, n_heads] on the cache's device")
    return lse.data_ptr()


def op_branch_attention(cache: KVCache, layer, seqs, n_q, q, o, shared_len=0, causal=False, scale=0.0,
                        workspace=None, stream=None, lse=None):
    """q, o [len(seqs) * n_q, n_heads * head_dim] (row-strided views allowed); seqs int32 CUDA tensor.
    lse: float32 [len(seqs) * n_q, n_heads], receives the log of each row's sum of exponentials, or None.
    workspace: a device tensor of op_branch_attention_workspace_bytes, or None for the cache's own."""
    B, hd, dt = seqs.numel(), cache.head_dim, cache.torch_dtype
    T, dq = q.shape
    if T != B * n_q or dq % hd or o.shape != q.shape or q.dtype is not dt or o.dtype is not dt:
        raise ValueError("q, o [len(seqs) * n_q, n_heads * head_dim] of the cache's dtype")
    (sq, u0), (so, u1) = q.stride(), o.stride()
    if u0 != 1 or u1 != 1:
        raise ValueError("rows must have unit column stride")
    if not (q.get_device() == o.get_device() == cache.device):
        raise ValueError("expected CUDA tensors on the cache's device")
    if T == 1:
        sq = so = dq
    if lse is not None:
        lse = _lse(cache, lse, T, dq // hd)
    cuda = cache.stream(stream)
    if workspace is None:
        key = (B, n_q, dq, shared_len)
        need = cache._attn_bytes.get(key)
        if need is None:
            need = cache.note(cache._attn_bytes, key,
                              op_branch_attention_workspace_bytes(cache, B, n_q, dq // hd, shared_len))
        buf, ws, nbytes = cache.workspace(need, cuda)
    else:
        buf, ws, nbytes = _given(workspace)
    st = LIB.xc_op_branch_attention_lse(cache.ptr, layer, B, cache.int32(seqs, B), n_q, dq // hd, q.data_ptr(), sq,
                                        shared_len, causal, scale, o.data_ptr(), so, lse, ws, nbytes, cuda)
    if st:
        check(st)


def op_key_weights_workspace_bytes(cache: KVCache, n_branches, n_q, n_heads, shared_len=0) -> int:
    return LIB.xc_op_key_weights_workspace_bytes(cache.ptr, n_branches, n_q, n_heads, shared_len)


def _weights(cache: KVCache, weights) -> tuple:
    """(pointer, row stride) of the keys' weights."""
    if weights.dim() != 2 or weights.shape[0] != cache.table.shape[0] or \
            weights.shape[1] < cache.table.shape[1] * cache.page_size or weights.dtype is not cache._float32 or \
            weights.get_device() != cache.device or weights.stride(1) != 1 or \
            (weights.shape[0] > 1 and weights.stride(0) < weights.shape[1]):
        raise ValueError("weights: float32 tensor [max_seqs, max_pages * page_size] with unit column stride on the "
                         "cache's device")
    return weights.data_ptr(), max(weights.stride(0), weights.shape[1])


def op_key_weights(cache: KVCache, layer, seqs, n_q, q, lse, weights, shared_len=0, causal=False, scale=0.0, decay=1.0,
                   workspace=None, stream=None):
    """Adds to weights [max_seqs, max_pages * page_size] (float32), after decaying them, the weight that the rows of q
    gave to each key; lse [len(seqs) * n_q, n_heads] from op_branch_attention of the same q.  workspace: a device tensor
    of op_key_weights_workspace_bytes, or None for the cache's own."""
    B, hd = seqs.numel(), cache.head_dim
    T, dq = q.shape
    if T != B * n_q or dq % hd or q.dtype is not cache.torch_dtype or q.get_device() != cache.device:
        raise ValueError("q: [len(seqs) * n_q, n_heads * head_dim] of the cache's dtype, on its device")
    sq, u0 = q.stride()
    if u0 != 1:
        raise ValueError("rows must have unit column stride")
    if T == 1:
        sq = dq
    w, sw = _weights(cache, weights)
    cuda = cache.stream(stream)
    if workspace is None:
        key = (B, n_q, dq, shared_len)
        need = cache._weigh_bytes.get(key)
        if need is None:
            need = cache.note(cache._weigh_bytes, key, op_key_weights_workspace_bytes(cache, B, n_q, dq // hd, shared_len))
        buf, ws, nbytes = cache.workspace(need, cuda)
    else:
        buf, ws, nbytes = _given(workspace)
    st = LIB.xc_op_key_weights(cache.ptr, layer, B, cache.int32(seqs, B), n_q, dq // hd, q.data_ptr(), sq,
                               _lse(cache, lse, T, dq // hd), shared_len, causal, scale, decay, w, sw, ws, nbytes, cuda)
    if st:
        check(st)


def op_kv_evict_workspace_bytes(cache: KVCache, n, keep) -> int:
    return LIB.xc_op_kv_evict_workspace_bytes(cache.ptr, n, keep)


def op_kv_evict(cache: KVCache, seqs, keep: int, weights=None, n_first=0, n_last=0, kept=None, workspace=None, stream=None):
    """Shortens every listed sequence that is longer than keep to its first n_first tokens, its last n_last and those of
    the largest weights between (weights as of op_key_weights; None if n_first + n_last == keep).  kept: int32 CUDA tensor
    [len(seqs), keep], receives the tokens that stayed, or None.  workspace: a device tensor of
    op_kv_evict_workspace_bytes, or None for the cache's own."""
    n = seqs.numel()
    w, sw = _weights(cache, weights) if weights is not None else (None, 0)
    cuda = cache.stream(stream)
    if workspace is None:
        need = cache._evict_bytes.get((n, keep))
        if need is None:
            need = cache.note(cache._evict_bytes, (n, keep), op_kv_evict_workspace_bytes(cache, n, keep))
        buf, ws, nbytes = cache.workspace(need, cuda)
    else:
        buf, ws, nbytes = _given(workspace)
    st = LIB.xc_op_kv_evict(cache.ptr, n, cache.int32(seqs, n), keep, n_first, n_last, w, sw,
                            cache.int32(kept, n * keep) if kept is not None else None, ws, nbytes, cuda)
    if st:
        check(st)
