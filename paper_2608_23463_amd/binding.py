"""ctypes binding of libproxyformer.so (the C ABI in include/proxyformer.h).

Argument marshalling only: PyTorch provides device memory (tensor.data_ptr())
and the stream; every step of the computation runs in the library's HIP
kernels. Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libproxyformer.so")
MAX_LEVELS = 4

PF_OK = 0
PF_ERR_INVALID_ARG = -1
PF_ERR_UNSUPPORTED = -2
PF_ERR_CAPACITY = -3
PF_ERR_WORKSPACE = -4
PF_ERR_HIP = -5
PF_FP32 = 0
PF_BF16 = 1
PF_INJECT_GATED = 0
PF_INJECT_ADD = 1
PF_INJECT_AFFINE = 2
PF_INJECT_GATED_HEAD = 3
PF_PRECISION_EXTENDED = 0
PF_PRECISION_BF16 = 1
PF_GATE_SEPARATE = 0
PF_GATE_FUSED = 1
MAX_AXES = 3
PF_NORM_NONE = 0
PF_NORM_RMS = 1
PF_ROPE_HALVES = 0
PF_ROPE_PAIRS = 1

EXPORTS = (
    "proxy_layer_workspace_size", "proxy_layer_saved_size", "proxy_layer_forward",
    "proxy_layer_backward", "proxy_decode_workspace_size", "proxy_decode_step",
    "proxy_cache_append", "proxy_prefill_workspace_size", "proxy_decode_prefill",
    "proxy_last_error", "proxy_version",
    "proxy_trace_enable", "proxy_trace_collect", "proxy_trace_get", "proxy_trace_reset",
    "proxy_ceiling_mfma", "proxy_decode_step_static", "proxy_ceiling_read",
    "proxy_qk_norm_rope_forward", "proxy_qk_workspace_size", "proxy_qk_norm_rope_backward",
    "proxy_paged_append", "proxy_paged_workspace_size", "proxy_paged_attention",
)

c_void_p = ctypes.c_void_p
c_int32 = ctypes.c_int32
c_int64 = ctypes.c_int64
c_size_t = ctypes.c_size_t


class PfLinear(ctypes.Structure):
    _fields_ = [("w", c_void_p), ("b", c_void_p)]


class PfLayerConfig(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("seq_len", c_int64), ("d_fine", c_int32), ("d_proxy", c_int32),
                ("n_heads", c_int32), ("head_dim", c_int32), ("n_levels", c_int32),
                ("factors", c_int32 * MAX_LEVELS), ("level_dims", c_int32 * MAX_LEVELS),
                ("dtype", c_int32), ("mask", c_int32), ("injection", c_int32), ("image_width", c_int32),
                ("precision", c_int32), ("gate_fusion", c_int32)]


class PfLayerWeights(ctypes.Structure):
    _fields_ = [("compress", PfLinear * MAX_LEVELS), ("q", PfLinear), ("k", PfLinear), ("v", PfLinear),
                ("o", PfLinear), ("decompress", PfLinear * MAX_LEVELS), ("gate", PfLinear), ("affine", PfLinear)]


class PfLinearGrad(ctypes.Structure):
    _fields_ = [("dw", c_void_p), ("db", c_void_p)]


class PfLayerGrads(ctypes.Structure):
    _fields_ = [("compress", PfLinearGrad * MAX_LEVELS), ("q", PfLinearGrad), ("k", PfLinearGrad),
                ("v", PfLinearGrad), ("o", PfLinearGrad), ("decompress", PfLinearGrad * MAX_LEVELS),
                ("gate", PfLinearGrad), ("affine", PfLinearGrad)]


class PfDecodeConfig(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("d_model", c_int32), ("n_heads", c_int32), ("head_dim", c_int32),
                ("n_levels", c_int32), ("factors", c_int32 * MAX_LEVELS),
                ("level_dims", c_int32 * MAX_LEVELS), ("dtype", c_int32), ("rms_eps", ctypes.c_float)]


class PfDecodeWeights(ctypes.Structure):
    _fields_ = [("rms_gamma", c_void_p), ("q", PfLinear), ("k", PfLinear), ("v", PfLinear), ("o", PfLinear),
                ("alpha", PfLinear), ("compress", PfLinear * MAX_LEVELS), ("k_proxy", PfLinear),
                ("v_proxy", PfLinear)]


class PfDecodeState(ctypes.Structure):
    _fields_ = [("k_cache", c_void_p), ("v_cache", c_void_p), ("n_cap", c_int64), ("n", c_int64),
                ("x_blk", c_void_p), ("k_loc", c_void_p), ("v_loc", c_void_p), ("j", c_int32),
                ("n_seq", ctypes.POINTER(c_int64)), ("j_seq", ctypes.POINTER(c_int32))]


class PfHeadsConfig(ctypes.Structure):
    _fields_ = [("n_heads", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32), ("dtype", c_int32),
                ("norm", c_int32), ("eps", ctypes.c_float), ("rot_dim", c_int32), ("rope_style", c_int32),
                ("n_axes", c_int32), ("axis_pairs", c_int32 * MAX_AXES)]


class PfHeadsWeights(ctypes.Structure):
    _fields_ = [("gamma_q", c_void_p), ("gamma_k", c_void_p), ("freqs", c_void_p)]


class PfRows(ctypes.Structure):
    _fields_ = [("p", c_void_p), ("token_stride", c_int64), ("head_stride", c_int64)]


class PfPagedCache(ctypes.Structure):
    _fields_ = [("k_pages", c_void_p), ("v_pages", c_void_p), ("n_pages", c_int32), ("page_size", c_int32),
                ("page_table", c_void_p), ("max_pages", c_int32), ("kv_len", c_void_p), ("batch", c_int32)]


_lib = None

# Allocation policy of the helpers below (a test aid): when on, every buffer
# they allocate for the library to write (outputs, gradients, saved
# activations, workspace, decode state slots) starts as all-ones bytes, a NaN
# in both bf16 and fp32, and the decode and prefill workspaces are refilled
# before every call. An element the library fails to write then cannot pass
# a comparison on stale memory that happens to hold a correct value.
_poison = False


def set_poison(on: bool) -> bool:
    """Turn NaN-filled allocation on or off; returns the previous setting."""
    global _poison
    prev, _poison = _poison, bool(on)
    return prev


def _fresh(t):
    """Apply the allocation policy to a new (contiguous) buffer; returns it."""
    if _poison:
        import torch
        t.view(torch.uint8).fill_(255)
    return t


def _fresh_on(t, stream):
    """_fresh with the fill enqueued on `stream` (the stream the library call
    that reads the buffer runs on; None = the current stream)."""
    if _poison and stream is not None:
        import torch
        with torch.cuda.stream(stream):
            return _fresh(t)
    return _fresh(t)


def _empty(shape, dtype, device):
    import torch
    return _fresh(torch.empty(shape, dtype=dtype, device=device))


class ProxyFormerError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"status {status}: {msg}")
        self.status = status


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2608_23463_amd.build.build()")
    # torch first: the library then binds to the HIP runtime torch has loaded
    # (its buffers and streams are torch's). Loaded before torch, the library
    # would map the system runtime and torch its own, two runtimes in one
    # process, and the library's launches fail.
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    lib.proxy_layer_workspace_size.argtypes = [P(PfLayerConfig), c_int32]
    lib.proxy_layer_workspace_size.restype = c_size_t
    lib.proxy_layer_saved_size.argtypes = [P(PfLayerConfig)]
    lib.proxy_layer_saved_size.restype = c_size_t
    lib.proxy_layer_forward.argtypes = [P(PfLayerConfig), P(PfLayerWeights), c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.proxy_layer_forward.restype = c_int32
    lib.proxy_layer_backward.argtypes = [P(PfLayerConfig), P(PfLayerWeights), c_void_p, c_void_p, c_void_p,
                                         c_void_p, c_void_p, c_void_p, c_void_p, P(PfLayerGrads), c_void_p,
                                         c_size_t, c_void_p]
    lib.proxy_layer_backward.restype = c_int32
    lib.proxy_decode_workspace_size.argtypes = [P(PfDecodeConfig)]
    lib.proxy_decode_workspace_size.restype = c_size_t
    lib.proxy_decode_step.argtypes = [P(PfDecodeConfig), P(PfDecodeWeights), P(PfDecodeState), c_void_p,
                                      c_void_p, c_void_p, c_size_t, c_void_p]
    lib.proxy_decode_step.restype = c_int32
    lib.proxy_cache_append.argtypes = [P(PfDecodeConfig), P(PfDecodeWeights), P(PfDecodeState), c_void_p,
                                       c_int64, c_void_p, c_size_t, c_void_p]
    lib.proxy_cache_append.restype = c_int32
    lib.proxy_prefill_workspace_size.argtypes = [P(PfDecodeConfig), c_int64, c_int64]
    lib.proxy_prefill_workspace_size.restype = c_size_t
    lib.proxy_decode_prefill.argtypes = [P(PfDecodeConfig), P(PfDecodeWeights), P(PfDecodeState), c_void_p,
                                         c_int64, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.proxy_decode_prefill.restype = c_int32
    lib.proxy_last_error.argtypes = []
    lib.proxy_last_error.restype = ctypes.c_char_p
    lib.proxy_version.argtypes = []
    lib.proxy_version.restype = c_int32
    lib.proxy_trace_enable.argtypes = [c_int32]
    lib.proxy_trace_enable.restype = c_int32
    lib.proxy_trace_collect.argtypes = []
    lib.proxy_trace_collect.restype = c_int32
    lib.proxy_trace_get.argtypes = [c_int32, ctypes.c_char_p, c_size_t, ctypes.POINTER(c_int64),
                                    ctypes.POINTER(ctypes.c_double)]
    lib.proxy_trace_get.restype = c_int32
    lib.proxy_trace_reset.argtypes = []
    lib.proxy_trace_reset.restype = None
    lib.proxy_ceiling_mfma.argtypes = [c_void_p, c_int64, c_int32, c_void_p]
    lib.proxy_ceiling_mfma.restype = c_int32
    lib.proxy_ceiling_read.argtypes = [c_void_p, ctypes.c_size_t, c_void_p, c_int64, c_void_p]
    lib.proxy_ceiling_read.restype = c_int32
    lib.proxy_decode_step_static.argtypes = [P(PfDecodeConfig), P(PfDecodeWeights), P(PfDecodeState), c_void_p,
                                             c_void_p, c_void_p]
    lib.proxy_decode_step_static.restype = c_int32
    rows = P(PfRows)
    lib.proxy_qk_norm_rope_forward.argtypes = [P(PfHeadsConfig), P(PfHeadsWeights), c_int64, rows, rows, c_void_p,
                                               rows, rows, c_void_p]
    lib.proxy_qk_norm_rope_forward.restype = c_int32
    lib.proxy_qk_workspace_size.argtypes = [P(PfHeadsConfig), c_int64]
    lib.proxy_qk_workspace_size.restype = c_size_t
    lib.proxy_qk_norm_rope_backward.argtypes = [P(PfHeadsConfig), P(PfHeadsWeights), c_int64, rows, rows, c_void_p,
                                                rows, rows, rows, rows, c_void_p, c_void_p, c_void_p, c_size_t,
                                                c_void_p]
    lib.proxy_qk_norm_rope_backward.restype = c_int32
    lib.proxy_paged_append.argtypes = [P(PfHeadsConfig), P(PfHeadsWeights), P(PfPagedCache), c_int64, c_void_p, rows,
                                       rows, rows, c_void_p, rows, c_void_p]
    lib.proxy_paged_append.restype = c_int32
    lib.proxy_paged_workspace_size.argtypes = [P(PfHeadsConfig), c_int32, c_int64, c_int32, c_int64, c_int64, c_int64,
                                               c_int64]
    lib.proxy_paged_workspace_size.restype = c_size_t
    lib.proxy_paged_attention.argtypes = [P(PfHeadsConfig), P(PfPagedCache), c_int64, c_void_p, rows, c_int64, c_int64,
                                          c_int64, c_int64, ctypes.c_float, c_void_p, c_void_p, c_void_p, c_size_t,
                                          c_void_p]
    lib.proxy_paged_attention.restype = c_int32
    _lib = lib
    return lib


def last_error() -> str:
    return load().proxy_last_error().decode()


def _check(status: int):
    if status != PF_OK:
        raise ProxyFormerError(status, last_error())


def ceiling_mfma(out, n_workgroups: int, iters: int, stream=None) -> None:
    """Enqueue the matrix-core ceiling loop (see proxy_ceiling_mfma) on
    `stream` (torch's current stream if None); out is a device float32
    tensor of n_workgroups * 256 elements."""
    if out.numel() < n_workgroups * 256 or out.dtype.itemsize != 4 or not out.is_cuda:
        raise ValueError("out must be a device float32 tensor of n_workgroups * 256 elements")
    _check(load().proxy_ceiling_mfma(c_void_p(out.data_ptr()), n_workgroups, iters, c_void_p(_stream(stream))))


def ceiling_read(src, out, n_workgroups: int, stream=None) -> None:
    """Enqueue the HBM read probe (see proxy_ceiling_read) over all bytes of
    the device tensor src on `stream` (torch's current stream if None); out is
    a device int32 tensor of at least n_workgroups elements."""
    if not src.is_cuda or not src.is_contiguous() or (src.numel() * src.element_size()) % 16 != 0:
        raise ValueError("src must be a contiguous device tensor whose size is a multiple of 16 bytes")
    if out.numel() < n_workgroups or out.element_size() != 4 or not out.is_cuda:
        raise ValueError("out must be a device 32-bit tensor of n_workgroups elements")
    _check(load().proxy_ceiling_read(c_void_p(src.data_ptr()), src.numel() * src.element_size(),
                                     c_void_p(out.data_ptr()), n_workgroups, c_void_p(_stream(stream))))


def trace_enable(on: bool) -> bool:
    return bool(load().proxy_trace_enable(int(on)))


def trace_reset() -> None:
    load().proxy_trace_reset()


def trace_collect() -> Dict[str, tuple]:
    """{label: (launches, total_ms)} of everything traced since the last reset."""
    lib = load()
    n = lib.proxy_trace_collect()
    if n < 0:
        raise ProxyFormerError(n, "trace collection failed")
    out = {}
    buf = ctypes.create_string_buffer(128)
    for i in range(n):
        cnt = c_int64()
        ms = ctypes.c_double()
        _check(lib.proxy_trace_get(i, buf, 128, ctypes.byref(cnt), ctypes.byref(ms)))
        out[buf.value.decode()] = (int(cnt.value), float(ms.value))
    return out


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


# ---------------------------------------------------------------- layer

def layer_config(batch: int, seq_len: int, d_fine: int, d_proxy: int, n_heads: int, head_dim: int,
                 factors: Sequence[int], level_dims: Sequence[int] = (), dtype: str = "bf16",
                 mask: int = 0, injection: int = 0, image_width: int = 0, precision: int = 0,
                 gate_fusion: int = 0) -> PfLayerConfig:
    c = PfLayerConfig()
    c.batch = batch
    c.seq_len = seq_len
    c.d_fine = d_fine
    c.d_proxy = d_proxy
    c.n_heads = n_heads
    c.head_dim = head_dim
    c.n_levels = len(factors)
    for i, k in enumerate(factors):
        c.factors[i] = k
    for i, v in enumerate(level_dims):
        c.level_dims[i] = v
    c.dtype = PF_BF16 if dtype == "bf16" else PF_FP32
    c.mask = mask
    c.injection = injection
    c.image_width = image_width
    c.precision = precision
    c.gate_fusion = gate_fusion
    return c


def config_from_shape(shape) -> PfLayerConfig:
    """PfLayerConfig of a synth.LayerShape."""
    dims = list(shape.level_dims) if shape.level_dims else []
    return layer_config(shape.batch, shape.seq_len, shape.d_fine, shape.d_proxy, shape.n_heads,
                        shape.head_dim, shape.factors, dims, shape.dtype, shape.mask,
                        getattr(shape, "injection", 0), getattr(shape, "image_width", 0),
                        getattr(shape, "precision", 0), getattr(shape, "gate_fusion", 0))


def _lin(pair) -> PfLinear:
    if pair is None:
        return PfLinear(None, None)
    w, b = pair
    return PfLinear(_ptr(w), _ptr(b))


def layer_weights(w: Dict[str, object]) -> PfLayerWeights:
    """Weight struct from {"compress": [(W, b)...], "q": (W, b), ...} of device tensors."""
    s = PfLayerWeights()
    for i, pair in enumerate(w["compress"]):
        s.compress[i] = _lin(pair)
    for i, pair in enumerate(w["decompress"]):
        s.decompress[i] = _lin(pair)
    for name in ("q", "k", "v", "o", "gate", "affine"):
        setattr(s, name, _lin(w.get(name)))
    return s


def layer_workspace_size(cfg: PfLayerConfig, for_backward: bool = False) -> int:
    return int(load().proxy_layer_workspace_size(ctypes.byref(cfg), int(for_backward)))


def layer_saved_size(cfg: PfLayerConfig) -> int:
    return int(load().proxy_layer_saved_size(ctypes.byref(cfg)))


def _bytes(n: int, device):
    import torch
    return _fresh(torch.empty(max(n, 256), dtype=torch.uint8, device=device))


def layer_forward_raw(cfg, wstruct, x, h_in, x_out, h_out, saved, workspace, stream=None):
    """Direct call of proxy_layer_forward on preallocated tensors."""
    ws_bytes = workspace.numel() if workspace is not None else 0
    _check(load().proxy_layer_forward(ctypes.byref(cfg), ctypes.byref(wstruct), _ptr(x), _ptr(h_in),
                                      _ptr(x_out), _ptr(h_out), _ptr(saved), _ptr(workspace), ws_bytes,
                                      _stream(stream)))


def layer_forward(cfg: PfLayerConfig, weights: Dict[str, object], x, h_in=None, save: bool = False,
                  workspace=None, stream=None):
    """Allocate outputs (and workspace), run the forward; returns (x_out, h_out, saved)."""
    import torch
    m = -(-cfg.seq_len // _block(cfg))  # ceil(L / P): a partial last block has a proxy
    x_out = _empty(x.shape, x.dtype, x.device)
    h_out = _empty((cfg.batch, m, cfg.d_proxy), x.dtype, x.device)
    saved = _bytes(layer_saved_size(cfg), x.device) if save else None
    if workspace is None:
        workspace = _bytes(layer_workspace_size(cfg, False), x.device)
    layer_forward_raw(cfg, layer_weights(weights), x, h_in, x_out, h_out, saved, workspace, stream)
    return x_out, h_out, saved


def _block(cfg) -> int:
    p = 1
    for i in range(cfg.n_levels):
        p *= cfg.factors[i]
    return p


def layer_grads(g: Dict[str, object]) -> PfLayerGrads:
    s = PfLayerGrads()

    def lg(pair):
        if pair is None:
            return PfLinearGrad(None, None)
        dw, db = pair
        return PfLinearGrad(_ptr(dw), _ptr(db))

    for i, pair in enumerate(g["compress"]):
        s.compress[i] = lg(pair)
    for i, pair in enumerate(g["decompress"]):
        s.decompress[i] = lg(pair)
    for name in ("q", "k", "v", "o", "gate", "affine"):
        setattr(s, name, lg(g.get(name)))
    return s


def layer_backward(cfg: PfLayerConfig, weights: Dict[str, object], x, h_in, saved, dy, dh_out=None,
                   workspace=None, stream=None):
    """Run the backward; returns (dx, dh_in, grads) with fp32 weight gradients."""
    import torch
    dev = x.device
    dx = _empty(x.shape, x.dtype, dev)
    dh_in = _empty(h_in.shape, h_in.dtype, dev) if h_in is not None else None

    def g_like(pair):
        w, b = pair
        return (_empty(w.shape, torch.float32, dev), _empty((w.shape[0],), torch.float32, dev))

    grads = {"compress": [g_like(p) for p in weights["compress"]],
             "decompress": [g_like(p) for p in weights["decompress"]]}
    for name in ("q", "k", "v", "o"):
        grads[name] = g_like(weights[name])
    # the gate is only read (and differentiated) by gated injection
    grads["gate"] = g_like(weights["gate"]) if cfg.injection in (PF_INJECT_GATED, PF_INJECT_GATED_HEAD) else None
    grads["affine"] = g_like(weights["affine"]) if cfg.injection == PF_INJECT_AFFINE else None
    if workspace is None:
        workspace = _bytes(layer_workspace_size(cfg, True), dev)
    _check(load().proxy_layer_backward(ctypes.byref(cfg), ctypes.byref(layer_weights(weights)), _ptr(x),
                                       _ptr(h_in), _ptr(saved), _ptr(dy), _ptr(dh_out), _ptr(dx), _ptr(dh_in),
                                       ctypes.byref(layer_grads(grads)), _ptr(workspace), workspace.numel(),
                                       _stream(stream)))
    return dx, dh_in, grads


# ---------------------------------------------------------------- decode

def decode_config(batch: int, d_model: int, n_heads: int, head_dim: int, factors: Sequence[int],
                  level_dims: Sequence[int] = (), dtype: str = "bf16", rms_eps: float = 1e-6) -> PfDecodeConfig:
    c = PfDecodeConfig()
    c.batch = batch
    c.d_model = d_model
    c.n_heads = n_heads
    c.head_dim = head_dim
    c.n_levels = len(factors)
    for i, k in enumerate(factors):
        c.factors[i] = k
    for i, v in enumerate(level_dims):
        c.level_dims[i] = v
    c.dtype = PF_BF16 if dtype == "bf16" else PF_FP32
    c.rms_eps = rms_eps
    return c


def decode_weights(w: Dict[str, object]) -> PfDecodeWeights:
    s = PfDecodeWeights()
    s.rms_gamma = _ptr(w["rms_gamma"])
    for name in ("q", "k", "v", "o", "alpha", "k_proxy", "v_proxy"):
        setattr(s, name, _lin(w[name]))
    for i, pair in enumerate(w["compress"]):
        s.compress[i] = _lin(pair)
    return s


class DecodeSession:
    """Caller-owned decode state on the device plus the host counters n, j.

    With ``ragged=True`` every sequence keeps its own position: ``n_seq`` and
    ``j_seq`` (host int64 / int32 arrays of batch entries) replace n and j."""

    def __init__(self, cfg: PfDecodeConfig, weights: Dict[str, object], k_cache, v_cache, n: int = 0,
                 device="cuda", ragged: bool = False, n_seq=None, j_seq=None):
        import torch
        self.cfg = cfg
        self.weights = weights            # keeps the device tensors alive
        self.wstruct = decode_weights(weights)
        p = _block(cfg)
        dt = k_cache.dtype
        self.k_cache = k_cache
        self.v_cache = v_cache
        # slots at or past j are never read: they start as NaN under poisoning
        self.x_blk = _fresh(torch.zeros((cfg.batch, p, cfg.d_model), dtype=dt, device=device))
        self.k_loc = _fresh(torch.zeros((cfg.batch, cfg.n_heads, p, cfg.head_dim), dtype=dt, device=device))
        self.v_loc = _fresh(torch.zeros_like(self.k_loc))
        self.state = PfDecodeState(k_cache.data_ptr(), v_cache.data_ptr(), k_cache.shape[2], n,
                                   self.x_blk.data_ptr(), self.k_loc.data_ptr(), self.v_loc.data_ptr(), 0)
        self.n_seq = self.j_seq = None
        if ragged:
            import numpy as np
            # own copies: the library advances these counters in place
            self.n_seq = np.array(np.full(cfg.batch, n) if n_seq is None else n_seq, dtype=np.int64, copy=True)
            self.j_seq = np.array(np.zeros(cfg.batch) if j_seq is None else j_seq, dtype=np.int32, copy=True)
            self.state.n_seq = self.n_seq.ctypes.data_as(ctypes.POINTER(c_int64))
            self.state.j_seq = self.j_seq.ctypes.data_as(ctypes.POINTER(c_int32))
        self.workspace = _bytes(int(load().proxy_decode_workspace_size(ctypes.byref(cfg))), device)

    @property
    def n(self) -> int:
        return int(self.state.n)

    @property
    def j(self) -> int:
        return int(self.state.j)

    def step(self, x_t, y_t=None, stream=None):
        if y_t is None:
            y_t = _empty(x_t.shape, x_t.dtype, x_t.device)
        _fresh_on(self.workspace, stream)
        _check(load().proxy_decode_step(ctypes.byref(self.cfg), ctypes.byref(self.wstruct),
                                        ctypes.byref(self.state), _ptr(x_t), _ptr(y_t),
                                        _ptr(self.workspace), self.workspace.numel(), _stream(stream)))
        return y_t

    def step_static(self, x_t, y_t=None, stream=None):
        """The same step through proxy_decode_step_static (no workspace)."""
        if y_t is None:
            y_t = _empty(x_t.shape, x_t.dtype, x_t.device)
        _check(load().proxy_decode_step_static(ctypes.byref(self.cfg), ctypes.byref(self.wstruct),
                                               ctypes.byref(self.state), _ptr(x_t), _ptr(y_t), _stream(stream)))
        return y_t

    def prefill(self, x, y=None, stream=None):
        """Parallel form of the generation block over x [B, T, d] (the next T
        tokens of every sequence, from a block boundary); returns y [B, T, d].
        The prefill workspace is allocated on first use and grown as needed."""
        if y is None:
            y = _empty(x.shape, x.dtype, x.device)
        lib = load()
        need = int(lib.proxy_prefill_workspace_size(ctypes.byref(self.cfg), x.shape[1], self.state.n_cap))
        if need == 0:
            raise ProxyFormerError(-2, "prefill sizes beyond the library's limits")
        if getattr(self, "prefill_ws", None) is None or self.prefill_ws.numel() < need:
            self.prefill_ws = _bytes(need, x.device)
        _fresh_on(self.prefill_ws, stream)
        _check(lib.proxy_decode_prefill(ctypes.byref(self.cfg), ctypes.byref(self.wstruct), ctypes.byref(self.state),
                                        _ptr(x), x.shape[1], _ptr(y), _ptr(self.prefill_ws),
                                        self.prefill_ws.numel(), _stream(stream)))
        return y

    def append(self, x_blocks, nblk: int, stream=None):
        _fresh_on(self.workspace, stream)
        _check(load().proxy_cache_append(ctypes.byref(self.cfg), ctypes.byref(self.wstruct),
                                         ctypes.byref(self.state), _ptr(x_blocks), nblk,
                                         _ptr(self.workspace), self.workspace.numel(), _stream(stream)))


# ---------------------------------------------------------------- heads

def heads_config(n_heads: int, n_kv_heads: int, head_dim: int, dtype: str = "bf16", norm: bool = True,
                 eps: float = 1e-6, rot_dim: Optional[int] = None, style: int = PF_ROPE_HALVES,
                 axis_pairs: Sequence[int] = ()) -> PfHeadsConfig:
    """Heads of the fine tokens' own attention. rot_dim: elements that are
    turned (all of head_dim unless given); axis_pairs: pairs that turn by each
    coordinate of a position (one coordinate unless given)."""
    if dtype not in ("bf16", "fp32"):
        raise ValueError("dtype must be 'bf16' or 'fp32'")
    if len(axis_pairs) > MAX_AXES:
        raise ValueError(f"at most {MAX_AXES} axes")
    c = PfHeadsConfig()
    c.n_heads = n_heads
    c.n_kv_heads = n_kv_heads
    c.head_dim = head_dim
    c.dtype = PF_BF16 if dtype == "bf16" else PF_FP32
    c.norm = PF_NORM_RMS if norm else PF_NORM_NONE
    c.eps = eps
    c.rot_dim = head_dim if rot_dim is None else rot_dim
    c.rope_style = style
    pairs = list(axis_pairs) if len(axis_pairs) else [c.rot_dim // 2]
    c.n_axes = len(pairs)
    for i, n in enumerate(pairs):
        c.axis_pairs[i] = n
    return c


def rope_freqs(cfg: PfHeadsConfig, base: float = 10000.0, device="cuda"):
    """freqs [rot_dim / 2] fp64: base ** (-p / n) for pair p of an axis' n pairs."""
    import torch
    return torch.cat([base ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))
                      for n in cfg.axis_pairs[:cfg.n_axes]]).to(device)


def _heads_dtype(cfg):
    import torch
    return torch.bfloat16 if cfg.dtype == PF_BF16 else torch.float32


def _want(name, t, dtype, device, shape, contiguous=True):
    """Data pointer of a tensor of a call, whose type, place and shape (None:
    any size) are as told."""
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on the call's GPU {device}, got {t.device}")
    if t.shape != shape and (t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape))):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(cfg, name, t, n, heads, device) -> PfRows:
    """The rows of a tensor [tokens, heads, head_dim]; only a row itself must be contiguous."""
    dtype, shape = _heads_dtype(cfg), (n, heads, cfg.head_dim)
    if t.dtype != dtype or t.shape != shape or t.device != device:
        _want(name, t, dtype, device, shape, contiguous=False)  # raises
    ts, hs, es = t.stride()
    if es != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    return PfRows(t.data_ptr(), ts if n > 1 else 0, hs if heads > 1 else 0)


def _heads_weights(cfg, weights: Dict[str, object], device) -> PfHeadsWeights:
    import torch
    s = PfHeadsWeights()
    for name in ("gamma_q", "gamma_k"):
        t = weights.get(name)
        if t is not None:
            setattr(s, name, _want(name, t, _heads_dtype(cfg), device, (cfg.head_dim,)))
    t = weights.get("freqs")
    if t is not None:
        s.freqs = _want("freqs", t, torch.float64, device, (cfg.rot_dim // 2,))
    return s


def _positions(cfg, positions, n, device):
    import torch
    if positions is None:
        return None
    if positions.dim() == 1:
        positions = positions[None]
    return _want("positions", positions, torch.int32, device, (cfg.n_axes, n))


def _workspace(t, device):
    """Data pointer and bytes of a call's workspace (None, 0 without one)."""
    if t is None:
        return None, 0
    if t.device != device:
        raise ValueError(f"workspace must be on the call's GPU {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _elsewhere(device, stream):
    """None where a call on `device` with `stream` (None: the current one) can
    go out as it is; else the context that makes that GPU and stream current,
    for kernels and for buffers allocated on the way."""
    import torch
    if device.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, got {device}")
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"the stream belongs to {stream.device}, the tensors to {device}")
        return torch.cuda.stream(stream)
    return None if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _current(device) -> int:
    """The device's current stream."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def qk_norm_rope_forward(cfg: PfHeadsConfig, weights: Dict[str, object], q, k, positions=None, q_out=None, k_out=None,
                         stream=None):
    """Queries [T, n_heads, head_dim] and keys [T, n_kv_heads, head_dim]
    normed per head and turned by positions (int32 [n_axes, T] or [T]);
    weights {"gamma_q", "gamma_k", "freqs"}. Returns (q_out, k_out)."""
    dev, n = q.device, q.shape[0]
    ctx = _elsewhere(dev, stream)
    if ctx is not None:
        with ctx:
            return qk_norm_rope_forward(cfg, weights, q, k, positions, q_out, k_out)
    w = _heads_weights(cfg, weights, dev)
    rq, rk = _rows(cfg, "q", q, n, cfg.n_heads, dev), _rows(cfg, "k", k, n, cfg.n_kv_heads, dev)
    at = _positions(cfg, positions, n, dev)
    if q_out is None:
        q_out = _empty(q.shape, q.dtype, dev)
    if k_out is None:
        k_out = _empty(k.shape, k.dtype, dev)
    ro, rp = _rows(cfg, "q_out", q_out, n, cfg.n_heads, dev), _rows(cfg, "k_out", k_out, n, cfg.n_kv_heads, dev)
    _check(load().proxy_qk_norm_rope_forward(cfg, w, n, rq, rk, at, ro, rp, _current(dev)))
    return q_out, k_out


def qk_norm_rope_backward(cfg: PfHeadsConfig, weights: Dict[str, object], q, k, positions, dq_out, dk_out, dq=None,
                          dk=None, workspace=None, stream=None):
    """Gradients of qk_norm_rope_forward's q and k (of their dtype) and of the
    gains (fp32; None without a norm). q and k are the forward's inputs."""
    import torch
    dev, n = dq_out.device, dq_out.shape[0]
    ctx = _elsewhere(dev, stream)
    if ctx is not None:
        with ctx:
            return qk_norm_rope_backward(cfg, weights, q, k, positions, dq_out, dk_out, dq, dk, workspace)
    lib = load()
    norm = cfg.norm == PF_NORM_RMS
    w = _heads_weights(cfg, weights, dev)
    rq = rk = None
    if norm:
        rq, rk = _rows(cfg, "q", q, n, cfg.n_heads, dev), _rows(cfg, "k", k, n, cfg.n_kv_heads, dev)
    at = _positions(cfg, positions, n, dev)
    ro = _rows(cfg, "dq_out", dq_out, n, cfg.n_heads, dev)
    rp = _rows(cfg, "dk_out", dk_out, n, cfg.n_kv_heads, dev)
    if dq is None:
        dq = _empty(dq_out.shape, dq_out.dtype, dev)
    if dk is None:
        dk = _empty(dk_out.shape, dk_out.dtype, dev)
    da, db = _rows(cfg, "dq", dq, n, cfg.n_heads, dev), _rows(cfg, "dk", dk, n, cfg.n_kv_heads, dev)
    gq = gk = None
    ws, ws_bytes = None, 0
    if norm:
        gq, gk = _empty((2, cfg.head_dim), torch.float32, dev).unbind()
        if workspace is None:
            workspace = _bytes(int(lib.proxy_qk_workspace_size(cfg, n)), dev)
        ws, ws_bytes = _workspace(workspace, dev)
    _check(lib.proxy_qk_norm_rope_backward(cfg, w, n, rq, rk, at, ro, rp, da, db, _ptr(gq), _ptr(gk), ws, ws_bytes,
                                           _current(dev)))
    return dq, dk, gq, gk


class PagedCache:
    """A cache of the fine tokens' keys and values in pages (one per layer).

    k_pages, v_pages [n_pages, n_kv_heads, page_size, head_dim]; page_table
    int32 [batch, max_pages] and kv_len int32 [batch] on the device, the
    caller's own: it hands out pages and sets kv_len (the new tokens counted)
    before a step's append, and the step's attention reads the same lengths.
    cfg and weights are taken as they are when the cache is made: later changes
    of the config or of the dict's entries do not reach it."""

    def __init__(self, cfg: PfHeadsConfig, weights: Dict[str, object], k_pages, v_pages, page_table, kv_len):
        import torch
        dev, dt = k_pages.device, _heads_dtype(cfg)
        if dev.type != "cuda":
            raise ValueError(f"tensors must be on a GPU, got {dev}")
        shape = (k_pages.shape[0], cfg.n_kv_heads, None, cfg.head_dim)
        batch = kv_len.shape[0]
        self.cfg = PfHeadsConfig.from_buffer_copy(cfg)
        self.device = dev
        self.tensors = (k_pages, v_pages, page_table, kv_len)  # kept alive, like the weights as they are now
        self.weights = dict(weights)
        self.batch = batch
        self.wstruct = _heads_weights(cfg, weights, dev)
        self.state = PfPagedCache(_want("k_pages", k_pages, dt, dev, shape),
                                  _want("v_pages", v_pages, dt, dev, tuple(k_pages.shape)), k_pages.shape[0],
                                  k_pages.shape[2], _want("page_table", page_table, torch.int32, dev, (batch, None)),
                                  page_table.shape[1], _want("kv_len", kv_len, torch.int32, dev, (batch,)), batch)

    def append(self, k, v, q=None, cu_tokens=None, positions=None, q_out=None, stream=None):
        """New tokens' keys and values [T, n_kv_heads, head_dim] into the pages,
        and their queries [T, n_heads, head_dim] normed and turned into q_out
        (returned). cu_tokens int32 [batch + 1]: which tokens are whose (None:
        one of every sequence); positions as in qk_norm_rope_forward (None:
        the tokens' rows). Tokens without a place are left alone: pass a
        q_out of your own where that can be."""
        import torch
        cfg, dev, n = self.cfg, self.device, k.shape[0]
        ctx = _elsewhere(dev, stream)
        if ctx is not None:
            with ctx:
                return self.append(k, v, q, cu_tokens, positions, q_out)
        rk, rv = _rows(cfg, "k", k, n, cfg.n_kv_heads, dev), _rows(cfg, "v", v, n, cfg.n_kv_heads, dev)
        cu = None if cu_tokens is None else _want("cu_tokens", cu_tokens, torch.int32, dev, (self.batch + 1,))
        at = _positions(cfg, positions, n, dev)
        rq = ro = None
        if q is not None:
            rq = _rows(cfg, "q", q, n, cfg.n_heads, dev)
            if q_out is None:
                q_out = _empty(q.shape, q.dtype, dev)
            ro = _rows(cfg, "q_out", q_out, n, cfg.n_heads, dev)
        elif q_out is not None:
            raise ValueError("q_out without q")
        _check(load().proxy_paged_append(cfg, self.wstruct, self.state, n, cu, rq, rk, rv, at, ro, _current(dev)))
        return q_out

    def attend(self, q, max_kv_len: int, cu_tokens=None, max_new: Optional[int] = None, window: int = 0,
               sinks: int = 0, scale: Optional[float] = None, out=None, lse=None, workspace=None, stream=None):
        """Attention of new tokens, q [T, n_heads, head_dim] laid out as append's,
        over the rows up to their own: all of them, or (window > 0) the last
        `window` and the first `sinks`. max_kv_len, max_new: most rows and new
        tokens of a sequence, to lay the launch out for (max_new: 1 without
        cu_tokens, T with it unless given; bf16 prompts laid out for 32 or more
        round their weights to bf16, for 31 or fewer keep them in two terms,
        more exact and slower). scale: 1 / sqrt(head_dim) unless
        given. lse: an fp32 [T, n_heads] tensor for the log-sums. workspace: a
        byte tensor that no call running at the same time uses (allocated
        unless given). Returns out; rows of tokens behind the last sequence are
        left alone."""
        import torch
        cfg, dev, n = self.cfg, self.device, q.shape[0]
        ctx = _elsewhere(dev, stream)
        if ctx is not None:
            with ctx:
                return self.attend(q, max_kv_len, cu_tokens, max_new, window, sinks, scale, out, lse, workspace)
        lib = load()
        if max_new is None:
            max_new = 1 if cu_tokens is None else max(n, 1)
        rq = _rows(cfg, "q", q, n, cfg.n_heads, dev)
        cu = None if cu_tokens is None else _want("cu_tokens", cu_tokens, torch.int32, dev, (self.batch + 1,))
        shape = (n, cfg.n_heads, cfg.head_dim)
        if out is None:
            out = _empty(shape, q.dtype, dev)
        to = _want("out", out, q.dtype, dev, shape)
        tl = None if lse is None else _want("lse", lse, torch.float32, dev, (n, cfg.n_heads))
        if workspace is None:
            need = lib.proxy_paged_workspace_size(cfg, self.batch, n, cu is not None, max_new, max_kv_len, window, sinks)
            workspace = _bytes(need, dev) if need else None
        ws, ws_bytes = _workspace(workspace, dev)
        _check(lib.proxy_paged_attention(cfg, self.state, n, cu, rq, max_new, max_kv_len, window, sinks,
                                         cfg.head_dim ** -0.5 if scale is None else scale, to, tl, ws, ws_bytes,
                                         _current(dev)))
        return out
