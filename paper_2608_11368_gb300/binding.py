"""ctypes binding of libpair.so for torch tensors: argument marshalling only.

The functions carry the C-ABI names (include/pair.h). Every step of the
estimator runs in the library's CUDA kernels; this module only checks
tensor placement/dtypes, allocates outputs with torch when the caller does
not pass them, and forwards raw device pointers plus the current CUDA stream.
There is no CPU fallback: if libpair.so is missing, importing the binding's
library raises.
"""
from __future__ import annotations

import ctypes
import os
import re

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libpair.so")
HEADER = os.path.join(os.path.dirname(_PKG), "include", "pair.h")

PAIR_OK = 0
PAIR_F32, PAIR_BF16 = 0, 1
PAIR_CENTER = 1
PAIR_STANDARDIZE = 2
STATUS_NAMES = {0: "PAIR_OK", 1: "PAIR_ERR_INVALID_ARG", 2: "PAIR_ERR_UNSUPPORTED",
                3: "PAIR_ERR_WORKSPACE", 4: "PAIR_ERR_NONPOSITIVE_INCLUSION",
                5: "PAIR_ERR_TARGET_RANGE", 6: "PAIR_ERR_CUDA",
                7: "PAIR_ERR_DEVICE_TIMEOUT", 8: "PAIR_ERR_ALLOC_INPUT",
                9: "PAIR_ERR_ALLOC_INFEASIBLE", 10: "PAIR_ERR_PAGES",
                11: "PAIR_ERR_PROBABILITY"}


class PairError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (%s)" % (where, STATUS_NAMES.get(status, status),
                                          pair_status_string(status)))


class CacheStrides(ctypes.Structure):
    """pair_cache_strides (include/pair.h), in elements."""
    _fields_ = [("for_page", ctypes.c_int64), ("for_token", ctypes.c_int64),
                ("for_head", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libpair.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libpair.so is not built (run __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, I64, F32, U32, SZ = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                 ctypes.c_float, ctypes.c_uint32, ctypes.c_size_t)
    L.pair_coeffs.argtypes = [I32, I32, P, P, P, F32, U32, P, P, P, P, P, P]
    L.pair_coeffs.restype = ctypes.c_int
    L.pair_estimate_dense.argtypes = [I32, I32, I32, P, P, P, P, F32, P, P, P, P]
    L.pair_estimate_dense.restype = ctypes.c_int
    L.pair_grad_workspace_size.argtypes = [I64, I32, I32, I32, ctypes.c_int]
    L.pair_grad_workspace_size.restype = SZ
    L.pair_grad_workspace_min_size.argtypes = [I64, I32, I32, I32, ctypes.c_int]
    L.pair_grad_workspace_min_size.restype = SZ
    L.pair_grad.argtypes = [I64, I32, I32, ctypes.c_int, P, P, P, P, P, I32, P,
                            P, P, P, P, P, SZ, P, P]
    L.pair_grad.restype = ctypes.c_int
    L.pair_status_sync.argtypes = [P, P]
    L.pair_status_sync.restype = ctypes.c_int
    L.pair_status_string.argtypes = [ctypes.c_int]
    L.pair_status_string.restype = ctypes.c_char_p
    L.pair_last_launch_count.argtypes = []
    L.pair_last_launch_count.restype = I32
    L.pair_grad_clipped.argtypes = [I64, I32, I32, ctypes.c_int, P, P, P, P, P, I32, P, P, F32,
                                    P, P, P, P, P, P, SZ, P, P]
    L.pair_grad_clipped.restype = ctypes.c_int
    L.pair_grad_noalloc.argtypes = [I64, I32, I32, ctypes.c_int, P, P, P, P, P,
                                    I32, P, P, P, P, P, P, P]
    L.pair_grad_noalloc.restype = ctypes.c_int
    L.pair_timing_enable.argtypes = [I32]
    L.pair_timing_enable.restype = None
    L.pair_timing_read.argtypes = [I32, P, P]
    L.pair_timing_read.restype = I32
    L.pair_coeffs_weighted.argtypes = [I32, I32, P, P, P, F32, U32, ctypes.c_int, F32,
                                       P, P, P, P, P, P, P, P]
    L.pair_coeffs_weighted.restype = ctypes.c_int
    L.pair_coeffs_product.argtypes = [I32, I32, P, P, P, F32, U32, P, P, P, P, P, P, P, P]
    L.pair_coeffs_product.restype = ctypes.c_int
    L.pair_audit_workspace_size.argtypes = [I32, I32, I32]
    L.pair_audit_workspace_size.restype = SZ
    L.pair_audit.argtypes = [I32, I32, I32, P, P, P, P, P, F32, U32, ctypes.c_int, F32, P, P,
                             P, SZ, P, P]
    L.pair_audit.restype = ctypes.c_int
    L.pair_allocate.argtypes = [I32, I32, P, P, P, P, P, F32, P, P, P, P]
    L.pair_allocate.restype = ctypes.c_int
    L.pair_grad_token_logp.argtypes = [I64, I32, I32, I32, ctypes.c_int, P, SZ, P, P]
    L.pair_grad_token_logp.restype = ctypes.c_int
    L.pair_pages_extend.argtypes = [I32, I32, I32, P, P, P, P, I32, P, I64, P, P, P, P, P, P, P,
                                    P]
    L.pair_pages_extend.restype = ctypes.c_int
    L.pair_cache_append.argtypes = [I64, I32, I32, ctypes.c_int, P, I64, I64, P, I64, I64, P, I32,
                                    I32, P, CacheStrides, P, CacheStrides, P, P]
    L.pair_cache_append.restype = ctypes.c_int
    L.pair_attend_workspace_size.argtypes = [I32, I32, I32, I32, ctypes.c_int]
    L.pair_attend_workspace_size.restype = SZ
    L.pair_attend_paged.argtypes = [I64, I32, I32, I32, I32, ctypes.c_int, P, I64, I64, P,
                                    CacheStrides, P, CacheStrides, I32, I32, P, I32, P, P, F32,
                                    I32, P, P, P, SZ, P, P]
    L.pair_attend_paged.restype = ctypes.c_int
    L.pair_verify_drafts.argtypes = [I64, I32, I32, ctypes.c_int, P, I64, P, I64, P, P, P, P, P,
                                     P, P, P, P]
    L.pair_verify_drafts.restype = ctypes.c_int
    L.pair_selftest_wait_timeout.argtypes = [I64, P, P, P]
    L.pair_selftest_wait_timeout.restype = ctypes.c_int
    _lib = L
    return L


def header_functions():
    """Names of the functions declared in include/pair.h."""
    txt = open(HEADER).read()
    return sorted(set(re.findall(r"^\s*(?:[\w\s\*]+?)\b(pair_\w+)\s*\(", txt,
                                 flags=re.M)))


def pair_status_string(status: int) -> str:
    return lib().pair_status_string(int(status)).decode()


def pair_last_launch_count() -> int:
    return int(lib().pair_last_launch_count())


def pair_timing_enable(on: bool) -> None:
    """Start (or stop) recording per-kernel CUDA events for this thread."""
    lib().pair_timing_enable(1 if on else 0)


def pair_timing_read(max_launches: int = 4096):
    """[(kernel name, milliseconds)] of the launches recorded since the last
    enable/read (waits for their events)."""
    ms = (ctypes.c_float * max_launches)()
    names = (ctypes.c_char_p * max_launches)()
    n = lib().pair_timing_read(max_launches, ms, names)
    return [(names[i].decode(), float(ms[i])) for i in range(n)]


# Device pointers and streams go to the library as plain integers (the
# functions' argtypes convert them; None is a null pointer). A call on a small
# batch is over in a few microseconds on the GPU, so the path to it is kept
# short: coefficients of 8 x 8 groups took 24 us with a context manager for the
# device, a stream object and a c_void_p per argument, 17 us without.
def _p(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _need(t, name, dtype, shape=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape),
                                                            tuple(t.shape)))


def _check(st, where):
    if st != PAIR_OK:
        raise PairError(st, where)


def _on_device(t):
    """Context manager making t's device current for the call: the library
    launches on the current device and takes its stream from there."""
    return torch.cuda.device(t.device)


def _call(where, t, stream, *args):
    """Library function `where` with args and the stream, on t's device (made
    current for the call if it is not): `stream`, or that device's current
    one. Raises PairError for any status but PAIR_OK."""
    fn = getattr(_lib or lib(), where)
    dev = t.get_device()
    if dev == torch._C._cuda_getDevice():
        st = fn(*args, torch._C._cuda_getCurrentRawStream(dev) if stream is None
                else stream.cuda_stream)
    else:
        with _on_device(t):
            st = fn(*args, _stream(stream))
    if st != PAIR_OK:
        raise PairError(st, where)


def _out(t, name, shape, dtype, dev):
    """Caller-passed output (checked) or a fresh torch allocation."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    _need(t, name, dtype, shape)
    if t.device != dev:
        raise ValueError("%s must be on %s, got %s" % (name, dev, t.device))
    return t


def pair_coeffs(r, J, rho, scale=1.0, flags=0, a=None, active=None, edges=None,
                contrast_edges=None, dev_err=None, stream=None):
    """Coefficients of Eq. (pair-advantage) (times `scale`, see pair.h), on
    r's device. Returns (a, active, edges, contrast_edges)."""
    B, G = r.shape
    dev = r.device
    _need(r, "r", torch.float32)
    _need(J, "J", torch.uint8, (B, G))
    _need(rho, "rho", torch.float32, (B, G, G))
    a = _out(a, "a", (B, G), torch.float32, dev)
    active = _out(active, "active", (B, G), torch.uint8, dev)
    edges = _out(edges, "edges", (B,), torch.int32, dev)
    contrast_edges = _out(contrast_edges, "contrast_edges", (B,), torch.int32, dev)
    _call("pair_coeffs", r, stream, B, G, _p(r), _p(J), _p(rho), float(scale), int(flags),
          _p(a), _p(active), _p(edges), _p(contrast_edges), _p(dev_err))
    return a, active, edges, contrast_edges


PAIR_W_HT, PAIR_W_UNWEIGHTED, PAIR_W_MARGINAL, PAIR_W_CLIPPED, PAIR_W_HAJEK = 0, 1, 2, 3, 4


def _coeffs_outputs(B, G, dev, a, active, edges, contrast_edges, ess, max_w):
    return (_out(a, "a", (B, G), torch.float32, dev),
            _out(active, "active", (B, G), torch.uint8, dev),
            _out(edges, "edges", (B,), torch.int32, dev),
            _out(contrast_edges, "contrast_edges", (B,), torch.int32, dev),
            _out(ess, "ess", (B,), torch.float32, dev),
            _out(max_w, "max_w", (B,), torch.float32, dev))


def pair_coeffs_weighted(r, J, rho, wmode=PAIR_W_HT, w_max=0.0, scale=1.0, flags=0, a=None,
                         active=None, edges=None, contrast_edges=None, ess=None, max_w=None,
                         dev_err=None, stream=None):
    """pair_coeffs under a weighting variant (see pair.h), with per-group ESS
    and largest weight. Returns (a, active, edges, contrast_edges, ess, max_w)."""
    B, G = r.shape
    _need(r, "r", torch.float32)
    _need(J, "J", torch.uint8, (B, G))
    if rho is not None:
        _need(rho, "rho", torch.float32, (B, G, G))
    outs = _coeffs_outputs(B, G, r.device, a, active, edges, contrast_edges, ess, max_w)
    _call("pair_coeffs_weighted", r, stream, B, G, _p(r), _p(J), _p(rho), float(scale),
          int(flags), int(wmode), float(w_max), *[_p(t) for t in outs], _p(dev_err))
    return outs


def pair_coeffs_product(r, J, p, scale=1.0, flags=0, a=None, active=None, edges=None,
                        contrast_edges=None, ess=None, max_w=None, dev_err=None, stream=None):
    """Coefficients of the independent design rho_ij = p_i p_j from the
    marginals p [B, G]. Returns (a, active, edges, contrast_edges, ess, max_w)."""
    B, G = r.shape
    _need(r, "r", torch.float32)
    _need(J, "J", torch.uint8, (B, G))
    _need(p, "p", torch.float32, (B, G))
    outs = _coeffs_outputs(B, G, r.device, a, active, edges, contrast_edges, ess, max_w)
    _call("pair_coeffs_product", r, stream, B, G, _p(r), _p(J), _p(p), float(scale), int(flags),
          *[_p(t) for t in outs], _p(dev_err))
    return outs


AUDIT_STATS = ("bias_norm", "mse", "cos", "vertices", "edges", "ess", "target_sq", "weight")


def pair_audit(r, rho, S, Jdraws, draw_weight=None, wmode=PAIR_W_HT, w_max=0.0, scale=1.0,
               flags=0, stats=None, bias=None, ws=None, dev_err=None, stream=None):
    """Frozen-population audit of one group over design draws (see pair.h).
    r [G], rho [G, G] (None for PAIR_W_UNWEIGHTED), S [G, D], Jdraws [N, G]
    uint8, draw_weight [N] float64 or None. Returns (stats [8] f64, bias [D] f64)."""
    N, G = Jdraws.shape
    D = S.shape[1]
    _need(r, "r", torch.float32, (G,))
    if rho is not None:
        _need(rho, "rho", torch.float32, (G, G))
    _need(S, "S", torch.float32, (G, D))
    _need(Jdraws, "Jdraws", torch.uint8, (N, G))
    if draw_weight is not None:
        _need(draw_weight, "draw_weight", torch.float64, (N,))
    dev = r.device
    stats = _out(stats, "stats", (8,), torch.float64, dev)
    bias = _out(bias, "bias", (D,), torch.float64, dev)
    need = int(lib().pair_audit_workspace_size(N, G, D))
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    _need(ws, "ws", torch.uint8)
    _call("pair_audit", r, stream, N, G, D, _p(r), _p(rho), _p(S), _p(Jdraws), _p(draw_weight),
          float(scale), int(flags), int(wmode), float(w_max), _p(stats), _p(bias), _p(ws),
          ws.numel(), _p(dev_err))
    return stats, bias


ALLOC_OK, ALLOC_SLACK, ALLOC_FLOOR, ALLOC_INFEASIBLE, ALLOC_FALLBACK, ALLOC_FLAT, \
    ALLOC_INVALID = range(7)
ALLOC_STATS = ("phi", "spent", "gap", "newton", "status")


def pair_allocate(c_hat, budget, pi_min, p_hat=None, m_hat=None, a=None, pi=None, stats=None,
                  dev_err=None, stream=None):
    """Continuation probabilities of the convex design (see pair.h).
    c_hat [B, G], budget [B], p_hat [B, G] (or a [B, G, G]), m_hat [B, G] or
    None. Returns (pi [B, G] f32, stats [B, 5] f64: phi, spent, gap, newton,
    status)."""
    B, G = c_hat.shape
    _need(c_hat, "c_hat", torch.float32, (B, G))
    _need(budget, "budget", torch.float32, (B,))
    if p_hat is not None:
        _need(p_hat, "p_hat", torch.float32, (B, G))
    if m_hat is not None:
        _need(m_hat, "m_hat", torch.float32, (B, G))
    if a is not None:
        _need(a, "a", torch.float32, (B, G, G))
    dev = c_hat.device
    pi = _out(pi, "pi", (B, G), torch.float32, dev)
    stats = _out(stats, "stats", (B, 5), torch.float64, dev)
    if dev_err is None:
        dev_err = torch.zeros(1, dtype=torch.int32, device=dev)
    _call("pair_allocate", c_hat, stream, B, G, _p(p_hat), _p(m_hat), _p(a), _p(c_hat),
          _p(budget), float(pi_min), _p(pi), _p(stats), _p(dev_err))
    return pi, stats


def pair_estimate_dense(r, J, rho, S, scale=1.0, g=None, a=None, dev_err=None,
                        stream=None):
    """Eq. (pair-ht) for explicit scores S [B,G,D], on S's device. Returns (g, a)."""
    B, G, D = S.shape
    _need(r, "r", torch.float32, (B, G))
    _need(J, "J", torch.uint8, (B, G))
    _need(rho, "rho", torch.float32, (B, G, G))
    _need(S, "S", torch.float32)
    g = _out(g, "g", (B, D), torch.float32, S.device)
    if a is not None:
        a = _out(a, "a", (B, G), torch.float32, S.device)
    _call("pair_estimate_dense", S, stream, B, G, D, _p(r), _p(J), _p(rho), _p(S), float(scale),
          _p(g), _p(a), _p(dev_err))
    return g, a


def pair_grad_workspace_size(T, d, V, R, dtype) -> int:
    return int(lib().pair_grad_workspace_size(int(T), int(d), int(V), int(R),
                                              int(dtype)))


def pair_grad_workspace_min_size(T, d, V, R, dtype) -> int:
    return int(lib().pair_grad_workspace_min_size(int(T), int(d), int(V), int(R),
                                                  int(dtype)))


def _pair_dtype(t, name="H/W"):
    if t.dtype == torch.bfloat16:
        return PAIR_BF16
    if t.dtype == torch.float32:
        return PAIR_F32
    raise TypeError("%s must be bfloat16 or float32" % name)


def _grad_inputs(H, W, y, mask, cu_seqlens, a):
    T, d = H.shape
    V = W.shape[0]
    R = cu_seqlens.numel() - 1
    dt = _pair_dtype(H)
    _need(H, "H", H.dtype, (T, d))
    _need(W, "W", H.dtype, (V, d))
    _need(y, "y", torch.int32, (T,))
    _need(mask, "mask", torch.uint8, (T,))
    _need(cu_seqlens, "cu_seqlens", torch.int32, (R + 1,))
    _need(a, "a", torch.float32, (R,))
    for t, nm in ((W, "W"), (y, "y"), (mask, "mask"), (cu_seqlens, "cu_seqlens"), (a, "a")):
        if t.device != H.device:
            raise ValueError("%s must be on %s like H, got %s" % (nm, H.device, t.device))
    return T, d, V, R, dt


def _grad_outputs(T, d, V, R, dev, dH, dW, Jobj, logp_seq):
    return (_out(dH, "dH", (T, d), torch.float32, dev), _out(dW, "dW", (V, d), torch.float32, dev),
            _out(Jobj, "Jobj", (1,), torch.float64, dev),
            _out(logp_seq, "logp_seq", (R,), torch.float32, dev))


def pair_grad(H, W, y, mask, cu_seqlens, a, dH=None, dW=None, Jobj=None,
              logp_seq=None, ws=None, dev_err=None, stream=None):
    """LM-head realisation of sum_i a_i log pi(o_i|q) and its gradients.
    Runs on H's device. Returns (Jobj [1] f64, dH [T,d] f32, dW [V,d] f32,
    logp_seq [R] f32)."""
    T, d, V, R, dt = _grad_inputs(H, W, y, mask, cu_seqlens, a)
    dev = H.device
    dH, dW, Jobj, logp_seq = _grad_outputs(T, d, V, R, dev, dH, dW, Jobj, logp_seq)
    if ws is None:
        need = pair_grad_workspace_size(T, d, V, R, dt)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    _need(ws, "ws", torch.uint8)
    _call("pair_grad", H, stream, T, d, V, dt, _p(H), _p(W), _p(y), _p(mask), _p(cu_seqlens), R,
          _p(a), _p(dH), _p(dW), _p(Jobj), _p(logp_seq), _p(ws), ws.numel(), _p(dev_err))
    return Jobj, dH, dW, logp_seq


def pair_grad_token_logp(T, d, V, R, dtype, ws, logp_tok=None, stream=None):
    """Per-token log-probabilities [T] left in `ws` by the last pair_grad (or
    pair_grad_clipped) call with these shapes (see pair.h): logp_t for active
    tokens, 0 elsewhere."""
    _need(ws, "ws", torch.uint8)
    logp_tok = _out(logp_tok, "logp_tok", (int(T),), torch.float32, ws.device)
    _call("pair_grad_token_logp", ws, stream, int(T), int(d), int(V), int(R), int(dtype), _p(ws),
          ws.numel(), _p(logp_tok))
    return logp_tok


def pair_grad_clipped(H, W, y, mask, cu_seqlens, a, logp_old, clip_eps=0.2, dH=None, dW=None,
                      Jobj=None, logp_seq=None, coef=None, ws=None, dev_err=None, stream=None):
    """Clipped trajectory-ratio surrogate (see pair.h). Runs on H's device.
    Returns (Jobj [1] f64, dH [T,d] f32, dW [V,d] f32, logp_seq [R] f32, coef [R] f32)."""
    T, d, V, R, dt = _grad_inputs(H, W, y, mask, cu_seqlens, a)
    _need(logp_old, "logp_old", torch.float32, (R,))
    dev = H.device
    dH, dW, Jobj, logp_seq = _grad_outputs(T, d, V, R, dev, dH, dW, Jobj, logp_seq)
    coef = _out(coef, "coef", (R,), torch.float32, dev)
    if ws is None:
        need = pair_grad_workspace_size(T, d, V, R, dt)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    _need(ws, "ws", torch.uint8)
    _call("pair_grad_clipped", H, stream, T, d, V, dt, _p(H), _p(W), _p(y), _p(mask),
          _p(cu_seqlens), R, _p(a), _p(logp_old), float(clip_eps), _p(dH), _p(dW), _p(Jobj),
          _p(logp_seq), _p(coef), _p(ws), ws.numel(), _p(dev_err))
    return Jobj, dH, dW, logp_seq, coef


NOALLOC_MAX_WORKSPACE = 32 << 20


def pair_grad_noalloc(H, W, y, mask, cu_seqlens, a, dH=None, dW=None,
                      Jobj=None, logp_seq=None, dev_err=None, stream=None):
    """pair_grad on the library's fixed device workspace (no workspace
    argument; see pair.h for the size limit and the sharing rules). Runs on
    H's device. Output tensors not passed in are allocated here by torch, as
    in pair_grad; pass all four (checked for shape, dtype and device) to keep
    the call allocation-free. Returns (Jobj, dH, dW, logp_seq)."""
    T, d, V, R, dt = _grad_inputs(H, W, y, mask, cu_seqlens, a)
    dev = H.device
    dH, dW, Jobj, logp_seq = _grad_outputs(T, d, V, R, dev, dH, dW, Jobj, logp_seq)
    _call("pair_grad_noalloc", H, stream, T, d, V, dt, _p(H), _p(W), _p(y), _p(mask),
          _p(cu_seqlens), R, _p(a), _p(dH), _p(dW), _p(Jobj), _p(logp_seq), _p(dev_err))
    return Jobj, dH, dW, logp_seq


# The rollout step's calls are made once per generated chunk and a small one is
# over in a few microseconds on the GPU, so each tensor is checked by one
# expression; what fails it goes through the checks that say why.
def _index(t, name):
    """Index of the device that a call's leading tensor is on."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    return t.get_device()


def _same_device(like, name, t):
    if t.device != like.device:
        raise ValueError("%s must be on %s, got %s" % (name, like.device, t.device))


def _ptr(t, name, dtype, shape, like, at):
    """Pointer of a contiguous tensor on like's device, whose index is `at`."""
    if not (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape
            and t.is_contiguous() and t.get_device() == at):
        _need(t, name, dtype, shape)
        _same_device(like, name, t)
    return t.data_ptr()


def _fresh(shape, dtype, like, stream):
    """Tensor on like's device, of the memory of the stream that will write it:
    memory of another one may still be in use there, or be given out again there
    before the call has run."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _out_ptr(t, name, dtype, shape, like, at, stream):
    """Output tensor (allocated where it is None) and its pointer."""
    if t is None:
        t = _fresh(shape, dtype, like, stream)
        return t, t.data_ptr()
    return t, _ptr(t, name, dtype, shape, like, at)


def _err_ptr(dev_err, like, at):
    return None if dev_err is None else _ptr(dev_err, "dev_err", torch.int32, (1,), like, at)


def _strided(t, name, dtype, shape, like, at):
    """Pointer of a tensor on like's device whose last dimension is contiguous
    (rows of a wider array are fine); the library checks alignment."""
    if not (type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape
            and t.get_device() == at and t.stride(-1) == 1):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError("%s must be a CUDA tensor" % name)
        if t.dtype is not dtype:
            raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
        if t.shape != shape:
            raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape),
                                                                tuple(t.shape)))
        _same_device(like, name, t)
        if t.stride(-1) != 1 and t.shape[-1] != 1:
            raise ValueError("%s must be contiguous in its last dimension" % name)
    return t.data_ptr()


def _cache(k_cache, v_cache, like, at):
    """Pointers and strides of both caches, their shape."""
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be [num_pages, page_size, Hkv, D]")
    shape, dtype = k_cache.shape, like.dtype
    k, v = (_strided(k_cache, "k_cache", dtype, shape, like, at),
            _strided(v_cache, "v_cache", dtype, shape, like, at))
    return (k, CacheStrides(*k_cache.stride()[:3]), v, CacheStrides(*v_cache.stride()[:3]), shape)


def pair_pages_extend(lens, held, n_new, free_pages, free_count, block_table, page_size, T,
                      kv_len=None, held_out=None, cu_new=None, slots=None, taken=None,
                      dev_err=None, stream=None):
    """Pages and slots of a step's new tokens (see pair.h). lens, held, n_new
    [R], free_pages [F], free_count [1], block_table [R, width], all int32;
    block_table gets the new pages in place. Returns (kv_len [R], held_out
    [R], cu_new [R+1], slots [T] int64, taken [1])."""
    R, width = block_table.shape
    i32, T, at, per = torch.int32, int(T), _index(lens, "lens"), (R,)
    F = free_pages.numel()
    ins = (_ptr(lens, "lens", i32, per, lens, at), _ptr(held, "held", i32, per, lens, at),
           _ptr(n_new, "n_new", i32, per, lens, at),
           _ptr(free_pages, "free_pages", i32, (F,), lens, at))
    count = _ptr(free_count, "free_count", i32, (1,), lens, at)
    table = _ptr(block_table, "block_table", i32, (R, width), lens, at)
    kv_len, kv_p = _out_ptr(kv_len, "kv_len", i32, per, lens, at, stream)
    held_out, held_p = _out_ptr(held_out, "held_out", i32, per, lens, at, stream)
    cu_new, cu_p = _out_ptr(cu_new, "cu_new", i32, (R + 1,), lens, at, stream)
    slots, slots_p = _out_ptr(slots, "slots", torch.int64, (T,), lens, at, stream)
    taken, taken_p = _out_ptr(taken, "taken", i32, (1,), lens, at, stream)
    _call("pair_pages_extend", lens, stream, R, int(page_size), width, *ins, F, count, T, table,
          kv_p, held_p, cu_p, slots_p, taken_p, _err_ptr(dev_err, lens, at))
    return kv_len, held_out, cu_new, slots, taken


def pair_cache_append(k, v, slots, k_cache, v_cache, dev_err=None, stream=None):
    """Keys and values k, v [T, Hkv, D] into their slots [T] (int64, -1: left
    out) of the caches [num_pages, page_size, Hkv, D] (see pair.h). k, v and
    the caches may be views with other strides. Returns (k_cache, v_cache)."""
    T, H, D = k.shape
    dt, at = _pair_dtype(k, "k"), _index(k, "k")
    kp, vp = (_strided(k, "k", k.dtype, (T, H, D), k, at),
              _strided(v, "v", k.dtype, (T, H, D), k, at))
    slots_p = _ptr(slots, "slots", torch.int64, (T,), k, at)
    kc, ks, vc, vs, shape = _cache(k_cache, v_cache, k, at)
    if shape[2] != H or shape[3] != D:
        raise ValueError("k_cache must have %d heads of %d, got %s" % (H, D, tuple(shape)))
    _call("pair_cache_append", k, stream, T, H, D, dt, kp, k.stride(0), k.stride(1), vp,
          v.stride(0), v.stride(1), slots_p, shape[0], shape[1], kc, ks, vc, vs,
          _err_ptr(dev_err, k, at))
    return k_cache, v_cache


def pair_attend_workspace_size(R, Hq, Hkv, D, dtype) -> int:
    return int(lib().pair_attend_workspace_size(int(R), int(Hq), int(Hkv), int(D), int(dtype)))


def pair_attend_paged(q, k_cache, v_cache, block_table, kv_len, cu_new, scale=None, max_new=0,
                      out=None, lse=None, ws=None, dev_err=None, stream=None):
    """Attention of every request's chunk of new tokens over its paged cache
    (see pair.h). q [T, Hq, D], caches [num_pages, page_size, Hkv, D] (views
    with other strides too), block_table [R, width], kv_len [R], cu_new [R+1]
    int32; scale is D ** -0.5 by default; max_new is the longest chunk if the
    host knows it. Returns (out [T, Hq, D], lse [T, Hq] float32)."""
    T, Hq, D = q.shape
    dt, at, i32 = _pair_dtype(q, "q"), _index(q, "q"), torch.int32
    qp = _strided(q, "q", q.dtype, (T, Hq, D), q, at)
    kc, ks, vc, vs, shape = _cache(k_cache, v_cache, q, at)
    if shape[3] != D:
        raise ValueError("k_cache must have heads of %d, got %s" % (D, tuple(shape)))
    R, width = block_table.shape
    table = _ptr(block_table, "block_table", i32, (R, width), q, at)
    lens = _ptr(kv_len, "kv_len", i32, (R,), q, at)
    cu = _ptr(cu_new, "cu_new", i32, (R + 1,), q, at)
    out, out_p = _out_ptr(out, "out", q.dtype, (T, Hq, D), q, at, stream)
    lse, lse_p = _out_ptr(lse, "lse", torch.float32, (T, Hq), q, at, stream)
    if ws is None:
        need = pair_attend_workspace_size(R, Hq, shape[2], D, dt)
        ws = _fresh((max(need, 256),), torch.uint8, q, stream)
    n = ws.numel()
    _call("pair_attend_paged", q, stream, T, R, Hq, shape[2], D, dt, qp, q.stride(0), q.stride(1),
          kc, ks, vc, vs, shape[0], shape[1], table, width, lens, cu,
          D ** -0.5 if scale is None else float(scale), int(max_new), out_p, lse_p,
          _ptr(ws, "ws", torch.uint8, (n,), q, at), n, _err_ptr(dev_err, q, at))
    return out, lse


def pair_verify_drafts(p, ids, cu_new, u, u_draw, q=None, out_ids=None, logp=None, n_emit=None,
                       dev_err=None, stream=None):
    """Drafted tokens against the target's probabilities p [T, V], and the
    token that follows (see pair.h). ids [T], cu_new [R+1] int32; u [T], u_draw
    [R] float32; q [T, V] the drafter's probabilities, or None for drafts that
    were looked up. Returns (out_ids [T] int32, logp [T] float32, n_emit [R]
    int32)."""
    T, V = p.shape
    dt, at, i32, f32 = _pair_dtype(p, "p"), _index(p, "p"), torch.int32, torch.float32
    pp = _strided(p, "p", p.dtype, (T, V), p, at)
    qp, q_row = (None, 0) if q is None else (_strided(q, "q", p.dtype, (T, V), p, at), q.stride(0))
    R = cu_new.numel() - 1
    ids_p = _ptr(ids, "ids", i32, (T,), p, at)
    cu = _ptr(cu_new, "cu_new", i32, (R + 1,), p, at)
    up, dp = _ptr(u, "u", f32, (T,), p, at), _ptr(u_draw, "u_draw", f32, (R,), p, at)
    out_ids, out_p = _out_ptr(out_ids, "out_ids", i32, (T,), p, at, stream)
    logp, logp_p = _out_ptr(logp, "logp", f32, (T,), p, at, stream)
    n_emit, n_p = _out_ptr(n_emit, "n_emit", i32, (R,), p, at, stream)
    _call("pair_verify_drafts", p, stream, T, R, V, dt, pp, p.stride(0), qp, q_row, ids_p, cu, up,
          dp, out_p, logp_p, n_p, _err_ptr(dev_err, p, at))
    return out_ids, logp, n_emit


def pair_selftest_wait_timeout(limit_cycles, dev_err, seen, stream=None):
    """Launch the bounded-wait failure-path check (see pair.h)."""
    _need(dev_err, "dev_err", torch.int32)
    _need(seen, "seen", torch.int32, (2,))
    st = lib().pair_selftest_wait_timeout(int(limit_cycles), _p(dev_err), _p(seen),
                                          _stream(stream))
    _check(st, "pair_selftest_wait_timeout")


def pair_status_sync(dev_err=None, stream=None) -> int:
    """Synchronise the stream and decode/reset the device error word (on
    dev_err's device when it is given)."""
    if dev_err is None:
        return int(lib().pair_status_sync(_stream(stream), None))
    with _on_device(dev_err):
        return int(lib().pair_status_sync(_stream(stream), _p(dev_err)))
