"""Python binding of the C ABI in include/mca.h (ctypes; argument marshalling only).

Every step of the trial loop runs in libmca.so's CUDA kernels. PyTorch provides device memory
(the library's workspace is a torch tensor) and the stream. There is no CPU fallback: if the
library is missing or no GPU is present, the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import (POINTER, Structure, c_char_p, c_double, c_float, c_int8, c_int32, c_int64,
                    c_size_t, c_uint8, c_uint32, c_uint64, c_void_p)
from contextlib import contextmanager
from typing import NamedTuple, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmca.so")

MCA_OK, MCA_ERR_INVALID, MCA_ERR_CUDA, MCA_ERR_OOM, MCA_ERR_TIMEOUT, MCA_ERR_NUMERIC, \
    MCA_ERR_UNSUPPORTED = range(7)
ACT = {"identity": 0, "tanh": 1, "sigmoid": 2, "relu": 3, "gaussian": 4, "gelu": 5}
LOSS = {"mse_onehot": 0, "softmax_ce": 1}
WKIND = {"fp32": 0, "ternary_i8": 1, "masked_fp32": 2}
OP = {"replace": 0, "perturb": 1}
DTYPE = {"float32": 0, "float16": 1, "bfloat16": 2}
MAX_TOP = 32


class mca_layer(Structure):
    _fields_ = [("n_in", c_int32), ("n_out", c_int32), ("act", c_int32), ("act_param", c_float),
                ("wkind", c_int32), ("scale", c_float)]


class mca_domain(Structure):
    _fields_ = [("op", c_int32), ("lo", c_float), ("hi", c_float), ("delta", c_float),
                ("bound", c_float), ("strict", c_int32), ("temperature", c_float),
                ("layer_stretch", c_int32)]


class mca_dataset(Structure):
    _fields_ = [("x", c_void_p), ("y", c_void_p), ("n", c_int64), ("d", c_int32)]


class mca_options(Structure):
    _fields_ = [("K", c_int32), ("resync_period", c_int32), ("stream", c_void_p),
                ("trace_cap", c_int32), ("grid", c_int32), ("workspace", c_void_p),
                ("workspace_bytes", c_size_t), ("fixed_K", c_int32)]


class mca_tfm_spec(Structure):
    _fields_ = [("vocab", c_int32), ("ctx", c_int32), ("d_model", c_int32), ("n_layer", c_int32),
                ("n_head", c_int32), ("d_ff", c_int32), ("act", c_int32), ("act_param", c_float),
                ("ln_eps", c_float)]


class mca_run_stats(Structure):
    _fields_ = [("trials", c_uint64), ("accepts", c_uint64), ("candidates", c_uint64),
                ("batches", c_uint64), ("wasted", c_uint64), ("forced", c_uint64),
                ("resyncs", c_uint64), ("launches", c_uint64), ("tau", c_uint64), ("S", c_double),
                ("alg_bytes", c_uint64), ("phase_ns", c_uint64 * 8), ("alg_flops", c_uint64),
                ("tensor_cores", c_uint32), ("reserved", c_uint32)]

    def asdict(self):
        d = {f: getattr(self, f) for f, _ in self._fields_ if f != "phase_ns"}
        d["phase_ns"] = list(self.phase_ns)
        return d


class mca_trace_rec(Structure):
    _fields_ = [("tau", c_uint64), ("idx", c_uint32), ("accept", c_int32), ("old_w", c_float),
                ("new_w", c_float), ("valid", c_int32), ("forced", c_int32), ("dS", c_double),
                ("S", c_double)]


class mca_code_linear_args(Structure):
    _fields_ = [("rows", c_int64), ("n_in", c_int32), ("n_out", c_int32), ("x", c_void_p),
                ("ldx", c_int64), ("x_scale", c_void_p), ("w", c_void_p), ("ldw", c_int64),
                ("w_scale", c_void_p), ("bias", c_void_p), ("y", c_void_p), ("ldy", c_int64),
                ("dtype", c_int32), ("act", c_int32), ("act_param", c_float),
                ("workspace", c_void_p), ("workspace_bytes", c_size_t), ("stream", c_void_p)]


class mca_token_logprobs_args(Structure):
    _fields_ = [("logits", c_void_p), ("dtype", c_int32), ("vocab", c_int32), ("rows", c_int64),
                ("ld", c_int64), ("targets", c_void_p), ("logprob", c_void_p),
                ("entropy", c_void_p), ("lse", c_void_p), ("top", c_int32),
                ("top_logprob", c_void_p), ("top_index", c_void_p), ("stream", c_void_p)]


class mca_token_logprobs_backward_args(Structure):
    _fields_ = [("logits", c_void_p), ("dtype", c_int32), ("vocab", c_int32), ("rows", c_int64),
                ("ld", c_int64), ("targets", c_void_p), ("lse", c_void_p), ("entropy", c_void_p),
                ("g_logprob", c_void_p), ("g_entropy", c_void_p), ("grad", c_void_p),
                ("ldg", c_int64), ("stream", c_void_p)]


TRACE_DTYPE = np.dtype([("tau", np.uint64), ("idx", np.uint32), ("accept", np.int32),
                        ("old_w", np.float32), ("new_w", np.float32), ("valid", np.int32),
                        ("forced", np.int32), ("dS", np.float64), ("S", np.float64)])
assert TRACE_DTYPE.itemsize == ctypes.sizeof(mca_trace_rec)

# Every function the header declares, with its ctypes signature.
SIGNATURES = {
    "mca_workspace_size": (c_int32, [POINTER(mca_layer), c_int32, c_int32, POINTER(mca_dataset),
                                     POINTER(mca_options), POINTER(c_size_t)]),
    "mca_create": (c_int32, [POINTER(mca_layer), c_int32, c_int32, POINTER(mca_domain),
                             POINTER(mca_dataset), c_void_p, POINTER(mca_options),
                             POINTER(c_void_p)]),
    "mca_tfm_workspace_size": (c_int32, [POINTER(mca_tfm_spec), c_int64, POINTER(mca_options),
                                         POINTER(c_size_t)]),
    "mca_create_transformer": (c_int32, [POINTER(mca_tfm_spec), POINTER(mca_domain), c_void_p,
                                         c_int64, c_void_p, POINTER(mca_options),
                                         POINTER(c_void_p)]),
    "mca_run": (c_int32, [c_void_p, c_uint64, c_uint64, POINTER(mca_run_stats)]),
    "mca_loss": (c_int32, [c_void_p, POINTER(c_double)]),
    "mca_get_params": (c_int32, [c_void_p, c_void_p, c_size_t]),
    "mca_get_codes": (c_int32, [c_void_p, c_void_p, c_size_t]),
    "mca_set_params": (c_int32, [c_void_p, c_void_p, c_void_p, c_size_t, c_uint64]),
    "mca_resync": (c_int32, [c_void_p]),
    "mca_get_trace": (c_int32, [c_void_p, c_void_p, c_size_t, POINTER(c_size_t)]),
    "mca_force_decisions": (c_int32, [c_void_p, c_void_p, c_void_p, c_size_t]),
    "mca_get_stats": (c_int32, [c_void_p, POINTER(mca_run_stats)]),
    "mca_eval_candidates": (c_int32, [c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "mca_eval_candidates_noalloc": (c_int32, [c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "mca_eval_trials": (c_int32, [c_void_p, c_uint64, c_uint64, c_size_t, c_void_p]),
    "mca_decide_batch": (c_int32, [c_void_p, c_uint64, c_uint64, c_size_t, c_void_p, c_void_p,
                                   c_int64, POINTER(c_int32)]),
    "mca_run_channels": (c_int32, [c_void_p, c_uint64, c_uint64, c_int32, c_void_p, c_void_p]),
    "mca_selftest_wait_timeout": (c_int32, [POINTER(c_int32), POINTER(c_double)]),
    "mca_quantize_rows": (c_int32, [c_void_p, c_int32, c_int64, c_int64, c_int64, c_void_p,
                                    c_int64, c_void_p, c_void_p]),
    "mca_code_linear_workspace_size": (c_int32, [POINTER(mca_code_linear_args),
                                                 POINTER(c_size_t)]),
    "mca_code_linear": (c_int32, [POINTER(mca_code_linear_args)]),
    "mca_token_logprobs": (c_int32, [POINTER(mca_token_logprobs_args)]),
    "mca_token_logprobs_backward": (c_int32, [POINTER(mca_token_logprobs_backward_args)]),
    "mca_score": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                            c_void_p]),
    "mca_predict_workspace_size": (c_int32, [c_void_p, c_int64, POINTER(c_size_t)]),
    "mca_predict": (c_int32, [c_void_p, c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_size_t]),
    "mca_destroy": (None, [c_void_p]),
    "mca_last_error": (c_char_p, [c_void_p]),
}

_lib = None


def load_library(path: str = LIB_PATH):
    """Load libmca.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        lib = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


class MCAError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"mca status {status}: {msg}")
        self.status = status


def _check(status: int, handle=None):
    if status != MCA_OK:
        msg = load_library().mca_last_error(handle)
        raise MCAError(status, msg.decode() if msg else "")


def _ptr(a):
    """Address of a torch tensor or numpy array (host or device), keeping it contiguous."""
    import torch
    if isinstance(a, torch.Tensor):
        assert a.is_contiguous()
        return a.data_ptr()
    assert isinstance(a, np.ndarray) and a.flags.c_contiguous
    return a.ctypes.data


def _layers(layers) -> "ctypes.Array":
    arr = (mca_layer * len(layers))()
    for k, L in enumerate(layers):
        arr[k] = mca_layer(L.n_in, L.n_out, ACT[L.act], float(L.act_param), WKIND[L.wkind],
                           float(L.scale))
    return arr


def _domain(d) -> mca_domain:
    beta = float(getattr(d, "beta", float("inf")))
    if not beta > 0.0:
        raise ValueError(f"beta = {beta}: the selection intensity must be > 0 (inf: greedy rule)")
    return mca_domain(OP[d.op], d.lo, d.hi, d.delta, d.bound, int(bool(d.strict)),
                      0.0 if beta == float("inf") else 1.0 / beta,
                      int(getattr(d, "layer_stretch", 0)))


class Handle:
    """Owns one mca_handle plus the torch tensors the library borrows (workspace, dataset)."""

    def __init__(self, ptr, keep, stream=0, rows=0, classes=0, n_in=0):
        self.ptr = ptr
        self._keep = keep
        self.stream = stream or 0        # cudaStream_t of the handle's work
        self.rows, self.classes = rows, classes     # samples or predicted positions, and their classes
        self.n_in = n_in                 # MLP: input features

    def close(self):
        if self.ptr:
            load_library().mca_destroy(self.ptr)
            self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def mca_workspace_size(layers, loss: str, X, y, K: int = 32, trace_cap: int = 0,
                       stream=None) -> int:
    lib = load_library()
    L = _layers(layers)
    ds = mca_dataset(_ptr(X), _ptr(y), int(X.shape[0]), int(X.shape[1]))
    opt = mca_options(K, 0, stream, trace_cap, 0, None, 0, 0)
    out = c_size_t(0)
    _check(lib.mca_workspace_size(L, len(layers), LOSS[loss], ctypes.byref(ds), ctypes.byref(opt),
                                  ctypes.byref(out)))
    return out.value


def mca_create(layers, loss: str, domain, X, y, init, K: int = 32, resync_period: int = 0,
               trace_cap: int = 0, grid: int = 0, stream=None, torch_workspace: bool = True,
               fixed_K: bool = False):
    """X: [N, D] float32, y: [N] int32, init: [P] float32 -- torch tensors (CUDA or CPU) or numpy
    arrays. The workspace is a torch CUDA tensor the handle keeps alive."""
    import torch
    lib = load_library()
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    L = _layers(layers)
    dom = _domain(domain)
    ds = mca_dataset(_ptr(X), _ptr(y), int(X.shape[0]), int(X.shape[1]))
    keep = [X, y, init]
    ws_ptr, ws_bytes = None, 0
    if torch_workspace:
        nbytes = mca_workspace_size(layers, loss, X, y, K, trace_cap, stream)
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
        base = ws.data_ptr()
        ws_ptr = (base + 255) // 256 * 256
        ws_bytes = nbytes
        keep.append(ws)
    opt = mca_options(K, resync_period, stream, trace_cap, grid, ws_ptr, ws_bytes, int(fixed_K))
    h = c_void_p(None)
    _check(lib.mca_create(L, len(layers), LOSS[loss], ctypes.byref(dom), ctypes.byref(ds),
                          _ptr(init), ctypes.byref(opt), ctypes.byref(h)))
    return Handle(h, keep, stream, int(X.shape[0]), int(layers[-1].n_out), int(layers[0].n_in))


def _tfm_spec(sp) -> mca_tfm_spec:
    return mca_tfm_spec(sp.vocab, sp.ctx, sp.d_model, sp.n_layer, sp.n_head, sp.d_ff, ACT[sp.act],
                        float(sp.act_param), float(sp.ln_eps))


def mca_tfm_workspace_size(spec, n_seq: int, K: int = 32, trace_cap: int = 0) -> int:
    opt = mca_options(K, 0, None, trace_cap, 0, None, 0, 0)
    out = c_size_t(0)
    sp = _tfm_spec(spec)
    _check(load_library().mca_tfm_workspace_size(ctypes.byref(sp), n_seq, ctypes.byref(opt),
                                                 ctypes.byref(out)))
    return out.value


def mca_create_transformer(spec, domain, tokens, init, K: int = 32, resync_period: int = 0,
                           trace_cap: int = 0, stream=None, fixed_K: bool = False):
    """tokens: [B, ctx + 1] int32, init: [P] float32 (torch tensors or numpy arrays, host or
    device). The workspace is a torch CUDA tensor the handle keeps alive."""
    import torch
    lib = load_library()
    if stream is None:
        stream = torch.cuda.current_stream().cuda_stream
    n_seq = int(tokens.shape[0])
    nbytes = mca_tfm_workspace_size(spec, n_seq, K, trace_cap)
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
    ws_ptr = (ws.data_ptr() + 255) // 256 * 256
    opt = mca_options(K, resync_period, stream, trace_cap, 0, ws_ptr, nbytes, int(fixed_K))
    sp = _tfm_spec(spec)
    dom = _domain(domain)
    h = c_void_p(None)
    _check(lib.mca_create_transformer(ctypes.byref(sp), ctypes.byref(dom), _ptr(tokens), n_seq,
                                      _ptr(init), ctypes.byref(opt), ctypes.byref(h)))
    return Handle(h, [tokens, init, ws], stream, n_seq * int(spec.ctx), int(spec.vocab))


def create_from_tfm_workload(wl, device: bool = True, **kw) -> Handle:
    import torch
    tokens, init = wl.tokens, wl.init
    if device:
        tokens = torch.from_numpy(tokens).cuda()
        init = torch.from_numpy(init).cuda()
    kw.setdefault("K", wl.K)
    return mca_create_transformer(wl.spec, wl.domain, tokens, init, **kw)


def mca_run(h: Handle, n_trials: int, seed: int) -> dict:
    st = mca_run_stats()
    _check(load_library().mca_run(h.ptr, n_trials, seed, ctypes.byref(st)), h.ptr)
    return st.asdict()


def mca_loss(h: Handle) -> float:
    v = c_double(0.0)
    _check(load_library().mca_loss(h.ptr, ctypes.byref(v)), h.ptr)
    return v.value


def mca_get_params(h: Handle, P: int, out=None):
    """Effective weights [P] float32 into `out` (numpy or torch, host or device) or a new array."""
    dst = np.empty(P, np.float32) if out is None else out
    _check(load_library().mca_get_params(h.ptr, _ptr(dst), P), h.ptr)
    return dst


def mca_get_codes(h: Handle, P: int) -> np.ndarray:
    dst = np.empty(P, np.int8)
    _check(load_library().mca_get_codes(h.ptr, dst.ctypes.data, P), h.ptr)
    return dst


def mca_set_params(h: Handle, params, codes=None, tau: int = 0):
    P = int(params.shape[0])
    _check(load_library().mca_set_params(h.ptr, _ptr(params),
                                         None if codes is None else _ptr(codes), P, tau), h.ptr)


def mca_resync(h: Handle):
    _check(load_library().mca_resync(h.ptr), h.ptr)


def mca_get_trace(h: Handle, cap: int) -> np.ndarray:
    buf = np.zeros(cap, TRACE_DTYPE)
    n = c_size_t(0)
    _check(load_library().mca_get_trace(h.ptr, buf.ctypes.data, cap, ctypes.byref(n)), h.ptr)
    return buf[:n.value]


def mca_force_decisions(h: Handle, taus: Sequence[int], accepts: Sequence[bool]):
    t = np.ascontiguousarray(np.asarray(taus, dtype=np.uint64))
    a = np.ascontiguousarray(np.asarray(accepts, dtype=np.uint8))
    _check(load_library().mca_force_decisions(h.ptr, t.ctypes.data if len(t) else None,
                                              a.ctypes.data if len(a) else None, len(t)), h.ptr)


def mca_get_stats(h: Handle) -> dict:
    st = mca_run_stats()
    _check(load_library().mca_get_stats(h.ptr, ctypes.byref(st)), h.ptr)
    return st.asdict()


def mca_eval_candidates(h: Handle, flat_idx, new_w) -> np.ndarray:
    idx = np.ascontiguousarray(np.asarray(flat_idx, dtype=np.uint32))
    nw = np.ascontiguousarray(np.asarray(new_w, dtype=np.float32))
    out = np.zeros(len(idx), np.float64)
    _check(load_library().mca_eval_candidates(h.ptr, idx.ctypes.data, nw.ctypes.data, len(idx),
                                              out.ctypes.data), h.ptr)
    return out


def mca_eval_candidates_noalloc(h: Handle, flat_idx, new_w, dS):
    """flat_idx (int32/uint32 bits), new_w (float32) and dS (float64): CUDA tensors of equal length
    owned by the caller; the library allocates nothing for this call."""
    n = int(flat_idx.numel())
    _check(load_library().mca_eval_candidates_noalloc(h.ptr, flat_idx.data_ptr(), new_w.data_ptr(),
                                                      n, dS.data_ptr()), h.ptr)
    return dS


def mca_eval_trials(h: Handle, seed: int, tau: int, n: int) -> np.ndarray:
    """Proposals of trials tau .. tau+n-1 and their loss changes on this handle's samples (no
    commit): a structured array of TRACE_DTYPE records."""
    buf = np.zeros(n, TRACE_DTYPE)
    _check(load_library().mca_eval_trials(h.ptr, seed, tau, n, buf.ctypes.data), h.ptr)
    return buf


def mca_decide_batch(h: Handle, seed: int, tau: int, valid, dS, n_samples: int = 0) -> int:
    """Index of the accepted trial of a batch under the handle's rule (Eq. 6 / Eq. 7), -1 if none."""
    v = np.ascontiguousarray(np.asarray(valid, dtype=np.uint8))
    d = np.ascontiguousarray(np.asarray(dS, dtype=np.float64))
    k = c_int32(-1)
    _check(load_library().mca_decide_batch(h.ptr, seed, tau, len(v), v.ctypes.data, d.ctypes.data,
                                           n_samples, ctypes.byref(k)), h.ptr)
    return k.value


CHANNEL = {"he": 0, "zero": 1}


def mca_run_channels(h: Handle, n_trials: int, seed: int, scheme: str):
    """Channel-mutation trials (Section 2.3); returns (accepted [n] bool, dS [n] float64)."""
    acc = np.zeros(n_trials, np.uint8)
    dS = np.zeros(n_trials, np.float64)
    _check(load_library().mca_run_channels(h.ptr, n_trials, seed, CHANNEL[scheme],
                                           acc.ctypes.data, dS.ctypes.data), h.ptr)
    return acc.astype(bool), dS


def mca_selftest_wait_timeout():
    """(status recorded by the kernel, host milliseconds): the trial loop's bounded grid barrier
    waiting for a peer CTA that never arrives must give up with MCA_ERR_TIMEOUT."""
    st, ms = ctypes.c_int32(-1), ctypes.c_double(0.0)
    _check(load_library().mca_selftest_wait_timeout(ctypes.byref(st), ctypes.byref(ms)))
    return st.value, ms.value


# ------------------------------------------------------------------------------------------------
# A trained net's answers. Tensors are CUDA tensors of one device, matrices with unit column stride;
# results are new tensors (or the ones given). Work is queued on `stream` (a torch.cuda.Stream or
# cudaStream_t, default: the device's current torch stream), and tensors made here belong to it. On
# another stream than the current one the tensors given are recorded there, so that their memory is not
# handed out again before the work is done; that they are ready is for the caller to see to
# (stream.wait_stream), as for any other work on a stream.
# ------------------------------------------------------------------------------------------------

torch = None             # the module, once one of the calls below has needed it
_dtypes: dict = {}       # torch dtype -> mca_dtype
_fn: dict = {}           # entry points by name


def _ready():
    """torch and the library, looked up once: a call's marshalling is what a small call costs."""
    global torch
    if not _fn:
        import torch as t
        lib = load_library()
        torch = t
        _dtypes.update({getattr(t, n): c for n, c in DTYPE.items()})
        _fn.update({n: getattr(lib, n) for n in SIGNATURES})


def _refuse(name, t, dtypes, device, ndim):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: not a CUDA tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(str(d) for d in dtypes)}")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name}: on {t.device}, expected device {device}")
    if t.dim() != ndim:
        raise ValueError(f"{name}: {t.dim()} dimensions, expected {ndim}")
    raise ValueError(f"{name}: stride {t.stride(-1)} between elements of a row, expected 1")


def _matrix(name, t, dtypes, device=None):
    """Checks a matrix argument: (rows, columns, distance of rows)."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.dim() == 2:
        d = t.get_device()
        if d >= 0 and (device is None or d == device):
            rows, cols = t.shape
            ld, unit = t.stride()
            if unit == 1 or cols <= 1:
                return rows, cols, ld if rows > 1 else cols
    _refuse(name, t, dtypes, device, 2)


def _vector(name, t, n, dtype, device):
    """Address of a vector argument of n elements (None: NULL)."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device
            and t.dim() == 1 and (n <= 1 or t.stride(0) == 1 or t.numel() <= 1)):
        _refuse(name, t, (dtype,), device, 1)
    if t.numel() != n:
        raise ValueError(f"{name}: {t.numel()} elements, expected {n}")
    return t.data_ptr()


def _dtype_code(dtype) -> int:
    _ready()
    try:
        return _dtypes[dtype]
    except KeyError:
        raise ValueError(f"dtype {dtype}: expected float32, float16 or bfloat16") from None


def _on(index, stream, given, call):
    """call(stream's cudaStream_t) with device `index` current and tensors allocated on the stream; the
    tensors `given` (None: none) are recorded on it."""
    if stream is not None:
        stream = getattr(stream, "cuda_stream", stream)
    if torch._C._cuda_getDevice() == index:
        cur = torch._C._cuda_getCurrentRawStream(index)
        if stream is None or stream == cur:
            return call(cur)
    with torch.cuda.device(index):
        if stream is None or stream == torch.cuda.current_stream().cuda_stream:
            return call(torch.cuda.current_stream().cuda_stream)
        st = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
        try:
            with torch.cuda.stream(st):
                return call(stream)
        finally:
            for t in given:
                if t is not None:
                    t.record_stream(st)


def mca_quantize_rows(x, codes=None, scale=None, stream=None):
    """Rows of x [rows, cols] in 8 bits: (codes [rows, cols] int8, scale [rows] float32), x ~ scale *
    codes. New codes' rows start on 16-byte boundaries (a view of a wider matrix when cols is not a
    multiple of 16). stream, here and below: where the work is queued; the tensors have to be ready there
    (stream.wait_stream), and their memory is kept until it is done."""
    _ready()
    rows, cols, ldx = _matrix("x", x, _dtypes)
    dev = x.get_device()
    if codes is not None:
        crows, ccols, ldc = _matrix("codes", codes, (torch.int8,), dev)
        if crows != rows or ccols != cols:
            raise ValueError(f"codes: shape {tuple(codes.shape)}, expected {tuple(x.shape)}")
    if scale is not None:
        _vector("scale", scale, rows, torch.float32, dev)

    def call(s):
        c, ld, sc = codes, 0, scale
        if c is None:
            ld = (cols + 15) // 16 * 16
            c = torch.empty_strided((rows, cols), (ld, 1), dtype=torch.int8, device=x.device)
        else:
            ld = ldc
        if sc is None:
            sc = torch.empty(rows, dtype=torch.float32, device=x.device)
        _check(_fn["mca_quantize_rows"](x.data_ptr(), _dtypes[x.dtype], rows, cols, ldx,
                                        c.data_ptr(), ld, sc.data_ptr(), s))
        return c, sc

    return _on(dev, stream, (x, codes, scale), call)


def _linear_args(x_codes, x_scale, w_codes, w_scale, bias, act, act_param, dtype):
    _ready()
    i8, f32 = (torch.int8,), torch.float32
    rows, n_in, ldx = _matrix("x_codes", x_codes, i8)
    dev = x_codes.get_device()
    n_out, w_in, ldw = _matrix("w_codes", w_codes, i8, dev)
    if w_in != n_in:
        raise ValueError(f"w_codes: {w_in} columns, x_codes has {n_in}")
    return mca_code_linear_args(
        rows, n_in, n_out, x_codes.data_ptr(), ldx, _vector("x_scale", x_scale, rows, f32, dev),
        w_codes.data_ptr(), ldw, _vector("w_scale", w_scale, n_out, f32, dev),
        _vector("bias", bias, n_out, f32, dev), None, n_out,
        0 if dtype is None else _dtype_code(dtype), ACT[act], act_param)


def mca_code_linear_workspace_size(x_codes, x_scale, w_codes, w_scale, bias=None, act="identity",
                                   act_param: float = 0.0, dtype=None) -> int:
    """Bytes of workspace of mca_code_linear for these operands."""
    a = _linear_args(x_codes, x_scale, w_codes, w_scale, bias, act, act_param, dtype)
    n = c_size_t(0)
    _check(_fn["mca_code_linear_workspace_size"](ctypes.byref(a), ctypes.byref(n)))
    return n.value


def mca_code_linear(x_codes, x_scale, w_codes, w_scale, bias=None, act="identity",
                    act_param: float = 0.0, dtype=None, out=None, workspace=None, stream=None):
    """act((x_codes w_codes^T) * x_scale[:, None] * w_scale + bias), sums exact: [rows, n_out] of
    `dtype` (default: out's, or float32). workspace: a uint8 CUDA tensor of at least
    mca_code_linear_workspace_size bytes on a 256-byte boundary (default: allocated for the call)."""
    _ready()
    if out is not None:
        if dtype is not None and dtype != out.dtype:
            raise ValueError(f"out: dtype {out.dtype}, expected {dtype}")
        dtype = out.dtype
    a = _linear_args(x_codes, x_scale, w_codes, w_scale, bias, act, act_param, dtype)
    dev = x_codes.get_device()
    if out is not None:
        rows, n_out, a.ldy = _matrix("out", out, _dtypes, dev)
        if rows != a.rows or n_out != a.n_out:
            raise ValueError(f"out: shape {tuple(out.shape)}, expected {(a.rows, a.n_out)}")
    if workspace is not None:
        _vector("workspace", workspace, workspace.numel(), torch.uint8, dev)
        if workspace.numel():
            a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    ref = ctypes.byref(a)

    def call(s):
        y = out if out is not None else torch.empty(
            (a.rows, a.n_out), dtype=dtype or torch.float32, device=x_codes.device)
        a.y, a.stream = y.data_ptr(), s
        status = _fn["mca_code_linear"](ref)
        if status == MCA_ERR_OOM and workspace is None:      # it wants workspace
            n = c_size_t(0)
            _check(_fn["mca_code_linear_workspace_size"](ref, ctypes.byref(n)))
            ws = torch.empty(n.value, dtype=torch.uint8, device=x_codes.device)
            a.workspace, a.workspace_bytes = ws.data_ptr(), n.value
            status = _fn["mca_code_linear"](ref)
        if status:
            _check(status)
        return y

    return _on(dev, stream, (x_codes, x_scale, w_codes, w_scale, bias, out, workspace), call)


class TokenLogprobs(NamedTuple):
    """Of every row of logits; None for what was not asked for."""
    logprob: object          # [rows] float32, of the target
    entropy: object          # [rows] float32
    lse: object              # [rows] float32
    top_logprob: object      # [rows, top] float32
    top_index: object        # [rows, top] int32


def _logprob_outputs(rows, top, targets, dev):
    f32 = torch.float32
    logprob = torch.empty(rows, dtype=f32, device=dev) if targets else None
    entropy = torch.empty(rows, dtype=f32, device=dev)
    lse = torch.empty(rows, dtype=f32, device=dev)
    if not top:
        return TokenLogprobs(logprob, entropy, lse, None, None)
    return TokenLogprobs(logprob, entropy, lse, torch.empty((rows, top), dtype=f32, device=dev),
                         torch.empty((rows, top), dtype=torch.int32, device=dev))


def _addr(t):
    return None if t is None else t.data_ptr()


def mca_token_logprobs(logits, targets=None, top: int = 0, stream=None) -> TokenLogprobs:
    """Log probabilities of targets [rows] (int32, -1: none) under softmax of each row of logits [rows,
    vocab], entropies, log-sum-exps and the `top` most probable symbols (at most 32). No operation of
    torch's autograd: of logits that require a gradient the results carry none;
    mca_token_logprobs_backward computes it."""
    _ready()
    rows, vocab, ld = _matrix("logits", logits, _dtypes)
    dev = logits.get_device()
    t = _vector("targets", targets, rows, torch.int32, dev)
    if not 0 <= top <= MAX_TOP:
        raise ValueError(f"top = {top} outside 0..{MAX_TOP}")

    def call(s):
        r = _logprob_outputs(rows, top, t is not None, logits.device)
        a = mca_token_logprobs_args(
            logits.data_ptr(), _dtypes[logits.dtype], vocab, rows, ld, t, _addr(r.logprob),
            r.entropy.data_ptr(), r.lse.data_ptr(), top, _addr(r.top_logprob), _addr(r.top_index),
            s)
        _check(_fn["mca_token_logprobs"](ctypes.byref(a)))
        return r

    return _on(dev, stream, (logits, targets), call)


def mca_token_logprobs_backward(logits, targets, lse, entropy, g_logprob, g_entropy=None, out=None,
                                stream=None):
    """Gradient of sum(g_logprob * logprob + g_entropy * entropy) with respect to the logits, from the
    lse and entropy of mca_token_logprobs. g_logprob (with targets) or g_entropy (with entropy) may be
    None. out: [rows, vocab] of the logits' dtype, which may be `logits` itself."""
    _ready()
    rows, vocab, ld = _matrix("logits", logits, _dtypes)
    dev = logits.get_device()
    f32 = torch.float32
    a = mca_token_logprobs_backward_args(
        logits.data_ptr(), _dtypes[logits.dtype], vocab, rows, ld,
        _vector("targets", targets, rows, torch.int32, dev), _vector("lse", lse, rows, f32, dev),
        _vector("entropy", entropy, rows, f32, dev),
        _vector("g_logprob", g_logprob, rows, f32, dev),
        _vector("g_entropy", g_entropy, rows, f32, dev), None, vocab)
    if out is not None:
        orows, ocols, a.ldg = _matrix("out", out, (logits.dtype,), dev)
        if orows != rows or ocols != vocab:
            raise ValueError(f"out: shape {tuple(out.shape)}, expected {tuple(logits.shape)}")

    def call(s):
        g = out if out is not None else torch.empty((rows, vocab), dtype=logits.dtype,
                                                    device=logits.device)
        a.grad, a.stream = g.data_ptr(), s
        _check(_fn["mca_token_logprobs_backward"](ctypes.byref(a)))
        return g

    return _on(dev, stream, (logits, targets, lse, entropy, g_logprob, g_entropy, out), call)


@contextmanager
def _handle_stream(h: Handle, *inputs):
    """The handle's stream as the current one: its work follows what is queued on the caller's stream
    (which made the inputs), and the caller's stream goes on after it."""
    cur = torch.cuda.current_stream()
    if cur.cuda_stream == h.stream:
        yield []
        return
    st = torch.cuda.ExternalStream(h.stream) if h.stream else torch.cuda.default_stream()
    st.wait_stream(cur)
    made = []
    try:
        with torch.cuda.stream(st):
            yield made
    finally:
        for t in inputs:
            t.record_stream(st)
        cur.wait_stream(st)
    for t in made:
        t.record_stream(cur)


def mca_score(h: Handle, top: int = 0):
    """(logits [rows, classes], TokenLogprobs of the labels / next tokens) of the handle's own samples
    under its present weights."""
    _ready()
    if not 0 <= top <= MAX_TOP:
        raise ValueError(f"top = {top} outside 0..{MAX_TOP}")
    with _handle_stream(h) as made:
        logits = torch.empty((h.rows, h.classes), dtype=torch.float32, device="cuda")
        r = _logprob_outputs(h.rows, top, True, "cuda")
        _check(load_library().mca_score(h.ptr, logits.data_ptr(), top, _addr(r.logprob),
                                        _addr(r.entropy), _addr(r.lse), _addr(r.top_logprob),
                                        _addr(r.top_index)), h.ptr)
        made += [logits] + [t for t in r if t is not None]
    return logits, r


def mca_predict_workspace_size(h: Handle, n: int) -> int:
    b = c_size_t(0)
    _check(load_library().mca_predict_workspace_size(h.ptr, n, ctypes.byref(b)), h.ptr)
    return b.value


def mca_predict(h: Handle, x):
    """Activations [n, n_out] float32 of an MLP handle's last layer for new samples x [n, n_in]
    (float32), every layer in 8-bit integers."""
    _ready()
    n, cols, ldx = _matrix("x", x, (torch.float32,))
    if h.n_in and cols != h.n_in:
        raise ValueError(f"x: {cols} columns, the net has {h.n_in} inputs")
    with _handle_stream(h, x) as made:
        nbytes = mca_predict_workspace_size(h, n)
        out = torch.empty((n, h.classes), dtype=torch.float32, device="cuda")
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        _check(load_library().mca_predict(h.ptr, x.data_ptr(), n, ldx, out.data_ptr(),
                                          ws.data_ptr() if nbytes else None, nbytes), h.ptr)
        made.append(out)
    return out


def mca_destroy(h: Handle):
    h.close()


def create_from_workload(wl, device: bool = True, **kw) -> Handle:
    """mca_create for a workloads.MLPWorkload, with its arrays moved to the GPU by torch."""
    import torch
    X, y, init = wl.X, wl.y, wl.init
    if device:
        X = torch.from_numpy(X).cuda()
        y = torch.from_numpy(y).cuda()
        init = torch.from_numpy(init).cuda()
    kw.setdefault("K", wl.K)
    return mca_create(wl.layers, wl.loss, wl.domain, X, y, init, **kw)
