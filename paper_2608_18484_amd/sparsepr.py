"""Thin ctypes binding of the SparsePR C ABI (include/sparsepr.h).

Argument marshalling only: every step of the operator runs in the HIP
library.  torch supplies device memory (inputs, outputs, the workspace) and
the stream.  Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
# SPARSEPR_LIB selects another build of the same library (the host-side
# sanitizer build of build.py --sanitize); the default is the in-tree build
LIB_PATH = os.environ.get("SPARSEPR_LIB") or os.path.join(HERE, "libsparsepr.so")

F32, BF16 = 0, 1
FLAG_NONFINITE_INPUT, FLAG_FIT_NOT_PD, FLAG_BUDGET_BELOW_FORCED, FLAG_EIG_JACOBI = 1, 2, 4, 8
STATUS = {0: "OK", 1: "INVALID_ARGUMENT", 2: "UNSUPPORTED", 3: "WORKSPACE_TOO_SMALL", 4: "HIP",
          5: "NUMERICAL"}


class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("n_q", ctypes.c_int32),
                ("n_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("d_v", ctypes.c_int32),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("heads_kv", ctypes.c_int32), ("kv_stride_b", ctypes.c_int64),
                ("kv_stride_h", ctypes.c_int64)]


class Params(ctypes.Structure):
    _fields_ = [("n_sampled_queries", ctypes.c_int32), ("r_k", ctypes.c_int32),
                ("r_q", ctypes.c_int32), ("n_kv_groups", ctypes.c_int32),
                ("n_q_groups", ctypes.c_int32), ("kmeans_iters", ctypes.c_int32),
                ("target_exec_density", ctypes.c_float), ("n_probes", ctypes.c_int32),
                ("resid_rank", ctypes.c_int32), ("ridge", ctypes.c_float),
                ("eps_q", ctypes.c_float), ("eps_x", ctypes.c_float),
                ("n_dense_prefix", ctypes.c_int32), ("warm_start", ctypes.c_int32),
                ("warm_iters", ctypes.c_int32), ("partition", ctypes.c_int32),
                ("probe_rule", ctypes.c_int32), ("probe_seed", ctypes.c_uint32),
                ("ridge_only", ctypes.c_int32), ("routing", ctypes.c_int32)]


class Stats(ctypes.Structure):
    _fields_ = [("rho_route", ctypes.c_double), ("rho_exec", ctypes.c_double),
                ("routed_pairs", ctypes.c_int64), ("exec_pairs", ctypes.c_int64),
                ("forced_pairs", ctypes.c_int64), ("routed_cells", ctypes.c_int32),
                ("forced_cells", ctypes.c_int32), ("nonempty_q_groups", ctypes.c_int32),
                ("nonempty_kv_groups", ctypes.c_int32), ("n_probes", ctypes.c_int32),
                ("kmeans_iters_kv", ctypes.c_int32), ("kmeans_iters_q", ctypes.c_int32),
                ("status_flags", ctypes.c_int32), ("kmeans_rescans", ctypes.c_int64)]


class Timings(ctypes.Structure):
    _fields_ = [("plan_ms", ctypes.c_double), ("sparse_attn_ms", ctypes.c_double),
                ("probe_ms", ctypes.c_double), ("fit_ms", ctypes.c_double),
                ("correct_ms", ctypes.c_double), ("plan_calls", ctypes.c_int32),
                ("attend_calls", ctypes.c_int32), ("attn_launches", ctypes.c_int32)]


_P = ctypes.c_void_p


class Cache(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("d", ctypes.c_int32),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64), ("dtype", ctypes.c_int32), ("k", _P), ("v", _P),
                ("lengths", _P), ("scores", _P), ("positions", _P), ("flags", _P)]


class Tokens(ctypes.Structure):
    _fields_ = [("heads", ctypes.c_int32), ("n", ctypes.c_int32),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64), ("out_stride_b", ctypes.c_int64),
                ("out_stride_h", ctypes.c_int64), ("out_stride_n", ctypes.c_int64),
                ("kv_stride_b", ctypes.c_int64), ("kv_stride_h", ctypes.c_int64),
                ("kv_stride_n", ctypes.c_int64), ("mask", ctypes.c_int32)]


TOKENS_CAUSAL, TOKENS_FULL, TOKENS_TREE = 0, 1, 2
CACHE_FLAG_OVERFLOW, CACHE_FLAG_BAD_INDEX, CACHE_FLAG_REFUSED = 1, 2, 4
HOST_FIELDS = [
    ("labels_q", "i4"), ("labels_kv", "i4"), ("routes", "u1"), ("probes", "i4"),
    ("n_probes", None),
    ("probe_weights", "f4"), ("perm_q", "i4"), ("off_q", "i4"), ("perm_kv", "i4"),
    ("off_kv", "i4"), ("m_k", "f4"), ("m_q", "f4"), ("f_k", "f4"), ("f_q", "f4"),
    ("phi_k", "f4"), ("phi_q", "f4"), ("cent_k", "f4"), ("cent_q", "f4"), ("kbar", "f4"),
    ("qbar", "f4"), ("route_prio", "f4"), ("o_sparse", "f4"), ("o_dense_probes", "f4"),
    ("fit_mu_x", "f4"), ("fit_s_x", "f4"), ("fit_mu_r", "f4"), ("fit_bpsi", "f4"),
    ("fit_psi", "f4"), ("fit_rank", None), ("route_key", "f4"),
]


class PlanHost(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32 if kind is None else _P) for name, kind in HOST_FIELDS]


EXPORTED = ["sparsepr_params_default", "sparsepr_workspace_size", "sparsepr_plan_create",
            "sparsepr_plan", "sparsepr_attend", "sparsepr_dense_workspace_size",
            "sparsepr_dense_attend", "sparsepr_get_stats", "sparsepr_plan_export",
            "sparsepr_plan_import", "sparsepr_set_profiling", "sparsepr_get_timings",
            "sparsepr_plan_destroy", "sparsepr_last_error", "sparsepr_plan_create_static",
            "sparsepr_cache_attend_workspace_size", "sparsepr_cache_attend",
            "sparsepr_cache_append", "sparsepr_cache_accumulate_workspace_size",
            "sparsepr_cache_accumulate", "sparsepr_cache_evict_workspace_size",
            "sparsepr_cache_evict"]

# argument kinds of the cache operators: p = pointer, i = int32, z = size_t
CACHE_CALLS = {"sparsepr_cache_attend_workspace_size": "ppp",
               "sparsepr_cache_attend": "ppppppppppzp",
               "sparsepr_cache_append": "ppppppippp",
               "sparsepr_cache_accumulate_workspace_size": "ppip",
               "sparsepr_cache_accumulate": "pppppippzp",
               "sparsepr_cache_evict_workspace_size": "pip",
               "sparsepr_cache_evict": "ppiiipzp"}

_lib = None


def lib():
    """Load libsparsepr.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"SparsePR HIP library not built: {LIB_PATH} is missing "
                               "(run __graft_entry__.build() or paper_2608_18484_amd/build.py)")
        L = ctypes.CDLL(LIB_PATH)
        L.sparsepr_last_error.restype = ctypes.c_char_p
        for name, n_args in CACHE_CALLS.items():  # every argument a pointer or an int
            getattr(L, name).argtypes = [ctypes.c_int32 if c == "i" else ctypes.c_size_t if c == "z"
                                         else ctypes.c_void_p for c in n_args]
        for name in EXPORTED:
            if name not in ("sparsepr_last_error", "sparsepr_params_default", "sparsepr_plan_destroy"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


class SparsePRError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


def _check(st):
    if st != 0:
        raise SparsePRError(st, lib().sparsepr_last_error().decode())


PARTITION_RESPONSE, PARTITION_SEMANTIC, PARTITION_KEY_RESPONSE = 0, 1, 2
PROBES_STRATIFIED, PROBES_RANDOM, PROBES_UNIFORM = 0, 1, 2
ROUTING_PRIORITY, ROUTING_TOP_P = 0, 1


def default_params(**kw) -> Params:
    p = Params()
    lib().sparsepr_params_default(ctypes.byref(p))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def shape_of(t, dtype=None, kv=None) -> Shape:
    """Shape struct for a [B, H, N, d] torch tensor (last dim contiguous).
    `kv`: the [B, H_kv, N, d] K tensor (V must share its strides) for
    grouped-query attention, where H_kv divides H."""
    import torch
    b, h, n, d = t.shape
    sb, sh, sn, sd = t.stride()
    if sd != 1:
        raise ValueError("last dimension must be contiguous")
    dt = dtype if dtype is not None else (BF16 if t.dtype == torch.bfloat16 else F32)
    hkv, ksb, ksh = 0, 0, 0
    if kv is not None:
        bk, hkv, nk, dk = kv.shape
        ksb, ksh, ksn, ksd = kv.stride()
        if (bk, nk, dk) != (b, n, d) or ksn != sn or ksd != 1:
            raise ValueError("K/V must be [B, H_kv, N, d] with Q's row stride")
    return Shape(b, h, n, n, d, d, sb, sh, sn, dt, hkv, ksb, ksh)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def check_tensors(shape: Shape, q=None, k=None, v=None, out=None, device_type="cuda"):
    """Check tensors against the geometry a plan was created with, before any
    launch: the C side sees only pointers, so a tensor with another dtype,
    fewer heads or rows, or other strides would make the kernels read or write
    past its end.  Q and the output are [batch, heads, n, d] with the shape's
    strides; K and V are [batch, heads_kv, n, d] with the K/V strides (the Q
    strides when heads_kv is 0).  Raises ValueError on any mismatch."""
    import torch
    want_dtype = torch.bfloat16 if shape.dtype == BF16 else torch.float32
    hkv = shape.heads_kv or shape.heads
    kvsb = shape.kv_stride_b or shape.stride_b
    kvsh = shape.kv_stride_h or shape.stride_h
    geo = {
        "q": ((shape.batch, shape.heads, shape.n_q, shape.d),
              (shape.stride_b, shape.stride_h, shape.stride_n, 1)),
        "out": ((shape.batch, shape.heads, shape.n_q, shape.d_v),
                (shape.stride_b, shape.stride_h, shape.stride_n, 1)),
        "k": ((shape.batch, hkv, shape.n_kv, shape.d), (kvsb, kvsh, shape.stride_n, 1)),
        "v": ((shape.batch, hkv, shape.n_kv, shape.d_v), (kvsb, kvsh, shape.stride_n, 1)),
    }
    device = None
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        if t is None:
            continue
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
        if t.device.type != device_type:
            raise ValueError(f"{name}: tensor on {t.device}, expected a {device_type} tensor")
        if device is None:
            device = t.device
        elif t.device != device:
            raise ValueError(f"{name}: tensor on {t.device}, the others on {device}")
        if t.dtype != want_dtype:
            raise ValueError(f"{name}: dtype {t.dtype}, the plan was made for {want_dtype}")
        dims, strides = geo[name]
        if tuple(t.shape) != dims:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, the plan was made for {dims}")
        # a dimension of extent 1 is never stepped over, so its stride is free
        for ax, (got, exp) in enumerate(zip(t.stride(), strides)):
            if dims[ax] > 1 and got != exp:
                raise ValueError(f"{name}: strides {tuple(t.stride())}, the plan was made for "
                                 f"{strides}")


def _stream(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


class SparsePR:
    """One SparsePR operator instance bound to a shape, parameters and a workspace."""

    def __init__(self, shape: Shape, params: Params, device="cuda", static=False):
        """static=True binds the plan to the library's static scratch array of
        the current device (sparsepr_plan_create_static: nothing is
        allocated; one such plan per device at a time, small shapes only)."""
        import torch
        self.shape, self.params = shape, params
        nbytes = ctypes.c_size_t(0)
        _check(lib().sparsepr_workspace_size(ctypes.byref(shape), ctypes.byref(params),
                                             ctypes.byref(nbytes)))
        self.workspace_bytes = nbytes.value
        self.handle = ctypes.c_void_p()
        if static:
            self.workspace = None
            _check(lib().sparsepr_plan_create_static(ctypes.byref(shape), ctypes.byref(params),
                                                     ctypes.byref(self.handle)))
        else:
            self.workspace = torch.empty(max(nbytes.value, 256), dtype=torch.uint8, device=device)
            _check(lib().sparsepr_plan_create(ctypes.byref(shape), ctypes.byref(params),
                                              _ptr(self.workspace),
                                              ctypes.c_size_t(self.workspace.numel()),
                                              ctypes.byref(self.handle)))
        n = shape.n_q
        ntext = params.n_dense_prefix
        nv = n - ntext
        self.ck = params.n_kv_groups or -(-nv // 64)
        self.cq = params.n_q_groups or -(-nv // 64)
        self.ck_t = self.ck + (ntext > 0)
        self.cq_t = self.cq + (ntext > 0)
        self.m = min(params.n_probes, nv)

    def close(self):
        """Destroy the plan handle now (a static plan releases its device's array)."""
        h = getattr(self, "handle", None)
        if h is not None and h.value and _lib is not None:
            _lib.sparsepr_plan_destroy(h)
        self.handle = None

    def __del__(self):
        self.close()

    def plan(self, q, k, stream=None):
        check_tensors(self.shape, q=q, k=k)
        _check(lib().sparsepr_plan(self.handle, _ptr(q), _ptr(k), _stream(stream)))

    def attend(self, q, k, v, out, stream=None):
        check_tensors(self.shape, q=q, k=k, v=v, out=out)
        _check(lib().sparsepr_attend(self.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                     _stream(stream)))

    def __call__(self, q, k, v, out=None, stream=None):
        import torch
        if out is None:
            out = torch.empty_like(q)
        self.plan(q, k, stream)
        self.attend(q, k, v, out, stream)
        return out

    def stats(self, stream=None) -> dict:
        s = Stats()
        _check(lib().sparsepr_get_stats(self.handle, ctypes.byref(s), _stream(stream)))
        return {name: getattr(s, name) for name, _ in Stats._fields_}

    def set_profiling(self, enable=True):
        _check(lib().sparsepr_set_profiling(self.handle, ctypes.c_int32(int(enable))))

    def timings(self, reset=True, stream=None) -> dict:
        t = Timings()
        _check(lib().sparsepr_get_timings(self.handle, ctypes.byref(t), ctypes.c_int32(int(reset)),
                                          _stream(stream)))
        return {name: getattr(t, name) for name, _ in Timings._fields_}

    def _sizes(self):
        sh, p = self.shape, self.params
        n, d, dv = sh.n_q, sh.d, sh.d_v
        nv = n - p.n_dense_prefix
        rk, rq = min(p.r_k, d), min(p.r_q, d)
        if p.partition == PARTITION_SEMANTIC:
            rk = d
        if p.partition != PARTITION_RESPONSE:
            rq = d
        r = dv if p.ridge_only else p.resid_rank
        m = max(self.m, 1)
        return {
            "labels_q": n, "labels_kv": n, "routes": self.cq_t * self.ck_t, "probes": m,
            "probe_weights": m, "perm_q": n, "off_q": self.cq_t + 1, "perm_kv": n,
            "off_kv": self.ck_t + 1, "m_k": d * d, "m_q": d * d, "f_k": d * rk, "f_q": d * rq,
            "phi_k": nv * rk, "phi_q": nv * rq, "cent_k": self.ck * rk, "cent_q": self.cq * rq,
            "kbar": self.ck * d, "qbar": self.cq * d, "route_prio": self.cq * self.ck,
            "route_key": self.cq * self.ck, "o_sparse": n * dv, "o_dense_probes": m * dv,
            "fit_mu_x": dv, "fit_s_x": dv,
            "fit_mu_r": dv, "fit_bpsi": dv * r, "fit_psi": dv * r,
        }

    def export(self, bh: int = 0, fields=None, stream=None) -> dict:
        """Copy the plan used by query head bh (and that head's attend outputs)
        to numpy arrays."""
        sizes = self._sizes()
        want = [name for name, kind in HOST_FIELDS if kind is not None and
                (fields is None or name in fields)]
        bufs = {}
        ph = PlanHost()
        for name, kind in HOST_FIELDS:
            if kind is None or name not in want:
                continue
            arr = np.zeros(sizes[name], dtype=np.dtype(kind))
            bufs[name] = arr
            setattr(ph, name, arr.ctypes.data_as(ctypes.c_void_p))
        _check(lib().sparsepr_plan_export(self.handle, ctypes.c_int32(bh), ctypes.byref(ph),
                                          _stream(stream)))
        sh, p = self.shape, self.params
        d, dv = sh.d, sh.d_v
        r = dv if p.ridge_only else p.resid_rank
        rk, rq = min(p.r_k, d), min(p.r_q, d)
        if p.partition == PARTITION_SEMANTIC:
            rk = d
        if p.partition != PARTITION_RESPONSE:
            rq = d
        npr = ph.n_probes
        shapes = {"routes": (self.cq_t, self.ck_t), "m_k": (d, d), "m_q": (d, d),
                  "f_k": (d, rk), "f_q": (d, rq), "phi_k": (-1, rk), "phi_q": (-1, rq),
                  "cent_k": (self.ck, rk), "cent_q": (self.cq, rq), "kbar": (self.ck, d),
                  "qbar": (self.cq, d), "route_prio": (self.cq, self.ck),
                  "route_key": (self.cq, self.ck), "o_sparse": (-1, dv),
                  "o_dense_probes": (-1, dv), "fit_bpsi": (dv, r), "fit_psi": (dv, r)}
        out = {}
        for name, arr in bufs.items():
            if name in ("probes", "probe_weights"):
                arr = arr[:npr]
            if name == "o_dense_probes":
                arr = arr[:npr * dv]
            out[name] = arr.reshape(shapes[name]) if name in shapes else arr
        out["n_probes"] = npr
        out["fit_rank"] = ph.fit_rank
        return out

    def import_plan(self, bh: int, labels_q, labels_kv, routes, probes, stream=None):
        """Replace the plan used by query head bh (shared by its K/V head's
        group) by host arrays (labels, route matrix, probes)."""
        lq = np.ascontiguousarray(labels_q, np.int32)
        lk = np.ascontiguousarray(labels_kv, np.int32)
        z = np.ascontiguousarray(routes, np.uint8)
        pr = np.ascontiguousarray(probes, np.int32)
        ph = PlanHost()
        ph.labels_q = lq.ctypes.data_as(ctypes.c_void_p)
        ph.labels_kv = lk.ctypes.data_as(ctypes.c_void_p)
        ph.routes = z.ctypes.data_as(ctypes.c_void_p)
        ph.probes = pr.ctypes.data_as(ctypes.c_void_p) if len(pr) else None
        ph.n_probes = len(pr)
        _check(lib().sparsepr_plan_import(self.handle, ctypes.c_int32(bh), ctypes.byref(ph),
                                          _stream(stream)))


def dense_attention(q, k, v, out=None, stream=None):
    """Dense attention (Sec. 3) for every query head (K and V may have fewer
    heads: grouped-query attention)."""
    import torch
    if out is None:
        out = torch.empty_like(q)
    sh = shape_of(q, kv=k if k.shape[1] != q.shape[1] else None)
    check_tensors(sh, q=q, k=k, v=v, out=out)
    _check(lib().sparsepr_dense_attend(ctypes.byref(sh), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                       None, ctypes.c_size_t(0), _stream(stream)))
    return out


def _tensor(name, t, shape, dtype, device, contiguous=True):
    """Raises ValueError unless t is a tensor of this shape, dtype and device,
    contiguous or with a contiguous last dimension, that asks for no gradient."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
    if t.requires_grad:
        _no_grad(name, t)
    if t.device == device and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return
    if t.device != device:
        raise ValueError(f"{name}: tensor on {t.device}, the cache is on {device}")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: last dimension must be contiguous")


def _too_long(name, t):
    """The library takes extents as int32."""
    return ValueError(f"{name}: shape {tuple(t.shape)}, extents must be below 2^31")


def _no_grad(name, t):
    """What the cache's operators write has no graph: a gradient would be lost."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: requires grad, and the operators on a cache have no backward "
                         "(call them under torch.no_grad())")


def _same_strides(name, a, other, b):
    """Strides of dimensions that are stepped over."""
    if a.stride() != b.stride() and any(n > 1 and x != y for n, x, y in
                                        zip(a.shape, a.stride(), b.stride())):
        raise ValueError(f"{name}: strides {a.stride()}, those of {other} are {b.stride()}")


# Flags that a captured graph writes: a replay may come after the cache object's end.
_captured = []


def _opt(t):
    return None if t is None else t.data_ptr()


class KVCache:
    """A cache of keys and values with the operators on it (the cache section
    of include/sparsepr.h): attention of new tokens, append, accumulated
    attention weights, eviction.  The tensors are the caller's:

      k, v       [B, H_kv, capacity, d] bfloat16 or float32, last dim contiguous,
                 equal strides
      lengths    [B] int32: slots in use
      scores     [B, H_kv, capacity] float32 contiguous, or None: accumulated
                 weights (accumulate, evict)
      positions  [B, H_kv, capacity] int32 contiguous, or None: token positions
                 (evict's n_sink and n_recent)

    Calls are enqueued on `stream` (default: the current stream of the cache's
    device) and never synchronise; flags() does.  A graph that captured calls needs
    the tensors alone: it may be replayed after this object's end.  Inference only:
    tensors that require gradients are refused outside torch.no_grad()."""

    def __init__(self, k, v, lengths, scores=None, positions=None):
        global torch
        import torch  # once for the module: the calls below look it up as a global
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k: expected a [B, H_kv, capacity, d] torch.Tensor")
        if k.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"k: dtype {k.dtype}, expected bfloat16 or float32")
        if k.device.type != self._device_type:
            raise ValueError(f"k: tensor on {k.device}, expected a {self._device_type} tensor")
        self.device, self.dtype = k.device, k.dtype
        if max(k.shape) >= 2 ** 31:
            raise _too_long("k", k)
        b, hkv, cap, d = k.shape
        _tensor("k", k, k.shape, k.dtype, k.device, contiguous=False)
        _tensor("v", v, k.shape, k.dtype, k.device, contiguous=False)
        _same_strides("v", v, "k", k)
        _tensor("lengths", lengths, (b,), torch.int32, k.device)
        if scores is not None:
            _tensor("scores", scores, (b, hkv, cap), torch.float32, k.device)
        if positions is not None:
            _tensor("positions", positions, (b, hkv, cap), torch.int32, k.device)
        self.k, self.v, self.lengths = k, v, lengths
        self.scores, self.positions = scores, positions
        self._flags = torch.zeros(b, dtype=torch.int32, device=k.device)
        self._kept, self._streams, self._cleared = False, set(), None
        if self._device_type == "cuda":
            self._streams.add(torch._C._cuda_getCurrentRawStream(k.device.index))
            if not torch.cuda.is_current_stream_capturing():
                self._cleared = torch.cuda.current_stream(k.device).record_event()
        self._default = 0 in self._streams
        sb, sh, sn, _ = k.stride()
        self.desc = Cache(b, hkv, cap, d, sb, sh, sn, BF16 if k.dtype == torch.bfloat16 else F32,
                          k.data_ptr(), v.data_ptr(), lengths.data_ptr(), _opt(scores),
                          _opt(positions), self._flags.data_ptr())
        self._desc = ctypes.addressof(self.desc)

    _device_type = "cuda"

    def flags(self) -> list:
        """CACHE_FLAG_OVERFLOW and _BAD_INDEX raised on the device since the
        last call, per batch entry; clears them.  Waits for the device."""
        torch.cuda.synchronize(self.device)
        got = self._flags.tolist()
        # (append's own note for accumulate stays; an object made in inference mode
        # has flags that can be written there alone)
        with torch.inference_mode():
            self._flags.bitwise_and_(CACHE_FLAG_REFUSED)
        torch.cuda.synchronize(self.device)
        return [x & ~CACHE_FLAG_REFUSED for x in got]

    # -- marshalling --------------------------------------------------------

    def _run(self, stream, launch):
        """launch(stream handle), with the stream and the cache's device current
        where they are not, so that scratch memory and outputs made by the call
        belong to the stream that uses them."""
        if self.k.requires_grad or self.v.requires_grad:
            _no_grad("k", self.k)
            _no_grad("v", self.v)
        if stream is None:
            # (the handle alone: the stream object takes longer than a short kernel's launch)
            handle = torch._C._cuda_getCurrentRawStream(self.device.index)
            if self.device.index == torch._C._cuda_getDevice():
                if handle or not self._default:
                    self._order(handle)
                return launch(handle)
            with torch.cuda.device(self.device):
                self._order(handle)
                return launch(handle)
        if stream.device != self.device:
            raise ValueError(f"stream on {stream.device}, the cache is on {self.device}")
        with torch.cuda.stream(stream):
            self._order(stream.cuda_stream)
            return launch(stream.cuda_stream)

    def _order(self, handle):
        """The flags' memory in order with a call on that (current) stream."""
        if handle in self._streams and (self._kept or handle == 0):
            return
        # (the default stream, 0, captures nothing)
        if handle and torch.cuda.is_current_stream_capturing():
            if not self._kept:
                self._kept = True
                _captured.append(self._flags)
        elif handle not in self._streams:
            # first call on a stream: after the flags were cleared on the one that was
            # current then, and before their memory is used again
            here = torch.cuda.current_stream(self.device)
            if self._cleared is not None:
                here.wait_event(self._cleared)
            self._flags.record_stream(here)
            self._streams.add(handle)
            self._default = 0 in self._streams

    def _scratch(self, size_fn, *args):
        """Scratch memory of one call from torch's allocator (None if it needs none)."""
        need = ctypes.c_size_t(0)
        _check(size_fn(self._desc, *args, ctypes.addressof(need)))
        if need.value == 0:
            return None, 0
        return torch.empty(need.value, dtype=torch.uint8, device=self.device), need.value

    def _q(self, q):
        c = self.desc
        if not isinstance(q, torch.Tensor) or q.dim() != 4:
            raise ValueError("q: expected a [B, H, n, d] torch.Tensor")
        _, h, n, _ = q.shape
        if n >= 2 ** 31 or h >= 2 ** 31:
            raise _too_long("q", q)
        _tensor("q", q, (c.batch, h, n, c.d), self.dtype, self.device, contiguous=False)
        if n < 1 or h < 1 or h % c.heads_kv != 0:
            raise ValueError(f"q: {h} heads of {n} tokens; heads must be a multiple of the "
                             f"cache's {c.heads_kv}, tokens at least 1")
        return h, n

    def _new(self, k_new, v_new, n):
        c = self.desc
        _tensor("k_new", k_new, (c.batch, c.heads_kv, n, c.d), self.dtype, self.device, False)
        _tensor("v_new", v_new, k_new.shape, self.dtype, self.device, False)
        _same_strides("v_new", v_new, "k_new", k_new)
        return k_new.stride()[:3]

    def _list(self, rows, counts, n):
        """Checks an accepted-rows list and the counts; the list's width."""
        b, width = self.desc.batch, n
        if rows is not None:
            if not isinstance(rows, torch.Tensor) or rows.dim() != 2 or rows.shape[1] < 1:
                raise ValueError("rows: expected a [B, n_rows] torch.Tensor")
            width = rows.shape[1]
            if width >= 2 ** 31:
                raise _too_long("rows", rows)
            _tensor("rows", rows, (b, width), torch.int32, self.device)
        if counts is not None:
            _tensor("counts", counts, (b,), torch.int32, self.device)
        return width

    # -- operators ----------------------------------------------------------

    def attend(self, q, k_new, v_new, parents=None, counts=None, causal=True, out=None, lse=None,
               stream=None):
        """Attention of the new tokens q [B, H, n, d] (their keys and values
        k_new, v_new [B, H_kv, n, d]) over the slots in use and each other; see
        sparsepr_cache_attend.  parents [B, n] int32 makes them a tree; without
        it they are a chain (causal) or all see each other.  counts [B] int32:
        tokens of each entry.  Returns (out, lse); rows behind counts keep what
        the given out and lse hold (zeros where they are made here)."""
        h, n = self._q(q)
        ks = self._new(k_new, v_new, n)
        b = self.desc.batch
        self._list(None, counts, n)
        mask = TOKENS_CAUSAL if causal else TOKENS_FULL
        if parents is not None:
            if not causal:
                raise ValueError("parents: a tree's tokens see their ancestors only (causal=True)")
            _tensor("parents", parents, (b, n), torch.int32, self.device)
            mask = TOKENS_TREE
        if out is not None:
            _tensor("out", out, q.shape, self.dtype, self.device, contiguous=False)
        if lse is not None:
            _tensor("lse", lse, (b, h, n), torch.float32, self.device)

        def launch(handle):
            o, z = out, lse
            make = torch.empty if counts is None else torch.zeros
            if o is None:
                o = make(q.shape, dtype=self.dtype, device=self.device)
            if z is None:
                z = make((b, h, n), dtype=torch.float32, device=self.device)
            t = Tokens(h, n, *q.stride()[:3], *o.stride()[:3], *ks, mask)
            at, L = ctypes.addressof(t), lib()
            ws, nbytes = self._scratch(L.sparsepr_cache_attend_workspace_size, at)
            _check(L.sparsepr_cache_attend(
                self._desc, at, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), _opt(parents),
                _opt(counts), o.data_ptr(), z.data_ptr(), _opt(ws), nbytes, handle))
            return o, z

        return self._run(stream, launch)

    def append(self, k_new, v_new, positions=None, rows=None, counts=None, lengths_out=None,
               stream=None):
        """Append the rows of k_new, v_new [B, H_kv, n, d] named by rows [B, n_rows]
        int32 (None: all, in order), counts[b] of them, behind the slots in use;
        see sparsepr_cache_append.  positions [B, n] int32: the tokens'
        positions (with a cache that keeps them).  The new lengths go to
        lengths_out [B] int32, or into the cache's own."""
        if not isinstance(k_new, torch.Tensor) or k_new.dim() != 4 or k_new.shape[2] < 1:
            raise ValueError("k_new: expected a [B, H_kv, n, d] torch.Tensor with n >= 1")
        c, n = self.desc, k_new.shape[2]
        if n >= 2 ** 31:
            raise _too_long("k_new", k_new)
        ks = self._new(k_new, v_new, n)
        width = self._list(rows, counts, n)
        if (positions is None) != (self.positions is None):
            raise ValueError("positions: given when the cache has positions, and only then")
        if positions is not None:
            _tensor("positions", positions, (c.batch, n), torch.int32, self.device)
        if lengths_out is None:
            lengths_out = self.lengths
        _tensor("lengths_out", lengths_out, (c.batch,), torch.int32, self.device)
        t = Tokens(c.heads_kv, n, 0, 0, 0, 0, 0, 0, *ks, TOKENS_CAUSAL)
        self._run(stream, lambda handle: _check(lib().sparsepr_cache_append(
            self._desc, ctypes.addressof(t), k_new.data_ptr(), v_new.data_ptr(), _opt(positions),
            _opt(rows), width, _opt(counts), lengths_out.data_ptr(), handle)))

    def accumulate(self, q, lse, rows=None, counts=None, causal=True, stream=None):
        """Add the attention weights of the rows that were just appended (rows
        and counts as in append; q and lse as in attend) to the scores of the
        slots that they see; see sparsepr_cache_accumulate.  Entries whose last
        append by this object was refused (flags()) keep their scores."""
        h, n = self._q(q)
        c = self.desc
        width = self._list(rows, counts, n)
        _tensor("lse", lse, (c.batch, h, n), torch.float32, self.device)
        if self.scores is None:
            raise ValueError("accumulate: the cache has no scores")
        t = Tokens(h, n, *q.stride()[:3], 0, 0, 0, 0, 0, 0,
                   TOKENS_CAUSAL if causal else TOKENS_FULL)

        def launch(handle):
            at, L = ctypes.addressof(t), lib()
            ws, nbytes = self._scratch(L.sparsepr_cache_accumulate_workspace_size, at, width)
            _check(L.sparsepr_cache_accumulate(
                self._desc, at, q.data_ptr(), lse.data_ptr(), _opt(rows), width, _opt(counts),
                _opt(ws), nbytes, handle))

        self._run(stream, launch)

    def evict(self, budget, n_sink=0, n_recent=0, out=None, stream=None):
        """Keep at most `budget` slots of every K/V head: the first n_sink
        positions, the n_recent newest and the largest scores, in place or in
        another KVCache `out`; see sparsepr_cache_evict."""
        if self.scores is None:
            raise ValueError("evict: the cache has no scores")
        if out is not None and out.device != self.device:
            raise ValueError(f"out: cache on {out.device}, this one on {self.device}")
        for name, x in (("budget", budget), ("n_sink", n_sink), ("n_recent", n_recent)):
            if not 0 <= x < 2 ** 31:
                raise ValueError(f"{name}: {x} is out of range")

        def launch(handle):
            L = lib()
            ws, nbytes = self._scratch(L.sparsepr_cache_evict_workspace_size, budget)
            _check(L.sparsepr_cache_evict(self._desc, None if out is None else out._desc, budget,
                                          n_sink, n_recent, _opt(ws), nbytes, handle))

        self._run(stream, launch)
