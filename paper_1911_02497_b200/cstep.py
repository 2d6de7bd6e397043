"""Thin ctypes binding of ``libcondensa_cstep.so`` (argument marshalling only).

Every step of the C-step runs in the library's CUDA kernels; PyTorch is used
by callers for device memory and streams. There is no CPU fallback: if the
shared library is missing or no CUDA device is present the calls raise.
Function names and arguments mirror ``include/condensa_cstep.h``.
"""
from __future__ import annotations

import ctypes as C
import os
import warnings
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcondensa_cstep.so")

FUSE_FP16, FUSE_LAMBDA, FUSE_PENALTY, NO_SAMPLING = 1, 2, 4, 64
OP_PRUNE, OP_FILTER, OP_BLOCK, OP_QUANTIZE, OP_LAGRANGE = 0, 1, 2, 3, 4
DTYPE_FP16, DTYPE_BF16, DTYPE_FP8_E4M3, DTYPE_FP8_E5M2 = 1, 2, 3, 4
FUSE_BF16, FUSE_E4M3, FUSE_E5M2 = 8, 16, 32
STRUCT_FILTER, STRUCT_NEURON = 1, 2
OK, ERR_INVALID_ARG, ERR_WORKSPACE, ERR_CUDA, ERR_UNSUPPORTED, ERR_INTERNAL = 0, -1, -2, -3, -4, -5
ERR_TOO_LARGE = -6
NOALLOC_MAX_NUMEL = 1048576

EXPORTS = ["condensa_create", "condensa_destroy", "condensa_cstep_prune", "condensa_cstep_filter",
           "condensa_cstep_block", "condensa_cstep_quantize", "condensa_cstep_lagrange_update",
           "condensa_cstep_host", "condensa_get_result", "condensa_launch_count",
           "condensa_last_error", "condensa_profile_enable", "condensa_profile_read",
           "condensa_cstep_prune_noalloc", "condensa_lstep_update",
           "condensa_cstep_structure", "condensa_thin_flags", "condensa_thin_compact",
           "condensa_count_nonzero", "condensa_set_seed", "condensa_noalloc_status",
           "condensa_cstep_structured", "condensa_workspace_bytes", "condensa_thin_list",
           "condensa_lstep_adamw", "condensa_grad_norm", "condensa_adapter_forward", "condensa_adapter_backward"]


class CondensaError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__("condensa error %d: %s" % (code, text))
        self.code = code


class Tensor(C.Structure):
    """Mirror of ``condensa_tensor``."""
    _fields_ = [("w", C.c_void_p), ("lam", C.c_void_p), ("theta", C.c_void_p),
                ("mask", C.c_void_p), ("grad", C.c_void_p), ("theta_h", C.c_void_p),
                ("numel", C.c_int64), ("ndim", C.c_int32), ("shape", C.c_int64 * 4)]


class Result(C.Structure):
    """Mirror of ``condensa_result``."""
    _fields_ = [("status", C.c_int32), ("passes", C.c_int32), ("n_units", C.c_int64),
                ("n_zero", C.c_int64), ("n_keep", C.c_int64), ("tau_key", C.c_uint64),
                ("tau_id", C.c_int64), ("n_gt", C.c_int64), ("n_tie", C.c_int64),
                ("n_tie_kept", C.c_int64), ("tau_norm", C.c_float), ("sampled", C.c_int32),
                ("n_candidates", C.c_int64), ("n_repaired", C.c_int64), ("seed", C.c_uint64)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class StructureSpec(C.Structure):
    """Mirror of ``condensa_structure_spec``."""
    _fields_ = [("kind", C.c_int32), ("kinds", C.c_int32), ("criterion", C.c_int32), ("ndim", C.c_int32),
                ("block", C.c_int64 * 4)]


SPEC_SLICES, SPEC_BLOCKS = 0, 1
CRITERIA = {"l2": 0, "l1": 1, "max": 2}


class ThinLayer(C.Structure):
    """Mirror of ``condensa_thin_layer``."""
    _fields_ = [("src", C.c_void_p), ("d0", C.c_int64), ("d1", C.c_int64), ("inner", C.c_int64),
                ("keep0", C.c_void_p), ("remove_axis0", C.c_int32), ("keep1_from", C.c_int32),
                ("dst", C.c_void_p), ("dims_out", C.c_void_p)]


class OptTensor(C.Structure):
    """Mirror of ``condensa_opt_tensor``."""
    _fields_ = [("w", C.c_void_p), ("theta", C.c_void_p), ("lam", C.c_void_p), ("grad", C.c_void_p),
                ("buf1", C.c_void_p), ("buf2", C.c_void_p), ("numel", C.c_int64)]


class Opt(C.Structure):
    """Mirror of ``condensa_opt``."""
    _fields_ = [("kind", C.c_int32), ("lr", C.c_float), ("momentum", C.c_float),
                ("weight_decay", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("step", C.c_int64)]


OPT_SGD, OPT_ADAM = 0, 1


DTYPE_FP32 = 0
STATE_BLOCK = 256               # elements that share a scale of the 8-bit states


class AdamwTensor(C.Structure):
    """Mirror of ``condensa_adamw_tensor``."""
    _fields_ = [("w", C.c_void_p), ("theta", C.c_void_p), ("lam", C.c_void_p), ("grad", C.c_void_p),
                ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("w_h", C.c_void_p), ("numel", C.c_int64)]


class Adamw(C.Structure):
    """Mirror of ``condensa_adamw``."""
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("grad_scale", C.c_float), ("step", C.c_int64),
                ("grad_dtype", C.c_int32), ("state_dtype", C.c_int32), ("w_h_dtype", C.c_int32), ("state_seed", C.c_uint32)]


ADAPTER_MAX_RANK = 128


class Adapter(C.Structure):
    """Mirror of ``condensa_adapter``."""
    _fields_ = [("a", C.c_void_p), ("b", C.c_void_p), ("grad_a", C.c_void_p), ("grad_b", C.c_void_p),
                ("scale", C.c_float), ("rank", C.c_int32)]


class AdapterBatch(C.Structure):
    """Mirror of ``condensa_adapter_batch``."""
    _fields_ = [("adapters", C.c_void_p), ("n_adapters", C.c_int32), ("n_requests", C.c_int32), ("request_rows", C.c_void_p),
                ("request_adapter", C.c_void_p), ("rows", C.c_int64), ("k", C.c_int64), ("n", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


class KernelTime(C.Structure):
    """Mirror of ``condensa_kernel_time``."""
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int64), ("total_ms", C.c_double)]


_lib = None


def load():
    """Load the shared library (no GPU needed for this) and declare signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s is missing: run `python -m paper_1911_02497_b200.build`" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i32, u32, f32, f64 = C.c_void_p, C.c_int, C.c_uint, C.c_float, C.c_double
    L.condensa_create.argtypes = [C.POINTER(vp), i32, C.c_size_t]
    L.condensa_destroy.argtypes = [vp]
    L.condensa_cstep_prune.argtypes = [vp, vp, i32, f64, f32, u32, vp]
    L.condensa_cstep_filter.argtypes = [vp, vp, i32, f64, f32, u32, vp]
    L.condensa_cstep_block.argtypes = [vp, vp, i32, f64, f32, i32, i32, u32, vp]
    L.condensa_cstep_structure.argtypes = [vp, vp, i32, f64, f32, i32, u32, vp]
    L.condensa_cstep_quantize.argtypes = [vp, vp, i32, f32, i32, u32, vp]
    L.condensa_cstep_structured.argtypes = [vp, vp, i32, f64, f32, C.POINTER(StructureSpec), u32, vp]
    L.condensa_cstep_lagrange_update.argtypes = [vp, vp, i32, f32, u32, vp]
    L.condensa_cstep_host.argtypes = [vp, i32, vp, i32, f64, f32, i32, i32, u32, vp]
    L.condensa_get_result.argtypes = [vp, C.POINTER(Result)]
    L.condensa_profile_enable.argtypes = [vp, i32]
    L.condensa_profile_read.argtypes = [vp, C.POINTER(KernelTime), i32, C.POINTER(i32)]
    L.condensa_cstep_prune_noalloc.argtypes = [vp, f64, f32, u32, vp]
    L.condensa_noalloc_status.argtypes = []
    L.condensa_workspace_bytes.argtypes = [i32, vp, i32, C.POINTER(StructureSpec), u32, C.POINTER(C.c_size_t)]
    L.condensa_set_seed.argtypes = [vp, C.c_uint64]
    L.condensa_lstep_update.argtypes = [vp, vp, i32, f32, C.POINTER(Opt), vp]
    i64 = C.c_int64
    L.condensa_thin_flags.argtypes = [vp, vp, i64, i64, i64, i32, vp, vp]
    L.condensa_thin_compact.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, vp, vp]
    L.condensa_count_nonzero.argtypes = [vp, C.POINTER(vp), C.POINTER(i64), i32, vp, vp]
    L.condensa_thin_list.argtypes = [vp, C.POINTER(ThinLayer), i32, vp]
    L.condensa_lstep_adamw.argtypes = [vp, vp, i32, f32, C.POINTER(Adamw), vp, vp]
    L.condensa_grad_norm.argtypes = [vp, vp, i32, f32, i32, f32, f32, vp, vp, vp]
    L.condensa_adapter_forward.argtypes = [vp, C.POINTER(AdapterBatch), vp, i64, vp, i64, vp, i64, vp]
    L.condensa_adapter_backward.argtypes = [vp, C.POINTER(AdapterBatch), vp, i64, vp, i64, vp, i64, vp, i64, i32, vp]
    L.condensa_launch_count.argtypes = [vp]
    L.condensa_launch_count.restype = C.c_int64
    L.condensa_last_error.argtypes = [vp]
    L.condensa_last_error.restype = C.c_char_p
    for name in EXPORTS:
        getattr(L, name)
    _lib = L
    return L


def fuse_bits(fuse) -> int:
    if isinstance(fuse, int):
        return fuse
    table = {"fp16": FUSE_FP16, "lambda": FUSE_LAMBDA, "penalty": FUSE_PENALTY, "bf16": FUSE_BF16,
             "e4m3": FUSE_E4M3, "e5m2": FUSE_E5M2, "no_sampling": NO_SAMPLING}
    b = 0
    for f in fuse:
        b |= table[f]
    return b


def _addr(x) -> Optional[int]:
    """Address of a torch tensor, a numpy array, an int, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x.ctypes.data)


def tensor_table(w: Sequence, lam: Optional[Sequence] = None, theta: Optional[Sequence] = None,
                 mask: Optional[Sequence] = None, grad: Optional[Sequence] = None,
                 theta_h: Optional[Sequence] = None, shapes: Optional[Sequence] = None):
    """Build a ``condensa_tensor[T]`` array from per-tensor buffers (torch tensors
    on the device, or numpy arrays for the host entry point). Buffers must be
    contiguous; the caller keeps them alive."""
    T = len(w)
    tab = (Tensor * max(T, 1))()
    for t in range(T):
        e = tab[t]
        shp = tuple(shapes[t]) if shapes is not None else tuple(w[t].shape)
        n = 1
        for d in shp:
            n *= int(d)
        e.w = _addr(w[t])
        e.lam = _addr(lam[t]) if lam is not None else None
        e.theta = _addr(theta[t]) if theta is not None else None
        e.mask = _addr(mask[t]) if mask is not None else None
        e.grad = _addr(grad[t]) if grad is not None else None
        e.theta_h = _addr(theta_h[t]) if theta_h is not None else None
        e.numel, e.ndim = n, len(shp)
        for d in range(4):
            e.shape[d] = int(shp[d]) if d < len(shp) else 1
    return tab


def opt_table(w, theta, lam, grad, buf1=None, buf2=None):
    """``condensa_opt_tensor[T]`` from per-tensor device buffers (entries of lam/buf1/buf2 may be None)."""
    T = len(w)
    tab = (OptTensor * max(T, 1))()
    for t in range(T):
        e = tab[t]
        e.w, e.theta, e.grad = _addr(w[t]), _addr(theta[t]), _addr(grad[t])
        e.lam = _addr(lam[t]) if lam is not None else None
        e.buf1 = _addr(buf1[t]) if buf1 is not None else None
        e.buf2 = _addr(buf2[t]) if buf2 is not None else None
        e.numel = int(w[t].numel()) if hasattr(w[t], "numel") else int(w[t].size)
    return tab


_DTYPES = {"float32": DTYPE_FP32, "float16": DTYPE_FP16, "bfloat16": DTYPE_BF16, "float8_e4m3fn": DTYPE_FP8_E4M3,
           "uint8": DTYPE_FP8_E4M3}


_codes = {}                     # type object (torch's or numpy's) -> code


def _dtype_code(x, allowed, what: str, *args) -> int:
    dtype = x.dtype
    code = _codes.get(dtype)
    if code is None:
        code = _codes[dtype] = _DTYPES.get(str(dtype).replace("torch.", ""), -1)
    if code not in allowed:
        raise TypeError((what + ": type %s is not supported") % (args + (dtype,)))
    return code


def _contiguous(x) -> bool:
    return x.is_contiguous() if hasattr(x, "is_contiguous") else bool(x.flags["C_CONTIGUOUS"])


def _numel(x) -> int:
    return int(x.numel()) if hasattr(x, "numel") else int(x.size)


class AdamwTable:
    """A ``condensa_adamw_tensor[T]`` array with the types of its gradients, states and copies."""

    def __init__(self, T: int):
        self.T, self.entries = T, (AdamwTensor * max(T, 1))()
        self.grad_dtype, self.state_dtype, self.w_h_dtype = DTYPE_FP32, DTYPE_FP32, DTYPE_FP16


def adamw_table(w, grad, m=None, v=None, m_scale=None, v_scale=None, theta=None, lam=None, w_h=None) -> AdamwTable:
    """Table for :meth:`Context.lstep_adamw` and :meth:`Context.grad_norm` from per-tensor device buffers; a list or an
    entry of it may be None where the header allows NULL. ``grad`` float32, float16 or bfloat16; ``m`` and ``v`` float32, or
    float8_e4m3fn (uint8) with a float32 scale per ``STATE_BLOCK`` elements; ``w_h`` float16 or bfloat16. The caller keeps the
    buffers alive."""
    tab = AdamwTable(len(grad))
    kinds = {"grad": set(), "state": set(), "w_h": set()}
    groups = [("w", w, (DTYPE_FP32,), None), ("theta", theta, (DTYPE_FP32,), None), ("lam", lam, (DTYPE_FP32,), None),
              ("grad", grad, (DTYPE_FP32, DTYPE_FP16, DTYPE_BF16), "grad"), ("m", m, (DTYPE_FP32, DTYPE_FP8_E4M3), "state"),
              ("v", v, (DTYPE_FP32, DTYPE_FP8_E4M3), "state"), ("m_scale", m_scale, (DTYPE_FP32,), None),
              ("v_scale", v_scale, (DTYPE_FP32,), None), ("w_h", w_h, (DTYPE_FP16, DTYPE_BF16), "w_h")]
    for t in range(tab.T):
        e = tab.entries[t]
        e.numel = n = _numel(grad[t])
        for name, group, allowed, kind in groups:
            x = group[t] if group is not None else None
            if x is None:
                continue
            code = _dtype_code(x, allowed, "tensor %d: %s", t, name)
            want = -(-n // STATE_BLOCK) if name.endswith("_scale") else n
            if _numel(x) != want or not _contiguous(x):
                raise ValueError("tensor %d: %s must be contiguous and hold %d elements" % (t, name, want))
            setattr(e, name, _addr(x))
            if kind:
                kinds[kind].add(code)
    for kind, codes in kinds.items():
        if len(codes) > 1:
            raise TypeError("all tensors of a list share one type of %s" % kind)
        for code in codes:
            setattr(tab, kind + "_dtype", code)
    return tab


class AdapterTable:
    """A ``condensa_adapter`` array: the adapters that are loaded beside one projection of ``k`` to ``n``."""

    def __init__(self, entries, count: int, k: int, n: int, dtype):
        self.entries, self.count, self.k, self.n, self.dtype = entries, count, k, n, dtype
        self.code = _DTYPES[str(dtype).replace("torch.", "")]
        self.address = C.addressof(entries)
        self.max_rank = max(entries[i].rank for i in range(count))


def adapter_table(a, b, scale, grad_a=None, grad_b=None) -> AdapterTable:
    """Table for :meth:`Context.adapter_forward` and :meth:`Context.adapter_backward`: ``a[i]`` [rank_i, k] and ``b[i]`` [n, rank_i] of
    one type (float32, float16, bfloat16) on the device, ``scale[i]`` a number; ``grad_a[i]`` and ``grad_b[i]`` float32 of the same
    shapes, or None. The caller keeps the buffers alive."""
    if not len(a) or len(a) != len(b) or len(a) != len(scale):
        raise ValueError("a, b and scale need one entry per adapter, and at least one")
    k, n, dtype = int(a[0].shape[1]), int(b[0].shape[0]), a[0].dtype
    _dtype_code(a[0], (DTYPE_FP32, DTYPE_FP16, DTYPE_BF16), "adapters")
    entries = (Adapter * len(a))()
    for i, e in enumerate(entries):
        rank = int(a[i].shape[0])
        wanted = [("a", a[i], (rank, k), dtype), ("b", b[i], (n, rank), dtype)]
        for name, group, shape in (("grad_a", grad_a, (rank, k)), ("grad_b", grad_b, (n, rank))):
            if group is not None and group[i] is not None:
                wanted.append((name, group[i], shape, None))
        for name, x, shape, kind in wanted:
            if kind is None:
                _dtype_code(x, (DTYPE_FP32,), "adapter %d: %s", i, name)
            elif x.dtype != kind:
                raise TypeError("adapter %d: %s has type %s, the table's is %s" % (i, name, x.dtype, kind))
            if tuple(x.shape) != shape or not _contiguous(x):
                raise ValueError("adapter %d: %s must be contiguous, of shape %s" % (i, name, shape))
            setattr(e, name, _addr(x))
        e.scale, e.rank = float(scale[i]), rank
    return AdapterTable(entries, len(a), k, n, dtype)


_INT64, _INT32 = np.dtype(np.int64), np.dtype(np.int32)


def _host_array(x, dtype):
    if type(x) is np.ndarray and x.dtype == dtype and x.flags.c_contiguous:
        return x
    return np.ascontiguousarray(x, dtype=dtype)


def _rows_of(x, rows: int, width: int, dtype, name: str):
    """Address and row stride of a [rows, width] matrix whose rows are contiguous."""
    if x is None:
        return None, 0
    shape, (ld, step) = x.shape, (x.stride() if x.dim() == 2 else (0, 0))
    if x.dtype != dtype or len(shape) != 2 or shape[0] != rows or shape[1] < width or (width > 1 and step != 1):
        raise ValueError("%s must be a [%d, %d] matrix of %s with contiguous rows" % (name, rows, width, dtype))
    return x.data_ptr(), (ld if rows > 1 else max(width, ld))


def _kept_rows(h, rows: int, tab, batch, backward: bool):
    """Address and row stride of h, which has a column for every rank of the adapters that the call uses it for."""
    if h is None:
        return None, 0
    _dtype_code(h, (DTYPE_FP32,), "h")
    if h.dim() != 2 or h.shape[0] != rows or (h.shape[1] > 1 and h.stride(1) != 1):
        raise ValueError("h must be a float32 matrix of %d contiguous rows" % rows)
    width = h.shape[1]
    if width < tab.max_rank:            # (the library sees the stride alone, which may be a wider matrix's)
        lengths, which = batch
        used = (tab.entries[a] for a in set(which[lengths > 0].tolist()) if 0 <= a < tab.count)
        need = max([e.rank for e in used if not backward or e.grad_b] or [0])
        if width < need:
            raise CondensaError(ERR_INVALID_ARG, "h has %d columns, the adapters' ranks go to %d" % (width, need))
        if need == 0:
            return h.data_ptr(), max(width, h.stride(0))
    return h.data_ptr(), (h.stride(0) if rows > 1 else width)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)          # torch.cuda.Stream


def cstep_prune_noalloc(tab, sparsity, mu, fuse=(), stream=None):
    """``condensa_cstep_prune_noalloc``: magnitude pruning of ONE tensor (entry 0 of
    ``tab``) on the current CUDA device without any device allocation by the
    library - for callers whose memory pool owns the whole device or who cannot
    take cudaMalloc's synchronisation. At most ``NOALLOC_MAX_NUMEL`` elements;
    calls on one device must not overlap (they share one built-in scratch)."""
    L = load()
    rc = L.condensa_cstep_prune_noalloc(tab, float(sparsity), float(mu), fuse_bits(fuse),
                                        _stream_handle(stream))
    if rc != OK:
        raise CondensaError(rc, (L.condensa_last_error(None) or b"").decode())


def workspace_bytes(op: int, tab, T: int, fuse=(), spec=None) -> int:
    """``condensa_workspace_bytes``: what ``Context(device, workspace_bytes)`` must reserve so that
    calls of this shape never allocate."""
    L = load()
    n = C.c_size_t(0)
    rc = L.condensa_workspace_bytes(int(op), tab, int(T), spec, fuse_bits(fuse), C.byref(n))
    if rc != OK:
        raise CondensaError(rc, (L.condensa_last_error(None) or b"").decode())
    return int(n.value)


def noalloc_status():
    """``condensa_noalloc_status``: waits for the last allocation-free call on the current
    device and raises if one of its device-side checks failed."""
    L = load()
    rc = L.condensa_noalloc_status()
    if rc != OK:
        raise CondensaError(rc, (L.condensa_last_error(None) or b"").decode())


class Context:
    """Owns a ``condensa_ctx`` (workspace and descriptor cache of one device)."""

    _told_rounding = False

    def __init__(self, device: int = 0, workspace_bytes: int = 0):
        self._lib = load()
        h = C.c_void_p()
        rc = self._lib.condensa_create(C.byref(h), int(device), int(workspace_bytes))
        if rc != OK:
            raise CondensaError(rc, (self._lib.condensa_last_error(None) or b"").decode())
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            self._lib.condensa_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != OK:
            raise CondensaError(rc, (self._lib.condensa_last_error(self._h) or b"").decode())

    def set_seed(self, seed: int):
        self._check(self._lib.condensa_set_seed(self._h, int(seed) & ((1 << 64) - 1)))

    def cstep_prune(self, tab, T, sparsity, mu, fuse=(), stream=None):
        self._check(self._lib.condensa_cstep_prune(self._h, tab, T, float(sparsity), float(mu),
                                                   fuse_bits(fuse), _stream_handle(stream)))

    def cstep_filter(self, tab, T, sparsity, mu, fuse=(), stream=None):
        self._check(self._lib.condensa_cstep_filter(self._h, tab, T, float(sparsity), float(mu),
                                                    fuse_bits(fuse), _stream_handle(stream)))

    def cstep_structure(self, tab, T, sparsity, mu, kinds=("filter", "neuron"), fuse=(), stream=None):
        mask = sum({"filter": STRUCT_FILTER, "neuron": STRUCT_NEURON}[k] for k in set(kinds))
        self._check(self._lib.condensa_cstep_structure(self._h, tab, T, float(sparsity), float(mu), mask,
                                                       fuse_bits(fuse), _stream_handle(stream)))

    def cstep_structured(self, tab, T, sparsity, mu, kind="filter", block=None, criterion="l2", fuse=(), stream=None):
        """``kind``: 'filter', 'neuron', 'structure' (both) or 'block' with ``block`` = the extents."""
        sp = StructureSpec()
        sp.criterion = CRITERIA[criterion]
        if kind == "block":
            sp.kind, sp.ndim = SPEC_BLOCKS, len(block)
            for d, b in enumerate(block):
                sp.block[d] = int(b)
        else:
            sp.kind, sp.kinds = SPEC_SLICES, {"filter": 1, "neuron": 2, "structure": 3}[kind]
        self._check(self._lib.condensa_cstep_structured(self._h, tab, T, float(sparsity), float(mu), C.byref(sp),
                                                        fuse_bits(fuse), _stream_handle(stream)))

    def cstep_block(self, tab, T, sparsity, mu, bh=4, bw=4, fuse=(), stream=None):
        self._check(self._lib.condensa_cstep_block(self._h, tab, T, float(sparsity), float(mu),
                                                   int(bh), int(bw), fuse_bits(fuse),
                                                   _stream_handle(stream)))

    def cstep_quantize(self, tab, T, mu, dtype=DTYPE_FP16, fuse=(), stream=None):
        self._check(self._lib.condensa_cstep_quantize(self._h, tab, T, float(mu), int(dtype),
                                                      fuse_bits(fuse), _stream_handle(stream)))

    def cstep_lagrange_update(self, tab, T, mu, fuse=("lambda",), stream=None):
        self._check(self._lib.condensa_cstep_lagrange_update(self._h, tab, T, float(mu),
                                                             fuse_bits(fuse), _stream_handle(stream)))

    def cstep_host(self, op, tab, T, sparsity, mu, bh=4, bw=4, fuse=(), stream=None):
        self._check(self._lib.condensa_cstep_host(self._h, int(op), tab, T, float(sparsity),
                                                  float(mu), int(bh), int(bw), fuse_bits(fuse),
                                                  _stream_handle(stream)))

    def lstep_update(self, tab, T, mu, kind="sgd", lr=0.1, momentum=0.9, weight_decay=0.0, beta1=0.9,
                     beta2=0.999, eps=1e-8, step=1, stream=None):
        o = Opt({"sgd": OPT_SGD, "adam": OPT_ADAM}[kind], lr, momentum, weight_decay, beta1, beta2, eps, step)
        self._check(self._lib.condensa_lstep_update(self._h, tab, T, float(mu), C.byref(o),
                                                    _stream_handle(stream)))

    def lstep_adamw(self, tab: AdamwTable, mu=0.0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, step=1,
                    grad_scale=1.0, clip=None, stream=None, state_seed=0):
        """One AdamW step over the list. ``clip``: the device record of :meth:`grad_norm` (4 float32), or None. ``state_seed``: 8-bit
        states are rounded by chance with this seed (1 to 2^32 - 1; any number, the same for all steps), as training needs; with
        0 to nearest, where moments do not follow the gradients over many steps (a warning says so once). A captured call keeps
        its ``lr``, ``step`` and seed in every replay."""
        if not 0 <= state_seed < 1 << 32:
            raise ValueError("state_seed must lie in 0 .. 2^32 - 1")
        if not state_seed and step > 1 and tab.state_dtype == DTYPE_FP8_E4M3 and not self._told_rounding:
            self._told_rounding = True
            warnings.warn("8-bit moments rounded to nearest do not follow the gradients over many steps: pass a state_seed to train", stacklevel=2)
        o = Adamw(lr, beta1, beta2, eps, weight_decay, grad_scale, step, tab.grad_dtype, tab.state_dtype, tab.w_h_dtype, state_seed)
        self._check(self._lib.condensa_lstep_adamw(self._h, tab.entries, tab.T, mu, C.byref(o), _addr(clip),
                                                   _stream_handle(stream)))

    def grad_norm(self, tab: AdamwTable, mu, max_norm, clip, norms=None, grad_scale=1.0, stream=None):
        """Gradient norm of the list: ``clip`` (4 float32 on the device) receives norm, coefficient, finite flag, 0;
        ``norms`` (T float32, may be None) the norm of each tensor."""
        self._check(self._lib.condensa_grad_norm(self._h, tab.entries, tab.T, mu, tab.grad_dtype, grad_scale, max_norm,
                                                 _addr(clip), _addr(norms), _stream_handle(stream)))

    def _adapter_batch(self, tab: AdapterTable, request_rows, request_adapter, rows: int):
        """The batch, and the arrays that must live through the call."""
        lengths = _host_array(request_rows, _INT64)
        which = _host_array(request_adapter, _INT32)
        if lengths.shape != which.shape or lengths.ndim != 1:
            raise ValueError("request_rows and request_adapter need one entry per request")
        return AdapterBatch(tab.address, tab.count, lengths.size, lengths.__array_interface__["data"][0],
                            which.__array_interface__["data"][0], rows, tab.k, tab.n, tab.code, 0), (lengths, which)

    def adapter_forward(self, tab: AdapterTable, request_rows, request_adapter, x, y, h=None, stream=None):
        """``y += scale (x A^T) B^T`` row by row, each request with its adapter (-1: none). ``request_rows`` and ``request_adapter``:
        host arrays; ``x`` [rows, k] and ``y`` [rows, n] of the table's type; ``h`` [rows, max rank] float32 receives x A^T for
        :meth:`adapter_backward`, or None."""
        m = x.shape[0]
        batch, keep = self._adapter_batch(tab, request_rows, request_adapter, m)
        px, ldx = _rows_of(x, m, tab.k, tab.dtype, "x")
        py, ldy = _rows_of(y, m, tab.n, tab.dtype, "y")
        ph, ldh = _kept_rows(h, m, tab, keep, False)
        self._check(self._lib.condensa_adapter_forward(self._h, C.byref(batch), px, ldx, py, ldy, ph, ldh, _stream_handle(stream)))

    def adapter_backward(self, tab: AdapterTable, request_rows, request_adapter, x, dy, h=None, dx=None, accumulate=False, stream=None):
        """Gradients of :meth:`adapter_forward`: ``dx`` (may be None) is added to, the table's ``grad_a`` and ``grad_b`` are
        overwritten, or added to with ``accumulate``."""
        m = dy.shape[0]
        batch, keep = self._adapter_batch(tab, request_rows, request_adapter, m)
        px, ldx = _rows_of(x, m, tab.k, tab.dtype, "x")
        pdy, lddy = _rows_of(dy, m, tab.n, tab.dtype, "dy")
        pdx, lddx = _rows_of(dx, m, tab.k, tab.dtype, "dx")
        ph, ldh = _kept_rows(h, m, tab, keep, True)
        self._check(self._lib.condensa_adapter_backward(self._h, C.byref(batch), px, ldx, pdy, lddy, ph, ldh, pdx, lddx,
                                                        1 if accumulate else 0, _stream_handle(stream)))

    def thin_flags(self, theta, d0, d1, inner, axis, keep, stream=None):
        self._check(self._lib.condensa_thin_flags(self._h, _addr(theta), int(d0), int(d1), int(inner), int(axis),
                                                  _addr(keep), _stream_handle(stream)))

    def thin_compact(self, src, d0, d1, inner, keep0, keep1, dst, dims_out, stream=None):
        self._check(self._lib.condensa_thin_compact(self._h, _addr(src), int(d0), int(d1), int(inner),
                                                    _addr(keep0), _addr(keep1), _addr(dst), _addr(dims_out),
                                                    _stream_handle(stream)))

    def thin_list(self, layers, stream=None):
        """``layers``: dicts with src, d0, d1, inner, keep0, remove_axis0, keep1_from, dst, dims_out."""
        n = len(layers)
        tab = (ThinLayer * max(n, 1))()
        for e, x in zip(tab, layers):
            e.src, e.dst, e.keep0, e.dims_out = _addr(x["src"]), _addr(x["dst"]), _addr(x["keep0"]), _addr(x["dims_out"])
            e.d0, e.d1, e.inner = int(x["d0"]), int(x["d1"]), int(x["inner"])
            e.remove_axis0, e.keep1_from = int(bool(x.get("remove_axis0", True))), int(x.get("keep1_from", -1))
        self._check(self._lib.condensa_thin_list(self._h, tab, n, _stream_handle(stream)))

    def count_nonzero(self, arrays, counts, stream=None):
        """``arrays``: device float32 tensors; ``counts``: device int64 tensor of len(arrays) + 1."""
        T = len(arrays)
        ptrs = (C.c_void_p * max(T, 1))(*[_addr(a) for a in arrays])
        numel = (C.c_int64 * max(T, 1))(*[int(a.numel()) for a in arrays])
        self._check(self._lib.condensa_count_nonzero(self._h, ptrs, numel, T, _addr(counts),
                                                     _stream_handle(stream)))

    def get_result(self) -> Result:
        r = Result()
        self._check(self._lib.condensa_get_result(self._h, C.byref(r)))
        return r

    def profile_enable(self, on: bool):
        self._check(self._lib.condensa_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        """{kernel name: (launches, total ms)} since profiling was enabled."""
        buf = (KernelTime * 32)()
        n = C.c_int(0)
        self._check(self._lib.condensa_profile_read(self._h, buf, 32, C.byref(n)))
        return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms))
                for i in range(n.value)}

    def launch_count(self) -> int:
        return int(self._lib.condensa_launch_count(self._h))
