"""Python binding of libfstcompose.so (argument marshalling only).

Every step of the composition runs in the library's HIP kernels; this module
only passes device pointers and the current HIP stream across the C ABI
declared in ``include/fst_compose.h``.  PyTorch supplies device memory and
streams.  There is no fallback: if the library is missing or cannot be loaded
the calls raise.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfstcompose.so")

FST_OK = 0
FST_ERR_INVALID_ARG = 1
FST_ERR_INVALID_GRAPH = 2
FST_ERR_TOO_LARGE = 3
FST_ERR_NOMEM = 4
FST_ERR_HIP = 5
FST_ERR_STATE = 6
FST_ERR_CYCLIC = 7
FST_ERR_NOT_CONVERGED = 8

FST_OPT_MAX_WORKSPACE = 1
FST_OPT_TIMING = 2
FST_OPT_LABEL_BUCKETS = 3
FST_OPT_CHAIN_DEPTH = 4
FST_OPT_COUNT_MOVES = 5
FST_OPT_ORDER = 6
FST_OPT_VALIDATE = 7
FST_OPT_LIST_CAPACITY = 8

FST_SCATTER_NOALLOC_MAX_TARGETS = 1 << 20

FST_ORDER_FORWARD_FIRST = 0
FST_ORDER_COACCESSIBLE_FIRST = 1
FST_ORDER_CONCURRENT = 2

FST_F32 = 0
FST_F16 = 1
FST_BF16 = 2

FST_RECURRENCE_MAX_SEQS = 1 << 22
FST_RECURRENCE_SAVE_ROWS = 64
FST_HEAD_MAX_ROWS = 1 << 25
FST_HEAD_MAX_COLS = 1 << 22

PHASES = ("preprocess", "forward", "backward", "count", "fill")

# kernels timed one by one (enum fst_kernel): a composition's, then a score's
KERNELS = ("search_forward", "search_backward", "count", "fill")
SCORE_KERNELS = ("score_gen", "score_prep")
KERNELS3 = ("search3", "compact3")


class FstError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {_strerror(code)} (code {code})")


class _Graph(ctypes.Structure):
    _fields_ = [("num_states", ctypes.c_int32), ("num_arcs", ctypes.c_int32),
                ("arc_offset", ctypes.c_void_p), ("src", ctypes.c_void_p),
                ("dst", ctypes.c_void_p), ("ilabel", ctypes.c_void_p),
                ("olabel", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("start", ctypes.c_void_p), ("accept", ctypes.c_void_p)]


class _GraphOut(ctypes.Structure):
    _fields_ = [("arc_offset", ctypes.c_void_p), ("src", ctypes.c_void_p),
                ("dst", ctypes.c_void_p), ("ilabel", ctypes.c_void_p),
                ("olabel", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("start", ctypes.c_void_p), ("accept", ctypes.c_void_p),
                ("key_a", ctypes.c_void_p), ("key_b", ctypes.c_void_p),
                ("key_f", ctypes.c_void_p), ("arc_a", ctypes.c_void_p),
                ("arc_b", ctypes.c_void_p)]


class _GraphOut3(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "arc_offset", "src", "dst", "ilabel", "olabel", "weight", "start", "accept", "key_a",
        "key_b", "key_fab", "key_d", "key_f", "arc_a", "arc_b", "arc_d")]


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("stride", ctypes.c_int64), ("type", ctypes.c_int32)]


class _Recurrence(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("offset", ctypes.c_void_p),
                ("reverse", ctypes.c_int32), ("x", _Matrix), ("gate", _Matrix),
                ("state", ctypes.c_void_p)]


class _Stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in (
        "key_space", "accessible", "coaccessible", "generated", "fwd_levels",
        "bwd_levels", "heavy_states", "num_states", "num_arcs", "generated_backward")]


_lib = None


def load():
    """Load the HIP library (raises if it was not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "or python -m paper_2110_02848_amd.build")
    lib = ctypes.CDLL(LIB_PATH)
    lib.fst_ctx_create.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_void_p)]
    lib.fst_ctx_create.restype = ctypes.c_int
    lib.fst_ctx_destroy.argtypes = [ctypes.c_void_p]
    lib.fst_ctx_destroy.restype = None
    lib.fst_ctx_set_option.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64]
    lib.fst_ctx_set_option.restype = ctypes.c_int
    lib.fst_compose_run.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Graph),
                                    ctypes.POINTER(_Graph), ctypes.c_void_p,
                                    ctypes.POINTER(ctypes.c_int64),
                                    ctypes.POINTER(ctypes.c_int64)]
    lib.fst_compose_run.restype = ctypes.c_int
    lib.fst_compose_fill.argtypes = [ctypes.c_void_p, ctypes.POINTER(_GraphOut), ctypes.c_void_p]
    lib.fst_compose_fill.restype = ctypes.c_int
    lib.fst_compose_stats.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Stats)]
    lib.fst_compose_stats.restype = ctypes.c_int
    lib.fst_compose_phase_times.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_float),
                                            ctypes.c_int]
    lib.fst_compose_phase_times.restype = ctypes.c_int
    lib.fst_compose_kernel_time.argtypes = [ctypes.c_void_p, ctypes.c_int,
                                            ctypes.POINTER(ctypes.c_float),
                                            ctypes.POINTER(ctypes.c_int64)]
    lib.fst_compose_kernel_time.restype = ctypes.c_int
    lib.fst_score.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Graph), ctypes.c_void_p,
                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.fst_score.restype = ctypes.c_int
    lib.fst_score_cyclic.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Graph), ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                                     ctypes.c_double, ctypes.POINTER(ctypes.c_int32),
                                     ctypes.c_void_p]
    lib.fst_score_cyclic.restype = ctypes.c_int
    lib.fst_score_posterior.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Graph),
                                        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p]
    lib.fst_score_posterior.restype = ctypes.c_int
    lib.fst_grad_scatter.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                     ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p,
                                     ctypes.c_void_p]
    lib.fst_grad_scatter.restype = ctypes.c_int
    lib.fst_grad_scatter_noalloc.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p,
                                             ctypes.c_void_p]
    lib.fst_grad_scatter_noalloc.restype = ctypes.c_int
    lib.fst_compose_batch_run.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Graph), ctypes.c_int32,
                                          ctypes.POINTER(_Graph), ctypes.c_void_p,
                                          ctypes.POINTER(ctypes.c_int64),
                                          ctypes.POINTER(ctypes.c_int64), ctypes.c_void_p,
                                          ctypes.c_void_p]
    lib.fst_compose_batch_run.restype = ctypes.c_int
    lib.fst_segment_logsum.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p]
    lib.fst_segment_logsum.restype = ctypes.c_int
    lib.fst_compose3_run.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Graph),
                                     ctypes.POINTER(_Graph), ctypes.POINTER(_Graph),
                                     ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                     ctypes.POINTER(ctypes.c_int64)]
    lib.fst_compose3_run.restype = ctypes.c_int
    lib.fst_compose3_fill.argtypes = [ctypes.c_void_p, ctypes.POINTER(_GraphOut3),
                                      ctypes.c_void_p]
    lib.fst_compose3_fill.restype = ctypes.c_int
    lib.fst_compose3_stats.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Stats)]
    lib.fst_compose3_stats.restype = ctypes.c_int
    P = ctypes.c_void_p
    M = ctypes.POINTER(_Matrix)
    R = ctypes.POINTER(_Recurrence)
    for name, args in dict(
            fst_recurrence_run=[P, R, M, P, P, P],
            fst_recurrence_grads=[P, R, P, M, P, M, M, P, P],
            fst_recurrence_step=[P, M, M, P, P, P, ctypes.c_int32, M, P],
            fst_emission_weights=[P, M, M, P, P],
            fst_emission_grads=[P, M, M, P, P, M, M, P],
            fst_cross_entropy=[P, M, M, P, P, P, P],
            fst_cross_entropy_grads=[P, M, M, P, P, P, M, M, P]).items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = ctypes.c_int
    lib.fst_strerror.argtypes = [ctypes.c_int]
    lib.fst_strerror.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _strerror(code):
    try:
        return load().fst_strerror(code).decode()
    except Exception:  # pragma: no cover - message only
        return "error"


def _check(rc, where):
    if rc != FST_OK:
        raise FstError(rc, where)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr() if t is not None and t.numel() else None)


def _stream_handle(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


_types = {}  # torch type -> enum fst_type


def _view(t, name):
    """(address, rows, cols, stride, type) of a 2-D device tensor whose rows are
    contiguous."""
    typ = _types.get(t.dtype)
    if typ is None and not _types:
        import torch
        _types.update({torch.float32: FST_F32, torch.float16: FST_F16,
                       torch.bfloat16: FST_BF16})
        typ = _types.get(t.dtype)
    if typ is None or not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{name}: a 2-D device tensor of float32, float16 or bfloat16 is needed")
    rows, cols = t.shape
    step, inner = t.stride()
    if inner != 1 and cols > 1 and rows > 0:
        raise ValueError(f"{name}: the elements of a row must lie side by side")
    if step < cols:
        if rows > 1:
            raise ValueError(f"{name}: rows overlap")
        step = cols
    return t.data_ptr() if rows and cols else 0, rows, cols, step, typ


def _matrix(t, name):
    return _Matrix(*_view(t, name))


class _Marshal:
    """The structures that the calls of a context pass, made once and filled for
    each call (a context is one thread's)."""
    _VIEW = struct.Struct("<Qqqqi")
    _RECURRENCE = struct.Struct("<i4xQi4xQqqqi4xQqqqi4xQ")

    def __init__(self):
        self._m = [_Matrix() for _ in range(4)]
        self._ref = [ctypes.byref(m) for m in self._m]
        self._r = _Recurrence()

    def matrix(self, i, t, name):
        self._VIEW.pack_into(self._m[i], 0, *_view(t, name))
        return self._ref[i]

    def made(self, i, t, typ):
        """The same of a tensor made for the call."""
        rows, cols = t.shape
        self._VIEW.pack_into(self._m[i], 0, t.data_ptr() if rows and cols else 0, rows, cols, cols,
                             typ)
        return self._ref[i]

    def recurrence(self, n, offset, reverse, x, gate, state):
        self._RECURRENCE.pack_into(self._r, 0, n, offset or 0, reverse, *_view(x, "x"),
                                   *_view(gate, "gate"), state or 0)
        return self._r


def _array(t, name, dtype, n):
    """Address of a contiguous device tensor of n elements (None: NULL)."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous device tensor of {n} {dtype} is needed")
    return t.data_ptr() if n else None


def _address(t):
    """Address of a tensor made here (None, or nothing in it: NULL)."""
    return t.data_ptr() if t is not None and t.numel() else None


GRAPH_DTYPES = dict(arc_offset=np.int32, src=np.int32, dst=np.int32, ilabel=np.int32,
                    olabel=np.int32, weight=np.float32, start=np.uint8, accept=np.uint8)


def to_device(g, device="cuda:0"):
    """Copy a numpy graph dict to device tensors (dict with the same keys)."""
    import torch
    out = {"num_states": int(g["num_states"])}
    for k, dt in GRAPH_DTYPES.items():
        out[k] = torch.from_numpy(np.ascontiguousarray(g[k], dtype=dt)).to(device)
    return out


def _graph_struct(g):
    s = _Graph()
    s.num_states = int(g["num_states"])
    s.num_arcs = int(g["src"].numel())
    for k in GRAPH_DTYPES:
        setattr(s, k, _ptr(g[k]))
    return s


class Composer:
    """Owns one library context on one device (reuse it across calls)."""

    def __init__(self, device=0):
        self._lib = load()
        self.device = int(device)
        h = ctypes.c_void_p()
        _check(self._lib.fst_ctx_create(self.device, ctypes.byref(h)), "fst_ctx_create")
        self._h = h
        self.options = {}  # options set on this context (option -> value)
        import torch
        self._dev = torch.device("cuda", self.device)
        self._pass = _Marshal()
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self._empty = torch.empty
        self._f32, self._i32 = torch.float32, torch.int32

    def close(self):
        if getattr(self, "_h", None):
            self._lib.fst_ctx_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover - interpreter shutdown order
        try:
            self.close()
        except Exception:
            pass

    def set_option(self, option, value):
        _check(self._lib.fst_ctx_set_option(self._h, option, int(value)), "fst_ctx_set_option")
        self.options[option] = int(value)

    def run(self, A, B, stream=None):
        """Phase 1: search, trim, number and count.  Returns (V_C, E_C)."""
        ga, gb = _graph_struct(A), _graph_struct(B)
        nv, ne = ctypes.c_int64(), ctypes.c_int64()
        rc = self._lib.fst_compose_run(self._h, ctypes.byref(ga), ctypes.byref(gb),
                                       _stream_handle(stream), ctypes.byref(nv), ctypes.byref(ne))
        _check(rc, "fst_compose_run")
        return int(nv.value), int(ne.value)

    def alloc_output(self, nv, ne, provenance=True, keys=True):
        import torch
        dev = f"cuda:{self.device}"
        i32 = dict(dtype=torch.int32, device=dev)
        u8 = dict(dtype=torch.uint8, device=dev)
        C = dict(num_states=nv, num_arcs=ne,
                 arc_offset=torch.empty(nv + 1, **i32),
                 src=torch.empty(ne, **i32), dst=torch.empty(ne, **i32),
                 ilabel=torch.empty(ne, **i32), olabel=torch.empty(ne, **i32),
                 weight=torch.empty(ne, dtype=torch.float32, device=dev),
                 start=torch.empty(nv, **u8), accept=torch.empty(nv, **u8))
        if keys:
            C.update(key_a=torch.empty(nv, **i32), key_b=torch.empty(nv, **i32),
                     key_f=torch.empty(nv, **u8))
        if provenance:
            C.update(arc_a=torch.empty(ne, **i32), arc_b=torch.empty(ne, **i32))
        return C

    def fill(self, C, stream=None):
        """Phase 2: write C into the tensors of ``alloc_output`` (async)."""
        o = _GraphOut()
        o.arc_offset = ctypes.c_void_p(C["arc_offset"].data_ptr())
        for k in ("src", "dst", "ilabel", "olabel", "weight", "start", "accept",
                  "key_a", "key_b", "key_f", "arc_a", "arc_b"):
            setattr(o, k, _ptr(C.get(k)))
        _check(self._lib.fst_compose_fill(self._h, ctypes.byref(o), _stream_handle(stream)),
               "fst_compose_fill")
        return C

    def compose(self, A, B, provenance=True, keys=True, stream=None):
        """C = A o B as a dict of device tensors (asynchronous fill)."""
        nv, ne = self.run(A, B, stream)
        C = self.alloc_output(nv, ne, provenance, keys)
        return self.fill(C, stream)

    def run_batch(self, As, B, stream=None):
        """Phase 1 of C_i = A_i o B for every A_i of the list, in one pass.
        Returns (V_C, E_C, item_states, item_arcs): the sizes of the one C
        (the union of the C_i) and the numpy int64 [n + 1] ranges of each
        item's states and arcs in it."""
        n = len(As)
        arr = (_Graph * max(n, 1))()
        for i, A in enumerate(As):
            arr[i] = _graph_struct(A)
        gb = _graph_struct(B)
        nv, ne = ctypes.c_int64(), ctypes.c_int64()
        st = np.zeros(n + 1, np.int64)
        ar = np.zeros(n + 1, np.int64)
        rc = self._lib.fst_compose_batch_run(self._h, arr, n, ctypes.byref(gb),
                                             _stream_handle(stream), ctypes.byref(nv),
                                             ctypes.byref(ne), st.ctypes.data, ar.ctypes.data)
        _check(rc, "fst_compose_batch_run")
        return int(nv.value), int(ne.value), st, ar

    def compose_batch(self, As, B, provenance=True, keys=True, stream=None):
        """C = union of A_i o B as one dict of device tensors (ids of the
        union), with the per-item ranges: (C, item_states, item_arcs)."""
        nv, ne, st, ar = self.run_batch(As, B, stream)
        C = self.alloc_output(nv, ne, provenance, keys)
        return self.fill(C, stream), st, ar

    def segment_logsum(self, val, flag, bounds, stream=None):
        """totals[i] = log-sum of exp(val[v]) over flagged v in
        [bounds[i], bounds[i + 1]) (float64 [n] tensor)."""
        import torch
        b = np.ascontiguousarray(bounds, dtype=np.int64)
        n = len(b) - 1
        out = torch.empty(max(n, 0), dtype=torch.float64, device=f"cuda:{self.device}")
        rc = self._lib.fst_segment_logsum(self._h, _ptr(val), _ptr(flag), n, b.ctypes.data,
                                          _ptr(out), _stream_handle(stream))
        _check(rc, "fst_segment_logsum")
        return out

    def stats(self):
        st = _Stats()
        _check(self._lib.fst_compose_stats(self._h, ctypes.byref(st)), "fst_compose_stats")
        return {n: int(getattr(st, n)) for n, _ in _Stats._fields_}

    def phase_times(self):
        buf = (ctypes.c_float * len(PHASES))()
        _check(self._lib.fst_compose_phase_times(self._h, buf, len(PHASES)),
               "fst_compose_phase_times")
        return dict(zip(PHASES, [float(x) for x in buf]))

    def kernel_times(self):
        """{kernel: (ms, launches)} of the last timed run + fill."""
        out = {}
        for i, name in enumerate(KERNELS):
            ms, n = ctypes.c_float(), ctypes.c_int64()
            _check(self._lib.fst_compose_kernel_time(self._h, i, ctypes.byref(ms), ctypes.byref(n)),
                   "fst_compose_kernel_time")
            out[name] = (float(ms.value), int(n.value))
        return out


    # ---- three inputs at once: C = A o B o D ----

    def run3(self, A, B, D, stream=None):
        """Phase 1 of C = A o B o D.  Returns (V_C, E_C)."""
        ga, gb, gd = _graph_struct(A), _graph_struct(B), _graph_struct(D)
        nv, ne = ctypes.c_int64(), ctypes.c_int64()
        rc = self._lib.fst_compose3_run(self._h, ctypes.byref(ga), ctypes.byref(gb),
                                        ctypes.byref(gd), _stream_handle(stream),
                                        ctypes.byref(nv), ctypes.byref(ne))
        _check(rc, "fst_compose3_run")
        return int(nv.value), int(ne.value)

    def alloc_output3(self, nv, ne, provenance=True, keys=True):
        import torch
        C = self.alloc_output(nv, ne, provenance=provenance, keys=keys)
        dev = f"cuda:{self.device}"
        if keys:
            C.update(key_fab=torch.empty(nv, dtype=torch.uint8, device=dev),
                     key_d=torch.empty(nv, dtype=torch.int32, device=dev))
        if provenance:
            C["arc_d"] = torch.empty(ne, dtype=torch.int32, device=dev)
        return C

    def fill3(self, C, stream=None):
        o = _GraphOut3()
        for k, _ in _GraphOut3._fields_:
            setattr(o, k, _ptr(C.get(k)))
        o.arc_offset = ctypes.c_void_p(C["arc_offset"].data_ptr())
        _check(self._lib.fst_compose3_fill(self._h, ctypes.byref(o), _stream_handle(stream)),
               "fst_compose3_fill")
        return C

    def compose3(self, A, B, D, provenance=True, keys=True, stream=None):
        """C = A o B o D (composed at once) as a dict of device tensors."""
        nv, ne = self.run3(A, B, D, stream)
        C = self.alloc_output3(nv, ne, provenance, keys)
        return self.fill3(C, stream)

    def stats3(self):
        st = _Stats()
        _check(self._lib.fst_compose3_stats(self._h, ctypes.byref(st)), "fst_compose3_stats")
        return {n: int(getattr(st, n)) for n, _ in _Stats._fields_}

    def kernel_times3(self):
        """{kernel: (ms, launches)} of the last timed fst_compose3_run + fill."""
        out = {}
        for i, name in enumerate(KERNELS3):
            ms, n = ctypes.c_float(), ctypes.c_int64()
            _check(self._lib.fst_compose_kernel_time(self._h, 6 + i, ctypes.byref(ms),
                                                     ctypes.byref(n)),
                   "fst_compose_kernel_time")
            out[name] = (float(ms.value), int(n.value))
        return out

    # ---- scores of an acyclic graph and their gradient ----

    def score(self, G, alpha=True, beta=True, stream=None):
        """Forward / backward log-semiring scores of an acyclic graph of
        device tensors: dict(alpha, beta: float64 [V] tensors or None, total:
        float64 [1] tensor).  Raises FstError(FST_ERR_CYCLIC) on a cycle."""
        import torch
        dev = f"cuda:{self.device}"
        V = int(G["num_states"])
        a = torch.empty(V, dtype=torch.float64, device=dev) if alpha else None
        b = torch.empty(V, dtype=torch.float64, device=dev) if beta else None
        total = torch.empty(1, dtype=torch.float64, device=dev)
        g = _graph_struct(G)
        rc = self._lib.fst_score(self._h, ctypes.byref(g), _ptr(a), _ptr(b),
                                 ctypes.c_void_p(total.data_ptr()), _stream_handle(stream))
        _check(rc, "fst_score")
        return dict(alpha=a, beta=b, total=total)

    def score_cyclic(self, G, alpha=True, beta=True, max_sweeps=10000, tol=0.0, stream=None):
        """The same scores of a graph that may have cycles, by relaxation
        sweeps: dict(alpha, beta, total as in ``score``, sweeps: the number
        of sweeps until none raised a value by more than ``tol``).  Raises
        FstError(FST_ERR_NOT_CONVERGED) if that took more than max_sweeps."""
        import torch
        dev = f"cuda:{self.device}"
        V = int(G["num_states"])
        a = torch.empty(V, dtype=torch.float64, device=dev) if alpha else None
        b = torch.empty(V, dtype=torch.float64, device=dev) if beta else None
        total = torch.empty(1, dtype=torch.float64, device=dev)
        n = ctypes.c_int32(0)
        g = _graph_struct(G)
        rc = self._lib.fst_score_cyclic(self._h, ctypes.byref(g), _ptr(a), _ptr(b),
                                        ctypes.c_void_p(total.data_ptr()), int(max_sweeps),
                                        float(tol), ctypes.byref(n), _stream_handle(stream))
        _check(rc, "fst_score_cyclic")
        return dict(alpha=a, beta=b, total=total, sweeps=int(n.value))

    def posterior(self, G, alpha, beta, total, scale=1.0, stream=None):
        """scale * d total / d w for every arc (float32 [E] tensor)."""
        import torch
        grad = torch.empty(int(G["src"].numel()), dtype=torch.float32,
                           device=f"cuda:{self.device}")
        g = _graph_struct(G)
        rc = self._lib.fst_score_posterior(self._h, ctypes.byref(g), _ptr(alpha), _ptr(beta),
                                           ctypes.c_void_p(total.data_ptr()), float(scale),
                                           _ptr(grad), _stream_handle(stream))
        _check(rc, "fst_score_posterior")
        return grad

    def grad_scatter(self, grad, idx, m, stream=None):
        """out[i] = sum of grad[e] over idx[e] = i (float32 [m] tensor)."""
        import torch
        out = torch.empty(int(m), dtype=torch.float32, device=f"cuda:{self.device}")
        rc = self._lib.fst_grad_scatter(self._h, int(grad.numel()), _ptr(grad), _ptr(idx),
                                        int(m), _ptr(out), _stream_handle(stream))
        _check(rc, "fst_grad_scatter")
        return out

    def grad_scatter_noalloc(self, grad, idx, m, out=None, stream=None):
        """grad_scatter through the entry point that allocates no device
        memory (m <= FST_SCATTER_NOALLOC_MAX_TARGETS); ``out`` (float32 [m])
        may be passed in, so that the call itself allocates nothing."""
        import torch
        if out is None:
            out = torch.empty(int(m), dtype=torch.float32, device=f"cuda:{self.device}")
        rc = self._lib.fst_grad_scatter_noalloc(self._h, int(grad.numel()), _ptr(grad), _ptr(idx),
                                                int(m), _ptr(out), _stream_handle(stream))
        _check(rc, "fst_grad_scatter_noalloc")
        return out

    def operand_grads(self, C, A_arcs, B_arcs, scale=1.0, stream=None):
        """Gradient of scale * total(C) by the arc weights of A and B (C
        filled with provenance): (grad_A [A_arcs], grad_B [B_arcs])."""
        sc = self.score(C, stream=stream)
        post = self.posterior(C, sc["alpha"], sc["beta"], sc["total"], scale, stream)
        return (self.grad_scatter(post, C["arc_a"], A_arcs, stream),
                self.grad_scatter(post, C["arc_b"], B_arcs, stream))

    # ---- between a network and its graphs ----
    # Gradients are calls of their own: results carry no autograd history, whether
    # or not an argument requires a gradient.

    def _call_stream(self, stream):
        return self._raw_stream(self.device) if stream is None else stream.cuda_stream

    def _new(self, stream, shape, dtype):
        """A tensor that belongs to the stream of the call."""
        if stream is None:
            return self._empty(shape, dtype=dtype, device=self._dev)
        import torch
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=self._dev)

    def _copy(self, stream, to, from_):
        if stream is None:
            to.copy_(from_)
            return
        import torch
        with torch.cuda.stream(stream):
            to.copy_(from_)

    def _uses(self, stream, *tensors):
        """Tells the allocator that the stream of the call uses these."""
        if stream is not None:
            for t in tensors:
                if t is not None and t.numel():
                    t.record_stream(stream)

    def recurrence(self, x, gate, offset, state=None, reverse=False, save=False, stream=None):
        """Gated linear recurrence over the sequences offset[s] .. offset[s + 1]
        of rows of x and gate ([N, D], offset int32 [n + 1]) from state
        (float32 [n, D], None: 0): dict(y: as x, last: the states after each
        sequence, saved: what ``recurrence_grads`` needs, with ``save``)."""
        R, n = self._recurrence(x, gate, offset, state, reverse)
        N, D = x.shape
        y = self._new(stream, (N, D), x.dtype)
        last = self._new(stream, (n, D), self._f32)
        saved = self._new(stream, (N // FST_RECURRENCE_SAVE_ROWS + n, D),
                          self._f32) if save else None
        self._uses(stream, x, gate, offset, state)
        rc = self._lib.fst_recurrence_run(self._h, R, self._pass.made(0, y, _types[y.dtype]),
                                          _address(last), _address(saved),
                                          self._call_stream(stream))
        _check(rc, "fst_recurrence_run")
        return dict(y=y, last=last, saved=saved)

    def recurrence_grads(self, x, gate, offset, grad_y, saved, state=None, grad_last=None,
                         reverse=False, stream=None):
        """Gradients of a loss by x, gate and state from those by y and last
        (``recurrence`` of the same arguments with ``save``): dict(x, gate:
        as x, state: float32 [n, D])."""
        R, n = self._recurrence(x, gate, offset, state, reverse)
        N, D = x.shape
        rows = N // FST_RECURRENCE_SAVE_ROWS + n
        gx, gu = self._new(stream, (N, D), x.dtype), self._new(stream, (N, D), x.dtype)
        gs = self._new(stream, (n, D), self._f32)
        self._uses(stream, x, gate, offset, grad_y, saved, state, grad_last)
        rc = self._lib.fst_recurrence_grads(
            self._h, R, _array(saved, "saved", self._f32, rows * D),
            self._pass.matrix(0, grad_y, "grad_y"),
            _array(grad_last, "grad_last", self._f32, n * D),
            self._pass.made(1, gx, _types[x.dtype]), self._pass.made(2, gu, _types[x.dtype]),
            _address(gs), self._call_stream(stream))
        _check(rc, "fst_recurrence_grads")
        return dict(x=gx, gate=gu, state=gs)

    def _recurrence(self, x, gate, offset, state, reverse):
        n = int(offset.numel()) - 1
        if n < 0:
            raise ValueError("offset: at least one entry is needed")
        R = self._pass.recurrence(n, _array(offset, "offset", self._i32, n + 1),
                                  int(bool(reverse)), x, gate,
                                  _array(state, "state", self._f32, n * x.shape[-1]))
        return R, n

    def recurrence_step(self, x, gate, state, slot=None, out=None, stream=None):
        """One step of the rows of x and gate ([n, D]): (y, new states).
        state: float32 [n, D], or more rows, which stay as they are; the new
        states go to ``out`` (may be state) or a new tensor.  With slot (int32
        [n]) state holds any number of rows, row i's is slot[i] (an idle row's
        lies outside), and the new states replace the old ones unless ``out``
        is given.  Rows of ``out`` that no row of x names are not written."""
        shape = x.shape
        slots, D = state.shape[0], shape[-1]
        from_ = _array(state, "state", self._f32, slots * D)
        if out is not None and out is not state:
            to = _array(out, "out", self._f32, slots * D)
        elif out is state or slot is not None:
            out, to = state, from_
        else:
            out = self._new(stream, (slots, D), self._f32)
            to = _address(out)
            if slots > shape[0]:  # states that this step leaves alone
                self._copy(stream, out[shape[0]:], state.view(slots, D)[shape[0]:])
        y = self._new(stream, shape, x.dtype)
        if stream is not None:
            self._uses(stream, x, gate, state, slot, out)
        rc = self._lib.fst_recurrence_step(
            self._h, self._pass.matrix(0, x, "x"), self._pass.matrix(1, gate, "gate"), from_, to,
            _array(slot, "slot", self._i32, shape[0]), slots,
            self._pass.made(2, y, _types[x.dtype]), self._call_stream(stream))
        _check(rc, "fst_recurrence_step")
        return y, out

    def emission_weights(self, x, w, out=None, stream=None):
        """Log-softmax of x w^T, float32 [N, C] (x [N, H], w [C, H]): the arc
        weights of emission graphs.  ``out`` may be a graph's weight tensor."""
        N, C = x.shape[0], w.shape[0]
        if out is None:
            out = self._new(stream, (N, C), self._f32)
            to = _address(out)
        else:
            to = _array(out, "out", self._f32, N * C)
        self._uses(stream, x, w, out)
        rc = self._lib.fst_emission_weights(self._h, self._pass.matrix(0, x, "x"),
                                            self._pass.matrix(1, w, "w"), to,
                                            self._call_stream(stream))
        _check(rc, "fst_emission_weights")
        return out

    def emission_grads(self, x, w, weight, grad, need_x=True, need_w=True, stream=None):
        """Gradients by x and w (None where not needed) from the gradient by
        the weights of ``emission_weights`` (grad: float32, N * C)."""
        n = int(x.shape[0]) * int(w.shape[0])
        gx, gw = self._head_grads(x, w, need_x, need_w, stream)
        self._uses(stream, x, w, weight, grad)
        rc = self._lib.fst_emission_grads(
            self._h, self._pass.matrix(0, x, "x"), self._pass.matrix(1, w, "w"),
            _array(weight, "weight", self._f32, n), _array(grad, "grad", self._f32, n),
            self._pass.made(2, gx, _types[x.dtype]) if need_x else None,
            self._pass.made(3, gw, _types[w.dtype]) if need_w else None, self._call_stream(stream))
        _check(rc, "fst_emission_grads")
        return gx, gw

    def cross_entropy(self, x, w, target, stream=None):
        """Cross entropy of x w^T (x [N, H], w [V, H]) against target (int32
        [N], -1: no word): dict(loss, lse: float32 [N])."""
        N = int(x.shape[0])
        loss = self._new(stream, (N,), self._f32)
        lse = self._new(stream, (N,), self._f32)
        self._uses(stream, x, w, target)
        rc = self._lib.fst_cross_entropy(self._h, self._pass.matrix(0, x, "x"),
                                         self._pass.matrix(1, w, "w"),
                                         _array(target, "target", self._i32, N),
                                         _address(loss), _address(lse),
                                         self._call_stream(stream))
        _check(rc, "fst_cross_entropy")
        return dict(loss=loss, lse=lse)

    def cross_entropy_grads(self, x, w, target, lse, grad=None, need_x=True, need_w=True,
                            stream=None):
        """Gradients of sum(grad * loss) by x and w (None where not needed);
        grad: float32 [N], None: 1."""
        N = int(x.shape[0])
        gx, gw = self._head_grads(x, w, need_x, need_w, stream)
        self._uses(stream, x, w, target, lse, grad)
        rc = self._lib.fst_cross_entropy_grads(
            self._h, self._pass.matrix(0, x, "x"), self._pass.matrix(1, w, "w"),
            _array(target, "target", self._i32, N), _array(lse, "lse", self._f32, N),
            _array(grad, "grad", self._f32, N),
            self._pass.made(2, gx, _types[x.dtype]) if need_x else None,
            self._pass.made(3, gw, _types[w.dtype]) if need_w else None, self._call_stream(stream))
        _check(rc, "fst_cross_entropy_grads")
        return gx, gw

    def _head_grads(self, x, w, need_x, need_w, stream):
        return (self._new(stream, x.shape, x.dtype) if need_x else None,
                self._new(stream, w.shape, w.dtype) if need_w else None)

    def score_kernel_times(self):
        """{kernel: (ms, launches)} of the last timed fst_score."""
        out = {}
        for i, name in enumerate(SCORE_KERNELS):
            ms, n = ctypes.c_float(), ctypes.c_int64()
            _check(self._lib.fst_compose_kernel_time(self._h, len(KERNELS) + i, ctypes.byref(ms),
                                                     ctypes.byref(n)),
                   "fst_compose_kernel_time")
            out[name] = (float(ms.value), int(n.value))
        return out


def to_numpy(C):
    """Device result dict -> numpy dict (synchronises)."""
    out = {}
    for k, v in C.items():
        out[k] = v.cpu().numpy() if hasattr(v, "cpu") else v
    return out


def compose_numpy(A, B, device=0, composer=None):
    """Convenience: numpy graphs in, numpy canonical C out (via the GPU)."""
    comp = composer or Composer(device)
    dev = f"cuda:{comp.device}"
    C = comp.compose(to_device(A, dev), to_device(B, dev))
    return to_numpy(C)
