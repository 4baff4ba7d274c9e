"""ctypes binding of libgcada.so: the same entry points as include/gcada.h.

Only argument marshalling happens here; every step of the method runs in the
library's CUDA kernels.  `load()` fails loudly when the shared library is
missing or cannot be loaded: there is no fallback implementation.
"""
import ctypes as C
import functools
import os
import threading

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgcada.so")
DEBUG_LIB_PATH = os.path.join(HERE, "libgcada_dbg.so")   # the same source with every computed store index checked

OK, EINVAL, ENOMEM, ECUDA, ESTATE, ETIMEOUT = range(6)
MODEL_LOGISTIC, MODEL_MLP, MODEL_QUADRATIC = 0, 1, 2
COMPUTE_FP32, COMPUTE_BF16 = 0, 1
(OPT_RULE, OPT_REDUCTION, OPT_HISTORY, OPT_KEEP_STALE, OPT_GRAPH, OPT_TIMING, _OPT_UNUSED,
 OPT_PERSISTENT, OPT_UPLOAD, OPT_SERVER_PRECISION) = range(10)
UPLOAD_FULL, UPLOAD_MXFP4 = 0, 1
(DBG_FRESH, DBG_STALE, DBG_LHS, DBG_RHS, DBG_TAU, DBG_AGG, DBG_H, DBG_VHAT, DBG_TGROUP, DBG_GLAST,
 DBG_SRING) = range(11)
MODEL_KINDS = {"logistic": MODEL_LOGISTIC, "mlp": MODEL_MLP, "quadratic": MODEL_QUADRATIC}
COMPUTE_KINDS = {"fp32": COMPUTE_FP32, "bf16": COMPUTE_BF16}
DELAY_LAWS = {"exp": 0, "pareto": 1, "uniform": 2}
SCHEDULES = {"const": 0, "poly": 1, "step": 2}
SERVER_RULES = {"amsgrad": 0, "muon": 1}


class Model(C.Structure):
    _fields_ = [("kind", C.c_int), ("n_dims", C.c_int), ("dims", C.POINTER(C.c_int)), ("compute", C.c_int)]


class GCadaError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("gcada status %d: %s" % (status, text))
        self.status = status


# name -> (restype, argtypes): every symbol include/gcada.h declares
_VP, _LL, _ULLP = C.c_void_p, C.c_longlong, C.POINTER(C.c_ulonglong)
SIGNATURES = {
    "gcada_create": (C.c_int, [C.POINTER(Model), C.c_int, C.c_int, C.c_int, C.c_double, C.c_double, C.c_double,
                               C.c_double, C.c_double, C.POINTER(_VP)]),
    "gcada_set_stream": (C.c_int, [_VP, _VP]),
    "gcada_set_data": (C.c_int, [_VP, _VP, _VP, _LL, _LL, C.c_int]),
    "gcada_set_theta": (C.c_int, [_VP, _VP, _LL, C.c_int]),
    "gcada_set_seed": (C.c_int, [_VP, C.c_ulonglong]),
    "gcada_set_delay_model": (C.c_int, [_VP, C.c_double, C.c_double]),
    "gcada_set_option": (C.c_int, [_VP, C.c_int, C.c_double]),
    "gcada_set_delay_law": (C.c_int, [_VP, C.c_int]),
    "gcada_set_lag_weights": (C.c_int, [_VP, C.POINTER(C.c_double), C.c_int]),
    "gcada_set_step_schedule": (C.c_int, [_VP, C.c_int, C.c_double, C.c_double]),
    "gcada_set_server_rule": (C.c_int, [_VP, C.c_int, C.c_double, C.c_double, C.c_int, C.c_int]),
    "gcada_set_smoothness": (C.c_int, [_VP, C.POINTER(C.c_double), C.c_int]),
    "gcada_step": (C.c_int, [_VP, C.c_int]),
    "gcada_step_forced": (C.c_int, [_VP, C.c_int, _VP]),
    "gcada_step_host_batch": (C.c_int, [_VP, _VP, _VP]),
    "gcada_set_batch": (C.c_int, [_VP, C.c_int]),
    "gcada_get_theta": (C.c_int, [_VP, _VP, _LL]),
    "gcada_get_selection_mask": (C.c_int, [_VP, _VP, _LL, C.c_int]),
    "gcada_get_comm_count": (C.c_int, [_VP, _ULLP, _ULLP, _ULLP]),
    "gcada_get_wallclock": (C.c_int, [_VP, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "gcada_get_iteration": (C.c_int, [_VP, C.POINTER(_LL)]),
    "gcada_get_debug": (C.c_int, [_VP, C.c_int, _VP, _LL]),
    "gcada_get_group_gradient": (C.c_int, [_VP, C.c_int, C.c_int, _VP, _LL]),
    "gcada_get_launch_count": (C.c_int, [_VP, _ULLP]),
    "gcada_get_kernel_times": (C.c_int, [_VP, C.POINTER(C.c_double), C.POINTER(C.c_int)]),
    "gcada_innovation_norms_noalloc": (C.c_int, [_VP, _VP, C.c_int, _LL, _LL, _VP, _VP, C.c_char_p, C.c_size_t]),
    "gcada_operator_status": (C.c_int, [C.POINTER(_VP)]),
    "gcada_orthogonalize_work": (C.c_int, [C.c_int, C.c_int, C.c_int, C.POINTER(C.c_size_t)]),
    "gcada_orthogonalize": (C.c_int, [_VP, _VP] + [C.c_int] * 4 + [_LL] * 4 + [C.c_int] * 2 +
                            [C.POINTER(C.c_double), C.c_double, _VP, C.c_size_t, _VP, _VP, C.c_char_p, C.c_size_t]),
    "gcada_muon_update": (C.c_int, [_VP, C.c_int, _VP, _VP, C.c_int, C.c_int, C.c_int, _LL, _LL, _LL, C.c_double,
                                    C.c_double, C.c_int, C.c_double, C.c_double, C.c_int, C.c_int,
                                    C.POINTER(C.c_double), C.c_double, _VP, C.c_size_t, _VP, _VP, C.c_char_p,
                                    C.c_size_t]),
    "gcada_mx_size": (C.c_int, [_LL, _LL, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "gcada_mx_quantize": (C.c_int, [_VP, C.c_int, _LL, _LL, _LL, C.c_int, _VP, _VP, _VP, C.c_char_p, C.c_size_t]),
    "gcada_mx_dequantize": (C.c_int, [_VP, _VP, _LL, _LL, _VP, C.c_int, _LL, _VP, C.c_char_p, C.c_size_t]),
    "gcada_mx_gemm": (C.c_int, [_VP, _VP, _LL, _VP, _VP, _LL, _LL, _VP, C.c_int, _LL, C.c_double, C.c_double, _VP, _VP,
                                _VP, C.c_char_p, C.c_size_t]),
    "gcada_time_gradient": (C.c_int, [_VP, C.c_int, C.POINTER(C.c_double)]),
    "gcada_time_empty_chain": (C.c_int, [_VP, C.c_int, C.POINTER(C.c_double)]),
    "gcada_eval_loss": (C.c_int, [_VP, _LL, _LL, C.POINTER(C.c_double)]),
    "gcada_checkpoint_size": (C.c_int, [_VP, _ULLP]),
    "gcada_checkpoint_save": (C.c_int, [_VP, _VP, C.c_ulonglong]),
    "gcada_checkpoint_load": (C.c_int, [_VP, _VP, C.c_ulonglong]),
    "gcada_is_debug_build": (C.c_int, []),
    "gcada_debug_set_error": (C.c_int, [_VP, C.c_int]),
    "gcada_last_error": (C.c_char_p, [_VP]),
    "gcada_destroy": (None, [_VP]),
}

_lib = None


def load(path=None):
    """dlopen the library and attach prototypes.  Raises if it is not there."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(
            "%s is missing: build it with `python -m paper_2201_04301_b200.build` (there is no fallback)" % path)
    lib = C.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


class GCada:
    """One G-CADA context.  Method names follow the C entry points."""

    def __init__(self, kind, dims, M, M_G, D, c, alpha, beta1, beta2, eps, compute="fp32", stream=None):
        self.lib = load()
        self.dims = [int(x) for x in dims]
        arr = (C.c_int * len(self.dims))(*self.dims)
        model = Model(MODEL_KINDS[kind], len(self.dims), arr, COMPUTE_KINDS[compute])
        h = _VP()
        st = self.lib.gcada_create(C.byref(model), M, M_G, D, c, alpha, beta1, beta2, eps, C.byref(h))
        if st != OK:
            raise GCadaError(st, self.lib.gcada_last_error(None).decode())
        self.h = h
        self.G = M // M_G
        self.M, self.M_G, self.D = M, M_G, D
        if kind == "mlp":
            self.p = sum(self.dims[l] * self.dims[l - 1] + self.dims[l] for l in range(1, len(self.dims)))
        else:
            self.p = self.dims[0]
        self._keep = []
        if stream is not None:
            self.set_stream(stream)

    def _ck(self, st):
        if st != OK:
            raise GCadaError(st, self.lib.gcada_last_error(self.h).decode())

    def close(self):
        if getattr(self, "h", None):
            self.lib.gcada_destroy(self.h)
            self.h = None

    __del__ = close

    # -- setters ----------------------------------------------------------
    def set_stream(self, stream):
        """`stream`: a torch.cuda.Stream, a raw cudaStream_t integer, or None."""
        raw = getattr(stream, "cuda_stream", stream)
        self._ck(self.lib.gcada_set_stream(self.h, _VP(raw or 0)))

    def set_data(self, X, y, batch, ld=None):
        """X, y: CUDA torch tensors (borrowed; kept alive by this object)."""
        assert X.is_cuda and y.is_cuda and X.stride(-1) == 1
        self._keep = [X, y]
        ld = int(ld if ld is not None else X.stride(0))
        self._ck(self.lib.gcada_set_data(self.h, _VP(X.data_ptr()), _VP(y.data_ptr()), X.shape[0], ld, int(batch)))

    def set_batch(self, batch):
        self._ck(self.lib.gcada_set_batch(self.h, int(batch)))

    def set_theta(self, theta0):
        """theta0: float32 torch tensor (CPU or CUDA) or numpy array."""
        if hasattr(theta0, "is_cuda"):
            t = theta0.detach().contiguous()
            assert str(t.dtype) == "torch.float32"
            self._ck(self.lib.gcada_set_theta(self.h, _VP(t.data_ptr()), t.numel(), 1 if t.is_cuda else 0))
        else:
            a = np.ascontiguousarray(theta0, dtype=np.float32)
            self._ck(self.lib.gcada_set_theta(self.h, _VP(a.ctypes.data), a.size, 0))

    def set_seed(self, seed):
        self._ck(self.lib.gcada_set_seed(self.h, int(seed)))

    def set_delay_model(self, shift, rate):
        self._ck(self.lib.gcada_set_delay_model(self.h, float(shift), float(rate)))

    def set_option(self, key, value):
        self._ck(self.lib.gcada_set_option(self.h, int(key), float(value)))

    def set_delay_law(self, law):
        self._ck(self.lib.gcada_set_delay_law(self.h, DELAY_LAWS.get(law, law)))

    def set_lag_weights(self, c_d):
        if c_d is None:
            self._ck(self.lib.gcada_set_lag_weights(self.h, None, 0))
        else:
            a = (C.c_double * len(c_d))(*[float(v) for v in c_d])
            self._ck(self.lib.gcada_set_lag_weights(self.h, a, len(c_d)))

    def set_step_schedule(self, kind, a=1.0, b=0.0):
        self._ck(self.lib.gcada_set_step_schedule(self.h, SCHEDULES.get(kind, kind), float(a), float(b)))

    def set_server_rule(self, rule, weight_decay=0.0, scale=1.0, nesterov=True, steps=5):
        """`rule`: "amsgrad" (Eq. 8) or "muon" (MLPs: orthogonalised momentum for the weight matrices)."""
        self._ck(self.lib.gcada_set_server_rule(self.h, SERVER_RULES.get(rule, rule), float(weight_decay), float(scale),
                                                int(bool(nesterov)), int(steps)))

    def set_smoothness(self, L):
        a = (C.c_double * len(L))(*[float(v) for v in L])
        self._ck(self.lib.gcada_set_smoothness(self.h, a, len(L)))

    # -- stepping ----------------------------------------------------------
    def step(self, n_iters=1):
        self._ck(self.lib.gcada_step(self.h, int(n_iters)))

    def step_forced(self, mask):
        m = np.ascontiguousarray(mask, dtype=np.uint8).reshape(-1, self.G)
        self._ck(self.lib.gcada_step_forced(self.h, m.shape[0], _VP(m.ctypes.data)))

    def step_host_batch(self, Xb, yb):
        """Xb, yb: host buffers (pinned torch CPU tensors or numpy arrays)."""
        xp = Xb.data_ptr() if hasattr(Xb, "data_ptr") else Xb.ctypes.data
        yp = yb.data_ptr() if hasattr(yb, "data_ptr") else yb.ctypes.data
        self._ck(self.lib.gcada_step_host_batch(self.h, _VP(xp), _VP(yp)))

    # -- getters -----------------------------------------------------------
    def get_theta(self, out=None):
        """theta^k as p floats on the host.  `out`: an optional float32 host buffer of p elements to fill
        (a numpy array or a CPU torch tensor; a pinned one is copied into without a staging pass)."""
        if out is None:
            out = np.empty(self.p, dtype=np.float32)
        n = out.numel() if hasattr(out, "numel") else out.size
        contiguous = out.is_contiguous() if hasattr(out, "is_contiguous") else out.flags["C_CONTIGUOUS"]
        if n != self.p or "float32" not in str(out.dtype) or not contiguous or getattr(out, "is_cuda", False):
            raise ValueError("get_theta: out must be a contiguous host buffer of p = %d float32 values" % self.p)
        ptr = out.data_ptr() if hasattr(out, "data_ptr") else out.ctypes.data
        self._ck(self.lib.gcada_get_theta(self.h, _VP(ptr), self.p))
        return out

    def get_selection_mask(self, first_iter, n_iters):
        out = np.empty((n_iters, self.G), dtype=np.uint8)
        self._ck(self.lib.gcada_get_selection_mask(self.h, _VP(out.ctypes.data), int(first_iter), int(n_iters)))
        return out

    def get_comm_count(self):
        a, b, c = C.c_ulonglong(), C.c_ulonglong(), C.c_ulonglong()
        self._ck(self.lib.gcada_get_comm_count(self.h, C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def get_wallclock(self):
        a, b = C.c_double(), C.c_double()
        self._ck(self.lib.gcada_get_wallclock(self.h, C.byref(a), C.byref(b)))
        return a.value, b.value

    def get_iteration(self):
        k = _LL()
        self._ck(self.lib.gcada_get_iteration(self.h, C.byref(k)))
        return k.value

    def get_launch_count(self):
        n = C.c_ulonglong()
        self._ck(self.lib.gcada_get_launch_count(self.h, C.byref(n)))
        return n.value

    def get_group_gradient(self, what, g):
        out = np.empty(self.p, dtype=np.float32)
        self._ck(self.lib.gcada_get_group_gradient(self.h, int(what), int(g), _VP(out.ctypes.data), self.p))
        return out

    def time_gradient(self, reps):
        """Mean device time (ms) of the gradient kernel(s) over `reps` back-to-back repetitions."""
        ms = C.c_double()
        self._ck(self.lib.gcada_time_gradient(self.h, int(reps), C.byref(ms)))
        return ms.value

    def time_empty_chain(self, n_iters):
        """Device time per iteration (microseconds) of the iteration's launch structure with empty kernels."""
        us = C.c_double()
        self._ck(self.lib.gcada_time_empty_chain(self.h, int(n_iters), C.byref(us)))
        return us.value

    def get_kernel_times(self):
        """(ms_gradient, ms_select, ms_update), n_timed: see GCADA_OPT_TIMING."""
        ms = (C.c_double * 3)()
        n = C.c_int()
        self._ck(self.lib.gcada_get_kernel_times(self.h, ms, C.byref(n)))
        return (ms[0], ms[1], ms[2]), n.value

    def eval_loss(self, first_row, n_rows):
        """Mean loss of the current iterate over a range of training rows (linear models)."""
        v = C.c_double()
        self._ck(self.lib.gcada_eval_loss(self.h, int(first_row), int(n_rows), C.byref(v)))
        return v.value

    def checkpoint_save(self):
        """The run's state as a numpy byte array (see gcada_checkpoint_save)."""
        n = C.c_ulonglong()
        self._ck(self.lib.gcada_checkpoint_size(self.h, C.byref(n)))
        buf = np.empty(n.value, dtype=np.uint8)
        self._ck(self.lib.gcada_checkpoint_save(self.h, _VP(buf.ctypes.data), n.value))
        return buf

    def checkpoint_load(self, buf):
        buf = np.ascontiguousarray(buf, dtype=np.uint8)
        self._ck(self.lib.gcada_checkpoint_load(self.h, _VP(buf.ctypes.data), buf.size))

    def debug_set_error(self, dev_err):
        """Debug library only: write the device error word (0 none, 1 a wait gave up, 2 an index check failed)."""
        self._ck(self.lib.gcada_debug_set_error(self.h, int(dev_err)))

    def get_debug(self, what):
        G, p, D = self.G, self.p, self.D
        shape, dt = {
            DBG_FRESH: ((G, p), np.float32), DBG_STALE: ((G, p), np.float32), DBG_GLAST: ((G, p), np.float32),
            DBG_LHS: ((G,), np.float64), DBG_RHS: ((1,), np.float64), DBG_TAU: ((G,), np.int32),
            DBG_AGG: ((p,), np.float32), DBG_H: ((p,), np.float32), DBG_VHAT: ((p,), np.float32),
            DBG_TGROUP: ((G,), np.float64), DBG_SRING: ((D,), np.float64),
        }[what]
        out = np.empty(shape, dtype=dt)
        self._ck(self.lib.gcada_get_debug(self.h, int(what), _VP(out.ctypes.data), out.nbytes))
        return out


NOALLOC_MAX_GROUPS = 1024


def innovation_norms_noalloc(fresh, stale, lhs_out, stream=None):
    """lhs_out[g] = ||fresh[g] - stale[g]||^2 through gcada_innovation_norms_noalloc.

    fresh, stale: CUDA float32 tensors [G, p] with the same row stride; lhs_out:
    CUDA float64 tensor [G].  All of them are the caller's; the call itself
    allocates nothing on the device (its scratch is a fixed array inside the
    library, shared by every call: do not overlap calls on one GPU)."""
    lib = load()
    G, p = fresh.shape
    assert stale.shape == fresh.shape and fresh.stride(0) == stale.stride(0) and fresh.stride(1) == 1
    buf = C.create_string_buffer(256)
    raw = getattr(stream, "cuda_stream", stream)
    st = lib.gcada_innovation_norms_noalloc(_VP(fresh.data_ptr()), _VP(stale.data_ptr()), int(G), int(p),
                                            int(fresh.stride(0)), _VP(lhs_out.data_ptr()), _VP(raw or 0), buf, 256)
    if st != OK:
        raise GCadaError(st, buf.value.decode())


# ---------------------------------------------------------------------------
# Matrix operators (gcada_orthogonalize, gcada_muon_update, gcada_mx_*).  Tensors live on one CUDA device, which
# need not be the current one; their last dimension is contiguous.  stream: a torch.cuda.Stream, a raw cudaStream_t
# integer, or None for torch's current stream of that device.  On another stream than the current one the caller orders the
# inputs' writers before the call; what the call itself takes from torch's allocator (a result without `out`, a work area
# without `work`) makes that stream wait for all that the current one holds, so calls that are to run beside it bring both.
# None of them is differentiable: results carry no gradient, whatever the inputs require.  Tensors that a call writes
# have their version counters raised, as by torch's own in-place operations.
# ---------------------------------------------------------------------------
PRECISIONS = {"full": 0, "half": 1}
MUON_COEF = (3.4445, -4.7750, 2.0315)
_NO_WORK = 256       # a work area of this size is asked for, but not used (narrow matrices stay on chip)
_unused_work = {}    # device index -> one such area, shared by every call
_status_words = {}   # device index -> address of the word that a kernel whose bounded wait gave up makes non-zero


def _compute_type(t, what):
    import torch
    if t.dtype is torch.float32:
        return COMPUTE_FP32
    if t.dtype is torch.bfloat16:
        return COMPUTE_BF16
    raise ValueError("%s must be float32 or bfloat16, not %s" % (what, t.dtype))


def _matrix(t, what, dims=(2,)):
    """Checks a row-major device matrix; its row stride."""
    shape, stride = t.shape, t.stride()
    if not t.is_cuda:
        raise ValueError("%s must be a CUDA tensor" % what)
    if len(shape) not in dims:
        raise ValueError("%s must have %s dimensions, not %d" % (what, " or ".join(map(str, dims)), len(shape)))
    rows, cols = shape[-2:]
    if cols > 1 and stride[-1] != 1:
        raise ValueError("%s: the last dimension must be contiguous" % what)
    if rows <= 1:
        return cols
    if stride[-2] < cols:
        raise ValueError("%s: rows overlap" % what)
    return stride[-2]


_messages = threading.local()


class _Launch:
    """Device, stream and message buffer of one operator call on `first`'s device."""

    def __init__(self, first, others, stream):
        import torch
        self.torch, self.first, self.device, self.lib = torch, first, first.device, _lib or load()
        for t in others:
            if t is not None and t.device != self.device:
                raise ValueError("tensors on different devices: %s and %s" % (self.device, t.device))
        self.index = self.device.index
        current = torch._C._cuda_getCurrentRawStream(self.index)
        self.raw, self.other = current, None
        if stream is not None:
            self.raw = int(getattr(stream, "cuda_stream", stream))
            if self.raw != current:
                # memory taken from torch's allocator belongs to the current stream; a call on another one says so
                self.other = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(self.raw, self.device)

    def fresh(self, *shape, dtype):
        t = self.first.new_empty(shape, dtype=dtype)
        if self.other is not None:  # the caching allocator may hand out memory that the current stream still uses
            self.other.wait_stream(self.torch.cuda.current_stream(self.device))
            t.record_stream(self.other)
        return t

    def status(self):
        w = _status_words.get(self.index)
        if w is None:
            word = _VP()
            with self.torch.cuda.device(self.index):
                st = self.lib.gcada_operator_status(C.byref(word))
            if st != OK:
                raise GCadaError(st, "no status word on device %d" % self.index)
            w = _status_words[self.index] = word.value
        return w

    def call(self, fn, args, tensors, written=()):
        """`written`: what the caller gave to be written."""
        buf = getattr(_messages, "buf", None)
        if buf is None:
            buf = _messages.buf = C.create_string_buffer(256)   # one a thread
        if self.torch._C._cuda_getDevice() == self.index:
            st = fn(*args, self.raw, buf, 256)
        else:
            with self.torch.cuda.device(self.index):
                st = fn(*args, self.raw, buf, 256)
        if st != OK:
            raise GCadaError(st, buf.value.decode())
        if written:
            self.torch.autograd.graph.increment_version(written)
        if self.other is not None:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.other)


class _Word:
    """One int32 at a device address, for torch.as_tensor."""

    def __init__(self, address):
        self.__cuda_array_interface__ = dict(shape=(1,), typestr="<i4", data=(address, False), version=2)


def _status_word(index):
    """The device's status word as a tensor, or None if no operator has run there."""
    import torch
    w = _status_words.get(index)
    return None if w is None else torch.as_tensor(_Word(w), device=torch.device("cuda", index))


def check_operators(device=None):
    """Waits for the device (by default, and for "cuda", the current one) and raises (GCADA_ETIMEOUT) if a kernel of the
    matrix operators ever gave up a wait there since the last check, in the replay of a graph too."""
    import torch
    index = device if isinstance(device, int) else None if device is None else torch.device(device).index
    if index is None:
        index = torch.cuda.current_device()
    torch.cuda.synchronize(index)
    w = _status_word(index)
    if w is not None and int(w.item()):
        w.zero_()
        raise GCadaError(ETIMEOUT, "a bounded device-side wait of a matrix operator gave up")


_coef_arrays = {}


def _steps(steps, coef, eps, precision):
    if precision is None:
        precision = "full"
    if precision not in PRECISIONS:
        raise ValueError("precision must be 'full' or 'half', not %r" % (precision,))
    array = _coef_arrays.get(coef) if type(coef) is tuple else None
    if array is None:
        if len(coef) != 3:
            raise ValueError("coef must hold three values")
        array = (C.c_double * 3)(*[float(v) for v in coef])
        if coef == MUON_COEF:
            _coef_arrays[MUON_COEF] = array
    return PRECISIONS[precision], int(steps), array, float(eps)


@functools.lru_cache(maxsize=256)
def _work_bytes(batch, rows, cols):
    n = C.c_size_t()
    st = load().gcada_orthogonalize_work(batch, rows, cols, C.byref(n))
    if st != OK:
        raise GCadaError(st, "matrix sizes out of range")
    return n.value


def _ns_work(run, batch, rows, cols, work):
    if work is None:
        need = _work_bytes(batch, rows, cols)
        if need > _NO_WORK:
            work = run.fresh(need, dtype=run.torch.uint8)
        else:
            work = _unused_work.get(run.index)
            if work is None:
                work = run.fresh(_NO_WORK, dtype=run.torch.uint8)
                if not run.torch.cuda.is_current_stream_capturing():   # (a graph's own memory goes with the graph)
                    _unused_work[run.index] = work
    elif not work.is_contiguous():
        raise ValueError("work must be contiguous")
    return work, work.data_ptr(), work.numel() * work.element_size()


def orthogonalize(g, out=None, steps=5, coef=MUON_COEF, eps=1e-7, precision=None, work=None, stream=None):
    """`g` ([rows, cols] or [batch, rows, cols], float32 or bfloat16) after `steps` Newton-Schulz steps: a matrix of
    the same singular vectors whose singular values are near one.  See gcada_orthogonalize.  `precision`: "full" (the
    default, for either type) or "half", up to three times as fast but with an error that can be above half a step of
    bfloat16 (GCADA_PRECISION_HALF).  `out` may be `g`.  `work`: a tensor of at least
    orthogonalize_work(g) bytes to use as the work area, by default taken from torch's allocator."""
    kind, ld_g = _compute_type(g, "g"), _matrix(g, "g", (2, 3))
    run = _Launch(g, (out, work), stream)
    shape, written = g.shape, () if out is None else (out,)
    if out is None:
        out = run.torch.empty_like(g) if run.other is None and g.is_contiguous() else run.fresh(*shape, dtype=g.dtype)
    elif out.shape != shape or out.dtype != g.dtype:
        raise ValueError("out must have g's shape and type")
    ld_o = _matrix(out, "out", (2, 3))
    rows, cols = shape[-2:]
    batch, stride_g, stride_o = (shape[0], g.stride(0), out.stride(0)) if len(shape) == 3 else (1, 0, 0)
    precision, steps, coef, eps = _steps(steps, coef, eps, precision)
    work, ptr, size = _ns_work(run, batch, rows, cols, work)
    run.call(run.lib.gcada_orthogonalize,
             (g.data_ptr(), out.data_ptr(), kind, batch, rows, cols, ld_g, stride_g, ld_o, stride_o, precision, steps,
              coef, eps, ptr, size, run.status()), (g, out, work), written)
    return out


def orthogonalize_work(g):
    """Bytes of the work area that orthogonalize(g) or muon_update(w=g) needs."""
    rows, cols = g.shape[-2:]
    return _work_bytes(g.shape[0] if g.dim() == 3 else 1, rows, cols)


def muon_update(w, m, g, lr, beta=0.95, nesterov=True, weight_decay=0.0, scale=None, steps=5, coef=MUON_COEF,
                eps=1e-7, precision=None, work=None, stream=None):
    """One optimiser step of the weight matrix `w`, in place with its momentum `m` (float32); `g` is the gradient.
    See gcada_muon_update.  `scale`: by default sqrt(max(1, rows / cols)).  `precision`: "full" (the default) or
    "half", see orthogonalize."""
    w_kind, g_kind = _compute_type(w, "w"), _compute_type(g, "g")
    ld_w, ld_m, ld_g = _matrix(w, "w"), _matrix(m, "m"), _matrix(g, "g")
    if _compute_type(m, "m") != COMPUTE_FP32:
        raise ValueError("m must be float32")
    rows, cols = w.shape
    if m.shape != w.shape or g.shape != w.shape:
        raise ValueError("w, m and g must have the same shape")
    run = _Launch(w, (m, g, work), stream)
    if scale is None:
        scale = max(1.0, rows / max(1, cols)) ** 0.5
    precision, steps, coef, eps = _steps(steps, coef, eps, precision)
    work, ptr, size = _ns_work(run, 1, rows, cols, work)
    run.call(run.lib.gcada_muon_update,
             (w.data_ptr(), w_kind, m.data_ptr(), g.data_ptr(), g_kind, rows, cols, ld_w, ld_m, ld_g, float(lr),
              float(beta), int(bool(nesterov)), float(weight_decay), float(scale), precision, steps, coef, eps, ptr,
              size, run.status()), (w, m, g, work), (w, m))


@functools.lru_cache(maxsize=256)
def _mx_bytes(rows, cols):
    n, s = C.c_size_t(), C.c_size_t()
    st = load().gcada_mx_size(rows, cols, C.byref(n), C.byref(s))
    if st != OK:
        raise GCadaError(st, "matrix sizes out of range")
    return n.value, s.value


class MxMatrix:
    """A rows x cols matrix in microscaled 4-bit floating point (layout: include/gcada.h).  `codes`, `scales`: uint8
    CUDA tensors of the sizes that gcada_mx_size gives, any shape, contiguous."""

    def __init__(self, rows, cols, codes, scales):
        self.rows, self.cols = int(rows), int(cols)
        for t, want, name in zip((codes, scales), _mx_bytes(self.rows, self.cols), ("codes", "scales")):
            if not t.is_cuda or str(t.dtype) != "torch.uint8" or not t.is_contiguous() or t.numel() != want:
                raise ValueError("%s of a %d x %d matrix must be a contiguous CUDA tensor of %d bytes"
                                 % (name, self.rows, self.cols, want))
        if codes.device != scales.device:
            raise ValueError("codes and scales on different devices")
        self._parts = codes, scales
        self._where = codes.data_ptr(), scales.data_ptr()

    @classmethod
    def _fresh(cls, run, rows, cols):
        """One allocation for both arrays (a row of codes is a multiple of 16 bytes, so the scales are aligned)."""
        self = cls.__new__(cls)
        self.rows, self.cols = rows, cols
        n, s = _mx_bytes(rows, cols)
        both = run.fresh(n + s, dtype=run.torch.uint8)
        self._parts, at = (both,), both.data_ptr()
        self._where = at, at + n
        return self

    def _part(self, i):
        if len(self._parts) == 1:
            self._parts = self._parts[0].split(_mx_bytes(self.rows, self.cols))
        return self._parts[i]

    codes = property(lambda self: self._part(0), doc="the elements, two to a byte")
    scales = property(lambda self: self._part(1), doc="the blocks' scales")

    def dequantize(self, dtype=None, out=None, stream=None):
        """The values as a float32 (default) or bfloat16 tensor.  See gcada_mx_dequantize."""
        run, written = _Launch(self._parts[0], (out,), stream), () if out is None else (out,)
        if out is None:
            out = run.fresh(self.rows, self.cols, dtype=dtype or run.torch.float32)
        elif tuple(out.shape) != (self.rows, self.cols) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be a %d x %d matrix of the type asked for" % (self.rows, self.cols))
        ld = _matrix(out, "out")
        run.call(run.lib.gcada_mx_dequantize,
                 (*self._where, self.rows, self.cols, out.data_ptr(), _compute_type(out, "out"), ld),
                 (*self._parts, out), written)
        return out


def mx_quantize(x, transpose=False, out=None, stream=None):
    """`x` (float32 or bfloat16 [rows, cols]), or with `transpose` its transpose, as an MxMatrix.  See
    gcada_mx_quantize.  `out`: an MxMatrix of the result's shape to fill."""
    kind, ld = _compute_type(x, "x"), _matrix(x, "x")
    rows, cols = x.shape
    shape = (cols, rows) if transpose else (rows, cols)
    written = () if out is None else out._parts
    run = _Launch(x, written, stream)
    if out is None:
        out = MxMatrix._fresh(run, *shape)
    elif (out.rows, out.cols) != shape:
        raise ValueError("out must be %d x %d" % shape)
    run.call(run.lib.gcada_mx_quantize,
             (x.data_ptr(), kind, rows, cols, ld, 1 if transpose else 0, *out._where), (x, *out._parts), written)
    return out


def mx_gemm(a, b, out=None, dtype=None, alpha=1.0, beta=0.0, bias=None, stream=None):
    """alpha a b^T + bias + beta out for MxMatrix operands a (m x k) and b (n x k), as a float32 (default) or bfloat16
    tensor.  See gcada_mx_gemm.  `bias`: float32, n values."""
    if a.cols != b.cols:
        raise ValueError("a has %d columns and b %d" % (a.cols, b.cols))
    run, written = _Launch(a._parts[0], (b._parts[0], out, bias), stream), () if out is None else (out,)
    if out is None:
        if beta != 0:
            raise ValueError("beta needs out")
        out = run.fresh(a.rows, b.rows, dtype=dtype or run.torch.float32)
    elif tuple(out.shape) != (a.rows, b.rows) or (dtype is not None and out.dtype != dtype):
        raise ValueError("out must be a %d x %d matrix of the type asked for" % (a.rows, b.rows))
    if bias is not None and (str(bias.dtype) != "torch.float32" or bias.numel() != b.rows or not bias.is_contiguous()):
        raise ValueError("bias must hold %d contiguous float32 values" % b.rows)
    ld = _matrix(out, "out")
    run.call(run.lib.gcada_mx_gemm,
             (*a._where, a.rows, *b._where, b.rows, a.cols, out.data_ptr(), _compute_type(out, "out"), ld, float(alpha),
              float(beta), None if bias is None else bias.data_ptr(), run.status()),
             (*a._parts, *b._parts, out, bias), written)
    return out


def from_workload(w, stream=None, options=None, smoothness=None, c_d=None, schedule=None, delay_law=None,
                  server_rule=None):
    """Context for a dict made by workloads.make_workload (tensors on CUDA)."""
    g = GCada(w["kind"], w["dims"], w["M"], w["M_G"], w["D"], w["c"], w["alpha"], w["beta1"], w["beta2"],
              w["eps"], compute=w["compute"], stream=stream)
    g.set_seed(w["seed"])
    g.set_delay_model(w["shift"], w["rate"])
    for key, val in (options or {}).items():
        g.set_option(key, val)
    if smoothness is not None:
        g.set_smoothness(smoothness)
    if c_d is not None:
        g.set_lag_weights(c_d)
    if schedule is not None:
        g.set_step_schedule(*schedule)
    if delay_law is not None:
        g.set_delay_law(delay_law)
    if server_rule is not None:
        g.set_server_rule(**server_rule)
    g.set_data(w["X"], w["y"], w["batch"], ld=w["ld"])
    g.set_theta(w["theta0"])
    return g
