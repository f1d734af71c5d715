"""Thin ctypes binding of libadapm (include/adapm.h): argument marshalling only.

Every entry point of the C ABI has a method of the same name (without the
``adapm_`` prefix) on ParameterManager.  Arrays may be torch tensors on the
GPU or on the host (pinned or not) or numpy arrays; keys are passed as
32-bit integers, rows as float32.  All work runs in the library's CUDA
kernels; if the library is missing this module raises instead of falling
back to anything else.
"""
import collections
import contextlib
import ctypes
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libadapm.so")

OK, EINVAL, ERANGE, ENOMEM, ESTATE, ECUDA, ETIMEOUT = range(7)
STATUS_NAMES = {0: "OK", 1: "EINVAL", 2: "ERANGE", 3: "ENOMEM", 4: "ESTATE", 5: "ECUDA", 6: "ETIMEOUT"}
NUM_OPS = 8
OP_NAMES = ["intent", "advance", "pull", "push", "sync", "step", "push_kernel", "pull_kernel"]
NO_KEY = 0xFFFFFFFF
_CUDA_STREAM_LEGACY = 0x1

EXPORTS = [
    "adapm_create", "adapm_destroy", "adapm_intent", "adapm_advance_clock", "adapm_pull",
    "adapm_push", "adapm_sync", "adapm_wait", "adapm_mf_step", "adapm_complex_step",
    "adapm_sgns_step", "adapm_clock", "adapm_replica_keys", "adapm_replica_rows",
    "adapm_refcounts", "adapm_owners", "adapm_poisson_quantile", "adapm_read_main", "adapm_get_stats", "adapm_profile_enable",
    "adapm_profile_read", "adapm_kernel_launches", "adapm_push_noalloc", "adapm_last_error",
    "adapm_debug_fail_next_barrier", "adapm_debug_fail_next_launch",
    "adapm_embed", "adapm_embed_grad", "adapm_grad_norm", "adapm_clip_grads", "adapm_push_grads",
    "adapm_layer_norm", "adapm_layer_norm_grad", "adapm_linear", "adapm_linear_grad", "adapm_distill",
]


class Config(ctypes.Structure):
    _fields_ = [
        ("num_keys", ctypes.c_uint64),
        ("value_len", ctypes.c_uint32),
        ("num_workers", ctypes.c_uint32),
        ("replica_capacity", ctypes.c_uint64),
        ("init_values", ctypes.c_void_p),
        ("stream", ctypes.c_void_p),
        ("relocate", ctypes.c_int32),
        ("action_timing", ctypes.c_int32),
        ("timing_alpha", ctypes.c_double),
        ("timing_p", ctypes.c_double),
        ("timing_lambda0", ctypes.c_double),
        ("delta_refresh", ctypes.c_int32),
        ("no_push_plans", ctypes.c_int32),
        ("pull_staging", ctypes.c_int32),
        ("no_early_events", ctypes.c_int32),
    ]


ACTION_TIMING = {"start": 0, "adaptive": 1, "signal": 2}


class Stats(ctypes.Structure):
    _fields_ = [
        ("live_replicas", ctypes.c_uint64),
        ("high_water", ctypes.c_uint64),
        ("capacity", ctypes.c_uint64),
        ("created", ctypes.c_uint64),
        ("destroyed", ctypes.c_uint64),
        ("last_push_unique", ctypes.c_uint64),
        ("push_rows", ctypes.c_uint64),
        ("push_unique", ctypes.c_uint64),
        ("sync_keys", ctypes.c_uint64),
        ("sync_replicas", ctypes.c_uint64),
        ("relocations", ctypes.c_uint64),
        ("sync_refreshed", ctypes.c_uint64),
        ("planned_pushes", ctypes.c_uint64),
        ("plan_misses", ctypes.c_uint64),
        ("early_advances", ctypes.c_uint64),
        ("early_undone", ctypes.c_uint64),
    ]


F32, F16, BF16 = range(3)


class _Tokens(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("id_bits", ctypes.c_int32), ("has_pad", ctypes.c_int32),
                ("pad", ctypes.c_int64), ("outer", ctypes.c_uint64), ("inner", ctypes.c_uint64),
                ("outer_stride", ctypes.c_int64), ("inner_stride", ctypes.c_int64)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("type", ctypes.c_int32), ("outer_stride", ctypes.c_int64),
                ("inner_stride", ctypes.c_int64)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_uint64), ("live", ctypes.c_void_p),
                ("row_len", ctypes.c_uint32), ("type", ctypes.c_int32)]


class _Shape(ctypes.Structure):
    _fields_ = [("outer", ctypes.c_uint64), ("inner", ctypes.c_uint64), ("dim", ctypes.c_uint32)]


class _Vector(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("type", ctypes.c_int32)]


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("type", ctypes.c_int32), ("row_stride", ctypes.c_int64),
                ("col_stride", ctypes.c_int64)]


class _Layer(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint64), ("ins", ctypes.c_uint32), ("outs", ctypes.c_uint32)]


class _Teacher(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("id_bits", ctypes.c_int32), ("logits", ctypes.c_void_p),
                ("type", ctypes.c_int32), ("top", ctypes.c_uint32)]


class _Labels(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("id_bits", ctypes.c_int32), ("has_pad", ctypes.c_int32),
                ("pad", ctypes.c_int64)]


class AdaPMError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


_lib = None


def load(path=LIB_PATH):
    """Load libadapm.so and declare its signatures (raises if it is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build()")
    L = ctypes.CDLL(path)
    P, U32, U64, I64, F, I = (ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int64,
                              ctypes.c_float, ctypes.c_int)
    sig = {
        "adapm_create": [ctypes.POINTER(Config), ctypes.POINTER(P)],
        "adapm_destroy": [P],
        "adapm_intent": [P, U32, P, U64, I64, I64],
        "adapm_advance_clock": [P, U32],
        "adapm_pull": [P, U32, P, U64, P],
        "adapm_push": [P, U32, P, U64, P],
        "adapm_sync": [P],
        "adapm_wait": [P],
        "adapm_mf_step": [P, U32, P, P, P, U64, U32, I, F, F, P],
        "adapm_complex_step": [P, U32, P, P, P, P, U64, U32, U32, F, F, P],
        "adapm_sgns_step": [P, U32, P, P, P, U64, U32, U32, U32, U32, F, P],
        "adapm_clock": [P, U32, ctypes.POINTER(I64)],
        "adapm_replica_keys": [P, U32, P, U64, ctypes.POINTER(U64)],
        "adapm_replica_rows": [P, U32, P, U64, P, P, P],
        "adapm_refcounts": [P, U32, P, U64, P],
        "adapm_owners": [P, P, U64, P],
        "adapm_poisson_quantile": [ctypes.c_double, ctypes.c_double, ctypes.POINTER(I64)],
        "adapm_read_main": [P, P, U64, P],
        "adapm_get_stats": [P, ctypes.POINTER(Stats)],
        "adapm_profile_enable": [P, I],
        "adapm_profile_read": [P, P, P],
        "adapm_kernel_launches": [ctypes.POINTER(U64)],
        "adapm_push_noalloc": [P, U32, P, U64, P],
        "adapm_debug_fail_next_barrier": [P],
        "adapm_debug_fail_next_launch": [P],
        "adapm_embed": [P, U32, P, U32, F, P],
        "adapm_embed_grad": [P, U32, P, U32, F, P, P, P, P],
        "adapm_grad_norm": [P, P, U64, F, P],
        "adapm_clip_grads": [P, P, P, U64, F, F, P],
        "adapm_push_grads": [P, U32, P, P, U64, U32, I, F, F, F, F, P],
        "adapm_layer_norm": [P, P, P, P, P, F, P, P],
        "adapm_layer_norm_grad": [P, P, P, P, P, P, P, P, P],
        "adapm_linear": [P, P, P, P, P, ctypes.c_int32, P, P, P],
        "adapm_linear_grad": [P, P, P, P, P, P, ctypes.c_int32, P, P, P],
        "adapm_distill": [P, P, P, P, F, F, P, F, F, P, P, P],
    }
    for name, args in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    L.adapm_last_error.argtypes = [P]
    L.adapm_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


def kernel_launches():
    """Kernels launched by libadapm in this process so far."""
    v = ctypes.c_uint64()
    st = load().adapm_kernel_launches(ctypes.byref(v))
    if st != OK:
        raise AdaPMError(st, "adapm_kernel_launches")
    return v.value


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_torch_types = None   # (Tensor, int32, float32), once torch is needed


def _plain_tensor(a, which):
    """Whether `a` is a contiguous tensor of int32 (which = 1) or float32 (2): passed on as it is."""
    global _torch_types
    if _torch_types is None:
        torch = _torch()
        _torch_types = (torch.Tensor, torch.int32, torch.float32)
    return isinstance(a, _torch_types[0]) and a.dtype is _torch_types[which] and a.is_contiguous()


class _Arr:
    """A pointer to a contiguous array and the object that keeps it alive."""

    __slots__ = ("ptr", "keep", "n")

    def __init__(self, ptr, keep, n):
        self.ptr, self.keep, self.n = ptr, keep, n


def _keys(a):
    if a is None:
        return _Arr(None, None, 0)
    if _plain_tensor(a, 1):
        n = a.numel()
        return _Arr(a.data_ptr() if n else None, a, n)
    if isinstance(a, np.ndarray) or isinstance(a, (list, tuple)):
        arr = np.ascontiguousarray(np.asarray(a, dtype=np.int64).astype(np.uint32))
        return _Arr(arr.ctypes.data if arr.size else None, arr, arr.size)
    torch = _torch()
    t = a.reshape(-1)
    if t.dtype != torch.int32:
        t = t.to(torch.int32)
    t = t.contiguous()
    return _Arr(t.data_ptr() if t.numel() else None, t, t.numel())


def _floats(a, dtype_np=np.float32):
    if a is None:
        return _Arr(None, None, 0)
    if _plain_tensor(a, 2):
        n = a.numel()
        return _Arr(a.data_ptr() if n else None, a, n)
    if isinstance(a, np.ndarray) or isinstance(a, (list, tuple)):
        arr = np.ascontiguousarray(np.asarray(a, dtype=dtype_np))
        return _Arr(arr.ctypes.data if arr.size else None, arr, arr.size)
    torch = _torch()
    t = a.contiguous()
    if t.dtype != torch.float32:
        t = t.to(torch.float32)
    return _Arr(t.data_ptr() if t.numel() else None, t, t.numel())


def _out_ptr(t):
    if isinstance(t, np.ndarray):
        assert t.flags["C_CONTIGUOUS"]
        return t.ctypes.data if t.size else None
    assert t.is_contiguous()
    return t.data_ptr() if t.numel() else None


# -- token embeddings --------------------------------------------------------------
_NOTHING = contextlib.nullcontext()
_float_types = {}   # torch dtype -> element type of the ABI


def _type_of(dtype):
    known = _float_types.get(dtype)
    if known is None:
        torch = _torch()
        _float_types.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
        if dtype not in _float_types:
            raise ValueError(f"rows and gradients are float32, float16 or bfloat16, not {dtype}")
        known = _float_types[dtype]
    return known


def _one_stride(shape, strides):
    """The step that walks these dimensions in order, None if there is none (0 where nothing is stepped over)."""
    step, size = 0, 1
    for n, s in zip(reversed(shape), reversed(strides)):
        if n == 1:
            continue
        if size > 1 and s != step * size:
            return None
        if size == 1:
            step = s
        size *= n
    return step


def _two_levels(shape, *strides):
    """(outer, inner, (outer stride, inner stride) of each), or None: an outer and an inner step for all of them."""
    if len(shape) == 1:
        return (1, shape[0], *((0, s[0]) for s in strides))
    for cut in range(len(shape) + 1):
        steps = [(_one_stride(shape[:cut], s[:cut]), _one_stride(shape[cut:], s[cut:])) for s in strides]
        if all(a is not None and b is not None for a, b in steps):
            outer = inner = 1
            for n in shape[:cut]:
                outer *= n
            for n in shape[cut:]:
                inner *= n
            return (outer, inner, *steps)
    return None


class RowGrads(collections.namedtuple("RowGrads", ["keys", "rows", "count"])):
    """Gradient rows of distinct keys (adapm_embed_grad): keys (int32, ascending, then -1), rows (float32, one per
    key) and count (int32, one element: how many of them there are)."""

    __slots__ = ()


class GradList:
    """Gradients for grad_norm and clip_grads: CUDA tensors without gaps (float32, float16, bfloat16) and RowGrads.
    A program whose gradient buffers stay can make its list once; the list keeps its tensors alive."""

    def __init__(self, grads):
        self.grads = list(grads)
        self.array = (_Tensor * max(1, len(self.grads)))()
        self.n = len(self.grads)
        for a, g in zip(self.array, self.grads):
            rows = g
            if isinstance(g, RowGrads):
                rows = g.rows
                a.live, a.row_len = g.count.data_ptr(), rows.shape[-1]
            if not rows.is_cuda or not rows.is_contiguous():
                raise ValueError("gradients are CUDA tensors without gaps")
            a.data, a.count, a.type = rows.data_ptr(), rows.numel(), _type_of(rows.dtype)


def _check_norm(norm):
    if norm is not None and not (norm.is_cuda and norm.dtype is _torch().float32 and norm.numel() == 1):
        raise ValueError("norm is a float32 scalar on the GPU")


def _grad_list(grads):
    return grads if isinstance(grads, GradList) else GradList(grads)


# -- dense layers ------------------------------------------------------------------
class NormGrads(collections.namedtuple("NormGrads", ["x", "weight", "bias"])):
    """Gradients of a layer norm's input, weight and bias (adapm_layer_norm_grad); None where one is not wanted."""

    __slots__ = ()


class LinearGrads(collections.namedtuple("LinearGrads", ["x", "weight", "bias"])):
    """Gradients of a dense layer's input, weight and bias (adapm_linear_grad); None where one is not wanted."""

    __slots__ = ()


ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4, "tanh": 5}


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(a for a in ACTIVATIONS if a)}")
    return ACTIVATIONS[name]


class _Dense:
    """Descriptors that the calls on dense layers refill (making one anew takes longer than filling it)."""

    __slots__ = ("shape", "layer", "rows", "matrices", "vectors", "teacher", "labels", "shape_ref", "layer_ref",
                 "rows_ref", "other_rows", "matrices_ref", "vectors_ref", "teacher_ref", "labels_ref")

    def __init__(self):
        self.shape, self.layer, self.teacher, self.labels = _Shape(), _Layer(), _Teacher(), _Labels()
        self.rows, self.vectors = [_Rows() for _ in range(3)], [_Vector() for _ in range(3)]
        self.matrices = [_Matrix() for _ in range(6)]
        for name in ("shape", "layer", "teacher", "labels"):
            setattr(self, name + "_ref", ctypes.byref(getattr(self, name)))
        self.other_rows = self.rows[1:]
        for name in ("rows", "vectors", "matrices"):
            setattr(self, name + "_ref", [ctypes.byref(a) for a in getattr(self, name)])


def poisson_quantile(lam, p):
    """The p quantile of Poisson(lam) as the library's adaptive action timing computes it (host only)."""
    out = ctypes.c_int64()
    st = load().adapm_poisson_quantile(float(lam), float(p), ctypes.byref(out))
    if st != OK:
        raise AdaPMError(st, "adapm_poisson_quantile: need lam > 0 and 0 < p < 1")
    return out.value


class ParameterManager:
    """One adapm context (adapm_create).  Device arrays are used in place; host arrays are copied.

    relocate        move a key to its only worker with active intent instead of replicating it (Sec. 4.1)
    action_timing   "start" (act when an intent becomes active), "adaptive" (Algorithm 1 at each sync, with
                    timing_alpha / timing_p / timing_lambda0, 0 = the paper's 0.1 / 0.9999 / 10) or "signal"
    delta_refresh   versioned refresh: sync leaves a sole holder's value when nobody else wrote the key
    push_plans      sort each intent's keys beside the library stream and let a push with the same keys
                    use that sort (adapm_intent); False sorts every push itself
    pull_staging    pull rows through shared memory with bulk copies instead of through registers
    early_events    compute the refcount changes of a worker's next advance beside its pull and push
                    (adapm_advance_clock); False computes them in the advance
    """

    def __init__(self, num_keys, value_len, num_workers, replica_capacity=0, init_values=None,
                 stream=None, relocate=False, action_timing="start", timing_alpha=0.0, timing_p=0.0,
                 timing_lambda0=0.0, delta_refresh=False, push_plans=True, pull_staging=False,
                 early_events=True):
        self._lib = load()
        torch = _torch()
        if stream is None:
            stream = torch.cuda.current_stream()
        self.stream = stream
        self.K, self.D, self.W = int(num_keys), int(value_len), int(num_workers)
        init = _floats(init_values)
        if init.ptr is not None and init.n != self.K * self.D:
            raise ValueError("init_values must hold num_keys * value_len floats")
        # torch's default stream has handle 0; the ABI reads NULL as "make a
        # stream of your own", so name the legacy default stream (0x1) instead
        handle = stream.cuda_stream or _CUDA_STREAM_LEGACY
        self.relocate = bool(relocate)
        if action_timing not in ACTION_TIMING:
            raise ValueError(f"action_timing must be one of {sorted(ACTION_TIMING)}")
        self.action_timing = action_timing
        cfg = Config(self.K, self.D, self.W, int(replica_capacity), init.ptr,
                     ctypes.c_void_p(handle), int(self.relocate), ACTION_TIMING[action_timing],
                     float(timing_alpha), float(timing_p), float(timing_lambda0), int(bool(delta_refresh)),
                     int(not push_plans), int(bool(pull_staging)), int(not early_events))
        h = ctypes.c_void_p()
        st = self._lib.adapm_create(ctypes.byref(cfg), ctypes.byref(h))
        if st != OK:
            raise AdaPMError(st, "adapm_create failed")
        self._h = h
        self._handle = stream.cuda_stream
        self._device = torch.device("cuda", torch.cuda.current_device())
        _type_of(torch.float32)   # (fills the table of types)
        self._t, self._r = _Tokens(), _Rows()   # refilled by every call that takes tokens
        self._t_ref, self._r_ref = ctypes.byref(self._t), ctypes.byref(self._r)
        self._d = _Dense()
        self._index = self._device.index

    # -- plumbing ------------------------------------------------------------
    def _check(self, st):
        if st != OK:
            msg = self._lib.adapm_last_error(self._h)
            raise AdaPMError(st, msg.decode() if msg else "")

    def close(self):
        if getattr(self, "_h", None):
            self._lib.adapm_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _new_rows(self, n, like):
        torch = _torch()
        if isinstance(like, torch.Tensor) and like.is_cuda:
            return torch.empty((n, self.D), dtype=torch.float32, device=like.device)
        if isinstance(like, np.ndarray):
            return np.empty((n, self.D), dtype=np.float32)
        dev = like.device if like is not None and hasattr(like, "device") else torch.device("cuda")
        pin = dev.type == "cpu"
        return torch.empty((n, self.D), dtype=torch.float32, device=dev, pin_memory=pin)

    # -- the ABI -------------------------------------------------------------
    def intent(self, worker, keys, clock_start, clock_end):
        k = _keys(keys)
        self._check(self._lib.adapm_intent(self._h, worker, k.ptr, k.n, int(clock_start), int(clock_end)))

    def advance_clock(self, worker):
        self._check(self._lib.adapm_advance_clock(self._h, worker))

    def pull(self, worker, keys, out=None):
        k = _keys(keys)
        if out is None:
            out = self._new_rows(k.n, keys)
        self._check(self._lib.adapm_pull(self._h, worker, k.ptr, k.n, _out_ptr(out)))
        return out

    def push(self, worker, keys, deltas):
        k = _keys(keys)
        d = _floats(deltas)
        if d.n != k.n * self.D:
            raise ValueError("deltas must hold len(keys) * value_len floats")
        self._check(self._lib.adapm_push(self._h, worker, k.ptr, k.n, d.ptr))

    def push_noalloc(self, worker, keys, deltas):
        """adapm_push_noalloc: device tensors only; no allocation by the library."""
        k = _keys(keys)
        d = _floats(deltas)
        if d.n != k.n * self.D:
            raise ValueError("deltas must hold len(keys) * value_len floats")
        self._check(self._lib.adapm_push_noalloc(self._h, worker, k.ptr, k.n, d.ptr))

    def last_error(self):
        """adapm_last_error: the message of the last error returned on this context ("" if none)."""
        msg = self._lib.adapm_last_error(self._h)
        return msg.decode() if msg else ""

    def debug_fail_next_barrier(self):
        """Test hook: the next push's sort gives up its grid-barrier wait (ADAPM_ETIMEOUT at wait)."""
        self._check(self._lib.adapm_debug_fail_next_barrier(self._h))

    def debug_fail_next_launch(self):
        """Test hook: the next call that launches kernels returns ADAPM_ECUDA as after a launch failure."""
        self._check(self._lib.adapm_debug_fail_next_launch(self._h))

    def sync(self):
        self._check(self._lib.adapm_sync(self._h))

    def wait(self):
        self._check(self._lib.adapm_wait(self._h))

    def _loss_buf(self, loss_out):
        if loss_out is not None:
            return loss_out, _out_ptr(loss_out)
        return None, None

    def mf_step(self, worker, row_keys, col_keys, vals, dim, adagrad, lr, eps=1e-8, loss_out=None):
        r, c, v = _keys(row_keys), _keys(col_keys), _floats(vals)
        lo, lp = self._loss_buf(loss_out)
        self._check(self._lib.adapm_mf_step(self._h, worker, r.ptr, c.ptr, v.ptr, r.n, dim,
                                            int(bool(adagrad)), lr, eps, lp))
        return lo

    def complex_step(self, worker, heads, rels, tails, neg_tails, n_neg, dim, lr, eps=1e-8,
                     loss_out=None):
        h, r, t, ng = _keys(heads), _keys(rels), _keys(tails), _keys(neg_tails)
        lo, lp = self._loss_buf(loss_out)
        self._check(self._lib.adapm_complex_step(self._h, worker, h.ptr, r.ptr, t.ptr, ng.ptr, h.n,
                                                 n_neg, dim, lr, eps, lp))
        return lo

    def sgns_step(self, worker, centres, contexts, negatives, n_ctx, n_neg, vocab, dim, lr,
                  loss_out=None):
        c, x, ng = _keys(centres), _keys(contexts), _keys(negatives)
        lo, lp = self._loss_buf(loss_out)
        self._check(self._lib.adapm_sgns_step(self._h, worker, c.ptr, x.ptr, ng.ptr, c.n, n_ctx,
                                              n_neg, vocab, dim, lr, lp))
        return lo

    # -- token embeddings --------------------------------------------------------
    def _on_stream(self):
        """Temporaries and new outputs are made on, and belong to, the library's stream."""
        torch = _torch()
        if torch._C._cuda_getCurrentRawStream(self._device.index) == self._handle:
            return _NOTHING
        return torch.cuda.stream(self.stream)

    def _describe(self, tokens, pad, rows, what):
        """Fills the descriptors of tokens and of the rows (..., dim) that belong to them; returns the two, or the
        temporaries that stand for them."""
        torch = _torch()
        if not isinstance(tokens, torch.Tensor):
            tokens = torch.from_numpy(np.ascontiguousarray(np.asarray(tokens, dtype=np.int64)))
        wide = tokens.dtype is torch.int64
        if not wide and tokens.dtype is not torch.int32:
            if tokens.is_floating_point() or tokens.is_complex() or tokens.dtype == torch.bool:
                raise ValueError(f"tokens are integers, not {tokens.dtype}")
            with self._on_stream():
                tokens = tokens.to(torch.int64)
            wide = True
        shape, row_shape = tokens.shape, rows.shape
        if not row_shape or row_shape[:-1] != shape:
            raise ValueError(f"{what} must have shape {(*shape, 'dim')}, not {tuple(row_shape)}")
        steps = rows.stride()
        if steps[-1] != 1 and row_shape[-1] > 1:
            if what == "out":
                raise ValueError("elements of a row of out must follow each other")
            with self._on_stream():
                rows = rows.contiguous()
            steps = rows.stride()
        t, r = self._t, self._r
        if len(shape) == 2:
            t.outer, t.inner = shape
            t.outer_stride, t.inner_stride = tokens.stride()
            r.outer_stride, r.inner_stride, _ = steps
        else:
            got = _two_levels(shape, tokens.stride(), steps[:-1])
            if got is None:
                with self._on_stream():
                    tokens = tokens.contiguous()
                got = _two_levels(shape, tokens.stride(), steps[:-1])
            if got is None:
                if what == "out":
                    raise ValueError("out's rows are not reached by an outer and an inner stride")
                with self._on_stream():
                    rows = rows.contiguous()
                got = _two_levels(shape, tokens.stride(), rows.stride()[:-1])
            t.outer, t.inner, (t.outer_stride, t.inner_stride), (r.outer_stride, r.inner_stride) = got
        t.ids, t.id_bits = tokens.data_ptr(), 64 if wide else 32
        if pad is None or not -2 ** 63 <= pad < 2 ** 63:   # (no id equals a larger one; a field would be cut)
            t.has_pad = 0
        else:
            t.has_pad, t.pad = 1, pad
        r.data, r.type = rows.data_ptr(), _type_of(rows.dtype)
        return tokens, rows

    def embed(self, worker, tokens, dim=None, scale=1.0, pad=None, out=None, dtype=None):
        """scale * the first dim floats of the worker's value of every token, as (*tokens.shape, dim) in dtype
        (float32 unless given, or out's).  Tokens: int32 or int64, any shape, strided or not; pad: the token whose
        rows are zeros."""
        torch = _torch()
        if out is None:
            shape = tokens.shape if hasattr(tokens, "shape") else np.shape(tokens)
            on_gpu = isinstance(tokens, torch.Tensor) and tokens.is_cuda
            with self._on_stream():
                out = torch.empty((*shape, self.D if dim is None else dim), dtype=dtype or torch.float32,
                                  device=self._device if on_gpu else "cpu", pin_memory=not on_gpu)
        elif (dim is not None and out.shape[-1] != dim) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out has another dim or dtype")
        keep = self._describe(tokens, pad, out, "out")   # (until the call has taken its arguments)
        self._check(self._lib.adapm_embed(self._h, worker, self._t_ref, out.shape[-1], scale, self._r_ref))
        del keep
        return out

    def embed_grad(self, worker, tokens, grad, scale=1.0, pad=None, out=None):
        """RowGrads of the distinct tokens: scale times the sum of the rows of grad (*tokens.shape, dim) that belong
        to each.  out: RowGrads with room for tokens.numel() keys and rows, of which the result is the front."""
        torch = _torch()
        tokens, grad = self._describe(tokens, pad, grad, "grad")
        n, dim = tokens.numel(), grad.shape[-1]
        if out is None:
            where = {"device": self._device} if grad.is_cuda else {"device": "cpu", "pin_memory": True}
            with self._on_stream():
                out = RowGrads(torch.empty(n, dtype=torch.int32, **where), torch.empty((n, dim), **where),
                               torch.empty(1, dtype=torch.int32, **where))
        elif (out.keys.numel() < n or out.rows.numel() < n * dim or out.count.numel() < 1
              or out.keys.dtype != torch.int32 or out.rows.dtype != torch.float32 or out.count.dtype != torch.int32
              or (n > 0 and out.rows.shape[-1] != dim)):
            raise ValueError("out needs int32 keys, float32 rows of dim elements for every token, and an int32 count")
        self._check(self._lib.adapm_embed_grad(self._h, worker, self._t_ref, dim, scale, self._r_ref, _out_ptr(out.keys),
                                               _out_ptr(out.rows), _out_ptr(out.count)))
        if out.keys.numel() != n or out.rows.numel() != n * dim:   # (what lies behind is another batch's)
            out = RowGrads(out.keys.view(-1)[:n], out.rows.view(-1)[:n * dim].view(n, dim), out.count)
        return out

    def grad_norm(self, grads, scale=1.0, out=None):
        """|scale| times the Euclidean norm over all elements of grads (a GradList, or what makes one), as a float32
        scalar on the GPU, or into out (a float32 scalar, on the host too)."""
        g, torch = _grad_list(grads), _torch()
        if out is None:
            with self._on_stream():
                out = torch.empty((), dtype=torch.float32, device=self._device)
        elif out.dtype is not torch.float32 or out.numel() != 1:
            raise ValueError("out is a float32 scalar")
        self._check(self._lib.adapm_grad_norm(self._h, g.array, g.n, scale, out.data_ptr()))
        return out

    def clip_grads(self, grads, norm, max_norm, scale=1.0, out=None):
        """scale * min(1, max_norm / norm) times every gradient, in place or into out (a GradList, or what makes one).
        norm: a float32 scalar on the GPU, as grad_norm returns it for the same scale."""
        g = _grad_list(grads)
        o = None if out is None else _grad_list(out)
        if o is not None and o.n != g.n:
            raise ValueError("out needs a tensor for every gradient")
        _check_norm(norm)
        self._check(self._lib.adapm_clip_grads(self._h, g.array, None if o is None else o.array, g.n, scale, max_norm,
                                               norm.data_ptr()))

    def push_grads(self, worker, keys, rows, lr, adagrad=False, eps=1e-8, scale=1.0, norm=None,
                   max_norm=float("inf")):
        """Update the worker's values of distinct ascending keys (-1: none) by their gradient rows, as embed_grad
        leaves both: SGD, or AdaGrad on [theta | a] rows, after clipping to max_norm by norm."""
        if _plain_tensor(keys, 1) and _plain_tensor(rows, 2):
            k, r, n, m = keys.data_ptr(), rows.data_ptr(), keys.numel(), rows.numel()   # (0 for none: a null pointer)
        else:
            with self._on_stream():
                keep = _keys(keys), _floats(rows)
            (k, n), (r, m) = ((a.ptr, a.n) for a in keep)
        dim = rows.shape[-1]
        if m != n * dim:
            raise ValueError("rows must hold a row for every key")
        _check_norm(norm)
        self._check(self._lib.adapm_push_grads(self._h, worker, k, r, n, dim, bool(adagrad), lr, eps, scale, max_norm,
                                               None if norm is None else norm.data_ptr()))

    # -- dense layers --------------------------------------------------------------
    def _gpu(self, t, what, dtype=None):
        if t.get_device() != self._index:
            raise ValueError(f"{what} is a tensor on {self._device}, not on {t.device}")
        if dtype is not None and t.dtype is not dtype:
            raise ValueError(f"{what} is {dtype}, not {t.dtype}")
        return t

    def _same_rows(self, x, *others):
        """_dense_rows where all are of one shape without gaps on the GPU, None where that takes a closer look."""
        shape, index = x.shape, self._index
        if not shape or x.get_device() != index or not x.is_contiguous():
            return None
        dim = shape[-1]
        d, n = self._d, x.numel()
        s = d.shape
        s.outer, s.inner, s.dim = 1, n // dim if dim else 0, dim
        r = d.rows[0]
        r.data, r.type, r.outer_stride, r.inner_stride = x.data_ptr(), _float_types.get(x.dtype, -1), 0, dim
        for r, t in zip(d.other_rows, others):
            if t.shape != shape or t.get_device() != index or not t.is_contiguous():
                return None
            r.data, r.type, r.outer_stride, r.inner_stride = t.data_ptr(), _float_types.get(t.dtype, -1), 0, dim
        return dim

    def _dense_rows(self, named):
        """Fills the shape and a descriptor of rows for each (tensor, name, written): all (..., dim), of one shape.
        Inputs that no outer and inner stride reach are copied; returns the tensors."""
        first = named[0][0]
        shape, flat = first.shape, True
        if not shape:
            raise ValueError(f"{named[0][1]} needs a dimension")
        tensors = []
        for t, what, written in named:
            self._gpu(t, what)
            if t.shape != shape:
                raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
            if shape[-1] > 1 and t.stride(-1) != 1 and t.numel() > 0:
                if written:
                    raise ValueError(f"elements of a row of {what} must follow each other")
                with self._on_stream():
                    t = t.contiguous()
            flat = flat and t.is_contiguous()
            tensors.append(t)
        d, dim = self._d, shape[-1]
        d.shape.dim = dim
        if flat:
            d.shape.outer, d.shape.inner = 1, (first.numel() // dim if dim else 0)
            steps = [(0, dim)] * len(tensors)
        else:
            got = _two_levels(shape[:-1], *(t.stride()[:-1] for t in tensors))
            if got is None:   # (outputs stay as they are)
                with self._on_stream():
                    tensors = [t if w else t.contiguous() for t, (_, _, w) in zip(tensors, named)]
                got = _two_levels(shape[:-1], *(t.stride()[:-1] for t in tensors))
            if got is None:
                raise ValueError("rows of the output are not reached by an outer and an inner stride")
            d.shape.outer, d.shape.inner, *steps = got
        for r, t, (outer, inner) in zip(d.rows, tensors, steps):
            r.data, r.type, r.outer_stride, r.inner_stride = t.data_ptr(), _type_of(t.dtype), outer, inner
        return tensors

    def _dense_vector(self, i, t, dim, what):
        """The descriptor of a vector of dim elements (None: none)."""
        if t is None:
            return None
        if t.get_device() != self._index or t.numel() != dim or not t.is_contiguous():
            raise ValueError(f"{what} holds {dim} elements without gaps on {self._device}")
        d = self._d
        v = d.vectors[i]
        v.data, v.type = t.data_ptr(), _float_types.get(t.dtype, -1)   # (the library refuses other types)
        return d.vectors_ref[i]

    def layer_norm(self, x, weight=None, bias=None, eps=1e-5, out=None, dtype=None, stats=None):
        """(x - mean) / sqrt(variance + eps) * weight + bias for every row of x (..., dim), in dtype (x's unless
        given, or out's).  stats (float32, two per row): receives every row's mean and reciprocal deviation, which
        layer_norm_grad needs.  out may be x."""
        torch, d = _torch(), self._d
        if out is None:
            with self._on_stream():
                out = torch.empty(x.shape, dtype=dtype or x.dtype, device=self._device)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError("out has another dtype")
        dim, keep = self._same_rows(x, out), None
        if dim is None:
            keep = self._dense_rows(((x, "x", False), (out, "out", True)))
            dim = x.shape[-1]
        w, b = self._dense_vector(0, weight, dim, "weight"), self._dense_vector(1, bias, dim, "bias")
        if stats is not None:
            self._check_stats(stats, x, dim)
        self._check(self._lib.adapm_layer_norm(self._h, d.shape_ref, d.rows_ref[0], w, b, eps, d.rows_ref[1],
                                               None if stats is None else stats.data_ptr()))
        del keep
        return out

    def _check_stats(self, stats, x, dim):
        if (stats.dtype is not _torch().float32 or stats.get_device() != self._index
                or stats.numel() * dim != 2 * x.numel() or not stats.is_contiguous()):
            raise ValueError(f"stats holds two float32 elements for every row, without gaps, on {self._device}")

    def layer_norm_grad(self, x, grad, stats, weight=None, bias=None, out=None):
        """NormGrads of layer_norm(x, weight, ..., stats=stats) for the gradient of its output: of x in x's dtype, of
        the weight (unless None) in the weight's, and of the bias (bias=True, and by default with a weight) in the
        weight's.  out: NormGrads to fill, None for those not wanted; its x may be x or grad."""
        torch, d = _torch(), self._d
        dim = x.shape[-1] if x.dim() else 0
        if out is None:
            like = torch.float32 if weight is None else weight.dtype
            with self._on_stream():
                dw, db = (torch.empty(dim, dtype=like, device=self._device) if want else None
                          for want in (weight is not None, weight is not None if bias is None else bias))
                out = NormGrads(torch.empty(x.shape, dtype=x.dtype, device=self._device), dw, db)
        dx, keep = out.x, None
        if (self._same_rows(x, grad) if dx is None else self._same_rows(x, grad, dx)) is None:
            rows = [(x, "x", False), (grad, "grad", False)]
            if dx is not None:
                rows.append((dx, "out.x", True))
            keep = self._dense_rows(rows)
        self._check_stats(stats, x, dim)
        w = self._dense_vector(0, weight, dim, "weight")
        dw, db = self._dense_vector(1, out.weight, dim, "out.weight"), self._dense_vector(2, out.bias, dim, "out.bias")
        self._check(self._lib.adapm_layer_norm_grad(self._h, d.shape_ref, d.rows_ref[0], d.rows_ref[1], stats.data_ptr(),
                                                    w, None if dx is None else d.rows_ref[2], dw, db))
        del keep
        return out

    def _matrix(self, i, t, rows, columns, what, written=False):
        """The descriptor of (..., columns), taken as so many rows; an input whose rows are not one step apart is
        copied, and the copy returned beside it (None otherwise)."""
        if t is None:
            return None, None
        shape, copy = t.shape, None
        if not shape or shape[-1] != columns or t.numel() != rows * columns or t.get_device() != self._index:
            raise ValueError(f"{what} must be (..., {columns}) with {rows} rows on {self._device}, not {tuple(shape)} on "
                             f"{t.device}")
        if t.is_contiguous():
            step, one = columns, 1
        else:
            *steps, one = t.stride()
            step = steps[0] if len(steps) == 1 else _one_stride(shape[:-1], steps)
            if step is None:
                if written:
                    raise ValueError(f"rows of {what} are not one step apart")
                with self._on_stream():
                    copy = t = t.contiguous()
                step, one = columns, 1
        d = self._d
        m = d.matrices[i]
        m.data, m.type, m.row_stride, m.col_stride = t.data_ptr(), _float_types.get(t.dtype, -1), step, one
        return d.matrices_ref[i], copy

    def _layer(self, x, weight):
        shape = weight.shape
        if len(shape) != 2 or not x.shape or x.shape[-1] != shape[0]:
            raise ValueError(f"x (..., ins) and weight (ins, outs) do not fit: {tuple(x.shape)}, {tuple(shape)}")
        ins, outs = shape
        n = x.numel() // ins if ins else 0
        layer = self._d.layer
        layer.rows, layer.ins, layer.outs = n, ins, outs
        return n, ins, outs

    def linear(self, x, weight, bias=None, activation=None, residual=None, out=None, dtype=None, pre=None):
        """activation(x weight + bias) + residual for x (..., ins) and weight (ins, outs), both float16 or bfloat16,
        as (..., outs) in dtype (x's unless given, or out's; or float32).  A weight stored by output is passed as its
        .t().  activation: "relu", "gelu", "gelu_tanh", "silu", "tanh" or None.  pre (x's dtype): receives
        x weight + bias, which linear_grad needs with an activation.  out may be the residual."""
        torch, d = _torch(), self._d
        n, ins, outs = self._layer(x, weight)
        if out is None:
            with self._on_stream():
                out = torch.empty((*x.shape[:-1], outs), dtype=dtype or x.dtype, device=self._device)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError("out has another dtype")
        xm, x = self._matrix(0, x, n, ins, "x")          # (copies stay until the call has taken its arguments)
        wm, weight = self._matrix(1, weight, ins, outs, "weight")
        rm, residual = self._matrix(2, residual, n, outs, "residual") if residual is not None else (None, None)
        om, _ = self._matrix(3, out, n, outs, "out", True)
        pm, _ = self._matrix(4, pre, n, outs, "pre", True) if pre is not None else (None, None)
        b = None if bias is None else self._dense_vector(0, bias, outs, "bias")
        self._check(self._lib.adapm_linear(self._h, d.layer_ref, xm, wm, b, _activation(activation), rm, om, pm))
        return out

    def linear_grad(self, x, weight, grad, pre=None, activation=None, bias=None, out=None):
        """LinearGrads of linear(x, weight, ..., pre=pre) for grad, the gradient of its output (that of the residual is
        grad itself): of x and weight in their dtype, the weight's stored as the weight is, and of the bias (bias=True,
        and by default) in the weight's.  out: LinearGrads to fill, None for those not wanted."""
        torch, d = _torch(), self._d
        n, ins, outs = self._layer(x, weight)
        kind = _activation(activation)
        if kind and pre is None:
            raise ValueError("an activation's gradient needs pre, what linear left there")
        if out is None:
            with self._on_stream():
                out = LinearGrads(torch.empty(x.shape, dtype=x.dtype, device=self._device),
                                  torch.empty_like(weight),
                                  torch.empty(outs, dtype=weight.dtype, device=self._device) if bias in (None, True) else None)
        xm, x = self._matrix(0, x, n, ins, "x")          # (copies stay until the call has taken its arguments)
        wm, weight = self._matrix(1, weight, ins, outs, "weight")
        gm, grad = self._matrix(2, grad, n, outs, "grad")
        pm, pre = self._matrix(3, pre if kind else None, n, outs, "pre")
        dx, _ = self._matrix(4, out.x, n, ins, "out.x", True)
        dw, _ = self._matrix(5, out.weight, ins, outs, "out.weight", True)
        db = self._dense_vector(0, out.bias, outs, "out.bias")
        self._check(self._lib.adapm_linear_grad(self._h, d.layer_ref, xm, wm, gm, pm, kind, dx, dw, db))
        return out

    def _ids(self, t, count, what):
        """Signed ids without gaps, and their bits."""
        torch = _torch()
        if t.dtype is not torch.int32 and t.dtype is not torch.int64:
            raise ValueError(f"{what} are int32 or int64, not {t.dtype}")
        if self._gpu(t, what).numel() != count:
            raise ValueError(f"{what}: {count} are needed, not {t.numel()}")
        if not t.is_contiguous():
            with self._on_stream():
                t = t.contiguous()
        return t, 32 if t.dtype is torch.int32 else 64

    def distill(self, logits, ids=None, teacher=None, temperature=1.0, soft=1.0, labels=None, hard=0.0, pad=None,
                scale=1.0, weights=None, grad=None, loss=None):
        """The loss of every row of student logits (..., vocabulary) against a teacher's top logits and labels:
        soft T^2 KL(softmax(teacher / T) || softmax(logits / T)) + hard * cross entropy, as float32 (...).

        ids, teacher    (..., top): the vocabulary ids (int32 or int64; -1: no entry) of the teacher's top logits
        labels, pad     (...): token ids; those equal to pad are none
        grad            a tensor like the logits (or the logits themselves) that receives scale * weights * the
                        gradient of the loss; weights: float32, one factor per row"""
        torch, d = _torch(), self._d
        lead = logits.shape[:-1]
        keep = []
        if (self._same_rows(logits) if grad is None else self._same_rows(logits, grad)) is None:
            rows = [(logits, "logits", False)]
            if grad is not None:
                rows.append((grad, "grad", True))
            keep.append(self._dense_rows(rows))
        n = logits.numel() // max(1, logits.shape[-1])
        t = y = None
        if teacher is not None or ids is not None:
            if teacher is None or ids is None or teacher.shape != ids.shape or teacher.shape[:-1] != lead:
                raise ValueError(f"ids and teacher both have shape {(*lead, 'top')}")
            top = teacher.shape[-1]
            at, d.teacher.id_bits = self._ids(ids, n * top, "ids")
            if not self._gpu(teacher, "teacher").is_contiguous():
                with self._on_stream():
                    teacher = teacher.contiguous()
            e = d.teacher
            e.ids, e.logits, e.top, e.type = at.data_ptr(), teacher.data_ptr(), top, _float_types.get(teacher.dtype, -1)
            keep.append((at, teacher))
            t = d.teacher_ref
        if labels is not None:
            if labels.shape != lead:
                raise ValueError(f"labels must have shape {tuple(lead)}, not {tuple(labels.shape)}")
            at, d.labels.id_bits = self._ids(labels, n, "labels")
            d.labels.ids = at.data_ptr()
            if pad is None or not -2 ** 63 <= pad < 2 ** 63:
                d.labels.has_pad = 0
            else:
                d.labels.has_pad, d.labels.pad = 1, pad
            keep.append(at)
            y = d.labels_ref
        if weights is not None and (self._gpu(weights, "weights", torch.float32).numel() != n
                                    or not weights.is_contiguous()):
            raise ValueError("weights holds one element for every row, without gaps")
        if loss is None:
            with self._on_stream():
                loss = torch.empty(lead, dtype=torch.float32, device=self._device)
        elif self._gpu(loss, "loss", torch.float32).numel() != n or not loss.is_contiguous():
            raise ValueError("loss holds one element for every row, without gaps")
        self._check(self._lib.adapm_distill(self._h, d.shape_ref, d.rows_ref[0], t, temperature, soft, y, hard, scale,
                                            None if weights is None else weights.data_ptr(),
                                            None if grad is None else d.rows_ref[1], loss.data_ptr()))
        del keep
        return loss

    # -- inspection ------------------------------------------------------------
    def clock(self, worker):
        v = ctypes.c_int64()
        self._check(self._lib.adapm_clock(self._h, worker, ctypes.byref(v)))
        return v.value

    def replica_keys(self, worker):
        n = ctypes.c_uint64()
        self._check(self._lib.adapm_replica_keys(self._h, worker, None, 0, ctypes.byref(n)))
        out = np.empty(n.value, dtype=np.uint32)
        if n.value:
            self._check(self._lib.adapm_replica_keys(self._h, worker, out.ctypes.data, n.value,
                                                     ctypes.byref(n)))
        return out.astype(np.int64)

    def replica_rows(self, worker, keys):
        k = _keys(keys)
        val = np.zeros((k.n, self.D), np.float32)
        acc = np.zeros((k.n, self.D), np.float32)
        has = np.zeros(k.n, np.uint8)
        self._check(self._lib.adapm_replica_rows(self._h, worker, k.ptr, k.n, _out_ptr(val),
                                                 _out_ptr(acc), _out_ptr(has)))
        return val, acc, has.astype(bool)

    def refcounts(self, worker, keys):
        k = _keys(keys)
        out = np.zeros(k.n, np.uint32)
        self._check(self._lib.adapm_refcounts(self._h, worker, k.ptr, k.n, _out_ptr(out)))
        return out.astype(np.int64)

    def owners(self, keys):
        """Owner worker of each key, -1 while it is at its home."""
        k = _keys(keys)
        out = np.zeros(k.n, np.int32)
        self._check(self._lib.adapm_owners(self._h, k.ptr, k.n, _out_ptr(out)))
        return out

    def read_main(self, keys):
        k = _keys(keys)
        out = np.zeros((k.n, self.D), np.float32)
        self._check(self._lib.adapm_read_main(self._h, k.ptr, k.n, _out_ptr(out)))
        return out

    def stats(self):
        s = Stats()
        self._check(self._lib.adapm_get_stats(self._h, ctypes.byref(s)))
        return {f: getattr(s, f) for f, _ in Stats._fields_}

    def profile_enable(self, enable=True):
        self._check(self._lib.adapm_profile_enable(self._h, int(bool(enable))))

    def profile_read(self):
        ms = (ctypes.c_double * NUM_OPS)()
        calls = (ctypes.c_uint64 * NUM_OPS)()
        self._check(self._lib.adapm_profile_read(self._h, ms, calls))
        return {OP_NAMES[i]: (ms[i], calls[i]) for i in range(NUM_OPS)}
