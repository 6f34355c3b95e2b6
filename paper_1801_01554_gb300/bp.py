"""ctypes binding of libbp.so (the C ABI declared in include/bp.h and include/bp_experts.h).

Argument marshalling only: every step of the back-propagation path runs in the
library's CUDA kernels.  Functions keep the C names; device buffers are passed
as torch CUDA tensors (or raw integer addresses), host buffers as numpy arrays
or CPU tensors.  A missing library raises at first use: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbp.so")
_lib = None

BP_OK, BP_EINVAL, BP_ENOMEM, BP_ECUDA, BP_ESHAPE, BP_ETIMEOUT, BP_ENONFINITE, BP_ESTATE = range(8)
STATUS_NAMES = ["BP_OK", "BP_EINVAL", "BP_ENOMEM", "BP_ECUDA", "BP_ESHAPE", "BP_ETIMEOUT",
                "BP_ENONFINITE", "BP_ESTATE"]
BP_F32, BP_BF16 = 0, 1
BP_SIGMOID_LOGISTIC, BP_SIGMOID_TABLE = 0, 1
BP_MAX_SIZES = 9
BP_MAX_EXPERTS, BP_MAX_CHOICES, BP_MAX_RANK = 512, 16, 128
BP_GATES_CHOSEN, BP_GATES_ALL = 0, 1

# name -> (restype, argtypes); every symbol declared in include/bp.h and include/bp_experts.h
_VP = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float
_FP = ctypes.POINTER(ctypes.c_float)
SIGNATURES = {
    "bp_create": (_I, [ctypes.POINTER(_I), _I, _F, _F, _I, _I, ctypes.POINTER(_VP)]),
    "bp_destroy": (None, [_VP]),
    "bp_set_hparams": (_I, [_VP, _F, _F, _F]),
    "bp_set_sigmoid": (_I, [_VP, _I]),
    "bp_set_guard": (_I, [_VP, _F]),
    "bp_get_faults": (_I, [_VP, ctypes.POINTER(ctypes.c_int64), _I]),
    "bp_diagnose": (_I, [_VP, _VP, _VP, _I, _FP, ctypes.POINTER(_I), _I, ctypes.POINTER(_I),
                         ctypes.POINTER(_I)]),
    "bp_vote": (_I, [_FP, _I, _FP, ctypes.POINTER(_I)]),
    "bp_num_params": (ctypes.c_int64, [_VP]),
    "bp_set_weights": (_I, [_VP, _FP]),
    "bp_get_weights": (_I, [_VP, _FP]),
    "bp_set_velocity": (_I, [_VP, _FP]),
    "bp_get_velocity": (_I, [_VP, _FP]),
    "bp_get_grads": (_I, [_VP, _FP]),
    "bp_forward": (_I, [_VP, _VP, _I, _VP, _VP]),
    "bp_backward": (_I, [_VP, _VP, _I, _VP, _VP]),
    "bp_update": (_I, [_VP, _VP]),
    "bp_train_batch": (_I, [_VP, _VP, _VP, _I, _VP, _VP]),
    "bp_train_epoch": (_I, [_VP, _VP, _VP, _I, _I, _VP, _VP]),
    "bp_train_epoch_host": (_I, [_VP, _VP, _VP, _I, _I, _FP, _VP]),
    "bp_check": (_I, [_VP, _VP]),
    "bp_train_epoch_noalloc": (_I, [ctypes.POINTER(_I), _I, _F, _F, _F, _VP, _VP, _VP, _VP, _I, _I,
                                    _VP, _VP, _VP]),
    "bp_debug_wait_test": (_I, [_VP, ctypes.c_ulonglong, _I]),
    "bp_last_error": (ctypes.c_char_p, []),
    "bp_router_create": (_I, [_I, _I, _I, _I, _I, ctypes.POINTER(_VP)]),
    "bp_router_destroy": (None, [_VP]),
    "bp_route": (_I, [_VP, _VP, _I, _VP, _VP, _VP, _VP, _VP, _VP]),
    "bp_route_backward": (_I, [_VP, _VP, _I, _VP, _VP, _VP, _VP, _VP]),
    "bp_mix": (_I, [_VP, _I, _VP, _VP, _I, _I, _I, _I, _VP, _VP]),
    "bp_mix_backward": (_I, [_VP, _VP, _I, _VP, _VP, _I, _I, _I, _I, _VP, _VP, _VP]),
    "bp_experts_create": (_I, [_I, _I, _I, _I, _I, ctypes.POINTER(_VP)]),
    "bp_experts_destroy": (None, [_VP]),
    "bp_experts_forward": (_I, [_VP, _VP, _VP, _VP, _I, _VP, _VP, _I, _I, _VP, _VP]),
    "bp_experts_backward": (_I, [_VP, _VP, _VP, _I, _VP, _VP, _I, _VP, _I, _VP, _VP, _VP, _I, _VP]),
    "bp_experts_check": (_I, [_VP, _VP]),
    "bp_adapters_create": (_I, [_I, _I, _I, _I, _I, _I, _I, ctypes.POINTER(_VP)]),
    "bp_adapters_destroy": (None, [_VP]),
    "bp_adapters_forward": (_I, [_VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _I, _I, _I, _VP, _VP, _VP]),
    "bp_adapters_backward": (_I, [_VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _I, _I, _VP, _I, _VP, _VP,
                                  _VP, _I, _VP]),
    "bp_adapters_check": (_I, [_VP, _VP]),
}


class BPError(RuntimeError):
    def __init__(self, status: int, message: str):
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{name}: {message}")
        self.status = status


def lib_path() -> str:
    return _LIB_PATH


def load(path: str | None = None):
    """Load libbp.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    p = path or _LIB_PATH
    if not os.path.exists(p):
        raise ImportError(f"{p} is missing: build it first (python -c 'import __graft_entry__ as g; "
                          "g.build()')")
    lib = ctypes.CDLL(p)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(status: int):
    if status != BP_OK:
        raise BPError(status, load().bp_last_error().decode())


def _dptr(x):
    """Device address of a CUDA tensor (or an int address, or None -> NULL)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not x.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return x.data_ptr()


def _hptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("expected a C-contiguous array")
        return x.ctypes.data
    if x.is_cuda or not x.is_contiguous():
        raise ValueError("expected a contiguous CPU tensor")
    return x.data_ptr()


def _stream(stream):
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _f32_host(arr, n):
    a = np.ascontiguousarray(arr, dtype=np.float32)
    if a.size != n:
        raise ValueError(f"expected {n} parameters, got {a.size}")
    return a


# ------------------------------------------------------------------ C names
def bp_create(sizes, lr, momentum, dtype=BP_F32, max_batch=1024):
    sizes = [int(s) for s in sizes]
    arr = (ctypes.c_int * len(sizes))(*sizes)
    out = ctypes.c_void_p()
    _check(load().bp_create(arr, len(sizes), float(lr), float(momentum), int(dtype),
                            int(max_batch), ctypes.byref(out)))
    return out.value


def bp_destroy(h):
    load().bp_destroy(h)


def bp_set_hparams(h, lr, momentum, grad_scale=1.0):
    _check(load().bp_set_hparams(h, float(lr), float(momentum), float(grad_scale)))


def bp_set_sigmoid(h, mode):
    _check(load().bp_set_sigmoid(h, int(mode)))


def bp_set_guard(h, threshold):
    _check(load().bp_set_guard(h, float(threshold)))


def bp_get_faults(h, reset=False) -> int:
    c = ctypes.c_int64(0)
    _check(load().bp_get_faults(h, ctypes.byref(c), 1 if reset else 0))
    return int(c.value)


def bp_diagnose(h, X, T, batch, capacity=1024):
    """Diagnostic mode: (per-CTA error sums, SM ids, number agreeing with the vote)."""
    sse = np.zeros(capacity, dtype=np.float32)
    sm = np.zeros(capacity, dtype=np.int32)
    n = ctypes.c_int(0)
    agree = ctypes.c_int(0)
    _check(load().bp_diagnose(h, _dptr(X), _dptr(T), int(batch), sse.ctypes.data_as(_FP),
                              sm.ctypes.data_as(ctypes.POINTER(_I)), capacity, ctypes.byref(n),
                              ctypes.byref(agree)))
    return sse[:n.value], sm[:n.value], agree.value


def bp_vote(values):
    """(the value most entries equal bit for bit, how many equal it)."""
    a = np.ascontiguousarray(values, dtype=np.float32)
    mode = ctypes.c_float(0.0)
    agree = ctypes.c_int(0)
    _check(load().bp_vote(a.ctypes.data_as(_FP), int(a.size), ctypes.byref(mode), ctypes.byref(agree)))
    return float(mode.value), agree.value


def bp_num_params(h) -> int:
    return int(load().bp_num_params(h))


def bp_set_weights(h, theta):
    a = _f32_host(theta, bp_num_params(h))
    _check(load().bp_set_weights(h, a.ctypes.data_as(_FP)))


def bp_get_weights(h) -> np.ndarray:
    a = np.empty(bp_num_params(h), dtype=np.float32)
    _check(load().bp_get_weights(h, a.ctypes.data_as(_FP)))
    return a


def bp_set_velocity(h, v):
    a = _f32_host(v, bp_num_params(h))
    _check(load().bp_set_velocity(h, a.ctypes.data_as(_FP)))


def bp_get_velocity(h) -> np.ndarray:
    a = np.empty(bp_num_params(h), dtype=np.float32)
    _check(load().bp_get_velocity(h, a.ctypes.data_as(_FP)))
    return a


def bp_get_grads(h) -> np.ndarray:
    a = np.empty(bp_num_params(h), dtype=np.float32)
    _check(load().bp_get_grads(h, a.ctypes.data_as(_FP)))
    return a


def bp_forward(h, X, batch, Y=None, stream=None):
    _check(load().bp_forward(h, _dptr(X), int(batch), _dptr(Y), _stream(stream)))


def bp_backward(h, T, batch, sse=None, stream=None):
    _check(load().bp_backward(h, _dptr(T), int(batch), _dptr(sse), _stream(stream)))


def bp_update(h, stream=None):
    _check(load().bp_update(h, _stream(stream)))


def bp_train_batch(h, X, T, batch, sse=None, stream=None):
    _check(load().bp_train_batch(h, _dptr(X), _dptr(T), int(batch), _dptr(sse), _stream(stream)))


def bp_train_epoch(h, X, T, n_patterns, minibatch, sse=None, stream=None):
    _check(load().bp_train_epoch(h, _dptr(X), _dptr(T), int(n_patterns), int(minibatch),
                                 _dptr(sse), _stream(stream)))


def bp_train_epoch_host(h, X, T, n_patterns, minibatch, sse=None, stream=None):
    sp = None
    if sse is not None:
        if isinstance(sse, np.ndarray):
            if sse.dtype != np.float32 or not sse.flags["C_CONTIGUOUS"]:
                raise ValueError("sse must be a C-contiguous float32 array")
            sp = sse.ctypes.data_as(_FP)
        else:
            sp = ctypes.cast(_hptr(sse), _FP)
    _check(load().bp_train_epoch_host(h, _hptr(X), _hptr(T), int(n_patterns), int(minibatch), sp,
                                      _stream(stream)))


def bp_check(h, stream=None):
    _check(load().bp_check(h, _stream(stream)))


def bp_train_epoch_noalloc(sizes, lr, momentum, grad_scale, theta, V, X, T, n_patterns, minibatch,
                           sse=None, status=None, stream=None):
    """Training epoch that allocates nothing: every buffer is the caller's
    (float32 CUDA tensors theta and V are updated in place)."""
    sizes = [int(s) for s in sizes]
    arr = (ctypes.c_int * len(sizes))(*sizes)
    _check(load().bp_train_epoch_noalloc(arr, len(sizes), float(lr), float(momentum),
                                         float(grad_scale), _dptr(theta), _dptr(V), _dptr(X),
                                         _dptr(T), int(n_patterns), int(minibatch), _dptr(sse),
                                         _dptr(status), _stream(stream)))


def bp_debug_wait_test(h, wait_ns, unreachable):
    """Checked builds only: grid-barrier and weight-phase wait limit (0 =
    default); unreachable = 1: a first grid barrier that the next training
    launch cannot pass; 2: a first weight-phase chunk copy that never comes."""
    _check(load().bp_debug_wait_test(h, int(wait_ns), int(unreachable)))


def bp_last_error() -> str:
    return load().bp_last_error().decode()


# ------------------------------------------------- C names of include/bp_experts.h
# Each call's tensors are checked for their element type (the kernels read raw memory: an int64
# index or a float64 gate would be read as something else) and for room for what the call reads or
# writes there, where the layer's sizes are known (`room`: values needed, from the classes below).
_dtypes = None


def _torch_types():
    """(float32, bfloat16, int32) of torch, looked up once: bp itself imports without torch."""
    global _dtypes
    if _dtypes is None:
        import torch

        _dtypes = (torch.float32, torch.bfloat16, torch.int32)
    return _dtypes


def _typed(x, kind, what, n=0):
    """Device address of a tensor of element type `kind` (an index of _torch_types) with n values."""
    if x is None or type(x) is int:
        return x
    if x.dtype is not _torch_types()[kind]:
        raise ValueError(f"{what} must be {_torch_types()[kind]} (got {x.dtype})")
    if x.numel() < n:
        raise ValueError(f"{what} holds {x.numel()} values; the call needs {n}")
    if not x.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return x.data_ptr()


def _values(x, dtype, what, n=0):
    return _typed(x, 1 if dtype == BP_BF16 else 0, what, n)


def _ints(x, what, n=0):
    return _typed(x, 2, what, n)


def _floats(x, what, n=0):
    return _typed(x, 0, what, n)


_NO_ROOM = (0,) * 12


def bp_router_create(n_experts, k, dtype=BP_F32, max_patterns=1024, gates=BP_GATES_CHOSEN):
    out = ctypes.c_void_p()
    _check(load().bp_router_create(int(n_experts), int(k), int(dtype), int(max_patterns), int(gates),
                                   ctypes.byref(out)))
    return out.value


def bp_router_destroy(h):
    load().bp_router_destroy(h)


def bp_route(h, logits, n, expert, gate, offsets, source, place, dtype=BP_F32, stream=None, room=_NO_ROOM):
    _check(load().bp_route(h, _values(logits, dtype, "logits", room[0]), n, _ints(expert, "expert", room[1]),
                           _floats(gate, "gate", room[1]), _ints(offsets, "offsets", room[2]),
                           _ints(source, "source", room[1]), _ints(place, "place", room[1]), _stream(stream)))


def bp_route_backward(h, logits, n, expert, gate, dgate, dlogits, dtype=BP_F32, stream=None, room=_NO_ROOM):
    _check(load().bp_route_backward(h, _values(logits, dtype, "logits", room[0]), n,
                                    _ints(expert, "expert", room[1]), _floats(gate, "gate", room[1]),
                                    _floats(dgate, "dgate", room[1]), _values(dlogits, dtype, "dlogits", room[0]),
                                    _stream(stream)))


def bp_mix(H, n_rows, place, gate, n, k, n_out, dtype, Y, stream=None):
    _check(load().bp_mix(_values(H, dtype, "H", n_rows * n_out), n_rows, _ints(place, "place", n * k),
                         _floats(gate, "gate", n * k), n, k, n_out, dtype, _values(Y, dtype, "Y", n * n_out),
                         _stream(stream)))


def bp_mix_backward(D, H, n_rows, place, gate, n, k, n_out, dtype, dH, dgate=None, stream=None):
    _check(load().bp_mix_backward(_values(D, dtype, "D", n * n_out), _values(H, dtype, "H", n_rows * n_out),
                                  n_rows, _ints(place, "place", n * k), _floats(gate, "gate", n * k), n, k,
                                  n_out, dtype, _values(dH, dtype, "dH", n_rows * n_out),
                                  _floats(dgate, "dgate", n * k), _stream(stream)))


def bp_experts_create(n_experts, n_in, n_out, dtype=BP_F32, max_rows=1024):
    out = ctypes.c_void_p()
    _check(load().bp_experts_create(int(n_experts), int(n_in), int(n_out), int(dtype), int(max_rows),
                                    ctypes.byref(out)))
    return out.value


def bp_experts_destroy(h):
    load().bp_experts_destroy(h)


def bp_experts_forward(h, W, b, X, n_x, source, offsets, n_rows, Y, squash=False, dtype=BP_F32, stream=None,
                       room=_NO_ROOM):
    _check(load().bp_experts_forward(h, _values(W, dtype, "W", room[0]), _floats(b, "b", room[1]),
                                     _values(X, dtype, "X", room[2]), n_x, _ints(source, "source", room[3]),
                                     _ints(offsets, "offsets", room[4]), n_rows, 1 if squash else 0,
                                     _values(Y, dtype, "Y", room[5]), _stream(stream)))


def bp_experts_backward(h, W, X, n_x, source, offsets, n_rows, D, dX=None, GW=None, Gb=None, squash=False,
                        accumulate=False, dtype=BP_F32, stream=None, room=_NO_ROOM):
    _check(load().bp_experts_backward(h, _values(W, dtype, "W", room[0]), _values(X, dtype, "X", room[2]), n_x,
                                      _ints(source, "source", room[3]), _ints(offsets, "offsets", room[4]),
                                      n_rows, _values(D, dtype, "D", room[5]), 1 if squash else 0,
                                      _values(dX, dtype, "dX", room[6]), _floats(GW, "GW", room[0]),
                                      _floats(Gb, "Gb", room[1]), 1 if accumulate else 0, _stream(stream)))


def bp_experts_check(h, stream=None):
    _check(load().bp_experts_check(h, _stream(stream)))


def bp_adapters_create(n_adapters, rank, n_in, n_out, dtype=BP_F32, max_rows=1024, max_requests=64):
    out = ctypes.c_void_p()
    _check(load().bp_adapters_create(int(n_adapters), int(rank), int(n_in), int(n_out), int(dtype),
                                     int(max_rows), int(max_requests), ctypes.byref(out)))
    return out.value


def bp_adapters_destroy(h):
    load().bp_adapters_destroy(h)


def bp_adapters_forward(h, W, b, A, B, scale, X, offsets, adapter, n_requests, n_rows, U, Y, squash=False,
                        dtype=BP_F32, stream=None, room=_NO_ROOM):
    _check(load().bp_adapters_forward(h, _values(W, dtype, "W", room[0]), _floats(b, "b", room[1]),
                                      _values(A, dtype, "A", room[2]), _values(B, dtype, "B", room[3]),
                                      _floats(scale, "scale", room[4]), _values(X, dtype, "X", room[5]),
                                      _ints(offsets, "offsets", room[6]), _ints(adapter, "adapter", room[7]),
                                      n_requests, n_rows, 1 if squash else 0, _floats(U, "U", room[8]),
                                      _values(Y, dtype, "Y", room[9]), _stream(stream)))


def bp_adapters_backward(h, W, A, B, scale, X, U, offsets, adapter, n_requests, n_rows, D, dX=None, GA=None,
                         GB=None, squash=False, accumulate=False, dtype=BP_F32, stream=None, room=_NO_ROOM):
    _check(load().bp_adapters_backward(h, _values(W, dtype, "W", room[0]), _values(A, dtype, "A", room[2]),
                                       _values(B, dtype, "B", room[3]), _floats(scale, "scale", room[4]),
                                       _values(X, dtype, "X", room[5]), _floats(U, "U", room[8]),
                                       _ints(offsets, "offsets", room[6]), _ints(adapter, "adapter", room[7]),
                                       n_requests, n_rows, _values(D, dtype, "D", room[9]), 1 if squash else 0,
                                       _values(dX, dtype, "dX", room[5]), _floats(GA, "GA", room[2]),
                                       _floats(GB, "GB", room[3]), 1 if accumulate else 0, _stream(stream)))


def bp_adapters_check(h, stream=None):
    _check(load().bp_adapters_check(h, _stream(stream)))


# ------------------------------------------------------------------ convenience
class _Handle:
    """A handle of the library, freed by close() or at the end of a with block."""

    _free = None

    def close(self):
        if getattr(self, "h", None):
            type(self)._free(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Router(_Handle):
    """Owns one bp_router handle; methods forward to bp_route and bp_route_backward."""

    _free = staticmethod(bp_router_destroy)

    def __init__(self, n_experts, k, dtype=BP_F32, max_patterns=1024, gates=BP_GATES_CHOSEN):
        self.n_experts, self.k, self.dtype = int(n_experts), int(k), dtype
        self.h = bp_router_create(n_experts, k, dtype, max_patterns, gates)

    def forward(self, logits, n, expert, gate, offsets, source, place, stream=None):
        bp_route(self.h, logits, n, expert, gate, offsets, source, place, self.dtype, stream,
                 (n * self.n_experts, n * self.k, self.n_experts + 1))

    def backward(self, logits, n, expert, gate, dgate, dlogits, stream=None):
        bp_route_backward(self.h, logits, n, expert, gate, dgate, dlogits, self.dtype, stream,
                          (n * self.n_experts, n * self.k))


class Experts(_Handle):
    """Owns one bp_experts handle; methods forward to the C names above."""

    _free = staticmethod(bp_experts_destroy)

    def __init__(self, n_experts, n_in, n_out, dtype=BP_F32, max_rows=1024):
        self.n_experts, self.n_in, self.n_out, self.dtype = int(n_experts), int(n_in), int(n_out), dtype
        self.h = bp_experts_create(n_experts, n_in, n_out, dtype, max_rows)

    def _room(self, n_x, n_rows):
        E, i, o = self.n_experts, self.n_in, self.n_out
        return E * o * i, E * o, n_x * i, n_rows, E + 1, n_rows * o, n_rows * i

    def forward(self, W, b, X, n_x, source, offsets, n_rows, Y, squash=False, stream=None):
        bp_experts_forward(self.h, W, b, X, n_x, source, offsets, n_rows, Y, squash, self.dtype, stream,
                           self._room(n_x, n_rows))

    def backward(self, W, X, n_x, source, offsets, n_rows, D, dX=None, GW=None, Gb=None, squash=False,
                 accumulate=False, stream=None):
        bp_experts_backward(self.h, W, X, n_x, source, offsets, n_rows, D, dX, GW, Gb, squash, accumulate,
                            self.dtype, stream, self._room(n_x, n_rows))

    def check(self, stream=None):
        bp_experts_check(self.h, stream)


class Adapters(_Handle):
    """Owns one bp_adapters handle; methods forward to the C names above."""

    _free = staticmethod(bp_adapters_destroy)

    def __init__(self, n_adapters, rank, n_in, n_out, dtype=BP_F32, max_rows=1024, max_requests=64):
        self.n_adapters, self.rank, self.dtype = int(n_adapters), int(rank), dtype
        self.n_in, self.n_out = int(n_in), int(n_out)
        self.h = bp_adapters_create(n_adapters, rank, n_in, n_out, dtype, max_rows, max_requests)

    def _room(self, n_requests, n_rows):
        a, r, i, o = self.n_adapters, self.rank, self.n_in, self.n_out
        return (o * i, o, a * r * i, a * r * o, a, n_rows * i, n_requests + 1 if n_requests > 0 else 0,
                n_requests, n_rows * r, n_rows * o)

    def forward(self, W, b, A, B, scale, X, offsets, adapter, n_requests, n_rows, U, Y, squash=False,
                stream=None):
        bp_adapters_forward(self.h, W, b, A, B, scale, X, offsets, adapter, n_requests, n_rows, U, Y, squash,
                            self.dtype, stream, self._room(n_requests, n_rows))

    def backward(self, W, A, B, scale, X, U, offsets, adapter, n_requests, n_rows, D, dX=None, GA=None,
                 GB=None, squash=False, accumulate=False, stream=None):
        bp_adapters_backward(self.h, W, A, B, scale, X, U, offsets, adapter, n_requests, n_rows, D, dX, GA, GB,
                             squash, accumulate, self.dtype, stream, self._room(n_requests, n_rows))

    def check(self, stream=None):
        bp_adapters_check(self.h, stream)


class Net:
    """Owns one bp_net handle; methods forward to the C names above."""

    def __init__(self, sizes, lr, momentum, dtype=BP_F32, max_batch=1024, grad_scale=1.0):
        self.sizes = tuple(int(s) for s in sizes)
        self.dtype = dtype
        self.h = bp_create(self.sizes, lr, momentum, dtype, max_batch)
        if grad_scale != 1.0:
            bp_set_hparams(self.h, lr, momentum, grad_scale)

    def close(self):
        if self.h:
            bp_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def num_params(self):
        return bp_num_params(self.h)

    def set_hparams(self, lr, momentum, grad_scale=1.0):
        bp_set_hparams(self.h, lr, momentum, grad_scale)

    def set_sigmoid(self, mode):
        bp_set_sigmoid(self.h, mode)

    def set_guard(self, threshold):
        bp_set_guard(self.h, threshold)

    def get_faults(self, reset=False):
        return bp_get_faults(self.h, reset)

    def diagnose(self, X, T, batch):
        return bp_diagnose(self.h, X, T, batch)

    def set_weights(self, theta):
        bp_set_weights(self.h, theta)

    def get_weights(self):
        return bp_get_weights(self.h)

    def set_velocity(self, v):
        bp_set_velocity(self.h, v)

    def get_velocity(self):
        return bp_get_velocity(self.h)

    def get_grads(self):
        return bp_get_grads(self.h)

    def forward(self, X, batch, Y=None, stream=None):
        bp_forward(self.h, X, batch, Y, stream)

    def backward(self, T, batch, sse=None, stream=None):
        bp_backward(self.h, T, batch, sse, stream)

    def update(self, stream=None):
        bp_update(self.h, stream)

    def train_batch(self, X, T, batch, sse=None, stream=None):
        bp_train_batch(self.h, X, T, batch, sse, stream)

    def train_epoch(self, X, T, n_patterns, minibatch, sse=None, stream=None):
        bp_train_epoch(self.h, X, T, n_patterns, minibatch, sse, stream)

    def train_epoch_host(self, X, T, n_patterns, minibatch, sse=None, stream=None):
        bp_train_epoch_host(self.h, X, T, n_patterns, minibatch, sse, stream)

    def check(self, stream=None):
        bp_check(self.h, stream)


def connections(sizes) -> int:
    """Connections counted as the paper counts them, bias connections included."""
    return sum((sizes[l - 1] + 1) * sizes[l] for l in range(1, len(sizes)))
