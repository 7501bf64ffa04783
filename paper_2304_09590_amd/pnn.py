"""Python binding of libpnn.so (the C ABI declared in include/pnn.h).

Argument marshalling only: every step of training, merging and inference runs in the
library's HIP kernels.  Device tensors come from PyTorch (memory and streams only).  There
is no fallback: if the compiled library is missing, importing the binding raises.

Every call that takes tensors takes `stream`: None for the current one; a torch.cuda.Stream, on which the
tensors are then recorded, so that their memory is not given to others before the call's work has ended;
or a raw handle, whose caller keeps the tensors until then.  New results belong to that stream.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpnn.so")

PNN_OK, PNN_EINVAL, PNN_ESHAPE, PNN_ENOMEM, PNN_EHIP, PNN_ESTATE = 0, -1, -2, -3, -4, -5
SIGMOID, TANH, RELU, LEAKY_RELU, SOFTMAX = 0, 1, 2, 3, 4
LOSS_MSE, LOSS_XENT = 0, 1
FP32, BF16_MIXED = 0, 1

STATUS_NAMES = {0: "PNN_OK", -1: "PNN_EINVAL", -2: "PNN_ESHAPE", -3: "PNN_ENOMEM", -4: "PNN_EHIP", -5: "PNN_ESTATE"}


class PnnConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32),
        ("sizes", ctypes.c_int32 * 9),
        ("act", ctypes.c_int32 * 8),
        ("loss", ctypes.c_int32),
        ("precision", ctypes.c_int32),
        ("replicas", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("lr", ctypes.c_float),
    ]


class PnnGroups(ctypes.Structure):
    _fields_ = [("plan", ctypes.c_void_p), ("n", ctypes.c_int64), ("per_row", ctypes.c_int32),
                ("networks", ctypes.c_int32)]


class PnnGroupLayer(ctypes.Structure):
    _fields_ = [("inputs", ctypes.c_int32), ("outputs", ctypes.c_int32), ("type", ctypes.c_int32),
                ("w", ctypes.c_void_p), ("w_net", ctypes.c_int64), ("w_ld", ctypes.c_int64), ("b", ctypes.c_void_p),
                ("b_net", ctypes.c_int64)]


class PnnDistill(ctypes.Structure):
    _fields_ = [("z", ctypes.c_void_p), ("z_ld", ctypes.c_int64), ("type", ctypes.c_int32), ("classes", ctypes.c_int32),
                ("n", ctypes.c_int64), ("idx", ctypes.c_void_p), ("t", ctypes.c_void_p), ("top", ctypes.c_int32),
                ("y", ctypes.c_void_p), ("temperature", ctypes.c_float), ("alpha", ctypes.c_float)]


class PnnError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Load libpnn.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2304_09590_amd/build.py "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER
        i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
        cfg = P(PnnConfig)
        L.pnn_config_check.argtypes = [cfg]
        L.pnn_config_check.restype = i32
        L.pnn_param_count.argtypes = [cfg]
        L.pnn_param_count.restype = i64
        L.pnn_shard.argtypes = [i64, i32, i32, P(i64), P(i64)]
        L.pnn_shard.restype = i32
        L.pnn_init.argtypes = [cfg, P(ctypes.c_float), vp, P(vp)]
        L.pnn_init.restype = i32
        L.pnn_train_epoch.argtypes = [vp, vp, vp, i64, vp]
        L.pnn_train_epoch.restype = i32
        L.pnn_merge.argtypes = [vp, i32, vp]
        L.pnn_merge.restype = i32
        L.pnn_infer.argtypes = [vp, i32, vp, i64, vp, vp, P(i64), vp, vp]
        L.pnn_infer.restype = i32
        L.pnn_eval.argtypes = [vp, i32, vp, vp, i64, P(i64), P(ctypes.c_double), vp]
        L.pnn_eval_noalloc.argtypes = [vp, i32, vp, vp, i64, P(i64), P(ctypes.c_double), vp]
        L.pnn_eval_noalloc.restype = i32
        L.pnn_merge_weighted.argtypes = [vp, P(ctypes.c_double), i32, vp]
        L.pnn_train_epoch_order.argtypes = [vp, vp, vp, i64, vp, vp]
        L.pnn_train_epoch_order.restype = i32
        L.pnn_merge_weighted.restype = i32
        L.pnn_eval.restype = i32
        L.pnn_get_params.argtypes = [vp, i32, P(ctypes.c_float)]
        L.pnn_get_params.restype = i32
        L.pnn_set_params.argtypes = [vp, i32, P(ctypes.c_float)]
        L.pnn_set_params.restype = i32
        L.pnn_last_error.argtypes = [vp]
        L.pnn_last_error.restype = ctypes.c_char_p
        L.pnn_plan.argtypes = [vp]
        L.pnn_plan.restype = ctypes.c_char_p
        L.pnn_profile.argtypes = [vp, i32]
        L.pnn_profile.restype = i32
        L.pnn_profile_read.argtypes = [vp, P(ctypes.c_char_p), P(ctypes.c_double), P(i64), i32]
        L.pnn_profile_read.restype = i32
        L.pnn_destroy.argtypes = [vp]
        L.pnn_destroy.restype = None
        groups, layer = P(PnnGroups), P(PnnGroupLayer)
        L.pnn_group_bytes.argtypes = [i64, i32, i32, P(i64)]
        L.pnn_group_rows.argtypes = [vp, i64, i32, i32, vp, i64, vp]
        L.pnn_grouped_forward.argtypes = [groups, layer, vp, i64, i32, vp, i64, i32, vp]
        L.pnn_grouped_workspace.argtypes = [groups, layer, P(i64), P(i64)]
        L.pnn_grouped_backward_input.argtypes = [groups, layer, vp, i64, vp, i64, i32, vp, i64, i32, vp, i64, vp]
        L.pnn_grouped_backward_weights.argtypes = [groups, layer, vp, i64, vp, i64, vp, i64, i64, vp, i64, vp, i64, vp]
        for name in ("pnn_group_bytes", "pnn_group_rows", "pnn_grouped_forward", "pnn_grouped_workspace",
                     "pnn_grouped_backward_input", "pnn_grouped_backward_weights"):
            getattr(L, name).restype = i32
        distill = P(PnnDistill)
        L.pnn_distill_bytes.argtypes = [i64, i32, P(i64)]
        L.pnn_distill_loss.argtypes = [distill, vp, vp, i64, vp]
        L.pnn_distill_grad.argtypes = [distill, vp, vp, i64, vp, i64, vp]
        for name in ("pnn_distill_bytes", "pnn_distill_loss", "pnn_distill_grad"):
            getattr(L, name).restype = i32
        L.pnn_infer_routed.argtypes = [vp, vp, i64, vp, i32, vp, vp, vp, vp]
        L.pnn_infer_routed.restype = i32
        L.pnn_train_routed.argtypes = [vp, vp, i64, vp, i32, vp, vp, i32, vp, ctypes.c_float, ctypes.c_float, vp, vp]
        L.pnn_train_routed.restype = i32
        _lib = L
    return _lib


def make_config(sizes: Sequence[int], acts: Sequence[int], loss: int, precision: int = FP32, replicas: int = 1,
                batch: int = 1, lr: float = 0.1) -> PnnConfig:
    c = PnnConfig()
    c.n_layers = len(sizes) - 1
    for i, s in enumerate(sizes):
        c.sizes[i] = int(s)
    for i, a in enumerate(acts):
        c.act[i] = int(a)
    c.loss, c.precision, c.replicas, c.batch = int(loss), int(precision), int(replicas), int(batch)
    c.lr = float(lr)
    return c


def config_from_workload(w, **over) -> PnnConfig:
    kw = dict(sizes=w.sizes, acts=w.acts, loss=w.loss, precision=w.precision, replicas=w.replicas, batch=w.batch,
              lr=w.lr)
    kw.update(over)
    return make_config(**kw)


def param_count(cfg: PnnConfig) -> int:
    return int(lib().pnn_param_count(ctypes.byref(cfg)))


def config_check(cfg: PnnConfig) -> int:
    return int(lib().pnn_config_check(ctypes.byref(cfg)))


def shard(n: int, k_total: int, k: int) -> Tuple[int, int]:
    s, ln = ctypes.c_int64(), ctypes.c_int64()
    st = lib().pnn_shard(n, k_total, k, ctypes.byref(s), ctypes.byref(ln))
    if st != PNN_OK:
        raise PnnError(st, "pnn_shard")
    return s.value, ln.value


_torch = None


def _t():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _stream_handle(stream, *tensors) -> Optional[int]:
    """The stream's handle; the tensors are recorded on a torch.cuda.Stream."""
    if stream is None:
        return _t().cuda.current_stream().cuda_stream
    _record(stream, tensors)
    return getattr(stream, "cuda_stream", stream)


def _record(stream, tensors) -> None:
    """Memory of tensors that work on a torch.cuda.Stream uses is not given to others before that work has ended."""
    if isinstance(stream, _t().cuda.Stream):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _dev_ptr(t, dtype_name: str):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous() or str(t.dtype) != dtype_name:
        raise ValueError(f"expected a contiguous CUDA tensor of {dtype_name}, got {t.dtype} on {t.device}")
    return t.data_ptr()


class PNN:
    """One handle of the library: K child networks plus the merged network."""

    def __init__(self, cfg: PnnConfig, theta0: np.ndarray, stream=None):
        self._lib = lib()
        self.cfg = cfg
        self.P = param_count(cfg)
        self.K = int(cfg.replicas)
        if self.P == 0:
            raise PnnError(PNN_EINVAL, "invalid configuration")
        th = np.ascontiguousarray(theta0, dtype=np.float32)
        if th.size != self.P:
            raise ValueError(f"theta0 has {th.size} values, the configuration needs {self.P}")
        h = ctypes.c_void_p()
        st = self._lib.pnn_init(ctypes.byref(cfg), th.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                _stream_handle(stream), ctypes.byref(h))
        if st != PNN_OK:
            raise PnnError(st, self._lib.pnn_last_error(None).decode())
        self.h = h

    def _check(self, st: int, what: str):
        if st != PNN_OK:
            raise PnnError(st, f"{what}: {self._lib.pnn_last_error(self.h).decode()}")

    def train_epoch(self, x, y, stream=None) -> None:
        self._check(self._lib.pnn_train_epoch(self.h, _dev_ptr(x, "torch.float32"), _dev_ptr(y, "torch.int32"),
                                              x.shape[0], _stream_handle(stream, x, y)), "pnn_train_epoch")

    def train_epoch_order(self, x, y, order, stream=None) -> None:
        """One epoch over x[order], y[order] (order: int32 device tensor of N row indices)."""
        self._check(self._lib.pnn_train_epoch_order(self.h, _dev_ptr(x, "torch.float32"), _dev_ptr(y, "torch.int32"),
                                                    x.shape[0], _dev_ptr(order, "torch.int32"),
                                                    _stream_handle(stream, x, y, order)), "pnn_train_epoch_order")

    def merge(self, broadcast: bool = False, stream=None) -> None:
        self._check(self._lib.pnn_merge(self.h, 1 if broadcast else 0, _stream_handle(stream)), "pnn_merge")

    def infer(self, x, pred, which: int = -1, out=None, y=None, count: bool = False, stream=None) -> Optional[int]:
        c = ctypes.c_int64(-1)
        self._check(self._lib.pnn_infer(self.h, which, _dev_ptr(x, "torch.float32"), x.shape[0],
                                        _dev_ptr(pred, "torch.int32"), _dev_ptr(out, "torch.float32"),
                                        ctypes.byref(c) if count else None, _dev_ptr(y, "torch.int32"),
                                        _stream_handle(stream, x, pred, out, y)), "pnn_infer")
        return c.value if count else None

    def merge_weighted(self, weights, broadcast: bool = False, stream=None) -> None:
        w = np.ascontiguousarray(weights, dtype=np.float64)
        if w.shape != (self.K,):
            raise ValueError(f"expected {self.K} weights, got shape {w.shape}")
        self._check(self._lib.pnn_merge_weighted(self.h, w.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                                 1 if broadcast else 0, _stream_handle(stream)), "pnn_merge_weighted")

    def evaluate(self, x, y, which: int = -1, stream=None):
        """(correct count, mean cost) of one network on labelled rows (pnn_eval)."""
        c = ctypes.c_int64(-1)
        cost = ctypes.c_double(float("nan"))
        self._check(self._lib.pnn_eval(self.h, which, _dev_ptr(x, "torch.float32"), _dev_ptr(y, "torch.int32"),
                                       x.shape[0], ctypes.byref(c), ctypes.byref(cost), _stream_handle(stream, x, y)),
                    "pnn_eval")
        return c.value, cost.value

    def evaluate_noalloc(self, x, y, which: int = -1, stream=None):
        """(correct count, mean cost) as evaluate, on the library's fixed workspace
        (pnn_eval_noalloc: no device allocation)."""
        c = ctypes.c_int64(-1)
        cost = ctypes.c_double(float("nan"))
        self._check(self._lib.pnn_eval_noalloc(self.h, which, _dev_ptr(x, "torch.float32"),
                                               _dev_ptr(y, "torch.int32"), x.shape[0], ctypes.byref(c),
                                               ctypes.byref(cost), _stream_handle(stream, x, y)), "pnn_eval_noalloc")
        return c.value, cost.value

    def get_params(self, which: int = -1) -> np.ndarray:
        out = np.empty(self.P, dtype=np.float32)
        self._check(self._lib.pnn_get_params(self.h, which, out.ctypes.data_as(ctypes.POINTER(ctypes.c_float))),
                    "pnn_get_params")
        return out

    def set_params(self, which: int, theta: np.ndarray) -> None:
        th = np.ascontiguousarray(theta, dtype=np.float32)
        assert th.size == self.P
        self._check(self._lib.pnn_set_params(self.h, which, th.ctypes.data_as(ctypes.POINTER(ctypes.c_float))),
                    "pnn_set_params")

    def infer_routed(self, x, ids, pred, weights=None, out=None, stream=None) -> None:
        """Answers of the CNs that each row names (ids int32 [rows, per_row]), combined by weights (None: the mean)."""
        rows, per_row = ids.shape
        self._shapes((x, (rows, self.cfg.sizes[0])), (pred, (rows,)), (weights, (rows, per_row)),
                     (out, (rows, self.cfg.sizes[self.cfg.n_layers])))
        self._check(self._lib.pnn_infer_routed(self.h, _dev_ptr(x, "torch.float32"), rows, _dev_ptr(ids, "torch.int32"), per_row,
                                               _dev_ptr(weights, "torch.float32"), _dev_ptr(pred, "torch.int32"),
                                               _dev_ptr(out, "torch.float32"), _stream_handle(stream, x, ids, weights, pred, out)),
                    "pnn_infer_routed")

    def train_routed(self, x, ids, idx=None, t=None, y=None, temperature: float = 1.0, alpha: float = 0.0, loss=None,
                     stream=None) -> None:
        """One mini-batch step of every CN on the rows that name it, towards a teacher's top logits (idx, t) and labels."""
        rows, per_row = ids.shape
        top = idx.shape[1] if idx is not None else 0
        self._shapes((x, (rows, self.cfg.sizes[0])), (idx, (rows, top)), (t, (rows, top)), (y, (rows,)), (loss, (rows, per_row)))
        self._check(self._lib.pnn_train_routed(self.h, _dev_ptr(x, "torch.float32"), rows, _dev_ptr(ids, "torch.int32"), per_row,
                                               _dev_ptr(idx, "torch.int32"), _dev_ptr(t, "torch.float32"), top,
                                               _dev_ptr(y, "torch.int32"), temperature, alpha, _dev_ptr(loss, "torch.float32"),
                                               _stream_handle(stream, x, ids, idx, t, y, loss)), "pnn_train_routed")

    @staticmethod
    def _shapes(*given) -> None:
        for t, shape in given:
            if t is not None and tuple(t.shape) != shape:
                raise ValueError(f"a tensor of shape {tuple(t.shape)}, expected {shape}")

    def profile(self, enable: bool) -> None:
        self._check(self._lib.pnn_profile(self.h, 1 if enable else 0), "pnn_profile")

    def profile_read(self) -> dict:
        cap = 64
        names = (ctypes.c_char_p * cap)()
        ms = (ctypes.c_double * cap)()
        cnt = (ctypes.c_int64 * cap)()
        n = self._lib.pnn_profile_read(self.h, names, ms, cnt, cap)
        return {names[i].decode(): (ms[i], cnt[i]) for i in range(min(n, cap))}

    @property
    def plan(self) -> str:
        """Training plan chosen at init (see pnn_plan in include/pnn.h)."""
        return self._lib.pnn_plan(self.h).decode()

    def close(self) -> None:
        if getattr(self, "h", None):
            self._lib.pnn_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- calls without a handle: rows that name their network, distillation ----------------------

def _call(what: str, *args) -> None:
    st = getattr(lib(), what)(*args)
    if st != PNN_OK:
        raise PnnError(st, f"{what}: {lib().pnn_last_error(None).decode()}")


def _on(stream, body, first, *others, groups=None):
    """body(stream handle) with the tensors' device current and, for allocations, the stream; the tensors have to
    be on one GPU.  The tensors, and a plan that another stream's memory holds, are recorded on the stream."""
    torch = _t()
    dev = first.get_device()
    if dev < 0:
        raise ValueError(f"expected CUDA tensors, got one on {first.device}")
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors on {first.device} and on {t.device}")
    if groups is not None and groups.plan.get_device() != dev:
        raise ValueError(f"tensors on {first.device} and a plan on {groups.plan.device}")
    if stream is None:
        s = torch._C._cuda_getCurrentRawStream(dev)
        if groups is not None and groups.stream != s:
            _record(torch.cuda.current_stream(dev), (groups.plan,))
        if torch._C._cuda_getDevice() == dev:
            return body(s)
    with torch.cuda.device(dev):
        if stream is None:
            return body(s)
        raw = not isinstance(stream, torch.cuda.Stream)
        if raw:
            stream = torch.cuda.ExternalStream(stream, device=first.device)
        if stream.device != first.device:
            raise ValueError(f"a stream of {stream.device} for tensors on {first.device}")
        if not raw:
            _record(stream, (first, *others, groups.plan if groups is not None else None))
        with torch.cuda.stream(stream):
            return body(stream.cuda_stream)


_TYPES = {}


def _type_of(t) -> int:
    if not _TYPES:
        _TYPES.update({_t().float32: FP32, _t().bfloat16: BF16_MIXED})
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"expected float32 or bfloat16, got {t.dtype}")
    return code


def _empty(like, shape, dtype=None):
    """New memory beside a tensor (new_empty, which costs less than a device and a type to parse)."""
    return like.new_empty(shape) if dtype is None or dtype is like.dtype else like.new_empty(shape, dtype=dtype)


def _rows(t, name: str, shape, dtype):
    """(pointer, distance between rows) of a matrix (or a stack of matrices) whose rows' values are contiguous."""
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} is {t.dtype}, expected {dtype}")
    strides = t.stride()
    width = shape[-1]
    if strides[-1] != 1 and width > 1:
        raise ValueError(f"the values of a row of {name} are not contiguous")
    return t.data_ptr(), (strides[-2] if shape[-2] > 1 else width)


def _values(t, name: str, shape, dtype):
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} is {tuple(t.shape)} of {t.dtype}, expected {tuple(shape)} of {dtype}, contiguous")
    return t.data_ptr()


@functools.lru_cache(maxsize=1024)
def _group_bytes(n: int, per_row: int, networks: int) -> int:
    size = ctypes.c_int64()
    _call("pnn_group_bytes", n, per_row, networks, ctypes.byref(size))
    return size.value


@functools.lru_cache(maxsize=1024)
def _group_workspace(n: int, per_row: int, networks: int, inputs: int, outputs: int, dtype: int) -> Tuple[int, int]:
    one, two = ctypes.c_int64(), ctypes.c_int64()
    groups, layer = PnnGroups(None, n, per_row, networks), PnnGroupLayer(inputs, outputs, dtype, None, 0, 0, None, 0)
    _call("pnn_grouped_workspace", ctypes.byref(groups), ctypes.byref(layer), ctypes.byref(one), ctypes.byref(two))
    return one.value, two.value


class RowGroups:
    """Rows grouped by the networks that they name (pnn_group_rows)."""

    def __init__(self, plan, n: int, per_row: int, networks: int, stream: Optional[int] = None):
        self.plan, self.n, self.per_row, self.networks = plan, n, per_row, networks
        self.stream = stream  # the handle of the stream that the plan's memory belongs to, if known
        self.struct = PnnGroups(plan.data_ptr(), n, per_row, networks)

    @property
    def offsets(self):
        """[networks + 1] int32: network e's pairs are positions offsets[e] to offsets[e + 1]."""
        return self.plan[:self.networks + 1]

    @property
    def pairs(self):
        """[n * per_row] int32 pair numbers by network, the dropped ones last."""
        first = -(-(self.networks + 1) // 4) * 4
        return self.plan[first:first + self.n * self.per_row]


def group_rows(ids, networks: int, stream=None) -> RowGroups:
    """Group rows by network: ids int32 [n] or [n, per_row], an id outside [0, networks) drops the pair."""
    torch = _t()
    shape = ids.shape
    if ids.dtype is not torch.int32 or len(shape) not in (1, 2) or not ids.is_contiguous():
        raise ValueError(f"ids: expected contiguous int32 [n] or [n, per_row], got {tuple(shape)} of {ids.dtype}")
    n, per_row = shape[0], (shape[1] if len(shape) == 2 else 1)

    def body(s):
        size = _group_bytes(n, per_row, networks)
        plan = _empty(ids, size // 4)
        _call("pnn_group_rows", ids.data_ptr(), n, per_row, networks, plan.data_ptr(), size, s)
        return plan, s

    plan, s = _on(stream, body, ids)
    return RowGroups(plan, n, per_row, networks, s)


def _weights(groups: RowGroups, w, b=None) -> PnnGroupLayer:
    shape = w.shape
    if len(shape) != 3 or shape[0] != groups.networks:
        raise ValueError(f"w has shape {tuple(shape)}, expected ({groups.networks}, outputs, inputs)")
    net, ld, one = w.stride()
    if one != 1 and shape[2] > 1:
        raise ValueError("the values of a row of w are not contiguous")
    pb, b_net = _rows(b, "b", shape[:2], _t().float32) if b is not None else (None, 0)
    return PnnGroupLayer(shape[2], shape[1], _type_of(w), w.data_ptr(), net, ld if shape[1] > 1 else shape[2], pb, b_net)


def grouped_forward(groups: RowGroups, x, w, b=None, act: Optional[int] = None, out=None, out_dtype=None, stream=None):
    """y[p] = act(w[e] x[p // per_row] + b[e]) for every pair p of network e; dropped pairs give 0.
    x [n, inputs], w [networks, outputs, inputs] of x's type (float32 or bfloat16), b fp32."""
    layer = _weights(groups, w, b)
    shape = (groups.n * groups.per_row, layer.outputs)

    def body(s):
        y = out if out is not None else _empty(x, shape, out_dtype)
        px, ldx = _rows(x, "x", (groups.n, layer.inputs), w.dtype)
        py, ldy = _rows(y, "out", shape, out_dtype or y.dtype)
        _call("pnn_grouped_forward", ctypes.byref(groups.struct), ctypes.byref(layer), px, ldx, -1 if act is None else act,
              py, ldy, _type_of(y), s)
        return y

    return _on(stream, body, x, w, b, out, groups=groups)


def _workspace(groups: RowGroups, layer: PnnGroupLayer, like, which: int):
    size = _group_workspace(groups.n, groups.per_row, groups.networks, layer.inputs, layer.outputs, layer.type)[which]
    if size == 0:
        return None, None, 0
    ws = _empty(like, size, _t().uint8)
    return ws, ws.data_ptr(), size


def grouped_backward_input(groups: RowGroups, dy, w, a=None, act: Optional[int] = None, out=None, out_dtype=None,
                           stream=None):
    """dx[r] = (sum over row r's pairs of w[e]^T dy[pair]) * act'(a[r]) (the slope from stored activations)."""
    layer = _weights(groups, w)
    shape = (groups.n, layer.inputs)
    if (a is None) != (act is None):
        raise ValueError("a and act go together")

    def body(s):
        dx = out if out is not None else _empty(dy, shape, out_dtype)
        pd, ldd = _rows(dy, "dy", (groups.n * groups.per_row, layer.outputs), w.dtype)
        pa, lda = _rows(a, "a", shape, w.dtype) if a is not None else (None, 0)
        po, ldo = _rows(dx, "out", shape, out_dtype or dx.dtype)
        ws, pw, size = _workspace(groups, layer, dy, 0)
        _call("pnn_grouped_backward_input", ctypes.byref(groups.struct), ctypes.byref(layer), pd, ldd, pa, lda,
              -1 if act is None else act, po, ldo, _type_of(dx), pw, size, s)
        return dx

    return _on(stream, body, dy, w, a, out, groups=groups)


def grouped_backward_weights(groups: RowGroups, dy, x, dw=None, db=None, bias: bool = True, stream=None):
    """(dw, db): dw[e] = sum over network e's pairs of dy[p] x[p // per_row]^T and db[e] = sum of dy[p], fp32;
    zeros for a network without pairs; bias=False leaves db out (None)."""
    torch = _t()
    if dy.dim() != 2 or x.dim() != 2:
        raise ValueError("dy and x are matrices")
    layer = PnnGroupLayer(x.shape[1], dy.shape[1], _type_of(x), None, 0, 0, None, 0)
    shape = (groups.networks, layer.outputs, layer.inputs)

    def body(s):
        w = dw if dw is not None else _empty(x, shape, torch.float32)
        b = db if db is not None or not bias else _empty(x, shape[:2], torch.float32)
        pd, ldd = _rows(dy, "dy", (groups.n * groups.per_row, layer.outputs), x.dtype)
        px, ldx = _rows(x, "x", (groups.n, layer.inputs), x.dtype)
        pw, ldw = _rows(w, "dw", shape, torch.float32)
        pb, netb = _rows(b, "db", shape[:2], torch.float32) if b is not None else (None, 0)
        ws, ps, size = _workspace(groups, layer, x, 1)
        _call("pnn_grouped_backward_weights", ctypes.byref(groups.struct), ctypes.byref(layer), pd, ldd, px, ldx, pw,
              w.stride(0), ldw, pb, netb, ps, size, s)
        return w, b

    return _on(stream, body, x, dy, dw, db, groups=groups)


@functools.lru_cache(maxsize=1024)
def _distill_bytes(n: int, classes: int) -> int:
    size = ctypes.c_int64()
    _call("pnn_distill_bytes", n, classes, ctypes.byref(size))
    return size.value


def _distill(z, idx, t, y, temperature, alpha) -> PnnDistill:
    torch = _t()
    if z.dim() != 2:
        raise ValueError(f"z has shape {tuple(z.shape)}, expected a matrix")
    if (idx is None) != (t is None):
        raise ValueError("idx and t go together")
    n, top = z.shape[0], (idx.shape[-1] if idx is not None else 0)
    pz, ldz = _rows(z, "z", z.shape, z.dtype)
    return PnnDistill(pz, ldz, _type_of(z), z.shape[1], n, None if idx is None else _values(idx, "idx", (n, top), torch.int32),
                      None if idx is None else _values(t, "t", (n, top), z.dtype), top,
                      None if y is None else _values(y, "y", (n,), torch.int32), temperature, alpha)


def distill_loss(z, idx, t, y=None, temperature: float = 1.0, alpha: float = 0.0, stream=None):
    """(loss [n] fp32, stats for distill_grad) of logits z [n, classes] against the teacher's entries: classes
    idx int32 [n, top], logits t [n, top] of z's type; labels y int32 [n] weigh alpha (see pnn_distill in pnn.h)."""
    torch = _t()
    a = _distill(z, idx, t, y, temperature, alpha)

    def body(s):
        size = _distill_bytes(a.n, a.classes)
        loss = _empty(z, a.n, torch.float32)
        stats = _empty(z, size // 4, torch.float32)
        _call("pnn_distill_loss", ctypes.byref(a), loss.data_ptr(), stats.data_ptr(), size, s)
        return loss, stats

    return _on(stream, body, z, idx, t, y)


def distill_grad(z, idx, t, stats, g=None, y=None, temperature: float = 1.0, alpha: float = 0.0, out=None, stream=None):
    """The gradient of z from distill_loss's arguments and statistics; g fp32 [n] is the gradient of each row's
    loss (None: 1).  out may be z."""
    torch = _t()
    a = _distill(z, idx, t, y, temperature, alpha)

    def body(s):
        dz = out if out is not None else _empty(z, z.shape)
        pg = _values(g, "g", (a.n,), torch.float32) if g is not None else None
        ps = _values(stats, "stats", stats.shape, torch.float32)
        po, ldo = _rows(dz, "out", z.shape, z.dtype)
        _call("pnn_distill_grad", ctypes.byref(a), pg, ps, 4 * stats.numel(), po, ldo, s)
        return dz

    return _on(stream, body, z, idx, t, stats, g, y, out)
