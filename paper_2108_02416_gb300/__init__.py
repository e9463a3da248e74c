"""Python binding of libaspis (C ABI in ``include/aspis.h``).

Argument marshalling only: every step of the PS round runs in the library's
CUDA kernels.  PyTorch supplies device memory and streams.  There is no CPU
fallback; if ``libaspis.so`` is missing, importing the binding raises.
Build it with ``python paper_2108_02416_gb300/build.py`` (or
``__graft_entry__.build()``).

The call names mirror the C entry points:

  aspis_assign(K, r) -> Assignment          Algorithm 2
  aspis_check(copies, d, a, file_neq, adj)  per-file agreement + graph G
  aspis_detect(adj, K, det)                 Algorithm 3 (maximum cliques)
  aspis_select(file_neq, det, a, sel)       Algorithm 1 (Case 1 / Case 2)
  aspis_aggregate(copies, d, a, sel, det, out, mode)   coordinate-wise median / mean
  aspis_round(...)                          the four device steps on one stream
  aspis_round_host(...)                     the same from pinned host memory
  aspis_round_static(copies, d, a, det, out, mode)   the round with no device allocation
  aspis_sgd(g, w, v, eta, mu)               the model update with the aggregate (Eq. 1, momentum)
  aspis_detect_wide(adj, K, det)            Algorithm 3 for K <= 128 (graph given directly)
  aspis_round_tolerant(copies, d, a, tau, ...)   the round for copies that are not bit-identical

and those of ``include/aspis_optim.h``, the end of a training step over a
model's many tensors:

  aspis_grad_norm(grads, norm, work)             their global norm
  aspis_clip_grads(grads, max_norm, norm, work)  the norm and clipping by it
  aspis_adamw(params, step, lr, ...)             AdamW with the clipping inside
"""
from __future__ import annotations

import ctypes
import os
import struct

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libaspis.so")

OK, E_INVAL, E_RANGE, E_ALIGN, E_CUDA, E_LIMIT, E_EMPTY, E_NOT_IMPLEMENTED = range(8)
MAX_K, MAX_R, MAX_AGG_FILES = 31, 8, 6144
STATIC_MAX_FILES = 6144
MEDIAN, MEAN = 0, 1


class AspisError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} ({status})")


class _Assignment(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("r", ctypes.c_int32), ("f", ctypes.c_int64),
                ("l", ctypes.c_int64), ("pair_share", ctypes.c_int64),
                ("file_workers", ctypes.POINTER(ctypes.c_uint8)),
                ("worker_files", ctypes.POINTER(ctypes.c_int32)),
                ("slot_of", ctypes.POINTER(ctypes.c_uint8)),
                ("dev_file_workers", ctypes.c_void_p)]


class Detection(ctypes.Structure):
    """Host image of ``aspis_detection`` (36 bytes)."""
    _fields_ = [("clique_mask", ctypes.c_uint32), ("omega", ctypes.c_int32),
                ("n_max_cliques", ctypes.c_uint32), ("success", ctypes.c_int32),
                ("n_sel", ctypes.c_int32), ("status", ctypes.c_int32),
                ("search_nodes", ctypes.c_uint32), ("node_budget", ctypes.c_uint32),
                ("median_exact", ctypes.c_uint32)]

    @classmethod
    def from_tensor(cls, t):
        """Read a device/host uint8 tensor holding an aspis_detection."""
        raw = bytes(t.detach().to("cpu").contiguous().numpy().tobytes())
        return cls.from_buffer_copy(raw)

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


DETECTION_BYTES = ctypes.sizeof(Detection)

WIDE_MAX_K = 128
WIDE_ALL_MAXIMAL = 1


class DetectionWide(ctypes.Structure):
    """Host image of ``aspis_detection_wide`` (64 bytes)."""
    _fields_ = [("clique_words", ctypes.c_uint32 * 4), ("n_max_cliques", ctypes.c_uint64),
                ("n_maximal", ctypes.c_uint64), ("search_nodes", ctypes.c_uint64),
                ("omega", ctypes.c_int32), ("success", ctypes.c_int32),
                ("status", ctypes.c_int32), ("node_budget", ctypes.c_uint32),
                ("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]

    @classmethod
    def from_tensor(cls, t):
        raw = bytes(t.detach().to("cpu").contiguous().numpy().tobytes())
        return cls.from_buffer_copy(raw)

    @property
    def clique_mask(self) -> int:
        """the reported clique as one integer, bit k = worker k"""
        return sum(int(self.clique_words[i]) << (32 * i) for i in range(4))


WIDE_DETECTION_BYTES = ctypes.sizeof(DetectionWide)


def wide_detection_buffer(device, node_budget: int = 0, flags: int = 0):
    """A device uint8 tensor holding an aspis_detection_wide with the inputs set."""
    import torch
    d = DetectionWide()
    d.node_budget = node_budget
    d.flags = flags
    host = torch.frombuffer(bytearray(bytes(d)), dtype=torch.uint8)
    return host.to(device)


NORM_WORKSPACE_BYTES = 40960
F32, BF16, F16 = 0, 1, 2


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("type", ctypes.c_int32), ("out_type", ctypes.c_int32)]


class _Param(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("master", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("exp_avg", ctypes.c_void_p), ("exp_avg_sq", ctypes.c_void_p),
                ("numel", ctypes.c_int64), ("param_type", ctypes.c_int32),
                ("grad_type", ctypes.c_int32), ("weight_decay", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


# the same two, as list constructors write them
_TENSOR, _PARAM = struct.Struct("=QQqii"), struct.Struct("=QQQQQqiifi")
assert _TENSOR.size == ctypes.sizeof(_Tensor) and _PARAM.size == ctypes.sizeof(_Param)


class _AdamwArgs(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("max_norm", ctypes.c_float),
                ("scale", ctypes.c_float), ("skip_nonfinite", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python "
                          "paper_2108_02416_gb300/build.py or __graft_entry__.build()); "
                          "there is no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    P, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    A = ctypes.POINTER(_Assignment)
    sig = {
        "aspis_status_str": ([i32], ctypes.c_char_p),
        "aspis_abi_version": ([], i32),
        "aspis_workspace_bytes": ([A], ctypes.c_size_t),
        "aspis_assign": ([i32, i32, A], i32),
        "aspis_assignment_to_device": ([A], i32),
        "aspis_assignment_free": ([A], None),
        "aspis_check": ([P, i64, i64, A, P, P, P], i32),
        "aspis_graph": ([P, A, P, P], i32),
        "aspis_detect": ([P, i32, P, P], i32),
        "aspis_select": ([P, P, A, P, P], i32),
        "aspis_aggregate": ([P, i64, i64, A, P, P, i32, P, P], i32),
        "aspis_round": ([P, i64, i64, A, P, P, P, P, i32, P, P], i32),
        "aspis_round_host": ([P, P, i64, i64, A, P, P, P, P, i32, P, P, P, P], i32),
        "aspis_round_static": ([P, i64, i64, A, P, i32, P, P], i32),
        "aspis_sgd": ([P, P, P, i64, ctypes.c_float, ctypes.c_float, P], i32),
        "aspis_detect_wide": ([P, i32, P, P], i32),
        "aspis_round_tolerant": ([P, i64, i64, A, ctypes.c_float, P, P, P, P, P, P, i64, i32, P, P],
                                 i32),
    }
    f32 = ctypes.c_float
    sig.update({
        "aspis_tensors_create": ([ctypes.POINTER(_Tensor), i64, ctypes.POINTER(P)], i32),
        "aspis_tensors_destroy": ([P], None),
        "aspis_params_create": ([ctypes.POINTER(_Param), i64, ctypes.POINTER(P)], i32),
        "aspis_params_destroy": ([P], None),
        "aspis_grad_norm": ([P, f32, P, P, P, P], i32),
        "aspis_clip_grads": ([P, f32, f32, P, P, P], i32),
        "aspis_adamw": ([P, ctypes.POINTER(_AdamwArgs), P, P, P], i32),
    })
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    return lib


lib = _load()


def status_str(status: int) -> str:
    return lib.aspis_status_str(int(status)).decode()


def _ok(status: int, where: str):
    if status != OK:
        raise AspisError(status, where)


class Assignment:
    """Owns an ``aspis_assignment`` (host tables + device mirror)."""

    def __init__(self, K: int, r: int, device: bool = True):
        self._a = _Assignment()
        _ok(lib.aspis_assign(K, r, ctypes.byref(self._a)), "aspis_assign")
        if device:
            self.to_device()

    def to_device(self):
        _ok(lib.aspis_assignment_to_device(ctypes.byref(self._a)), "aspis_assignment_to_device")
        return self

    @property
    def ref(self):
        return ctypes.byref(self._a)

    K = property(lambda s: s._a.K)
    r = property(lambda s: s._a.r)
    f = property(lambda s: s._a.f)
    l = property(lambda s: s._a.l)
    pair_share = property(lambda s: s._a.pair_share)

    def file_workers(self):
        import numpy as np
        return np.ctypeslib.as_array(self._a.file_workers, (self.f * self.r,)).reshape(self.f, self.r).copy()

    def worker_files(self):
        import numpy as np
        return np.ctypeslib.as_array(self._a.worker_files, (self.K * self.l,)).reshape(self.K, self.l).copy()

    def slot_of(self):
        import numpy as np
        return np.ctypeslib.as_array(self._a.slot_of, (self.K * self.l,)).reshape(self.K, self.l).copy()

    def close(self):
        if getattr(self, "_a", None) is not None and self._a.K:
            lib.aspis_assignment_free(ctypes.byref(self._a))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def aspis_assign(K: int, r: int, device: bool = True) -> Assignment:
    return Assignment(K, r, device)


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t, dtype=None, name="tensor"):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _ld(copies, a: Assignment):
    if copies.dim() != 3 or copies.shape[0] != a.f or copies.shape[1] != a.r:
        raise ValueError(f"copies must be [f={a.f}, r={a.r}, ld], got {tuple(copies.shape)}")
    return int(copies.shape[2])


def aspis_check(copies, d: int, a: Assignment, file_neq, adj, stream=None):
    import torch
    ld = _ld(copies, a)
    _ok(lib.aspis_check(_dev(copies, torch.float32, "copies"), d, ld, a.ref,
                        _dev(file_neq, torch.int32, "file_neq"), _dev(adj, torch.int32, "adj"),
                        _stream(stream)), "aspis_check")


def aspis_graph(file_neq, a: Assignment, adj, stream=None):
    import torch
    _ok(lib.aspis_graph(_dev(file_neq, torch.int32, "file_neq"), a.ref,
                        _dev(adj, torch.int32, "adj"), _stream(stream)), "aspis_graph")


def aspis_detect(adj, K: int, det, stream=None):
    import torch
    _ok(lib.aspis_detect(_dev(adj, torch.int32, "adj"), K, _dev(det, torch.uint8, "det"),
                         _stream(stream)), "aspis_detect")


def aspis_select(file_neq, det, a: Assignment, sel, stream=None):
    import torch
    _ok(lib.aspis_select(_dev(file_neq, torch.int32, "file_neq"), _dev(det, torch.uint8, "det"),
                         a.ref, _dev(sel, torch.int8, "sel"), _stream(stream)), "aspis_select")


def aspis_aggregate(copies, d: int, a: Assignment, sel, det, out, mode: int = MEDIAN, stream=None):
    import torch
    ld = _ld(copies, a)
    _ok(lib.aspis_aggregate(_dev(copies, torch.float32, "copies"), d, ld, a.ref,
                            _dev(sel, torch.int8, "sel"), _dev(det, torch.uint8, "det"), mode,
                            _dev(out, torch.float32, "out"), _stream(stream)), "aspis_aggregate")


def aspis_round(copies, d: int, a: Assignment, file_neq, adj, det, sel, out, mode: int = MEDIAN,
                stream=None):
    import torch
    ld = _ld(copies, a)
    _ok(lib.aspis_round(_dev(copies, torch.float32, "copies"), d, ld, a.ref,
                        _dev(file_neq, torch.int32, "file_neq"), _dev(adj, torch.int32, "adj"),
                        _dev(det, torch.uint8, "det"), _dev(sel, torch.int8, "sel"), mode,
                        _dev(out, torch.float32, "out"), _stream(stream)), "aspis_round")


def aspis_round_host(host_copies, dev_copies, d: int, a: Assignment, file_neq, adj, det, sel,
                     dev_out, host_out, host_det, mode: int = MEDIAN, stream=None):
    """host_copies / host_out / host_det: CPU tensors (pinned for full speed)."""
    import torch
    ld = _ld(dev_copies, a)
    for t, nm in ((host_copies, "host_copies"), (host_out, "host_out"), (host_det, "host_det")):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{nm} must be a contiguous CPU tensor")
    if host_copies.numel() != dev_copies.numel() or host_copies.dtype != torch.float32:
        raise ValueError("host_copies must match dev_copies (float32)")
    _ok(lib.aspis_round_host(ctypes.c_void_p(host_copies.data_ptr()),
                             _dev(dev_copies, torch.float32, "dev_copies"), d, ld, a.ref,
                             _dev(file_neq, torch.int32, "file_neq"), _dev(adj, torch.int32, "adj"),
                             _dev(det, torch.uint8, "det"), _dev(sel, torch.int8, "sel"), mode,
                             _dev(dev_out, torch.float32, "dev_out"),
                             ctypes.c_void_p(host_out.data_ptr()),
                             ctypes.c_void_p(host_det.data_ptr()), _stream(stream)),
        "aspis_round_host")


def aspis_round_static(copies, d: int, a: Assignment, det, out, mode: int = MEDIAN, stream=None):
    """The round for callers that cannot allocate device memory: the
    intermediates live in the library's fixed device array (see aspis.h);
    ``a`` needs no device mirror.  Calls that may overlap on the GPU race."""
    import torch
    ld = _ld(copies, a)
    _ok(lib.aspis_round_static(_dev(copies, torch.float32, "copies"), d, ld, a.ref,
                               _dev(det, torch.uint8, "det"), mode,
                               _dev(out, torch.float32, "out"), _stream(stream)),
        "aspis_round_static")


def aspis_detect_wide(adj, K: int, det, stream=None):
    """Algorithm 3 for K <= 128 workers: ``adj`` is a device uint32 [K, 4]
    tensor (worker k = bit k % 32 of word k // 32), ``det`` a device uint8
    tensor from :func:`wide_detection_buffer`."""
    import torch
    if adj.numel() < 4 * K:
        raise ValueError("adj must hold K rows of 4 words")
    if adj.dtype not in (torch.int32, getattr(torch, "uint32", torch.int32)):
        raise ValueError(f"adj must hold 32-bit words, got {adj.dtype}")
    _ok(lib.aspis_detect_wide(_dev(adj, None, "adj"), K, _dev(det, torch.uint8, "det"),
                              _stream(stream)),
        "aspis_detect_wide")


def aspis_round_tolerant(copies, d: int, a: Assignment, tau: float, file_neq, adj, det, slot_mask,
                         sel, means, out, mode: int = MEDIAN, stream=None):
    """The round with "close within tau" in place of bitwise equality and the
    kept files' averaged copies aggregated (see aspis.h).  ``means`` is a
    device float32 [f, ldm] tensor with ldm >= d."""
    import torch
    ld = _ld(copies, a)
    if means.dim() != 2 or means.shape[0] != a.f or means.shape[1] < d:
        raise ValueError(f"means must be [f={a.f}, ldm >= d], got {tuple(means.shape)}")
    _ok(lib.aspis_round_tolerant(_dev(copies, torch.float32, "copies"), d, ld, a.ref, float(tau),
                                 _dev(file_neq, torch.int32, "file_neq"), _dev(adj, torch.int32, "adj"),
                                 _dev(det, torch.uint8, "det"), _dev(slot_mask, torch.uint8, "slot_mask"),
                                 _dev(sel, torch.int8, "sel"), _dev(means, torch.float32, "means"),
                                 int(means.shape[1]), mode, _dev(out, torch.float32, "out"),
                                 _stream(stream)),
        "aspis_round_tolerant")


def aspis_sgd(g, w, v, eta: float, mu: float = 0.9, stream=None):
    """w, v <- one SGD step with heavy-ball momentum on the aggregate g
    (in place; see aspis.h).  ``v`` may be None when ``mu == 0``."""
    import torch
    n = g.numel()
    if w.numel() != n or (v is not None and v.numel() != n):
        raise ValueError("g, w and v must have the same number of elements")
    vp = None if v is None else _dev(v, torch.float32, "v")
    _ok(lib.aspis_sgd(_dev(g, torch.float32, "g"), _dev(w, torch.float32, "w"), vp, n,
                      float(eta), float(mu), _stream(stream)),
        "aspis_sgd")


class RoundBuffers:
    """Device buffers of one round for an assignment (allocated by torch)."""

    def __init__(self, a: Assignment, d: int, device="cuda"):
        import torch
        self.file_neq = torch.zeros(a.f, dtype=torch.int32, device=device)
        self.adj = torch.zeros(a.K, dtype=torch.int32, device=device)
        self.det = torch.zeros(DETECTION_BYTES, dtype=torch.uint8, device=device)
        self.sel = torch.zeros(a.f, dtype=torch.int8, device=device)
        self.out = torch.zeros(d, dtype=torch.float32, device=device)

    def detection(self) -> Detection:
        return Detection.from_tensor(self.det)


class TolerantBuffers(RoundBuffers):
    """RoundBuffers plus the slot masks and the [f, round_up(d, 4)] averages
    of the tolerant round."""

    def __init__(self, a: Assignment, d: int, device):
        import torch
        super().__init__(a, d, device)
        self.slot_mask = torch.zeros(a.f, dtype=torch.uint8, device=device)
        self.means = torch.zeros((a.f, (d + 3) // 4 * 4), dtype=torch.float32, device=device)


# ------------------------------------------------ many tensors (aspis_optim.h)


def _types():
    import torch
    return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}, torch.strided


def _gapless(t):
    """True when the tensor's elements fill its range of memory, in any order of dimensions."""
    at = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n > 1):
        if stride != at:
            return False
        at *= size
    return True


class _List:
    """Owns a list handle, and keeps its tensors' memory."""
    _create = _destroy = None

    def _start(self, first):
        import torch
        self._torch = torch
        self._codes, self._strided = _types()
        self._current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self._stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
        self.device = None if first is None else first.device
        self._index = -1 if first is None else first.get_device()
        self._kept = []

    def _take(self, t, name):
        """Checks a tensor, keeps its memory and gives its type's code and whether it is contiguous."""
        if t is None:
            raise ValueError(f"{name}: None is no tensor (leave parameters without a gradient out)")
        if t.layout is not self._strided or t.get_device() < 0:
            raise ValueError(f"{name} must be dense CUDA tensors")
        if t.get_device() != self._index:
            raise ValueError(f"{name} must be on one device: got {t.device} and {self.device}")
        code = self._codes.get(t.dtype)
        if code is None:
            raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
        plain = t.is_contiguous()
        if not plain and not _gapless(t):
            raise ValueError(f"{name} must fill their memory without gaps")
        self._kept.append(t.untyped_storage())
        return code, plain

    def _pair(self, t, plain, other, name):
        """Checks the tensor that goes with t element by element: the same shape, and the same order in memory."""
        code, plain_other = self._take(other, name)
        if t.shape != other.shape:
            raise ValueError(f"{name}: shapes {tuple(t.shape)} and {tuple(other.shape)} differ")
        if not (plain and plain_other) and any(a != b and n > 1 for a, b, n in zip(t.stride(), other.stride(), t.shape)):
            raise ValueError(f"{name}: orders in memory (strides) differ")
        return code

    def _make(self, items, n):
        self.n = n
        self._h = ctypes.c_void_p()
        _ok(getattr(lib, self._create)(items, n, ctypes.byref(self._h)), self._create)

    def __len__(self):
        return self.n

    def close(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            getattr(lib, self._destroy)(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class TensorList(_List):
    """Gradients for :func:`aspis_grad_norm` and :func:`aspis_clip_grads`.

    ``out``: tensors of the same shapes for the clipped values (any of the three
    types), or None to clip in place.  The list holds the tensors' memory as it is
    now: make another when a gradient moves to other memory.  Calls run on the current
    stream of the tensors' device, whichever device is current, or on ``stream``; norm,
    workspace and stream belong to that device.  What other streams still do with
    the tensors has to be waited for by the caller, as with any kernel."""
    _create, _destroy = "aspis_tensors_create", "aspis_tensors_destroy"

    def __init__(self, tensors, out=None):
        tensors = list(tensors)
        outs = [None] * len(tensors) if out is None else list(out)
        if len(outs) != len(tensors):
            raise ValueError(f"{len(tensors)} tensors and {len(outs)} outputs")
        self._start(tensors[0] if tensors else None)
        items, at = (_Tensor * len(tensors))(), 0
        for t, o in zip(tensors, outs):
            code, plain = self._take(t, "tensors")
            out_code = 0 if o is None else self._pair(t, plain, o, "out")
            _TENSOR.pack_into(items, at, t.data_ptr(), 0 if o is None else o.data_ptr(), t.numel(), code, out_code)
            at += _TENSOR.size
        self._make(items, len(tensors))


class ParamList(_List):
    """Parameters with their gradients and moments for :func:`aspis_adamw`.

    ``exp_avg``, ``exp_avg_sq`` and ``masters`` are float32; ``masters`` (of the 16-bit
    parameters, with None in the place of others, or None for none) hold the weights that
    the step is made on.  ``weight_decay``: one value, or one per tensor.  The list
    holds the tensors' memory as it is now."""
    _create, _destroy = "aspis_params_create", "aspis_params_destroy"

    def __init__(self, params, grads, exp_avg, exp_avg_sq, masters=None, weight_decay=0.0):
        params, grads, exp_avg, exp_avg_sq = (list(x) for x in (params, grads, exp_avg, exp_avg_sq))
        n = len(params)
        masters = [None] * n if masters is None else list(masters)
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else list(weight_decay)
        for name, x in (("grads", grads), ("exp_avg", exp_avg), ("exp_avg_sq", exp_avg_sq),
                        ("masters", masters), ("weight_decay", decay)):
            if len(x) != n:
                raise ValueError(f"{n} params and {len(x)} {name}")
        self._start(params[0] if n else None)
        items, at = (_Param * n)(), 0
        for p, g, m, v, w, k in zip(params, grads, exp_avg, exp_avg_sq, masters, decay):
            code, plain = self._take(p, "params")
            grad_code = self._pair(p, plain, g, "grads")
            if (self._pair(p, plain, m, "exp_avg") != F32 or self._pair(p, plain, v, "exp_avg_sq") != F32 or
                    (w is not None and self._pair(p, plain, w, "masters") != F32)):
                raise ValueError("exp_avg, exp_avg_sq and masters must be float32")
            _PARAM.pack_into(items, at, p.data_ptr(), 0 if w is None else w.data_ptr(), g.data_ptr(),
                             m.data_ptr(), v.data_ptr(), p.numel(), code, grad_code, k, 0)
            at += _PARAM.size
        self._make(items, n)


class NormBuffers:
    """Device buffers of a norm: ``norm`` (float32 [1]) and ``work``."""

    def __init__(self, device="cuda"):
        import torch
        self.norm = torch.zeros(1, dtype=torch.float32, device=device)
        self.work = torch.zeros(NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=device)


def _open(x, kind, name, norm):
    """The list's handle (the library cannot tell one kind of list from another), torch, and the device of the
    call: the list's, or of an empty one its buffers'; -1 where there is none."""
    if not isinstance(x, kind):
        raise ValueError(f"{name} must be a {kind.__name__}, got {type(x).__name__}")
    index = x._index
    return x._h, x._torch, index if index >= 0 or norm is None else norm.get_device()


def _buffer(t, dtype, least, index, name):
    """The address of a call's buffer on the call's device, or None."""
    if t is None:
        return None
    if t.get_device() != index or index < 0:
        raise ValueError(f"{name} must be a CUDA tensor on the list's device, got {t.device}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.numel() < least:
        raise ValueError(f"{name} must have {least} elements")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _launch(name, x, index, stream, *args):
    """Calls the library on ``stream`` or the device's current stream, with the device current, as it launches
    on the current one.  (Handles and device numbers alone: a Stream object takes 2 us, a third of a small call.)"""
    if stream is None:
        raw = x._stream_of(index) if index >= 0 else _stream(None)
    else:
        own = getattr(getattr(stream, "device", None), "index", None)
        if index >= 0 and own is not None and own != index:
            raise ValueError(f"stream must be on the list's device {index}, got {own}")
        raw = _stream(stream)
    if index < 0 or index == x._current():
        status = getattr(lib, name)(*args, raw)
    else:
        with x._torch.cuda.device(index):
            status = getattr(lib, name)(*args, raw)
    if status != OK:
        raise AspisError(status, name)


def aspis_grad_norm(grads: TensorList, norm, work, tensor_norms=None, scale: float = 1.0, stream=None):
    """norm <- scale * the global L2 norm of ``grads``; ``tensor_norms`` (float32 [n]):
    every tensor's own."""
    handle, torch, index = _open(grads, TensorList, "grads", norm)
    _launch("aspis_grad_norm", grads, index, stream, handle, scale, _buffer(norm, torch.float32, 1, index, "norm"),
            _buffer(tensor_norms, torch.float32, grads.n, index, "tensor_norms"),
            _buffer(work, torch.uint8, NORM_WORKSPACE_BYTES, index, "work"))


def aspis_clip_grads(grads: TensorList, max_norm: float, norm, work=None, scale: float = 1.0, stream=None):
    """Clips ``grads`` to ``max_norm`` (into the list's outputs, or in place) and writes
    their norm; without ``work`` the norm is given in ``norm``."""
    handle, torch, index = _open(grads, TensorList, "grads", norm)
    _launch("aspis_clip_grads", grads, index, stream, handle, max_norm, scale,
            _buffer(norm, torch.float32, 1, index, "norm"), _buffer(work, torch.uint8, NORM_WORKSPACE_BYTES, index, "work"))


def aspis_adamw(params: ParamList, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
                max_norm=None, norm=None, work=None, scale: float = 1.0, skip_nonfinite: bool = False,
                stream=None):
    """One AdamW step (``step`` counts from 1).  ``max_norm``: clip by the global norm,
    which is written to ``norm``, or given there where ``work`` is None; None: no
    clipping.  ``skip_nonfinite``: change nothing where the norm is not finite."""
    handle, torch, index = _open(params, ParamList, "params", norm)
    args = _AdamwArgs(lr, betas[0], betas[1], eps, step, -1.0 if max_norm is None else max_norm, scale,
                      skip_nonfinite, 0)
    if max_norm is not None and max_norm < 0:
        raise ValueError("max_norm must not be negative")
    _launch("aspis_adamw", params, index, stream, handle, ctypes.byref(args),
            _buffer(norm, torch.float32, 1, index, "norm"), _buffer(work, torch.uint8, NORM_WORKSPACE_BYTES, index, "work"))
