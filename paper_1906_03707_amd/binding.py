"""ctypes front end of libhag: argument marshalling only.

Function names follow include/hag.h.  Host arrays are numpy; device arrays are
torch tensors used purely as device memory (data_ptr) and for the current
stream.  Every step of the aggregation path runs in the library's HIP kernels;
there is no fallback: if libhag.so is missing or fails to load, importing a
symbol from it raises.
"""
from __future__ import annotations

import array
import ctypes
import os
import sys

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("HAG_LIB", os.path.join(_HERE, "libhag.so"))

HAG_SUM, HAG_MEAN, HAG_MAX, HAG_GCN = 0, 1, 2, 3
HAG_F32, HAG_I32, HAG_BF16, HAG_F16, HAG_I64 = 0, 1, 2, 3, 4
HAG_NO_PADDING = -1 << 63
HAG_OK, HAG_EINVAL, HAG_ENOMEM, HAG_EHIP, HAG_ESTATE, HAG_ETIMEOUT = 0, -1, -2, -3, -4, -5
HAG_OPT_ONE_LAUNCH_MAX_ITEMS, HAG_OPT_SPIN_LIMIT, HAG_OPT_TEST_WAIT_UNREACHABLE, HAG_OPT_DETERMINISTIC_MAX_BACKWARD = 1, 2, 3, 4
HAG_OPT_SEQ_ONE_LAUNCH = 6
HAG_OPT_PARTITION_SHIFT = 5
HAG_OPT_LIST_FORMS = 7
HAG_SEARCH_CANONICAL, HAG_SEARCH_DEDUP, HAG_SEARCH_DEVICE = 1, 2, 4
HAG_PHASE_LEVELS, HAG_PHASE_GATHER, HAG_PHASE_FOLD, HAG_PHASE_ALL = 1, 2, 4, 7
OPS = {"sum": HAG_SUM, "mean": HAG_MEAN, "max": HAG_MAX, "gcn": HAG_GCN}

EXPORTS = [
    "hag_search", "hag_search_batched", "hag_from_merges", "hag_prefix", "hag_free", "hag_stats",
    "hag_get_merges", "hag_get_forward", "hag_upload", "hag_workspace_bytes", "hag_forward",
    "hag_backward", "hag_forward_phases", "hag_backward_phases", "hag_naive_forward", "hag_naive_backward",
    "hag_algorithmic_bytes", "hag_last_error", "hag_forward_static_scratch", "hag_probe_rows", "hag_probe_copy", "hag_probe_mfma_f32", "hag_set_option", "hag_check", "hag_seq_search",
    "hag_seq_create", "hag_seq_free", "hag_seq_cells", "hag_seq_ranks", "hag_seq_launches", "hag_seq_get_plan", "hag_seq_set_option", "hag_seq_check", "hag_seq_train_workspace_bytes", "hag_seq_lstm_forward_train", "hag_seq_lstm_backward", "hag_seq_merges", "hag_seq_upload", "hag_seq_workspace_bytes",
    "hag_seq_lstm_forward", "hag_seq_weight_grad_slabs", "hag_route", "hag_naive_route", "hag_forward_workspace_bytes",
    "hag_weight_grad_workspace_bytes", "hag_weight_grad", "hag_narrow_product", "hag_softmax_loss_workspace_bytes", "hag_softmax_loss", "hag_softmax_loss_grad",
    "hag_embedding", "hag_embedding_grad_workspace_bytes", "hag_embedding_grad", "hag_layer_norm", "hag_layer_norm_grad_workspace_bytes", "hag_layer_norm_grad",
    "hag_clip_workspace_bytes", "hag_clip_gradients",
    "hag_rms_norm", "hag_rms_norm_fp8", "hag_rms_norm_grad_workspace_bytes", "hag_rms_norm_grad", "hag_fp8_product", "hag_adamw",
]
ROUTES = ("hag", "lists", "component_hag", "component_lists", "dense", "one_launch", "scatter")   # HAG_ROUTE_*
HAG_STATIC_SCRATCH_BYTES = 64 << 20


class HagError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libhag error {code}: {msg}")
        self.code = code


class hag_adamw_options_t(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_double) for k in ("lr", "beta1", "beta2", "eps", "weight_decay", "max_norm")] + [("step", ctypes.c_int64)]
                + [(k, ctypes.c_void_p) for k in ("lr_device", "step_device", "norm")] + [("seed", ctypes.c_uint32), ("bits", ctypes.c_int32)])


class hag_stats_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int64) for k in (
        "n", "e", "a", "levels", "h", "e_hag", "aggr_naive", "aggr_hag", "xfer_naive", "xfer_hag",
        "max_degree", "max_hag_degree", "stages", "components")]


_lib = None


def lib():
    """Load libhag.so (built by paper_1906_03707_amd.build); fails loudly if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: run `python -m paper_1906_03707_amd.build` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32, u32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32
        L.hag_search.argtypes = [i64, vp, vp, i64, u32, i32, ctypes.POINTER(vp)]
        L.hag_search_batched.argtypes = [i64, vp, vp, i64, vp, ctypes.c_double, u32, i32, ctypes.POINTER(vp)]
        L.hag_from_merges.argtypes = [i64, vp, vp, i64, vp, vp, u32, ctypes.POINTER(vp)]
        L.hag_prefix.argtypes = [vp, i64, ctypes.POINTER(vp)]
        L.hag_free.argtypes = [vp]
        L.hag_free.restype = None
        L.hag_stats.argtypes = [vp, ctypes.POINTER(hag_stats_t)]
        L.hag_get_merges.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
        L.hag_get_forward.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                      ctypes.POINTER(i32), ctypes.POINTER(vp), ctypes.POINTER(vp)]
        L.hag_upload.argtypes = [vp, vp]
        for name in ("hag_workspace_bytes", "hag_forward_workspace_bytes"):
            getattr(L, name).argtypes = [vp, ctypes.c_int, ctypes.c_int, i64]
            getattr(L, name).restype = ctypes.c_size_t
        for name in ("hag_forward", "hag_naive_forward"):
            getattr(L, name).argtypes = [vp, ctypes.c_int, ctypes.c_int, i64, vp, vp, vp, vp, vp]
        for name in ("hag_backward", "hag_naive_backward"):
            getattr(L, name).argtypes = [vp, ctypes.c_int, ctypes.c_int, i64, vp, vp, vp, vp, vp]
        for name in ("hag_forward_phases", "hag_backward_phases"):
            getattr(L, name).argtypes = [vp, ctypes.c_int, ctypes.c_int, i64, vp, vp, vp, vp, vp, u32]
        L.hag_algorithmic_bytes.argtypes = [vp, ctypes.c_int, ctypes.c_int, i64]
        L.hag_algorithmic_bytes.restype = i64
        L.hag_last_error.restype = ctypes.c_char_p
        L.hag_forward_static_scratch.argtypes = [vp, ctypes.c_int, ctypes.c_int, i64, vp, vp, vp, vp]
        L.hag_probe_rows.argtypes = [vp, i64, i64, i64, i32, i64, vp, vp]
        L.hag_probe_rows.restype = i64
        L.hag_probe_copy.argtypes = [vp, vp, i64, vp]
        L.hag_probe_mfma_f32.argtypes = [i64, i64, vp, vp]
        L.hag_probe_mfma_f32.restype = i64
        L.hag_seq_search.argtypes = [i64, vp, vp, i64, ctypes.POINTER(i64), vp, vp, vp, vp, vp]
        L.hag_seq_create.argtypes = [i64, vp, vp, i64, ctypes.POINTER(vp)]
        L.hag_seq_free.argtypes = [vp]
        L.hag_seq_free.restype = None
        for name in ("hag_seq_cells", "hag_seq_ranks", "hag_seq_launches", "hag_seq_merges"):
            getattr(L, name).argtypes = [vp]
            getattr(L, name).restype = i64
        L.hag_seq_weight_grad_slabs.argtypes = [i64, i32, ctypes.POINTER(i64)]
        L.hag_seq_weight_grad_slabs.restype = i64
        L.hag_seq_upload.argtypes = [vp]
        L.hag_seq_get_plan.argtypes = [vp, i32] + [vp] * 8
        L.hag_seq_set_option.argtypes = [vp, i32, i64]
        L.hag_seq_check.argtypes = [vp, vp]
        L.hag_seq_train_workspace_bytes.argtypes = [vp, i64, i64]
        L.hag_seq_train_workspace_bytes.restype = ctypes.c_size_t
        L.hag_seq_lstm_forward_train.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp]
        L.hag_seq_lstm_backward.argtypes = [vp, i64, i64] + [vp] * 10
        L.hag_seq_workspace_bytes.argtypes = [vp, i64, i64]
        L.hag_seq_workspace_bytes.restype = ctypes.c_size_t
        L.hag_seq_lstm_forward.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp, vp]
        L.hag_set_option.argtypes = [vp, i32, i64]
        L.hag_check.argtypes = [vp, vp]
        for name in ("hag_route", "hag_naive_route"):
            getattr(L, name).argtypes = [vp, ctypes.c_int, ctypes.c_int, i64, i32]
        L.hag_weight_grad_workspace_bytes.argtypes = [i64, i64, i64]
        L.hag_weight_grad_workspace_bytes.restype = ctypes.c_size_t
        L.hag_weight_grad.argtypes = [i64, i64, i64, vp, i32] + [vp] * 4
        L.hag_narrow_product.argtypes = [i64, i64, i64, vp, i32, vp, i32, vp, vp, vp]
        L.hag_softmax_loss_workspace_bytes.argtypes = []
        L.hag_softmax_loss_workspace_bytes.restype = ctypes.c_size_t
        L.hag_softmax_loss.argtypes = [i64, i64, vp, vp, i64] + [vp] * 4
        L.hag_softmax_loss_grad.argtypes = [i64, i64, vp, vp, i64] + [vp] * 4
        f32, size_t = ctypes.c_float, ctypes.c_size_t
        L.hag_embedding.argtypes = [i64, i64, i64, i32, vp, i64, i32, vp, i64, f32, vp, vp]
        L.hag_embedding_grad_workspace_bytes.argtypes = [i64, i64, i64]
        L.hag_embedding_grad_workspace_bytes.restype = size_t
        L.hag_embedding_grad.argtypes = [i64, i64, i64, i32, vp, i64, i32, vp, i64, f32, i32, vp, vp, vp]
        L.hag_layer_norm.argtypes = [i64, i64, i32, vp, i64, i32, vp, vp, f32, vp, vp, vp, vp]
        L.hag_layer_norm_grad_workspace_bytes.argtypes = [i64, i64]
        L.hag_layer_norm_grad_workspace_bytes.restype = size_t
        L.hag_layer_norm_grad.argtypes = [i64, i64, i32, vp, i64, vp, i64, i32] + [vp] * 8
        L.hag_clip_workspace_bytes.argtypes = [i64]
        L.hag_clip_workspace_bytes.restype = size_t
        L.hag_clip_gradients.argtypes = [i64, vp, ctypes.c_double, vp, vp, vp]
        L.hag_rms_norm.argtypes = [i64, i64, i32, vp, i64, vp, i64, i32, vp, f32, vp, vp, vp, vp]
        L.hag_rms_norm_fp8.argtypes = [i64, i64, i32, vp, i64, vp, i64, i32, vp, f32, vp, vp, i64, vp, i64, vp]
        L.hag_rms_norm_grad_workspace_bytes.argtypes = [i64, i64]
        L.hag_rms_norm_grad_workspace_bytes.restype = size_t
        L.hag_rms_norm_grad.argtypes = [i64, i64, i32, vp, i64, vp, i64, vp, i64, i32] + [vp] * 6
        L.hag_fp8_product.argtypes = [i64, i64, i64] + [vp, i64] * 4 + [i32] + [vp] * 2
        L.hag_adamw.argtypes = [i64, vp, ctypes.POINTER(hag_adamw_options_t), vp]
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise HagError(rc, lib().hag_last_error().decode())


def _np(a, dtype):
    return np.ascontiguousarray(a, dtype=dtype)


def _view(ptr, count, dtype):
    if count == 0 or not ptr:
        return np.zeros(0, dtype=dtype)
    ct = {np.int32: ctypes.c_int32, np.int64: ctypes.c_int64}[dtype]
    return np.ctypeslib.as_array(ctypes.cast(ptr, ctypes.POINTER(ct)), shape=(count,)).copy()


def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return HAG_F32
    if t.dtype == torch.int32:
        return HAG_I32
    raise TypeError(f"unsupported dtype {t.dtype}")


_torch_calls = None


def _resolve_torch_calls():
    """(current_device, current raw stream of a device): torch's short forms where this build of it has them, else the public ones, which
    take 0.2 us and 0.6 us more (a Stream object is built first)."""
    import torch
    global _torch_calls
    device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch_calls = device, stream
    return _torch_calls


def _stream_ptr():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev_ptr(t):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("device tensors must be contiguous and on the GPU")
    return ctypes.c_void_p(t.data_ptr())


_ended = []                                 # (free, handle) of objects that are gone


def _free_ended(*more):
    """Frees the handles of objects that are gone.  Garbage is collected at any time: while this thread's stream is captured they wait, for the next ones or the next call of a handle (what other
    threads and streams capture is left alone by hag_free itself)."""
    _ended.extend(more)
    torch = sys.modules.get("torch")
    if _ended and not (torch is not None and torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing()):
        while True:
            try:
                free, handle = _ended.pop()
            except IndexError:                  # (or another thread's, or garbage collected meanwhile)
                return
            free(handle)


class Hag:
    """Owner of one hag_t handle."""

    def __init__(self, handle):
        self._h = ctypes.c_void_p(handle)
        self._ws = {}
        self._shapes = {}
        self._n = None

    def __del__(self):
        try:
            if self._h:
                handle, self._h = self._h, None
                _free_ended((lib().hag_free, handle))
        except Exception:
            pass

    # ---- host side ---------------------------------------------------------------------------
    def stats(self) -> dict:
        s = hag_stats_t()
        _check(lib().hag_stats(self._h, ctypes.byref(s)))
        return {k: getattr(s, k) for k, _ in s._fields_}

    def get_merges(self):
        n = ctypes.c_int64()
        l, r, red = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        _check(lib().hag_get_merges(self._h, ctypes.byref(n), ctypes.byref(l), ctypes.byref(r), ctypes.byref(red)))
        return _view(l.value, n.value, np.int32), _view(r.value, n.value, np.int32), _view(red.value, n.value, np.int32)

    def get_forward(self):
        st = self.stats()
        l, r, lp, hp, hc = (ctypes.c_void_p() for _ in range(5))
        nl = ctypes.c_int32()
        _check(lib().hag_get_forward(self._h, ctypes.byref(l), ctypes.byref(r), ctypes.byref(lp), ctypes.byref(nl),
                                     ctypes.byref(hp), ctypes.byref(hc)))
        return dict(agg_left=_view(l.value, st["a"], np.int32), agg_right=_view(r.value, st["a"], np.int32),
                    level_ptr=_view(lp.value, nl.value + 1, np.int32), n_levels=nl.value,
                    hrowptr=_view(hp.value, st["n"] + 1, np.int64), hcol=_view(hc.value, st["h"], np.int32))

    def prefix(self, n_merges) -> "Hag":
        out = ctypes.c_void_p()
        _check(lib().hag_prefix(self._h, int(n_merges), ctypes.byref(out)))
        return Hag(out.value)

    def algorithmic_bytes(self, which, op, d) -> int:
        return int(lib().hag_algorithmic_bytes(self._h, which, OPS[op], int(d)))

    # ---- device side -------------------------------------------------------------------------
    def upload(self):
        _free_ended()
        _check(lib().hag_upload(self._h, _stream_ptr()))
        return self

    def set_option(self, option, value):
        _check(lib().hag_set_option(self._h, int(option), int(value)))
        return self

    def check(self):
        """Synchronises the current stream; raises HagError(HAG_ETIMEOUT) if a one-launch pass gave up waiting."""
        _check(lib().hag_check(self._h, _stream_ptr()))

    def route(self, op="sum", dtype_code=HAG_F32, d=64, backward=False, naive=False) -> str:
        """The way forward or backward (naive: naive_forward or naive_backward) takes for this op, dtype and width: one of ROUTES."""
        query = lib().hag_naive_route if naive else lib().hag_route
        rc = int(query(self._h, OPS[op], dtype_code, int(d), int(backward)))
        if rc < 0:
            _check(rc)
        return ROUTES[rc]

    def workspace_bytes(self, op, dtype_code, d) -> int:
        return int(lib().hag_workspace_bytes(self._h, OPS[op], dtype_code, int(d)))

    def _check_args(self, what, a, op, out, argmax, workspace, needs_argmax):
        """Everything the C ABI cannot check from raw pointers: the library takes no row count, so a
        matrix with too few rows, a narrower dtype or a short workspace would make a kernel read or
        write out of bounds."""
        import torch
        if op not in OPS:
            raise ValueError(f"unknown op {op!r}")
        if self._n is None:
            self._n = self.stats()["n"]
        if a.dim() != 2 or a.shape[0] != self._n:
            raise ValueError(f"{what} must have shape [{self._n}, d], got {tuple(a.shape)}")
        code = _dtype_code(a)
        for name, t in (("output", out),):
            if t is not None and (t.shape != a.shape or t.dtype != a.dtype or t.device != a.device):
                raise ValueError(f"{name} must match {what}: shape {tuple(a.shape)}, dtype {a.dtype}, device {a.device}; "
                                 f"got {tuple(t.shape)}, {t.dtype}, {t.device}")
        if argmax is not None and (argmax.shape != a.shape or argmax.dtype != torch.int32 or argmax.device != a.device):
            raise ValueError(f"argmax must be int32 of shape {tuple(a.shape)} on {a.device}, got {argmax.dtype} "
                             f"{tuple(argmax.shape)} on {argmax.device}")
        if needs_argmax and argmax is None:
            raise ValueError("argmax is required for max")
        if workspace is not None:
            need = self.workspace_bytes(op, code, a.shape[1])
            have = workspace.numel() * workspace.element_size()
            if have < need or workspace.device != a.device:
                raise ValueError(f"workspace holds {have} bytes on {workspace.device}, {need} needed on {a.device}")

    def _shape(self, what, a, op):
        """(op code, dtype code, d, workspace bytes, forward workspace bytes) of a call on a matrix of a's shape and dtype; raises what _check_args
        raises for `a`.  Looked up by value: a handle's sizes never change, so neither do the answers."""
        key = (op, a.dtype, a.shape)
        got = self._shapes.get(key)
        if got is None:
            self._check_args(what, a, op, None, None, None, False)
            code, d = _dtype_code(a), int(a.shape[1])
            got = (OPS[op], code, d, self.workspace_bytes(op, code, d), int(lib().hag_forward_workspace_bytes(self._h, OPS[op], code, d)))
            if len(self._shapes) >= 256:
                self._shapes.clear()
            self._shapes[key] = got
        return got

    def _launch(self, fn, what, a, op, out, argmax, workspace, needs_argmax, backward, extra):
        # A call on a small graph takes about as long as preparing it, so everything that depends on sizes only is looked up, and
        # the stream is asked for once.
        import torch
        if _ended:
            _free_ended()
        op_code, code, d, nbytes, forward_nbytes = self._shape(what, a, op)
        if out is not None or argmax is not None or workspace is not None or needs_argmax:
            self._check_args(what, a, op, out, argmax, workspace, needs_argmax)
        if not a.is_cuda or not a.is_contiguous():
            raise ValueError("device tensors must be contiguous and on the GPU")
        if out is None:
            out = torch.empty_like(a)
        if op == "max" and argmax is None:
            argmax = torch.empty_like(a, dtype=torch.int32)
        current_device, raw_stream = _torch_calls or _resolve_torch_calls()
        device = current_device()
        stream = raw_stream(device)
        if workspace is None:
            # one buffer per (device, stream): calls enqueued on different streams may overlap.  The transposed pass of max, where it needs more than
            # forward passes brought, has one of its own: theirs may be in use by a captured graph and is not replaced
            index = a.get_device()
            key = (index, stream if index == device else raw_stream(index))
            if op == "max":
                if not backward:
                    nbytes = forward_nbytes
                elif nbytes > forward_nbytes and (key not in self._ws or self._ws[key].numel() < nbytes):
                    key = (*key, "sorted")
            workspace = self._ws.get(key)
            if workspace is None or workspace.numel() < nbytes:
                workspace = self._ws[key] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=a.device)
        rest = (argmax, out) if backward else (out, argmax)
        for t in (out, argmax, workspace):
            if t is not None and (not t.is_cuda or not t.is_contiguous()):
                raise ValueError("device tensors must be contiguous and on the GPU")
        rc = fn(self._h, op_code, code, d, a.data_ptr(), *(None if t is None else t.data_ptr() for t in rest), workspace.data_ptr(), stream, *extra)
        if rc != 0:
            _check(rc)
        return out, argmax

    def _fwd(self, fn, x, op, y, argmax, workspace, *extra):
        y, argmax = self._launch(fn, "x", x, op, y, argmax, workspace, False, False, extra)
        return (y, argmax) if op == "max" else y

    def _bwd(self, fn, gy, op, argmax, gx, workspace, *extra):
        return self._launch(fn, "gy", gy, op, gx, argmax, workspace, op == "max", True, extra)[0]

    def forward(self, x, op="sum", y=None, argmax=None, workspace=None):
        return self._fwd(lib().hag_forward, x, op, y, argmax, workspace)

    def backward(self, gy, op="sum", argmax=None, gx=None, workspace=None):
        return self._bwd(lib().hag_backward, gy, op, argmax, gx, workspace)

    def forward_static_scratch(self, x, op="sum", y=None, argmax=None):
        """hag_forward with the library's fixed scratch array as workspace (no workspace argument)."""
        import torch
        self._check_args("x", x, op, y, argmax, None, False)
        n, d = x.shape
        if y is None:
            y = torch.empty_like(x)
        if op == "max" and argmax is None:
            argmax = torch.empty((n, d), dtype=torch.int32, device=x.device)
        _check(lib().hag_forward_static_scratch(self._h, OPS[op], _dtype_code(x), d, _dev_ptr(x), _dev_ptr(y),
                                                _dev_ptr(argmax), _stream_ptr()))
        return (y, argmax) if op == "max" else y

    def forward_phases(self, x, phases, op="sum", y=None, argmax=None, workspace=None):
        return self._fwd(lib().hag_forward_phases, x, op, y, argmax, workspace, int(phases))

    def backward_phases(self, gy, phases, op="sum", argmax=None, gx=None, workspace=None):
        return self._bwd(lib().hag_backward_phases, gy, op, argmax, gx, workspace, int(phases))

    def naive_forward(self, x, op="sum", y=None, argmax=None, workspace=None):
        return self._fwd(lib().hag_naive_forward, x, op, y, argmax, workspace)

    def naive_backward(self, gy, op="sum", argmax=None, gx=None, workspace=None):
        return self._bwd(lib().hag_naive_backward, gy, op, argmax, gx, workspace)


def hag_search(rowptr, col, capacity, flags=HAG_SEARCH_CANONICAL, max_depth=0) -> Hag:
    rowptr, col = _np(rowptr, np.int64), _np(col, np.int32)
    out = ctypes.c_void_p()
    _check(lib().hag_search(rowptr.size - 1, rowptr.ctypes.data, col.ctypes.data, int(capacity), flags, max_depth,
                            ctypes.byref(out)))
    return Hag(out.value)


def hag_search_batched(rowptr, col, graph_ptr, capacity_fraction, flags=HAG_SEARCH_CANONICAL, max_depth=0) -> Hag:
    rowptr, col, graph_ptr = _np(rowptr, np.int64), _np(col, np.int32), _np(graph_ptr, np.int64)
    out = ctypes.c_void_p()
    _check(lib().hag_search_batched(rowptr.size - 1, rowptr.ctypes.data, col.ctypes.data, graph_ptr.size - 1,
                                    graph_ptr.ctypes.data, float(capacity_fraction), flags, max_depth,
                                    ctypes.byref(out)))
    return Hag(out.value)


def hag_from_merges(rowptr, col, left, right, flags=0) -> Hag:
    rowptr, col = _np(rowptr, np.int64), _np(col, np.int32)
    left, right = _np(left, np.int32), _np(right, np.int32)
    out = ctypes.c_void_p()
    _check(lib().hag_from_merges(rowptr.size - 1, rowptr.ctypes.data, col.ctypes.data, left.size,
                                 left.ctypes.data, right.ctypes.data, flags, ctypes.byref(out)))
    return Hag(out.value)


def _raw_stream():
    """The current stream of the current device, as a number."""
    current_device, raw_stream = _torch_calls or _resolve_torch_calls()
    return raw_stream(current_device())


def _matrices(*tensors):
    import torch
    for t in tensors:
        if t.dim() != 2 or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.device != tensors[0].device:
            raise ValueError("contiguous float32 matrices on one device are needed")


def narrow_product(x, w, transposed=False, relu=False, mask=None):
    """x w [n, k] of x [n, d] and a small w [d, k] (transposed: w [k, d]), on the current device; relu: of relu(x); mask [n, k]: 0 where it is not positive
    (hag_narrow_product)."""
    import torch
    _matrices(x, w)
    n, d = x.shape
    k = w.shape[0 if transposed else 1]
    if w.shape[1 if transposed else 0] != d:
        raise ValueError(f"x {tuple(x.shape)} and w {tuple(w.shape)} do not match")
    if mask is not None:
        _matrices(x, mask)
        if mask.shape != (n, k):
            raise ValueError(f"mask must have shape {(n, k)}")
    y = torch.empty((n, k), dtype=torch.float32, device=x.device)
    _check(lib().hag_narrow_product(n, d, k, x.data_ptr(), int(relu), w.data_ptr(), int(transposed), None if mask is None else mask.data_ptr(), y.data_ptr(),
                                    _raw_stream()))
    return y


def weight_grad(x, g, relu=False):
    """x^T g [d, k] (relu: relu(x)^T g) of float32 device matrices x [n, d] and g [n, k] on the current device (hag_weight_grad)."""
    import torch
    _matrices(x, g)
    n, d, k = *x.shape, g.shape[1]
    if g.shape[0] != n:
        raise ValueError("x and g must have the same number of rows")
    out = torch.empty((d, k), dtype=torch.float32, device=x.device)
    ws = torch.empty(max(lib().hag_weight_grad_workspace_bytes(n, d, k), 16), dtype=torch.uint8, device=x.device)
    _check(lib().hag_weight_grad(n, d, k, x.data_ptr(), int(relu), g.data_ptr(), out.data_ptr(), ws.data_ptr(), _raw_stream()))
    return out


def _check_loss_args(z, labels):
    import torch
    _matrices(z)
    if labels.dim() != 1 or labels.dtype != torch.int64 or labels.shape[0] != z.shape[0] or labels.device != z.device or not labels.is_contiguous():
        raise ValueError("labels must be contiguous int64, one per row of z, on its device")
    return z.shape


def _scalar(t, like):
    import torch
    if t.numel() != 1 or t.dtype != torch.float32 or t.device != like.device:
        raise ValueError("a float32 scalar on z's device is needed")
    return t.data_ptr()


def softmax_loss(z, labels, ignore=-100):
    """(loss, rows that count), scalars on the device: SoftMax cross-entropy of z [n, classes], mean over the rows whose label is not `ignore`."""
    import torch
    n, classes = _check_loss_args(z, labels)
    loss, counted = (torch.empty((), dtype=torch.float32, device=z.device) for _ in range(2))
    ws = torch.empty(lib().hag_softmax_loss_workspace_bytes(), dtype=torch.uint8, device=z.device)
    _check(lib().hag_softmax_loss(n, classes, z.data_ptr(), labels.data_ptr(), int(ignore), loss.data_ptr(), counted.data_ptr(), ws.data_ptr(), _raw_stream()))
    return loss, counted


def softmax_loss_grad(z, labels, counted, g_loss, ignore=-100):
    """Gradient of g_loss * softmax_loss at z."""
    import torch
    n, classes = _check_loss_args(z, labels)
    out = torch.empty_like(z)
    _check(lib().hag_softmax_loss_grad(n, classes, z.data_ptr(), labels.data_ptr(), int(ignore), _scalar(counted, z), _scalar(g_loss, z), out.data_ptr(), _raw_stream()))
    return out


_elements = None


def _element_codes():
    """{torch dtype: HAG code} of what lookups, layer norm and clipping take."""
    import torch
    global _elements
    _elements = {torch.float32: HAG_F32, torch.bfloat16: HAG_BF16, torch.float16: HAG_F16}
    return _elements


def _device():
    return (_torch_calls or _resolve_torch_calls())[0]()


def _rows(name, t, device):
    """(element code, row stride) of a matrix with contiguous rows on the current device."""
    code = (_elements or _element_codes()).get(t.dtype)
    if code is None or t.dim() != 2 or t.get_device() != device:
        raise ValueError(f"{name} must be a float32, bfloat16 or float16 matrix on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    n, d = t.shape
    stride, step = t.stride()
    if step != 1 and d > 1 and n > 0:
        raise ValueError(f"the rows of {name} must be contiguous, got strides {tuple(t.stride())}")
    return code, stride if n > 1 else d


def _ids(ids, device):
    import torch
    if ids.dtype not in (torch.int64, torch.int32) or ids.get_device() != device or not ids.is_contiguous():
        raise ValueError(f"ids must be contiguous int64 or int32 on the current device, got {ids.dtype} {tuple(ids.shape)} on {ids.device}")
    return HAG_I64 if ids.dtype == torch.int64 else HAG_I32


def _padding(padding):
    """As a 64-bit number; one that no id can be is no padding (ctypes would pass its low 64 bits)."""
    padding = int(padding)
    if padding == HAG_NO_PADDING:
        raise ValueError("a padding of -2**63 cannot be told from none")
    return padding if HAG_NO_PADDING < padding < 1 << 63 else HAG_NO_PADDING


def embedding(table, ids, scale=1.0, padding=None):
    """scale * table[ids] [*ids.shape, d] of a table [rows, d] (hag_embedding).  Ids equal to `padding` (any number but -2**63, a row or not) give rows of zeros, ids that
    are no row of the table rows of NaN."""
    device = _device()
    code, stride = _rows("table", table, device)
    id_code, (rows, d) = _ids(ids, device), table.shape
    y = table.new_empty((*ids.shape, d))
    rc = lib().hag_embedding(ids.numel(), rows, d, code, table.data_ptr(), stride, id_code, ids.data_ptr(), HAG_NO_PADDING if padding is None else _padding(padding), scale,
                             y.data_ptr(), _raw_stream())
    if rc != 0:
        _check(rc)
    return y


def embedding_grad(g_y, ids, rows, scale=1.0, padding=None, dtype=None):
    """Gradient [rows, d] at the table of embedding(table, ids, scale, padding), for the gradient g_y [n, d] at its rows, n = ids.numel() (hag_embedding_grad);
    dtype: that of g_y (the default) or float32."""
    device = _device()
    code, stride = _rows("g_y", g_y, device)
    id_code, (n, d) = _ids(ids, device), g_y.shape
    if ids.numel() != n:
        raise ValueError(f"g_y has {n} rows for {ids.numel()} ids")
    if dtype is not None and dtype not in _elements:
        raise ValueError(f"unsupported dtype {dtype}")
    if rows < 0:
        raise ValueError("rows must not be negative")
    L = lib()
    nbytes = 0 if rows >> 31 else L.hag_embedding_grad_workspace_bytes(n, rows, d)
    if not nbytes:                                         # sizes that are refused, before anything of that size is made
        _check(L.hag_embedding_grad(n, min(rows, 1 << 31), d, code, None, stride, id_code, None, HAG_NO_PADDING, scale, code, None, None, None))
    out, ws = g_y.new_empty((rows, d), dtype=dtype), g_y.new_empty(_elements_of(nbytes, code))
    rc = L.hag_embedding_grad(n, rows, d, code, g_y.data_ptr(), stride, id_code, ids.data_ptr(), HAG_NO_PADDING if padding is None else _padding(padding), scale,
                              code if dtype is None else _elements[dtype], out.data_ptr(), ws.data_ptr(), _raw_stream())
    if rc != 0:
        _check(rc)
    return out


def _elements_of(nbytes, code):
    """Elements of the type that take so many bytes: a workspace made as a tensor like the call's own takes half as long to make as one of bytes."""
    return nbytes // 4 if code == HAG_F32 else nbytes // 2


def _norm_params(x, weight, bias):
    """The element code of weight and bias, which have the type of x or are float32, and their addresses."""
    code, ptrs, d = None, [None, None], x.shape[1]
    for k, t in enumerate((weight, bias)):
        if t is None:
            continue
        got = _elements.get(t.dtype)
        if t.shape != (d,) or t.get_device() != x.get_device() or not t.is_contiguous() or (got != HAG_F32 and t.dtype != x.dtype) or (code is not None and got != code):
            raise ValueError(f"{('weight', 'bias')[k]} must have one contiguous element for each of the {d} columns, float32 or of the type of x, on its device (and both the "
                             f"same); got {t.dtype} {tuple(t.shape)} on {t.device}")
        code = got
        ptrs[k] = t.data_ptr()
    return HAG_F32 if code is None else code, ptrs


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of x [n, d]: every row less its mean, over its standard deviation, times weight plus bias (hag_layer_norm)."""
    import torch
    code, stride = _rows("x", x, _device())
    n, d = x.shape
    param_code, (w, b) = _norm_params(x, weight, bias)
    f32 = None if code == HAG_F32 else torch.float32       # (of x, or)
    y, mean, rstd = x.new_empty((n, d)), x.new_empty(n, dtype=f32), x.new_empty(n, dtype=f32)
    rc = lib().hag_layer_norm(n, d, code, x.data_ptr(), stride, param_code, w, b, eps, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _raw_stream())
    if rc != 0:
        _check(rc)
    return y, mean, rstd


def layer_norm_grad(g_y, x, mean, rstd, weight=None, params=True):
    """(g_x, g_weight, g_bias): the gradients of layer_norm for the gradient g_y at y, mean and rstd as it returned them; the latter two of the type of weight
    (float32 without one), None if not params (hag_layer_norm_grad)."""
    device = _device()
    code, stride = _rows("x", x, device)
    g_code, g_stride = _rows("g_y", g_y, device)
    if g_code != code or g_y.shape != x.shape:
        raise ValueError(f"g_y must match x: {x.dtype} {tuple(x.shape)}, got {g_y.dtype} {tuple(g_y.shape)}")
    n, d = x.shape
    for name, t in (("mean", mean), ("rstd", rstd)):
        if _elements.get(t.dtype) != HAG_F32 or t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous float32, one for each of the {n} rows, on the current device")
    param_code, (w, _) = _norm_params(x, weight, None)
    g_x, g_w, g_b, where = x.new_empty((n, d)), None, None, (None, None, None)
    L = lib()
    if params:
        like = mean if weight is None else weight
        g_w, g_b, ws = like.new_empty(d), like.new_empty(d), mean.new_empty(L.hag_layer_norm_grad_workspace_bytes(n, d) // 4)
        where = g_w.data_ptr(), g_b.data_ptr(), ws.data_ptr()
    rc = L.hag_layer_norm_grad(n, d, code, g_y.data_ptr(), g_stride, x.data_ptr(), stride, param_code, w, mean.data_ptr(), rstd.data_ptr(), g_x.data_ptr(), *where, _raw_stream())
    if rc != 0:
        _check(rc)
    return g_x, g_w, g_b


def _dense(t):
    """Its elements fill a piece of memory, in whatever order of the dimensions."""
    count = 1
    for stride, size in sorted((stride, size) for stride, size in zip(t.stride(), t.shape) if size != 1):
        if stride != count:
            return False
        count *= size
    return True


def clip_gradients(tensors, max_norm, out=None):
    """The 2-norm (float32, on the device) of all elements of `tensors` as one vector; where it is above max_norm they are scaled down to it, in place or into the
    tensors of `out`, which get them unchanged where it is not (hag_clip_gradients).  The tensors fill their memory and do not overlap, each is float32, bfloat16 or float16."""
    import torch
    tensors = list(tensors)
    outs = tensors if out is None else list(out)
    if len(outs) != len(tensors):
        raise ValueError(f"{len(outs)} outputs for {len(tensors)} tensors")
    device, codes = _device(), _elements or _element_codes()
    entries = []
    for t, o in zip(tensors, outs):
        code, whole = codes.get(t.dtype), t.is_contiguous()
        if code is None or t.get_device() != device or not (whole or _dense(t)):
            raise ValueError(f"dense float32, bfloat16 or float16 tensors on the current device are needed, got {t.dtype} {tuple(t.shape)} with strides {tuple(t.stride())} on {t.device}")
        if o is not t and (o.dtype != t.dtype or o.shape != t.shape or o.get_device() != device or not (whole and o.is_contiguous() or o.stride() == t.stride())):
            raise ValueError(f"an output must match its tensor: {t.dtype} {tuple(t.shape)} with strides {tuple(t.stride())}, got {o.dtype} {tuple(o.shape)} with {tuple(o.stride())}")
        count = t.numel()
        if count:
            at = t.data_ptr()
            entries += (at, at if o is t else o.data_ptr(), count, code)
    count = len(entries) // 4
    if len(set(entries[1::4])) != count:
        raise ValueError("a tensor is named twice")
    L = lib()
    ws = torch.empty(L.hag_clip_workspace_bytes(count), dtype=torch.uint8, device="cuda")
    norm = torch.empty((), dtype=torch.float32, device="cuda")
    table = array.array("q", entries)
    rc = L.hag_clip_gradients(count, table.buffer_info()[0], max_norm, norm.data_ptr(), ws.data_ptr(), _raw_stream())
    if rc != 0:
        _check(rc)
    return norm


def _norm_input(x, weight, residual):
    """(element code, row stride, residual's address and row stride, code and address of the weight) of an RMS norm's arguments."""
    device = _device()
    code, stride = _rows("x", x, device)
    param_code, (w, _) = _norm_params(x, weight, None)
    if residual is None:
        return code, stride, None, 0, param_code, w
    res_code, res_stride = _rows("residual", residual, device)
    if res_code != code or residual.shape != x.shape:
        raise ValueError(f"residual must match x: {x.dtype} {tuple(x.shape)}, got {residual.dtype} {tuple(residual.shape)}")
    return code, stride, residual.data_ptr(), res_stride, param_code, w


def rms_norm(x, weight=None, eps=1e-5, residual=None):
    """(y, h, rstd) of x [n, d]: h = x + residual (x itself without one), rstd = 1 / sqrt(mean of h^2 + eps) of every row, y = h * rstd * weight (hag_rms_norm)."""
    import torch
    code, stride, res, res_stride, param_code, w = _norm_input(x, weight, residual)
    n, d = x.shape
    y, rstd = x.new_empty((n, d)), x.new_empty(n, dtype=None if code == HAG_F32 else torch.float32)
    h = x if residual is None else x.new_empty((n, d))
    rc = lib().hag_rms_norm(n, d, code, x.data_ptr(), stride, res, res_stride, param_code, w, eps, h.data_ptr(), y.data_ptr(), rstd.data_ptr(), _raw_stream())
    if rc != 0:
        _check(rc)
    return y, h, rstd


def rms_norm_fp8(x, weight=None, eps=1e-5, residual=None):
    """(codes, scales, h): rms_norm with y in 8 bits, codes [n, d] float8_e4m3fn, whose rows begin at multiples of 16 elements, and scales [n, ceil(d / 32)] float8_e8m0fnu, a power of two
    for every 32 columns: y is about codes * scales (hag_rms_norm_fp8)."""
    import torch
    code, stride, res, res_stride, param_code, w = _norm_input(x, weight, residual)
    n, d = x.shape
    wide, blocks = (d + 15) // 16 * 16, (d + 31) // 32
    codes, scales = x.new_empty((n, wide), dtype=torch.float8_e4m3fn), x.new_empty((n, blocks), dtype=torch.float8_e8m0fnu)
    h = x if residual is None else x.new_empty((n, d))
    rc = lib().hag_rms_norm_fp8(n, d, code, x.data_ptr(), stride, res, res_stride, param_code, w, eps, h.data_ptr(), codes.data_ptr(), wide, scales.data_ptr(), blocks, _raw_stream())
    if rc != 0:
        _check(rc)
    return codes if wide == d else codes[:, :d], scales, h


def rms_norm_grad(g_y, h, rstd, weight=None, g_h=None, params=True):
    """(g_x, g_weight): the gradients of rms_norm for the gradient g_y at y and, where h is used further, g_h at h; h and rstd as it returned them.  g_x is the gradient at x
    and at the residual; g_weight has the type of weight (float32 without one), None if not params (hag_rms_norm_grad)."""
    device = _device()
    code, stride = _rows("h", h, device)
    n, d = h.shape
    more = [None, 0]
    g_code, g_stride = _rows("g_y", g_y, device)
    if g_code != code or g_y.shape != h.shape:
        raise ValueError(f"g_y must match h: {h.dtype} {tuple(h.shape)}, got {g_y.dtype} {tuple(g_y.shape)}")
    if g_h is not None:
        more_code, more_stride = _rows("g_h", g_h, device)
        if more_code != code or g_h.shape != h.shape:
            raise ValueError(f"g_h must match h: {h.dtype} {tuple(h.shape)}, got {g_h.dtype} {tuple(g_h.shape)}")
        more = [g_h.data_ptr(), more_stride]
    if _elements.get(rstd.dtype) != HAG_F32 or rstd.shape != (n,) or rstd.get_device() != device or not rstd.is_contiguous():
        raise ValueError(f"rstd must be contiguous float32, one for each of the {n} rows, on the current device")
    param_code, (w, _) = _norm_params(h, weight, None)
    g_x, g_w, ws, where = h.new_empty((n, d)), None, None, (None, None)
    L = lib()
    if params:
        g_w, ws = (rstd if weight is None else weight).new_empty(d), rstd.new_empty(L.hag_rms_norm_grad_workspace_bytes(n, d) // 4)
        where = g_w.data_ptr(), ws.data_ptr()
    rc = L.hag_rms_norm_grad(n, d, code, g_y.data_ptr(), g_stride, *more, h.data_ptr(), stride, param_code, w, rstd.data_ptr(), g_x.data_ptr(), *where, _raw_stream())
    if rc != 0:
        _check(rc)
    return g_x, g_w


def _rows_fp8(name, codes, scales, device):
    """Row strides of rows in 8 bits and of their scales."""
    import torch
    if codes.dtype != torch.float8_e4m3fn or scales.dtype != torch.float8_e8m0fnu or codes.dim() != 2 or codes.get_device() != device or scales.get_device() != device:
        raise ValueError(f"{name} must be a float8_e4m3fn matrix with float8_e8m0fnu scales on the current device, got {codes.dtype} {tuple(codes.shape)} on {codes.device} "
                         f"and {scales.dtype} on {scales.device}")
    n, d = codes.shape
    if scales.shape != (n, (d + 31) // 32):
        raise ValueError(f"the scales of {name} {(n, d)} must have shape {(n, (d + 31) // 32)}, got {tuple(scales.shape)}")
    if (codes.stride(1) != 1 and d > 1 or scales.stride(1) != 1 and d > 32) and n > 0:
        raise ValueError(f"the rows of {name} and its scales must be contiguous, got strides {tuple(codes.stride())} and {tuple(scales.stride())}")
    return (codes.stride(0), scales.stride(0)) if n > 1 else (d, scales.shape[1])


def fp8_product(x, x_scales, w, w_scales, dtype=None):
    """x w^T [n, k] of rows in 8 bits, x [n, d] and w [k, d] as rms_norm_fp8 and layers.quantize_fp8 give them; dtype: float32 (the default), bfloat16 or float16 (hag_fp8_product).

    float32 adds up exact products.  For 16 bits products lose what is below 2^-13 of the largest of their neighbours: 1.5e-5 to 5e-5 of the result's norm, before it is rounded (2^-8 or 2^-11)."""
    import torch
    device = _device()
    dtype = torch.float32 if dtype is None else dtype
    code = (_elements or _element_codes()).get(dtype)
    if code is None:
        raise ValueError(f"unsupported dtype {dtype}")
    x_strides, w_strides = _rows_fp8("x", x, x_scales, device), _rows_fp8("w", w, w_scales, device)
    (n, d), k = x.shape, w.shape[0]
    if w.shape[1] != d:
        raise ValueError(f"x {tuple(x.shape)} and w {tuple(w.shape)} do not match")
    y = x.new_empty((n, k), dtype=dtype)
    rc = lib().hag_fp8_product(n, d, k, x.data_ptr(), x_strides[0], x_scales.data_ptr(), x_strides[1], w.data_ptr(), w_strides[0], w_scales.data_ptr(), w_strides[1], code, y.data_ptr(),
                               _raw_stream())
    if rc != 0:
        _check(rc)
    return y


def adamw_states(params, bits=32):
    """States of adamw for the tensors `params` that have seen no gradient: {"m": ..., "v": ...}, lists of tensors of zeros, float32 for 32 bits and float8_e4m3fn for 8, then with
    "m_scales" and "v_scales", float8_e8m0fnu, one for every 32 elements in the order of memory."""
    import torch
    if bits not in (8, 32):
        raise ValueError("states have 32 or 8 bits")
    dtype = torch.float32 if bits == 32 else torch.float8_e4m3fn
    # (their elements are in the order of the parameter's memory: what shape they have says nothing)
    states = {k: [torch.zeros(p.numel(), dtype=torch.float32 if bits == 32 else torch.uint8, device=p.device).view(dtype) for p in params] for k in ("m", "v")}
    if bits == 8:
        states.update({k: [torch.full(((p.numel() + 31) // 32,), 127, dtype=torch.uint8, device=p.device).view(torch.float8_e8m0fnu) for p in params] for k in ("m_scales", "v_scales")})
    return states


def _scalar_at(name, t, dtype, device):
    if t.numel() != 1 or t.dtype != dtype or t.get_device() != device:
        raise ValueError(f"{name} must be one {dtype} on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _adamw_check(p, g, states, scales, copy, device):
    """Raises what is wrong with one tensor of adamw and what belongs to it."""
    import torch
    codes, whole, count = _elements, p.is_contiguous(), p.numel()
    if p.dtype not in codes or p.get_device() != device or not (whole or _dense(p)):
        raise ValueError(f"dense float32, bfloat16 or float16 parameters on the current device are needed, got {p.dtype} {tuple(p.shape)} with strides {tuple(p.stride())} on {p.device}")
    if g.dtype not in codes or (g.dtype != p.dtype and p.dtype != torch.float32) or g.shape != p.shape or g.get_device() != device or not (whole and g.is_contiguous() or g.stride() == p.stride()):
        raise ValueError(f"a gradient must match its parameter: {p.dtype} {tuple(p.shape)} with strides {tuple(p.stride())}, got {g.dtype} {tuple(g.shape)} with {tuple(g.stride())}")
    state_dtype = torch.float8_e4m3fn if scales else torch.float32
    for t in states:
        if t.dtype != state_dtype or t.numel() != count or t.get_device() != device or not (t.is_contiguous() or t.shape == p.shape and t.stride() == p.stride()):
            raise ValueError(f"a state must be {state_dtype}, dense, of its parameter's {count} elements, on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    for t in scales:
        if t.dtype != torch.float8_e8m0fnu or t.numel() != (count + 31) // 32 or t.get_device() != device or not t.is_contiguous():
            raise ValueError(f"scales must be contiguous float8_e8m0fnu, {(count + 31) // 32} of them, on the current device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if copy is not None and (copy.dtype not in codes or copy.shape != p.shape or copy.get_device() != device or not (whole and copy.is_contiguous() or copy.stride() == p.stride())):
        raise ValueError(f"a copy must match its parameter {tuple(p.shape)} with strides {tuple(p.stride())}, got {copy.dtype} {tuple(copy.shape)} with {tuple(copy.stride())}")


def adamw(params, grads, m, v, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, norm=None, max_norm=None, copies=None, m_scales=None, v_scales=None, seed=0):
    """One step of AdamW on the tensors `params`, in place, with their gradients and states, lists of one tensor each (hag_adamw).

    params float32, bfloat16 or float16, dense; gradients of the same shape and order in memory and, but for float32 parameters, type.  m and v as adamw_states makes them, with
    m_scales and v_scales for 8 bits.  step: a number, from 1 on, or an int64 scalar on the device; lr: a number or a float32 scalar on the device.  With norm (a float32 scalar on the
    device, as clip_gradients returns it) the gradients count as if scaled down to max_norm where it is above, and nothing changes where it is no finite number.  copies: tensors (or
    None) of any of the three types that get the new parameters too.  seed: of the rounding of 8-bit states."""
    import torch
    device = _device()
    _elements or _element_codes()
    bits = 32 if m_scales is None else 8
    params, grads = list(params), list(grads)
    m, v = list(m), list(v)
    copies = [None] * len(params) if copies is None else list(copies)
    scales = [()] * len(params) if bits == 32 else list(zip(m_scales, v_scales or ()))
    if not len(params) == len(grads) == len(m) == len(v) == len(scales) == len(copies) or (bits == 32 and v_scales is not None):
        raise ValueError(f"{len(params)} parameters need as many gradients, states, scales of 8-bit states and copies")
    options = hag_adamw_options_t(0.0, betas[0], betas[1], eps, weight_decay, 1.0, 0, None, None, None, seed & 0xFFFFFFFF, bits)
    if isinstance(step, torch.Tensor):
        options.step_device = _scalar_at("step", step, torch.int64, device)
    else:
        options.step = step
    if isinstance(lr, torch.Tensor):
        options.lr_device = _scalar_at("lr", lr, torch.float32, device)
    else:
        options.lr = lr
    if (norm is None) != (max_norm is None):
        raise ValueError("norm and max_norm go together")
    if norm is not None:
        options.norm, options.max_norm = _scalar_at("norm", norm, torch.float32, device), max_norm
    codes, state_dtype, entries, written = _elements, torch.float32 if bits == 32 else torch.float8_e4m3fn, [], []
    for p, g, a, b, sc, copy in zip(params, grads, m, v, scales, copies):
        code, g_code, count = codes.get(p.dtype), codes.get(g.dtype), p.numel()
        # tensors of the ordinary kind pass at once, others are looked at one by one
        if not (code is not None and g_code is not None and (code == g_code or code == HAG_F32) and p.get_device() == g.get_device() == a.get_device() == b.get_device() == device
                and p.is_contiguous() and g.is_contiguous() and a.is_contiguous() and b.is_contiguous() and a.dtype == b.dtype == state_dtype and a.numel() == b.numel() == count and p.shape == g.shape
                and (copy is None or copy.dtype in codes and copy.get_device() == device and copy.is_contiguous() and copy.shape == p.shape)
                and (not sc or sc[0].get_device() == sc[1].get_device() == device and sc[0].is_contiguous() and sc[1].is_contiguous() and sc[0].dtype == sc[1].dtype == torch.float8_e8m0fnu
                     and sc[0].numel() == sc[1].numel() == (count + 31) // 32)):
            _adamw_check(p, g, (a, b), sc, copy, device)
        if count:
            at_p, at_a, at_b, at_copy = p.data_ptr(), a.data_ptr(), b.data_ptr(), 0 if copy is None else copy.data_ptr()
            at_sa, at_sb = (sc[0].data_ptr(), sc[1].data_ptr()) if sc else (0, 0)
            entries += (at_p, g.data_ptr(), at_a, at_b, at_copy, at_sa, at_sb, count, code | g_code << 32, 0 if copy is None else codes[copy.dtype])
            written += (at_p, at_a, at_b)
            if at_copy:
                written.append(at_copy)
            if sc:
                written += (at_sa, at_sb)
    if len(set(written)) != len(written):
        raise ValueError("a tensor is named twice")
    table = array.array("q", entries)
    rc = lib().hag_adamw(len(entries) // 10, table.buffer_info()[0], ctypes.byref(options), _raw_stream())
    if rc != 0:
        _check(rc)


def probe_rows(src, n_rows, d, reads, from_lds, workgroups, sink) -> int:
    """hag_probe_rows on torch device tensors; returns the row bytes the launch reads."""
    if src.numel() < n_rows * d or sink.numel() < workgroups * 1024:
        raise ValueError("probe buffers too small")
    rc = lib().hag_probe_rows(_dev_ptr(src), int(n_rows), int(d), int(reads), int(from_lds), int(workgroups),
                              _dev_ptr(sink), _stream_ptr())
    if rc < 0:
        _check(rc)
    return int(rc)


def probe_copy(src, dst, nbytes):
    if src.numel() * src.element_size() < nbytes or dst.numel() * dst.element_size() < nbytes:
        raise ValueError("copy buffers too small")
    _check(lib().hag_probe_copy(_dev_ptr(src), _dev_ptr(dst), int(nbytes), _stream_ptr()))


def probe_mfma_f32(iters, workgroups, sink) -> int:
    """hag_probe_mfma_f32; returns the flops of the launch."""
    if sink.numel() * sink.element_size() < workgroups * 1024:
        raise ValueError("sink too small")
    rc = lib().hag_probe_mfma_f32(int(iters), int(workgroups), _dev_ptr(sink), _stream_ptr())
    if rc < 0:
        _check(int(rc))
    return int(rc)


def hag_seq_search(rowptr, col, capacity):
    """Algorithm 3 for a sequential Aggregate (ordered lists): (left, right, redundancy, hrowptr, hcol)."""
    rowptr, col = _np(rowptr, np.int64), _np(col, np.int32)
    n, e = rowptr.size - 1, int(rowptr[-1]) if rowptr.size else 0
    cap = int(min(max(capacity, 0), e))
    left, right, red = (np.zeros(max(cap, 1), dtype=np.int32) for _ in range(3))
    hrowptr = np.zeros(n + 1, dtype=np.int64)
    hcol = np.zeros(max(e, 1), dtype=np.int32)
    a = ctypes.c_int64()
    _check(lib().hag_seq_search(n, rowptr.ctypes.data, col.ctypes.data, int(capacity), ctypes.byref(a), left.ctypes.data,
                                right.ctypes.data, red.ctypes.data, hrowptr.ctypes.data, hcol.ctypes.data))
    return left[:a.value], right[:a.value], red[:a.value], hrowptr, hcol[:hrowptr[n]]


class SeqHag:
    """Plan of an LSTM aggregator over ordered neighbour lists (hag_seq_create): a prefix HAG when capacity > 0,
    the plain lists when capacity == 0."""

    def __init__(self, rowptr, col, capacity):
        rowptr, col = _np(rowptr, np.int64), _np(col, np.int32)
        self.n = rowptr.size - 1
        h = ctypes.c_void_p()
        _check(lib().hag_seq_create(self.n, rowptr.ctypes.data, col.ctypes.data, int(capacity), ctypes.byref(h)))
        self._h = h
        self._ws = {}

    def __del__(self):
        try:                                # at interpreter shutdown the module's globals may be gone already
            if getattr(self, "_h", None):
                handle, self._h = self._h, None
                _free_ended((lib().hag_seq_free, handle))
        except Exception:
            pass

    @property
    def cells(self) -> int:
        return int(lib().hag_seq_cells(self._h))

    @property
    def ranks(self) -> int:
        return int(lib().hag_seq_ranks(self._h))

    @property
    def launches(self) -> int:
        return int(lib().hag_seq_launches(self._h))

    @property
    def merges(self) -> int:
        return int(lib().hag_seq_merges(self._h))

    def plan(self, order=0):
        """(n_states, paths [n_paths, 4], step_x, step_out, level_ptr, final_state) as copies (hag_seq_get_plan);
        order 0: paths grouped by level, 1: by the depth of their start state (the one-launch pass)."""
        i64, p32, p64 = ctypes.c_int64, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int64)
        ns, npaths, nl = i64(), i64(), i64()
        paths, sx, so, fs, lp = p32(), p32(), p32(), p32(), p64()
        _check(lib().hag_seq_get_plan(self._h, int(order), ctypes.byref(ns), ctypes.byref(npaths), ctypes.byref(paths), ctypes.byref(sx),
                                      ctypes.byref(so), ctypes.byref(nl), ctypes.byref(lp), ctypes.byref(fs)))
        take = lambda ptr, count, dt: (np.ctypeslib.as_array(ptr, shape=(count,)).astype(dt, copy=True) if count else np.zeros(0, dt))
        cells = self.cells
        return (ns.value, take(paths, 4 * npaths.value, np.int32).reshape(-1, 4), take(sx, cells, np.int32), take(so, cells, np.int32),
                take(lp, nl.value + 1, np.int64), take(fs, self.n, np.int32))

    def upload(self):
        _free_ended()
        _check(lib().hag_seq_upload(self._h))
        return self

    def set_option(self, option, value):
        _check(lib().hag_seq_set_option(self._h, int(option), int(value)))
        return self

    def train_workspace_bytes(self, d, hidden) -> int:
        return int(lib().hag_seq_train_workspace_bytes(self._h, int(d), int(hidden)))

    def lstm_forward_train(self, x, w_ih, w_hh, b, workspace=None):
        """As lstm_forward, keeping what lstm_backward needs; returns (a [n, H], workspace)."""
        import torch
        if _ended:
            _free_ended()
        hidden, d = int(w_hh.shape[1]), int(x.shape[1])
        for name, t, shape in (("x", x, (self.n, d)), ("w_ih", w_ih, (4 * hidden, d)), ("w_hh", w_hh, (4 * hidden, hidden)),
                               ("b", b, (4 * hidden,))):
            if tuple(t.shape) != shape or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous float32 device tensor of shape {shape}")
        need = self.train_workspace_bytes(d, hidden)
        if need == 0:
            raise ValueError("d must be a multiple of 4, hidden a multiple of 8 up to 128, d + hidden at most 256")
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        elif workspace.numel() * workspace.element_size() < need or workspace.device != x.device:
            raise ValueError("workspace too small or on another device")
        out = torch.empty((self.n, hidden), dtype=torch.float32, device=x.device)
        _check(lib().hag_seq_lstm_forward_train(self._h, d, hidden, _dev_ptr(x), _dev_ptr(w_ih), _dev_ptr(w_hh), _dev_ptr(b),
                                                _dev_ptr(out), _dev_ptr(workspace), _stream_ptr()))
        return out, workspace

    def lstm_backward(self, x, w_ih, w_hh, g_a, workspace):
        """Gradients (g_x, g_w_ih, g_w_hh, g_b) of a loss with gradient g_a [n, H] at a_out, after lstm_forward_train with
        the same x, w_ih, w_hh and workspace."""
        import torch
        hidden, d = int(w_hh.shape[1]), int(x.shape[1])
        for name, t, shape in (("x", x, (self.n, d)), ("w_ih", w_ih, (4 * hidden, d)), ("w_hh", w_hh, (4 * hidden, hidden)),
                               ("g_a", g_a, (self.n, hidden))):
            if tuple(t.shape) != shape or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous float32 device tensor of shape {shape}")
        need = self.train_workspace_bytes(d, hidden)
        if need == 0 or workspace.numel() * workspace.element_size() < need or workspace.device != x.device:
            raise ValueError("workspace too small or on another device")
        new = lambda *shape: torch.empty(shape, dtype=torch.float32, device=x.device)
        g_x, g_w_ih, g_w_hh, g_b = new(self.n, d), new(4 * hidden, d), new(4 * hidden, hidden), new(4 * hidden)
        _check(lib().hag_seq_lstm_backward(self._h, d, hidden, _dev_ptr(x), _dev_ptr(w_ih), _dev_ptr(w_hh), _dev_ptr(g_a), _dev_ptr(g_x),
                                           _dev_ptr(g_w_ih), _dev_ptr(g_w_hh), _dev_ptr(g_b), _dev_ptr(workspace), _stream_ptr()))
        return g_x, g_w_ih, g_w_hh, g_b

    def check(self):
        """Synchronise the current stream; raises HagError(HAG_ETIMEOUT) if a wait of a one-launch pass gave up."""
        _check(lib().hag_seq_check(self._h, _stream_ptr()))

    def workspace_bytes(self, d, hidden) -> int:
        return int(lib().hag_seq_workspace_bytes(self._h, int(d), int(hidden)))

    def lstm_forward(self, x, w_ih, w_hh, b, out=None, workspace=None):
        """a [n, H] = LSTM aggregate of every node's ordered list; torch float32 device tensors."""
        import torch
        if _ended:
            _free_ended()
        hidden, d = int(w_hh.shape[1]), int(x.shape[1])
        for name, t, shape in (("x", x, (self.n, d)), ("w_ih", w_ih, (4 * hidden, d)), ("w_hh", w_hh, (4 * hidden, hidden)),
                               ("b", b, (4 * hidden,))):
            if tuple(t.shape) != shape or t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous float32 device tensor of shape {shape}")
        if out is None:
            out = torch.empty((self.n, hidden), dtype=torch.float32, device=x.device)
        elif tuple(out.shape) != (self.n, hidden) or out.dtype != torch.float32 or not out.is_contiguous() or out.device != x.device:
            raise ValueError("out must be a contiguous float32 tensor [n, hidden] on x's device")
        need = self.workspace_bytes(d, hidden)
        if workspace is None:
            key = (x.device, torch.cuda.current_stream(x.device).cuda_stream, d, hidden)
            workspace = self._ws.get(key)
            if workspace is None:
                workspace = self._ws[key] = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
        elif workspace.numel() * workspace.element_size() < need or workspace.device != x.device:
            raise ValueError("workspace too small or on another device")
        _check(lib().hag_seq_lstm_forward(self._h, d, hidden, _dev_ptr(x), _dev_ptr(w_ih), _dev_ptr(w_hh), _dev_ptr(b),
                                          _dev_ptr(out), _dev_ptr(workspace), _stream_ptr()))
        return out
