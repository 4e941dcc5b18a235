"""MI355X library for synchronous model averaging (SMA) of k learners on one GPU.

A thin ctypes binding over ``libcrossbow_sma.so`` whose C ABI is declared in
``include/crossbow_sma.h``.  The functions keep the C names (``cb_create``,
``cb_step``, ``cb_sync``, ``cb_get_central`` ...); they only marshal
arguments.  Every step of the computation runs in the HIP kernels of the
library.  torch supplies the device memory (the workspace, images, labels)
and the stream.

Importing this package does not need a GPU; calling into the library does.
If the shared library has not been built the import of the native symbols
raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcrossbow_sma.so")

CB_OK, CB_EINVAL, CB_ENOMEM, CB_EDEVICE, CB_ESTATE, CB_ENONFINITE = 0, -1, -2, -3, -4, -5
ARCH = {"lenet5": 1, "resnet32": 2, "resnet50": 3}
KIND_NAMES = {0: "conv_w", 1: "bias", 2: "bn_gamma", 3: "bn_beta", 4: "fc_w"}

# The interface version these bindings are written for (CB_ABI_VERSION in
# include/crossbow_sma.h); a library built from other sources is refused.
ABI_VERSION = 4

# every symbol the header declares
EXPORTS = (
    "cb_abi_version", "cb_local_apply", "cb_test_conv_static", "cb_test_conv_fwd_parts", "cb_test_head_ok",
    "cb_test_head", "cb_num_params", "cb_num_tensors", "cb_tensor_info", "cb_workspace_bytes", "cb_create",
    "cb_step", "cb_sync", "cb_wait", "cb_get_central", "cb_get_replica", "cb_get_prev_central",
    "cb_get_grad", "cb_get_loss", "cb_sma_apply", "cb_set_state", "cb_last_error", "cb_destroy",
    "cb_profile_enable", "cb_profile_collect", "cb_profile_entry", "cb_profile_clear",
    "cb_test_conv_scratch_bytes", "cb_test_conv", "cb_test_bn_scratch_bytes", "cb_test_bn_fwd",
    "cb_test_bn_bwd", "cb_test_maxpool", "cb_test_softmax_xent",
    "cb_set_lr", "cb_restart", "cb_set_learners", "cb_learners", "cb_tuner_next",
    "cb_test_conv_dgrad_parts", "cb_test_conv_dgrad", "cb_set_graphs", "cb_test_conv_by_pointer",
    "cb_test_conv_pointers", "cb_test_conv_dgrad_pointers", "cb_test_conv_kernel",
    "cb_test_bn_fwd_two", "cb_test_bn_bwd_two",
    "cb_vocab_xent_workspace_bytes", "cb_vocab_xent_fwd", "cb_vocab_xent_bwd",
    "cb_gated_norm_workspace_bytes", "cb_gated_norm_fwd", "cb_gated_norm_bwd",
    "cb_ckpt_bytes", "cb_ckpt_pack", "cb_ckpt_unpack", "cb_ckpt_wgrad_workspace_bytes",
    "cb_ckpt_wgrad",
)


class CBError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{msg} (code {code})")
        self.code = code


class cb_model(ctypes.Structure):
    _fields_ = [("arch", ctypes.c_int32), ("in_c", ctypes.c_int32), ("in_h", ctypes.c_int32),
                ("in_w", ctypes.c_int32), ("num_classes", ctypes.c_int32),
                ("learner_momentum", ctypes.c_float), ("check_finite", ctypes.c_int32)]


class cb_vocab_xent(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("k", ctypes.c_int32), ("n", ctypes.c_int32),
                ("d", ctypes.c_int32), ("v", ctypes.c_int32), ("ignore", ctypes.c_int32),
                ("h", ctypes.c_void_p), ("ldh", ctypes.c_int64), ("w", ctypes.c_void_p),
                ("pstride", ctypes.c_int64), ("labels", ctypes.c_void_p)]


class cb_gated_norm(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("k", ctypes.c_int32), ("n", ctypes.c_int32),
                ("d", ctypes.c_int32), ("gate_rows", ctypes.c_int32),
                ("res_scale", ctypes.c_float), ("eps", ctypes.c_float),
                ("block", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("post", ctypes.c_void_p),
                ("pre", ctypes.c_void_p), ("post_stride", ctypes.c_int64),
                ("pre_stride", ctypes.c_int64)]


_lib = None
_P = ctypes.c_void_p


def check_abi(L, path):
    """Raises ImportError unless the loaded library L reports ABI_VERSION."""
    try:
        fn = L.cb_abi_version
    except AttributeError:
        raise ImportError(f"{path} predates interface version {ABI_VERSION} (no cb_abi_version): "
                          "rebuild it with `python -m paper_1901_02244_amd.build`") from None
    fn.restype = ctypes.c_int
    fn.argtypes = []
    v = fn()
    if v != ABI_VERSION:
        raise ImportError(f"{path} implements interface version {v}, these bindings version "
                          f"{ABI_VERSION}: rebuild it with `python -m paper_1901_02244_amd.build`")


def lib():
    """The loaded library; raises if it is missing (build it first) or was
    built from other sources than these bindings."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_1901_02244_amd.build` "
                              "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        check_abi(L, LIB_PATH)
        L.cb_num_params.restype = ctypes.c_int64
        L.cb_num_params.argtypes = [_P]
        L.cb_num_tensors.argtypes = [_P]
        L.cb_tensor_info.argtypes = [_P, ctypes.c_int, _P, _P, _P, _P]
        L.cb_workspace_bytes.restype = ctypes.c_size_t
        L.cb_workspace_bytes.argtypes = [_P, ctypes.c_int, ctypes.c_int]
        L.cb_create.argtypes = [_P, ctypes.c_int, ctypes.c_int, ctypes.c_float, ctypes.c_float,
                                ctypes.c_float, _P, ctypes.c_int64, _P, ctypes.c_size_t, _P, _P]
        L.cb_step.argtypes = [_P, _P, _P]
        for n in ("cb_sync", "cb_wait"):
            getattr(L, n).argtypes = [_P]
        for n in ("cb_get_central", "cb_get_prev_central"):
            getattr(L, n).argtypes = [_P, _P, ctypes.c_int64]
        for n in ("cb_get_replica", "cb_get_grad"):
            getattr(L, n).argtypes = [_P, ctypes.c_int, _P, ctypes.c_int64]
        L.cb_get_loss.argtypes = [_P, _P]
        L.cb_sma_apply.argtypes = [_P, _P]
        L.cb_local_apply.argtypes = [_P, _P]
        L.cb_set_state.argtypes = [_P, _P, _P, _P]
        L.cb_last_error.restype = ctypes.c_char_p
        L.cb_last_error.argtypes = [_P]
        L.cb_destroy.argtypes = [_P]
        L.cb_destroy.restype = None
        L.cb_profile_enable.argtypes = [_P, ctypes.c_int]
        L.cb_profile_collect.argtypes = [_P]
        L.cb_profile_entry.argtypes = [_P, ctypes.c_int, _P, _P, _P, _P, _P]
        L.cb_profile_clear.argtypes = [_P]
        _i = ctypes.c_int
        L.cb_test_conv_scratch_bytes.restype = ctypes.c_size_t
        L.cb_test_conv_scratch_bytes.argtypes = [_i] * 9
        L.cb_test_conv_fwd_parts.argtypes = [_i] * 9
        L.cb_test_conv.argtypes = [_i] * 11 + [_P, _P, ctypes.c_int64, _P, _P, _P, _P, _P, _P,
                                               ctypes.c_size_t, _P]
        L.cb_test_conv_pointers.argtypes = L.cb_test_conv.argtypes
        L.cb_test_conv_by_pointer.argtypes = [_i] * 10
        L.cb_test_conv_kernel.argtypes = [_i]
        L.cb_test_conv_kernel.restype = ctypes.c_char_p
        L.cb_test_conv_static.argtypes = [_i] * 11 + [_P, _P, ctypes.c_int64, _P, _P, _P, _P,
                                                      _P, _P]
        L.cb_test_head_ok.argtypes = [_i] * 4
        L.cb_test_head.argtypes = [_i] * 6 + [_P, _P, ctypes.c_int64, _P, _P, _P, _P, _P, _P, _P,
                                              _P, _i, _P, _P]
        L.cb_test_bn_scratch_bytes.restype = ctypes.c_size_t
        L.cb_test_bn_scratch_bytes.argtypes = [_i] * 5
        L.cb_test_bn_fwd.argtypes = [_i] * 6 + [_P, _P, ctypes.c_int64, _P, _P, _P, _P,
                                                ctypes.c_size_t, _P]
        L.cb_test_bn_bwd.argtypes = [_i] * 5 + [_P, _P, _i, _P, _P, ctypes.c_int64, _P, _P, _P,
                                                _P, _P, ctypes.c_size_t, _P]
        L.cb_test_bn_fwd_two.argtypes = L.cb_test_bn_fwd.argtypes
        L.cb_test_bn_bwd_two.argtypes = L.cb_test_bn_bwd.argtypes
        L.cb_test_maxpool.argtypes = [_i] * 7 + [_P, _P, _P, _P, _i, _P, _P]
        L.cb_test_softmax_xent.argtypes = [_i] * 3 + [_P, _P, _P, _P, _P]
        L.cb_test_conv_dgrad_parts.argtypes = [_i] * 9
        L.cb_test_conv_dgrad.argtypes = [_i] * 9 + [_P, _P, ctypes.c_int64, _P, _i, _P, _P, _i, _i,
                                                    _P, _P, _P, _P, _P, _P, _P]
        L.cb_test_conv_dgrad_pointers.argtypes = L.cb_test_conv_dgrad.argtypes
        L.cb_set_lr.argtypes = [_P, ctypes.c_float]
        L.cb_restart.argtypes = [_P]
        L.cb_set_learners.argtypes = [_P, _i, ctypes.c_float]
        L.cb_learners.argtypes = [_P]
        L.cb_set_graphs.argtypes = [_P, _i]
        L.cb_tuner_next.argtypes = [_i, ctypes.c_double, ctypes.c_double, ctypes.c_double, _i]
        _z, _q = ctypes.c_size_t, ctypes.c_int64
        L.cb_vocab_xent_workspace_bytes.restype = _z
        L.cb_vocab_xent_workspace_bytes.argtypes = [_P, _i]
        L.cb_vocab_xent_fwd.argtypes = [_P] * 4 + [_z, _P]
        L.cb_vocab_xent_bwd.argtypes = [_P, _P, ctypes.c_float, _P, _P, _q, _P, _z, _P]
        L.cb_gated_norm_workspace_bytes.restype = _z
        L.cb_gated_norm_workspace_bytes.argtypes = [_P]
        L.cb_gated_norm_fwd.argtypes = [_P] * 6
        L.cb_gated_norm_bwd.argtypes = [_P] * 8 + [_q, _P, _q, _P, _z, _P]
        L.cb_ckpt_bytes.restype = _z
        L.cb_ckpt_bytes.argtypes = [_q, _i]
        L.cb_ckpt_pack.argtypes = [_i, _q, _i, _P, _P, _P]
        L.cb_ckpt_unpack.argtypes = [_i, _q, _i, _P, _P, _P]
        L.cb_ckpt_wgrad_workspace_bytes.restype = _z
        L.cb_ckpt_wgrad_workspace_bytes.argtypes = [_i] * 5 + [_P]
        L.cb_ckpt_wgrad.argtypes = [_i] * 5 + [_P, _P, _P, _q, _P, _z, _P]
        _lib = L
    return _lib


def model(arch: str, in_c: int, in_h: int, in_w: int, num_classes: int,
          learner_momentum: float = 0.0, check_finite: bool = False) -> cb_model:
    return cb_model(ARCH[arch], in_c, in_h, in_w, num_classes, learner_momentum,
                    1 if check_finite else 0)


def cb_num_params(m: cb_model) -> int:
    n = lib().cb_num_params(ctypes.byref(m))
    if n < 0:
        raise CBError(n, "unsupported model")
    return int(n)


def cb_tuner_next(l: int, t: float, t_prev: float, threshold: float, l_max: int) -> int:
    """Algorithm 2, one observation (the library's decision rule)."""
    return int(lib().cb_tuner_next(l, t, t_prev, threshold, l_max))


def cb_tensor_layout(m: cb_model):
    """[(offset, kind, shape)] for every parameter tensor, in order."""
    L = lib()
    out = []
    for i in range(L.cb_num_tensors(ctypes.byref(m))):
        off, kind, nd = ctypes.c_int64(), ctypes.c_int(), ctypes.c_int()
        dims = (ctypes.c_int * 4)()
        rc = L.cb_tensor_info(ctypes.byref(m), i, ctypes.byref(off), ctypes.byref(kind),
                              ctypes.byref(nd), dims)
        if rc:
            raise CBError(rc, "cb_tensor_info")
        out.append((off.value, KIND_NAMES[kind.value], tuple(dims[: nd.value])))
    return out


def cb_workspace_bytes(m: cb_model, k: int, b: int) -> int:
    return int(lib().cb_workspace_bytes(ctypes.byref(m), k, b))


def _host_f32(a):
    return np.ascontiguousarray(a, dtype=np.float32)


class Context:
    """One SMA job: k learners of batch b on the current GPU.

    The workspace is one torch uint8 tensor on the device; the stream is
    torch's current stream unless one is given."""

    def __init__(self, m: cb_model, k: int, b: int, alpha: float, lr: float, momentum: float,
                 w0, stream=None):
        import torch

        L = lib()
        self.m, self.k, self.b = m, k, b
        self.capacity = k
        self.P = cb_num_params(m)
        w0 = _host_f32(w0)
        if w0.size != self.P:
            raise CBError(CB_EINVAL, f"w0 has {w0.size} elements, the model has {self.P}")
        nbytes = cb_workspace_bytes(m, k, b)
        if nbytes == 0:
            raise CBError(CB_EINVAL, "cb_workspace_bytes rejected the model, k or b")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._c = ctypes.c_void_p()
        rc = L.cb_create(ctypes.byref(m), k, b, alpha, lr, momentum, w0.ctypes.data, self.P,
                         self.workspace.data_ptr(), nbytes, ctypes.c_void_p(self.stream.cuda_stream),
                         ctypes.byref(self._c))
        if rc:
            raise CBError(rc, "cb_create: " + L.cb_last_error(None).decode())

    # -- errors -----------------------------------------------------------
    def _check(self, rc, what):
        if rc:
            raise CBError(rc, f"{what}: " + lib().cb_last_error(self._c).decode())
        return rc

    def close(self):
        # at interpreter exit the module globals may already be gone
        if getattr(self, "_c", None) and _lib is not None:
            _lib.cb_destroy(self._c)
        self._c = None

    __del__ = close

    # -- the method -------------------------------------------------------
    def cb_step(self, x, y):
        """x: cuda float32 [k*b][C][H][W] contiguous, y: cuda int32 [k*b]."""
        assert x.is_cuda and y.is_cuda and x.is_contiguous() and y.is_contiguous()
        assert x.dtype.is_floating_point and x.element_size() == 4 and y.element_size() == 4
        assert x.shape[0] == self.k * self.b and y.shape[0] == self.k * self.b
        assert tuple(x.shape[1:]) == (self.m.in_c, self.m.in_h, self.m.in_w)
        return self._check(lib().cb_step(self._c, x.data_ptr(), y.data_ptr()), "cb_step")

    def cb_sync(self):
        return self._check(lib().cb_sync(self._c), "cb_sync")

    def cb_wait(self):
        return self._check(lib().cb_wait(self._c), "cb_wait")

    # -- control between iterations -----------------------------------------
    def cb_set_lr(self, lr):
        return self._check(lib().cb_set_lr(self._c, lr), "cb_set_lr")

    def cb_restart(self):
        return self._check(lib().cb_restart(self._c), "cb_restart")

    def cb_set_learners(self, k, alpha):
        self._check(lib().cb_set_learners(self._c, k, alpha), "cb_set_learners")
        self.k = lib().cb_learners(self._c)
        return 0

    def cb_set_graphs(self, on=True):
        """Replay each step's launches as a HIP graph per input buffer pair."""
        return self._check(lib().cb_set_graphs(self._c, 1 if on else 0), "cb_set_graphs")

    def cb_get_central(self):
        out = np.empty(self.P, dtype=np.float32)
        self._check(lib().cb_get_central(self._c, out.ctypes.data, self.P), "cb_get_central")
        return out

    # -- test hooks -------------------------------------------------------
    def cb_get_prev_central(self):
        out = np.empty(self.P, dtype=np.float32)
        self._check(lib().cb_get_prev_central(self._c, out.ctypes.data, self.P),
                    "cb_get_prev_central")
        return out

    def cb_get_replica(self, j):
        out = np.empty(self.P, dtype=np.float32)
        self._check(lib().cb_get_replica(self._c, j, out.ctypes.data, self.P), "cb_get_replica")
        return out

    def cb_get_grad(self, j):
        out = np.empty(self.P, dtype=np.float32)
        self._check(lib().cb_get_grad(self._c, j, out.ctypes.data, self.P), "cb_get_grad")
        return out

    def cb_get_loss(self):
        out = np.empty(self.k, dtype=np.float32)
        self._check(lib().cb_get_loss(self._c, out.ctypes.data), "cb_get_loss")
        return out

    def cb_sma_apply(self, grads):
        """grads: cuda float32 [k][P] contiguous raw gradients."""
        assert grads.is_cuda and grads.is_contiguous() and grads.numel() == self.k * self.P
        return self._check(lib().cb_sma_apply(self._c, grads.data_ptr()), "cb_sma_apply")

    def cb_local_apply(self, grads):
        """A local step (no correction) with grads: cuda float32 [k][P]."""
        assert grads.is_cuda and grads.is_contiguous() and grads.numel() == self.k * self.P
        return self._check(lib().cb_local_apply(self._c, grads.data_ptr()), "cb_local_apply")

    # -- instrumentation --------------------------------------------------
    def cb_profile_enable(self, on=True):
        return self._check(lib().cb_profile_enable(self._c, 1 if on else 0), "cb_profile_enable")

    def cb_profile(self):
        """{kernel name: (launches, ms, flops, bytes)} accumulated so far."""
        L = lib()
        n = L.cb_profile_collect(self._c)
        self._check(min(n, 0), "cb_profile_collect")
        out = {}
        for i in range(n):
            name = ctypes.c_char_p()
            la, ms, fl, by = ctypes.c_int64(), ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
            self._check(L.cb_profile_entry(self._c, i, ctypes.byref(name), ctypes.byref(la),
                                           ctypes.byref(ms), ctypes.byref(fl), ctypes.byref(by)),
                        "cb_profile_entry")
            out[name.value.decode()] = (la.value, ms.value, fl.value, by.value)
        return out

    def cb_profile_clear(self):
        return self._check(lib().cb_profile_clear(self._c), "cb_profile_clear")

    def cb_set_state(self, W, z, zprev):
        W, z, zprev = _host_f32(W), _host_f32(z), _host_f32(zprev)
        assert W.size == self.k * self.P and z.size == self.P and zprev.size == self.P
        return self._check(lib().cb_set_state(self._c, W.ctypes.data, z.ctypes.data,
                                              zprev.ctypes.data), "cb_set_state")


# --- operators for language-model learners -------------------------------------
# Tensors of k learners: activations [k, n, width], parameters and gradients with
# the learner as their first dimension, which may be strided (a slice of a flat
# [k, P] vector).  Outputs are allocated on the inputs' device; the work goes to
# `stream`, or to torch's current stream of that device.  `stream` waits for nothing by
# itself: the caller has it wait for the inputs, and waits for it before using the
# outputs.  A workspace is a uint8 tensor that the caller keeps; without one each call
# takes its own from torch's allocator.

def _refuse(who, why):
    raise CBError(CB_EINVAL, f"{who}: {why}")


_torch = None          # torch, and what every call needs of it, after the first call
_type_codes = {}
_F32 = _I32 = _U8 = None


def _type_code(who, dtype):
    code = _type_codes.get(dtype)
    if code is None:
        global _torch, _F32, _I32, _U8
        import torch

        _torch, _F32, _I32, _U8 = torch, torch.float32, torch.int32, torch.uint8
        _type_codes.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
        code = _type_codes.get(dtype)
        if code is None:
            _refuse(who, f"{dtype} is none of float32, float16, bfloat16")
    return code


# Sizes are 32-bit numbers in the library, and ctypes would cut larger ones off:
# (a | b | c) >> 31 is 0 where none of them is negative or takes more.
_PAST = "a size or label past 32 bits"


def _need(who, name, t, shape, dtype, device, outer=False):
    """Checks one tensor: its shape, type, device, and that it is contiguous (with
    `outer`: apart from the stride of its first dimension)."""
    if t.shape == shape and t.dtype is dtype and t.device == device and t.is_cuda \
            and t.is_contiguous():
        return
    if t.shape != tuple(shape):
        _refuse(who, f"{name} is {tuple(t.shape)}, not {tuple(shape)}")
    if t.dtype != dtype:
        _refuse(who, f"{name} is {t.dtype}, not {dtype}")
    if not t.is_cuda or t.device != device:
        _refuse(who, f"{name} is on {t.device}, not on {device}, or not on a GPU")
    if not t.is_contiguous() and not (outer and t.dim() > 1 and t.numel()
                                      and t[0].is_contiguous()):
        _refuse(who, f"{name} is not contiguous" + (" within a learner" if outer else ""))


def _outer(t):
    """Elements from one learner to the next."""
    return t.stride(0) if t.shape[0] > 1 else t.numel()


def _begin(who, stream, t, *more):
    """Makes the device of t current, and `stream` if one is given, so that new tensors
    are that stream's memory: a block of another stream's may have been freed while
    work queued there still reads it.  For the same reason t and the call's other
    tensors (or None) are marked as used on that stream.  Returns the handle of the
    call's stream, what was torch's current stream (where results are used next, which
    the allocator has to know) if it was another one or None, and the device to return
    to or -1."""
    cuda, index = _torch.cuda, t.get_device()
    if stream is not None and stream.device_index != index:
        _refuse(who, f"the stream is not one of {t.device}")
    handle, before = _current_stream(index), None
    if stream is not None and stream.cuda_stream != handle:
        for used in (t, *more):
            if used is not None:
                used.record_stream(stream)
        handle, before = stream.cuda_stream, cuda.current_stream(index)
    back = cuda.current_device()
    if back != index:
        cuda.set_device(index)
    else:
        back = -1
    if before is not None:
        cuda.set_stream(stream)
    return handle, before, back


def _end(before, back):
    if before is not None:
        _torch.cuda.set_stream(before)
    if back >= 0:
        _torch.cuda.set_device(back)


def _current_stream(index):
    """The handle of torch's current stream of a device (the stream object itself
    takes microseconds to make)."""
    raw = getattr(_torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else _torch.cuda.current_stream(index).cuda_stream


def _like(t, before):
    n = _torch.empty_like(t)
    if before is not None:
        n.record_stream(before)
    return n


def _new(t, shape, dtype, before):
    n = t.new_empty(shape, dtype=dtype)
    if before is not None:
        n.record_stream(before)
    return n


def _check_workspace(who, t, given):
    if given is not None and (given.dtype != _U8 or not given.is_contiguous()
                              or given.device != t.device):
        _refuse(who, "the workspace is not a contiguous uint8 tensor on the inputs' device")


def _workspace(t, nbytes, given):
    return _new(t, (nbytes or 1,), _U8, None) if given is None else given


def _check(who, rc):
    if rc:
        raise CBError(rc, lib().cb_last_error(None).decode() or who)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _xent(who, h, w, labels, ignore):
    code = _type_code(who, h.dtype)
    if h.dim() != 3 or w.dim() != 3:
        _refuse(who, "h is [k, n, d] and w [k, v, d]")
    k, n, d = h.shape
    v = w.shape[1]
    if (k | n | d | v) >> 31 or not -2**31 <= ignore < 2**31:
        _refuse(who, _PAST)
    if not h.is_cuda:
        _refuse(who, "h is not on a GPU")
    if min(k, n, d, v) < 1:
        _refuse(who, "an empty dimension")
    ldh = d
    if not h.is_contiguous():
        # rows may lie further apart than d, the same for all learners
        ldh = h.stride(1) if n > 1 else h.stride(0) if k > 1 else d
        if (d > 1 and h.stride(2) != 1) or ldh < d or (k > 1 and h.stride(0) != n * ldh):
            _refuse(who, "h is not rows at one stride")
    dev = h.device
    _need(who, "w", w, (k, v, d), h.dtype, dev, outer=True)
    _need(who, "labels", labels, (k, n), _I32, dev)
    return cb_vocab_xent(code, k, n, d, v, ignore, h.data_ptr(), ldh, w.data_ptr(), _outer(w),
                         labels.data_ptr())


def cb_vocab_xent_fwd(h, w, labels, ignore=-100, workspace=None, stream=None):
    """Softmax cross-entropy of the logits h W^T over a large vocabulary, without
    storing them.  h [k, n, d] and w [k, v, d] of one type (float32, float16,
    bfloat16), labels int32 [k, n]; rows labelled `ignore` do not count.

    Returns (loss [k], lse [k, n]) in float32: each learner's mean over its counted
    rows (0 if none counts) and the rows' log-sum-exp, which the backward takes."""
    who = "cb_vocab_xent_fwd"
    L = lib()
    x = _xent(who, h, w, labels, ignore)
    r = ctypes.byref(x)
    _check_workspace(who, h, workspace)
    handle, before, back = _begin(who, stream, h, w, labels, workspace)
    try:
        loss, lse = _new(h, (x.k,), _F32, before), _new(h, (x.k, x.n), _F32, before)
        ws = _workspace(h, L.cb_vocab_xent_workspace_bytes(r, 0), workspace)
        _check(who, L.cb_vocab_xent_fwd(r, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(),
                                        ws.numel(), handle))
    finally:
        _end(before, back)
    return loss, lse


def cb_vocab_xent_bwd(h, w, labels, lse, grad_scale=1.0, ignore=-100, dw=None, workspace=None,
                      stream=None):
    """The gradients of grad_scale * loss of cb_vocab_xent_fwd, given its lse:
    (dh [k, n, d], dw [k, v, d]) in the inputs' type, which also holds the logits'
    gradients on the way.  dw may be given, for instance as a view of a flat gradient
    vector; it is overwritten."""
    who = "cb_vocab_xent_bwd"
    L = lib()
    x = _xent(who, h, w, labels, ignore)
    r = ctypes.byref(x)
    _need(who, "lse", lse, (x.k, x.n), _F32, h.device)
    if dw is not None:
        _need(who, "dw", dw, (x.k, x.v, x.d), h.dtype, h.device, outer=True)
    _check_workspace(who, h, workspace)
    handle, before, back = _begin(who, stream, h, w, labels, lse, dw, workspace)
    try:
        dh = _new(h, (x.k, x.n, x.d), h.dtype, before)
        if dw is None:
            dw = _new(h, (x.k, x.v, x.d), h.dtype, before)
        ws = _workspace(h, L.cb_vocab_xent_workspace_bytes(r, 1), workspace)
        _check(who, L.cb_vocab_xent_bwd(r, lse.data_ptr(), grad_scale, dh.data_ptr(),
                                        dw.data_ptr(), _outer(dw), ws.data_ptr(), ws.numel(),
                                        handle))
    finally:
        _end(before, back)
    return dh, dw


def _norm(who, x, block, gate, gate_rows, res_scale, post, pre, eps):
    dtype, shape, dev = x.dtype, x.shape, x.device
    code = _type_code(who, dtype)
    if len(shape) != 3 or min(shape) < 1:
        _refuse(who, "x is [k, n, d], none of them 0")
    k, n, d = shape
    if (k | n | d) >> 31:
        _refuse(who, _PAST)
    _need(who, "x", x, shape, dtype, dev)
    if block is not None:
        _need(who, "block", block, shape, dtype, dev)
    if gate is not None:
        if not 1 <= gate_rows < 2**31:
            _refuse(who, "gate_rows is out of range")
        _need(who, "gate", gate, (k, -(-n // gate_rows), d), dtype, dev)
    if post is not None:
        _need(who, "post", post, (k, d), _F32, dev, outer=True)
    if pre is not None:
        _need(who, "pre", pre, (k, d), _F32, dev, outer=True)
    return cb_gated_norm(code, k, n, d, gate_rows if gate is not None else 1, res_scale, eps,
                         _ptr(block), _ptr(gate), _ptr(post), _ptr(pre),
                         _outer(post) if post is not None else 0,
                         _outer(pre) if pre is not None else 0)


def cb_gated_norm_fwd(x, block=None, gate=None, gate_rows=1, res_scale=1.0, post=None, pre=None,
                      eps=1e-5, keep=False, stream=None):
    """The norm after a block, its gate and residual scale, the addition to the
    residual stream, and the norm before the next block, in one pass:

        x_out = x + res_scale * gate * (post * rms(block));  y = pre * rms(x_out)

    x, block [k, n, d] and gate [k, ceil(n/gate_rows), d] of one type, post and pre
    float32 [k, d]; each of block, gate, post and pre may be None.

    Returns (x_out, y), x_out being x without a block and y None without pre; with
    keep also y in 8 bits, as cb_ckpt_pack gives it."""
    who = "cb_gated_norm_fwd"
    L = lib()
    g = _norm(who, x, block, gate, gate_rows, res_scale, post, pre, eps)
    if keep and pre is None:
        _refuse(who, "keep without pre")
    handle, before, back = _begin(who, stream, x, block, gate, post, pre)
    try:
        xo = _like(x, before) if block is not None else x
        y = _like(x, before) if pre is not None else None
        kept = _new_kept(x, before) if keep else None
        _check(who, L.cb_gated_norm_fwd(ctypes.byref(g), x.data_ptr(), xo.data_ptr(), _ptr(y),
                                        kept.data.data_ptr() if keep else None, handle))
    finally:
        _end(before, back)
    return (xo, y, kept) if keep else (xo, y)


def cb_gated_norm_bwd(x_out, dy=None, dres=None, block=None, gate=None, gate_rows=1, res_scale=1.0,
                      post=None, pre=None, eps=1e-5, dpost=None, dpre=None, workspace=None,
                      stream=None):
    """Backward of cb_gated_norm_fwd, given its x_out, the gradient dy at y (with
    pre) and the gradient dres that reaches x_out along the stream (or None).

    Returns a dict: dx, and where their parts are there dblock, dgate (summed over
    the rows that share a gate row), dpost, dpre (float32 [k, d]; may be given as
    views of a flat gradient vector, and are overwritten)."""
    who = "cb_gated_norm_bwd"
    L = lib()
    g = _norm(who, x_out, block, gate, gate_rows, res_scale, post, pre, eps)
    r = ctypes.byref(g)
    if (dy is None) != (pre is None):
        _refuse(who, "dy goes with pre")
    if dy is not None:
        _need(who, "dy", dy, x_out.shape, x_out.dtype, x_out.device)
    if dres is not None:
        _need(who, "dres", dres, x_out.shape, x_out.dtype, x_out.device)
    for name, t, of in (("dpost", dpost, post), ("dpre", dpre, pre)):
        if t is not None:
            if of is None:
                _refuse(who, f"{name} without its gamma")
            _need(who, name, t, (g.k, g.d), _F32, x_out.device, outer=True)
    _check_workspace(who, x_out, workspace)
    handle, before, back = _begin(who, stream, x_out, dy, dres, block, gate, post, pre, dpost,
                                  dpre, workspace)
    try:
        dx = _like(x_out, before)
        dblock = dgate = None
        if block is not None:
            dblock = _like(block, before)
        if gate is not None:
            dgate = _like(gate, before)
        if post is not None and dpost is None:
            dpost = _new(post, (g.k, g.d), _F32, before)
        if pre is not None and dpre is None:
            dpre = _new(pre, (g.k, g.d), _F32, before)
        ws = _workspace(x_out, L.cb_gated_norm_workspace_bytes(r), workspace)
        _check(who, L.cb_gated_norm_bwd(
            r, x_out.data_ptr(), _ptr(dy), _ptr(dres), dx.data_ptr(), _ptr(dblock), _ptr(dgate),
            _ptr(dpost), _outer(dpost) if dpost is not None else 0, _ptr(dpre),
            _outer(dpre) if dpre is not None else 0, ws.data_ptr(), ws.numel(), handle))
    finally:
        _end(before, back)
    out = {"dx": dx, "dblock": dblock, "dgate": dgate, "dpost": dpost, "dpre": dpre}
    return {name: t for name, t in out.items() if t is not None}


class Kept:
    """Activations [k, n, d] of `dtype` in 8 bits: `data` is the library's buffer."""

    __slots__ = ("data", "shape", "dtype")

    def __init__(self, data, shape, dtype):
        self.data, self.shape, self.dtype = data, tuple(shape), dtype


def _new_kept(x, before):
    k, n, d = x.shape
    nbytes = lib().cb_ckpt_bytes(k * n, d)
    if nbytes == 0:
        _refuse("cb_ckpt_bytes", f"{tuple(x.shape)} is out of range")
    return Kept(_new(x, (nbytes,), _U8, before), x.shape, x.dtype)


def _check_kept(who, kept):
    """The type code of a Kept whose buffer is as long as its shape says."""
    code = _type_code(who, kept.dtype)
    k, n, d = kept.shape
    if (k | n | d) >> 31:
        _refuse(who, _PAST)
    need = lib().cb_ckpt_bytes(k * n, d)
    b = kept.data
    if not b.is_cuda or b.dtype != _U8 or not b.is_contiguous() or need == 0 or b.numel() < need:
        _refuse(who, f"the kept buffer is not {need} bytes on a GPU")
    return code


def cb_ckpt_pack(x, stream=None):
    """x [k, n, d] (float32, float16, bfloat16) in 8 bits a value and a power of two
    for every 32 columns.  Returns a Kept."""
    who = "cb_ckpt_pack"
    code = _type_code(who, x.dtype)
    if x.dim() != 3 or min(x.shape) < 1:
        _refuse(who, "x is [k, n, d], none of them 0")
    k, n, d = x.shape
    if (k | n | d) >> 31:
        _refuse(who, _PAST)
    _need(who, "x", x, x.shape, x.dtype, x.device)
    handle, before, back = _begin(who, stream, x)
    try:
        kept = _new_kept(x, before)
        _check(who, lib().cb_ckpt_pack(code, k * n, d, x.data_ptr(), kept.data.data_ptr(), handle))
    finally:
        _end(before, back)
    return kept


def cb_ckpt_unpack(kept, stream=None):
    """The values that `kept` stands for, [k, n, d] in its type."""
    who = "cb_ckpt_unpack"
    code = _check_kept(who, kept)
    k, n, d = kept.shape
    handle, before, back = _begin(who, stream, kept.data)
    try:
        x = _new(kept.data, kept.shape, kept.dtype, before)
        _check(who, lib().cb_ckpt_unpack(code, k * n, d, kept.data.data_ptr(), x.data_ptr(),
                                         handle))
    finally:
        _end(before, back)
    return x


def cb_ckpt_wgrad(kept, dy, dw=None, workspace=None, stream=None):
    """The weight gradient of a linear layer whose input [k, n, d] was kept in 8
    bits: dw [k, out, d] = dy^T x for dy [k, n, out] of the same type.  dw may be
    given, for instance as a view of a flat gradient vector; it is overwritten."""
    who = "cb_ckpt_wgrad"
    if dy.dim() != 3 or dy.shape[2] < 1:
        _refuse(who, "dy is [k, n, out]")
    out = dy.shape[2]
    if out >> 31:
        _refuse(who, _PAST)
    code = _check_kept(who, kept)
    k, n, d = kept.shape
    _need(who, "dy", dy, (k, n, out), kept.dtype, kept.data.device)
    if dw is not None:
        _need(who, "dw", dw, (k, out, d), kept.dtype, dy.device, outer=True)
    L = lib()
    _check_workspace(who, dy, workspace)
    handle, before, back = _begin(who, stream, dy, kept.data, dw, workspace)
    try:
        if dw is None:
            dw = _new(dy, (k, out, d), kept.dtype, before)
        need = L.cb_ckpt_wgrad_workspace_bytes(code, k, n, d, out, dy.data_ptr())
        ws = _workspace(dy, need, workspace)
        _check(who, L.cb_ckpt_wgrad(code, k, n, d, out, kept.data.data_ptr(), dy.data_ptr(),
                                    dw.data_ptr(), _outer(dw), ws.data_ptr(), ws.numel(), handle))
    finally:
        _end(before, back)
    return dw
