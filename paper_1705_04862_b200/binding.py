"""Thin ctypes binding of libpaac_b200.so: argument marshalling only.

Every step of the PAAC iteration runs in the library's CUDA kernels; this module
allocates nothing but host result buffers and (through torch) the device workspace.
If the shared library is missing or cannot be loaded the import of `lib()` raises:
there is no other implementation to fall back to.
"""
import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpaac_b200.so")

ARCH_NIPS, ARCH_NATURE = 0, 1
FP32, BF16 = 0, 1
ALGO_A2C, ALGO_NSTEP_Q = 0, 1
ENV_HASHED, ENV_PATTERN = 0, 1
SCAN_LINEAR, SCAN_SIGMOID = 0, 1
SELECTIVE_SPAN = 16
ACT_NONE, ACT_RELU, ACT_SILU = 0, 1, 2
OK, ERR_ARG, ERR_WORKSPACE, ERR_CUDA, ERR_NONFINITE, ERR_TIMEOUT, ERR_STATE, ERR_LIMIT, ERR_RANGE = range(9)
(DBG_FRAMES, DBG_NEXT_FRAMES, DBG_ACTIONS, DBG_REWARDS, DBG_TERMINALS, DBG_VALUES, DBG_LOGITS, DBG_UNIFORMS,
 DBG_COUNTERS, DBG_RETURNS, DBG_ADVANTAGES, DBG_DLOGITS, DBG_DVALUES, DBG_GRAD, DBG_RMS, DBG_SAMPLED,
 DBG_ERROR_WORD) = range(17)
DBG_ACT0, DBG_GACT0 = 32, 48
(OPT_CUDA_CORES_ONLY, OPT_TC_WGRAD_LAYERS, OPT_CUDA_GRAPHS, OPT_DEPENDENT_LAUNCH, OPT_FP32_TENSOR_CORES,
 OPT_UPDATE_CHUNKS, OPT_WAIT_POLLS) = 1, 2, 3, 4, 5, 6, 7

_DBG_DTYPE = {DBG_FRAMES: np.uint8, DBG_NEXT_FRAMES: np.uint8, DBG_ACTIONS: np.int32, DBG_REWARDS: np.int8,
              DBG_TERMINALS: np.uint8, DBG_COUNTERS: np.int32, DBG_SAMPLED: np.int32, DBG_ERROR_WORD: np.uint32}


class HParams(C.Structure):
    _fields_ = [("gamma", C.c_float), ("lr", C.c_float), ("rms_decay", C.c_float), ("rms_eps", C.c_float),
                ("clip_norm", C.c_float), ("entropy_beta", C.c_float), ("value_coef", C.c_float),
                ("term_denom", C.c_uint32), ("precision", C.c_int), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p), ("algorithm", C.c_int),
                ("epsilon", C.c_float), ("environment", C.c_int)]


class RolloutView(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("frames", "next_frames", "actions", "rewards", "terminals", "values",
                                          "logits", "uniforms")]


class UpdateStats(C.Structure):
    _fields_ = [("policy_loss", C.c_float), ("value_loss", C.c_float), ("entropy", C.c_float),
                ("grad_norm", C.c_float), ("clip_scale", C.c_float), ("status", C.c_int32),
                ("timesteps", C.c_uint64)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("outer", C.c_int64), ("inner", C.c_int64)]


class Tensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("n", C.c_uint64), ("src_type", C.c_int32), ("dst_type", C.c_int32)]


class Scan(C.Structure):
    _fields_ = [("t", C.c_int32), ("n", C.c_int32), ("c", C.c_int32), ("type", C.c_int32), ("kind", C.c_int32), ("reverse", C.c_int32),
                ("restart", C.c_void_p), ("restart_n", C.c_int64), ("restart_t", C.c_int64)]


class Norm(C.Structure):
    _fields_ = [("n", C.c_int32), ("pixels", C.c_int32), ("c", C.c_int32), ("groups", C.c_int32), ("type", C.c_int32),
                ("activation", C.c_int32), ("eps", C.c_float)]


EXPORTS = ["paac_default_hparams", "paac_workspace_bytes", "paac_init", "paac_rollout", "paac_update",
           "paac_param_count", "paac_params", "paac_destroy", "paac_strerror", "paac_act_host",
           "paac_observe_host", "paac_set_params", "paac_force_actions", "paac_debug_bytes", "paac_debug_read",
           "paac_debug_write", "paac_debug_wait_probe", "paac_preprocess", "paac_stack_push", "paac_act_host_newest", "paac_launch_count", "paac_profile", "paac_profile_read", "paac_set_option", "paac_clip_rmsprop_noalloc",
           "paac_noalloc_max_params", "paac_clip_tensors_workspace_bytes", "paac_clip_tensors", "paac_gated_scan",
           "paac_gated_scan_backward", "paac_group_norm_workspace_bytes", "paac_group_norm", "paac_group_norm_backward", "paac_causal_conv",
           "paac_causal_conv_workspace_bytes", "paac_causal_conv_backward", "paac_selective_scan_workspace_bytes", "paac_selective_scan",
           "paac_selective_scan_backward", "paac_sample"]

_lib = None


def lib():
    """The loaded library; raises OSError if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError("libpaac_b200.so is not built: run `python -m paper_1705_04862_b200.build` "
                          "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i, u64, sz = C.c_void_p, C.c_int, C.c_uint64, C.c_size_t
        L.paac_default_hparams.argtypes = [C.POINTER(HParams)]
        L.paac_default_hparams.restype = None
        L.paac_workspace_bytes.argtypes = [i, i, i, i, C.POINTER(HParams)]
        L.paac_workspace_bytes.restype = sz
        L.paac_init.argtypes = [C.POINTER(vp), i, i, i, i, C.POINTER(HParams), u64]
        L.paac_rollout.argtypes = [vp, C.POINTER(RolloutView)]
        L.paac_update.argtypes = [vp, C.POINTER(UpdateStats)]
        L.paac_param_count.argtypes = [vp]
        L.paac_param_count.restype = sz
        L.paac_params.argtypes = [vp, vp, sz]
        L.paac_destroy.argtypes = [vp]
        L.paac_strerror.argtypes = [i]
        L.paac_strerror.restype = C.c_char_p
        L.paac_act_host.argtypes = [vp, i, vp, vp, vp]
        L.paac_observe_host.argtypes = [vp, i, vp, vp]
        L.paac_set_params.argtypes = [vp, vp, sz]
        L.paac_force_actions.argtypes = [vp, vp]
        L.paac_debug_bytes.argtypes = [vp, i]
        L.paac_debug_bytes.restype = sz
        L.paac_debug_read.argtypes = [vp, i, vp, sz]
        L.paac_debug_write.argtypes = [vp, i, vp, sz]
        L.paac_debug_wait_probe.argtypes = [vp, C.c_uint32]
        L.paac_preprocess.argtypes = [vp, vp, vp, vp, i, vp]
        L.paac_stack_push.argtypes = [vp, vp, vp, vp, i, vp]
        L.paac_act_host_newest.argtypes = [vp, i, vp, vp, vp, vp]
        L.paac_launch_count.argtypes = [vp]
        L.paac_launch_count.restype = u64
        L.paac_profile.argtypes = [vp, i]
        L.paac_set_option.argtypes = [vp, i, i]
        f = C.c_float
        L.paac_clip_rmsprop_noalloc.argtypes = [vp, vp, vp, vp, sz, f, f, f, f, vp, vp]
        L.paac_noalloc_max_params.argtypes = []
        L.paac_noalloc_max_params.restype = sz
        L.paac_clip_tensors_workspace_bytes.argtypes = [sz]
        L.paac_clip_tensors_workspace_bytes.restype = sz
        L.paac_clip_tensors.argtypes = [vp, sz, f, vp, vp, sz, vp]
        L.paac_gated_scan.argtypes = [C.POINTER(Scan), Rows, Rows, vp, Rows, vp, vp]
        L.paac_gated_scan_backward.argtypes = [C.POINTER(Scan), Rows, Rows, Rows, Rows, vp, vp, Rows, Rows, vp, vp]
        L.paac_group_norm_workspace_bytes.argtypes = [C.POINTER(Norm)]
        L.paac_group_norm_workspace_bytes.restype = sz
        L.paac_group_norm.argtypes = [C.POINTER(Norm), Rows, vp, vp, Rows, vp, vp, vp, sz, vp]
        L.paac_group_norm_backward.argtypes = [C.POINTER(Norm), Rows, Rows, vp, vp, vp, vp, Rows, vp, vp, vp, sz, vp]
        L.paac_causal_conv.argtypes = [vp, vp, vp]
        L.paac_causal_conv_workspace_bytes.argtypes = [vp]
        L.paac_causal_conv_workspace_bytes.restype = sz
        L.paac_causal_conv_backward.argtypes = [vp, vp, vp]
        L.paac_selective_scan_workspace_bytes.argtypes = [vp, i]
        L.paac_selective_scan_workspace_bytes.restype = sz
        L.paac_selective_scan.argtypes = [vp, vp, vp]
        L.paac_selective_scan_backward.argtypes = [vp, vp, vp]
        L.paac_sample.argtypes = [vp, vp]
        L.paac_profile_read.argtypes = [vp, i, C.POINTER(C.c_char_p), C.POINTER(C.c_double), C.POINTER(u64)]
        _lib = L
    return _lib


class PaacError(RuntimeError):
    def __init__(self, status):
        self.status = status
        super().__init__("paac: %s (status %d)" % (lib().paac_strerror(status).decode(), status))


def _check(status, allow=()):
    if status != OK and status not in allow:
        raise PaacError(status)
    return status


def default_hparams(**over):
    hp = HParams()
    lib().paac_default_hparams(C.byref(hp))
    for k, v in over.items():
        setattr(hp, k, v)
    return hp


def workspace_bytes(arch, n_e, t_max, n_actions, hp):
    return int(lib().paac_workspace_bytes(arch, n_e, t_max, n_actions, C.byref(hp)))


def _host_ptr(a):
    """Address of a numpy array or a (pinned) CPU torch tensor."""
    if isinstance(a, np.ndarray):
        assert a.flags["C_CONTIGUOUS"]
        return a.ctypes.data
    return a.data_ptr()


def _addr(x):
    """Device address of a torch CUDA tensor or a raw address; None stays None."""
    return x if x is None or isinstance(x, int) else x.data_ptr()


def clip_rmsprop_noalloc(theta, rms, grad, n, lr, rms_decay, rms_eps, clip_norm, theta_bf16=None,
                         norm_and_scale=None, stream=None):
    """Optimiser step on caller-owned device arrays for hosts that may not allocate device memory (see
    paac_clip_rmsprop_noalloc in include/paac.h).  Arguments are torch CUDA tensors (or raw device
    addresses); returns the library status without raising, so callers can test for ERR_LIMIT."""
    return int(lib().paac_clip_rmsprop_noalloc(_addr(theta), _addr(rms), _addr(grad), _addr(theta_bf16), n, lr, rms_decay,
                                               rms_eps, clip_norm, _addr(norm_and_scale), _addr(stream)))


def preprocess(raw_prev, raw_last, state_in, state_out, n, stream=None):
    """Section 5.1 pre-processing on device buffers (torch CUDA uint8 tensors or raw addresses): see paac_preprocess
    in include/paac.h.  Returns the library status."""
    return int(lib().paac_preprocess(_addr(raw_prev), _addr(raw_last), _addr(state_in), _addr(state_out), n, _addr(stream)))


def stack_push(state_in, newest, restart, state_out, n, stream=None):
    """The four-frame stack on device buffers: see paac_stack_push in include/paac.h.  Returns the library status."""
    return int(lib().paac_stack_push(_addr(state_in), _addr(newest), _addr(restart), _addr(state_out), n, _addr(stream)))


# -- operators for networks of the caller's own: torch CUDA tensors in, the library's status out ------------------------
# Tensors that do not go together (type, shape, device, a last axis that is not contiguous) are ERR_ARG.  The work goes to
# `stream` (an address) on the tensors' device, by default torch's current stream there.

_torch, _TYPES, _stream_of, _current = None, {}, None, None


def _with_torch():
    """torch, and the storage types' numbers by its types (asked for at every call, so looked up once)."""
    global _torch, _stream_of, _current
    if _torch is None:
        import torch
        _TYPES.update({torch.float32: FP32, torch.bfloat16: BF16})
        # the current stream's address without an object around it, where this torch has that (0.06 us instead of 2.6)
        _stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        # the current device's number, likewise
        _current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        _torch = torch
    return _torch


def _status(index, stream, call, args):
    """call(*args, stream address) with device `index` current; None = torch's current stream of that device."""
    if stream is None:
        stream = _stream_of(index)
    if _current() == index:
        return call(*args, stream)
    with _torch.cuda.device(index):
        return call(*args, stream)


class _Apart(Exception):
    """Tensors do not go together."""


def _floats(t, index, count):
    """Address of `count` contiguous floats on device `index`, or None."""
    if t is None:
        return None
    if t.dtype is not _torch.float32 or t.get_device() != index or t.numel() != count or not t.is_contiguous():
        raise _Apart
    return t.data_ptr()


class TensorList:
    """The tensors of a network's gradient and where each goes clipped, for clip_tensors: made once, while the tensors stay where
    they are (a microsecond a tensor: 18 us for twelve, 330 for 300, beside calls of 9 and 16; gradients that are new tensors at every
    step need a new list, and that time, at every step).  src: contiguous float32 / bfloat16 CUDA tensors of one device; dst: as
    many of the same sizes, the same ones for clipping in place, None in the place of one (or of all) that only counts for the norm.
    Holds the tensors and the scratch, so calls with one list may not overlap on the GPU, and one that is used on another stream
    than it was made on is kept until those calls have run."""

    def __init__(self, src, dst=None):
        torch, types = _with_torch(), _TYPES
        src = list(src)
        dst = [None] * len(src) if dst is None else list(dst)
        self.device = src[0].device if src else torch.device("cuda", torch.cuda.current_device())
        ok = len(src) == len(dst) and self.device.type == "cuda"
        for t in src + [t for t in dst if t is not None]:
            ok = ok and t.dtype in types and t.device == self.device and t.is_contiguous()
        if not ok or any(d is not None and d.numel() != s.numel() for s, d in zip(src, dst)):
            raise PaacError(ERR_ARG)
        self.tensors = (src, dst)
        self.array = (Tensor * max(1, len(src)))()
        for a, s, d in zip(self.array, src, dst):
            a.src, a.n, a.src_type = s.data_ptr(), s.numel(), types[s.dtype]
            a.dst, a.dst_type = (None, a.src_type) if d is None else (d.data_ptr(), types[d.dtype])
        self.count = len(src)
        need = int(lib().paac_clip_tensors_workspace_bytes(self.count))
        if need == 0:
            raise PaacError(ERR_LIMIT)
        self.workspace = torch.empty(need, dtype=torch.uint8, device=self.device)


def clip_tensors(tensors, clip_norm, norm_and_scale=None, stream=None):
    """The global norm of a TensorList and its clipping: see paac_clip_tensors in include/paac.h."""
    index = tensors.device.index
    try:
        told = _floats(norm_and_scale, index, 2)
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_clip_tensors, (tensors.array, tensors.count, clip_norm, told, tensors.workspace.data_ptr(),
                                                            tensors.workspace.nbytes))


_NO_ROWS = Rows(None, 0, 0)
_MOST = 2 ** 31 - 1             # what an int32 field holds; a larger number would be cut off without a word


def _rows(t, shape, dtype, index, outer, inner):
    """Rows of the last axis along the axes `outer` and `inner` (4 axes: the middle two as one) of a tensor of this shape, type and device."""
    if t is None:
        return _NO_ROWS
    stride = t.stride()
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or (stride[-1] != 1 and shape[-1] > 1):
        raise _Apart
    if len(stride) == 4:
        if shape[1] > 1 and shape[2] > 1 and stride[1] != shape[2] * stride[2]:
            raise _Apart
        inner = 2 if shape[2] > 1 else 1
    return Rows(t.data_ptr(), stride[outer], stride[inner])


def _scan(lead, restart, kind, reverse):
    """(shape, type, device, the scan's own) of a call whose first tensor leads."""
    if _torch is None:
        _with_torch()
    shape, dtype, index = lead.shape, lead.dtype, lead.get_device()
    if len(shape) != 3 or dtype not in _TYPES or index < 0 or max(shape) > _MOST or not 0 <= kind <= _MOST:
        raise _Apart
    t, n, c = shape
    if restart is None:
        return shape, dtype, index, Scan(t, n, c, _TYPES[dtype], kind, 1 if reverse else 0, None, 0, 0)
    if restart.element_size() != 1 or restart.get_device() != index or restart.shape != (t, n):
        raise _Apart
    by_step, by_sequence = restart.stride()
    return shape, dtype, index, Scan(t, n, c, _TYPES[dtype], kind, 1 if reverse else 0, restart.data_ptr(), by_sequence, by_step)


def gated_scan(gate, x, h, h0=None, h_last=None, restart=None, kind=SCAN_SIGMOID, reverse=False, stream=None):
    """The gated linear recurrence: see paac_gated_scan in include/paac.h.  gate, x, h [steps][sequences][channels] with strides of
    their own (the last axis contiguous), h0 and h_last float32 [sequences][channels], restart one byte [steps][sequences]."""
    try:
        shape, dtype, index, s = _scan(gate, restart, kind, reverse)
        states = s.n * s.c
        args = (s, _rows(gate, shape, dtype, index, 1, 0), _rows(x, shape, dtype, index, 1, 0), _floats(h0, index, states),
                _rows(h, shape, dtype, index, 1, 0), _floats(h_last, index, states))
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_gated_scan, args)


def gated_scan_backward(gate, x, h, dh, dgate, dx, h0=None, dh_last=None, dh0=None, restart=None, kind=SCAN_SIGMOID, reverse=False,
                        stream=None):
    """Its gradient: see paac_gated_scan_backward in include/paac.h.  x may be None for SCAN_LINEAR, dgate, dx, dh0 where not wanted."""
    try:
        shape, dtype, index, s = _scan(gate, restart, kind, reverse)
        states = s.n * s.c
        args = (s, _rows(gate, shape, dtype, index, 1, 0), _rows(x, shape, dtype, index, 1, 0), _rows(h, shape, dtype, index, 1, 0),
                _rows(dh, shape, dtype, index, 1, 0), _floats(h0, index, states), _floats(dh_last, index, states),
                _rows(dgate, shape, dtype, index, 1, 0), _rows(dx, shape, dtype, index, 1, 0), _floats(dh0, index, states))
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_gated_scan_backward, args)


def group_norm_workspace_bytes(n, pixels, c, groups, precision):
    """Bytes of scratch group_norm and group_norm_backward need for this shape (0 on bad arguments)."""
    shape = (n, pixels, c, groups, precision)
    if min(shape) < 0 or max(shape) > _MOST:
        return 0
    return int(lib().paac_group_norm_workspace_bytes(Norm(*shape, ACT_NONE, 1.0)))


def _norm(lead, groups, activation, eps, workspace):
    """(shape, type, device, the normalisation's own) of a call whose first tensor leads."""
    if _torch is None:
        _with_torch()
    shape, dtype, index = lead.shape, lead.dtype, lead.get_device()
    if not 3 <= len(shape) <= 4 or dtype not in _TYPES or index < 0 or workspace.get_device() != index or not workspace.is_contiguous():
        raise _Apart
    pixels = shape[1] if len(shape) == 3 else shape[1] * shape[2]
    if pixels > _MOST or max(shape) > _MOST or not 0 <= groups <= _MOST or not 0 <= activation <= _MOST:
        raise _Apart
    return shape, dtype, index, Norm(shape[0], pixels, shape[-1], groups, _TYPES[dtype], activation, eps)


def group_norm(x, gamma, beta, y, mean, rstd, groups, workspace, activation=ACT_NONE, eps=1e-5, stream=None):
    """Group normalisation, channels last: see paac_group_norm in include/paac.h.  x, y [samples][pixels][channels] or
    [samples][rows][columns][channels] with strides of their own (the last axis contiguous); gamma, beta float32 [channels] or None;
    mean, rstd float32 [samples][groups] or None; workspace a contiguous byte tensor."""
    try:
        shape, dtype, index, s = _norm(x, groups, activation, eps, workspace)
        c, g = s.c, s.n * groups
        args = (s, _rows(x, shape, dtype, index, 0, 1), _floats(gamma, index, c), _floats(beta, index, c), _rows(y, shape, dtype, index, 0, 1),
                _floats(mean, index, g), _floats(rstd, index, g), workspace.data_ptr(), workspace.nbytes)
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_group_norm, args)


def group_norm_backward(x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, groups, workspace, activation=ACT_NONE, stream=None):
    """Its gradient: see paac_group_norm_backward in include/paac.h.  dx, dgamma, dbeta may be None where not wanted."""
    try:
        shape, dtype, index, s = _norm(x, groups, activation, 1.0, workspace)
        c, g = s.c, s.n * groups
        args = (s, _rows(x, shape, dtype, index, 0, 1), _rows(dy, shape, dtype, index, 0, 1), _floats(gamma, index, c), _floats(beta, index, c),
                _floats(mean, index, g), _floats(rstd, index, g), _rows(dx, shape, dtype, index, 0, 1), _floats(dgamma, index, c),
                _floats(dbeta, index, c), workspace.data_ptr(), workspace.nbytes)
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_group_norm_backward, args)


# The structures of the operators below as bytes: an object for each of their rows, and a call that hands them over one by one, take several times as long.
_CONV, _CONV_OUT, _CONV_GRADS = (struct.Struct("<" + f) for f in ("6i3q3q3q", "3qq", "3qq3q2qqqQ"))
_SELECTIVE, _SELECTIVE_OUT, _SELECTIVE_GRADS = (struct.Struct("<" + f) for f in ("7i4x3q15q3q", "q3q2qqQ", "q3qq15q4qqQ"))
_DRAW = struct.Struct("<3i4x11q")


def _flags(restart, index, t, n):
    """(address, by sequence, by step) of flags [steps][sequences], one byte each."""
    if restart is None:
        return 0, 0, 0
    if restart.element_size() != 1 or restart.get_device() != index or restart.shape != (t, n):
        raise _Apart
    by_step, by_sequence = restart.stride()
    return restart.data_ptr(), by_sequence, by_step


def _steps(t, shape, dtype, index):
    """(address, by sequence, by step) of the rows of a tensor [steps][sequences][channels]."""
    if t is None:
        return 0, 0, 0
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        raise _Apart
    by_step, by_sequence, one = t.stride()
    if one != 1 and shape[2] > 1:
        raise _Apart
    return t.data_ptr(), by_sequence, by_step


def _inputs(t, shape, dtype, index):
    """The same of a tensor [steps][sequences][groups][state], or without the groups."""
    if t is None:
        return 0, 0, 0
    stride = t.stride()
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or (stride[-1] != 1 and shape[-1] > 1):
        raise _Apart
    if len(stride) == 4 and shape[2] > 1 and stride[2] != shape[3]:
        raise _Apart
    return t.data_ptr(), stride[1], stride[0]


def _whole(t, dtype, index, count):
    """Address of a contiguous tensor of `count` elements of this type on device `index`, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != index or t.numel() != count or not t.is_contiguous():
        raise _Apart
    return t.data_ptr()


def _same(t, shape, dtype, index):
    """Address of a contiguous tensor of this shape and type on device `index`, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        raise _Apart
    return t.data_ptr()


def _room(workspace, index):
    """(address, bytes) of a call's scratch."""
    if workspace is None:
        return 0, 0
    if workspace.get_device() != index or not workspace.is_contiguous():
        raise _Apart
    return workspace.data_ptr(), workspace.nbytes


def _conv(x, weight, bias, before, activation, restart):
    """(shape, type, device, shape of what is carried, the convolution's own) of a call on x."""
    if _torch is None:
        _with_torch()
    shape, dtype, index = x.shape, x.dtype, x.get_device()
    if len(shape) != 3 or dtype not in _TYPES or index < 0 or max(shape) > _MOST or not 0 <= activation <= _MOST:
        raise _Apart
    if weight is None or weight.dim() != 2 or not 1 <= weight.shape[1] <= _MOST:
        raise _Apart
    t, n, c = shape
    width, f = weight.shape[1], _torch.float32
    held = (n, width - 1, c)
    return shape, dtype, index, held, _CONV.pack(t, n, c, width, _TYPES[dtype], activation, *_flags(restart, index, t, n), *_steps(x, shape, dtype, index),
                                                 _whole(weight, f, index, c * width), _whole(bias, f, index, c), _same(before, held, dtype, index))


def causal_conv(x, weight, bias, y, before=None, after=None, restart=None, activation=ACT_SILU, stream=None):
    """A short causal convolution of every channel by itself: see paac_causal_conv in include/paac.h.  x, y [steps][sequences][channels] with
    strides of their own (the last axis contiguous), weight float32 [channels][width], bias float32 [channels] or None, before and after
    [sequences][width - 1][channels] of x's type (after may be before), restart one byte [steps][sequences]."""
    try:
        shape, dtype, index, held, s = _conv(x, weight, bias, before, activation, restart)
        args = (s, _CONV_OUT.pack(*_steps(y, shape, dtype, index), _same(after, held, dtype, index)))
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_causal_conv, args)


def causal_conv_workspace_bytes(t, n, c, width, precision):
    """Bytes of scratch causal_conv_backward needs (0 on bad arguments)."""
    sizes = (t, n, c, width, precision)
    if min(sizes) < 0 or max(sizes) > _MOST:
        return 0
    return int(lib().paac_causal_conv_workspace_bytes(_CONV.pack(*sizes, ACT_NONE, *[0] * 9)))


def causal_conv_backward(x, dy, weight, bias, dx, dweight, dbias, workspace, before=None, dafter=None, dbefore=None, restart=None, activation=ACT_SILU,
                         stream=None):
    """Its gradient: see paac_causal_conv_backward in include/paac.h.  dx, dweight, dbias, dbefore may be None where not wanted."""
    try:
        shape, dtype, index, held, s = _conv(x, weight, bias, before, activation, restart)
        c, f = shape[2], _torch.float32
        args = (s, _CONV_GRADS.pack(*_steps(dy, shape, dtype, index), _same(dafter, held, dtype, index), *_steps(dx, shape, dtype, index),
                                    _whole(dweight, f, index, c * (held[1] + 1)), _whole(dbias, f, index, c), _same(dbefore, held, dtype, index), *_room(workspace, index)))
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_causal_conv_backward, args)


def selective_scan_workspace_bytes(t, n, c, state, groups, precision, backward=False):
    """Bytes of scratch selective_scan, or its gradient, needs (0: on bad arguments, or none)."""
    sizes = (t, n, c, state, groups, precision)
    if min(sizes) < 0 or max(sizes) > _MOST:
        return 0
    return int(lib().paac_selective_scan_workspace_bytes(_SELECTIVE.pack(*sizes, 1, *[0] * 21), 1 if backward else 0))


def _selective(x, dt, A, B, C, D, z, dt_bias, softplus, restart):
    """(shape, shape of B and C, type, device, elements of a state, the scan's own) of a call on x."""
    if _torch is None:
        _with_torch()
    if A is None or B is None:
        raise _Apart
    shape, dtype, index, inputs, rates = x.shape, x.dtype, x.get_device(), B.shape, A.shape
    if len(shape) != 3 or dtype not in _TYPES or index < 0 or max(shape) > _MOST or len(rates) != 2 or not 3 <= len(inputs) <= 4 or max(inputs) > _MOST:
        raise _Apart
    t, n, c = shape
    state, groups, f = inputs[-1], inputs[2] if len(inputs) == 4 else 1, _torch.float32
    if rates[0] != c or rates[1] != state or inputs[0] != t or inputs[1] != n:
        raise _Apart
    s = _SELECTIVE.pack(t, n, c, state, groups, _TYPES[dtype], 1 if softplus else 0, *_flags(restart, index, t, n), *_steps(x, shape, dtype, index),
                        *_steps(dt, shape, dtype, index), *_inputs(B, inputs, dtype, index), *_inputs(C, inputs, dtype, index), *_steps(z, shape, dtype, index),
                        _whole(A, f, index, c * state), _whole(D, f, index, c), _whole(dt_bias, f, index, c))
    return shape, inputs, dtype, index, n * c * state, s


def selective_scan(x, dt, A, B, C, y, workspace=None, D=None, z=None, dt_bias=None, h0=None, h_last=None, states=None, restart=None, softplus=True, stream=None):
    """The selective state space scan: see paac_selective_scan in include/paac.h.  x, dt, z, y [steps][sequences][channels] and B, C
    [steps][sequences][groups][state] (or without the groups) with strides of their own (what is said of a step and sequence contiguous), A float32
    [channels][state], D and dt_bias float32 [channels] or None, h0 and h_last float32 [sequences][channels][state] (h_last may be h0), states float32
    [ceil(steps / SELECTIVE_SPAN)][sequences][channels][state] where the gradient is wanted later, restart one byte [steps][sequences]; workspace a
    contiguous byte tensor of selective_scan_workspace_bytes(), None where that is 0."""
    try:
        shape, inputs, dtype, index, held, s = _selective(x, dt, A, B, C, D, z, dt_bias, softplus, restart)
        f = _torch.float32
        args = (s, _SELECTIVE_OUT.pack(_whole(h0, f, index, held), *_steps(y, shape, dtype, index), _whole(h_last, f, index, held),
                                       _whole(states, f, index, -(-shape[0] // SELECTIVE_SPAN) * held), *_room(workspace, index)))
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_selective_scan, args)


def selective_scan_backward(x, dt, A, B, C, dy, states, dx, ddt, dA, dB, dC, workspace, D=None, z=None, dt_bias=None, dD=None, dz=None, ddt_bias=None,
                            dh_last=None, dh0=None, restart=None, softplus=True, stream=None):
    """Its gradient: see paac_selective_scan_backward in include/paac.h.  Gradients that are not wanted may be None."""
    try:
        shape, inputs, dtype, index, held, s = _selective(x, dt, A, B, C, D, z, dt_bias, softplus, restart)
        c, f = shape[2], _torch.float32
        args = (s, _SELECTIVE_GRADS.pack(_whole(states, f, index, -(-shape[0] // SELECTIVE_SPAN) * held), *_steps(dy, shape, dtype, index), _whole(dh_last, f, index, held),
                                         *_steps(dx, shape, dtype, index), *_steps(ddt, shape, dtype, index), *_inputs(dB, inputs, dtype, index),
                                         *_inputs(dC, inputs, dtype, index), *_steps(dz, shape, dtype, index), _whole(dA, f, index, c * inputs[-1]), _whole(dD, f, index, c),
                                         _whole(ddt_bias, f, index, c), _whole(dh0, f, index, held), *_room(workspace, index)))
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_selective_scan_backward, args)


def _each(t, dtype, index, n):
    """Address of one number a row, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != index or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise _Apart
    return t.data_ptr()


def sample(logits, uniforms, actions, logprob=None, temperature=None, top_k=None, top_p=None, min_p=None, allowed=None, stream=None):
    """An action out of many for each row: see paac_sample in include/paac.h.  logits [rows][actions] with a row stride of its own, uniforms, logprob,
    temperature, top_p, min_p float32 [rows], top_k and actions int32 [rows], allowed one byte [rows][actions]."""
    try:
        if _torch is None:
            _with_torch()
        shape, dtype, index, f, i = logits.shape, logits.dtype, logits.get_device(), _torch.float32, _torch.int32
        if len(shape) != 2 or dtype not in _TYPES or index < 0 or max(shape) > _MOST or uniforms is None or actions is None:
            raise _Apart
        n, v = shape
        row, one = logits.stride()
        mask = mask_row = 0
        if allowed is not None:
            if allowed.element_size() != 1 or allowed.get_device() != index or allowed.shape != shape:
                raise _Apart
            mask_row, mask_one = allowed.stride()
            if mask_one != 1 and v > 1:
                raise _Apart
            mask = allowed.data_ptr()
        if one != 1 and v > 1:
            raise _Apart
        args = (_DRAW.pack(n, v, _TYPES[dtype], logits.data_ptr(), row, mask, mask_row, _each(uniforms, f, index, n), _each(temperature, f, index, n),
                           _each(top_k, i, index, n), _each(top_p, f, index, n), _each(min_p, f, index, n), _each(actions, i, index, n), _each(logprob, f, index, n)),)
    except _Apart:
        return ERR_ARG
    return _status(index, stream, lib().paac_sample, args)


class Paac:
    """One learner.  The device workspace is a torch uint8 tensor on `device`; kernels run on
    torch's current stream at construction time."""

    def __init__(self, arch, n_e, t_max, n_actions, seed, precision=FP32, device="cuda:0", **hparams):
        import torch
        L = lib()
        self.arch = {"nips": ARCH_NIPS, "nature": ARCH_NATURE}.get(arch, arch)
        self.n_e, self.t_max, self.A, self.seed, self.precision = n_e, t_max, n_actions, seed, precision
        self.B = n_e * t_max
        self.hp = default_hparams(precision=precision, **hparams)
        need = workspace_bytes(self.arch, n_e, t_max, n_actions, self.hp)
        if need == 0:
            raise PaacError(ERR_ARG)
        self.device = torch.device(device)
        with torch.cuda.device(self.device):
            self._ws = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
            base = (self._ws.data_ptr() + 255) // 256 * 256
            self.hp.workspace, self.hp.workspace_bytes = base, need
            self._stream = torch.cuda.current_stream(self.device)
            self.hp.stream = self._stream.cuda_stream
            h = C.c_void_p()
            _check(L.paac_init(C.byref(h), self.arch, n_e, t_max, n_actions, C.byref(self.hp), seed))
        self._h = h
        self.P = int(L.paac_param_count(h))

    # -- Algorithm 1 ------------------------------------------------------------------------
    def rollout(self):
        v = RolloutView()
        _check(lib().paac_rollout(self._h, C.byref(v)))
        return v

    def update(self, sync=True):
        if not sync:
            _check(lib().paac_update(self._h, None))
            return None
        s = UpdateStats()
        _check(lib().paac_update(self._h, C.byref(s)), allow=(ERR_NONFINITE, ERR_TIMEOUT, ERR_RANGE))
        return {n: getattr(s, n) for n, _ in UpdateStats._fields_}

    def params(self):
        out = np.empty(self.P, np.float32)
        _check(lib().paac_params(self._h, out.ctypes.data, self.P))
        return out

    # -- external environments -----------------------------------------------------------------
    def act_host(self, t, frames, actions=None, values=None):
        _check(lib().paac_act_host(self._h, t, _host_ptr(frames) if frames is not None else None,
                                   _host_ptr(actions) if actions is not None else None,
                                   _host_ptr(values) if values is not None else None))

    def act_host_newest(self, t, newest, restart=None, actions=None, values=None):
        _check(lib().paac_act_host_newest(self._h, t, _host_ptr(newest), _host_ptr(restart) if restart is not None else None,
                                          _host_ptr(actions) if actions is not None else None,
                                          _host_ptr(values) if values is not None else None))

    def observe_host(self, t, rewards, terminals):
        _check(lib().paac_observe_host(self._h, t, _host_ptr(rewards), _host_ptr(terminals)))

    # -- hooks ---------------------------------------------------------------------------------
    def set_params(self, theta):
        theta = np.ascontiguousarray(theta, np.float32)
        _check(lib().paac_set_params(self._h, theta.ctypes.data, theta.size))

    def force_actions(self, actions):
        if actions is None:
            _check(lib().paac_force_actions(self._h, None))
            return
        a = np.ascontiguousarray(actions, np.int32)
        assert a.size == self.B
        _check(lib().paac_force_actions(self._h, a.ctypes.data))

    def debug_read(self, which):
        """Tensor `which` as a flat numpy array (bf16 tensors are widened to float32)."""
        n = int(lib().paac_debug_bytes(self._h, which))
        if n == 0:
            raise PaacError(ERR_ARG)
        raw = np.empty(n, np.uint8)
        _check(lib().paac_debug_read(self._h, which, raw.ctypes.data, n))
        if which in _DBG_DTYPE:
            return raw.view(_DBG_DTYPE[which])
        if which >= DBG_ACT0 and self.precision == BF16:
            return (raw.view(np.uint16).astype(np.uint32) << 16).view(np.float32)
        return raw.view(np.float32)

    def debug_write(self, which, arr):
        arr = np.ascontiguousarray(arr)
        _check(lib().paac_debug_write(self._h, which, arr.ctypes.data, arr.nbytes))

    def debug_write_act(self, layer, arr):
        """Overwrite stored activation `layer` from float32 values (which, with bf16 storage, must
        already be bf16-representable)."""
        arr = np.ascontiguousarray(arr, np.float32)
        if self.precision == BF16:
            bits = arr.view(np.uint32)
            assert not np.any(bits & 0xFFFF), "not bf16 values"
            arr = (bits >> 16).astype(np.uint16)
        self.debug_write(DBG_ACT0 + layer, arr)

    def error_word(self):
        """The sticky device error bits (0 when every kernel so far ran to the end)."""
        w = np.zeros(1, np.uint32)
        lib().paac_debug_read(self._h, DBG_ERROR_WORD, w.ctypes.data, 4)      # the status only repeats the word
        return int(w[0])

    def clear_error_word(self):
        self.debug_write(DBG_ERROR_WORD, np.zeros(1, np.uint32))

    def wait_probe(self, max_polls):
        """Status of a wait that is made to run out (ERR_TIMEOUT when the device-side bound works)."""
        return int(lib().paac_debug_wait_probe(self._h, max_polls))

    def launch_count(self):
        return int(lib().paac_launch_count(self._h))

    def set_option(self, option, value):
        _check(lib().paac_set_option(self._h, option, value))

    def profile(self, enable):
        _check(lib().paac_profile(self._h, 1 if enable else 0))

    def profile_read(self):
        """{kernel family: (device ms, launches)} since profiling was enabled."""
        n = 64
        names, ms, cnt = (C.c_char_p * n)(), (C.c_double * n)(), (C.c_uint64 * n)()
        k = lib().paac_profile_read(self._h, n, names, ms, cnt)
        if k < 0:
            raise PaacError(ERR_ARG)
        return {names[j].decode(): (ms[j], int(cnt[j])) for j in range(k)}

    def close(self):
        if getattr(self, "_h", None):
            lib().paac_destroy(self._h)
            self._h = None
            self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
