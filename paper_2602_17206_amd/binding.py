"""ctypes binding of ``libsdtw_hip.so`` (the C-ABI of ``include/sdtw.h``).

Argument marshalling only: every function here checks shapes and dtypes, passes device
pointers through, and raises :class:`SdtwError` on a non-zero status.  PyTorch supplies
device memory and the current stream; nothing is computed in Python and there is no
fallback: if the library has not been built, the first call raises.
"""
import array
import contextlib
import ctypes
import functools
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsdtw_hip.so")
_lib = None

UNFUSED = 0
FUSED = 1
FLAG_VALUE_ONLY = 1
FLAG_MIN_MEMORY = 2
FLAG_DENSE_E = 4
EXPORT_COST, EXPORT_R, EXPORT_E = 0, 1, 2

STATUS_OK = 0
STATUS_INVALID_ARG = 1
STATUS_WORKSPACE = 2
STATUS_UNSUPPORTED = 3
STATUS_STATE = 4
STATUS_HIP = 5
STATUS_TIMEOUT = 6


class SdtwError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__("%s: status %d (%s)" % (where, status, sdtw_status_string(status)))


class Desc(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("M", ctypes.c_int32), ("D", ctypes.c_int32),
        ("gamma", ctypes.c_float), ("mode", ctypes.c_int32),
        ("x_batch_stride", ctypes.c_int64), ("y_batch_stride", ctypes.c_int64),
        ("bandwidth", ctypes.c_int32), ("flags", ctypes.c_uint32),
    ]


class BaryDesc(ctypes.Structure):
    _fields_ = [
        ("K", ctypes.c_int32), ("Lz", ctypes.c_int32), ("Lx", ctypes.c_int32), ("D", ctypes.c_int32),
        ("gamma", ctypes.c_float), ("mode", ctypes.c_int32),
        ("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
        ("step", ctypes.c_int32), ("flags", ctypes.c_uint32),
    ]


class DistillDesc(ctypes.Structure):
    _fields_ = [
        ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("top", ctypes.c_int32), ("teacher_rows", ctypes.c_int32),
        ("temperature", ctypes.c_float), ("target", ctypes.c_int32),
        ("logit_type", ctypes.c_int32), ("teacher_type", ctypes.c_int32), ("id_type", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("logit_stride", ctypes.c_int64), ("grad_stride", ctypes.c_int64), ("teacher_stride", ctypes.c_int64),
        ("id_stride", ctypes.c_int64),
    ]


class BiasDesc(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("M", ctypes.c_int32),
        ("buckets", ctypes.c_int32), ("max_distance", ctypes.c_int32), ("two_sided", ctypes.c_int32),
        ("plane_type", ctypes.c_int32), ("table_type", ctypes.c_int32), ("flags", ctypes.c_uint32),
        ("offset", ctypes.c_int64), ("in_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
        ("table_stride", ctypes.c_int64 * 2),
    ]


class AttentionDesc(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hk", ctypes.c_int32), ("N", ctypes.c_int32), ("M", ctypes.c_int32),
        ("D", ctypes.c_int32), ("type", ctypes.c_int32), ("table_type", ctypes.c_int32), ("buckets", ctypes.c_int32),
        ("max_distance", ctypes.c_int32), ("two_sided", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("scale", ctypes.c_float), ("cap", ctypes.c_float), ("flags", ctypes.c_uint32),
        ("offset", ctypes.c_int64), ("prefix", ctypes.c_int64),
        ("q_stride", ctypes.c_int64 * 4), ("k_stride", ctypes.c_int64 * 4), ("v_stride", ctypes.c_int64 * 4),
        ("out_stride", ctypes.c_int64 * 4), ("dout_stride", ctypes.c_int64 * 4), ("dq_stride", ctypes.c_int64 * 4),
        ("dk_stride", ctypes.c_int64 * 4), ("dv_stride", ctypes.c_int64 * 4), ("table_stride", ctypes.c_int64 * 2),
    ]


class AttentionLists(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("offsets", "prefixes", "row_len", "col_len", "row_document", "col_document")]


EXPORTED_SYMBOLS = (
    "sdtw_version", "sdtw_status_string", "sdtw_workspace_bytes", "sdtw_forward", "sdtw_backward",
    "sdtw_barycenter_workspace_bytes", "sdtw_barycenter_step", "sdtw_workspace_status",
    "sdtw_normalized_workspace_bytes", "sdtw_normalized_forward", "sdtw_normalized_backward",
    "sdtw_forward_ragged", "sdtw_backward_ragged",
    "sdtw_debug_export", "sdtw_debug_lane_shift", "sdtw_debug_set_spin_limit",
    "sdtw_debug_profile", "sdtw_debug_profile_read", "sdtw_debug_force_workgroup_shape",
    "sdtw_debug_rate_probe", "sdtw_forward_static_scratch", "sdtw_debug_set_pool_blocks",
    "sdtw_half_workspace_bytes", "sdtw_forward_half", "sdtw_backward_half",
    "sdtw_distill_workspace_bytes", "sdtw_distill_forward", "sdtw_distill_backward", "sdtw_distill_step",
    "sdtw_position_bias_starts", "sdtw_position_bias_forward", "sdtw_position_bias_workspace_bytes",
    "sdtw_position_bias_backward", "sdtw_biased_workspace_bytes", "sdtw_forward_biased", "sdtw_backward_biased",
    "sdtw_attention_forward_workspace_bytes", "sdtw_attention_backward_workspace_bytes", "sdtw_attention_forward",
    "sdtw_attention_backward", "sdtw_gradient_clip_workspace_bytes", "sdtw_gradient_clip",
)


def library_path():
    return _LIB_PATH


def load_library():
    """Loads the HIP library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            "libsdtw_hip.so is missing at %s: run `python -c 'import __graft_entry__ as g; g.build()'` "
            "from the repository root" % _LIB_PATH)
    # PyTorch first: its wheel brings a HIP runtime of its own, and the tensors this binding hands over
    # live in that runtime.  Loaded after it, this library binds to the same one; loaded before it, the
    # process would end up with two (the calls then fail with a HIP runtime error).
    import torch  # noqa: F401

    lib = ctypes.CDLL(_LIB_PATH)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    lib.sdtw_version.restype = i32
    lib.sdtw_status_string.restype = ctypes.c_char_p
    lib.sdtw_status_string.argtypes = [i32]
    lib.sdtw_workspace_bytes.restype = sz
    lib.sdtw_workspace_bytes.argtypes = [ctypes.POINTER(Desc)]
    lib.sdtw_forward.restype = i32
    lib.sdtw_forward.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, sz, vp]
    lib.sdtw_forward_static_scratch.restype = i32
    lib.sdtw_forward_static_scratch.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp]
    lib.sdtw_backward.restype = i32
    lib.sdtw_backward.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_barycenter_workspace_bytes.restype = sz
    lib.sdtw_barycenter_workspace_bytes.argtypes = [ctypes.POINTER(BaryDesc)]
    lib.sdtw_barycenter_step.restype = i32
    lib.sdtw_barycenter_step.argtypes = [ctypes.POINTER(BaryDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_forward_ragged.restype = i32
    lib.sdtw_forward_ragged.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_backward_ragged.restype = i32
    lib.sdtw_backward_ragged.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_normalized_workspace_bytes.restype = sz
    lib.sdtw_normalized_workspace_bytes.argtypes = [ctypes.POINTER(Desc)]
    lib.sdtw_normalized_forward.restype = i32
    lib.sdtw_normalized_forward.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, sz, vp]
    lib.sdtw_normalized_backward.restype = i32
    lib.sdtw_normalized_backward.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_workspace_status.restype = i32
    lib.sdtw_workspace_status.argtypes = [vp, sz, vp, ctypes.POINTER(ctypes.c_int32)]
    lib.sdtw_debug_export.restype = i32
    lib.sdtw_debug_export.argtypes = [ctypes.POINTER(Desc), vp, sz, i32, vp, vp]
    lib.sdtw_debug_lane_shift.restype = i32
    lib.sdtw_debug_lane_shift.argtypes = [vp, vp]
    lib.sdtw_debug_set_spin_limit.restype = i32
    lib.sdtw_debug_set_spin_limit.argtypes = [ctypes.c_uint32]
    lib.sdtw_debug_force_workgroup_shape.restype = i32
    lib.sdtw_debug_force_workgroup_shape.argtypes = [i32]
    lib.sdtw_debug_profile.restype = i32
    lib.sdtw_debug_profile.argtypes = [i32]
    lib.sdtw_debug_profile_read.restype = i32
    lib.sdtw_debug_profile_read.argtypes = [ctypes.c_char_p, sz, ctypes.POINTER(ctypes.c_float), i32,
                                            ctypes.POINTER(ctypes.c_int)]
    lib.sdtw_half_workspace_bytes.restype = sz
    lib.sdtw_half_workspace_bytes.argtypes = [ctypes.POINTER(Desc)]
    lib.sdtw_forward_half.restype = i32
    lib.sdtw_forward_half.argtypes = [ctypes.POINTER(Desc), vp, vp, i32, vp, vp, sz, vp]
    lib.sdtw_backward_half.restype = i32
    lib.sdtw_backward_half.argtypes = [ctypes.POINTER(Desc), vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_debug_set_pool_blocks.restype = i32
    lib.sdtw_debug_set_pool_blocks.argtypes = [ctypes.c_longlong]
    lib.sdtw_debug_rate_probe.restype = i32
    lib.sdtw_debug_rate_probe.argtypes = [i32, i32, i32, i32, vp, sz, ctypes.POINTER(ctypes.c_float), vp]
    pd, pb = ctypes.POINTER(DistillDesc), ctypes.POINTER(BiasDesc)
    lib.sdtw_distill_workspace_bytes.restype = sz
    lib.sdtw_distill_workspace_bytes.argtypes = [pd]
    lib.sdtw_distill_forward.restype = i32
    lib.sdtw_distill_forward.argtypes = [pd, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_distill_backward.restype = i32
    lib.sdtw_distill_backward.argtypes = [pd, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.sdtw_distill_step.restype = i32
    lib.sdtw_distill_step.argtypes = [pd, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_position_bias_starts.restype = i32
    lib.sdtw_position_bias_starts.argtypes = [pb, vp]
    lib.sdtw_position_bias_forward.restype = i32
    lib.sdtw_position_bias_forward.argtypes = [pb, vp, vp, vp, vp, vp, vp, vp]
    lib.sdtw_position_bias_workspace_bytes.restype = sz
    lib.sdtw_position_bias_workspace_bytes.argtypes = [pb]
    lib.sdtw_position_bias_backward.restype = i32
    lib.sdtw_position_bias_backward.argtypes = [pb, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    pdesc = ctypes.POINTER(Desc)
    lib.sdtw_biased_workspace_bytes.restype = sz
    lib.sdtw_biased_workspace_bytes.argtypes = [pdesc, pb]
    lib.sdtw_forward_biased.restype = i32
    lib.sdtw_forward_biased.argtypes = [pdesc, pb, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_backward_biased.restype = i32
    lib.sdtw_backward_biased.argtypes = [pdesc, pb, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    # (descriptors and lists as structures by reference, or as their bytes)
    for name in ("sdtw_attention_forward_workspace_bytes", "sdtw_attention_backward_workspace_bytes"):
        getattr(lib, name).restype, getattr(lib, name).argtypes = sz, [vp]
    lib.sdtw_attention_forward.restype = i32
    lib.sdtw_attention_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_attention_backward.restype = i32
    lib.sdtw_attention_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.sdtw_gradient_clip_workspace_bytes.restype = sz
    lib.sdtw_gradient_clip_workspace_bytes.argtypes = [vp, i32]
    lib.sdtw_gradient_clip.restype = i32
    lib.sdtw_gradient_clip.argtypes = [vp, i32, ctypes.c_float, vp, vp, sz, vp]
    _lib = lib
    return lib


def sdtw_version():
    return int(load_library().sdtw_version())


def sdtw_status_string(status):
    return load_library().sdtw_status_string(int(status)).decode()


def make_desc(B, N, M, D, gamma, mode, x_shared=False, y_shared=False, bandwidth=0, flags=0):
    return Desc(B, N, M, D, float(gamma), int(mode), 0 if x_shared else N * D, 0 if y_shared else M * D,
                bandwidth, flags)


def sdtw_workspace_bytes(desc):
    return int(load_library().sdtw_workspace_bytes(ctypes.byref(desc)))


def sdtw_barycenter_workspace_bytes(bdesc):
    return int(load_library().sdtw_barycenter_workspace_bytes(ctypes.byref(bdesc)))


def _stream_ptr(stream):
    if stream is not None:
        return ctypes.c_void_p(int(stream))
    import torch

    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t, dtype=None, shape=None, name="tensor", device=None):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return ctypes.c_void_p(0)
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous device tensor" % name)
    if device is not None and t.device != device:
        raise ValueError("%s must be on %s" % (name, device))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must have dtype %s" % (name, dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return ctypes.c_void_p(t.data_ptr())


class Workspace:
    """A device buffer of ``sdtw_workspace_bytes(desc)`` bytes allocated through PyTorch."""

    def __init__(self, nbytes, device="cuda"):
        import torch

        self.nbytes = int(nbytes)
        # torch's caching allocator returns 512-byte aligned blocks
        self.buffer = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        assert self.buffer.data_ptr() % 256 == 0

    @property
    def ptr(self):
        return ctypes.c_void_p(self.buffer.data_ptr())


def _desc_for(x, y, gamma, mode, check_dtype=True):
    import torch

    if x.dim() == 2:
        N, D = x.shape
        x_shared = True
    else:
        _, N, D = x.shape
        x_shared = False
    if y.dim() == 2:
        M = y.shape[0]
        y_shared = True
    else:
        M = y.shape[1]
        y_shared = False
    if x_shared and y_shared:
        B = 1
    else:
        B = y.shape[0] if not y_shared else x.shape[0]
    if y.shape[-1] != D:
        raise ValueError("x and y must have the same feature dimension")
    if not x_shared and not y_shared and x.shape[0] != y.shape[0]:
        raise ValueError("x and y must have the same batch size")
    assert not check_dtype or (x.dtype == torch.float32 and y.dtype == torch.float32)
    return make_desc(B, N, M, D, gamma, mode, x_shared, y_shared)


def sdtw_forward(x, y, gamma, mode=FUSED, workspace=None, value=None, stream=None, value_only=False,
                 bandwidth=0, min_memory=False):
    """value[b] = sdtw_gamma(x_b, y_b).  Returns (value, desc, workspace); keep the last two for
    :func:`sdtw_backward`.  x [B,N,D] or [N,D]; y [B,M,D] or [M,D]; float32 device tensors.
    ``value_only=True`` sets SDTW_FLAG_VALUE_ONLY: no backward call will follow.
    ``bandwidth`` w > 0: only cells with |i-j| <= w belong to the grid."""
    import torch

    lib = load_library()
    desc = _desc_for(x, y, gamma, mode)
    desc.bandwidth = int(bandwidth)
    if value_only:
        desc.flags |= FLAG_VALUE_ONLY
    if min_memory:
        desc.flags |= FLAG_MIN_MEMORY
    if workspace is None:
        nbytes = sdtw_workspace_bytes(desc)
        if nbytes == 0:
            raise SdtwError(STATUS_INVALID_ARG, "sdtw_workspace_bytes")
        workspace = Workspace(nbytes, x.device)
    if value is None:
        value = torch.empty(desc.B, dtype=torch.float32, device=x.device)
    rc = lib.sdtw_forward(ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
                          _ptr(value, torch.float32, (desc.B,), "value"), workspace.ptr, workspace.nbytes,
                          _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_forward")
    return value, desc, workspace


def sdtw_forward_desc(desc, x, y, workspace, value, stream=None):
    """sdtw_forward with a descriptor the caller made (make_desc): nothing is allocated here."""
    import torch

    rc = load_library().sdtw_forward(ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
                                     _ptr(value, torch.float32, (desc.B,), "value"), workspace.ptr, workspace.nbytes,
                                     _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_forward")
    return value


STATIC_SCRATCH_BYTES = 64 << 20


def sdtw_forward_static_scratch(desc, x, y, value, stream=None):
    """sdtw_forward's values through the entry point that uses the library's own scratch buffer
    (nothing is allocated, here or in the library).  Returns the status code."""
    import torch

    return int(load_library().sdtw_forward_static_scratch(
        ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
        _ptr(value, torch.float32, (desc.B,), "value"), _stream_ptr(stream)))


def sdtw_backward(desc, x, y, workspace, grad_value=None, want_dx=True, want_dy=True, want_E=False,
                  dx=None, dy=None, E=None, stream=None):
    """Gradients of the values produced by the forward call that filled ``workspace``.
    Returns (dx [B,N,D] or None, dy [B,M,D] or None, E [B,N,M] or None)."""
    import torch

    lib = load_library()
    dev = x.device
    if want_dx and dx is None:
        dx = torch.empty((desc.B, desc.N, desc.D), dtype=torch.float32, device=dev)
    if want_dy and dy is None:
        dy = torch.empty((desc.B, desc.M, desc.D), dtype=torch.float32, device=dev)
    if want_E and E is None:
        E = torch.empty((desc.B, desc.N, desc.M), dtype=torch.float32, device=dev)
    rc = lib.sdtw_backward(
        ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
        _ptr(grad_value, torch.float32, (desc.B,), "grad_value"),
        _ptr(dx, torch.float32, (desc.B, desc.N, desc.D), "dx"),
        _ptr(dy, torch.float32, (desc.B, desc.M, desc.D), "dy"),
        _ptr(E, torch.float32, (desc.B, desc.N, desc.M), "E"),
        workspace.ptr, workspace.nbytes, _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_backward")
    return dx, dy, E


def sdtw_forward_ragged(x, y, x_len, y_len, gamma, mode=FUSED, workspace=None, value=None, stream=None,
                        bandwidth=0, min_memory=False):
    """As :func:`sdtw_forward` for pairs of individual lengths: x_len, y_len are int32 device tensors
    [B] (or None).  Returns (value, desc, workspace)."""
    import torch

    lib = load_library()
    desc = _desc_for(x, y, gamma, mode)
    desc.bandwidth = int(bandwidth)
    if min_memory:
        desc.flags |= FLAG_MIN_MEMORY
    if workspace is None:
        nbytes = sdtw_workspace_bytes(desc)
        if nbytes == 0:
            raise SdtwError(STATUS_INVALID_ARG, "sdtw_workspace_bytes")
        workspace = Workspace(nbytes, x.device)
    if value is None:
        value = torch.empty(desc.B, dtype=torch.float32, device=x.device)
    rc = lib.sdtw_forward_ragged(ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
                                 _ptr(x_len, torch.int32, (desc.B,), "x_len"), _ptr(y_len, torch.int32, (desc.B,), "y_len"),
                                 _ptr(value, torch.float32, (desc.B,), "value"), workspace.ptr, workspace.nbytes,
                                 _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_forward_ragged")
    return value, desc, workspace


def sdtw_backward_ragged(desc, x, y, x_len, y_len, workspace, grad_value=None, want_E=False, dx=None, dy=None,
                         E=None, stream=None):
    """Gradients for :func:`sdtw_forward_ragged` (same length vectors).  Returns (dx, dy, E or None)."""
    import torch

    lib = load_library()
    dev = x.device
    if dx is None:
        dx = torch.empty((desc.B, desc.N, desc.D), dtype=torch.float32, device=dev)
    if dy is None:
        dy = torch.empty((desc.B, desc.M, desc.D), dtype=torch.float32, device=dev)
    if want_E and E is None:
        E = torch.empty((desc.B, desc.N, desc.M), dtype=torch.float32, device=dev)
    rc = lib.sdtw_backward_ragged(
        ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
        _ptr(x_len, torch.int32, (desc.B,), "x_len"), _ptr(y_len, torch.int32, (desc.B,), "y_len"),
        _ptr(grad_value, torch.float32, (desc.B,), "grad_value"),
        _ptr(dx, torch.float32, (desc.B, desc.N, desc.D), "dx"),
        _ptr(dy, torch.float32, (desc.B, desc.M, desc.D), "dy"),
        _ptr(E, torch.float32, (desc.B, desc.N, desc.M), "E"),
        workspace.ptr, workspace.nbytes, _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_backward_ragged")
    return dx, dy, E


def sdtw_normalized_workspace_bytes(desc):
    return int(load_library().sdtw_normalized_workspace_bytes(ctypes.byref(desc)))


def sdtw_normalized_forward(x, y, gamma, mode=FUSED, workspace=None, value=None, stream=None, min_memory=False):
    """value[b] = sdtw(x_b,y_b) - (sdtw(x_b,x_b) + sdtw(y_b,y_b)) / 2.  Returns (value, desc, workspace)."""
    import torch

    lib = load_library()
    desc = _desc_for(x, y, gamma, mode)
    if min_memory:
        desc.flags |= FLAG_MIN_MEMORY
    if workspace is None:
        nbytes = sdtw_normalized_workspace_bytes(desc)
        if nbytes == 0:
            raise SdtwError(STATUS_INVALID_ARG, "sdtw_normalized_workspace_bytes")
        workspace = Workspace(nbytes, x.device)
    if value is None:
        value = torch.empty(desc.B, dtype=torch.float32, device=x.device)
    rc = lib.sdtw_normalized_forward(ctypes.byref(desc), _ptr(x, torch.float32, name="x"),
                                     _ptr(y, torch.float32, name="y"), _ptr(value, torch.float32, (desc.B,), "value"),
                                     workspace.ptr, workspace.nbytes, _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_normalized_forward")
    return value, desc, workspace


def sdtw_normalized_backward(desc, x, y, workspace, grad_value=None, want_dx=True, want_dy=True, dx=None, dy=None,
                             stream=None):
    """Gradients of the normalised values.  Returns (dx [B,N,D] or None, dy [B,M,D] or None)."""
    import torch

    lib = load_library()
    dev = x.device
    if want_dx and dx is None:
        dx = torch.empty((desc.B, desc.N, desc.D), dtype=torch.float32, device=dev)
    if want_dy and dy is None:
        dy = torch.empty((desc.B, desc.M, desc.D), dtype=torch.float32, device=dev)
    rc = lib.sdtw_normalized_backward(
        ctypes.byref(desc), _ptr(x, torch.float32, name="x"), _ptr(y, torch.float32, name="y"),
        _ptr(grad_value, torch.float32, (desc.B,), "grad_value"),
        _ptr(dx, torch.float32, (desc.B, desc.N, desc.D), "dx"),
        _ptr(dy, torch.float32, (desc.B, desc.M, desc.D), "dy"),
        workspace.ptr, workspace.nbytes, _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_normalized_backward")
    return dx, dy


def make_bary_desc(K, Lz, Lx, D, gamma, mode, lr, beta1, beta2, eps, step, flags=0):
    return BaryDesc(K, Lz, Lx, D, float(gamma), int(mode), float(lr), float(beta1), float(beta2), float(eps),
                    int(step), int(flags))


def sdtw_barycenter_step(z, X, adam_m, adam_v, gamma, step, lr=0.05, beta1=0.9, beta2=0.999, eps=1e-8,
                         mode=FUSED, workspace=None, loss=None, dz=None, want_dz=False, stream=None, min_memory=False):
    """One in-place Adam step on z [Lz,D] against X [K,Lx,D].  Returns (loss [1], dz or None, workspace)."""
    import torch

    lib = load_library()
    K, Lx, D = X.shape
    Lz = z.shape[0]
    bdesc = make_bary_desc(K, Lz, Lx, D, gamma, mode, lr, beta1, beta2, eps, step, FLAG_MIN_MEMORY if min_memory else 0)
    if workspace is None:
        nbytes = sdtw_barycenter_workspace_bytes(bdesc)
        if nbytes == 0:
            raise SdtwError(STATUS_INVALID_ARG, "sdtw_barycenter_workspace_bytes")
        workspace = Workspace(nbytes, z.device)
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=z.device)
    if want_dz and dz is None:
        dz = torch.empty((Lz, D), dtype=torch.float32, device=z.device)
    rc = lib.sdtw_barycenter_step(
        ctypes.byref(bdesc), _ptr(z, torch.float32, (Lz, D), "z"), _ptr(X, torch.float32, name="X"),
        _ptr(adam_m, torch.float32, (Lz, D), "adam_m"), _ptr(adam_v, torch.float32, (Lz, D), "adam_v"),
        _ptr(loss, torch.float32, (1,), "loss"), _ptr(dz, torch.float32, (Lz, D), "dz"),
        workspace.ptr, workspace.nbytes, _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_barycenter_step")
    return loss, dz, workspace


def workspace_status(workspace, stream=None):
    """Synchronises and returns the device-side status word of a workspace."""
    out = ctypes.c_int32(-1)
    rc = load_library().sdtw_workspace_status(workspace.ptr, workspace.nbytes, _stream_ptr(stream), ctypes.byref(out))
    if rc != 0:
        raise SdtwError(rc, "sdtw_workspace_status")
    return int(out.value)


def debug_export(desc, workspace, what, stream=None):
    """Row-major copy of an intermediate (cost: float32, R: float64, E: float32), shape [B,N,M]."""
    import torch

    dtype = torch.float64 if what == EXPORT_R else torch.float32
    out = torch.empty((desc.B, desc.N, desc.M), dtype=dtype, device=workspace.buffer.device)
    rc = load_library().sdtw_debug_export(ctypes.byref(desc), workspace.ptr, workspace.nbytes, int(what),
                                          ctypes.c_void_p(out.data_ptr()), _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_debug_export")
    return out


def debug_lane_shift(stream=None):
    import torch

    out = torch.empty(128, dtype=torch.int32, device="cuda")
    rc = load_library().sdtw_debug_lane_shift(ctypes.c_void_p(out.data_ptr()), _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_debug_lane_shift")
    return out


def debug_set_spin_limit(polls):
    load_library().sdtw_debug_set_spin_limit(int(polls))


def debug_profile(enable):
    load_library().sdtw_debug_profile(1 if enable else 0)


def debug_profile_read(max_entries=4096):
    """[(kernel label, milliseconds)] of every launch since profiling was switched on."""
    names = ctypes.create_string_buffer(64 * max_entries)
    ms = (ctypes.c_float * max_entries)()
    count = ctypes.c_int(0)
    rc = load_library().sdtw_debug_profile_read(names, len(names), ms, max_entries, ctypes.byref(count))
    if rc != 0:
        raise SdtwError(rc, "sdtw_debug_profile_read")
    labels = names.value.decode().split(";")[:count.value]
    return [(labels[i], float(ms[i])) for i in range(count.value)]


def debug_force_workgroup_shape(bands_per_workgroup):
    rc = load_library().sdtw_debug_force_workgroup_shape(int(bands_per_workgroup))
    if rc != 0:
        raise SdtwError(rc, "sdtw_debug_force_workgroup_shape")


RATE_PROBE_SCRATCH_BYTES = 16 << 20


def debug_rate_probe(probe, variant, waves_per_simd, iters, scratch, stream=None):
    """Milliseconds one calibration micro-kernel took (see sdtw_debug_rate_probe in sdtw.h)."""
    ms = ctypes.c_float(0.0)
    rc = load_library().sdtw_debug_rate_probe(int(probe), int(variant), int(waves_per_simd), int(iters), scratch.ptr,
                                              scratch.nbytes, ctypes.byref(ms), _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_debug_rate_probe")
    return float(ms.value)


def debug_set_pool_blocks(blocks):
    load_library().sdtw_debug_set_pool_blocks(int(blocks))


INPUT_F16, INPUT_BF16 = 1, 2


def sdtw_forward_half(x, y, gamma, mode=FUSED, workspace=None, value=None, stream=None, min_memory=False):
    """sdtw_forward for float16 or bfloat16 device tensors x [B,N,D] / [N,D], y [B,M,D] / [M,D] (same dtype).
    Returns (value float32 [B], desc, workspace); keep the last two for :func:`sdtw_backward_half`."""
    import torch

    lib = load_library()
    if x.dtype != y.dtype or x.dtype not in (torch.float16, torch.bfloat16):
        raise ValueError("x and y must both be float16 or both bfloat16")
    desc = _desc_for(x, y, gamma, mode, check_dtype=False)
    if min_memory:
        desc.flags |= FLAG_MIN_MEMORY
    if workspace is None:
        nbytes = int(lib.sdtw_half_workspace_bytes(ctypes.byref(desc)))
        if nbytes == 0:
            raise SdtwError(STATUS_INVALID_ARG, "sdtw_half_workspace_bytes")
        workspace = Workspace(nbytes, x.device)
    if value is None:
        value = torch.empty(desc.B, dtype=torch.float32, device=x.device)
    kind = INPUT_F16 if x.dtype == torch.float16 else INPUT_BF16
    rc = lib.sdtw_forward_half(ctypes.byref(desc), _ptr(x, name="x"), _ptr(y, name="y"), kind,
                               _ptr(value, torch.float32, (desc.B,), "value"), workspace.ptr, workspace.nbytes,
                               _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_forward_half")
    return value, desc, workspace


def sdtw_backward_half(desc, workspace, grad_value=None, want_dx=True, want_dy=True, want_E=False, stream=None):
    """Gradients (float32) of the values :func:`sdtw_forward_half` produced.  Returns (dx, dy, E or None)."""
    import torch

    lib = load_library()
    dev = workspace.buffer.device
    dx = torch.empty((desc.B, desc.N, desc.D), dtype=torch.float32, device=dev) if want_dx else None
    dy = torch.empty((desc.B, desc.M, desc.D), dtype=torch.float32, device=dev) if want_dy else None
    E = torch.empty((desc.B, desc.N, desc.M), dtype=torch.float32, device=dev) if want_E else None
    rc = lib.sdtw_backward_half(ctypes.byref(desc), _ptr(grad_value, torch.float32, (desc.B,), "grad_value"),
                                _ptr(dx), _ptr(dy), _ptr(E), workspace.ptr, workspace.nbytes, _stream_ptr(stream))
    if rc != 0:
        raise SdtwError(rc, "sdtw_backward_half")
    return dx, dy, E


# ---------------------------------------------------------------- operators of a model trained with Soft-DTW

TYPE_F32, TYPE_F16, TYPE_BF16 = 0, 1, 2
ID_I32, ID_I64 = 0, 1
DISTILL_RENORMALIZED, DISTILL_TAIL = 0, 1
DISTILL_STATS = 8


_type_codes = {}


def _type_of(t, name):
    if not _type_codes:
        import torch

        _type_codes.update({torch.float32: TYPE_F32, torch.float16: TYPE_F16, torch.bfloat16: TYPE_BF16})
    kind = _type_codes.get(t.dtype)
    if kind is None:
        raise ValueError("%s must be float32, float16 or bfloat16" % name)
    return kind


def _given_stream(stream, device):
    """With ``stream`` (a raw handle) the calls in this context run as on that stream: what they allocate belongs to it too, so
    that no other stream is given the memory while the kernels are still at work, and no memory is taken that is in use elsewhere."""
    if stream is None:
        return contextlib.nullcontext()
    import torch

    handle = int(stream)
    return torch.cuda.stream(torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device))


def _on_given_stream(call):
    """The call with ``stream=``: see :func:`_given_stream`."""
    @functools.wraps(call)
    def on_stream(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        import torch

        device = next((a.device for a in (*args, *kw.values()) if torch.is_tensor(a)), None)
        with _given_stream(stream, device):
            return call(*args, **kw)
    return on_stream


def _stream_of(device):
    """The current stream of the tensors' device, which has to be the current one."""
    import torch

    if device.index != torch._C._cuda_getDevice():
        raise ValueError("the tensors must be on the current device")
    return torch._C._cuda_getCurrentRawStream(device.index)


def _rows_ptr(t, T, K, device, name, dtype=None):
    """Device pointer and row stride of a matrix [T, K] whose rows are contiguous."""
    if t.device != device or t.shape != (T, K) or (dtype is not None and t.dtype != dtype):
        raise ValueError("%s must be%s [%d, %d] on %s" % (name, " %s" % dtype if dtype else "", T, K, device))
    step, along = t.stride()
    if (along != 1 and K > 1) or (step < K and T > 1):
        raise ValueError("%s must have contiguous rows that do not overlap" % name)
    return t.data_ptr(), step if step > K else K


def _vector_ptr(t, n, device, dtype, name):
    if t is None:
        return None
    if t.device != device or t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s [%d] on %s" % (name, dtype, n, device))
    return t.data_ptr()


_I32, _I64 = 1 << 31, 1 << 63


def _whole(v, limit, name):
    """v as a whole number of [-limit, limit): a descriptor's field would drop what it does not hold."""
    if type(v) is int and -limit <= v < limit:
        return v
    n = int(v)
    if n != v or not -limit <= n < limit:
        raise ValueError("%s must be a whole number below 2^%d" % (name, limit.bit_length() - 1))
    return n


def _distill_args(logits, teacher_logits, teacher_ids, temperature, teacher_lse, teacher_row):
    """(descriptor, the pointers every distillation call begins with)"""
    import torch

    if logits.dim() != 2 or teacher_logits.dim() != 2 or not logits.is_cuda:
        raise ValueError("logits [T, V] and teacher_logits [R, K] must be device matrices")
    dev, (T, V), (R, K) = logits.device, logits.shape, teacher_logits.shape
    wide_ids = teacher_ids.dtype == torch.int64
    if not wide_ids and teacher_ids.dtype != torch.int32:
        raise ValueError("teacher_ids must be int32 or int64")
    zp, zs = _rows_ptr(logits, T, V, dev, "logits")
    tp, ts = _rows_ptr(teacher_logits, R, K, dev, "teacher_logits")
    ip, ids = _rows_ptr(teacher_ids, R, K, dev, "teacher_ids")
    desc = DistillDesc(T, V, K, R, temperature, DISTILL_RENORMALIZED if teacher_lse is None else DISTILL_TAIL,
                       _type_of(logits, "logits"), _type_of(teacher_logits, "teacher_logits"), ID_I64 if wide_ids else ID_I32, 0,
                       zs, V, ts, ids)
    return desc, (zp, tp, ip, _vector_ptr(teacher_lse, R, dev, torch.float32, "teacher_lse"),
                  _vector_ptr(teacher_row, T, dev, torch.int32, "teacher_row"))


def _distill_grad_out(desc, logits, dlogits):
    """(dlogits, its pointer), with its row stride in the descriptor"""
    import torch

    if dlogits is None:  # (the descriptor's stride is that of whole rows)
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        return dlogits, dlogits.data_ptr()
    ptr, desc.grad_stride = _rows_ptr(dlogits, desc.rows, desc.vocab, logits.device, "dlogits", logits.dtype)
    return dlogits, ptr


def _loss_out(rows, loss, device):
    """(loss, its pointer)"""
    import torch

    if loss is None:
        loss = torch.empty(rows, dtype=torch.float32, device=device)
        return loss, loss.data_ptr()
    return loss, _vector_ptr(loss, rows, device, torch.float32, "loss")


def _operator_workspace(nbytes, workspace, device, where):
    """(what keeps the workspace alive, its pointer, its size)"""
    import torch

    if workspace is not None:
        if workspace.buffer.device != device:
            raise ValueError("workspace must be on %s" % device)
        return workspace, workspace.ptr, workspace.nbytes
    if nbytes == 0:
        raise SdtwError(STATUS_INVALID_ARG, where)
    buffer = torch.empty(nbytes, dtype=torch.uint8, device=device)  # (aligned to 512 bytes by torch's allocator)
    return buffer, buffer.data_ptr(), nbytes


def sdtw_distill_workspace_bytes(desc):
    return int(load_library().sdtw_distill_workspace_bytes(ctypes.byref(desc)))


@_on_given_stream
def sdtw_distill_forward(logits, teacher_logits, teacher_ids, temperature=1.0, teacher_lse=None, teacher_row=None,
                         loss=None, stats=None, workspace=None):
    """Divergence of every row of ``logits`` [T, V] from the teacher's top logits [R, K] at the tokens ``teacher_ids``
    [R, K] (negative: unused).  Row t goes with the teacher's row ``teacher_row[t]`` (int32; negative: no target), or t.
    The teacher's probabilities are renormalised over the kept tokens, or, with ``teacher_lse`` [R] (float32, the log-sum-exp
    of all of its logits over the temperature), the rest of its mass is held against the student's outside the kept tokens.
    Returns (loss [T] float32, stats); keep stats for :func:`sdtw_distill_backward`."""
    import torch

    lib = load_library()
    desc, args = _distill_args(logits, teacher_logits, teacher_ids, temperature, teacher_lse, teacher_row)
    dev = logits.device
    ref = ctypes.byref(desc)
    keep, wp, wn = _operator_workspace(lib.sdtw_distill_workspace_bytes(ref), workspace, dev, "sdtw_distill_forward")
    loss, lp = _loss_out(desc.rows, loss, dev)
    if stats is None:
        stats = torch.empty((desc.rows, DISTILL_STATS), dtype=torch.float32, device=dev)
        sp = stats.data_ptr()
    else:
        sp = _ptr(stats, torch.float32, (desc.rows, DISTILL_STATS), "stats")
    rc = lib.sdtw_distill_forward(ref, *args, lp, sp, wp, wn, _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_distill_forward")
    return loss, stats


@_on_given_stream
def sdtw_distill_backward(logits, teacher_logits, teacher_ids, stats, grad_loss=None, temperature=1.0, teacher_lse=None,
                          teacher_row=None, dlogits=None):
    """Gradient [T, V] (of the logits' type) of the losses :func:`sdtw_distill_forward` produced, weighted by ``grad_loss``
    [T] (float32; None: ones).  ``dlogits`` may be ``logits`` itself."""
    import torch

    lib = load_library()
    desc, args = _distill_args(logits, teacher_logits, teacher_ids, temperature, teacher_lse, teacher_row)
    dev = logits.device
    dlogits, dp = _distill_grad_out(desc, logits, dlogits)
    rc = lib.sdtw_distill_backward(ctypes.byref(desc), *args, _vector_ptr(grad_loss, desc.rows, dev, torch.float32, "grad_loss"),
                                   _ptr(stats, torch.float32, (desc.rows, DISTILL_STATS), "stats"), dp, _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_distill_backward")
    return dlogits


@_on_given_stream
def sdtw_distill_step(logits, teacher_logits, teacher_ids, grad_loss=None, temperature=1.0, teacher_lse=None,
                      teacher_row=None, loss=None, dlogits=None, workspace=None):
    """Loss and gradient in one call, for a caller who knows ``grad_loss`` beforehand.  Returns (loss [T], dlogits [T, V])."""
    import torch

    lib = load_library()
    desc, args = _distill_args(logits, teacher_logits, teacher_ids, temperature, teacher_lse, teacher_row)
    dev = logits.device
    ref = ctypes.byref(desc)
    keep, wp, wn = _operator_workspace(lib.sdtw_distill_workspace_bytes(ref), workspace, dev, "sdtw_distill_step")
    loss, lp = _loss_out(desc.rows, loss, dev)
    dlogits, dp = _distill_grad_out(desc, logits, dlogits)
    rc = lib.sdtw_distill_step(ref, *args, _vector_ptr(grad_loss, desc.rows, dev, torch.float32, "grad_loss"), lp, dp, wp, wn,
                               _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_distill_step")
    return loss, dlogits


def _bias_args(plane, shape, dtype, device, buckets, max_distance, two_sided, offset, row_len, col_len, name):
    """(descriptor without output and table, pointers of offsets, row_len, col_len)"""
    import torch

    B, H, N, M = shape
    desc = BiasDesc(B, H, N, M, _whole(buckets, _I32, "buckets"), _whole(max_distance, _I32, "max_distance"), 1 if two_sided else 0, 0, 0, 0)
    if plane is not None:
        if plane.dim() != 4 or not plane.is_cuda:
            raise ValueError("%s must be a device tensor [B, H, N, M]" % name)
        if M > 1 and plane.stride(3) != 1:
            raise ValueError("%s must have contiguous rows" % name)
        desc.in_stride[:] = [plane.stride(0), plane.stride(1), plane.stride(2)]
    offsets = None
    if torch.is_tensor(offset):
        offsets = _vector_ptr(offset, B, device, torch.int32, "offset")
    else:
        desc.offset = _whole(offset, _I64, "offset")
    return desc, (offsets, _vector_ptr(row_len, B, device, torch.int32, "row_len"),
                  _vector_ptr(col_len, B, device, torch.int32, "col_len"))


def sdtw_position_bias_starts(buckets, max_distance=128, two_sided=True):
    """First distance of each bucket of a side (host)."""
    buckets = _whole(buckets, _I32, "buckets")
    desc = BiasDesc(1, 1, 1, 1, buckets, _whole(max_distance, _I32, "max_distance"), 1 if two_sided else 0, 0, 0, 0)
    starts = (ctypes.c_int32 * 256)()  # (more buckets are refused)
    rc = load_library().sdtw_position_bias_starts(ctypes.byref(desc), starts)
    if rc != 0:
        raise SdtwError(rc, "sdtw_position_bias_starts")
    return list(starts)[:buckets // 2 if two_sided else buckets]


@_on_given_stream
def sdtw_position_bias_forward(table, plane=None, max_distance=128, two_sided=True, offset=0, row_len=None, col_len=None,
                               out=None):
    """plane [B, H, N, M] + table[h, bucket(j - i - offset)], ``table`` [H, buckets] of any strides (an embedding's transpose).
    ``offset``: a number, or int32 [B]: where every sequence's row 0 stands.  ``row_len``, ``col_len`` [B] int32: cells beyond
    keep what ``plane`` holds.  Without ``plane`` the bias alone goes to ``out``.  ``out`` may be ``plane`` itself."""
    import torch

    lib = load_library()
    if plane is None and out is None:
        raise ValueError("one of plane and out is needed")
    like = plane if plane is not None else out
    if like.dim() != 4 or table.dim() != 2 or not like.is_cuda or table.device != like.device or table.shape[0] != like.shape[1]:
        raise ValueError("plane [B, H, N, M] and table [H, buckets] must be on one device")
    if out is None:
        out = torch.empty(plane.shape, dtype=plane.dtype, device=plane.device)
    elif out.shape != like.shape or out.dtype != like.dtype or out.device != like.device or (out.shape[3] > 1 and out.stride(3) != 1):
        raise ValueError("out must have the shape and type of plane and contiguous rows")
    desc, args = _bias_args(plane, like.shape, like.dtype, like.device, table.shape[1], max_distance, two_sided, offset, row_len,
                            col_len, "plane")
    desc.plane_type, desc.table_type = _type_of(like, "plane"), _type_of(table, "table")
    desc.out_stride[:] = [out.stride(0), out.stride(1), out.stride(2)]
    desc.table_stride[:] = [table.stride(0), table.stride(1)]
    rc = lib.sdtw_position_bias_forward(ctypes.byref(desc), table.data_ptr(), None if plane is None else plane.data_ptr(), *args,
                                        out.data_ptr(), _stream_of(like.device))
    if rc != 0:
        raise SdtwError(rc, "sdtw_position_bias_forward")
    return out


@_on_given_stream
def sdtw_position_bias_backward(grad, buckets, max_distance=128, two_sided=True, offset=0, row_len=None, col_len=None, scale=None,
                                dtable=None, workspace=None):
    """Gradient [H, buckets] (float32) of the table from ``grad`` [B, H, N, M] of the planes (any strides, broadcast ones too),
    each sequence's times ``scale[b]`` (float32 [B]; None: ones)."""
    import torch

    lib = load_library()
    if grad.dim() != 4 or not grad.is_cuda:
        raise ValueError("grad must be a device tensor [B, H, N, M]")
    dev = grad.device
    desc, args = _bias_args(grad, grad.shape, grad.dtype, dev, buckets, max_distance, two_sided, offset, row_len, col_len, "grad")
    desc.plane_type = _type_of(grad, "grad")
    ref = ctypes.byref(desc)
    keep, wp, wn = _operator_workspace(lib.sdtw_position_bias_workspace_bytes(ref), workspace, dev, "sdtw_position_bias_backward")
    if dtable is None:
        dtable = torch.empty((desc.H, desc.buckets), dtype=torch.float32, device=dev)
        dp = dtable.data_ptr()
    else:
        dp = _ptr(dtable, torch.float32, (desc.H, desc.buckets), "dtable")
    rc = lib.sdtw_position_bias_backward(ref, grad.data_ptr(), _vector_ptr(scale, desc.B, dev, torch.float32, "scale"), *args, dp, wp, wn,
                                         _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_position_bias_backward")
    return dtable


def sdtw_biased_workspace_bytes(desc, bias_desc):
    return int(load_library().sdtw_biased_workspace_bytes(ctypes.byref(desc), ctypes.byref(bias_desc)))


def sdtw_forward_biased(x, y, table, gamma, max_distance=128, two_sided=True, offset=0, x_len=None, y_len=None, bandwidth=0,
                        workspace=None, value=None, stream=None, value_only=False, min_memory=False):
    """value[b] = sdtw_gamma(x_b, y_b) with max(0, table[b mod H, bucket(j - i - offset)]) added to the cost of cell (i, j): a
    learned position penalty, ``table`` [H, buckets] of any strides.  Unfused mode.
    Returns (value, state, workspace); keep the last two for :func:`sdtw_backward_biased`."""
    import torch

    lib = load_library()
    desc = _desc_for(x, y, gamma, UNFUSED)
    desc.bandwidth = int(bandwidth)
    desc.flags |= (FLAG_VALUE_ONLY if value_only else 0) | (FLAG_MIN_MEMORY if min_memory else 0)
    dev = x.device
    if not x.is_cuda:
        raise ValueError("x must be a contiguous device tensor")
    if table.dim() != 2 or table.device != dev or table.shape[0] < 1 or desc.B % table.shape[0]:
        raise ValueError("table must be [H, buckets] on the sequences' device, the number of pairs a multiple of H")
    H, buckets = table.shape
    bias = BiasDesc(desc.B // H, H, desc.N, desc.M, buckets, _whole(max_distance, _I32, "max_distance"), 1 if two_sided else 0, TYPE_F32,
                    _type_of(table, "table"), 0, _whole(offset, _I64, "offset"))
    bias.table_stride[:] = [table.stride(0), table.stride(1)]
    if workspace is None:
        nbytes = sdtw_biased_workspace_bytes(desc, bias)
        if nbytes == 0:
            raise SdtwError(STATUS_INVALID_ARG, "sdtw_biased_workspace_bytes")
    with _given_stream(stream, dev):
        handle = _stream_of(dev)
        if workspace is None:
            workspace = Workspace(nbytes, dev)
        if value is None:
            value = torch.empty(desc.B, dtype=torch.float32, device=dev)
        rc = lib.sdtw_forward_biased(ctypes.byref(desc), ctypes.byref(bias), _ptr(x, torch.float32, name="x"),
                                     _ptr(y, torch.float32, name="y"), table.data_ptr(),
                                     _vector_ptr(x_len, desc.B, dev, torch.int32, "x_len"), _vector_ptr(y_len, desc.B, dev, torch.int32, "y_len"),
                                     _ptr(value, torch.float32, (desc.B,), "value"), workspace.ptr, workspace.nbytes, handle)
    if rc != 0:
        raise SdtwError(rc, "sdtw_forward_biased")
    return value, (desc, bias), workspace


def sdtw_backward_biased(state, x, y, table, workspace, grad_value=None, x_len=None, y_len=None, want_E=False, dx=None, dy=None,
                         dtable=None, E=None, stream=None):
    """Gradients of the values :func:`sdtw_forward_biased` produced (same tensors; the table may have another type or layout by now).
    Returns (dx, dy, dtable [H, buckets] float32, E or None)."""
    import torch

    lib = load_library()
    desc, bias = state
    dev = x.device
    if not x.is_cuda:
        raise ValueError("x must be a contiguous device tensor")
    if table.shape != (bias.H, bias.buckets) or table.device != dev:
        raise ValueError("table must be [%d, %d] on %s" % (bias.H, bias.buckets, dev))
    bias = BiasDesc.from_buffer_copy(bias)
    bias.table_type, bias.table_stride[:] = _type_of(table, "table"), table.stride()
    x_shape = (desc.N, desc.D) if desc.x_batch_stride == 0 else (desc.B, desc.N, desc.D)
    y_shape = (desc.M, desc.D) if desc.y_batch_stride == 0 else (desc.B, desc.M, desc.D)
    with _given_stream(stream, dev):
        handle = _stream_of(dev)
        if dx is None:
            dx = torch.empty((desc.B, desc.N, desc.D), dtype=torch.float32, device=dev)
        if dy is None:
            dy = torch.empty((desc.B, desc.M, desc.D), dtype=torch.float32, device=dev)
        if dtable is None:
            dtable = torch.empty((bias.H, bias.buckets), dtype=torch.float32, device=dev)
        if want_E and E is None:
            E = torch.empty((desc.B, desc.N, desc.M), dtype=torch.float32, device=dev)
        rc = lib.sdtw_backward_biased(
            ctypes.byref(desc), ctypes.byref(bias), _ptr(x, torch.float32, x_shape, "x"), _ptr(y, torch.float32, y_shape, "y"), table.data_ptr(),
            _vector_ptr(x_len, desc.B, dev, torch.int32, "x_len"), _vector_ptr(y_len, desc.B, dev, torch.int32, "y_len"),
            _ptr(grad_value, torch.float32, (desc.B,), "grad_value"), _ptr(dx, torch.float32, (desc.B, desc.N, desc.D), "dx"),
            _ptr(dy, torch.float32, (desc.B, desc.M, desc.D), "dy"), _ptr(dtable, torch.float32, (bias.H, bias.buckets), "dtable"),
            _ptr(E, torch.float32, (desc.B, desc.N, desc.M), "E"), workspace.ptr, workspace.nbytes, handle)
    if rc != 0:
        raise SdtwError(rc, "sdtw_backward_biased")
    return dx, dy, dtable, E


def _positions_ptr(t, B, n, device, name):
    if t is None:
        return None
    import torch

    if t.device != device or t.dtype != torch.int32 or t.shape != (B, n) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 [%d, %d] on %s" % (name, B, n, device))
    return t.data_ptr()


# struct sdtw_attention_desc and sdtw_attention_lists, put together at once: field by field takes several times as long
_attention_desc = struct.Struct("=12i2fI4x2q32q2q").pack
_attention_lists = struct.Struct("=6Q").pack
_NO_STRIDES = (0, 0, 0, 0)


def _attention_args(q, k, v, table, scale, cap, causal, max_distance, two_sided, offset, prefix, row_len, col_len, row_document,
                    col_document, out=_NO_STRIDES, dout=_NO_STRIDES, dq=_NO_STRIDES, dk=_NO_STRIDES, dv=_NO_STRIDES):
    """(descriptor, lists or None, pointers of q, k, v, table); `out` and on: the strides of the tensors that a call has beside them"""
    import torch

    if q.dim() != 4 or k.dim() != 4 or not q.is_cuda:
        raise ValueError("q [B, H, N, D] and k, v [B, Hk, M, D] must be device tensors")
    dev, dtype, (B, H, N, D), (_, Hk, M, _) = q.device, q.dtype, q.shape, k.shape
    if k.shape != (B, Hk, M, D) or v.shape != k.shape or k.device != dev or v.device != dev or k.dtype != dtype or v.dtype != dtype:
        raise ValueError("k and v must be [B, Hk, M, D] with q's B and D, on its device and of its type")
    if Hk < 1 or H % Hk:
        raise ValueError("the number of q's heads must be a multiple of that of k's")
    if max(B, H, N, M, D) >= _I32:
        raise ValueError("a dimension is too large")
    table_type = buckets = 0
    tp, table_strides = None, (0, 0)
    if table is not None:
        if table.dim() != 2 or table.shape[0] != H or table.device != dev:
            raise ValueError("table must be [%d, buckets] on %s" % (H, dev))
        buckets = table.shape[1]
        if not 1 <= buckets < _I32:
            raise ValueError("table must have buckets")
        table_type, table_strides, tp = _type_of(table, "table"), table.stride(), table.data_ptr()
        max_distance = _whole(max_distance, _I32, "max_distance")
    else:
        max_distance = two_sided = 0
    lists = [0, 0, 0, 0, 0, 0]
    if torch.is_tensor(offset):
        lists[0] = _vector_ptr(offset, B, dev, torch.int32, "offset")
        offset = 0
    else:
        offset = _whole(offset, _I64, "offset")
    if prefix is None:
        prefix = 0
    else:
        if not causal:
            raise ValueError("a prefix belongs to a causal mask")
        if torch.is_tensor(prefix):
            lists[1] = _vector_ptr(prefix, B, dev, torch.int32, "prefix")
            prefix = 0
        else:
            prefix = _whole(prefix, _I64, "prefix")
    if row_len is not None:
        lists[2] = _vector_ptr(row_len, B, dev, torch.int32, "row_len")
    if col_len is not None:
        lists[3] = _vector_ptr(col_len, B, dev, torch.int32, "col_len")
    if (row_document is None) != (col_document is None):
        raise ValueError("row_document and col_document go together")
    if row_document is not None:
        lists[4] = _positions_ptr(row_document, B, N, dev, "row_document")
        lists[5] = _positions_ptr(col_document, B, M, dev, "col_document")
    try:
        desc = _attention_desc(B, H, Hk, N, M, D, _type_of(q, "q"), table_type, buckets, max_distance, 1 if two_sided else 0, 1 if causal else 0,
                               max(D, 1) ** -0.5 if scale is None else scale, cap, 0, offset, prefix, *q.stride(), *k.stride(), *v.stride(), *out, *dout,
                               *dq, *dk, *dv, *table_strides)
    except (OverflowError, struct.error):
        raise ValueError("scale and cap must be float32 numbers") from None
    return desc, _attention_lists(*lists) if any(lists) else None, (q.data_ptr(), k.data_ptr(), v.data_ptr(), tp)


def _like(given, like, name):
    """(a tensor as ``like``, with contiguous features)"""
    import torch

    if like.dim() != 4:
        raise ValueError("q [B, H, N, D] and k, v [B, Hk, M, D] must be device tensors")
    if given is None:
        given = torch.empty_like(like)  # (the same order of dimensions in memory)
        return given if given.shape[3] <= 1 or given.stride(3) == 1 else torch.empty(like.shape, dtype=like.dtype, device=like.device)
    if given.shape != like.shape or given.dtype != like.dtype or given.device != like.device:
        raise ValueError("%s must be %s of %s on %s" % (name, tuple(like.shape), like.dtype, like.device))
    return given


@_on_given_stream
def sdtw_attention_forward(q, k, v, table=None, scale=None, cap=0.0, causal=False, max_distance=128, two_sided=True, offset=0, prefix=None,
                           row_len=None, col_len=None, row_document=None, col_document=None, out=None, lse=None, workspace=None):
    """Softmax attention of ``q`` [B, H, N, D] over ``k``, ``v`` [B, Hk, M, D] (any strides; H a multiple of Hk: heads share keys
    in groups; D <= 128).  Scores are ``scale`` (None: 1 / sqrt(D)) times the products, ``cap`` > 0: cap * tanh(score / cap), plus
    ``table`` [H, buckets] by the distance j - i - offset as in :func:`sdtw_position_bias_forward`.
    Row i sees the keys j < col_len[b]; ``causal``: of these, j <= i + offset or j < ``prefix``; with documents (int32
    [B, N] and [B, M], negative: none) those of its own.  ``offset`` and ``prefix``: numbers, or int32 [B].
    One new token per sequence against a cache: N = 1, ``offset`` = its position, ``causal``.
    Returns (out [B, H, N, D], lse [B, H, N] float32): 0 and -inf for a row that sees nothing or lies behind ``row_len``."""
    import torch

    lib = load_library()
    dev = q.device
    out = _like(out, q, "out")
    desc, lists, args = _attention_args(q, k, v, table, scale, cap, causal, max_distance, two_sided, offset, prefix, row_len, col_len,
                                        row_document, col_document, out.stride())
    keep, wp, wn = _operator_workspace(lib.sdtw_attention_forward_workspace_bytes(desc), workspace, dev, "sdtw_attention_forward")
    if lse is None:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=dev)
        lp = lse.data_ptr()
    else:
        lp = _ptr(lse, torch.float32, q.shape[:3], "lse", dev)
    rc = lib.sdtw_attention_forward(desc, *args, lists, out.data_ptr(), lp, wp, wn, _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_attention_forward")
    return out, lse


@_on_given_stream
def sdtw_attention_backward(q, k, v, out, lse, dout, table=None, scale=None, cap=0.0, causal=False, max_distance=128, two_sided=True,
                            offset=0, prefix=None, row_len=None, col_len=None, row_document=None, col_document=None, want_dtable=True,
                            dq=None, dk=None, dv=None, dtable=None, workspace=None):
    """Gradients of what :func:`sdtw_attention_forward` returned as ``out`` and ``lse`` (the same tensors and options), from ``dout``
    [B, H, N, D] of any strides, broadcast ones too.  Returns (dq, dk, dv, dtable [H, buckets] float32, or None without a
    table or with ``want_dtable=False``)."""
    import torch

    lib = load_library()
    dev = q.device
    for t, name in ((out, "out"), (dout, "dout")):
        if t.shape != q.shape or t.dtype != q.dtype or t.device != dev:
            raise ValueError("%s must be %s of %s on %s" % (name, tuple(q.shape), q.dtype, dev))
    dq, dk, dv = _like(dq, q, "dq"), _like(dk, k, "dk"), _like(dv, v, "dv")
    desc, lists, args = _attention_args(q, k, v, table, scale, cap, causal, max_distance, two_sided, offset, prefix, row_len, col_len,
                                        row_document, col_document, out.stride(), dout.stride(), dq.stride(), dk.stride(), dv.stride())
    dp = None
    if table is None or not want_dtable:
        dtable = None
    elif dtable is None:
        dtable = torch.empty(table.shape, dtype=torch.float32, device=dev)
        dp = dtable.data_ptr()
    else:
        dp = _ptr(dtable, torch.float32, table.shape, "dtable", dev)
    keep, wp, wn = _operator_workspace(lib.sdtw_attention_backward_workspace_bytes(desc), workspace, dev, "sdtw_attention_backward")
    rc = lib.sdtw_attention_backward(desc, *args, lists, out.data_ptr(), _ptr(lse, torch.float32, q.shape[:3], "lse", dev), dout.data_ptr(),
                                     dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dp, wp, wn, _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_attention_backward")
    return dq, dk, dv, dtable


def _tensor_types(tensors, name):
    kinds = {t.dtype for t in tensors}
    if len(kinds) == 1:
        return [_type_of(tensors[0], name)] * len(tensors)
    return [_type_of(t, name) for t in tensors]


def _without_gaps(t):
    """Whether the elements fill their memory, in whatever order of the dimensions."""
    span = 1
    for size, stride in sorted(((n, s) for n, s in zip(t.shape, t.stride()) if n != 1), key=lambda x: x[1]):
        if stride != span:
            return t.numel() == 0
        span *= size
    return True


@_on_given_stream
def sdtw_gradient_clip(grads, max_norm, out=None, norm=None, workspace=None):
    """Scales the tensors ``grads`` (a sequence; float32, float16 and bfloat16 mixed, any of them empty) down so that all of their elements
    together have a 2-norm of at most ``max_norm``, in place or into the tensors ``out``: as many elements each, of any of the types.
    If the norm is not finite they stay as they are.  A tensor's elements fill its memory; one that does so in another order
    than its shape's goes with an ``out`` of its strides.  No tensor may stand in the list twice.
    Returns the norm before, a float32 scalar on the device: nothing waits for it.  It is not finite only if an element is not."""
    import torch

    lib = load_library()
    grads = list(grads)
    outs = grads if out is None else list(out)
    n = len(grads)
    if len(outs) != n:
        raise ValueError("out must have a tensor for each of grads")
    if n == 0 and norm is None:
        raise ValueError("without gradients norm has to be given: its device is not known otherwise")
    dev = (grads[0] if n else norm).device
    if dev.type != "cuda" or any(set(map(torch.Tensor.get_device, x)) - {dev.index} for x in (grads, outs)):
        raise ValueError("the gradients must be on one device")
    counts = list(map(torch.Tensor.numel, grads))
    if outs is not grads and counts != list(map(torch.Tensor.numel, outs)):
        raise ValueError("out must have as many elements as the gradients")
    for k in range(n) if not all(map(torch.Tensor.is_contiguous, grads)) or not all(map(torch.Tensor.is_contiguous, outs)) else ():
        g, o = grads[k], outs[k]
        if g.is_contiguous() and o.is_contiguous():
            continue
        if g.shape != o.shape or not _without_gaps(g) or any(a != b for a, b, m in zip(g.stride(), o.stride(), g.shape) if m != 1):
            raise ValueError("a gradient's elements must fill its memory, and its out must have the same strides")
    # struct sdtw_gradient as four 64-bit words
    words = array.array("q", bytes(32 * n))
    words[0::4] = array.array("q", map(torch.Tensor.data_ptr, grads))
    words[1::4] = words[0::4] if outs is grads else array.array("q", map(torch.Tensor.data_ptr, outs))
    words[2::4] = array.array("q", counts)
    kinds = _tensor_types(grads, "grads") if n else []
    out_kinds = kinds if outs is grads else _tensor_types(outs, "out") if n else []
    words[3::4] = array.array("q", [a | b << 32 for a, b in zip(kinds, out_kinds)])
    ptr = words.buffer_info()[0] if n else None
    keep, wp, wn = _operator_workspace(lib.sdtw_gradient_clip_workspace_bytes(ptr, n), workspace, dev, "sdtw_gradient_clip")
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=dev)
    np = _ptr(norm, torch.float32, (), "norm", dev)
    rc = lib.sdtw_gradient_clip(ptr, n, max_norm, np, wp, wn, _stream_of(dev))
    if rc != 0:
        raise SdtwError(rc, "sdtw_gradient_clip")
    return norm


def sdtw_gradient_norm(grads, norm=None, workspace=None, stream=None):
    """The 2-norm of all elements of the tensors ``grads`` together, a float32 scalar on the device.  They are only read."""
    return sdtw_gradient_clip(grads, float("inf"), norm=norm, workspace=workspace, stream=stream)
