"""ctypes binding with the same names as the C ABI in include/la.h.

Argument marshalling only; for calls on plain tensors without a trace it is done in native code
(csrc/la_bind.cpp, _marshal.so), by the same rules.  There is no CPU fallback: if libla.so has not been
built, loading fails with an error that says how to build it.
"""
import ctypes
import importlib.util
import os
import sys
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libla.so")
_MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")
_lib = None
_native = None  # the module of _marshal.so once the library is loaded

LA_F32 = 0
LA_BF16 = 1
LA_E4M3 = 2
LA_I8 = 3

LA_GATE_VALUE = 0
LA_GATE_SIGMOID = 1

LA_MAX_TRACE = 8

EXPORTS = ("la_version", "la_status_string", "la_workspace_bytes", "la_forward", "la_backward",
           "la_forward_traced", "la_backward_traced", "la_saved_state_bytes", "la_forward_save",
           "la_backward_saved", "la_debug_override", "la_forward_static", "la_decode_state_bytes",
           "la_decode_step", "la_decode_prefill", "la_backward_ab", "la_forward_qknorm",
           "la_backward_qknorm", "la_forward_qknorm_save", "la_backward_qknorm_saved",
           "la_recurrence_workspace_bytes", "la_recurrence_forward", "la_recurrence_backward",
           "la_recurrence_step", "la_pack_rows", "la_pack_tensors", "la_unpack_rows", "la_rmsnorm_workspace_bytes",
           "la_rmsnorm_forward", "la_rmsnorm_backward")


class la_trace(ctypes.Structure):
    """struct la_trace of include/la.h."""
    _fields_ = [("events", ctypes.POINTER(ctypes.c_void_p)),
                ("capacity", ctypes.c_int),
                ("recorded", ctypes.c_int),
                ("names", ctypes.c_char_p * LA_MAX_TRACE)]


class LaError(RuntimeError):
    def __init__(self, code, where):
        self.code = int(code)
        super().__init__("%s failed: %s" % (where, la_status_string(code)))


def library_path():
    return _LIB_PATH


def load_library():
    """Load libla.so (built by paper_2510_21956_amd/build.py).  Raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            "HIP library %s not found; build it with "
            "`python -c 'import __graft_entry__ as g; g.build()'` "
            "(or python paper_2510_21956_amd/build.py).  There is no CPU fallback." % _LIB_PATH)
    lib = ctypes.CDLL(_LIB_PATH)
    vp, sz, i, f = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
    lib.la_version.restype = i
    lib.la_version.argtypes = []
    lib.la_status_string.restype = ctypes.c_char_p
    lib.la_status_string.argtypes = [i]
    lib.la_workspace_bytes.restype = sz
    lib.la_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
    lib.la_forward.restype = i
    lib.la_forward.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, f, f, i, i, vp, sz, vp]
    lib.la_backward.restype = i
    lib.la_backward.argtypes = [vp] * 9 + [i, i, i, i, f, f, i, i, vp, sz, vp]
    tp = ctypes.POINTER(la_trace)
    lib.la_forward_traced.restype = i
    lib.la_forward_traced.argtypes = lib.la_forward.argtypes + [tp]
    lib.la_backward_traced.restype = i
    lib.la_backward_traced.argtypes = lib.la_backward.argtypes + [tp]
    lib.la_saved_state_bytes.restype = sz
    lib.la_saved_state_bytes.argtypes = [i, i, i, i, i, i]
    lib.la_forward_save.restype = i
    lib.la_forward_save.argtypes = lib.la_forward.argtypes[:-1] + [vp, sz, vp, tp]
    lib.la_backward_saved.restype = i
    lib.la_backward_saved.argtypes = lib.la_backward.argtypes[:-1] + [vp, sz, vp, tp]
    lib.la_forward_static.restype = i
    lib.la_forward_static.argtypes = lib.la_forward.argtypes[:-3] + [vp]
    lib.la_decode_state_bytes.restype = sz
    lib.la_decode_state_bytes.argtypes = [i, i, i]
    lib.la_decode_step.restype = i
    lib.la_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, sz, i, i, i, i, f, f, i, vp]
    lib.la_decode_prefill.restype = i
    lib.la_decode_prefill.argtypes = [vp, vp, vp, sz, i, i, i, i, i, i, vp, sz, vp]
    lib.la_forward_qknorm.restype = i
    lib.la_forward_qknorm.argtypes = lib.la_forward_traced.argtypes
    lib.la_backward_qknorm.restype = i
    lib.la_backward_qknorm.argtypes = lib.la_backward_traced.argtypes
    lib.la_forward_qknorm_save.restype = i
    lib.la_forward_qknorm_save.argtypes = lib.la_forward_save.argtypes
    lib.la_backward_qknorm_saved.restype = i
    lib.la_backward_qknorm_saved.argtypes = lib.la_backward_saved.argtypes
    lib.la_backward_ab.restype = i
    lib.la_backward_ab.argtypes = [vp] * 7 + [i, i, i, i, f, f, i, i, vp, sz, vp]
    lib.la_recurrence_workspace_bytes.restype = sz
    lib.la_recurrence_workspace_bytes.argtypes = [i] * 5
    lib.la_recurrence_forward.restype = i
    lib.la_recurrence_forward.argtypes = [vp] * 6 + [i] * 5 + [vp, sz, vp]
    lib.la_recurrence_backward.restype = i
    lib.la_recurrence_backward.argtypes = [vp] * 10 + [i] * 5 + [vp, sz, vp]
    lib.la_recurrence_step.restype = i
    lib.la_recurrence_step.argtypes = [vp] * 4 + [i] * 5 + [vp]
    lib.la_pack_rows.restype = i
    lib.la_pack_rows.argtypes = [vp, vp, vp, sz, i, i, i, vp]
    lib.la_pack_tensors.restype = i
    lib.la_pack_tensors.argtypes = [i, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), sz, i, i, i, vp]
    lib.la_unpack_rows.restype = i
    lib.la_unpack_rows.argtypes = [vp, vp, vp, sz, i, i, i, vp]
    lib.la_rmsnorm_workspace_bytes.restype = sz
    lib.la_rmsnorm_workspace_bytes.argtypes = [sz, i]
    lib.la_rmsnorm_forward.restype = i
    lib.la_rmsnorm_forward.argtypes = [vp] * 9 + [sz, i, f, i, i, i, i, vp]
    lib.la_rmsnorm_backward.restype = i
    lib.la_rmsnorm_backward.argtypes = [vp] * 8 + [sz, i, i, i, i, vp, sz, vp]
    lib.la_debug_override.restype = None
    lib.la_debug_override.argtypes = [i, i]
    _lib = lib
    _load_native(lib)
    return lib


def _load_native(lib):
    """The native marshalling, if there is one that fits; a file that does not load, or that was built for
    another torch or Python (whose tensors it would misread), is reported and left out: the Python functions
    below do all of it."""
    global _native
    if not os.path.exists(_MARSHAL_PATH):
        return
    try:
        _native = _open_native(lib)
    except Exception as e:
        warnings.warn("%s is not used, calls take a few microseconds longer: %s" % (_MARSHAL_PATH, e),
                      RuntimeWarning, stacklevel=3)


def _open_native(lib):
    spec = importlib.util.spec_from_file_location("_marshal", _MARSHAL_PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    here = "torch %s, Python %d.%d" % (torch.__version__, *sys.version_info[:2])
    if getattr(module, "built_for", None) != here:
        raise ImportError("built for %s, not for %s" % (getattr(module, "built_for", "another version"), here))
    from . import autograd  # imports this module; by the first call both are there
    module.init(autograd.python_backward, _device_stream, *(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.la_forward_traced, lib.la_forward_qknorm, lib.la_forward_save, lib.la_forward_qknorm_save,
        lib.la_backward_traced, lib.la_backward_qknorm, lib.la_backward_saved,
        lib.la_backward_qknorm_saved, lib.la_decode_step, lib.la_decode_prefill, lib.la_workspace_bytes,
        lib.la_saved_state_bytes)))
    module.init_layer(autograd.recurrence_backward, autograd.norm_backward, autograd.checkpointed_backward, *(
        ctypes.cast(f, ctypes.c_void_p).value for f in (
            lib.la_recurrence_workspace_bytes, lib.la_recurrence_forward, lib.la_recurrence_backward, lib.la_recurrence_step,
            lib.la_pack_tensors, lib.la_unpack_rows, lib.la_rmsnorm_workspace_bytes, lib.la_rmsnorm_forward,
            lib.la_rmsnorm_backward, lib.la_forward_traced, lib.la_forward_qknorm, lib.la_forward_save,
            lib.la_forward_qknorm_save, lib.la_backward_saved, lib.la_backward_qknorm_saved, lib.la_workspace_bytes,
            lib.la_saved_state_bytes)))
    return module


def la_version():
    return int(load_library().la_version())


def la_status_string(code):
    return load_library().la_status_string(int(code)).decode()


def la_debug_override(seg_len=0, force_generic=0):
    """la_debug_override of include/la.h (test / profiling hook; 0, 0 = automatic)."""
    load_library().la_debug_override(int(seg_len), int(bool(force_generic)))


def _dtype_code(t):
    if t.dtype == torch.float32:
        return LA_F32
    if t.dtype == torch.bfloat16:
        return LA_BF16
    raise TypeError("Q/K/V must be float32 or bfloat16, got %s" % t.dtype)


def la_workspace_bytes(B, H, N, D, dt, causal, is_backward):
    """is_backward: 0 forward, 1 backward, 2 backward that recomputes O / G (given as None)."""
    return int(load_library().la_workspace_bytes(B, H, N, D, dt, int(bool(causal)),
                                                 int(is_backward)))


def la_saved_state_bytes(B, H, N, D, dt, causal):
    return int(load_library().la_saved_state_bytes(B, H, N, D, dt, int(bool(causal))))


# A small call (a decode step, a toy layer) cost more in this file than on the GPU: a decode step of 128
# slices at D = 128, whose kernel takes 4.6 us, 7.4 us with the functions below and 4.8 us with the native
# ones, which return None for what they leave to these (other objects than tensors, a missing tensor, whatever
# is to be refused).
# What is done per tensor and per call is kept to integers: device indices, raw stream handles and
# addresses, which ctypes converts by the declared argument types.

def _check_tensors(ref, *ts):
    """Every tensor of a call, the first one included, is packed and on ref's device: the
    kernels read B*H*N*D elements from its address, whatever its strides say."""
    dev = ref.get_device()
    if not ref.is_cuda or not ref.is_contiguous():
        raise ValueError("tensors must be contiguous device tensors")
    for t in ts:
        if t is None:
            continue
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous device tensors")
        if t.get_device() != dev:
            raise ValueError("tensors must live on one device")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _device_stream(index):
    """hipStream_t of the current stream of device ``index``."""
    if _raw_stream is not None:
        return _raw_stream(index)
    return torch.cuda.current_stream(index).cuda_stream


def _stream_ptr(stream, ref):
    """hipStream_t of ``stream``, or of the current stream of ref's device."""
    if stream is not None:
        return stream.cuda_stream
    return _device_stream(ref.get_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def la_forward(Q, K, V, O, G, a, b, causal, workspace, stream=None):
    """la_forward of include/la.h on torch device tensors.

    Q, K, V, O: [B, H, N, D] float32 or bfloat16; G: [B, H, N] float32;
    workspace: uint8 device tensor of at least la_workspace_bytes(..., 0) bytes."""
    la_forward_traced(Q, K, V, O, G, a, b, causal, workspace, stream, None)


LA_STATIC_SCRATCH_BYTES = 32 << 20


def la_forward_static(Q, K, V, O, G, a, b, causal, stream=None):
    """la_forward_static of include/la.h: la_forward with the library's own static scratch."""
    if Q.dim() != 4:
        raise ValueError("Q must be [B, H, N, D]")
    B, H, N, D = Q.shape
    _check_tensors(Q, K, V, O, G)
    if K.shape != Q.shape or V.shape != Q.shape or O.shape != Q.shape:
        raise ValueError("shape mismatch")
    if not (K.dtype == V.dtype == O.dtype == Q.dtype):
        raise TypeError("dtype mismatch")
    if G is not None and (G.shape != Q.shape[:3] or G.dtype != torch.float32):
        raise ValueError("G must be [B, H, N] float32 (or None)")
    rc = load_library().la_forward_static(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(G), B, H, N, D,
                                          float(a), float(b), int(bool(causal)), _dtype_code(Q),
                                          _stream_ptr(stream, Q))
    if rc != 0:
        raise LaError(rc, "la_forward_static")


def la_forward_traced(Q, K, V, O, G, a, b, causal, workspace, stream=None, trace=None):
    """la_forward_traced of include/la.h; ``trace`` is a la_trace structure or None."""
    _forward(Q, K, V, O, G, a, b, causal, workspace, None, stream, trace, False)


def la_forward_save(Q, K, V, O, G, a, b, causal, workspace, saved, stream=None, trace=None):
    """la_forward_save of include/la.h; ``saved`` is a uint8 device tensor of at least
    la_saved_state_bytes(...) bytes (None when that is 0)."""
    _forward(Q, K, V, O, G, a, b, causal, workspace, saved, stream, trace, True)


def _saved_args(saved, ref):
    if saved is None:
        return None, 0
    _check_tensors(ref, saved)
    return _ptr(saved), saved.numel() * saved.element_size()


_KIND = {False: 0, True: 1, "qknorm": 2, "qknorm_save": 3}


def _forward(Q, K, V, O, G, a, b, causal, workspace, saved, stream, trace, save):
    if _native is not None and trace is None:
        rc = _native.forward(_KIND[save], Q, K, V, O, G, a, b, causal, workspace, saved, stream)
        if rc == 0:
            return
        if rc is not None:
            raise LaError(rc, "la_forward_save" if save else "la_forward")
    if Q.dim() != 4:
        raise ValueError("Q must be [B, H, N, D]")
    shape = Q.shape
    B, H, N, D = shape
    _check_tensors(Q, K, V, O, G, workspace)
    if K.shape != shape or V.shape != shape or O.shape != shape:
        raise ValueError("shape mismatch")
    if not (K.dtype == V.dtype == O.dtype == Q.dtype):
        raise TypeError("dtype mismatch")
    if G is not None and (G.shape != Q.shape[:3] or G.dtype != torch.float32):
        raise ValueError("G must be [B, H, N] float32 (or None)")
    lib = load_library()
    head = (_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(G), B, H, N, D, float(a), float(b),
            int(bool(causal)), _dtype_code(Q), _ptr(workspace),
            workspace.numel() * workspace.element_size())
    tr = ctypes.byref(trace) if trace is not None else None
    if save == "qknorm":
        rc = lib.la_forward_qknorm(*head, _stream_ptr(stream, Q), tr)
    elif save == "qknorm_save":
        sp, sb = _saved_args(saved, Q)
        rc = lib.la_forward_qknorm_save(*head, sp, sb, _stream_ptr(stream, Q), tr)
    elif save:
        sp, sb = _saved_args(saved, Q)
        rc = lib.la_forward_save(*head, sp, sb, _stream_ptr(stream, Q), tr)
    else:
        rc = lib.la_forward_traced(*head, _stream_ptr(stream, Q), tr)
    if rc != 0:
        raise LaError(rc, "la_forward_save" if save else "la_forward")


def la_backward(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, stream=None):
    """la_backward of include/la.h on torch device tensors (see la_forward)."""
    la_backward_traced(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, stream, None)


def la_backward_traced(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, stream=None,
                       trace=None):
    """la_backward_traced of include/la.h; ``trace`` is a la_trace structure or None."""
    _backward(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, None, stream, trace, False)


def la_backward_saved(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, saved, stream=None,
                      trace=None):
    """la_backward_saved of include/la.h; ``saved`` as filled by la_forward_save."""
    _backward(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, saved, stream, trace, True)


def _backward(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, saved, stream, trace,
              use_saved):
    if _native is not None and trace is None:
        rc = _native.backward(_KIND[use_saved], Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace,
                              saved, stream)
        if rc == 0:
            return
        if rc is not None:
            raise LaError(rc, "la_backward_saved" if use_saved else "la_backward")
    if Q.dim() != 4:
        raise ValueError("Q must be [B, H, N, D]")
    B, H, N, D = Q.shape
    _check_tensors(Q, K, V, O, G, dO, dQ, dK, dV, workspace)
    for name, t in (("K", K), ("V", V), ("O", O), ("dO", dO), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        if t is None:
            if name == "O":
                continue  # recomputed inside the call
            raise ValueError("%s is required" % name)
        if t.shape != Q.shape:
            raise ValueError("shape mismatch")
        if t.dtype != Q.dtype:
            raise TypeError("dtype mismatch")
    if G is not None and (G.shape != Q.shape[:3] or G.dtype != torch.float32):
        raise ValueError("G must be [B, H, N] float32 (or None)")
    lib = load_library()
    head = (_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(G), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
            B, H, N, D, float(a), float(b), int(bool(causal)), _dtype_code(Q), _ptr(workspace),
            workspace.numel() * workspace.element_size())
    tr = ctypes.byref(trace) if trace is not None else None
    if use_saved == "qknorm":
        rc = lib.la_backward_qknorm(*head, _stream_ptr(stream, Q), tr)
    elif use_saved == "qknorm_save":
        sp, sb = _saved_args(saved, Q)
        rc = lib.la_backward_qknorm_saved(*head, sp, sb, _stream_ptr(stream, Q), tr)
    elif use_saved:
        sp, sb = _saved_args(saved, Q)
        rc = lib.la_backward_saved(*head, sp, sb, _stream_ptr(stream, Q), tr)
    else:
        rc = lib.la_backward_traced(*head, _stream_ptr(stream, Q), tr)
    if rc != 0:
        raise LaError(rc, "la_backward_saved" if use_saved else "la_backward")


def attention(Q, K, V, a, b, causal, normalize):
    """O of linear_attention (autograd.py) through the autograd node in native code; None where that is left to
    the Python one."""
    if _native is None:
        load_library()
        if _native is None:
            return None
    O = _native.attention(Q, K, V, a, b, causal, normalize)
    if type(O) is int:
        raise LaError(O, "la_forward_save")
    return O


def la_decode_state_bytes(B, H, D):
    return int(load_library().la_decode_state_bytes(B, H, D))


def la_decode_step(q, k, v, o, g, state, a, b, stream=None):
    """la_decode_step of include/la.h: q, k, v, o [B, H, T, D]; g [B, H, T] float32 or None;
    state: float32 device tensor of la_decode_state_bytes(B, H, D) bytes, updated in place."""
    if _native is not None:
        rc = _native.decode_step(q, k, v, o, g, state, a, b, stream)
        if rc == 0:
            return
        if rc is not None:
            raise LaError(rc, "la_decode_step")
    if q.dim() != 4:
        raise ValueError("q must be [B, H, T, D]")
    shape = q.shape
    B, H, T, D = shape
    _check_tensors(q, k, v, o, g, state)
    if k.shape != shape or v.shape != shape or o.shape != shape:
        raise ValueError("shape mismatch")
    if not (k.dtype == v.dtype == o.dtype == q.dtype) or state.dtype != torch.float32:
        raise TypeError("dtype mismatch")
    if g is not None and (g.shape != q.shape[:3] or g.dtype != torch.float32):
        raise ValueError("g must be [B, H, T] float32 (or None)")
    rc = load_library().la_decode_step(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(g), _ptr(state),
                                       state.numel() * 4, B, H, T, D, float(a), float(b),
                                       _dtype_code(q), _stream_ptr(stream, q))
    if rc != 0:
        raise LaError(rc, "la_decode_step")


def la_decode_prefill(K, V, state, accumulate, workspace, stream=None):
    """la_decode_prefill of include/la.h: K, V [B, H, N, D]."""
    if _native is not None:
        rc = _native.decode_prefill(K, V, state, accumulate, workspace, stream)
        if rc == 0:
            return
        if rc is not None:
            raise LaError(rc, "la_decode_prefill")
    if K.dim() != 4:
        raise ValueError("K must be [B, H, N, D]")
    B, H, N, D = K.shape
    _check_tensors(K, V, state, workspace)
    if V.shape != K.shape or V.dtype != K.dtype or state.dtype != torch.float32:
        raise ValueError("shape or dtype mismatch")
    rc = load_library().la_decode_prefill(_ptr(K), _ptr(V), _ptr(state), state.numel() * 4, B, H,
                                          N, D, _dtype_code(K), int(bool(accumulate)),
                                          _ptr(workspace),
                                          workspace.numel() * workspace.element_size(),
                                          _stream_ptr(stream, K))
    if rc != 0:
        raise LaError(rc, "la_decode_prefill")


def la_backward_ab(Q, K, V, O, G, dO, dab, a, b, causal, workspace, stream=None):
    """la_backward_ab of include/la.h; ``dab``: float32 device tensor of two elements."""
    if Q.dim() != 4:
        raise ValueError("Q must be [B, H, N, D]")
    B, H, N, D = Q.shape
    _check_tensors(Q, K, V, O, G, dO, dab, workspace)
    for t in (K, V, O, dO):
        if t.shape != Q.shape or t.dtype != Q.dtype:
            raise ValueError("shape or dtype mismatch")
    if G.shape != Q.shape[:3] or G.dtype != torch.float32:
        raise ValueError("G must be [B, H, N] float32")
    if dab.dtype != torch.float32 or dab.numel() < 2:
        raise ValueError("dab must hold two float32")
    rc = load_library().la_backward_ab(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(G), _ptr(dO),
                                       _ptr(dab), B, H, N, D, float(a), float(b),
                                       int(bool(causal)), _dtype_code(Q), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(),
                                       _stream_ptr(stream, Q))
    if rc != 0:
        raise LaError(rc, "la_backward_ab")


def la_forward_qknorm(Q, K, V, O, G, a, b, causal, workspace, stream=None, trace=None):
    """la_forward_qknorm of include/la.h: la_forward on raw Q, K, normalised row by row inside."""
    _forward(Q, K, V, O, G, a, b, causal, workspace, None, stream, trace, "qknorm")


def la_backward_qknorm(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, stream=None,
                       trace=None):
    """la_backward_qknorm of include/la.h: gradients for the raw Q, K."""
    _backward(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, None, stream, trace,
              "qknorm")


def la_forward_qknorm_save(Q, K, V, O, G, a, b, causal, workspace, saved, stream=None, trace=None):
    """la_forward_qknorm_save of include/la.h (``saved`` as for la_forward_save)."""
    _forward(Q, K, V, O, G, a, b, causal, workspace, saved, stream, trace, "qknorm_save")


def la_backward_qknorm_saved(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, saved,
                             stream=None, trace=None):
    """la_backward_qknorm_saved of include/la.h; ``saved`` as filled by la_forward_qknorm_save."""
    _backward(Q, K, V, O, G, dO, dQ, dK, dV, a, b, causal, workspace, saved, stream, trace,
              "qknorm_save")


# ---- the operators around the attention ---------------------------------------------------------

def _call(name, ref, stream, written, *args):
    """Calls the entry point with the stream behind its arguments, on ref's device.  `written`: the tensors that it
    writes, which autograd has to know of: a node that saved one of them must not go on with the new values."""
    f = getattr(load_library(), name)
    index = ref.get_device()
    if torch.cuda.current_device() == index:
        rc = f(*args, _stream_ptr(stream, ref))
    else:
        with torch.cuda.device(index):
            rc = f(*args, _stream_ptr(stream, ref))
    if rc != 0:
        raise LaError(rc, name)
    torch.autograd.graph.increment_version([t for t in written if t is not None and not t.is_inference()])


def _room(t):
    return (None, 0) if t is None else (_ptr(t), t.numel() * t.element_size())


def _like(ref, **ts):
    """Every tensor given has ref's shape and type."""
    for name, t in ts.items():
        if t is None:
            continue
        if t.shape != ref.shape:
            raise ValueError("%s must be %s, got %s" % (name, tuple(ref.shape), tuple(t.shape)))
        if t.dtype != ref.dtype:
            raise TypeError("%s must be %s, got %s" % (name, ref.dtype, t.dtype))


def _needed(**ts):
    for name, t in ts.items():
        if t is None:
            raise ValueError("%s is required" % name)


def _real_code(t):
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("tensors must be float32 or bfloat16, got %s" % t.dtype)
    return LA_F32 if t.dtype == torch.float32 else LA_BF16


_INTS = 1 << 31  # what the library's sizes stay below; ctypes would cut larger ones off


def _fit(**sizes):
    for name, n in sizes.items():
        if n >= _INTS:
            raise ValueError("%s must be less than 2^31, got %d" % (name, n))


def la_recurrence_workspace_bytes(B, N, C, dt, is_backward):
    if max(B, N, C) >= _INTS:
        return 0
    return int(load_library().la_recurrence_workspace_bytes(B, N, C, dt, int(bool(is_backward))))


def _sequences(x, **states):
    """B, N, C of x [..., N, C]; states are float32 of one row a sequence."""
    if x.dim() < 2:
        raise ValueError("x must be [..., N, C]")
    N, C = x.shape[-2:]
    for name, t in states.items():
        if t is not None and (t.shape != x.shape[:-2] + x.shape[-1:] or t.dtype != torch.float32):
            raise ValueError("%s must be float32 %s" % (name, tuple(x.shape[:-2] + x.shape[-1:])))
    B = x.numel() // (N * C) if x.numel() else 0
    _fit(B=B, N=N, C=C)
    return B, N, C


def _lengths_ptr(lengths, x):
    if lengths is None:
        return None
    if lengths.dtype != torch.int32 or lengths.shape != x.shape[:-2]:
        raise ValueError("lengths must be int32 %s" % (tuple(x.shape[:-2]),))
    return _ptr(lengths)


def la_recurrence_forward(x, gates, h0, h, last, lengths, gate, workspace, stream=None):
    """la_recurrence_forward of include/la.h: x, gates, h [..., N, C] float32 or bfloat16; h0, last
    [..., C] float32 or None; lengths [...] int32 or None; gate LA_GATE_VALUE or LA_GATE_SIGMOID;
    workspace: uint8 device tensor of la_recurrence_workspace_bytes(..., 0) bytes (None where that is 0)."""
    _needed(x=x, gates=gates, h=h)
    _check_tensors(x, gates, h0, h, last, lengths, workspace)
    _like(x, gates=gates, h=h)
    B, N, C = _sequences(x, h0=h0, last=last)
    _call("la_recurrence_forward", x, stream, (h, last), _ptr(x), _ptr(gates), _ptr(h0), _ptr(h), _ptr(last),
          _lengths_ptr(lengths, x), B, N, C, int(gate), _real_code(x), *_room(workspace))


def la_recurrence_backward(x, gates, h0, h, dh, dlast, dx, dgates, dh0, lengths, gate, workspace, stream=None):
    """la_recurrence_backward of include/la.h (see la_recurrence_forward; dlast, dh0 [..., C] float32 or None)."""
    _needed(x=x, gates=gates, h=h, dh=dh, dx=dx, dgates=dgates)
    _check_tensors(x, gates, h0, h, dh, dlast, dx, dgates, dh0, lengths, workspace)
    _like(x, gates=gates, h=h, dh=dh, dx=dx, dgates=dgates)
    B, N, C = _sequences(x, h0=h0, dlast=dlast, dh0=dh0)
    _call("la_recurrence_backward", x, stream, (dx, dgates, dh0), _ptr(x), _ptr(gates), _ptr(h0), _ptr(h), _ptr(dh), _ptr(dlast),
          _ptr(dx), _ptr(dgates), _ptr(dh0), _lengths_ptr(lengths, x), B, N, C, int(gate), _real_code(x),
          *_room(workspace))


def la_recurrence_step(x, gates, h, state, gate, stream=None):
    """la_recurrence_step of include/la.h: x, gates, h [..., T, C]; state [..., C] float32, updated in place (as a change
    that autograd sees, and outside of any graph: a state with a history is left with that of its values before)."""
    if _native is not None:
        rc = _native.recurrence_step(x, gates, h, state, gate, stream)
        if rc == 0:
            return
        if rc is not None:
            raise LaError(rc, "la_recurrence_step")
    _needed(x=x, gates=gates, h=h, state=state)
    _check_tensors(x, gates, h, state)
    _like(x, gates=gates, h=h)
    B, T, C = _sequences(x, state=state)
    _call("la_recurrence_step", x, stream, (h, state), _ptr(x), _ptr(gates), _ptr(h), _ptr(state), B, T, C, int(gate),
          _real_code(x))


LA_GROUP = 32  # neighbours of a row that share a power of two
_EIGHT = {"e4m3": LA_E4M3, "int8": LA_I8}


def eight_bit_code(name):
    """LA_E4M3 or LA_I8 from a type's name."""
    if name not in _EIGHT:
        raise ValueError("8-bit types are %s, got %r" % (" and ".join(map(repr, _EIGHT)), name))
    return _EIGHT[name]


def powers_shape(shape):
    """The shape of the powers of rows of ``shape``, one for every 32 elements."""
    if len(shape) < 1:
        raise ValueError("rows of [..., C] are needed")
    return (*shape[:-1], -(-shape[-1] // LA_GROUP))


def _eight(codes, scales, x, code, what):
    """Checks codes like x and a power for every 32 elements of a row; both of one byte an element."""
    if code not in (LA_E4M3, LA_I8):
        raise ValueError("%s: the code is LA_E4M3 or LA_I8, got %r" % (what, code))
    _needed(**{what + " codes": codes, what + " scales": scales})
    if codes.shape != x.shape or codes.element_size() != 1:
        raise ValueError("%s codes must be %s of one byte an element" % (what, tuple(x.shape)))
    groups = powers_shape(x.shape)
    if scales.shape != groups or scales.element_size() != 1:
        raise ValueError("%s scales must be %s of one byte an element" % (what, groups))


def _rows(x):
    if x.dim() < 1:
        raise ValueError("rows of [..., C] are needed")
    C = x.shape[-1]
    _fit(C=C)
    return (x.numel() // C if x.numel() else 0), C


def la_pack_rows(x, codes, scales, code, stream=None):
    """la_pack_rows of include/la.h: x [..., C] float32 or bfloat16 -> codes [..., C], scales
    [..., ceil(C / 32)], any types of one byte; code LA_E4M3 or LA_I8."""
    _needed(x=x)
    _check_tensors(x, codes, scales)
    _eight(codes, scales, x, code, "packed")
    rows, C = _rows(x)
    _call("la_pack_rows", x, stream, (codes, scales), _ptr(x), _ptr(codes), _ptr(scales), rows, C, _real_code(x), int(code))


def la_pack_tensors(xs, codes, scales, code, stream=None):
    """la_pack_tensors of include/la.h: lists of one to four tensors of one shape, as for la_pack_rows."""
    if not len(xs) == len(codes) == len(scales) or not xs:
        raise ValueError("as many codes and scales as tensors are needed")
    _needed(x=xs[0])
    _check_tensors(xs[0], *xs, *codes, *scales)
    for x, c, s in zip(xs, codes, scales):
        _needed(x=x)
        _like(xs[0], x=x)
        _eight(c, s, x, code, "packed")
    rows, C = _rows(xs[0])
    lists = [(ctypes.c_void_p * len(ts))(*map(_ptr, ts)) for ts in (xs, codes, scales)]
    _call("la_pack_tensors", xs[0], stream, (*codes, *scales), len(xs), *lists, rows, C, _real_code(xs[0]), int(code))


def la_unpack_rows(codes, scales, x, code, stream=None):
    """la_unpack_rows of include/la.h: the way back, into x."""
    _needed(x=x)
    _check_tensors(x, codes, scales)
    _eight(codes, scales, x, code, "packed")
    rows, C = _rows(x)
    _call("la_unpack_rows", x, stream, (x,), _ptr(codes), _ptr(scales), _ptr(x), rows, C, int(code), _real_code(x))


def la_rmsnorm_workspace_bytes(rows, C):
    if C >= _INTS:
        return 0
    return int(load_library().la_rmsnorm_workspace_bytes(rows, C))


def _weight_code(weight, x):
    if weight is None:
        return LA_F32
    if weight.shape != x.shape[-1:]:
        raise ValueError("the weight must be [%d], got %s" % (x.shape[-1], tuple(weight.shape)))
    if weight.dtype not in (torch.float32, x.dtype):
        raise TypeError("the weight must be float32 or %s, got %s" % (x.dtype, weight.dtype))
    return LA_F32 if weight.dtype == torch.float32 else LA_BF16


def _per_row(x, **ts):
    for name, t in ts.items():
        if t is not None and (t.shape != x.shape[:-1] or t.dtype != torch.float32):
            raise ValueError("%s must be float32 %s" % (name, tuple(x.shape[:-1])))


def la_rmsnorm_forward(x, residual, weight, y, yscales, total, kept, kscales, rstd, eps, ycode=None, kcode=None,
                       stream=None):
    """la_rmsnorm_forward of include/la.h: x, residual, total [..., C] float32 or bfloat16 (residual and
    total together, or both None); weight [C] float32 or x's type, or None; y like x (yscales, ycode None)
    or 8-bit codes; kept, kscales, kcode: the sum in 8 bits, or None; rstd [...] float32 or None."""
    _needed(x=x, y=y)
    _check_tensors(x, residual, weight, y, yscales, total, kept, kscales, rstd)
    _like(x, residual=residual, total=total)
    if (residual is None) != (total is None):
        raise ValueError("residual and total go together")
    dt, wt = _real_code(x), _weight_code(weight, x)
    if ycode is None:
        _like(x, y=y)
        if yscales is not None:
            raise ValueError("yscales belong to 8-bit codes (ycode)")
    else:
        _eight(y, yscales, x, ycode, "y")
    if kcode is not None:
        _eight(kept, kscales, x, kcode, "kept")
    elif kept is not None or kscales is not None:
        raise ValueError("kept and kscales need kcode")
    _per_row(x, rstd=rstd)
    rows, C = _rows(x)
    _call("la_rmsnorm_forward", x, stream, (y, yscales, total, kept, kscales, rstd), _ptr(x), _ptr(residual),
          _ptr(weight), _ptr(y), _ptr(yscales), _ptr(total), _ptr(kept), _ptr(kscales), _ptr(rstd), rows, C, float(eps), dt, wt, dt if ycode is None else int(ycode),
          LA_E4M3 if kcode is None else int(kcode))


def la_rmsnorm_backward(total, scales, weight, rstd, dy, dtotal, dx, dweight, workspace, code=None, stream=None):
    """la_rmsnorm_backward of include/la.h: total like dy (scales, code None) or the 8-bit codes that
    la_rmsnorm_forward kept; dy, dtotal (or None), dx [..., C]; dweight [C] float32 or None; workspace: uint8
    device tensor of la_rmsnorm_workspace_bytes(rows, C) bytes where dweight is given."""
    _needed(total=total, rstd=rstd, dy=dy, dx=dx)
    _check_tensors(dy, total, scales, weight, rstd, dtotal, dx, dweight, workspace)
    _like(dy, dtotal=dtotal, dx=dx)
    if code is None:
        _like(dy, total=total)
        if scales is not None:
            raise ValueError("scales belong to 8-bit codes (code)")
    else:
        _eight(total, scales, dy, code, "total")
    dt, wt = _real_code(dy), _weight_code(weight, dy)
    if dweight is not None and (weight is None or dweight.shape != weight.shape or dweight.dtype != torch.float32):
        raise ValueError("dweight must be float32, of the weight's shape")
    _per_row(dy, rstd=rstd)
    rows, C = _rows(dy)
    _call("la_rmsnorm_backward", dy, stream, (dx, dweight), _ptr(total), _ptr(scales), _ptr(weight), _ptr(rstd), _ptr(dy),
          _ptr(dtotal), _ptr(dx), _ptr(dweight), rows, C, dt, wt, dt if code is None else int(code), *_room(workspace))


def in_native_code(name, where, *args):
    """The result of one of the native functions of csrc/la_bind_layer.cpp; None where there is none, or what it is
    given is left to the Python code."""
    if _native is None:
        load_library()
        if _native is None:
            return None
    out = getattr(_native, name)(*args)
    if type(out) is int:
        raise LaError(out, where)
    return out
