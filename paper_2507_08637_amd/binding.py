"""ctypes binding of libwersa.so: argument marshalling only.

Function names mirror the C entry points of include/wersa.h.  Tensors are torch CUDA tensors
(torch supplies device memory and the stream; every step of the computation runs inside the
library's HIP kernels).  There is no CPU fallback: if the shared library is missing, loading
raises.
"""
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwersa.so")

WERSA_F32, WERSA_BF16 = 0, 1
WERSA_FLAG_GENERIC_PATH = 1
EXPORTS = ["wersa_workspace_bytes", "wersa_saved_bytes", "wersa_forward", "wersa_backward",
           "wersa_forward_static", "wersa_static_scratch_bytes",
           "wersa_haar_filter", "wersa_haar_filter_ws", "wersa_haar_filter_workspace_bytes", "wersa_saved_offset", "wersa_selected_path", "wersa_status_string", "wersa_version",
           "wersa_profile_enable", "wersa_profile_only", "wersa_profile_reset", "wersa_profile_collect", "wersa_profile_get",
           "wersa_peak_copy", "wersa_peak_mfma",
           "wersa_block_workspace_bytes", "wersa_block_saved_bytes", "wersa_block_saved_offset",
           "wersa_block_workspace_offset",
           "wersa_block_forward", "wersa_block_backward",
           "wersa_decay_workspace_bytes", "wersa_decay_saved_bytes", "wersa_decay_forward", "wersa_decay_backward", "wersa_decay_step",
           "wersa_rms_norm_forward", "wersa_rms_norm_eight_bit", "wersa_rms_norm_workspace_bytes", "wersa_rms_norm_backward"]


class WersaDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("n", ctypes.c_int32),
                ("d", ctypes.c_int32), ("L", ctypes.c_int32), ("m", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("bw_floor", ctypes.c_float),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64), ("flags", ctypes.c_int32)]


class WersaDecayDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("n", ctypes.c_int32), ("dk", ctypes.c_int32),
                ("dv", ctypes.c_int32), ("dtype", ctypes.c_int32), ("packed", ctypes.c_int32), ("scale", ctypes.c_float)] + \
               [(name, ctypes.c_int64 * 3) for name in ("stride_q", "stride_k", "stride_v", "stride_o", "stride_dq", "stride_dk", "stride_dv")] + \
               [("clear", ctypes.c_int32)]


class WersaNormDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("stride_x", ctypes.c_int64), ("stride_residual", ctypes.c_int64)]


class WersaError(RuntimeError):
    def __init__(self, status, text):
        super().__init__(f"wersa status {status}: {text}")
        self.status = status


_lib = None


def load_library():
    """Load libwersa.so (built by paper_2507_08637_amd.build); raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} not found: build it with `python -m paper_2507_08637_amd.build` "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, fp, dp = ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(WersaDesc)
    lib.wersa_workspace_bytes.restype = ctypes.c_size_t
    lib.wersa_workspace_bytes.argtypes = [dp, ctypes.c_int]
    lib.wersa_saved_bytes.restype = ctypes.c_size_t
    lib.wersa_saved_bytes.argtypes = [dp]
    lib.wersa_selected_path.restype = ctypes.c_int32
    lib.wersa_selected_path.argtypes = [dp]
    lib.wersa_saved_offset.restype = ctypes.c_int64
    lib.wersa_saved_offset.argtypes = [dp, ctypes.c_int]
    lib.wersa_forward.restype = ctypes.c_int
    lib.wersa_forward.argtypes = [dp, vp, vp, vp, vp, fp, fp, fp, fp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.wersa_forward_static.restype = ctypes.c_int
    lib.wersa_forward_static.argtypes = [dp, vp, vp, vp, vp, fp, fp, fp, fp, vp, vp, vp]
    lib.wersa_static_scratch_bytes.restype = ctypes.c_size_t
    lib.wersa_static_scratch_bytes.argtypes = []
    lib.wersa_backward.restype = ctypes.c_int
    lib.wersa_backward.argtypes = [dp] + [vp] * 4 + [fp] * 4 + [vp] * 3 + [vp] * 3 + [fp] * 4 + \
        [vp, ctypes.c_size_t, vp]
    lib.wersa_haar_filter.restype = ctypes.c_int
    lib.wersa_haar_filter.argtypes = [dp, vp, fp, vp, vp]
    lib.wersa_haar_filter_workspace_bytes.restype = ctypes.c_size_t
    lib.wersa_haar_filter_workspace_bytes.argtypes = [dp]
    lib.wersa_haar_filter_ws.restype = ctypes.c_int
    lib.wersa_haar_filter_ws.argtypes = [dp, vp, fp, vp, vp, ctypes.c_size_t, vp]
    lib.wersa_block_workspace_bytes.restype = ctypes.c_size_t
    lib.wersa_block_workspace_bytes.argtypes = [dp, ctypes.c_int]
    lib.wersa_block_saved_bytes.restype = ctypes.c_size_t
    lib.wersa_block_saved_bytes.argtypes = [dp]
    lib.wersa_block_saved_offset.restype = ctypes.c_int64
    lib.wersa_block_saved_offset.argtypes = [dp, ctypes.c_int]
    lib.wersa_block_workspace_offset.restype = ctypes.c_int64
    lib.wersa_block_workspace_offset.argtypes = [dp, ctypes.c_int]
    lib.wersa_block_forward.restype = ctypes.c_int
    lib.wersa_block_forward.argtypes = [dp] + [vp] * 6 + [fp] * 4 + [vp, vp, vp, ctypes.c_size_t, vp]
    lib.wersa_block_backward.restype = ctypes.c_int
    lib.wersa_block_backward.argtypes = [dp] + [vp] * 6 + [fp] * 4 + [vp, vp, vp] + [fp] * 8 + \
        [vp, ctypes.c_size_t, vp]
    ddp, ndp = ctypes.POINTER(WersaDecayDesc), ctypes.POINTER(WersaNormDesc)
    lib.wersa_decay_workspace_bytes.restype = ctypes.c_size_t
    lib.wersa_decay_workspace_bytes.argtypes = [ddp, ctypes.c_int]
    lib.wersa_decay_saved_bytes.restype = ctypes.c_size_t
    lib.wersa_decay_saved_bytes.argtypes = [ddp]
    lib.wersa_decay_forward.restype = ctypes.c_int
    lib.wersa_decay_forward.argtypes = [ddp] + [vp] * 8 + [ctypes.c_int32] + [vp] * 3 + [ctypes.c_size_t, vp]
    lib.wersa_decay_backward.restype = ctypes.c_int
    lib.wersa_decay_backward.argtypes = [ddp] + [vp] * 14 + [ctypes.c_size_t, vp]
    lib.wersa_decay_step.restype = ctypes.c_int
    lib.wersa_decay_step.argtypes = [ddp] + [vp] * 6 + [ctypes.c_int32, vp, vp]
    lib.wersa_rms_norm_forward.restype = ctypes.c_int
    lib.wersa_rms_norm_forward.argtypes = [ndp] + [vp] * 7
    lib.wersa_rms_norm_eight_bit.restype = ctypes.c_int
    lib.wersa_rms_norm_eight_bit.argtypes = [ndp] + [vp] * 7
    lib.wersa_rms_norm_workspace_bytes.restype = ctypes.c_size_t
    lib.wersa_rms_norm_workspace_bytes.argtypes = [ndp]
    lib.wersa_rms_norm_backward.restype = ctypes.c_int
    lib.wersa_rms_norm_backward.argtypes = [ndp] + [vp] * 8 + [ctypes.c_size_t, vp]
    lib.wersa_status_string.restype = ctypes.c_char_p
    lib.wersa_status_string.argtypes = [ctypes.c_int]
    lib.wersa_version.restype = ctypes.c_int32
    lib.wersa_version.argtypes = []
    lib.wersa_profile_enable.restype = None
    lib.wersa_profile_enable.argtypes = [ctypes.c_int]
    lib.wersa_profile_only.restype = None
    lib.wersa_profile_only.argtypes = [ctypes.c_char_p]
    lib.wersa_profile_reset.restype = None
    lib.wersa_profile_reset.argtypes = []
    lib.wersa_profile_collect.restype = ctypes.c_int32
    lib.wersa_profile_collect.argtypes = []
    lib.wersa_profile_get.restype = ctypes.c_int32
    lib.wersa_profile_get.argtypes = [ctypes.c_int32, ctypes.c_char_p, ctypes.c_int32,
                                      ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int32)]
    lib.wersa_peak_copy.restype = ctypes.c_double
    lib.wersa_peak_copy.argtypes = [vp, vp, ctypes.c_size_t, ctypes.c_int32, vp]
    lib.wersa_peak_mfma.restype = ctypes.c_double
    lib.wersa_peak_mfma.argtypes = [fp, ctypes.c_int32, vp]
    _lib = lib
    return lib


def _check(status):
    if status != 0:
        raise WersaError(status, load_library().wersa_status_string(status).decode())


def wersa_path_name(desc):
    return {1: "mfma", 0: "generic"}.get(load_library().wersa_selected_path(ctypes.byref(desc)), "rejected")


def make_desc(x, L, m, eps=1e-6, bw_floor=1e-6, flags=0):
    """Descriptor for a (B, H, n, d) tensor x (last dim contiguous)."""
    assert x.dim() == 4 and x.stride(3) == 1, "expect (B, H, n, d) with contiguous last dim"
    B, H, n, d = x.shape
    if x.dtype == torch.float32:
        dt = WERSA_F32
    elif x.dtype == torch.bfloat16:
        dt = WERSA_BF16
    else:
        raise TypeError("dtype must be float32 or bfloat16")
    return WersaDesc(B, H, n, d, L, m, dt, eps, bw_floor, x.stride(0), x.stride(1), x.stride(2), flags)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    # (the handle alone: building a torch.cuda.Stream for it takes 3 us)
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _nbytes(t):
    return t.numel() * t.element_size()


def _scratch(nbytes, like, stream):
    """Temporary device buffer for one call.  The kernels that use it are only queued when the call
    returns, so the buffer must not go back to torch's allocator for reuse before they have run:
    with an explicit `stream` it is tied to that stream (the caching allocator then waits for the
    stream's queued work before handing the block to anyone else)."""
    buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=like.device)
    if stream is not None:
        buf.record_stream(stream)
    return buf


def _same_layout(ref, *others):
    shape, stride, dtype = ref.shape, ref.stride(), ref.dtype
    for t in others:
        assert t.shape == shape and t.stride() == stride and t.dtype == dtype, \
            "q, k, v, out and gradients must share shape, strides and dtype"


FLAG_GENERIC_PATH = 1
FLAG_SEPARATE_OMEGA = 2
FLAG_POOLED_GATE = 4
FLAG_LAYERNORM = 8


def _check_omega(omega_rf, q, flags):
    """(d, m), or (2, d, m) with FLAG_SEPARATE_OMEGA: the query-side matrix, then the key-side one."""
    d = q.shape[3]
    assert omega_rf.is_contiguous() and omega_rf.dtype == q.dtype
    if flags & FLAG_SEPARATE_OMEGA:
        assert omega_rf.dim() == 3 and omega_rf.shape[0] == 2 and omega_rf.shape[1] == d
    else:
        assert omega_rf.dim() == 2 and omega_rf.shape[0] == d


def wersa_workspace_bytes(desc, for_backward):
    return load_library().wersa_workspace_bytes(ctypes.byref(desc), int(for_backward))


def wersa_saved_bytes(desc):
    return load_library().wersa_saved_bytes(ctypes.byref(desc))


def saved_views(desc, saved):
    """Named float32 views into the saved buffer: S, z, qbar, s, F, D."""
    lib = load_library()
    sl = desc.B * desc.H
    shapes = [("S", (sl, desc.m, desc.d)), ("z", (sl, desc.m)), ("qbar", (sl, desc.d)),
              ("s", (sl, desc.L + 1)), ("F", (sl, desc.L + 1)), ("D", (sl, desc.n))]
    out = {}
    for which, (name, shape) in enumerate(shapes):
        off = lib.wersa_saved_offset(ctypes.byref(desc), which)
        cnt = 1
        for s in shape:
            cnt *= s
        out[name] = saved[off:off + cnt].view(*shape)
    return out


def alloc_like(desc, ref, for_backward):
    """Allocate (saved, workspace) float32 buffers on ref's device."""
    lib = load_library()
    sb = lib.wersa_saved_bytes(ctypes.byref(desc))
    wb = lib.wersa_workspace_bytes(ctypes.byref(desc), int(for_backward))
    if sb == 0 or wb == 0:
        raise WersaError(2, "descriptor rejected (invalid or unsupported shape)")
    saved = torch.empty(sb // 4, dtype=torch.float32, device=ref.device)
    ws = torch.empty(wb // 4, dtype=torch.float32, device=ref.device)
    return saved, ws


def checked_desc(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor, flags):
    """(descriptor, bytes of saved, bytes of the forward's workspace) of a forward call's arguments, which are checked."""
    lib = load_library()
    _same_layout(q, k, v)
    desc = make_desc(q, L, omega_rf.shape[-1], eps, bw_floor, flags)
    _check_omega(omega_rf, q, flags)
    for p in (sigma, gate_w, gate_b, scale_w):
        assert p.dtype == torch.float32 and p.is_contiguous()
    sb = lib.wersa_saved_bytes(ctypes.byref(desc))
    if sb == 0:
        _check(_probe(desc))
    return desc, sb, lib.wersa_workspace_bytes(ctypes.byref(desc), 0)


def wersa_forward(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps=1e-6, bw_floor=1e-6,
                  out=None, saved=None, workspace=None, stream=None, flags=0):
    """Returns (out, saved).  All tensor arguments live on one CUDA device."""
    lib = load_library()
    desc, sb, wb = checked_desc(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor, flags)
    if out is None:
        out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
    else:
        _same_layout(q, out)
    if saved is None:
        saved = torch.empty(sb // 4, dtype=torch.float32, device=q.device)
    else:   # the C ABI takes no size for `saved`: checked here
        assert _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_saved_bytes asks for {sb}"
    if workspace is None:
        workspace = _scratch(wb, q, stream)
    _check(lib.wersa_forward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(omega_rf), _ptr(sigma),
                             _ptr(gate_w), _ptr(gate_b), _ptr(scale_w), _ptr(out), _ptr(saved),
                             _ptr(workspace), _nbytes(workspace), _stream(stream)))
    return out, saved


def wersa_forward_static(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, out, saved, eps=1e-6,
                         bw_floor=1e-6, stream=None, flags=0):
    """wersa_forward with the library's built-in scratch as the workspace: `out` and `saved` come
    from the caller and nothing is allocated here or in the library.  Returns (out, saved)."""
    lib = load_library()
    _same_layout(q, k, v, out)
    desc = make_desc(q, L, omega_rf.shape[-1], eps, bw_floor, flags)
    _check_omega(omega_rf, q, flags)
    sb = lib.wersa_saved_bytes(ctypes.byref(desc))
    assert sb == 0 or _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_saved_bytes asks for {sb}"
    _check(lib.wersa_forward_static(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(omega_rf), _ptr(sigma),
                                    _ptr(gate_w), _ptr(gate_b), _ptr(scale_w), _ptr(out), _ptr(saved),
                                    _stream(stream)))
    return out, saved


def _probe(desc):
    # wersa_saved_bytes returned 0: ask the forward entry point for the precise status
    return load_library().wersa_forward(ctypes.byref(desc), *([None] * 11), 0, None)


def wersa_backward(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, out, dout, saved, L,
                   eps=1e-6, bw_floor=1e-6, workspace=None, stream=None, param_grads=True, grads=None,
                   flags=0):
    """Returns dict(dq, dk, dv, dgate_w, dgate_b, dscale_w, dsigma).

    `grads` may be a dict from an earlier call: its tensors are then overwritten in place."""
    lib = load_library()
    _same_layout(q, k, v, out, dout)
    desc = make_desc(q, L, omega_rf.shape[-1], eps, bw_floor, flags)
    _check_omega(omega_rf, q, flags)
    if grads is not None:
        dq, dk, dv = grads["dq"], grads["dk"], grads["dv"]
        _same_layout(q, dq, dk, dv)
        dgw, dgb, dsw, dsg = grads["dgate_w"], grads["dgate_b"], grads["dscale_w"], grads["dsigma"]
    else:
        dq = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
        dk = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
        dv = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
    if grads is not None:
        pass
    elif param_grads:
        dgw = torch.empty_like(gate_w)
        dgb = torch.empty_like(gate_b)
        dsw = torch.empty_like(scale_w)
        dsg = torch.empty(1, dtype=torch.float32, device=q.device)
    else:
        dgw = dgb = dsw = dsg = None
    wb = lib.wersa_workspace_bytes(ctypes.byref(desc), 1)
    if workspace is None:
        workspace = _scratch(wb, q, stream)
    sb = lib.wersa_saved_bytes(ctypes.byref(desc))
    assert sb == 0 or _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_saved_bytes asks for {sb}"
    _check(lib.wersa_backward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(omega_rf), _ptr(sigma),
                              _ptr(gate_w), _ptr(gate_b), _ptr(scale_w), _ptr(out), _ptr(dout),
                              _ptr(saved), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgw), _ptr(dgb),
                              _ptr(dsw), _ptr(dsg), _ptr(workspace), _nbytes(workspace),
                              _stream(stream)))
    return dict(dq=dq, dk=dk, dv=dv, dgate_w=dgw, dgate_b=dgb, dscale_w=dsw, dsigma=dsg)


def wersa_haar_filter(x, filt, L, out=None, stream=None):
    """X_F = W^-1(F (.) W X) for x (B, H, n, d) and filt (B*H, L+1) float32."""
    lib = load_library()
    desc = make_desc(x, L, 16)
    assert filt.dtype == torch.float32 and filt.is_contiguous() and filt.numel() == x.shape[0] * x.shape[1] * (L + 1)
    if out is None:
        out = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    wb = lib.wersa_haar_filter_workspace_bytes(ctypes.byref(desc))
    if wb == 0:
        _check(lib.wersa_haar_filter(ctypes.byref(desc), _ptr(x), _ptr(filt), _ptr(out), _stream(stream)))
    else:   # levels above 6: the tiles' approximation coefficients go through a workspace
        ws = _scratch(wb, x, stream)
        _check(lib.wersa_haar_filter_ws(ctypes.byref(desc), _ptr(x), _ptr(filt), _ptr(out), _ptr(ws), wb,
                                        _stream(stream)))
    return out


def make_block_desc(x, H, L, m, eps=1e-6, bw_floor=1e-6, flags=0):
    """Descriptor for the attention block on x (B, n, hidden), hidden = H * d, dense bf16."""
    assert x.dim() == 3 and x.is_contiguous() and x.shape[2] % H == 0
    if x.dtype != torch.bfloat16:
        raise TypeError("the attention block takes bfloat16 tensors")
    B, n, hidden = x.shape
    d = hidden // H
    return WersaDesc(B, H, n, d, L, m, WERSA_BF16, eps, bw_floor, n * hidden, d, hidden, flags)


def block_saved_views(desc, saved):
    """bf16 views (B, n, hidden) of Q', K', V', A inside the block's saved byte buffer, and the
    core's saved buffer as float32."""
    lib = load_library()
    B, n, hidden = desc.B, desc.n, desc.H * desc.d
    out = {}
    for which, name in enumerate(("Qp", "Kp", "Vp", "A")):
        off = lib.wersa_block_saved_offset(ctypes.byref(desc), which)
        out[name] = saved[off:off + B * n * hidden * 2].view(torch.bfloat16).view(B, n, hidden)
    off = lib.wersa_block_saved_offset(ctypes.byref(desc), 4)
    out["core"] = saved[off:].view(torch.float32)
    return out


def block_workspace_views(desc, workspace):
    """bf16 views (B, n, hidden) of dA, dQ', dK', dV' left in the backward workspace."""
    lib = load_library()
    B, n, hidden = desc.B, desc.n, desc.H * desc.d
    out = {}
    for which, name in enumerate(("dA", "dQp", "dKp", "dVp")):
        off = lib.wersa_block_workspace_offset(ctypes.byref(desc), which)
        out[name] = workspace[off:off + B * n * hidden * 2].view(torch.bfloat16).view(B, n, hidden)
    return out


def _block_check_args(x, weights, omega_rf, params):
    hidden = x.shape[2]
    for w in weights:
        assert w.shape == (hidden, hidden) and w.is_contiguous() and w.dtype == x.dtype
    assert omega_rf.is_contiguous() and omega_rf.dtype == x.dtype
    for p in params:
        assert p.dtype == torch.float32 and p.is_contiguous()


def wersa_block_forward(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps=1e-6,
                        bw_floor=1e-6, y=None, saved=None, workspace=None, stream=None, flags=0):
    """Returns (y, saved): y (B, n, hidden) bf16, saved a uint8 buffer for wersa_block_backward."""
    lib = load_library()
    desc = make_block_desc(x, H, L, omega_rf.shape[1], eps, bw_floor, flags)
    _block_check_args(x, (wq, wk, wv, wo), omega_rf, (sigma, gate_w, gate_b, scale_w))
    sb = lib.wersa_block_saved_bytes(ctypes.byref(desc))
    wb = lib.wersa_block_workspace_bytes(ctypes.byref(desc), 0)
    if sb == 0 or wb == 0:
        _check(lib.wersa_block_forward(ctypes.byref(desc), *([None] * 13), 0, None) or 2)
    if y is None:
        y = torch.empty_like(x)
    if saved is None:
        saved = torch.empty(sb, dtype=torch.uint8, device=x.device)
    else:
        assert _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_block_saved_bytes asks for {sb}"
    if workspace is None:
        workspace = _scratch(wb, x, stream)
    _check(lib.wersa_block_forward(ctypes.byref(desc), _ptr(x), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(wo),
                                   _ptr(omega_rf), _ptr(sigma), _ptr(gate_w), _ptr(gate_b), _ptr(scale_w),
                                   _ptr(y), _ptr(saved), _ptr(workspace), _nbytes(workspace), _stream(stream)))
    return y, saved


def wersa_block_backward(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, dy, saved, L,
                         eps=1e-6, bw_floor=1e-6, workspace=None, stream=None, grads=None, flags=0):
    """Returns dict(dx, dwq, dwk, dwv, dwo, dgate_w, dgate_b, dscale_w, dsigma); weight gradients are
    float32.  `grads` may be a dict from an earlier call: its tensors are then overwritten."""
    lib = load_library()
    desc = make_block_desc(x, H, L, omega_rf.shape[1], eps, bw_floor, flags)
    _block_check_args(x, (wq, wk, wv, wo), omega_rf, (sigma, gate_w, gate_b, scale_w))
    assert dy.shape == x.shape and dy.is_contiguous() and dy.dtype == x.dtype
    wb = lib.wersa_block_workspace_bytes(ctypes.byref(desc), 1)
    if wb == 0:
        _check(lib.wersa_block_backward(ctypes.byref(desc), *([None] * 21), 0, None) or 2)
    if grads is None:
        f32 = dict(dtype=torch.float32, device=x.device)
        grads = dict(dx=torch.empty_like(x), dwq=torch.empty(wq.shape, **f32), dwk=torch.empty(wq.shape, **f32),
                     dwv=torch.empty(wq.shape, **f32), dwo=torch.empty(wq.shape, **f32),
                     dgate_w=torch.empty_like(gate_w), dgate_b=torch.empty_like(gate_b),
                     dscale_w=torch.empty_like(scale_w), dsigma=torch.empty(1, **f32))
    if workspace is None:
        workspace = _scratch(wb, x, stream)
    sb = lib.wersa_block_saved_bytes(ctypes.byref(desc))
    assert _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_block_saved_bytes asks for {sb}"
    g = grads
    _check(lib.wersa_block_backward(ctypes.byref(desc), _ptr(x), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(wo),
                                    _ptr(omega_rf), _ptr(sigma), _ptr(gate_w), _ptr(gate_b), _ptr(scale_w),
                                    _ptr(dy), _ptr(saved), _ptr(g["dx"]), _ptr(g["dwq"]), _ptr(g["dwk"]),
                                    _ptr(g["dwv"]), _ptr(g["dwo"]), _ptr(g["dgate_w"]), _ptr(g["dgate_b"]),
                                    _ptr(g["dscale_w"]), _ptr(g["dsigma"]), _ptr(workspace),
                                    _nbytes(workspace), _stream(stream)))
    return grads


# ---- causal linear attention with a decay for each head -------------------------------------------

def _dtype_code(x):
    if x.dtype == torch.float32:
        return WERSA_F32
    if x.dtype == torch.bfloat16:
        return WERSA_BF16
    raise TypeError("dtype must be float32 or bfloat16")


# (a structure of ctypes takes several times as long to fill in field by field)
_DECAY_DESC = struct.Struct("7if12q72xi4x")   # without the gradients' strides
_GRAD_STRIDES = struct.Struct("9q")


def make_decay_desc(q, k, v, out, scale=None, offsets=None, clear=False):
    """Descriptor for q, k (B, H, n, dk) and v, out (B, H, n, dv), last dimension contiguous; with offsets (B + 1) the tensors
    have one batch entry that holds the rows of all B sequences.  scale: 1 / sqrt(dk) by default.  clear: the forward writes zeros to rows of no sequence."""
    assert q.dim() == 4 and v.dim() == 4, "expect q, k (B, H, n, dk) and v, out (B, H, n, dv)"
    (N, H, n, dk), dv = q.shape, v.shape[3]
    assert k.shape == q.shape and v.shape == (N, H, n, dv) and out.shape == v.shape, "expect q, k (B, H, n, dk) and v, out (B, H, n, dv)"
    dtype = q.dtype
    assert k.dtype == dtype and v.dtype == dtype and out.dtype == dtype, "q, k, v and out must share a dtype"
    (qb, qh, qn, q1), (kb, kh, kn, k1), (vb, vh, vn, v1), (ob, oh, on, o1) = q.stride(), k.stride(), v.stride(), out.stride()
    assert q1 == k1 == v1 == o1 == 1, "expect a contiguous last dim"
    B = N
    if offsets is not None:
        assert N == 1 and offsets.dim() == 1 and offsets.numel() >= 2 and offsets.dtype == torch.int32 and offsets.is_contiguous(), \
            "packed sequences: tensors of one batch entry and int32 offsets (B + 1)"
        B = offsets.numel() - 1
    return WersaDecayDesc.from_buffer_copy(_DECAY_DESC.pack(
        B, H, n, dk, dv, _dtype_code(q), offsets is not None, dk ** -0.5 if scale is None else scale,
        qb, qh, qn, kb, kh, kn, vb, vh, vn, ob, oh, on, clear))


def _dense_like(x):
    """A new tensor of x's shape, with its dimensions in x's order in memory but none apart from or on another: x may be a slice, or windows that overlap."""
    shape = N, H, n, d = x.shape
    b, h, r, _ = x.stride()
    if (r == d and h == n * d or h == d and r == H * d) and b == H * n * d:
        return torch.empty_like(x)
    step, strides = d, [1] * 4
    for i in sorted(range(3), key=x.stride):
        strides[i] = step
        step *= max(1, shape[i])
    return torch.empty_strided(shape, strides, dtype=x.dtype, device=x.device)


def _not_broadcast(x, stream):
    """x, or a copy where it is expanded over sequences, heads or rows: the library takes strides above 0."""
    if 0 not in x.stride():
        return x
    if stream is None:
        return x.contiguous()
    with torch.cuda.stream(stream):
        return x.contiguous()


def _addr(t):
    return None if t is None else t.data_ptr()


def _on_one_gpu(first, *others):
    """An address of host memory, or of another device's, would fault on the GPU."""
    device = first.get_device()
    assert device >= 0, "expect tensors on the GPU"
    for t in others:
        assert t is None or t.get_device() == device, "expect all tensors on one GPU"


def _check_states(desc, slots, *states):
    """float32 (rows, H, dk, dv); rows = B, or any number with slots (B).  Returns the rows."""
    rows = desc.B
    if slots is not None:
        assert slots.dtype == torch.int32 and slots.is_contiguous() and slots.numel() == desc.B, "slots: int32, one per sequence"
        rows = max([s.shape[0] for s in states if s is not None], default=0)
    for s in states:
        if s is not None:
            assert s.shape == (rows, desc.H, desc.dk, desc.dv) and s.is_contiguous() and s.dtype == torch.float32, \
                "states are contiguous float32 (sequences or slots, H, dk, dv)"
    return rows


def _check_log_decay(log_decay, desc):
    assert log_decay.dtype == torch.float32 and log_decay.is_contiguous() and log_decay.numel() == desc.H, "log_decay: float32, one per head"


def checked_decay_desc(q, k, v, log_decay, scale, offsets, initial_state):
    """(descriptor, bytes of saved) of a forward call, whose output's strides the caller fills in; the arguments are checked."""
    desc = make_decay_desc(q, k, v, v, scale, offsets)
    _check_log_decay(log_decay, desc)
    _check_states(desc, None, initial_state)
    _on_one_gpu(q, k, v, log_decay, offsets, initial_state)
    sb = load_library().wersa_decay_saved_bytes(ctypes.byref(desc))
    if sb == 0:   # the precise status
        _check(load_library().wersa_decay_forward(ctypes.byref(desc), *([None] * 8), 0, *([None] * 3), 0, None))
    return desc, sb


def wersa_decay_forward(q, k, v, log_decay, scale=None, offsets=None, initial_state=None, final_state=None, slots=None, out=None,
                        want_state=False, want_saved=False, saved=None, workspace=None, stream=None):
    """Returns (out, final_state, saved).  final_state: a buffer to write, or want_state=True for a new one (else None);
    want_saved=True leaves what wersa_decay_backward needs (else None).  Rows of no sequence are zeros in a new out, and left as they are in
    the caller's."""
    lib = load_library()
    clear = out is None and offsets is not None
    if 0 in q.stride() or 0 in k.stride() or 0 in v.stride():
        q, k, v = _not_broadcast(q, stream), _not_broadcast(k, stream), _not_broadcast(v, stream)
    if out is None:
        out = _dense_like(v)
    desc = make_decay_desc(q, k, v, out, scale, offsets, clear=clear)
    _check_log_decay(log_decay, desc)
    if want_state and final_state is None:
        assert slots is None, "with slots the states lie in a buffer of the caller's"
        final_state = torch.empty(desc.B, desc.H, desc.dk, desc.dv, dtype=torch.float32, device=q.device)
    rows = _check_states(desc, slots, initial_state, final_state)
    _on_one_gpu(q, k, v, log_decay, offsets, initial_state, final_state, slots, out, saved, workspace)
    sb = lib.wersa_decay_saved_bytes(ctypes.byref(desc))
    if saved is not None:
        assert _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_decay_saved_bytes asks for {sb}"
    elif want_saved:
        saved = torch.empty(max(sb // 4, 64), dtype=torch.float32, device=q.device)
    elif workspace is None:
        wb = lib.wersa_decay_workspace_bytes(ctypes.byref(desc), 0)
        workspace = _scratch(wb, q, stream) if wb > 256 else None   # (256: no scratch in it)
    _check(lib.wersa_decay_forward(ctypes.byref(desc), _addr(q), _addr(k), _addr(v), _addr(log_decay), _addr(offsets), _addr(initial_state),
                                   _addr(final_state), _addr(slots), rows, _addr(out), _addr(saved), _addr(workspace),
                                   0 if workspace is None else _nbytes(workspace), _stream(stream)))
    return out, final_state, saved


def wersa_decay_backward(q, k, v, log_decay, dout, saved, scale=None, offsets=None, initial_state=None, dfinal_state=None,
                         want_dinitial=False, workspace=None, stream=None, grads=None):
    """Returns dict(dq, dk, dv, dinitial_state); rows of no sequence are zeros.  `grads` may be a dict from an earlier call, of any strides: its tensors are then
    overwritten."""
    lib = load_library()
    fresh = grads is None
    q, k, v, dout = (_not_broadcast(x, stream) for x in (q, k, v, dout))
    if fresh:
        grads = dict(dq=_dense_like(q), dk=_dense_like(k), dv=_dense_like(v))
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        g = grads[name]
        assert g.shape == x.shape and g.dtype == x.dtype and g.stride(3) == 1, f"{name} has its tensor's shape and dtype, and a contiguous last dim"
    desc = make_decay_desc(q, k, v, dout, scale, offsets)
    _GRAD_STRIDES.pack_into(desc, WersaDecayDesc.stride_dq.offset, *(s for name in ("dq", "dk", "dv") for s in grads[name].stride()[:3]))
    _check_log_decay(log_decay, desc)
    _check_states(desc, None, initial_state, dfinal_state)
    sb = lib.wersa_decay_saved_bytes(ctypes.byref(desc))
    assert _nbytes(saved) >= sb, f"saved buffer holds {_nbytes(saved)} bytes, wersa_decay_saved_bytes asks for {sb}"
    if fresh:
        grads["dinitial_state"] = torch.empty(desc.B, desc.H, desc.dk, desc.dv, dtype=torch.float32, device=q.device) if want_dinitial else None
    _check_states(desc, None, grads["dinitial_state"])
    _on_one_gpu(q, k, v, log_decay, offsets, initial_state, dout, dfinal_state, saved, workspace, *grads.values())
    if workspace is None:
        workspace = _scratch(lib.wersa_decay_workspace_bytes(ctypes.byref(desc), 1), q, stream)
    _check(lib.wersa_decay_backward(ctypes.byref(desc), _addr(q), _addr(k), _addr(v), _addr(log_decay), _addr(offsets), _addr(initial_state),
                                    _addr(dout), _addr(dfinal_state), _addr(saved), _addr(grads["dq"]), _addr(grads["dk"]), _addr(grads["dv"]),
                                    _addr(grads["dinitial_state"]), _addr(workspace), _nbytes(workspace), _stream(stream)))
    return grads


def wersa_decay_step(q, k, v, log_decay, state, scale=None, slots=None, out=None, stream=None):
    """One token of each of B sequences: q, k (B, H, dk), v (B, H, dv), state (B or slots, H, dk, dv) float32, updated in place.  Returns out."""
    lib = load_library()
    if out is None:
        out = torch.empty(v.shape, dtype=v.dtype, device=v.device)
    assert q.dim() == 3 and v.dim() == 3, "expect q, k (B, H, dk) and v, out (B, H, dv)"
    (B, H, dk), dv, dtype = q.shape, v.shape[2], q.dtype
    assert k.shape == q.shape and v.shape == (B, H, dv) and out.shape == v.shape, "expect q, k (B, H, dk) and v, out (B, H, dv)"
    assert k.dtype == dtype and v.dtype == dtype and out.dtype == dtype, "q, k, v and out must share a dtype"
    (qb, qh, q1), (kb, kh, k1), (vb, vh, v1), (ob, oh, o1) = q.stride(), k.stride(), v.stride(), out.stride()
    if not (qb and qh and kb and kh and vb and vh):
        q, k, v = _not_broadcast(q, stream), _not_broadcast(k, stream), _not_broadcast(v, stream)
        (qb, qh, q1), (kb, kh, k1), (vb, vh, v1) = q.stride(), k.stride(), v.stride()
    assert q1 == k1 == v1 == o1 == 1, "expect a contiguous last dim"
    desc = WersaDecayDesc.from_buffer_copy(_DECAY_DESC.pack(B, H, 1, dk, dv, _dtype_code(q), 0, dk ** -0.5 if scale is None else scale,
                                                            qb, qh, 0, kb, kh, 0, vb, vh, 0, ob, oh, 0, 0))
    _check_log_decay(log_decay, desc)
    rows = _check_states(desc, slots, state)
    _on_one_gpu(q, k, v, log_decay, state, slots, out)
    _check(lib.wersa_decay_step(ctypes.byref(desc), q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), state.data_ptr(), _addr(slots),
                                rows, out.data_ptr(), _stream(stream)))
    return out


# ---- root-mean-square norm with the residual's addition --------------------------------------------

_NORM_DESC = struct.Struct("qiif4xqq")


def checked_norm_args(x, weight, residual):
    """(rows, cols) tensors, columns contiguous."""
    assert x.dim() == 2 and x.stride(1) == 1, "expect (rows, cols) with contiguous columns"
    if weight is not None:
        assert weight.dtype == torch.float32 and weight.is_contiguous() and weight.numel() == x.shape[1], "weight: float32, one per column"
    if residual is not None:
        assert residual.shape == x.shape and residual.dtype == x.dtype and residual.stride(1) == 1, "the residual has x's shape and dtype"
    _dtype_code(x)
    _on_one_gpu(x, weight, residual)


def _norm_args(x, weight, residual, eps, r):
    """Returns the descriptor and the stream's buffer (None without a residual)."""
    checked_norm_args(x, weight, residual)
    rows, cols = x.shape
    step = cols
    if residual is not None:
        step = residual.stride(0)
        if r is None:
            r = x.new_empty((rows, cols))
        else:
            _dense(x, r, x.shape, x.dtype, "r")
    return WersaNormDesc.from_buffer_copy(_NORM_DESC.pack(rows, cols, _dtype_code(x), eps, x.stride(0), step)), r if residual is not None else None


def _dense(like, t, shape, dtype, name):
    _on_one_gpu(like, t)
    assert t.shape == shape and t.dtype == dtype and t.is_contiguous(), f"{name} is dense, {tuple(shape)} of {dtype}"
    return t


def wersa_rms_norm_forward(x, weight=None, residual=None, eps=1e-6, r=None, y=None, rstd=None, want_rstd=False, stream=None):
    """Returns (y, r, rstd): r = x + residual (x itself without one), rstd (rows) float32 or None."""
    desc, stream_out = _norm_args(x, weight, residual, eps, r)
    y = x.new_empty(x.shape) if y is None else _dense(x, y, x.shape, x.dtype, "y")
    if rstd is not None:
        _dense(x, rstd, x.shape[:1], torch.float32, "rstd")
    elif want_rstd:
        rstd = x.new_empty(x.shape[0], dtype=torch.float32)
    _check(load_library().wersa_rms_norm_forward(ctypes.byref(desc), x.data_ptr(), _addr(residual), _addr(weight), _addr(stream_out), y.data_ptr(),
                                                 _addr(rstd), _stream(stream)))
    return y, x if residual is None else stream_out, rstd


def wersa_rms_norm_eight_bit(x, weight=None, residual=None, eps=1e-6, r=None, y=None, scales=None, stream=None):
    """Returns (y, r, scales): y (rows, cols) float8_e4m3fn, to be multiplied by scales (rows) float32."""
    desc, stream_out = _norm_args(x, weight, residual, eps, r)
    y = x.new_empty(x.shape, dtype=torch.float8_e4m3fn) if y is None else _dense(x, y, x.shape, torch.float8_e4m3fn, "y")
    scales = x.new_empty(x.shape[0], dtype=torch.float32) if scales is None else _dense(x, scales, x.shape[:1], torch.float32, "scales")
    _check(load_library().wersa_rms_norm_eight_bit(ctypes.byref(desc), x.data_ptr(), _addr(residual), _addr(weight), _addr(stream_out), y.data_ptr(),
                                                   scales.data_ptr(), _stream(stream)))
    return y, x if residual is None else stream_out, scales


def wersa_rms_norm_backward(r, rstd, dy, weight=None, dr=None, dx=None, want_dweight=True, dweight=None, workspace=None, stream=None):
    """Returns (dx, dweight): dx is the gradient of x and of the residual; dr: what reaches the stream r from elsewhere."""
    lib = load_library()
    desc, _ = _norm_args(r, weight, None, 0.0, None)
    for t in (dy, dr):
        assert t is None or (t.shape == r.shape and t.dtype == r.dtype and t.is_contiguous()), "dy and dr are dense, of r's shape and dtype"
    assert rstd.numel() == r.shape[0] and rstd.dtype == torch.float32 and rstd.is_contiguous()
    if dx is None:
        dx = torch.empty(r.shape, dtype=r.dtype, device=r.device)
    assert dx.shape == r.shape and dx.dtype == r.dtype and dx.is_contiguous()
    _on_one_gpu(r, rstd, dy, weight, dr, dx, dweight, workspace)
    if want_dweight and dweight is None:
        dweight = torch.empty(r.shape[1], dtype=torch.float32, device=r.device)
    if dweight is not None:
        assert dweight.numel() == r.shape[1] and dweight.dtype == torch.float32 and dweight.is_contiguous()
        if workspace is None:
            workspace = _scratch(lib.wersa_rms_norm_workspace_bytes(ctypes.byref(desc)), r, stream)
    _check(lib.wersa_rms_norm_backward(ctypes.byref(desc), _addr(r), _addr(weight), _addr(rstd), _addr(dy), _addr(dr), _addr(dx), _addr(dweight),
                                       _addr(workspace), 0 if workspace is None else _nbytes(workspace), _stream(stream)))
    return dx, dweight


def wersa_profile_enable(on, only=None):
    """Switch the event bracketing on or off; `only` restricts it to one kernel name."""
    lib = load_library()
    lib.wersa_profile_reset()
    lib.wersa_profile_only(only.encode() if only else None)
    lib.wersa_profile_enable(int(bool(on)))


def wersa_profile_collect():
    """{kernel name: (total_ms, launches)} for everything recorded since the last collect."""
    lib = load_library()
    cnt = lib.wersa_profile_collect()
    out = {}
    buf = ctypes.create_string_buffer(128)
    ms, launches = ctypes.c_double(), ctypes.c_int32()
    for i in range(cnt):
        if lib.wersa_profile_get(i, buf, 128, ctypes.byref(ms), ctypes.byref(launches)) == 0:
            out[buf.value.decode()] = (ms.value, launches.value)
    return out


def wersa_peak_copy(dst, src, reps=10, stream=None):
    """GB/s (read + written) of a plain streaming copy src -> dst, measured now on this device."""
    assert dst.is_contiguous() and src.is_contiguous() and dst.numel() * dst.element_size() == src.numel() * src.element_size()
    return load_library().wersa_peak_copy(_ptr(dst), _ptr(src), src.numel() * src.element_size() // 16 * 16, reps,
                                          _stream(stream))


def wersa_peak_mfma(reps=3, stream=None):
    """TFLOP/s of a loop of independent bf16 32x32x16 matrix instructions on every compute unit."""
    sink = torch.zeros(64, dtype=torch.float32, device="cuda")
    return load_library().wersa_peak_mfma(_ptr(sink), reps, _stream(stream))
