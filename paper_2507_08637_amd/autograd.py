"""torch.autograd bindings of the WERSA hot path (argument marshalling only: every step runs in
the HIP kernels behind the C ABI).

    out = wersa_attention(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L)
    y = wersa_attention_block(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, L)

q, k, v: (B, H, n, d) with a shared layout (any strides, last dimension contiguous); gradients
flow to q, k, v, sigma, gate_w, gate_b, scale_w (omega_rf is a fixed random matrix) and, for the
block, to x and the four weight matrices (float32 gradients cast to the weights' dtype).

    out, final_state = wersa_decay_attention(q, k, v, log_decay, scale, initial_state, offsets)
    y = wersa_rms_norm(x, weight, eps=eps)
    y, r = wersa_rms_norm(x, weight, residual, eps)

q, k (B, H, n, dk), v (B, H, n, dv), each with strides of its own; gradients flow to q, k, v and initial_state (log_decay
is fixed: one that wants a gradient is refused).  x, residual (..., cols), weight float32 (cols) or None; gradients flow to all three.
"""
import ctypes
import warnings

import torch

from . import binding


_node = None   # (False: it does not load)


def _load_node():
    """The extension that holds the operators' nodes of the autograd graph (csrc/wersa_torch.cpp), on the library that the
    binding has loaded.  It is bound to one version of torch where the library is not: without it the node in Python makes the same
    calls, and a warning says that its host path is the slower one."""
    global _node
    if _node is None:
        lib = binding.load_library()
        try:
            from . import _wersa_torch as node
        except ImportError as e:
            warnings.warn("the autograd extension _wersa_torch.so is missing or does not load, training steps take up to 100 us longer on "
                          f"the host: build it with `python -m paper_2507_08637_amd.build` ({e})", RuntimeWarning, stacklevel=3)
            _node = False
            return _node
        node.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (lib.wersa_forward, lib.wersa_backward, lib.wersa_workspace_bytes,
                                                                    lib.wersa_saved_bytes, lib.wersa_selected_path)))
        node.bind_causal([ctypes.cast(f, ctypes.c_void_p).value for f in (
            lib.wersa_decay_forward, lib.wersa_decay_backward, lib.wersa_decay_workspace_bytes, lib.wersa_decay_saved_bytes,
            lib.wersa_rms_norm_forward, lib.wersa_rms_norm_backward, lib.wersa_rms_norm_workspace_bytes)])
        _node = node
    return _node


class _WersaAttention(torch.autograd.Function):
    """The same node in Python, for torch.jit.trace (the tracer records its call, and of the one in C++ only the allocation of the output) and where
    the extension does not load."""

    @staticmethod
    def forward(ctx, q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor):
        out, saved = binding.wersa_forward(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps=eps,
                                           bw_floor=bw_floor)
        ctx.save_for_backward(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, out, saved)
        ctx.cfg = (L, eps, bw_floor, q.stride())
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, out, saved = ctx.saved_tensors
        L, eps, bw_floor, strides = ctx.cfg
        # (saved-tensor hooks may have made them dense; `saved` is laid out for the path that the forward's strides select)
        q, k, v, out, dout = (x if x.stride() == strides else torch.empty_strided(x.shape, strides, dtype=x.dtype, device=x.device).copy_(x)
                              for x in (q, k, v, out, dout))
        g = binding.wersa_backward(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, out, dout, saved, L,
                                   eps=eps, bw_floor=bw_floor)
        return (g["dq"], g["dk"], g["dv"], None, g["dsigma"], g["dgate_w"], g["dgate_b"], g["dscale_w"],
                None, None, None)


def wersa_attention(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps=1e-6, bw_floor=1e-6):
    node = _load_node() if _node is None else _node
    if not node or torch.jit.is_tracing():
        return _WersaAttention.apply(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor)
    desc, saved_bytes, workspace = binding.checked_desc(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor, 0)
    return node.attention(q, k, v, omega_rf, sigma, gate_w, gate_b, scale_w, bytes(desc), saved_bytes, workspace)


class _WersaBlock(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor):
        y, saved = binding.wersa_block_forward(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, L,
                                               eps=eps, bw_floor=bw_floor)
        ctx.save_for_backward(x, wq, wk, wv, wo, omega_rf, sigma, gate_w, gate_b, scale_w, saved)
        ctx.cfg = (H, L, eps, bw_floor)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, wq, wk, wv, wo, omega_rf, sigma, gate_w, gate_b, scale_w, saved = ctx.saved_tensors
        H, L, eps, bw_floor = ctx.cfg
        g = binding.wersa_block_backward(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w,
                                         dy.contiguous(), saved, L, eps=eps, bw_floor=bw_floor)
        cast = lambda t: t.to(wq.dtype)
        return (g["dx"], cast(g["dwq"]), cast(g["dwk"]), cast(g["dwv"]), cast(g["dwo"]), None, None, g["dsigma"],
                g["dgate_w"], g["dgate_b"], g["dscale_w"], None, None, None)


def wersa_attention_block(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps=1e-6,
                          bw_floor=1e-6):
    return _WersaBlock.apply(x, wq, wk, wv, wo, H, omega_rf, sigma, gate_w, gate_b, scale_w, L, eps, bw_floor)


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, scale, initial_state, offsets):
        out, final_state, saved = binding.wersa_decay_forward(q, k, v, log_decay, scale=scale, offsets=offsets, initial_state=initial_state,
                                                              want_state=True, want_saved=True)
        ctx.save_for_backward(q, k, v, log_decay, initial_state, offsets, saved)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return out, final_state

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dfinal):
        q, k, v, log_decay, initial_state, offsets, saved = ctx.saved_tensors
        dout = torch.zeros_like(v) if dout is None else _rows_apart(dout)
        g = binding.wersa_decay_backward(q, k, v, log_decay, dout, saved, scale=ctx.scale, offsets=offsets, initial_state=initial_state,
                                         dfinal_state=None if dfinal is None else dfinal.contiguous(), want_dinitial=ctx.needs_input_grad[5])
        return g["dq"], g["dk"], g["dv"], None, None, g["dinitial_state"], None


def _rows_apart(x):
    """x with contiguous columns, and strides as the library reads them: rows that do not share memory, heads and sequences that are not one (an
    expanded tensor is copied)."""
    apart = x.stride(3) == 1 and all(x.stride(i) > 0 or x.shape[i] == 1 for i in range(2)) and (x.stride(2) >= x.shape[3] or x.shape[2] <= 1)
    return x if apart else x.contiguous()


def wersa_decay_attention(q, k, v, log_decay, scale=None, initial_state=None, offsets=None):
    """Causal linear attention with a decay for each head.  Returns (out, final states (B, H, dk, dv) in float32).  Rows of no sequence (offsets that
    begin behind the first row or end before the last one) are zeros in out and in the gradients, whatever they hold in q, k, v and out's gradient."""
    assert not (log_decay.requires_grad and torch.is_grad_enabled()), "log_decay is fixed and has no gradient: pass log_decay.detach() if none is wanted"
    q, k, v = _rows_apart(q), _rows_apart(k), _rows_apart(v)
    node = _load_node() if _node is None else _node
    if not node or torch.jit.is_tracing():
        return _DecayAttention.apply(q, k, v, log_decay, scale, initial_state, offsets)
    desc, saved_bytes = binding.checked_decay_desc(q, k, v, log_decay, scale, offsets, initial_state)
    return tuple(node.decay_attention(q, k, v, log_decay, initial_state, offsets, bytes(desc), saved_bytes))


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, r, rstd = binding.wersa_rms_norm_forward(x, weight, residual=residual, eps=eps, want_rstd=True)
        ctx.save_for_backward(x if residual is None else r, weight, rstd)
        ctx.set_materialize_grads(False)
        return y if residual is None else (y, r)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dr=None):
        r, weight, rstd = ctx.saved_tensors
        dense = lambda t: None if t is None else t.contiguous()
        if dy is None:
            dy = torch.zeros(r.shape, dtype=r.dtype, device=r.device)
        dx, dw = binding.wersa_rms_norm_backward(r, rstd, dense(dy), weight, dense(dr), want_dweight=weight is not None and ctx.needs_input_grad[1])
        return dx, dw, dx if ctx.needs_input_grad[2] else None, None


def _as_rows(x):
    """(rows, cols), columns contiguous, rows that do not share memory: a view, or a copy of what is not laid out so (transposed, broadcast)."""
    if x.dim() != 2:
        x = x.reshape(-1, x.shape[-1])
    apart = x.stride(1) == 1 and (x.stride(0) >= x.shape[1] or x.shape[0] <= 1)
    return x if apart else x.clone(memory_format=torch.contiguous_format)


def wersa_rms_norm(x, weight=None, residual=None, eps=1e-6):
    """RMS norm over the last dimension: y, or (y, x + residual)."""
    shape = x.shape
    assert residual is None or residual.shape == shape, "the residual has x's shape and dtype"
    x, residual = _as_rows(x), None if residual is None else _as_rows(residual)
    node = _load_node() if _node is None else _node
    if not node or torch.jit.is_tracing():
        outs = _RmsNorm.apply(x, weight, residual, eps)
        outs = (outs,) if residual is None else outs
    else:
        binding.checked_norm_args(x, weight, residual)
        outs = node.rms_norm(x, weight, residual, eps)
    if len(shape) != 2:
        outs = [t.view(shape) for t in outs]
    return outs[0] if residual is None else tuple(outs)
