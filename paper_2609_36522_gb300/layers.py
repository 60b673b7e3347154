"""Layers of a text-conditioned denoiser on the solver's batch, forward and backward.

``layer_norm`` and ``cross_attention`` with their gradients, as kernels of
libparaanya.so behind plain functions: tensors in, tensors out, on the current
stream (or ``stream``). A denoiser for ``Solver`` gets the rows of the batch
with their (trajectory, timestep) pairs; ``cross_attention`` takes the states of
the text encoder once per trajectory and ``source=miss_bt[:, 0]``, so that the
rows of a trajectory share them. Inside a captured loop (``Solver.generate``)
give ``count`` (the device address of the miss count), the output buffers and
``workspace``: then nothing is allocated. There is no fallback implementation.
"""
from __future__ import annotations

import torch

from . import abi

_DTYPES = {torch.float32: abi.PA_F32, torch.float16: abi.PA_F16, torch.bfloat16: abi.PA_BF16}


def _on(x, stream):
    """The stream's address; allocations must be made with that stream current."""
    if stream is None:
        stream = torch.cuda.current_stream(x.device)
    return stream.cuda_stream


class _Place:
    """The tensors' device and the given stream as the current ones."""

    def __init__(self, x, stream):
        self.guards = []
        if x.device.index != torch.cuda.current_device():
            self.guards.append(torch.cuda.device(x.device))
        if stream is not None:
            self.guards.append(torch.cuda.stream(stream))

    def __enter__(self):
        for g in self.guards:
            g.__enter__()

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _check(ok, what):
    if not ok:
        raise ValueError(what)


def _device(name, t, like):
    _check(isinstance(t, torch.Tensor) and t.is_cuda and t.device == like.device, f"{name} must be a tensor on x's GPU")


def _count(count, like):
    """Device address of an int32: a tensor or, as the solver hands it out, an address."""
    if count is None or isinstance(count, int):
        return count
    _device("count", count, like)
    _check(count.dtype == torch.int32 and count.numel() == 1, "count must be one int32 on the device")
    return count.data_ptr()


def _workspace(workspace, need, like):
    if need == 0:
        return None, 0, None
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    else:
        _device("workspace", workspace, like)
        _check(workspace.is_contiguous(), "workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


# ---- layer norm ----------------------------------------------------------------

def _rows(name, x, like=None):
    """(rows, row stride) of a tensor [..., cols] whose rows lie at one distance."""
    _check(isinstance(x, torch.Tensor) and x.is_cuda and x.dim() >= 1, f"{name} must be a CUDA tensor")
    if like is not None:
        _check(x.shape == like.shape and x.dtype == like.dtype and x.device == like.device,
               f"{name} must have x's shape, type and device")
    cols = x.shape[-1]
    if x.is_contiguous():
        return x.numel() // cols if cols else 0, cols
    _check(x.stride(-1) == 1 or cols == 1, f"{name}'s last axis must be contiguous")
    rows, step = 1, None
    for n, s in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
        if n == 1:
            continue
        _check(step is None or s == step * rows, f"{name}'s rows must lie at one distance")
        step = s if step is None else step
        rows *= n
    return rows, cols if step is None else step


def _weights(x, **named):
    for name, w in named.items():
        if w is not None:
            _device(name, w, x)
            _check(w.dtype == x.dtype and w.is_contiguous() and w.shape == x.shape[-1:],
                   f"{name} must be contiguous, of x's type and last size")


def _ptr(t):
    return None if t is None else t.data_ptr()


def layer_norm(x, weight=None, bias=None, eps=1e-5, stats=False, out=None, mean=None, rstd=None, count=None, stream=None):
    """Layer norm over the last axis of x (float32, float16 or bfloat16):
    y = (x - mean) rstd weight + bias. Returns y, with ``stats`` (or with
    buffers ``mean`` and ``rstd``) (y, mean, rstd) for ``layer_norm_backward``.
    ``out``: where y goes (x itself is allowed). ``count``: device int32, only
    the first ``count`` entries of x's first axis are computed."""
    rows, xs = _rows("x", x)
    _check(x.dtype in _DTYPES, "x must be float32, float16 or bfloat16")
    _weights(x, weight=weight, bias=bias)
    with _Place(x, stream):
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _, ys = _rows("out", out, x)
        if stats or mean is not None or rstd is not None:
            if mean is None:
                mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
            if rstd is None:
                rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
            _stats(x, mean, rstd)
        abi.pa_layer_norm(_DTYPES[x.dtype], rows, x.shape[-1], x.data_ptr(), xs, _ptr(weight), _ptr(bias), eps,
                          out.data_ptr(), ys, _ptr(mean), _ptr(rstd), _count(count, x),
                          _per_item(x, rows), _on(x, stream))
    return out if mean is None else (out, mean, rstd)


def _per_item(x, rows):
    return max(1, rows // x.shape[0]) if x.dim() > 1 and x.shape[0] else 1


def _stats(x, mean, rstd):
    for name, t in (("mean", mean), ("rstd", rstd)):
        _device(name, t, x)
        _check(t.dtype == torch.float32 and t.is_contiguous() and t.shape == x.shape[:-1],
               f"{name} must be contiguous float32 of x's shape without the last axis")


def layer_norm_backward(dy, x, mean, rstd, weight=None, weight_grad=True, bias_grad=True, dx=None, count=None,
                        workspace=None, stream=None):
    """Gradients of ``layer_norm`` for dy: (dx, dweight, dbias), None where
    ``weight_grad`` or ``bias_grad`` is False. mean and rstd are the forward
    call's. ``dx``: where it goes (dy or x themselves are allowed).
    ``workspace``: a CUDA tensor of at least
    ``abi.pa_layer_norm_backward_workspace_bytes(rows, cols)`` bytes."""
    rows, xs = _rows("x", x)
    _check(x.dtype in _DTYPES, "x must be float32, float16 or bfloat16")
    _, dys = _rows("dy", dy, x)
    _weights(x, weight=weight)
    _stats(x, mean, rstd)
    cols = x.shape[-1]
    with _Place(x, stream):
        if dx is None:
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        _, dxs = _rows("dx", dx, x)
        dw = torch.empty(cols, dtype=x.dtype, device=x.device) if weight_grad else None
        db = torch.empty(cols, dtype=x.dtype, device=x.device) if bias_grad else None
        need = abi.pa_layer_norm_backward_workspace_bytes(rows, cols) if weight_grad or bias_grad else 0
        ws, nbytes, keep = _workspace(workspace, need, x)
        abi.pa_layer_norm_backward(_DTYPES[x.dtype], rows, cols, dy.data_ptr(), dys, x.data_ptr(), xs, _ptr(weight),
                                   mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dxs, _ptr(dw), _ptr(db),
                                   _count(count, x), _per_item(x, rows), ws, nbytes, _on(x, stream))
    return dx, dw, db


# ---- cross attention --------------------------------------------------------------

def _arguments(q, k, v, scale, source, lengths, mask, count):
    """The argument block's first part: what both directions share."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 4, f"{name} must be a CUDA tensor of four axes")
        _check(t.dtype == q.dtype and t.device == q.device, f"{name} must have q's type and device")
    _check(q.dtype in (torch.float16, torch.bfloat16), "q, k and v must be float16 or bfloat16")
    _check(k.shape == v.shape and k.shape[3] == q.shape[3], "k and v need one shape, and q's last size")
    a = abi.PaAttention()
    a.dtype = _DTYPES[q.dtype]
    a.items, a.tokens, a.heads, a.head_dim = q.shape
    a.sources, a.keys, a.kv_heads = k.shape[:3]
    a.scale = q.shape[3] ** -0.5 if scale is None else scale
    a.q, a.q_stride = _tensor("q", q)
    a.k, a.k_stride = _tensor("k", k)
    a.v, a.v_stride = _tensor("v", v)
    if source is not None:
        _device("source", source, q)
        _check(source.dtype == torch.int32 and source.dim() == 1 and source.shape[0] >= q.shape[0],
               "source must be an int32 vector with an entry per item")
        a.source, a.source_stride = source.data_ptr(), source.stride(0)
    if lengths is not None:
        _device("lengths", lengths, q)
        _check(lengths.dtype == torch.int32 and lengths.is_contiguous() and lengths.shape == k.shape[:1],
               "lengths must be a contiguous int32 vector with an entry per source")
        a.lengths = lengths.data_ptr()
    if mask is not None:
        _device("mask", mask, q)
        _check(mask.dtype in (torch.bool, torch.uint8) and mask.shape == k.shape[:2]
               and (mask.stride(1) == 1 or mask.shape[1] <= 1),
               "mask must be bool or uint8 [sources][keys], its last axis contiguous")
        a.mask, a.mask_stride = mask.data_ptr() or None, mask.stride(0)
    a.n_items_dev = _count(count, q)
    return a


# an axis of one entry has no stride that matters (torch leaves any value there)
def _tensor(name, t, like=None):
    if like is not None:
        _check(isinstance(t, torch.Tensor) and t.is_cuda and t.shape == like.shape and t.dtype == like.dtype
               and t.device == like.device, f"{name} must have the shape, type and device of what it belongs to")
    shape, s = t.shape, t.stride()
    _check(s[3] == 1 or shape[3] == 1, f"{name}'s last axis must be contiguous")
    return t.data_ptr(), (s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0)


def cross_attention(q, k, v, scale=None, source=None, lengths=None, mask=None, count=None, stats=False, out=None, lse=None,
                    workspace=None, stream=None):
    """Attention of q [items][tokens][heads][dim] to k, v [sources][keys][kv_heads][dim]
    (float16 or bfloat16): softmax(scale q k^T) v over the keys of the item's source.

    ``scale``: default dim ** -0.5. ``source``: int32 per item (a strided view
    such as ``miss_bt[:, 0]`` will do), default item n attends to source n.
    ``lengths``: int32 per source, keys past it do not count; ``mask``: bool
    [sources][keys], False does not count; such keys are not read. Rows without
    keys give zeros. ``heads`` may be a multiple of ``kv_heads``: neighbouring
    heads share a key head. ``count``: device int32, only the first ``count``
    items are computed. Returns out, with ``stats`` (or a buffer ``lse``)
    (out, lse) for ``cross_attention_backward``: lse float32 [items][tokens][heads].
    ``workspace``: a CUDA tensor, see ``cross_attention_workspace_bytes``."""
    a = _arguments(q, k, v, scale, source, lengths, mask, count)
    with _Place(q, stream):
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        a.out, a.out_stride = _tensor("out", out, q)
        if stats and lse is None:
            lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        if lse is not None:
            _lse(lse, q)
            a.lse = lse.data_ptr()
        ws, nbytes, keep = _workspace(workspace, abi.pa_attention_workspace_bytes(a, 0), q)
        abi.pa_attention(a, ws, nbytes, _on(q, stream))
    return out if lse is None else (out, lse)


def _lse(lse, q):
    _device("lse", lse, q)
    _check(lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == q.shape[:3],
           "lse must be contiguous float32 [items][tokens][heads]")


def cross_attention_backward(dout, q, k, v, out, lse, scale=None, source=None, lengths=None, mask=None, count=None,
                             dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Gradients of ``cross_attention`` for dout: (dq, dk, dv). The arguments and
    out and lse are the forward call's; dk and dv are sums over all rows that
    attend to a source, and zero for keys that do not count."""
    a = _arguments(q, k, v, scale, source, lengths, mask, count)
    a.out, a.out_stride = _tensor("out", out, q)
    a.dout, a.dout_stride = _tensor("dout", dout, q)
    _lse(lse, q)
    a.lse = lse.data_ptr()
    with _Place(q, stream):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device) if dk is None else dk
        dv = torch.empty(v.shape, dtype=q.dtype, device=q.device) if dv is None else dv
        a.dq, a.dq_stride = _tensor("dq", dq, q)
        a.dk, a.dk_stride = _tensor("dk", dk, k)
        a.dv, a.dv_stride = _tensor("dv", dv, v)
        ws, nbytes, keep = _workspace(workspace, abi.pa_attention_workspace_bytes(a, 1), q)
        abi.pa_attention_backward(a, ws, nbytes, _on(q, stream))
    return dq, dk, dv


def cross_attention_workspace_bytes(q, k, mask=False, backward=False):
    """Bytes of workspace of a call on tensors of these shapes."""
    a = abi.PaAttention()
    a.dtype = abi.PA_BF16
    a.items, a.tokens, a.heads, a.head_dim = q.shape
    a.sources, a.keys, a.kv_heads = k.shape[:3]
    a.mask = 1 if mask else None
    return abi.pa_attention_workspace_bytes(a, backward)


def check(stream=None):
    """Wait for ``stream`` (default: the current one) and raise PaError if an
    attention call met a source index out of range or a wait that ran out."""
    if stream is None:
        stream = torch.cuda.current_stream()
    abi.pa_attention_check(stream.cuda_stream)
