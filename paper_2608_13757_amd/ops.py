"""The operators beside the plans (include/bfs.h): a mixture of experts'
router, dispatch and combination with their gradients, and the global gradient
norm with clipping.

Argument checks and marshalling only.  Tensors are torch tensors on the
current device; a refused argument raises BfsError (E_INVALID or E_RESOURCE)
before anything is launched.  An output must not share memory with an input or
another output, except where it is said.  Outputs that are not given are
allocated on the current stream.  ``stream``: a torch stream or handle, None
the current one; on another stream than the current one every output (and the
workspace) has to be given, since an allocation belongs to the stream that it
was made on.  No autograd graph is recorded: the gradients are calls of their
own.

Calls of a few tokens are bound by the host (some 2.5 us of a call are the launch),
so the checks stand in the calls themselves; the functions they call say what
is wrong.
"""
from __future__ import annotations

import ctypes as C
import functools
import struct

import torch

from . import bfs
from .bfs import E_INVALID, E_RESOURCE, OK, BfsError

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
MOE_RENORMALIZE = 1
MAX_EXPERTS = 1024
DISPATCH_ALONE = 8192            # slots up to which a dispatch needs no workspace
# bfs_call's words: the operator, the number of its arguments, the arguments
_ROUTE, _ROUTE_GRAD, _DISPATCH, _COMBINE, _COMBINE_GRAD, _NORM, _CLIP = (
    struct.Struct(f).pack for f in ("12q", "14q", "18q", "14q", "17q", "8q", "4qd4q"))
_I32, _F32 = torch.int32, torch.float32

# The current device and its current stream's handle, by the bindings that
# torch.cuda's functions wrap (which take most of a microsecond together).
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: bfs._stream_handle(None))


def _refuse(name, what):
    raise BfsError(E_INVALID, f"{name}: {what}")


def _refuse_matrix(name, what, t):
    _refuse(name, f"{what} must be a matrix on the current device with unit stride in its rows, not {tuple(t.shape)} with "
                  f"strides {t.stride()} on {t.device}")


def _refuse_like(name, what, t, shape, dtype):
    _refuse(name, f"{what} must be {dtype} of shape {tuple(shape)} on the current device with unit stride in rows that do "
                  f"not overlap, not {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _refuse_dense(name, what, t, shape, dtype):
    _refuse(name, f"{what} must be contiguous {dtype} of shape {tuple(shape)} on the current device, not {t.dtype} "
                  f"{tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _refuse_type(name, what, t):
    _refuse(name, f"{what} of type {t.dtype} (float32, bfloat16 and float16 are supported)")


def _refuse_experts(name, n_experts):
    raise BfsError(E_INVALID if n_experts < 1 else E_RESOURCE, f"{name}: n_experts = {n_experts} (1 .. {MAX_EXPERTS})")


def _stream(name, stream, device, given):
    """Handle of a stream; ``given``: whether nothing has to be allocated."""
    handle = bfs._stream_handle(stream)
    if getattr(stream, "device_index", device) != device:
        _refuse(name, "the stream belongs to another device")
    if not given and handle != _raw_stream(device):
        _refuse(name, "on another stream than the current one every output and the workspace must be given")
    return handle


def _call(function, *args):
    status = function(*args)
    if status != OK:
        bfs._check(status)


def moe_route(logits, k, *, renormalize=True, experts=None, weights=None, stream=None):
    """(experts int32 [T, k], weights float32 [T, k]): the k experts of each
    token with the largest logits ([T, E]; equal ones by the lower index) and
    their softmax over the chosen ones (``renormalize``) or over all experts.
    A logit of -inf masks its expert; slots left without one hold -1 and
    weight 0."""
    name = "moe_route"
    device, size = logits.get_device(), logits.shape
    if device < 0 or device != _device() or len(size) != 2:
        _refuse_matrix(name, "logits", logits)
    t, e = size
    stride, unit = logits.stride()
    if unit != 1 and e > 1:
        _refuse_matrix(name, "logits", logits)
    dtype = DTYPES.get(logits.dtype)
    if dtype is None:
        _refuse_type(name, "logits", logits)
    if not 1 <= k <= e:
        _refuse(name, f"k = {k} of {e} experts")
    handle = _raw_stream(device) if stream is None else _stream(name, stream, device, experts is not None and weights is not None)
    shape = (t, k)
    if experts is None:
        experts = logits.new_empty(shape, dtype=_I32)
    elif experts.dtype is not _I32 or experts.shape != shape or experts.get_device() != device or not experts.is_contiguous():
        _refuse_dense(name, "experts", experts, shape, _I32)
    if weights is None:
        weights = logits.new_empty(shape, dtype=_F32)
    elif weights.dtype is not _F32 or weights.shape != shape or weights.get_device() != device or not weights.is_contiguous():
        _refuse_dense(name, "weights", weights, shape, _F32)
    status = (bfs._lib or bfs.lib()).bfs_call(_ROUTE(
        0, 10, logits.data_ptr(), dtype, t, e, stride, k, MOE_RENORMALIZE if renormalize else 0, experts.data_ptr(),
        weights.data_ptr(), handle))
    if status:
        bfs._check(status)
    return experts, weights


def moe_route_grad(logits, experts, grad_weights, *, renormalize=True, grad_logits=None, stream=None):
    """The gradient of the logits (of their type) for the gradient of the
    router's weights; ``experts`` and ``renormalize`` as the router had them."""
    name = "moe_route_grad"
    device, size = logits.get_device(), logits.shape
    if device < 0 or device != _device() or len(size) != 2:
        _refuse_matrix(name, "logits", logits)
    t, e = size
    stride, unit = logits.stride()
    if unit != 1 and e > 1:
        _refuse_matrix(name, "logits", logits)
    dtype = DTYPES.get(logits.dtype)
    if dtype is None:
        _refuse_type(name, "logits", logits)
    k = experts.shape[-1] if experts.shape else 1
    shape = (t, k)
    if experts.dtype is not _I32 or experts.shape != shape or experts.get_device() != device or not experts.is_contiguous():
        _refuse_dense(name, "experts", experts, shape, _I32)
    if (grad_weights.dtype is not _F32 or grad_weights.shape != shape or grad_weights.get_device() != device
            or not grad_weights.is_contiguous()):
        _refuse_dense(name, "grad_weights", grad_weights, shape, _F32)
    handle = _raw_stream(device) if stream is None else _stream(name, stream, device, grad_logits is not None)
    if grad_logits is None:
        grad_logits = logits.new_empty(size)
    elif grad_logits.dtype is not logits.dtype or grad_logits.shape != size or grad_logits.get_device() != device:
        _refuse_like(name, "grad_logits", grad_logits, size, logits.dtype)
    out_stride, unit = grad_logits.stride()
    if (unit != 1 and e > 1) or (out_stride < e and t > 1):
        _refuse_like(name, "grad_logits", grad_logits, size, logits.dtype)
    status = (bfs._lib or bfs.lib()).bfs_call(_ROUTE_GRAD(
        1, 12, logits.data_ptr(), dtype, t, e, stride, experts.data_ptr(), k, grad_weights.data_ptr(),
        MOE_RENORMALIZE if renormalize else 0, grad_logits.data_ptr(), out_stride if t > 1 else e, handle))
    if status:
        bfs._check(status)
    return grad_logits


@functools.lru_cache(maxsize=1024)
def moe_dispatch_workspace(n_tokens, k, n_experts):
    """Bytes of device memory that a dispatch of these sizes works in."""
    if n_experts > MAX_EXPERTS:
        _refuse_experts("moe_dispatch_workspace", n_experts)
    n = C.c_int64()
    _call(bfs.lib().bfs_moe_dispatch_workspace, n_tokens, k, n_experts, C.byref(n))
    return n.value


def moe_dispatch(experts, n_experts, x=None, *, perm=None, expert_off=None, pos=None, rows=None, workspace=None,
                 stream=None):
    """(perm, expert_off, pos, rows): the slots of ``experts`` (int32 [T, k],
    ids outside 0 .. n_experts - 1: none) in a stable order by expert.  perm
    int32 [T * k]: each row's token; expert_off int32 [n_experts + 1]: each
    expert's first row, last the number of rows (the MoE plans' buffers); pos
    int32 [T, k]: each slot's row or -1; rows [T * k, width]: x[token], None
    without x [T, width].  Entries of perm and rows behind the last row are
    left as they were."""
    name = "moe_dispatch"
    device, shape = experts.get_device(), experts.shape
    if device < 0 or device != _device() or len(shape) != 2 or experts.dtype is not _I32 or not experts.is_contiguous():
        _refuse(name, f"experts must be a contiguous int32 matrix on the current device, not {experts.dtype} {tuple(shape)}")
    if not 1 <= n_experts <= MAX_EXPERTS:
        _refuse_experts(name, n_experts)
    t, k = shape
    slots = t * k
    alone = k and slots <= DISPATCH_ALONE
    handle = _raw_stream(device) if stream is None else _stream(
        name, stream, device, perm is not None and expert_off is not None and pos is not None
        and (x is None or rows is not None) and (alone or workspace is not None))
    if perm is None:
        perm = experts.new_empty(slots)
    elif perm.dtype is not _I32 or perm.shape != (slots,) or perm.get_device() != device or not perm.is_contiguous():
        _refuse_dense(name, "perm", perm, (slots,), _I32)
    if expert_off is None:
        expert_off = experts.new_empty(n_experts + 1)
    elif (expert_off.dtype is not _I32 or expert_off.shape != (n_experts + 1,) or expert_off.get_device() != device
          or not expert_off.is_contiguous()):
        _refuse_dense(name, "expert_off", expert_off, (n_experts + 1,), _I32)
    if pos is None:
        pos = experts.new_empty(shape)
    elif pos.dtype is not _I32 or pos.shape != shape or pos.get_device() != device or not pos.is_contiguous():
        _refuse_dense(name, "pos", pos, shape, _I32)
    x_ptr = rows_ptr = ws_ptr = dtype = width = x_stride = rows_stride = ws_bytes = 0
    if x is not None:
        size = x.shape
        if x.get_device() != device or len(size) != 2 or size[0] != t:
            _refuse(name, f"x must be a matrix of {t} rows on the current device, not {tuple(size)}")
        width = size[1]
        x_stride, unit = x.stride()
        if unit != 1 and width > 1:
            _refuse_matrix(name, "x", x)
        dtype = DTYPES.get(x.dtype)
        if dtype is None:
            _refuse_type(name, "x", x)
        if rows is None:
            rows = x.new_empty((slots, width))
        elif rows.dtype is not x.dtype or rows.shape != (slots, width) or rows.get_device() != device:
            _refuse_like(name, "rows", rows, (slots, width), x.dtype)
        rows_stride, unit = rows.stride()
        if (unit != 1 and width > 1) or (rows_stride < width and slots > 1):
            _refuse_like(name, "rows", rows, (slots, width), x.dtype)
        if slots <= 1:
            rows_stride = width
        x_ptr, rows_ptr = x.data_ptr(), rows.data_ptr()
    elif rows is not None:
        _refuse(name, "rows without x")
    if not alone:
        if workspace is None:
            workspace = experts.new_empty((moe_dispatch_workspace(t, k, n_experts) + 3) // 4)
        elif workspace.get_device() != device or not workspace.is_contiguous():
            _refuse(name, "workspace must be a contiguous tensor on the current device")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    status = (bfs._lib or bfs.lib()).bfs_call(_DISPATCH(
        2, 16, experts.data_ptr(), t, k, n_experts, perm.data_ptr(), expert_off.data_ptr(), pos.data_ptr(), x_ptr, dtype, width,
        x_stride, rows_ptr, rows_stride, ws_ptr, ws_bytes, handle))
    if status:
        bfs._check(status)
    return perm, expert_off, pos, rows


def _combine(name, rows, pos, weights, out, stream):
    device, size, shape = rows.get_device(), rows.shape, pos.shape
    if device < 0 or device != _device() or len(size) != 2:
        _refuse_matrix(name, "rows", rows)
    n, width = size
    stride, unit = rows.stride()
    if unit != 1 and width > 1:
        _refuse_matrix(name, "rows", rows)
    dtype = DTYPES.get(rows.dtype)
    if dtype is None:
        _refuse_type(name, "rows", rows)
    if pos.dtype is not _I32 or len(shape) != 2 or pos.get_device() != device or not pos.is_contiguous():
        _refuse(name, f"pos must be a contiguous int32 matrix on the current device, not {pos.dtype} {tuple(shape)}")
    t, k = shape
    w_ptr = 0
    if weights is not None:
        if weights.dtype is not _F32 or weights.shape != shape or weights.get_device() != device or not weights.is_contiguous():
            _refuse_dense(name, "weights", weights, shape, _F32)
        w_ptr = weights.data_ptr()
    handle = _raw_stream(device) if stream is None else _stream(name, stream, device, out is not None)
    if out is None:
        out = rows.new_empty((t, width))
    elif out.dtype is not rows.dtype or out.shape != (t, width) or out.get_device() != device:
        _refuse_like(name, "out", out, (t, width), rows.dtype)
    out_stride, unit = out.stride()
    if (unit != 1 and width > 1) or (out_stride < width and t > 1):
        _refuse_like(name, "out", out, (t, width), rows.dtype)
    status = (bfs._lib or bfs.lib()).bfs_call(_COMBINE(
        3, 12, rows.data_ptr(), dtype, n, width, stride, pos.data_ptr(), w_ptr, t, k, out.data_ptr(),
        out_stride if t > 1 else width, handle))
    if status:
        bfs._check(status)
    return out


def moe_combine(rows, pos, weights, *, out=None, stream=None):
    """[T, width]: the sum over j of weights[t, j] * rows[pos[t, j]]; slots
    without a row (pos outside the rows) add nothing."""
    if weights is None:
        _refuse("moe_combine", "weights are needed")
    return _combine("moe_combine", rows, pos, weights, out, stream)


def moe_dispatch_grad(grad_rows, pos, *, out=None, stream=None):
    """The gradient of the dispatch's x: the sum of each token's rows."""
    return _combine("moe_dispatch_grad", grad_rows, pos, None, out, stream)


def moe_combine_grad(grad_y, rows, pos, weights, *, grad_rows=None, grad_weights=None, stream=None):
    """(grad_rows, grad_weights) of the combination: grad_rows[pos[t, j]] =
    weights[t, j] * grad_y[t], grad_weights[t, j] = <grad_y[t],
    rows[pos[t, j]]>.  Slots have different rows, as the dispatch gives them;
    rows that no slot names are left as they were (zeros in a grad_rows that
    the call allocates, which costs a pass over it)."""
    name = "moe_combine_grad"
    device, size, shape = grad_y.get_device(), grad_y.shape, rows.shape
    if device < 0 or device != _device() or len(size) != 2:
        _refuse_matrix(name, "grad_y", grad_y)
    t, width = size
    dy_stride, unit = grad_y.stride()
    if unit != 1 and width > 1:
        _refuse_matrix(name, "grad_y", grad_y)
    dtype = DTYPES.get(grad_y.dtype)
    if dtype is None:
        _refuse_type(name, "grad_y", grad_y)
    if rows.dtype is not grad_y.dtype or len(shape) != 2 or shape[1] != width or rows.get_device() != device:
        _refuse(name, f"rows must be {grad_y.dtype} of {width} columns on the current device, not {rows.dtype} {tuple(shape)}")
    n = shape[0]
    rows_stride, unit = rows.stride()
    if unit != 1 and width > 1:
        _refuse_matrix(name, "rows", rows)
    k = pos.shape[-1] if pos.shape else 1
    slots = (t, k)
    if pos.dtype is not _I32 or pos.shape != slots or pos.get_device() != device or not pos.is_contiguous():
        _refuse_dense(name, "pos", pos, slots, _I32)
    if weights.dtype is not _F32 or weights.shape != slots or weights.get_device() != device or not weights.is_contiguous():
        _refuse_dense(name, "weights", weights, slots, _F32)
    handle = _raw_stream(device) if stream is None else _stream(name, stream, device,
                                                                grad_rows is not None and grad_weights is not None)
    if grad_rows is None:
        grad_rows = rows.new_zeros(shape)
    elif grad_rows.dtype is not grad_y.dtype or grad_rows.shape != shape or grad_rows.get_device() != device:
        _refuse_like(name, "grad_rows", grad_rows, shape, grad_y.dtype)
    out_stride, unit = grad_rows.stride()
    if (unit != 1 and width > 1) or (out_stride < width and n > 1):
        _refuse_like(name, "grad_rows", grad_rows, shape, grad_y.dtype)
    if grad_weights is None:
        grad_weights = weights.new_empty(slots)
    elif (grad_weights.dtype is not _F32 or grad_weights.shape != slots or grad_weights.get_device() != device
          or not grad_weights.is_contiguous()):
        _refuse_dense(name, "grad_weights", grad_weights, slots, _F32)
    status = (bfs._lib or bfs.lib()).bfs_call(_COMBINE_GRAD(
        4, 15, grad_y.data_ptr(), dtype, t, width, dy_stride, rows.data_ptr(), n, rows_stride, pos.data_ptr(), weights.data_ptr(),
        k, grad_rows.data_ptr(), out_stride if n > 1 else width, grad_weights.data_ptr(), handle))
    if status:
        bfs._check(status)
    return grad_rows, grad_weights


class GradSet:
    """The gradients of a model, for their global norm and clipping.

    ``grads``: contiguous float32, bfloat16 or float16 tensors.  ``out``: None
    (they are clipped in place), a flat tensor that takes them one after the
    other (float32, or the type of all of them: the gradient buffer of an
    AdamW plan), or a tensor for each.  Like a plan its program, the set keeps
    a table of the tensors on the device, and their memory: a gradient that is
    allocated anew (as torch's zero_grad() lets them be) needs a new set, the
    old one goes on with the old memory.  A gradient named twice counts twice in the
    norm; a set whose outputs overlap (that one in place, say) is not clipped.
    Making one copies the table (it waits for the copy, some 60 us of the host
    for 24 tensors, 470 for 290, and cannot be captured); the calls can be.  A set may be dropped while a call of it is under way, on
    whatever stream: its memory is used again only behind that stream's work.
    A stream given by its handle has to exist until the set is gone, and a set
    whose calls were captured has to be kept as long as the graph."""

    def __init__(self, grads, out=None):
        name = "GradSet"
        grads = list(grads)
        for g in grads:
            if not isinstance(g, torch.Tensor) or not g.is_cuda or not g.is_contiguous():
                _refuse(name, "gradients must be contiguous tensors on a device")
            if g.dtype not in DTYPES:
                _refuse_type(name, "a gradient", g)
        types = [DTYPES[g.dtype] for g in grads]
        sizes = [g.numel() for g in grads]
        if out is None:
            outs = grads
        elif isinstance(out, torch.Tensor):
            if out.dim() != 1 or out.numel() != sum(sizes) or not out.is_cuda or not out.is_contiguous():
                _refuse(name, f"out must be a contiguous vector of {sum(sizes)} elements on a device")
            outs = out.split(sizes) if grads else []
        else:
            outs = list(out)
            if len(outs) != len(grads):
                _refuse(name, f"{len(outs)} outputs for {len(grads)} gradients")
            for o, g in zip(outs, grads):
                if not isinstance(o, torch.Tensor) or not o.is_cuda or not o.is_contiguous() or o.shape != g.shape:
                    _refuse(name, "an output must be contiguous and of its gradient's shape")
        devices = {t.get_device() for t in [*grads, *outs]}
        if len(devices) > 1:
            _refuse(name, "tensors on several devices")
        for o, g in zip(outs, grads):
            if o.dtype is not torch.float32 and o.dtype is not g.dtype:
                _refuse(name, f"an output is float32 or has its gradient's type, not {o.dtype} for {g.dtype}")
        # aliases: the memory stays even where a tensor's data is exchanged
        self._keep = [t.detach() for t in [*grads, *outs]]
        self._device = devices.pop() if devices else None
        # The stream that the table's memory belongs to, and the other ones that calls ran on.
        self._made_on = None if self._device is None else _raw_stream(self._device)
        self._used_on = set()
        n = len(grads)
        arrays = (struct.pack("%dP" % n, *[g.data_ptr() for g in grads]), struct.pack("%dP" % n, *[o.data_ptr() for o in outs]),
                  struct.pack("%dq" % n, *sizes), struct.pack("%di" % n, *types),
                  struct.pack("%di" % n, *[DTYPES[o.dtype] for o in outs]), n)
        table = bfs.lib().bfs_grad_table
        self._set = bfs.GradSetStruct()
        _call(table, *arrays, C.byref(self._set), None, 0)
        size = self._set.image_bytes
        self._table = None
        if size:
            image = bytearray(size)
            _call(table, *arrays, C.byref(self._set), (C.c_char * size).from_buffer(image), size)
            self._table = torch.frombuffer(image, dtype=torch.uint8).to(grads[0].device)     # waits for the copy
            self._keep.append(self._table)
        self._args = C.addressof(self._set), 0 if self._table is None else self._table.data_ptr()
        self.workspace_bytes = self._set.workspace_bytes
        self._words = (self.workspace_bytes + 3) // 4

    def _record(self, stream, handle):
        """The allocator is told that a stream uses the set's memory: once for
        each stream, it holds until the memory goes back."""
        if stream is None:
            stream = torch.cuda.current_stream()
        elif isinstance(stream, int):                  # (no handle of torch's wrapper: 0, the default stream)
            stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
        for t in self._keep:
            t.record_stream(stream)
        self._used_on.add(handle)

    def _buffers(self, name, norm, workspace, stream):
        device = _device()
        if device != self._device and self._device is not None:
            _refuse(name, "the gradients are not on the current device")
        handle = _raw_stream(device) if stream is None else _stream(name, stream, device,
                                                                    norm is not None and workspace is not None)
        if norm is None:
            norm = torch.empty((), dtype=_F32, device="cuda")
        elif norm.dtype is not _F32 or norm.dim() != 0 or norm.get_device() != device:
            _refuse_dense(name, "norm", norm, (), _F32)
        if workspace is not None and (workspace.get_device() != device or not workspace.is_contiguous()):
            _refuse(name, "workspace must be a contiguous tensor on the current device")
        if handle != self._made_on and handle not in self._used_on:
            self._record(stream, handle)
        if workspace is None:
            return norm, norm.new_empty(self._words), self.workspace_bytes, handle
        return norm, workspace, workspace.numel() * workspace.element_size(), handle

    def norm(self, norm=None, workspace=None, stream=None):
        """The global norm, a float32 scalar on the device."""
        norm, workspace, size, handle = self._buffers("grad_norm", norm, workspace, stream)
        address, table = self._args
        status = bfs._lib.bfs_call(_NORM(5, 6, address, table, norm.data_ptr(), workspace.data_ptr(), size, handle))
        if status:
            bfs._check(status)
        return norm

    def clip(self, max_norm, norm=None, workspace=None, stream=None):
        """Writes grads * min(1, max_norm / (norm + 1e-6)) to the outputs and
        returns the norm before clipping.  A norm that is not finite in
        float32, as it is returned, scales by 1, also where only float32 does
        not hold it: gradients beside an infinite norm are as they were."""
        norm, workspace, size, handle = self._buffers("grad_clip", norm, workspace, stream)
        address, table = self._args
        status = bfs._lib.bfs_call(_CLIP(6, 7, address, table, max_norm, norm.data_ptr(), workspace.data_ptr(), size, handle))
        if status:
            bfs._check(status)
        return norm


def grad_norm(grads, **kw):
    """GradSet(grads).norm(), for gradients that are used once (not captured)."""
    return GradSet(grads).norm(**kw)


def grad_clip(grads, max_norm, out=None, **kw):
    """GradSet(grads, out).clip(max_norm), for gradients that are used once (not captured)."""
    return GradSet(grads, out).clip(max_norm, **kw)
