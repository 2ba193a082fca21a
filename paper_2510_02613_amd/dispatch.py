"""Tokens sorted by expert and back over torch tensors, with gradients: for expert products that are not the layer's (those of four_bit.py,
a library's, adapters).

    rows, order = sort_tokens(x, ids, n_groups, expert_map=map)      # group g has rows order.offsets[g] .. order.offsets[g + 1] - 1
    y = ...                                                          # what the experts make of them, row by row
    out = combine_tokens(y, order, weights)

torch is plumbing here: it holds device memory, names the stream and records who needs a gradient.  Every function enqueues its kernels on
`stream` (the current one of the tensors' device by default) and returns the tensors that hold the results; results that are given are written
in place, and their rows behind the last one are not touched; results that a call makes itself are zeros there.  What a call allocates belongs
to `stream`.  Matrices are [rows, cols] with contiguous rows that start on 16 bytes; rows may lie further apart (`stride(0)`).

Where grad mode is on and x, y or weights require gradients, they are computed by kernels of this library, on the stream that is current in the call;
`stream` and results that are given are refused then, and so are gradients of gradients.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .layer import _owned_by
from .scaled import _DTYPE, _current_device, _current_stream, _device_of, _matrix, _whole


class Order(NamedTuple):
    """Where the assignments (token t, its j-th expert) stand: int32 tensors offsets [n_groups + 1], the groups' rows; source [tokens * top_k],
    the assignment t * top_k + j of every row, -1 behind the last; row [tokens, top_k], the row of every assignment, -1 where it has none."""
    offsets: torch.Tensor
    source: torch.Tensor
    row: torch.Tensor


class Sorted(NamedTuple):
    rows: torch.Tensor
    order: Order


_pack_sort, _pack_combine = B.packer(B.MoESortTokens), B.packer(B.MoECombineTokens)
_pack_backward = B.packer(B.MoECombineTokensBackward)


def sort_workspace(tokens: int, top_k: int, n_groups: int, device="cuda") -> Optional[torch.Tensor]:
    """A workspace for sort_tokens() of these sizes, or None when it needs none.  One for more tokens is enough for fewer."""
    n = B.moe_sort_tokens_workspace_bytes(tokens, top_k, n_groups)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _overwritten(tensors) -> None:
    """Results that were given count as changed in place: a backward pass that was to read what they held refuses."""
    if tensors:
        torch.autograd.graph.increment_version(tensors)


def _check_routing(ids: torch.Tensor, tokens: int, dev: int):
    if ids.dim() != 2 or ids.shape[0] != tokens:
        raise ValueError(f"ids must be [{tokens}, top_k], is {list(ids.shape)}")
    return ids.shape[1], _whole(ids, ids.shape, torch.int32, dev, "ids")


def _sort(x, ids, n_groups, expert_map, rows, order, workspace, stream, dev):
    if x.dim() != 2 or x.dtype not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    tokens, cols = x.shape
    top_k, pi = _check_routing(ids, tokens, dev)
    A, dt = tokens * top_k, x.dtype
    pm, n_experts = 0, 0
    if expert_map is not None:
        if expert_map.dim() != 1:
            raise ValueError("expert_map must be [n_experts]")
        n_experts = expert_map.shape[0]
        pm = _whole(expert_map, (n_experts,), torch.int32, dev, "expert_map")
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError("the workspace must be contiguous and on the device of x")
    if n_groups <= 0:
        raise ValueError(f"n_groups must be positive, is {n_groups}")
    zero_rest, written = rows is None, [t for t in (rows, *(order or ())) if t is not None]
    if rows is None or order is None or workspace is None:
        with _owned_by(stream):
            if rows is None:
                rows = torch.empty((A, cols), dtype=dt, device=x.device)
            if order is None:
                order = Order(*(torch.empty(shape, dtype=torch.int32, device=x.device) for shape in ((n_groups + 1,), (A,), (tokens, top_k))))
            if workspace is None:
                workspace = sort_workspace(tokens, top_k, n_groups, x.device)
    po = _whole(order.offsets, (n_groups + 1,), torch.int32, dev, "offsets")
    ps = _whole(order.source, (A,), torch.int32, dev, "source")
    pr = _whole(order.row, (tokens, top_k), torch.int32, dev, "row")
    px, ld_x = _matrix(x, (tokens, cols), dt, dev, "x")
    pt, ld_t = _matrix(rows, (A, cols), dt, dev, "rows")
    pk, nk = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    B.moe_sort_tokens(_pack_sort(tokens, top_k, n_groups, n_experts, cols, _DTYPE[dt], zero_rest, pi, pm, px, ld_x, pt, ld_t, po, ps, pr, pk, nk),
                      _current_stream(dev) if stream is None else stream.cuda_stream)
    _overwritten(written)
    return rows, order


def _combine(y, row, weights, out, stream, dev):
    if y.dim() != 2 or y.dtype not in _DTYPE:
        raise ValueError("y must be a bfloat16 or float32 matrix")
    if row.dim() != 2:
        raise ValueError("row must be [tokens, top_k]")
    tokens, top_k = row.shape
    cols, dt = y.shape[1], y.dtype
    written = [] if out is None else [out]
    if out is None:
        with _owned_by(stream):
            out = torch.empty((tokens, cols), dtype=dt, device=y.device)
    pr = _whole(row, row.shape, torch.int32, dev, "row")
    pw = 0 if weights is None else _whole(weights, (tokens, top_k), torch.float32, dev, "weights")
    py, ld_y = _matrix(y, (tokens * top_k, cols), dt, dev, "y")
    po, ld_o = _matrix(out, (tokens, cols), dt, dev, "out")
    B.moe_combine_tokens(_pack_combine(tokens, top_k, cols, _DTYPE[dt], py, ld_y, pr, pw, po, ld_o),
                         _current_stream(dev) if stream is None else stream.cuda_stream)
    _overwritten(written)
    return out


def _rows16(t: torch.Tensor) -> torch.Tensor:
    """A gradient as the kernels read it: autograd's may be broadcast or start anywhere."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _SortTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, ids, n_groups, expert_map, workspace):
        rows, order = _sort(x, ids, n_groups, expert_map, None, None, workspace, None, x.get_device())
        ctx.save_for_backward(order.row)
        ctx.mark_non_differentiable(*order)
        ctx.set_materialize_grads(False)
        return rows, order.offsets, order.source, order.row

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_rows, *_):
        if grad_rows is None:
            return None, None, None, None, None
        row, = ctx.saved_tensors
        return _combine(_rows16(grad_rows), row, None, None, None, grad_rows.get_device()), None, None, None, None


class _CombineTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, offsets, row):
        ctx.save_for_backward(y if ctx.needs_input_grad[1] else None, weights, offsets, row)
        ctx.set_materialize_grads(False)
        return _combine(y, row, weights, None, None, y.get_device())

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        if grad is None:
            return None, None, None, None
        y, weights, offsets, row = ctx.saved_tensors
        grad, dev, dt = _rows16(grad), grad.get_device(), grad.dtype
        tokens, top_k = row.shape
        cols = grad.shape[1]
        dy = torch.empty((tokens * top_k, cols), dtype=dt, device=grad.device) if ctx.needs_input_grad[0] else None
        dw = torch.empty((tokens, top_k), dtype=torch.float32, device=grad.device) if ctx.needs_input_grad[1] else None
        pg, ld_g = _matrix(grad, (tokens, cols), dt, dev, "grad")
        py, ld_y = (0, 0) if dw is None else _matrix(y, (tokens * top_k, cols), dt, dev, "y")
        pd, ld_d = (0, 0) if dy is None else _matrix(dy, dy.shape, dt, dev, "grad_y")
        B.moe_combine_tokens_backward(
            _pack_backward(tokens, top_k, cols, _DTYPE[dt], pg, ld_g, py, ld_y, row.data_ptr(), 0 if weights is None else weights.data_ptr(),
                           offsets.data_ptr() + 4 * (offsets.shape[0] - 1), pd, ld_d, 0 if dw is None else dw.data_ptr()), _current_stream(dev))
        return dy, dw, None, None


def _wants_gradient(what, *tensors) -> bool:
    if not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in tensors):
        return False
    if any(w is not None for w in what):
        raise ValueError("results that are given and a stream are for calls without a gradient")
    return True


def sort_tokens(x: torch.Tensor, ids: torch.Tensor, n_groups: int, *, expert_map: Optional[torch.Tensor] = None,
                rows: Optional[torch.Tensor] = None, order: Optional[Order] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> Sorted:
    """The rows of x [tokens, cols] in the order of their groups, one for every assignment ids [tokens, top_k] (int32) to a group of this rank:
    group expert_map[id] (int32 [n_experts], other ranks' -1), or the id itself without a map.  Groups outside [0, n_groups) are not this rank's."""
    dev = _device_of(x)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return sort_tokens(x, ids, n_groups, expert_map=expert_map, rows=rows, order=order, workspace=workspace, stream=stream)
    if _wants_gradient((rows, order, stream), x):
        got = _SortTokens.apply(x, ids, n_groups, expert_map, workspace)
        return Sorted(got[0], Order(*got[1:]))
    return Sorted(*_sort(x, ids, n_groups, expert_map, rows, order, workspace, stream, dev))


def combine_tokens(y: torch.Tensor, order: Order, weights: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out[t] = sum over j of weights[t, j] * y[order.row[t, j]], of the assignments that have a row; weights float32 [tokens, top_k], None: ones."""
    dev = _device_of(y)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return combine_tokens(y, order, weights, out=out, stream=stream)
    if _wants_gradient((out, stream), y, weights):
        if order.offsets.dim() != 1 or order.offsets.numel() == 0:
            raise ValueError("offsets must be [n_groups + 1]")
        _whole(order.offsets, order.offsets.shape, torch.int32, dev, "offsets")
        return _CombineTokens.apply(y, weights, order.offsets, order.row)
    return _combine(y, order.row, weights, out, stream, dev)
