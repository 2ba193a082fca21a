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
`stream` and results that are given are refused then, and so are gradients of gradients; derivatives in forward mode and traces are refused always.  A step that is captured into a graph together with its
backward pass takes leaves that no eager graph still holds (torch keeps one accumulation node a leaf, on the stream of its first use).
"""
from __future__ import annotations

import functools
from typing import NamedTuple, Optional

import torch

from . import binding as B
from .derivatives import refuse_duals, refuse_watched, watched
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
# results that were given count as changed in place: a backward pass that was to read what they held refuses
_increment_version, _grad_enabled = torch._C._increment_version, torch.is_grad_enabled


_workspace_bytes = functools.lru_cache(maxsize=1024)(B.moe_sort_tokens_workspace_bytes)      # of sizes alone


def sort_workspace(tokens: int, top_k: int, n_groups: int, device="cuda") -> Optional[torch.Tensor]:
    """A workspace for sort_tokens() of these sizes, or None when it needs none.  One for more tokens is enough for fewer."""
    n = _workspace_bytes(tokens, top_k, n_groups)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _new_order(n_groups, routing, device) -> Order:
    empty, i32 = torch.empty, torch.int32
    return Order(empty(n_groups + 1, dtype=i32, device=device), empty(routing[0] * routing[1], dtype=i32, device=device), empty(routing, dtype=i32, device=device))


def _sort(x, ids, n_groups, expert_map, rows, order, workspace, stream, dev, zero_rest=False):
    shape, dt = x.shape, x.dtype
    if len(shape) != 2 or dt not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    tokens, cols = shape
    if ids.dim() != 2 or ids.shape[0] != tokens:
        raise ValueError(f"ids must be [{tokens}, top_k], is {list(ids.shape)}")
    if n_groups <= 0:
        raise ValueError(f"n_groups must be positive, is {n_groups}")
    routing = ids.shape
    top_k = routing[1]
    A = tokens * top_k
    pi = _whole(ids, routing, torch.int32, dev, "ids")
    pm, n_experts = 0, 0
    if expert_map is not None:
        if expert_map.dim() != 1:
            raise ValueError("expert_map must be [n_experts]")
        n_experts = expert_map.shape[0]
        pm = _whole(expert_map, expert_map.shape, torch.int32, dev, "expert_map")
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError("the workspace must be contiguous and on the device of x")
    written = (rows, *order) if rows is not None and order is not None else order or (() if rows is None else (rows,))
    if rows is None or order is None or (workspace is None and _workspace_bytes(tokens, top_k, n_groups)):
        with _owned_by(stream):
            if rows is None:
                rows, zero_rest = torch.empty((A, cols), dtype=dt, device=x.device), True
            if order is None:
                order = _new_order(n_groups, routing, x.device)
            if workspace is None:
                workspace = sort_workspace(tokens, top_k, n_groups, x.device)
    offsets, source, row = order
    po = _whole(offsets, (n_groups + 1,), torch.int32, dev, "offsets")
    ps = _whole(source, (A,), torch.int32, dev, "source")
    pr = _whole(row, routing, torch.int32, dev, "row")
    px, ld_x = _matrix(x, shape, dt, dev, "x")
    pt, ld_t = _matrix(rows, (A, cols), dt, dev, "rows")
    pk, nk = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    B.moe_sort_tokens(_pack_sort(tokens, top_k, n_groups, n_experts, cols, _DTYPE[dt], zero_rest, pi, pm, px, ld_x, pt, ld_t, po, ps, pr, pk, nk),
                      _current_stream(dev) if stream is None else stream.cuda_stream)
    if written:
        _increment_version(written)
    return rows, order


def _combine(y, row, weights, out, stream, dev):
    shape, dt, routing = y.shape, y.dtype, row.shape
    if len(shape) != 2 or dt not in _DTYPE:
        raise ValueError("y must be a bfloat16 or float32 matrix")
    if len(routing) != 2:
        raise ValueError("row must be [tokens, top_k]")
    tokens, top_k = routing
    cols, given = shape[1], out is not None
    if not given:
        with _owned_by(stream):
            out = torch.empty((tokens, cols), dtype=dt, device=y.device)
    pr = _whole(row, routing, torch.int32, dev, "row")
    pw = 0 if weights is None else _whole(weights, routing, torch.float32, dev, "weights")
    py, ld_y = _matrix(y, (tokens * top_k, cols), dt, dev, "y")
    po, ld_o = _matrix(out, (tokens, cols), dt, dev, "out")
    B.moe_combine_tokens(_pack_combine(tokens, top_k, cols, _DTYPE[dt], py, ld_y, pr, pw, po, ld_o),
                         _current_stream(dev) if stream is None else stream.cuda_stream)
    if given:
        _increment_version((out,))
    return out


def _rows16(t: torch.Tensor) -> torch.Tensor:
    """A gradient as the kernels read it: autograd's may be broadcast or start anywhere."""
    if watched():
        refuse_duals(t)
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _unchanged(t: torch.Tensor, version: int) -> None:
    if t._version != version:
        raise RuntimeError("the order of the tokens was changed in place since the call whose gradient is wanted, by the caller or by a call that its buffers were given to")


def _places(source: torch.Tensor, routing) -> torch.Tensor:
    """row of an Order, from its source: places behind the last one have a spare entry each, so that no two write to one."""
    A = source.numel()
    at = torch.arange(A, dtype=torch.int64, device=source.device)
    places = torch.full((2 * A,), -1, dtype=torch.int32, device=source.device)
    return places.scatter_(0, torch.where(source >= 0, source, at + A), at.int())[:A].view(routing)


def _sort_backward(ctx, grad_rows):
    if grad_rows is None:
        return None, None, None, None, None, None
    source, row, *versions = ctx.order
    if row._version != versions[1]:                     # entries were set to -1: what combine_tokens drops, the rows' gradient may still have from elsewhere
        _unchanged(source, versions[0])
        row = _places(source, row.shape)
    return _combine(_rows16(grad_rows), row, None, None, None, grad_rows.get_device()), None, None, None, None, None


def _combine_backward(ctx, grad):
    if grad is None:
        return None, None, None, None
    source, row, *versions = ctx.order
    _unchanged(source, versions[0])
    _unchanged(row, versions[1])
    y, weights = ctx.saved_tensors
    grad, dev, dt = _rows16(grad), grad.get_device(), grad.dtype
    wants_y, wants_w, *_ = ctx.needs_input_grad
    tokens, top_k = row.shape
    cols = grad.shape[1]
    shape = (tokens * top_k, cols)
    dy = torch.empty(shape, dtype=dt, device=grad.device) if wants_y else None
    dw = torch.empty(row.shape, dtype=torch.float32, device=grad.device) if wants_w else None
    py, ld_y = _matrix(y, shape, dt, dev, "y") if wants_w else (0, 0)
    B.moe_combine_tokens_backward(
        _pack_backward(tokens, top_k, cols, _DTYPE[dt], grad.data_ptr(), cols, py, ld_y, row.data_ptr(), 0 if weights is None else weights.data_ptr(),
                       source.data_ptr(), dy.data_ptr() if wants_y else 0, cols, dw.data_ptr() if wants_w else 0), _current_stream(dev))
    return dy, dw, None, None


class _FirstOrder(torch.autograd.Function):
    """A gradient in a graph of the backward pass (create_graph): it depends on `of`, and has no gradient of its own to them."""

    @staticmethod
    def forward(ctx, gradient, *of):
        return gradient

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("sort_tokens and combine_tokens have no gradient of a gradient")


# What each gradient depends on: dx on the rows' gradient; dy = w dout on the weights too, dw = <dout, y> on y too, also where dout is a constant
def _sort_backward_graph(ctx, grad_rows):
    with torch.no_grad():
        dx, *rest = _sort_backward(ctx, grad_rows)
    return dx if dx is None else _FirstOrder.apply(dx, grad_rows), *rest


def _combine_backward_graph(ctx, grad):
    with torch.no_grad():
        dy, dw, *rest = _combine_backward(ctx, grad)
    if grad is not None:
        y, weights = ctx.saved_tensors
        dy = dy if dy is None else _FirstOrder.apply(dy, grad, weights)
        dw = dw if dw is None else _FirstOrder.apply(dw, grad, y)
    return dy, dw, *rest


class _SortTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, ids, n_groups, expert_map, order, workspace):
        ctx.set_materialize_grads(False)
        rows = torch.empty((ids.numel(), x.shape[1]), dtype=x.dtype, device=x.device)
        _sort(x, ids, n_groups, expert_map, rows, order, workspace, None, x.get_device(), zero_rest=True)
        ctx.order = order.source, order.row, order.source._version, order.row._version
        return rows

    @staticmethod
    def backward(ctx, grad_rows):
        return (_sort_backward_graph if torch.is_grad_enabled() else _sort_backward)(ctx, grad_rows)


class _CombineTokens(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, source, row):
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(y if ctx.needs_input_grad[1] else None, weights)
        ctx.order = source, row, source._version, row._version
        return _combine(y, row, weights, None, None, y.get_device())

    @staticmethod
    def backward(ctx, grad):
        return (_combine_backward_graph if torch.is_grad_enabled() else _combine_backward)(ctx, grad)


def _refuse_given():
    raise ValueError("results that are given and a stream are for calls without a gradient")


def _refuse_leaf(given):
    if given.requires_grad and _grad_enabled():
        raise ValueError("results that are given must not require a gradient")


def sort_tokens(x: torch.Tensor, ids: torch.Tensor, n_groups: int, *, expert_map: Optional[torch.Tensor] = None,
                rows: Optional[torch.Tensor] = None, order: Optional[Order] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> Sorted:
    """The rows of x [tokens, cols] in the order of their groups, one for every assignment ids [tokens, top_k] (int32) to a group of this rank:
    group expert_map[id] (int32 [n_experts], other ranks' -1), or the id itself without a map.  Groups outside [0, n_groups) are not this rank's."""
    dev = _device_of(x)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return sort_tokens(x, ids, n_groups, expert_map=expert_map, rows=rows, order=order, workspace=workspace, stream=stream)
    if watched():
        refuse_watched(x, rows)
    if x.requires_grad and _grad_enabled():
        if rows is not None or order is not None or stream is not None:
            _refuse_given()
        if ids.dim() != 2 or n_groups <= 0 or x.dim() != 2:
            raise ValueError("x must be [tokens, cols], ids [tokens, top_k] and n_groups positive")
        order = _new_order(n_groups, ids.shape, x.device)
        return Sorted(_SortTokens.apply(x, ids, n_groups, expert_map, order, workspace), order)
    if rows is not None:
        _refuse_leaf(rows)
    return Sorted(*_sort(x, ids, n_groups, expert_map, rows, order, workspace, stream, dev))


def combine_tokens(y: torch.Tensor, order: Order, weights: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """out[t] = sum over j of weights[t, j] * y[order.row[t, j]], of the assignments that have a row; weights float32 [tokens, top_k], None: ones.
    Entries of order.row may be set to -1 before (assignments that are dropped), in place or in another Order; rows that none names have a gradient of zeros."""
    dev = _device_of(y)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return combine_tokens(y, order, weights, out=out, stream=stream)
    if watched():
        refuse_watched(y, weights, out)
    if (y.requires_grad or (weights is not None and weights.requires_grad)) and _grad_enabled():
        if out is not None or stream is not None:
            _refuse_given()
        if order.source is None:
            raise ValueError("a gradient wants the order's source, [tokens * top_k]")
        _whole(order.source, (order.row.numel(),), torch.int32, dev, "source")
        return _CombineTokens.apply(y, weights, order.source, order.row)
    if out is not None:
        _refuse_leaf(out)
    return _combine(y, order.row, weights, out, stream, dev)
