"""Experts held in 4 bits, over torch tensors: e2m1 values, two a byte, with a power of two (e8m0) for each row and 32 columns.

torch is plumbing here: it holds device memory and names the stream.  Every function enqueues its kernel on `stream` (the current one of the
tensors' device by default) and returns the tensors that hold the results; results that are given are written in place.  What a call allocates
itself belongs to `stream`.  Matrices are [rows, cols] with contiguous rows that start on 16 bytes; rows may lie further apart (`stride(0)`); weights
are contiguous, [n, k / 2] or, for sorted rows, [groups, n, k / 2], their powers [..., n, k / 32].  The bytes may be torch.uint8 or the types
that name them, torch.float4_e2m1fn_x2 and torch.float8_e8m0fnu.

The products are for serving: they have no gradient, and refuse tensors that ask for one while grad mode is on, and those that carry a
derivative in forward mode; and they refuse to be traced.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B
from .derivatives import any_requires_grad, refuse_watched, watched
from .layer import _owned_by
from .scaled import _DTYPE, _current_device, _current_stream, _device_of, _matrix, _whole

GROUP = 32
_CODES = (torch.uint8, torch.float4_e2m1fn_x2)
_POWERS = (torch.uint8, torch.float8_e8m0fnu)


class FourBit(NamedTuple):
    """A 4-bit matrix: element (i, j) stands for the e2m1 value in half j % 2 of q[i, j // 2], times 2^(scale[i, j // 32] - 127)."""
    q: torch.Tensor
    scale: torch.Tensor


_pack_quantize, _pack_matmul = B.packer(B.MoEFourBitQuantize), B.packer(B.MoEFourBitMatmul)
_pack_swiglu = B.packer(B.MoEFourBitSwiglu)


def _named(t: torch.Tensor, dtypes):
    """t's type where it is one that names such bytes, else the plain one, for the check that refuses it."""
    return t.dtype if t.dtype in dtypes else torch.uint8


# results that were given count as changed in place
_increment_version, _grad_enabled = torch._C._increment_version, torch.is_grad_enabled


def _refuse_gradient():
    raise ValueError("4-bit operators have no gradient: call them under torch.no_grad()")


def quantize(x: torch.Tensor, *, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, values: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> FourBit:
    """x [rows, cols] in 4 bits; values, where given, gets the numbers that they stand for, in x's type (it may be x itself)."""
    dev = _device_of(x)
    if dev != _current_device():      # kernels run on the tensors' device, whichever is current
        with torch.cuda.device(dev):
            return quantize(x, q=q, scale=scale, values=values, stream=stream)
    if watched():
        refuse_watched(x, q, scale, values)
    if _grad_enabled() and any_requires_grad(x, q, scale, values):
        _refuse_gradient()
    shape, dt = x.shape, x.dtype
    if len(shape) != 2 or dt not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    rows, cols = shape
    written = (q, scale) if values is None else (q, scale, values)
    if q is None or scale is None:
        written = [t for t in written if t is not None]
        with _owned_by(stream):
            q = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device) if q is None else q
            scale = torch.empty((rows, cols // GROUP), dtype=torch.uint8, device=x.device) if scale is None else scale
    px, ld_x = _matrix(x, shape, dt, dev, "x")
    pq, ld_q = _matrix(q, (rows, cols // 2), _named(q, _CODES), dev, "q")
    ps, ld_s = _matrix(scale, (rows, cols // GROUP), _named(scale, _POWERS), dev, "scale")
    pv, ld_v = (0, 0) if values is None else _matrix(values, shape, dt, dev, "values")
    B.moe_four_bit_quantize(_pack_quantize(rows, cols, _DTYPE[dt], px, ld_x, pq, ld_q, ps, ld_s, pv, ld_v),
                            _current_stream(dev) if stream is None else stream.cuda_stream)
    if written:
        _increment_version(written)
    return FourBit(q, scale)


def _weights(w, w_scale, offsets, k, dev):
    """Checks the weights; (groups, weight rows of a group, addresses of offsets, w and w_scale)."""
    if offsets is None:
        if w.dim() != 2:
            raise ValueError("w must be [n, k / 2] without offsets")
        n = w.shape[0]
        return (1, n, 0, _whole(w, (n, k // 2), _named(w, _CODES), dev, "w"), _whole(w_scale, (n, k // GROUP), _named(w_scale, _POWERS), dev, "w_scale"))
    if w.dim() != 3:
        raise ValueError("w must be [groups, n, k / 2] with offsets")
    groups, n, _ = w.shape
    return (groups, n, _whole(offsets, (groups + 1,), torch.int32, dev, "offsets"), _whole(w, (groups, n, k // 2), _named(w, _CODES), dev, "w"),
            _whole(w_scale, (groups, n, k // GROUP), _named(w_scale, _POWERS), dev, "w_scale"))


def _result(m, cols, dtype, device, offsets, stream):
    """Rows of the result start on 16 bytes whatever their width; those in no group are zeros."""
    with _owned_by(stream):
        return (torch.empty if offsets is None else torch.zeros)((m, (cols + 7) // 8 * 8), dtype=dtype, device=device)[:, :cols]


def matmul(a: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, offsets: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """a w^T (+ add) of bf16 rows a [m, k] and 4-bit weights; out may be add itself.  offsets (int32 [groups + 1], as sort_tokens makes them): rows
    offsets[g] .. offsets[g + 1] - 1 take w[g]; rows in no group are not touched, zeros where the call makes the result."""
    dev = _device_of(a)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return matmul(a, w, w_scale, offsets=offsets, add=add, out=out, out_dtype=out_dtype, stream=stream)
    if watched():
        refuse_watched(a, w, w_scale, add, out)
    if _grad_enabled() and any_requires_grad(a, w, w_scale, add, out):
        _refuse_gradient()
    m, k = a.shape
    groups, n, po, pw, ps = _weights(w, w_scale, offsets, k, dev)
    given = out is not None
    if not given:
        out = _result(m, n, out_dtype if add is None else add.dtype, a.device, offsets, stream)
    dt = out.dtype
    if dt not in _DTYPE:
        raise ValueError("out must be bfloat16 or float32")
    pa, ld_a = _matrix(a, (m, k), torch.bfloat16, dev, "a")
    pd, ld_d = (0, 0) if add is None else _matrix(add, (m, n), dt, dev, "add")
    pt, ld_t = _matrix(out, (m, n), dt, dev, "out")
    B.moe_four_bit_matmul(_pack_matmul(m, n, k, groups, _DTYPE[dt], pa, ld_a, po, pw, ps, pd, ld_d, pt, ld_t),
                          _current_stream(dev) if stream is None else stream.cuda_stream)
    if given:
        _increment_version((out,))
    return out


def swiglu(a: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, offsets: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
           out_dtype: torch.dtype = torch.bfloat16, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """silu(a Wg^T) * (a Wu^T); w [2 inter, k / 2] (with offsets [groups, 2 inter, k / 2]) holds the gate rows, then the up rows."""
    dev = _device_of(a)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return swiglu(a, w, w_scale, offsets=offsets, out=out, out_dtype=out_dtype, stream=stream)
    if watched():
        refuse_watched(a, w, w_scale, out)
    if _grad_enabled() and any_requires_grad(a, w, w_scale, out):
        _refuse_gradient()
    m, k = a.shape
    groups, n, po, pw, ps = _weights(w, w_scale, offsets, k, dev)
    if n % 2:
        raise ValueError("w must hold as many gate rows as up rows")
    inter = n // 2
    given = out is not None
    if not given:
        out = _result(m, inter, out_dtype, a.device, offsets, stream)
    dt = out.dtype
    if dt not in _DTYPE:
        raise ValueError("out must be bfloat16 or float32")
    pa, ld_a = _matrix(a, (m, k), torch.bfloat16, dev, "a")
    pt, ld_t = _matrix(out, (m, inter), dt, dev, "out")
    B.moe_four_bit_swiglu(_pack_swiglu(m, inter, k, groups, _DTYPE[dt], pa, ld_a, po, pw, ps, pt, ld_t),
                          _current_stream(dev) if stream is None else stream.cuda_stream)
    if given:
        _increment_version((out,))
    return out
