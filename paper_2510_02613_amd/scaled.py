"""The operators of the 8-bit path over torch tensors: e4m3 values (torch.float8_e4m3fn) with fp32 scales, one for each row
and 128 columns of an activation, one for each block of 128 x 128 of a weight matrix.

torch is plumbing here: it holds device memory and names the stream.  Every function enqueues its kernels on `stream` (the current
one of the tensors' device by default) and returns the tensors that hold the results; results that are given are written in place.
What a call allocates itself, results and workspace, belongs to `stream`, as if the call stood under torch.cuda.stream(stream).
Matrices are [rows, cols] with contiguous rows; rows may lie further apart (`stride(0)`), weights and their scales are contiguous.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B
from .layer import _owned_by

BLOCK = 128
E4M3 = torch.float8_e4m3fn
_DTYPE = {torch.float32: B.MOE_F32, torch.bfloat16: B.MOE_BF16}


class Scaled(NamedTuple):
    """An 8-bit matrix: element (i, j) stands for q[i, j] * scale[its block]."""
    q: torch.Tensor
    scale: torch.Tensor


class Normed(NamedTuple):
    sum: Optional[torch.Tensor]
    out: Optional[torch.Tensor]
    q: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]


def blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream
_pack_norm, _pack_quantize = B.packer(B.MoERmsNorm), B.packer(B.MoEQuantize)
_pack_matmul, _pack_swiglu = B.packer(B.MoEScaledMatmul), B.packer(B.MoEScaledSwiglu)


def _device_of(t: torch.Tensor) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError("the tensors must be on the GPU")
    return dev


def _matrix(t: torch.Tensor, shape, dtype, dev: int, what: str):
    """Checks a matrix with contiguous rows; (address, elements from one row to the next)."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        raise ValueError(f"{what} must be {dtype} {list(shape)} on device {dev}, is {t.dtype} {list(t.shape)} on {t.device}")
    if shape[0] > 1:
        if t.is_contiguous():
            return t.data_ptr(), shape[1]
        ld, one = t.stride()
    else:
        ld, one = (shape[1] + 15) // 16 * 16, t.stride(1)                       # one row: its stride says nothing
    if one != 1 and shape[1] > 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return t.data_ptr(), ld


def _whole(t: torch.Tensor, shape, dtype, dev: int, what: str) -> int:
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} {list(shape)}, is {t.dtype} {list(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, not on device {dev}")
    return t.data_ptr()


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
             sum_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
             q_scale: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Normed:
    """r = x + residual; sum_out = r, out = r / sqrt(mean(r^2) + eps) * weight, (q, q_scale) = the same in 8 bits.

    Those of sum_out, out and (q, q_scale) that are given are computed; with none given, out is allocated, and with a residual sum_out too.
    sum_out and out may be x or residual themselves."""
    dev = _device_of(x)
    if dev != _current_device():      # kernels run on the tensors' device, whichever is current
        with torch.cuda.device(dev):
            return rms_norm(x, weight, residual=residual, eps=eps, sum_out=sum_out, out=out, q=q, q_scale=q_scale, stream=stream)
    if x.dim() != 2 or x.dtype not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    shape, dt = x.shape, x.dtype
    rows, cols = shape
    if sum_out is None and out is None and q is None:
        with _owned_by(stream):
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
            sum_out = None if residual is None else torch.empty_like(out)
    px, ld_x = _matrix(x, shape, dt, dev, "x")
    pr, ld_r = (0, 0) if residual is None else _matrix(residual, shape, dt, dev, "residual")
    pw = 0 if weight is None else _whole(weight, (cols,), dt, dev, "weight")
    ps, ld_s = (0, 0) if sum_out is None else _matrix(sum_out, shape, dt, dev, "sum_out")
    po, ld_o = (0, 0) if out is None else _matrix(out, shape, dt, dev, "out")
    pq, ld_q = (0, 0) if q is None else _matrix(q, shape, E4M3, dev, "q")
    pc, ld_c = (0, 0) if q_scale is None else _matrix(q_scale, (rows, (cols + 127) // 128), torch.float32, dev, "q_scale")
    B.moe_rms_norm(_pack_norm(rows, cols, _DTYPE[dt], eps, px, ld_x, pr, ld_r, pw, ps, ld_s, po, ld_o, pq, ld_q, pc, ld_c),
                   _current_stream(dev) if stream is None else stream.cuda_stream)
    return Normed(sum_out, out, q, q_scale)


def quantize(x: torch.Tensor, *, block_rows: int = 1, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> Scaled:
    """x in 8 bits: rows of activations (block_rows 1) or a weight matrix (block_rows 128)."""
    dev = _device_of(x)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return quantize(x, block_rows=block_rows, q=q, scale=scale, stream=stream)
    if x.dim() != 2 or x.dtype not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    shape, dt = x.shape, x.dtype
    rows, cols = shape
    groups = (rows if block_rows == 1 else blocks(rows), blocks(cols))
    if q is None or scale is None:
        with _owned_by(stream):
            q = torch.empty(shape, dtype=E4M3, device=x.device) if q is None else q
            scale = torch.empty(groups, dtype=torch.float32, device=x.device) if scale is None else scale
    px, ld_x = _matrix(x, shape, dt, dev, "x")
    pq, ld_q = _matrix(q, shape, E4M3, dev, "q")
    pc, ld_c = _matrix(scale, groups, torch.float32, dev, "scale")
    B.moe_quantize(_pack_quantize(rows, cols, _DTYPE[dt], block_rows, px, ld_x, pq, ld_q, pc, ld_c),
                   _current_stream(dev) if stream is None else stream.cuda_stream)
    return Scaled(q, scale)


def matmul(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, add: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16, fast: bool = False,
           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """a w^T (+ add) of 8-bit rows a [m, k] and 8-bit weights w [n, k]; out may be add itself.  fast: bf16 results of many rows
    from the 8-bit matrix instructions, at up to twice the rate, which drop of eight products what lies 2^-14 below the largest."""
    dev = _device_of(a)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return matmul(a, a_scale, w, w_scale, add=add, out=out, out_dtype=out_dtype, fast=fast, stream=stream)
    m, k = a.shape
    n = w.shape[0]
    if out is None:
        # rows of the result start on 16 bytes whatever n is
        with _owned_by(stream):
            out = torch.empty((m, (n + 7) // 8 * 8), dtype=add.dtype if add is not None else out_dtype, device=a.device)[:, :n]
    dt = out.dtype
    if dt not in _DTYPE:
        raise ValueError("out must be bfloat16 or float32")
    kb = (k + 127) // 128
    pa, ld_a = _matrix(a, (m, k), E4M3, dev, "a")
    pas, ld_as = _matrix(a_scale, (m, kb), torch.float32, dev, "a_scale")
    pw = _whole(w, (n, k), E4M3, dev, "w")
    pws = _whole(w_scale, ((n + 127) // 128, kb), torch.float32, dev, "w_scale")
    pad, ld_ad = (0, 0) if add is None else _matrix(add, (m, n), dt, dev, "add")
    po, ld_o = _matrix(out, (m, n), dt, dev, "out")
    B.moe_scaled_matmul(_pack_matmul(m, n, k, _DTYPE[dt] | (B.MOE_FAST_PRODUCTS if fast else 0), pa, ld_a, pas, ld_as, pw, pws, pad, ld_ad, po, ld_o),
                        _current_stream(dev) if stream is None else stream.cuda_stream)
    return out


def swiglu_workspace(m: int, inter: int, k: int, device="cuda", up_to: bool = False) -> Optional[torch.Tensor]:
    """A workspace for swiglu() of these sizes, or None when it needs none.  up_to: for any number of rows up to m (a call of m rows may need
    none where one of fewer needs some)."""
    n = (B.moe_scaled_swiglu_max_workspace_bytes if up_to else B.moe_scaled_swiglu_workspace_bytes)(m, inter, k)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def swiglu(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, q: Optional[torch.Tensor] = None,
           scale: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> Scaled:
    """silu(a Wg^T) * (a Wu^T) in 8 bits; w [2 inter, k] holds the gate rows, then the up rows, w_scale their blocks in that order."""
    dev = _device_of(a)
    if dev != _current_device():
        with torch.cuda.device(dev):
            return swiglu(a, a_scale, w, w_scale, q=q, scale=scale, workspace=workspace, stream=stream)
    m, k = a.shape
    inter = w.shape[0] // 2
    if workspace is not None and (workspace.get_device() != dev or not workspace.is_contiguous()):
        raise ValueError("the workspace must be contiguous and on the device of a")
    if q is None or scale is None or workspace is None:
        with _owned_by(stream):
            q = torch.empty((m, inter), dtype=E4M3, device=a.device) if q is None else q
            scale = torch.empty((m, blocks(inter)), dtype=torch.float32, device=a.device) if scale is None else scale
            workspace = swiglu_workspace(m, inter, k, a.device) if workspace is None else workspace
    kb, nb = (k + 127) // 128, (inter + 127) // 128
    pa, ld_a = _matrix(a, (m, k), E4M3, dev, "a")
    pas, ld_as = _matrix(a_scale, (m, kb), torch.float32, dev, "a_scale")
    pw = _whole(w, (2 * inter, k), E4M3, dev, "w")
    pws = _whole(w_scale, (2 * nb, kb), torch.float32, dev, "w_scale")
    pq, ld_q = _matrix(q, (m, inter), E4M3, dev, "q")
    pc, ld_c = _matrix(scale, (m, nb), torch.float32, dev, "scale")
    pk, nk = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    B.moe_scaled_swiglu(_pack_swiglu(m, inter, k, pa, ld_a, pas, ld_as, pw, pws, pq, ld_q, pc, ld_c, pk, nk),
                        _current_stream(dev) if stream is None else stream.cuda_stream)
    return Scaled(q, scale)
