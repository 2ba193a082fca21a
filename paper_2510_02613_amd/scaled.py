"""The operators of the 8-bit path over torch tensors: e4m3 values (torch.float8_e4m3fn) with fp32 scales, one for each row
and 128 columns of an activation, one for each block of 128 x 128 of a weight matrix.

torch is plumbing here: it holds device memory and names the stream.  Every function enqueues its kernels on `stream` (the current
one of the tensors' device by default) and returns the tensors that hold the results; results that are given are written in place.
Matrices are [rows, cols] with contiguous rows; rows may lie further apart (`stride(0)`), weights and their scales are contiguous.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B

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


def _on_its_device(fn):
    """Runs a call on the device of its first tensor, whichever is current."""
    def call(x, *args, **kw):
        if not x.is_cuda:
            raise ValueError(f"{fn.__name__} takes tensors on the GPU")
        dev = x.device.index
        if dev == torch._C._cuda_getDevice():
            return fn(x, *args, **kw)
        with torch.cuda.device(dev):
            return fn(x, *args, **kw)
    call.__name__, call.__doc__, call.__wrapped__ = fn.__name__, fn.__doc__, fn
    return call


def _stream(stream, t) -> int:
    return torch._C._cuda_getCurrentRawStream(t.device.index) if stream is None else stream.cuda_stream


def _matrix(t: torch.Tensor, rows: int, cols: int, dtype, like: torch.Tensor, what: str):
    """Checks a matrix [rows, cols] with contiguous rows; (address, elements from one row to the next)."""
    if t.dtype != dtype or t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{what} must be {dtype} [{rows}, {cols}], is {t.dtype} {list(t.shape)}")
    if t.device != like.device:
        raise ValueError(f"{what} is on {t.device}, not on {like.device}")
    ld, one = t.stride()
    if cols > 1 and one != 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return t.data_ptr(), (ld if rows > 1 else (cols + 15) // 16 * 16)   # one row: its stride says nothing


def _whole(t: torch.Tensor, shape, dtype, like: torch.Tensor, what: str) -> int:
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} {list(shape)}, is {t.dtype} {list(t.shape)}")
    if t.device != like.device:
        raise ValueError(f"{what} is on {t.device}, not on {like.device}")
    return t.data_ptr()


def _empty(rows, cols, dtype, like):
    return torch.empty((rows, cols), dtype=dtype, device=like.device)


@_on_its_device
def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
             sum_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
             q_scale: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Normed:
    """r = x + residual; sum_out = r, out = r / sqrt(mean(r^2) + eps) * weight, (q, q_scale) = the same in 8 bits.

    Those of sum_out, out and (q, q_scale) that are given are computed; with none given, out is allocated, and with a residual sum_out too.
    sum_out and out may be x or residual themselves."""
    if x.dim() != 2 or x.dtype not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    rows, cols = x.shape
    if sum_out is None and out is None and q is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        sum_out = None if residual is None else torch.empty_like(out)
    px, ld_x = _matrix(x, rows, cols, x.dtype, x, "x")
    pr, ld_r = (0, 0) if residual is None else _matrix(residual, rows, cols, x.dtype, x, "residual")
    pw = 0 if weight is None else _whole(weight, (cols,), x.dtype, x, "weight")
    ps, ld_s = (0, 0) if sum_out is None else _matrix(sum_out, rows, cols, x.dtype, x, "sum_out")
    po, ld_o = (0, 0) if out is None else _matrix(out, rows, cols, x.dtype, x, "out")
    pq, ld_q = (0, 0) if q is None else _matrix(q, rows, cols, E4M3, x, "q")
    pc, ld_c = (0, 0) if q_scale is None else _matrix(q_scale, rows, blocks(cols), torch.float32, x, "q_scale")
    B.moe_rms_norm(B.MoERmsNorm(rows, cols, _DTYPE[x.dtype], eps, px, ld_x, pr, ld_r, pw, ps, ld_s, po, ld_o, pq, ld_q, pc, ld_c),
                   _stream(stream, x))
    return Normed(sum_out, out, q, q_scale)


@_on_its_device
def quantize(x: torch.Tensor, *, block_rows: int = 1, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> Scaled:
    """x in 8 bits: rows of activations (block_rows 1) or a weight matrix (block_rows 128)."""
    if x.dim() != 2 or x.dtype not in _DTYPE:
        raise ValueError("x must be a bfloat16 or float32 matrix")
    rows, cols = x.shape
    scale_rows = rows if block_rows == 1 else blocks(rows)
    if q is None:
        q = _empty(rows, cols, E4M3, x)
    if scale is None:
        scale = _empty(scale_rows, blocks(cols), torch.float32, x)
    px, ld_x = _matrix(x, rows, cols, x.dtype, x, "x")
    pq, ld_q = _matrix(q, rows, cols, E4M3, x, "q")
    pc, ld_c = _matrix(scale, scale_rows, blocks(cols), torch.float32, x, "scale")
    B.moe_quantize(B.MoEQuantize(rows, cols, _DTYPE[x.dtype], block_rows, px, ld_x, pq, ld_q, pc, ld_c), _stream(stream, x))
    return Scaled(q, scale)


@_on_its_device
def matmul(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, add: Optional[torch.Tensor] = None,
           out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """a w^T (+ add) of 8-bit rows a [m, k] and 8-bit weights w [n, k]; out may be add itself."""
    (m, k), n = a.shape, w.shape[0]
    if out is None:
        # rows of the result start on 16 bytes whatever n is
        dt = add.dtype if add is not None else out_dtype
        out = torch.empty((m, (n + 7) // 8 * 8), dtype=dt, device=a.device)[:, :n]
    if out.dtype not in _DTYPE:
        raise ValueError("out must be bfloat16 or float32")
    pa, ld_a = _matrix(a, m, k, E4M3, a, "a")
    pas, ld_as = _matrix(a_scale, m, blocks(k), torch.float32, a, "a_scale")
    pw = _whole(w, (n, k), E4M3, a, "w")
    pws = _whole(w_scale, (blocks(n), blocks(k)), torch.float32, a, "w_scale")
    pad, ld_ad = (0, 0) if add is None else _matrix(add, m, n, out.dtype, a, "add")
    po, ld_o = _matrix(out, m, n, out.dtype, a, "out")
    B.moe_scaled_matmul(B.MoEScaledMatmul(m, n, k, _DTYPE[out.dtype], pa, ld_a, pas, ld_as, pw, pws, pad, ld_ad, po, ld_o), _stream(stream, a))
    return out


def swiglu_workspace(m: int, inter: int, k: int, device="cuda") -> Optional[torch.Tensor]:
    """A workspace for swiglu() of these sizes, or None when it needs none."""
    n = B.moe_scaled_swiglu_workspace_bytes(m, inter, k)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


@_on_its_device
def swiglu(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, *, q: Optional[torch.Tensor] = None,
           scale: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> Scaled:
    """silu(a Wg^T) * (a Wu^T) in 8 bits; w [2 inter, k] holds the gate rows, then the up rows, w_scale their blocks in that order."""
    (m, k), inter = a.shape, w.shape[0] // 2
    if q is None:
        q = _empty(m, inter, E4M3, a)
    if scale is None:
        scale = _empty(m, blocks(inter), torch.float32, a)
    if workspace is None:
        workspace = swiglu_workspace(m, inter, k, a.device)
    pa, ld_a = _matrix(a, m, k, E4M3, a, "a")
    pas, ld_as = _matrix(a_scale, m, blocks(k), torch.float32, a, "a_scale")
    pw = _whole(w, (2 * inter, k), E4M3, a, "w")
    pws = _whole(w_scale, (2 * blocks(inter), blocks(k)), torch.float32, a, "w_scale")
    pq, ld_q = _matrix(q, m, inter, E4M3, a, "q")
    pc, ld_c = _matrix(scale, m, blocks(inter), torch.float32, a, "scale")
    pws_, nws = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    B.moe_scaled_swiglu(B.MoEScaledSwiglu(m, inter, k, pa, ld_a, pas, ld_as, pw, pws, pq, ld_q, pc, ld_c, pws_, nws), _stream(stream, a))
    return Scaled(q, scale)
