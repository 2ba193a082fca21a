"""Derivatives that torch would lose without a word: its forward mode sees neither the kernels nor that a result which a call makes or is given depends on its arguments."""
from __future__ import annotations

from torch.autograd import forward_ad


def forward_mode() -> bool:
    """Whether any tensor may carry a derivative in forward mode: what a call asks first, for most have none."""
    return forward_ad._current_level >= 0


def refuse_duals(*tensors) -> None:
    """torch.no_grad() does not turn forward mode off, so that it is refused there too."""
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError("there is no derivative in forward mode: call with the primal tensor")
