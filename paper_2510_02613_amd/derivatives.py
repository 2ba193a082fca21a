"""What torch would lose without a word: it sees neither the kernels nor that a result which a call makes or is given depends on its arguments.  Its forward mode
would leave a derivative out, a trace would hold the result's allocation and no call."""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

_is_tracing, _count_modes = torch._C._is_tracing, torch._C._len_torch_dispatch_stack
any_requires_grad = torch._C._any_requires_grad      # of its arguments, tensors or None: 0.3 us for five


def watched() -> bool:
    """Whether something of this sort may be going on, for most calls nothing is: 0.2 us."""
    return forward_ad._current_level >= 0 or _is_tracing() or _count_modes() > 0


def refuse_duals(*tensors) -> None:
    """torch.no_grad() does not turn forward mode off, so that it is refused there too."""
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise ValueError("there is no derivative in forward mode: call with the primal tensor")


def refuse_watched(*tensors) -> None:
    """Traces are torch.jit.trace's and those of make_fx on tensors with values.  Without such values (export, compilation) tensors have no address, which torch refuses."""
    if _is_tracing() or (_count_modes() and torch._C._get_dispatch_mode(torch._C._TorchDispatchModeKey.PROXY) is not None):
        raise ValueError("the library's calls cannot be traced: a trace would hold their results' allocation only")
    refuse_duals(*tensors)
