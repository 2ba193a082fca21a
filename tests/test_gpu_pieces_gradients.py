"""Training steps through sorted tokens on the GPU: assignments that are dropped between the sort and the combination, and gradients of gradients."""
import pytest
import torch

import dispatch_ref as R
from test_gpu_dispatch import BF16, D, F32, routing

pytestmark = pytest.mark.gpu


def dropped(order, drop, in_place):
    if in_place:
        order.row.masked_fill_(drop, -1)
        return order
    return order._replace(row=order.row.masked_fill(drop, -1))


@pytest.mark.parametrize("share", [0.3, 1.0])
@pytest.mark.parametrize("T,k,E,S,cols,dt,kind", [(70, 4, 16, 12, 264, BF16, "map"), (70, 4, 16, 12, 264, F32, "map"), (1, 8, 32, 8, 64, BF16, "plain"), (600, 8, 64, 64, 24, F32, "wild"),
                                                  (5, 2, 8, 8, 40, F32, "none")])
def test_assignments_dropped_after_the_sort(T, k, E, S, cols, dt, kind, share):
    ids, m = routing(T, T, k, E, S, kind)
    g = torch.Generator().manual_seed(T)
    x, grad = torch.randn(T, cols, generator=g).to(dt), torch.randn(T, cols, generator=g).to(dt)
    w, drop = torch.rand(T, k, generator=g) - 0.2, torch.rand(T, k, generator=g) < share
    got = []
    for in_place in (True, False):
        xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
        rows, order = D().sort_tokens(xg, ids.cuda(), S, expert_map=None if m is None else m.cuda())
        order = dropped(order, drop.cuda(), in_place)
        out = D().combine_tokens(rows, order, wg)
        got.append((out.detach(), rows.detach(), *torch.autograd.grad(out, (rows, wg, xg), grad.cuda())))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    out, rows, drows, dw, dx = got[0]
    _, _, row = R.order(ids, S, m)
    kept = torch.where(drop, -1, row).int()
    R.check(out, *R.combine(rows.cpu(), kept, w), "out")
    dy, off_y, want, off = R.backward(grad, rows.cpu(), kept, w)
    R.check(drows, dy, off_y, "drows")
    R.check(dw, want, off, "dweights")
    R.check(dx, *R.combine(drows.cpu(), row), "dx")


def test_dropped_in_place_in_a_captured_step():
    """The drop is part of the graph; every replay is the eager step on a copy of the order."""
    T, k, S, cols = 40, 4, 8, 128
    ids, drop = torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(T, k, dtype=torch.bool, device="cuda")
    grad = torch.zeros(T, cols, device="cuda")
    values = [torch.randn(T, cols, device="cuda"), torch.rand(T, k, device="cuda")]

    def step(x, w, in_place):
        rows, order = D().sort_tokens(x, ids, S)
        out = D().combine_tokens(rows * 2, dropped(order, drop, in_place), w)
        return (out, *torch.autograd.grad(out, (x, w), grad))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*(v.clone().requires_grad_() for v in values), True)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    leaves = [v.clone().requires_grad_() for v in values]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*leaves, True)
    for seed in range(4):
        ids.copy_(routing(seed, T, k, S + 1, S, "plain")[0])
        drop.copy_(torch.rand(T, k, generator=torch.Generator().manual_seed(seed)) < 0.4)
        grad.copy_(torch.randn(T, cols))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.detach().clone() for t in captured]
        for a, b in zip(got, step(*(v.clone().requires_grad_() for v in values), False)):
            assert torch.equal(a, b.detach())


def test_gradients_of_the_gradients_of_combine_are_refused():
    T, k, S, cols = 6, 2, 4, 64
    ids, _ = routing(1, T, k, S, S, "plain")
    _, order = D().sort_tokens(torch.randn(T, cols, device="cuda"), ids.cuda(), S)
    y, w = torch.randn(T * k, cols, device="cuda", requires_grad=True), torch.rand(T, k, device="cuda", requires_grad=True)
    first = torch.autograd.grad(D().combine_tokens(y, order, w).sum(), (y, w))
    for got, want in zip(torch.autograd.grad(D().combine_tokens(y, order, w).sum(), (y, w), create_graph=True), first):
        assert torch.equal(got.detach(), want)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(got.square().sum(), (y, w), allow_unused=True)
