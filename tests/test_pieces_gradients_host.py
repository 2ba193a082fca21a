"""What the torch functions of a layer in pieces do about derivatives that their kernels do not compute, without a GPU: the library's calls compute on the CPU here."""
import ctypes

import pytest
import torch

import dispatch_ref as R
from paper_2510_02613_amd import binding as B
from paper_2510_02613_amd import dispatch as D

T, K, COLS, S = 4, 2, 64, 3


def at(address, *shape, dt=torch.float32):
    """Memory of a tensor as a tensor."""
    n = 1
    for d in shape:
        n *= d
    return torch.frombuffer((ctypes.c_char * (n * dt.itemsize)).from_address(address), dtype=dt).view(shape)


@pytest.fixture(autouse=True)
def on_the_cpu(monkeypatch):
    monkeypatch.setattr(D, "_device_of", lambda t: -1)
    monkeypatch.setattr(D, "_current_device", lambda: -1)
    monkeypatch.setattr(D, "_current_stream", lambda dev: 0)

    def sort(packed, stream):
        p = B.MoESortTokens.from_buffer_copy(packed)
        offsets, source, row = R.order(at(p.ids, p.tokens, p.top_k, dt=torch.int32), p.n_groups)
        for address, t in ((p.offsets, offsets), (p.source, source), (p.row, row)):
            at(address, *t.shape, dt=torch.int32).copy_(t)
        rows = at(p.rows, p.tokens * p.top_k, p.ld_rows)
        rows.copy_(torch.where(source[:, None] >= 0, at(p.x, p.tokens, p.ld_x)[source.clamp(min=0).long() // p.top_k], 0.0))

    def combine(packed, stream):
        p = B.MoECombineTokens.from_buffer_copy(packed)
        weights = at(p.weights, p.tokens, p.top_k) if p.weights else None
        out, _ = R.combine(at(p.y, p.tokens * p.top_k, p.ld_y), at(p.row, p.tokens, p.top_k, dt=torch.int32), weights)
        at(p.out, p.tokens, p.ld_out).copy_(out)

    def backward(packed, stream):
        p = B.MoECombineTokensBackward.from_buffer_copy(packed)
        A = p.tokens * p.top_k
        y = at(p.y, A, p.ld_y) if p.y else torch.zeros(A, p.cols)
        dy, _, dw, _ = R.backward(at(p.grad_out, p.tokens, p.ld_grad_out), y, at(p.row, p.tokens, p.top_k, dt=torch.int32),
                                  at(p.weights, p.tokens, p.top_k) if p.weights else None)
        if p.grad_y:
            at(p.grad_y, A, p.ld_grad_y).copy_(dy)
        if p.grad_weights:
            at(p.grad_weights, p.tokens, p.top_k).copy_(dw)

    for name, f in (("moe_sort_tokens", sort), ("moe_combine_tokens", combine), ("moe_combine_tokens_backward", backward)):
        monkeypatch.setattr(D.B, name, torch.no_grad()(f))


def inputs():
    ids = torch.tensor([[0, 2], [1, 5], [2, 0], [0, 0]], dtype=torch.int32)
    _, order = D.sort_tokens(torch.randn(T, COLS), ids, S)
    return torch.randn(T * K, COLS), torch.rand(T, K), order, ids


# ---- gradients of gradients ----

@pytest.mark.parametrize("wants", ["y", "weights", "both"])
def test_gradients_of_the_gradients_of_combine_are_refused(wants):
    """dy depends on the weights and dweights on y, also where the result's gradient is a constant."""
    y, w, order, _ = inputs()
    y.requires_grad_(), w.requires_grad_()
    leaves = {"y": (y,), "weights": (w,), "both": (y, w)}[wants]
    grads = torch.autograd.grad(D.combine_tokens(y, order, w).sum(), leaves, create_graph=True)
    for g in grads:
        with pytest.raises(RuntimeError, match="gradient of a gradient"):
            torch.autograd.grad(g.square().sum(), (y, w), allow_unused=True, retain_graph=True)
    with pytest.raises(RuntimeError, match="gradient of a gradient"):
        (D.combine_tokens(y, order, w).sum() + sum(g.square().sum() for g in grads)).backward()


def test_gradients_that_depend_on_nothing_else_are_plain():
    """With a constant gradient of the result: dy of constant weights, dweights of constant rows.  And without create_graph all of them."""
    y, w, order, _ = inputs()
    yg, wg = y.clone().requires_grad_(), w.clone().requires_grad_()
    dy, = torch.autograd.grad(D.combine_tokens(yg, order, w).sum(), yg, create_graph=True)
    dw, = torch.autograd.grad(D.combine_tokens(y, order, wg).sum(), wg, create_graph=True)
    alone, = torch.autograd.grad(D.combine_tokens(yg, order).sum(), yg, create_graph=True)
    assert not (dy.requires_grad or dw.requires_grad or alone.requires_grad)
    first = torch.autograd.grad(D.combine_tokens(yg, order, wg).sum(), (yg, wg))
    asked = torch.autograd.grad(D.combine_tokens(yg, order, wg).sum(), (yg, wg), create_graph=True)
    assert torch.equal(first[0], dy) and torch.equal(first[1], dw) and not any(t.requires_grad for t in first)
    assert all(torch.equal(a, b.detach()) and b.requires_grad for a, b in zip(first, asked))


@pytest.mark.parametrize("weighted", [True, False])
def test_gradients_by_way_of_the_result_are_refused(weighted):
    """The result's gradient depends on what is differentiated."""
    y, w, order, _ = inputs()
    y.requires_grad_()
    dy, = torch.autograd.grad(D.combine_tokens(y, order, w if weighted else None).square().sum(), y, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dy.sum(), y)
