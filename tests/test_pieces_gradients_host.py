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


# ---- derivatives in forward mode ----

def four_bit(monkeypatch):
    from paper_2510_02613_amd import four_bit as Q
    monkeypatch.setattr(Q, "_device_of", lambda t: -1)
    monkeypatch.setattr(Q, "_current_device", lambda: -1)
    monkeypatch.setattr(Q, "_current_stream", lambda dev: 0)
    for name in ("moe_four_bit_quantize", "moe_four_bit_matmul", "moe_four_bit_swiglu"):
        monkeypatch.setattr(Q.B, name, lambda *a: None)
    return Q


def calls_of(Q):
    """Calls by name, each of the tensor that its results depend on, and what to call them with."""
    y, w, order, ids = inputs()
    q, s = torch.zeros(64, 32, dtype=torch.uint8), torch.zeros(64, 2, dtype=torch.uint8)
    half = torch.zeros(T, COLS, dtype=torch.bfloat16)
    new = lambda rows, cols=COLS, dt=torch.float32: torch.zeros(rows, cols, dtype=dt)  # noqa: E731
    return {
        "sort": (lambda x: D.sort_tokens(x, ids, S).rows, new(T)),
        "sort, given": (lambda x: D.sort_tokens(new(T), ids, S, rows=x).rows, new(T * K)),
        "combine": (lambda x: D.combine_tokens(x, order, w), y),
        "combine, weights": (lambda x: D.combine_tokens(y, order, x), w),
        "combine, given": (lambda x: D.combine_tokens(y, order, w, out=x), new(T)),
        "quantize": (lambda x: Q.quantize(x).q, new(T)),
        "quantize, values": (lambda x: Q.quantize(new(T), values=x).q, new(T)),
        "matmul": (lambda x: Q.matmul(x, q, s), half),
        "matmul, addend": (lambda x: Q.matmul(half, q, s, add=x), new(T)),
        "matmul, given": (lambda x: Q.matmul(half, q, s, out=x), new(T)),
        "swiglu": (lambda x: Q.swiglu(x, q, s), half),
        "swiglu, given": (lambda x: Q.swiglu(half, q, s, out=x), new(T, 32)),
    }


CALLS = ["sort", "sort, given", "combine", "combine, weights", "combine, given", "quantize", "quantize, values", "matmul", "matmul, addend", "matmul, given", "swiglu",
         "swiglu, given"]


@pytest.mark.parametrize("no_grad", [False, True])
@pytest.mark.parametrize("name", CALLS)
def test_derivatives_in_forward_mode_are_refused(monkeypatch, name, no_grad):
    """A dual number's derivative would be missing from the result, with no error; torch.no_grad() does not turn this mode off."""
    f, x = calls_of(four_bit(monkeypatch))[name]
    f(x)
    with torch.autograd.forward_ad.dual_level(), torch.set_grad_enabled(not no_grad):
        f(x)                                        # only tensors that carry one
        with pytest.raises(ValueError, match="forward"):
            f(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
    f(x)


@pytest.mark.parametrize("of", ["sort", "combine"])
def test_derivatives_in_forward_mode_of_gradients_are_refused(of):
    y, w, order, ids = inputs()
    leaf = torch.zeros(T, COLS, requires_grad=True) if of == "sort" else y.requires_grad_()
    out = D.sort_tokens(leaf, ids, S).rows if of == "sort" else D.combine_tokens(leaf, order, w)
    with torch.autograd.forward_ad.dual_level():
        grad = torch.autograd.forward_ad.make_dual(torch.ones_like(out), torch.ones_like(out))
        with pytest.raises(ValueError, match="forward"):
            torch.autograd.grad(out, leaf, grad, retain_graph=True)
        torch.autograd.grad(out, leaf, torch.ones_like(out))


def test_tensors_of_other_types_are_refused_as_ever():
    with torch.autograd.forward_ad.dual_level():
        for dt in (torch.int32, torch.float16):
            with pytest.raises(ValueError, match="x must be"):
                D.sort_tokens(torch.zeros(T, COLS, dtype=dt), torch.zeros(T, K, dtype=torch.int32), S)


# ---- traces ----

@pytest.mark.parametrize("name", CALLS)
def test_traces_are_refused(monkeypatch, name):
    """What is traced would hold the allocation of the result and no call."""
    from torch.fx.experimental.proxy_tensor import make_fx
    f, x = calls_of(four_bit(monkeypatch))[name]
    with pytest.raises(ValueError, match="trace"):
        torch.jit.trace(f, (x,), check_trace=False)
    with pytest.raises(ValueError, match="trace"):
        make_fx(f)(x)
    f(x)


def test_other_modes_of_torch_are_not_in_the_way(monkeypatch):
    from torch.utils.flop_counter import FlopCounterMode
    with FlopCounterMode(display=False):
        for f, x in calls_of(four_bit(monkeypatch)).values():
            f(x)


# ---- powers whose type could have a gradient ----

@pytest.mark.parametrize("which", ["scale", "w_scale"])
def test_powers_that_ask_for_a_gradient_are_refused(monkeypatch, which):
    Q = four_bit(monkeypatch)
    powers = torch.zeros(64, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    x = torch.zeros(64, 64, dtype=torch.bfloat16)
    call = {"scale": lambda p: Q.quantize(x, scale=p), "w_scale": lambda p: Q.matmul(x, torch.zeros(64, 32, dtype=torch.uint8), p)}[which]
    with torch.autograd.forward_ad.dual_level(), pytest.raises(ValueError, match="forward"):
        call(torch.autograd.forward_ad.make_dual(powers, powers.clone()))
    powers.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        call(powers)
    with torch.no_grad():
        call(powers)


# ---- assignments that are dropped between the sort and the combination ----

def dropping_step(x, w, ids, drop, how):
    """(out, rows) of x with assignments dropped, by torch's own operations where `how` is "plain"."""
    if how == "plain":
        rows = x[:, None].expand(T, K, COLS)
        kept = torch.where((ids >= 0) & (ids < S) & ~drop, w, torch.zeros(()))
        return (kept[..., None] * (2 * rows)).sum(1), torch.where(((ids >= 0) & (ids < S))[..., None], rows, 0.0)
    rows, order = D.sort_tokens(x, ids, S)
    if how == "in place":
        order.row[drop] = -1
    else:
        order = order._replace(row=order.row.masked_fill(drop, -1))
    return D.combine_tokens(2 * rows, order, w), rows


@pytest.mark.parametrize("how", ["in place", "copy"])
def test_assignments_dropped_after_the_sort(how):
    """Gradients of tokens and weights through sort, drop and combine; rows that are used elsewhere too keep that part of their gradient, dropped or not."""
    _, w, _, ids = inputs()
    x, drop = torch.randn(T, COLS), torch.tensor([[True, False], [False, False], [True, True], [False, True]])
    grad, more = torch.randn(T, COLS), torch.randn(COLS)
    got, want = [], []
    for to, h in ((got, how), (want, "plain")):
        xs, ws = x.clone().requires_grad_(), w.clone().requires_grad_()
        out, rows = dropping_step(xs, ws, ids, drop, h)
        to.extend((out.detach(), *torch.autograd.grad((out * grad).sum() + (rows * more).sum(), (xs, ws))))
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-5)


def test_what_else_is_changed_after_the_sort_is_refused():
    """The rows' assignments tell the sort where its rows came from: with them gone it has no gradient, and says so.  So has the combination when its entries change behind it."""
    _, w, _, ids = inputs()
    x = torch.randn(T, COLS, requires_grad=True)
    rows, order = D.sort_tokens(x, ids, S)
    order.row[0] = -1
    order.source[0] = -1
    with pytest.raises(RuntimeError, match="changed in place"):
        torch.autograd.grad(rows.sum(), x)
    rows, order = D.sort_tokens(x, ids, S)
    out = D.combine_tokens(rows, order, w)
    order.row[0] = -1
    with pytest.raises(RuntimeError, match="changed in place"):
        torch.autograd.grad(out.sum(), x)


@pytest.mark.parametrize("tokens,k,n_groups", [(0, 2, 3), (1, 1, 1), (7, 3, 4), (40, 8, 5)])
def test_places_from_the_rows_assignments(tokens, k, n_groups):
    ids = torch.randint(-1, n_groups + 2, (tokens, k), generator=torch.Generator().manual_seed(tokens), dtype=torch.int32)
    _, source, row = R.order(ids, n_groups)
    got = D._places(source, ids.shape)
    assert got.dtype == torch.int32 and got.is_contiguous() and torch.equal(got, row)
