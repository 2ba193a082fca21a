"""Tokens sorted by expert and back, with their gradients, on the GPU against the definition."""
import pytest
import torch

import dispatch_ref as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def D():
    from paper_2510_02613_amd import dispatch
    return dispatch


def routing(seed, T, k, E, S, kind):
    """(ids, map) on the CPU: `kind` says what is unusual about them."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(E, (T, k), generator=g, dtype=torch.int32)
    m = None
    if kind == "map":                    # some experts here, in shuffled groups
        m = torch.full((E,), -1, dtype=torch.int32)
        here = torch.randperm(E, generator=g)[:min(E, S)]
        m[here] = torch.randperm(S, generator=g)[:len(here)].to(torch.int32)
    elif kind == "none":                 # nobody here
        m = torch.full((E,), -1, dtype=torch.int32)
    elif kind == "one":                  # everybody in one group
        m = torch.full((E,), S - 1, dtype=torch.int32)
    elif kind == "wild":                 # ids and entries of the map that do not exist
        m = torch.randint(-3, S + 3, (E,), generator=g, dtype=torch.int32)
        m[0], m[-1] = 2 ** 31 - 1, -2 ** 31
        ids = torch.randint(-2, E + 2, (T, k), generator=g, dtype=torch.int32)
        if T:
            ids[0, 0], ids[-1, -1] = -2 ** 31, 2 ** 31 - 1
    return ids, m


def padded(t, fill=float("nan")):
    """The same matrix with rows further apart and `fill` between them."""
    rows, cols = t.shape
    wide = torch.full((rows, cols + 16), fill, dtype=t.dtype, device=t.device)
    wide[:, :cols] = t
    return wide[:, :cols]


SORTS = [
    (0, 8, 16, 16, 64, BF16, "plain"), (1, 1, 4, 4, 8, BF16, "plain"), (1, 8, 256, 32, 7168, BF16, "map"), (2, 32, 64, 64, 8, F32, "map"), (3, 6, 64, 1, 72, F32, "plain"),
    (17, 8, 128, 128, 768, BF16, "map"), (63, 8, 256, 257, 520, BF16, "plain"), (64, 4, 16, 16, 136, F32, "one"), (65, 2, 8, 8, 1032, BF16, "none"),
    (333, 6, 64, 64, 2048, F32, "map"), (200, 20, 300, 255, 24, BF16, "wild"), (512, 8, 128, 128, 16, BF16, "plain"),          # 4096 assignments: one launch
    (513, 8, 128, 2047, 16, BF16, "wild"), (585, 7, 64, 63, 40, F32, "map"), (1000, 31, 256, 256, 8, BF16, "one"), (5000, 8, 128, 128, 264, BF16, "map"),   # counted first
    (3001, 32, 2047, 2047, 8, BF16, "map"), (9000, 8, 2047, 2047, 16, F32, "wild"), (40000, 2, 4, 2, 8, BF16, "plain"),     # more counts than a workgroup adds up
]


@pytest.mark.parametrize("T,k,E,S,cols,dt,kind", SORTS)
def test_sort(T, k, E, S, cols, dt, kind):
    ids, m = routing(T + k, T, k, E, S, kind)
    want = R.order(ids, S, m)
    total = int(want[0][-1])
    x = torch.randn(T, cols, device="cuda").to(dt)
    dm = None if m is None else m.cuda()
    # what the call makes itself: zeros behind the last row
    rows, order = D().sort_tokens(padded(x), ids.cuda(), S, expert_map=dm)
    for got, w, name in zip(order, want, order._fields):
        assert got.dtype == torch.int32 and torch.equal(got.cpu(), w), name
    xr = x.cpu()[(want[1][:total].long() // k)]
    assert torch.equal(rows[:total].cpu(), xr)
    assert rows.shape[0] == T * k and not rows[total:].any()
    # what is given: nothing behind the last row is touched, nor between the rows
    given = padded(torch.full((T * k, cols), 7.0, dtype=dt, device="cuda"), 3.0)
    again = D().Order(*(torch.full_like(t, 99) for t in order))
    got = D().sort_tokens(x, ids.cuda(), S, expert_map=dm, rows=given, order=again)
    assert got.rows is given and torch.equal(given[:total].cpu(), xr) and given[total:].eq(7.0).all()
    if T * k:
        wide = given.as_strided((T * k, 16), given.stride(), cols)
        assert wide.eq(3.0).all()
    for a, b in zip(again, order):
        assert torch.equal(a, b)


def made(T, k, E, S, cols, dt, kind, seed=5):
    ids, m = routing(seed, T, k, E, S, kind)
    _, _, row = R.order(ids, S, m)
    g = torch.Generator().manual_seed(seed)
    y = (torch.randn(T * k, cols, generator=g) * torch.exp(2 * torch.randn(T * k, 1, generator=g))).to(dt)
    y[~torch.isin(torch.arange(T * k), row.flatten())] = float("nan")        # no entry names these
    w = torch.rand(T, k, generator=g) - 0.2
    w[row < 0] = float("nan")
    return ids, m, row, y, w


COMBINES = [(1, 1, 4, 4, 8, BF16, "plain"), (1, 8, 256, 32, 7168, BF16, "map"), (2, 32, 64, 64, 520, F32, "map"), (5, 9, 16, 16, 72, F32, "plain"), (64, 8, 256, 32, 7168, BF16, "map"),
            (33, 6, 64, 64, 2048, F32, "plain"), (65, 2, 8, 8, 1032, BF16, "none"), (40, 20, 300, 255, 24, BF16, "wild"), (77, 17, 8, 8, 264, BF16, "one")]


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("T,k,E,S,cols,dt,kind", COMBINES)
def test_combine(T, k, E, S, cols, dt, kind, weighted):
    _, _, row, y, w = made(T, k, E, S, cols, dt, kind)
    want, off = R.combine(y, row, w if weighted else None)
    order = D().Order(None, None, row.cuda())
    out = D().combine_tokens(y.cuda(), order, w.cuda() if weighted else None)
    R.check(out, want, off, "out")
    given = padded(torch.full((T, cols), 7.0, dtype=dt, device="cuda"), 3.0)
    got = D().combine_tokens(padded(y.cuda()), order, w.cuda() if weighted else None, out=given)
    assert got is given and torch.equal(given, out)
    assert given.as_strided((T, 16), given.stride(), cols).eq(3.0).all()


def test_combine_leaves_rows_out_that_do_not_exist():
    T, k, cols = 3, 4, 64
    y = torch.randn(T * k, cols, device="cuda")
    row = torch.tensor([[0, 12, -1, -2 ** 31], [2 ** 31 - 1, 11, 3, 13], [-5, -1, 100, 12]], dtype=torch.int32)
    out = D().combine_tokens(y, D().Order(None, None, row.cuda()))
    assert torch.equal(out[0], y[0]) and torch.equal(out[1], y[11] + y[3]) and not out[2].any()


@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("T,k,E,S,cols,dt,kind", COMBINES)
def test_gradients_of_combine(T, k, E, S, cols, dt, kind, weighted):
    ids, m, row, y, w = made(T, k, E, S, cols, dt, kind)
    offsets, source, _ = R.order(ids, S, m)
    order = D().Order(offsets.cuda(), source.cuda(), row.cuda())
    g = torch.randn(T, cols, generator=torch.Generator().manual_seed(9)).to(dt)
    dy, off_y, dw, off_w = R.backward(g, y, row, w if weighted else None)
    yg, wg = y.cuda().requires_grad_(), w.cuda().requires_grad_() if weighted else None
    out = D().combine_tokens(yg, order, wg)
    got = torch.autograd.grad(out, (yg, wg) if weighted else (yg,), g.cuda())
    assert got[0].dtype == dt
    R.check(got[0], dy, off_y, "dy")                       # zeros behind the last row
    assert not got[0][int(offsets[-1]):].any()
    if weighted:
        assert got[1].dtype == F32
        R.check(got[1], dw, off_w, "dweights")
        alone = torch.autograd.grad(D().combine_tokens(y.cuda(), order, wg), wg, g.cuda())[0]
        assert torch.equal(alone, got[1])
        alone = torch.autograd.grad(D().combine_tokens(yg, order, w.cuda()), yg, g.cuda())[0]
        assert torch.equal(alone, got[0])


@pytest.mark.parametrize("T,k,E,S,cols,dt,kind", [c for c in SORTS if 0 < c[0] <= 600])
def test_gradient_of_sort(T, k, E, S, cols, dt, kind):
    ids, m = routing(T + k, T, k, E, S, kind)
    _, _, row = R.order(ids, S, m)
    x = torch.randn(T, cols, device="cuda").to(dt).requires_grad_()
    rows, order = D().sort_tokens(x, ids.cuda(), S, expert_map=None if m is None else m.cuda())
    assert rows.requires_grad and not any(t.requires_grad for t in order)
    g = torch.randn(T * k, cols, generator=torch.Generator().manual_seed(9)).to(dt)
    g[order.offsets[-1].item():] = float("nan")            # what is behind the last row counts nowhere
    want, off = R.combine(g, row)
    dx, = torch.autograd.grad(rows, x, g.cuda())
    R.check(dx, want, off, "dx")


def test_backward_leaves_the_rest_alone_without_the_sources():
    """The call itself: rows of grad_y that no entry names are touched only where the sources are given; either result alone."""
    from paper_2510_02613_amd import binding as B
    T, k, E, S, cols, dt = 33, 6, 64, 20, 520, BF16
    ids, m, row, y, w = made(T, k, E, S, cols, dt, "map")
    offsets, sources, _ = R.order(ids, S, m)
    total = int(offsets[-1])
    g = torch.randn(T, cols, generator=torch.Generator().manual_seed(9)).to(dt)
    dy, off_y, dw, off_w = R.backward(g, y, row, w)
    dev = [t.cuda() for t in (g, y, row, w, sources)]
    for source in (0, dev[4].data_ptr()):
        for wants in ((True, True), (True, False), (False, True)):
            gy = padded(torch.full((T * k, cols), 7.0, dtype=dt, device="cuda"), 3.0)
            gw = torch.full((T, k), 7.0, device="cuda")
            B.moe_combine_tokens_backward(B.MoECombineTokensBackward(
                tokens=T, top_k=k, cols=cols, dtype=B.MOE_BF16, grad_out=dev[0].data_ptr(), ld_grad_out=cols, y=dev[1].data_ptr(), ld_y=cols, row=dev[2].data_ptr(),
                weights=dev[3].data_ptr(), source=source, grad_y=gy.data_ptr() if wants[0] else 0, ld_grad_y=gy.stride(0), grad_weights=gw.data_ptr() if wants[1] else 0),
                torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            if wants[0]:
                R.check(gy[:total], dy[:total], off_y[:total], "grad_y")
                assert gy[total:].eq(0.0 if source else 7.0).all() and gy.as_strided((T * k, 16), gy.stride(), cols).eq(3.0).all()
            else:
                assert gy.eq(7.0).all()
            if wants[1]:
                R.check(gw, dw, off_w, "grad_weights")
            else:
                assert gw.eq(7.0).all()


def test_gradients_by_differences():
    """Sorting and adding up again is linear in x and in the weights: its differences along a direction are the gradient's products with it."""
    T, k, E, S, cols = 37, 4, 16, 11, 96
    ids, m = routing(3, T, k, E, S, "map")
    gen = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    x, w, scale, grad = new(T, cols).requires_grad_(), new(T, k).requires_grad_(), new(T * k, 1), new(T, cols)

    def f(x, w):
        rows, order = D().sort_tokens(x, ids.cuda(), S, expert_map=m.cuda())
        return D().combine_tokens(rows * scale, order, w)

    dx, dw = torch.autograd.grad(f(x, w), (x, w), grad)
    directions = {"x": (dx, new(T, cols)), "w": (dw, new(T, k))}
    with torch.no_grad():
        # the magnitudes of all terms that either side adds up: a result's are off by k + 2 half steps each, twice; dx by k + 3, dw by its dot product's 18
        rows, order = D().sort_tokens(x.abs() + directions["x"][1].abs(), ids.cuda(), S, expert_map=m.cuda())
        size = (D().combine_tokens(rows * scale.abs(), order, w.abs() + directions["w"][1].abs()) * grad.abs()).double().sum()
    for at, (d, direction) in directions.items():
        with torch.no_grad():
            lo, hi = [f(x + s * direction, w) if at == "x" else f(x, w + s * direction) for s in (-0.5, 0.5)]
        by_difference = ((hi.double() - lo.double()) * grad.double()).sum()
        by_gradient = (d.double() * direction.double()).sum()
        assert (by_difference - by_gradient).abs() <= (2 * (k + 2) + (k + 3) + 18) * R.F32 * size, at


def test_gradients_of_broadcast_and_shared_results():
    T, k, S, cols = 12, 2, 4, 64
    ids, _ = routing(1, T, k, S, S, "plain")
    x = torch.randn(T, cols, device="cuda", requires_grad=True)
    w = torch.rand(T, k, device="cuda", requires_grad=True)
    rows, order = D().sort_tokens(x, ids.cuda(), S)
    out = D().combine_tokens(rows, order, w)
    dx, dw = torch.autograd.grad(out.sum() + rows.sum(), (x, w))             # gradients with strides of zero, two uses of rows
    assert torch.allclose(dx, (w.sum(1, keepdim=True) + k).expand(T, cols).detach(), rtol=1e-5)
    assert torch.allclose(dw, x.detach().sum(1, keepdim=True).expand(T, k), rtol=1e-4, atol=1e-4)
    # a gradient that starts off the 16 bytes
    flat = torch.randn(T * cols + 1, device="cuda")

    def dx_of(grad):
        rows, order = D().sort_tokens(x, ids.cuda(), S)
        return torch.autograd.grad(D().combine_tokens(rows, order, w), x, grad)[0]

    assert torch.equal(dx_of(flat[1:].view(T, cols)), dx_of(flat[1:].view(T, cols).clone()))


@pytest.mark.parametrize("dt", [BF16, F32])
def test_dropped_assignments(dt):
    """Entries of row that the caller sets to -1: nothing is added for them, and the gradient of their rows is zeros."""
    T, k, E, S, cols = 70, 4, 16, 12, 264
    ids, m, row, y, w = made(T, k, E, S, cols, dt, "map")
    offsets, source, _ = R.order(ids, S, m)
    for share in (0.3, 1.0):
        kept = torch.where(torch.rand(T, k, generator=torch.Generator().manual_seed(3)) < share, -1, row).to(torch.int32)
        order = D().Order(offsets.cuda(), source.cuda(), kept.cuda())
        g = torch.randn(T, cols, generator=torch.Generator().manual_seed(9)).to(dt)
        yg, wg = y.cuda().requires_grad_(), w.cuda().requires_grad_()
        junk = [torch.full((T * k, cols), float("nan"), dtype=dt, device="cuda") for _ in range(4)]
        del junk                                            # what the gradient may be allocated on
        out = D().combine_tokens(yg, order, wg)
        want, off = R.combine(y, kept, w)
        R.check(out.detach(), want, off, "out")
        got = torch.autograd.grad(out, (yg, wg), g.cuda())
        dy, off_y, dw, off_w = R.backward(g, y, kept, w)
        R.check(got[0], dy, off_y, "dy")
        R.check(got[1], dw, off_w, "dweights")


def test_a_gradient_of_a_gradient_is_refused():
    x = torch.randn(4, 64, device="cuda", requires_grad=True)
    ids = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    dx, = torch.autograd.grad(D().sort_tokens(x, ids, 1).rows.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dx.sum(), x)


def test_an_order_that_was_overwritten_has_no_gradient():
    T, k, S, cols = 8, 2, 4, 64
    a, b = (routing(s, T, k, S, S, "plain")[0].cuda() for s in (1, 2))
    x = torch.randn(T, cols, device="cuda")
    y = torch.randn(T * k, cols, device="cuda", requires_grad=True)
    rows, order = D().sort_tokens(x, a, S)
    out = D().combine_tokens(y, order)
    D().sort_tokens(x, b, S, rows=rows, order=order)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(out.sum(), y)


def test_a_captured_step_with_its_backward():
    """Sort, an expert's product of torch's, combine and all gradients in one graph, on leaves that no eager graph holds."""
    T, k, S, cols = 40, 4, 8, 128
    ids = torch.zeros(T, k, dtype=torch.int32, device="cuda")
    grad = torch.zeros(T, cols, device="cuda")
    values = [torch.randn(T, cols, device="cuda"), torch.rand(T, k, device="cuda"), torch.randn(T * k, 1, device="cuda")]

    def step(x, w, scale):
        rows, order = D().sort_tokens(x, ids, S)
        out = D().combine_tokens(rows * scale, order, w)
        return (out, *torch.autograd.grad(out, (x, w, scale), grad))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*(v.clone().requires_grad_() for v in values))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    leaves = [v.clone().requires_grad_() for v in values]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*leaves)
    for seed in range(3):
        ids.copy_(routing(seed, T, k, S + 1, S, "plain")[0])
        grad.copy_(torch.randn(T, cols))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.detach().clone() for t in captured]
        want = step(*(v.clone().requires_grad_() for v in values))
        for a, b in zip(got, want):
            assert torch.equal(a, b.detach())


@pytest.mark.parametrize("T", [64, 1200])
def test_replays_of_a_graph(T):
    """Sort and combine captured on buffers; every replay is the eager result for what the buffers hold by then."""
    k, E, S, cols = 8, 32, 24, 256
    x, w = torch.randn(T, cols, device="cuda"), torch.rand(T, k, device="cuda")
    ids = torch.zeros(T, k, dtype=torch.int32, device="cuda")
    m = torch.arange(E, dtype=torch.int32, device="cuda")
    rows = torch.zeros(T * k, cols, device="cuda")
    order = D().Order(*(torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((S + 1,), (T * k,), (T, k))))
    out, space = torch.zeros(T, cols, device="cuda"), D().sort_workspace(T, k, S)
    call = lambda: (D().sort_tokens(x, ids, S, expert_map=m, rows=rows, order=order, workspace=space), D().combine_tokens(rows, order, w, out=out))  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        new, _ = routing(seed, T, k, E, S, "plain")
        ids.copy_(new)
        x.copy_(torch.randn(T, cols))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        r2, o2 = D().sort_tokens(x, ids, S, expert_map=m)
        assert torch.equal(o2.row, order.row) and torch.equal(o2.offsets, order.offsets)
        assert torch.equal(D().combine_tokens(r2, o2, w), got)


def test_two_streams_with_workspaces_of_their_own():
    T, k, S, cols = 3000, 8, 64, 128
    got = []
    xs = [torch.randn(T, cols, device="cuda") for _ in range(2)]
    ids = [routing(s, T, k, S, S, "plain")[0].cuda() for s in range(2)]
    want = [D().sort_tokens(x, i, S) for x, i in zip(xs, ids)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [D().sort_tokens(x, i, S, stream=st) for x, i, st in zip(xs, ids, streams)]
        outs = [D().combine_tokens(g.rows, g.order, stream=st) for g, st in zip(got, streams)]
    torch.cuda.synchronize()
    for g, w, o in zip(got, want, outs):
        assert torch.equal(g.rows, w.rows) and torch.equal(g.order.row, w.order.row)
        assert torch.equal(o, D().combine_tokens(w.rows, w.order))


def test_threads_with_gradients():
    """Several threads at once, each on a stream of its own: x is copied k times, doubled and added up again."""
    import threading
    ids, _ = routing(2, 64, 8, 16, 16, "plain")
    ids, wrong = ids.cuda(), []
    torch.cuda.synchronize()

    def steps():
        with torch.cuda.stream(torch.cuda.Stream()):
            for n in range(1, 21):
                x = torch.randn(64, 8 * n, device="cuda", requires_grad=True)
                rows, order = D().sort_tokens(x, ids, 16)
                D().combine_tokens(rows * 2, order).sum().backward()
                if not x.grad.eq(16.0).all():
                    wrong.append(n)

    threads = [threading.Thread(target=steps) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong


def test_rows_behind_2_to_the_32_bytes():
    """140000 assignments of 32 KB rows: the last ones lie past 2^32 bytes."""
    T, k, S, cols = 17500, 8, 3, 16384
    ids, _ = routing(2, T, k, S, S, "plain")
    x = torch.randn(T, cols, device="cuda", dtype=BF16)
    rows, order = D().sort_tokens(x, ids.cuda(), S)
    source = order.source.long()
    assert torch.equal(torch.sort(source).values, torch.arange(T * k, device="cuda"))
    for lo in (0, 65530, T * k - 64):
        assert torch.equal(rows[lo:lo + 64], x[source[lo:lo + 64] // k])
    out = D().combine_tokens(rows, order)
    assert torch.equal(out, (x.float() * 8).to(BF16))
