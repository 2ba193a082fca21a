"""The 4-bit operators on the GPU against 64 bits; whole numbers whose sums fp32 holds have to come out exactly."""
import pytest
import torch

import dispatch_ref
import four_bit_ref as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def Q():
    from paper_2510_02613_amd import four_bit
    return four_bit


def padded(t, fill=float("nan")):
    """The same matrix with rows further apart and `fill` between them."""
    rows, cols = t.shape
    wide = torch.full((rows, (cols + 7) // 8 * 8 + 16), fill, dtype=t.dtype, device=t.device)
    wide[:, :cols] = t
    return wide[:, :cols]


# ---- quantising ----

def rows_of(kind, rows, cols, dt, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, cols // 32, generator=g)).repeat_interleave(32, 1)
    if kind == "borders":            # whole eighths: half of them ties
        x = torch.randint(-48, 49, (rows, cols), generator=g) / 8 * torch.exp2(torch.randint(-20, 20, (rows, cols // 32), generator=g).float()).repeat_interleave(32, 1)
        x[:, ::32] = 6 * torch.exp2(torch.randint(-3, 4, (rows, cols // 32), generator=g).float())
    elif kind == "tiny":             # groups whose power would be below 2^-127, in numbers that a type may hold as subnormal ones
        x = torch.randint(-200, 201, (rows, cols), generator=g) * 2.0 ** -133
        x[:, :32] = 0.0
        x[:1, 3] = -0.0
    elif kind == "huge":
        x = torch.sign(x) * torch.rand(rows, cols, generator=g) * 3.3e38
    x = x.to(dt)
    if kind == "holes":
        x[0, 5], x[-1, 40], x[rows // 2, cols - 1] = float("nan"), float("inf"), float("-inf")
    return x


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("rows,cols,kind", [(1, 32, "normal"), (3, 64, "borders"), (17, 1408, "normal"), (2, 8224, "borders"), (333, 544, "normal"), (65, 2048, "borders"), (4, 96, "tiny"),
                                            (4, 96, "huge"), (6, 160, "holes"), (5000, 32, "normal"), (0, 64, "normal")])
def test_quantize(rows, cols, kind, dt):
    x = rows_of(kind, rows, cols, dt) if rows else torch.zeros(0, cols, dtype=dt)
    codes, powers = R.quantize(x) if rows else (torch.zeros(0, cols, dtype=torch.uint8), torch.zeros(0, cols // 32, dtype=torch.uint8))
    got = Q().quantize(padded(x.cuda()))
    assert torch.equal(got.scale.cpu(), powers) and torch.equal(got.q.cpu(), R.packed(codes))
    q = torch.full((rows + 1, cols // 2 + 4), 77, dtype=torch.uint8, device="cuda")
    scale = torch.full((rows + 1, cols // 32 + 3), 77, dtype=torch.uint8, device="cuda")
    values = padded(torch.full((rows + 1, cols), 7.0, dtype=dt, device="cuda"), 3.0)
    Q().quantize(x.cuda(), q=q[:rows, :cols // 2], scale=scale[:rows, :cols // 32], values=values[:rows])
    assert torch.equal(q[:rows, :cols // 2], got.q) and torch.equal(scale[:rows, :cols // 32], got.scale)
    assert q[rows:].eq(77).all() and q[:, cols // 2:].eq(77).all() and scale[rows:].eq(77).all() and scale[:, cols // 32:].eq(77).all()
    assert values[rows:].eq(7.0).all()
    want = R.values(got.q, got.scale).to(dt)
    assert torch.equal(values[:rows].cpu().nan_to_num(9.0, 8.0, -8.0), want.nan_to_num(9.0, 8.0, -8.0))
    if rows:
        assert values.as_strided((rows + 1, 8), values.stride(), cols).eq(3.0).all()
        again = x.cuda()
        Q().quantize(again, q=got.q.clone(), scale=got.scale.clone(), values=again)
        assert torch.equal(again.cpu().nan_to_num(9.0, 8.0, -8.0), want.nan_to_num(9.0, 8.0, -8.0))


# ---- products ----

def whole_weights(g, *shape):
    """Codes and powers of a matrix whose products with whole numbers up to 8 add up exactly in fp32: multiples of 2^-3, below 2^21 in all."""
    n, k = shape[-2:]
    q = torch.randint(256, (*shape[:-1], k // 2), generator=g, dtype=torch.uint8)
    return q, torch.randint(125, 129, (*shape[:-1], k // 32), generator=g, dtype=torch.uint8)


def whole_rows(g, m, k):
    return torch.randint(-8, 9, (m, k), generator=g).to(BF16)


DENSE = [(1, 1, 32), (1, 7168, 2048), (2, 17, 96), (3, 2816, 2048), (15, 16, 128), (16, 100, 160), (17, 1543, 1440), (31, 72, 7168), (33, 64, 4128), (64, 256, 512), (65, 40, 7168), (100, 2056, 768),
         (129, 129, 1056), (173, 1543, 1440), (513, 48, 256), (700, 1000, 352), (2000, 264, 96), (0, 32, 64)]


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("m,n,k", DENSE)
def test_products_of_whole_numbers(m, n, k, out):
    g = torch.Generator().manual_seed(m + n + k)
    (q, s), a = whole_weights(g, n, k), whole_rows(g, m, k)
    want = a.double() @ R.values(q, s).t()
    assert want.abs().max() < 2 ** 20 if m else True
    got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), out_dtype=out)
    assert got.dtype == out and torch.equal(got.cpu(), want.float().to(out))
    # on strided buffers, with an addend, in place of it, nothing beside it touched
    add = torch.randint(-64, 65, (m, n), generator=g).to(out)
    given = padded(torch.cat((add, torch.full((2, n), 7.0, dtype=out))).cuda(), 3.0)
    res = Q().matmul(padded(a.cuda()), q.cuda(), s.cuda(), add=given[:m], out=given[:m])
    assert (m == 0 or res.data_ptr() == given.data_ptr()) and torch.equal(res.cpu(), (want + add.double()).float().to(out))
    assert given[m:].eq(7.0).all() and given.as_strided((m + 2, 16), given.stride(), n).eq(3.0).all()


GROUPED = [([3], 1, 100, 96), ([0, 5, 0, 1, 17, 16, 0], 7, 264, 544), ([1] * 40, 40, 48, 2048), ([33, 0, 64, 2, 100], 5, 1543, 768), ([0] * 9, 9, 64, 64), ([0] * 300 + [300], 301, 16, 32),
           ([20, 21, 22, 0, 19] * 8, 40, 256, 768), ([700, 1, 0, 0, 300], 5, 72, 160), ([1, 0] * 500, 1000, 24, 64)]


def offsets_of(counts):
    return torch.tensor([0] + counts).cumsum(0).int()


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("counts,groups,n,k", GROUPED)
def test_grouped_products_of_whole_numbers(counts, groups, n, k, out):
    g = torch.Generator().manual_seed(n + k)
    total, m = sum(counts), sum(counts) + 21
    (q, s), a = whole_weights(g, groups, n, k), whole_rows(g, m, k)
    off = offsets_of(counts)
    for e, c in enumerate(counts):
        if c == 0:
            s[e] = 255                    # weights that nobody's rows take
    a[total:] = float("nan")
    want = torch.zeros(m, n, dtype=torch.float64)
    for e in range(groups):
        want[off[e]:off[e + 1]] = a[off[e]:off[e + 1]].double() @ R.values(q[e], s[e]).t()
    got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out_dtype=out)
    assert torch.equal(got.cpu(), want.float().to(out))
    given = padded(torch.full((m, n), 7.0, dtype=out, device="cuda"), 3.0)
    add = padded(torch.randint(-64, 65, (m, n), generator=g).to(out).cuda())
    Q().matmul(padded(a.cuda()), q.cuda(), s.cuda(), offsets=off.cuda(), add=add, out=given)
    assert torch.equal(given[:total].cpu(), (want + add.cpu().double())[:total].float().to(out)) and given[total:].eq(7.0).all()
    assert given.as_strided((m, 16), given.stride(), n).eq(3.0).all()


# Every form of the kernel, k in whole lines of 256 columns and not: which one runs goes by the workgroups it would have
FORMS = [(2100, 1600, 512), (2100, 1600, 288), (1300, 1100, 512), (1300, 1100, 352), (1300, 1100, 1280), (1300, 1100, 1120), (160, 1800, 512), (160, 1800, 544), (100, 2056, 800),
         (16, 100, 2816), (16, 100, 2848), (40, 33, 7168), (1, 64, 8192)]


@pytest.mark.parametrize("m,n,k", FORMS)
def test_every_form_of_the_product(m, n, k):
    g = torch.Generator().manual_seed(m + n + k)
    (q, s), a = whole_weights(g, n, k), whole_rows(g, m, k)
    want = a.double() @ R.values(q, s).t()
    for out in (BF16, F32):
        assert torch.equal(Q().matmul(a.cuda(), q.cuda(), s.cuda(), out_dtype=out).cpu(), want.float().to(out))


GROUP_FORMS = [([3] * 40, 2048, 768), ([3] * 40, 2048, 544), ([2, 3, 4, 0] * 10, 2048, 1312), ([3] * 40, 2048, 1536), ([20, 40, 0, 17] * 10, 1024, 512), ([20, 40, 0, 17] * 10, 1024, 1120),
               ([1] + [0] * 70 + [5] + [0] * 200, 48, 160), ([0] * 500 + [2] + [0] * 300 + [1] + [0] * 99, 272, 96), ([0] * 1999 + [40], 16, 32), ([200] * 3 + [0] * 4 + [1000], 520, 96),
               # several slices of weight rows with the same rows, one tile of them after the other; groups much longer than the others
               ([20, 40, 0, 17] * 10, 4100, 288), ([12] * 38 + [0, 900], 1100, 736), ([12] * 38 + [0, 900], 2200, 768), ([2] * 39 + [150], 2100, 1024), ([2] * 39 + [150], 2100, 992),
               ([1, 0] * 40, 2048, 512), ([1, 0] * 40, 2048, 544), ([20, 40, 0, 17] * 10, 1024, 1024), ([20, 40, 0, 17] * 10, 1024, 800)]


@pytest.mark.parametrize("counts,n,k", GROUP_FORMS)
def test_every_form_of_the_grouped_product(counts, n, k):
    g = torch.Generator().manual_seed(n + k)
    groups, total = len(counts), sum(counts)
    (q, s), a = whole_weights(g, groups, n, k), whole_rows(g, total + 3, k)
    off = offsets_of(counts)
    got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out_dtype=F32).cpu()
    assert not got[total:].any()
    for e in range(groups):
        lo, hi = off[e], off[e + 1]
        if hi > lo:
            assert torch.equal(got[lo:hi].double(), a[lo:hi].double() @ R.values(q[e], s[e]).t()), e


def test_offsets_that_leave_the_rows_are_cut():
    g = torch.Generator().manual_seed(3)
    (q, s), a = whole_weights(g, 4, 32, 64), whole_rows(g, 10, 64)
    off = torch.tensor([-5, 4, 2, 8, 99], dtype=torch.int32)      # rows 0..3, none, rows 2..7, rows 8..9
    got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out_dtype=F32).cpu()
    w = [R.values(q[e], s[e]) for e in range(4)]
    assert torch.equal(got[:2].double(), a[:2].double() @ w[0].t()) and torch.equal(got[4:8].double(), a[4:8].double() @ w[2].t())
    assert torch.equal(got[8:].double(), a[8:].double() @ w[3].t())


@pytest.mark.parametrize("m,n,k", [(1, 512, 7168), (5, 96, 2048), (40, 200, 1440), (300, 300, 4096)])
def test_products_of_normal_values(m, n, k):
    g = torch.Generator().manual_seed(k)
    a = (torch.randn(m, k, generator=g) * torch.exp(0.6 * torch.randn(k, generator=g))).to(BF16)
    q, s = Q().quantize((0.02 * torch.randn(n, k, generator=g)).cuda())
    want, off = R.product(a.double(), torch.zeros(m, k).double(), R.values(q, s))
    for out in (BF16, F32):
        got = Q().matmul(a.cuda(), q, s, out_dtype=out)
        R.check(got, want, off)
        R.check_norm(got, want, out)
    # the same bytes under the names of their types
    again = Q().matmul(a.cuda(), q.view(torch.float4_e2m1fn_x2), s.view(torch.float8_e8m0fnu), out_dtype=F32)
    assert torch.equal(again, got)


def test_powers_from_end_to_end():
    """Powers of 2^-127 to 2^126 and NaN, each in a weight row of its own; activations bring the sums back into range."""
    k = 64
    q = torch.randint(256, (256, k // 2), generator=torch.Generator().manual_seed(1), dtype=torch.uint8)
    s = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 2)
    for scale in (2.0 ** 100, 1.0, 2.0 ** -100):
        a = torch.full((3, k), scale, dtype=BF16)
        w = R.values(q, s)
        want = a.double() @ w.t()
        got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), out_dtype=F32).cpu()
        fine = (w.abs().amax(1) * scale * k < 3e38) & (w.abs().amax(1) < 3e38) & ((want[0].abs() > 1e-37) | (want[0] == 0))
        assert fine.sum() > 140 and torch.equal(got[:, fine], want[:, fine].float())
        assert got[:, 255].isnan().all()


def test_not_a_number_stays_in_its_row():
    g = torch.Generator().manual_seed(3)
    (q, s), a = whole_weights(g, 40, 256), whole_rows(g, 20, 256)
    want = a.double() @ R.values(q, s).t()
    a[3, 17], a[19, 255] = float("nan"), float("inf")
    got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), out_dtype=F32).cpu()
    other = [r for r in range(20) if r not in (3, 19)]
    assert torch.equal(got[other].double(), want[other]) and got[3].isnan().all() and not torch.isfinite(got[19]).any()


# ---- SwiGLU ----

def case(seed, m, inter, k, groups=None):
    g = torch.Generator().manual_seed(seed)
    a = torch.randn(m, k, generator=g).to(BF16)
    shape = (2 * inter, k) if groups is None else (groups, 2 * inter, k)
    codes = torch.randint(256, (*shape[:-1], k // 2), generator=g, dtype=torch.uint8)
    return a, codes, torch.randint(118, 122, (*shape[:-1], k // 32), generator=g, dtype=torch.uint8)


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("m,inter,k", [(1, 1, 32), (1, 2048, 7168), (3, 1408, 2048), (16, 100, 544), (17, 33, 96), (50, 768, 2048), (200, 264, 1056), (1030, 40, 64), (0, 16, 32)])
def test_swiglu(m, inter, k, out):
    a, q, s = case(m + k, m, inter, k)
    want, off = R.swiglu(a.double(), torch.zeros(m, k).double(), R.values(q, s))
    got = Q().swiglu(a.cuda(), q.cuda(), s.cuda(), out_dtype=out)
    R.check(got, want, off)
    if m * inter > 100:
        R.check_norm(got, want, out)
    given = padded(torch.full((m + 2, inter), 7.0, dtype=out, device="cuda"), 3.0)
    Q().swiglu(padded(a.cuda()), q.cuda(), s.cuda(), out=given[:m])
    assert torch.equal(given[:m], got) and given[m:].eq(7.0).all() and given.as_strided((m + 2, 16), given.stride(), inter).eq(3.0).all()


@pytest.mark.parametrize("m,inter,k", [(1300, 1100, 64), (1300, 1100, 288), (2500, 500, 4128), (200, 800, 512), (200, 800, 544), (200, 520, 1024), (200, 520, 1056), (16, 100, 7168), (17, 33, 4128),
                                       (300, 2100, 4352)])
def test_every_form_of_swiglu(m, inter, k):
    a, q, s = case(m + k, m, inter, k)
    rows = torch.randperm(m, generator=torch.Generator().manual_seed(1))[:64]
    want, off = R.swiglu(a[rows].double(), torch.zeros(len(rows), k).double(), R.values(q, s))
    for out in (BF16, F32):
        got = Q().swiglu(a.cuda(), q.cuda(), s.cuda(), out_dtype=out)[rows.cuda()]
        R.check(got, want, off)
        R.check_norm(got, want, out)


@pytest.mark.parametrize("counts,inter,k", [([20, 40, 0, 17] * 10, 512, 544), ([20, 40, 0, 17] * 10, 512, 512), ([3] * 40, 1024, 4352), ([3] * 40, 1024, 4128), ([20, 40, 0, 17] * 5, 2048, 4128),
                                            ([3] * 20, 640, 2048), ([0] * 500 + [2] + [0] * 399, 48, 96), ([1, 0, 0, 0] * 8, 2048, 4352),
                                            ([20, 40, 0, 17] * 10, 1700, 288), ([20, 40, 0, 17] * 10, 1664, 2048), ([9] * 70, 1000, 96), ([12] * 38 + [0, 900], 2100, 1056)])
def test_every_form_of_grouped_swiglu(counts, inter, k):
    groups, total = len(counts), sum(counts)
    a, q, s = case(k, total + 3, inter, k, groups)
    off = offsets_of(counts)
    got = Q().swiglu(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out_dtype=F32)
    assert not got[total:].any()
    for e in [e for e in range(groups) if counts[e]][::max(1, groups // 5)]:
        lo, hi = off[e], off[e + 1]
        want, far = R.swiglu(a[lo:hi].double(), torch.zeros(hi - lo, k).double(), R.values(q[e], s[e]))
        R.check(got[lo:hi], want, far)
        R.check_norm(got[lo:hi], want, F32)


@pytest.mark.parametrize("counts,groups,n,k", GROUPED)
def test_grouped_swiglu(counts, groups, n, k):
    m, off = sum(counts) + 5, offsets_of(counts)
    a, q, s = case(n, m, n, k, groups)
    a[off[-1]:] = float("nan")
    got = Q().swiglu(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out_dtype=F32)
    assert not got[off[-1]:].any()
    for e in range(groups):
        lo, hi = off[e], off[e + 1]
        if hi > lo:
            want, far = R.swiglu(a[lo:hi].double(), torch.zeros(hi - lo, k).double(), R.values(q[e], s[e]))
            R.check(got[lo:hi], want, far)
    given = torch.full((m, (n + 7) // 8 * 8), 7.0, dtype=F32, device="cuda")[:, :n]
    Q().swiglu(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out=given)
    assert torch.equal(given[:off[-1]], got[:off[-1]]) and given[off[-1]:].eq(7.0).all()


# ---- together ----

@pytest.mark.parametrize("T,k,E,S,H,I", [(1, 8, 32, 8, 256, 96), (37, 4, 16, 11, 544, 160), (300, 6, 16, 16, 256, 352)])
def test_a_layer_in_pieces(T, k, E, S, H, I):
    """Sorted, through 4-bit experts, added up again: the whole of a layer whose routing is given, against 64 bits with the roundings in between."""
    from paper_2510_02613_amd import dispatch
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, H, generator=g).to(BF16)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).int()
    m = torch.full((E,), -1, dtype=torch.int32)
    m[torch.randperm(E, generator=g)[:S]] = torch.randperm(S, generator=g).int()
    w = torch.softmax(torch.randn(T, k, generator=g), 1)
    q13, s13 = Q().quantize((0.05 * torch.randn(S * 2 * I, H, generator=g)).cuda())
    q2, s2 = Q().quantize((0.05 * torch.randn(S * H, I, generator=g)).cuda())
    q13, s13, q2, s2 = q13.view(S, 2 * I, -1), s13.view(S, 2 * I, -1), q2.view(S, H, -1), s2.view(S, H, -1)
    rows, order = dispatch.sort_tokens(x.cuda(), ids.cuda(), S, expert_map=m.cuda())
    h = Q().swiglu(rows, q13, s13, offsets=order.offsets)
    y = Q().matmul(h, q2, s2, offsets=order.offsets, out_dtype=F32)
    out = dispatch.combine_tokens(y, order, w.cuda())
    assert out.dtype == F32
    want, off = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    _, _, row = dispatch_ref.order(ids, S, m)
    for e in range(S):
        for t, j in (dispatch_ref.groups(ids, S, m).view(T, k) == e).nonzero().tolist():
            hw, dh = R.swiglu(x[t:t + 1].double(), torch.zeros(1, H).double(), R.values(q13[e], s13[e]))
            yw, dy = R.product(hw, dh + R.BF16 * (hw.abs() + dh), R.values(q2[e], s2[e]))
            want[t] += w[t, j].double() * yw[0]
            off[t] += w[t, j].double() * (dy + (k + 2) * R.F32 * yw.abs())[0]
    assert torch.equal(order.row.cpu(), row)
    R.check(out, want, off)


def test_replays_of_a_graph():
    """A layer in pieces captured on buffers; every replay is the eager result for what the buffers hold by then."""
    from paper_2510_02613_amd import dispatch
    T, k, S, H, I = 24, 4, 8, 256, 128
    x, ids = torch.zeros(T, H, dtype=BF16, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda")
    w = torch.rand(T, k, device="cuda")
    (q13, s13), (q2, s2) = (Q().quantize(0.05 * torch.randn(S * n, c, device="cuda")) for n, c in ((2 * I, H), (H, I)))
    q13, s13, q2, s2 = q13.view(S, 2 * I, -1), s13.view(S, 2 * I, -1), q2.view(S, H, -1), s2.view(S, H, -1)
    new = lambda *s, dt=BF16: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    rows, h, y, out = new(T * k, H), new(T * k, I), new(T * k, H), new(T, H)
    order = dispatch.Order(new(S + 1, dt=torch.int32), new(T * k, dt=torch.int32), new(T, k, dt=torch.int32))

    def call(rows=rows, order=order, h=h, y=y, out=out):
        dispatch.sort_tokens(x, ids, S, rows=rows, order=order)
        Q().swiglu(rows, q13, s13, offsets=order.offsets, out=h)
        Q().matmul(h, q2, s2, offsets=order.offsets, out=y)
        return dispatch.combine_tokens(y, order, w, out=out)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        ids.copy_(torch.randint(-1, S if seed else 1, (T, k), generator=g).int())
        x.copy_(torch.randn(T, H, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(call(new(T * k, H), dispatch.Order(*(torch.zeros_like(t) for t in order)), new(T * k, I), new(T * k, H), new(T, H)), got)


def test_two_streams():
    g = torch.Generator().manual_seed(2)
    cases = [(whole_rows(g, m, 512).cuda(), *(t.cuda() for t in whole_weights(g, 300, 512))) for m in (5, 90)]
    want = [Q().matmul(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [Q().matmul(*c, stream=st) for c, st in zip(cases, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_behind_2_to_the_32_bytes():
    groups, n, k = 300, 4096, 7168
    q = torch.empty(groups, n, k // 2, dtype=torch.uint8, device="cuda")
    s = torch.full((groups, n, k // 32), 126, dtype=torch.uint8, device="cuda")
    g = torch.Generator().manual_seed(2)
    last, _ = whole_weights(g, n, k)
    q[-1] = last.cuda()
    a = whole_rows(g, 3, k)
    off = torch.tensor([0] * groups + [3], dtype=torch.int32, device="cuda")
    got = Q().matmul(a.cuda(), q, s, offsets=off, out_dtype=F32)
    want = a.double() @ R.values(last, torch.full((n, k // 32), 126, dtype=torch.uint8)).t()
    assert torch.equal(got.cpu().double(), want)
