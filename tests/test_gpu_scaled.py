"""The operators of the 8-bit path against their definitions in 64 bits: norm with residual, quantising, the block-scaled product and its SwiGLU form."""
import pytest
import torch

import scaled_ref as R

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def S():
    from paper_2510_02613_amd import scaled
    return scaled


def randn(seed, *shape):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g)


def strided(t, ld):
    """t on the GPU with rows ld elements apart; what lies between the rows is NaN."""
    fill = torch.full((t.shape[0], ld), float("nan"), dtype=torch.float32).to(t.dtype).cuda()
    fill[:, :t.shape[1]] = t.cuda()
    return fill[:, :t.shape[1]]


def eight_bit_rows(seed, m, k, zero_rows=False):
    """8-bit rows with random scales of a wide range, on the CPU: (q, scale, their values)."""
    q = (randn(seed, m, k) * 100).clamp(-448, 448).to(E4M3)
    scale = torch.exp(randn(seed + 1, m, R.blocks(k))) * 0.01
    if zero_rows and m:
        scale[m // 2] = 0.0
    return q, scale, q.double() * R.spread_rows(scale, k)


def eight_bit_weights(seed, n, k, parts=1):
    q = (randn(seed, n, k) * 100).clamp(-448, 448).to(E4M3)
    scale = torch.exp(0.5 * randn(seed + 1, parts * R.blocks(n // parts), R.blocks(k))) * 2e-4
    nb = R.blocks(n // parts)
    values = torch.cat([q[i * (n // parts):(i + 1) * (n // parts)].double() * R.spread_blocks(scale[i * nb:(i + 1) * nb], n // parts, k)
                        for i in range(parts)])
    return q, scale, values


# ---- norm ----

NORM = [(1, 8), (1, 7168), (3, 128), (5, 136), (64, 1024), (7, 1032), (33, 2048), (2, 2056), (9, 8192), (3, 8200), (2, 32768), (300, 264)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", NORM)
def test_rms_norm(S, rows, cols, dtype):
    x, res = (randn(rows + cols, rows, cols) * 2).to(dtype), randn(rows * cols, rows, cols).to(dtype)
    w = (1 + 0.3 * randn(cols, cols)).to(dtype)
    if rows > 2:
        x[1] = 0
        res[1] = 0                                       # a row of zeros: scale 0, zeros
    xd, rd = strided(x, cols + 8), strided(res, cols + 16)
    out, total = strided(x, cols + 24), strided(x, cols + 8)
    q, scale = strided(torch.zeros(rows, cols).to(E4M3), cols + 8), torch.full((rows, R.blocks(cols) + 1), float("nan")).cuda()[:, :R.blocks(cols)]
    S.rms_norm(xd, w.cuda(), residual=rd, eps=1e-5, sum_out=total, out=out, q=q, q_scale=scale)
    r = x.double() + res.double()
    y = r / torch.sqrt((r * r).mean(1, keepdim=True) + 1e-5) * w.double()
    # fp32: the addition, at most 64 additions in a chain of squares, the square root and four products
    fp32 = 80 * R.F32
    half = R.HALF_STEP[dtype]
    assert ((total.cpu().double() - r).abs() <= (half + R.F32) * r.abs()).all()
    assert ((out.cpu().double() - y).abs() <= (half + 2 * fp32) * y.abs() + 1e-30).all()
    R.check_quantized(q.cpu(), scale.cpu(), y, fp32 * y.abs())
    assert torch.isnan(xd.as_strided((rows, 8), (xd.stride(0), 1), cols)).all()      # nothing was written between the rows
    for t, n in ((out, 24), (total, 8)):
        assert torch.isnan(t.as_strided((rows, n), (t.stride(0), 1), cols)).all()


def test_rms_norm_in_place_and_without_residual(S):
    x, res, w = randn(1, 37, 2048).bfloat16(), randn(2, 37, 2048).bfloat16(), randn(3, 2048).bfloat16()
    want = S.rms_norm(x.cuda(), w.cuda(), residual=res.cuda())
    xd, rd = x.cuda(), res.cuda()
    got = S.rms_norm(xd, w.cuda(), residual=rd, sum_out=rd, out=xd)
    assert torch.equal(got.sum, want.sum) and torch.equal(got.out, want.out) and got.out is xd and got.sum is rd
    plain = S.rms_norm(x.cuda())
    y = x.double() / torch.sqrt((x.double() ** 2).mean(1, keepdim=True) + 1e-6)
    assert plain.sum is None and ((plain.out.cpu().double() - y).abs() <= (R.BF16 + 160 * R.F32) * y.abs()).all()


# ---- quantising ----

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,block_rows", [(1, 8, 1), (5, 136, 1), (130, 2048, 1), (3, 8200, 1), (1, 8, 128), (128, 128, 128),
                                                  (129, 136, 128), (300, 1032, 128), (64, 40, 128)])
def test_quantize(S, rows, cols, block_rows, dtype):
    x = (randn(rows + cols, rows, cols) * torch.exp(2 * randn(cols, 1, cols))).to(dtype)
    x[0, 0] = 0.0
    got = S.quantize(strided(x, cols + 8), block_rows=block_rows)
    R.check_quantized(got.q.cpu(), got.scale.cpu(), x.double(), torch.zeros(rows, cols, dtype=torch.float64), block_rows)
    if dtype == torch.bfloat16:
        # quotients of bf16 numbers meet half-way points exactly, or miss them by far more than fp32 is off: every byte is certain
        _, per = R.group_max(x.double(), block_rows)
        t = torch.where(per > 0, x.double() * 448 / per, 0.0)
        assert torch.equal(got.q.cpu().double().abs(), R.e4m3_round(t).abs())


def test_quantize_ties_go_to_even(S):
    x = torch.zeros(1, 128)
    x[0, 0] = 448.0
    steps = torch.arange(8, 16).float()
    x[0, 1:9] = steps * 2 + 1                     # half way between neighbours 2 apart, from 17 to 31
    x[0, 9:17] = -(steps * 2 + 1)
    x[0, 17:19] = torch.tensor([2.0 ** -10, 3 * 2.0 ** -10])    # half of the smallest value, and between the first two
    got = S.quantize(x.bfloat16().cuda())
    assert got.scale.item() == 1.0
    want = R.e4m3_round(x.double())
    assert torch.equal(got.q.cpu().double(), want) and want[0, 17] == 0 and want[0, 18] == 2.0 ** -8


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_extremes(S, block_rows):
    """Groups of zeros, of tiny and of huge numbers, and groups that hold an infinity or a NaN."""
    x = torch.zeros(2, 7 * 128)
    x[:, 128:256] = 1e-38                       # below 2^-110: counts as zero
    x[:, 256:384] = torch.linspace(1e30, 3e38, 128)
    x[:, 384:512] = 1.0
    x[0, 400] = float("inf")
    x[:, 512:640] = 2.0
    x[0, 600] = float("nan")
    x[:, 640:768] = torch.linspace(2.0 ** -109, 2.0 ** -106, 128)
    x[:, 768:] = torch.linspace(-3, 3, 128)
    got = S.quantize(x.cuda(), block_rows=block_rows)
    q, scale = got.q.cpu().float(), got.scale.cpu()
    value = q.double() * scale.double().repeat_interleave(128, 1)
    assert (q[:, :256] == 0).all() and (scale[:, :2] == 0).all()
    for b in (2, 5, 6):
        cols = slice(128 * b, 128 * b + 128)
        R.check_quantized(got.q.cpu()[:, cols], scale[:, b:b + 1], x[:, cols].double(), torch.zeros(2, 128, dtype=torch.float64), block_rows)
    assert torch.isnan(value[0, 384:640]).all()
    if block_rows == 1:
        # 448 times the rounded a / 448: off by half a step of fp32 at most
        assert ((value[1, 384:512] - 1).abs() <= R.F32).all() and ((value[1, 512:640] - 2).abs() <= 2 * R.F32).all()


# ---- products ----

MATMUL = [(1, 1, 16), (1, 7168, 2048), (3, 17, 128), (16, 128, 144), (17, 130, 256), (33, 264, 400), (64, 200, 1024), (65, 136, 272),
          (100, 384, 128), (129, 257, 1168), (257, 520, 640), (300, 1000, 48), (513, 256, 512), (1000, 129, 2048), (40, 768, 7168),
          # tiles of 32, 64, 128, 192 and 256 rows (fp32 results: up to 128), the last tile one of few rows
          (2001, 520, 1168), (2000, 1032, 2048), (3000, 1001, 400), (5000, 1100, 272), (4100, 2050, 528), (8201, 1300, 400), (9000, 2100, 112), (8190, 1288, 512)]


@pytest.mark.parametrize("m,n,k", MATMUL)
def test_matmul(S, m, n, k):
    q, scale, a = eight_bit_rows(m + k, m, k, zero_rows=True)
    wq, ws, w = eight_bit_weights(n + k, n, k)
    y, exact = R.product(a, torch.zeros_like(a), w)
    fast = R.product(a, torch.zeros_like(a), w, fast=True)[1]       # what bf16 results of many rows may come from
    # rows further apart than they are long, with NaN bytes between them
    wide = torch.full((m, k + 32), float("nan")).to(E4M3).cuda()
    wide[:, :k] = q.cuda()
    sw = torch.full((m, R.blocks(k) + 3), float("nan")).cuda()
    sw[:, :R.blocks(k)] = scale.cuda()
    for dtype, dy in ((torch.float32, exact), (torch.bfloat16, fast)):
        add = randn(m * n, m, n).to(dtype)
        ld = (n + 7) // 8 * 8 + 8
        for with_add in (False, True):
            out = strided(torch.zeros(m, n, dtype=dtype), ld)
            if with_add:
                out.copy_(add.cuda())
            S.matmul(wide[:, :k], sw[:, :R.blocks(k)], wq.cuda(), ws.cuda(), add=out if with_add else None, out=out)
            want = y + add.double() if with_add else y
            off = (out.cpu().double() - want).abs() - (dy + R.F32 * want.abs()) * (1 + R.BF16) - R.HALF_STEP[dtype] * want.abs()
            assert (off <= 0).all(), (dtype, with_add, off.max().item())
            assert torch.isnan(out.as_strided((m, ld - n), (ld, 1), n)).all()


SWIGLU = [(1, 16, 16), (1, 2048, 512), (2, 128, 128), (17, 1408, 256), (16, 144, 272), (63, 256, 400), (64, 768, 128), (65, 272, 144), (130, 128, 1024),
          (257, 400, 384), (300, 2048, 128), (600, 136 + 8, 640), (700, 1040, 2064), (2000, 528, 1168), (3001, 400, 400), (2100, 912, 512), (1500, 1040, 96)]


@pytest.mark.parametrize("m,inter,k", SWIGLU)
def test_swiglu(S, m, inter, k):
    q, scale, a = eight_bit_rows(m + k, m, k, zero_rows=m > 4)
    wq, ws, w = eight_bit_weights(inter + k, 2 * inter, k, parts=2)
    h, dh = R.swiglu(a, torch.zeros_like(a), w)
    rows = torch.full((m + 2, inter + 16), float("nan")).to(E4M3).cuda()
    scales = torch.full((m + 2, R.blocks(inter)), 7.0).cuda()
    S.swiglu(q.cuda(), scale.cuda(), wq.cuda(), ws.cuda(), q=rows[:m, :inter], scale=scales[:m])
    R.check_quantized(rows[:m, :inter].cpu(), scales[:m].cpu(), h, dh)
    assert torch.isnan(rows[m:].float()).all() and torch.isnan(rows[:, inter:].float()).all() and (scales[m:] == 7).all()


@pytest.mark.parametrize("m", [3, 300])
def test_matmul_of_weights_past_32_bits(S, m):
    """4.3 GB of weights: rows behind the first 2^32 bytes, streamed and in tiles."""
    n, k = 66048, 65552
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.empty(n, k, dtype=E4M3, device="cuda")
    for at in range(0, n, 4128):      # 0 .. 0x77: finite values
        w[at:at + 4128].view(torch.uint8).copy_(torch.randint(0, 0x60, (4128, k), dtype=torch.uint8, device="cuda", generator=g))
    ws = torch.rand(R.blocks(n), R.blocks(k), device="cuda", generator=g) * 1e-3
    q, scale, a = eight_bit_rows(3, m, k)
    out = S.matmul(q.cuda(), scale.cuda(), w, ws, out_dtype=torch.float32)
    cols = [0, 65535, 65536, 65537, 66000, n - 1]
    wv = torch.stack([w[c].cpu().double() * ws[c // 128].cpu().double().repeat_interleave(128)[:k] for c in cols])
    y, dy = R.product(a, torch.zeros_like(a), wv)
    assert ((out[:, cols].cpu().double() - y).abs() <= dy).all()


def test_matmul_of_rows_past_32_bits(S):
    """Rows four million bytes apart, 1100 of them."""
    m, n, k, ld = 1100, 1536, 1024, 1 << 22
    q, scale, a = eight_bit_rows(4, m, k)
    wq, ws, w = eight_bit_weights(5, n, k)
    wide = torch.empty(m * ld, dtype=torch.uint8, device="cuda").view(E4M3).view(m, ld)[:, :k]
    wide.view(torch.uint8).copy_(q.view(torch.uint8).cuda())
    for dtype, fast in ((torch.float32, False), (torch.bfloat16, True)):
        out = S.matmul(wide, scale.cuda(), wq.cuda(), ws.cuda(), out_dtype=dtype)
        y, dy = R.product(a, torch.zeros_like(a), w, fast=fast)
        assert ((out.cpu().double() - y).abs() <= (dy + R.F32 * y.abs()) * (1 + R.BF16) + R.HALF_STEP[dtype] * y.abs()).all()


def test_both_forms_of_the_products_run():
    """What the sizes above are for: some are streamed, some go through tiles."""
    from gpu_util import kernels_of
    from paper_2510_02613_amd import scaled as S

    def names(m, n, k, dtype):
        q, scale, _ = eight_bit_rows(1, m, k)
        wq, ws, _ = eight_bit_weights(2, n, k)
        q, scale, wq, ws, out = q.cuda(), scale.cuda(), wq.cuda(), ws.cuda(), torch.empty(m, n, dtype=dtype, device="cuda")
        return kernels_of(lambda stream: S.matmul(q, scale, wq, ws, out=out, stream=stream))

    for dtype in (torch.bfloat16, torch.float32):
        assert ["k_scaled_stream" in n for n in names(16, 128, 144, dtype)] == [True]
        for m, n, k in ((3000, 1000, 400), (5000, 1104, 272)):
            assert ["k_scaled_tiles" in n_ for n_ in names(m, n, k, dtype)] == [True]


@pytest.mark.parametrize("m", [70, 2100])
def test_nan_stays_in_its_row_and_column(S, m):
    q, scale, a = eight_bit_rows(5, m, 384)
    wq, ws, w = eight_bit_weights(6, 520, 384)
    qn, wn = q.float(), wq.float()
    qn[3, 200] = float("nan")
    wn[150, 7] = float("nan")
    out = S.matmul(qn.to(E4M3).cuda(), scale.cuda(), wn.to(E4M3).cuda(), ws.cuda(), out_dtype=torch.float32).cpu()
    bad = torch.zeros(m, 520, dtype=torch.bool)
    bad[3], bad[:, 150] = True, True
    assert torch.equal(torch.isnan(out), bad)
    out = S.matmul(qn.to(E4M3).cuda(), scale.cuda(), wn.to(E4M3).cuda(), ws.cuda()).cpu()
    assert torch.equal(torch.isnan(out), bad)


@pytest.mark.parametrize("m,n,k", [(1000, 1032, 1152), (4500, 2100, 1152), (9000, 4100, 384)])
def test_a_row_is_the_same_wherever_it_stands(S, m, n, k):
    """Rows of whole tiles, of the last one and of tiles that several workgroups share: the second half repeats the first."""
    q, scale, _ = eight_bit_rows(m + k, m // 2, k)
    q, scale = torch.cat([q.view(torch.uint8)] * 2).view(q.dtype).cuda(), torch.cat([scale] * 2).cuda()
    wq, ws, _ = eight_bit_weights(n + k, n, k)
    for dtype in (torch.bfloat16, torch.float32):
        out = S.matmul(q, scale, wq.cuda(), ws.cuda(), out_dtype=dtype)
        assert torch.equal(out[:m // 2], out[m // 2:])
    wq, ws, _ = eight_bit_weights(n, 2 * n - n % 16 * 2, k, parts=2)
    got = S.swiglu(q, scale, wq.cuda(), ws.cuda())
    assert torch.equal(got.q[:m // 2].view(torch.uint8), got.q[m // 2:].view(torch.uint8)) and torch.equal(got.scale[:m // 2], got.scale[m // 2:])


@pytest.mark.parametrize("m,n,k", [(5, 136, 256), (3001, 1000, 400)])
def test_rows_behind_the_last_are_left_alone(S, m, n, k):
    q, scale, _ = eight_bit_rows(5, m, k)
    wq, ws, _ = eight_bit_weights(6, n, k)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((m + 3, n), 7.0, dtype=dtype, device="cuda")
        S.matmul(q.cuda(), scale.cuda(), wq.cuda(), ws.cuda(), out=out[:m])
        assert (out[m:] == 7).all() and not (out[:m] == 7).all(1).any()


def test_two_streams_at_once(S):
    """Products on two streams, each with a workspace of its own, beside each other: what they are one after the other."""
    sizes = [(9, 768, 2048), (700, 1040, 2064)]
    args, want = [], []
    for m, inter, k in sizes:
        q, scale, _ = eight_bit_rows(m, m, k)
        w, ws, _ = eight_bit_weights(k, 2 * inter, k, parts=2)
        args.append([t.cuda() for t in (q, scale, w, ws)])
        want.append([t.clone() for t in S.swiglu(*args[-1])])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    spaces = [S.swiglu_workspace(*s) for s in sizes]
    assert spaces[0] is not None and spaces[1] is None
    got = [[torch.empty_like(t) for t in w] for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for a, s, ws, (q, sc) in zip(args, streams, spaces, got):
            S.swiglu(*a, q=q, scale=sc, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0].view(torch.uint8), w[0].view(torch.uint8)) and torch.equal(g[1], w[1])


def test_zero_rows_are_a_no_op(S):
    e = lambda *s, dt=E4M3: torch.empty(s, dtype=torch.float32).to(dt).cuda()  # noqa: E731
    assert S.rms_norm(e(0, 128, dt=torch.bfloat16)).out.shape == (0, 128)
    assert S.quantize(e(0, 128, dt=torch.bfloat16)).q.shape == (0, 128)
    w, ws = e(256, 128), e(2, 1, dt=torch.float32)
    assert S.matmul(e(0, 128), e(0, 1, dt=torch.float32), w, ws).shape == (0, 256)
    assert S.swiglu(e(0, 128), e(0, 1, dt=torch.float32), w, ws).q.shape == (0, 128)


def test_dense_expert_in_a_graph_and_on_another_stream(S):
    """Norm, both halves of a dense expert and the addition to the residual stream: eager, captured and replayed on changed inputs."""
    T, H, I = 40, 256, 384
    w13, s13, _ = eight_bit_weights(1, 2 * I, H, parts=2)
    w2, s2, _ = eight_bit_weights(2, H, I)
    w13, s13, w2, s2 = w13.cuda(), s13.cuda(), w2.cuda(), s2.cuda()
    x, res = torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    q, sc = torch.empty(T, H, dtype=E4M3, device="cuda"), torch.empty(T, 2, device="cuda")
    h, hs = torch.empty(T, I, dtype=E4M3, device="cuda"), torch.empty(T, 3, device="cuda")
    total, out = torch.empty_like(x), torch.empty_like(x)
    ws = S.swiglu_workspace(T, I, H)

    def chain():
        S.rms_norm(x, residual=res, sum_out=total, q=q, q_scale=sc)
        S.swiglu(q, sc, w13, s13, q=h, scale=hs, workspace=ws)
        S.matmul(h, hs, w2, s2, add=total, out=out)

    def fill(seed):
        x.copy_(randn(seed, T, H))
        res.copy_(randn(seed + 1, T, H))

    side = torch.cuda.Stream()
    fill(10)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        chain()
    side.synchronize()
    first = out.clone()
    chain()
    assert torch.equal(out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for seed in (20, 30, 10, 10):
        fill(seed)
        chain()
        want = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    assert torch.equal(out, first)
    # and the chain is what its parts say, in 64 bits
    fill(10)
    chain()
    r = x.cpu().double() + res.cpu().double()
    y = r / torch.sqrt((r * r).mean(1, keepdim=True) + 1e-6)
    v, dv = R.quantize(y, 80 * R.F32 * y.abs())
    hh, dh = R.swiglu(v, dv, torch.cat([w13.cpu()[:I].double() * R.spread_blocks(s13.cpu()[:3], I, H), w13.cpu()[I:].double() * R.spread_blocks(s13.cpu()[3:], I, H)]))
    v, dv = R.quantize(hh, dh)
    o, do = R.product(v, dv, w2.cpu().double() * R.spread_blocks(s2.cpu(), H, I))
    o = o + total.cpu().double()
    assert ((out.cpu().double() - o).abs() <= do + (R.BF16 + 2 * R.F32) * o.abs()).all()
