"""Instances of the 4-bit products' kernel that the sizes of the other tests do not reach, for results of both types and for sorted rows."""
import pytest
import torch

import four_bit_ref as R
from test_gpu_four_bit import BF16, F32, Q, case, offsets_of, whole_rows, whole_weights

pytestmark = pytest.mark.gpu

# counts: rows of each group
PRODUCTS = [([3] * 40, 2048, 768), ([3] * 40, 2052, 768), ([3] * 40, 2048, 544), ([2, 3, 4, 0] * 10, 2048, 1312), ([2, 3, 4, 0] * 10, 2050, 1312), ([3] * 40, 2048, 1536),
            ([3] * 40, 2041, 1536), ([20, 40, 0, 17] * 10, 1024, 512), ([20, 40, 0, 17] * 10, 1020, 352), ([20, 40, 0, 17] * 10, 1024, 1280), ([20, 40, 0, 17] * 10, 1028, 1120),
            ([1, 0] * 40, 2048, 512), ([1, 0] * 40, 2048, 544), ([2] * 39 + [150], 2100, 1024), ([2] * 39 + [150], 2100, 992),
            ([3, 0, 40, 1, 2] * 2, 1664, 512), ([3, 0, 40, 1, 2] * 2, 1660, 544), ([3, 0, 40, 1, 2] * 2, 2048, 1120), ([3, 0, 20, 1, 2] * 2, 2044, 544), ([30, 0, 17], 100, 2816), ([30, 0, 17], 104, 2848)]
# m rows, or counts
SWIGLUS = [(1300, 1100, 256), (2500, 500, 4352), (300, 1100, 544), (300, 1100, 512), ([20, 40, 0, 17] * 5, 2048, 4352), ([20, 40, 0, 17] * 5, 2044, 4352), ([20, 40, 0, 17] * 5, 2048, 4128), ([70] * 10, 1000, 512),
           ([70] * 10, 1004, 288), ([20, 40, 0, 17] * 10, 512, 544), ([20, 40, 0, 17] * 10, 508, 512), ([3] * 40, 1024, 4352), ([3] * 40, 1028, 4352), ([3] * 40, 1024, 4128), ([9] * 70, 1000, 96),
           ([3] * 20, 640, 2048), ([3] * 20, 640, 2080), ([1, 0, 0, 0] * 8, 2048, 4352),
           ([3, 2, 1, 0, 4, 2, 3, 3], 800, 4352), ([3, 2, 1, 0, 4, 2, 30, 3], 796, 4128), ([30, 0, 17], 33, 4352), ([30, 0, 17], 36, 4128), ([1, 0, 2, 1], 100, 512), ([1, 0, 2, 1], 97, 544)]


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("counts,n,k", PRODUCTS)
def test_sorted_products_of_whole_numbers(counts, n, k, out):
    g = torch.Generator().manual_seed(n + k)
    groups, total = len(counts), sum(counts)
    (q, s), a = whole_weights(g, groups, n, k), whole_rows(g, total + 3, k)
    off = offsets_of(counts)
    got = Q().matmul(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda(), out_dtype=out).cpu()
    assert got.dtype == out and not got[total:].any()
    for e in range(groups):
        lo, hi = off[e], off[e + 1]
        if hi > lo:
            assert torch.equal(got[lo:hi], (a[lo:hi].double() @ R.values(q[e], s[e]).t()).float().to(out)), e


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("rows,inter,k", SWIGLUS)
def test_swiglu(rows, inter, k, out):
    counts = rows if isinstance(rows, list) else None
    total = sum(counts) if counts else rows
    groups = len(counts) if counts else None
    a, q, s = case(k, total + (3 if counts else 0), inter, k, groups)
    off = offsets_of(counts or [total])
    got = Q().swiglu(a.cuda(), q.cuda(), s.cuda(), offsets=off.cuda() if counts else None, out_dtype=out)
    assert got.dtype == out and not got[total:].any()
    some = [e for e in range(len(off) - 1) if off[e + 1] > off[e]]
    for e in some[::max(1, len(some) // 5)]:
        lo, hi = int(off[e]), int(off[e + 1])
        at = torch.arange(lo, hi)[torch.randperm(hi - lo, generator=torch.Generator().manual_seed(1))[:64]]
        want, far = R.swiglu(a[at].double(), torch.zeros(len(at), k).double(), R.values(q, s) if groups is None else R.values(q[e], s[e]))
        R.check(got[at.cuda()], want, far)
        if out == F32 or want.numel() >= 1000:      # of fewer, large values with the same roundings by chance
            R.check_norm(got[at.cuda()], want, out)
