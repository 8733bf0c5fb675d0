"""Products of 8-bit rows and weights whose scales lie far apart: a result that fp32 holds is not lost on the way to it."""
import pytest
import torch

import paper_2408_05676_amd as laser
from tests import eight_bit_ref as ref
from tests.test_gpu_eight_bit import gen, made, padded

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
# scales of weights and of rows: either's products with a sum pass fp32 or fall below it, both together do not
FAR = [(1e31, 1e-30), (2e36, 1e-37), (1e-44, 1e38), (1e-39, 1e38), (1e-30, 1e31), (1e-37, 2e36), (1e38, 1e-44), (1e38, 1e-39)]


def inside(p):
    """Results that fp32 holds as normal numbers; the others are infinite, or rounded to the fewer bits of the numbers below them."""
    return (p.abs() < torch.finfo(F32).max * (1 - 2.0 ** -20)) & (p.abs() > 2.0 ** -126)


@pytest.mark.parametrize("sw, sx", FAR)
@pytest.mark.parametrize("M, N, Kd", [(1, 40, 200), (9, 100, 1000), (40, 300, 256), (200, 700, 512), (704, 6144, 384)])
def test_scales_far_apart(M, N, Kd, sw, sx):
    g = gen(M)
    w, a = made(g, N, Kd)
    x, b = made(g, M, Kd)
    a, b = (a.double() * 1e3 * sw).float(), (b.double() * 1e3 * sx).float()
    a[:3], b[1:2] = 1.0, 1.0                                               # ordinary ones beside them
    x = padded(x, 127)
    p = ref.product(x, b, w, a)
    ok = inside(p)
    assert bool(ok.any())
    out = laser.w8_matmul(laser.W8(w, a), x, b, dtype=F32)
    assert ref.product_close(torch.where(ok, out, 0.0), torch.where(ok, p, 0.0))
    assert bool(out[p.abs() > torch.finfo(F32).max * (1 + 2.0 ** -20)].isinf().all())
    low = p.abs() <= 2.0 ** -126
    assert bool(((out.double() - p).abs()[low] <= 2.1 * 2.0 ** -149).all())      # three roundings of 2^-24 above that step, half of it below


@pytest.mark.parametrize("sw, sx", [f for f in FAR if f[0] > 1e-40])      # (rows' scales would pass fp32)
@pytest.mark.parametrize("M, N, Kd", [(1, 40, 200), (9, 100, 1000), (40, 300, 256), (249, 700, 512)])
def test_gates_of_scales_far_apart(M, N, Kd, sw, sx):
    """Gates of some units, and up projections as large."""
    g = gen(M + 1)
    w, a = made(g, 2 * N, Kd)
    x, b = made(g, M, Kd)
    a, b = (a.double() * 1e3 * sw).float(), b.double() * 1e3
    x = padded(x, -128)
    b = (b * (3.0 / (float(a.double().mean()) * Kd ** 0.5 * 73 * 73 * 0.6))).float()
    assert bool(b.isfinite().all()) and float(b.min()) > 0
    o, before = ref.gated(x, b, w, a)
    h = laser.W8(w, a, gated=True)
    for t in (F16, BF16, F32):
        assert ref.gated_close(laser.w8_matmul(h, x, b, dtype=t), o, before), t


def test_scales_of_nothing_and_numbers_that_are_not_finite():
    """Zeros, infinities and NaN among scales, sums of zero beside the largest scales."""
    w = torch.ones((40, 128), dtype=torch.int8, device="cuda")
    w[20:] = 0
    a = torch.tensor([0.0, 1.0, float("inf"), float("nan"), 3e38, 1e-45, -2.0, -0.0] * 5, device="cuda")
    for M in (3, 20, 130):
        x = torch.ones((M, 128), dtype=torch.int8, device="cuda")
        b = torch.tensor([0.0, 1.0, 3e38, 1e-45, -1.0, float("inf"), float("nan")], device="cuda").repeat(M // 7 + 1)[:M].contiguous()
        out = laser.w8_matmul(laser.W8(w, a), x, b, dtype=F32)
        p = ref.product(x, b, w, a)
        want = p.float()
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.isinf(), want.isinf())
        ok = want.isfinite()
        assert bool(((out.double() - p).abs()[ok] <= 3.01 * 2.0 ** -24 * p.abs()[ok] + 2.0 ** -149).all())
