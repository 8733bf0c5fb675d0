"""Products of rows in which one activation is far larger than the others."""
import pytest
import torch

import paper_2408_05676_amd as laser
from tests import four_bit_ref as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("M", [1, 3, 9, 40, 100])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_with_one_large_activation(M, group, dtype):
    """The weights that it meets stand for little, so that the results are of the size that the others make: the bound is that of fp32 sums, as for
    other rows: two roundings a group and some sixty within it and at the joints."""
    gen = torch.Generator(device="cuda").manual_seed(M + group)
    N, Kd, at = 512, 512, 77
    w = torch.empty((N, Kd), device="cuda").normal_(0, 0.05, generator=gen)
    w[:, at] = 0
    codes, s, m = laser.w4_quantize(w.bfloat16(), group)
    x = torch.empty((M, Kd), device="cuda").normal_(0, 1, generator=gen)
    x[:, at] = 3000.0
    x = x.to(dtype)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(1).double()
    want, got = x.double() @ ref.values(c, s, m).T, laser.w4_matmul(laser.W4(codes, s, m), x).double()
    size = x.double().abs() @ (ref.values(c, s, m.abs()) + (256 * s.double().repeat_interleave(group, 1) if dtype == BF16 else 0)).T
    tol = (2 * Kd / group + 64) * 2.0 ** -24 * size
    bound = tol + ref.EPS[dtype] * (want.abs() + tol) + (2.0 ** -25 if dtype == F16 else 0)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
    # in the mean: an eighth of that and the last rounding
    rms = lambda t: float(t.square().mean().sqrt())  # noqa: E731
    rounding = rms(want.to(dtype).double() - want)
    assert rms(got - want) <= rounding + rms(tol) / 8, (rms(got - want) / rounding, rms(tol) / rounding)
