"""Every kernel of the operators on rows and weights in 8-bit integers, also those that sizes of the other tests do not reach."""
import pytest
import torch

import paper_2408_05676_amd as laser
from tests import eight_bit_ref as ref
from tests.eight_bit_shapes import GATED, PLAIN
from tests.test_gpu_eight_bit import activations, gen, made, normal, padded

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def framed(M, N, dtype):
    """([M][N] inside a larger tensor, a check that the rest of that is as it was)."""
    buf = torch.full((M + 2, N + 13), 9.0, dtype=dtype, device="cuda")
    out = buf[1:M + 1, 5:5 + N]

    def untouched():
        out.fill_(9)
        return bool((buf == 9).all())
    return out, untouched


@pytest.mark.parametrize("M, N, Kd", PLAIN)
def test_products(M, N, Kd):
    g = gen(M + N + Kd)
    w, sw = made(g, N, Kd)
    x, sx = made(g, M, Kd)
    x = padded(x, 127)
    p = ref.product(x, sx, w, sw)
    h = laser.W8(w, sw)
    for t in (F16, BF16, F32):
        out, untouched = framed(M, N, t)
        laser.w8_matmul(h, x, sx, out=out)
        assert ref.product_close(out, p), t
        whole = laser.w8_matmul(h, x, sx, dtype=t)
        assert torch.equal(out, whole) and untouched()


@pytest.mark.parametrize("M, N, Kd", GATED)
def test_gated_products(M, N, Kd):
    g = gen(M + N + Kd + 1)
    w, sw = made(g, 2 * N, Kd)
    x, sx = made(g, M, Kd)
    x, sx = padded(x, -128), sx * (3.0 / (Kd ** 0.5 * 73 * 73 * 5.5e-4 * 6e-4))  # gates of some units
    o, before = ref.gated(x, sx, w, sw)
    h = laser.W8(w, sw, gated=True)
    for t in (F16, BF16, F32):
        out, untouched = framed(M, N, t)
        laser.w8_matmul(h, x, sx, out=out)
        assert ref.gated_close(out, o, before), t
        whole = laser.w8_matmul(h, x, sx, dtype=t)
        assert torch.equal(out, whole) and untouched()


# more than 256 rows, by their lengths: one wave, four, eight with one to three pieces a thread, sixteen with two and four, and those that are read twice
MANY = [(257, 505), (300, 2041), (300, 2049), (704, 4096), (257, 4095), (300, 4097), (300, 8191), (300, 8193), (704, 11008), (257, 12281), (257, 12290), (257, 16383), (257, 16386),
        (257, 32761), (257, 32770)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M, N", MANY)
def test_many_rows(M, N, dtype):
    x = activations(gen(M + N), M, N, dtype)
    codes, scales = laser.q8_rows(x)
    c, s = ref.rows(x)
    assert torch.equal(codes, c) and torch.equal(scales, s)
    for t in (F16, BF16, F32):
        assert ref.values_close(laser.q8_read(codes, scales, dtype=t), codes, scales)


@pytest.mark.parametrize("dtype, res", [(F16, None), (F16, F16), (F16, F32), (BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)])
@pytest.mark.parametrize("M, N", MANY)
def test_norms_of_many_rows(M, N, dtype, res):
    g = gen(M + N + 1)
    x, gain = activations(g, M, N, dtype), 1 + 0.1 * normal(g, N)
    r = activations(g, M, N, res) if res else None
    c, s, h = ref.norm(x, gain, 1e-6, r)
    out = None if r is None else torch.empty_like(r)
    codes, scales = laser.q8_norm(x, gain, 1e-6, residual=r, residual_out=out)
    assert torch.equal(codes, c) and ref.scales_close(scales, s)
    if r is None:
        return
    total = h.float().to(res)
    assert torch.equal(out, total)
    for to in ("r", "x") if dtype == res else ("r",):                          # the sum in the residual's place, and in x's
        x2, r2 = x.clone(), r.clone()
        again, s2 = laser.q8_norm(x2, gain, 1e-6, residual=r2, residual_out=r2 if to == "r" else x2)
        assert torch.equal(again, codes) and torch.equal(s2, scales)
        assert torch.equal(r2 if to == "r" else x2, total) and torch.equal(x2 if to == "r" else r2, x if to == "r" else r)


def test_norm_in_place_past_32_bits():
    """The sum over x itself, 300000 rows of 8192 in bf16 (4.9 GB): codes, scales and sums of the first and last rows and of those where a byte offset passes 2^31 and 2^32."""
    g = gen(40)
    M, N = 300000, 8192
    x = torch.empty((M, N), dtype=BF16, device="cuda").normal_(0, 1, generator=g)
    gain = 1 + 0.1 * normal(g, N)
    at = [0, 1, M - 2, M - 1] + [b // (2 * N) + d for b in (2 ** 31, 2 ** 32) for d in (-1, 0, 1)] + [b // N + d for b in (2 ** 31,) for d in (-1, 0, 1)]
    at = torch.tensor(sorted(at), device="cuda")
    was = x[at].clone()
    codes, scales = laser.q8_norm(x, gain, residual=x)
    c, s, h = ref.norm(was, gain, 1e-6, was)
    assert torch.equal(codes[at], c) and ref.scales_close(scales[at], s) and torch.equal(x[at], h.float().to(BF16))
    values = laser.q8_read(codes, scales, dtype=BF16, out=x)
    assert ref.values_close(values[at], codes[at], scales[at])
