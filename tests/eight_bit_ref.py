"""Plain 64-bit forms of the operators on rows and weights in 8-bit integers, and how far a result may be off them."""
import torch

EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -149}  # and below the normal numbers


def quantize(u):
    """(codes, largest magnitudes [M][1], rows that are not finite [M]) of float64 u."""
    bad = ~torch.isfinite(u).all(-1)
    m = u.abs().amax(-1, keepdim=True)
    ok = ((m > 0) & ~bad[:, None])
    c = torch.where(ok, (127 * u / torch.where(ok, m, 1.0)).round(), 0.0)
    return c, m, bad


def rows(x):
    """codes and scales of rows: the scales are one rounding of a quotient, so they are these bit for bit."""
    c, m, bad = quantize(x.double())
    s = (m / 127).float().flatten()
    return c.to(torch.int8), torch.where(bad, torch.nan, s)


def norm(x, gain, eps, res):
    """codes, scales in float64, h in float64."""
    h = x.double() + (0 if res is None else res.double())
    c, m, bad = quantize(h * gain.double())
    bad |= ~torch.isfinite(h).all(-1)
    s = (m / 127 / (h.square().mean(-1, keepdim=True) + eps).sqrt()).flatten()
    s = torch.where(m.flatten() == 0, 0.0, s)
    return torch.where(bad[:, None], 0.0, c).to(torch.int8), torch.where(bad, torch.nan, s), h


def scales_close(got, want):
    """One rounding to fp32 of what 64-bit sums in any order make (2^-40 covers their own)."""
    bound = (2.0 ** -24 + 2.0 ** -40) * want.abs() + 2.0 ** -149
    return bool((((got.double() - want).abs() <= bound) | (got.isnan() & want.isnan())).all())


def values_close(got, codes, scales):
    """s c (exact in 64 bits) rounded to the result's type, either at once or by way of fp32: at most half a step of each."""
    v = scales.double()[:, None] * codes.double()
    e = EPS[got.dtype] + (2.0 ** -24 if got.dtype != torch.float32 else 0)
    return bool(((got.double() - v).abs() <= e * v.abs() + TINY[got.dtype]).all())


def product(x, sx, w, sw):
    """float64 sums of codes (exact) times both scales."""
    return (x.double() @ w.double().T.contiguous()) * sx.double()[:, None] * sw.double()


def product_close(got, p):
    """The sum becomes fp32 (2^-24) and is multiplied twice (2^-24 each), then rounded to the result's type."""
    e = EPS[got.dtype]
    before = 3.01 * 2.0 ** -24 * p.abs()
    err = (got.double() - p).abs()
    return bool((err <= before + e * (p.abs() + before) + TINY[got.dtype]).all())


def gated(x, sx, w, sw):
    """(float64 result, bound on a kernel's error before its last rounding)."""
    p = product(x, sx, w, sw)
    gate, up = p.chunk(2, -1)
    o = gate * torch.sigmoid(gate) * up
    # gate and up are 3 roundings off; silu takes a relative change d of its argument g to at most d (1 + |g|). exp(-g) is 2^(-g log2 e): the product and the
    # constant are a rounding each, absolute in the exponent (2 |g| roundings), its own error a last place, 2 more; a sum (1), a reciprocal within
    # a last place (2), two products (2).
    return o, 2.0 ** -24 * (3 * (1 + gate.abs()) + 3 + 2 * gate.abs() + 2 + 5) * o.abs() + 2.0 ** -110 * up.abs()


def gated_close(got, o, before):
    e = EPS[got.dtype]
    return bool(((got.double() - o).abs() <= before + e * (o.abs() + before) + TINY[got.dtype]).all())
