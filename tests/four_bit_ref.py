"""Plain 64-bit forms of the operators on 4-bit caches and weights, and how far a result may be off them."""
import math

import torch

EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative


def quantize(x, group):
    """(codes float64, s fp16, m fp16) of float64 x along its last dimension."""
    g = x.unflatten(-1, (-1, group))
    lo, hi = g.amin(-1), g.amax(-1)
    s = ((hi - lo) / 15).clamp(max=65504.0).float().half()
    m = lo.clamp(-65504.0, 65504.0).float().half()
    sd, md = s.double().unsqueeze(-1), m.double().unsqueeze(-1)
    c = torch.where(sd > 0, ((g - md) / torch.where(sd > 0, sd, 1.0)).round().clamp(0, 15), 0.0)
    return c.flatten(-2), s, m


def values(c, s, m):
    g = c.unflatten(-1, (s.shape[-1], -1))
    return (m.double().unsqueeze(-1) + s.double().unsqueeze(-1) * g).flatten(-2)


def held(x):
    return values(*quantize(x.double(), 32))


def paths(parent, R):
    """Rows that each row of a step sees, from the parents of its nodes (None: a chain); itself last."""
    out = [[0]]
    for i in range(R - 1):
        p = i - 1 if parent is None else int(parent[i])
        if p < -1 or p >= i:
            p = -1
        out.append(out[p + 1] + [i + 1])
    return out


def rotate(x, table, dim, pos):
    """x [R][H][dh] float64 at positions pos [R]."""
    if not dim:
        return x
    t = table.double()[pos].unsqueeze(1)
    co, si = t[..., 0], t[..., 1]
    a, b = x[..., :dim // 2], x[..., dim // 2:dim]
    return torch.cat([a * co - b * si, a * si + b * co, x[..., dim:]], -1)


def attend(q, k, v, len_, see, scale, v_span, k_span, two_planes):
    """q [R][Hq][dh], k, v [len + R][H][dh] (what the cache stands for), all float64; see: paths. -> result and the bound on what
    a kernel may be off it before its last rounding.

    Weights p are rounded to fp16 (half a step 2^-11, two planes 2^-22) before they meet codes and offsets, whose sizes v_span =
    s c + |m| bound: (2^-11 or 2^-21) sum(p v_span) / sum(p). Below fp16's smallest numbers the rounding is absolute, 2^-25 of a weight whose
    largest is 1 or more, for codes up to 15 behind a factor of 16 (or 1/16 where scales pass 511: then 2^-17) and for offsets:
    T 2^-25 (1 + max v_span). Scores are fp32 sums of under 2^6 roundings of terms k_span |q|: 2^-18 of that sum, to the result as twice the
    relative change of the weights."""
    R, Hq, dh = q.shape
    G = Hq // k.shape[1]
    T = len_ + R
    mask = torch.full((R, T), -math.inf, dtype=torch.float64, device=q.device)
    mask[:, :len_] = 0
    for r, rows in enumerate(see):
        mask[r, [len_ + j for j in rows]] = 0
    out, tol = torch.empty_like(q), torch.empty_like(q)
    for h in range(Hq):
        s = q[:, h] @ k[:, h // G].T * scale + mask
        p = (s - s.amax(-1, keepdim=True)).exp()
        n = p.sum(-1, keepdim=True)
        out[:, h] = p @ v[:, h // G] / n
        span = v_span[:, h // G]
        delta = 2.0 ** -18 * abs(scale) * (q[:, h].abs() @ k_span[:, h // G].T).amax(-1, keepdim=True)
        floor = 2.0 ** -25 if float(span.max()) < 15 * 511 else 2.0 ** -17
        tol[:, h] = ((2.0 ** -21 if two_planes else 2.0 ** -11) + 2 * delta) * (p @ span / n) + T * floor * (1 + span.amax())
    return out, tol


def spans(x):
    c, s, m = quantize(x.double(), 32)
    return values(c, s, m.abs())
