"""Operators on rows and weights held in 8-bit integers, as measurable cases.

  rows     rows put into 8 bits with a scale each (laser.q8_rows), and the values they stand for (laser.q8_read)
  norm     the residual's addition, the root-mean-square norm and the same 8 bits in one pass (laser.q8_norm), and the values
  product  such rows times a matrix of 8-bit weights with a scale for every output (laser.w8_matmul)
  gated    the same with a gate and an up matrix: silu(gate) * up (laser.w8_matmul with a gated W8)

Eight bits: codes c in -127..127 and one fp32 scale s for a row of activations or of weights; an element stands for s c, the row's
largest magnitude for 127 s. c = 127 x / max|x| rounded to nearest even.
"""
from __future__ import annotations

import math

import torch

own = False            # True: run() calls the framework's operators; False: plain torch operations

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
PAD = 128              # rows of codes start at multiples of this many bytes


def listed():
    return [
        # the FFN activation of a throughput step (64 users, chains of 10 drafts) on its way into the down projection, 7B width
        dict(name="rows_7b_m704", kind="rows", M=704, d=11008, dtype="f16"),
        # attention's result of a single token, 7B width: latency is all there is
        dict(name="rows_7b_m1", kind="rows", M=1, d=4096, dtype="bf16"),
        # two users' verify steps of the two-layer model
        dict(name="norm_tiny_m10", kind="norm", M=10, d=256, dtype="f16", residual="f16"),
        # verify steps of eight users at the 1B width, residual stream in fp32
        dict(name="norm_1b_m72", kind="norm", M=72, d=2048, dtype="bf16", residual="f32"),
        # a throughput step at the 7B width
        dict(name="norm_7b_m704", kind="norm", M=704, d=4096, dtype="bf16", residual="bf16"),
        # the smallest product: fused query/key/value projection of two users, two-layer model
        dict(name="product_tiny_m2", kind="product", M=2, N=768, Kd=256, dtype="f16"),
        # a verify step of one user (8 drafts), down projection
        dict(name="product_7b_down_m9", kind="product", M=9, N=4096, Kd=11008, dtype="f16"),
        # verify steps of eight users, query/key/value projection at the 1B width
        dict(name="product_1b_qkv_m72", kind="product", M=72, N=6144, Kd=2048, dtype="bf16"),
        # a throughput step, query/key/value projection at the 7B width
        dict(name="product_7b_qkv_m704", kind="product", M=704, N=12288, Kd=4096, dtype="f16"),
        # plain decoding of one user, gate and up projection at the 7B width
        dict(name="gated_7b_m1", kind="gated", M=1, N=11008, Kd=4096, dtype="f16"),
        # pieces of prompts, gate and up projection at the 1B width; odd number of rows
        dict(name="gated_1b_m249", kind="gated", M=249, N=5632, Kd=2048, dtype="bf16"),
        # a throughput step, gate and up projection at the 7B width
        dict(name="gated_7b_m704", kind="gated", M=704, N=11008, Kd=4096, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rows", "norm", "product", "product", "gated"])
    dtype = rng.choice(["f16", "bf16"])
    if kind in ("rows", "norm"):
        # no more elements than the listed throughput steps have
        d = _log_int(rng, 64, 11008 if kind == "rows" else 8192)
        M = min(_log_int(rng, 1, 1024), 704 * (11008 if kind == "rows" else 4096) // d)
        case = dict(kind=kind, M=M, d=d, dtype=dtype)
        if kind == "norm":
            case["residual"] = rng.choice(["f32", dtype, "none"])
        return case
    Kd = rng.choice([_log_int(rng, 64, 11008), 128 * _log_int(rng, 1, 86)])
    N = _log_int(rng, 100, 12288 if kind == "product" else 11008)
    N = min(N, (12288 if kind == "product" else 11008) * 4096 // Kd)
    M = min(_log_int(rng, 1, 1024), 704 * (12288 if kind == "product" else 11008) * 4096 // (N * Kd))
    return dict(kind=kind, M=M, N=N, Kd=Kd, dtype=dtype)


def work(case):
    M = case["M"]
    if case["kind"] in ("rows", "norm"):
        d, b = case["d"], 2
        if case["kind"] == "rows":
            return dict(bytes=M * d * (b + 1 + b) + 4 * M, flops=4 * M * d)
        r = 0 if case["residual"] == "none" else 4 if case["residual"] == "f32" else 2
        return dict(bytes=M * d * (b + 2 * r + 1 + b) + 4 * (M + d), flops=8 * M * d)
    N, Kd, two = case["N"], case["Kd"], 2 if case["kind"] == "gated" else 1
    return dict(bytes=two * N * Kd + M * Kd + 2 * M * N + 4 * (M + two * N), flops=2 * two * M * N * Kd)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *dims):
    return torch.empty(dims, device="cuda").normal_(0.0, 1.0, generator=gen)


def _activations(gen, M, d):
    """Rows of different sizes, with channels that are larger than the others in every row, as in trained models."""
    return _normal(gen, M, d) * torch.exp(0.6 * _normal(gen, d)) * torch.exp(0.3 * _normal(gen, M, 1))


def _codes(u):
    """(codes float64, largest magnitudes [..., 1]) of float64 u along its last dimension."""
    m = u.abs().amax(-1, keepdim=True)
    return (127 * u / torch.where(m > 0, m, 1.0)).round(), m


def _padded(codes):
    """Codes as the operators lay them out: rows that start at multiples of PAD bytes."""
    M, K = codes.shape
    t = torch.zeros((M, -(-K // PAD) * PAD), dtype=torch.int8, device="cuda")
    t[:, :K] = codes
    return t[:, :K]


def prepare(case, seed):
    gen = _gen(seed)
    dt = DTYPES[case["dtype"]]
    M = case["M"]
    st = dict(case=case)
    if case["kind"] in ("rows", "norm"):
        d = case["d"]
        st["x"] = _activations(gen, M, d).to(dt)
        st["codes"] = _padded(torch.zeros((M, d), device="cuda"))
        st["scales"] = torch.zeros(M, device="cuda")
        st["out"] = torch.zeros((M, d), dtype=dt, device="cuda")
        if case["kind"] == "norm":
            st["gain"] = 1.0 + 0.1 * _normal(gen, d)
            st["r"] = st["r_out"] = None
            if case["residual"] != "none":
                st["r"] = (4.0 * _activations(gen, M, d)).to(DTYPES[case["residual"]])
                st["r_out"] = torch.zeros_like(st["r"])
        return st
    N, Kd, gated = case["N"], case["Kd"], case["kind"] == "gated"
    c, m = _codes(_activations(gen, M, Kd).double())
    st["x"], st["s"] = _padded(c), (m / 127).float().flatten()
    rows = 2 * N if gated else N
    st["w"], st["ws"] = torch.empty((rows, Kd), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    for lo in range(0, rows, 4096):
        c, m = _codes((0.02 * _normal(gen, min(4096, rows - lo), Kd)).to(torch.bfloat16).double())
        st["w"][lo:lo + 4096], st["ws"][lo:lo + 4096] = c, (m / 127).float().flatten()
    st["out"] = torch.zeros((M, N), dtype=dt, device="cuda")
    if own:
        import paper_2408_05676_amd as laser
        st["w8"] = laser.W8(st["w"], st["ws"], gated=gated)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if own:
        import paper_2408_05676_amd as laser
        if kind in ("product", "gated"):
            return laser.w8_matmul(st["w8"], st["x"], st["s"], out=st["out"])
        if kind == "rows":
            q = laser.q8_rows(st["x"], out=(st["codes"], st["scales"]))
            return laser.q8_read(*q, out=st["out"])
        q = laser.q8_norm(st["x"], st["gain"], EPS, residual=st["r"], residual_out=st["r_out"], out=(st["codes"], st["scales"]))
        values = laser.q8_read(*q, out=st["out"])
        return values if st["r"] is None else (values, st["r_out"])
    if kind in ("product", "gated"):
        acc = st["x"].float() @ st["w"].float().T
        o = acc * st["s"][:, None] * st["ws"]
        if kind == "gated":
            gate, up = o.chunk(2, -1)
            o = gate / (1 + (-gate).exp()) * up
        return o.to(st["out"].dtype)
    # codes in 64 bits: a value half-way between two of them falls to one side or the other by its last bits
    if kind == "rows":
        c, m = _codes(st["x"].double())
        return (c.float() * (m / 127).float()).to(st["x"].dtype)
    h = st["x"].double() + (0 if st["r"] is None else st["r"].double())
    c, m = _codes(h * st["gain"].double())
    s = (m / 127 / (h.square().mean(-1, keepdim=True) + EPS).sqrt()).float()
    values = (c.float() * s).to(st["x"].dtype)
    return values if st["r"] is None else (values, h.to(st["r"].dtype))


# ------------------------------------------------------------------------------------------------ in 64 bits, from the definitions
def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64

    def held(u, factor):
        """What a row's codes stand for: multiples of a 127th of its largest magnitude."""
        top = torch.linalg.vector_norm(u, math.inf, dim=1)
        n = torch.round(torch.div(torch.mul(u, 127), top.clamp(min=1e-300).unsqueeze(1)))
        return n * (top / 127 * factor).unsqueeze(1)

    if case["kind"] in ("product", "gated"):
        # row by row of scales: diag(s) X W^T diag(w), the integers' products in 64 bits
        full = torch.mm(st["x"].to(f64) * st["s"].to(f64).unsqueeze(1), st["w"].to(f64).t().contiguous()).mul_(st["ws"].to(f64))
        if case["kind"] == "product":
            return full
        F = case["N"]
        return torch.sigmoid(full[:, :F]) * full[:, :F] * full[:, F:]
    x = st["x"].to(f64)
    if case["kind"] == "rows":
        return held(x, 1.0)
    if st["r"] is not None:
        x = torch.add(x, st["r"].to(f64))
    rms = (torch.linalg.vector_norm(x, dim=1).square() / case["d"] + EPS).sqrt()
    values = held(x * st["gain"].to(f64), 1 / rms)
    return values if st["r"] is None else (values, x)
