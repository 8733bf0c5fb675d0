"""Operators on weights and caches held in four bits, as measurable cases.

  product  rows times a matrix of 4-bit weights with group scales (laser.w4_matmul)
  append   a step's keys and values into a paged 4-bit cache, rotary positions applied on the way (laser.kv_append)
  attend   attention of a step's rows over such a cache: single tokens, draft chains, token trees (laser.kv_attend)

Four bits: codes c in 0..15 with a scale s and an offset m in fp16 for every group of consecutive elements; an element stands for
m + s c. Cache groups are 32 channels of one token and head; weight groups are 32, 64 or 128 inputs of one output.
"""
from __future__ import annotations

import math

import torch

own = False            # True: run() calls the framework's operators; False: plain torch operations

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
GROUP = 32             # channels of a token and head that share a scale in the cache
PAGE = 16              # tokens per cache page


def listed():
    return [
        # smallest calls, where latency is all there is: the two-layer model's fused query/key/value projection of two users
        dict(name="product_tiny_m2", kind="product", N=768, Kd=256, M=2, group=32, dtype="f16"),
        # plain decoding of one user, gate/up projection at the 7B width
        dict(name="product_7b_gateup_m1", kind="product", N=22016, Kd=4096, M=1, group=128, dtype="bf16"),
        # a verify step of one user (8 drafts), down projection
        dict(name="product_7b_down_m9", kind="product", N=4096, Kd=11008, M=9, group=64, dtype="f16"),
        # verify steps of eight users, 72 rows, query/key/value projection at the 1B width
        dict(name="product_1b_qkv_m72", kind="product", N=6144, Kd=2048, M=72, group=128, dtype="bf16"),
        # two users' verify steps of the two-layer model
        dict(name="append_tiny_b2_r5", kind="append", B=2, R=5, kv_heads=4, per_kv=1, dh=64, ctx=64, dtype="f16", tree=False),
        # plain decoding of 64 users, one token each, a layer at the 7B width
        dict(name="append_7b_b64_r1", kind="append", B=64, R=1, kv_heads=32, per_kv=1, dh=128, ctx=512, dtype="bf16", tree=False),
        # prompts in pieces of 64 rows, grouped heads
        dict(name="append_prompt_b16_r64", kind="append", B=16, R=64, kv_heads=8, per_kv=4, dh=128, ctx=1000, dtype="bf16", tree=False),
        # a token tree over a short cache, the two-layer model
        dict(name="attend_tiny_tree_b2_r5", kind="attend", B=2, R=5, kv_heads=4, per_kv=1, dh=64, ctx=64, dtype="f16", tree=True),
        # the latency workload: one user, chain of 8 drafts, context 1024
        dict(name="attend_7b_b1_r9", kind="attend", B=1, R=9, kv_heads=32, per_kv=1, dh=128, ctx=1024, dtype="f16", tree=False),
        # plain decoding of one user far into a long text, grouped heads
        dict(name="attend_long_b1_r1", kind="attend", B=1, R=1, kv_heads=8, per_kv=4, dh=128, ctx=65000, dtype="bf16", tree=False),
        # the throughput workload: 64 users, chains of 10, contexts up to 512
        dict(name="attend_7b_b64_r11", kind="attend", B=64, R=11, kv_heads=32, per_kv=1, dh=128, ctx=512, dtype="bf16", tree=False),
        # pieces of 64 prompt rows behind a long text, grouped heads: 256 query rows per key/value head
        dict(name="attend_prompt_b4_r64", kind="attend", B=4, R=64, kv_heads=8, per_kv=4, dh=128, ctx=8000, dtype="bf16", tree=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["product", "append", "attend"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "product":
        group = rng.choice([32, 64, 128])
        N, Kd = _log_int(rng, 200, 22016), 128 * _log_int(rng, 2, 86)
        # no more weights than the largest listed matrix, no more products than the listed 72 rows take
        N = min(N, 22016 * 4096 // Kd)
        M = max(1, min(_log_int(rng, 1, 80), 72 * 6144 * 2048 // (N * Kd)))
        return dict(kind=kind, N=N, Kd=Kd, M=M, group=group, dtype=dtype)
    dh = rng.choice([64, 128, 128])
    kv_heads, per_kv = rng.choice([(4, 1), (16, 1), (32, 1), (8, 4), (8, 8), (2, 5), (3, 7)])
    tree = rng.random() < 0.3
    R = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 2, 17)])
    if kind == "append":
        B = max(1, min(_log_int(rng, 1, 200), 16 * 64 * 48 // (R * kv_heads * (per_kv + 2))))
        return dict(kind=kind, B=B, R=R, kv_heads=kv_heads, per_kv=per_kv, dh=dh, ctx=_log_int(rng, 1, 2000), dtype=dtype, tree=tree and R > 1)
    B, ctx = _log_int(rng, 1, 64), _log_int(rng, 1, 65000)
    # no more cached tokens than the listed 64 users hold, no more scores than the listed prompts have
    ctx = max(1, min(ctx, 64 * 512 * 32 // (B * kv_heads), 4 * 64 * 32 * 8000 // (B * R * kv_heads * per_kv)))
    return dict(kind=kind, B=B, R=R, kv_heads=kv_heads, per_kv=per_kv, dh=dh, ctx=ctx, dtype=dtype, tree=tree and R > 1)


def work(case):
    if case["kind"] == "product":
        N, Kd, M = case["N"], case["Kd"], case["M"]
        return dict(bytes=N * Kd // 2 + 4 * N * (Kd // case["group"]) + 2 * M * (Kd + N), flops=2 * M * N * Kd)
    B, R, H, dh = case["B"], case["R"], case["kv_heads"], case["dh"]
    Hq, packed = H * case["per_kv"], 2 * H * dh * 5 // 8          # bytes of a token's keys and values in the cache
    if case["kind"] == "append":
        # rows and their positions' (cos, sin) in; rotated queries and packed rows out; the values they stand for
        return dict(bytes=B * R * (2 * dh * (2 * Hq + 2 * H) + 4 * dh + packed + 4 * H * dh), flops=B * R * dh * (3 * (Hq + H) + 8 * H))
    tokens = int(B * case["ctx"] * (1.0 if B == 1 else 0.875)) + B * R
    return dict(bytes=tokens * packed + 4 * B * R * Hq * dh, flops=4 * R * Hq * dh * tokens)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *dims):
    return torch.empty(dims, device="cuda").normal_(0.0, 1.0, generator=gen)


def _quantize(x, group):
    """(codes uint8, scales fp16, offsets fp16) of float64 x, groups along the last dimension."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // group, group)
    lo, hi = g.amin(-1), g.amax(-1)
    s, m = ((hi - lo) / 15).float().half(), lo.float().half()
    sd = s.double().unsqueeze(-1)
    c = ((g - m.double().unsqueeze(-1)) / torch.where(sd > 0, sd, 1.0)).round().clamp(0, 15) * (sd > 0)
    return c.to(torch.uint8).reshape(x.shape), s, m


def _values(codes, s, m):
    """What codes, scales and offsets stand for, in float32 (exact: 4 + 11 bits, one rounding of the sum)."""
    g = codes.reshape(*s.shape, codes.shape[-1] // s.shape[-1]).float()
    return (m.float().unsqueeze(-1) + s.float().unsqueeze(-1) * g).reshape(codes.shape)


def _heads(gen, scale, *dims):
    """Keys, values or queries: a few channels of each head are larger than the others, as in trained models."""
    channel = torch.exp(0.5 * _normal(gen, *dims[-2:]))
    return _normal(gen, *dims) * channel * scale


def _rope_table(max_pos, dim):
    angle = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def _lens(gen, case):
    """Running texts have different lengths: the named context is the longest."""
    n = case["ctx"] - torch.randint(0, max(1, case["ctx"] // 4), (case["B"],), generator=gen, device="cuda")
    n[0] = case["ctx"]
    return n.to(torch.int32)


def _parents(gen, B, K):
    """Token trees: a node hangs off the pending token (-1) or off an earlier node, the last ones more often."""
    back = torch.empty((B, K), device="cuda").exponential_(0.7, generator=gen).long() + 1
    return (torch.arange(K, device="cuda") - back).clamp(min=-1).to(torch.int32)


def prepare(case, seed):
    gen = _gen(seed)
    dt = DTYPES[case["dtype"]]
    st = dict(case=case)
    if case["kind"] == "product":
        N, Kd, G = case["N"], case["Kd"], case["group"]
        st["codes"], st["s"], st["m"] = _quantize((0.02 * _normal(gen, N, Kd)).double(), G)
        packed = st["codes"].reshape(N, Kd // 2, 2)
        st["packed"] = packed[..., 0] | (packed[..., 1] << 4)
        st["x"] = _normal(gen, case["M"], Kd).to(dt)
        st["out"] = torch.zeros((case["M"], N), dtype=dt, device="cuda")
        if own:
            import paper_2408_05676_amd as laser
            st["w"] = laser.W4(st["packed"], st["s"], st["m"])
        return st
    B, R, H, G, dh = (case[n] for n in ("B", "R", "kv_heads", "per_kv", "dh"))
    st["lens"], st["ids"] = _lens(gen, case), list(range(B))
    st["parent"] = _parents(gen, B, R - 1) if case["tree"] else None
    st["q"] = _heads(gen, 1.0, B, R, H * G, dh).to(dt)
    st["out"] = torch.zeros((B, R, H * G, dh), dtype=dt, device="cuda")
    rows = R if case["kind"] == "append" else int(st["lens"].max()) + R
    k, v = _heads(gen, 1.0, B, rows, H, dh), _heads(gen, 0.5, B, rows, H, dh)
    if case["kind"] == "append":
        st["k"], st["v"], st["table"] = k.to(dt), v.to(dt), _rope_table(case["ctx"] + R, dh)
        st["values"] = tuple(torch.zeros((B, R, H, dh), dtype=torch.float16, device="cuda") for _ in range(2))
    else:
        k, v = k.half(), v.half()
        st["cache"] = (*_quantize(k.double(), GROUP), *_quantize(v.double(), GROUP))
    if own:
        import paper_2408_05676_amd as laser
        pages = -(-(case["ctx"] + R) // PAGE)
        st["kv"] = kv = laser.KVCache4(1, H, dh, B * pages, B, pages)
        for b, n in enumerate(st["lens"].tolist()):
            kv.reserve(b, n + R)
            if case["kind"] == "attend":
                kv.import_layer(b, 0, k[b, :n + R].contiguous(), v[b, :n + R].contiguous())
            kv.set_len(b, n)
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    kind = state["case"]["kind"]
    return _run_product(state) if kind == "product" else _run_append(state) if kind == "append" else _run_attend(state)


def _run_product(st):
    if own:
        import paper_2408_05676_amd as laser
        return laser.w4_matmul(st["w"], st["x"], out=st["out"])
    return (st["x"].float() @ _values(st["codes"], st["s"], st["m"]).T).to(st["x"].dtype)


def _visible(parent, B, R):
    """[B][R][R]: whether row i attends to row j of its own step: row 0 is the pending token, row 1 + i node i of the tree
    (None: a chain). A row sees itself and its ancestors."""
    if parent is None:
        return torch.ones((R, R), device="cuda").tril().bool().expand(B, R, R)
    up = torch.zeros((B, R, R), dtype=torch.float64, device="cuda")
    up[:, 1:] = torch.nn.functional.one_hot(parent.long() + 1, R)
    return torch.linalg.matrix_power(up + torch.eye(R, dtype=torch.float64, device="cuda"), R) > 0


def _rotate(x, angle):
    """x [B][R][H][dh] in float64, angle [B][R][dh/2][2]: channel i is paired with channel i + dh/2."""
    a, b = x.chunk(2, -1)
    co, si = angle[..., 0].unsqueeze(2), angle[..., 1].unsqueeze(2)
    return torch.cat([a * co - b * si, a * si + b * co], -1)


def _run_append(st):
    if own:
        import paper_2408_05676_amd as laser
        q = laser.kv_append(st["kv"], 0, st["ids"], st["k"], st["v"], q=st["q"], rope=st["table"], tree_parent=st["parent"], q_out=st["out"])
        return (q, *laser.kv_read(st["kv"], 0, st["ids"], st["q"].shape[1], out=st["values"]))
    B, R = st["q"].shape[:2]
    depth = _visible(st["parent"], B, R).sum(-1) - 1
    angle = st["table"][st["lens"].long()[:, None] + depth].double()
    # in 64 bits: a value half-way between two codes falls to one side or the other by its last bits
    k = _values(*_quantize(_rotate(st["k"].double(), angle), GROUP))
    v = _values(*_quantize(st["v"].double(), GROUP))
    return _rotate(st["q"].double(), angle).to(st["q"].dtype), k.half(), v.half()


def _run_attend(st):
    if own:
        import paper_2408_05676_amd as laser
        return laser.kv_attend(st["kv"], 0, st["ids"], st["q"], tree_parent=st["parent"], out=st["out"])
    kc, ks, km, vc, vs, vm = st["cache"]
    B, R, Hq, dh = st["q"].shape
    T, H = kc.shape[1], kc.shape[2]
    k, v = _values(kc, ks, km).permute(0, 2, 3, 1), _values(vc, vs, vm).permute(0, 2, 1, 3)
    q = st["q"].float().reshape(B, R, H, Hq // H, dh).permute(0, 2, 3, 1, 4).reshape(B, H, Hq // H * R, dh)
    s = (q @ k.contiguous()).reshape(B, H, Hq // H, R, T) * dh ** -0.5
    slot = torch.arange(T, device="cuda") - st["lens"].long()[:, None]                       # [B][T], 0 .. R-1: the step's rows
    seen = _visible(st["parent"], B, R).gather(2, slot.clamp(0, R - 1)[:, None].expand(B, R, T)) & (slot < R)[:, None] | (slot < 0)[:, None]
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    p = (s - s.amax(-1, keepdim=True)).exp()
    o = (p.reshape(B, H, -1, T) @ v.contiguous()).reshape(B, H, Hq // H, R, dh) / p.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4).reshape(B, R, Hq, dh).to(st["q"].dtype)


# ------------------------------------------------------------------------------------------------ in 64 bits, from the definitions
def _depths(parent, B, R):
    if parent is None:
        return [[list(range(r + 1)) for r in range(R)] for _ in range(B)]
    paths = []
    for p in parent.tolist():
        rows = [[0]]
        for i, up in enumerate(p):
            rows.append(rows[up + 1] + [i + 1])
        paths.append(rows)
    return paths


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    if case["kind"] == "product":
        G = case["group"]
        s, m = st["s"].to(f64).repeat_interleave(G, 1), st["m"].to(f64).repeat_interleave(G, 1)
        return torch.mm(st["x"].to(f64), torch.addcmul(m, s, st["codes"].to(f64)).t())
    B, R, H, G, dh = (case[n] for n in ("B", "R", "kv_heads", "per_kv", "dh"))
    paths, lens = _depths(st["parent"], B, R), st["lens"].tolist()
    if case["kind"] == "append":
        pos = torch.tensor([[lens[b] + len(paths[b][r]) - 1 for r in range(R)] for b in range(B)], device="cuda")
        z = torch.view_as_complex(st["table"].to(f64))[pos][:, :, None]                      # e^(i angle)
        turn = lambda x: torch.view_as_real(torch.complex(x[..., :dh // 2], x[..., dh // 2:]) * z)  # noqa: E731

        def held(x):
            x = x.unflatten(-1, (-1, GROUP))
            low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            step, low = ((high - low) / 15).to(torch.float32).to(torch.float16).to(f64), low.to(torch.float32).to(torch.float16).to(f64)
            n = torch.where(step > 0, torch.round((x - low) / step.clamp(min=1e-30)), 0.0)
            return (low + step * n.clamp(0, 15)).flatten(-2)

        q, k = (torch.cat(turn(st[n].to(f64)).unbind(-1), -1) for n in ("q", "k"))
        return q, held(k), held(st["v"].to(f64))
    if B * R * H * G * (case["ctx"] + R) > 1 << 31:
        return None
    kc, ks, km, vc, vs, vm = st["cache"]
    out = torch.zeros((B, R, H * G, dh), dtype=f64, device="cuda")
    for b in range(B):
        n = lens[b] + R
        k, v = (torch.addcmul(o[b, :n].to(f64)[..., None], t[b, :n].to(f64)[..., None], c[b, :n].to(f64).unflatten(-1, (-1, GROUP))).flatten(-2)
                for c, t, o in ((kc, ks, km), (vc, vs, vm)))
        bias = torch.full((R, n), -math.inf, dtype=f64, device="cuda")
        bias[:, :lens[b]] = 0
        for r in range(R):
            bias[r, [lens[b] + j for j in paths[b][r]]] = 0
        for h in range(H * G):
            w = torch.softmax(torch.mm(st["q"][b, :, h].to(f64), k[:, h // G].t()) / math.sqrt(dh) + bias, -1)
            out[b, :, h] = torch.mm(w, v[:, h // G])
    return out
