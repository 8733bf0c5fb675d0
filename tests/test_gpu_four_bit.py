"""The 4-bit cache (append, attend, read, commit, use by the model) and products with 4-bit weights against plain 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2408_05676_amd as laser
from tests import four_bit_ref as ref

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *dims, dtype=F32, scale=1.0):
    return (torch.empty(dims, device="cuda").normal_(0, 1, generator=g) * scale).to(dtype)


def make_kv(n, H, dh, lens, extra, layers=1):
    pages = [-(-(t + extra) // 16) for t in lens]
    kv = laser.KVCache4(layers, H, dh, sum(pages) + 2, n, max(pages))
    order = np.random.default_rng(5).permutation(n)              # pages of a sequence need not lie side by side
    for part in (0.5, 1.0):
        for b in order:
            kv.reserve(int(b), int((lens[b] + extra) * part))
    return kv


def fill(kv, lens, H, dh, g, layer=0, scale=1.0):
    """Imported tokens; returns what the cache stands for, and the spans, as float64 [T][H][dh] per sequence."""
    ks, vs = [], []
    for b, n in enumerate(lens):
        k, v = normal(g, n, H, dh, dtype=F16, scale=scale), normal(g, n, H, dh, dtype=F16, scale=scale)
        kv.import_layer(b, layer, k, v)
        kv.set_len(b, n)
        ks.append(k.double())
        vs.append(v.double())
    return ks, vs


def cat_steps(cached, new):
    return torch.cat([cached, new]) if cached.shape[0] else new


def check_attend(kv, lens, ks, vs, new_k, new_v, q, parent, n_rows, scale, got, before, two_planes):
    for b, n in enumerate(lens):
        R = q.shape[1] if n_rows is None else max(0, min(int(n_rows[b]), q.shape[1]))
        if R < q.shape[1]:
            assert torch.equal(got[b, R:], before[b, R:])
        if R == 0:
            continue
        see = ref.paths(None if parent is None else parent[b].tolist(), R)
        k, v = cat_steps(ks[b], new_k[b, :R]), cat_steps(vs[b], new_v[b, :R])
        want, tol = ref.attend(q[b, :R].double(), ref.held(k), ref.held(v), n, see, scale, ref.spans(v), ref.spans(k), two_planes)
        err = (got[b, :R].double() - want).abs()
        bound = tol + ref.EPS[q.dtype] * (want.abs() + tol)
        assert bool((err <= bound).all()), (b, n, float((err / bound).max()))


CASES = [
    # B, R, H, G, dh, dtype, lens, tree
    (1, 1, 1, 1, 64, F16, [0], False),
    (1, 1, 2, 1, 128, BF16, [1], False),
    (3, 1, 2, 4, 128, F16, [15, 16, 17], False),
    (3, 5, 4, 1, 64, BF16, [31, 0, 33], True),
    (2, 9, 2, 5, 128, F16, [127, 128], True),
    (4, 2, 3, 7, 128, BF16, [129, 250, 511, 12], False),
    (2, 64, 2, 1, 128, F16, [0, 40], True),
    (2, 64, 1, 8, 64, BF16, [100, 3], False),
    (1, 17, 2, 4, 128, F32, [300], True),
    (1, 1, 2, 8, 64, F32, [1000], False),
    (1, 11, 32, 1, 128, F16, [1030], False),
    (1, 1, 8, 4, 128, F16, [9000], False),
    (2, 33, 8, 4, 128, BF16, [700, 1500], False),
]


@pytest.mark.parametrize("B, R, H, G, dh, dtype, lens, tree", CASES)
def test_append_read_attend(B, R, H, G, dh, dtype, lens, tree):
    g = gen(len(lens) + R)
    kv = make_kv(B, H, dh, lens, R)
    ks, vs = fill(kv, lens, H, dh, g)
    table = laser.rope_table(max(lens) + R, dh)
    q, k, v = normal(g, B, R, H * G, dh, dtype=dtype), normal(g, B, R, H, dh, dtype=dtype), normal(g, B, R, H, dh, dtype=dtype)
    parent = None
    if tree:
        parent = (torch.rand((B, R - 1), device="cuda", generator=g) * (torch.arange(R - 1, device="cuda") + 1)).int() - 1
    ids = list(range(B))
    qr = laser.kv_append(kv, 0, ids, k, v, q=q, rope=table, tree_parent=parent)
    rk, rv = laser.kv_read(kv, 0, ids, R, dtype=F32)
    new_k = torch.empty((B, R, H, dh), dtype=torch.float64, device="cuda")
    for b in range(B):
        see = ref.paths(None if parent is None else parent[b].tolist(), R)
        pos = torch.tensor([lens[b] + len(s) - 1 for s in see], device="cuda")
        new_k[b] = ref.rotate(k[b].double(), table, dh, pos)
        wq = ref.rotate(q[b].double(), table, dh, pos)
        # two products and a sum in fp32, then the last rounding
        size = q[b].double().abs()
        size = size + torch.cat([size[..., dh // 2:], size[..., :dh // 2]], -1)
        assert bool(((qr[b].double() - wq).abs() <= ref.EPS[dtype] * wq.abs() + 2.0 ** -22 * size).all())
    assert torch.equal(rk, ref.held(new_k).float())              # codes are exact, and so is m + s c up to its one rounding
    assert torch.equal(rv, ref.held(v).float())
    for b, n in enumerate(lens):                                 # imported tokens too
        if n:
            ik, iv = laser.kv_read(kv, 0, [b], n, start=0, dtype=F32)
            assert torch.equal(ik[0], ref.held(ks[b]).float()) and torch.equal(iv[0], ref.held(vs[b]).float())
    out = laser.kv_attend(kv, 0, ids, qr, tree_parent=parent)
    check_attend(kv, lens, ks, vs, new_k, v.double(), qr, parent, None, dh ** -0.5, out, out, dtype != BF16)
    again = laser.kv_attend(kv, 0, ids, qr, tree_parent=parent)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_that_are_not_there_are_left_alone(dtype):
    B, R, H, G, dh, lens = 4, 6, 2, 3, 128, [20, 0, 64, 5]
    g = gen(1)
    kv = make_kv(B, H, dh, lens, R)
    ks, vs = fill(kv, lens, H, dh, g)
    n_rows = torch.tensor([6, 3, 0, 99], dtype=torch.int32, device="cuda")       # 99 is cut to R
    q, k, v = normal(g, B, R, H * G, dh, dtype=dtype), normal(g, B, R, H, dh, dtype=dtype), normal(g, B, R, H, dh, dtype=dtype)
    k[1, 3:], v[1, 3:], q[1, 3:] = float("nan"), float("inf"), float("nan")      # padding may hold anything
    before_k, before_v = laser.kv_read(kv, 0, range(B), R, dtype=F32)
    q_out = torch.full_like(q, 7.0)
    laser.kv_append(kv, 0, range(B), k, v, q=q, q_out=q_out, n_rows=n_rows)
    rk, rv = laser.kv_read(kv, 0, range(B), R, dtype=F32)
    for b, n in enumerate([6, 3, 0, 6]):
        assert torch.equal(rk[b, :n], ref.held(k[b, :n]).float()) and torch.equal(rk[b, n:], before_k[b, n:]) and torch.equal(rv[b, n:], before_v[b, n:])
        assert torch.equal(q_out[b, :n], q[b, :n]) and bool((q_out[b, n:] == 7).all())
    out = torch.full_like(q, -3.0)
    before = out.clone()
    laser.kv_attend(kv, 0, range(B), q, n_rows=n_rows, out=out)
    check_attend(kv, lens, ks, vs, k.double(), v.double(), q, None, n_rows, dh ** -0.5, out, before, dtype != BF16)


def test_strides_orders_and_in_place():
    B, R, H, G, dh, lens = 2, 3, 4, 2, 64, [37, 70]
    g = gen(2)
    kv = make_kv(B, H, dh, lens, R)
    ks, vs = fill(kv, lens, H, dh, g)
    fused = normal(g, B * R * (H * G + 2 * H) * dh + 1, dtype=F16)[1:].view(B, R, H * G + 2 * H, dh)     # one element off any grid
    q, k, v = fused[:, :, :H * G], fused[:, :, H * G:H * G + H], fused[:, :, H * G + H:]
    kd, vd, qd = k.double().clone(), v.double().clone(), q.clone()
    heads_first = q.transpose(1, 2).contiguous().transpose(1, 2)                 # [B][H][R][dh] in memory
    table = laser.rope_table(128, 64)
    want = laser.kv_append(kv, 0, [0, 1], k, v, q=heads_first, rope=table)
    got = laser.kv_append(kv, 0, [0, 1], k, v, q=q, rope=table, q_out=q)         # in place, within the fused rows
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want) and torch.equal(fused[:, :, H * G:].double(), torch.cat([kd, vd], 2))
    assert not torch.equal(got, qd)
    a = laser.kv_attend(kv, 0, [0, 1], want)
    odd = torch.zeros(B * H * G * R * dh + 1, dtype=F16, device="cuda")[1:].view(B, H * G, R, dh).transpose(1, 2)
    assert torch.equal(a, laser.kv_attend(kv, 0, [0, 1], q, out=odd))
    assert torch.equal(a, laser.kv_attend(kv, 0, [0, 1], q, out=q))
    same = normal(g, 1, 1, 1, dh, dtype=F16).expand(B, R, H, dh)                 # stride 0
    laser.kv_append(kv, 0, [0, 1], same, same)
    rk, rv = laser.kv_read(kv, 0, [0, 1], R, dtype=F32)
    assert torch.equal(rk, ref.held(same).float()) and torch.equal(rv, rk)


@pytest.mark.parametrize("dh, dim", [(128, 64), (128, 128), (64, 64)])
def test_partial_rotation_and_far_positions(dh, dim):
    H, n = 2, 40000
    kv = make_kv(1, H, dh, [n], 2)
    kv.set_len(0, n)
    g = gen(3)
    k, v = normal(g, 1, 2, H, dh, dtype=BF16), normal(g, 1, 2, H, dh, dtype=BF16)
    table = laser.rope_table(n + 2, dim, base=500000.0)
    i = torch.arange(dim // 2, dtype=torch.float64)
    ang = n * 500000.0 ** (-2 * i / dim)
    assert float((table[n].cpu().double() - torch.stack([ang.cos(), ang.sin()], -1)).abs().max()) <= 2.0 ** -24      # |cos| <= 1: half a step
    laser.kv_append(kv, 0, [0], k, v, rope=table)
    rk, _ = laser.kv_read(kv, 0, [0], 2, dtype=F32)
    want = ref.rotate(k[0].double(), table, dim, torch.tensor([n, n + 1], device="cuda"))
    assert torch.equal(rk[0], ref.held(want).float())


@pytest.mark.parametrize("scale", [1e-4, 1.0, 3000.0, 60000.0])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_sizes_of_values(scale, dtype):
    """Tiny and huge values: scales beyond 511 change the factor that weights carry, within one context."""
    B, R, H, G, dh, lens = 1, 2, 2, 2, 128, [600]
    g = gen(4)
    kv = make_kv(B, H, dh, lens, R)
    k = normal(g, 600, H, dh, dtype=F16)
    grow = torch.where(torch.arange(600, device="cuda") < 300, 1.0, scale)[:, None, None]
    v = (normal(g, 600, H, dh).clamp(-1, 1) * grow).to(F16)
    kv.import_layer(0, 0, k, v)
    kv.set_len(0, 600)
    q, nk, nv = normal(g, B, R, H * G, dh, dtype=dtype), normal(g, B, R, H, dh, dtype=dtype), normal(g, B, R, H, dh, dtype=dtype)
    laser.kv_append(kv, 0, [0], nk, nv)
    out = laser.kv_attend(kv, 0, [0], q)
    check_attend(kv, lens, [k.double()], [v.double()], nk.double(), nv.double(), q, None, None, dh ** -0.5, out, out, dtype != BF16)


@pytest.mark.parametrize("q_scale, softmax_scale", [(1e-6, 1e4), (3e4, 1e-4), (1.0, 0.0), (1.0, -0.3), (30.0, 1.0)])
def test_sizes_of_queries(q_scale, softmax_scale):
    B, R, H, dh, lens = 1, 3, 2, 64, [200]
    g = gen(5)
    kv = make_kv(B, H, dh, lens, R)
    ks, vs = fill(kv, lens, H, dh, g)
    q, k, v = normal(g, B, R, H, dh, scale=q_scale), normal(g, B, R, H, dh), normal(g, B, R, H, dh)
    laser.kv_append(kv, 0, [0], k, v)
    out = laser.kv_attend(kv, 0, [0], q, scale=softmax_scale)
    check_attend(kv, lens, ks, vs, k.double(), v.double(), q, None, None, softmax_scale, out, out, True)


def test_values_beyond_fp16_saturate():
    g = gen(6)
    kv = make_kv(1, 1, 64, [0], 3)
    k, v = normal(g, 1, 3, 1, 64, scale=1e30), normal(g, 1, 3, 1, 64, scale=1e6)
    k[0, 1], v[0, 1] = 5.0, 0.0                                                  # a constant group: scale 0
    laser.kv_append(kv, 0, [0], k, v)
    rk, rv = laser.kv_read(kv, 0, [0], 3, dtype=F32)
    assert torch.equal(rk, ref.held(k).float()) and torch.equal(rv, ref.held(v).float()) and bool(torch.isfinite(rk).all())


def test_what_is_not_finite_reaches_the_rows_that_see_it_and_no_others():
    R, H, G, dh, n = 5, 2, 2, 128, 50
    g = gen(7)
    kv = make_kv(1, H, dh, [n], R)
    ks, vs = fill(kv, [n], H, dh, g)
    parent = torch.tensor([[-1, -1, 0, 1]], dtype=torch.int32, device="cuda")    # rows 1 and 2 hang off row 0, 3 off 1, 4 off 2
    q, k, v = normal(g, 1, R, H * G, dh, dtype=F16), normal(g, 1, R, H, dh, dtype=F16), normal(g, 1, R, H, dh, dtype=F16)
    laser.kv_append(kv, 0, [0], k, v, tree_parent=parent)
    clean = laser.kv_attend(kv, 0, [0], q, tree_parent=parent)
    for bad in (float("nan"), float("inf"), float("-inf")):
        for what in (k, v):
            kk, vv = k.clone(), v.clone()
            (kk if what is k else vv)[0, 1, 0, 77] = bad                         # row 1, head 0
            laser.kv_append(kv, 0, [0], kk, vv, tree_parent=parent)
            out = laser.kv_attend(kv, 0, [0], q, tree_parent=parent)
            hit = torch.zeros(1, R, H * G, dtype=torch.bool, device="cuda")
            hit[0, [1, 3], :G] = True                                            # its own row and its child, query heads of head 0
            assert bool(torch.isnan(out[hit]).all()) and torch.equal(out[~hit], clean[~hit])
    # a query that is not finite: its own row only
    qq = q.clone()
    qq[0, 2, 1, 3] = float("nan")
    laser.kv_append(kv, 0, [0], k, v, tree_parent=parent)
    out = laser.kv_attend(kv, 0, [0], qq, tree_parent=parent)
    assert bool(torch.isnan(out[0, 2, 1]).all()) and int(torch.isnan(out).any(-1).sum()) == 1
    # stale rows behind the step, left by a longer one, are nobody's
    kk = k.clone()
    kk[0, 3:] = float("nan")
    laser.kv_append(kv, 0, [0], kk, v)
    laser.kv_append(kv, 0, [0], k[:, :2], v[:, :2])
    out = laser.kv_attend(kv, 0, [0], q[:, :2])
    assert bool(torch.isfinite(out).all())


def test_pages_that_another_sequence_left():
    H, dh = 2, 64
    g = gen(8)
    kv = laser.KVCache4(1, H, dh, 4, 2, 4)
    kv.reserve(0, 64)
    bad = torch.full((64, H, dh), float("nan"), dtype=F16, device="cuda")
    kv.import_layer(0, 0, bad, bad)
    kv.set_len(0, 60)
    kv.release(0)
    kv.reserve(1, 40)
    q, k, v = (normal(g, 1, 1, H, dh, dtype=F16) for _ in range(3))
    laser.kv_append(kv, 0, [1], k, v)
    out = laser.kv_attend(kv, 0, [1], q)
    check_attend(kv, [0], [k[0, :0].double()], [v[0, :0].double()], k.double(), v.double(), q, None, None, dh ** -0.5, out, out, True)


@pytest.mark.parametrize("G", [1, 4, 16])
def test_what_lies_behind_the_last_token_changes_nothing(G):
    """Values whose scales pass 511 switch the factor of the weights: not if they are in slots behind the step's."""
    H, dh, n = 2, 128, 37
    g = gen(14)
    k, v = normal(g, n, H, dh, dtype=F16), normal(g, n, H, dh, dtype=F16, scale=1e-3)
    q, nk, nv = normal(g, 1, 2, H * G, dh, dtype=F16), normal(g, 1, 2, H, dh, dtype=F16), normal(g, 1, 2, H, dh, dtype=F16, scale=1e-3)
    outs = []
    for stale in (0.0, 60000.0):
        kv = make_kv(1, H, dh, [n], 11)
        full = torch.full((48, H, dh), stale, dtype=F16, device="cuda")
        full[:, :, ::2] = -stale
        kv.import_layer(0, 0, full, full)
        kv.import_layer(0, 0, k, v)
        kv.set_len(0, n)
        laser.kv_append(kv, 0, [0], nk, nv)
        outs.append(laser.kv_attend(kv, 0, [0], q))
    assert torch.equal(outs[0], outs[1])
    check_attend(kv, [n], [k.double()], [v.double()], nk.double(), nv.double(), q, None, None, dh ** -0.5, outs[1], outs[1], True)


def test_many_sequences_in_one_call():
    """More sequences than ride in one launch's arguments."""
    B, H, dh = 300, 1, 64
    g = gen(9)
    lens = [i % 23 for i in range(B)]
    kv = make_kv(B, H, dh, lens, 2)
    ks, vs = fill(kv, lens, H, dh, g)
    q, k, v = (normal(g, B, 2, H, dh, dtype=F16) for _ in range(3))
    n_rows = torch.tensor([i % 3 for i in range(B)], dtype=torch.int32, device="cuda")
    parent = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    laser.kv_append(kv, 0, range(B), k, v, n_rows=n_rows, tree_parent=parent)
    out = torch.zeros_like(q)
    before = out.clone()
    laser.kv_attend(kv, 0, range(B), q, n_rows=n_rows, tree_parent=parent, out=out)
    check_attend(kv, lens, ks, vs, k.double(), v.double(), q, parent, n_rows, dh ** -0.5, out, before, True)


def test_commits_of_chains_and_trees():
    B, H, dh, lens = 2, 2, 128, [14, 30]
    g = gen(10)
    kv = make_kv(B, H, dh, lens, 40, layers=2)
    for layer in (0, 1):
        fill(kv, lens, H, dh, g, layer)
    k, v = (normal(g, B, 6, H, dh, dtype=BF16) for _ in range(2))
    parent = torch.tensor([[-1, 0, -1, 2, 3], [-1, -1, 1, -1, 3]], dtype=torch.int32, device="cuda")
    for layer in (0, 1):
        laser.kv_append(kv, layer, [1, 0], k + layer, v - layer, tree_parent=parent)
    accept = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    path = torch.tensor([[2, 3, 4, -1, -1], [1, 2, -1, -1, -1]], dtype=torch.int32, device="cuda")
    laser.kv_commit_tree(kv, [1, 0], accept, path)
    assert kv.read_lens([0, 1]).tolist() == [14 + 3, 30 + 4]
    for layer in (0, 1):
        for seq, b, rows in ((1, 0, [0, 3, 4, 5]), (0, 1, [0, 2, 3])):
            rk, rv = laser.kv_read(kv, layer, [seq], len(rows), start=lens[seq], dtype=F32)
            assert torch.equal(rk[0], ref.held((k + layer)[b, rows]).float()) and torch.equal(rv[0], ref.held((v - layer)[b, rows]).float())
    laser.kv_append(kv, 0, [0, 1], k[:, :3], v[:, :3])
    laser.kv_commit(kv, [0, 1], torch.tensor([2, 0], dtype=torch.int32, device="cuda"))
    assert kv.read_lens([0, 1]).tolist() == [20, 35]


def test_refusals():
    H, dh = 2, 64
    kv = laser.KVCache4(1, H, dh, 4, 2, 2)
    kv.reserve(0, 20)
    g = gen(11)
    q, k, v = normal(g, 1, 2, 4, dh, dtype=F16), normal(g, 1, 2, H, dh, dtype=F16), normal(g, 1, 2, H, dh, dtype=F16)
    two = lambda t: t.expand(2, *t.shape[1:])  # noqa: E731
    table = laser.rope_table(8, dh)

    def refused(match, f, *a, **kw):
        with pytest.raises(laser.LaserError, match=match):
            f(*a, **kw)
    refused("code -4|reserved", laser.kv_append, kv, 0, [1], k, v)                         # nothing reserved
    refused("twice", laser.kv_append, kv, 0, [0, 0], two(k), two(v))
    refused("out of range", laser.kv_append, kv, 0, [2], k, v)
    refused("layer", laser.kv_append, kv, 1, [0], k, v)
    refused("contiguous", laser.kv_append, kv, 0, [0], k, v.float())
    refused("contiguous", laser.kv_append, kv, 0, [0], k, v[:, :1])
    refused("R 65", laser.kv_append, kv, 0, [0], k[:, :1].expand(1, 65, H, dh), v[:, :1].expand(1, 65, H, dh))
    refused("n_rows", laser.kv_append, kv, 0, [0], k, v, n_rows=torch.ones(2, dtype=torch.int32, device="cuda"))
    refused("tree_parent", laser.kv_append, kv, 0, [0], k, v, tree_parent=torch.zeros((1, 2), dtype=torch.int32, device="cuda"))
    refused("tree_parent", laser.kv_append, kv, 0, [0], k, v, tree_parent=torch.zeros((1, 1), dtype=torch.int64, device="cuda"))
    refused("rope_dim", laser.kv_append, kv, 0, [0], k, v, rope=laser.rope_table(8, 32))
    kv.set_len(0, 7)
    refused("max_pos", laser.kv_append, kv, 0, [0], k, v, rope=table)
    kv.set_len(0, 31)
    refused("reserved", laser.kv_append, kv, 0, [0], k, v)
    refused("reserved", laser.kv_attend, kv, 0, [0], q)
    refused("reserved", laser.kv_read, kv, 0, [0], 2)
    kv.set_len(0, 0)
    refused("multiple", laser.kv_attend, kv, 0, [0], q[:, :, :3])
    refused("finite", laser.kv_attend, kv, 0, [0], q, scale=float("nan"))
    refused("float64", laser.kv_attend, kv, 0, [0], q.double())
    refused("seq_ids", laser.kv_attend, kv, 0, [0, 1], q)
    refused("contiguous", laser.kv_attend, kv, 0, [0], q.transpose(2, 3).contiguous().transpose(2, 3))
    refused("start", laser.kv_read, kv, 0, [0], 2, start=-2)
    plain = laser.KVCache(1, H, dh, 4, 2, 2)
    refused("KVCache4", laser.kv_append, plain, 0, [0], k, v)
    plain._h, kv._h = kv._h, plain._h                                                      # the library itself refuses it too
    try:
        refused("laser_kv_create_4bit", laser.kv_append, kv, 0, [0], k, v)
    finally:
        plain._h, kv._h = kv._h, plain._h
    refused("commit", laser.kv_commit, kv, [0], torch.zeros(1, dtype=torch.int32, device="cuda"))
    empty = torch.zeros((0, 1, H, dh), dtype=F16, device="cuda")
    laser.kv_append(kv, 0, [], empty, empty)
    assert laser.kv_attend(kv, 0, [], torch.zeros((0, 1, 4, dh), dtype=F16, device="cuda")).shape[0] == 0


def test_on_another_stream_and_captured():
    """A layer's step on a stream of its own, and as a captured graph replayed over changing inputs and growing lengths."""
    B, R, H, G, dh, lens = 2, 2, 2, 4, 128, [100, 33]
    g = gen(12)
    ids = list(range(B))
    table = laser.rope_table(256, dh)
    wq = laser.W4(*laser.w4_quantize(normal(g, (G + 2) * H * dh, 256, dtype=BF16, scale=0.05), 64))
    wo = laser.W4(*laser.w4_quantize(normal(g, 256, G * H * dh, dtype=BF16, scale=0.05), 128))
    x = normal(g, B * R, 256, dtype=BF16)
    accept = torch.full((B,), R - 1, dtype=torch.int32, device="cuda")
    caches = [make_kv(B, H, dh, lens, 40) for _ in range(2)]
    for kv in caches:
        fill(kv, lens, H, dh, gen(13))

    def step(kv, bufs, stream=None):
        qkv, qo, o, y = bufs
        laser.w4_matmul(wq, x, out=qkv, stream=stream)
        rows = qkv.view(B, R, (G + 2) * H, dh)
        laser.kv_append(kv, 0, ids, rows[:, :, G * H:(G + 1) * H], rows[:, :, (G + 1) * H:], q=rows[:, :, :G * H], rope=table, q_out=qo, stream=stream)
        laser.kv_attend(kv, 0, ids, qo, out=o, stream=stream)
        laser.kv_commit(kv, ids, accept, stream=stream)
        return laser.w4_matmul(wo, o.view(B * R, G * H * dh), out=y, stream=stream)

    def buffers():
        return (torch.empty((B * R, (G + 2) * H * dh), dtype=BF16, device="cuda"), *(torch.empty((B, R, G * H, dh), dtype=BF16, device="cuda") for _ in range(2)),
                torch.empty((B * R, 256), dtype=BF16, device="cuda"))
    torch.cuda.synchronize()
    graph, side, mine = torch.cuda.CUDAGraph(), torch.cuda.Stream(), buffers()
    step(caches[1], mine)                                        # warm up; then back to the start
    for b, n in enumerate(lens):
        caches[1].set_len(b, n)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(caches[1], mine)
    for i in range(4):
        x.copy_(normal(g, B * R, 256, dtype=BF16))
        theirs = buffers()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = step(caches[0], theirs)
        graph.replay()
        torch.cuda.synchronize()
        # the same tokens; the eager launches may cut the context elsewhere, as their bounds grow: the last bits of fp32 sums, so a
        # step of bf16 here and there, which the next product averages
        assert torch.equal(mine[0], theirs[0]) and torch.equal(mine[1], theirs[1])
        a, b = mine[2].double(), theirs[2].double()
        assert bool(((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -10).all())
        assert bool(((mine[3].double() - want.double()).abs() <= 2.0 ** -6 * want.double().abs().max()).all())
        assert caches[0].read_lens(ids).tolist() == [n + R * (i + 1) for n in lens]
    # replays beyond what was reserved at the capture: no row is written there, none is read
    for _ in range(30):
        graph.replay()
    torch.cuda.synchronize()
    caches[1].set_len(0, 0)
    assert bool(torch.isfinite(laser.kv_attend(caches[1], 0, [0], mine[1][:1])).all())


# ------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("N, Kd, group", [(1, 32, 32), (17, 96, 32), (40, 64, 64), (33, 320, 64), (200, 128, 128), (768, 256, 32), (1000, 1152, 128)])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 40, 63, 80, 81, 200])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_products(N, Kd, group, M, dtype):
    g = gen(N + M)
    w = normal(g, N, Kd, dtype=BF16, scale=0.3)
    w[:, ::7] *= 6
    codes, s, m = laser.w4_quantize(w, group)
    c, rs, rm = ref.quantize(w.double(), group)
    assert torch.equal(s, rs) and torch.equal(m, rm)
    unpacked = torch.stack([codes & 15, codes >> 4], -1).flatten(1)
    assert torch.equal(unpacked.double(), c)
    h = laser.W4(codes, s, m)
    big = torch.full((M + 1, Kd + 3), 50.0, dtype=dtype, device="cuda")
    x = big[:M, 1:Kd + 1]                                        # rows off any grid, a stride of their own
    x.copy_(normal(g, M, Kd, dtype=dtype))
    out = torch.full((M + 1, N + 5), 3.0, dtype=dtype, device="cuda")
    laser.w4_matmul(h, x, out=out[:M, 2:N + 2])
    assert bool((out[M] == 3).all()) and bool((out[:, :2] == 3).all()) and bool((out[:, N + 2:] == 3).all())
    want = x.double() @ ref.values(c, s, m).T
    # fp32 sums: two roundings a group and some sixty within it and at the joints, of terms |x| (s c + |m|); bf16 rows meet codes as
    # 128 + c, and an offset of m - 128 s
    size = x.double().abs() @ (ref.values(c, s, m.abs()) + (256 * s.double().repeat_interleave(group, 1) if dtype == BF16 else 0)).T
    tol = (2 * Kd / group + 64) * 2.0 ** -24 * size
    err = (out[:M, 2:N + 2].double() - want).abs()
    bound = tol + ref.EPS[dtype] * (want.abs() + tol)
    if dtype == F16:
        bound = bound + 2.0 ** -25                               # half of fp16's smallest step
    assert bool((err <= bound).all()), float((err / bound).max())
    assert torch.equal(laser.w4_matmul(h, x), out[:M, 2:N + 2])


@pytest.mark.parametrize("N, M", [(4100, 17), (4100, 65), (8185, 33), (6150, 50), (11260, 20), (12270, 40), (22010, 24), (22010, 35), (22010, 75), (9003, 170)])
@pytest.mark.parametrize("Kd, group", [(160, 32), (320, 64), (384, 128)])
def test_products_of_every_tile_of_a_wave(N, Kd, group, M):
    """Widths and rows that the choice of tiles falls to either side for, neither whole tiles."""
    test_products(N, Kd, group, M, F16)
    test_products(N, Kd, group, M, BF16)


def test_products_at_the_model_widths():
    g = gen(20)
    for N, Kd, group, M, dtype in ((22016, 4096, 128, 1, BF16), (4096, 11008, 64, 9, F16), (6144, 2048, 128, 72, BF16), (12288, 4096, 32, 33, F16)):
        c = torch.randint(0, 16, (N, Kd), device="cuda", generator=g)
        s, m = normal(g, N, Kd // group, scale=0.01).abs().to(F16), normal(g, N, Kd // group, dtype=F16, scale=0.05)
        h = laser.W4((c[:, ::2] | (c[:, 1::2] << 4)).to(torch.uint8), s, m)
        x = normal(g, M, Kd, dtype=dtype)
        w = ref.values(c.double(), s, m)
        want, got = x.double() @ w.T, laser.w4_matmul(h, x).double()
        size = x.double().abs() @ (ref.values(c.double(), s, m.abs()) + (256 * s.double().repeat_interleave(group, 1) if dtype == BF16 else 0)).T
        tol = (2 * Kd / group + 64) * 2.0 ** -24 * size
        assert bool(((got - want).abs() <= tol + ref.EPS[dtype] * (want.abs() + tol) + 2.0 ** -25).all()), (N, Kd)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_weights_that_are_not_finite_reach_their_own_output_only(dtype, group):
    """A group with such a weight is NaN: so is its output, and no other."""
    g = gen(15)
    w, x = normal(g, 48, 256, dtype=BF16, scale=0.05), normal(g, 7, 256, dtype=dtype)
    want = laser.w4_matmul(laser.W4(*laser.w4_quantize(w, group)), x)
    bad = {3: (0, float("nan")), 17: (255, float("inf")), 40: (130, float("-inf"))}
    for n, (i, value) in bad.items():
        w[n, i] = value
    w[33, :group] = float("nan")
    codes, s, m = laser.w4_quantize(w, group)
    assert s.isfinite().all()
    for n, (i, _) in bad.items():
        assert m[n].isnan().nonzero().tolist() == [[i // group]] and s[n, i // group] == 0
        assert not codes[n, i // group * group // 2:(i // group + 1) * group // 2].any()
    got = laser.w4_matmul(laser.W4(codes, s, m), x)
    rows = torch.tensor([*bad, 33], device="cuda")
    assert got[:, rows].isnan().all()
    keep = torch.ones(48, dtype=torch.bool, device="cuda")
    keep[rows] = False
    assert torch.equal(got[:, keep], want[:, keep])


def test_product_refusals():
    g = gen(21)
    h = laser.W4(*laser.w4_quantize(normal(g, 32, 128, dtype=BF16), 64))
    x = normal(g, 2, 128, dtype=F16)
    for bad in (x.float(), x[:, :64], x.cpu(), x.T, x[0]):
        with pytest.raises(laser.LaserError):
            laser.w4_matmul(h, bad)
    for out in (x, torch.empty((2, 32), dtype=BF16, device="cuda"), torch.empty((32, 2), dtype=F16, device="cuda").T):
        with pytest.raises(laser.LaserError):
            laser.w4_matmul(h, x, out=out)
    with pytest.raises(laser.LaserError, match="overlap"):
        laser.w4_matmul(h, x[:1].expand(2, 128))
    with pytest.raises(laser.LaserError):
        laser.w4_quantize(normal(g, 32, 96, dtype=BF16), 64)
    assert laser.w4_matmul(h, x[:0]).shape == (0, 32)


# ------------------------------------------------------------------------------------------------ the model on a 4-bit cache
def reference_step(w, sh, kv, lens, tokens, parent, stored=True):
    """Logits [B][R][V] of a step in 64 bits, with the keys and values that the cache holds after it, and the largest distance of these from
    the step's own keys and values, in steps of their group's codes. stored False: with the step's own keys and values as they are."""
    L, d, H, dh = sh.n_layers, sh.d, sh.n_heads, sh.head_dim
    B, R = tokens.shape
    f = {n: t.double() for n, t in w.items()}
    x = f["emb"][tokens.long()]
    norm = lambda y, gain: y * (y.square().mean(-1, keepdim=True) + sh.eps).rsqrt() * gain  # noqa: E731
    table = laser.rope_table(max(lens) + R, dh, base=sh.rope_base)
    worst = 0.0
    for layer in range(L):
        qkv = norm(x, f["g1"][layer]) @ f["wqkv"][layer].T
        att = torch.empty((B, R, H, dh), dtype=torch.float64, device="cuda")
        for b in range(B):
            see = ref.paths(None if parent is None else parent[b].tolist(), R)
            pos = torch.tensor([lens[b] + len(s) - 1 for s in see], device="cuda")
            q, k, v = qkv[b].view(R, 3, H, dh).unbind(1)
            q, k = ref.rotate(q, table, dh, pos), ref.rotate(k, table, dh, pos)
            ck, cv = laser.kv_read(kv, layer, [b], lens[b] + R, start=0, dtype=F32)
            if not stored:
                ck, cv = ck.double(), cv.double()
                ck[0, lens[b]:], cv[0, lens[b]:] = k, v
            for own, have in ((k, ck[0, lens[b]:].double()), (v, cv[0, lens[b]:].double())):
                span = own.unflatten(-1, (-1, 32))
                span = (span.amax(-1) - span.amin(-1)).repeat_interleave(32, -1) / 15
                worst = max(worst, float(((own - have).abs() / span).max()))
            att[b], _ = ref.attend(q, ck[0].double(), cv[0].double(), lens[b], see, dh ** -0.5, cv[0].double().abs(), ck[0].double().abs(), True)
        x = x + att.reshape(B, R, d) @ f["wo"][layer].T
        gu = norm(x, f["g2"][layer]) @ f["wgu"][layer].T
        gate, up = gu.chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ f["wdown"][layer].T
    return norm(x, f["gf"]) @ f["wlm"].T, worst


@pytest.mark.parametrize("B, K, tree", [(2, 4, False), (2, 4, True), (1, 0, False), (5, 7, True), (3, 40, False)])
def test_model_steps_on_a_four_bit_cache(B, K, tree):
    import synth
    from tests.gpu_util import gpu_weights, logits_close
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    lens = [33 + 20 * b for b in range(B)]
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * (K + 1), B, 512, eps=sh.eps, rope_base=sh.rope_base)
    kv = make_kv(B, sh.n_heads, sh.head_dim, lens, 2 * (K + 1), layers=sh.n_layers)
    g = gen(30 + K)
    for layer in range(sh.n_layers):
        fill(kv, lens, sh.n_heads, sh.head_dim, g, layer)
    r = np.random.default_rng(K)
    tokens = torch.tensor(r.integers(0, sh.vocab, (B, K + 1)), dtype=torch.int32, device="cuda")
    n = torch.full((B,), K, dtype=torch.int32, device="cuda")
    drafts = tokens[:, 1:].contiguous()
    parent = None
    if tree:
        parent = torch.tensor([[int(r.integers(-1, i)) if i else -1 for i in range(K)] for _ in range(B)], dtype=torch.int32, device="cuda")
        acc, out, path, logits = laser.verify_tree(model, kv, range(B), tokens[:, 0].contiguous(), drafts, parent, n, 2, 0.1, 0, want_logits=True)
    else:
        acc, out, logits = laser.verify_step(model, kv, range(B), tokens[:, 0].contiguous(), drafts, n, 2, 0.1, 0, want_logits=True)
    want, worst = reference_step(w, sh, kv, lens, tokens, parent)
    ok, err, rel = logits_close(logits.cpu().double().numpy(), want.cpu().numpy())
    assert ok, (err, rel)
    # half a step for the nearest code, one part in 2^11 of an offset up to 15 steps from zero (or more where a group lies off it:
    # these are centred), and a scale that fp16 rounds by 2^-11 over 15 steps; the rows' own rounding is far below
    assert worst <= 0.5 + 3 * 15 * 2.0 ** -11, worst
    laser.kv_commit_tree(kv, range(B), acc, path) if tree else laser.kv_commit(kv, range(B), acc)
    assert kv.read_lens(range(B)).tolist() == [t + int(a) + 1 for t, a in zip(lens, acc.tolist())]


@pytest.mark.parametrize("B, K, tree, four_bit_cache, which", [
    (2, 4, False, True, "wqkv wo wgu wdown"), (1, 0, False, False, "wqkv wo wgu wdown"), (4, 10, True, True, "wqkv wo wgu wdown"),
    (3, 40, False, False, "wqkv wo wgu wdown"), (2, 7, False, False, "wgu"), (5, 7, True, False, "wo wdown"), (2, 2, False, True, "wqkv")])
def test_model_steps_with_four_bit_weights(B, K, tree, four_bit_cache, which):
    import synth
    from tests.gpu_util import gpu_weights, logits_close
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    lens = [20 + 9 * b for b in range(B)]
    R = K + 1
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * R, B, 512, eps=sh.eps, rope_base=sh.rope_base)
    what = dict(w)
    groups = dict(wqkv=32, wo=64, wgu=128, wdown=128)
    for name in which.split():
        what[name] = torch.empty(w[name].shape, dtype=torch.float64, device="cuda")
        for layer in range(sh.n_layers):
            codes, s, m = laser.w4_quantize(w[name][layer].contiguous(), groups[name])
            model.set_w4(layer, name, laser.W4(codes, s, m))
            what[name][layer] = ref.values(torch.stack([codes & 15, codes >> 4], -1).flatten(1).double(), s, m)
    g = gen(40 + K)
    # the reference takes its cache contents from laser_kv_read: a 4-bit copy of a plain cache's imports would differ, so these are what
    # a 4-bit cache stands for in both
    kv = make_kv(B, sh.n_heads, sh.head_dim, lens, 2 * R, layers=sh.n_layers)
    plain = laser.KVCache(sh.n_layers, sh.n_heads, sh.head_dim, 200, B, 40)
    for b in range(B):
        plain.reserve(b, lens[b] + 2 * R)
        plain.set_len(b, lens[b])
    for layer in range(sh.n_layers):
        fill(kv, lens, sh.n_heads, sh.head_dim, g, layer)
        for b in range(B):
            k, v = laser.kv_read(kv, layer, [b], lens[b], start=0)
            plain.import_layer(b, layer, k[0], v[0])
    r = np.random.default_rng(K)
    tokens = torch.tensor(r.integers(0, sh.vocab, (B, R)), dtype=torch.int32, device="cuda")
    n = torch.full((B,), K, dtype=torch.int32, device="cuda")
    drafts = tokens[:, 1:].contiguous()
    parent = torch.tensor([[int(r.integers(-1, i)) if i else -1 for i in range(K)] for _ in range(B)], dtype=torch.int32, device="cuda") if tree else None
    use = kv if four_bit_cache else plain

    def step():
        if tree:
            return laser.verify_tree(model, use, range(B), tokens[:, 0].contiguous(), drafts, parent, n, 2, 0.1, 0, want_logits=True)[-1]
        return laser.verify_step(model, use, range(B), tokens[:, 0].contiguous(), drafts, n, 2, 0.1, 0, want_logits=True)[-1]
    logits = step()
    want = reference_step(what, sh, kv, lens, tokens, parent, stored=four_bit_cache)[0]
    ok, err, rel = logits_close(logits.cpu().double().numpy(), want.cpu().numpy())
    assert ok, (err, rel)
    for name in which.split():                                   # and back
        for layer in range(sh.n_layers):
            model.set_w4(layer, name, None)
    want = reference_step(w, sh, kv, lens, tokens, parent, stored=False)[0]
    if not four_bit_cache:
        ok, err, rel = logits_close(step().cpu().double().numpy(), want.cpu().numpy())
        assert ok, (err, rel)
    with pytest.raises(laser.LaserError, match="not"):
        model.set_w4(0, "wo", laser.W4(*laser.w4_quantize(w["wqkv"][0].contiguous(), 128)))
    with pytest.raises(laser.LaserError, match="layer"):
        model.set_w4(sh.n_layers, "wo", None)


def test_engine_in_four_bits():
    """Prompts in pieces, then a step, all through the Engine, with 4-bit weights and a 4-bit cache."""
    import synth
    from paper_2408_05676_amd.harness import Engine
    from tests.gpu_util import gpu_weights, logits_close
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    what = dict(w)
    for name in ("wqkv", "wo", "wgu", "wdown"):
        what[name] = torch.stack([ref.values(*ref.quantize(w[name][layer].double(), 64)) for layer in range(sh.n_layers)])
    B, K, T = 3, 5, 40
    eng = Engine(sh, w, B, K, T + 20, prefill_chunk=16, four_bit_cache=True, w4_group=64)
    r = np.random.default_rng(8)
    prompts = r.integers(0, sh.vocab, (B, T))
    eng.prefill(prompts)
    assert eng.kv.read_lens(eng.seq_ids).tolist() == [T - 1] * B
    drafts = torch.tensor(r.integers(0, sh.vocab, (B, K)), dtype=torch.int32, device="cuda")
    n = torch.full((B,), K, dtype=torch.int32, device="cuda")
    logits = laser.verify_step(eng.model, eng.kv, eng.seq_ids, eng.pending, drafts, n, 2, 0.1, want_logits=True)[-1]
    want, worst = reference_step(what, sh, eng.kv, [T - 1] * B, torch.cat([eng.pending[:, None], drafts], 1), None)
    ok, err, rel = logits_close(logits.cpu().double().numpy(), want.cpu().numpy())
    assert ok, (err, rel)
    assert worst <= 0.5 + 3 * 15 * 2.0 ** -11, worst
    eng.close()


def test_generation_on_a_four_bit_cache():
    """laser_generate with strict acceptance emits what one-token steps on the same kind of cache emit, drafts or not: a row's scores
    are the same numbers however many rows its step has, up to the order of fp32 sums."""
    import synth
    from tests.gpu_util import gpu_weights
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    w["gf"] = w["gf"] * 5
    B, T, new = 2, 24, 20
    r = np.random.default_rng(3)
    prompt = r.integers(0, sh.vocab, (B, T))
    texts = []
    for K in (0, 4):
        model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * (K + 1), B, 512, eps=sh.eps, rope_base=sh.rope_base)
        kv = make_kv(B, sh.n_heads, sh.head_dim, [T] * B, new + K + 2, layers=sh.n_layers)
        for t in range(T - 1):
            one = torch.tensor(prompt[:, t], dtype=torch.int32, device="cuda")
            none = torch.empty((B, 0), dtype=torch.int32, device="cuda")
            acc, _, _ = laser.verify_step(model, kv, range(B), one, none, torch.zeros(B, dtype=torch.int32, device="cuda"), 1, -1.0)
            laser.kv_commit(kv, range(B), acc)
        pool = None
        if K:
            seqs = np.concatenate([texts[0][b] for b in range(B)]).astype(np.int32)        # drafts that are right
            pool = laser.Pool(seqs, np.arange(B + 1) * new, np.arange(B), 3)
        tail = torch.tensor(prompt[:, -3:], dtype=torch.int32, device="cuda")
        pending = torch.tensor(prompt[:, -1], dtype=torch.int32, device="cuda")
        keys = torch.arange(B, dtype=torch.int64, device="cuda")
        text, n, *_ = laser.generate(model, kv, pool, range(B), keys, tail, pending, K, 1, 1, -1.0, 0, max_new_tokens=new)
        assert n.tolist() == [new] * B
        texts.append(text.cpu().numpy())
    assert (texts[0] == texts[1]).mean() > 0.5                   # (a code may fall to the other side of a border, and the texts part)
    assert (texts[0][:, 0] == texts[1][:, 0]).all()
