"""Steps of models whose projections are held in 8-bit integers: the operators one after the other, mixtures with other weights, replays, the Engine."""
import numpy as np
import pytest
import torch

import paper_2408_05676_amd as laser
import synth
from tests import eight_bit_ref as ref
from tests import test_gpu_four_bit as four
from tests.gpu_util import gpu_weights, logits_close

pytestmark = pytest.mark.gpu

F16, F32 = torch.float16, torch.float32
NAMES = ("wqkv", "wo", "wgu", "wdown")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def held(w, which=NAMES):
    """{(layer, name): W8} and the weights that these stand for."""
    what, made = dict(w), {}
    for name in which:
        what[name] = torch.empty(w[name].shape, dtype=torch.float64, device="cuda")
        for layer in range(w[name].shape[0]):
            codes, s = laser.w8_quantize(w[name][layer].contiguous())
            made[layer, name] = laser.W8(codes, s, gated=name == "wgu")
            what[name][layer] = codes.double() * s.double()[:, None]
    return made, what


def tree_or_chain(r, B, K, tree):
    return i32([[int(r.integers(-1, i)) if i else -1 for i in range(K)] for _ in range(B)]) if tree and K else None


def caches(sh, lens, extra, seed, n=2):
    """n 4-bit caches with the same contents."""
    out = []
    for _ in range(n):
        kv = four.make_kv(len(lens), sh.n_heads, sh.head_dim, lens, extra, layers=sh.n_layers)
        g = four.gen(seed)
        for layer in range(sh.n_layers):
            four.fill(kv, lens, sh.n_heads, sh.head_dim, g, layer)
        out.append(kv)
    return out


def step(model, kv, tokens, parent):
    B, R = tokens.shape
    n, pending, drafts = i32([R - 1] * B), tokens[:, 0].contiguous(), tokens[:, 1:].contiguous()
    if parent is not None:
        return laser.verify_tree(model, kv, range(B), pending, drafts, parent, n, 2, 0.1, 0, want_logits=True)[-1]
    return laser.verify_step(model, kv, range(B), pending, drafts, n, 2, 0.1, 0, want_logits=True)[-1]


def by_operators(sh, w, w8, kv, lens, tokens, parent):
    """Residual stream [B R][d] of a step, by calls of the operators."""
    B, R = tokens.shape
    M, d, H, dh = B * R, sh.d, sh.n_heads, sh.head_dim
    x = w["emb"][tokens.long()].float().view(M, d)
    table = laser.rope_table(max(lens) + R, dh, base=sh.rope_base)
    down = None
    for layer in range(sh.n_layers):
        q = laser.q8_norm(x if down is None else down, w["g1"][layer], sh.eps, residual=None if down is None else x)
        qkv = laser.w8_matmul(w8[layer, "wqkv"], *q, dtype=F32).view(B, R, 3, H, dh)
        qr = laser.kv_append(kv, layer, range(B), qkv[:, :, 1], qkv[:, :, 2], q=qkv[:, :, 0], rope=table, tree_parent=parent)
        att = laser.kv_attend(kv, layer, range(B), qr, tree_parent=parent).view(M, d)
        o = laser.w8_matmul(w8[layer, "wo"], *laser.q8_rows(att.half()), dtype=F32)
        act = laser.w8_matmul(w8[layer, "wgu"], *laser.q8_norm(o, w["g2"][layer], sh.eps, residual=x))
        down = laser.w8_matmul(w8[layer, "wdown"], *laser.q8_rows(act), dtype=F32)
    return x + down


@pytest.mark.parametrize("shape", ["tiny", "tiny128"])
@pytest.mark.parametrize("B, K, tree", [(1, 0, False), (2, 4, True), (3, 10, False), (5, 7, True), (3, 40, False), (6, 63, True)])
def test_a_step_is_its_operators(shape, B, K, tree):
    """1 to 384 rows. Everything up to the final norm is the same calls, so that the logits differ by that norm's rounding alone: its fp32 sums and fp16 results
    are within a place of the 64-bit ones, 2^-10 of each element of the head's input, and the head adds fp32 sums of as many products.
    At 128 channels a head the step multiplies scores with fp32(log2 e) / fp32(sqrt(128)), the operator with the product of log2 e and the caller's 1 / sqrt(128), three
    roundings in another order (at 64 channels the root is a power of two). A value may then round to the next code, as in test_steps_beside_other_weights; what comes before
    the first attention is the same."""
    sh = synth.SHAPES[shape]
    w = gpu_weights(sh)
    w8, _ = held(w)
    r = np.random.default_rng(K)
    lens = [20 + 9 * b for b in range(B)]
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * (K + 1), B, 512, eps=sh.eps, rope_base=sh.rope_base)
    for (layer, name), m in w8.items():
        model.set_w8(layer, name, m)
    kv, twin = caches(sh, lens, K + 1, 7)
    tokens, parent = i32(r.integers(0, sh.vocab, (B, K + 1))), tree_or_chain(r, B, K, tree)
    logits = step(model, kv, tokens, parent).double().view(B * (K + 1), -1)
    x = by_operators(sh, w, w8, twin, lens, tokens, parent).double()
    for layer in range(sh.n_layers if sh.head_dim == 64 else 1):
        for a, b in zip(laser.kv_read(kv, layer, range(B), K + 1), laser.kv_read(twin, layer, range(B), K + 1)):
            assert torch.equal(a, b)
    h = x * (x.square().mean(-1, keepdim=True) + sh.eps).rsqrt() * w["gf"].double()
    head = w["wlm"].double().T.contiguous()
    bound = (2.0 ** -10 + sh.d * 2.0 ** -24) * (h.abs() @ head.abs())
    if sh.head_dim == 64:
        assert bool(((logits - h @ head).abs() <= bound).all())
    else:
        assert float((logits - h @ head).norm() / logits.norm()) < 0.06


@pytest.mark.parametrize("B, K, tree, four_bit_cache, which", [
    (2, 4, False, False, "wqkv wo wgu wdown"), (1, 0, False, False, "wqkv"), (1, 8, True, False, "wo"), (3, 9, False, False, "wgu"), (4, 10, True, False, "wdown"),
    (3, 40, False, False, "wo wdown"), (3, 40, True, True, "wqkv wgu"), (2, 63, False, False, "wqkv wo wgu wdown")])
def test_steps_beside_other_weights(B, K, tree, four_bit_cache, which):
    """Single projections in 8 bits, the others in bf16, on either cache, against 64-bit steps with the weights that the codes stand for.
    A row's 8 bits are steps of its largest / 127, here 4.5 standard deviations / 127 = 0.035 of one, a rounding error of 0.035 / sqrt(12) = 0.01; a layer has four
    such tensors, the model two layers, and each meets the others' through a norm or a softmax: 0.01 sqrt(8) = 0.03 of the logits' norm, held to twice that."""
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    names = which.split()
    w8, what = held(w, names)
    lens = [20 + 9 * b for b in range(B)]
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * (K + 1), B, 512, eps=sh.eps, rope_base=sh.rope_base)
    kv, = caches(sh, lens, 2 * (K + 1), 9, n=1)
    plain = laser.KVCache(sh.n_layers, sh.n_heads, sh.head_dim, 200, B, 40)
    for b in range(B):
        plain.reserve(b, lens[b] + 2 * (K + 1))
        for layer in range(sh.n_layers):
            k, v = laser.kv_read(kv, layer, [b], lens[b], start=0)
            plain.import_layer(b, layer, k[0], v[0])
        plain.set_len(b, lens[b])
    use = kv if four_bit_cache else plain
    r = np.random.default_rng(K + 1)
    tokens, parent = i32(r.integers(0, sh.vocab, (B, K + 1))), tree_or_chain(r, B, K, tree)
    before = step(model, use, tokens, parent)
    for (layer, name), m in w8.items():
        model.set_w8(layer, name, m)
    logits = step(model, use, tokens, parent)
    want = four.reference_step(what, sh, kv, lens, tokens, parent, stored=four_bit_cache)[0]
    off = float((logits.double() - want).norm() / want.norm())
    assert 1e-4 < off < 0.06, off
    for layer, name in w8:
        model.set_w8(layer, name, None)
    after = step(model, use, tokens, parent)
    if B * (K + 1) > 16:
        assert torch.equal(after, before)
    ok, err, rel = logits_close(after.cpu().double().numpy(), before.cpu().double().numpy())
    assert ok, (err, rel)


def test_one_kind_of_weights_takes_the_others_place():
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    lens, r = [30, 12], np.random.default_rng(3)
    tokens = i32(r.integers(0, sh.vocab, (2, 12)))

    def fresh(setter):
        model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, 24, 2, 512, eps=sh.eps, rope_base=sh.rope_base)
        setter(model)
        kv, = caches(sh, lens, 12, 4, n=1)
        return step(model, kv, tokens, None)
    eight = lambda m: m.set_w8(1, "wo", laser.W8(*laser.w8_quantize(w["wo"][1].contiguous())))  # noqa: E731
    four_ = lambda m: m.set_w4(1, "wo", laser.W4(*laser.w4_quantize(w["wo"][1].contiguous(), 64)))  # noqa: E731
    a, b, none = fresh(eight), fresh(four_), fresh(lambda m: None)
    assert not torch.equal(a, b) and not torch.equal(a, none)
    assert torch.equal(fresh(lambda m: (four_(m), eight(m))), a)
    assert torch.equal(fresh(lambda m: (eight(m), four_(m))), b)
    assert torch.equal(fresh(lambda m: (four_(m), eight(m), m.set_w8(1, "wo", None))), none)
    assert torch.equal(fresh(lambda m: (eight(m), m.set_w4(1, "wo", None))), a)              # (takes away 4-bit weights only)


def test_matrices_of_a_model(monkeypatch):
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, 4, 1, 64, eps=sh.eps, rope_base=sh.rope_base)
    make = lambda name, **k: laser.W8(*laser.w8_quantize(w[name][0].contiguous()), **k)  # noqa: E731
    closed, first, second = make("wo"), make("wo"), make("wo")
    closed.close()
    with pytest.raises(laser.LaserError, match="closed"):
        model.set_w8(0, "wo", closed)
    with pytest.raises(laser.LaserError, match="W8"):
        model.set_w8(0, "wo", laser.W4(*laser.w4_quantize(w["wo"][0].contiguous(), 64)))
    with pytest.raises(laser.LaserError, match="W4"):
        model.set_w4(0, "wo", first)
    with pytest.raises(laser.LaserError, match="wq"):
        model.set_w8(0, "wq", first)
    with pytest.raises(laser.LaserError, match="layer"):
        model.set_w8(sh.n_layers, "wo", first)
    with pytest.raises(laser.LaserError, match="not"):
        model.set_w8(0, "wqkv", first)
    with pytest.raises(laser.LaserError, match="gated"):
        model.set_w8(0, "wgu", make("wgu"))
    with pytest.raises(laser.LaserError, match="gated"):
        model.set_w8(0, "wo", make("wo", gated=True))
    monkeypatch.setattr(second, "device", 1)
    with pytest.raises(laser.LaserError, match="device"):
        model.set_w8(0, "wo", second)
    monkeypatch.undo()
    model.set_w8(0, "wo", first)
    model.set_w8(0, "wo", second)
    for m in (first, second):                                              # (a captured step may still read the first)
        with pytest.raises(laser.LaserError, match="in use"):
            m.close()
    model.close()
    first.close()
    second.close()


@pytest.mark.parametrize("B, K", [(2, 3), (3, 30)])
def test_captured_steps(B, K):
    """A step and its commit, captured once and replayed as lengths grow, against eager steps of a second model with the same matrices."""
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    w8, _ = held(w)
    lens = [17 + 5 * b for b in range(B)]
    models = [laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * (K + 1), B, 512, eps=sh.eps, rope_base=sh.rope_base) for _ in range(2)]
    for model in models:
        for (layer, name), m in w8.items():
            model.set_w8(layer, name, m)
    kvs = caches(sh, lens, 8 * (K + 1), 5)
    r = np.random.default_rng(1)
    all_tokens = [i32(r.integers(0, sh.vocab, (B, K + 1))) for _ in range(6)]
    pending, drafts, n, keep = all_tokens[0][:, 0].contiguous(), all_tokens[0][:, 1:].contiguous(), i32([K] * B), i32([K] * B)
    out = [torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty((B, K + 1), dtype=torch.int32, device="cuda")]

    def both(model, kv, out):
        logits = laser.verify_step(model, kv, range(B), pending, drafts, n, 1, -1.0, want_logits=True, out=out)[-1]
        laser.kv_commit(kv, range(B), keep)
        return logits
    both(models[0], kvs[0], out)
    for b in range(B):
        kvs[0].set_len(b, lens[b])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = both(models[0], kvs[0], out)
    for b in range(B):
        kvs[0].set_len(b, lens[b])
    for tokens in all_tokens:
        pending.copy_(tokens[:, 0])
        drafts.copy_(tokens[:, 1:])
        graph.replay()
        torch.cuda.synchronize()
        want = both(models[1], kvs[1], [torch.empty_like(t) for t in out])
        kvs[1].read_lens(range(B))
        # contexts are split over workgroups by the host's bounds of their lengths, which the capture keeps: other orders of sums, after which a value may round
        # to the next code, as in test_steps_beside_other_weights
        assert float((logits - want).norm() / want.norm()) < 0.06
    assert kvs[0].read_lens(range(B)).tolist() == kvs[1].read_lens(range(B)).tolist() == [t + 6 * (K + 1) for t in lens]


def test_engine():
    from paper_2408_05676_amd.harness import Engine
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    w8, _ = held(w)
    B, K, T = 3, 5, 40
    with pytest.raises(laser.LaserError, match="not both"):
        Engine(sh, w, B, K, T + 20, w8=True, w4_group=64)
    eng = Engine(sh, w, B, K, T + 20, prefill_chunk=16, four_bit_cache=True, w8=True)
    r = np.random.default_rng(8)
    prompts = r.integers(0, sh.vocab, (B, T))
    eng.prefill(prompts)
    drafts = i32(r.integers(0, sh.vocab, (B, K)))
    tokens = torch.cat([eng.pending[:, None], drafts], 1)
    logits = step(eng.model, eng.kv, tokens, None).double().view(B * (K + 1), -1)
    x = by_operators(sh, w, w8, eng.kv, [T - 1] * B, tokens, None).double()    # the same rows again, into the same slots
    h = x * (x.square().mean(-1, keepdim=True) + sh.eps).rsqrt() * w["gf"].double()
    head = w["wlm"].double().T.contiguous()
    assert bool(((logits - h @ head).abs() <= (2.0 ** -10 + sh.d * 2.0 ** -24) * (h.abs() @ head.abs())).all())
    eng.close()
