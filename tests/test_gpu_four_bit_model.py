"""Steps of models with 4-bit weights and caches at the widths and rows whose tiles the small models do not reach, and at 128 channels a head."""
import numpy as np
import pytest
import torch

import paper_2408_05676_amd as laser
import synth
from tests import four_bit_ref as ref
from tests import test_gpu_four_bit as base
from tests.gpu_util import ATOL, RTOL, gpu_weights, logits_close

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("B, K, tree", [(2, 4, False), (2, 4, True), (1, 0, False), (1, 2, True), (5, 7, True), (3, 40, False)])
def test_steps_on_a_four_bit_cache_at_128_channels(B, K, tree, monkeypatch):
    monkeypatch.setitem(synth.SHAPES, "tiny", synth.SHAPES["tiny128"])
    base.test_model_steps_on_a_four_bit_cache(B, K, tree)


@pytest.mark.parametrize("B, K, tree, four_bit_cache, which", [(2, 4, False, True, "wqkv wo wgu wdown"), (1, 0, True, True, "wqkv wo wgu wdown"),
                                                              (4, 10, True, True, "wo wdown"), (3, 40, False, False, "wqkv wo wgu wdown")])
def test_steps_with_four_bit_weights_at_128_channels(B, K, tree, four_bit_cache, which, monkeypatch):
    monkeypatch.setitem(synth.SHAPES, "tiny", synth.SHAPES["tiny128"])
    base.test_model_steps_with_four_bit_weights(B, K, tree, four_bit_cache, which)


WIDTHS = {"7b": dict(n_layers=1, d=4096, n_heads=32, ffn=11008, vocab=1040), "1b": dict(n_layers=1, d=2048, n_heads=16, ffn=8192, vocab=1040)}


@pytest.fixture(scope="module")
def wide():
    made = {}

    def get(name):
        if name not in made:
            made.clear()
            sh = synth.SHAPES["tiny"].with_(**WIDTHS[name])
            made[name] = sh, gpu_weights(sh)
        return made[name]
    yield get
    made.clear()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("B, K", [(2, 3), (3, 7), (4, 9), (8, 8), (10, 16)])
@pytest.mark.parametrize("width", ["7b", "1b"])
def test_every_projection_of_a_wide_layer(wide, width, B, K, group):
    """8 to 170 rows: gate and up tiles that share a wave in pairs and in fours, sums added to the residual, of every tile shape of the products."""
    sh, w = wide(width)
    R, lens = K + 1, [5 + 3 * b for b in range(B)]
    model = laser.Model(1, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * R, B, 128, eps=sh.eps, rope_base=sh.rope_base)
    what = dict(w)
    for name in ("wqkv", "wo", "wgu", "wdown"):
        codes, s, m = laser.w4_quantize(w[name][0].contiguous(), group)
        model.set_w4(0, name, laser.W4(codes, s, m))
        what[name] = ref.values(torch.stack([codes & 15, codes >> 4], -1).flatten(1).double(), s, m)[None]
    kv = base.make_kv(B, sh.n_heads, sh.head_dim, lens, R)
    base.fill(kv, lens, sh.n_heads, sh.head_dim, base.gen(50 + K))
    r = np.random.default_rng(B)
    tokens = i32(r.integers(0, sh.vocab, (B, R)))
    logits = laser.verify_step(model, kv, range(B), tokens[:, 0].contiguous(), tokens[:, 1:].contiguous(), i32([K] * B), 2, 0.1, 0, want_logits=True)[-1]
    want, worst = base.reference_step(what, sh, kv, lens, tokens, None)
    ok, err, rel = logits_close(logits.cpu().double().numpy(), want.cpu().numpy())
    assert ok, (err, rel)
    assert worst <= 0.5 + 3 * 15 * 2.0 ** -11, worst
    model.close()


@pytest.mark.parametrize("shape", ["tiny", "tiny128"])
def test_generated_texts_part_only_where_two_tokens_are_close(shape):
    """laser_generate with right drafts against one-token steps, all greedy: the first token that differs is one whose logit and the next's are
    within what two paths may differ by (each the tolerance off the 64-bit logits)."""
    sh = synth.SHAPES[shape]
    w = gpu_weights(sh)
    w["gf"] = w["gf"] * 5
    B, T, new = 3, 24, 40
    prompt = np.random.default_rng(4).integers(0, sh.vocab, (B, T))
    none, zero = torch.empty((B, 0), dtype=torch.int32, device="cuda"), i32([0] * B)

    def start(K):
        model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, B * (K + 1), B, 512, eps=sh.eps, rope_base=sh.rope_base)
        kv = base.make_kv(B, sh.n_heads, sh.head_dim, [T] * B, new + K + 2, layers=sh.n_layers)
        for t in range(T - 1):
            acc, *_ = laser.verify_step(model, kv, range(B), i32(prompt[:, t]), none, zero, 1, -1.0)
            laser.kv_commit(kv, range(B), acc)
            kv.read_lens(range(B))
        return model, kv
    model, kv = start(0)
    pending, plain, gaps, bounds, every = i32(prompt[:, -1]), [], [], [], []
    for _ in range(new):
        acc, out, logits = laser.verify_step(model, kv, range(B), pending, none, zero, 1, -1.0, 0, want_logits=True)
        laser.kv_commit(kv, range(B), acc)
        kv.read_lens(range(B))
        every.append(logits[:, 0].double().cpu().numpy())
        top = logits[:, 0].double().topk(2, -1)
        pending = out[:, 0].contiguous()
        assert torch.equal(pending.long(), top.indices[:, 0])
        plain.append(pending.cpu().numpy())
        gaps.append((top.values[:, 0] - top.values[:, 1]).cpu().numpy())
        bounds.append(4 * (ATOL + RTOL * top.values.abs().amax(-1)).cpu().numpy())
    plain, gaps, bounds = (np.stack(x, 1) for x in (plain, gaps, bounds))
    for K in (0, 4, 9):
        model, kv = start(K)
        pool = laser.Pool(plain.reshape(-1).astype(np.int32), np.arange(B + 1) * new, np.arange(B), 3) if K else None
        text, n, *_ = laser.generate(model, kv, pool, range(B), torch.arange(B, dtype=torch.int64, device="cuda"), i32(prompt[:, -3:]), i32(prompt[:, -1]),
                                     K, 1, 1, -1.0, 0, max_new_tokens=new)
        text = text.cpu().numpy()
        assert n.tolist() == [new] * B
        for b in range(B):
            differ = np.flatnonzero(text[b] != plain[b])
            if K == 0:
                assert not differ.size
            elif differ.size:
                assert gaps[b, differ[0]] <= bounds[b, differ[0]], (K, b, differ[0], gaps[b, differ[0]])
    # and every position's logits, with the same text before it
    rows = np.concatenate([prompt[:, -1:], plain], 1)
    for K in (4, 9):
        model, kv = start(K)
        for t in range(0, new - K, K + 1):
            drafts = i32(rows[:, t + 1:t + K + 1])
            logits = laser.verify_step(model, kv, range(B), i32(rows[:, t]), drafts, i32([K] * B), 1, -1.0, 0, want_logits=True)[-1].double().cpu().numpy()
            one = np.stack(every[t:t + K + 1], 1)
            assert (np.abs(logits - one) <= 2 * (ATOL + RTOL * np.abs(one))).all(), (K, t)
            laser.kv_commit(kv, range(B), i32([K] * B))
            kv.read_lens(range(B))
