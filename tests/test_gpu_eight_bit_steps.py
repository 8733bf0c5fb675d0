"""Steps of models with 8-bit weights at the widths and rows whose kernels the small models do not reach, beside products split along their inputs, and generated texts."""
import numpy as np
import pytest
import torch

import paper_2408_05676_amd as laser
import synth
from tests import test_gpu_four_bit as four
from tests.gpu_util import gpu_weights
from tests.test_gpu_eight_bit_model import by_operators, caches, held, i32, step, tree_or_chain

pytestmark = pytest.mark.gpu

WIDTHS = {"7b": dict(n_layers=1, d=4096, n_heads=32, ffn=11008, vocab=1040), "1b": dict(n_layers=1, d=2048, n_heads=16, ffn=5632, vocab=1040)}


@pytest.fixture(scope="module")
def wide():
    made = {}

    def get(name):
        if name not in made:
            made.clear()
            sh = synth.SHAPES["tiny"].with_(**WIDTHS[name])
            w = gpu_weights(sh)
            made[name] = sh, w, held(w)[0]
        return made[name]
    yield get
    made.clear()


def with_w8(sh, w, w8, rows, B, **options):
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, rows, B, 512, eps=sh.eps, rope_base=sh.rope_base)
    for k, v in options.items():
        model.set_option(k, v)
    for (layer, name), m in w8.items():
        model.set_w8(layer, name, m)
    return model


def same_as_its_operators(sh, w, w8, B, K, tree):
    """The first layer's cache bit for bit. The step rounds attention's last product to fp16 at once, the operator and .half() by way of fp32: these differ for 2^-13 of the
    elements, by a step of 2^-11, which takes 127 |x| / max 2^-11 = some 0.014 of those to the next code, d 2^-13 0.014 = 0.0004 (256 elements) to 0.007 (4096) of the
    rows: a count that comes to a hundredth of them at most on average, held to that, five deviations of such a count and three. Such a code moves its row by 0.035 (4.5
    standard deviations / 127) of an element's deviation, 0.0022 (256) to 0.0005 of its norm, and what a tensor is off by takes 127 |x| / max = 28 times as many of the next
    one's codes to their neighbours, 1 to 6 %, and so on: in the end up to what the rounding of all the codes amounts to, 0.03 (see test_steps_beside_other_weights), held to
    twice that, in four-bit caches as in logits. A second layer's attention carries it to the rows of the same sequence. The other rows' logits are off by the head's input in
    fp16 (2^-11 / sqrt 3 of its norm) and the order of fp32 sums, held to 2^-10."""
    r = np.random.default_rng(K)
    M, lens = B * (K + 1), [20 + 9 * b % 97 for b in range(B)]
    some = 0.01 * M + 5 * (0.01 * M) ** 0.5 + 3
    model = with_w8(sh, w, w8, M, B)
    kv, twin = caches(sh, lens, K + 1, 7)
    tokens, parent = i32(r.integers(0, sh.vocab, (B, K + 1))), tree_or_chain(r, B, K, tree)
    logits = step(model, kv, tokens, parent).double().view(M, -1)
    x = by_operators(sh, w, w8, twin, lens, tokens, parent).double()
    moved = torch.zeros(B, dtype=torch.bool, device="cuda")                     # sequences whose caches have such rows
    for layer in range(sh.n_layers):
        for a, b in zip(laser.kv_read(kv, layer, range(B), K + 1), laser.kv_read(twin, layer, range(B), K + 1)):
            a, b = a.double().view(M, -1), b.double().view(M, -1)
            differ = (a != b).any(-1)
            assert int(differ.sum()) <= (some if layer else 0)
            assert float(((a - b).norm(dim=-1) / b.norm(dim=-1)).max()) < 0.06
            moved |= differ.view(B, -1).any(-1)
    h = x * (x.square().mean(-1, keepdim=True) + sh.eps).rsqrt() * w["gf"].double()
    want = h @ w["wlm"].double().T.contiguous()
    off = (logits - want).norm(dim=-1) / want.norm(dim=-1)
    assert float(off.max()) < 0.06
    assert int((off.view(B, -1)[~moved] > 2.0 ** -10).sum()) <= some
    model.close()


@pytest.mark.parametrize("B, K, tree", [(1, 0, False), (2, 4, True), (3, 10, False), (5, 7, True), (3, 40, False), (6, 63, True)])
def test_a_step_is_its_operators_at_128_channels(B, K, tree):
    sh = synth.SHAPES["tiny128"]
    w = gpu_weights(sh)
    same_as_its_operators(sh, w, held(w)[0], B, K, tree)


@pytest.mark.parametrize("B, K, tree", [(1, 0, False), (1, 8, False), (2, 7, True), (3, 7, False), (4, 9, False), (8, 8, True), (10, 16, False), (16, 15, False), (64, 10, False)])
@pytest.mark.parametrize("width", ["7b", "1b"])
def test_every_projection_of_a_wide_layer(wide, width, B, K, tree):
    """1 to 704 rows: kernels of few rows, tiles, norms and rows of one wave to sixteen."""
    same_as_its_operators(*wide(width), B, K, tree)


@pytest.mark.parametrize("B, K", [(3, 10), (4, 31), (5, 63)])
@pytest.mark.parametrize("four_bit_cache", [False, True])
def test_beside_products_split_along_their_inputs(B, K, four_bit_cache):
    """O and down projections in bf16 whose inputs are split into 1, 2 and 4 parts: the norm before an 8-bit product adds them up. Parts are fp32 sums in another order: a
    value of the residual stream moves by some 2^-22 of itself, and a code with it where it was that close to a half: 127 2^-21 of the 256 of a row, one row in sixty, by
    0.035 / 16 = 0.0022 of the row's norm. 0.01 for a row is several of them; a part that is missing, or added twice, is of the size of the row."""
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    w8, _ = held(w, ("wqkv", "wgu"))
    r = np.random.default_rng(K)
    lens = [20 + 9 * b for b in range(B)]
    tokens, results, keys = i32(r.integers(0, sh.vocab, (B, K + 1))), [], []
    for parts in (1, 2, 4):
        model = with_w8(sh, w, w8, B * (K + 1), B, ksplit_o=parts, ksplit_down=parts)
        kv, = caches(sh, lens, K + 1, 9, n=1)
        if not four_bit_cache:
            plain = laser.KVCache(sh.n_layers, sh.n_heads, sh.head_dim, 200, B, 40)
            for b in range(B):
                plain.reserve(b, lens[b] + K + 1)
                for layer in range(sh.n_layers):
                    k, v = laser.kv_read(kv, layer, [b], lens[b], start=0)
                    plain.import_layer(b, layer, k[0], v[0])
                plain.set_len(b, lens[b])
            kv = plain
        results.append(step(model, kv, tokens, None).double().flatten(0, 1))
        if four_bit_cache:
            keys.append(laser.kv_read(kv, 1, range(B), K + 1)[0].double().flatten(0, 1).flatten(1))
        model.close()
    assert B * (K + 1) <= 80 or not torch.equal(results[0], results[2])          # (the split took place)
    for other in results[1:]:
        off = (other - results[0]).norm(dim=-1) / results[0].norm(dim=-1)
        assert float(off.max()) < 0.01
    for other in keys[1:]:                                                       # four bits: a code of these is a fifteenth of its group
        assert float((other - keys[0]).norm() / keys[0].norm()) < 0.01


@pytest.mark.parametrize("four_bit_cache", [False, True])
@pytest.mark.parametrize("shape", ["tiny", "tiny128"])
def test_generated_texts_part_only_where_two_tokens_are_close(shape, four_bit_cache):
    """laser_generate with right drafts against one-token steps, all greedy. Products are sums of integers and rows have codes of their own, so that other rows beside one change
    the order of attention's and the head's sums alone. A code may then be the next one: 0.0022 of a row's norm (see above), in some of eight tensors, and again where the
    cache holds such a row: 0.006 of the head's input, which is 0.006 of the logits' deviation for each, 4.5 times that for the furthest of 2048: 0.03; two logits may both be off."""
    sh = synth.SHAPES[shape]
    w = gpu_weights(sh)
    w["gf"] = w["gf"] * 5
    w8, _ = held(w)
    B, T, new = 3, 24, 40
    prompt = np.random.default_rng(4).integers(0, sh.vocab, (B, T))
    none, zero = torch.empty((B, 0), dtype=torch.int32, device="cuda"), i32([0] * B)

    def start(K):
        model = with_w8(sh, w, w8, B * (K + 1), B)
        if four_bit_cache:
            kv = four.make_kv(B, sh.n_heads, sh.head_dim, [T] * B, new + K + 2, layers=sh.n_layers)
        else:
            kv = laser.KVCache(sh.n_layers, sh.n_heads, sh.head_dim, 60, B, 20)
            for b in range(B):
                kv.reserve(b, T + new + K + 2)
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
        bounds.append(0.06 * logits[:, 0].double().std(-1).cpu().numpy())
    plain, gaps, bounds = (np.stack(x, 1) for x in (plain, gaps, bounds))
    assert np.median(gaps / bounds) > 1                                    # (most tokens are not close)
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
                assert gaps[b, differ[0]] <= bounds[b, differ[0]], (K, b, differ[0], gaps[b, differ[0]], bounds[b, differ[0]])
    rows = np.concatenate([prompt[:, -1:], plain], 1)                      # and every position's logits, with the same text before it
    for K in (4, 9):
        model, kv = start(K)
        for t in range(0, new - K, K + 1):
            drafts = i32(rows[:, t + 1:t + K + 1])
            logits = laser.verify_step(model, kv, range(B), i32(rows[:, t]), drafts, i32([K] * B), 1, -1.0, 0, want_logits=True)[-1].double().cpu().numpy()
            one = np.stack(every[t:t + K + 1], 1)
            assert (np.abs(logits - one).max(-1) <= 0.06 * one.std(-1)).all(), (K, t, (np.abs(logits - one).max(-1) / one.std(-1)).max())
            laser.kv_commit(kv, range(B), i32([K] * B))
            kv.read_lens(range(B))


@pytest.mark.parametrize("B, K", [(2, 3), (3, 30), (8, 40)])
def test_captured_steps_are_eager_steps(B, K):
    """A step captured and replayed at the lengths it was captured at, with other tokens each time: bit for bit the eager step's logits and cache (the host's bounds of the
    lengths, by which contexts are split, are the same)."""
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    w8, _ = held(w)
    lens = [17 + 5 * b for b in range(B)]
    models = [with_w8(sh, w, w8, B * (K + 1), B) for _ in range(2)]
    kvs = caches(sh, lens, K + 1, 5)
    r = np.random.default_rng(1)
    every = [i32(r.integers(0, sh.vocab, (B, K + 1))) for _ in range(5)]
    pending, drafts, n = every[0][:, 0].contiguous(), every[0][:, 1:].contiguous(), i32([K] * B)
    run = lambda model, kv: laser.verify_step(model, kv, range(B), pending, drafts, n, 1, -1.0, want_logits=True)[-1]  # noqa: E731
    run(models[0], kvs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = run(models[0], kvs[0])
    for tokens in every:
        pending.copy_(tokens[:, 0])
        drafts.copy_(tokens[:, 1:])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(run(models[1], kvs[1]), logits)
        for layer in range(sh.n_layers):
            assert all(torch.equal(a, b) for a, b in zip(*(laser.kv_read(kv, layer, range(B), K + 1) for kv in kvs)))
