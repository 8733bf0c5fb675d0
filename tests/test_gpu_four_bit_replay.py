"""Captured steps on paged caches whose lengths grow under replays, past what is reserved: other sequences keep their tokens."""
import numpy as np
import pytest
import torch

import paper_2408_05676_amd as laser
import synth
from tests import four_bit_ref as ref
from tests.gpu_util import gpu_weights

pytestmark = pytest.mark.gpu

F16, F32 = torch.float16, torch.float32


def normal(seed, *dims):
    return torch.empty(dims, device="cuda").normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(seed)).half()


def capture(f):
    """f has run once (what it allocates, it has)."""
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f()
    return graph


def small_cache(make, layers, H, dh):
    """Two sequences, two pages each at most, the second's behind the first's in the table: sequence 0 holds 3 tokens, 1 all its 32."""
    kv = make(layers, H, dh, 4, 2, 2)
    kv.reserve(0, 32)
    kv.reserve(1, 32)
    for layer in range(layers):
        for b in (0, 1):
            kv.import_layer(b, layer, normal(10 * layer + b, 32, H, dh), normal(100 + 10 * layer + b, 32, H, dh))
    kv.set_len(0, 3)
    kv.set_len(1, 25)
    return kv


def contents(kv, layers, seq=1):
    return [t for layer in range(layers) for t in laser.kv_read(kv, layer, [seq], 32, start=0, dtype=F32)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


PARENT, ACCEPT, PATH = [[-1, -1, 1, 1, 3]], [3], [[1, 3, 4, -1, -1]]         # nodes 1, 3 and 4 of the tree's five: four tokens more a step


@pytest.mark.parametrize("dh", [64, 128])
def test_appends_and_tree_commits(dh):
    H = 2
    kv, twin = (small_cache(laser.KVCache4, 1, H, dh) for _ in range(2))
    before = contents(kv, 1)
    k, v, parent, accept, path = normal(3, 1, 6, H, dh), normal(4, 1, 6, H, dh), i32(PARENT), i32(ACCEPT), i32(PATH)

    def step(kv):
        laser.kv_append(kv, 0, [0], k, v, tree_parent=parent)
        laser.kv_commit_tree(kv, [0], accept, path)
    step(kv)
    kv.set_len(0, 3)
    graph = capture(lambda: step(kv))
    for _ in range(5):                                           # slots 3 .. 22 and one step's rows: within the 32
        graph.replay()
        step(twin)
        twin.read_lens([0])                                      # (the host's bound back to the length)
    torch.cuda.synchronize()
    assert kv.read_lens([0]).tolist() == [23]
    assert all(torch.equal(a[:, :23], b[:, :23]) for a, b in zip(contents(kv, 1, 0), contents(twin, 1, 0)))
    moved = [0, 2, 4, 5]                                         # rows of the accepted branch, behind one another
    assert torch.equal(contents(kv, 1, 0)[1][0, 19:23], ref.held(v[0, moved]).float())
    for _ in range(20):                                          # to slot 103: past the reservation, the table's row and the table
        graph.replay()
    torch.cuda.synchronize()
    assert kv.read_lens([0, 1]).tolist() == [103, 25]
    kv.set_len(0, 0)
    assert all(torch.equal(a, b) for a, b in zip(before, contents(kv, 1)))


def test_released_slots_and_later_reservations():
    """A replayed append goes by what is reserved as it runs: nothing for a released slot, whose pages are another sequence's now."""
    H, dh = 2, 64
    kv = laser.KVCache4(1, H, dh, 3, 2, 3)
    kv.reserve(0, 16)
    k, v = normal(5, 1, 4, H, dh), normal(6, 1, 4, H, dh)
    run = lambda: laser.kv_append(kv, 0, [0], k, v)  # noqa: E731
    run()
    graph = capture(run)
    kv.release(0)
    kv.reserve(1, 48)                                            # all pages
    kv.import_layer(1, 0, normal(7, 48, H, dh), normal(8, 48, H, dh))
    kv.set_len(1, 48)
    before = laser.kv_read(kv, 0, [1], 48, start=0, dtype=F32)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, laser.kv_read(kv, 0, [1], 48, start=0, dtype=F32)))
    kv.release(1)
    kv.reserve(0, 40)
    kv.set_len(0, 30)                                            # slots that the capture's reservation did not have
    graph.replay()
    rk, rv = laser.kv_read(kv, 0, [0], 4, dtype=F32)
    assert torch.equal(rk, ref.held(k).float()) and torch.equal(rv, ref.held(v).float())


def test_tree_steps_of_a_model_on_a_four_bit_cache():
    sh = synth.SHAPES["tiny"]
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, gpu_weights(sh), 6, 1, 512, eps=sh.eps, rope_base=sh.rope_base)
    kv = small_cache(laser.KVCache4, sh.n_layers, sh.n_heads, sh.head_dim)
    before = contents(kv, sh.n_layers)
    r = np.random.default_rng(1)
    tokens, n, pending = i32(r.integers(0, sh.vocab, (1, 5))), i32([5]), i32([7])
    parent, accept, path = i32(PARENT), i32(ACCEPT), i32(PATH)

    def step():
        laser.verify_tree(model, kv, [0], pending, tokens, parent, n, 2, 0.1, 0)
        laser.kv_commit_tree(kv, [0], accept, path)
    step()
    kv.set_len(0, 3)
    graph = capture(step)
    for _ in range(25):
        graph.replay()
    torch.cuda.synchronize()
    assert kv.read_lens([0, 1]).tolist() == [103, 25]
    kv.set_len(0, 0)
    assert all(torch.equal(a, b) for a, b in zip(before, contents(kv, sh.n_layers)))


def test_tree_commits_on_a_cache_of_sixteen_bits():
    """The commit alone (its step's lengths stay within the reservation): what sequence 1 answers does not change."""
    sh = synth.SHAPES["tiny"]
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, gpu_weights(sh), 6, 1, 512, eps=sh.eps, rope_base=sh.rope_base)
    kv = small_cache(laser.KVCache, sh.n_layers, sh.n_heads, sh.head_dim)
    r = np.random.default_rng(1)
    tokens, n, pending = i32(r.integers(0, sh.vocab, (1, 5))), i32([5]), i32([7])
    parent, accept, path = i32(PARENT), i32(ACCEPT), i32(PATH)
    answer = lambda: laser.verify_tree(model, kv, [1], pending, tokens, parent, n, 2, 0.1, 0, want_logits=True)[-1].clone()  # noqa: E731
    want = answer()
    laser.verify_tree(model, kv, [0], pending, tokens, parent, n, 2, 0.1, 0)
    graph = capture(lambda: laser.kv_commit_tree(kv, [0], accept, path))
    for _ in range(25):
        graph.replay()
    torch.cuda.synchronize()
    assert kv.read_lens([0, 1]).tolist() == [103, 25]
    kv.set_len(0, 0)
    assert torch.equal(answer(), want)


@pytest.mark.parametrize("same_stream", [False, True])
def test_captured_commits_keep_their_sequences(same_stream):
    """Calls for other sequences on the same handle come in between, more of them than the host stages lists of ids for."""
    H, dh = 1, 64
    kv = laser.KVCache4(1, H, dh, 6, 3, 2)
    for s in range(3):
        kv.reserve(s, 32)
    k, none, two = normal(9, 1, 2, H, dh), i32([-1]), i32([1])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        def step(s, accept):
            laser.kv_append(kv, 0, [s], k, k)
            laser.kv_commit(kv, [s], accept)
        step(0, none)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream if same_stream else None):
            step(0, two)
        assert kv.read_lens([0, 1, 2]).tolist() == [0, 0, 0]
        step(0, none)                                            # what the capture staged was not copied by it
        for rounds in range(3):
            graph.replay()
            assert kv.read_lens([0, 1, 2]).tolist() == [2 * rounds + 2, 0, 0]
            for i in range(70):
                step(1 + i % 2, none)
                kv.read_lens([1, 2])
            step(1, none)
            graph.replay()                                       # must not change the ids that the next call finds staged
            kv.set_len(0, 2 * rounds + 2)
            step(1, two)
            assert kv.read_lens([0, 1, 2]).tolist() == [2 * rounds + 2, 2, 0]
            kv.set_len(1, 0)
        stream.synchronize()
