"""Arguments of the calls on 4-bit caches and weights that must be refused, and the layouts next to them that must not."""
import pytest
import torch

import paper_2408_05676_amd as laser

pytestmark = pytest.mark.gpu

F16 = torch.float16


def normal(seed, *dims):
    return torch.empty(dims, device="cuda").normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(seed)).half()


@pytest.fixture
def step():
    B, R, H, dh = 2, 3, 2, 64
    kv = laser.KVCache4(1, H, dh, 4, B, 2)
    for b in range(B):
        kv.reserve(b, 32)
    return kv, normal(1, B, R, 2 * H, dh), normal(2, B, R, H, dh), normal(3, B, R, H, dh)


def strided(*strides, shape=(2, 3, 4, 64)):
    n = 1 + sum(s * (d - 1) for s, d in zip(strides, shape))
    return torch.zeros(n, dtype=F16, device="cuda").as_strided(shape, strides)


@pytest.mark.parametrize("strides", [(0, 256, 64, 1), (768, 0, 64, 1), (768, 256, 0, 1), (768, 64, 64, 1), (768, 256, 63, 1), (767, 256, 64, 1), (768, 255, 64, 1),
                                     (64, 128, 192, 1), (128, 128, 384, 1)])
def test_results_whose_rows_overlap(step, strides):
    kv, q, k, v = step
    out = strided(*strides)
    with pytest.raises(laser.LaserError, match="overlap"):
        laser.kv_append(kv, 0, [0, 1], k, v, q=q, q_out=out)
    laser.kv_append(kv, 0, [0, 1], k, v)
    with pytest.raises(laser.LaserError, match="overlap"):
        laser.kv_attend(kv, 0, [0, 1], q, out=out)


@pytest.mark.parametrize("strides", [(0, 256, 64, 1), (768, 0, 64, 1), (768, 256, 0, 1), (768, 64, 64, 1), (768, 256, 63, 1), (64, 128, 192, 1)])
def test_reads_into_rows_that_overlap(step, strides):
    bad, good = strided(*strides, shape=(2, 3, 2, 64)), strided(768, 256, 64, 1, shape=(2, 3, 2, 64))
    for out in ((bad, good), (good, bad)):
        with pytest.raises(laser.LaserError, match="overlap"):
            laser.kv_read(step[0], 0, [0, 1], 3, out=out)


@pytest.mark.parametrize("strides", [(768, 256, 64, 1), (64, 128, 384, 1), (64, 512, 128, 1), (1000, 300, 64, 1), (192, 64, 1000, 1), (192, 128, 1000, 1)])
def test_results_in_any_order_of_rows(step, strides):
    """The last: sequences and rows interleave (0, 128, 192, 256, 320, 448) and share nothing."""
    kv, q, k, v = step
    want_q = laser.kv_append(kv, 0, [0, 1], k, v, q=q)
    assert torch.equal(laser.kv_append(kv, 0, [0, 1], k, v, q=q, q_out=strided(*strides)), want_q)
    assert torch.equal(laser.kv_attend(kv, 0, [0, 1], q, out=strided(*strides)), laser.kv_attend(kv, 0, [0, 1], q))
    got = laser.kv_read(kv, 0, [0, 1], 3, out=tuple(strided(*strides)[:, :, :2] for _ in range(2)))
    assert all(torch.equal(a, b) for a, b in zip(got, laser.kv_read(kv, 0, [0, 1], 3)))


def test_keys_read_into_the_memory_of_the_values(step):
    kv = step[0]
    t = torch.zeros((2, 3, 2, 64), dtype=F16, device="cuda")
    with pytest.raises(laser.LaserError, match="same memory"):
        laser.kv_read(kv, 0, [0, 1], 3, out=(t, t))


def test_matrices_of_a_model(monkeypatch):
    import gc
    import weakref

    import synth
    from tests.gpu_util import gpu_weights
    sh = synth.SHAPES["tiny"]
    w = gpu_weights(sh)
    model = laser.Model(sh.n_layers, sh.d, sh.n_heads, sh.ffn, sh.vocab, w, 4, 1, 64, eps=sh.eps, rope_base=sh.rope_base)
    make = lambda: laser.W4(*laser.w4_quantize(w["wo"][0].contiguous(), 64))  # noqa: E731
    closed, first, second = make(), make(), make()
    closed.close()
    with pytest.raises(laser.LaserError, match="closed"):            # not the bf16 matrix in silence
        model.set_w4(0, "wo", closed)
    with pytest.raises(laser.LaserError, match="closed"):
        model.set_w4(0, "wo", w["wo"][0])
    with pytest.raises(laser.LaserError, match="wq"):
        model.set_w4(0, "wq", first)
    monkeypatch.setattr(second, "device", 1)
    with pytest.raises(laser.LaserError, match="device"):
        model.set_w4(0, "wo", second)
    monkeypatch.undo()
    model.set_w4(0, "wo", first)
    with pytest.raises(laser.LaserError, match="in use"):
        first.close()
    model.set_w4(0, "wo", second)
    alive = weakref.ref(first)
    del first
    gc.collect()
    assert alive() is not None and alive()._h                        # a captured step may read it
    model.set_w4(0, "wo", None)
    with pytest.raises(laser.LaserError, match="in use"):
        second.close()
    model.close()
    gc.collect()
    assert alive() is None
    second.close()
    second.close()
