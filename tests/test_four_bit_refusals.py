"""What the calls on 4-bit caches and weights refuse, before any of them touches a device."""
import ctypes as C
import os

import pytest

E_ARG, E_SHAPE, E_LIMIT = -1, -2, -5


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("seq", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


@pytest.fixture(scope="module")
def lib():
    from paper_2408_05676_amd import build as b
    if not os.path.exists(b.LIB):
        b.build(verbose=False)
    L = C.CDLL(b.LIB)
    L.laser_last_error.restype = C.c_char_p
    return L


def test_without_a_cache(lib):
    h = Heads(64, 1, 1, 1)
    ids = (C.c_int32 * 1)(0)
    assert lib.laser_kv_append(None, 0, ids, None, None, 1, 1, 0, C.byref(h), C.byref(h), None, None, 0, None, 0, 0, None) == E_ARG
    assert lib.laser_kv_attend(None, 0, ids, None, None, 1, 1, 1, 0, C.byref(h), C.c_float(1), C.byref(h), None) == E_ARG
    assert lib.laser_kv_read(None, 0, ids, 1, 0, 1, 0, C.byref(h), C.byref(h), None) == E_ARG
    assert b"kv is NULL" in lib.laser_last_error()
    out = C.c_void_p()
    assert lib.laser_kv_create_4bit(None, None, C.byref(out)) == E_ARG


@pytest.mark.parametrize("field, value, code", [("page_size", 32, E_SHAPE), ("head_dim", 96, E_SHAPE), ("n_heads", 0, E_ARG), ("n_pages", 0, E_ARG),
                                                ("max_seqs", 0, E_ARG), ("max_pages_per_seq", 0, E_ARG), ("n_layers", -1, E_ARG)])
def test_cache_shapes(lib, field, value, code):
    class Desc(C.Structure):
        _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_heads", "head_dim", "page_size", "n_pages", "max_seqs", "max_pages_per_seq")]
    d = Desc(1, 2, 64, 16, 4, 1, 4)
    setattr(d, field, value)
    out = C.c_void_p()
    assert lib.laser_kv_create_4bit(C.byref(d), None, C.byref(out)) == code and not out.value


@pytest.mark.parametrize("N, Kd, group, code", [(16, 128, 16, E_SHAPE), (16, 128, 256, E_SHAPE), (16, 96, 64, E_SHAPE), (16, 0, 32, E_ARG), (0, 128, 32, E_ARG),
                                                (-1, 128, 32, E_ARG), (16, 100, 32, E_SHAPE), (2 ** 31 - 1, 2 ** 31 - 128, 128, E_LIMIT),
                                                (2 ** 27, 128, 128, E_LIMIT), (16, 2 ** 30, 32, E_LIMIT)])
def test_weight_shapes(lib, N, Kd, group, code):
    out, p = C.c_void_p(), C.c_void_p(64)
    assert lib.laser_w4_create(p, p, p, N, Kd, group, None, C.byref(out)) == code and not out.value
    assert lib.laser_w4_quantize(p, N, Kd, group, p, p, p, None) == code


def test_null_and_misaligned_arguments(lib):
    out, p = C.c_void_p(), C.c_void_p(64)
    assert lib.laser_w4_create(None, p, p, 16, 128, 32, None, C.byref(out)) == E_ARG
    assert lib.laser_w4_create(p, p, p, 16, 128, 32, None, None) == E_ARG
    assert lib.laser_w4_create(p, C.c_void_p(65), p, 16, 128, 32, None, C.byref(out)) == E_ARG
    assert lib.laser_w4_matmul(None, p, C.c_int64(128), 1, 0, p, C.c_int64(16), None) == E_ARG
    assert lib.laser_w4_destroy(None) == 0
    assert lib.laser_model_set_w4(None, 0, 0, None) == E_ARG
    assert lib.laser_rope_table(None, 4, 64, C.c_double(1e4), None) == E_ARG
    assert lib.laser_rope_table(p, 2 ** 27, 64, C.c_double(1e4), None) == E_LIMIT
    for size, dim, base in ((0, 64, 1e4), (4, 63, 1e4), (4, 0, 1e4), (4, 64, 0.0)):
        assert lib.laser_rope_table(p, size, dim, C.c_double(base), None) == E_ARG


def test_binding_refuses_host_tensors_and_wrong_types():
    import torch

    import paper_2408_05676_amd as laser
    w = torch.zeros(16, 128, dtype=torch.bfloat16)
    with pytest.raises(laser.LaserError):
        laser.w4_quantize(w)
    with pytest.raises(laser.LaserError):
        laser.W4(torch.zeros(16, 64, dtype=torch.uint8), torch.zeros(16, 4, dtype=torch.float16), torch.zeros(16, 4, dtype=torch.float16))
    with pytest.raises(laser.LaserError):
        laser.W4(torch.zeros(16, 64, dtype=torch.uint8), torch.zeros(16, 4, dtype=torch.float16), torch.zeros(16, 3, dtype=torch.float16))
    with pytest.raises(laser.LaserError, match="KVCache4"):
        laser.kv_append(object(), 0, [0], torch.zeros(1, 1, 2, 64), torch.zeros(1, 1, 2, 64))
    with pytest.raises(laser.LaserError, match="KVCache4"):
        laser.kv_attend(object(), 0, [0], torch.zeros(1, 1, 2, 64))
