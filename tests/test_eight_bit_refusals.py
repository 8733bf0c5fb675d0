"""What the calls on rows and weights in 8-bit integers refuse, before any of them touches a device."""
import ctypes as C
import os

import pytest

E_ARG, E_SHAPE, E_LIMIT = -1, -2, -5
I64, F32 = C.c_int64, C.c_float


@pytest.fixture(scope="module")
def lib():
    from paper_2408_05676_amd import build as b
    if not os.path.exists(b.LIB):
        b.build(verbose=False)
    L = C.CDLL(b.LIB)
    L.laser_last_error.restype = C.c_char_p
    return L


P = [C.c_void_p(k << 20) for k in range(1, 8)]                    # addresses far from each other, never used


def rows(lib, x=P[0], step=64, M=4, N=64, dtype=0, codes=P[1], cs=128, scales=P[2]):
    return lib.laser_q8_rows(x, I64(step), M, N, dtype, codes, I64(cs), scales, None)


def norm(lib, x=P[0], step=64, dtype=0, res=P[1], rs=64, ro=P[1], ros=64, rdt=0, gain=P[2], eps=1e-6, M=4, N=64, codes=P[3], cs=128, scales=P[4]):
    return lib.laser_q8_norm(x, I64(step), dtype, res, I64(rs), ro, I64(ros), rdt, gain, F32(eps), M, N, codes, I64(cs), scales, None)


def at(p, n):
    return C.c_void_p(p.value + n)


@pytest.mark.parametrize("bad", [dict(x=None), dict(codes=None), dict(scales=None), dict(dtype=3), dict(dtype=-1), dict(M=-1), dict(M=65535 * 32 + 1), dict(N=0),
                                 dict(N=2 ** 30 + 1), dict(step=-1), dict(cs=63), dict(cs=2 ** 36), dict(step=2 ** 36), dict(x=at(P[0], 1)), dict(scales=at(P[2], 2)),
                                 dict(codes=P[0]), dict(codes=at(P[0], 500)), dict(scales=at(P[1], 400)), dict(scales=P[0])])
def test_rows(lib, bad):
    assert rows(lib, **bad) == E_ARG


@pytest.mark.parametrize("bad", [dict(gain=None), dict(gain=at(P[2], 2)), dict(res=None), dict(ro=None), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                 dict(rdt=1), dict(rdt=3), dict(dtype=2), dict(rs=-1), dict(ros=63), dict(ros=128), dict(ro=at(P[1], 2)), dict(ro=P[0], ros=128),
                                 dict(res=at(P[1], 1)), dict(ro=P[2], ros=64), dict(ro=P[3]), dict(ro=P[4]), dict(codes=P[1]), dict(codes=P[2]), dict(scales=P[2]),
                                 dict(ro=P[0], rdt=2)])
def test_norm(lib, bad):
    assert norm(lib, **bad) == E_ARG


def test_read(lib):
    def read(codes=P[0], cs=128, scales=P[1], M=4, N=64, dtype=0, out=P[2], os=64):
        return lib.laser_q8_read(codes, I64(cs), scales, M, N, dtype, out, I64(os), None)
    for bad in (dict(codes=None), dict(scales=None), dict(out=None), dict(dtype=3), dict(M=-1), dict(N=0), dict(cs=-1), dict(os=63), dict(out=at(P[2], 1)),
                dict(scales=at(P[1], 1)), dict(out=P[0]), dict(out=P[1])):
        assert read(**bad) == E_ARG, bad


@pytest.mark.parametrize("N, Kd, gated, code", [(0, 128, 0, E_ARG), (16, 0, 0, E_ARG), (-1, 128, 0, E_ARG), (16, 2 ** 17, 0, E_LIMIT), (2 ** 27, 128, 0, E_LIMIT),
                                                (2 ** 31 - 1, 2 ** 17 - 1, 0, E_LIMIT), (17, 128, 1, E_SHAPE), (16, 128, 2, E_ARG), (16, 128, -1, E_ARG)])
def test_weights(lib, N, Kd, gated, code):
    out = C.c_void_p()
    assert lib.laser_w8_create(P[0], P[1], N, Kd, gated, None, C.byref(out)) == code and not out.value
    if gated == 0:
        assert lib.laser_w8_quantize(P[0], N, Kd, P[1], P[2], None) == code


def test_null_and_misaligned_arguments(lib):
    out = C.c_void_p()
    assert lib.laser_w8_create(None, P[1], 16, 128, 0, None, C.byref(out)) == E_ARG
    assert lib.laser_w8_create(P[0], None, 16, 128, 0, None, C.byref(out)) == E_ARG
    assert lib.laser_w8_create(P[0], P[1], 16, 128, 0, None, None) == E_ARG
    assert lib.laser_w8_create(P[0], at(P[1], 2), 16, 128, 0, None, C.byref(out)) == E_ARG
    assert lib.laser_w8_quantize(P[0], 16, 128, None, P[2], None) == E_ARG
    assert lib.laser_w8_quantize(at(P[0], 1), 16, 128, P[1], P[2], None) == E_ARG
    assert lib.laser_w8_destroy(None) == 0
    assert lib.laser_w8_matmul(None, P[0], I64(128), P[1], 1, 0, P[2], I64(16), None) == E_ARG
    assert b"w is NULL" in lib.laser_last_error()


def test_nothing_to_do(lib):
    assert rows(lib, M=0, x=None, codes=None, scales=None) == 0
    assert norm(lib, M=0, x=None, codes=None, scales=None, gain=None) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    import torch

    import paper_2408_05676_amd as laser
    x = torch.zeros(4, 64, dtype=torch.float16)
    for call in (lambda: laser.q8_rows(x), lambda: laser.q8_rows(x.double()), lambda: laser.q8_rows(x[0]), lambda: laser.q8_norm(x, torch.ones(64)),
                 lambda: laser.q8_read(x.to(torch.int8), torch.zeros(4)), lambda: laser.w8_quantize(x.bfloat16()), lambda: laser.w8_matmul(object(), x, x),
                 lambda: laser.W8(x.to(torch.int8), torch.zeros(4)), lambda: laser.W8(x.to(torch.int8), torch.zeros(3))):
        with pytest.raises(laser.LaserError):
            call()
