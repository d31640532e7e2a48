"""The 8-bit building blocks without a GPU: the format, and every refusal."""
import ctypes
import math

import pytest
import torch

import fp8_oracle as F
from paper_2508_17588_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2508_17588_amd.build import BINDING_PATH, build
    if not (os.path.exists(B.LIB_PATH) and os.path.exists(BINDING_PATH)):
        build(verbose=False)
    return B.load_library()


def test_oracle_codes_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.isnan(want), torch.isnan(F.TABLE))
    fine = ~torch.isnan(want)
    assert torch.equal(want[fine], F.TABLE[fine])
    # to the nearest, ties to even, as the type's own conversion does it
    t = torch.cat([torch.linspace(-448, 448, 20001, dtype=torch.float64), F.TABLE[:126] + (F.TABLE[1:127] - F.TABLE[:126]) / 2])
    assert torch.equal(F.TABLE[F.encode(t).long()], t.float().to(torch.float8_e4m3fn).double())


def test_oracle_scales():
    y = torch.zeros(5, 256, dtype=torch.float64)
    y[0, 3], y[1, 130], y[2, 0], y[3, 5] = 448.0, 448.0000001, -3.5e-38, float("inf")
    y[4, 7], y[4, 8] = float("nan"), 1.0
    b = F.scale_bytes(y)
    assert b[0, 0] == 127 and b[0, 1] == 127 and b[1, 1] == 128 and b[3, 0] == 127
    assert b[2, 0] == 0 and b[4, 0] == 127 - 8 and b.shape == (5, 4)
    assert F.pitch(512) == 4 and F.pitch(528) == 8 and B.fp8_scale_pitch(528) == 8 and B.fp8_scale_pitch(16) == 4


P, ODD = ctypes.c_void_p(256), ctypes.c_void_p(264)


def test_quantize_refusals(lib):
    def rc(x=P, dtype=1, rows=4, cols=64, block=1, q=P, s=P):
        return lib.hero_quantize_fp8(x, dtype, rows, cols, block, q, s, None)
    assert rc(x=None) == rc(q=None) == rc(s=None) == B.HERO_ERR_INVALID_ARG
    assert rc(dtype=2) == rc(rows=-1) == rc(block=0) == rc(block=64) == B.HERO_ERR_INVALID_ARG
    assert rc(cols=0) == rc(cols=8) == rc(cols=72) == B.HERO_ERR_SHAPE
    assert b"multiple of 16" in lib.hero_last_error()
    assert rc(rows=1 << 30, cols=4096) == B.HERO_ERR_SHAPE
    assert rc(x=ODD) == rc(q=ODD) == rc(s=ctypes.c_void_p(258)) == B.HERO_ERR_INVALID_ARG
    assert rc(rows=0, x=None, q=None, s=None) == B.HERO_OK


def test_rms_refusals(lib):
    def rc(x=P, dtype=1, add=None, rows=None, n=4, hidden=64, gain=P, eps=1e-6, total=None, q=P, s=P):
        return lib.hero_gather_rms_fp8(x, dtype, add, rows, n, hidden, gain, eps, total, q, s, None)
    assert rc(x=None) == rc(gain=None) == rc(q=None) == rc(s=None) == B.HERO_ERR_INVALID_ARG
    assert rc(dtype=7) == rc(n=-1) == rc(eps=-1.0) == rc(eps=math.nan) == B.HERO_ERR_INVALID_ARG
    assert rc(hidden=8) == rc(hidden=100) == rc(hidden=16400) == rc(hidden=0) == B.HERO_ERR_SHAPE
    assert rc(x=ODD) == rc(add=ODD) == rc(gain=ODD) == rc(total=ODD) == rc(q=ODD) == B.HERO_ERR_INVALID_ARG
    assert rc(rows=ctypes.c_void_p(257)) == rc(s=ctypes.c_void_p(257)) == B.HERO_ERR_INVALID_ARG
    assert rc(rows=P, total=P) == B.HERO_ERR_INVALID_ARG and b"listed" in lib.hero_last_error()
    assert rc(total=ctypes.c_void_p(256 + 512)) == B.HERO_ERR_INVALID_ARG and b"overlap" in lib.hero_last_error()
    assert rc(n=0, x=None, q=None, s=None) == B.HERO_OK


@pytest.mark.parametrize("quantized", [False, True])
def test_linear_refusals(lib, quantized):
    def rc(a=P, sa=P, w=P, sw=P, bias=P, c=P, s=P, m=4, n=64, k=64, act=0, scratch=None, size=0):
        if quantized:
            return lib.hero_linear_fp8_quantized(a, sa, w, sw, bias, c, s, m, n, k, act, scratch, size, None)
        return lib.hero_linear_fp8(a, sa, w, sw, bias, c, m, n, k, act, scratch, size, None)
    for name in ("a", "sa", "w", "sw", "c") + (("s",) if quantized else ()):
        assert rc(**{name: None}) == B.HERO_ERR_INVALID_ARG, name
        assert rc(**{name: ctypes.c_void_p(258)}) == B.HERO_ERR_INVALID_ARG, name
    assert rc(bias=ODD) == rc(scratch=ODD, size=1 << 20) == B.HERO_ERR_INVALID_ARG
    assert rc(m=-1) == rc(n=0) == rc(k=0) == rc(act=2) == B.HERO_ERR_INVALID_ARG
    assert rc(n=24) == rc(k=40) == rc(k=8) == B.HERO_ERR_SHAPE
    assert rc(m=1 << 20, k=4096) == rc(n=1 << 20, k=4096) == B.HERO_ERR_SHAPE and b"2^32" in lib.hero_last_error()
    assert rc(m=0, a=None, sa=None, c=None, s=None) == B.HERO_OK


@pytest.mark.parametrize("m,n,k,what", [(300, 1 << 23, 16, b"2^23"), (1, (1 << 23) - 16, 16, None), (1 << 27, 1 << 20, 16, b"tiles"),
                                        (1 << 28, 16, 16, b"2^32"), ((1 << 28) - 528, 16, 16, None)])
def test_largest_products(lib, m, n, k, what):
    if what is None:
        assert B.hero_linear_fp8_route(m, n, k)
        return
    out = [ctypes.byref(ctypes.c_int32()) for _ in range(3)]
    assert lib.hero_linear_fp8_route(m, n, k, 0, 0, *out) == B.HERO_ERR_SHAPE and what in lib.hero_last_error()
    assert lib.hero_linear_fp8(P, P, P, P, P, P, m, n, k, 0, None, 0, None) == B.HERO_ERR_SHAPE and what in lib.hero_last_error()


def test_route(lib):
    t = [ctypes.c_int32() for _ in range(3)]
    p = [ctypes.byref(v) for v in t]
    assert lib.hero_linear_fp8_route(0, 64, 64, 0, 0, *p) == lib.hero_linear_fp8_route(1, 64, 64, 0, 0, None, *p[1:]) == B.HERO_ERR_INVALID_ARG
    assert lib.hero_linear_fp8_route(1, 24, 64, 0, 0, *p) == lib.hero_linear_fp8_route(1 << 20, 64, 4096, 0, 0, *p) == B.HERO_ERR_SHAPE
    for m, n, k, q in ((1, 1920, 7680, False), (17776, 7680, 1920, True), (550, 720, 3008, False), (4, 16, 1 << 20, True)):
        # without scratch nothing is cut, and a little more of it never makes a tile that does not fit
        assert B.hero_linear_fp8_route(m, n, k, q, 0)[2] in (1, -1)
        for scratch in (1 << 10, 1 << 22, 1 << 26):
            bm, bn, last = B.hero_linear_fp8_route(m, n, k, q, scratch)
            if last > 1:
                tiles = -(-m // bm) * -(-n // bn)
                assert -(-tiles // 8) * 8 % 256 * last * bm * bn * 4 <= scratch


def test_binding_refuses_what_does_not_fit(lib):
    q, s = B.empty_fp8(4, 64, device="cpu")
    x = torch.zeros(4, 64)
    assert s.shape == (4, 4) and B.empty_fp8(300, 64, 128, device="cpu")[1].shape == (3, 4)
    with pytest.raises(TypeError):
        B.hero_quantize_fp8(x, q, s)                  # not on a device
    with pytest.raises(TypeError):
        B.hero_linear_fp8(q, s, q, s, None, x)
    with pytest.raises((TypeError, ValueError)):
        B.hero_gather_rms_fp8(x, None, None, 4, torch.zeros(64, dtype=torch.bfloat16), 1e-6, q, s)
    with pytest.raises(TypeError, match="c must be a tensor|not a device tensor"):
        B.hero_linear_fp8(q, s, q, s, None, None)
    with pytest.raises(TypeError, match="x must be a tensor"):
        B.hero_quantize_fp8([1.0], q, s)
