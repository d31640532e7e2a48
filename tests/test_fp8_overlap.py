"""Outputs of the 8-bit building blocks that overlap what a call still reads are refused before anything is launched."""
import ctypes

import pytest
import torch

from paper_2508_17588_amd import binding as B

AT = 1 << 20                           # where the made-up buffers begin


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2508_17588_amd.build import BINDING_PATH, build
    if not (os.path.exists(B.LIB_PATH) and os.path.exists(BINDING_PATH)):
        build(verbose=False)
    return B.load_library()


def at(offset):
    return None if offset is None else ctypes.c_void_p(offset)


# ---- the norm's sum (no GPU: a call that is not refused reaches the runtime, and that is no HERO_ERR_INVALID_ARG) ----------

N, H = 4, 64
ROW = {1: 4 * H, 0: 2 * H}             # bytes of a row of x by its type
X, ADD, ROWS, GAIN, Q, S, FAR = (AT + (i << 14) for i in range(7))


def rms(lib, total, dtype=1, listed=False, add=ADD, n=N, gain=GAIN):
    rc = lib.hero_gather_rms_fp8(at(X), dtype, at(add), at(ROWS if listed else None), n, H, at(gain), 1e-6, at(total), at(Q), at(S), None)
    return rc, lib.hero_last_error()


@pytest.mark.parametrize("dtype", [0, 1])
def test_sum_that_overlaps_an_input_is_refused(lib, dtype):
    row = ROW[dtype]
    for listed in (False, True):
        whole = N * row
        # the last byte of the sum on an input's first, and with rows not listed the sum's first on an input's last
        for start, bytes_ in ((X, N * row), (ADD, N * 2 * H), (ROWS, 4 * N), (GAIN, 2 * H)):
            if start == ROWS and not listed:
                continue
            places = [start - whole + 16, start + (0 if start != X or listed else 16)]
            if not listed or start in (ROWS, GAIN):
                places.append(start + bytes_ - 16)
            for total in places:
                if not listed and dtype == 0 and total == ADD:
                    continue
                rc, why = rms(lib, total, dtype, listed)
                assert rc == B.HERO_ERR_INVALID_ARG and b"overlap" in why, (listed, start, total)
        # listed rows: x and add have one row at least
        if listed:
            for start, bytes_ in ((X, row), (ADD, 2 * H)):
                rc, why = rms(lib, start + bytes_ - 16, dtype, True)
                assert rc == B.HERO_ERR_INVALID_ARG and b"overlap" in why


def without_a_gpu(call):
    """Not refused: without a device the call ends in the runtime's error, which is the library's own code for that."""
    rc, why = call
    assert rc != B.HERO_ERR_INVALID_ARG and rc != B.HERO_ERR_SHAPE, why


@pytest.mark.skipif(torch.cuda.is_available(), reason="the buffers are made up")
@pytest.mark.parametrize("dtype", [0, 1])
def test_sum_beside_the_inputs_is_accepted(lib, dtype):
    row = ROW[dtype]
    for listed in (False, True):
        for total in (FAR, X - N * row, X + N * row, ADD - N * row, ADD + 2 * N * H, GAIN + 2 * H, ROWS + 4 * N):
            without_a_gpu(rms(lib, total, dtype, listed))
    without_a_gpu(rms(lib, X, dtype))                                   # in place
    if dtype == 0:
        without_a_gpu(rms(lib, ADD, 0))
    assert rms(lib, X, dtype, True, n=0)[0] == B.HERO_OK                # nothing is read or written


# ---- the binding, which knows how many rows x and add have ------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_binding_looks_at_all_rows_of_x_and_add(dtype):
    n, total, hidden = 3, 9, 64
    arena = torch.randn(4 * total, hidden, device="cuda").to(dtype)
    x, gain = arena[:total], torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([8, 0, 8], dtype=torch.int32, device="cuda")
    q, s = B.empty_fp8(n, hidden)
    # another slice of the same allocation holds no row of x
    for first in (total, 2 * total, 4 * total - n):
        B.hero_gather_rms_fp8(x, None, rows, n, gain, 1e-6, q, s, arena[first:first + n])
        torch.cuda.synchronize()
        assert torch.equal(arena[first:first + n], x[rows.long()])
    for first in (0, 1, total - n, total - 1):
        with pytest.raises(ValueError, match="share memory"):
            B.hero_gather_rms_fp8(x, None, rows, n, gain, 1e-6, q, s, arena[first:first + n])
    add = torch.randn(total, hidden, dtype=torch.bfloat16, device="cuda")
    if dtype == torch.bfloat16:
        for first in (0, total - n):
            with pytest.raises(ValueError, match="share memory"):
                B.hero_gather_rms_fp8(x, add, rows, n, gain, 1e-6, q, s, add[first:first + n])
        # without a list of rows each is read before it is written
        want = (x.float() + add.float()).to(dtype)
        q, s = B.empty_fp8(total, hidden)
        B.hero_gather_rms_fp8(x, add, None, total, gain, 1e-6, q, s, add)
        torch.cuda.synchronize()
        assert torch.equal(add, want)
    # nothing listed: two tensors without memory do not overlap
    none = torch.empty(0, hidden, dtype=dtype, device="cuda")
    B.hero_gather_rms_fp8(none, None, rows[:0], 0, gain, 1e-6, *B.empty_fp8(0, hidden), none.clone())


# ---- every other output, and scratch ----------------------------------------------------------------------------------------

def overlaps(sizes, written, call):
    """`call(places)` with one buffer of `written` moved onto another: the last bytes of one on the first of the other."""
    base = {name: AT + (i << 20) for i, name in enumerate(sizes)}
    for w in written:
        for other in sizes:
            if other == w:
                continue
            places = dict(base, **{w: base[other] - sizes[w] + 16 if sizes[w] % 16 == 0 else base[other]})
            if places[w] % 16:
                places[w] = base[other]
            yield w, other, call(places)
            yield w, other, call(dict(base, **{w: base[other] + (sizes[other] - 1) // 16 * 16}))


def refused(lib, sizes, written, call):
    for w, other, rc in overlaps(sizes, written, call):
        assert rc == B.HERO_ERR_INVALID_ARG and b"overlap" in lib.hero_last_error(), (w, other)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_outputs(lib, dtype, block_rows):
    n, cols = 256, 640
    sizes = {"x": n * cols * (4 if dtype else 2), "q": n * cols, "scales": n // block_rows * 8}
    refused(lib, sizes, ("q", "scales"), lambda p: lib.hero_quantize_fp8(at(p["x"]), dtype, n, cols, block_rows, at(p["q"]), at(p["scales"]), None))


@pytest.mark.parametrize("listed", [False, True])
def test_norm_outputs(lib, listed):
    n, hidden = 16, 640
    reads = 1 if listed else n
    sizes = {"x": reads * hidden * 4, "add": reads * hidden * 2, "gain": hidden * 2, "sum": n * hidden * 4, "q": n * hidden, "scales": n * 8}
    if listed:
        sizes["rows"] = 4 * n
    refused(lib, sizes, ("q", "scales"),
            lambda p: lib.hero_gather_rms_fp8(at(p["x"]), 1, at(p["add"]), at(p.get("rows")), n, hidden, at(p["gain"]), 1e-6, at(p["sum"]),
                                              at(p["q"]), at(p["scales"]), None))


@pytest.mark.parametrize("bias", [False, True])
def test_product_outputs(lib, bias):
    m, n, k, scratch = 32, 272, 640, 4096
    sizes = {"a": m * k, "a_scales": m * 8, "w": n * k, "w_scales": 3 * 8, "scratch": scratch}
    if bias:
        sizes["bias"] = 2 * n
    first = lambda p: (at(p["a"]), at(p["a_scales"]), at(p["w"]), at(p["w_scales"]), at(p.get("bias")))
    refused(lib, dict(sizes, c=2 * m * n), ("c", "scratch"),
            lambda p: lib.hero_linear_fp8(*first(p), at(p["c"]), m, n, k, 0, at(p["scratch"]), scratch, None))
    refused(lib, dict(sizes, q=m * n, scales=m * 4), ("q", "scales", "scratch"),
            lambda p: lib.hero_linear_fp8_quantized(*first(p), at(p["q"]), at(p["scales"]), m, n, k, 0, at(p["scratch"]), scratch, None))


@pytest.mark.skipif(torch.cuda.is_available(), reason="the buffers are made up")
def test_buffers_side_by_side_are_accepted(lib):
    m, n, k = 32, 256, 512
    sizes = (("a", m * k), ("a_scales", m * 4), ("w", n * k), ("w_scales", 2 * 4 + 8), ("bias", 2 * n), ("q", m * n), ("scales", m * 4), ("scratch", 4096))
    p, end = {}, AT
    for name, size in sizes:
        p[name], end = at(end), end + size
    args = (p["a"], p["a_scales"], p["w"], p["w_scales"], p["bias"])
    without_a_gpu((lib.hero_linear_fp8_quantized(*args, p["q"], p["scales"], m, n, k, 0, p["scratch"], 4096, None), lib.hero_last_error()))
    without_a_gpu((lib.hero_quantize_fp8(at(AT), 0, m, k, 1, at(AT + 2 * m * k), at(AT + 3 * m * k), None), lib.hero_last_error()))


@pytest.mark.gpu
def test_binding_looks_at_all_rows_for_q_and_scales_too():
    n, total, hidden = 2, 40, 64
    x = torch.randn(total, hidden, device="cuda")
    gain, rows = torch.ones(hidden, dtype=torch.bfloat16, device="cuda"), torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    q, s = B.empty_fp8(n, hidden)
    inside = x.view(torch.uint8)[30].view(torch.float8_e4m3fn)[:n * hidden].view(n, hidden)
    with pytest.raises(ValueError, match="share memory"):
        B.hero_gather_rms_fp8(x, None, rows, n, gain, 1e-6, inside, s)
    with pytest.raises(ValueError, match="share memory"):
        B.hero_gather_rms_fp8(x, None, rows, n, gain, 1e-6, q, inside.view(torch.float8_e8m0fnu))
    with pytest.raises(B.HeroError, match="overlap"):
        B.hero_quantize_fp8(x[30:31], inside[:1], s)
