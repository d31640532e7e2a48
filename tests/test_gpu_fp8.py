"""The 8-bit building blocks against their plain 64-bit forms."""
import pytest
import torch

import fp8_oracle as F
from paper_2508_17588_amd import binding as B

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def say(msg):
    print(f"[case] {msg}", flush=True)


def normal(seed, *shape, scale=1.0, dtype=torch.float32):
    gen = torch.Generator()
    gen.manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def room(rows, columns, block_rows=1, spare=2):
    """Elements and scales with rows behind the last that have to stay as they are."""
    q = torch.full((rows + spare, columns), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    s = torch.full((-(-rows // block_rows) + spare, F.pitch(columns)), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    return q, s


def written(q, s, rows, block_rows=1):
    blocks = -(-rows // block_rows)
    assert bool((q[rows:].view(torch.uint8) == 0x55).all()) and bool((s[blocks:].view(torch.uint8) == 0x55).all()), "rows behind the last"
    return q[:rows], s[:blocks]


# ---- quantiser: every bit --------------------------------------------------------------------------

@pytest.mark.parametrize("rows,columns,block_rows", [
    (1, 16, 1), (1, 1920, 1), (3, 48, 1), (5, 128, 1), (2, 144, 1), (7, 512, 1), (4, 528, 1), (33, 1008, 1), (2, 8208, 1), (600, 640, 1),
    (1, 16, 128), (127, 112, 128), (128, 128, 128), (129, 144, 128), (300, 528, 128), (257, 1920, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_is_exact(rows, columns, block_rows, dtype):
    say(f"quantize {rows} x {columns} blocks of {block_rows} {dtype}")
    # magnitudes over many binades, rows of zeros, exact borders
    x = normal(rows + columns, rows, columns) * torch.exp2(torch.randint(-30, 30, (rows, columns // 16), generator=torch.Generator().manual_seed(7)).float()).repeat_interleave(16, dim=1)
    x[rows // 2, : columns // 2] = 0.0
    x[0, 0] = 448.0 * 2.0 ** 40
    x = x.to(dtype)
    q, s = room(rows, columns, block_rows)
    B.hero_quantize_fp8(x.cuda(), q, s, block_rows)
    torch.cuda.synchronize()
    q, s = written(q, s, rows, block_rows)
    code, byte = F.quantized(x.double(), block_rows)
    assert torch.equal(s.view(torch.uint8).cpu(), byte)
    assert torch.equal(F.codes(q), code)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_extremes(block_rows):
    say(f"quantize extremes, blocks of {block_rows}")
    x = torch.zeros(6, 256)
    x[0, 5], x[0, 6], x[0, 7] = INF, 3.0, -INF
    x[1, 3], x[1, 4] = NAN, 2.0 ** -140
    x[2, 0], x[2, 200] = 3.4028234e38, -1e-45
    x[3, :128] = 448.0
    x[3, 128:] = 449.0
    x[4, 9] = -0.0
    x[5, :] = torch.linspace(-1, 1, 256)
    x = x.repeat_interleave(block_rows, dim=0) if block_rows > 1 else x
    q, s = room(x.shape[0], 256, block_rows)
    B.hero_quantize_fp8(x.cuda(), q, s, block_rows)
    torch.cuda.synchronize()
    q, s = written(q, s, x.shape[0], block_rows)
    code, byte = F.quantized(x.double(), block_rows)
    assert torch.equal(s.view(torch.uint8).cpu(), byte)
    got, want = F.TABLE[F.codes(q).long()], F.TABLE[code.long()]
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(9e9), want.nan_to_num(9e9))


# ---- norm ------------------------------------------------------------------------------------------

def run_rms(x, add, rows, n, gain, eps, want_sum, spare=2):
    hidden = x.shape[1]
    q, s = room(n, hidden, spare=spare)
    total = torch.full((n + spare, hidden), 7.0, dtype=x.dtype, device="cuda") if want_sum else None
    dev = lambda t: None if t is None else t.cuda()
    B.hero_gather_rms_fp8(dev(x), dev(add), dev(rows), n, dev(gain), eps, q, s, total)
    torch.cuda.synchronize()
    q, s = written(q, s, n)
    y, h = F.rms(x, add, rows, gain, eps)
    y, h = y[:n], h[:n]
    F.check_fp8(q, s, y, F.RMS_ERROR * y.abs(), "rms")
    if want_sum:
        assert bool((total[n:] == 7.0).all())
        got = total[:n].double().cpu()
        step = F.U32 if x.dtype == torch.float32 else F.U32 + 2.0 ** -8
        assert bool(((got - h).abs() <= step * h.abs()).all())


@pytest.mark.parametrize("n,hidden,listed,add,want_sum", [
    (1, 16, False, False, False), (1, 1920, False, True, True), (2, 64, True, True, False), (5, 112, False, True, True),
    (9, 512, True, False, True), (3, 528, False, True, True), (6, 1008, False, False, False), (4, 1024, False, True, True),
    (7, 1040, True, True, True), (3, 1920, True, True, False), (2, 2560, False, True, True), (5, 4096, True, True, True),
    (3, 6000, False, True, False), (2, 8192, False, True, True), (2, 8208, True, True, True), (1, 16384, False, True, True),
    (1003, 1920, True, True, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rms(n, hidden, listed, add, want_sum, dtype):
    say(f"rms {n} x {hidden} listed {listed} add {add} sum {want_sum} {dtype}")
    total = 2 * n + 1 if listed else n
    x = normal(n + hidden, total, hidden)
    x[:, hidden // 3] *= 40.0
    rows = torch.randint(0, total, (n,), generator=torch.Generator().manual_seed(3), dtype=torch.int32) if listed else None   # rows may repeat
    run_rms(x.to(dtype), normal(5, total, hidden, dtype=torch.bfloat16) if add else None, rows, n,
            (1 + normal(6, hidden, scale=0.1)).to(torch.bfloat16), 1e-6, want_sum)


def test_rms_of_zero_rows_infinities_and_nan():
    say("rms special rows")
    x = normal(1, 5, 640)
    x[0] = 0.0
    x[2, 17] = NAN
    gain = torch.ones(640, dtype=torch.bfloat16)
    q, s = room(5, 640)
    B.hero_gather_rms_fp8(x.cuda(), None, None, 5, gain.cuda(), 1e-6, q, s)
    torch.cuda.synchronize()
    got = F.values(*written(q, s, 5))
    assert bool((got[0] == 0).all()) and bool(torch.isnan(got[2]).all()) and bool(torch.isfinite(got[[1, 3, 4]]).all())
    # eps 0 and a row of zeros: 0 / 0, and nothing of it past the end of the row
    q, s = room(1, 144)
    B.hero_gather_rms_fp8(torch.zeros(1, 144, device="cuda"), None, None, 1, gain[:144].cuda(), 0.0, q, s)
    torch.cuda.synchronize()
    assert bool(torch.isnan(F.values(*written(q, s, 1))).all())
    assert s[:1].view(torch.uint8).cpu().tolist() == [[127] * 4]
    # an infinity: its own element is inf / inf, the others 0
    x = torch.ones(1, 144)
    x[0, 3] = INF
    q, s = room(1, 144)
    B.hero_gather_rms_fp8(x.cuda(), None, None, 1, gain[:144].cuda(), 1e-6, q, s)
    torch.cuda.synchronize()
    got = F.values(*written(q, s, 1))
    assert bool(torch.isnan(got[0, 3])) and bool((torch.cat([got[0, :3], got[0, 4:]]) == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rms_adds_the_branch_in_place(dtype):
    say(f"rms in place {dtype}")
    for hidden in (912, 3008):
        x, add = normal(3, 50, hidden).to(dtype), normal(4, 50, hidden, dtype=torch.bfloat16)
        gain = torch.ones(hidden, dtype=torch.bfloat16)
        xd = x.cuda()
        q, s = room(50, hidden)
        B.hero_gather_rms_fp8(xd, add.cuda(), None, 50, gain.cuda(), 1e-6, q, s, xd)
        torch.cuda.synchronize()
        y, h = F.rms(x, add, None, gain, 1e-6)
        F.check_fp8(*written(q, s, 50), y, F.RMS_ERROR * y.abs(), "rms in place")
        assert torch.equal(xd.cpu(), (x.float() + add.float()).to(dtype))


# ---- product ---------------------------------------------------------------------------------------

def operands(m, n, k, seed=0, bias=True):
    a = normal(seed + 1, m, k) * torch.exp2(torch.randint(-3, 4, (m, 1), generator=torch.Generator().manual_seed(seed)).float())
    a[:, k // 2] *= 30.0
    w = normal(seed + 2, n, k, scale=k ** -0.5)
    if m * k + n * k > 1 << 22:                    # (the plain quantiser walks over its blocks)
        pairs = []
        for t, block_rows in ((a, 1), (w, 128)):
            pairs.append(B.empty_fp8(*t.shape, block_rows))
            B.hero_quantize_fp8(t.cuda(), *pairs[-1], block_rows)
        pairs = tuple(pairs)
    else:
        pairs = F.to_device(*F.quantized(a.double())), F.to_device(*F.quantized(w.double(), 128))
    return pairs[0], pairs[1], normal(seed + 3, n, scale=0.5, dtype=torch.bfloat16).cuda() if bias else None


def run_linear(a, w, bias, act, quantized, scratch=None, rows=None, spare=2):
    (aq, as_), (wq, ws) = a, w
    m, n = aq.shape[0], wq.shape[0]
    what = f"linear {m} x {n} x {aq.shape[1]} act {act} quantized {quantized}"
    if quantized:
        q, s = room(m, n, spare=spare)
        B.hero_linear_fp8_quantized(aq, as_, wq, ws, bias, q, s, act, scratch)
        torch.cuda.synchronize()
        out = written(q, s, m)
    else:
        c = torch.full((m + spare, n), 7.0, dtype=torch.bfloat16, device="cuda")
        B.hero_linear_fp8(aq, as_, wq, ws, bias, c, act, scratch)
        torch.cuda.synchronize()
        assert bool((c[m:] == 7.0).all()), "rows behind the last"
        out = c[:m]
    pick = torch.arange(m) if rows is None else rows
    v, off = F.linear(F.values(aq, as_)[pick], F.values(wq, ws, 128), bias, act)
    if quantized:
        F.check_fp8(out[0][pick.cuda()] if rows is None else out[0].view(torch.uint8)[pick.cuda()].view(torch.float8_e4m3fn),
                    out[1].view(torch.uint8)[pick.cuda()].view(torch.float8_e8m0fnu), v, off, what)
    else:
        F.check_bf16(out[pick.cuda()], v, off, what)
    return out


SIZES = [
    (1, 16, 16), (1, 128, 128), (1, 1920, 400), (2, 48, 64), (3, 144, 80), (5, 112, 512), (16, 256, 640), (17, 272, 528),
    (31, 400, 48), (32, 128, 1040), (33, 384, 192), (64, 64, 64), (65, 640, 144), (100, 528, 1920), (127, 256, 256),
    (128, 128, 128), (129, 272, 272), (200, 208, 2064), (255, 384, 96), (256, 256, 1024), (257, 512, 384), (300, 1040, 320),
    (513, 144, 160), (700, 656, 208),
]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("quantized", [False, True])
def test_linear(m, n, k, quantized):
    say(f"linear {m} x {n} x {k} quantized {quantized}")
    a, w, bias = operands(m, n, k, seed=m + n + k)
    run_linear(a, w, bias, (m + n) % 2, quantized)


# long k: several groups of scale words, tiles cut along k (scratch) or not
LONG = [(300, 272, 4112), (256, 528, 6160), (130, 144, 8208), (4, 64, 5008), (70, 128, 4096), (16, 48, 7696), (20, 272, 2064), (32, 144, 1936),
        (1, 16, 70000), (2, 144, 8272)]


@pytest.mark.parametrize("m,n,k", LONG)
@pytest.mark.parametrize("quantized", [False, True])
def test_linear_long_k(m, n, k, quantized):
    say(f"linear {m} x {n} x {k} quantized {quantized}")
    a, w, bias = operands(m, n, k)
    scratch = torch.full((64 << 18,), float("nan"), device="cuda")
    outs = [run_linear(a, w, bias, 1, quantized, scratch=s) for s in (None, scratch, scratch[: 1 << 10], scratch)]
    for o in zip(*outs) if quantized else [outs]:
        assert torch.equal(o[1].view(torch.uint8), o[3].view(torch.uint8)), "two calls differ"


@pytest.mark.parametrize("m,n,k", [(4485, 4112, 272), (9001, 1920, 144), (2900, 2064, 4128), (1755, 528, 640)])
@pytest.mark.parametrize("quantized", [False, True])
def test_linear_many_tiles(m, n, k, quantized):
    say(f"linear {m} x {n} x {k} quantized {quantized}")
    a, w, bias = operands(m, n, k)
    rows = torch.unique(torch.cat([torch.randint(0, m, (150,), generator=torch.Generator().manual_seed(9)), torch.tensor([0, m - 1])]))
    run_linear(a, w, bias, 0, quantized, scratch=torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), rows=rows)


# Every kernel that a product can go to: the tile and what becomes of the last round's tiles, with 64 MiB of scratch
SCRATCH = 64 << 20
ROUTES = [
    (1, 16, 16, False, (16, 16, 1)), (4, 928, 2064, False, (16, 16, 1)), (9, 7520, 1936, False, (16, 16, 1)),
    (65, 832, 16, False, (32, 32, 1)), (61, 1920, 7696, False, (32, 32, 1)), (161, 1888, 16, False, (32, 64, 1)),
    (550, 720, 3008, False, (32, 64, 1)), (137, 2608, 8160, False, (32, 64, 1)), (12309, 16, 16, False, (64, 64, 1)),
    (400, 1936, 1920, False, (64, 64, 1)), (329, 2192, 3792, False, (64, 64, 1)), (5475, 144, 496, False, (64, 128, 1)),
    (7262, 160, 6688, False, (64, 128, 1)), (2047, 2048, 2032, False, (128, 128, 1)), (974, 544, 7072, False, (128, 128, 5)),
    (16590, 160, 16, False, (192, 128, 1)), (138, 7120, 7424, False, (192, 128, 4)), (1217, 4688, 528, False, (192, 192, 1)),
    (5794, 160, 7968, False, (192, 192, 6)), (626, 8864, 16, False, (256, 256, 1)), (17311, 784, 144, False, (256, 256, -1)),
    (2958, 7024, 3776, False, (256, 256, 2)), (1, 16, 16, True, (16, 128, 1)), (13, 1936, 1936, True, (16, 128, 1)),
    (137, 2608, 8160, True, (16, 128, 1)), (4135, 16, 16, True, (32, 128, 1)), (400, 1936, 1920, True, (32, 128, 1)),
    (9164, 16, 400, True, (64, 128, 1)), (1406, 4144, 5088, True, (64, 128, 1)), (8363, 16, 16, True, (128, 128, 1)),
    (1, 16, 7792, True, (128, 128, 7)), (16505, 176, 400, True, (192, 128, 1)), (3357, 384, 7920, True, (192, 128, 4)),
    (16590, 160, 16, True, (256, 256, 1)), (14604, 1056, 544, True, (256, 256, -1)), (10879, 1296, 4848, True, (256, 256, 4)),
]


@pytest.mark.parametrize("m,n,k,quantized,route", ROUTES)
def test_linear_every_kernel(m, n, k, quantized, route):
    say(f"linear {m} x {n} x {k} quantized {quantized}: {route}")
    assert B.hero_linear_fp8_route(m, n, k, quantized, SCRATCH) == route
    a, w, bias = operands(m, n, k)
    rows = torch.unique(torch.cat([torch.randint(0, m, (120,), generator=torch.Generator().manual_seed(m)), torch.tensor([0, m - 1])]))
    scratch = torch.full((SCRATCH // 4,), float("nan"), device="cuda")
    for act in (0, 1):
        run_linear(a, w, bias, act, quantized, scratch=scratch, rows=rows)


@pytest.mark.parametrize("quantized", [False, True])
def test_linear_without_bias(quantized):
    say(f"linear without bias, quantized {quantized}")
    for m, n, k in ((3, 64, 96), (150, 272, 400)):
        a, w, _ = operands(m, n, k, bias=False)
        run_linear(a, w, None, 0, quantized)
        run_linear(a, w, None, 1, quantized)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_linear_special_values(m):
    """A NaN element or a NaN scale of a row reaches that row only, of a weight's row its column only; scales from 2^-127 on."""
    say(f"linear special values, {m} rows")
    n, k = 272, 400
    (aq, as_), (wq, ws), bias = operands(m, n, k)
    clean = run_linear((aq, as_), (wq, ws), bias, 0, False).clone()
    qa, sa = aq.view(torch.uint8).clone(), as_.view(torch.uint8).clone()
    qa[m // 2, 333] = 0x7F
    qw = wq.view(torch.uint8).clone()
    qw[200, 5] = 0xFF
    out = run_linear((qa.view(torch.float8_e4m3fn), as_), (qw.view(torch.float8_e4m3fn), ws), bias, 0, False)
    bad = torch.isnan(out)
    assert bool(bad[m // 2].all()) and bool(bad[:, 200].all())
    bad[m // 2], bad[:, 200] = False, False
    keep = torch.ones_like(bad)
    keep[m // 2], keep[:, 200] = False, False
    assert not bool(bad.any()) and torch.equal(out[keep], clean[keep])
    # a NaN scale
    sa2 = sa.clone()
    sa2[m - 1, 2] = 255
    out = run_linear((aq, sa2.view(torch.float8_e8m0fnu)), (wq, ws), bias, 0, False)
    assert bool(torch.isnan(out[m - 1]).all()) and torch.equal(out[: m - 1], clean[: m - 1])
    # tiny scales: that block counts for nothing beside the others, but is no NaN
    sa2 = sa.clone()
    sa2[:, 1] = 0
    run_linear((aq, sa2.view(torch.float8_e8m0fnu)), (wq, ws), bias, 0, False)
    # large ones
    sa2 = sa.clone()
    sa2[:, 1] += 60
    run_linear((aq, sa2.view(torch.float8_e8m0fnu)), (wq, ws), bias, 0, True)


@pytest.mark.parametrize("m,n,k", [(3, 272, 160), (200, 272, 160), (700, 1040, 2048), (40, 144, 4112)])
def test_infinite_results_in_8_bits(m, n, k):
    """An infinite result is a NaN element and does not count for its block's scale."""
    say(f"infinite results {m} x {n} x {k}")
    a, w, bias = operands(m, n, k)
    bias[5], bias[140], bias[141] = INF, -INF, NAN
    scratch = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    for act in (0, 1):
        run_linear(a, w, bias, act, True, scratch=scratch)
        run_linear(a, w, bias, act, False, scratch=scratch)


def test_padding_bytes_of_scales_are_not_used():
    say("padding of the scales")
    m, n, k = 70, 144, 272
    (aq, as_), (wq, ws), bias = operands(m, n, k)
    want = run_linear((aq, as_), (wq, ws), bias, 0, False).clone()
    sa, sw = as_.view(torch.uint8).clone(), ws.view(torch.uint8).clone()
    sa[:, 3:], sw[:, 3:] = 255, 255
    got = run_linear((aq, sa.view(torch.float8_e8m0fnu)), (wq, sw.view(torch.float8_e8m0fnu)), bias, 0, False)
    assert torch.equal(got, want)


# ---- beyond one launch, beyond 32 bits -------------------------------------------------------------

MANY = (1 << 21) + 133


def some_rows(rows, *borders):
    """The first rows, the last and those on both sides of the borders."""
    near = [torch.arange(max(0, b - 3), min(rows, b + 4)) for b in (0, rows, *borders)]
    return torch.cat(near).unique()


@pytest.mark.parametrize("rows,columns,borders", [(MANY, 16, (1 << 21,)), (9, 1 << 22, ()), (70000, 1040, (1 << 16,)), (300, 16 << 20, (256,))])
def test_quantize_of_many_rows(rows, columns, borders):
    say(f"quantize {rows} x {columns}")
    x = torch.randn(rows, columns, device="cuda", dtype=torch.bfloat16, generator=torch.Generator("cuda").manual_seed(1))
    q, s = room(rows, columns)
    B.hero_quantize_fp8(x, q, s)
    torch.cuda.synchronize()
    q, s = written(q, s, rows)
    pick, last = some_rows(rows, *borders), max(0, (columns - 1024) // 512 * 512)
    code, byte = F.quantized(x[pick.cuda(), last:].cpu().double())
    assert torch.equal(F.codes(q.view(torch.uint8)[pick.cuda(), last:]), code)
    assert torch.equal(s.view(torch.uint8)[pick.cuda(), last // 128: F.pitch(columns)].cpu(), byte)


@pytest.mark.parametrize("rows", [MANY, (1 << 23) + 1])
def test_quantize_blocks_of_many_rows(rows):
    say(f"quantize {rows} x 16 in blocks")
    x = torch.randn(rows, 16, device="cuda", dtype=torch.bfloat16, generator=torch.Generator("cuda").manual_seed(1))
    q, s = room(rows, 16, 128)
    B.hero_quantize_fp8(x, q, s, 128)
    torch.cuda.synchronize()
    q, s = written(q, s, rows, 128)
    for b in (0, (1 << 14) - 1, 1 << 14, s.shape[0] - 2, s.shape[0] - 1):
        part = slice(128 * b, min(rows, 128 * b + 128))
        code, byte = F.quantized(x[part].cpu().double(), 128)
        assert torch.equal(F.codes(q[part]), code) and torch.equal(s[b: b + 1].view(torch.uint8).cpu(), byte)


@pytest.mark.parametrize("listed", [False, True])
def test_rms_of_many_rows(listed):
    say(f"rms {MANY} x 32 listed {listed}")
    gen = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(MANY, 32, device="cuda", generator=gen)
    add = torch.randn(MANY, 32, device="cuda", generator=gen).bfloat16()
    rows = torch.arange(MANY - 1, -1, -1, dtype=torch.int32, device="cuda") if listed else None
    gain = torch.ones(32, dtype=torch.bfloat16)
    total = torch.full((MANY + 2, 32), 7.0, device="cuda")
    q, s = room(MANY, 32)
    B.hero_gather_rms_fp8(x, add, rows, MANY, gain.cuda(), 1e-6, q, s, total)
    torch.cuda.synchronize()
    q, s = written(q, s, MANY)
    pick = some_rows(MANY, 1 << 21).cuda()
    src = rows[pick].long() if listed else pick
    y, h = F.rms(x[src].cpu(), add[src].cpu(), None, gain, 1e-6)
    F.check_fp8(q.view(torch.uint8)[pick].view(q.dtype), s.view(torch.uint8)[pick].view(s.dtype), y, F.RMS_ERROR * y.abs(), "rms")
    assert bool((total[MANY:] == 7.0).all())
    assert torch.equal(total[pick], x[src] + add[src].float())


@pytest.mark.parametrize("m,n,quantized", [(270000, 8192, False), (530000, 8192, True), (300, (8 << 20) - 16, False), (560, (8 << 20) - 16, True)])
def test_results_past_4_gib(m, n, quantized):
    say(f"linear {m} x {n} x 16 quantized {quantized}")
    a, w, bias = operands(m, n, 16)
    (aq, as_), (wq, ws) = a, w
    border = (1 << 32) // (n * (1 if quantized else 2))
    rows, cols = some_rows(m, border), slice(max(0, (n - 1600) // 512 * 512), n)
    if quantized:
        out = room(m, n)
        B.hero_linear_fp8_quantized(aq, as_, wq, ws, bias, *out)
        torch.cuda.synchronize()
        out = written(*out, m)
    else:
        c = torch.full((m + 2, n), 7.0, dtype=torch.bfloat16, device="cuda")
        B.hero_linear_fp8(aq, as_, wq, ws, bias, c)
        torch.cuda.synchronize()
        assert bool((c[m:] == 7.0).all()), "rows behind the last"
    at = rows.cuda()
    some_a = F.values(aq.view(torch.uint8)[at].view(aq.dtype), as_.view(torch.uint8)[at].view(as_.dtype))
    v, off = F.linear(some_a, F.values(wq[cols], ws[cols.start // 128:], 128), bias[cols], 0)
    if quantized:
        scales = out[1].view(torch.uint8)[at][:, cols.start // 128: F.pitch(n)].view(torch.float8_e8m0fnu)
        F.check_fp8(out[0].view(torch.uint8)[at][:, cols].view(torch.float8_e4m3fn), scales, v, off, "past 4 GiB")
    else:
        F.check_bf16(c[at][:, cols], v, off, "past 4 GiB")


# ---- together --------------------------------------------------------------------------------------

def branch(x, add, rows, n, gain, w1, b1, w2, b2, room_, scratch=None):
    (q, s), (mid, ms), c = room_
    B.hero_gather_rms_fp8(x, add, rows, n, gain, 1e-6, q, s)
    B.hero_linear_fp8_quantized(q, s, *w1, b1, mid, ms, 1, scratch)
    B.hero_linear_fp8(mid, ms, *w2, b2, c, 0, scratch)


@pytest.mark.parametrize("n,hidden", [(1, 128), (77, 320), (300, 512)])
def test_feed_forward_branch(n, hidden):
    """Norm, product with GELU into 8 bits, product: each step against its plain form on what the step before stored."""
    say(f"branch {n} x {hidden}")
    ffn, total = 4 * hidden, 2 * n
    x, add = normal(1, total, hidden), normal(2, total, hidden, dtype=torch.bfloat16)
    rows = torch.randperm(total, generator=torch.Generator().manual_seed(5))[:n].to(torch.int32)
    gain = (1 + normal(3, hidden, scale=0.1)).to(torch.bfloat16)
    weights = []
    for seed, out, into in ((4, ffn, hidden), (5, hidden, ffn)):
        w = normal(seed, out, into, scale=into ** -0.5, dtype=torch.bfloat16).cuda()
        q, s = B.empty_fp8(out, into, 128)
        B.hero_quantize_fp8(w, q, s, 128)
        weights.append((q, s))
    b1, b2 = normal(6, ffn, scale=0.1, dtype=torch.bfloat16).cuda(), normal(7, hidden, scale=0.1, dtype=torch.bfloat16).cuda()
    got = (B.empty_fp8(n, hidden), B.empty_fp8(n, ffn), torch.empty(n, hidden, dtype=torch.bfloat16, device="cuda"))
    branch(x.cuda(), add.cuda(), rows.cuda(), n, gain.cuda(), weights[0], b1, weights[1], b2, got)
    torch.cuda.synchronize()
    y, _ = F.rms(x, add, rows, gain, 1e-6)
    F.check_fp8(*got[0], y, F.RMS_ERROR * y.abs(), "norm")
    v, off = F.linear(F.values(*got[0]), F.values(*weights[0], 128), b1, 1)
    F.check_fp8(*got[1], v, off, "first product")
    v, off = F.linear(F.values(*got[1]), F.values(*weights[1], 128), b2, 0)
    F.check_bf16(got[2], v, off, "second product")


def test_captured_branch_replays_with_new_inputs():
    say("captured branch")
    n, hidden, ffn = 150, 256, 1024
    gain = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    w = []
    for seed, out, into in ((4, ffn, hidden), (5, hidden, ffn)):
        q, s = B.empty_fp8(out, into, 128)
        B.hero_quantize_fp8(normal(seed, out, into, scale=0.05).cuda(), q, s, 128)
        w.append((q, s))
    x = torch.empty(n, hidden, device="cuda")
    add = torch.empty(n, hidden, dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")

    def rooms():
        return B.empty_fp8(n, hidden), B.empty_fp8(n, ffn), torch.zeros(n, hidden, dtype=torch.bfloat16, device="cuda")
    eager, held = rooms(), rooms()

    def fill(seed):
        x.copy_(normal(seed, n, hidden))
        add.copy_(normal(seed + 50, n, hidden, dtype=torch.bfloat16))

    fill(0)
    branch(x, add, None, n, gain, w[0], None, w[1], None, held, scratch)      # every kernel has run once
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        branch(x, add, None, n, gain, w[0], None, w[1], None, held, scratch)
    for seed in (1, 2, 3, 4):
        fill(seed)
        branch(x, add, None, n, gain, w[0], None, w[1], None, eager, scratch)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[2], eager[2]) and torch.equal(held[1][0].view(torch.uint8), eager[1][0].view(torch.uint8))


def test_on_another_stream():
    say("another stream")
    m, n, k = 90, 256, 512
    a, w, bias = operands(m, n, k)
    c = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    want = run_linear(a, w, bias, 0, False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.hero_linear_fp8(a[0], a[1], w[0], w[1], bias, c)
    side.synchronize()
    assert torch.equal(c, want)


@pytest.mark.parametrize("m,n,k,quantized", [(974, 544, 7072, False), (200, 400, 7120, True), (33, 272, 1040, False)])
def test_two_streams_at_once(m, n, k, quantized):
    """Calls that overlap, each with its own scratch and result."""
    say(f"two streams {m} x {n} x {k} quantized {quantized}")
    a, w, bias = operands(m, n, k)
    bounds = [torch.full((16 << 20,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]

    def call(out, scratch):
        if quantized:
            B.hero_linear_fp8_quantized(*a, *w, bias, *out, 1, scratch)
        else:
            B.hero_linear_fp8(*a, *w, bias, out[0], 1, scratch)
    outs = [B.empty_fp8(m, n) if quantized else (torch.empty(m, n, dtype=torch.bfloat16, device="cuda"),) for _ in range(9)]
    call(outs[8], bounds[0])
    torch.cuda.synchronize()
    for i in range(8):
        with torch.cuda.stream(sides[i % 2]):
            call(outs[i], bounds[i % 2])
    torch.cuda.synchronize()
    for out in outs[:8]:
        assert all(torch.equal(t.view(torch.uint8), u.view(torch.uint8)) for t, u in zip(out, outs[8]))


def test_two_graphs_with_one_scratch():
    """Captured calls that share scratch, replayed one after the other, with eager work between them."""
    say("two graphs, one scratch")
    scratch = torch.full((32 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    problems, graphs = [], []
    for i, (m, n, k) in enumerate(((974, 544, 7072), (900, 640, 7264))):
        a, w, bias = operands(m, n, k, seed=10 * i)
        c, want = (torch.zeros(m, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        assert B.hero_linear_fp8_route(m, n, k, False, scratch.numel())[2] > 1          # (cut: the scratch is used)
        B.hero_linear_fp8(*a, *w, bias, want, 0, scratch)
        problems.append((a, w, bias, c, want))
    torch.cuda.synchronize()
    for a, w, bias, c, _ in problems:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.hero_linear_fp8(*a, *w, bias, c, 0, scratch)
        graphs.append(graph)
    for turn in range(4):
        for graph, (a, w, bias, c, want) in zip(graphs, problems):
            c.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c, want), turn
        scratch.fill_(0xFF)


# ---- what the binding refuses before anything is launched ------------------------------------------

def test_binding_refusals():
    m, n, k = 4, 32, 64
    a, w, bias = operands(m, n, k)
    c = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    q, s = B.empty_fp8(m, n)
    x, add = torch.randn(m, k, device="cuda"), torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
    gain, rows = torch.ones(k, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    xq, xs = B.empty_fp8(m, k)

    def refused(kind, match, call, *args):
        with pytest.raises(kind, match=match):
            call(*args)
    rms, linear, both, quantize = B.hero_gather_rms_fp8, B.hero_linear_fp8, B.hero_linear_fp8_quantized, B.hero_quantize_fp8
    # type, order, place and size of each tensor
    refused(TypeError, "q must be", quantize, x, xs, xs)
    refused(TypeError, "scales must be", quantize, x, xq, xq)
    refused(ValueError, "q is too small", quantize, x, xq[:3], xs)
    refused(ValueError, "scales is too small", quantize, x, xq, xs[:3])
    refused(ValueError, "rows, columns", quantize, x[0], xq, xs)
    refused(ValueError, "block_rows", quantize, x, xq, xs, 64)
    refused(TypeError, "x must be", quantize, x[:, ::2], xq, xs)
    refused(TypeError, "unsupported", quantize, x.double(), xq, xs)
    refused(TypeError, "q must be", quantize, x, xq.cpu(), xs)
    refused(TypeError, "an integer|integer", quantize, x, xq, xs, None)
    refused(ValueError, "shape", rms, x, add[:3], None, m, gain, 1e-6, xq, xs)
    refused(ValueError, "shape", rms, x, None, None, m + 1, gain, 1e-6, xq, xs)
    refused(ValueError, "shape", rms, x, None, None, m, gain[:32], 1e-6, xq, xs)
    refused(TypeError, "add must be", rms, x, x, None, m, gain, 1e-6, xq, xs)
    refused(TypeError, "rows must be", rms, x, None, rows.long(), 2, gain, 1e-6, xq, xs)
    refused(ValueError, "rows is too small", rms, x, None, rows, 3, gain, 1e-6, xq, xs)
    refused(ValueError, "share memory", rms, x, None, rows, 2, gain, 1e-6, xq, xs, x)
    refused(TypeError, "sum must be", rms, x, None, None, m, gain, 1e-6, xq, xs, add)
    refused(TypeError, "real number", rms, x, None, None, m, gain, "1e-6", xq, xs)
    refused(ValueError, "shape", linear, *a, w[0][:, :32].contiguous(), w[1], bias, c)
    refused(ValueError, "shape", linear, *a, *w, bias[:16], c)
    refused(ValueError, "w_scales is too small", linear, *a, w[0], w[1][:0], bias, c)
    refused(ValueError, "c is too small", linear, *a, *w, bias, c[:3])
    refused(TypeError, "bias must be", linear, *a, *w, bias.float(), c)
    refused(TypeError, "scratch must be a tensor", linear, *a, *w, bias, c, 0, 4096)
    refused(TypeError, "w must be", linear, *a, torch.empty(k, n, dtype=torch.float8_e4m3fn, device="cuda").t(), w[1], None, c)
    refused(ValueError, "q is too small", both, *a, *w, bias, q[:3], s)
    refused(ValueError, "scales is too small", both, *a, *w, bias, q, s[:3])
    refused(TypeError, "a_scales must be a tensor", both, a[0], None, *w, bias, q, s)
    # the library's own refusals arrive as its error
    refused(B.HeroError, "act must be", linear, *a, *w, bias, c, 2)
    refused(B.HeroError, "eps", rms, x, None, None, m, gain, -1.0, xq, xs)
    refused(B.HeroError, "16-byte", linear, *a, *w, bias, torch.zeros(m * n + 4, dtype=torch.bfloat16, device="cuda")[4:].view(m, n))
    # sizes past 31 bits do not arrive as their low 32 bits
    refused(ValueError, "2.31", quantize, torch.zeros(1, 16, device="cuda").expand((1 << 32) + 1, 16), xq, xs)
    refused(ValueError, "2.31", rms, x, None, rows, (1 << 32) + 1, gain, 1e-6, xq, xs)
    refused(ValueError, "2.31", linear, a[0][:1].expand((1 << 32) + 1, k), a[1], *w, None, c)
    torch.cuda.synchronize()


def test_calls_on_no_rows():
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    empty, (q, s) = torch.empty(0, 64, device="cuda"), B.empty_fp8(0, 64)
    B.hero_quantize_fp8(empty, q, s)
    B.hero_gather_rms_fp8(empty, None, None, 0, gain, 1e-6, q, s, empty.clone())
    w = operands(1, 32, 64)[1]
    B.hero_linear_fp8(q, s, *w, None, torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"))
    B.hero_linear_fp8_quantized(q, s, *w, None, *B.empty_fp8(0, 32))
    torch.cuda.synchronize()


def test_two_threads():
    """Calls from two threads, each on its own stream with its own results; a refusal in one leaves the other alone."""
    import threading
    say("two threads")
    problems = [operands(226, 400, 1920), operands(40, 528, 4112, seed=20)]
    wants = [run_linear(a, w, bias, 1, False).clone() for a, w, bias in problems]
    failures = []

    def work(i):
        try:
            a, w, bias = problems[i]
            side = torch.cuda.Stream()
            scratch = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for turn in range(40):
                    c = torch.zeros_like(wants[i])
                    B.hero_linear_fp8(*a, *w, bias, c, 1, scratch)
                    if turn % 8 == i:
                        with pytest.raises(B.HeroError, match="act must be" if i else "16-byte"):
                            B.hero_linear_fp8(*a, *w, bias, c if i else torch.empty(c.numel() + 1, dtype=c.dtype, device="cuda")[1:], 2 if i else 0)
                    side.synchronize()
                    assert torch.equal(c, wants[i]), turn
        except BaseException as e:      # (a thread's own failure would pass unseen)
            failures.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
