"""The 8-bit norm over the whole range of fp32: the mean square of a row is neither lost where squares are too small for
fp32 nor infinite where they are too large."""
import pytest
import torch

import fp8_oracle as F
from paper_2508_17588_amd import binding as B

pytestmark = pytest.mark.gpu

# log2 of the rows' magnitudes (in bf16 nothing lies below 2^-133): subnormal, squares of zero, subnormal squares, both sides of where the row is scaled, ordinary ones,
# squares whose sum passes fp32, squares that pass it
MAGNITUDES = (-146, -130, -110, -75, -70, -64, -50, -48, -47, -20, 0, 50, 58, 60, 63, 64, 100, 125)


def check(x, add, rows, gain, eps):
    n, hidden = (x.shape[0] if rows is None else rows.shape[0]), x.shape[1]
    q, s = B.empty_fp8(n, hidden)
    total = torch.full((n, hidden), 7.0, dtype=x.dtype, device="cuda")
    dev = lambda t: None if t is None else t.cuda()
    B.hero_gather_rms_fp8(x.cuda(), dev(add), dev(rows), n, gain.cuda(), eps, q, s, total)
    torch.cuda.synchronize()
    y, h = F.rms(x, add, rows, gain, eps)
    assert bool(torch.isfinite(y).all())
    # What lies below half of fp32's least number, 2^-150, is 0 there, and a block of zeros has the scale byte 127 and not 0: both
    # stand for 0, since the least element is 2^-136 (a row of 2^-110 over the root of an eps of 1e30).  Nothing here lies near 2^-150.
    assert not bool(((y.abs() > 2.0 ** -155) & (y.abs() < 2.0 ** -145)).any())
    y = torch.where(y.abs() < 2.0 ** -150, torch.zeros_like(y), y)
    F.check_fp8(q, s, y, F.RMS_ERROR * y.abs(), f"rms {n} x {hidden} eps {eps}")
    got = total.double().cpu()
    # half a step of the type, of a subnormal one: 2^-150 in fp32, 2^-134 in bf16
    step, least = (F.U32, 2.0 ** -150) if x.dtype == torch.float32 else (F.U32 + 2.0 ** -8, 2.0 ** -134)
    assert bool(((got - h).abs() <= step * h.abs() + least).all())


@pytest.mark.parametrize("hidden", [16, 496, 1040, 1920, 6000, 16384])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-30, 1e-6, 1e30])
def test_rows_of_every_magnitude(hidden, dtype, eps):
    print(f"[case] hidden {hidden} {dtype} eps {eps}", flush=True)
    gen = torch.Generator().manual_seed(hidden)
    magnitudes = torch.tensor(MAGNITUDES, dtype=torch.float64).clamp(min=-146.0 if dtype == torch.float32 else -131.0)
    sign = torch.where(torch.rand(len(MAGNITUDES), hidden, generator=gen) < 0.5, -1.0, 1.0)
    x = (1.0 + torch.rand(len(MAGNITUDES), hidden, generator=gen, dtype=torch.float64)) * sign
    x = (x * torch.exp2(magnitudes)[:, None]).to(dtype)
    gain = (1 + 0.1 * torch.randn(hidden, generator=gen)).to(torch.bfloat16)
    check(x, None, None, gain, eps)


@pytest.mark.parametrize("hidden", [272, 2048])
def test_one_large_or_small_element(hidden):
    print(f"[case] one element, hidden {hidden}", flush=True)
    x = torch.zeros(8, hidden)
    x[0, 3], x[1, 5], x[2, 7] = 3.4028234e38, 1e-45, -1.2e-38
    x[3, 1], x[3, 2] = 1e30, 1e-20                     # far apart in one row
    x[4, :] = 1e-24
    x[4, 9] = 1e-19
    x[5, :] = 3e38
    x[6, :] = 1e-45
    x[7, 0] = 1.0
    check(x, None, None, torch.ones(hidden, dtype=torch.bfloat16), 0.0)
    rows = torch.tensor([5, 1, 1, 6, 0, 3], dtype=torch.int32)
    check(x, torch.zeros(8, hidden, dtype=torch.bfloat16), rows, torch.ones(hidden, dtype=torch.bfloat16), 0.0)


@pytest.mark.parametrize("hidden", [144, 1920])
def test_rows_without_a_mean_square(hidden):
    print(f"[case] zeros, infinities, NaN, hidden {hidden}", flush=True)
    inf, nan = float("inf"), float("nan")
    x = torch.ones(5, hidden)
    x[0], x[1, 3], x[2, 3], x[3, 3], x[3, 5], x[4] = 0.0, inf, nan, -inf, nan, 1e-20
    q, s = B.empty_fp8(5, hidden)
    B.hero_gather_rms_fp8(x.cuda(), None, None, 5, torch.ones(hidden, dtype=torch.bfloat16, device="cuda"), 0.0, q, s)
    torch.cuda.synchronize()
    got = F.values(q, s)
    bad = torch.isnan(got)
    assert bool(bad[0].all()) and bool(bad[2].all()) and bool(bad[3].all())              # 0 / 0, and NaN
    assert bool(bad[1, 3]) and int(bad[1].sum()) == 1 and float(got[1].nan_to_num(0.0).abs().max()) == 0.0      # 1 / inf
    assert not bool(bad[4].any()) and float((got[4] - 1.0).abs().max()) <= 2.0 ** -4 + F.RMS_ERROR
