"""8-bit products over very long k, with sums that are exact: a block of k that is lost, taken twice, or meets another block's
scale changes results that have to come out to the last bit.

A is +-1 everywhere; a column of W has a single 1 in each of a few neighbouring blocks of 128 k and zeros elsewhere.  The scales make
the products of those blocks neighbouring powers of two, so that a result is an odd whole number below 2^8 (8-bit results: 2^4) times a
power of two that differs from row to row and from group of blocks to group: exact in fp32, in bf16 (8 bits) and in e4m3 (4 bits, with
groups within 2^6 of each other in a block of the result)."""
import pytest
import torch

import fp8_oracle as F
from paper_2508_17588_amd import binding as B

SCRATCH = 64 << 20
ONE, MINUS_ONE = 0x38, 0xB8            # 1.0 and -1.0 in e4m3


class Problem:
    def __init__(self, m, n, k, quantized, device):
        gen = torch.Generator(device).manual_seed(m + n + k)
        some = lambda low, high, *shape: torch.randint(low, high + 1, shape, generator=gen, device=device)
        self.m, self.n, self.k, self.few = m, n, k, 4 if quantized else 8
        self.stages = -(-k // 128)
        groups = -(-self.stages // self.few)
        assert n >= groups, "a column to each group of blocks"
        self.a = (some(0, 1, m, k) * (MINUS_ONE - ONE) + ONE).to(torch.uint8)
        block = torch.arange(self.stages, device=device)
        self.group = torch.arange(n, device=device) % groups                  # the group of a column
        self.at = some(0, 127, n, self.few)                                   # where in each block its 1 is
        self.place = (self.group[:, None] * self.few + torch.arange(self.few, device=device)) * 128 + self.at
        self.place = torch.where((self.place >= k) & (self.place - self.at < k), (self.place - self.at), self.place)   # (the last block may be short)
        self.present = self.place < k
        self.w = torch.zeros(n, k, dtype=torch.uint8, device=device)
        rows = torch.arange(n, device=device)[:, None].expand(n, self.few)
        self.w[rows[self.present], self.place[self.present]] = ONE
        # exponents: of a block of W random; of A what makes it the block's place in its group, and 2^base of row and group
        of_w = some(-9, 9, self.stages)
        by_block = some(-5, 5, -(-n // 128))                                  # 128 rows of W each
        base = some(0, 6, m, groups) if quantized else some(-20, 20, m, groups)
        self.a_exponents = block % self.few + base[:, block // self.few] - of_w
        self.w_exponents = of_w[None] + by_block[:, None]
        assert int(self.a_exponents.abs().max()) < 120

    def operands(self):
        def scales(exponents):
            out = torch.full((exponents.shape[0], F.pitch(self.k)), 255, dtype=torch.uint8, device=exponents.device)    # (NaN past the row)
            out[:, :self.stages] = (exponents + 127).to(torch.uint8)
            return out.view(torch.float8_e8m0fnu)
        return ((self.a.view(torch.float8_e4m3fn), scales(self.a_exponents)), (self.w.view(torch.float8_e4m3fn), scales(self.w_exponents)))

    def result(self, a_exponents=None, lost=None):
        """The exact sums; a_exponents: others than the scales say; lost: a block that is left out."""
        e = self.a_exponents if a_exponents is None else a_exponents
        out = torch.zeros(self.m, self.n, dtype=torch.float64, device=self.a.device)
        for t in range(self.few):
            place, present = self.place[:, t].clamp(max=self.k - 1), self.present[:, t]
            b = place // 128
            sign = torch.where(self.a[:, place] == ONE, 1.0, -1.0).double()
            power = torch.exp2((e[:, b] + self.w_exponents[torch.arange(self.n, device=b.device) // 128, b]).double())
            out += torch.where(present & (b != lost if lost is not None else True), sign * power, 0.0)
        return out


@pytest.mark.parametrize("quantized", [False, True])
def test_a_lost_or_misplaced_block_shows(quantized):
    """(no GPU) The sums are exact, and every mistake that these tests are for changes some of them."""
    p = Problem(3, 144, 128 * 67 + 48, quantized, "cpu")
    (a, sa), (w, sw) = p.operands()
    want = p.result()
    dense = F.values(a, sa) @ F.values(w, sw, 128).t()
    assert torch.equal(dense, want) and torch.equal(want.float().double(), want)
    if quantized:
        code, byte = F.quantized(want)
        f = torch.exp2(byte.double() - 127.0).repeat_interleave(128, dim=1)[:, :p.n]
        assert torch.equal(F.TABLE[code.long()] * f, want)
    else:
        assert torch.equal(want.bfloat16().double(), want)
    assert bool((want != 0).all())
    for b in range(p.stages):
        assert not torch.equal(p.result(lost=b), want)
        e = p.a_exponents.clone()
        e[:, b] += 1
        assert not torch.equal(p.result(a_exponents=e), want)
    for shift in (1, 4, 16, 64):
        assert not torch.equal(p.result(a_exponents=p.a_exponents.roll(shift, 1)), want)
    assert not torch.equal(p.result(a_exponents=p.a_exponents.roll(1, 0)), want)


# The kernel of each: shared-k tiles up to their 60 stages a wave, and past them; groups of scale words of the others; cut and not
CASES = [
    (1, 64, 61440, False, 0, (16, 16, 1)), (1, 64, 61424, False, 0, (16, 16, 1)), (1, 4096, 14336, False, 0, (16, 16, 1)),
    (16, 4096, 28672, False, 0, (16, 16, 1)), (64, 1024, 20000, False, 0, (16, 16, 1)), (300, 256, 61424, False, 0, (32, 32, 1)),
    (500, 528, 61424, False, 0, (32, 64, 1)), (1000, 528, 30704, False, 0, (64, 64, 1)), (2000, 528, 30704, False, 0, (64, 128, 1)),
    (1, 128, 61440, True, 0, (16, 128, 1)), (17, 144, 30000, True, 0, (16, 128, 1)), (1000, 528, 46000, True, 0, (32, 128, 1)),
    (2000, 528, 30704, True, 0, (64, 128, 1)), (1, 128, 61456, False, 0, (128, 128, 1)), (1, 144, 61456, True, 0, (128, 128, 1)),
    (1, 80, 70000, False, SCRATCH, (128, 128, 8)), (1000, 528, 70000, False, SCRATCH, (192, 128, 8)),
    (4000, 528, 7696, False, SCRATCH, (192, 192, 3)), (2000, 1024, 14336, False, SCRATCH, (256, 256, 6)),
    (4000, 2048, 70000, False, 0, (192, 192, 1)), (4000, 4096, 70000, False, 0, (256, 256, 1)), (500, 1024, 46000, True, SCRATCH, (128, 128, 7)),
    (2000, 528, 70000, True, SCRATCH, (192, 128, 4)), (2000, 1024, 30704, True, SCRATCH, (256, 256, 7)),
    (4000, 2048, 70000, True, 0, (256, 256, 1)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,quantized,scratch_bytes,route", CASES)
def test_exact_sums(m, n, k, quantized, scratch_bytes, route):
    print(f"[case] {m} x {n} x {k} quantized {quantized} scratch {scratch_bytes}: {route}", flush=True)
    assert B.hero_linear_fp8_route(m, n, k, quantized, scratch_bytes) == route
    p = Problem(m, n, k, quantized, "cuda")
    (a, sa), (w, sw) = p.operands()
    scratch = torch.full((scratch_bytes // 4,), float("nan"), device="cuda") if scratch_bytes else None
    want = p.result()
    if quantized:
        q, s = B.empty_fp8(m, n)
        B.hero_linear_fp8_quantized(a, sa, w, sw, None, q, s, 0, scratch)
        torch.cuda.synchronize()
        got = F.values(q, s)
    else:
        c = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
        B.hero_linear_fp8(a, sa, w, sw, None, c, 0, scratch)
        torch.cuda.synchronize()
        got = c.double()
    wrong = got != want.to(got.device)
    assert not bool(wrong.any()), f"{int(wrong.sum())} of {m * n} sums are off, the first at {wrong.nonzero()[0].tolist()}"
