"""8-bit products of operands whose scales lie far apart: neither scale is applied by itself where only both together leave
ordinary numbers."""
import pytest
import torch

import fp8_oracle as F
from paper_2508_17588_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", [40, 100, 115, -40, -100, -115])
@pytest.mark.parametrize("m,n,k,quantized", [(3, 272, 400, False), (40, 144, 1040, False), (100, 1936, 1920, False), (300, 1040, 320, False),
                                             (626, 8864, 16, False), (3, 272, 400, True), (300, 1040, 320, True), (1406, 1040, 640, True)])
def test_scales_far_apart(m, n, k, quantized, far):
    print(f"[case] {m} x {n} x {k} quantized {quantized}: scales 2^{far} and 2^{-far} apart", flush=True)
    gen = torch.Generator().manual_seed(m)
    a, w = torch.randn(m, k, generator=gen).double(), torch.randn(n, k, generator=gen).double() * k ** -0.5
    pairs = []
    for t, block_rows, by in ((a, 1, far), (w, 128, -far)):
        code, byte = F.quantized(t, block_rows)
        moved = byte.clone()
        moved[:, : -(-k // 128)] = (byte[:, : -(-k // 128)].int() + by).to(torch.uint8)
        assert int(moved.max()) < 255 and int((byte.int() + by)[:, : -(-k // 128)].min()) >= 0
        pairs.append((F.to_device(code, byte), F.to_device(code, moved)))
    (near_a, far_a), (near_w, far_w) = pairs
    bias = (torch.randn(n, generator=gen) * 0.5).bfloat16().cuda()
    if quantized:
        outs = [B.empty_fp8(m, n) for _ in range(2)]
        for out, x, y in zip(outs, (near_a, far_a), (near_w, far_w)):
            B.hero_linear_fp8_quantized(*x, *y, bias, *out)
    else:
        outs = [(torch.zeros(m, n, dtype=torch.bfloat16, device="cuda"),) for _ in range(2)]
        for out, x, y in zip(outs, (near_a, far_a), (near_w, far_w)):
            B.hero_linear_fp8(*x, *y, bias, *out)
    torch.cuda.synchronize()
    # powers of two that cancel: every product is the same number
    for one, other in zip(*outs):
        assert torch.equal(one.view(torch.uint8), other.view(torch.uint8))
