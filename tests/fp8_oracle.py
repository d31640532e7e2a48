"""Plain 64-bit forms of the 8-bit building blocks, on the CPU, written from the format's definition, and the bounds that
results are held to.

Rounding: e4m3 has three fraction bits, so a stored element is off by at most 2^-4 of its value, or by half of the
smallest step 2^-9 below 2^-6 (both times the block's scale).  bf16: 2^-8 of the value."""
import math

import numpy as np
import torch

U32 = 2.0 ** -24                      # half a step of fp32, relative


def pitch(columns):
    return -(-columns // 512) * 4


def e4m3_table():
    """Value of each of the 256 codes."""
    v = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v[c] = math.ldexp(1 + f / 8, e - 7) if e else math.ldexp(f / 8, -6)
        if c & 0x7F == 0x7F:
            v[c] = np.nan
        if c & 0x80:
            v[c] = -v[c]
    return v


TABLE = torch.from_numpy(e4m3_table())


def codes(q):
    return q.contiguous().view(torch.uint8).cpu()


def scale_values(scales):
    b = scales.contiguous().view(torch.uint8).cpu().to(torch.float64)
    return torch.where(b == 255, torch.full_like(b, float("nan")), torch.exp2(b - 127.0))


def values(q, scales, block_rows=1):
    """What [rows, columns] elements and their scales stand for, in float64."""
    rows, columns = q.shape
    f = scale_values(scales).repeat_interleave(128, dim=1)[:, :columns].repeat_interleave(block_rows, dim=0)[:rows]
    return TABLE[codes(q).long()] * f


def encode(t):
    """Codes of float64 values by search in the table: nearest, ties to the even code; NaN and infinities NaN."""
    pos = TABLE[:127]
    size = t.abs().clamp(max=448.0)
    size = torch.where(torch.isnan(t), torch.zeros_like(t), size)
    hi = torch.searchsorted(pos, size.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = pos[hi] - size, size - pos[lo]
    pick = torch.where(up < down, hi, torch.where(down < up, lo, torch.where(hi % 2 == 0, hi, lo)))
    code = torch.where(torch.signbit(t), pick + 128, pick)
    return torch.where(torch.isfinite(t), code, torch.full_like(code, 127)).to(torch.uint8)


def scale_bytes(y, block_rows=1):
    """Bytes [row blocks, pitch] of float64 y: the least power of two that takes a block's largest finite magnitude to 448
    or below, by trying them."""
    rows, columns = y.shape
    out = torch.full((-(-rows // block_rows), pitch(columns)), 127, dtype=torch.uint8)
    size = torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y))
    for i in range(out.shape[0]):
        for b in range(-(-columns // 128)):
            largest = float(size[i * block_rows:(i + 1) * block_rows, b * 128:(b + 1) * 128].max())
            if largest == 0.0:
                continue
            e = max(-127, math.frexp(largest)[1] - 12)
            while largest > math.ldexp(448.0, e):
                e += 1
            out[i, b] = e + 127
    return out


def quantized(y, block_rows=1):
    """(codes, scale bytes) of float64 y."""
    rows, columns = y.shape
    bytes_ = scale_bytes(y, block_rows)
    f = torch.exp2(bytes_.to(torch.float64) - 127.0)
    f = f.repeat_interleave(128, dim=1)[:, :columns].repeat_interleave(block_rows, dim=0)[:rows]
    return encode(y / f), bytes_


def to_device(code, bytes_):
    return code.cuda().view(torch.float8_e4m3fn), bytes_.cuda().view(torch.float8_e8m0fnu)


def gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))


def rms(x, add, rows, gain, eps):
    """(y, h) in float64."""
    h = x.double().cpu()
    if add is not None:
        h = h + add.double().cpu()
    if rows is not None:
        h = h[rows.cpu().long()]
    return h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps) * gain.double().cpu(), h


# The norm in fp32, relative to y: h 1, its square 3, at most 46 additions of positive numbers (16 in a lane, 6 over the
# lanes, 16 waves: 38), the division 1 and eps 1: 52 units of 2^-24 on the mean square, 26 on its root; the reciprocal root 4;
# two products 2.  33 in all.
RMS_ERROR = 33 * U32


def linear(a, w, bias, gelu_act):
    """act(a w^T + bias) in float64 and how far the fp32 sums may be off.  Matrix instructions add the products of eight
    neighbouring k after aligning them to the largest, 13 bits below its leading one: each of the other seven loses less
    than 2^-13 of the largest.  Then k / 8 + 2 additions of partial sums that stay below sum |a w| each round by 2^-24."""
    a, w = a.double(), w.double()
    v = a @ w.t()
    size = a.abs() @ w.abs().t()
    m, k = a.shape
    aligned = torch.zeros_like(v)
    pad = -k % 8
    ap = torch.nn.functional.pad(a.abs(), (0, pad)).view(m, -1, 8)
    wp = torch.nn.functional.pad(w.abs(), (0, pad)).view(w.shape[0], -1, 8)
    for g in range(ap.shape[1]):                  # largest product of a group: at most the product of the largest
        aligned += ap[:, g].amax(dim=1)[:, None] * wp[:, g].amax(dim=1)[None]
    off = torch.minimum(7 * 2.0 ** -13 * aligned, 7 * 2.0 ** -13 * size) + (k / 8 + 2) * U32 * size
    if bias is not None:
        v = v + bias.double().cpu()
        off = off + U32 * v.abs()
    if gelu_act:
        off = 1.13 * off + 16 * U32 * v.abs()     # |gelu'| <= 1.13; eight operations of 2 units each
        v = gelu(v)
    return v, off


def check_bf16(got, want, off, what):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    fine = torch.isfinite(want)
    err = (got - want).abs()[fine]
    bound = (off + 2.0 ** -8 * (want.abs() + off))[fine]
    worst = float((err - bound).max()) if err.numel() else 0.0
    assert worst <= 0, f"{what}: {worst:.3g} beyond the bound, at {int((err - bound).argmax())}"
    if err.numel() >= 1000:
        # bf16 rounding alone: at most 2^-8 / sqrt(3) = 2.3e-3 of the norm; 1e-3 more for the sums
        rel = float(err.norm() / want[fine].norm())
        assert rel <= 3.3e-3, f"{what}: {rel:.3g} of the norm"


def check_fp8(q, scales, want, off, what):
    """Stored rows against float64 `want` that the kernel knows to within `off`."""
    rows, columns = want.shape
    byte = scales.contiguous().view(torch.uint8).cpu()
    assert byte.shape == (rows, pitch(columns)), what
    ok = byte == scale_bytes(want)
    sure = torch.isfinite(want)
    if not bool(ok.all()):                        # next to a border either scale may come out
        near = (byte == scale_bytes(want + torch.sign(want) * off)) | (byte == scale_bytes(torch.sign(want) * (want.abs() - off).clamp(min=0)))
        assert bool((ok | near).all()), f"{what}: a scale is off"
    got = values(q, scales)
    assert torch.equal(torch.isnan(got), ~sure), f"{what}: NaN elsewhere"
    step = scale_values(scales).repeat_interleave(128, dim=1)[:, :columns] * 2.0 ** -10
    bound = off + torch.maximum(2.0 ** -4 * (want.abs() + off), step)
    excess = ((got - want).abs() - bound)[sure]
    assert not excess.numel() or float(excess.max()) <= 0, f"{what}: {float(excess.max()):.3g} beyond the bound"
