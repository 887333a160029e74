"""Matrices in 8 bits restated in 64 bits on the host's side of the tests: format, rounding, error bounds."""
import math

import torch

import paper_1806_08054_b200 as ecq

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
KINDS = {E4M3: (3, -6, 448.0), E5M2: (2, -14, 57344.0)}          # mantissa bits, lowest exponent, largest


def pair(rows, cols, dtype=E4M3, extra=0, fill=0xA5):
    """An 8-bit matrix's room, filled with a pattern that results have to leave behind the last column."""
    stride = -(-cols // 16) * 16 + 16 * extra
    whole = torch.full((rows, stride), fill, dtype=torch.uint8, device="cuda")
    scales = torch.full((ecq.ecq_act8_scale_bytes(rows, cols),), fill, dtype=torch.uint8, device="cuda")
    return whole.view(dtype)[:, :cols], scales


def bytes_of(p):
    q = p[0]
    return torch.as_strided(q.view(torch.uint8), (q.shape[0], q.stride(0)), (q.stride(0), 1))


def scale_places(rows, cols):
    """Index of row r's block b in the scales."""
    r = torch.arange(rows, device="cuda")[:, None]
    b = torch.arange(-(-cols // 128), device="cuda")[None, :]
    return ((r // 128) * -(-cols // 512) + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4


def scale_bytes(p):
    return p[1][scale_places(*p[0].shape)]


def expand(blocks, cols):
    return blocks.repeat_interleave(128, dim=1)[:, :cols]


def values(p):
    """What a pair stands for, in 64 bits."""
    b = expand(scale_bytes(p).double(), p[0].shape[1])
    return torch.where(b == 255, math.nan, p[0].to(torch.float64) * torch.exp2(b - 127))


def block_scales(x, dtype=E4M3):
    """Scale bytes of a matrix in 64 bits: the smallest power of two that brings a block into range."""
    _, _, largest = KINDS[dtype]
    rows, cols = x.shape
    wide = torch.nn.functional.pad(x, (0, -cols % 128)).view(rows, -1, 128)
    top = wide.abs().amax(2)
    e = torch.full_like(top, -127.0)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):
        e = torch.where(top > largest * torch.exp2(e + step - 1), e + step, e)
    e = torch.where(top > largest * torch.exp2(e), e + 1, e)
    ok = torch.isfinite(wide).all(2)
    return torch.where(ok, e + 127, 255.0).to(torch.uint8)


def rounded(x, blocks, dtype=E4M3):
    """Entries on their block's grid, in 64 bits: nearest, ties to even."""
    m, lowest, _ = KINDS[dtype]
    unit = torch.exp2(expand(blocks.double(), x.shape[1]) - 127)
    v = x / unit
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp(min=lowest).double() - m)
    r = torch.round(v / step) * step * unit
    return torch.where(expand(blocks, x.shape[1]) == 255, math.nan, r)


def stored(x, dtype=E4M3, extra=0):
    """A pair made by the definition, not by the library."""
    p = pair(*x.shape, dtype, extra)
    x = x.double()
    b = block_scales(x, dtype)
    r = rounded(x, b, dtype) / torch.exp2(expand(b.double(), x.shape[1]) - 127)
    p[0].view(torch.uint8).copy_(r.float().to(dtype).view(torch.uint8))
    p[1][scale_places(*x.shape)] = b
    return p


def half_step(x, dtype):
    """Half of the distance between neighbours of a plain type at x (64 bits)."""
    if dtype == torch.float32:
        return x.abs() * 2.0 ** -24 + 2.0 ** -150
    return x.abs() * torch.finfo(dtype).eps / 2 + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)


def check_pair(p, want, err, what=""):
    """A pair against values in 64 bits that the kernel knows within `err`: scales are those of values
    within err, entries within half a step of the grid that the scale byte gives, and err."""
    dtype = p[0].dtype
    m, lowest, largest = KINDS[dtype]
    b = scale_bytes(p)
    rows, cols = want.shape
    size = want.abs()
    low, high = block_scales((size - err).clamp(min=0), dtype), block_scales(size + err, dtype)
    assert bool(((b >= low) & (b <= high)).all()), what + ": scales"
    unit = torch.exp2(expand(b.double(), cols) - 127)
    half = torch.maximum(size * 2.0 ** -(m + 1), unit * 2.0 ** (lowest - m - 1))
    bad = (values(p) - want).abs() > half * (1 + 2.0 ** -20) + 2 * err
    assert not bool(bad.any()), "%s: %d entries, first %s" % (what, int(bad.sum()), bad.nonzero()[0].tolist())


def check_plain(got, want, err, what=""):
    bad = ~((got.double() - want).abs() <= half_step(want, got.dtype) * (1 + 2.0 ** -8) + err)
    assert not bool(bad.any()), "%s: %d entries, first %s" % (what, int(bad.sum()), bad.nonzero()[0].tolist())


def strided(rows, cols, dtype, stride=None, offset=0, fill=float("nan")):
    """A plain matrix whose rows may begin anywhere; what is around it is NaN."""
    stride = stride or cols
    flat = torch.full((rows * stride + offset + 16,), fill, dtype=dtype, device="cuda")
    return torch.as_strided(flat, (rows, cols), (stride, 1), offset)


def random(rows, cols, seed, size=1.0):
    """Values over many powers of two."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen, device="cuda", dtype=torch.float64)
    return x * torch.exp(1.5 * torch.randn(rows, cols, generator=gen, device="cuda", dtype=torch.float64)) * size
