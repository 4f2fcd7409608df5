"""Matrices in 8 bits, norm and dropout in numpy, from the definitions: what the GPU tests compare with."""
import numpy as np
import torch

DEV = "cuda:0"
U = 2.0 ** -24            # half a step of fp32
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def values_of_codes():
    """The 256 e4m3 values."""
    b = np.arange(256)
    e, f = (b >> 3) & 15, b & 7
    v = np.where(e > 0, np.ldexp(8.0 + f, e - 10), np.ldexp(1.0 * f, -9))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b > 127, -v, v)


CODES = values_of_codes()


def scale_exponents(largest):
    """k of the smallest 2^k, k >= -127, with largest <= 448 2^k; 0 for zero."""
    f, e = np.frexp(largest)                   # largest = f 2^e, f in [1/2, 1); 448 = 0.875 2^9
    k = e - 9 + (f > 0.875)
    return np.where(largest > 0, np.maximum(k, -127), 0)


def nearest_codes(x):
    """The bytes of the e4m3 values nearest to |x| <= 448 (ties to even); what is not finite: NaN with its sign."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    _, e = np.frexp(a)
    e = np.where(a > 0, np.maximum(e - 1, -6), -6)  # a in [2^e, 2^(e+1)), or below the normal range
    q = np.rint(np.ldexp(a, 3 - e))            # 8 .. 16 eighths (0 .. 8 below): np.rint rounds ties to even
    byte = ((e + 6) * 8 + q).astype(np.int64)  # (a q of 16 carries into the exponent, 8 of the lowest is its first)
    byte = np.where(np.isfinite(x), byte, 127)
    return (byte + 128 * np.signbit(x)).astype(np.uint8)


def quantize(x, square=False):
    """Codes and scale bytes (unpadded) of a float64 matrix."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    finite = np.where(np.isfinite(x), np.abs(x), 0.0)
    top = np.zeros((rows, nb))
    for b in range(nb):
        top[:, b] = finite[:, b * 128:(b + 1) * 128].max(1)
    if square:
        for t in range(0, rows, 128):
            top[t:t + 128] = top[t:t + 128].max(0)
    k = scale_exponents(top)
    codes = nearest_codes(np.ldexp(x, -np.repeat(k, 128, 1)[:, :cols]))
    return codes, (k + 127).astype(np.uint8)


def decode(codes, scales, cols):
    with np.errstate(invalid="ignore"):
        return np.ldexp(CODES[codes[:, :cols]], np.repeat(scales.astype(np.int64), 128, 1)[:, :cols] - 127)


def kept(total, p, seed, offset):
    """The mask of `total` elements: Philox 4x32 with ten rounds on whole numbers."""
    n = -(-total // 8)
    m32 = np.uint64(0xFFFFFFFF)
    at = np.arange(n, dtype=np.uint64)
    c = [at & m32, at >> np.uint64(32), np.full(n, offset & 0xFFFFFFFF, np.uint64), np.full(n, offset >> 32, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & m32, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & m32]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    bits = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in c for s in (0, 16)], 1).reshape(-1)[:total]
    return bits >= round(p * 65536)


def matrix(gen, rows, cols, dtype, std=1.0, pad=0, shift=0):
    """A device matrix of `rows` rows, `pad` elements apart and `shift` elements into an array of NaN."""
    wide = cols + pad
    full = torch.full((rows * wide + shift + 8,), float("nan"), dtype=dtype)
    view = full[shift:shift + rows * wide].view(rows, wide)[:, :cols]
    view.copy_((torch.randn(rows, cols, generator=gen, dtype=torch.float64) * std).to(dtype))
    full = full.to(DEV)
    return full[shift:shift + rows * wide].view(rows, wide)[:, :cols]


def around(t, rows, cols):
    """What lies around a view that `matrix` made."""
    full = t._base if t._base is not None else t
    flat = full.reshape(-1)
    mask = torch.ones(flat.numel(), dtype=torch.bool, device=flat.device)
    at = t.storage_offset() + torch.arange(rows, device=flat.device)[:, None] * t.stride(0) + torch.arange(cols, device=flat.device)
    mask[at.reshape(-1)] = False
    return flat[mask]


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()
