"""Reference of the 8-bit operands in 64 bits, from the definitions: numpy only, nothing of the library."""
import numpy as np
import torch

U = 2.0 ** -24            # unit roundoff of fp32
BF16 = 2.0 ** -8          # half a step of bf16, relative
GROUP = 128

# the 127 non-negative finite e4m3 values in code order: code c has exponent field c >> 3 (bias 7) and three mantissa bits
TABLE = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def encode(v):
    """e4m3 codes of v (64 bits), nearest, ties to the even code."""
    a = np.abs(v)
    lo = np.clip(np.searchsorted(TABLE, a, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    down, up = a - TABLE[lo], TABLE[hi] - a
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = np.where(np.signbit(v) & (v != 0), code | 0x80, code)
    return np.where(np.isnan(v), 0x7F, code).astype(np.uint8)


def decode(codes):
    c = codes.astype(np.int64)
    v = np.where((c & 127) == 127, np.nan, TABLE[np.minimum(c & 127, 126)])
    return np.where(c & 128, -v, v)


def spread(s, block_rows, rows, K):
    return s[np.arange(rows) // block_rows][:, np.arange(K) // GROUP]


def quantize(x, block_rows):
    """codes (uint8), scales (64 bits) of a float array."""
    x = x.astype(np.float64)
    rows, K = x.shape
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    amax = np.stack([fin[:, k:k + GROUP].max(axis=1) for k in range(0, K, GROUP)], axis=1)
    amax = np.stack([amax[r:r + block_rows].max(axis=0) for r in range(0, rows, block_rows)], axis=0)
    m, e = np.frexp(amax)                                  # amax = m 2^e, 448 = 0.875 2^9
    e = np.where(amax > 0, e - 9 + (m > 0.875), -117)
    s = np.ldexp(1.0, np.maximum(e, -117))
    v = np.where(np.isfinite(x), x, np.nan) / spread(s, block_rows, rows, K)
    return encode(v), s


def values(codes, s, block_rows):
    rows, K = codes.shape
    return decode(codes) * spread(s.astype(np.float64), block_rows, rows, K)


def binarize_backward(codes, s, gy, beta):
    """Eq. 6 with the dequantized values for x and the codes' sign bits for Sign(x); and the magnitude its rounding follows."""
    x, g = values(codes, s, 1), gy.astype(np.float64)
    sign = np.where(codes & 0x80, -1.0, 1.0)
    out, mag = np.empty_like(g), np.empty_like(g)
    for k in range(0, x.shape[1], beta):
        sl = slice(k, min(k + beta, x.shape[1]))
        delta = np.abs(x[:, sl]).mean(axis=1, keepdims=True)
        back = (g[:, sl] * sign[:, sl]).mean(axis=1, keepdims=True)
        with np.errstate(invalid="ignore"):
            out[:, sl] = sign[:, sl] * back + np.where(np.abs(x[:, sl]) <= 1, delta * g[:, sl], 0.0)
        mag[:, sl] = np.abs(g[:, sl]).mean(axis=1, keepdims=True) + delta * np.abs(g[:, sl])
    return out, mag


def held(x, block_rows, scales="pow2", pad=0):
    """An 8-bit operand of x, made here: (Fp8Operand on the device, its values in 64 bits, codes, scales).  `pad`: columns more
    than a whole number of 16 bytes, filled with NaN codes, and scales behind the last group filled with NaN."""
    from paper_1905_10759_b200 import hbmm
    rows, K = x.shape
    codes, s = quantize(x, block_rows)
    if scales == "any":                                    # scales of another program: no powers of two
        s = s * np.random.default_rng(rows + K).uniform(1.0, 1.99, s.shape)
    s = s.astype(np.float32)
    c = np.full((rows, -(-K // 16) * 16 + pad), 0x7F, dtype=np.uint8)
    c[:, :K] = codes
    t = np.full((s.shape[0], -(-s.shape[1] // 4) * 4), np.nan, dtype=np.float32)
    t[:, :s.shape[1]] = s
    op = hbmm.Fp8Operand(torch.from_numpy(c).cuda(), torch.from_numpy(t).cuda(), K, block_rows)
    return op, values(codes, s, block_rows), codes, s


def framed(rows, cols, dtype, step):
    """A NaN-filled [rows, cols] view inside a larger NaN-filled buffer, rows `step`-aligned, and a check that nothing outside was
    written."""
    ld = -(-cols // step) * step + step
    buf = torch.full((rows + 2, ld), float("nan"), dtype=dtype, device="cuda")
    view = buf[1:rows + 1, :cols]

    def clean():
        rest = buf.clone()
        rest[1:rows + 1, :cols] = float("nan")
        return bool(torch.isnan(rest).all())
    return view, clean
