"""Plain references of the 8-bit operators, in numpy: E4M3 by searching its table of values, block scales by trying
exponents, Philox4x32-10 in 64-bit words, AdamW's sequence operation by operation in binary32 (which numpy rounds as
IEEE asks, so its bits are the canonical ones) and once more in binary64."""
import math

import numpy as np

BLOCK = 128


def _e4m3_values():
    v = []
    for c in range(127):
        e, m = c >> 3, c & 7
        v.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(v)


E4M3 = _e4m3_values()  # of codes 0 .. 126, ascending


def e4m3_value(codes):
    codes = np.asarray(codes, np.uint8)
    mag = codes & 0x7F
    v = np.where(mag == 0x7F, np.nan, E4M3[np.minimum(mag, 126)])
    return np.where(codes & 0x80, -v, v)


def e4m3_nearest(y):
    """Codes of binary64 values: nearest, ties to the even code, saturating; NaN is 0x7F."""
    y = np.asarray(y, np.float64)
    a = np.minimum(np.nan_to_num(np.abs(y), nan=0.0, posinf=448.0), 448.0)
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    c = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    c = np.where(np.isnan(y), 0x7F, c | np.where(np.signbit(y), 0x80, 0))
    return c.astype(np.uint8)


def e4m3_stochastic(y, r):
    """Codes of binary32 values y by 16 random bits each: the value at or below |y| + r 2^-16 steps of the grid; below
    2^-6, where the grid's step is 2^-9, after |y| + 2^-6 is rounded to binary32."""
    y = np.asarray(y, np.float32)
    a = np.abs(y)
    small = a < np.float32(2.0 ** -6)
    z = np.where(small, a + np.float32(2.0 ** -6), a).astype(np.float64)
    ok = a <= 448.0
    z = np.where(ok, z, 1.0)
    step = 2.0 ** (np.frexp(np.maximum(z, 2.0 ** -6))[1] - 4.0)
    q = np.floor(z / step + np.asarray(r, np.float64) / 65536.0) * step - np.where(small, 2.0 ** -6, 0.0)
    c = np.searchsorted(E4M3, q)
    assert np.array_equal(E4M3[np.minimum(c, 126)][ok], q[ok])  # on the grid
    return np.where(ok, c | np.where(np.signbit(y), 0x80, 0), e4m3_nearest(y)).astype(np.uint8)


def exponent(a):
    """The smallest k in [-127, 127] with a <= 448 * 2^k; 0 for 0."""
    if a == 0:
        return 0
    k = -127
    while a > math.ldexp(448.0, k):
        k += 1
    return k


def finite_max(x):
    x = np.asarray(x, np.float64)
    x = np.abs(x[np.isfinite(x)])
    return float(x.max()) if x.size else 0.0


def quantize(x, square):
    """(codes [rows, cols], exponents [rows, blocks]) of the float matrix x."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    k = np.zeros((rows, nb), np.int64)
    codes = np.zeros((rows, cols), np.uint8)
    for c in range(nb):
        sl = slice(c * BLOCK, min(cols, (c + 1) * BLOCK))
        if square:
            for r in range(0, rows, BLOCK):
                k[r:r + BLOCK, c] = exponent(finite_max(x[r:r + BLOCK, sl]))
        else:
            for r in range(rows):
                k[r, c] = exponent(finite_max(x[r, sl]))
        codes[:, sl] = e4m3_nearest(np.ldexp(x[:, sl].astype(np.float64), -k[:, c:c + 1]))
    return codes, k


def stored_scales(k):
    """E8M0 bytes of the exponents k [rows, blocks] in the stored order, 127 in the padding."""
    rows, nb = k.shape
    out = np.full((-(-rows // BLOCK), -(-nb // 4), 32, 4, 4), 127, np.uint8)
    for r in range(rows):
        for c in range(nb):
            out[r // 128, c // 4, r % 32, r % 128 // 32, c % 4] = k[r, c] + 127
    return out


def philox(blocks, word1_high, t, seed):
    """[n, 4] words of counters (block lo, block hi | word1_high << 31, t lo, t hi) under the key `seed`."""
    m = np.uint64(0xFFFFFFFF)
    b = np.asarray(blocks, np.uint64)
    s32 = np.uint64(32)
    x = [b & m, (b >> s32) | np.uint64(word1_high << 31), np.full_like(b, t & 0xFFFFFFFF), np.full_like(b, t >> 32)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> s32) ^ x[1] ^ np.uint64(k0), q & m, (p >> s32) ^ x[3] ^ np.uint64(k1), p & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(x, 1)


def weight_lanes(first, n, t, seed):
    """16 random bits of the global elements first .. first + n - 1 (first a multiple of 8)."""
    w = philox(np.arange(first // 8, (first + n + 7) // 8), 0, t, seed)
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[:n]


def state_lanes(first, n, t, seed):
    w = philox(np.arange(first // 4, (first + n + 3) // 4), 1, t, seed).reshape(-1)[:n]
    return w & np.uint64(0xFFFF), w >> np.uint64(16)


def bf16_nearest(x):
    """BF16 bits of binary32 values, nearest-even; NaN is 0x7FFF."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = (b + np.uint64(0x7FFF) + ((b >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16)
    return np.where(np.isnan(x), 0x7FFF, r).astype(np.uint16)


def bf16_stochastic(x, lanes):
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = (b >> np.uint64(16)) + (lanes < (b & np.uint64(0xFFFF))).astype(np.uint64)
    return np.where(np.isnan(x), 0x7FFF, r).astype(np.uint16)


def bf16_value(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)


def blocks_of(x):
    return [x[i:i + BLOCK] for i in range(0, len(x), BLOCK)]


def decode_blocks(codes, scales):
    s = np.repeat(np.ldexp(1.0, scales.astype(np.int64) - 127), BLOCK)[:len(codes)]
    return (e4m3_value(codes) * s).astype(np.float32)  # exact, but for subnormal results


def encode_blocks(x, lanes, keep):
    codes, scales = [], []
    for i, b in enumerate(blocks_of(x)):
        k = exponent(finite_max(b))
        with np.errstate(over="ignore", under="ignore", invalid="ignore"):
            y = (b * np.float32(math.ldexp(1.0, -k))).astype(np.float32)
        c = e4m3_nearest(y) if lanes is None else e4m3_stochastic(y, lanes[i * BLOCK:i * BLOCK + len(b)])
        if keep:
            c = np.where((b > 0) & (c == 0), 1, c).astype(np.uint8)
        codes.append(c)
        scales.append(k + 127)
    return np.concatenate(codes), np.array(scales, np.uint8)


def adamw(w, g, m, v, *, t, lr, beta1, beta2, eps, weight_decay, mult=None, dtype=np.float32):
    """(w', m', r', v') in `dtype`; with binary32, every operation rounded on its own, in the canonical order."""
    f = dtype
    b1, b2 = float(np.float32(beta1)), float(np.float32(beta2))
    lr = float(np.float32(lr))
    omb1, omb2, ka = f(1.0 - b1), f(1.0 - b2), f(lr / (1.0 - b1 ** t))
    c2, kwd = f(1.0 / math.sqrt(1.0 - b2 ** t)), f(lr * float(np.float32(weight_decay)))
    w, g, m, v = (np.asarray(x, f) for x in (w, g, m, v))
    with np.errstate(all="ignore"):
        if mult is not None:
            g = g * f(mult)
        m = m * f(b1) + g * omb1
        v = v * f(b2) + (g * g) * omb2
        r = np.sqrt(v)
        u = (m * ka) / (r * c2 + f(np.float32(eps)))
        return ((w - w * kwd) if kwd else w) - u, m, r, v
