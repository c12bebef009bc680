"""The AdamW step's formulas in numpy, operation by operation: states bit for bit (every fp32 operation of numpy
rounds as the formulas say), the parameters in 64 bits."""
import numpy as np

BLOCK = 256
F = np.float32


def mix(x):
    x = np.asarray(x, dtype=np.uint64) & 0xFFFFFFFF
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0xBB67AE85)) & np.uint64(0xFFFFFFFF)
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0xA54FF53B)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(n, block0, seed, t):
    k = np.uint64(0)
    for w in (seed & 0xFFFFFFFF, seed >> 32, t & 0xFFFFFFFF, t >> 32):
        k = mix((int(k) ^ w) + 0x3C6EF373)
    i = np.arange(n, dtype=np.uint64)
    b = mix(k + (np.uint64(block0) + i // np.uint64(BLOCK)) * np.uint64(0x9E3779B9))
    return mix(b + (i % np.uint64(BLOCK)) * np.uint64(0x9E3779B9))


def values_of(fraction_bits):
    """Value of every code 0 .. 127: e4m3 (3; the last one is NaN) or e5m2 (2; the last four are infinity and NaN)."""
    exponent_bits = 7 - fraction_bits
    bias = (1 << (exponent_bits - 1)) - 1
    out = np.empty(128, dtype=np.float64)
    for c in range(128):
        e, f = c >> fraction_bits, c & ((1 << fraction_bits) - 1)
        out[c] = np.ldexp(f, 1 - bias - fraction_bits) if e == 0 else np.ldexp(f + (1 << fraction_bits), e - bias - fraction_bits)
    out[127] = np.nan
    if fraction_bits == 2:
        out[124], out[125:] = np.inf, np.nan
    return out


E4M3, E5M2 = values_of(3), values_of(2)


def decode(codes, scales, table, signed):
    n = len(codes)
    v = table[codes & 0x7F].astype(F) * np.repeat(np.ldexp(F(1), scales.astype(np.int32) - 127), BLOCK)[:n].astype(F)
    return np.where(codes & 0x80, -v, v).astype(F) if signed else v.astype(F)


def encode(x, r16, table, top, signed):
    """Codes and scales; the neighbours are looked up in the table of values, not made from bits."""
    n, blocks = len(x), -(-len(x) // BLOCK)
    mag = np.abs(x)
    fine = np.isfinite(mag)
    padded = np.zeros(blocks * BLOCK, dtype=F)
    padded[:n] = np.where(fine, mag, 0)
    most = padded.reshape(blocks, BLOCK).max(1)
    scales = np.maximum((most.view(np.int32) >> 23) - top, 0).astype(np.int64)
    z = np.where(fine, mag, 0).astype(np.float64) / np.repeat(np.ldexp(1.0, scales - 127), BLOCK)[:n]
    values = table[:124]
    low = np.searchsorted(values, z, side="right") - 1
    spacing = values[low + 1] - values[low]
    # far below the smallest spacing fp32 has no bits left: its smallest unit is 2^-20 (e4m3), 2^-21 (e5m2) of it
    unit = spacing[:] * 2.0 ** -(20 if top == 7 else 21)
    rest = np.rint((z - values[low]) / unit) * unit if n else z
    up = rest / spacing + (r16.astype(np.float64) + 0.5) / 65536 >= 1
    codes = low + up
    if not signed:
        codes = np.where((mag > 0) & (codes == 0), 1, codes)
        codes = np.where(np.isposinf(x), 124, np.where(np.isnan(x), 127, codes))
    else:
        codes = np.where(fine, codes | np.where(np.signbit(x), 128, 0), 127)       # (a NaN's sign says nothing)
    return codes.astype(np.uint8), scales.astype(np.uint8)


def step(p, g, m, v, hp, t, scale=1.0, decay=True):
    """p (float64, not rounded), m, v (fp32, as the formulas round them) and how far p may be off."""
    b1, c1, b2, c2 = F(hp["beta1"]), F(1 - hp["beta1"]), F(hp["beta2"]), F(1 - hp["beta2"])
    with np.errstate(all="ignore"):
        g = (g.astype(F) * F(scale)).astype(F)
        a, b = b1 * m, c1 * g
        m, v = (a + b).astype(F), (b2 * v + c2 * (g * g)).astype(F)
        m64, v64, p64 = m.astype(np.float64), v.astype(np.float64), p.astype(np.float64)
        up = hp["lr"] / (1 - hp["beta1"] ** t) * m64 / (np.sqrt(v64 / (1 - hp["beta2"] ** t)) + hp["eps"])
        wd = hp["lr"] * hp.get("weight_decay", 0.0) * p64 * decay
        # root and reciprocal 2^-22 each; factors, products and sums 8 x 2^-24 of the update; the decay's factor, product and
        # sum 4 x 2^-24; the parameter's own rounding 2^-24 of the result
        tol = np.abs(up) * (2.0 ** -21 + 8 * 2.0 ** -24) + np.abs(wd) * 4 * 2.0 ** -24 + np.abs(p64 - wd - up) * 2.0 ** -24 + 1e-44
    return p64 - wd - up, m, v, tol
