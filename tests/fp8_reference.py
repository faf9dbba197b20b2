"""8-bit blocks in 64 bits on the CPU, from their definition: what the library's kernels are compared with."""
import math

import numpy as np

BLOCK = 128


def code_values():
    """The 256 values of e4m3: sign, exponent field (bias 7), three fraction bits; no infinities, all ones is NaN."""
    v = np.empty(256)
    for c in range(256):
        field, fraction = (c >> 3) & 15, c & 7
        x = fraction * 2.0 ** -9 if field == 0 else (8 + fraction) * 2.0 ** (field - 10)
        v[c] = math.nan if c & 127 == 127 else -x if c & 128 else x
    return v


VALUES = code_values()
MAGNITUDES = VALUES[:127]          # ascending, codes 0 .. 126


def planes(rows, cols):
    """(columns of the code plane, columns of the exponent plane)"""
    blocks = -(-cols // BLOCK)
    return blocks * BLOCK, -(-blocks // 4) * 4


def encode(x):
    """(codes, exponents) of a float64 matrix that holds values of a narrower type."""
    rows, cols = x.shape
    C, E = planes(rows, cols)
    codes, exps = np.zeros((rows, C), np.uint8), np.zeros((rows, E), np.uint8)
    for b in range(C // BLOCK):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        top = np.where(np.isfinite(part), np.abs(part), 0.0).max(axis=1, initial=0.0)
        # the least s with top <= 448 * 2^s: 448 2^s = 0.875 * 2^(s + 9)
        fraction, e = np.frexp(top)
        s = np.where(top == 0, -110, np.clip(e - 9 + (fraction > 0.875), -110, 120)).astype(int)
        exps[:, b] = s + 127
        scaled = np.ldexp(np.where(np.isfinite(part), part, 0.0), -s[:, None])
        # the nearest magnitude; of two equally near ones the even code
        at = np.clip(np.searchsorted(MAGNITUDES, np.abs(scaled)), 1, 126)
        low, high = MAGNITUDES[at - 1], MAGNITUDES[at]
        below, above = np.abs(scaled) - low, high - np.abs(scaled)
        up = (above < below) | ((above == below) & (at % 2 == 0))
        c = np.where(up, at, at - 1) | (np.signbit(part) * 128)
        codes[:, b * BLOCK:b * BLOCK + part.shape[1]] = np.where(np.isfinite(part), c, 127)
    return codes, exps


def decode(codes, exps, cols):
    rows, C = codes.shape
    scale = np.ldexp(1.0, np.repeat(exps[:, :C // BLOCK].astype(int) - 127, BLOCK, axis=1))
    return (VALUES[codes] * scale)[:, :cols]


def same_codes(got, want):
    """Codes are equal, a NaN of either sign to a NaN."""
    return np.array_equal(np.where(got & 127 == 127, 127, got), np.where(want & 127 == 127, 127, want))


def sigma(x):
    return 1 / (1 + np.exp(-x))


def act(name, g):
    """(value, derivative)"""
    if name == "silu":
        s = sigma(g)
        return g * s, s + g * s * (1 - s)
    c = math.sqrt(2 / math.pi)
    w, dw = c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g ** 2)
    return 0.5 * g * (1 + np.tanh(w)), 0.5 * (1 + np.tanh(w)) + 0.5 * g * (1 - np.tanh(w) ** 2) * dw


def random_blocks(rng, rows, cols, scale=1.0):
    """(codes, exponents, values) of a Gaussian matrix with a few loud columns and rows of different size."""
    x = rng.standard_normal((rows, cols)) * scale * np.exp(0.5 * rng.standard_normal((rows, 1)))
    if cols:
        x[:, rng.integers(0, cols, max(1, cols // 100))] *= 10
    c, e = encode(x)
    return c, e, decode(c, e, cols)
