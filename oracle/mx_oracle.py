"""Independent fp64 CPU oracle of the microscaled layers (NumPy; shares no code
with the library): blocks of 32 values, one power of two each, E2M1 ("fp4") or
E2M3 ("fp6") elements. The rotation is the HIGGS layers'."""
from __future__ import annotations

import math

import numpy as np

from . import higgs_oracle as O

BLOCK = 32
FORMATS = {"fp4": (2, 1), "fp6": (2, 3)}    # exponent bits, mantissa bits


def magnitudes(fmt: str) -> np.ndarray:
    """The format's magnitudes in the order of their codes (bias 1, subnormals,
    no infinity and no NaN)."""
    exp_bits, man_bits = FORMATS[fmt]
    out = []
    for code in range(1 << (exp_bits + man_bits)):
        e, m = code >> man_bits, code & ((1 << man_bits) - 1)
        frac = m / (1 << man_bits)
        out.append(frac if e == 0 else 2.0 ** (e - 1) * (1 + frac))
    return np.array(out)


def code_bits(fmt: str) -> int:
    return 1 + sum(FORMATS[fmt])


def blocks(inp: int) -> int:
    return -(-inp // BLOCK)


def row_bytes(inp: int, fmt: str) -> int:
    return blocks(inp) * BLOCK * code_bits(fmt) // 8


def rotated(w: np.ndarray, g: int, seed: int) -> np.ndarray:
    # (+ 0.0: a rotated zero is positive)
    return O.rht_activations(w, g, seed) + 0.0 if g else np.asarray(w, dtype=np.float64)


def quantize(w: np.ndarray, fmt: str, g: int = 0, seed: int = 0):
    """(codes int [rows, blocks, 32], scale bytes uint8 [rows, blocks])."""
    with np.errstate(invalid="ignore", over="ignore"):
        v = rotated(w, g, seed)
    rows, inp = v.shape
    nb = blocks(inp)
    full = np.zeros((rows, nb * BLOCK))
    full[:, :inp] = v
    full = full.reshape(rows, nb, BLOCK)
    mag = np.abs(full)
    bad = ~(mag.max(axis=2) < 2.0 ** 128)           # NaN compares false
    mag[bad] = 0.0
    top = mag.max(axis=2)
    e = np.full((rows, nb), -127)
    some = top > 0
    e[some] = np.frexp(top[some])[1] - 1 - 2        # floor(log2) less the format's top exponent
    e = np.maximum(e, -127)
    scaled = np.ldexp(mag, -e[:, :, None])
    table = magnitudes(fmt)
    codes = np.zeros(scaled.shape, dtype=np.int64)
    for k in range(len(table) - 1):                 # past every border between neighbours
        mid = (table[k] + table[k + 1]) / 2
        codes += (scaled > mid) | ((scaled == mid) & (k % 2 == 1))
    codes |= np.signbit(full).astype(np.int64) << (code_bits(fmt) - 1)
    codes[bad] = 0
    scales = (e + 127).astype(np.uint8)
    scales[bad] = 255
    return codes, scales


def pack(codes: np.ndarray, fmt: str) -> np.ndarray:
    """uint8 [rows, row_bytes]: the rows' codes as bits, least significant first."""
    bits = code_bits(fmt)
    rows = codes.shape[0]
    b = (codes[..., None] >> np.arange(bits)) & 1
    return np.packbits(b.reshape(rows, -1).astype(np.uint8), axis=1, bitorder="little")


def unpack(packed: np.ndarray, fmt: str) -> np.ndarray:
    bits = code_bits(fmt)
    rows = packed.shape[0]
    b = np.unpackbits(packed, axis=1, bitorder="little").reshape(rows, -1, BLOCK, bits)
    return (b.astype(np.int64) << np.arange(bits)).sum(axis=3)


def values(codes: np.ndarray, scales: np.ndarray, fmt: str, inp: int) -> np.ndarray:
    """fp64 [rows, inp]; a block of scale 255 is NaN."""
    table = magnitudes(fmt)
    n = len(table)
    v = np.where(codes >= n, -1.0, 1.0) * table[codes % n]
    s = np.ldexp(1.0, scales.astype(np.int64) - 127)
    s = np.where(scales == 255, np.nan, s)
    return (v * s[:, :, None]).reshape(codes.shape[0], -1)[:, :inp]


def rotate_back(v: np.ndarray, g: int, seed: int) -> np.ndarray:
    rows, inp = v.shape
    h = O.hadamard(g)
    sigma = O.rht_signs(seed, g).astype(np.float64)
    return (v.reshape(rows, inp // g, g) @ h / math.sqrt(g) * sigma).reshape(rows, inp)


def quantized(w: np.ndarray, fmt: str, g: int = 0, seed: int = 0) -> np.ndarray:
    """The values that quantize() stores (in the rotated space for g > 0)."""
    return values(*quantize(w, fmt, g, seed), fmt, w.shape[1])


def row_error(w: np.ndarray, w_values: np.ndarray, g: int, seed: int) -> np.ndarray:
    """[rows, 2]: squared error and squared norm."""
    d = rotated(w, g, seed) - w_values
    w = np.asarray(w, dtype=np.float64)
    return np.stack(((d * d).sum(axis=1), (w * w).sum(axis=1)), axis=1)
