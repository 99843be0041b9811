"""Pins of the microscaled oracle: the element formats by their definition, a
hand-worked block, rounding and packing."""
import numpy as np
import pytest

from oracle import higgs_oracle as O
from oracle import mx_oracle as M


def test_magnitudes():
    assert M.magnitudes("fp4").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    m6 = M.magnitudes("fp6")
    assert m6.tolist() == ([k / 8 for k in range(16)] + [2 + k / 4 for k in range(8)]
                           + [4 + k / 2 for k in range(8)])


def test_hand_worked_block():
    w = np.zeros((1, 34))
    # largest magnitude 7 -> 2^2 -> E = 0; 7 saturates at 6; ties to even codes
    w[0, :10] = [7, -7, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, 5.0, -0.2]
    w[0, 32:] = [0.011, -0.01]      # second block, of two values: 2^-7 -> E = -9
    codes, scales = M.quantize(w, "fp4")
    assert scales.tolist() == [[127, 118]]
    assert codes[0, 0, :10].tolist() == [7, 15, 0, 2, 10, 4, 4, 6, 6, 8]
    # 0.011 * 512 = 5.632 -> 6; 0.01 * 512 = 5.12 -> 6
    assert codes[0, 1, :3].tolist() == [7, 15, 0]
    packed = M.pack(codes, "fp4")
    assert packed.shape == (1, 32) == (1, M.row_bytes(34, "fp4"))
    assert packed[0, :5].tolist() == [0xF7, 0x20, 0x4A, 0x64, 0x86]
    assert np.array_equal(M.unpack(packed, "fp4"), codes)
    v = M.values(codes, scales, "fp4", 34)
    assert v[0, :10].tolist() == [6, -6, 0, 1, -1, 2, 2, 4, 4, 0]
    assert v[0, 32:].tolist() == [6 / 512, -6 / 512]


def test_fp6_packing():
    codes = np.zeros((1, 1, 32), dtype=np.int64)
    codes[0, 0, :4] = [0b000001, 0b100000, 0b111111, 0b000010]
    packed = M.pack(codes, "fp6")
    # 1 | 32 << 6 | 63 << 12 | 2 << 18
    word = 1 | 32 << 6 | 63 << 12 | 2 << 18
    assert packed.shape == (1, 24)
    assert packed[0, :3].tolist() == [word & 255, word >> 8 & 255, word >> 16]
    assert np.array_equal(M.unpack(packed, "fp6"), codes)


@pytest.mark.parametrize("fmt", ["fp4", "fp6"])
def test_nearest(fmt):
    """Every value is rounded to the nearest of its block's points."""
    rng = np.random.default_rng(1)
    w = rng.standard_normal((8, 96)) * np.exp(rng.standard_normal((8, 1)) * 4)
    codes, scales = M.quantize(w, fmt)
    v = M.values(codes, scales, fmt, 96)
    t = M.magnitudes(fmt)
    points = np.concatenate((-t, t))
    s = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, axis=1)
    best = np.abs(w[:, :, None] - points * s[:, :, None]).min(axis=2)
    assert np.array_equal(np.abs(w - v), best)


@pytest.mark.parametrize("fmt", ["fp4", "fp6"])
def test_special_blocks(fmt):
    w = np.ones((1, 32 * 6))
    w[0, 3] = np.nan
    w[0, 35] = -np.inf
    w[0, 64:96] = 0.0
    w[0, 96:128] = 2.0 ** -149
    w[0, 128] = np.finfo(np.float32).max
    codes, scales = M.quantize(w, fmt)
    assert scales[0].tolist() == [255, 255, 0, 0, 252, 125]
    assert not codes[0, :4].any()
    v = M.values(codes, scales, fmt, w.shape[1])[0]
    assert np.isnan(v[:64]).all() and not v[64:128].any() and (v[160:] == 1).all()


def test_rotation_keeps_norms_and_comes_back():
    rng = np.random.default_rng(3)
    w = rng.standard_normal((3, 256))
    r = M.rotated(w, 64, 5)
    assert np.allclose((r * r).sum(axis=1), (w * w).sum(axis=1), rtol=1e-13)
    assert np.allclose(M.rotate_back(r, 64, 5), w, atol=1e-13)
    q = M.quantized(w, "fp4", 64, 5)
    # the error is the same in both spaces
    err = M.row_error(w, q, 64, 5)[:, 0]
    back = M.rotate_back(q, 64, 5)
    assert np.allclose(err, ((w - back) ** 2).sum(axis=1), rtol=1e-12)
    assert abs(O.layer_error(w, back) - err.sum() / (w * w).sum()) < 1e-12
