"""The rotated way back of microscaled layers over the whole range of their scale
bytes: finite results stay finite, tiny ones keep their bits, sums that fp32 holds
are rounded once."""
import sys

import numpy as np
import pytest

from oracle import mx_oracle as M

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
FMTS = ["fp4", "fp6"]
GROUPS = [64, 128, 256, 512, 1024, 2048, 4096]
LARGEST = {"f32": float(np.finfo(np.float32).max), "bf16": float(2.0 ** 127 * (2 - 2.0 ** -7))}


def announce(msg):
    print(f"[gpu-case] mx range {msg}", file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def H():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2411_17525_amd import higgs
    higgs.lib()
    return higgs


def back(H, packed, scales, inp, fmt, g, seed, dtype):
    """The call's result in fp64."""
    return H.mx_dequantize(torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda(), inp,
                           H.MX_FP4 if fmt == "fp4" else H.MX_FP6, g, seed,
                           dtype=torch.bfloat16 if dtype == "bf16" else torch.float32
                           ).double().cpu().numpy()


def check(got, packed, scales, inp, fmt, g, seed, dtype):
    rows = packed.shape[0]
    v = M.values(M.unpack(packed, fmt), scales, fmt, inp)
    want = M.rotate_back(v, g, seed)
    # log2 g levels of fp32 sums, each off by 2^-24 of at most the group's sum |v|, and
    # the multiplication by 1 / sqrt(g) by 2^-24 (its factor by 2^-48, hence "2"); below
    # fp32's normal range by half its last bit, 2^-150, in each of two steps
    top = np.repeat(np.abs(v).reshape(rows, -1, g).sum(axis=2), g, axis=1) / np.sqrt(g)
    tol = (np.log2(g) + 2) * 2.0 ** -24 * top + 2.0 ** -149
    if dtype == "bf16":     # rounded once more: half a step, or half of bf16's last bit
        tol = tol + 2.0 ** -8 * np.abs(want) + 2.0 ** -134
    inside = np.abs(want) + tol < LARGEST[dtype]
    assert np.isfinite(got[inside]).all()
    assert (np.abs(got - want)[inside] <= tol[inside]).all()
    # (up to half a step above the largest value a result may be rounded to it)
    outside = np.abs(want) - tol > LARGEST[dtype] * (1 + 2.0 ** -8)
    assert np.array_equal(got[outside], np.copysign(np.inf, want[outside]))
    return inside, outside


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
def test_a_large_weight_comes_back(H, g, fmt, dtype):
    """One weight of 5e36 .. 2^127 among zeros, quantized and brought back."""
    for spike in (5e36, 2e37, -2.0 ** 124, 2.0 ** 127):
        announce(f"spike {spike:g} g={g} {fmt} {dtype}")
        w = np.zeros((2, 2 * g), dtype=np.float32)
        w[0, g // 3] = spike
        w[1, 2 * g - 1] = -spike
        t = torch.from_numpy(w).cuda()
        codes, scales = H.mx_quantize(t.bfloat16() if dtype == "bf16" else t,
                                      H.MX_FP4 if fmt == "fp4" else H.MX_FP6, g, 11)
        packed, sc = codes.cpu().numpy(), scales.cpu().numpy()
        assert sc.max() < 255
        got = back(H, packed, sc, 2 * g, fmt, g, 11, dtype)
        inside, _ = check(got, packed, sc, 2 * g, fmt, g, 11, dtype)
        assert inside.all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
@pytest.mark.parametrize("lo,hi", [(0, 1), (0, 40), (14, 19), (225, 255), (250, 255), (0, 255)])
def test_all_scale_bytes(H, g, fmt, dtype, lo, hi):
    """Any codes with scale bytes of lo .. hi - 1: the smallest, the largest, all."""
    announce(f"bytes {lo}..{hi} g={g} {fmt} {dtype}")
    rng = np.random.default_rng(g + lo + hi)
    rows, inp = 3, 5 * g
    packed = rng.integers(0, 256, (rows, M.row_bytes(inp, fmt)), dtype=np.uint8)
    scales = rng.integers(lo, hi, (rows, M.blocks(inp)), dtype=np.uint8)
    got = back(H, packed, scales, inp, fmt, g, 5, dtype)
    inside, outside = check(got, packed, scales, inp, fmt, g, 5, dtype)
    assert inside.any()
    if lo == 250:
        assert outside.any()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
def test_exact_sums_are_rounded_once(H, g, fmt):
    """Blocks of nearby exponents: fp32 holds every sum (multiples of 2^-3 of the smallest
    block's power of two, below 2^3 of the largest's times 4096: 18 bits and the exponents'
    spread of 3), so the result is off by one rounding, half a step."""
    announce(f"rounded once g={g} {fmt}")
    rng = np.random.default_rng(g)
    rows, inp = 7, 2 * g
    packed = rng.integers(0, 256, (rows, M.row_bytes(inp, fmt)), dtype=np.uint8)
    scales = rng.integers(118, 122, (rows, M.blocks(inp)), dtype=np.uint8)
    got = back(H, packed, scales, inp, fmt, g, 9, "f32")
    want = M.rotate_back(M.values(M.unpack(packed, fmt), scales, fmt, inp), g, 9)
    # (2^-16: the factor here, to 48 bits; 2^-40: the oracle's sums and factor in fp64, up to
    # 16 roundings of 2^-53 of a sum of 4096 values below 2^-3)
    assert (np.abs(got - want) <= 2.0 ** -24 * (1 + 2.0 ** -16) * np.abs(want) + 2.0 ** -40).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
def test_nan_stays_in_its_group(H, g, fmt):
    announce(f"NaN group g={g} {fmt}")
    rng = np.random.default_rng(g)
    inp = 4 * g
    packed = rng.integers(0, 256, (2, M.row_bytes(inp, fmt)), dtype=np.uint8)
    scales = rng.integers(100, 140, (2, M.blocks(inp)), dtype=np.uint8)
    scales[1, (2 * g + g // 2) // 32] = 255
    got = back(H, packed, scales, inp, fmt, g, 5, "f32")
    nan = np.zeros((2, inp), dtype=bool)
    nan[1, 2 * g:3 * g] = True
    assert np.array_equal(np.isnan(got), nan)
    clean = scales.copy()
    clean[1, (2 * g + g // 2) // 32] = 0
    assert np.array_equal(got[~nan], back(H, packed, clean, inp, fmt, g, 5, "f32")[~nan])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("batch", [1, 9, 24, 80, 300])
@pytest.mark.parametrize("x_power,lo,hi", [(-110, 225, 255), (110, 0, 16), (0, 100, 140),
                                           (-60, 40, 68)])
def test_product_over_the_range(H, batch, fmt, x_power, lo, hi):
    """Weights of the largest and the smallest scale bytes with activations that bring the
    products back into fp32's range, and sums just above its smallest normal value."""
    announce(f"product batch={batch} x 2^{x_power} bytes {lo}..{hi} {fmt}")
    out, inp = 70, 1088
    rng = np.random.default_rng(batch + lo)
    x = np.ldexp(rng.standard_normal((batch, inp)), x_power).astype(np.float32)
    packed = rng.integers(0, 256, (out, M.row_bytes(inp, "fp4")), dtype=np.uint8)
    scales = rng.integers(lo, hi, (out, M.blocks(inp)), dtype=np.uint8)
    y = H.mx_qmatmul(torch.from_numpy(x).cuda(), torch.from_numpy(packed).cuda(),
                     torch.from_numpy(scales).cuda(), H.MX_FP4 if fmt == "fp4" else H.MX_FP6, 0, 0,
                     out).double().cpu().numpy()
    xq = M.quantized(x.astype(np.float64), fmt)
    wq = M.values(M.unpack(packed, "fp4"), scales, "fp4", inp)
    want, size = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    # exact products; one rounding of a partial sum per 64 of K, one per part (at most 16)
    tol = (-(-inp // 64) + 16) * 2.0 ** -24 * size
    assert (np.abs(y - want) <= tol).all()
