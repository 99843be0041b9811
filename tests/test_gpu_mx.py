"""The microscaled operators on the GPU against the fp64 oracle: codes and scale
bytes exactly, stored values exactly, the rotation back, the layer error and the
product within bounds of fp32 / fp64 summation that are worked out here."""
import sys

import numpy as np
import pytest

from oracle import mx_oracle as M

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
FMTS = ["fp4", "fp6"]
GROUPS = [64, 128, 256, 512, 1024, 2048, 4096]


def announce(msg):
    print(f"[gpu-case] mx {msg}", file=sys.stderr, flush=True)


@pytest.fixture(scope="module")
def H():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2411_17525_amd import higgs
    higgs.lib()
    return higgs


def fmt_of(H, fmt):
    return H.MX_FP4 if fmt == "fp4" else H.MX_FP6


def cast(a, dtype):
    """(device tensor of dtype, its values in fp64)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    return t.cuda(), t.double().numpy()


def normal(rows, inp, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    a = rng.standard_normal((rows, inp))
    return a * np.exp(spread * rng.standard_normal((rows, inp)))


def same_codes(H, w, fmt, g, seed, dtype):
    t, v = cast(w, dtype)
    codes, scales = H.mx_quantize(t, fmt_of(H, fmt), g, seed)
    torch.cuda.synchronize()
    want_c, want_s = M.quantize(v, fmt, g, seed)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.cpu().numpy(), M.pack(want_c, fmt))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,inp", [(1, 1), (3, 15), (2, 16), (5, 17), (7, 31), (1, 32), (9, 33),
                                      (4, 47), (33, 100), (3, 4999), (300, 8), (17, 4096)])
def test_quantize_plain(H, rows, inp, fmt, dtype):
    announce(f"quantize {rows}x{inp} {fmt} {dtype}")
    same_codes(H, normal(rows, inp, rows + inp), fmt, 0, 0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
def test_quantize_rotated(H, g, fmt, dtype):
    # one group; rows that leave a segment of 1024 part empty; several segments
    for rows, inp in ((1, g), (3, 3 * g), (37, 5 * g if g < 1024 else g)):
        announce(f"quantize {rows}x{inp} g={g} {fmt} {dtype}")
        same_codes(H, normal(rows, inp, g + rows), fmt, g, 77 + g, dtype)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", [0, 64])
def test_quantize_borders(H, fmt, g):
    """Values on the borders between codes, and one step beside them, in blocks
    of every exponent; with a rotation whole numbers whose sums fall on borders."""
    announce(f"borders {fmt} g={g}")
    if g:
        rng = np.random.default_rng(5)
        w = rng.integers(-8, 9, (400, 128)).astype(np.float64)
        same_codes(H, w, fmt, g, 3, "bf16")
        same_codes(H, w, fmt, g, 3, "f32")
        return
    t = M.magnitudes(fmt)
    mid = (t[1:] + t[:-1]) / 2
    vals = np.concatenate((t, mid, np.nextafter(np.float32(mid), np.float32(9)),
                           np.nextafter(np.float32(mid), np.float32(0)), [7.0, 7.75, 7.99]))
    rows = []
    for e in list(range(-149, -120)) + list(range(-20, 21)) + list(range(118, 126)):
        v = np.ldexp(np.resize(vals, -(-len(vals) // 31) * 31).reshape(-1, 31), e)
        top = np.full((len(v), 1), np.ldexp(4.0, e))
        rows.append(np.concatenate((top, v * np.resize([1, -1], v.shape)), axis=1))
    w = np.concatenate(rows)
    w = w[np.abs(w).max(axis=1) < 3.3e38]
    same_codes(H, w, fmt, 0, 0, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_special_values(H, fmt, dtype):
    announce(f"special {fmt} {dtype}")
    w = normal(6, 192, 1)
    w[0, :32] = 0.0
    w[0, 32:64] = -0.0
    w[1, 5] = np.nan
    w[1, 40] = np.inf
    w[2, 191] = -np.inf
    w[3, 64:96] = 2.0 ** -133
    w[4, 0] = 3.3e38
    same_codes(H, w, fmt, 0, 0, dtype)
    w[4, 0] = 1.0
    codes, scales = H.mx_quantize(cast(w, dtype)[0], fmt_of(H, fmt), 64, 9)
    want_c, want_s = M.quantize(cast(w, dtype)[1], fmt, 64, 9)   # NaN spreads over its group
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.cpu().numpy(), M.pack(want_c, fmt))
    assert (want_s == 255).sum() == 4       # two groups of two blocks
    # finite inputs whose rotation leaves fp32's range
    big = np.full((1, 64), 3.0e38)
    same_codes(H, big * H.rht_signs(4, 64), fmt, 64, 4, dtype)


@pytest.mark.parametrize("fmt", FMTS)
def test_buffers_behind_the_last_row(H, fmt):
    announce(f"guards {fmt}")
    for rows, inp, g in ((3, 100, 0), (3, 192, 64), (5, 1024, 256), (1, 2048, 2048)):
        w, v = cast(normal(rows, inp, 3), "bf16")
        cb, sb = H.mx_codes_row_bytes(inp, fmt_of(H, fmt)), H.mx_scales_row_bytes(inp)
        codes = torch.full((rows + 2, cb), 0xA5, dtype=torch.uint8, device="cuda")
        scales = torch.full((rows + 2, sb), 0xA5, dtype=torch.uint8, device="cuda")
        H.mx_quantize(w, fmt_of(H, fmt), g, 1, codes=codes, scales=scales)
        assert (codes[rows:] == 0xA5).all() and (scales[rows:] == 0xA5).all()
        out = torch.full((rows + 2, inp), 7.25, device="cuda")
        H.mx_dequantize(codes[:rows], scales[:rows], inp, fmt_of(H, fmt), g, 1, out=out)
        assert (out[rows:] == 7.25).all()
        if fmt == "fp4":
            err = torch.full((rows + 2, 2), 7.25, dtype=torch.float64, device="cuda")
            H.mx_layer_error(w, codes, scales, g, 1, row_err=err)
            assert (err[rows:] == 7.25).all()
        codes4, scales4 = H.mx_quantize(cast(normal(19, inp, 4), "f32")[0], H.MX_FP4, g, 1)
        y = torch.full((rows + 2, 19), 7.25, device="cuda")
        H.mx_qmatmul(w, codes4, scales4, fmt_of(H, fmt), g, 1, 19, y=y)
        assert (y.view(-1)[rows * 19:] == 7.25).all()


def random_layer(rows, inp, fmt, seed, lo=100, hi=140):
    rng = np.random.default_rng(seed)
    packed = rng.integers(0, 256, (rows, M.row_bytes(inp, fmt)), dtype=np.uint8)
    scales = rng.integers(lo, hi, (rows, M.blocks(inp)), dtype=np.uint8)
    return packed, scales


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,inp", [(1, 1), (3, 33), (2, 47), (5, 64), (7, 1000), (65, 96)])
def test_dequantize_plain(H, rows, inp, fmt, dtype):
    """Every value exactly (bf16 holds them too), NaN blocks included."""
    announce(f"dequantize {rows}x{inp} {fmt} {dtype}")
    packed, scales = random_layer(rows, inp, fmt, rows + inp, 0, 256)
    out_type = torch.bfloat16 if dtype == "bf16" else torch.float32
    got = H.mx_dequantize(torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda(), inp,
                          fmt_of(H, fmt), dtype=out_type)
    assert got.dtype == out_type
    want = M.values(M.unpack(packed, fmt), scales, fmt, inp)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(want).float().to(out_type).double().numpy()   # exact, or infinite
    assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
def test_dequantize_rotates_back(H, g, fmt, dtype):
    for rows, inp in ((1, g), (5, 3 * g)):
        announce(f"dequantize {rows}x{inp} g={g} {fmt} {dtype}")
        packed, scales = random_layer(rows, inp, fmt, g + rows)
        out_type = torch.bfloat16 if dtype == "bf16" else torch.float32
        got = H.mx_dequantize(torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda(),
                              inp, fmt_of(H, fmt), g, 21, dtype=out_type).double().cpu().numpy()
        v = M.values(M.unpack(packed, fmt), scales, fmt, inp)
        want = M.rotate_back(v, g, 21)
        # fp32 butterflies: each of log2(g) levels, the factor and the rounding to
        # fp32 are off by 2^-24 of values up to sum |v| / sqrt(g) of their group
        top = np.repeat(np.abs(v).reshape(rows, -1, g).sum(axis=2), g, axis=1) / np.sqrt(g)
        tol = (np.log2(g) + 3) * 2.0 ** -24 * top
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * np.abs(want)
        assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,inp,g", [(1, 1, 0), (3, 47, 0), (20, 5000, 0), (2, 64, 64),
                                        (3, 1088, 64), (7, 1280, 128), (5, 2560, 512),
                                        (4, 4096, 1024), (2, 14336, 1024), (3, 4096, 2048),
                                        (3, 20480, 4096), (1100, 64, 64)])
def test_layer_error(H, rows, inp, g, dtype):
    announce(f"error {rows}x{inp} g={g} {dtype}")
    w, v = cast(0.02 * normal(rows, inp, g + rows, 0.3), dtype)
    codes, scales = H.mx_quantize(w, H.MX_FP4, g, 8)
    t2, rows_got = H.mx_layer_error(w, codes, scales, g, 8)
    q = M.values(M.unpack(codes.cpu().numpy(), "fp4"), scales.cpu().numpy(), "fp4", inp)
    want = M.row_error(v, q, g, 8)
    got = rows_got.cpu().numpy()
    u = 2.0 ** -53
    err, norm = want[:, 0], want[:, 1]
    # sums of `in` terms; the rotated values are off by (log2 g + 3) u of their
    # group's sum |w| / sqrt(g) <= its norm, which meets |d| once per value (both
    # sides have such errors)
    rot = 2 * (np.log2(g) + 3) * np.sqrt(g) * np.sqrt(norm * err) if g else 0.0
    assert (np.abs(got[:, 0] - err) <= 2 * u * ((inp + 8) * err + rot)).all()
    assert (np.abs(got[:, 1] - norm) <= 2 * u * (inp + 8) * norm).all()
    assert abs(t2 - got[:, 0].sum() / got[:, 1].sum()) <= 4 * u * (rows + 8) * t2
    assert 0.002 < t2 < 0.03 or inp < 64


def test_layer_error_of_nothing(H):
    announce("error of zeros")
    for g in (0, 64):
        w = torch.zeros((3, 128), device="cuda")
        codes, scales = H.mx_quantize(w, H.MX_FP4, g, 1)
        t2, rows = H.mx_layer_error(w, codes, scales, g, 1)
        assert t2 == 0.0 and not rows.any()


def product_reference(x, packed, scales, fmt, g, seed):
    """(y, sum of the magnitudes) in fp64, in the stored space."""
    inp = x.shape[1]
    xq = M.quantized(x, fmt, g, seed)
    wq = M.values(M.unpack(packed, "fp4"), scales, "fp4", inp)
    return xq @ wq.T, np.abs(xq) @ np.abs(wq).T


def check_product(H, batch, out, inp, fmt, g, x_type, y_type, seed=5, x=None):
    announce(f"product {batch}x{inp}->{out} {fmt} g={g} {x_type} {y_type}")
    x = normal(batch, inp, batch + out + inp) if x is None else x
    xt, xv = cast(x, x_type)
    packed, scales = random_layer(out, inp, "fp4", out + inp, 112, 124)
    dtype = torch.bfloat16 if y_type == "bf16" else torch.float32
    y = H.mx_qmatmul(xt, torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda(),
                     fmt_of(H, fmt), g, seed, out, dtype=dtype)
    assert y.shape == (batch, out) and y.dtype == dtype
    want, size = product_reference(xv, packed, scales, fmt, g, seed)
    # exact products; one fp32 rounding of a partial sum per 64 of K, one per
    # part of a split sum (at most 16)
    tol = (-(-inp // 64) + 16) * 2.0 ** -24 * size
    if y_type == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(want)
    got = y.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= tol).all()
    return y


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("inp", [1, 31, 32, 33, 96, 127, 128, 129, 160, 511, 512, 513, 640, 1000,
                                 2085, 5003])
@pytest.mark.parametrize("batch", [1, 3, 16, 80])
def test_product_row_lengths(H, inp, batch, fmt):
    check_product(H, batch, 37, inp, fmt, 0, "f32", "f32")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("batch", [1, 2, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100,
                                   127, 128, 129, 255, 256, 257, 300])
def test_product_batches(H, batch, fmt):
    check_product(H, batch, 272, 1184, fmt, 0, "bf16", "f32")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("out", [1, 2, 3, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 257,
                                 1001])
@pytest.mark.parametrize("batch", [1, 20, 260])
def test_product_outputs(H, out, batch, fmt):
    check_product(H, batch, out, 768, fmt, 0, "bf16", "bf16")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("g", GROUPS)
@pytest.mark.parametrize("batch", [1, 6, 16, 70])
def test_product_rotated(H, g, batch, fmt):
    for y_type, x_type in (("f32", "bf16"), ("bf16", "f32")):
        check_product(H, batch, 96, 3 * g if g < 4096 else 2 * g, fmt, g, x_type, y_type)


@pytest.mark.parametrize("batch,out,inp,fmt,g", [
    (1, 4096, 4096, "fp6", 1024), (2, 1024, 14336, "fp4", 512), (16, 512, 14336, "fp6", 1024),
    (64, 2048, 4096, "fp6", 0), (512, 1024, 8192, "fp4", 1024), (300, 1103, 5003, "fp6", 0),
    (2048, 512, 1024, "fp4", 64), (1030, 2050, 512, "fp6", 128), (1, 64, 40960, "fp6", 4096),
    (5, 40000, 64, "fp4", 64), (33, 48, 32768, "fp6", 0)])
def test_product_sizes(H, batch, out, inp, fmt, g):
    check_product(H, batch, out, inp, fmt, g, "bf16", "f32")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("batch", [1, 4, 16, 90, 300])
def test_product_nan_stays_in_its_row(H, batch, fmt):
    """A NaN activation makes its row NaN, a NaN block of weights its column,
    and no other output."""
    announce(f"NaN rows batch={batch} {fmt}")
    out, inp = 70, 1100
    x = normal(batch, inp, 1)
    packed, scales = random_layer(out, inp, "fp4", 2, 112, 124)
    packed[11, :16] = 0
    scales[11, 0] = 255
    scales[69, 34] = 255
    x[batch // 2, 1099] = np.nan
    xt, xv = cast(x, "f32")
    y = H.mx_qmatmul(xt, torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda(),
                     fmt_of(H, fmt), 0, 0, out).cpu().numpy()
    nan = np.zeros((batch, out), dtype=bool)
    nan[batch // 2] = True
    nan[:, [11, 69]] = True
    assert np.array_equal(np.isnan(y), nan)
    want, size = product_reference(np.nan_to_num(xv), packed, np.where(scales == 255, 0, scales),
                                   fmt, 0, 0)
    assert (np.abs(y - want)[~nan] <= ((1100 / 128 + 65) * 2.0 ** -24 * size)[~nan]).all()


@pytest.mark.parametrize("batch", [1, 16, 40, 200])
def test_product_of_zero_rows(H, batch):
    announce(f"zero rows batch={batch}")
    x = normal(batch, 640, 4)
    x[batch - 1] = 0.0
    y = check_product(H, batch, 50, 640, "fp6", 128, "f32", "f32", x=x)
    assert not y[batch - 1].any()


@pytest.mark.parametrize("batch,g", [(1, 1024), (4, 0), (16, 256), (48, 1024), (300, 64)])
def test_product_same_bits_each_time(H, batch, g):
    """Repeated, in a workspace of another content, on another stream, from an
    output buffer, and beside a second call on its own stream and workspace."""
    announce(f"repeat batch={batch} g={g}")
    inp, out = 4096, 1030
    x = cast(normal(batch, inp, 9), "bf16")[0]
    layer = H.MXLinear.from_weight(cast(0.02 * normal(out, inp, 10, 0.3), "bf16")[0], g, 3)
    first = layer.forward(x)
    need = H.mx_qmatmul_workspace_bytes(batch, out, inp, H.MX_FP6, g)
    ws = torch.full((max(need, 1),), 0xFF, dtype=torch.uint8, device="cuda")
    y = torch.full((batch, out), float("nan"), device="cuda")
    assert layer.forward(x, y=y, workspace=ws) is y
    assert torch.equal(y, first)
    other = layer.forward(x, dtype=torch.bfloat16)
    assert torch.equal(other, first.bfloat16())
    x2 = cast(normal(batch, inp, 19), "bf16")[0]
    second = layer.forward(x2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for k, (s, a) in enumerate(zip(streams, (x, x2))):
            with torch.cuda.stream(s):
                got[k].append(layer.forward(a))
    torch.cuda.synchronize()
    for k, want in enumerate((first, second)):
        assert all(torch.equal(t, want) for t in got[k])


@pytest.mark.parametrize("batch,g", [(1, 1024), (16, 0), (40, 512), (300, 1024)])
def test_calls_in_a_graph(H, batch, g):
    """Quantization, the way back, the error and the product captured once and
    replayed on new inputs, with eager calls between the replays."""
    announce(f"graph batch={batch} g={g}")
    inp, out = 2048, 192
    w = cast(0.02 * normal(out, inp, 1, 0.3), "bf16")[0]
    x = cast(normal(batch, inp, 2), "bf16")[0]
    xs = [cast(normal(batch, inp, 20 + k), "bf16")[0] for k in range(3)]
    codes, scales = H.mx_quantize(w, H.MX_FP4, g, 6)
    y = torch.empty((batch, out), device="cuda")
    ws = torch.empty(max(1, H.mx_qmatmul_workspace_bytes(batch, out, inp, H.MX_FP6, g)),
                     dtype=torch.uint8, device="cuda")
    xc = torch.empty((batch, H.mx_codes_row_bytes(inp, H.MX_FP6)), dtype=torch.uint8, device="cuda")
    sc = torch.empty((batch, H.mx_scales_row_bytes(inp)), dtype=torch.uint8, device="cuda")
    xv = torch.empty((batch, inp), device="cuda")

    def step():
        H.mx_qmatmul(x, codes, scales, H.MX_FP6, g, 6, out, y=y, workspace=ws)
        H.mx_quantize(x, H.MX_FP6, g, 6, codes=xc, scales=sc)
        H.mx_dequantize(xc, sc, inp, H.MX_FP6, out=xv)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for new in xs:
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got_y, got_v = y.clone(), xv.clone()
        y.fill_(float("nan"))
        xv.fill_(float("nan"))
        step()
        assert torch.equal(got_y, y) and torch.equal(got_v, xv)


def test_a_layer_from_weights_to_outputs(H):
    """The operators as a program uses them together, beside a HIGGS layer: error
    tables, the allocation, the chosen layers' outputs."""
    announce("layers together")
    from conftest import load_grid_fixture
    from oracle import higgs_oracle as O
    g, inp, outs = 256, 1024, (96, 160, 64)
    grid = torch.from_numpy(load_grid_fixture(2, 64)[0].astype(np.float32)).cuda()
    ws = [cast(0.02 * normal(o, inp, o, 0.3), "bf16") for o in outs]
    bits = [6 / 2 + 16 / g, 4 + 8 / 32]
    layers, t2 = [], []
    for w, _ in ws:
        hl = H.QuantizedLinear.from_weight(w, grid, g, 3)
        ml = H.MXLinear.from_weight(w, g, 3)
        t2.append([H.layer_error(w, hl.codes, hl.scales, grid, g, 3)[0], ml.error(w)])
        layers.append((hl, ml))
    t2 = np.array(t2)
    assert (t2[:, 1] < t2[:, 0]).all()      # 4.25 bits against 3.06
    choice, _, avg = H.allocate_bits([1.0, 2.0, 0.5], t2, bits, [o * inp for o in outs], 4.0)
    assert 0 < (choice == 1).sum() < 3 and avg <= 4.0
    x, xv = cast(normal(7, inp, 2, 0.0), "bf16")
    for (w, wv), pair, c in zip(ws, layers, choice):
        y = pair[c].forward(x).double().cpu().numpy()
        dense = xv @ wv.T
        rel = np.linalg.norm(y - dense) / np.linalg.norm(dense)
        assert rel < 0.25
        if c == 1:
            ml = pair[1]
            want, size = product_reference(xv, ml.codes.cpu().numpy(), ml.scales.cpu().numpy(),
                                           "fp6", g, 3)
            assert (np.abs(y - want) <= 72 * 2.0 ** -24 * size).all()
            back = ml.weight().double().cpu().numpy()
            assert abs(O.layer_error(wv, back) - ml.error(w)) < 1e-5


def test_binding_refuses(H):
    announce("refusals")
    w = torch.zeros((4, 128), device="cuda")
    codes, scales = H.mx_quantize(w)
    u8 = dict(dtype=torch.uint8, device="cuda")
    bad_values = [
        lambda: H.mx_quantize(w.half()), lambda: H.mx_quantize(w.t()), lambda: H.mx_quantize(w[0]),
        lambda: H.mx_quantize(w, codes=torch.empty(255, **u8)),
        lambda: H.mx_quantize(w, scales=torch.empty(15, **u8)),
        lambda: H.mx_dequantize(codes, scales, 129), lambda: H.mx_dequantize(codes[:, ::2], scales, 64),
        lambda: H.mx_dequantize(codes, scales, 128, dtype=torch.float16),
        lambda: H.mx_dequantize(codes, scales, 128, out=torch.empty((3, 128), device="cuda")),
        lambda: H.mx_layer_error(w, codes[:3], scales),
        lambda: H.mx_layer_error(w, codes, scales, row_err=torch.empty((3, 2), dtype=torch.float64,
                                                                       device="cuda")),
        lambda: H.mx_qmatmul(w, codes, scales, H.MX_FP6, 0, 0, 5),
        lambda: H.mx_qmatmul(w, codes, scales, H.MX_FP6, 0, 0, 4, dtype=torch.float16),
        lambda: H.mx_qmatmul(w, codes, scales, H.MX_FP6, 0, 0, 4, y=torch.empty((3, 4), device="cuda")),
        lambda: H.mx_qmatmul(w, codes, scales.cpu(), H.MX_FP6, 0, 0, 4),
    ]
    for k, call in enumerate(bad_values):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    bad_calls = [
        lambda: H.mx_quantize(w, 2), lambda: H.mx_quantize(w, g=256), lambda: H.mx_quantize(w, g=32),
        lambda: H.mx_quantize(w.new_zeros((0, 128))),
        lambda: H.mx_qmatmul(w, codes, scales, 3, 0, 0, 4),
        lambda: H.mx_qmatmul(w.new_zeros((0, 128)), codes, scales, H.MX_FP6, 0, 0, 4),
        lambda: H.mx_quantize(torch.zeros(4 * 128 + 1, device="cuda")[1:].view(4, 128)),
    ]
    for k, call in enumerate(bad_calls):
        with pytest.raises(H.HiggsError):
            call()
            pytest.fail(f"call {k} was taken")


def test_outputs_of_tensor_subclasses_are_plain(H):
    class Tagged(torch.Tensor):
        pass
    announce("subclass")
    w = torch.randn((8, 128), device="cuda")
    codes, scales = H.mx_quantize(w.as_subclass(Tagged))
    outs = [codes, scales, H.mx_dequantize(codes.as_subclass(Tagged), scales, 128),
            H.mx_layer_error(w.as_subclass(Tagged), codes, scales)[1],
            H.mx_qmatmul(w.as_subclass(Tagged), codes, scales, H.MX_FP6, 0, 0, 8)]
    assert all(type(t) is torch.Tensor for t in outs)


@pytest.mark.parametrize("batch,out,inp", [
    # columns in two parts: whole rounds of large tiles, the rest in smaller ones
    (2048, 9001, 1024), (3000, 6001, 512), (779, 20297, 593), (1499, 22329, 70),
    (872, 37387, 825), (1504, 23835, 64),
    # blocks that take several tiles
    (1131, 21806, 77), (313, 39341, 70), (560, 22555, 816), (33, 140001, 64), (17, 70003, 100),
    # parts of K
    (2814, 44, 4041), (149, 4363, 9963), (2352, 35, 5450), (141, 17813, 5935), (18, 513, 20000),
    # 17 .. 32 rows streamed and tiled
    (24, 20001, 2048), (20, 4097, 4096), (32, 512, 8192), (17, 37, 64)])
@pytest.mark.parametrize("fmt,y_type", [("fp6", "bf16"), ("fp4", "f32")])
def test_product_plans(H, batch, out, inp, fmt, y_type):
    check_product(H, batch, out, inp, fmt, 0, "bf16", y_type)


@pytest.mark.parametrize("batch", [3, 16, 30, 200])
def test_product_of_unaligned_scales(H, batch):
    """Scale bytes at any address, and g = 0 codes of rows that are no multiple of 64."""
    announce(f"unaligned scales batch={batch}")
    out, inp = 77, 1056
    packed, scales = random_layer(out, inp, "fp4", 4, 112, 124)
    x = cast(normal(batch, inp, 3), "bf16")[0]
    c = torch.from_numpy(packed).cuda()
    want = H.mx_qmatmul(x, c, torch.from_numpy(scales).cuda(), H.MX_FP6, 0, 0, out)
    w = H.mx_dequantize(c, torch.from_numpy(scales).cuda(), inp)
    for shift in (1, 2, 3, 7):
        room = torch.zeros(scales.size + 8, dtype=torch.uint8, device="cuda")
        view = room[shift:shift + scales.size].view(scales.shape)
        view.copy_(torch.from_numpy(scales))
        assert torch.equal(H.mx_qmatmul(x, c, view, H.MX_FP6, 0, 0, out), want)
        assert torch.equal(H.mx_dequantize(c, view, inp), w)
        assert H.mx_layer_error(w, c, view)[0] == 0.0
        c2, s2 = H.mx_quantize(w, scales=room[shift:shift + scales.size].view(scales.shape))
        assert torch.equal(H.mx_dequantize(c2, s2, inp), w)


@pytest.mark.parametrize("batch,out,inp,g", [
    (1, 33, 128, 64), (16, 100, 1024, 1024), (20, 50, 544, 0), (31, 130, 4096, 4096),
    (65, 127, 2048, 256), (40, 60, 16384, 0), (2048, 9001, 256, 0)])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_product_stays_in_its_buffers(H, batch, out, inp, g, y_type):
    """Memory behind y and behind the workspace keeps its bytes."""
    announce(f"buffers {batch}x{inp}->{out} g={g} {y_type}")
    packed, scales = random_layer(out, inp, "fp4", 4, 112, 124)
    c, s = torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda()
    x = cast(normal(batch, inp, 3), "bf16")[0]
    dtype = torch.bfloat16 if y_type == "bf16" else torch.float32
    want = H.mx_qmatmul(x, c, s, H.MX_FP6, g, 2, out, dtype=dtype)
    room = torch.full((batch * out + 4096,), 7.0, dtype=dtype, device="cuda")
    need = H.mx_qmatmul_workspace_bytes(batch, out, inp, H.MX_FP6, g)
    ws = torch.full((need + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    y = room[:batch * out].view(batch, out)
    H.mx_qmatmul(x, c, s, H.MX_FP6, g, 2, out, y=y, workspace=ws[:need])
    assert torch.equal(y, want)
    assert (room[batch * out:] == 7.0).all() and (ws[need:] == 0xA5).all()


def test_calls_on_a_given_stream(H):
    """stream=: the call runs there, with a workspace of its own that is not handed
    out again before it has ended."""
    announce("given stream")
    out, inp, g, batch = 1536, 4096, 1024, 96
    w = cast(0.02 * normal(out, inp, 1, 0.3), "bf16")[0]
    x = cast(normal(batch, inp, 2), "bf16")[0]
    codes, scales = H.mx_quantize(w, H.MX_FP4, g, 6)
    want = H.mx_qmatmul(x, codes, scales, H.MX_FP6, g, 6, out)
    back = H.mx_dequantize(codes, scales, inp)
    outs = [torch.empty_like(want) for _ in range(6)]
    c2, s2, b2 = torch.empty_like(codes), torch.empty_like(scales), torch.empty_like(back)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    need = H.mx_qmatmul_workspace_bytes(batch, out, inp, H.MX_FP6, g)
    for y in outs:
        H.mx_qmatmul(x, codes, scales, H.MX_FP6, g, 6, out, y=y, stream=s)
        # (takes the workspace's memory, if that has been handed back)
        torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    H.mx_quantize(w, H.MX_FP4, g, 6, codes=c2, scales=s2, stream=s)
    H.mx_dequantize(c2, s2, inp, out=b2, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in outs)
    assert torch.equal(c2, codes) and torch.equal(s2, scales) and torch.equal(b2, back)


@pytest.mark.parametrize("g", [0, 1024, 4096])
def test_rows_beyond_32_bit_offsets(H, g):
    """More than 2^32 bytes of weights, 2^31 values: the last rows as on their own."""
    announce(f"long tensors g={g}")
    inp, rows = 4096, (1 << 19) + 5
    w = torch.zeros((rows, inp), dtype=torch.bfloat16, device="cuda")
    tail = cast(normal(9, inp, 2), "bf16")[0]
    w[-9:] = tail
    w[:9] = tail.flip(0)
    for fmt in (H.MX_FP4, H.MX_FP6):
        codes, scales = H.mx_quantize(w, fmt, g, 3)
        c, s = H.mx_quantize(tail, fmt, g, 3)
        assert torch.equal(codes[-9:], c) and torch.equal(scales[-9:], s)
        assert torch.equal(codes[:9], c.flip(0)) and torch.equal(scales[:9], s.flip(0))
        assert not codes[9:-9].any() and not scales[9:-9].any()
        back = H.mx_dequantize(codes, scales, inp, fmt, g, 3, dtype=torch.bfloat16)
        want = H.mx_dequantize(c, s, inp, fmt, g, 3, dtype=torch.bfloat16)
        assert torch.equal(back[-9:], want) and torch.equal(back[:9], want.flip(0))
        if fmt == H.MX_FP4:
            rows_err = H.mx_layer_error(w, codes, scales, g, 3)[1]
            assert torch.equal(rows_err[-9:], H.mx_layer_error(tail, c, s, g, 3)[1])
        del codes, scales, back


@pytest.mark.parametrize("batch", [2, 16, 24, 48])
def test_product_of_the_largest_layer(H, batch):
    """Codes of almost 2 GiB: the first and the last outputs."""
    announce(f"largest layer batch={batch}")
    out, inp, n = (1 << 20) - 70, 4064, 200
    packed, scales = random_layer(2 * n, inp, "fp4", 4, 112, 124)
    codes = torch.zeros((out, packed.shape[1]), dtype=torch.uint8, device="cuda")
    sc = torch.zeros((out, scales.shape[1]), dtype=torch.uint8, device="cuda")
    for whole, part in ((codes, packed), (sc, scales)):
        whole[:n] = torch.from_numpy(part[:n]).cuda()
        whole[-n:] = torch.from_numpy(part[n:]).cuda()
    x, xv = cast(normal(batch, inp, 2), "bf16")
    y = H.mx_qmatmul(x, codes, sc, H.MX_FP6, 0, 0, out)
    want, size = product_reference(xv, packed, scales, "fp6", 0, 0)
    got = torch.cat([y[:, :n], y[:, -n:]], 1).double().cpu().numpy()
    assert (np.abs(got - want) <= (-(-inp // 64) + 16) * 2.0 ** -24 * size).all()
    assert not y[:, n:-n].any()


def test_product_of_very_many_rows(H):
    """More than 2^32 bytes of outputs: the first and the last rows."""
    announce("many rows")
    batch, out, inp, n = (1 << 21) + 77, 1040, 64, 300
    packed, scales = random_layer(out, inp, "fp4", 4, 112, 124)
    x, xv = cast(normal(2 * n, inp, 2), "bf16")
    many = torch.zeros((batch, inp), dtype=torch.bfloat16, device="cuda")
    many[:n], many[-n:] = x[:n], x[n:]
    y = H.mx_qmatmul(many, torch.from_numpy(packed).cuda(), torch.from_numpy(scales).cuda(),
                     H.MX_FP6, 64, 3, out, dtype=torch.bfloat16)
    want, size = product_reference(xv, packed, scales, "fp6", 64, 3)
    got = torch.cat([y[:n], y[-n:]]).double().cpu().numpy()
    assert (np.abs(got - want) <= 17 * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(want)).all()
    assert not y[n:-n].any()


def test_linear_captured_beside_an_eager_one(H):
    """MXLinear.forward captured with a workspace from the graph's pool, replayed with
    eager calls of the same layer between, two graphs in turn."""
    announce("linear in graphs")
    inp, out = 2048, 640
    layer = H.MXLinear.from_weight(cast(0.02 * normal(out, inp, 1, 0.3), "bf16")[0], 1024, 6)
    xs = [cast(normal(b, inp, b), "bf16")[0] for b in (8, 120)]
    want = [layer.forward(x) for x in xs]
    torch.cuda.synchronize()
    graphs = []
    for x in xs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layer.forward(x)
        graphs.append((graph, y))
    for _ in range(3):
        for (graph, y), w, x in zip(graphs, want, xs):
            y.fill_(float("nan"))
            graph.replay()
            eager = layer.forward(x)
            torch.cuda.synchronize()
            assert torch.equal(y, w) and torch.equal(eager, w)


def test_refuses_another_device(H, monkeypatch):
    """Tensors of one device on the current stream or a stream of another."""
    announce("other device")
    w = torch.zeros((4, 128), device="cuda")
    codes, scales = H.mx_quantize(w)

    class Elsewhere:
        device = torch.device("cuda", 1)
        cuda_stream = 0
    calls = [lambda s=None: H.mx_quantize(w, stream=s),
             lambda s=None: H.mx_dequantize(codes, scales, 128, stream=s),
             lambda s=None: H.mx_layer_error(w, codes, scales, stream=s),
             lambda s=None: H.mx_qmatmul(w, codes, scales, H.MX_FP6, 0, 0, 4, stream=s)]
    for call in calls:
        with pytest.raises(ValueError, match="stream"):
            call(Elsewhere())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="stream"):
            call()


def test_refuses_rows_of_another_length(H):
    announce("row length")
    x = torch.zeros((4, 64), device="cuda")
    codes, scales = H.mx_quantize(torch.zeros((4, 128), device="cuda"))
    for call in (lambda: H.mx_dequantize(codes, scales, 64),
                 lambda: H.mx_layer_error(x, codes, scales),
                 lambda: H.mx_qmatmul(x, codes, scales, H.MX_FP6, 0, 0, 4),
                 lambda: H.mx_quantize(x, codes=codes), lambda: H.mx_quantize(x, scales=scales)):
        with pytest.raises(ValueError, match="another length"):
            call()
    # buffers without rows, and with more of them, are taken
    flat = H.mx_dequantize(codes, scales.view(-1), 128)
    assert flat.shape == (4, 128) and not flat.any()
    y = H.mx_qmatmul(x[:1].repeat(1, 2), codes.view(-1), scales.view(-1), H.MX_FP6, 0, 0, 3)
    assert y.shape == (1, 3) and not y.any()


@pytest.mark.parametrize("batch,g", [(1, 4096), (16, 0), (32, 1024), (40, 0)])
def test_product_of_the_longest_rows(H, batch, g):
    check_product(H, batch, 24, 1 << 20, "fp6", g, "bf16", "f32")


@pytest.mark.parametrize("batch,inp,g", [
    (2, 4096, 1024), (3, 4096, 64), (4, 4096, 256), (1, 14336, 2048), (1, 14336, 512), (1, 15360, 1024),
    (4, 1024, 128), (5, 1024, 1024), (14, 1024, 64), (2, 7168, 1024), (4, 4096, 0), (5, 4096, 0),
    (16, 1024, 0), (16, 1088, 64)])
@pytest.mark.parametrize("fmt", FMTS)
def test_product_of_few_rows(H, batch, inp, g, fmt):
    """Calls on both sides of where the product converts its activations itself."""
    for out, x_type in ((50, "bf16"), (4100, "f32")):
        check_product(H, batch, out, inp, fmt, g, x_type, "f32")
