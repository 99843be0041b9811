"""Sizes and refusals of the microscaled entry points: everything invalid is
refused on the host, before anything reaches the GPU. No call here launches a
kernel."""
import pytest

from oracle import mx_oracle as M
from test_abi_cpu import FAKE, INVALID, UNSUPPORTED, L, no_gpu  # noqa: F401

H = pytest.importorskip("paper_2411_17525_amd.higgs")
FP4, FP6 = H.MX_FP4, H.MX_FP6


@pytest.mark.parametrize("inp", [1, 31, 32, 33, 4096, 4999, 14336])
def test_row_bytes_match_oracle(inp):
    assert H.mx_codes_row_bytes(inp, FP4) == M.row_bytes(inp, "fp4")
    assert H.mx_codes_row_bytes(inp, FP6) == M.row_bytes(inp, "fp6")
    assert H.mx_scales_row_bytes(inp) == M.blocks(inp)


def test_row_bytes_invalid(L):  # noqa: F811
    for inp in (0, -1, -(1 << 62), (1 << 62)):
        assert H.mx_codes_row_bytes(inp, FP4) == -1
        assert H.mx_scales_row_bytes(inp) == -1
    for fmt in (-1, 2, 1 << 30):
        assert H.mx_codes_row_bytes(64, fmt) == -1


def test_workspace_invalid(L):  # noqa: F811
    good = dict(batch=3, out=64, inp=128, fmt=FP6, g=64)
    assert H.mx_qmatmul_workspace_bytes(**good) >= 0
    for bad in (dict(batch=0), dict(out=0), dict(inp=0), dict(fmt=2), dict(g=3), dict(g=32),
                dict(g=8192), dict(g=256), dict(batch=1 << 62), dict(out=1 << 62),
                dict(inp=(1 << 20) + 64), dict(out=1 << 30, inp=4096)):
        assert H.mx_qmatmul_workspace_bytes(**{**good, **bad}) == -1, bad


BAD_LAYER = [
    (dict(dt=2), INVALID), (dict(dt=-1), INVALID), (dict(rows=0), INVALID),
    (dict(rows=-5), INVALID), (dict(inp=0), INVALID), (dict(g=100), INVALID),
    (dict(g=-64), INVALID), (dict(g=32), UNSUPPORTED), (dict(g=8192), UNSUPPORTED),
    (dict(g=256), INVALID),                      # in = 128 is no multiple of it
    (dict(rows=1 << 40), UNSUPPORTED), (dict(w=None), INVALID), (dict(codes=None), INVALID),
    (dict(scales=None), INVALID), (dict(w=FAKE + 8), INVALID), (dict(codes=FAKE + 4), INVALID),
]


@no_gpu
@pytest.mark.parametrize("bad,status", BAD_LAYER + [(dict(fmt=2), INVALID), (dict(fmt=-1), INVALID)])
def test_quantize_and_dequantize_reject(L, bad, status):  # noqa: F811
    a = dict(w=FAKE, dt=1, rows=16, inp=128, fmt=FP4, g=64, codes=FAKE, scales=FAKE)
    a.update(bad)
    assert L.higgs_mx_quantize(a["w"], a["dt"], a["rows"], a["inp"], a["fmt"], a["g"], 0,
                               a["codes"], a["scales"], None) == status
    assert L.higgs_last_error()
    assert L.higgs_mx_dequantize(a["codes"], a["scales"], a["rows"], a["inp"], a["fmt"], a["g"], 0,
                                 a["w"], a["dt"], None) == status


@no_gpu
@pytest.mark.parametrize("bad,status", BAD_LAYER + [
    (dict(err=None), INVALID), (dict(err=FAKE + 4), INVALID), (dict(t2=FAKE + 4), INVALID),
    (dict(rows=1 << 31), UNSUPPORTED)])
def test_layer_error_rejects(L, bad, status):  # noqa: F811
    a = dict(w=FAKE, dt=1, rows=16, inp=128, g=64, codes=FAKE, scales=FAKE, err=FAKE, t2=FAKE)
    a.update(bad)
    assert L.higgs_mx_layer_error(a["w"], a["dt"], a["rows"], a["inp"], a["codes"], a["scales"],
                                  a["g"], 0, a["err"], a["t2"], None) == status


@no_gpu
@pytest.mark.parametrize("bad,status", [
    (dict(x=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID),
    (dict(y=None), INVALID), (dict(x=FAKE + 8), INVALID), (dict(codes=FAKE + 8), INVALID),
    (dict(y=FAKE + 4), INVALID), (dict(ws=FAKE + 16), INVALID), (dict(xd=2), INVALID),
    (dict(yd=-1), INVALID), (dict(fmt=2), INVALID), (dict(fmt=-1), INVALID),
    (dict(batch=0), INVALID), (dict(out=0), INVALID), (dict(inp=0), INVALID),
    (dict(g=96), INVALID), (dict(g=32), UNSUPPORTED), (dict(g=8192), UNSUPPORTED),
    (dict(g=1024), INVALID), (dict(inp=(1 << 20) + 512), UNSUPPORTED),
    (dict(out=1 << 26), UNSUPPORTED), (dict(batch=1 << 40), UNSUPPORTED)])
def test_qmatmul_rejects(L, bad, status):  # noqa: F811
    a = dict(x=FAKE, xd=1, batch=40, fmt=FP6, codes=FAKE, scales=FAKE, g=512, out=256, inp=512,
             y=FAKE, yd=0, ws=FAKE, wb=1 << 40)
    a.update(bad)
    assert L.higgs_mx_qmatmul(a["x"], a["xd"], a["batch"], a["fmt"], a["codes"], a["scales"],
                              a["g"], 0, a["out"], a["inp"], a["y"], a["yd"], a["ws"], a["wb"],
                              None) == status
    assert L.higgs_last_error()


@no_gpu
def test_qmatmul_rejects_small_workspaces(L):  # noqa: F811
    args = (256, 4096, 8192)
    need = H.mx_qmatmul_workspace_bytes(*args, FP6, 1024)
    assert need > 0

    def call(ws, wb):
        return L.higgs_mx_qmatmul(FAKE, 1, 256, FP6, FAKE, FAKE, 1024, 0, 4096, 8192, FAKE, 0, ws,
                                  wb, None)
    assert call(FAKE, need - 1) == INVALID
    assert call(None, need) == INVALID
    assert call(FAKE, -1) == INVALID


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    w = torch.zeros((4, 64))
    c = torch.zeros((4, 32), dtype=torch.uint8)
    s = torch.zeros((4, 2), dtype=torch.uint8)
    for call in (lambda: H.mx_quantize(w), lambda: H.mx_dequantize(c, s, 64),
                 lambda: H.mx_layer_error(w, c, s),
                 lambda: H.mx_qmatmul(w, c, s, FP6, 0, 0, 4)):
        with pytest.raises(ValueError):
            call()


def test_limits_of_the_product(L):  # noqa: F811
    """Counts that the kernels hold in 32 bits: the largest calls taken, the next refused."""
    def need(batch, out, inp):
        return H.mx_qmatmul_workspace_bytes(batch, out, inp, FP6, 0)
    top = (1 << 24) - 1
    assert need(top, 1, 32) > 0 and need(top + 1, 1, 32) == -1
    assert need(40, top, 64) > 0 and need(40, top + 1, 64) == -1
    assert need(1 << 14, 16, 1 << 20) > 0 and need((1 << 14) + 1, 16, 1 << 20) == -1
    assert need(1 << 19, 1 << 19, 32) > 0 and need((1 << 19) + 1, 1 << 19, 32) == -1
    assert need(40, (1 << 20) - 1, 4096) > 0 and need(40, 1 << 20, 4096) == -1


@no_gpu
def test_layer_error_refuses_more_rows_than_a_launch_holds(L):  # noqa: F811
    assert L.higgs_mx_layer_error(FAKE, 1, 1 << 24, 64, FAKE, FAKE, 0, 0, FAKE, None,
                                  None) == UNSUPPORTED
