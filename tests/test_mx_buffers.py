"""Buffers that the microscaled product refuses, without a GPU (launches are recorded)."""
import pytest

from test_mx_streams import H, layer, streams, torch  # noqa: F401


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("make", [
    lambda n: torch.zeros(1, dtype=torch.uint8).expand(n),               # one byte, n times
    lambda n: torch.zeros((1, n // 8), dtype=torch.uint8).expand(16, n // 8),
    lambda n: torch.zeros(2 * n, dtype=torch.uint8)[::2]])
def test_workspace_that_is_no_run_of_memory(streams, make, given):  # noqa: F811
    log, there = streams
    w, c, s = layer()
    need = H.mx_qmatmul_workspace_bytes(40, 40, 512, H.MX_FP6, 0)
    ws = make(need)
    assert ws.numel() >= need > 0
    with pytest.raises(ValueError, match="workspace"):
        H.mx_qmatmul(w, c, s, H.MX_FP6, 0, 0, 40, y=torch.zeros((40, 40)), workspace=ws,
                     stream=there if given else None)
    assert not [e for e in log if e[0] == "launch"]
