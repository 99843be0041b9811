"""stream= of the microscaled calls, without a GPU: what a call allocates is the given
stream's memory, its kernels go there, and new results are kept until the work of the
stream that was current has ended too. The library's launches are recorded, not made."""
import contextlib
import types

import pytest

H = pytest.importorskip("paper_2411_17525_amd.higgs")
torch = pytest.importorskip("torch")

HERE, THERE = 11, 22    # raw streams


class Library:
    """Sizes from the library, launches into `log`."""

    def __init__(self, real, log, now):
        self.real, self.log, self.now = real, log, now

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)

        def launch(*args):
            self.log.append(("launch", name, args[-1], self.now[0]))
            return 0
        return launch


@pytest.fixture
def streams(monkeypatch):
    """(log of allocations, launches and records, the given stream)."""
    log, now = [], [HERE]
    real = H.lib()
    H._need_torch()
    monkeypatch.setattr(H, "lib", lambda: Library(real, log, now))
    monkeypatch.setattr(H, "_need_cuda", lambda *a: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: now[0])

    @contextlib.contextmanager
    def on(stream):
        before, now[0] = now[0], stream.cuda_stream
        yield
        now[0] = before
    monkeypatch.setattr(torch.cuda, "stream", on)
    empty, new_empty = torch.empty, torch.Tensor.new_empty

    def logged(make):
        def call(*args, **kw):
            t = make(*args, **kw)
            log.append(("allocation", t.data_ptr(), now[0]))
            return t
        return call
    monkeypatch.setattr(torch, "empty", logged(empty))
    monkeypatch.setattr(torch.Tensor, "new_empty", logged(new_empty))
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: log.append(("record", t.data_ptr(), s)))
    there = types.SimpleNamespace(cuda_stream=THERE, device=types.SimpleNamespace(index=-1))
    there.synchronize = lambda: None
    return log, there


def layer(rows=40, inp=512):
    return (torch.zeros((rows, inp)), torch.zeros((rows, inp // 2), dtype=torch.uint8),
            torch.zeros((rows, inp // 32), dtype=torch.uint8))


CALLS = {
    "quantize": lambda w, c, s, **kw: H.mx_quantize(w, **kw),
    "dequantize": lambda w, c, s, **kw: H.mx_dequantize(c, s, w.shape[1], **kw),
    "error": lambda w, c, s, **kw: H.mx_layer_error(w, c, s, **kw),
    "product": lambda w, c, s, **kw: H.mx_qmatmul(w, c, s, H.MX_FP6, 0, 0, len(w), **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_call_allocates_on_its_stream(streams, name):
    log, there = streams
    results = CALLS[name](*layer(), stream=there)
    made = [e for e in log if e[0] == "allocation"]
    # (the product of 40 rows has a workspace beside its output)
    assert len(made) == {"quantize": 2, "dequantize": 1, "error": 2, "product": 2}[name]
    assert all(where == THERE for *_, where in made), log
    launches = [e for e in log if e[0] == "launch"]
    assert [e[2] for e in launches] == [THERE], log
    for t in results if isinstance(results, tuple) else (results,):
        if isinstance(t, torch.Tensor):
            assert ("record", t.data_ptr(), HERE) in log, log


@pytest.mark.parametrize("name", CALLS)
def test_a_call_without_a_stream_stays_here(streams, name):
    log, _ = streams
    CALLS[name](*layer())
    assert all(e[2] == HERE for e in log), log
    assert not [e for e in log if e[0] == "record"]


def test_the_callers_outputs_are_the_callers(streams):
    """No record and no allocation for outputs and workspaces that the caller brings."""
    log, there = streams
    w, c, s = layer()
    y = torch.zeros((40, 40))
    ws = torch.zeros(H.mx_qmatmul_workspace_bytes(40, 40, 512, H.MX_FP6, 0), dtype=torch.uint8)
    assert H.mx_qmatmul(w, c, s, H.MX_FP6, 0, 0, 40, y=y, workspace=ws, stream=there) is y
    assert H.mx_quantize(w, codes=c, scales=s, stream=there) == (c, s)
    assert [e[0] for e in log] == ["launch", "launch"]


@pytest.mark.parametrize("name", CALLS)
def test_refuses_a_stream_of_another_device(streams, name):
    log, there = streams
    there.device.index = 1
    with pytest.raises(ValueError, match="stream"):
        CALLS[name](*layer(), stream=there)
    assert not log
