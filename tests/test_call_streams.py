"""stream= of the HIGGS calls, without a GPU: what a call allocates is the given stream's
memory, its kernels go there, and a result read on the host has been waited for. The
library's launches are recorded, not made."""
import pytest

from test_mx_streams import HERE, THERE, H, streams, torch  # noqa: F401

P, N, G, OUT, IN, BATCH = 2, 64, 256, 96, 512, 24


@pytest.fixture
def on(streams, monkeypatch):  # noqa: F811
    log, there = streams
    monkeypatch.setattr(torch.cuda, "Stream", type(there))
    return log, there


def arguments():
    return dict(w=torch.zeros((OUT, IN)), grid=torch.zeros((N, P)), x=torch.zeros((BATCH, IN)),
                codes=torch.zeros((OUT, H.codes_row_bytes(IN, P, N)), dtype=torch.uint8),
                scales=torch.zeros((OUT, IN // G), dtype=torch.float16),
                factor=torch.zeros((IN, IN), dtype=torch.float64))


CALLS = {
    "search_index": lambda a, **kw: H.search_index(a["grid"], **kw),
    "quantize": lambda a, **kw: H.quantize(a["w"], a["grid"], G, 1, **kw),
    "layer_error": lambda a, **kw: H.layer_error(a["w"], a["codes"], a["scales"], a["grid"], G, 1,
                                                 **kw),
    "gptq_factor": lambda a, **kw: H.gptq_factor(a["x"], **kw),
    "quantize_gptq": lambda a, **kw: H.quantize_gptq(a["w"], a["grid"], G, 1, a["factor"], **kw),
    "rht_activations": lambda a, **kw: H.rht_activations(a["x"], G, 1, **kw),
    "qmatmul": lambda a, **kw: H.qmatmul(a["x"], a["codes"], a["scales"], a["grid"], G, OUT, **kw),
    "qmatmul_fused": lambda a, **kw: H.qmatmul_fused(a["x"], a["codes"], a["scales"], a["grid"], G,
                                                     1, OUT, **kw),
    "qmatmul_fused_noalloc": lambda a, **kw: H.qmatmul_fused_noalloc(
        a["x"], a["codes"], a["scales"], a["grid"], G, 1, OUT, **kw),
    "qmatmul_fused_multi": lambda a, **kw: H.qmatmul_fused_multi(
        a["x"], [(a["codes"], a["scales"], s, OUT) for s in (1, 2)], a["grid"], G, **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_call_allocates_on_its_stream(on, name):
    log, there = on
    results = CALLS[name](arguments(), stream=there)
    made = [e for e in log if e[0] == "allocation"]
    assert made and all(where == THERE for *_, where in made), log
    launches = [e for e in log if e[0] == "launch"]
    # (the stream given to the library, and the one that a copy to the host would wait for)
    assert launches and all(e[2:] == (THERE, THERE) for e in launches), log
    for t in results if isinstance(results, (tuple, list)) else (results,):
        if isinstance(t, torch.Tensor):
            assert ("record", t.data_ptr(), HERE) in log, log


@pytest.mark.parametrize("name", CALLS)
def test_a_call_without_a_stream_stays_here(on, name):
    log, _ = on
    CALLS[name](arguments())
    assert log and all(e[2] == HERE for e in log), log
    assert not [e for e in log if e[0] == "record"]


@pytest.mark.parametrize("name", CALLS)
def test_another_kind_of_stream_names_one_for_the_kernels(streams, name):  # noqa: F811
    """Any object with a cuda_stream is taken, as ever."""
    log, there = streams
    CALLS[name](arguments(), stream=there)
    launches = [e for e in log if e[0] == "launch"]
    assert launches and all(e[2] == THERE for e in launches), log
