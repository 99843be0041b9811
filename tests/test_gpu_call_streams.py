"""stream= of the HIGGS calls on the GPU, beside calls on the current stream, without
buffers from the caller."""
import sys

import pytest

from test_gpu_parity import grid_f32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_calls_on_a_given_stream():
    from paper_2411_17525_amd import higgs as H
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print("[gpu-case] higgs calls on a given stream", file=sys.stderr, flush=True)
    p, n, g, out, inp, batch = 2, 256, 256, 1024, 4096, 96
    grid = torch.from_numpy(grid_f32(p, n)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn((out, inp), generator=gen, device="cuda").bfloat16()
    xs = [torch.randn((batch, inp), generator=gen, device="cuda") for _ in range(2)]
    index = H.search_index(grid)
    codes, scales = H.quantize(w, grid, g, 3, index=index)
    layer = (codes, scales, grid, g)
    t2, errors = H.layer_error(w, *layer, 3)

    def forms(x, stream=None):
        rot = H.rht_activations(x, g, 3, stream=stream)
        return [rot, H.qmatmul(rot, *layer, out, stream=stream),
                H.qmatmul_fused(x, *layer, 3, out, stream=stream),
                *H.qmatmul_fused_multi(x, [(codes, scales, 3, out)] * 2, grid, g, stream=stream)]
    want = [forms(x) for x in xs]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        got.append((forms(xs[0]), forms(xs[1], s)))
        c, sc = H.quantize(w, grid, g, 3, stream=s)
        i = H.search_index(grid, stream=s)
        t, e = H.layer_error(w, *layer, 3, stream=s)     # (waits for s)
        assert t == t2 and torch.equal(e, errors)
        # (an index's bytes behind its lists are not written: it is compared by its codes)
        assert torch.equal(c, codes) and torch.equal(sc, scales)
        assert torch.equal(H.quantize(w, grid, g, 3, index=i)[0], codes)
    torch.cuda.synchronize()
    for pair in got:
        for a, b in zip(pair, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))
