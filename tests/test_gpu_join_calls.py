"""Calls of the join of a layer and its gradient: what needs no scratch can be recorded at once; workgroups that take several rows in turn."""
import pytest
import torch

from test_gpu_layer import EPS, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def helios():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2310_00837_amd import helios as hl
    return hl


@pytest.fixture(scope="module")
def h(helios):
    ctx = helios.Helios(0)
    yield ctx
    ctx.close()


@pytest.mark.parametrize("d", [32, 9000])
def test_a_gradient_without_sums_needs_no_scratch(helios, d):
    """In a capture of a context that has made no call before: dx, dresidual and a gate of every row are written without sums over rows."""
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        n = 64
        x, dy, gate = (_rand(n, d, s).float().cuda() for s in (1, 2, 3))
        outs = [torch.full((n, d), -7.0, device="cuda") for _ in range(3)]

        def call():
            h.join_norm_grad(x, outs[0], EPS, total=x, dy=dy, gate=gate, dresidual=outs[1], dgate=outs[2])

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        got = []
        for _ in range(3):
            with torch.cuda.stream(stream):
                graph.replay()
            h.sync()
            got.append([o.clone() for o in outs])
            for o in outs:
                o.fill_(-7.0)
            torch.cuda.synchronize()
        call()
        h.sync()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, outs)) and bool((outs[0] != -7.0).all())
    finally:
        h.close()
