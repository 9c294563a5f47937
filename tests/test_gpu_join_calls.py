"""Calls of the join of a layer and its gradient: what needs no scratch can be recorded at once; workgroups that take several rows in turn."""
import pytest
import torch

from test_gpu_join import _join_case, _join_grad_case
from test_gpu_layer import BF16, E4M3, EPS, F16, F32, _rand

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


# rows beyond which a workgroup takes a second one: 65 536 where 16 lanes share a row, 32 768 (a wave), 16 384 (128 lanes), 8192, 4096, 2048 (1024)
@pytest.mark.parametrize("n,d", [(66_000, 3), (66_000, 12), (66_000, 16), (33_000, 130), (33_000, 136), (16_500, 520), (16_500, 521), (8300, 1032), (4200, 2050),
                                 (4200, 2056), (2100, 4104), (2100, 4105), (2100, 8200), (2100, 8203)])
def test_join_by_workgroups_that_take_several_rows(h, n, d):
    """Every row against the 64-bit form, with a residual and a gate for every row, rows in 16 bits and in 8, and a count that ends in the second turn."""
    print("join", n, d, flush=True)
    _join_case(h, n, d, BF16, BF16, "rows", True, True, 0.3, d, pads=(1, 0), count=n - 37)
    _join_case(h, n, d, F16, E4M3, "rows", False, True, 0.0, d + 1)
    if n * d < 9_000_000:
        _join_case(h, n, d, F32, E4M3, "row", True, True, 0.4, d + 2, count=n - 1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("d", [64, 512, 1024, 4096])
def test_the_last_rows_of_large_calls(h, d, dtype):
    """Of calls of more than 128 MB, which may go past the caches: they are those of a call on a view of these rows, nothing being dropped."""
    few = 100
    n = (150 << 20) // (2 * d * torch.empty(0, dtype=dtype).element_size())
    x, residual, gate, dy, dtotal = (torch.randn((n, d), device="cuda").to(dtype) for _ in range(5))
    gain_x, gain, one_gate = (torch.randn(d, device="cuda").to(dtype) for _ in range(3))

    def run(rows, g):
        at = lambda t: t[rows]  # noqa: E731
        m = at(x).shape[0]
        out = {k: torch.full((m, d), -7.0, dtype=dtype, device="cuda") for k in ("total", "y", "dx", "dresidual")}
        out["y8"], out["y_scale"] = torch.empty((m, d), dtype=E4M3, device="cuda"), torch.empty(m, device="cuda")
        args = dict(gain_x=gain_x, gate=at(g) if g.dim() == 2 else g, residual_scale=0.5, gain=gain)
        h.join_norm(at(x), EPS, y=out["y"], total=out["total"], residual=at(residual), **args)
        h.join_norm(at(x), EPS, y=out["y8"], y_scale=out["y_scale"], residual=at(residual), **args)
        h.join_norm_grad(at(x), out["dx"], EPS, total=out["total"], dy=at(dy), dtotal=at(dtotal), dresidual=out["dresidual"], **args)
        h.sync()
        return out

    for g in (one_gate, gate):
        large, last = run(slice(None), g), run(slice(n - few, n), g)
        for k, v in last.items():
            a, b = (t.view(torch.uint8) if t.dtype == E4M3 else t for t in (large[k][-few:], v))
            assert torch.equal(a, b), k


# ... in the gradient: 16 384 rows where 16 lanes share a row, 4096 (a wave), 2048, 1024, 512, 256 (1024 lanes, and rows that pass through memory)
@pytest.mark.parametrize("n,d", [(17_000, 5), (17_000, 13), (17_000, 24), (4200, 136), (4200, 200), (2100, 520), (2100, 521), (1030, 1032), (520, 2056), (300, 4104),
                                 (300, 4105), (300, 8200)])
def test_join_grad_by_workgroups_that_take_several_rows(h, n, d):
    print("join grad", n, d, flush=True)
    _join_grad_case(h, n, d, BF16, "rows", True, 0.3, d, pads=(1, 0), count=n - 7)
    _join_grad_case(h, n, d, F16, "row", True, 0.1, d + 1)
    _join_grad_case(h, n, d, F32, "rows", False, 0.4, d + 2, has_dy=False)
    _join_grad_case(h, n, d, F32, "none", True, 0.0, d + 3, has_dtotal=False, count=n - 1)
