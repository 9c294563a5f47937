"""Scratch memory of the operators of a layer: how much they take, and what happens where there is little left."""
import pytest
import torch

from test_gpu_layer import BF16, F32, U32, _close, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def helios():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2310_00837_amd import helios as hl
    return hl


@pytest.fixture()
def h(helios):
    ctx = helios.Helios(0)
    yield ctx
    ctx.close()


def _free():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


@pytest.mark.parametrize("n,k,m", [(1024, 8192, 8192), (4096, 4096, 4096)])
def test_gradient_of_large_weights_takes_no_copies_of_them(helios, h, n, k, m):
    """dw's own tiles fill the GPU: it is written at once, not summed from parts in scratch (of four times its size here, or eight)."""
    x, w, dy = (torch.randn(s, device="cuda").to(BF16) for s in ((n, k), (m, k), (n, m)))
    dw = torch.empty_like(w)
    h.linear_grad(x[:8], w, dy[:8], dw=dw)        # (the kernels are loaded, and memory for them is taken)
    before = _free()
    h.linear_grad(x, w, dy, dw=dw)
    assert before - _free() < 64 << 20
    # a row of the gradient in full, and a column
    for got, want, size in ((dw[7:8], dy[:, 7:8].t(), x), (dw[:, 9:10].t(), x[:, 9:10].t(), dy)):
        a, b = want.double().cpu(), size.double().cpu()
        _close(got, a @ b, (n + 8) * U32 * (a.abs() @ b.abs()), BF16)


@pytest.mark.parametrize("n", [1, 63, 64, 200, 300, 1000, 1100])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_gradients_of_few_rows_with_wide_weights(helios, h, n, dtype):
    """One to seven groups of tiles, which go to all XCDs, and eight and nine, which go to one each."""
    k, m = 1000, 520
    x, w, dy = _rand(n, k, 1).to(dtype), _rand(m, k, 2, 0.03).to(dtype), _rand(n, m, 3).to(dtype)
    dx, dw = torch.full((n, k), -7.0, dtype=dtype, device="cuda"), torch.full((m, k), -7.0, dtype=dtype, device="cuda")
    h.linear_grad(x.cuda(), w.cuda(), dy.cuda(), dx=dx, dw=dw)
    y = torch.full((n, m), -7.0, dtype=dtype, device="cuda")
    h.linear(x.cuda(), w.cuda(), y)
    h.sync()
    xd, wd, d = x.double(), w.double(), dy.double()
    _close(dx, d @ wd, (m + 8) * U32 * (d.abs() @ wd.abs()), dtype)
    _close(dw, d.t() @ xd, (n + 8) * U32 * (d.abs().t() @ xd.abs()), dtype)
    _close(y, xd @ wd.t(), (k + 8) * U32 * (xd.abs() @ wd.abs().t()), dtype)


def test_scratch_that_cannot_be_doubled_is_what_the_call_needs(helios, h):
    """1 GiB of scratch, and 1.25 GiB asked for where 2 GiB are not to be had; then more than there is, which is an error of this call only."""
    gib, width = 1 << 30, 1024
    w, row = torch.ones((width, 8), device="cuda"), torch.ones((1, width), device="cuda")
    rows = {q: int(q * gib / 4 / width) for q in (1.0, 1.25, 3.0)}
    dx = torch.empty((rows[3.0], 8), device="cuda")

    def call(q):                                  # (its scratch: dz, in single precision)
        n = rows[q]
        dx[:n].fill_(-7.0)
        h.linear_grad(dx[:n], w, row.expand(n, width), act=helios.ACT_RELU, pre=row.expand(n, width), dx=dx[:n])
        h.sync()
        return bool((dx[:n] == width).all())

    assert call(1.0)
    room = []
    try:
        for _ in range(4):                        # (what is free afterwards is not to the byte what was asked to be left)
            if _free() > 1.8 * gib:
                room.append(torch.empty(_free() - int(1.6 * gib), dtype=torch.uint8, device="cuda"))
        assert 1.3 * gib < _free() < 1.9 * gib
        assert call(1.25)
        with pytest.raises(helios.HeliosError) as e:
            call(3.0)
        assert e.value.code == helios.EHIP and "scratch" in str(e.value)
        assert call(1.25) and call(1.0)
    finally:
        room.clear()
        torch.cuda.empty_cache()
    assert call(3.0)


def test_rows_too_far_apart_are_refused(helios, h):
    """Where the bytes from the first row to the last are more than 64 bits hold, or than can be addressed: such rows' places cannot be told apart."""
    p, q = (torch.zeros(64, device="cuda").data_ptr() for _ in range(2))
    lib = helios._lib
    for rows, ld in ((1 << 30, 1 << 40), (1 << 30, 1 << 32), (1 << 20, 1 << 38)):
        assert lib.helios_quantize_rows(h._h, rows, None, 4, helios.F32, p, ld, q, 4, q) == helios.EINVAL
        assert b"too far apart" in lib.helios_last_error(h._h)
        assert lib.helios_linear(h._h, helios.LinearArgs(n_rows=rows, n_in=4, n_out=4, x=p, x_ld=4, w=p, w_ld=4, y=q, y_ld=ld)) == helios.EINVAL
        assert b"too far apart" in lib.helios_last_error(h._h)
