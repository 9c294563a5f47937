"""The operators of a layer (products, norm, neighbour mean, their gradients) against plain 64-bit forms.

Bounds are worked out from the formulas, per element.  With u the rounding of a type (half the distance between
neighbouring values, relative) and U = 2^-24 that of the 32-bit steps in between, a sum of k products is off by at most
(k + 8) U times the sum of the products' magnitudes; an activation of slope at most 1.13 passes that on, and its own
evaluation is good to 2^-20 of its argument; a result is rounded once to its type, which adds u times its magnitude (and half the
smallest subnormal)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
U32 = 2.0 ** -24
ROUND = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8, E4M3: 2.0 ** -4}
TINY = {F32: 2.0 ** -149, F16: 2.0 ** -25, BF16: 2.0 ** -134, E4M3: 2.0 ** -10}
ACTS = ["none", "relu", "gelu", "silu"]
EPS = 1e-6


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


def _rand(n, d, seed, scale=1.0):
    return scale * torch.from_numpy(np.random.default_rng(seed).standard_normal((n, d)))


def _on_gpu(t, dtype, pad=0, at=0, fill=float("nan")):
    """A copy of t on the GPU whose rows are t.shape[1] + pad apart and start `at` elements into the array; NaN everywhere else."""
    n, d = t.shape
    room = torch.full((n * (d + pad) + at + 16,), fill, dtype=torch.float32).to(dtype).cuda()
    view = room[at:at + n * (d + pad)].view(n, d + pad)[:, :d] if n else torch.empty((0, d), dtype=dtype, device="cuda")
    view.copy_(t.to(torch.float32).to(dtype))
    view.room = room
    return view


def _out(n, d, dtype, pad=0, at=0):
    return _on_gpu(torch.full((n, d), -7.0), dtype, pad, at, fill=-7.0)


def _untouched(t):
    """Whether what lies around t's rows still holds the fill value."""
    mark = t.room.float().cpu().clone()
    seen = torch.zeros(mark.numel(), dtype=torch.bool)
    off = t.storage_offset()
    for i in range(t.shape[0]):
        seen[off + i * t.stride(0):off + i * t.stride(0) + t.shape[1]] = True
    return bool((mark[~seen] == -7.0).all())


def _close(got, want, bound, dtype, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    limit = bound + ROUND[dtype] * (want.abs() + bound) + TINY[dtype]
    worse = (got - want).abs() - limit
    assert not torch.isnan(got).any() or torch.isnan(want).any(), what
    bad = ~((worse <= 0) | (torch.isnan(got) & torch.isnan(want)) | (got == want))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, the worst by {float(worse[bad].max()):.3g}"


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    return z * torch.sigmoid(z) if act == "silu" else z


def _slope(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


# ------------------------------------------------------------------ product


SHAPES = [(1, 1, 1), (1, 256, 256), (3, 5, 7), (16, 64, 16), (17, 33, 65), (31, 2048, 24), (64, 128, 64), (65, 200, 47), (129, 72, 130), (300, 513, 257),
          (777, 100, 172), (4100, 40, 1000), (33000, 24, 9)]


def _linear_case(helios, h, n, k, m, x_type, out_type, act, bias, residual, pre, pads, seed, count=None):
    x64, w64 = _rand(n, k, seed), _rand(m, k, seed + 1, k ** -0.5)
    scales, sx, sw = {}, 1.0, 1.0
    px, pw, py = pads
    x, w = _on_gpu(x64, x_type, px, px % 3), _on_gpu(w64, x_type, pw, pw % 5)
    if x_type == E4M3:
        sx, sw = _rand(n, 1, seed + 2).abs() + 0.1, _rand(m, 1, seed + 3).abs() + 0.1
        scales = {"x_scale": sx.float().cuda().view(-1), "w_scale": sw.float().cuda().view(-1)}
        sx, sw = scales["x_scale"].double().cpu()[:, None], scales["w_scale"].double().cpu()[None, :]
    b = _rand(1, m, seed + 4)[0].to(out_type).cuda() if bias else None
    r = _on_gpu(_rand(n, m, seed + 5), out_type, py, py % 2) if residual else None
    y, z = _out(n, m, out_type, py, py % 3), _out(n, m, out_type, py) if pre else None
    n_dev = None
    if count is not None:
        n_dev = torch.tensor([count], dtype=torch.int64, device="cuda")
        x[count:] = float("nan")
    h.linear(x, w, y, bias=b, act=getattr(helios, "ACT_" + act.upper()), residual=r, pre=z, n_rows_dev=n_dev, **scales)
    h.sync()
    live = n if count is None else count
    xd, wd = x.double().cpu()[:live], w.double().cpu()
    sx = sx[:live] if x_type == E4M3 else sx
    want_z, size = xd @ wd.t() * sx * sw, xd.abs() @ wd.abs().t() * sx * sw
    if b is not None:
        want_z, size = want_z + b.double().cpu(), size + b.double().abs().cpu()
    bound = 1.13 * (k + 8) * U32 * size + 2.0 ** -20 * want_z.abs()
    if z is not None:
        _close(z[:live], want_z, (k + 8) * U32 * size, out_type, "pre")
        assert _untouched(z) and bool((z[live:] == -7.0).all())
    want = _act(want_z, act)
    if r is not None:
        rd = r.double().cpu()[:live]
        want, bound = want + rd, bound + 2 * U32 * (rd.abs() + want.abs())
    _close(y[:live], want, bound, out_type, "y")
    assert _untouched(y) and bool((y[live:] == -7.0).all())


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("x_type,out_type", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32), (E4M3, F16), (E4M3, BF16), (E4M3, F32)], ids=str)
def test_linear(helios, h, shape, x_type, out_type):
    n, k, m = shape
    print("linear", shape, x_type, out_type, flush=True)
    seed = n + 3 * k + 7 * m
    _linear_case(helios, h, n, k, m, x_type, out_type, ACTS[seed % 4], True, True, True, (0, 0, 0), seed)
    _linear_case(helios, h, n, k, m, x_type, out_type, ACTS[(seed + 1) % 4], False, False, False, (3, 1, 5), seed + 10)
    _linear_case(helios, h, n, k, m, x_type, out_type, ACTS[(seed + 2) % 4], True, False, True, (16, 16, 8), seed + 20)


@pytest.mark.parametrize("x_type,out_type", [(F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)], ids=str)
def test_linear_of_long_lists(helios, h, x_type, out_type):
    """Lists of several rounds of tiles, where tiles are 160 rows high; the last one is cut short, in rows and columns."""
    print("linear long", x_type, out_type, flush=True)
    _linear_case(helios, h, 20400, 584, 1000, x_type, out_type, "relu", True, True, True, (0, 0, 0), 5)
    _linear_case(helios, h, 20391, 583, 1001, x_type, out_type, "silu", True, True, False, (3, 1, 5), 6, 20390)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("x_type", [F32, F16, BF16, E4M3], ids=str)
def test_linear_with_the_count_on_the_device(helios, h, x_type, act):
    """Rows behind the count hold NaN and are neither read nor written."""
    out_type = F16 if x_type == E4M3 else x_type
    for n, count in ((16, 3), (200, 0), (200, 77), (200, 200), (5000, 4097)):
        print("linear count", x_type, act, n, count, flush=True)
        _linear_case(helios, h, n, 72, 72 if n < 5000 else 900, x_type, out_type, act, True, True, True, (0, 0, 0), n + count, count)


def test_linear_repeats_a_row_and_writes_over_its_residual(helios, h):
    x64, w64, r64 = _rand(1, 96, 1), _rand(80, 96, 2, 0.1), _rand(50, 80, 3)
    x, w, y = x64.half().cuda().expand(50, 96), w64.half().cuda(), r64.half().cuda()
    want = (x.double().cpu() @ w.double().cpu().t()) + y.double().cpu()
    h.linear(x, w, y, residual=y)
    h.sync()
    _close(y, want, 2 * 104 * U32 * (x.double().abs().cpu() @ w.double().abs().cpu().t() + want.abs() + 4), F16)


@pytest.mark.parametrize("dtype", [F32, F16, BF16, E4M3], ids=str)
@pytest.mark.parametrize("n", [5, 100])
def test_linear_keeps_infinities_and_nan_to_their_rows(helios, h, n, dtype):
    """A row of x that is not finite makes its own row of y so, and no other."""
    out_type = F32 if dtype == E4M3 else dtype
    x64, w64 = _rand(n, 64, 5), _rand(40, 64, 6)
    x, w = x64.float().to(dtype).cuda(), w64.float().to(dtype).cuda()
    x[2, 7] = float("nan")
    if dtype != E4M3:
        x[3, 9] = float("inf")
    scales = {"x_scale": torch.ones(n, device="cuda"), "w_scale": torch.ones(40, device="cuda")} if dtype == E4M3 else {}
    y = torch.zeros((n, 40), dtype=out_type, device="cuda")
    h.linear(x, w, y, **scales)
    h.sync()
    want = x.double().cpu() @ w.double().cpu().t()
    got = y.double().cpu()
    assert torch.isnan(got[2]).all()
    if dtype != E4M3:
        assert torch.equal(got[3], want[3]) and torch.isinf(want[3]).all()
    rest = [i for i in range(n) if i not in (2, 3)]
    _close(y[rest], want[rest], 72 * U32 * (x[rest].double().abs().cpu() @ w.double().abs().cpu().t()), out_type)


def _linear_grad_case(helios, h, n, k, m, x_type, out_type, act, pads, seed, count=None, outs=("dx", "dw", "dbias")):
    px, pw, py = pads
    x, w = _on_gpu(_rand(n, k, seed), x_type, px, px % 3), _on_gpu(_rand(m, k, seed + 1), x_type, pw)
    dy, pre = _on_gpu(_rand(n, m, seed + 2), out_type, py, py % 3), _on_gpu(_rand(n, m, seed + 3), out_type, py)
    room = {"dx": _out(n, k, x_type, px, px % 2), "dw": _out(m, k, x_type, pw, pw % 3), "dbias": torch.full((m,), -7.0, dtype=out_type, device="cuda")}
    n_dev = None
    live = n if count is None else count
    if count is not None:
        n_dev = torch.tensor([count], dtype=torch.int64, device="cuda")
        for t in (x, dy, pre):
            t[count:] = float("nan")
    h.linear_grad(x, w, dy, act=getattr(helios, "ACT_" + act.upper()), pre=pre if act != "none" else None, n_rows_dev=n_dev, **{o: room[o] for o in outs})
    h.sync()
    xd, wd, d, p = (t.double().cpu() for t in (x[:live], w, dy[:live], pre[:live]))
    slope = _slope(p, act)
    dz, dz_off = d * slope, 2.0 ** -20 * d.abs() * (1 + p.abs())          # the slope is good to 2^-20 of its terms
    exact = act in ("none", "relu") and (out_type == x_type)
    rounded = dz_off + (0 if exact else ROUND[x_type] * dz.abs() + TINY[x_type])
    if "dx" in outs:
        _close(room["dx"][:live], dz @ wd, rounded @ wd.abs() + (m + 8) * U32 * (dz.abs() @ wd.abs()), x_type, "dx")
        assert _untouched(room["dx"]) and bool((room["dx"][live:] == -7.0).all())
    if "dw" in outs:
        _close(room["dw"], dz.t() @ xd, rounded.t() @ xd.abs() + (live + 8) * U32 * (dz.abs().t() @ xd.abs()), x_type, "dw")
        assert _untouched(room["dw"])
    if "dbias" in outs:
        _close(room["dbias"], dz.sum(0), (dz_off + (live + 8) * U32 * dz.abs()).sum(0), out_type, "dbias")


@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] != 33000] + [(0, 8, 8), (4100, 1000, 24), (9000, 65, 33)], ids=str)
@pytest.mark.parametrize("x_type,out_type", [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)], ids=str)
def test_linear_grad(helios, h, shape, x_type, out_type):
    n, k, m = shape
    print("linear_grad", shape, x_type, out_type, flush=True)
    seed = n + 3 * k + 7 * m
    _linear_grad_case(helios, h, n, k, m, x_type, out_type, ACTS[seed % 4], (0, 0, 0), seed)
    _linear_grad_case(helios, h, n, k, m, x_type, out_type, ACTS[(seed + 1) % 4], (3, 1, 5), seed + 10)
    _linear_grad_case(helios, h, n, k, m, x_type, out_type, ACTS[(seed + 2) % 4], (8, 8, 8), seed + 20)


@pytest.mark.parametrize("outs", [("dx",), ("dw",), ("dbias",), ("dw", "dbias"), ("dx", "dw")], ids=str)
def test_linear_grad_of_some(helios, h, outs):
    for act in ("none", "gelu"):
        _linear_grad_case(helios, h, 130, 72, 40, BF16, BF16, act, (0, 0, 0), 77, outs=outs)
        _linear_grad_case(helios, h, 130, 72, 40, F32, F32, act, (0, 0, 0), 78, outs=outs)


@pytest.mark.parametrize("x_type", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("outs", [("dw",), ("dx", "dw")], ids=str)
def test_linear_grad_of_long_lists(helios, h, x_type, outs):
    """Long slices of rows, as many as fill the GPU once or twice."""
    print("linear grad long", x_type, outs, flush=True)
    _linear_grad_case(helios, h, 12500, 1000, 504, x_type, x_type, "relu", (0, 0, 0), 7, outs=outs)
    _linear_grad_case(helios, h, 12501, 1001, 503, x_type, x_type, "none", (3, 1, 5), 8, 12500, outs=outs)


@pytest.mark.parametrize("x_type", [F32, F16, BF16], ids=str)
def test_linear_grad_with_the_count_on_the_device(helios, h, x_type):
    for n, count in ((200, 0), (200, 1), (200, 130), (3000, 2049)):
        for act in ("none", "silu"):
            print("linear_grad count", x_type, n, count, act, flush=True)
            _linear_grad_case(helios, h, n, 72, 136, x_type, x_type, act, (0, 0, 0), n + count, count)


@pytest.mark.parametrize("act", ACTS)
def test_linear_grad_against_differences(helios, h, act):
    """Single precision against central differences of the 64-bit forward form: a step of e leaves terms of e^2 (the third
    derivatives are below 2), and relu's corner is kept out of the steps' way."""
    n, k, m, e = 5, 6, 4, 1e-4
    x, w, b, dy = _rand(n, k, 1).float(), _rand(m, k, 2).float(), _rand(1, m, 3)[0].float(), _rand(n, m, 4).float()
    loss = lambda x, w, b: float((_act(x @ w.t() + b, act) * dy.double()).sum())  # noqa: E731
    xd, wd, bd = x.double(), w.double(), b.double()
    z = xd @ wd.t() + bd
    assert z.abs().min() > 10 * e * max(xd.abs().max(), wd.abs().max())
    y, pre = torch.empty((n, m), device="cuda"), torch.empty((n, m), device="cuda")
    code = getattr(helios, "ACT_" + act.upper())
    h.linear(x.cuda(), w.cuda(), y, bias=b.cuda(), act=code, pre=pre)
    dx, dw, db = torch.empty((n, k), device="cuda"), torch.empty((m, k), device="cuda"), torch.empty(m, device="cuda")
    h.linear_grad(x.cuda(), w.cuda(), dy.cuda(), act=code, pre=pre, dx=dx, dw=dw, dbias=db)
    h.sync()
    for got, at in ((dx, 0), (dw, 1), (db, 2)):
        got = got.double().cpu()
        for i in range(got.numel()):
            args = [xd, wd, bd]
            side = []
            for s in (e, -e):
                moved = args[at].clone()
                moved.view(-1)[i] += s
                side.append(loss(*[moved if q == at else v for q, v in enumerate(args)]))
            assert abs(float(got.view(-1)[i]) - (side[0] - side[1]) / (2 * e)) < 2e-5


# ------------------------------------------------------------------ norm


WIDTHS = [1, 2, 7, 8, 64, 100, 128, 129, 200, 512, 513, 1000, 1024, 1032, 2048, 2049, 4100, 8192, 8200, 32768]


def _norm_case(h, n, d, dtype, out8, residual, gain, pad, seed, count=None, total=True, scale=1.0):
    x = _on_gpu(_rand(n, d, seed, scale), dtype, pad, pad % 3)
    r = _on_gpu(_rand(n, d, seed + 1, 3 * scale), dtype, pad) if residual else None
    g = (_rand(1, d, seed + 2, 0.3)[0] + 1).to(dtype).cuda() if gain else None
    t = _out(n, d, dtype, pad) if total else None
    y = _out(n, d, E4M3 if out8 else dtype, pad, pad % 5)
    y_scale = torch.full((n,), -7.0, device="cuda") if out8 else None
    inv = torch.full((n,), -7.0, device="cuda")
    n_dev = None
    live = n if count is None else count
    if count is not None:
        n_dev = torch.tensor([count], dtype=torch.int64).pin_memory()
        x[count:] = float("nan")
    h.rms_norm(x, y, EPS, gain=g, residual=r, total=t, y_scale=y_scale, inv_rms=inv, n_rows_dev=n_dev)
    h.sync()
    xd = x.double().cpu()[:live]
    rd = r.double().cpu()[:live] if residual else torch.zeros_like(xd)
    td = xd + rd
    t_off = U32 * td.abs()
    if total:
        _close(t[:live], td, t_off, dtype, "total")
        assert _untouched(t) and bool((t[live:] == -7.0).all())
    q = 1 / torch.sqrt((td * td).mean(1, keepdim=True) + EPS)
    _close(inv[:live], q[:, 0], (d + 8) * U32 * q[:, 0], F32, "inv_rms")
    want = td * q * (g.double().cpu() if gain else 1.0)
    off = (d + 12) * U32 * want.abs()
    if not out8:
        _close(y[:live], want, off, dtype, "y")
    else:
        s = (want.abs().amax(1) / 448.0).clamp_min(2.0 ** -126) if live else torch.zeros(0, dtype=torch.float64)
        _close(y_scale[:live], s, (d + 16) * U32 * s, F32, "scale")
        _close(y[:live], want / s[:, None], (2 * d + 32) * U32 * (want / s[:, None]).abs(), E4M3, "y")
    assert _untouched(y) and bool((y[live:].float() == torch.full((1,), -7.0).to(y.dtype).float().cuda()).all())


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_norm(h, d, dtype):
    print("norm", d, dtype, flush=True)
    for k, (n, pad) in enumerate(((1, 0), (5, 3), (67, 8))):
        for out8 in (False, True):
            _norm_case(h, n, d, dtype, out8, k != 1, k != 2, pad, d + 10 * k + out8)
    _norm_case(h, 9, d, dtype, False, False, True, 0, d, total=False)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_norm_with_the_count_on_the_device(h, dtype):
    for d in (100, 700, 5000):
        for n, count in ((40, 0), (40, 1), (40, 33)):
            for out8 in (False, True):
                _norm_case(h, n, d, dtype, out8, True, True, 0, d + count, count)


@pytest.mark.parametrize("d", [64, 520, 3000])
def test_norm_of_rows_of_zeros_infinities_and_tiny_values(h, d):
    x = _rand(6, d, 9).float().cuda()
    x[1] = 0
    x[2, d // 2] = float("inf")
    x[3, d - 1] = float("nan")
    x[4] = 1e-30
    y = torch.empty((6, d), device="cuda")
    y8, s = torch.empty((6, d), dtype=E4M3, device="cuda"), torch.empty(6, device="cuda")
    h.rms_norm(x, y, EPS)
    h.rms_norm(x, y8, EPS, y_scale=s)
    h.sync()
    assert bool((y[1] == 0).all()) and bool((y8[1].float() == 0).all()) and float(s[1]) == 2.0 ** -126
    assert bool(torch.isnan(y[2, d // 2])) and bool((y[2, :d // 2] == 0).all()) and bool(torch.isnan(y[3]).all())
    assert bool(torch.isnan(s[2])) and bool(torch.isnan(s[3])) and bool(torch.isnan(y8[3].float()).all())
    want = 1e-30 / math.sqrt(EPS)
    assert abs(float(y[4, 0]) - want) < 1e-5 * want and bool((y8[4].float() == 448).all())
    for i in (0, 5):
        q = x[i].double() / torch.sqrt((x[i].double() ** 2).mean() + EPS)
        _close(y[i].cpu(), q.cpu(), (d + 12) * U32 * q.abs().cpu(), F32)


def test_norm_over_its_own_inputs(h):
    n, d = 33, 300
    x64, r64 = _rand(n, d, 1).float(), _rand(n, d, 2).float()
    want_t = x64.double() + r64.double()
    want = want_t / torch.sqrt((want_t ** 2).mean(1, keepdim=True) + EPS)
    x, r = x64.cuda(), r64.cuda()
    h.rms_norm(x, x, EPS, residual=r, total=r)            # total over the residual, y over x
    h.sync()
    _close(r, want_t, U32 * want_t.abs(), F32)
    _close(x, want, (d + 12) * U32 * want.abs(), F32)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_quantize_rows(h, d, dtype):
    for n, pad in ((1, 0), (37, 3)):
        x = _on_gpu(_rand(n, d, d, 5.0), dtype, pad)
        q, s = _out(n, d, E4M3, pad), torch.empty(n, device="cuda")
        h.quantize_rows(x, q, s)
        h.sync()
        xd = x.double().cpu()
        want = (xd.abs().amax(1) / 448).clamp_min(2.0 ** -126)
        _close(s, want, 2 * U32 * want, F32)
        _close(q, xd / want[:, None], 8 * U32 * (xd / want[:, None]).abs(), E4M3)
        assert _untouched(q)


def _norm_grad_case(h, n, d, dtype, dtotal, gain, use_inv, pad, seed, count=None, dgain=True):
    t, dy = _on_gpu(_rand(n, d, seed, 2.0), dtype, pad, pad % 3), _on_gpu(_rand(n, d, seed + 1), dtype, pad)
    dt = _on_gpu(_rand(n, d, seed + 2), dtype, pad) if dtotal else None
    g = (_rand(1, d, seed + 3, 0.3)[0] + 1).to(dtype).cuda() if gain else None
    live = n if count is None else count
    td, dyd = t.double().cpu()[:live], dy.double().cpu()[:live]
    q = 1 / torch.sqrt((td * td).mean(1, keepdim=True) + EPS)
    inv = torch.zeros(n, device="cuda")
    inv[:live] = q[:, 0].float().cuda()
    n_dev = None
    if count is not None:
        n_dev = torch.tensor([count], dtype=torch.int64, device="cuda")
        t[count:] = float("nan")
        dy[count:] = float("nan")
    dx, dg = _out(n, d, dtype, pad, pad % 2), torch.full((d,), -7.0, dtype=dtype, device="cuda") if dgain else None
    h.rms_norm_grad(t, dy, dx, EPS, gain=g, dtotal=dt, dgain=dg, inv_rms=inv if use_inv else None, n_rows_dev=n_dev)
    h.sync()
    u = dyd * (g.double().cpu() if gain else 1.0)
    back = td * q ** 3 * (u * td).mean(1, keepdim=True)
    want = q * u - back
    off = (2 * d + 24) * U32 * (q * u.abs() + td.abs() * q ** 3 * (u * td).abs().mean(1, keepdim=True))
    if dtotal:
        want = want + dt.double().cpu()[:live]
        off = off + 2 * U32 * (want.abs() + dt.double().abs().cpu()[:live])
    _close(dx[:live], want, off, dtype, "dx")
    assert _untouched(dx) and bool((dx[live:] == -7.0).all())
    if dgain:
        each = dyd * td * q
        _close(dg, each.sum(0), (live + d + 24) * U32 * each.abs().sum(0), dtype, "dgain")


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_norm_grad(h, d, dtype):
    print("norm_grad", d, dtype, flush=True)
    for k, (n, pad) in enumerate(((1, 0), (5, 3), (67, 8))):
        _norm_grad_case(h, n, d, dtype, k != 1, k != 2, k == 1, pad, d + 10 * k)
    _norm_grad_case(h, 9, d, dtype, False, True, False, 0, d, dgain=False)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_norm_grad_of_many_rows_and_of_a_count_on_the_device(h, dtype):
    _norm_grad_case(h, 20_011, 40, dtype, True, True, False, 0, 3)
    _norm_grad_case(h, 5_003, 260, dtype, True, True, False, 0, 4)
    for d in (100, 700, 5000):
        for n, count in ((40, 0), (40, 1), (40, 33)):
            _norm_grad_case(h, n, d, dtype, True, True, False, 0, d + count, count)


def test_norm_grad_of_no_rows(h):
    dg = torch.full((24,), -7.0, device="cuda")
    e = torch.empty((0, 24), device="cuda")
    h.rms_norm_grad(e, e, e, EPS, dgain=dg)
    h.sync()
    assert bool((dg == 0).all())


def test_norm_grad_against_differences(h):
    n, d, e = 4, 9, 1e-4
    t, dy, g = _rand(n, d, 1).float(), _rand(n, d, 2).float(), (_rand(1, d, 3)[0] + 1).float()
    loss = lambda t, g: float((t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS) * g * dy.double()).sum())  # noqa: E731
    dx, dg = torch.empty((n, d), device="cuda"), torch.empty(d, device="cuda")
    h.rms_norm_grad(t.cuda(), dy.cuda(), dx, EPS, gain=g.cuda(), dgain=dg)
    h.sync()
    td, gd = t.double(), g.double()
    for got, at in ((dx, 0), (dg, 1)):
        got = got.double().cpu()
        for i in range(got.numel()):
            side = []
            for s in (e, -e):
                args = [td.clone(), gd.clone()]
                args[at].view(-1)[i] += s
                side.append(loss(*args))
            assert abs(float(got.view(-1)[i]) - (side[0] - side[1]) / (2 * e)) < 1e-5


# ------------------------------------------------------------------ neighbours


def _block(n, n_src, fan, seed, popular=0):
    """A hop in local numbering: row i has 0 to fan samples; `popular` rows in ten also take source 0."""
    rng = np.random.default_rng(seed)
    deg = np.minimum(rng.integers(0, fan + 3, n), fan)
    deg[rng.random(n) < 0.1] = 0
    indptr = np.zeros(n + 1, np.int64)
    indptr[1:] = np.cumsum(deg)
    col = rng.integers(0, max(n_src, 1), indptr[-1]).astype(np.int32)
    if popular:
        first = indptr[:-1][deg > 0]
        col[first[rng.random(first.size) < popular / 10]] = 0
    row = rng.integers(0, max(n_src, 1), n).astype(np.int32)
    return torch.from_numpy(indptr), torch.from_numpy(col), torch.from_numpy(row)


def _dense(indptr, col, n, n_src):
    m = torch.zeros((n, n_src), dtype=torch.float64)
    for i in range(n):
        lo, hi = int(indptr[i]), int(indptr[i + 1])
        for e in range(lo, hi):
            m[i, int(col[e])] += 1.0 / (hi - lo)
    return m


BLOCKS = [(1, 1, 1), (1, 5, 3), (7, 3, 5), (128, 600, 5), (300, 40, 25), (90, 2000, 10)]


@pytest.mark.parametrize("d", [1, 8, 30, 64, 100, 128, 200, 256, 300, 512, 1024, 1100])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_block_mean_and_gradient(h, d, dtype):
    for n, n_src, fan in BLOCKS:
        for pad, with_row in ((0, True), (3, False), (8, True)):
            seed = n + n_src + d + pad
            indptr, col, row = _block(n, n_src, fan, seed, popular=9)
            use_row = with_row or n_src < n
            x = _on_gpu(_rand(n_src, d, seed), dtype, pad, pad % 3)
            both = torch.full((n, 2 * d + pad), -7.0, dtype=dtype, device="cuda")
            own, mean = both[:, :d], both[:, d:2 * d]
            ip, cl, rw = indptr.cuda(), col.cuda(), row.cuda() if use_row else None
            print("block", n, n_src, fan, d, dtype, pad, flush=True)
            h.block_mean(x, ip, cl, mean, row=rw, own=own)
            h.sync()
            m, xd = _dense(indptr, col, n, n_src), x.double().cpu()
            at = row.long() if use_row else torch.arange(n)
            assert torch.equal(own.cpu(), x.cpu()[at])
            _close(mean, m @ xd, (fan + 4) * U32 * (m @ xd.abs()), dtype, "mean")
            assert bool((both[:, 2 * d:] == -7.0).all())
            # gradient
            dmean, down = _on_gpu(_rand(n, d, seed + 1), dtype, pad, pad % 2), _on_gpu(_rand(n, d, seed + 2), dtype, pad)
            si = torch.full((n_src + 1,), -7, dtype=torch.int32, device="cuda")
            se = torch.full((max(1, col.numel() + (n if use_row else 0)),), -7, dtype=torch.int32, device="cuda")
            h.block_transpose(ip, cl, n_src, si, se, row=rw)
            dx = _out(n_src, d, dtype, pad)
            h.block_mean_grad(ip, si, se, dmean, dx, down=down if use_row else None)
            h.sync()
            dm, dn = dmean.double().cpu(), down.double().cpu()
            want, size = m.t() @ dm, m.t() @ dm.abs()
            if use_row:
                want = want.index_add(0, at, dn)
                size = size.index_add(0, at, dn.abs())
            entries = (si[1:] - si[:-1]).double().cpu()[:, None]
            _close(dx, want, (entries + 4) * U32 * size, dtype, "dx")
            assert _untouched(dx)
            if d == 8 and pad == 0:
                lists = [[] for _ in range(n_src)]
                for i in range(n):
                    for e in range(int(indptr[i]), int(indptr[i + 1])):
                        lists[int(col[e])].append(i)
                for i in range(n):
                    lists[int(row[i])].append(~i)
                assert si.tolist() == [0] + np.cumsum([len(v) for v in lists]).tolist()
                assert se.tolist() == sum(lists, [])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_block_with_the_count_on_the_device(h, dtype):
    """Worst-case buffers, as a batch has them: what lies behind the count and behind the last list is never looked at."""
    n, n_src, d = 200, 90, 72
    indptr, col, row = _block(n, n_src, 6, 4)
    x = _rand(n_src, d, 1).to(dtype).cuda()
    for count in (0, 1, 150, 200):
        used = int(indptr[count])
        ip, cl, rw = indptr.clone(), torch.cat([col, torch.zeros(50, dtype=torch.int32)]), row.clone()
        ip[count + 1:] = -5
        cl[used:] = 10 ** 9
        rw[count:] = -3
        ip, cl, rw, n_dev = ip.cuda(), cl.cuda(), rw.cuda(), torch.tensor([count], dtype=torch.int64, device="cuda")
        own, mean = torch.full((n, d), -7.0, dtype=dtype, device="cuda"), torch.full((n, d), -7.0, dtype=dtype, device="cuda")
        h.block_mean(x, ip, cl, mean, row=rw, own=own, n_rows_dev=n_dev)
        si, se = torch.empty(n_src + 1, dtype=torch.int32, device="cuda"), torch.empty(cl.numel() + n, dtype=torch.int32, device="cuda")
        h.block_transpose(ip, cl, n_src, si, se, row=rw, n_rows_dev=n_dev)
        dmean, down = _rand(n, d, 2).to(dtype).cuda(), _rand(n, d, 3).to(dtype).cuda()
        dx = torch.empty((n_src, d), dtype=dtype, device="cuda")
        h.block_mean_grad(ip, si, se, dmean, dx, down=down)
        h.sync()
        m = _dense(indptr, col, count, n_src)
        _close(mean[:count], m @ x.double().cpu(), 10 * U32 * (m @ x.double().abs().cpu()), dtype, "mean")
        assert torch.equal(own[:count].cpu(), x.cpu()[row[:count].long()])
        assert bool((mean[count:] == -7.0).all()) and bool((own[count:] == -7.0).all())
        want = (m.t() @ dmean.double().cpu()[:count]).index_add(0, row[:count].long(), down.double().cpu()[:count])
        size = (m.t() @ dmean.double().abs().cpu()[:count]).index_add(0, row[:count].long(), down.double().abs().cpu()[:count])
        _close(dx, want, 300 * U32 * size, dtype, "dx")


def test_block_of_one_source_with_a_very_long_list(h):
    n, n_src, d = 9000, 30, 136
    indptr = torch.arange(n + 1, dtype=torch.int64) * 2
    col = torch.stack([torch.full((n,), 17, dtype=torch.int32), torch.arange(n, dtype=torch.int32) % n_src], 1).reshape(-1)
    dmean, dx = _rand(n, d, 2).float().cuda(), torch.empty((n_src, d), device="cuda")
    si, se = torch.empty(n_src + 1, dtype=torch.int32, device="cuda"), torch.empty(2 * n, dtype=torch.int32, device="cuda")
    h.block_transpose(indptr.cuda(), col.cuda(), n_src, si, se)
    h.block_mean_grad(indptr.cuda(), si, se, dmean, dx)
    h.sync()
    each = dmean.double().cpu().repeat_interleave(2, 0) / 2
    want = torch.zeros((n_src, d), dtype=torch.float64).index_add(0, col.long(), each)
    size = torch.zeros((n_src, d), dtype=torch.float64).index_add(0, col.long(), each.abs())
    _close(dx, want, (n + 320) * U32 * size, F32)


def test_block_with_bad_indices_is_reported(helios, h):
    x = _rand(10, 16, 1).float().cuda()
    ip = torch.tensor([0, 2, 3], dtype=torch.int64, device="cuda")
    good_col, row = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    mean, own = torch.zeros((2, 16), device="cuda"), torch.zeros((2, 16), device="cuda")

    def fails(*args, **kw):
        h.block_mean(*args, **kw)
        with pytest.raises(helios.HeliosError) as e:
            h.sync()
        assert e.value.code == helios.EDATA

    for bad in (-1, 10, 2 ** 31 - 1):
        fails(x, ip, torch.tensor([1, bad, 3], dtype=torch.int32, device="cuda"), mean)
        assert torch.allclose(mean[0], x[1] / 2) and torch.equal(mean[1], x[3])
        fails(x, ip, good_col, mean, row=torch.tensor([0, bad], dtype=torch.int32, device="cuda"), own=own)
    for bad in ([0, 4, 3], [0, -1, 3], [0, 2, 9], [3, 2, 3]):
        fails(x, torch.tensor(bad, dtype=torch.int64, device="cuda"), good_col, mean)
    si, se = torch.empty(11, dtype=torch.int32, device="cuda"), torch.empty(5, dtype=torch.int32, device="cuda")
    h.block_transpose(ip, torch.tensor([1, 99, 3], dtype=torch.int32, device="cuda"), 10, si, se, row=row)
    with pytest.raises(helios.HeliosError) as e:
        h.sync()
    assert e.value.code == helios.EDATA
    dx = torch.empty((10, 16), device="cuda")
    h.block_transpose(ip, good_col, 10, si, se, row=row)
    h.sync()
    h.block_mean_grad(ip, si, se, mean, dx)               # own sources among the entries, and no gradient for them
    with pytest.raises(helios.HeliosError) as e:
        h.sync()
    assert e.value.code == helios.EDATA
    se.fill_(7)                                           # entries of rows that there are none of
    h.block_mean_grad(ip, si, se, mean, dx, down=own)
    with pytest.raises(helios.HeliosError) as e:
        h.sync()
    assert e.value.code == helios.EDATA
    assert bool((dx == 0).all())


def test_block_without_samples_or_sources(h):
    ip = torch.zeros(4, dtype=torch.int64, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    mean = torch.full((3, 24), -7.0, device="cuda")
    h.block_mean(torch.empty((0, 24), device="cuda"), ip, none, mean)
    si, se = torch.full((6,), -7, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    h.block_transpose(ip, none, 5, si, se)
    dx = torch.full((5, 24), -7.0, device="cuda")
    h.block_mean_grad(ip, si, se, mean, dx)
    h.sync()
    assert bool((mean == 0).all()) and si.tolist() == [0] * 6 and bool((dx == 0).all())


def test_block_gradient_against_differences(h):
    n, n_src, d, e = 6, 5, 3, 1e-3
    indptr, col, row = _block(n, n_src, 3, 8)
    x, dm, dn = _rand(n_src, d, 1), _rand(n, d, 2).float(), _rand(n, d, 3).float()
    m = _dense(indptr, col, n, n_src)
    loss = lambda x: float(((m @ x) * dm.double()).sum() + (x[row.long()] * dn.double()).sum())  # noqa: E731
    si, se = torch.empty(n_src + 1, dtype=torch.int32, device="cuda"), torch.empty(col.numel() + n, dtype=torch.int32, device="cuda")
    dx = torch.empty((n_src, d), device="cuda")
    h.block_transpose(indptr.cuda(), col.cuda(), n_src, si, se, row=row.cuda())
    h.block_mean_grad(indptr.cuda(), si, se, dm.cuda(), dx, down=dn.cuda())
    h.sync()
    for i in range(x.numel()):
        side = []
        for s in (e, -e):
            moved = x.clone()
            moved.view(-1)[i] += s
            side.append(loss(moved))
        assert abs(float(dx.view(-1)[i]) - (side[0] - side[1]) / (2 * e)) < 1e-5


# ------------------------------------------------------------------ the calls as calls


def test_the_same_call_gives_the_same_bits_on_another_stream_and_in_a_graph(helios):
    n, k, m = 3000, 200, 136
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        indptr, col, row = (t.cuda() for t in _block(n, 700, 7, 3, popular=9))
        x, w, b = _rand(700, k, 1).half().cuda(), _rand(m, 2 * k, 2, 0.05).half().cuda(), _rand(1, m, 3)[0].half().cuda()
        gain = (_rand(1, m, 4, 0.1)[0] + 1).half().cuda()
        new = lambda *s, dtype=F16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        both, y, pre, t8, s8, dpre = new(n, 2 * k), new(n, m), new(n, m), new(n, m, dtype=E4M3), new(n, dtype=F32), new(n, m)
        dboth, dw, db, dg, dx = new(n, 2 * k), new(m, 2 * k), new(m), new(m), new(700, k)
        si, se = new(701, dtype=torch.int32), new(col.numel() + n, dtype=torch.int32)
        outs = [both, y, pre, t8, s8, dpre, dboth, dw, db, dg, dx, si, se]
        torch.cuda.synchronize()

        def step():
            h.block_mean(x, indptr, col, both[:, k:], row=row, own=both[:, :k])
            h.linear(both, w, y, bias=b, act=helios.ACT_GELU, pre=pre)
            h.rms_norm(y, t8, EPS, gain=gain, y_scale=s8)
            h.rms_norm_grad(y, y, dpre, EPS, gain=gain, dgain=dg)
            h.linear_grad(both, w, dpre, act=helios.ACT_GELU, pre=pre, dx=dboth, dw=dw, dbias=db)
            h.block_transpose(indptr, col, 700, si, se, row=row)
            h.block_mean_grad(indptr, si, se, dboth[:, k:], dx, down=dboth[:, :k])

        step()
        h.sync()
        want = [t.clone() for t in outs]
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
        same = lambda: all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs, want))  # noqa: E731
        for turn in range(4):
            print("graph replay", turn, flush=True)
            for t in outs:
                t.zero_()
            torch.cuda.synchronize()
            if turn % 2:
                step()
            else:
                with torch.cuda.stream(stream):
                    graph.replay()
            h.sync()
            assert same(), turn
            h.linear_grad(x, w[:, :k].contiguous(), y[:700], dx=torch.empty_like(x), dw=torch.empty((m, k), dtype=F16, device="cuda"))
            h.sync()
    finally:
        h.close()


def test_a_capture_that_would_have_to_allocate_is_refused(helios):
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        x, w, dy, dw = (torch.zeros(s, device="cuda") for s in ((64, 32), (16, 32), (64, 16), (16, 32)))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(helios.HeliosError) as e:
                h.linear_grad(x, w, dy, dw=dw)
        assert e.value.code == helios.ESTATE and "capture" in str(e.value)
        h.linear_grad(x, w, dy, dw=dw)
        h.sync()
    finally:
        h.close()


def test_refusals(helios, h):
    x, w, y = torch.zeros((8, 16), device="cuda"), torch.zeros((4, 16), device="cuda"), torch.zeros((8, 4), device="cuda")

    def einval(call, *args, **kw):
        with pytest.raises(helios.HeliosError) as e:
            call(*args, **kw)
        assert e.value.code == helios.EINVAL
        return str(e.value)

    def typeerror(call, *args, **kw):
        with pytest.raises(TypeError):
            call(*args, **kw)

    typeerror(h.linear, x.cpu(), w, y)
    typeerror(h.linear, x.double(), w, y)
    typeerror(h.linear, x, w.half(), y)
    typeerror(h.linear, x, w[:, :15], y)
    typeerror(h.linear, x.t(), w, y)
    typeerror(h.linear, x, w, y, bias=torch.zeros(5, device="cuda"))
    typeerror(h.linear, x, w, y, bias=torch.zeros(4, device="cuda", dtype=F16))
    typeerror(h.linear, x, w, y, pre=torch.zeros((8, 5), device="cuda"))
    assert "activation" in einval(h.linear, x, w, y, act=9)
    assert "out_type" in einval(h.linear, x, w, y.half())
    assert "n_in" in einval(h.linear, x[:, :0], w[:, :0], y)
    assert "shares memory" in einval(h.linear, x, w, x[:, :4])
    assert "shares memory" in einval(h.linear, x, w, y, pre=y)
    wide = torch.zeros((8, 8), device="cuda")
    assert "shares memory" in einval(h.linear, x, w, wide[:, :4], residual=wide[:, 3:7])
    h.linear(x, w, wide[:, :4], residual=wide[:, 4:])     # side by side is apart
    assert "x_scale" in einval(h.linear, x, w, y, x_scale=torch.ones(8, device="cuda"))
    assert "x_scale" in einval(h.linear, x.to(E4M3), w.to(E4M3), y)
    assert "out_type" in einval(h.linear, x.to(E4M3), w.to(E4M3), y.to(E4M3))
    assert "narrower" in einval(h.linear, x, w, y[:1].expand(8, 4))
    dy = torch.zeros((8, 4), device="cuda")
    assert "NULL" in einval(h.linear_grad, x, w, dy, act=helios.ACT_GELU, dx=torch.zeros_like(x))
    assert "no gradient" in einval(h.linear_grad, x.to(E4M3), w.to(E4M3), dy, dx=torch.zeros_like(x).to(E4M3))
    assert "shares memory" in einval(h.linear_grad, x, w, dy, dx=x, dw=torch.zeros_like(w))
    h.linear_grad(x, w, dy)                               # nothing asked for
    assert "width" in einval(h.rms_norm, torch.zeros((1, 32769), device="cuda"), torch.zeros((1, 32769), device="cuda"), EPS)
    assert "eps" in einval(h.rms_norm, x, torch.zeros_like(x), -1.0)
    assert "eps" in einval(h.rms_norm, x, torch.zeros_like(x), float("nan"))
    assert "y_scale" in einval(h.rms_norm, x, torch.zeros_like(x).to(E4M3), EPS)
    assert "y_scale" in einval(h.rms_norm, x, torch.zeros_like(x), EPS, y_scale=torch.zeros(8, device="cuda"))
    assert "y_type" in einval(h.rms_norm, x, torch.zeros_like(x).half(), EPS)
    assert "shares memory" in einval(h.rms_norm, x, x, EPS, total=x)
    assert "shares memory" in einval(h.rms_norm, x[1:], x[:-1], EPS)
    ip, col = torch.zeros(9, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    assert "shares memory" in einval(h.block_mean, x, ip, col, x)
    typeerror(h.block_mean, x, ip.int(), col, torch.zeros_like(x))
    typeerror(h.block_mean, x, ip, col.long(), torch.zeros_like(x))
    lib = helios._lib
    assert lib.helios_linear(None, None) == helios.EINVAL and lib.helios_linear(h._h, None) == helios.EINVAL
    assert lib.helios_linear(h._h, helios.LinearArgs(n_rows=1, n_in=4, n_out=4, x_ld=4, w_ld=4, y_ld=4)) == helios.EINVAL
    assert lib.helios_linear(h._h, helios.LinearArgs(n_rows=-1, n_in=4, n_out=4)) == helios.EINVAL
    assert lib.helios_linear(h._h, helios.LinearArgs(n_rows=2 ** 31, n_in=4, n_out=4)) == helios.EINVAL
    assert lib.helios_linear(h._h, helios.LinearArgs(n_rows=0, n_in=4, n_out=4)) == helios.OK
    p = x.data_ptr()
    assert lib.helios_linear(h._h, helios.LinearArgs(n_rows=1, n_in=4, n_out=4, x=p + 2, x_ld=4, w=w.data_ptr(), w_ld=4, y=y.data_ptr(), y_ld=4)) == helios.EINVAL
    assert lib.helios_block_transpose(h._h, 1, None, None, None, 0, None, 4, si_ptr := torch.zeros(5, dtype=torch.int32, device="cuda").data_ptr(), None) == helios.EINVAL
    assert si_ptr
    assert lib.helios_block_mean_grad(h._h, helios.BlockMeanGradArgs(n_rows=1, width=4, n_src=-1)) == helios.EINVAL
    assert lib.helios_quantize_rows(h._h, 1, None, 4, helios.E4M3, p, 4, p, 4, p) == helios.EINVAL
    h.sync()


# ------------------------------------------------------------------ values that are not finite in tiles, lists of several pieces


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("n,k,m", [(3000, 64, 256), (5000, 72, 1024), (3001, 67, 255)])
def test_products_in_tiles_keep_infinities_and_nan_to_their_rows_and_columns(helios, h, dtype, n, k, m):
    """A row of x that is not finite makes its own row of y so, a row of w its own column, and nothing else; dw likewise."""
    x, w, dy = (_rand(*s, seed).to(dtype).cuda() for s, seed in (((n, k), 1), ((m, k), 2), ((n, m), 3)))
    x[70, 5], x[71, 6], w[3, 1] = float("inf"), float("nan"), -float("inf")
    y = torch.zeros((n, m), dtype=dtype, device="cuda")
    h.linear(x, w, y)
    h.sync()
    want, got = x.double().cpu() @ w.double().cpu().t(), y.double().cpu()
    assert torch.isnan(got[71]).all() and torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    rows, cols = [i for i in range(n) if i not in (70, 71)], [j for j in range(m) if j != 3]
    clean = (x[rows].double().abs().cpu() @ w[cols].double().abs().cpu().t())
    _close(y[rows][:, cols], want[rows][:, cols], (k + 8) * U32 * clean, dtype)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    h.linear_grad(x, w, dy, dx=dx, dw=dw)
    h.sync()
    ref = dy.double().cpu().t() @ x.double().cpu()
    got = dw.double().cpu()
    assert torch.isnan(got[:, 6]).all() and torch.isinf(got[:, 5]).all() and torch.equal(got[:, 5], ref[:, 5])
    cols = [j for j in range(k) if j not in (5, 6)]
    _close(dw[:, cols], ref[:, cols], (n + 8) * U32 * (dy.double().abs().cpu().t() @ x[:, cols].double().abs().cpu()), dtype)
    cols = [j for j in range(k) if j != 1]
    ref = dy.double().cpu() @ w.double().cpu()
    assert torch.equal(torch.isinf(dx[:, 1].cpu()), torch.isinf(ref[:, 1]))
    _close(dx[:, cols], ref[:, cols], (m + 8) * U32 * (dy.double().abs().cpu() @ w[:, cols].double().abs().cpu()), dtype)


@pytest.mark.parametrize("d", [40, 300, 1100])
@pytest.mark.parametrize("dtype", [F32, F16], ids=str)
def test_block_gradient_of_lists_of_several_pieces(h, d, dtype):
    """Lists of 30 to 3000 entries side by side, three times on the same scratch: the pieces are added in the same order every time."""
    n, n_src = 3000, 60
    rng = np.random.default_rng(d)
    lens = np.array([0, 1, 31, 32, 33, 64, 255, 256, 257, 511, 513, 1024, 1500, 2047, 3000] * 4)
    rows = [np.sort(rng.choice(n, k, replace=False)) for k in lens]
    src = np.concatenate([np.full(k, u) for u, k in enumerate(lens)])
    dst = np.concatenate(rows)
    order = np.argsort(dst, kind="stable")
    col = torch.from_numpy(src[order].astype(np.int32))
    indptr = torch.zeros(n + 1, dtype=torch.int64)
    indptr[1:] = torch.from_numpy(np.bincount(dst, minlength=n)).cumsum(0)
    dmean = _rand(n, d, 4).to(dtype).cuda()
    si, se = torch.empty(n_src + 1, dtype=torch.int32, device="cuda"), torch.empty(col.numel(), dtype=torch.int32, device="cuda")
    h.block_transpose(indptr.cuda(), col.cuda(), n_src, si, se)
    dx = [torch.full((n_src, d), -7.0, dtype=dtype, device="cuda") for _ in range(3)]
    for t in dx:
        h.block_mean_grad(indptr.cuda(), si, se, dmean, t)
    h.sync()
    assert se.tolist() == dst.tolist()                    # every source's rows, ascending
    m = _dense(indptr, col, n, n_src)
    want, size = m.t() @ dmean.double().cpu(), m.t() @ dmean.double().abs().cpu()
    _close(dx[0], want, 3100 * U32 * size, dtype)
    assert all(torch.equal(t, dx[0]) for t in dx)


@pytest.mark.parametrize("n,n_src,skew", [(9000, 5000, 1), (9000, 70_000, 4), (30_000, 2_000_000, 1), (6000, 40, 1), (200, 300_000, 1)])
def test_block_by_source_at_other_sizes(h, n, n_src, skew):
    """Both ways of sorting the entries, few and many of them for a range of sources: exactly the lists in order."""
    rng = np.random.default_rng(n)
    deg = rng.integers(0, 9, n)
    indptr = np.zeros(n + 1, np.int64)
    indptr[1:] = np.cumsum(deg)
    col = (n_src * rng.random(indptr[-1]) ** skew).astype(np.int32)
    row = rng.integers(0, n_src, n).astype(np.int32)
    for own in (False, True):
        si = torch.full((n_src + 1,), -7, dtype=torch.int32, device="cuda")
        se = torch.full((col.size + (n if own else 0),), -7, dtype=torch.int32, device="cuda")
        h.block_transpose(torch.from_numpy(indptr).cuda(), torch.from_numpy(col).cuda(), n_src, si, se, row=torch.from_numpy(row).cuda() if own else None)
        h.sync()
        source = np.concatenate([col, row]) if own else col
        entry = np.concatenate([np.repeat(np.arange(n), deg), ~np.arange(n)]) if own else np.repeat(np.arange(n), deg)
        order = np.argsort(source, kind="stable")
        assert np.array_equal(se.cpu().numpy(), entry[order].astype(np.int32))
        assert np.array_equal(si.cpu().numpy(), np.searchsorted(source[order], np.arange(n_src + 1)).astype(np.int32))
