"""Dropout and the join of a layer's output with what went around it, against plain 64-bit forms.

Which elements are dropped is worked out here from the generator's definition, and is the same to the element.  Bounds are
worked out from the formulas, per element, with U = 2^-24 for every 32-bit step.  A sum over a row is a chain of at most 32 products in a lane,
six or seven steps of a tree and 16 waves: at most 64 U of its magnitudes.  So a reciprocal root is good to 40 U, and what follows from it to a few
U more.  A result is rounded once to its type."""
import os

import numpy as np
import pytest
import torch

from test_gpu_layer import BF16, E4M3, EPS, F16, F32, ROUND, U32, _close, _on_gpu, _out, _rand, _untouched

gpu = pytest.mark.gpu
TAG = 0x44524F50


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


def _philox(counter, key):
    """Philox4x32-10 on four arrays of 32-bit words."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k = list(key)
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def _threshold(p):
    return int(p * 65536 + 0.5)


def _kept(n, d, p, seed, site):
    row, block = np.meshgrid(np.arange(n), np.arange((d + 7) // 8), indexing="ij")
    words = _philox([row, block, np.full_like(row, site), np.full_like(row, TAG)], [seed & 0xFFFFFFFF, seed >> 32])
    draws = np.stack([(words[e // 2] >> np.uint64(16 * (e % 2))) & np.uint64(0xFFFF) for e in range(8)], 2)
    return torch.from_numpy(draws.reshape(n, -1)[:, :d] >= _threshold(p))


def _factor(p):
    t = _threshold(p)
    return 65536 / (65536 - t) if t < 65536 else 0.0


def test_the_generator_of_these_tests():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")
    rows = [[int(w, 16) for w in line.split()] for line in open(path) if line.strip() and not line.startswith("#")]
    assert len(rows) == 3
    for r in rows:
        assert [int(v[0]) for v in _philox([[v] for v in r[:4]], r[4:6])] == r[6:]


# ------------------------------------------------------------------ dropout


@gpu
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("n,d", [(1, 1), (1, 8), (3, 7), (5, 9), (64, 64), (33, 100), (777, 256), (2, 5000), (1, 70_000), (3000, 3)])
def test_dropout(h, n, d, dtype):
    seed = 0x9876543210ABCDEF + n + d
    x = _on_gpu(_rand(n, d, n + d), dtype, d % 4, n % 3)
    for p, site in ((0.0, 0), (0.1, 5), (0.5, 0xFFFFFFFF), (0.9, 1), (1.0, 2)):
        y = _out(n, d, dtype, 3, d % 2)
        h.dropout(x, y, p, seed % 2 ** 64, site=site)
        h.sync()
        kept = _kept(n, d, p, seed % 2 ** 64, site)
        want = torch.where(kept, x.float().cpu() * np.float32(_factor(p)), 0.0).to(dtype)          # (the same two roundings)
        assert torch.equal(y.cpu(), want) and _untouched(y), (p, site)
        again = x.clone()
        h.dropout(again, again, p, seed % 2 ** 64, site=site)
        h.sync()
        assert torch.equal(again.cpu(), want)


@gpu
def test_dropout_drops_its_share(h):
    """Of 2^22 elements a share of p, to five standard deviations, and neighbours independently; another site, seed or row drops others."""
    n, d = 4096, 1024
    x, y = torch.ones((n, d), device="cuda"), torch.empty((n, d), device="cuda")
    for p in (0.1, 0.5, 2.0 ** -16):
        h.dropout(x, y, p, 12345)
        h.sync()
        gone = (y == 0).double().cpu()
        q = _threshold(p) / 65536
        assert abs(float(gone.mean()) - q) < 5 * (q * (1 - q) / (n * d)) ** 0.5
        for a, b in ((gone[:, 1:], gone[:, :-1]), (gone[1:], gone[:-1]), (gone[:, 8:], gone[:, :-8])):
            assert abs(float((a * b).mean()) - q * q) < 5 * (q * q * (1 - q * q) / a.numel()) ** 0.5 + 1e-6
    masks = []
    for seed, site in ((12345, 0), (12345, 1), (12346, 0), (12345 + 2 ** 32, 0)):
        h.dropout(x, y, 0.5, seed, site=site)
        h.sync()
        masks.append((y == 0).cpu())
    for i in range(4):
        for j in range(i):
            assert abs(float((masks[i] == masks[j]).double().mean()) - 0.5) < 5 * (0.25 / (n * d)) ** 0.5


@gpu
def test_dropout_with_the_count_and_the_seed_on_the_device(h):
    n, d, live = 50, 72, 33
    x = _rand(n, d, 1).float().cuda()
    x[live:] = float("nan")
    y = torch.full((n, d), -7.0, device="cuda")
    count = torch.tensor([live], dtype=torch.int64, device="cuda")
    for seed in (5, -1, 2 ** 62):                              # (the tensor holds the 64 bits of the seed)
        for where in (torch.tensor([seed], dtype=torch.int64, device="cuda"), torch.tensor([seed], dtype=torch.int64).pin_memory()):
            h.dropout(x, y, 0.5, where, site=9, n_rows_dev=count)
            h.sync()
            want = torch.where(_kept(live, d, 0.5, seed % 2 ** 64, 9), x[:live].cpu() * 2, 0.0)
            assert torch.equal(y[:live].cpu(), want) and bool((y[live:] == -7.0).all())
    h.dropout(x, y, 0.5, 5, n_rows_dev=torch.zeros(1, dtype=torch.int64, device="cuda"))
    h.dropout(x[:0], y[:0], 0.5, 5)
    h.sync()
    assert bool((y[live:] == -7.0).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
def test_dropped_infinities_and_nan_are_zeros(h, dtype):
    kept = _kept(4, 64, 0.5, 77, 0)
    x = torch.where(kept, 1.0, float("nan")).to(dtype).cuda()
    x[1][~kept[1].cuda()] = float("inf")
    y = torch.empty_like(x)
    h.dropout(x, y, 0.5, 77)
    h.sync()
    assert torch.equal(y.cpu(), torch.where(kept, 2.0, 0.0).to(dtype))
    x = torch.where(kept, float("nan"), 1.0).to(dtype).cuda()          # what is kept stays what it is
    h.dropout(x, y, 0.5, 77)
    h.sync()
    assert torch.equal(torch.isnan(y.cpu()), kept)
    # ... and they take no part in a join
    x = torch.where(kept, 1.0, float("inf")).to(dtype).cuda()
    total, one = torch.empty_like(x), torch.ones(64, dtype=dtype, device="cuda")
    h.join_norm(x, EPS, total=total, norm_x=False, p=0.5, seed=77, gate=one)
    dx, dgate = torch.empty_like(x), torch.empty_like(one)
    h.join_norm_grad(x, dx, EPS, dtotal=torch.ones_like(x), norm_x=False, p=0.5, seed=77, gate=one, dgate=dgate)
    h.sync()
    assert torch.equal(total.cpu(), torch.where(kept, 2.0, 0.0).to(dtype)) and torch.equal(dx.cpu(), torch.where(kept, 2.0, 0.0).to(dtype))
    assert torch.equal(dgate.cpu(), (2.0 * kept.sum(0)).to(dtype))


# ------------------------------------------------------------------ join


def _inputs(n, d, dtype, gate, seed, pads=(0, 0)):
    """What a case has, on the GPU (g) and in 64 bits (w)."""
    pad, at = pads
    g = {"x": _on_gpu(_rand(n, d, seed, 2.0), dtype, pad, at), "residual": _on_gpu(_rand(n, d, seed + 1, 3.0), dtype, at, pad),
         "gain_x": (_rand(1, d, seed + 2, 0.3)[0] + 1).to(dtype).cuda(), "gain": (_rand(1, d, seed + 3, 0.3)[0] + 1).to(dtype).cuda(),
         "gate": {"none": None, "row": _rand(1, d, seed + 4)[0].to(dtype).cuda(), "rows": _on_gpu(_rand(n, d, seed + 5), dtype, 2 * pad, at)}[gate],
         "dy": _on_gpu(_rand(n, d, seed + 6), dtype, pad, at), "dtotal": _on_gpu(_rand(n, d, seed + 7), dtype, at, at)}
    return g, {k: None if v is None else v.double().cpu() for k, v in g.items()}


def _root(t):
    return 1.0 / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)


def _forward(w, norm_x, gate, residual, scale, factor):
    """(total, its bound, y, its bound) in 64 bits; factor: of every element, 0 where it is dropped."""
    x = w["x"]
    q = _root(x) if norm_x else torch.ones(x.shape[0], 1, dtype=torch.float64)
    v = x * factor * (q * w["gain_x"] if norm_x else 1.0) * (w["gate"] if gate != "none" else 1.0)
    r = scale * w["residual"] if residual else torch.zeros_like(x)
    total = v + r
    off = (44 if norm_x else 4) * U32 * v.abs() + 3 * U32 * r.abs() + U32 * total.abs()
    q = _root(total)
    mean_off = (2 * total.abs() * off + off * off).mean(1, keepdim=True)            # of the mean of squares
    rel = 44 * U32 + 0.5 * mean_off * q * q
    y = total * q * w["gain"]
    return total, off, y, y.abs() * rel + q * w["gain"].abs() * off


WIDTHS = [1, 3, 8, 100, 128, 130, 256, 512, 520, 1000, 1024, 1030, 2048, 2050, 4100, 8192, 8200, 20_001, 32_768]


def _join_case(h, n, d, dtype, out, gate, norm_x, residual, p, seed, pads=(0, 0), count=None):
    g, w = _inputs(n, d, dtype, gate, seed, pads)
    live = n if count is None else count
    n_dev = None
    if count is not None:
        n_dev = torch.tensor([count], dtype=torch.int64, device="cuda")
        g["x"][count:] = float("nan")
    kept = _kept(n, d, p, seed, 3)
    total, y = _out(n, d, dtype, 1, pads[1]), _out(n, d, out, pads[0])
    y_scale = torch.full((n,), -7.0, device="cuda") if out == E4M3 else None
    root_x, root = (torch.full((n,), -7.0, device="cuda") for _ in range(2))
    h.join_norm(g["x"], EPS, y=y, total=total, norm_x=norm_x, gain_x=g["gain_x"] if norm_x else None, p=p, seed=seed, site=3, gate=g["gate"],
                residual=g["residual"] if residual else None, residual_scale=0.625, gain=g["gain"], y_scale=y_scale, inv_rms_x=root_x if norm_x else None,
                inv_rms=root, n_rows_dev=n_dev)
    h.sync()
    w = {k: v[:live] if v is not None and v.dim() == 2 else v for k, v in w.items()}
    t, t_off, want, off = _forward(w, norm_x, gate, residual, 0.625, torch.where(kept[:live], _factor(p), 0.0).double())
    _close(total[:live], t, t_off, dtype, "total")
    if norm_x:
        _close(root_x[:live, None], _root(w["x"]), 40 * U32 * _root(w["x"]), F32, "inv_rms_x")
    q = _root(t)
    _close(root[:live, None], q, q * (44 * U32 + 0.5 * (2 * t.abs() * t_off + t_off ** 2).mean(1, keepdim=True) * q * q), F32, "inv_rms")
    if out == E4M3:
        s = y_scale.double().cpu()[:live, None]
        most = (want.abs() / 448).amax(1, keepdim=True).clamp_min(2.0 ** -126)
        assert bool(((s - most).abs() <= (off / 448).amax(1, keepdim=True) + 2 * U32 * most).all())
        got = y.double().cpu()[:live] * s
        assert bool(((got - want).abs() <= off + ROUND[E4M3] * (1 + 1e-5) * (want.abs() + off) + s * 2.0 ** -10).all())
    else:
        _close(y[:live], want, off, dtype, "y")
    for o in [total, y]:
        assert _untouched(o) and bool((o[live:].float() == -7.0).all())
    for o in [root, root_x, y_scale]:
        assert o is None or bool((o[live:] == -7.0).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("d", WIDTHS)
def test_join(h, d, dtype):
    print("join", d, dtype, flush=True)
    n = 5 if d > 2000 else 37
    _join_case(h, n, d, dtype, dtype, "row", True, True, 0.1, d)
    _join_case(h, n, d, dtype, dtype, "rows", True, True, 0.5, d + 10, pads=(3, 1))
    _join_case(h, n, d, dtype, E4M3, "none", False, True, 0.0, d + 20, pads=(8, 0))
    _join_case(h, 1, d, dtype, E4M3, "row", True, False, 0.0, d + 30)
    _join_case(h, n, d, dtype, dtype, "rows", False, False, 0.3, d + 40, pads=(1, 2), count=n - 2)


@gpu
@pytest.mark.parametrize("dtype", [F32, F16], ids=str)
def test_join_of_many_rows_and_a_count_on_the_device(h, dtype):
    _join_case(h, 9000, 136, dtype, dtype, "row", True, True, 0.1, 1, count=8999)
    _join_case(h, 300, 72, dtype, E4M3, "rows", True, True, 0.5, 2, count=0)
    _join_case(h, 5000, 16, dtype, dtype, "none", True, True, 0.0, 3)


@gpu
def test_join_of_one_output_and_in_place(h):
    n, d = 20, 200
    g, w = _inputs(n, d, F32, "row", 4)
    want = [torch.empty((n, d), device="cuda") for _ in range(2)]
    args = dict(gain_x=g["gain_x"], p=0.25, seed=11, gate=g["gate"], residual_scale=0.5)
    h.join_norm(g["x"], EPS, y=want[0], total=want[1], residual=g["residual"], gain=g["gain"], **args)
    only_y, only_total = torch.empty((n, d), device="cuda"), torch.empty((n, d), device="cuda")
    h.join_norm(g["x"], EPS, y=only_y, residual=g["residual"], gain=g["gain"], **args)
    h.join_norm(g["x"], EPS, total=only_total, residual=g["residual"], **args)
    h.sync()
    assert torch.equal(only_y, want[0]) and torch.equal(only_total, want[1])
    for y_in, total_in in (("x", "residual"), ("residual", "x")):
        c = {k: g[k].clone() for k in ("x", "residual")}
        h.join_norm(c["x"], EPS, y=c[y_in], total=c[total_in], residual=c["residual"], gain=g["gain"], **args)
        h.sync()
        assert torch.equal(c[y_in], want[0]) and torch.equal(c[total_in], want[1])
    # without a layer's norm, dropout, gate and scale it is the norm with a residual (the mean by a reciprocal: 2 U, its root 1, a root to two units in the last
    # place 4, two products 2; the other call as much: 16 U)
    y, t, y2, t2 = (torch.empty((n, d), device="cuda") for _ in range(4))
    h.join_norm(g["x"], EPS, y=y, total=t, norm_x=False, residual=g["residual"], gain=g["gain"])
    h.rms_norm(g["x"], y2, EPS, gain=g["gain"], residual=g["residual"], total=t2)
    h.sync()
    assert bool(((y - y2).abs() <= 16 * U32 * y2.abs()).all()) and torch.equal(t, t2)


@gpu
@pytest.mark.parametrize("d", [64, 600, 9000])
def test_join_of_rows_of_zeros_and_rows_that_are_not_finite(h, d):
    """A row of zeros stays one; a row with an infinity or NaN spoils itself and no other."""
    n = 6
    x, r = _rand(n, d, 1).float().cuda(), _rand(n, d, 2).float().cuda()
    x[0], r[0] = 0, 0
    x[2, d // 2], r[3, 5], x[4] = float("nan"), float("inf"), 3e38
    y, t = torch.full((n, d), -7.0, device="cuda"), torch.full((n, d), -7.0, device="cuda")
    h.join_norm(x, EPS, y=y, total=t, residual=r)
    dx, dr = torch.full((n, d), -7.0, device="cuda"), torch.full((n, d), -7.0, device="cuda")
    h.join_norm_grad(x, dx, EPS, total=t, dy=torch.ones_like(x), dtotal=torch.ones_like(x), dresidual=dr)
    h.sync()
    assert bool((y[0] == 0).all()) and bool((t[0] == 0).all())
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(t[2]).all()) and bool(torch.isnan(dx[2]).all())
    assert bool(torch.isinf(t[3, 5])) and bool(torch.isnan(y[3, 5])) and bool((y[3, :5] == 0).all())
    for row in (1, 5):
        for o in (y, t, dx, dr):
            assert bool(torch.isfinite(o[row]).all())
    assert bool(torch.isfinite(dx[0]).all())


# ------------------------------------------------------------------ gradient of the join


def _backward(w, norm_x, gate, scale, factor, has_dy, has_dtotal):
    """{name: (gradient, its bound)} in 64 bits."""
    n, d = w["x"].shape
    x, t = w["x"], w["total"]
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    dt, size = torch.zeros_like(x), torch.zeros_like(x)
    out = {}
    if has_dy:
        q, a = _root(t), w["dy"] * w["gain"]
        dt = q * (a - t * q * q * mean(a * t))
        size = q * (a.abs() + t.abs() * q * q * mean((a * t).abs()))
        terms = w["dy"] * t * q
        out["dgain"] = (terms.sum(0), (n + 64 + 44) * U32 * terms.abs().sum(0))
    if has_dtotal:
        dt, size = dt + w["dtotal"], size + w["dtotal"].abs()
    off = 200 * U32 * size                                # the root 40, its square 80, the sum over the row 64, and the steps between
    out["dresidual"] = (scale * dt, abs(scale) * (off + 2 * U32 * dt.abs()))
    qx = _root(x) if norm_x else torch.ones(n, 1, dtype=torch.float64)
    gain_x = w["gain_x"] if norm_x else 1.0
    gates = w["gate"] if gate != "none" else 1.0
    slope = dt * factor * x * qx * gain_x
    slope_off = (off + 48 * U32 * dt.abs()) * (factor * x * qx * gain_x).abs()
    if gate == "rows":
        out["dgate"] = (slope, slope_off)
    elif gate == "row":
        out["dgate"] = (slope.sum(0), slope_off.sum(0) + (n + 64) * U32 * slope.abs().sum(0))
    dw = dt * factor * gates
    dw_off = (off + 4 * U32 * dt.abs()) * (factor * gates).abs()
    dx, dx_off = dw, dw_off
    if norm_x:
        terms = dw * x * qx
        out["dgain_x"] = (terms.sum(0), (dw_off * (x * qx).abs()).sum(0) + (n + 64 + 48) * U32 * terms.abs().sum(0))
        v, v_off = dw * gain_x, dw_off * gain_x.abs()
        dx = qx * (v - x * qx * qx * mean(v * x))
        dx_off = qx * (v_off + x.abs() * qx * qx * mean(v_off * x.abs())) + 200 * U32 * qx * (v.abs() + x.abs() * qx * qx * mean((v * x).abs()))
    out["dx"] = (dx, dx_off)
    return out


def _join_grad_case(h, n, d, dtype, gate, norm_x, p, seed, has_dy=True, has_dtotal=True, pads=(0, 0), count=None, roots=False, asked=None):
    g, w = _inputs(n, d, dtype, gate, seed, pads)
    g["total"] = _on_gpu(_rand(n, d, seed + 8, 3.0), dtype, pads[1], pads[0])
    w["total"] = g["total"].double().cpu()
    live = n if count is None else count
    n_dev = None
    if count is not None:
        n_dev = torch.tensor([count], dtype=torch.int64, device="cuda")
        for k in ("x", "dy", "total"):
            g[k][count:] = float("nan")
    vec = lambda: torch.full((d,), -7.0, dtype=dtype, device="cuda")  # noqa: E731
    outs = {"dx": _out(n, d, dtype, pads[0]), "dresidual": _out(n, d, dtype, 1, pads[1])}
    if gate != "none":
        outs["dgate"] = vec() if gate == "row" else _out(n, d, dtype, pads[1])
    if norm_x:
        outs["dgain_x"] = vec()
    if has_dy:
        outs["dgain"] = vec()
    if asked is not None:
        outs = {k: v for k, v in outs.items() if k == "dx" or k in asked}
    given = {}
    if roots:
        if norm_x:
            given["inv_rms_x"] = _root(w["x"])[:, 0].float().cuda()
        given["inv_rms"] = _root(w["total"])[:, 0].float().cuda()
    h.join_norm_grad(g["x"], outs["dx"], EPS, total=g["total"] if has_dy else None, dy=g["dy"] if has_dy else None, dtotal=g["dtotal"] if has_dtotal else None,
                     norm_x=norm_x, gain_x=g["gain_x"] if norm_x else None, p=p, seed=seed, site=3, gate=g["gate"], residual_scale=-0.625,
                     gain=g["gain"] if has_dy else None, **{k: v for k, v in outs.items() if k != "dx"}, **given, n_rows_dev=n_dev)
    h.sync()
    kept = _kept(n, d, p, seed, 3)
    w = {k: v[:live] if v is not None and v.dim() == 2 else v for k, v in w.items()}
    want = _backward(w, norm_x, gate, -0.625, torch.where(kept[:live], _factor(p), 0.0).double(), has_dy, has_dtotal)
    for name, got in outs.items():
        ref, off = want[name]
        if got.dim() == 2:
            _close(got[:live], ref, off, dtype, name)
            assert _untouched(got) and bool((got[live:].float() == -7.0).all()), name
        else:
            _close(got, ref, off, dtype, name)


@gpu
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("d", WIDTHS)
def test_join_grad(h, d, dtype):
    print("join grad", d, dtype, flush=True)
    n = 5 if d > 2000 else 37
    _join_grad_case(h, n, d, dtype, "row", True, 0.1, d)
    _join_grad_case(h, n, d, dtype, "rows", True, 0.5, d + 10, pads=(3, 1))
    _join_grad_case(h, n, d, dtype, "none", False, 0.0, d + 20, has_dtotal=False, pads=(8, 0), roots=True)
    _join_grad_case(h, 1, d, dtype, "row", True, 0.3, d + 30, has_dy=False, roots=False)
    _join_grad_case(h, n, d, dtype, "rows", False, 0.3, d + 40, pads=(1, 2), count=n - 2)
    _join_grad_case(h, n, d, dtype, "row", True, 0.0, d + 50, roots=True, asked=())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("n,d", [(9000, 136), (3001, 24), (1500, 1030), (1100, 2050), (300, 9000)])
def test_join_grad_of_many_rows_and_a_count_on_the_device(h, n, d, dtype):
    _join_grad_case(h, n, d, dtype, "row", True, 0.1, n)
    _join_grad_case(h, n, d, dtype, "row", True, 0.1, n + 1, count=n // 2, asked=("dgate", "dgain"))
    _join_grad_case(h, n, d, dtype, "row", True, 0.1, n + 2, count=0)


@gpu
def test_join_grad_over_its_own_inputs_and_of_no_rows(h):
    n, d = 33, 300
    for wide in (False, True):
        d = 9000 if wide else 300
        g, _ = _inputs(n, d, F16, "row", 5)
        g["total"] = _rand(n, d, 6).half().cuda()
        args = lambda c: dict(gain_x=g["gain_x"], p=0.25, seed=3, gate=g["gate"], residual_scale=0.5, gain=g["gain"], total=c["total"], dy=c["dy"], dtotal=c["dtotal"])  # noqa: E731
        dx, dr = torch.empty((n, d), dtype=F16, device="cuda"), torch.empty((n, d), dtype=F16, device="cuda")
        h.join_norm_grad(g["x"], dx, EPS, dresidual=dr, **args(g))
        for a, b in (("x", "dtotal"), ("dtotal", "dy"), ("total", "dtotal"), ("dy", "total")):
            c = {k: g[k].clone() for k in ("x", "dy", "total", "dtotal")}
            h.join_norm_grad(c["x"], c[a], EPS, dresidual=c[b], **args(c))
            h.sync()
            assert torch.equal(c[a], dx) and torch.equal(c[b], dr), (a, b)
    none = torch.empty((0, 24), device="cuda")
    sums = [torch.full((24,), -7.0, device="cuda") for _ in range(3)]
    h.join_norm_grad(none, none, EPS, total=none, dy=none, gate=torch.ones(24, device="cuda"), dgate=sums[0], dgain_x=sums[1], dgain=sums[2])
    h.join_norm(none, EPS, y=none)
    h.sync()
    assert all(bool((s == 0).all()) for s in sums)


@gpu
@pytest.mark.parametrize("gate", ["none", "row", "rows"])
def test_join_grad_against_differences(h, gate):
    """Central differences in 64 bits of the forward formula (h = 1e-5: off by some 1e-9), for every input element."""
    n, d, p, seed, e = 3, 10, 0.3, 21, 1e-5
    g, w = _inputs(n, d, F32, gate, seed)
    factor = torch.where(_kept(n, d, p, seed, 3), _factor(p), 0.0).double()

    def loss(v):
        total, _, y, _ = _forward(v, True, gate, True, 0.625, factor)
        return float((total * w["dtotal"]).sum() + (y * w["dy"]).sum())

    total = torch.empty((n, d), device="cuda")
    args = dict(gain_x=g["gain_x"], p=p, seed=seed, site=3, gate=g["gate"], residual_scale=0.625)
    h.join_norm(g["x"], EPS, total=total, residual=g["residual"], **args)
    outs = {"dx": torch.empty((n, d), device="cuda"), "dresidual": torch.empty((n, d), device="cuda"), "dgain_x": torch.empty(d, device="cuda"), "dgain": torch.empty(d, device="cuda")}
    if gate != "none":
        outs["dgate"] = torch.empty(g["gate"].shape, device="cuda")
    h.join_norm_grad(g["x"], outs["dx"], EPS, total=total, dy=g["dy"], dtotal=g["dtotal"], gain=g["gain"], **{k: v for k, v in outs.items() if k != "dx"}, **args)
    h.sync()
    for name, out in outs.items():
        of, got = name[1:], out.double().cpu().view(-1)
        for i in range(got.numel()):
            sides = []
            for step in (e, -e):
                moved = {k: None if v is None else v.clone() for k, v in w.items()}
                moved[of].view(-1)[i] += step
                sides.append(loss(moved))
            assert abs(float(got[i]) - (sides[0] - sides[1]) / (2 * e)) < 2e-5 * max(1.0, abs(float(got[i]))), (name, i)


# ------------------------------------------------------------------ the calls as calls


@gpu
def test_the_same_bits_on_another_stream_and_in_a_graph_with_other_seeds(helios):
    """A recorded forward and backward pass whose seed lies in memory: every replay drops what an eager call with that seed drops."""
    n, d = 3000, 200
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        g, _ = _inputs(n, d, BF16, "row", 8)
        seed = torch.tensor([1], dtype=torch.int64, device="cuda")
        new = lambda *s: torch.zeros(s, dtype=BF16, device="cuda")  # noqa: E731
        a, total, y, dx, dr, da = (new(n, d) for _ in range(6))
        sums = [new(d) for _ in range(3)]
        outs = [a, total, y, dx, dr, da] + sums

        def step(s):
            h.dropout(g["x"], a, 0.2, s, site=1)
            args = dict(gain_x=g["gain_x"], p=0.1, seed=s, site=2, gate=g["gate"], residual_scale=0.5)
            h.join_norm(a, EPS, y=y, total=total, residual=g["residual"], gain=g["gain"], **args)
            h.join_norm_grad(a, dx, EPS, total=total, dy=g["dy"], dtotal=g["dtotal"], gain=g["gain"], dresidual=dr, dgate=sums[0], dgain_x=sums[1], dgain=sums[2], **args)
            h.dropout(dx, da, 0.2, s, site=1)

        torch.cuda.synchronize()
        step(1)
        h.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(seed)
        for turn, value in enumerate((1, 7, 2 ** 40, 7)):
            print("graph replay", turn, flush=True)
            step(value)
            h.sync()
            want = [t.clone() for t in outs]
            for t in outs:
                t.zero_()
            seed.fill_(value)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            h.sync()
            assert all(torch.equal(p.view(torch.int16), q.view(torch.int16)) for p, q in zip(outs, want)), turn
    finally:
        h.close()


@gpu
def test_a_capture_that_would_have_to_allocate_is_refused(helios):
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        x, dx, dg = torch.zeros((64, 32), device="cuda"), torch.zeros((64, 32), device="cuda"), torch.zeros(32, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(helios.HeliosError) as e:
                h.join_norm_grad(x, dx, EPS, total=x, dy=x, dgain=dg)
        assert e.value.code == helios.ESTATE and "capture" in str(e.value)
        h.join_norm_grad(x, dx, EPS, total=x, dy=x, dgain=dg)
        h.sync()
    finally:
        h.close()


@gpu
@pytest.mark.parametrize("d", [16, 13])
def test_a_distance_between_rows_of_a_gate_that_is_not_there(helios, h, d):
    """It is not looked at: the gate is ones."""
    x, dy = _rand(8, d, 1).float().cuda(), _rand(8, d, 2).float().cuda()
    want, got, dx, got_dx = (torch.empty_like(x) for _ in range(4))
    h.join_norm(x, EPS, y=want)
    h.join_norm_grad(x, dx, EPS, dtotal=dy)
    p, q = x.data_ptr(), dy.data_ptr()
    args = dict(n_rows=8, width=d, norm_x=1, eps=EPS, residual_scale=1.0, x=p, x_ld=d, gate_ld=d)
    assert helios._lib.helios_join_norm(h._h, helios.JoinNormArgs(y=got.data_ptr(), y_ld=d, **args)) == helios.OK
    assert helios._lib.helios_join_norm_grad(h._h, helios.JoinNormGradArgs(dtotal=q, dtotal_ld=d, dx=got_dx.data_ptr(), dx_ld=d, **args)) == helios.OK
    dgate, dgain_x = (torch.full((d,), -7.0, device="cuda") for _ in range(2))
    args = dict(args, n_rows=0, dgate=dgate.data_ptr(), dgate_ld=d, dgain_x=dgain_x.data_ptr())
    assert helios._lib.helios_join_norm_grad(h._h, helios.JoinNormGradArgs(**args)) == helios.OK
    h.sync()
    assert torch.equal(got, want) and torch.equal(got_dx, dx)
    assert bool((dgate == -7.0).all()) and bool((dgain_x == 0).all())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_large_calls_give_the_bits_of_small_ones(h, dtype):
    """Calls of more than 128 MB, which may go past the caches, and their first rows by themselves."""
    d, few = 512, 100
    n = (150 << 20) // (2 * d * torch.empty(0, dtype=dtype).element_size())
    x, dy, dtotal, residual, gate = (torch.randn((n, d), device="cuda").to(dtype) for _ in range(5))
    gain_x, gain, one_gate = (torch.randn(d, device="cuda").to(dtype) for _ in range(3))

    def run(m, with_gates):
        out = {k: torch.full((m, d), -7.0, dtype=dtype, device="cuda") for k in ("dropout", "total", "y", "dx", "dresidual")}
        out["dgate"] = torch.empty((m, d) if with_gates else d, dtype=dtype, device="cuda")
        out["dgain"] = torch.empty(d, dtype=dtype, device="cuda")
        out["y8"], out["y_scale"] = torch.empty((m, d), dtype=E4M3, device="cuda"), torch.empty(m, device="cuda")
        g = gate[:m] if with_gates else one_gate
        h.dropout(x[:m], out["dropout"], 0.1, 5, 1)
        h.join_norm(x[:m], EPS, y=out["y"], total=out["total"], gain_x=gain_x, p=0.1, seed=5, gate=g, residual=residual[:m], gain=gain)
        h.join_norm(x[:m], EPS, y=out["y8"], y_scale=out["y_scale"], gain_x=gain_x, p=0.1, seed=5, gate=g, residual=residual[:m])
        h.join_norm_grad(x[:m], out["dx"], EPS, total=out["total"], dy=dy[:m], dtotal=dtotal[:m], gain_x=gain_x, p=0.1, seed=5, gate=g, gain=gain,
                         dresidual=out["dresidual"], dgate=out["dgate"], dgain=out["dgain"])
        h.sync()
        return out

    for with_gates in (False, True):
        large, small = run(n, with_gates), run(few, with_gates)
        for k in ("dropout", "total", "y", "y_scale", "dx", "dresidual") + (("dgate",) if with_gates else ()):
            assert torch.equal(large[k][:few], small[k]), k
            assert bool(torch.isfinite(large[k]).all()), k
        assert torch.equal(large["y8"].view(torch.uint8)[:few], small["y8"].view(torch.uint8))
        last = {k: v[-few:].float() for k, v in large.items() if v.dim() == 2}
        assert bool((last["dropout"] != -7.0).all()) and float((last["dropout"] == 0).float().mean()) < 0.2
        # the last rows, and a sum over all.  (y is made from the unrounded total, whose elements and root are each off by half a step of the type.)
        t = large["total"].double()
        q = _root(t)
        y = (t * q * gain.double())[-few:].cpu()
        _close(large["y"][-few:], y, (2.1 * ROUND[dtype] + 60 * U32) * y.abs(), dtype, "y")
        terms = dy.double() * t * q
        _close(large["dgain"], terms.sum(0).cpu(), ((n + 108) * U32 * terms.abs().sum(0)).cpu(), dtype, "dgain")


@gpu
def test_refusals(helios, h):
    x, z, one = torch.zeros((8, 16), device="cuda"), torch.zeros((8, 16), device="cuda"), torch.ones(16, device="cuda")

    def einval(call, *args, **kw):
        with pytest.raises(helios.HeliosError) as e:
            call(*args, **kw)
        assert e.value.code == helios.EINVAL
        return str(e.value)

    def typeerror(call, *args, **kw):
        with pytest.raises(TypeError):
            call(*args, **kw)

    for p in (-0.1, 1.1, float("nan"), float("inf")):
        assert "share" in einval(h.dropout, x, z, p, 1)
        assert "share" in einval(h.join_norm, x, EPS, y=z, p=p)
        assert "share" in einval(h.join_norm_grad, x, z, EPS, dtotal=x, p=p)
    typeerror(h.dropout, x, z.half(), 0.5, 1)
    typeerror(h.dropout, x, z, 0.5, torch.zeros(1, device="cuda"))
    typeerror(h.dropout, x, z, 0.5, torch.zeros(2, dtype=torch.int64, device="cuda"))
    typeerror(h.dropout, x, z, 0.5, torch.zeros(1, dtype=torch.int64))
    assert "x_type" in einval(h.dropout, x.to(E4M3), z.to(E4M3), 0.5, 1)
    assert "shares memory" in einval(h.dropout, x[1:], x[:-1], 0.5, 1)
    assert "shares memory" in einval(h.dropout, x, z, 0.5, z.view(torch.int64)[0, :1])
    assert "narrower" in einval(h.dropout, x, z[:1].expand(8, 16), 0.5, 1)
    wide = torch.zeros((1, 32_769), device="cuda")
    assert "width" in einval(h.join_norm, wide, EPS, y=torch.zeros_like(wide))
    assert "width" in einval(h.join_norm_grad, wide, torch.zeros_like(wide), EPS, dtotal=wide)
    assert "eps" in einval(h.join_norm, x, -1.0, y=z)
    assert "eps" in einval(h.join_norm_grad, x, z, float("nan"), dtotal=x)
    assert "NULL" in einval(h.join_norm, x, EPS)
    assert "y_type" in einval(h.join_norm, x, EPS, y=z.half())
    assert "y_scale" in einval(h.join_norm, x, EPS, y=z.to(E4M3))
    assert "y_scale" in einval(h.join_norm, x, EPS, y=z, y_scale=torch.zeros(8, device="cuda"))
    assert "norm_x" in einval(h.join_norm, x, EPS, y=z, norm_x=False, gain_x=one)
    assert "go with y" in einval(h.join_norm, x, EPS, total=z, gain=one)
    assert "shares memory" in einval(h.join_norm, x, EPS, y=z, total=z)
    assert "shares memory" in einval(h.join_norm, x, EPS, y=z, gate=z)
    assert "shares memory" in einval(h.join_norm, x, EPS, y=z, gain=z[0])
    typeerror(h.join_norm, x, EPS, y=z, gate=torch.ones(15, device="cuda"))
    typeerror(h.join_norm, x, EPS, y=z, gate=torch.ones((4, 16), device="cuda"))
    assert "NULL" in einval(h.join_norm_grad, x, z, EPS)
    assert "NULL" in einval(h.join_norm_grad, x, z, EPS, dy=x)
    assert "go with dy" in einval(h.join_norm_grad, x, z, EPS, dtotal=x, dgain=torch.zeros(16, device="cuda"))
    assert "gate" in einval(h.join_norm_grad, x, z, EPS, dtotal=x, dgate=torch.zeros(16, device="cuda"))
    assert "norm_x" in einval(h.join_norm_grad, x, z, EPS, dtotal=x, norm_x=False, dgain_x=torch.zeros(16, device="cuda"))
    assert "shares memory" in einval(h.join_norm_grad, x, z, EPS, dtotal=x, dresidual=z)
    assert "shares memory" in einval(h.join_norm_grad, x, z, EPS, dtotal=torch.ones_like(x), dresidual=x)
    assert "shares memory" in einval(h.join_norm_grad, x, z, EPS, dtotal=x, dgain_x=z[0])
    typeerror(h.join_norm_grad, x, z, EPS, dtotal=x, gate=one, dgate=torch.zeros((8, 16), device="cuda"))
    lib = helios._lib
    for call, args in (("dropout", helios.DropoutArgs), ("join_norm", helios.JoinNormArgs), ("join_norm_grad", helios.JoinNormGradArgs)):
        f = getattr(lib, "helios_" + call)
        assert f(None, None) == helios.EINVAL and f(h._h, None) == helios.EINVAL
        assert f(h._h, args(n_rows=-1, width=4)) == helios.EINVAL and f(h._h, args(n_rows=2 ** 31, width=4)) == helios.EINVAL
        assert f(h._h, args(n_rows=1, width=0)) == helios.EINVAL and f(h._h, args(n_rows=1, width=4)) == helios.EINVAL
        assert f(h._h, args(n_rows=0, width=4)) == helios.OK
    p, q = x.data_ptr(), z.data_ptr()
    assert lib.helios_dropout(h._h, helios.DropoutArgs(n_rows=1, width=4, x=p + 2, x_ld=4, y=q, y_ld=4)) == helios.EINVAL
    assert lib.helios_join_norm(h._h, helios.JoinNormArgs(n_rows=1, width=4, x=p, x_ld=4, y=q + 2, y_ld=4)) == helios.EINVAL
    assert lib.helios_join_norm_grad(h._h, helios.JoinNormGradArgs(n_rows=1, width=4, x=p, x_ld=4, dtotal=p + 2, dtotal_ld=4, dx=q, dx_ld=4)) == helios.EINVAL
    assert lib.helios_dropout(h._h, helios.DropoutArgs(n_rows=1 << 30, width=4, x=p, x_ld=1 << 40, y=q, y_ld=4)) == helios.EINVAL
    h.sync()
