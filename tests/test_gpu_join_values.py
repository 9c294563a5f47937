"""The join of a layer and its gradient where gates, gains and dropped elements are not finite.

The forms are those of test_gpu_join.py in 64 bits, with elements dropped by selection: what is dropped is 0 whatever it was."""
import pytest
import torch

from test_gpu_join import _factor, _kept, _root
from test_gpu_layer import BF16, E4M3, EPS, F16, F32, U32, _close, _rand

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
WIDTHS = [3, 24, 101, 512, 600, 1032, 4104, 8200]          # rows by 16 lanes (short ones among them), a wave, several waves; more than are kept in registers


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


def _same_kind(got, want, bound, dtype, what):
    """NaN where NaN belongs, the right infinity where one does, and what is finite within its bound."""
    got, finite = got.double().cpu(), torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), what
    _close(torch.where(finite, got, 0.0), torch.where(finite, want, 0.0), torch.where(finite, bound, 0.0), dtype, what)


def _gates(d, dtype):
    """A gate of one row with an infinity of each sign and NaN among its columns, the last one too."""
    gate = _rand(1, d, 4)[0]
    gate[d // 3], gate[d // 2], gate[d - 1] = INF, NAN, -INF
    return gate.to(dtype)


@pytest.mark.parametrize("norm_x", [False, True])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("d", WIDTHS)
def test_join_with_a_gate_that_is_not_finite(h, d, dtype, norm_x):
    """total = residual_scale * residual + gate * drop(u): a dropped element's product with an infinite gate is NaN, whether the gate is one row or a
    row for each; the other columns are what they are."""
    n, p, seed = 5, 0.4, d
    x, r, gain_x, gate = _rand(n, d, 1).to(dtype), _rand(n, d, 2).to(dtype), (_rand(1, d, 3, 0.3)[0] + 1).to(dtype), _gates(d, dtype)
    kept = _kept(n, d, p, seed, 3)
    x64, q = x.double(), _root(x.double()) if norm_x else torch.ones(n, 1, dtype=torch.float64)
    u = x64 * q * (gain_x.double() if norm_x else 1.0)
    moved = gate.double() * torch.where(kept, u * _factor(p), 0.0)
    want = moved + 0.5 * r.double()
    bound = 44 * U32 * moved.abs() + 3 * U32 * r.double().abs() + U32 * want.abs()
    for g in (gate.cuda(), gate[None].repeat(n, 1).cuda()):
        total, y = (torch.full((n, d), -7.0, dtype=dtype, device="cuda") for _ in range(2))
        h.join_norm(x.cuda(), EPS, y=y, total=total, norm_x=norm_x, gain_x=gain_x.cuda() if norm_x else None, p=p, seed=seed, site=3, gate=g, residual=r.cuda(),
                    residual_scale=0.5)
        h.sync()
        _same_kind(total, want, bound, dtype, "total")
        assert bool(torch.isnan(y).all())                      # (there is NaN in every row)


@pytest.mark.parametrize("norm_x", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("d", WIDTHS + [8193])
def test_join_grad_with_a_gate_that_is_not_finite(h, d, dtype, norm_x):
    """What is dropped adds nothing, whether the gate is one row or a row for each: columns of dgain_x in which all is dropped are 0 where every row has
    a gate of its own, and dx is 0 there; dgate, which the gate takes no part in, is finite everywhere."""
    n, p, seed = 6, 0.6, d
    x, dt, gain_x, gate = _rand(n, d, 1).to(dtype), _rand(n, d, 2).to(dtype), (_rand(1, d, 3, 0.3)[0] + 1).to(dtype), _gates(d, dtype)
    kept = _kept(n, d, p, seed, 3)
    x64, dt64 = x.double(), dt.double()
    q = _root(x64) if norm_x else torch.ones(n, 1, dtype=torch.float64)
    slope = torch.where(kept, dt64 * x64 * q * (gain_x.double() if norm_x else 1.0) * _factor(p), 0.0)
    w = torch.where(kept, dt64 * _factor(p) * gate.double(), 0.0)
    for rows in (False, True):
        g = (gate[None].repeat(n, 1) if rows else gate).cuda()
        dx, dgate = torch.full((n, d), -7.0, dtype=dtype, device="cuda"), torch.full(g.shape, -7.0, dtype=dtype, device="cuda")
        dgain_x = torch.full((d,), -7.0, dtype=dtype, device="cuda") if norm_x else None
        h.join_norm_grad(x.cuda(), dx, EPS, dtotal=dt.cuda(), norm_x=norm_x, gain_x=gain_x.cuda() if norm_x else None, p=p, seed=seed, site=3, gate=g, dgate=dgate,
                         dgain_x=dgain_x)
        h.sync()
        off = 52 * U32 * slope.abs()
        _close(dgate, slope if rows else slope.sum(0), off if rows else off.sum(0) + (n + 64) * U32 * slope.abs().sum(0), dtype, "dgate")
        if not norm_x:
            _same_kind(dx, w, 4 * U32 * w.abs(), dtype, "dx")
            continue
        terms = torch.where(kept, w * x64 * q, 0.0)
        finite = torch.isfinite(gate)
        bound = ((n + 64 + 52) * U32 * terms.abs()).sum(0)
        if rows:
            _same_kind(dgain_x, terms.sum(0), bound, dtype, "dgain_x")
        else:                                                # (the complete sum is multiplied by the gate)
            _close(dgain_x[finite.cuda()], terms.sum(0)[finite], bound[finite], dtype, "dgain_x")
            got, whole = dgain_x.double().cpu()[~finite], gate.double()[~finite] * torch.where(kept, dt64 * x64 * q, 0.0).sum(0)[~finite]
            assert torch.equal(torch.isnan(got), torch.isnan(whole)) and torch.equal(got[torch.isinf(whole)], whole[torch.isinf(whole)])


@pytest.mark.parametrize("d", [24, 600, 8193])
def test_what_is_dropped_adds_nothing_to_gradients(h, d):
    """Rows that are NaN through and through but for what is dropped, and rows whose dropped elements alone are NaN: one dgate for every row."""
    n, p, seed = 4, 0.5, 5
    kept = _kept(n, d, p, seed, 0)
    x, dt = _rand(n, d, 1).float(), _rand(n, d, 2).float()
    x[1], x[2][~kept[2]], dt[3][~kept[3]] = NAN, INF, NAN
    gate, dgate, dx = torch.ones((n, d), device="cuda"), torch.empty((n, d), device="cuda"), torch.empty((n, d), device="cuda")
    dgain_x = torch.empty(d, device="cuda")
    h.join_norm_grad(x.cuda(), dx, EPS, dtotal=dt.cuda(), p=p, seed=seed, gate=gate, dgate=dgate, dgain_x=dgain_x)
    h.sync()
    got = dgate.cpu()
    assert bool((got[~kept] == 0).all()) and torch.equal(torch.isnan(got[1]), kept[1]) and bool(torch.isfinite(got[[0, 3]]).all())
    assert torch.equal(torch.isnan(dgain_x.cpu()), kept[1])
    h.join_norm_grad(x.cuda(), dx, EPS, dtotal=dt.cuda(), norm_x=False, p=p, seed=seed, gate=gate, dgate=dgate)
    h.sync()
    got = dx.cpu()
    assert bool((got[~kept] == 0).all()) and bool(torch.isfinite(got).all())
    got = dgate.cpu()
    assert bool((got[~kept] == 0).all()) and bool(torch.isfinite(got[[0, 2, 3]]).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("d", WIDTHS + [16, 200, 264, 1024, 8192, 20_000])
def test_8_bits_with_a_gain_that_is_not_finite(h, d, dtype):
    """The scale of a row with an infinity is infinite, whatever lanes behind the row's end have loaded: what is finite becomes 0, and infinity over infinity
    NaN, as in the norm.  A gain that is NaN makes the scale NaN."""
    n = 3
    x = (_rand(n, d, 1).abs() + 0.5).to(dtype).cuda()
    for value, at in ((INF, d - 1), (-INF, max(0, d - 6)), (INF, 0), (NAN, d - 1)):
        gain = torch.ones(d, dtype=dtype, device="cuda")
        gain[at] = value
        y, y2 = (torch.zeros((n, d), dtype=E4M3, device="cuda") for _ in range(2))
        scale, scale2 = (torch.full((n,), -7.0, device="cuda") for _ in range(2))
        h.join_norm(x, EPS, y=y, norm_x=False, gain=gain, y_scale=scale)
        h.rms_norm(x, y2, EPS, gain=gain, y_scale=scale2)
        h.sync()
        for s, o in ((scale, y.float()), (scale2, y2.float())):
            if value != value:
                assert bool(torch.isnan(s).all()) and bool(torch.isnan(o).all()), (value, at)
                continue
            assert bool((s == INF).all()), (value, at)
            assert bool(torch.isnan(o[:, at]).all()) and float(o.nan_to_num(0.0).abs().max()) == 0 and int(torch.isnan(o).sum()) == n, (value, at)
