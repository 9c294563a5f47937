"""Blocks whose lists do not take all of col, or lie wrong: what helios_block_mean, _transpose and _mean_grad make of them."""
import numpy as np
import pytest
import torch

from test_gpu_layer import F32, U32, _close, _rand

pytestmark = pytest.mark.gpu
ONE_LAUNCH = 131_072                              # places up to which a block is put by source in one launch


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


def _hop(n, n_src, fan, seed):
    rng = np.random.default_rng(seed)
    deg = rng.integers(0, fan + 1, n)
    indptr = np.zeros(n + 1, np.int64)
    indptr[1:] = np.cumsum(deg)
    return indptr, rng.integers(0, n_src, indptr[-1]).astype(np.int32), rng.integers(0, n_src, n).astype(np.int32)


def _transposed(h, indptr, col, row, n_src):
    si = torch.full((n_src + 1,), -7, dtype=torch.int32, device="cuda")
    se = torch.full((max(1, len(col) + (0 if row is None else len(row))),), -7, dtype=torch.int32, device="cuda")
    h.block_transpose(torch.from_numpy(indptr).cuda(), torch.from_numpy(col).cuda(), n_src, si, se, row=None if row is None else torch.from_numpy(row).cuda())
    return si, se


# the shapes lie on both sides of ONE_LAUNCH; the parts leave out rows in front, behind, and all but a few
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("n,n_src,fan", [(40, 30, 4), (9000, 700, 9), (60_000, 5000, 8)])
@pytest.mark.parametrize("part", [(0.3, 1.0), (0.0, 0.6), (0.45, 0.5), (0.5, 0.5)], ids=str)
def test_block_of_part_of_a_hops_rows(h, n, n_src, fan, part, own):
    indptr, col, row = _hop(n, n_src, fan, n + int(own))
    lo, hi = int(part[0] * n), int(part[1] * n)
    print("part", n, n_src, lo, hi, own, len(col), flush=True)
    _transposed(h, indptr, col, row, n_src)       # (another call's entries in the scratch)
    cut, rows = indptr[lo:hi + 1].copy(), row[lo:hi].copy() if own else None
    si, se = _transposed(h, cut, col, rows, n_src)
    h.sync()
    deg = np.diff(cut)
    source, entry = col[cut[0]:cut[-1]], np.repeat(np.arange(hi - lo), deg)
    if own:
        source, entry = np.concatenate([source, rows]), np.concatenate([entry, ~np.arange(hi - lo)])
    order = np.argsort(source, kind="stable")
    assert np.array_equal(si.cpu().numpy(), np.searchsorted(source[order], np.arange(n_src + 1)))
    assert np.array_equal(se.cpu().numpy()[:len(entry)], entry[order])
    assert bool((se[len(entry):] == -7).all())
    # and the gradient of the mean over these rows
    d = 24
    dmean, down, dx = _rand(hi - lo, d, 1).float(), _rand(hi - lo, d, 2).float(), torch.empty((n_src, d), device="cuda")
    h.block_mean_grad(torch.from_numpy(cut).cuda(), si, se, dmean.cuda(), dx, down=down.cuda() if own else None)
    h.sync()
    each = torch.cat([(dmean.double() / torch.from_numpy(np.maximum(deg, 1))[:, None]).repeat_interleave(torch.from_numpy(deg), 0), down.double()])[:len(source)]
    at = torch.from_numpy(source).long()
    want, size = (torch.zeros((n_src, d), dtype=torch.float64).index_add(0, at, v) for v in (each, each.abs()))
    _close(dx, want, (np.bincount(source, minlength=n_src).max() + 4) * U32 * size if len(source) else want, F32)


@pytest.mark.parametrize("n,fan", [(6, 4), (40_000, 8)], ids=["one launch", "sort"])
def test_transposing_lists_that_lie_wrong_is_reported(helios, h, n, fan):
    """As by helios_block_mean: a list in front of col, behind it, or that ends before it begins, wherever it is."""
    n_src, d = 50, 16
    indptr, col, row = _hop(n, n_src, fan, 5)
    indptr[1:] += np.arange(n) // (n // 2) + 1    # (no list is empty by chance where it matters)
    col = np.resize(col, indptr[-1])
    assert (len(col) + n > ONE_LAUNCH) == (n > 6)
    x, mean = _rand(n_src, d, 1).float().cuda(), torch.empty((n, d), device="cuda")
    wrong = {"behind": (n, len(col) + 1), "before": (0, -1), "backwards": (n // 2, int(indptr[n // 2 + 1]) + 1), "first": (0, int(indptr[1]) + 1), "last": (n, int(indptr[n - 1]) - 1)}
    for name, (at, value) in wrong.items():
        bad = indptr.copy()
        bad[at] = value
        print(name, flush=True)
        for call in (lambda: h.block_mean(x, torch.from_numpy(bad).cuda(), torch.from_numpy(col).cuda(), mean),
                     lambda: _transposed(h, bad, col, None, n_src), lambda: _transposed(h, bad, col, row, n_src)):
            call()
            with pytest.raises(helios.HeliosError) as e:
                h.sync()
            assert e.value.code == helios.EDATA, name
    _transposed(h, indptr, col, row, n_src)
    h.sync()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("d", [1, 16, 300])
def test_own_row_of_a_source_that_there_is_none_of_is_zeros(helios, h, dtype, d):
    """Whatever own held before, with `row` and without; the rows around it are theirs."""
    x = _rand(10, d, 1).to(dtype).cuda()
    indptr, col = torch.zeros(13, dtype=torch.int64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    for bad in (-1, 10, 2 ** 31 - 1, None):
        mean, own = (torch.full((12, d), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        at = torch.arange(12, dtype=torch.int32) % 10
        row = None
        if bad is not None:
            at[[0, 7]] = bad
            row = at.cuda()
        else:
            at = torch.arange(12)
        h.block_mean(x, indptr, col, mean, row=row, own=own)
        with pytest.raises(helios.HeliosError) as e:
            h.sync()
        assert e.value.code == helios.EDATA
        there = (at >= 0) & (at < 10)
        want = torch.zeros((12, d), dtype=dtype)
        want[there] = x.cpu()[at[there].long()]
        assert torch.equal(own.cpu(), want) and bool((mean == 0).all())


def test_gradient_of_a_sample_of_a_row_without_samples_is_left_out(helios, h):
    """An entry that names row 1, whose list is empty (or backwards), adds nothing, and is reported; those of row 0 count."""
    dmean, si, se = _rand(3, 16, 1).float().cuda(), torch.tensor([0, 2, 3, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
    for indptr in ([0, 2, 2, 3], [0, 2, 1, 3]):
        dx = torch.full((3, 16), -7.0, device="cuda")
        h.block_mean_grad(torch.tensor(indptr, dtype=torch.int64, device="cuda"), si, se, dmean, dx)
        with pytest.raises(helios.HeliosError) as e:
            h.sync()
        assert e.value.code == helios.EDATA
        assert torch.equal(dx[0], dmean[0] / 2) and bool((dx[1:] == 0).all())
