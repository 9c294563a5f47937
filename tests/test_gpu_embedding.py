"""Learnt rows by ID and the gradient of their table, against plain 64-bit forms; and a block of a model from the rows' IDs to
their gradient.

With U = 2^-24 for every 32-bit step, a looked-up element is off by U of it, a sum over k positions by k U of its terms' magnitudes and U for the
scale; a result is rounded once to its type."""
import numpy as np
import pytest
import torch

from test_gpu_join import _factor, _kept
from test_gpu_layer import BF16, E4M3, EPS, F16, F32, U32, _close, _on_gpu, _out, _rand, _untouched

pytestmark = pytest.mark.gpu

TYPES = [(F32, F32), (F32, F16), (F32, BF16), (F16, F16), (BF16, BF16)]


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


def _ids(n, n_table, skew, missing, seed):
    rng = np.random.default_rng(seed)
    ids = rng.permutation(n_table)[(n_table * rng.random(n) ** skew).astype(np.int64)]
    ids[rng.random(n) < missing] = -1
    return torch.from_numpy(ids.astype(np.int32))


# ------------------------------------------------------------------ lookup


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("n,n_table,d", [(1, 1, 1), (1, 1000, 256), (7, 3, 9), (100, 50, 64), (777, 2000, 200), (3000, 100_000, 24), (33, 10, 5000), (2, 5, 70_001)])
def test_lookup(h, n, n_table, d, types):
    table_type, y_type = types
    ids = _ids(n, n_table, 2, 0.2, n + d)
    table, add = _on_gpu(_rand(n_table, d, 1), table_type, d % 5, n % 3), _on_gpu(_rand(n, d, 2), y_type, 3, 1)
    rows = torch.where(ids[:, None] >= 0, table.double().cpu()[ids.clamp_min(0).long()], 0.0)
    for scale, plus in ((1.0, False), (-11.3, True), (0.0, True)):
        scale = float(np.float32(scale))
        y = _out(n, d, y_type, d % 4, n % 2)
        h.embedding(table, ids.cuda(), y, scale=scale, add=add if plus else None)
        h.sync()
        want = rows * scale + (add.double().cpu() if plus else 0.0)
        _close(y, want, U32 * want.abs(), y_type)
        assert _untouched(y)
    y = add.clone()
    h.embedding(table, ids.cuda(), y, scale=2.0, add=y)
    h.sync()
    _close(y, rows * 2 + add.double().cpu(), U32 * (rows * 2 + add.double().cpu()).abs(), y_type)


def test_lookup_with_the_count_on_the_device_and_bad_ids(helios, h):
    n, d = 20, 40
    table, ids = _rand(9, d, 1).float().cuda(), torch.arange(n, dtype=torch.int32) % 9
    ids[13:] = 1000                                       # behind the count: not looked at
    y = torch.full((n, d), -7.0, device="cuda")
    h.embedding(table, ids.cuda(), y, n_rows_dev=torch.tensor([13], dtype=torch.int64, device="cuda"))
    h.sync()
    assert torch.equal(y[:13], table[ids[:13].long().cuda()]) and bool((y[13:] == -7.0).all())
    for bad in (-2, 9, 2 ** 31 - 1, -2 ** 31):
        wrong = ids.clone()
        wrong[13:], wrong[4] = 0, bad
        h.embedding(table, wrong.cuda(), y)
        with pytest.raises(helios.HeliosError) as e:
            h.sync()
        assert e.value.code == helios.EDATA
        assert bool((y[4] == 0).all()) and torch.equal(y[5], table[5])
    h.embedding(table[:0], torch.full((n,), -1, dtype=torch.int32, device="cuda"), y)
    h.embedding(table, ids[:0].cuda(), y[:0])
    h.sync()
    assert bool((y == 0).all())


def test_lookup_of_rows_that_are_not_finite(h):
    """-1 takes nothing from the table, whatever its rows hold, and a row that is not finite stays in its places."""
    table = torch.full((3, 16), float("nan"), device="cuda")
    table[1], table[2] = 1.0, float("inf")
    ids, y = torch.tensor([-1, 1, 0, 2], dtype=torch.int32, device="cuda"), torch.empty((4, 16), device="cuda")
    h.embedding(table, ids, y, scale=0.5)
    h.sync()
    assert bool((y[0] == 0).all()) and bool((y[1] == 0.5).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isinf(y[3]).all())


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_a_large_lookup(h, types):
    """One of more than 128 MB, which may go past the caches."""
    n, n_table, d = 120_000, 40_000, 256
    table, add, ids = torch.randn((n_table, d), device="cuda").to(types[0]), torch.randn((n, d), device="cuda").to(types[1]), _ids(n, n_table, 1.0, 0.1, 5).cuda()
    y = torch.full((n, d), -7.0, dtype=types[1], device="cuda")
    h.embedding(table, ids, y, add=add)
    h.sync()
    want = torch.where((ids >= 0)[:, None], table[ids.clamp_min(0).long()].float() + add.float(), add.float())
    assert torch.equal(y, want.to(types[1]))


def test_rows_beyond_32_bits(h):
    """A table of 5 000 000 x 1024 in half precision (elements and bytes past 2^32), few rows of which are looked up and get a gradient."""
    n_table, d = 5_000_000, 1024
    table = torch.empty((n_table, d), dtype=F16, device="cuda")
    ids = torch.tensor([4_999_999, 0, 4_194_304, 2_097_152, 4_999_999], dtype=torch.int32)
    rows = _rand(5, d, 3).half()
    rows[4] = rows[0]
    table[ids.long().cuda()] = rows.cuda()
    y = torch.empty((5, d), dtype=F16, device="cuda")
    h.embedding(table, ids.cuda(), y)
    h.sync()
    assert torch.equal(y.cpu(), rows)
    h.embedding_grad(ids.cuda(), y, n_table, dtable=table)
    h.sync()
    assert torch.equal(table[4_999_999].cpu(), (rows[0].float() * 2).half()) and torch.equal(table[4_194_304].cpu(), rows[2])
    assert int((table[::1000].abs().amax(1) > 0).sum()) == 1 and int((table.view(torch.int32).amax(1) != 0).sum()) <= 4


# ------------------------------------------------------------------ gradient


def _grad_case(h, n, n_table, d, types, ids, scale, seed, pads=(0, 0), count=None, runs=1):
    table_type, y_type = types
    live = n if count is None else count
    dy = _on_gpu(_rand(n, d, seed), y_type, pads[0], pads[1])
    if live < n:
        dy[live:] = float("nan")
    n_dev = None if count is None else torch.tensor([count], dtype=torch.int64, device="cuda")
    at = torch.nonzero(ids[:live] >= 0)[:, 0]
    scale = float(np.float32(scale))
    g = dy.double().cpu()[at]
    which = ids[at].long()
    want, size = (torch.zeros((n_table, d), dtype=torch.float64).index_add(0, which, v) for v in (g, g.abs()))
    times = torch.bincount(which, minlength=n_table)
    bound = abs(scale) * (times[:, None] + 2) * U32 * size
    want = want * scale
    ids_gpu = ids.cuda()
    seen = torch.nonzero(times > 0)[:, 0]
    rows = min(n, n_table)
    first = None
    for _ in range(runs):
        dtable, drow = _out(n_table, d, table_type, pads[1], pads[0]), _out(rows, d, table_type, pads[0])
        row_id = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
        n_distinct = torch.full((1,), -7, dtype=torch.int64, device="cuda")
        h.embedding_grad(ids_gpu, dy, n_table, scale=scale, dtable=dtable, n_rows_dev=n_dev)
        h.embedding_grad(ids_gpu, dy, n_table, scale=scale, drow=drow, row_id=row_id, n_distinct=n_distinct, n_rows_dev=n_dev)
        h.sync()
        u = int(n_distinct)
        assert u == seen.numel() and torch.equal(row_id[:u].cpu().long(), seen) and bool((row_id[u:] == -7).all())
        assert _untouched(dtable) and _untouched(drow) and bool((drow[u:].float() == -7.0).all())
        if first is None:
            first = (dtable, drow)
            _close(dtable, want, bound, table_type, "dtable")
            assert torch.equal(drow[:u], dtable[seen.cuda()])
        assert torch.equal(dtable, first[0]) and torch.equal(drow, first[1])            # the same bits in every call


CASES = [(1, 1, 1), (1, 500, 256), (2, 2, 7), (16, 4, 64), (17, 100, 100), (33, 1, 130), (777, 3000, 200), (777, 7, 24), (1000, 50, 520), (2048, 300, 40),
         (2049, 300, 40), (4096, 5000, 16), (5000, 2, 300), (12_289, 70_000, 72), (70_000, 400, 24), (300_000, 5000, 9)]


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("n,n_table,d", CASES)
def test_gradient(h, n, n_table, d, types):
    print("gradient", n, n_table, d, types, flush=True)
    _grad_case(h, n, n_table, d, types, _ids(n, n_table, 1, 0.0, n), 1.0, n)
    _grad_case(h, n, n_table, d, types, _ids(n, n_table, 4, 0.2, n + 1), -3.7, n + 1, pads=(3, 1))


@pytest.mark.parametrize("n,count", [(100, 0), (100, 37), (2048, 2047), (2049, 2048), (5000, 1), (9000, 4097), (20_000, 20_000)])
def test_gradient_with_the_count_on_the_device(h, n, count):
    """IDs behind the count are not looked at: they are none."""
    ids = _ids(n, 700, 2, 0.1, n)
    ids[count:] = 123_456
    _grad_case(h, n, 700, 40, (F32, F32), ids, 0.5, n, count=count)


@pytest.mark.parametrize("n,count", [(4095, None), (4096, None), (4097, None), (4096, 4095), (4097, 4096), (3000, 65)])
def test_gradient_of_the_longest_lists_that_are_not_sorted(h, n, count):
    """Distinct IDs only; one ID only; few; a few that are met often among many."""
    some = torch.from_numpy(np.random.default_rng(n).permutation(9000)[:n].astype(np.int32))
    mixed = torch.where(torch.arange(n) % 3 == 0, some, some % 5)
    for k, ids in enumerate((some, torch.full((n,), 8999, dtype=torch.int32), some % 70, mixed)):
        _grad_case(h, n, 9000, 72, (F32, BF16), ids, 1.5, n + k, **({} if count is None else dict(count=count)))


@pytest.mark.parametrize("d", [8, 200, 1000])
@pytest.mark.parametrize("n", [50, 2000, 9000, 40_000])
def test_gradient_of_long_runs(h, n, d):
    """One ID only; two that meet inside a chunk; runs of every length side by side; nothing but missing ones.  Three times, the same bits."""
    rng = np.random.default_rng(n)
    one = torch.full((n,), 3, dtype=torch.int32)
    two = one.clone()
    two[n // 3:] = 4
    lens = np.concatenate([np.arange(1, 70), [127, 128, 129, 511, 512, 513]])
    every = torch.from_numpy(np.repeat(np.arange(lens.size), lens)[:n].astype(np.int32))
    mixed = torch.full((n,), 90, dtype=torch.int32)
    mixed[:every.numel()] = every
    mixed = mixed[torch.from_numpy(rng.permutation(n))]
    for k, ids in enumerate((one, two, mixed, torch.full((n,), -1, dtype=torch.int32))):
        _grad_case(h, n, 100, d, (F32, F32), ids, 1.5, n + k, runs=3)


@pytest.mark.parametrize("n_table", [1, 15, 16, 255, 256, 257, 65_535, 65_536, 2 ** 24, 2 ** 31 - 1025])
def test_gradient_of_tables_of_any_size(h, n_table):
    """The numbers of bits that the sort has to look at; the largest IDs."""
    n, d = 5000, 16
    ids = torch.from_numpy(np.random.default_rng(n_table).integers(0, n_table, n).astype(np.int32))
    ids[7], ids[4000], ids[8] = n_table - 1, n_table - 1, -1
    dy = _rand(n, d, 1).float().cuda()
    rows = min(n, n_table)
    drow, row_id = torch.full((rows, d), -7.0, device="cuda"), torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    n_distinct = torch.zeros(1, dtype=torch.int64).pin_memory()
    h.embedding_grad(ids.cuda(), dy, n_table, drow=drow, row_id=row_id, n_distinct=n_distinct)
    h.sync()
    seen, where, times = torch.unique(ids[ids >= 0], return_inverse=True, return_counts=True)
    assert int(n_distinct) == seen.numel() and torch.equal(row_id[:seen.numel()].cpu(), seen)
    g = dy.double().cpu()[ids >= 0]
    want, size = (torch.zeros((seen.numel(), d), dtype=torch.float64).index_add(0, where, v) for v in (g, g.abs()))
    _close(drow[:seen.numel()], want, (times[:, None] + 2) * U32 * size, F32)


def test_gradient_of_bad_ids_is_reported(helios, h):
    for n in (50, 5000):
        ids = _ids(n, 30, 1, 0.0, n)
        dy = torch.ones((n, 24), device="cuda")
        for bad in (-2, 30, 2 ** 31 - 1, -2 ** 31):
            wrong = ids.clone()
            wrong[n // 2] = bad
            dtable = torch.full((30, 24), -7.0, device="cuda")
            h.embedding_grad(wrong.cuda(), dy, 30, dtable=dtable)
            with pytest.raises(helios.HeliosError) as e:
                h.sync()
            assert e.value.code == helios.EDATA
            wrong[n // 2] = -1
            assert torch.equal(dtable[:, 0].cpu().long(), torch.bincount(wrong[wrong >= 0].long(), minlength=30))


def test_gradient_of_empty_lists_and_tables_and_of_repeated_rows(h):
    none, ids = torch.empty(0, dtype=torch.int32, device="cuda"), torch.full((9,), -1, dtype=torch.int32, device="cuda")
    dtable, n_distinct = torch.full((5, 24), -7.0, device="cuda"), torch.full((1,), -7, dtype=torch.int64, device="cuda")
    rows, row_id = torch.empty((0, 24), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    h.embedding_grad(none, rows, 5, dtable=dtable)
    h.embedding_grad(none, rows, 5, drow=rows, row_id=row_id, n_distinct=n_distinct)
    h.sync()
    assert bool((dtable == 0).all()) and int(n_distinct) == 0
    n_distinct.fill_(-7)
    h.embedding_grad(ids, torch.ones((9, 24), device="cuda"), 0, drow=rows, row_id=row_id, n_distinct=n_distinct)
    h.embedding_grad(ids, torch.ones((9, 24), device="cuda"), 0, dtable=rows)
    h.sync()
    assert int(n_distinct) == 0
    ids[3:] = 2
    h.embedding_grad(ids, torch.full((1, 24), 0.25, device="cuda").expand(9, 24), 5, dtable=dtable)
    h.sync()
    assert bool((dtable[2] == 1.5).all()) and bool((dtable[[0, 1, 3, 4]] == 0).all())


def test_gradient_against_differences(h):
    n, n_table, d, e = 7, 4, 3, 1e-3
    ids = torch.tensor([3, 0, -1, 3, 1, 0, 3], dtype=torch.int32)
    table, dy = _rand(n_table, d, 1), _rand(n, d, 2).float()
    loss = lambda t: float(((t[ids.clamp_min(0).long()] * 0.5) * (ids >= 0)[:, None] * dy.double()).sum())  # noqa: E731
    dtable = torch.empty((n_table, d), device="cuda")
    h.embedding_grad(ids.cuda(), dy.cuda(), n_table, scale=0.5, dtable=dtable)
    h.sync()
    for i in range(table.numel()):
        sides = []
        for s in (e, -e):
            moved = table.clone()
            moved.view(-1)[i] += s
            sides.append(loss(moved))
        assert abs(float(dtable.view(-1)[i]) - (sides[0] - sides[1]) / (2 * e)) < 1e-5


# ------------------------------------------------------------------ the calls as calls


def test_in_a_graph_with_other_lists(helios):
    """A recorded lookup and gradient, dense and by row: replays on lists of other IDs and lengths in the same memory give what eager calls give."""
    n, n_table, d = 5000, 900, 72
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        table, dy, ids = _rand(n_table, d, 1).half().cuda(), _rand(n, d, 2).half().cuda(), torch.zeros(n, dtype=torch.int32, device="cuda")
        count = torch.zeros(1, dtype=torch.int64, device="cuda")
        y, dtable, drow = torch.zeros((n, d), dtype=F16, device="cuda"), torch.zeros((n_table, d), dtype=F16, device="cuda"), torch.zeros((n_table, d), dtype=F16, device="cuda")
        row_id, n_distinct = torch.zeros(n_table, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        outs = [y, dtable, drow, row_id, n_distinct]
        torch.cuda.synchronize()

        def step():
            h.embedding(table, ids, y, scale=3.0, n_rows_dev=count)
            h.embedding_grad(ids, dy, n_table, scale=3.0, dtable=dtable, n_rows_dev=count)
            h.embedding_grad(ids, dy, n_table, scale=3.0, drow=drow, row_id=row_id, n_distinct=n_distinct, n_rows_dev=count)

        step()
        h.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for turn, live in enumerate((5000, 1, 0, 3333, 5000)):
            print("graph replay", turn, flush=True)
            ids.copy_(_ids(n, n_table, 1 + turn, 0.1, turn).cuda())
            count.fill_(live)
            got = []
            for replay in (False, True):
                for t in outs:
                    t.zero_()
                torch.cuda.synchronize()
                if replay:
                    with torch.cuda.stream(stream):
                        graph.replay()
                else:
                    step()
                h.sync()
                got.append([t.clone() for t in outs])
            assert all(torch.equal(a, b) for a, b in zip(*got)), turn
            assert int(n_distinct) == torch.unique(ids[:live][ids[:live] >= 0]).numel()
    finally:
        h.close()


def test_refusals(helios, h):
    table, ids, y = torch.zeros((8, 16), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((4, 16), device="cuda")
    row_id, n_distinct = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")

    def einval(call, *args, **kw):
        with pytest.raises(helios.HeliosError) as e:
            call(*args, **kw)
        assert e.value.code == helios.EINVAL
        return str(e.value)

    def refused(kind, call, *args, **kw):
        with pytest.raises(kind):
            call(*args, **kw)

    refused(TypeError, h.embedding, table, ids.long(), y)
    refused(TypeError, h.embedding, table, ids, y[:, :15])
    refused(TypeError, h.embedding, table, ids, y, add=y.half())
    refused(AssertionError, h.embedding, table, ids[:3], y)
    assert "y_type" in einval(h.embedding, table.half(), ids, y)
    assert "y_type" in einval(h.embedding, table, ids, y.to(E4M3))
    assert "table_type" in einval(h.embedding, table.to(E4M3), ids, y)
    assert "shares memory" in einval(h.embedding, table, ids, table[:4])
    assert "shares memory" in einval(h.embedding, table, y.view(torch.int32)[0, :4], y)
    assert "width" in einval(h.embedding, table[:, :0], ids, y[:, :0])
    refused(TypeError, h.embedding_grad, ids, y, 8)
    refused(AssertionError, h.embedding_grad, ids, y, 8, drow=torch.zeros((3, 16), device="cuda"), row_id=row_id, n_distinct=n_distinct)
    refused(AssertionError, h.embedding_grad, ids, y, 8, drow=torch.zeros_like(y), row_id=row_id[:3], n_distinct=n_distinct)
    refused(TypeError, h.embedding_grad, ids, y, 8, dtable=y)
    assert "both" in einval(h.embedding_grad, ids, y, 8, dtable=table, n_distinct=n_distinct)
    assert "NULL" in einval(h.embedding_grad, ids, y, 8, drow=torch.zeros_like(y), row_id=row_id)
    assert "NULL" in einval(h.embedding_grad, ids, y, 8, drow=torch.zeros_like(y), n_distinct=n_distinct)
    assert "shares memory" in einval(h.embedding_grad, ids, y, 8, drow=y, row_id=row_id, n_distinct=n_distinct)
    assert "shares memory" in einval(h.embedding_grad, ids, y, 8, drow=torch.zeros_like(y), row_id=ids, n_distinct=n_distinct)
    assert "y_type" in einval(h.embedding_grad, ids, y, 8, dtable=table.half())
    assert "n_table" in einval(h.embedding_grad, ids, y, 2 ** 31, drow=torch.zeros_like(y), row_id=row_id, n_distinct=n_distinct)
    assert "n_table" in einval(h.embedding_grad, ids[:0], y[:0], -1, drow=torch.zeros_like(y), row_id=row_id, n_distinct=n_distinct)
    lib = helios._lib
    for f, args in ((lib.helios_embedding, helios.EmbeddingArgs), (lib.helios_embedding_grad, helios.EmbeddingGradArgs)):
        assert f(None, None) == helios.EINVAL and f(h._h, None) == helios.EINVAL
        assert f(h._h, args(n_rows=-1, width=4)) == helios.EINVAL and f(h._h, args(n_rows=1, width=4, n_table=1)) == helios.EINVAL
        assert f(h._h, args(n_rows=1, width=2 ** 25, n_table=1)) == helios.EINVAL
    assert lib.helios_embedding(h._h, helios.EmbeddingArgs(n_rows=0, width=4, n_table=4)) == helios.OK
    h.sync()


def test_a_capture_that_would_have_to_allocate_is_refused(helios):
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        ids, dy, dtable = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.ones((64, 32), device="cuda"), torch.zeros((4, 32), device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(helios.HeliosError) as e:
                h.embedding_grad(ids, dy, 4, dtable=dtable)
        assert e.value.code == helios.ESTATE and "capture" in str(e.value)
        h.embedding_grad(ids, dy, 4, dtable=dtable)
        h.sync()
        assert bool((dtable[0] == 64).all()) and bool((dtable[1:] == 0).all())
    finally:
        h.close()


def test_two_contexts_at_once(helios):
    """Long lists and a join's gradient on two streams, call by call in turn: scratch is a context's own."""
    n, n_table, d = 30_000, 500, 64
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [helios.Helios(0, stream=s) for s in streams]
    try:
        cases = []
        for k in range(2):
            ids, dy = _ids(n, n_table, 2, 0.1, 70 + k).cuda(), torch.randn((n, d), device="cuda")
            cases.append(dict(ids=ids, dy=dy, dtable=torch.empty((n_table, d), device="cuda"), dx=torch.empty_like(dy), dgain_x=torch.empty(d, device="cuda"),
                              x=torch.randn((n, d), device="cuda")))
        torch.cuda.synchronize()

        def call(h, c):
            h.embedding_grad(c["ids"], c["dy"], n_table, dtable=c["dtable"])
            h.join_norm_grad(c["x"], c["dx"], EPS, dtotal=c["dy"], p=0.3, seed=9, dgain_x=c["dgain_x"])

        want = []
        for h, c in zip(contexts, cases):
            call(h, c)
            h.sync()
            want.append([c[k].clone() for k in ("dtable", "dx", "dgain_x")])
        torch.cuda.synchronize()
        for _ in range(5):
            for c in cases:
                for k in ("dtable", "dx", "dgain_x"):
                    c[k].fill_(-7.0)
            torch.cuda.synchronize()
            for _ in range(3):
                for h, c in zip(contexts, cases):
                    call(h, c)
            for h in contexts:
                h.sync()
            for c, w in zip(cases, want):
                assert all(torch.equal(c[k], v) for k, v in zip(("dtable", "dx", "dgain_x"), w))
    finally:
        for h in contexts:
            h.close()


# ------------------------------------------------------------------ together


def test_a_block_of_a_model_and_its_gradients(helios, h):
    """ids -> learnt rows beside features -> product -> dropout -> product -> join with the residual, and back to the table's rows: every
    gradient against automatic differentiation in 64 bits with the same elements dropped.  Single precision: there are about ten steps, each good
    to some 1e-6 of its largest values."""
    n, n_table, d, seed, p = 500, 200, 48, 31, 0.2
    ids = _ids(n, n_table, 2, 0.05, 1)
    par = {"table": _rand(n_table, d, 1), "w1": _rand(2 * d, d, 2, d ** -0.5), "w2": _rand(d, 2 * d, 3, (2 * d) ** -0.5), "gain_x": _rand(1, d, 4, 0.2)[0] + 1,
           "gate": _rand(1, d, 5)[0], "gain": _rand(1, d, 6, 0.2)[0] + 1}
    g = {k: v.float().cuda() for k, v in par.items()}
    feats, dy, dtotal = (_rand(n, d, s).float().cuda() for s in (7, 8, 9))
    new = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    x, z, a, k, b, total, y = new(n, d), new(n, 2 * d), new(n, 2 * d), new(n, 2 * d), new(n, d), new(n, d), new(n, d)
    rows = ids.cuda()
    h.embedding(g["table"], rows, x, scale=d ** 0.5, add=feats)
    h.linear(x, g["w1"], a, act=helios.ACT_GELU, pre=z)
    h.dropout(a, k, p, seed, site=1)
    h.linear(k, g["w2"], b)
    join = dict(gain_x=g["gain_x"], p=p, seed=seed, site=2, gate=g["gate"], residual_scale=0.7)
    h.join_norm(b, EPS, y=y, total=total, residual=x, gain=g["gain"], **join)
    grad = {name: torch.empty_like(g[name]) for name in ("w1", "w2", "gain_x", "gate", "gain")}
    db, dres, dk, da, dx = new(n, d), new(n, d), new(n, 2 * d), new(n, 2 * d), new(n, d)
    h.join_norm_grad(b, db, EPS, total=total, dy=dy, dtotal=dtotal, gain=g["gain"], dresidual=dres, dgate=grad["gate"], dgain_x=grad["gain_x"], dgain=grad["gain"], **join)
    h.linear_grad(k, g["w2"], db, dx=dk, dw=grad["w2"])
    h.dropout(dk, da, p, seed, site=1)
    h.linear_grad(x, g["w1"], da, act=helios.ACT_GELU, pre=z, dx=dx, dw=grad["w1"])
    dx += dres
    drow, row_id, n_distinct = new(n_table, d), torch.empty(n_table, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int64, device="cuda")
    h.embedding_grad(rows, dx, n_table, scale=d ** 0.5, drow=drow, row_id=row_id, n_distinct=n_distinct)
    h.sync()
    w = {name: v.double().cpu().requires_grad_(True) for name, v in g.items()}
    mask = lambda cols, site: torch.where(_kept(n, cols, p, seed, site), _factor(p), 0.0).double()  # noqa: E731
    norm = lambda t, s: t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS) * s  # noqa: E731
    x64 = feats.double().cpu() + d ** 0.5 * w["table"][ids.clamp_min(0).long()] * (ids >= 0)[:, None]
    z64 = x64 @ w["w1"].t()
    b64 = (z64 * 0.5 * torch.special.erfc(-z64 / 2 ** 0.5) * mask(2 * d, 1)) @ w["w2"].t()
    t64 = 0.7 * x64 + w["gate"] * (norm(b64, w["gain_x"]) * mask(d, 2))
    y64 = norm(t64, w["gain"])
    assert float((y.double().cpu() - y64.detach()).abs().max()) < 1e-5 * float(y64.detach().abs().max())
    ((y64 * dy.double().cpu()).sum() + (t64 * dtotal.double().cpu()).sum()).backward()
    u = int(n_distinct)
    assert torch.equal(row_id[:u].cpu(), torch.unique(ids[ids >= 0]))
    grad["table"] = torch.zeros_like(g["table"])
    grad["table"][row_id[:u].long()] = drow[:u]
    for name, t in grad.items():
        ref = w[name].grad
        assert float((t.double().cpu() - ref).abs().max()) < 2e-5 * float(ref.abs().max()), name
