"""The gradient of learnt rows: lists that are sorted though they are short, for their rows are wide; tables that are cleared by a launch of their own; lists
long enough that a workgroup sorts several tiles and counts several spans."""
import pytest
import torch

from test_gpu_embedding import _grad_case, _ids
from test_gpu_layer import BF16, F16, F32

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


@pytest.mark.parametrize("types", [(F32, F32), (F32, BF16), (F16, F16)], ids=str)
@pytest.mark.parametrize("n,n_table,d", [(1, 3, 70_001), (100, 50, 40_000), (1000, 300, 4200), (2048, 100, 1300), (4096, 300, 256), (4096, 300, 257), (4096, 300, 513)])
def test_gradient_of_short_lists_with_wide_rows(h, n, n_table, d, types):
    """Both sides of the rule."""
    print("wide rows", n, n_table, d, types, flush=True)
    _grad_case(h, n, n_table, d, types, _ids(n, n_table, 2, 0.1, n + d), -1.7, n, pads=(3, 1), runs=2)
    _grad_case(h, n, n_table, d, types, torch.full((n,), n_table - 1, dtype=torch.int32), 1.0, n + 1, count=(n + 1) // 2)


@pytest.mark.parametrize("n,n_table,d", [(1, 300_000, 8), (300, 100_000, 33), (1000, 70_000, 72), (4096, 8000, 136)])
def test_gradient_of_large_tables(h, n, n_table, d):
    """A few rows of them are met, the others are cleared beforehand."""
    print("large tables", n, n_table, d, flush=True)
    _grad_case(h, n, n_table, d, (F32, F32), _ids(n, n_table, 1, 0.1, n), 1.5, n, pads=(1, 2), runs=2)
    _grad_case(h, n, n_table, d, (BF16, BF16), _ids(n, n_table, 3, 0.0, n + 1), 1.5, n, count=0)


def test_gradient_of_rows_of_millions_of_columns(helios):
    """4096 positions of one row of dy (its rows lie in the same place), 4 300 003 columns: sums of whole numbers, which are exact."""
    h = helios.Helios(0)
    try:
        n, d = 4096, 4_300_003
        row = (torch.arange(d, device="cuda") % 2047 - 1023).float()
        ids = torch.zeros(n, dtype=torch.int32, device="cuda")
        ids[::2] = 1
        dtable, drow = torch.full((3, d), -7.0, device="cuda"), torch.full((3, d), -7.0, device="cuda")
        row_id, n_distinct = torch.full((3,), -7, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        h.embedding_grad(ids, row.expand(n, d), 3, dtable=dtable)
        h.embedding_grad(ids, row.expand(n, d), 3, drow=drow, row_id=row_id, n_distinct=n_distinct)
        h.sync()
        assert int(n_distinct) == 2 and row_id.tolist() == [0, 1, -7]
        for k in range(2):
            assert torch.equal(dtable[k], row * (n // 2)) and torch.equal(drow[k], row * (n // 2))
        assert bool((dtable[2] == 0).all()) and bool((drow[2] == -7.0).all())
    finally:
        h.close()


def test_scratch_of_a_short_list_is_what_the_first_call_takes(helios):
    """After a call with one row a capture takes lists of up to 4096, and refuses one whose sums need more than 1 MB."""
    stream = torch.cuda.Stream()
    h = helios.Helios(0, stream=stream)
    try:
        dy, ids = torch.ones((4096, 64), device="cuda"), torch.arange(4096, dtype=torch.int32, device="cuda") % 7
        wide, dtable, wide_table = torch.ones((1, 4096), device="cuda").expand(4096, 4096), torch.zeros((9, 64), device="cuda"), torch.zeros((9, 4096), device="cuda")
        torch.cuda.synchronize()
        h.embedding_grad(ids[:1], dy[:1], 9, dtable=dtable)
        h.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            h.embedding_grad(ids, dy, 9, dtable=dtable)
            with pytest.raises(helios.HeliosError) as e:
                h.embedding_grad(ids, wide, 9, dtable=wide_table)
        assert e.value.code == helios.ESTATE and "capture" in str(e.value)
        want = torch.bincount(ids.long(), minlength=9)
        for _ in range(3):
            dtable.fill_(-7.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            h.sync()
            assert bool((dtable == want[:, None]).all())
        h.embedding_grad(ids, wide, 9, dtable=wide_table)
        h.sync()
        assert bool((wide_table == want[:, None]).all())
    finally:
        h.close()


@pytest.mark.parametrize("n,n_table,d,skew,count", [(600_000, 70_000, 3, 1, None), (600_000, 30, 8, 4, None), (600_000, 70_000, 5, 2, 550_001), (1_100_000, 1, 1, 1, None),
                                                    (2_200_000, 70_000, 2, 1, None), (2_200_000, 600, 4, 3, None), (2_200_000, 600, 1, 3, 2_097_153)])
def test_gradient_of_very_long_lists(h, n, n_table, d, skew, count):
    """More than 524 288 entries, of which a workgroup sorts two tiles and more, and more than 2 097 152, of which it counts two spans."""
    print("long lists", n, n_table, d, skew, count, flush=True)
    _grad_case(h, n, n_table, d, (F32, F32), _ids(n, n_table, skew, 0.1, n), 0.5, n, count=count, runs=2)
