"""Page calls where they can go wrong: arguments out of range anywhere among many rows, tables without places, the launches of large pools and
large tables together, arrays off 16 bytes, handles side by side."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_utils import dev_i32, make_handle
from paper_2607_13095_b200 import binding as hb
from test_gpu_packed import dims, no_error
from test_gpu_pages import FILL, check_fork, children, fork, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [5003, 70001])
@pytest.mark.parametrize("rows,hi", [(100, 40), (1500, 30), (100, 8000)])
def test_fork_refuses_a_bad_number_of_pages_in_any_row(rows, hi, pages):
    """A row that claims more pages than its table has places, or fewer than none, wherever it stands: nothing is done."""
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    rng = np.random.default_rng(rows)
    blocks = -(-hi // P) + 1
    table = rng.integers(0, pages, (rows, blocks)).astype(np.int32)
    counts = np.bincount(table.ravel(), minlength=pages).astype(np.int32)
    parent = np.arange(rows, dtype=np.int32)[::-1].copy()
    length = np.full(rows, P, np.int32)
    for row in (0, 31, 33, 64, rows // 2, rows - 1):
        for bad in (blocks + 1, 1 << 30, -1):
            held = np.full(rows, blocks, np.int32)
            held[row] = bad
            got = fork(h, counts, table, held, parent, length, length + 1, blocks)
            st = hb.hswa_get_async_error(h)
            assert st == (hb.HSWA_ERR_BOUNDS, row, -1, bad), st
            assert np.array_equal(got[0], counts) and all((g == FILL).all() for g in got[1:])


@pytest.mark.parametrize("pages", [9, 70001])
@pytest.mark.parametrize("blocks,out_blocks", [(0, 0), (0, 2), (2, 0)])
def test_fork_of_tables_without_places(blocks, out_blocks, pages):
    """Rows that hold no page, from or into tables of width 0: their numbers of pages and copies are written like any others."""
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts = np.zeros(pages, np.int32)
    counts[3] = 2
    need = [0, 0, P + 1 if out_blocks else 0]
    got = check_fork(h, P, counts, np.zeros((2, blocks), np.int32), np.zeros(2, np.int32), [0, -1, -1], [0, 0, 0], need, out_blocks)
    assert got[2].tolist() == [0, 0, out_blocks]


def test_compact_of_tables_without_places():
    h = make_handle(dims(1, 64, 16, 1))
    counts = dev_i32([0, 1, 0, 2])
    o = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((4,), (2, 0), (4,), (2,), (2,))]
    hb.hswa_pages_compact(h, counts, o[0], torch.zeros((2, 0), dtype=torch.int32, device="cuda"), dev_i32([0, 0]), o[1], o[2], o[3], o[4])
    no_error(h)
    assert [x.tolist() for x in (o[0], o[2], o[3], o[4])] == [[2, 1, 0, 0], [0, 1, 2, 0], [3, -1], [0, -1]]


def test_compact_refuses_a_table_over_the_counts():
    h = make_handle(dims(1, 64, 16, 1))
    counts = dev_i32([0, 1, 0, 2, 1, 0])
    before = counts.clone()
    o = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((6,), (6,), (2,), (2,))]
    with pytest.raises(hb.HswaError) as e:
        hb.hswa_pages_compact(h, counts, o[0], dev_i32([[1, 3, 0], [4, 0, 0]]), dev_i32([2, 1]), counts.reshape(2, 3), o[1], o[2], o[3])
    assert e.value.status == hb.HSWA_ERR_INVALID_ARG
    assert torch.equal(counts, before) and all((x == FILL).all() for x in o)
    no_error(h)
