"""Page calls where they can go wrong: arguments out of range anywhere among many rows, tables without places, the launches of large pools and
large tables together, arrays off 16 bytes, handles side by side."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl
from test_gpu_packed import dims, no_error, no_rings
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


@pytest.mark.parametrize("what", ["fork", "compact"])
def test_tables_written_through_another_handle_between_decode_calls(what):
    """Decode calls of one handle may overlap; a table that another handle's call writes between two of them is whole before the second reads it."""
    d, B, L = dims(4, 64, 16, 1), 8, 300
    P, blocks = 16, 20
    pages = 1 + B * blocks
    h, other = make_handle(d, torch.float32), make_handle(d, torch.float32)
    table = dev_i32(1 + np.random.default_rng(12).permutation(B * blocks).reshape(B, blocks))
    pools = [to_dev_bf16(wl.bf16_bits_normal(60 + i, (pages, 2, 1, P, 64))) for i in range(2)]
    q, k, v = (to_dev_bf16(wl.bf16_bits_normal(62 + i, (B, n, 64))) for i, n in enumerate((4, 1, 1)))
    ref_in, held = torch.ones((pages,), dtype=torch.int32, device="cuda"), dev_i32([blocks] * B)
    ref_out, page_map = torch.empty_like(ref_in), torch.empty_like(ref_in)
    seen = torch.zeros((B, blocks), dtype=torch.int32, device="cuda")  # the table that the decode calls read
    batch = hb.Batch(dev_i32([L] * B), seen, *no_rings(d, B), max_ctx_len=L)
    parent, length, need = dev_i32(np.arange(B)), dev_i32([L] * B), dev_i32([blocks * P] * B)
    small = [torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(3)]
    ws_pages = torch.empty((hb.hswa_pages_workspace_need(h, pages),), dtype=torch.uint8, device="cuda")
    ws = torch.empty((hb.hswa_workspace_bytes(h, B, B, L),), dtype=torch.uint8, device="cuda")
    layers = [hb.Layer(p, False) for p in pools]

    def step():
        seen.zero_()  # page 0: nobody's
        out = [torch.empty((B, 4, 64), device="cuda") for _ in range(2)]
        hb.hswa_decode_attn(h, layers[0], batch, q, k, v, out[0], None, ws)
        if what == "fork":
            hb.hswa_pages_fork(other, ref_in, ref_out, table, held, parent, length, need, seen, *small, ws_pages)
        else:
            hb.hswa_pages_compact(other, ref_in, ref_out, table, held, seen, page_map, small[0], small[1])
        hb.hswa_decode_attn(h, layers[1], batch, q, k, v, out[1], None, ws)
        return out[1]

    hb.hswa_set_overlap(h, False)
    want = step()
    hb.hswa_set_overlap(h, True)
    assert torch.isfinite(want).all()
    for _ in range(50):
        assert torch.equal(step(), want)
    assert torch.equal(seen, table)
    no_error(h)
    no_error(other)
