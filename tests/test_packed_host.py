"""Host-side answers of the 4-bit cache and page calls that need no GPU, and the 64-bit statement the GPU tests compare with,
pinned on inputs small enough to count by hand."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from paper_2607_13095_b200 import binding as hb


def test_null_handles_are_refused():
    lib, bad = hb.load(), hb.HSWA_ERR_INVALID_ARG
    assert lib.hswa_packed_append(None, None, None, None, None, None) == bad
    assert lib.hswa_packed_read(None, None, None, None, None, None) == bad
    assert lib.hswa_packed_attn(None, None, None, 0, None, None, None, None, 0, None) == bad
    assert lib.hswa_packed_workspace_need(None, 1, 1, 1, 100, 1) == 0
    assert lib.hswa_pages_workspace_need(None, 5) == 0
    assert lib.hswa_pages_fork(None, 5, None, None, 1, None, None, 1, 1, None, None, None, None, 1, None, None, None, None, 0, None) == bad
    assert lib.hswa_pages_compact(None, 5, None, None, 1, None, None, 1, None, None, 1, None, None, None) == bad
    assert lib.hswa_pages_copy(None, 1, None, 5, 16, 1, None, None, None) == bad


def test_tensors_of_wrong_types_and_shapes_are_refused():
    with pytest.raises(AssertionError):
        hb.PackedLayer(torch.zeros((2, 2, 1, 64), dtype=torch.int8))
    with pytest.raises(AssertionError):
        hb.PackedLayer(torch.zeros((2, 3, 1, 64), dtype=torch.uint8))
    with pytest.raises(AssertionError):
        hb.PackedLayer(torch.zeros((2, 2, 1, 64, 1), dtype=torch.uint8))
    i32, z = torch.int32, lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(AssertionError, match="fewer entries"):
        hb.hswa_pages_fork(None, z(4), z(4), z(2, 3), z(2), z(2), z(2), z(2), z(3, 3), z(3), z(3), z(3), z(9))
    with pytest.raises(AssertionError):
        hb.hswa_pages_fork(None, z(4), z(5), z(2, 3), z(2), z(2), z(2), z(2), z(2, 3), z(2), z(2), z(2), z(9))
    with pytest.raises(AssertionError):
        hb.hswa_pages_compact(None, z(4), z(4), z(2, 3), z(2), z(2, 4), z(4), z(1), z(1))
    with pytest.raises(AssertionError):
        hb.hswa_pages_copy(None, [], z(4), z(4).long())
    assert i32 == torch.int32


def test_reference_codes():
    assert ref.e4m3_value([0x00, 0x01, 0x08, 0x38, 0x7e, 0xb8]).tolist() == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -1.0]
    assert np.array_equal(ref.SCALES, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    # ties go to the even code: 0.25 -> 0, 0.75 -> 1.0, 1.25 -> 1.0, 1.75 -> 2.0, 2.5 -> 2.0, 3.5 -> 4.0, 5 -> 4.0
    assert ref.LEVELS[ref.nearest(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 9.0]), ref.LEVELS)].tolist() == [0, 1, 1, 2, 2, 4, 4, 6]
    x = np.zeros((1, 32))
    x[0, :3] = 6.0, -2.5, 0.1
    n, f = ref.round_rows(x, 1.0)
    assert ref.SCALES[f].tolist() == [[1.0, 0.0]] and n[0, :4].tolist() == [7, 12, 0, 0]
    assert ref.values(n, f, 2.0)[0, :4].tolist() == [12.0, -4.0, 0.0, 0.0]
    x[0, :3] = 6e-4, 0.0, 0.0      # a / 6 = 1e-4 is below half of the smallest scale
    assert (ref.values(*ref.round_rows(x, 1.0), 1.0) == 0).all()


def test_reference_pool_rows():
    pool = np.zeros((2, 2, 1, 16 * (32 + 4)), np.uint8)
    x = np.arange(64.0)[None] % 7 - 3
    n, f = ref.round_rows(x, 0.5)
    ref.put(pool, 1, 3, 0, 16, n, f)
    got = ref.rows(pool, np.array([[1]]), 0, 4, 0, 16, 64, 0.5)
    assert np.array_equal(got[3], ref.values(n, f, 0.5)) and (got[:3] == 0).all()


def test_reference_fork():
    """Pages of 4 tokens.  Row 0 holds pages 1, 2 (6 tokens); row 1 holds 3, 4 (8 tokens), page 3 also a prefix cache's."""
    counts = np.array([0, 1, 1, 2, 1, 0, 0, 0], np.int32)
    table, held = np.array([[1, 2, 9], [3, 4, 9]], np.int32), np.array([2, 2], np.int32)
    # two children of row 0: the first takes its partly filled page, the second a copy; row 1 ends
    got = ref.fork(counts, table, held, [0, 0], [6, 6], [7, 9], 4, 3, -7)
    assert got[1].tolist() == [[1, 2, -7], [1, 0, 5]] and got[2].tolist() == [2, 3]
    assert got[3].tolist() == [-1, 2] and got[4].tolist() == [-1, 0]
    assert got[0].tolist() == [1, 2, 1, 1, 0, 1, 0, 0]
    # row 1 taken back into a page that is not its own alone: a copy; a new request
    got = ref.fork(counts, table, held, [1, -1], [3, 0], [3, 5], 4, 2, -7)
    assert got[1].tolist() == [[0, -7], [5, 6]] and got[3].tolist() == [3, -1] and got[4].tolist() == [0, -1]
    assert got[0].tolist() == [1, 0, 0, 1, 0, 1, 1, 0]
    # a shorter child first, a longer one shares the page the first would have taken
    got = ref.fork(counts, table, held, [0, 0], [2, 6], [2, 6], 4, 2, -7)
    assert got[1].tolist() == [[0, -7], [1, 5]] and got[3].tolist() == [1, 2]
    assert ref.fork(counts, table, held, [0, 0, 0, 0, 0, 0], [6] * 6, [6] * 6, 4, 2, -7) is None


def test_reference_compact():
    counts = np.array([0, 1, 0, 0, 2, 0, 1], np.int32)
    got = ref.compact(counts, np.array([[6, 4, 9]], np.int32), np.array([2]), 4, -7)
    assert got[3].tolist() == [6, 4, -1, -1] and got[4].tolist() == [0, 2, -1, -1]
    assert got[0].tolist() == [1, 1, 2, 0, 0, 0, 0] and got[1].tolist() == [[0, 2, -7]]
    assert ref.compact(counts, np.zeros((0, 3), np.int32), [], 1, 0)[0].tolist() == [1, 1, 0, 0, 2, 0, 0]
