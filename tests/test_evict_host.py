"""Host-side answers of the cross-attention and eviction calls that need no GPU, and the 64-bit statement the GPU tests
compare with, pinned on inputs small enough to count by hand."""
import numpy as np

import evict_reference as ref
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl


def test_null_handles_are_refused():
    lib = hb.load()
    assert lib.hswa_cross_workspace_need(None, 1, 1, 1, 100) == 0
    assert lib.hswa_cross_attn(None, None, None, None, None, None, None, 0, None) == hb.HSWA_ERR_INVALID_ARG
    assert lib.hswa_attn_weights(None, None, None, 0, None, None, 1.0, None, 0, None) == hb.HSWA_ERR_INVALID_ARG
    assert lib.hswa_evict_select(None, 1, None, 1, None, 1, None, 1, 0, 0, None, None, None) == hb.HSWA_ERR_INVALID_ARG
    assert lib.hswa_evict_compact(None, None, None, None, None, 1, None, 1, None, 0, None, 0, None) == hb.HSWA_ERR_INVALID_ARG


def _cache():
    """Two pages of two slots, one head of two elements; request 0 has positions 0..2 in pages 1, 0."""
    pool = np.zeros((2, 2, 1, 2, 2), np.uint16)
    one, two = wl.bf16_bits_const(1.0, (1,))[0], wl.bf16_bits_const(2.0, (1,))[0]
    pool[1, 0, 0, 0, 0] = one   # k0 = (1, 0)
    pool[1, 0, 0, 1, 1] = one   # k1 = (0, 1)
    pool[1, 1, 0, 0, 0] = one   # v0 = (1, 0)
    pool[1, 1, 0, 1, 0] = two   # v1 = (2, 0)
    return pool, np.array([[1, 0]], np.int32), one      # k2 = v2 = 0


def test_reference_cross_attention_and_weights():
    pool, table, one = _cache()
    q = np.zeros((1, 1, 2), np.uint16)
    q[0, 0, 0] = one
    out, lse, _ = ref.cross_attention(pool, table, [3], [0, 1], q, 1.0)
    e = np.e
    assert np.allclose(lse[0, 0], np.log(e + 2)) and np.allclose(out[0, 0], [(e + 2) / (e + 2), 0])
    w = ref.attn_weights(pool, table, [3], [0, 1], q, lse, 1.0, False, 0.5, np.full((1, 1, 4), 2.0, np.float32))
    assert np.allclose(w[0, 0], [1 + e / (e + 2), 1 + 1 / (e + 2), 1 + 1 / (e + 2), 2.0])
    lse = ref.self_lse(pool, table, [2], [0, 1], q, 1.0)
    w = ref.attn_weights(pool, table, [2], [0, 1], q, lse, 1.0, True, 1.0, np.full((1, 1, 4), 2.0, np.float32))
    assert np.allclose(w[0, 0], [2 + e / (e + 2), 2 + 1 / (e + 2), 1 / (e + 2), 2.0])


def test_reference_select_and_compact():
    w = np.array([[[0.5, 0.1, 0.5, np.nan, 0.5, -np.inf, 9.0]]], np.float32)
    pick = lambda keep, first=0, last=0, ctx=6: ref.evict_select(w, np.array([ctx]), np.array([keep]), 6, first, last)[0][0, 0].tolist()  # noqa: E731
    assert pick(2) == [0, 2, -1, -1, -1, -1]          # ties from the lowest position on; position 6 is not cached
    assert pick(4) == [0, 1, 2, 4, -1, -1]
    assert pick(5) == [0, 1, 2, 4, 5, -1]             # NaN ranks below minus infinity
    assert pick(2, last=1) == [0, 5, -1, -1, -1, -1]
    assert pick(1, first=2, last=2) == [0, -1, -1, -1, -1, -1]
    assert pick(9) == [0, 1, 2, 3, 4, 5]
    pool, table, _ = _cache()
    pool = np.concatenate([pool, np.full((1, 2, 1, 2, 2), 7, np.uint16)])
    got = ref.evict_compact(pool, table, np.array([[[1]]]), [1], np.array([[2]]))
    assert np.array_equal(got[2, :, 0, 0], pool[1, :, 0, 1]) and (got[2, :, 0, 1] == 7).all() and np.array_equal(got[:2], pool[:2])
