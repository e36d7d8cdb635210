"""Cross attention, accumulated attention weights and cache eviction on the GPU, against their 64-bit statement.

Tolerances.  u = 2^-24 is fp32's half step, 2^-8 bf16's (relative to the value).  Inputs are N(0, 1) in bf16.
  - A score is a sum of D <= 128 exact products of bf16 numbers in fp32, off by at most D u sum |q k| <= 128 * 2^-24 *
    128 = 2^-10 before the scale of 1 / sqrt(D) <= 1/8, i.e. 2^-13; that is the relative error of a probability, next to
    which the exponential's own (2^-22) and the rounding of lse (|lse| < 16: 2^-20) are small: S = 2^-12 covers them.
  - lse: S.  out: probabilities are rounded to bf16 (2^-8) and off by S in numerator and denominator:
    (2^-8 + 2 S) * sum_j p_j |v_j|, and 2^-8 |out| more where the output itself is bf16.
  - a weight is a sum of `rows` non-negative terms: (S + rows u) * weight, and 2 u for the decayed old value.
  - chosen positions and moved rows are equal bit for bit.
"""
import numpy as np
import pytest
import torch

import evict_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16, to_host_bits
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl

pytestmark = pytest.mark.gpu
S_ERR = 2.0 ** -12
NAN_BITS, INF_BITS = 0x7FC0, 0x7F80


def dims(G, D, P, Hkv=2):
    return wl.Dims(num_q_heads=G * Hkv, num_kv_heads=Hkv, head_dim=D, page_size=P)


class Case:
    """A paged cache of `cached` positions per request; every slot that holds none of them is NaN (V) or infinity (K)."""

    def __init__(self, d, ctx, n, seed, causal=False, spare_blocks=0):
        self.d, self.causal = d, causal
        self.ctx, self.n = np.asarray(ctx, np.int32), np.asarray(n, np.int32)
        self.cached = self.ctx + (self.n if causal else 0)
        B, P = len(ctx), d.page_size
        rng = np.random.default_rng(seed)
        self.blocks = max(1, int(-(-self.cached.max() // P))) + spare_blocks
        used = [-(-int(c) // P) for c in self.cached]
        pages = sum(used) + 3
        perm = rng.permutation(pages)
        self.free = list(perm[sum(used):])
        self.table = np.full((B, self.blocks), -1, np.int32)
        self.pool = np.empty((pages, 2, d.num_kv_heads, P, d.head_dim), np.uint16)
        self.pool[:, 0], self.pool[:, 1] = INF_BITS, NAN_BITS
        at = 0
        for r in range(B):
            self.table[r, : used[r]] = perm[at:at + used[r]]
            at += used[r]
            kv = wl.bf16_bits_normal(seed * 100 + r, (int(self.cached[r]), 2, d.num_kv_heads, d.head_dim))
            pos = np.arange(int(self.cached[r]))
            self.pool[self.table[r, pos // P], :, :, pos % P] = kv
        self.indptr = np.zeros(B + 1, np.int32)
        self.indptr[1:] = np.cumsum(self.n)
        self.q = wl.bf16_bits_normal(seed * 100 + 77, (int(self.indptr[-1]), d.num_q_heads, d.head_dim))
        self.scale = 1.0 / np.sqrt(d.head_dim)

    def batch(self, single=None, max_ctx=None, max_q=None):
        single = bool((self.n == 1).all()) if single is None else single
        B = len(self.ctx)
        ring = torch.zeros((B, self.d.ring_pages), dtype=torch.int32, device="cuda")
        head = torch.zeros((B,), dtype=torch.int32, device="cuda")
        return hb.Batch(dev_i32(self.ctx), dev_i32(self.table), ring, head, None if single else dev_i32(self.indptr),
                        max_q_len=int(self.n.max()) if max_q is None else max_q, total_q=int(self.indptr[-1]),
                        max_ctx_len=int(self.ctx.max()) if max_ctx is None else max_ctx)


def workspace(h, b):
    need = hb.hswa_cross_workspace_need(h, b.batch, b.total_q, b.max_q_len, b.c.max_ctx_len)
    return torch.empty((max(need, 256),), dtype=torch.uint8, device="cuda")


def no_error(h):
    st = hb.hswa_get_async_error(h)
    assert st[0] == hb.HSWA_OK, st


def run_cross(c, out_dtype=torch.float32, single=None, **bounds):
    h = make_handle(c.d, out_dtype)
    b = c.batch(single, **bounds)
    T = int(c.indptr[-1])
    out = torch.full((T, c.d.num_q_heads, c.d.head_dim), float("nan"), dtype=out_dtype, device="cuda")
    lse = torch.full((T, c.d.num_q_heads), float("nan"), dtype=torch.float32, device="cuda")
    hb.hswa_cross_attn(h, hb.Layer(to_dev_bf16(c.pool), False), b, to_dev_bf16(c.q), out, lse, workspace(h, b))
    no_error(h)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def check_cross(c, out, lse, out_dtype=torch.float32):
    want, want_lse, mag = ref.cross_attention(c.pool, c.table, c.ctx, c.indptr, c.q, c.scale)
    tol = (2.0 ** -8 + 2 * S_ERR) * mag + (2.0 ** -8 * np.abs(want) if out_dtype == torch.bfloat16 else 0.0)
    assert (np.abs(out - want) <= tol + 1e-7).all(), np.abs(out - want).max()
    empty = np.isinf(want_lse)
    assert (lse[empty] == -np.inf).all() and (out[empty] == 0).all()
    assert (np.abs(lse[~empty] - want_lse[~empty]) <= S_ERR).all()


SHAPES = [dims(8, 128, 64), dims(4, 64, 16, 1), dims(1, 128, 32, 3), dims(3, 64, 32), dims(5, 128, 16), dims(7, 128, 64, 1),
          dims(6, 64, 64), dims(2, 128, 64)]
EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000]


@pytest.mark.parametrize("d", SHAPES, ids=str)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_cross_decode(d, out_dtype):
    c = Case(d, EDGES, [1] * len(EDGES), seed=1)
    check_cross(c, *run_cross(c, out_dtype), out_dtype)


@pytest.mark.parametrize("d", SHAPES, ids=str)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_cross_prompt(d, out_dtype):
    n = [3, 0, 1, 40, 8, 9, 0, 16, 2, 31, 130, 1, 17, 32, 33, 7, 70]
    c = Case(d, EDGES, n, seed=2)
    check_cross(c, *run_cross(c, out_dtype), out_dtype)


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 32)], ids=str)
@pytest.mark.parametrize("ctx,n", [([9000], [1]), ([9000], [5]), ([4097, 0], [300, 20]), ([0, 0], [1, 1]), ([0], [9]), ([1], [600])])
def test_cross_few_requests(d, ctx, n):
    """Batches that need key slices, and batches without any key."""
    c = Case(d, ctx, n, seed=3)
    check_cross(c, *run_cross(c))
    if all(x == 1 for x in n):  # the same step said with row offsets
        check_cross(c, *run_cross(c, single=False))


@pytest.mark.parametrize("d", [dims(8, 128, 64, 4), dims(3, 128, 16, 2), dims(6, 64, 32)], ids=str)
def test_cross_many_requests(d):
    rng = np.random.default_rng(40)
    B = 60
    c = Case(d, np.where(rng.random(B) < 0.2, 0, rng.integers(1, 900, B)), rng.integers(0, 40, B), seed=41)
    check_cross(c, *run_cross(c))
    c = Case(d, np.where(rng.random(B) < 0.2, 0, rng.integers(1, 900, B)), np.ones(B, np.int32), seed=42)
    check_cross(c, *run_cross(c))


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16, 1)], ids=str)
@pytest.mark.parametrize("n", [1, 3, 70])
def test_cross_shows_a_nan_among_its_inputs(d, n):
    """A NaN in a cached state shows in the rows of its KV head and nowhere else."""
    c = Case(d, [300, 200], [n, n], seed=43)
    kh = d.num_kv_heads - 1
    c.pool[c.table[0, 100 // d.page_size], 0, kh, 100 % d.page_size, 5] = NAN_BITS
    out, lse = run_cross(c)
    hit = slice(kh * d.group, (kh + 1) * d.group)
    assert np.isnan(out[:n, hit]).all() and np.isnan(lse[:n, hit]).all()
    out[:n, hit] = lse[:n, hit] = 0
    assert np.isfinite(out).all() and np.isfinite(lse).all()


def test_cross_bounds_wider_than_the_batch():
    d = dims(8, 128, 64)
    c = Case(d, [100, 0, 700], [5, 2, 0], seed=4, spare_blocks=40)
    check_cross(c, *run_cross(c, max_ctx=3000, max_q=7))


@pytest.mark.parametrize("d", SHAPES, ids=str)
@pytest.mark.parametrize("top", [192, 193, 512, 513])
def test_cross_decode_of_short_states(d, top):
    """Few requests whose states are one block's: every tile has a stage of its own, or not quite."""
    c = Case(d, [top, 0, 1, 63, 64, 65, 150, top - 1], [1] * 8, seed=45)
    check_cross(c, *run_cross(c))


@pytest.mark.parametrize("d", SHAPES, ids=str)
def test_cross_requests_of_one_tile(d):
    """No request has more rows than a tile: two blocks to an SM, many key tiles through one stage, with and without slices."""
    rng = np.random.default_rng(43)
    most = 128 // d.group
    for B, top in ((2, 5000), (40, 700), (90, 300)):
        n = np.minimum(rng.integers(0, most + 1, B), 16)
        n[0] = min(most, 37)
        c = Case(d, np.where(rng.random(B) < 0.2, 0, rng.integers(1, top, B)), n, seed=44)
        check_cross(c, *run_cross(c))


def no_rings(d, B):
    return torch.zeros((B, d.ring_pages), dtype=torch.int32, device="cuda"), torch.zeros((B,), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)], ids=str)
@pytest.mark.parametrize("ctx,n", [([100, 300, 40], [1, 0, 1]), ([100, 300, 0, 40, 5], [0, 1, 1, 0, 1]), ([9000, 700, 4100], [0, 1, 1]),
                                   ([300, 9000, 20], [1, 0, 1]), ([100, 300], [0, 0]), ([600, 40, 9], [5, 0, 2])])
@pytest.mark.parametrize("pad", ["batch", "more"])
def test_cross_and_weights_of_a_padded_batch(d, ctx, n, pad):
    """Requests without a token, and rows behind the last request's: those rows are left as they were."""
    c = Case(d, ctx, n, seed=9)
    used = int(c.indptr[-1])
    total = max(used, len(ctx)) + (0 if pad == "batch" else 3)
    h = make_handle(d)
    b = hb.Batch(dev_i32(c.ctx), dev_i32(c.table), *no_rings(d, len(ctx)), dev_i32(c.indptr), max_q_len=max(1, int(c.n.max())), total_q=total,
                 max_ctx_len=int(c.ctx.max()))
    q = np.full((total, d.num_q_heads, d.head_dim), NAN_BITS, np.uint16)
    q[:used] = c.q
    out = torch.full((total, d.num_q_heads, d.head_dim), 7.0, device="cuda")
    lse = torch.full((total, d.num_q_heads), 7.0, device="cuda")
    layer = hb.Layer(to_dev_bf16(c.pool), False)
    hb.hswa_cross_attn(h, layer, b, to_dev_bf16(q), out, lse, workspace(h, b))
    no_error(h)
    assert (out[used:] == 7).all() and (lse[used:] == 7).all()
    check_cross(c, out[:used].double().cpu().numpy(), lse[:used].double().cpu().numpy())
    old = np.random.default_rng(9).random((len(ctx), d.num_kv_heads, int(c.ctx.max()) + 3)).astype(np.float32)
    w = torch.from_numpy(old).cuda()
    lse[used:] = float("nan")
    hb.hswa_attn_weights(h, layer, b, False, to_dev_bf16(q), lse, 0.5, w)
    no_error(h)
    check_weights(c, 0.5, lse[:used].cpu().numpy(), old, w.cpu().numpy())


def test_cross_single_tokens_record_values_out_of_range():
    d = dims(8, 128, 64)
    c = Case(d, [100, 300], [1, 1], seed=10)
    h = make_handle(d)
    for ctx, indptr, index, value in ([[-5, 300], None, -1, -5], [[100, 301], None, -1, 301], [[100, 300], [0, 2, 2], -2, 2]):
        b = hb.Batch(dev_i32(np.asarray(ctx, np.int32)), dev_i32(c.table), *no_rings(d, 2),
                     None if indptr is None else dev_i32(np.asarray(indptr, np.int32)), max_q_len=1, total_q=2, max_ctx_len=300)
        out = torch.zeros((2, d.num_q_heads, d.head_dim), device="cuda")
        hb.hswa_cross_attn(h, hb.Layer(to_dev_bf16(c.pool), False), b, to_dev_bf16(c.q), out, None, workspace(h, b))
        st = hb.hswa_get_async_error(h)
        assert st[0] == hb.HSWA_ERR_BOUNDS and st[2] == index and st[3] == value, st


def test_lengths_past_the_limit_are_refused():
    d = dims(8, 128, 64)
    h = make_handle(d)
    assert hb.hswa_cross_workspace_need(h, 1, 1, 1, 2 ** 30 + 1) == 0
    assert hb.hswa_cross_workspace_need(h, 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1) == 0


def run_weights(c, decay, lse, old, stride_extra=3, single=None, **bounds):
    h = make_handle(c.d)
    w = torch.from_numpy(old).cuda()
    b = c.batch(single, **bounds)
    hb.hswa_attn_weights(h, hb.Layer(to_dev_bf16(c.pool), False), b, c.causal, to_dev_bf16(c.q),
                         torch.from_numpy(lse).cuda(), decay, w)
    no_error(h)
    return w.cpu().numpy()


def weights_inputs(c, seed, extra=3):
    lse = (ref.self_lse if c.causal else lambda *a: ref.cross_attention(*a)[1])(c.pool, c.table, c.ctx, c.indptr, c.q, c.scale)
    old = np.random.default_rng(seed).random((len(c.ctx), c.d.num_kv_heads, max(int(c.cached.max()), 1) + extra)).astype(np.float32)
    return lse.astype(np.float32), old


def check_weights(c, decay, lse, old, got):
    want = ref.attn_weights(c.pool, c.table, c.ctx, c.indptr, c.q, lse, c.scale, c.causal, decay, old)
    u = 2.0 ** -24
    n_rows = int(c.n.max()) * c.d.group
    tol = (S_ERR + (n_rows + 2) * u) * want
    for r in range(len(c.ctx)):
        L = int(c.cached[r])
        assert np.array_equal(got[r, :, L:], old[r, :, L:]), "columns behind the last position were written"
        assert (np.abs(got[r, :, :L] - want[r, :, :L]) <= tol[r, :, :L] + 1e-30).all(), (r, np.abs(got - want)[r, :, :L].max())


@pytest.mark.parametrize("d", SHAPES, ids=str)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("decay", [0.0, 0.75, 1.0])
def test_weights_single_token(d, causal, decay):
    c = Case(d, EDGES, [1] * len(EDGES), seed=5, causal=causal)
    lse, old = weights_inputs(c, 5)
    if decay == 0.0:
        old[:] = np.nan  # not read
    got = run_weights(c, decay, lse, old)
    if decay == 0.0:
        for r in range(len(c.ctx)):
            assert np.isnan(got[r, :, int(c.cached[r]):]).all()
            got[r, :, int(c.cached[r]):] = 0.0
        old[:] = 0.0
    check_weights(c, decay, lse, old, got)


@pytest.mark.parametrize("d", SHAPES, ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_weights_prompt(d, causal):
    n = [3, 0, 1, 40, 8, 9, 0, 16, 2, 31, 130, 1, 17, 32, 33, 7, 70]
    c = Case(d, EDGES, n, seed=6, causal=causal)
    lse, old = weights_inputs(c, 6)
    check_weights(c, 0.9, lse, old.copy(), run_weights(c, 0.9, lse, old))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ctx,n", [([9000, 77], [1, 1]), ([3000], [16]), ([5000, 100], [17, 300]), ([600], [600]), ([0], [500])])
def test_weights_long(causal, ctx, n):
    c = Case(dims(8, 128, 64), ctx, n, seed=7, causal=causal)
    lse, old = weights_inputs(c, 7)
    got = run_weights(c, 1.0, lse, old)
    check_weights(c, 1.0, lse, old.copy(), got)
    assert np.array_equal(got, run_weights(c, 1.0, lse, old)), "repeated calls differ"


@pytest.mark.parametrize("d", [dims(8, 128, 64, 8), dims(5, 64, 16, 3), dims(7, 128, 32, 8)], ids=str)
@pytest.mark.parametrize("kind", ["single", "few", "many", "mixed"])
@pytest.mark.parametrize("causal", [False, True])
def test_weights_many_requests(d, kind, causal):
    """More (request, KV head) pairs than blocks: a block's share crosses requests, with and without rows, whose Q tiles fit
    shared memory or are streamed."""
    rng = np.random.default_rng(70)
    B = 50
    n = {"single": np.ones(B), "few": rng.integers(0, 9, B), "many": rng.integers(0, 70, B),
         "mixed": np.where(rng.random(B) < 0.3, 0, np.where(rng.random(B) < 0.1, rng.integers(90, 200, B), rng.integers(1, 30, B)))}[kind]
    ctx = np.where(rng.random(B) < 0.2, rng.integers(0, 3, B), rng.integers(1, 700, B))
    c = Case(d, ctx, n.astype(np.int32), seed=71, causal=causal)
    lse, old = weights_inputs(c, 72)
    got = run_weights(c, 0.5, lse, old)
    check_weights(c, 0.5, lse, old.copy(), got)
    assert np.array_equal(got, run_weights(c, 0.5, lse, old)), "repeated calls differ"


def test_weights_of_a_causal_step_add_up_to_its_rows():
    """Every row's probabilities sum to one: the weights of a head pair add up to the rows it has."""
    c = Case(dims(8, 128, 64), [700, 0, 5], [33, 64, 1], seed=8, causal=True)
    lse, old = weights_inputs(c, 8)
    got = run_weights(c, 0.0, lse, old)
    for r in range(3):
        total = got[r, :, : int(c.cached[r])].sum(axis=-1, dtype=np.float64)
        assert np.allclose(total, c.n[r] * c.d.group, rtol=S_ERR + 600 * 2.0 ** -24, atol=0), total


# ---------------------------------------------------------------------------------------------------------------------
def run_select(w, ctx, keep, max_keep, first=0, last=0, max_ctx=None):
    B, Hkv, _ = w.shape
    h = make_handle(wl.Dims(Hkv * 2, Hkv, 64, 16))
    idx = torch.full((B, Hkv, max_keep), 7, dtype=torch.int32, device="cuda")
    kept = torch.full((B,), 7, dtype=torch.int32, device="cuda")
    hb.hswa_evict_select(h, B, dev_i32(ctx), int(max(ctx)) if max_ctx is None else max_ctx, torch.from_numpy(w).cuda(), dev_i32(keep), idx, kept,
                         protect_first=first, protect_last=last)
    no_error(h)
    return idx.cpu().numpy(), kept.cpu().numpy()


def check_select(w, ctx, keep, max_keep, first=0, last=0, max_ctx=None):
    got = run_select(w, ctx, keep, max_keep, first, last, max_ctx)
    want = ref.evict_select(w, np.asarray(ctx), np.asarray(keep), max_keep, first, last)
    assert np.array_equal(got[1], want[1])
    assert np.array_equal(got[0], want[0])


CTX = [0, 1, 2, 31, 32, 33, 100, 1023, 1024, 1025, 5000]


@pytest.mark.parametrize("first,last", [(0, 0), (4, 32), (1, 0), (0, 2000)])
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd values"])
def test_select(first, last, kind):
    rng = np.random.default_rng(9)
    w = rng.random((len(CTX), 3, 5003)).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 6).astype(np.float32)
    if kind == "equal":
        w[:] = 0.25
    if kind == "odd values":
        w = (w * 2 - 1).astype(np.float32)
        pick = rng.random(w.shape)
        w[pick < 0.3] = np.nan
        w[(pick >= 0.3) & (pick < 0.4)] = np.inf
        w[(pick >= 0.4) & (pick < 0.5)] = -np.inf
        w[(pick >= 0.5) & (pick < 0.55)] = 0.0
        w[(pick >= 0.55) & (pick < 0.6)] = -0.0
        w[(pick >= 0.6) & (pick < 0.62)] = np.finfo(np.float32).max
        w[(pick >= 0.62) & (pick < 0.64)] = -np.finfo(np.float32).max
        w[(pick >= 0.64) & (pick < 0.66)] = 1e-45
    for keep in ([0, 0, 1, 5, 32, 32, 64, 512, 1024, 3, 2500], [9] * len(CTX), [5000] * len(CTX)):
        check_select(w, CTX, keep, max(keep), first, last)
    check_select(w, CTX, [3] * len(CTX), 17, first, last, max_ctx=5003)


@pytest.mark.parametrize("batch,lo,hi,keep", [(100, 0, 3000, 300), (90, 1000, 9000, 2048), (100, 3000, 40000, 900), (85, 30000, 60000, 4096),
                                              (80, 100000, 140000, 512), (80, 50000, 70000, 12000), (60, 2000, 30000, 64), (6, 100000, 200000, 18000),
                                              (6, 20000, 50000, 24000)])
@pytest.mark.parametrize("kind", ["random", "skewed"])
def test_select_more_rows_than_sms(batch, lo, hi, keep, kind):
    """And just fewer: blocks of either size, several to an SM or one; weights spread evenly and as attention spreads them."""
    rng = np.random.default_rng(12)
    w = rng.random((batch, 2, hi + 1), dtype=np.float32)
    if kind == "skewed":
        w = np.exp(np.float32(9) * w) * (rng.random(w.shape, dtype=np.float32) < 0.7)
    ctx = rng.integers(lo, hi + 1, batch).astype(np.int32)
    check_select(w, ctx, np.where(rng.random(batch) < 0.2, keep // 3, keep), keep, 4, 64, hi)


@pytest.mark.parametrize("ctx", [16383, 16384, 16385, 49152, 65536, 200001, 262144, 300000])
def test_select_long(ctx):
    rng = np.random.default_rng(10)
    w = np.exp(2 * rng.standard_normal((2, 2, ctx + 1)) - 6).astype(np.float32)
    w[rng.random(w.shape) < 0.06] = 0.0
    check_select(w, [ctx, ctx // 3], [ctx // 7, 1], ctx // 7, 4, 128)
    check_select(np.round(w, 3), [ctx - 1, ctx], [1000, ctx - 5], ctx, 0, 1)


# ---------------------------------------------------------------------------------------------------------------------
def compact_case(d, ctx, keep, seed, max_keep=None):
    c = Case(d, ctx, [1] * len(ctx), seed=seed)
    rng = np.random.default_rng(seed)
    kept = np.minimum(keep, ctx).astype(np.int32)
    max_keep = max(1, int(max(keep))) if max_keep is None else max_keep
    idx = np.full((len(ctx), d.num_kv_heads, max_keep), -1, np.int32)
    for r in range(len(ctx)):
        for kh in range(d.num_kv_heads):
            idx[r, kh, : kept[r]] = np.sort(rng.permutation(int(ctx[r]))[: kept[r]])
    blocks = -(-max_keep // d.page_size)
    more = np.empty((len(ctx) * blocks, *c.pool.shape[1:]), np.uint16)
    more[:, 0], more[:, 1] = INF_BITS, NAN_BITS
    dst = (c.pool.shape[0] + rng.permutation(len(ctx) * blocks)).astype(np.int32).reshape(len(ctx), blocks)
    c.pool = np.concatenate([c.pool, more])
    return c, idx, kept, dst


@pytest.mark.parametrize("d", SHAPES, ids=str)
@pytest.mark.parametrize("with_weights", [True, False])
def test_compact(d, with_weights):
    ctx = [0, 1, 2, 33, 64, 65, 300, 1000]
    c, idx, kept, dst = compact_case(d, ctx, [5, 1, 1, 16, 64, 17, 129, 700], seed=11)
    h = make_handle(d)
    pool = to_dev_bf16(c.pool)
    rng = np.random.default_rng(12)
    w = rng.random((len(ctx), d.num_kv_heads, 1003)).astype(np.float32)
    out = np.full((len(ctx), d.num_kv_heads, idx.shape[2] + 2), -3.0, np.float32)
    w_out = torch.from_numpy(out).cuda()
    hb.hswa_evict_compact(h, hb.Layer(pool, False), c.batch(), dev_i32(idx), dev_i32(kept), dev_i32(dst),
                          torch.from_numpy(w).cuda() if with_weights else None, w_out if with_weights else None)
    no_error(h)
    assert np.array_equal(to_host_bits(pool), ref.evict_compact(c.pool, c.table, idx, kept, dst))
    for r in range(len(ctx)):
        for kh in range(d.num_kv_heads):
            if with_weights:
                out[r, kh, : kept[r]] = w[r, kh, idx[r, kh, : kept[r]]]
    assert np.array_equal(w_out.cpu().numpy(), out)


def test_compact_pages_far_into_a_large_pool():
    """Page offsets past 2^32 bytes (and 2^31 elements), for the whole run: weights, choice, move, attention."""
    d = dims(8, 128, 64)
    far = 5_000_000_000 // (d.page_bytes) + 1
    c = Case(d, [200], [1], seed=13)
    small, table = c.pool, c.table
    pool = torch.empty((far + small.shape[0] + 2, 2, d.num_kv_heads, 64, 128), dtype=torch.bfloat16, device="cuda")
    pool[far:far + small.shape[0]] = to_dev_bf16(small)
    c.table = np.where(table >= 0, table + far, table).astype(np.int32)
    h, layer, b = make_handle(d), hb.Layer(pool, False), c.batch()
    q, out = to_dev_bf16(c.q), torch.zeros((1, 16, 128), device="cuda")
    lse = torch.zeros((1, 16), device="cuda")
    hb.hswa_cross_attn(h, layer, b, q, out, lse, workspace(h, b))
    want, want_lse, mag = ref.cross_attention(small, table, c.ctx, c.indptr, c.q, c.scale)
    assert (np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -8 + 2 * S_ERR) * mag + 1e-7).all()
    w = torch.zeros((1, 2, 200), device="cuda")
    hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
    want_w = ref.attn_weights(small, table, c.ctx, c.indptr, c.q, lse.cpu().numpy(), c.scale, False, 0.0, np.zeros((1, 2, 200), np.float32))
    assert np.allclose(w.cpu().numpy(), want_w, rtol=2 * S_ERR, atol=0)
    idx = torch.arange(0, 200, 4, dtype=torch.int32, device="cuda").expand(1, 2, 50).contiguous()
    dst = dev_i32([[far + small.shape[0] + 1]])
    hb.hswa_evict_compact(h, layer, b, idx, dev_i32([50]), dst)
    no_error(h)
    got = to_host_bits(pool[far + small.shape[0] + 1])
    pos = np.arange(0, 200, 4)
    assert np.array_equal(got[:, :, :50], small[table[0, pos // 64], :, :, pos % 64].transpose(1, 2, 0, 3))


# ---------------------------------------------------------------------------------------------------------------------
def test_run_of_decode_steps_with_eviction():
    """Decode steps that accumulate weights, an eviction, and more decode steps on the compacted cache: every output is that
    of attention over the kept rows.  The second request's prompt pages are shared with the first and must not change."""
    d = dims(8, 128, 64)
    P, steps = 64, 4
    ctx0 = np.array([500, 300], np.int32)
    c = Case(d, ctx0, [1, 1], seed=14, spare_blocks=2)
    blocks = c.table.shape[1]
    shared = 2
    pages = c.pool.shape[0]
    extra = np.empty((24, *c.pool.shape[1:]), np.uint16)
    extra[:, 0], extra[:, 1] = INF_BITS, NAN_BITS
    c.pool = np.concatenate([c.pool, extra])
    c.table[1, :shared] = c.table[0, :shared]  # a common prefix of 128 tokens
    free = list(range(pages, pages + 24))
    for r in range(2):
        for k in range(blocks):
            if c.table[r, k] < 0 or (k >= -(-int(ctx0[r]) // P)):
                c.table[r, k] = free.pop()
    h = make_handle(d)
    pool = to_dev_bf16(c.pool)
    layer = hb.Layer(pool, False)
    K = [ref.rows(c.pool, c.table, r, int(ctx0[r]), 0) for r in range(2)]
    V = [ref.rows(c.pool, c.table, r, int(ctx0[r]), 1) for r in range(2)]
    K = [[K[r][:, kh] for kh in range(2)] for r in range(2)]
    V = [[V[r][:, kh] for kh in range(2)] for r in range(2)]
    W = [[np.zeros(int(ctx0[r])) for kh in range(2)] for r in range(2)]
    ctx, table = dev_i32(ctx0), dev_i32(c.table)
    ring, head = torch.zeros((2, d.ring_pages), dtype=torch.int32, device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")
    weights = torch.zeros((2, 2, 600), device="cuda")
    ws = torch.empty((hb.hswa_workspace_bytes(h, 2, 2, 600),), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros((2, 16, 128), device="cuda"), torch.zeros((2, 16), device="cuda")

    def step(k, bound):
        q, kn, vn = (wl.bf16_bits_normal(900 + 10 * k + i, (2, n, 128)) for i, n in enumerate((16, 2, 2)))
        b = hb.Batch(ctx, table, ring, head, None, max_ctx_len=bound)
        hb.hswa_decode_attn(h, layer, b, to_dev_bf16(q), to_dev_bf16(kn), to_dev_bf16(vn), out, lse, ws)
        hb.hswa_attn_weights(h, layer, b, True, to_dev_bf16(q), lse, 1.0, weights)
        hb.hswa_step_advance(h, 2, ctx, head)
        no_error(h)
        got = out.double().cpu().numpy()
        Q = wl.bits_to_f64(q)
        for r in range(2):
            for kh in range(2):
                K[r][kh] = np.concatenate([K[r][kh], wl.bits_to_f64(kn)[r, kh][None]])
                V[r][kh] = np.concatenate([V[r][kh], wl.bits_to_f64(vn)[r, kh][None]])
                W[r][kh] = np.append(W[r][kh], 0.0)
                for hh in range(kh * 8, kh * 8 + 8):
                    s = c.scale * (K[r][kh] @ Q[r, hh])
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    W[r][kh] += p
                    assert np.abs(got[r, hh] - p @ V[r][kh]).max() <= (2.0 ** -8 + 2 * S_ERR) * (p @ np.abs(V[r][kh])).max(), (k, r, hh)

    for k in range(steps):
        step(k, 520)
    got_w = weights.cpu().numpy()
    for r in range(2):
        for kh in range(2):
            # (the decode kernels' lse sums rounded probabilities: 2^-8 more)
            assert np.allclose(got_w[r, kh, : len(W[r][kh])], W[r][kh], rtol=2.0 ** -8 + 2 * S_ERR, atol=0)
    idx = torch.zeros((2, 2, 200), dtype=torch.int32, device="cuda")
    kept = torch.zeros((2,), dtype=torch.int32, device="cuda")
    hb.hswa_evict_select(h, 2, ctx, 520, weights, dev_i32([200, 130]), idx, kept, protect_first=4, protect_last=16)
    want_idx, want_kept = ref.evict_select(got_w, ctx0 + steps, np.array([200, 130]), 200, 4, 16)
    assert np.array_equal(idx.cpu().numpy(), want_idx) and np.array_equal(kept.cpu().numpy(), want_kept)
    dst = dev_i32([[free.pop() for _ in range(4)], [free.pop() for _ in range(4)]])
    w2 = torch.zeros_like(weights)
    before = to_host_bits(pool)
    hb.hswa_evict_compact(h, layer, hb.Batch(ctx, table, ring, head, None, max_ctx_len=520), idx, kept, dst, weights, w2)
    no_error(h)
    assert np.array_equal(to_host_bits(pool), ref.evict_compact(before, c.table, want_idx, want_kept, dst.cpu().numpy()))
    for r in range(2):
        for kh in range(2):
            at = want_idx[r, kh, : want_kept[r]]
            K[r][kh], V[r][kh], W[r][kh] = K[r][kh][at], V[r][kh][at], W[r][kh][at]
    ctx.copy_(kept)
    table, weights = dst, w2
    for k in range(steps, 2 * steps):
        step(k, 210)


def test_run_of_cross_attention_with_eviction_of_states():
    """Encoder states appended to pages, a decoder prompt, its weights, an eviction, and a decode step on what is left."""
    d = dims(5, 128, 32)
    lens, n = [150, 0, 77], [20, 3, 0]
    c = Case(d, lens, n, seed=15)
    h, b = make_handle(d), c.batch()
    pool = to_dev_bf16(c.pool)
    grown = torch.cat([pool, torch.full((6, *pool.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")])
    layer = hb.Layer(grown, False)
    T = int(c.indptr[-1])
    out, lse = torch.zeros((T, 10, 128), device="cuda"), torch.zeros((T, 10), device="cuda")
    hb.hswa_cross_attn(h, layer, b, to_dev_bf16(c.q), out, lse, workspace(h, b))
    w = torch.zeros((3, 2, 150), device="cuda")
    hb.hswa_attn_weights(h, layer, b, False, to_dev_bf16(c.q), lse, 0.0, w)
    idx, kept = torch.zeros((3, 2, 40), dtype=torch.int32, device="cuda"), torch.zeros((3,), dtype=torch.int32, device="cuda")
    hb.hswa_evict_select(h, 3, b.ctx_len, 150, w, dev_i32([40, 40, 40]), idx, kept)
    dst = dev_i32(pool.shape[0] + np.arange(6).reshape(3, 2))
    hb.hswa_evict_compact(h, layer, b, idx, kept, dst)
    after = Case(d, [40, 0, 40], [1, 1, 1], seed=16)
    after.pool, after.table, after.ctx = to_host_bits(grown), dst.cpu().numpy(), kept.cpu().numpy()
    no_error(h)
    assert list(after.ctx) == [40, 0, 40]
    pos = idx.cpu().numpy()[0, 0]
    assert np.array_equal(ref.rows(after.pool, after.table, 0, 40, 1)[:, 0], ref.rows(c.pool, c.table, 0, 150, 1)[pos, 0])
    check_cross(after, *run_cross(after))


# ---------------------------------------------------------------------------------------------------------------------
def test_captured_run_replays_on_new_data():
    """The whole run on a side stream, captured into a graph and replayed on changed inputs, equals an eager run on them."""
    d = dims(8, 128, 64)
    results = []
    for seed in (20, 21):
        c = Case(d, [300, 200], [4, 3], seed=seed)
        results.append(c)
    c = results[0]
    h, b = make_handle(d), c.batch()
    grown = torch.cat([to_dev_bf16(c.pool), torch.zeros((4, 2, 2, 64, 128), dtype=torch.bfloat16, device="cuda")])
    layer, q = hb.Layer(grown, False), to_dev_bf16(c.q)
    out, lse, ws = torch.zeros((7, 16, 128), device="cuda"), torch.zeros((7, 16), device="cuda"), workspace(h, b)
    w = torch.zeros((2, 2, 300), device="cuda")
    idx, kept = torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")
    keep, dst = dev_i32([100, 90]), dev_i32(len(c.pool) + np.arange(4).reshape(2, 2))

    def run():
        hb.hswa_cross_attn(h, layer, b, q, out, lse, ws)
        hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.5, w)
        hb.hswa_evict_select(h, 2, b.ctx_len, 300, w, keep, idx, kept, protect_last=3)
        hb.hswa_evict_compact(h, layer, b, idx, kept, dst)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (30, 31):
        g = torch.Generator(device="cuda").manual_seed(seed)
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        w.zero_()
        eager = []
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        eager = [t.clone() for t in (out, lse, w, idx, kept, grown)]
        for t in (out, lse, w):
            t.zero_()
        idx.zero_()
        grown[-4:] = 0
        graph.replay()
        torch.cuda.synchronize()
        got = [out, lse, w, idx, kept, grown]
        for a, e in zip(got, eager):
            assert torch.equal(a.contiguous().view(torch.uint8), e.contiguous().view(torch.uint8))
    no_error(h)


# ---------------------------------------------------------------------------------------------------------------------
def refused(status, fn, *a, **k):
    with pytest.raises(hb.HswaError) as e:
        fn(*a, **k)
    assert e.value.status == status, e.value


def test_refusals():
    d = dims(8, 128, 64)
    c = Case(d, [9000, 5], [2, 1], seed=17)
    h, b = make_handle(d), c.batch()
    layer, q = hb.Layer(to_dev_bf16(c.pool), False), to_dev_bf16(c.q)
    out, lse = torch.zeros((3, 16, 128), device="cuda"), torch.zeros((3, 16), device="cuda")
    ws = workspace(h, b)
    assert hb.hswa_cross_workspace_need(h, 2, 3, 2, 9000) > 0
    INV, WS = hb.HSWA_ERR_INVALID_ARG, hb.HSWA_ERR_WORKSPACE
    refused(WS, hb.hswa_cross_attn, h, layer, b, q, out, lse, None)
    refused(WS, hb.hswa_cross_attn, h, layer, b, q, out, lse, ws[: ws.numel() - 256])
    swa = hb.Layer(layer.pool, True)
    refused(INV, hb.hswa_cross_attn, h, swa, b, q, out, lse, ws)
    refused(INV, hb.hswa_cross_attn, h, layer, c.batch(max_ctx=c.blocks * 64 + 1), q, out, lse, ws)
    w = torch.zeros((2, 2, 9002), device="cuda")
    refused(INV, hb.hswa_attn_weights, h, swa, b, False, q, lse, 1.0, w)
    refused(INV, hb.hswa_attn_weights, h, layer, b, False, q, lse, -1.0, w)
    refused(INV, hb.hswa_attn_weights, h, layer, b, False, q, lse, float("nan"), w)
    refused(INV, hb.hswa_attn_weights, h, layer, b, False, q, lse, float("inf"), w)
    refused(INV, hb.hswa_attn_weights, h, layer, b, False, q, lse, 1.0, w[..., :8999].contiguous())
    ctx, keep = dev_i32([9000, 5]), dev_i32([8, 8])
    idx, kept = torch.zeros((2, 2, 8), dtype=torch.int32, device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")
    refused(INV, hb.hswa_evict_select, h, 2, ctx, 9003, w, keep, idx, kept)
    refused(INV, hb.hswa_evict_select, h, 2, ctx, 9000, w, keep, idx, kept, protect_first=-1)
    refused(INV, hb.hswa_evict_select, h, 2, ctx, 9000, w, keep, idx, kept, protect_last=-1)
    refused(INV, hb.hswa_evict_select, h, 2, ctx, 9000, w, keep, idx, ctx)
    refused(INV, hb.hswa_evict_compact, h, layer, b, idx, kept, b.block_table)
    refused(INV, hb.hswa_evict_compact, h, swa, b, idx, kept, dev_i32([[0], [1]]))
    refused(INV, hb.hswa_evict_compact, h, layer, b, idx, kept, dev_i32(np.zeros((2, 0))))
    refused(INV, hb.hswa_evict_compact, h, layer, b, idx, kept, dev_i32([[0], [1]]), w, None)
    refused(INV, hb.hswa_evict_compact, h, layer, b, idx, kept, dev_i32([[0], [1]]), w, w)
    refused(INV, hb.hswa_evict_compact, h, layer, b, idx, kept, dev_i32([[0], [1]]), w, torch.zeros((2, 2, 7), device="cuda"))
    no_error(h)


def test_values_out_of_range_are_recorded():
    """Bad ids and lengths end in the error word; nothing is read or written outside, and later calls work."""
    d = dims(8, 128, 64)
    c = Case(d, [300, 100], [2, 1], seed=18)
    h = make_handle(d)
    pool = to_dev_bf16(c.pool)
    layer, q = hb.Layer(pool, False), to_dev_bf16(c.q)
    out, lse = torch.zeros((3, 16, 128), device="cuda"), torch.zeros((3, 16), device="cuda")
    w = torch.zeros((2, 2, 400), device="cuda")
    BOUNDS = hb.HSWA_ERR_BOUNDS
    good = c.table.copy()
    for bad_page in (-5, len(c.pool)):
        c.table = good.copy()
        c.table[0, 2] = bad_page
        b = c.batch()
        hb.hswa_cross_attn(h, layer, b, q, out, lse, workspace(h, b))
        assert hb.hswa_get_async_error(h) == (BOUNDS, 0, 2, bad_page)
        hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
        assert hb.hswa_get_async_error(h) == (BOUNDS, 0, 2, bad_page)
        idx = dev_i32(np.full((2, 2, 1), 130))
        idx[1] = 3
        hb.hswa_evict_compact(h, layer, b, idx, dev_i32([1, 1]), dev_i32([[len(c.pool) - 1], [len(c.pool) - 2]]))
        assert hb.hswa_get_async_error(h)[0] == BOUNDS
    c.table = good
    b = c.batch(max_ctx=299)  # request 0 is longer than the bound
    hb.hswa_cross_attn(h, layer, b, q, out, lse, workspace(h, b))
    assert hb.hswa_get_async_error(h) == (BOUNDS, 0, -1, 300)
    hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
    assert hb.hswa_get_async_error(h) == (BOUNDS, 0, -1, 300)
    hb.hswa_attn_weights(h, layer, c.batch(), True, q, lse, 0.0, w[..., :301].contiguous())  # 302 positions
    assert hb.hswa_get_async_error(h) == (BOUNDS, 0, -3, 302)
    b = c.batch(max_q=1)
    hb.hswa_cross_attn(h, layer, b, q, out, lse, workspace(h, b))
    assert hb.hswa_get_async_error(h) == (BOUNDS, 0, -2, 2)
    hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
    assert hb.hswa_get_async_error(h) == (BOUNDS, 0, -2, 2)
    idx, kept = torch.zeros((2, 2, 8), dtype=torch.int32, device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")
    hb.hswa_evict_select(h, 2, dev_i32([300, 100]), 250, w, dev_i32([8, 8]), idx, kept)
    assert hb.hswa_get_async_error(h) == (BOUNDS, 0, -1, 300)
    hb.hswa_evict_select(h, 2, dev_i32([30, 100]), 250, w, dev_i32([8, 9]), idx, kept)
    assert hb.hswa_get_async_error(h) == (BOUNDS, 1, -2, 9)
    for idx_bad in (-1, 300):
        idx = dev_i32(np.full((2, 2, 1), 3))
        idx[0, 0, 0] = idx_bad
        hb.hswa_evict_compact(h, layer, c.batch(), idx, dev_i32([1, 1]), dev_i32([[len(c.pool) - 1], [len(c.pool) - 2]]))
        assert hb.hswa_get_async_error(h) == (BOUNDS, 0, 0, idx_bad)
    hb.hswa_evict_compact(h, layer, c.batch(), idx, dev_i32([1, 1]), dev_i32([[len(c.pool)], [-1]]))
    assert hb.hswa_get_async_error(h)[0] == BOUNDS
    check_cross(c, *run_cross(c))


def test_empty_calls():
    d = dims(8, 128, 64)
    c = Case(d, [100], [1], seed=19)
    h, layer = make_handle(d), hb.Layer(to_dev_bf16(c.pool), False)
    w = torch.full((1, 2, 200), 2.0, device="cuda")
    none = torch.zeros((0, 16, 128), dtype=torch.bfloat16, device="cuda")
    b = hb.Batch(dev_i32([100]), dev_i32(c.table), torch.zeros((1, d.ring_pages), dtype=torch.int32, device="cuda"), dev_i32([0]),
                 dev_i32([0, 0]), max_q_len=0, total_q=0, max_ctx_len=100)
    hb.hswa_cross_attn(h, layer, b, none, torch.zeros((0, 16, 128), device="cuda"), None, None)
    hb.hswa_attn_weights(h, layer, b, True, none, torch.zeros((0, 16), device="cuda"), 0.5, w)  # a step without rows only decays
    no_error(h)
    want = torch.full((1, 2, 200), 2.0)
    want[..., :100] = 1.0
    assert torch.equal(w.cpu(), want)


def test_tensors_too_small_for_the_batch_are_refused():
    d = dims(8, 128, 64)
    c = Case(d, [100, 200], [1, 1], seed=20)
    h, layer, b = make_handle(d), hb.Layer(to_dev_bf16(c.pool), False), c.batch()
    q, out, lse = to_dev_bf16(c.q), torch.zeros((2, 16, 128), device="cuda"), torch.zeros((2, 16), device="cuda")
    w, idx, kept = torch.zeros((2, 2, 200), device="cuda"), dev_i32(np.zeros((2, 2, 4), np.int32)), dev_i32([1, 1])
    dst = dev_i32([[0], [1]])
    for bad in ((q[:1], out, lse), (q, out[:1], lse), (q, out, lse[:1])):
        with pytest.raises(AssertionError):
            hb.hswa_cross_attn(h, layer, b, *bad)
    for bad in ((q[:1], lse, 0.0, w), (q, lse[:1], 0.0, w), (q, lse, 0.0, w[:1]), (q, lse, 0.0, w[:, :1])):
        with pytest.raises(AssertionError):
            hb.hswa_attn_weights(h, layer, b, False, *bad)
    for bad in ((kept[:1], 200, w, kept, idx, kept.clone()), (kept, 200, w, kept[:1], idx, kept.clone()), (kept, 200, w, kept, idx, kept[:1]),
                (kept, 200, w[:1], kept, idx, kept.clone()), (kept, 200, w, kept, idx[:, :1], kept.clone())):
        with pytest.raises(AssertionError):
            hb.hswa_evict_select(h, 2, *bad)
    for bad in ((idx[:1], kept, dst), (idx[:, :1], kept, dst), (idx, kept[:1], dst), (idx, kept, dst[:1]), (idx, kept, dst, w[:1], w.clone()),
                (idx, kept, dst, w, w[:, :1].clone())):
        with pytest.raises(AssertionError):
            hb.hswa_evict_compact(h, layer, b, *bad)
    no_error(h)
