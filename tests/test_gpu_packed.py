"""The 4-bit cache on the GPU, against its 64-bit statement.

Tolerances.  u = 2^-24 is fp32's half step, 2^-11 fp16's, 2^-8 bf16's (relative to the value).  Inputs are N(0, 1) in bf16.
  - held codes: equal.  The two scales are powers of two or have two significant bits, so that quotients halfway between two
    codes are exact in 32 bits as well.  Read back: the value rounded to bf16 (2^-8; exact where the scale is a power of two:
    2 + 4 significant bits).
  - A score is a sum of D <= 128 products in fp32 of fp16 values, each exact: off by at most D u sum |q k| <= 128 * 2^-24 *
    128 = 2^-10 before the scale of 1 / sqrt(D) <= 1/8, i.e. 2^-13, which is the relative error of a probability; with the
    exponential's own (2^-22) and the rounding of lse (2^-20) S = 2^-12 covers it.
  - out: probabilities are rounded to fp16, 2^-11 of their value or, below 2^-14 of the row's running maximum's, 2^-25 of that,
    whose share of the row's sum is at most 1: 2^-25 per key; sums of L terms in fp32 add L u.  Together
    (2^-11 + 2 S + L u) sum_j p_j |v_j| + L 2^-25 max |v|, and 2^-8 |out| more where the output itself is bf16.
"""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16, to_host_bits
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl

pytestmark = pytest.mark.gpu
S_ERR = 2.0 ** -12


def dims(G, D, P, Hkv=2):
    return wl.Dims(num_q_heads=G * Hkv, num_kv_heads=Hkv, head_dim=D, page_size=P)


def no_error(h):
    st = hb.hswa_get_async_error(h)
    assert st[0] == hb.HSWA_OK, st


def no_rings(d, B):
    return torch.zeros((B, d.ring_pages), dtype=torch.int32, device="cuda"), torch.zeros((B,), dtype=torch.int32, device="cuda")


class Case:
    """A 4-bit cache of `cached` positions per request; all other slots hold codes of any value and scales of NaN."""

    def __init__(self, d, ctx, n, seed, causal=True, spare_blocks=0, k_scale=1.0, v_scale=0.5):
        self.d, self.causal, self.k_scale, self.v_scale = d, causal, k_scale, v_scale
        self.ctx, self.n = np.asarray(ctx, np.int32), np.asarray(n, np.int32)
        self.cached = self.ctx + (self.n if causal else 0)
        B, P, D, H = len(ctx), d.page_size, d.head_dim, d.num_kv_heads
        rng = np.random.default_rng(seed)
        self.blocks = max(1, int(-(-self.cached.max() // P))) + spare_blocks
        used = [-(-int(c) // P) for c in self.cached]
        pages = sum(used) + 3
        perm = rng.permutation(pages)
        self.table = np.full((B, self.blocks), -1, np.int32)
        self.pool = rng.integers(0, 256, (pages, 2, H, P * (D // 2 + D // 16)), dtype=np.uint8)
        self.pool[..., P * D // 2:] = 0x7f
        at = 0
        self.kv = []
        for r in range(B):
            self.table[r, : used[r]] = perm[at:at + used[r]]
            at += used[r]
            L = int(self.cached[r])
            both = []
            for which, scale in ((0, k_scale), (1, v_scale)):
                n4, f = ref.round_rows(wl.bits_to_f64(wl.bf16_bits_normal(seed * 100 + 2 * r + which, (L, H, D))), scale)
                for j in range(L):
                    ref.put(self.pool, self.table[r, j // P], j % P, which, P, n4[j], f[j])
                both.append(ref.values(n4, f, scale))
            self.kv.append(both)
        self.indptr = np.zeros(B + 1, np.int32)
        self.indptr[1:] = np.cumsum(self.n)
        self.q = wl.bf16_bits_normal(seed * 100 + 77, (int(self.indptr[-1]), d.num_q_heads, D))
        self.scale = 1.0 / np.sqrt(D)

    def batch(self, single=None, max_ctx=None, max_q=None):
        single = bool((self.n == 1).all()) if single is None else single
        return hb.Batch(dev_i32(self.ctx), dev_i32(self.table), *no_rings(self.d, len(self.ctx)), None if single else dev_i32(self.indptr),
                        max_q_len=int(self.n.max()) if max_q is None else max_q, total_q=int(self.indptr[-1]),
                        max_ctx_len=int(self.ctx.max()) if max_ctx is None else max_ctx)

    def layer(self):
        return hb.PackedLayer(torch.from_numpy(self.pool).cuda(), self.k_scale, self.v_scale)

    def want(self, sm_scale=None):
        T = int(self.indptr[-1])
        out, mag = (np.zeros((T, self.d.num_q_heads, self.d.head_dim)) for _ in range(2))
        lse, slack = np.full((T, self.d.num_q_heads), -np.inf), np.zeros((T, 1, 1))
        q = wl.bits_to_f64(self.q)
        for r, (K, V) in enumerate(self.kv):
            a, b, c = self.indptr[r], self.indptr[r + 1], int(self.ctx[r])
            ends = [c + i + 1 if self.causal else c for i in range(b - a)]
            out[a:b], lse[a:b], mag[a:b] = ref.attention(K, V, q[a:b], ends, self.scale if sm_scale is None else sm_scale)
            slack[a:b] = len(K) * (2.0 ** -25 * (np.abs(V).max() if len(V) else 0.0))
            mag[a:b] *= 2.0 ** -11 + 2 * S_ERR + len(K) * 2.0 ** -24
        return out, lse, mag + slack


def workspace(h, b, causal):
    need = hb.hswa_packed_workspace_need(h, b.batch, b.total_q, b.max_q_len, b.c.max_ctx_len, causal)
    return torch.empty((max(need, 256),), dtype=torch.uint8, device="cuda")


def run(c, out_dtype=torch.float32, single=None, q=None, h=None, **bounds):
    h = h or make_handle(c.d, out_dtype)
    b = c.batch(single, **bounds)
    T = int(c.indptr[-1])
    out = torch.full((T, c.d.num_q_heads, c.d.head_dim), float("nan"), dtype=out_dtype, device="cuda")
    lse = torch.full((T, c.d.num_q_heads), float("nan"), dtype=torch.float32, device="cuda")
    ws = workspace(h, b, c.causal)
    ws.fill_(255)  # (partials of NaN, were any read that no block wrote)
    hb.hswa_packed_attn(h, c.layer(), b, c.causal, to_dev_bf16(c.q if q is None else q), out, lse, ws)
    no_error(h)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def check(c, out, lse, out_dtype=torch.float32, rows=slice(None)):
    want, want_lse, tol = c.want()
    if out_dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(want)
    off = np.abs(out - want)[rows]
    assert (off <= tol[rows] + 1e-7).all(), (off.max(), np.argwhere(off > tol[rows])[:5])
    empty = np.isinf(want_lse)[rows]
    assert (lse[rows][empty] == -np.inf).all() and (out[rows][empty] == 0).all()
    assert (np.abs(lse[rows][~empty] - want_lse[rows][~empty]) <= S_ERR).all()


SHAPES = [dims(8, 128, 64), dims(4, 64, 16, 1), dims(1, 128, 32, 3), dims(3, 64, 32), dims(5, 128, 16), dims(7, 128, 64, 1),
          dims(6, 64, 64), dims(2, 128, 64)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", SHAPES)
def test_single_tokens(d, causal):
    c = Case(d, [0, 1, 15, 16, 17, 63, 64, 65, 127, 300, 511, 700], [1] * 12, seed=1, causal=causal)
    check(c, *run(c))


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", SHAPES)
def test_few_tokens(d, causal, out_dtype):
    c = Case(d, [0, 1, 30, 64, 200, 333, 0], [3, 1, 0, 4, 2, 4, 0], seed=2, causal=causal, k_scale=0.046875)
    check(c, *run(c, out_dtype), out_dtype)


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", SHAPES)
def test_prompts(d, causal, out_dtype):
    c = Case(d, [0, 5, 129, 64, 70], [70, 33, 0, 131, 1], seed=3, causal=causal, v_scale=2.0)
    check(c, *run(c, out_dtype), out_dtype)


@pytest.mark.parametrize("ctx,n", [([1400], [1]), ([2100], [3]), ([1029, 10], [40, 2]), ([40] * 40, [1] * 40), ([100] * 9, [60] * 9)])
@pytest.mark.parametrize("d", [dims(8, 128, 64, 1), dims(2, 64, 16, 1)])
def test_slices_and_batches(d, ctx, n):
    c = Case(d, ctx, n, seed=4)
    check(c, *run(c))


@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)])
def test_bounds_wider_than_the_batch(d, n):
    """Bounds far above the lengths, a padded batch: rows and slices without a key."""
    c = Case(d, [3, 0, 90], [n, 1 if n == 1 else 0, n], seed=5, spare_blocks=200)
    check(c, *run(c, single=False, max_ctx=5000 * d.page_size // 64, max_q=min(n + 9, int(c.indptr[-1]))))


@pytest.mark.parametrize("n", [1, 2, 50])
@pytest.mark.parametrize("mag", [2.0 ** -120, 2.0 ** -30, 2.0 ** 40])
def test_queries_of_any_magnitude(n, mag):
    """Rows of tiny and of huge elements: the power of two that brings them into fp16 is taken back in the scores."""
    c = Case(dims(4, 128, 32), [40, 70], [n, n], seed=6)
    T = int(c.indptr[-1])
    small = wl.bits_to_f64(c.q) * mag
    h = make_handle(c.d, torch.float32, sm_scale=float(np.float32(min(1.0 / np.sqrt(128) / mag, 2.0 ** 100))))
    bits = to_host_bits(torch.from_numpy(small).to(torch.bfloat16))
    assert mag < 2.0 ** -100 or np.array_equal(wl.bits_to_f64(bits), small)  # (the smallest are no normal numbers any more)
    out, lse = run(c, q=bits, h=h)
    if mag > 2.0 ** -100:
        c.scale = float(h.cfg.sm_scale) * mag
        check(c, out, lse)
    else:  # scores of 2^100 * 2^-120 at most: equal weights
        for r in range(2):
            for i in range(n):
                L = int(c.ctx[r]) + i + 1
                assert np.abs(lse[c.indptr[r] + i] - np.log(L)).max() < 2.0 ** -10
    assert out.shape[0] == T


@pytest.mark.parametrize("n", [1, 3, 40])
def test_a_nan_query_shows_and_stays_in_its_row(n):
    c = Case(dims(8, 128, 64), [70, 20], [n, n], seed=7)
    q = c.q.copy()
    q[n - 1, 5, 3] = 0x7FC0
    out, lse = run(c, q=q)
    assert np.isnan(out[n - 1, 5]).all() and np.isnan(lse[n - 1, 5])
    out[n - 1, 5], lse[n - 1, 5] = c.want()[0][n - 1, 5], c.want()[1][n - 1, 5]
    check(c, out, lse)


@pytest.mark.parametrize("ctx,n", [([70, 20], 1), ([70, 20], 3), ([70, 20], 40), ([2400, 300], 1), ([2400, 300], 2), ([2400, 300], 4)])
def test_an_infinite_query_stays_in_its_row(ctx, n):
    """Rows of elements that fp16 does not reach beside one with an infinity."""
    c = Case(dims(8, 128, 64), ctx, [n, n], seed=41)
    big = wl.bits_to_f64(c.q) * 2.0 ** 20
    q = to_host_bits(torch.from_numpy(big).to(torch.bfloat16))
    assert np.array_equal(wl.bits_to_f64(q), big)
    q[n - 1, 5, 3] = 0x7F80
    h = make_handle(c.d, torch.float32, sm_scale=float(np.float32(1.0 / np.sqrt(128))) * 2.0 ** -20)
    c.scale = float(h.cfg.sm_scale) * 2.0 ** 20
    out, lse = run(c, q=q, h=h, single=False)
    out[n - 1, 5], lse[n - 1, 5] = c.want()[0][n - 1, 5], c.want()[1][n - 1, 5]
    check(c, out, lse)


@pytest.mark.parametrize("sm_scale", [1.0, 3.0])
@pytest.mark.parametrize("n", [1, 4, 40])
def test_peaked_rows_and_growing_maxima(n, sm_scale):
    """Larger scales: nearly one-hot rows whose maxima move from tile to tile.  The error of a score grows with the scale: S times
    8 and 24 (from 1 / sqrt(64))."""
    c = Case(dims(4, 64, 32), [500, 130], [n, n], seed=8)
    h = make_handle(c.d, torch.float32, sm_scale=sm_scale)
    out, lse = run(c, h=h)
    want, want_lse, tol = c.want(sm_scale)
    more = S_ERR * 8 * sm_scale
    assert (np.abs(out - want) <= tol + 2 * more * np.abs(np.concatenate([v for _, v in c.kv])).max()).all()
    assert (np.abs(lse - want_lse) <= more).all()


@pytest.mark.parametrize("ctx,n", [([100, 200], [2, 3]), ([2300, 200], [1, 1]), ([2300, 200], [2, 3]), ([100, 200], [40, 3])])
def test_offsets_past_32_bits_and_rows_left_alone(ctx, n):
    """A pool of more than 4 GB, requests in its last pages; rows of out behind the last request stay as they were."""
    d = dims(8, 128, 64, 8)
    c = Case(d, ctx, n, seed=9)
    pages = 60000  # x 73728 bytes
    pool = torch.zeros((pages, *c.pool.shape[1:]), dtype=torch.uint8, device="cuda")
    pool[pages - c.pool.shape[0]:] = torch.from_numpy(c.pool).cuda()
    c.table = np.where(c.table >= 0, c.table + pages - c.pool.shape[0], -1).astype(np.int32)
    h = make_handle(d, torch.float32)
    T = int(c.indptr[-1])
    b = hb.Batch(dev_i32(c.ctx), dev_i32(c.table), *no_rings(d, 2), dev_i32(c.indptr), max_q_len=max(n), total_q=T + 4, max_ctx_len=max(ctx))
    out = torch.full((T + 4, 64, 128), 7.0, device="cuda")
    lse = torch.full((T + 4, 64), 7.0, device="cuda")
    q = torch.zeros((T + 4, 64, 128), dtype=torch.bfloat16, device="cuda")
    q[:T] = to_dev_bf16(c.q)
    hb.hswa_packed_attn(h, hb.PackedLayer(pool, c.k_scale, c.v_scale), b, True, q, out, lse, workspace(h, b, True))
    no_error(h)
    assert (out[T:] == 7).all() and (lse[T:] == 7).all()
    check(c, out[:T].double().cpu().numpy(), lse[:T].double().cpu().numpy())


# ---- contexts past what a block takes as a whole ----
LONG = [2500, 0, 1, 2240, 130, 4005]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows", [8, 16, 32])
@pytest.mark.parametrize("d", SHAPES)
def test_long_contexts(d, rows, causal):
    """As many tokens as make up to 8, 16 and 32 rows for a KV head; some requests shorter by a token, one without any."""
    n = max(1, rows // (d.num_q_heads // d.num_kv_heads))
    c = Case(d, LONG, [n, n, max(1, n - 1), n, 0, n], seed=30 + rows, causal=causal, v_scale=3.0)
    check(c, *run(c))


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", SHAPES)
def test_long_single_tokens(d, out_dtype):
    """Without row offsets; a table with places to spare, a bound far above the lengths."""
    c = Case(d, [2113, 3000, 64, 0], [1] * 4, seed=31, spare_blocks=300, k_scale=0.046875)
    check(c, *run(c, out_dtype), out_dtype)
    check(c, *run(c, out_dtype, max_ctx=3000 + 100 * d.page_size), out_dtype)


@pytest.mark.parametrize("d,n", [(dims(1, 64, 16, 1), 1), (dims(8, 128, 64, 1), 2), (dims(8, 64, 32, 1), 4), (dims(3, 128, 16, 1), 3)])
def test_many_requests_of_all_lengths(d, n):
    """More streams than SMs, most of them short: runs that begin and end in the middle of streams, and hold several."""
    rng = np.random.default_rng(32)
    B = 170
    ctx = [int(x) for x in rng.integers(0, 400, B)]
    ctx[3], ctx[77], ctx[B - 1] = 2600, 0, 2301
    c = Case(d, ctx, [n if r % 5 else r % (n + 1) for r in range(B)], seed=33)
    check(c, *run(c, single=False))


@pytest.mark.parametrize("n", [1, 2])
def test_one_long_request_among_many_short_ones(n):
    """Most streams in a piece or two, a few in dozens."""
    ctx = [9] * 300
    ctx[150] = 12007
    c = Case(dims(8, 64, 64, 1), ctx, [n] * 300, seed=40)
    check(c, *run(c, single=False))


@pytest.mark.parametrize("n", [1, 2, 4])
def test_one_long_request(n):
    """A stream in many pieces."""
    c = Case(dims(8, 128, 64, 1), [20011], [n], seed=34)
    check(c, *run(c, single=False))


@pytest.mark.parametrize("n", [1, 2, 4])
def test_long_rows_of_nan_and_unlike_magnitudes(n):
    """A NaN stays in its row; a row 2^20 times smaller than its neighbour keeps its own maxima and sums."""
    c = Case(dims(8, 128, 64, 2), [2400, 300], [n, n], seed=35)
    q = c.q.copy()
    q[n - 1, 5, 3] = 0x7FC0
    q[0, 9] = to_host_bits(torch.from_numpy(wl.bits_to_f64(c.q[0, 9]) * 2.0 ** -20).to(torch.bfloat16))
    c.q[0, 9] = q[0, 9]
    out, lse = run(c, q=q, single=False)
    assert np.isnan(out[n - 1, 5]).all() and np.isnan(lse[n - 1, 5])
    out[n - 1, 5], lse[n - 1, 5] = c.want()[0][n - 1, 5], c.want()[1][n - 1, 5]
    check(c, out, lse)


@pytest.mark.parametrize("sm_scale", [1.0, 3.0])
@pytest.mark.parametrize("n", [1, 3, 8])
def test_long_peaked_rows(n, sm_scale):
    """As test_peaked_rows_and_growing_maxima."""
    c = Case(dims(4, 64, 32), [3500, 130], [n, n], seed=36)
    h = make_handle(c.d, torch.float32, sm_scale=sm_scale)
    out, lse = run(c, h=h, single=False)
    want, want_lse, tol = c.want(sm_scale)
    more = S_ERR * 8 * sm_scale
    assert (np.abs(out - want) <= tol + 2 * more * np.abs(np.concatenate([v for _, v in c.kv])).max()).all()
    assert (np.abs(lse - want_lse) <= more).all()


@pytest.mark.parametrize("n", [1, 2, 4])
def test_long_contexts_record_values_out_of_range(n):
    """What the bounds do not cover is recorded and left alone; the other requests' rows are computed."""
    d = dims(8, 64, 16, 1)
    c = Case(d, [2300, 40, 2200], [n, n, n], seed=37)
    good = run(c, single=False)
    h = make_handle(d, torch.float32)

    def record(ctx=None, indptr=None, table=None, max_q=n, total=3 * n):
        b = hb.Batch(dev_i32(c.ctx if ctx is None else ctx), dev_i32(c.table if table is None else table), *no_rings(d, 3),
                     dev_i32(c.indptr if indptr is None else indptr), max_q_len=max_q, total_q=total, max_ctx_len=2300)
        out, lse = torch.full((3 * n, 8, 64), 7.0, device="cuda"), torch.full((3 * n, 8), 7.0, device="cuda")
        hb.hswa_packed_attn(h, c.layer(), b, True, to_dev_bf16(c.q), out, lse, workspace(h, b, True))
        return hb.hswa_get_async_error(h), out.double().cpu().numpy(), lse.double().cpu().numpy()

    table = c.table.copy()
    table[1, 1] = 1 << 20
    st, out, _ = record(table=table)
    assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, 1, 1 << 20), st
    assert np.array_equal(out[:n], good[0][:n]) or np.abs(out[:n] - good[0][:n]).max() < 1e-2
    for bad in (-1, 2301):
        st, out, _ = record(ctx=[2300, bad, 2200])
        assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, -1, bad), st
        assert np.abs(out[2 * n:] - good[0][2 * n:]).max() < 1e-2  # (other runs, other roundings)
    if n > 1:
        st, out, lse = record(indptr=np.array([0, n - 1, 2 * n, 3 * n], np.int32))
        assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, -2, n + 1), st
        assert (out[2 * n - 1] == 7).all() and (lse[2 * n - 1] == 7).all()
    for indptr in ([0, n, 2 * n, 3 * n + 1], [-1, n, 2 * n, 3 * n]):
        st, _, _ = record(indptr=np.array(indptr, np.int32), max_q=n + 1 if n > 1 else 1)
        assert (st[0], st[2]) == (hb.HSWA_ERR_BOUNDS, -2), st


@pytest.mark.parametrize("n", [1, 4])
def test_long_calls_captured_and_repeated(n):
    """A captured call replayed on other data, twice: bit for bit what the call itself gives."""
    c, other = (Case(dims(8, 128, 64, 2), [2600, 900], [n, n], seed=s) for s in (38, 39))
    h = make_handle(c.d, torch.float32)
    b, layer, q = c.batch(single=False), c.layer(), to_dev_bf16(c.q)
    T = int(c.indptr[-1])
    out, lse, ws = torch.empty((T, 16, 128), device="cuda"), torch.empty((T, 16), device="cuda"), workspace(h, b, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.hswa_packed_attn(h, layer, b, True, q, out, lse, ws)
    layer.pool.copy_(torch.from_numpy(other.pool).cuda())
    q.copy_(to_dev_bf16(other.q))
    b.block_table.copy_(dev_i32(other.table))
    seen = []
    for _ in range(2):
        out.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        no_error(h)
        seen.append(out.double().cpu().numpy())
        check(other, seen[-1], lse.double().cpu().numpy())
    assert np.array_equal(*seen)


# ---- rows in and out --------------------------------------------------------------------------------------------------
def codes_of(pool, table, ctx, n, P, D):
    return [[ref.rows(pool, table, r, int(ctx[r] + n[r]), which, P, D, 1.0)[ctx[r]:] for which in (0, 1)] for r in range(len(ctx))]


@pytest.mark.parametrize("scales", [(1.0, 0.5), (0.046875, 3.0)])
@pytest.mark.parametrize("d", SHAPES)
def test_append_and_read(d, scales):
    ctx, n = np.array([0, 3, 60, 7, 100], np.int32), np.array([20, 1, 0, 70, 33], np.int32)
    P, D, H, T = d.page_size, d.head_dim, d.num_kv_heads, int(n.sum())
    rng = np.random.default_rng(10)
    blocks = -(-133 // P)
    table = rng.permutation(5 * blocks + 2)[: 5 * blocks].reshape(5, blocks).astype(np.int32)
    pool = rng.integers(0, 256, (5 * blocks + 2, 2, H, P * (D // 2 + D // 16)), dtype=np.uint8)
    k, v = (wl.bf16_bits_normal(s, (T, H, D)) for s in (11, 12))
    k[0, 0, :16] = 0                                                              # a block of zeros
    k[1, 0, :16] = to_host_bits(torch.full((16,), 2.0 ** -100).bfloat16())        # a scale below the smallest
    k[2, 0, :16] = to_host_bits(torch.arange(16.0).mul(1e30).bfloat16())          # past the largest
    k[3, 0, 1] |= 0x8000
    v[4, 0, :16] = to_host_bits(torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0]).mul(scales[1]).bfloat16())
    h = make_handle(d)
    indptr = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    b = hb.Batch(dev_i32(ctx), dev_i32(table), *no_rings(d, 5), dev_i32(indptr), max_q_len=70, total_q=T, max_ctx_len=100)
    layer = hb.PackedLayer(torch.from_numpy(pool).cuda(), *scales)
    hb.hswa_packed_append(h, layer, b, to_dev_bf16(k), to_dev_bf16(v))
    outs = [torch.full((T + 1, H, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    hb.hswa_packed_read(h, layer, b, *outs)
    no_error(h)
    want, values = pool.copy(), [np.zeros((T, H, D)) for _ in range(2)]
    for which, x in ((0, k), (1, v)):
        n4, f = ref.round_rows(wl.bits_to_f64(x), scales[which])
        values[which] = ref.values(n4, f, scales[which])
        for r in range(5):
            for i in range(n[r]):
                pos, t = ctx[r] + i, indptr[r] + i
                ref.put(want, table[r, pos // P], pos % P, which, P, n4[t], f[t])
    got = layer.pool.cpu().numpy()
    assert np.array_equal(got, want), np.argwhere(got != want)[:8]
    for o, w in zip(outs, values):
        assert (o[T:] == 9).all()
        x = o[:T].double().cpu().numpy()
        assert (np.abs(x - w) <= 2.0 ** -8 * np.abs(w)).all() and (scales != (1.0, 0.5) or np.array_equal(x, w))


def test_infinities_and_nan_are_held_as_finite_values():
    d = dims(2, 64, 16, 1)
    k = np.zeros((1, 1, 64), np.uint16)
    k[0, 0, 0], k[0, 0, 16], k[0, 0, 32], k[0, 0, 33] = 0x7F80, 0xFF80, 0x7FC0, 0x3F80
    h = make_handle(d)
    b = hb.Batch(dev_i32([0]), dev_i32([[1]]), *no_rings(d, 1), max_ctx_len=0)
    layer = hb.PackedLayer(torch.zeros((2, 2, 1, 16 * 36), dtype=torch.uint8, device="cuda"))
    hb.hswa_packed_append(h, layer, b, to_dev_bf16(k), to_dev_bf16(k))
    ko, vo = (torch.empty((1, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hb.hswa_packed_read(h, layer, b, ko, vo)
    no_error(h)
    assert torch.isfinite(ko).all() and ko[0, 0, 0] == 448 * 6 and ko[0, 0, 16] == -448 * 6 and torch.equal(ko, vo)


def test_every_finite_bf16_rounds_as_stated():
    """All magnitudes of bf16 next to a block's largest of several sizes, with a scale that divides none of them evenly."""
    d = dims(1, 128, 64, 1)
    every = np.arange(0x7F80, dtype=np.uint16)
    h = make_handle(d)
    for scale in (1.0, 0.7, 2.0 ** -60):
        rows = []
        for top in (0x3F80, 0x4049, 0x7F7F, 0x2345):
            x = np.concatenate([every, np.zeros(-len(every) % 15, np.uint16)]).reshape(-1, 15)
            x = np.minimum(x, top)
            x = np.concatenate([np.full((len(x), 1), top, np.uint16), x], axis=1)
            x[1::2] |= 0x8000
            rows.append(x.reshape(-1))
        flat = np.concatenate(rows)
        T = -(-len(flat) // 128)
        flat = np.concatenate([flat, np.zeros(T * 128 - len(flat), np.uint16)]).reshape(T, 1, 128)
        pages = -(-T // 64)
        b = hb.Batch(dev_i32([0]), dev_i32(np.arange(pages)[None]), *no_rings(d, 1), dev_i32([0, T]), max_q_len=T, total_q=T, max_ctx_len=0)
        layer = hb.PackedLayer(torch.zeros((pages, 2, 1, 64 * 72), dtype=torch.uint8, device="cuda"), scale, scale)
        x = to_dev_bf16(flat)
        hb.hswa_packed_append(h, layer, b, x, x)
        no_error(h)
        s32 = float(np.float32(scale))
        n4, f = ref.round_rows(wl.bits_to_f64(flat), s32)
        want = ref.values(n4, f, 1.0)
        got = ref.rows(layer.pool.cpu().numpy(), np.arange(pages)[None], 0, T, 1, 64, 128, 1.0)
        if scale == 0.7:  # (its quotients may lie within 2^-22 of a border: half a step of each rounding to 32 bits)
            differ = got != want
            y = np.abs(wl.bits_to_f64(flat)) / np.repeat(ref.SCALES[f] * s32 + 1e-300, 16, axis=-1)
            near = np.abs(y[..., None] / np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) - 1).min(axis=-1) < 2.0 ** -22
            assert (near | ~differ).all()
        else:
            assert np.array_equal(got, want)


# ---- refusals -----------------------------------------------------------------------------------------------------------
def test_refusals():
    c = Case(dims(2, 64, 16, 1), [20], [2], seed=13)
    h, b, layer = make_handle(c.d), c.batch(), c.layer()
    q, out = to_dev_bf16(c.q), torch.empty((2, 2, 64), device="cuda")
    k = torch.zeros((2, 1, 64), dtype=torch.bfloat16, device="cuda")
    ws = workspace(h, b, True)

    def status(call, *a):
        with pytest.raises(hb.HswaError) as e:
            call(h, *a)
        return e.value.status

    for bad in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** 65, 2.0 ** -65):
        for scales in ((bad, 1.0), (1.0, bad)):
            assert status(hb.hswa_packed_attn, hb.PackedLayer(layer.pool, *scales), b, True, q, out, None, ws) == hb.HSWA_ERR_INVALID_ARG
            assert status(hb.hswa_packed_append, hb.PackedLayer(layer.pool, *scales), b, k, k) == hb.HSWA_ERR_INVALID_ARG
    assert status(hb.hswa_packed_attn, layer, c.batch(max_ctx=1 << 20), True, q, out, None, ws) == hb.HSWA_ERR_INVALID_ARG  # table too small
    long = Case(dims(2, 64, 16, 1), [5000], [2], seed=13)
    need = hb.hswa_packed_workspace_need(h, 1, 2, 2, 5000, True)
    assert need > 0 and need % 256 == 0
    for w in (None, torch.empty((need - 256,), dtype=torch.uint8, device="cuda"), torch.empty((need + 16,), dtype=torch.uint8, device="cuda")[16:]):
        assert status(hb.hswa_packed_attn, long.layer(), long.batch(), True, q, out, None, w) == hb.HSWA_ERR_WORKSPACE
    with pytest.raises(AssertionError):  # of another page size
        hb.hswa_packed_attn(make_handle(dims(2, 64, 32, 1)), layer, b, True, q, out, None, ws)
    with pytest.raises(AssertionError):  # fewer rows than total_q
        hb.hswa_packed_append(h, layer, b, k[:1], k)
    with pytest.raises(AssertionError):
        hb.hswa_packed_attn(h, layer, b, True, q, out.bfloat16(), None, ws)
    with pytest.raises(AssertionError):
        hb.hswa_packed_attn(h, layer, b, True, q, out, None, ws.cpu())
    assert hb.hswa_packed_workspace_need(h, 1, 2, 2, 2 ** 30, True) == 0
    steep = make_handle(dims(2, 64, 16, 1), torch.float32, sm_scale=2.0 ** 100)
    with pytest.raises(hb.HswaError) as e:
        hb.hswa_packed_attn(steep, hb.PackedLayer(layer.pool, 2.0 ** 40, 1.0), b, True, q, out, None, ws)
    assert e.value.status == hb.HSWA_ERR_INVALID_ARG
    no_error(h)


@pytest.mark.parametrize("n", [1, 3, 40])
def test_values_out_of_range_are_recorded(n):
    d = dims(4, 64, 16, 1)
    c = Case(d, [40, 40, 40], [n, n, n], seed=14)
    good = run(c)
    h = make_handle(d, torch.float32)

    def record(ctx=None, indptr=None, table=None, max_q=None, call="attn"):
        b = hb.Batch(dev_i32(c.ctx if ctx is None else ctx), dev_i32(c.table if table is None else table), *no_rings(d, 3),
                     dev_i32(c.indptr if indptr is None else indptr), max_q_len=max_q or n, total_q=3 * n, max_ctx_len=40)
        out, lse = torch.full((3 * n, 4, 64), 7.0, device="cuda"), torch.full((3 * n, 4), 7.0, device="cuda")
        if call == "attn":
            hb.hswa_packed_attn(h, c.layer(), b, True, to_dev_bf16(c.q), out, lse, workspace(h, b, True))
        else:
            k = torch.zeros((3 * n, 1, 64), dtype=torch.bfloat16, device="cuda")
            hb.hswa_packed_append(h, c.layer(), b, k, k)
        return hb.hswa_get_async_error(h), out.double().cpu().numpy(), lse.double().cpu().numpy()

    table = c.table.copy()
    table[1, 1] = 1 << 20
    for call in ("attn", "append"):
        st, out, _ = record(table=table, call=call)
        if call == "attn" or n > 1:  # (one token goes to block 2)
            assert (st[0], st[1]) == ((hb.HSWA_ERR_BOUNDS, 1) if call == "attn" else (hb.HSWA_OK, 0)), st
        for bad in (-1, 41):
            st, out2, _ = record(ctx=[40, bad, 40], call=call)
            assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, -1, bad), st
        if call == "attn":
            assert np.array_equal(out[:n], good[0][:n]) and np.array_equal(out2[2 * n:], good[0][2 * n:])
    table[1, 2] = -5
    st, _, _ = record(table=table, call="append")
    assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, 2, -5), st
    if n > 1:  # a request longer than the bound: its rows past it stay as they were
        indptr = np.array([0, n - 1, 2 * n, 3 * n], np.int32)
        st, out, lse = record(indptr=indptr, max_q=n)
        assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, -2, n + 1), st
        assert (out[2 * n - 1] == 7).all() and (lse[2 * n - 1] == 7).all() and (out[: 2 * n - 1] != 7).any(axis=(1, 2)).all()
    for indptr in ([0, n, 2 * n, 3 * n + 1], [-1, n, 2 * n, 3 * n]):
        st, _, _ = record(indptr=np.array(indptr, np.int32), max_q=n + 1 if n > 1 else 1)
        assert (st[0], st[2]) == (hb.HSWA_ERR_BOUNDS, -2), st


def test_keys_past_the_block_table_are_recorded():
    """The longest context and the longest step may belong to different requests: only their sum within one has to fit the table."""
    d = dims(4, 64, 16, 1)
    c = Case(d, [32, 10], [1, 6], seed=15)
    c.table = c.table[:, :2].copy()
    h = make_handle(d, torch.float32)
    out, lse = torch.full((7, 4, 64), 7.0, device="cuda"), torch.full((7, 4), 7.0, device="cuda")
    b = c.batch(single=False)
    hb.hswa_packed_attn(h, c.layer(), b, True, to_dev_bf16(c.q), out, lse, workspace(h, b, True))
    st = hb.hswa_get_async_error(h)
    assert st[:3] == (hb.HSWA_ERR_BOUNDS, 0, -3), st
    check(c, out.double().cpu().numpy(), lse.double().cpu().numpy(), rows=slice(1, None))
    k = torch.zeros((7, 1, 64), dtype=torch.bfloat16, device="cuda")
    hb.hswa_packed_append(h, c.layer(), b, k, k)
    assert hb.hswa_get_async_error(h)[:3] == (hb.HSWA_ERR_BOUNDS, 0, 2)


def test_empty_calls():
    d = dims(2, 64, 16, 1)
    h = make_handle(d)
    layer = hb.PackedLayer(torch.zeros((1, 2, 1, 16 * 36), dtype=torch.uint8, device="cuda"))
    none = torch.empty((0, 2, 64), device="cuda")
    k = torch.empty((0, 1, 64), dtype=torch.bfloat16, device="cuda")
    for B in (0, 2):
        b = hb.Batch(dev_i32([0] * B), dev_i32([[0]] * B) if B else torch.zeros((0, 1), dtype=torch.int32, device="cuda"), *no_rings(d, B),
                     dev_i32([0] * (B + 1)), max_q_len=0, total_q=0, max_ctx_len=0)
        hb.hswa_packed_attn(h, layer, b, True, none.bfloat16(), none)
        hb.hswa_packed_append(h, layer, b, k, k)
        hb.hswa_packed_read(h, layer, b, k, k)
    no_error(h)


# ---- together -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16, 1)])
def test_a_run_of_steps(d):
    """Prompts, then drafts of three, then single tokens: appended and attended to, step by step, on a captured graph for the
    single tokens; another stream than the current one's default."""
    B, P, D, H = 3, d.page_size, d.head_dim, d.num_kv_heads
    h = make_handle(d, torch.float32)
    blocks = -(-260 // P)
    table = np.random.default_rng(16).permutation(B * blocks).reshape(B, blocks).astype(np.int32)
    layer = hb.PackedLayer(torch.zeros((B * blocks, 2, H, P * (D // 2 + D // 16)), dtype=torch.uint8, device="cuda"), 1.0, 0.5)
    ctx, table_d = dev_i32([0] * B), dev_i32(table)
    rings = no_rings(d, B)
    kv = [[np.zeros((0, H, D)) for _ in range(2)] for _ in range(B)]
    stream = torch.cuda.Stream()
    graph = None
    for step, lens in enumerate([[130, 7, 66], [3, 3, 3], [1, 1, 1], [1, 1, 1], [1, 1, 1]]):
        T = sum(lens)
        bits = [wl.bf16_bits_normal(200 + 10 * step + i, (T, hh, D)) for i, hh in ((0, H), (1, H), (2, d.num_q_heads))]
        indptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        single = lens[0] == 1
        if not single or graph is None:
            data = [to_dev_bf16(x) for x in bits]
            b = hb.Batch(ctx, table_d, *rings, None if single else dev_i32(indptr), max_q_len=max(lens), total_q=T, max_ctx_len=250)
            out, lse = torch.empty((T, d.num_q_heads, D), device="cuda"), torch.empty((T, d.num_q_heads), device="cuda")
            ws = workspace(h, b, True)

        def one_step():
            hb.hswa_packed_append(h, layer, b, data[0], data[1])
            hb.hswa_packed_attn(h, layer, b, True, data[2], out, lse, ws)
            hb.hswa_step_advance(h, B, ctx, rings[1], b.q_indptr)

        if single:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    one_step()
            for x, y in zip(data, bits):
                x.copy_(to_dev_bf16(y))
            graph.replay()
        else:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                one_step()
            torch.cuda.current_stream().wait_stream(stream)
        no_error(h)
        q = wl.bits_to_f64(bits[2])
        o, ls = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for r in range(B):
            a, e = indptr[r], indptr[r + 1]
            for which, scale in ((0, 1.0), (1, 0.5)):
                x = wl.bits_to_f64(bits[which][a:e])
                kv[r][which] = np.concatenate([kv[r][which], ref.values(*ref.round_rows(x, scale), scale)])
            L = len(kv[r][0])
            want, want_lse, mag = ref.attention(*kv[r], q[a:e], [L - (e - a) + i + 1 for i in range(e - a)], 1.0 / np.sqrt(D))
            tol = (2.0 ** -11 + 2 * S_ERR + L * 2.0 ** -24) * mag + L * 2.0 ** -25 * np.abs(kv[r][1]).max()
            assert (np.abs(o[a:e] - want) <= tol + 1e-7).all() and (np.abs(ls[a:e] - want_lse) <= S_ERR).all()


def test_calls_on_two_streams_at_once():
    cases = [Case(dims(8, 128, 64), [700, 300], [n, n], seed=17 + n) for n in (1, 40)]
    h = make_handle(cases[0].d, torch.float32)
    jobs = []
    for c in cases:
        b = c.batch()
        T = int(c.indptr[-1])
        jobs.append((c, b, c.layer(), to_dev_bf16(c.q), torch.empty((T, 16, 128), device="cuda"), torch.empty((T, 16), device="cuda"),
                     workspace(h, b, True), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for _, b, layer, q, out, lse, ws, s in jobs:
            with torch.cuda.stream(s):
                hb.hswa_packed_attn(h, layer, b, True, q, out, lse, ws)
    torch.cuda.synchronize()
    no_error(h)
    for c, _, _, _, out, lse, _, _ in jobs:
        check(c, out.double().cpu().numpy(), lse.double().cpu().numpy())


def test_repeated_calls_agree_bit_for_bit():
    c = Case(dims(8, 128, 64), [1500, 40, 900], [1, 1, 1], seed=20)
    a, b = run(c), run(c)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
