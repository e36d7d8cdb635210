"""The 4-bit cache's attention where it can go wrong, beside test_gpu_packed.py, whose tolerances hold here too."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16, to_host_bits
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl
from test_gpu_packed import S_ERR, Case, check, dims, no_error, no_rings, run, workspace

pytestmark = pytest.mark.gpu


class Filled:
    """A cache of many requests whose pages are filled on the GPU: random codes, scales between 2^-3 and 2^2."""

    def __init__(self, d, ctx, n, seed, sm_scale=0.0):
        P, D, H = d.page_size, d.head_dim, d.num_kv_heads
        g = torch.Generator(device="cuda").manual_seed(seed)
        used = [-(-(c + n) // P) for c in ctx]
        pages, B = sum(used), len(ctx)
        pool = torch.randint(0, 256, (pages, 2, H, P * (D // 2 + D // 16)), generator=g, device="cuda", dtype=torch.uint8)
        pool[..., P * D // 2:] = torch.randint(0x20, 0x48, (pages, 2, H, P * D // 16), generator=g, device="cuda", dtype=torch.uint8)
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros((B, max(used)), dtype=torch.int32, device="cuda")
        at = 0
        for r, u in enumerate(used):
            table[r, :u] = perm[at:at + u]
            at += u
        self.h, self.n, self.B = make_handle(d, torch.float32, sm_scale), n, B
        self.layer = hb.PackedLayer(pool, 0.5, 1.0)
        self.q = torch.randn((B * n, d.num_q_heads, D), generator=g, device="cuda", dtype=torch.bfloat16)
        self.batch = hb.Batch(dev_i32(ctx), table, *no_rings(d, B), dev_i32(np.arange(B + 1) * n), max_q_len=n, total_q=B * n, max_ctx_len=max(ctx))
        self.ws = workspace(self.h, self.batch, True)

    def run(self):
        out = torch.full(self.q.shape, 7.0, device="cuda")
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        hb.hswa_packed_attn(self.h, self.layer, self.batch, True, self.q, out, lse, self.ws)
        return out, lse


@pytest.mark.parametrize("d", [dims(8, 128, 64, 4), dims(8, 128, 32, 4), dims(4, 128, 16, 4), dims(8, 64, 64, 4), dims(3, 64, 32, 4), dims(8, 64, 16, 4)])
def test_full_machines_of_single_tokens_repeat_themselves(d):
    """Every warp of the machine fetches for itself, and the lanes that wait see a copy land at different polls: pages of each size, with one and
    with several copies a tile, give the same bits whenever they run."""
    rng = np.random.default_rng(1)
    c = Filled(d, [int(x) for x in rng.integers(1000, 9000, 48)], 1, seed=2)
    first = c.run()
    assert torch.isfinite(first[0]).all() and torch.isfinite(first[1]).all()
    for _ in range(20):
        again = c.run()
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    no_error(c.h)


@pytest.mark.parametrize("sm_scale", [0.0, 2.0])
@pytest.mark.parametrize("d,n", [(dims(8, 128, 64, 4), 2), (dims(8, 128, 16, 4), 4), (dims(8, 64, 32, 4), 4), (dims(3, 64, 64, 4), 5)])
def test_full_machines_of_drafts_repeat_themselves(d, n, sm_scale):
    """Runs of many pieces, in which two groups of warps take turns and vote on their maxima tile by tile (with the larger scale, maxima grow
    all along): the same bits whenever they run, and no wait runs out."""
    rng = np.random.default_rng(3)
    c = Filled(d, [int(x) for x in rng.integers(100, 9000, 48)], n, seed=4, sm_scale=sm_scale)
    first = c.run()
    assert torch.isfinite(first[0]).all() and torch.isfinite(first[1]).all()
    for _ in range(20):
        again = c.run()
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    no_error(c.h)


@pytest.mark.parametrize("d,n", [(dims(8, 128, 64, 4), 150), (dims(5, 64, 16, 4), 70)])
def test_full_machines_of_prompts_repeat_themselves(d, n):
    """Blocks of one and of two Q tiles, whose MMA issuers pass a token: the same bits whenever they run, and no wait runs out."""
    rng = np.random.default_rng(5)
    c = Filled(d, [int(x) for x in rng.integers(0, 3000, 24)], n, seed=6)
    first = c.run()
    assert torch.isfinite(first[0]).all() and torch.isfinite(first[1]).all()
    for _ in range(10):
        again = c.run()
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    no_error(c.h)


# ---- probabilities far below the row's largest ----
def levelled(d, L, n, k_of, v_of, sm_scale, ones=1.0):
    """One request of L cached keys (the step's n among them) whose K and V rows are constant, k_of[j] and v_of[j] (values of e2m1), and queries
    of ones: the score of key j is sm_scale * D * ones * k_of[j] for every row.  -> out, lse of the call."""
    P, D, H = d.page_size, d.head_dim, d.num_kv_heads
    pages = -(-L // P)
    pad = np.zeros(pages * P - L)
    codes = [np.searchsorted(ref.LEVELS, np.concatenate([x, pad])).astype(np.uint8) * 17 for x in (k_of, v_of)]
    pool = torch.full((pages, 2, H, P * (D // 2 + D // 16)), 0x38, dtype=torch.uint8, device="cuda")  # scales of 1
    for which, c in enumerate(codes):
        rows = torch.from_numpy(c).cuda().reshape(pages, 1, P, 1).expand(pages, H, P, D // 2)
        pool[:, which, :, : P * D // 2] = rows.reshape(pages, H, -1)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    pool = pool.flip(0).contiguous()
    h = make_handle(d, torch.float32, sm_scale=float(np.float32(sm_scale)))
    q = torch.full((n, d.num_q_heads, D), ones, dtype=torch.bfloat16, device="cuda")
    b = hb.Batch(dev_i32([L - n]), table, *no_rings(d, 1), dev_i32([0, n]), max_q_len=n, total_q=n, max_ctx_len=L - n)
    out, lse = torch.full(q.shape, 7.0, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    ws = workspace(h, b, True)
    ws.fill_(255)
    hb.hswa_packed_attn(h, hb.PackedLayer(pool), b, True, q, out, lse, ws)
    no_error(h)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


LEVEL_SHAPES = [(dims(8, 128, 64, 1), 1, 2000), (dims(8, 128, 64, 1), 1, 131072), (dims(4, 64, 16, 1), 1, 100000), (dims(8, 128, 64, 1), 2, 131072),
                (dims(8, 128, 32, 1), 4, 1000), (dims(8, 128, 64, 1), 4, 131072), (dims(8, 64, 64, 1), 4, 131072), (dims(8, 128, 64, 1), 40, 20000),
                (dims(5, 64, 32, 1), 30, 20000)]


@pytest.mark.parametrize("bits", [7.9, 8.1, 14.9, 25.1, 27.0])
@pytest.mark.parametrize("where", ["first", "middle", "late"])
@pytest.mark.parametrize("d,n,L", LEVEL_SHAPES)
def test_one_key_far_above_all_others_leaves_them_their_weight(d, n, L, where, bits):
    """One key `bits` powers of two above all others, whose V is 0 where theirs is 1: what comes out is their weight.  A score off by S = 2^-12
    (as in test_gpu_packed.py), fp16's 2^-11 and 2^-32 of the largest for each key, and sums of L terms."""
    at = {"first": 0, "middle": L // 2, "late": L - n - 1}[where]
    k, v = np.zeros(L), np.ones(L)
    k[at], v[at] = 1.0, 0.0
    scale = np.float32(bits * np.log(2.0) / d.head_dim)
    out, lse = levelled(d, L, n, k, v, scale)
    s = float(scale) * d.head_dim
    for i in range(n):
        others = L - n + i
        want = others * np.exp(-s) / (1.0 + others * np.exp(-s))
        tol = want * (2.0 ** -11 + 2 * S_ERR + L * 2.0 ** -24) + L * 2.0 ** -32
        assert np.abs(out[i] - want).max() <= tol, (i, out[i].min(), out[i].max(), want)
        assert np.abs(lse[i] - (s + np.log1p(others * np.exp(-s)))).max() <= S_ERR


@pytest.mark.parametrize("bits", [2.0 ** 12, 2.0 ** 20, 2.0 ** 24, 2.0 ** 26])
@pytest.mark.parametrize("d,n,L", LEVEL_SHAPES)
def test_scores_of_any_size_that_grow_from_key_to_key(d, n, L, bits):
    """Scores that grow in steps along the keys, up to sizes where a score's own rounding is several powers of two: the largest, one key, takes all."""
    k, v = np.zeros(L), np.full(L, 3.0)
    steps = [0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for i, x in enumerate(steps):
        k[(L - n) * (i + 1) // 8] = x
    v[(L - n) * 7 // 8] = 1.0
    scale = np.float32(bits * np.log(2.0) / d.head_dim / 6.0)
    out, lse = levelled(d, L, n, k, v, scale)
    assert (np.abs(out - 1.0) <= 2.0 ** -10).all()
    want = float(scale) * d.head_dim * 6.0
    assert (np.abs(lse - want) <= want * 2.0 ** -21).all()


@pytest.mark.parametrize("n,ctx", [(1, [40, 70]), (1, [2400, 70]), (2, [2400, 70]), (4, [40, 70]), (4, [2400, 70]), (50, [40, 70])])
@pytest.mark.parametrize("mag", [2.0 ** -90, 2.0 ** -112, 2.0 ** -118, 2.0 ** -121])
def test_queries_of_tiny_elements_and_a_large_scale(n, ctx, mag):
    """Elements around `mag` with a scale that makes scores of order 1: no element within 2^28 of the largest loses a bit on its way to fp16."""
    c = Case(dims(8, 128, 32), ctx, [n, n], seed=50)
    c.q = to_host_bits((torch.from_numpy(wl.bits_to_f64(c.q)) * mag).to(torch.bfloat16))
    h = make_handle(c.d, torch.float32, sm_scale=float(np.float32(1.0 / np.sqrt(128) / mag)))
    c.scale = float(h.cfg.sm_scale)
    check(c, *run(c, h=h, single=False))


# ---- layer scales of many bits ----
BORDERS = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])


@pytest.mark.parametrize("scale", [0.7001953125, 1.4998779296875 * 2.0 ** -9, 5.2119140625, 0.7, 4.0 / 3.0, 3.3895 / 2688.0, 1.9999998807907104, 2.0 ** -63 * 1.1])
def test_layer_scales_of_any_number_of_bits(scale):
    """Scales of up to 14 bits round as in exact arithmetic.  Longer ones make quotients that 32 bits round, two of them (2^-23 each) for the
    scale of a block, a product and one quotient for an element: within 2^-22 of a border either neighbour may be held.  The read-back rounds to
    32 bits, then to bf16."""
    d = dims(1, 128, 64, 1)
    s32 = float(np.float32(scale))
    exact = (np.float32(scale).view(np.uint32) & 0x3FF) == 0
    rng = np.random.default_rng(13)
    tops = np.concatenate([[0x3F80, 0x4049, 0x7F7F, 0x2345], rng.integers(0x3000, 0x4800, 4000)]).astype(np.uint16)
    x = np.stack([tops] + [np.maximum(tops.astype(int) - rng.integers(0, 700, len(tops)), 0).astype(np.uint16) for _ in range(15)], axis=1)
    x[:, 1:] |= rng.integers(0, 2, (len(tops), 15)).astype(np.uint16) << 15
    # elements next to the borders of their block's quotients
    f = ref.round_rows(wl.bits_to_f64(x), s32)[1]
    near = (BORDERS[rng.integers(0, 7, len(tops))] * ref.SCALES[f[:, 0]] * s32).astype(np.float32)
    near_bits = to_host_bits(torch.from_numpy(near).to(torch.bfloat16))
    x[:, 1] = np.minimum(near_bits, tops)
    flat = x.reshape(-1)
    T = -(-len(flat) // 128)
    flat = np.concatenate([flat, np.zeros(T * 128 - len(flat), np.uint16)]).reshape(T, 1, 128)
    pages = -(-T // 64)
    h = make_handle(d)
    b = hb.Batch(dev_i32([0]), dev_i32(np.arange(pages)[None]), *no_rings(d, 1), dev_i32([0, T]), max_q_len=T, total_q=T, max_ctx_len=0)
    layer = hb.PackedLayer(torch.zeros((pages, 2, 1, 64 * 72), dtype=torch.uint8, device="cuda"), scale, scale)
    data = to_dev_bf16(flat)
    hb.hswa_packed_append(h, layer, b, data, data)
    k, v = torch.empty_like(data), torch.empty_like(data)
    hb.hswa_packed_read(h, layer, b, k, v)
    no_error(h)
    pool, table = layer.pool.cpu().numpy(), np.arange(pages)[None]
    held = ref.rows(pool, table, 0, T, 1, 64, 128, 1.0)
    n4, f = ref.round_rows(wl.bits_to_f64(flat), s32)
    want = ref.values(n4, f, 1.0)
    if exact:
        assert np.array_equal(held, want)
    else:
        # a block's scale: the statement's, or its neighbour where the quotient is that near to the middle between them
        pos = np.arange(T)
        codes = pool[pos // 64, 1, 0][:, 64 * 64:].reshape(T, 64, 8)[pos, pos % 64]
        a = np.abs(wl.bits_to_f64(flat)).reshape(T, 8, 16).max(axis=-1) / s32 / 6.0
        other = codes != f[:, 0]
        middle = (ref.SCALES[codes] + ref.SCALES[f[:, 0]]) / 2
        assert (np.abs(a / np.where(other, middle, a + 1e-300) - 1)[other] < 2.0 ** -22).all() and (np.abs(codes.astype(int) - f[:, 0])[other] == 1).all()
        y = np.abs(wl.bits_to_f64(flat[:, 0])) / np.repeat(ref.SCALES[f[:, 0]] * s32 + 1e-300, 16, axis=-1)
        close = np.abs(y[..., None] / BORDERS - 1).min(axis=-1) < 2.0 ** -22
        differ = (held != want)[:, 0]
        assert (close | np.repeat(other, 16, axis=-1) | ~differ).all()
    got, stands_for = v.double().cpu().numpy(), held * s32
    assert (np.abs(got - stands_for) <= (2.0 ** -8 + 2.0 ** -24) * np.abs(stands_for)).all() and torch.equal(k, v)


# ---- on both sides of the lengths up to which a block takes a stream as a whole ----
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,n,keys", [(dims(8, 128, 64, 1), 1, 4096), (dims(1, 128, 16, 1), 8, 4096), (dims(8, 64, 32, 1), 1, 2112), (dims(8, 128, 32, 1), 2, 1600),
                                      (dims(8, 128, 64, 1), 4, 1600), (dims(4, 64, 16, 1), 8, 1600)])
def test_lengths_where_streams_begin_to_be_cut(d, n, keys, causal):
    step = n if causal else 0
    c = Case(d, [keys - step - 1, 70, keys - 300], [n] * 3, seed=60, causal=causal, spare_blocks=4)
    for bound in (keys - step - 1, keys - step, keys - step + 1):  # (host-known: it decides, whatever the lengths)
        check(c, *run(c, single=False, max_ctx=bound))


LONGER = [4500, 0, 1, 4240, 130, 6005]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(1, 128, 32, 3), dims(5, 128, 16), dims(3, 128, 64, 1), dims(2, 64, 32)])
def test_single_tokens_over_longer_contexts(d, causal, out_dtype):
    c = Case(d, LONGER, [1] * 6, seed=61, causal=causal, v_scale=3.0)
    check(c, *run(c, out_dtype), out_dtype)


def test_single_tokens_of_nan_over_longer_contexts():
    """As test_long_rows_of_nan_and_unlike_magnitudes."""
    c = Case(dims(8, 128, 64, 2), [4400, 300], [1, 1], seed=62)
    q = c.q.copy()
    q[0, 5, 3] = 0x7FC0
    q[0, 9] = to_host_bits(torch.from_numpy(wl.bits_to_f64(c.q[0, 9]) * 2.0 ** -20).to(torch.bfloat16))
    c.q[0, 9] = q[0, 9]
    out, lse = run(c, q=q, single=False)
    assert np.isnan(out[0, 5]).all() and np.isnan(lse[0, 5])
    out[0, 5], lse[0, 5] = c.want()[0][0, 5], c.want()[1][0, 5]
    check(c, out, lse)


def test_single_tokens_over_longer_contexts_record_values_out_of_range():
    """As test_long_contexts_record_values_out_of_range."""
    d = dims(8, 128, 16, 1)
    c = Case(d, [4300, 40, 4200], [1] * 3, seed=63)
    good = run(c, single=False)
    h = make_handle(d, torch.float32)

    def record(ctx=None, indptr=None, table=None):
        b = hb.Batch(dev_i32(c.ctx if ctx is None else ctx), dev_i32(c.table if table is None else table), *no_rings(d, 3),
                     dev_i32(c.indptr if indptr is None else indptr), max_q_len=1, total_q=3, max_ctx_len=4300)
        out, lse = torch.full((3, 8, 128), 7.0, device="cuda"), torch.full((3, 8), 7.0, device="cuda")
        hb.hswa_packed_attn(h, c.layer(), b, True, to_dev_bf16(c.q), out, lse, workspace(h, b, True))
        return hb.hswa_get_async_error(h), out.double().cpu().numpy()

    table = c.table.copy()
    table[1, 1] = 1 << 20
    st, out = record(table=table)
    assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, 1, 1 << 20), st
    assert np.abs(out[0] - good[0][0]).max() < 1e-2
    for bad in (-1, 4301):
        st, out = record(ctx=[4300, bad, 4200])
        assert st[:4] == (hb.HSWA_ERR_BOUNDS, 1, -1, bad), st
        assert np.abs(out[2] - good[0][2]).max() < 1e-2  # (other runs, other roundings)
    for indptr in ([0, 1, 2, 4], [-1, 1, 2, 3]):
        st, _ = record(indptr=np.array(indptr, np.int32))
        assert (st[0], st[2]) == (hb.HSWA_ERR_BOUNDS, -2), st


def test_single_tokens_over_longer_contexts_captured_and_repeated():
    """As test_long_calls_captured_and_repeated."""
    c, other = (Case(dims(8, 128, 64, 2), [4600, 900], [1, 1], seed=s) for s in (64, 65))
    h = make_handle(c.d, torch.float32)
    b, layer, q = c.batch(single=False), c.layer(), to_dev_bf16(c.q)
    out, lse, ws = torch.empty((2, 16, 128), device="cuda"), torch.empty((2, 16), device="cuda"), workspace(h, b, True)
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


@pytest.mark.parametrize("ctx,n", [([100, 200], [1, 1]), ([4500, 200], [1, 1]), ([100, 200], [2, 3]), ([2300, 200], [2, 3]), ([100, 200], [4, 4]), ([2300, 200], [4, 4]),
                                   ([100, 200], [40, 3]), ([3000, 200], [40, 30])])
def test_rows_before_the_first_request_and_calls_without_lse(ctx, n):
    """Row offsets that begin behind 0: rows before them and behind the last stay as they were, in the cache's calls too; no lse asked for."""
    d = dims(8, 128, 64)
    c = Case(d, ctx, n, seed=70)
    T, lead = int(c.indptr[-1]), 5
    h = make_handle(d, torch.float32)
    b = hb.Batch(dev_i32(c.ctx), dev_i32(c.table), *no_rings(d, 2), dev_i32(c.indptr + lead), max_q_len=max(n), total_q=T + lead + 3, max_ctx_len=max(ctx))
    q = torch.zeros((T + lead + 3, 16, 128), dtype=torch.bfloat16, device="cuda")
    q[lead:lead + T] = to_dev_bf16(c.q)
    outs = []
    for lse in (torch.full((T + lead + 3, 16), 7.0, device="cuda"), None):
        out, ws = torch.full(q.shape, 7.0, device="cuda"), workspace(h, b, True)
        ws.fill_(255)
        hb.hswa_packed_attn(h, c.layer(), b, True, q, out, lse, ws)
        no_error(h)
        assert (out[:lead] == 7).all() and (out[lead + T:] == 7).all()
        if lse is not None:
            assert (lse[:lead] == 7).all() and (lse[lead + T:] == 7).all()
            check(c, out[lead:lead + T].double().cpu().numpy(), lse[lead:lead + T].double().cpu().numpy())
        outs.append(out)
    assert torch.equal(*outs)
    # the step's rows back, and in again: nothing changes
    layer = c.layer()
    before = layer.pool.clone()
    k, v = (torch.full((T + lead + 3, 2, 128), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hb.hswa_packed_read(h, layer, b, k, v)
    no_error(h)
    for x in (k, v):
        assert (x[:lead] == 9).all() and (x[lead + T:] == 9).all() and (x[lead:lead + T] != 9).any(dim=(1, 2)).all()
    hb.hswa_packed_append(h, layer, b, k, v)
    no_error(h)
    again = [torch.empty_like(k) for _ in range(2)]
    hb.hswa_packed_read(h, layer, b, *again)
    no_error(h)
    assert all(torch.equal(x[lead:lead + T], y[lead:lead + T]) for x, y in zip((k, v), again))
    untouched = torch.ones_like(before, dtype=torch.bool)
    P, D = 64, 128
    for r in range(2):
        for i in range(n[r]):
            page, slot = int(c.table[r, (ctx[r] + i) // P]), (ctx[r] + i) % P
            untouched[page, :, :, slot * D // 2:(slot + 1) * D // 2] = False
            untouched[page, :, :, P * D // 2 + slot * D // 16:P * D // 2 + (slot + 1) * D // 16] = False
    assert torch.equal(layer.pool[untouched], before[untouched])


def test_append_and_read_refuse_more_heads_than_they_divide_by():
    for heads in (65536, 70001):
        d = dims(1, 64, 16, heads)
        h = make_handle(d)
        layer = hb.PackedLayer(torch.zeros((1, 2, heads, 16 * 36), dtype=torch.uint8, device="cuda"))
        k, v = (torch.zeros((1, heads, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        b = hb.Batch(dev_i32([0]), dev_i32([[0]]), *no_rings(d, 1), max_ctx_len=0)
        for call in (hb.hswa_packed_append, hb.hswa_packed_read):
            with pytest.raises(hb.HswaError) as e:
                call(h, layer, b, k, v)
            assert e.value.status == hb.HSWA_ERR_UNSUPPORTED
        no_error(h)


def test_append_and_read_of_many_heads():
    """The most heads that are taken: each head's row goes to its own slab and comes back."""
    heads = 65535
    d = dims(1, 64, 16, heads)
    h = make_handle(d)
    layer = hb.PackedLayer(torch.zeros((1, 2, heads, 16 * 36), dtype=torch.uint8, device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(14)
    k, v = (torch.randint(0, 2, (2, heads, 64), generator=g, device="cuda").mul(12).sub(6).to(torch.bfloat16) for _ in range(2))
    b = hb.Batch(dev_i32([3]), dev_i32([[0]]), *no_rings(d, 1), dev_i32([0, 2]), max_q_len=2, total_q=2, max_ctx_len=3)
    hb.hswa_packed_append(h, layer, b, k, v)
    back = [torch.empty_like(k) for _ in range(2)]
    hb.hswa_packed_read(h, layer, b, *back)
    no_error(h)
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
    touched = layer.pool.reshape(2, heads, -1)[:, :, : 16 * 32].reshape(2, heads, 16, 32).ne(0).any(dim=3)
    assert (touched[:, :, 3:5]).all() and not touched[:, :, :3].any() and not touched[:, :, 5:].any()
