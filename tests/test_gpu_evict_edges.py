"""Cross attention, accumulated attention weights and eviction at the edges of what their calls take: row counts that leave part
of a tile empty, contexts near the limit, rows of NaN, lengths past the bounds, drafts, hybrid stacks.  Tolerances as derived in
test_gpu_evict.py: S_ERR = 2^-12 is the relative error of a probability at a scale of 1 / sqrt(D)."""
import numpy as np
import pytest
import torch

import evict_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16, to_host_bits
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl
from test_gpu_evict import (NAN_BITS, S_ERR, Case, check_cross, check_weights, dims, no_error, no_rings, run_cross, run_weights,
                            weights_inputs, workspace)

pytestmark = pytest.mark.gpu


def leave_nan_in_the_accumulators():
    """Cross attention of many short prompts, whose key tiles end in slots of infinity: their raw scores stay behind in the
    accumulators of every SM."""
    c = Case(dims(8, 128, 64, 8), [9] * 40, [64] * 40, seed=100)
    run_cross(c)


@pytest.mark.parametrize("G,n", [(1, 65), (1, 96), (4, 17), (4, 24), (5, 13), (5, 19), (6, 11), (6, 16), (7, 10), (7, 13), (8, 9), (8, 12), (8, 13)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_weights_of_65_to_104_rows(G, n, D, causal):
    """Q tiles of 65 to 96 rows (and just more): columns behind them belong to no row, whatever an earlier kernel left there."""
    B = 80
    rng = np.random.default_rng(101)
    c = Case(dims(G, D, 64, 4), rng.integers(0, 500, B), [n if r % 3 else r % (n + 1) for r in range(B)], seed=102, causal=causal)
    lse, old = weights_inputs(c, 103)
    leave_nan_in_the_accumulators()
    check_weights(c, 0.5, lse, old.copy(), run_weights(c, 0.5, lse, old))


@pytest.mark.parametrize("n", [1, 5, 20])
def test_weights_of_the_oldest_keys_of_a_context_past_2_to_28(n):
    """2^28 and some positions behind a block table that names eight pages over and over: positions with equal slots of equal
    pages get equal weights, the oldest ones too."""
    d, L, pages = dims(8, 64, 64, 1), 2 ** 28 + 200, 8
    rng = np.random.default_rng(110)
    pool = wl.bf16_bits_normal(111, (pages, 2, 1, 64, 64))
    q = wl.bf16_bits_normal(112, (n, 8, 64))
    blocks = -(-(L + n) // 64)
    table = torch.arange(blocks, dtype=torch.int32, device="cuda") % pages
    lse = rng.uniform(2.0, 4.0, (n, 8)).astype(np.float32)
    b = hb.Batch(dev_i32([L]), table[None], *no_rings(d, 1), dev_i32([0, n]), max_q_len=n, total_q=n, max_ctx_len=L)
    w = torch.full((1, 1, L + n + 5), -1.0, device="cuda")
    h = make_handle(d)
    hb.hswa_attn_weights(h, hb.Layer(to_dev_bf16(pool), False), b, True, to_dev_bf16(q), torch.from_numpy(lse).cuda(), 0.0, w)
    no_error(h)
    s = wl.bits_to_f64(q).reshape(n * 8, 64) @ wl.bits_to_f64(pool[:, 0, 0]).reshape(pages * 64, 64).T / 8.0
    e = np.exp(s - lse.reshape(n * 8, 1))
    want = torch.from_numpy(e.sum(axis=0)).float().cuda()
    tol = (S_ERR + (8 * n + 4) * 2.0 ** -24) * want
    whole = L // (pages * 64) * (pages * 64)
    assert ((w[0, 0, :whole].view(-1, pages * 64) - want).abs_() <= tol).all()
    new = np.arange(n)[:, None] >= np.arange(n)[None, :]  # the step's own positions: causal
    at = (L + np.arange(n)) % (pages * 64)
    own = (e.reshape(n, 8, -1).sum(axis=1)[:, at] * new).sum(axis=0)
    assert np.allclose(w[0, 0, L:L + n].cpu().numpy(), own, rtol=S_ERR + (8 * n + 4) * 2.0 ** -24, atol=0)
    assert (w[0, 0, L + n:] == -1).all()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)], ids=str)
@pytest.mark.parametrize("ctx", [1, 300, 9000])
@pytest.mark.parametrize("n", [1, 3])
def test_cross_shows_a_row_of_nan(d, ctx, n):
    """A NaN in q makes every score of its row NaN: that row is NaN, with one slice of the keys and with many."""
    c = Case(d, [ctx, 5], [n, 1], seed=120)
    c.q[0, 1, 7] = NAN_BITS
    out, lse = run_cross(c)
    assert np.isnan(out[0, 1]).all() and np.isnan(lse[0, 1])
    out[0, 1] = lse[0, 1] = 0
    assert np.isfinite(out).all() and np.isfinite(lse).all()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)], ids=str)
@pytest.mark.parametrize("ctx", [1, 65, 129, 4097])
@pytest.mark.parametrize("n", [1, 3])
def test_cross_shows_a_nan_in_the_last_key(d, ctx, n):
    """Alone in the request, in its tile, or in its slice of the keys."""
    c = Case(d, [ctx, 5], [n, 1], seed=121)
    c.pool[c.table[0, (ctx - 1) // d.page_size], 0, 1, (ctx - 1) % d.page_size] = NAN_BITS
    out, lse = run_cross(c)
    assert np.isnan(out[:n, d.group:]).all() and np.isnan(lse[:n, d.group:]).all()
    assert np.isfinite(out[:n, :d.group]).all() and np.isfinite(out[n:]).all()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)], ids=str)
@pytest.mark.parametrize("ctx", [[300, 100, 50], [9000, 700, 0]])
@pytest.mark.parametrize("max_q,n", [(7, [90, 5, 100]), (50, [20, 200, 3])])
def test_cross_leaves_rows_past_the_bound_alone(d, ctx, max_q, n):
    """Requests longer than max_q_len, with and without slices of the keys: a row is right or as it was, and what the workspace
    held does not matter."""
    c = Case(d, ctx, n, seed=130)
    h, b, T = make_handle(d), c.batch(max_q=max_q), int(c.indptr[-1])
    out = torch.full((T, d.num_q_heads, d.head_dim), 7.0, device="cuda")
    lse = torch.full((T, d.num_q_heads), 7.0, device="cuda")
    ws = workspace(h, b)
    ws.view(torch.float32).fill_(float("nan"))
    hb.hswa_cross_attn(h, hb.Layer(to_dev_bf16(c.pool), False), b, to_dev_bf16(c.q), out, lse, ws)
    st = hb.hswa_get_async_error(h)
    assert st[0] == hb.HSWA_ERR_BOUNDS and st[2] == -2 and st[3] == n[st[1]] > max_q, st
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    want, want_lse, mag = ref.cross_attention(c.pool, c.table, c.ctx, c.indptr, c.q, c.scale)
    with np.errstate(invalid="ignore"):
        right = (np.abs(out - want) <= (2.0 ** -8 + 2 * S_ERR) * mag + 1e-7).all(axis=2) & ((np.abs(lse - want_lse) <= S_ERR) | (lse == want_lse))
    same = (out == 7).all(axis=2) & (lse == 7)
    for r in range(3):
        rows = slice(int(c.indptr[r]), int(c.indptr[r]) + min(int(c.n[r]), max_q))
        assert right[rows].all(), r
    assert (right | same).all()
    assert same.any()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)], ids=str)
@pytest.mark.parametrize("ctx", [[300, 100, 50], [9000, 700, 800]])
@pytest.mark.parametrize("n", [[1, 1, 1], [2, 3, 20], [30, 40, 50]])
def test_row_offsets_past_total_q_are_recorded(d, ctx, n):
    """The last request's rows pass total_q (and one request's begin there): they are neither read nor written."""
    c = Case(d, ctx, n, seed=140)
    h, T, cut = make_handle(d), int(c.indptr[-1]), int(c.indptr[2])
    q, layer = to_dev_bf16(c.q), hb.Layer(to_dev_bf16(c.pool), False)
    want, want_lse, mag = ref.cross_attention(c.pool, c.table, c.ctx, c.indptr, c.q, c.scale)
    for total in (cut, T - 1):
        if total < max(n):
            continue
        b = hb.Batch(dev_i32(c.ctx), dev_i32(c.table), *no_rings(d, 3), dev_i32(c.indptr), max_q_len=max(n), total_q=total, max_ctx_len=max(ctx))
        out = torch.full((T, d.num_q_heads, d.head_dim), 7.0, device="cuda")
        lse = torch.full((T, d.num_q_heads), 7.0, device="cuda")
        ws = torch.full((workspace(h, b).numel() // 4 + 64 * 1024,), 7.0, device="cuda")
        need = hb.hswa_cross_workspace_need(h, 3, total, max(n), max(ctx))
        hb.hswa_cross_attn(h, layer, b, q, out, lse, ws)
        assert hb.hswa_get_async_error(h) == (hb.HSWA_ERR_BOUNDS, 2, -2, n[2])
        assert (out[total:] == 7).all() and (lse[total:] == 7).all() and (ws[need // 4:] == 7).all()
        got, got_lse = out[:cut].double().cpu().numpy(), lse[:cut].double().cpu().numpy()
        assert (np.abs(got - want[:cut]) <= (2.0 ** -8 + 2 * S_ERR) * mag[:cut] + 1e-7).all() and (np.abs(got_lse - want_lse[:cut]) <= S_ERR).all()
        w = torch.full((3, d.num_kv_heads, max(ctx)), 7.0, device="cuda")
        hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
        assert hb.hswa_get_async_error(h) == (hb.HSWA_ERR_BOUNDS, 2, -2, n[2])
        assert (w[2] == 7).all() and not (w[:2, :, :50] == 7).any()


def test_negative_row_offsets_are_recorded():
    d = dims(8, 128, 64)
    for n in ([1, 1], [4, 30]):
        c = Case(d, [300, 100], n, seed=141)
        h, T = make_handle(d), int(c.indptr[-1])
        q, layer = to_dev_bf16(c.q), hb.Layer(to_dev_bf16(c.pool), False)
        b = hb.Batch(dev_i32(c.ctx), dev_i32(c.table), *no_rings(d, 2), dev_i32([n[0] - 2 * n[0], 0, n[1]]), max_q_len=max(n), total_q=T,
                     max_ctx_len=300)
        out, lse = torch.full((T, 16, 128), 7.0, device="cuda"), torch.full((T, 16), 7.0, device="cuda")
        hb.hswa_cross_attn(h, layer, b, q, out, lse, workspace(h, b))
        assert hb.hswa_get_async_error(h) == (hb.HSWA_ERR_BOUNDS, 0, -2, n[0])
        assert (out[n[1]:] == 7).all() and (out[:n[1]] != 7).any(dim=-1).all()
        w = torch.full((2, 2, 300), 7.0, device="cuda")
        hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
        assert hb.hswa_get_async_error(h) == (hb.HSWA_ERR_BOUNDS, 0, -2, n[0])
        assert (w[0] == 7).all() and not (w[1, :, :100] == 7).any()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16)], ids=str)
@pytest.mark.parametrize("n", [[9, 1, 1], [9, 3, 20], [30, 40, 50]])
def test_cross_of_the_last_requests_of_a_batch(d, n):
    """Row offsets that do not begin at 0 (the last requests of a longer batch): the rows before them stay as they were."""
    c = Case(d, [10, 9000, 700], n, seed=145)
    h, T, first = make_handle(d), int(c.indptr[-1]), int(c.indptr[1])
    q, layer, indptr = to_dev_bf16(c.q), hb.Layer(to_dev_bf16(c.pool), False), dev_i32(c.indptr)
    b = hb.Batch(dev_i32(c.ctx[1:]), dev_i32(c.table[1:]), *no_rings(d, 2), indptr[1:], max_q_len=max(n[1:]), total_q=T, max_ctx_len=9000)
    out, lse = torch.full((T, d.num_q_heads, d.head_dim), 7.0, device="cuda"), torch.full((T, d.num_q_heads), 7.0, device="cuda")
    ws = workspace(h, b)
    ws.view(torch.float32).fill_(float("nan"))
    hb.hswa_cross_attn(h, layer, b, q, out, lse, ws)
    no_error(h)
    assert (out[:first] == 7).all() and (lse[:first] == 7).all()
    want, want_lse, mag = ref.cross_attention(c.pool, c.table, c.ctx, c.indptr, c.q, c.scale)
    got, got_lse = out.double().cpu().numpy()[first:], lse.double().cpu().numpy()[first:]
    assert (np.abs(got - want[first:]) <= (2.0 ** -8 + 2 * S_ERR) * mag[first:] + 1e-7).all() and (np.abs(got_lse - want_lse[first:]) <= S_ERR).all()
    w = torch.full((2, d.num_kv_heads, 9000), 7.0, device="cuda")
    hb.hswa_attn_weights(h, layer, b, False, q, lse, 0.0, w)
    no_error(h)
    rows = torch.tensor(n[1:], device="cuda")[:, None] * d.group  # every row's probabilities sum to one
    assert torch.allclose(torch.stack([w[0].double().sum(-1), w[1, :, :700].double().sum(-1)]), rows.double().expand(2, d.num_kv_heads),
                          rtol=2 * S_ERR + 2.0 ** -11, atol=0)


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(3, 64, 16), dims(5, 128, 32)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [[1, 1, 1], [4, 0, 3], [9, 12, 2], [40, 16, 64], [300, 5, 500]])
@pytest.mark.parametrize("what", ["nan", "large"])
def test_weights_of_rows_without_a_vote(d, causal, n, what):
    """A row whose lse is minus infinity adds nothing, whatever its q is."""
    c = Case(d, [700, 90, 300], n, seed=150, causal=causal)
    lse, old = weights_inputs(c, 151)
    rng = np.random.default_rng(152)
    out = rng.random(lse.shape) < 0.3
    out[0, 0] = True
    lse[out] = -np.inf
    q = c.q.copy()
    q[out] = NAN_BITS if what == "nan" else wl.bf16_bits_const(3e38, (1,))[0]
    want_q, c.q = c.q, q
    got = run_weights(c, 0.5, lse, old)
    c.q = want_q
    check_weights(c, 0.5, lse, old.copy(), got)


def test_cross_of_a_padded_batch_without_any_token():
    """No request of the step has a token (max_q_len = 0), the tensors are padded: nothing to do, as for the weights."""
    d = dims(8, 128, 64)
    c = Case(d, [100, 200], [1, 1], seed=160)
    h, layer = make_handle(d), hb.Layer(to_dev_bf16(c.pool), False)
    b = hb.Batch(dev_i32(c.ctx), dev_i32(c.table), *no_rings(d, 2), dev_i32([0, 0, 0]), max_q_len=0, total_q=2, max_ctx_len=200)
    out, lse = torch.full((2, 16, 128), 7.0, device="cuda"), torch.full((2, 16), 7.0, device="cuda")
    assert hb.hswa_cross_workspace_need(h, 2, 2, 0, 200) == 0
    hb.hswa_cross_attn(h, layer, b, to_dev_bf16(c.q), out, lse, None)
    no_error(h)
    assert (out == 7).all() and (lse == 7).all()


def drafts(d, ctx0, q_len, seed):
    B = len(ctx0)
    c = Case(d, ctx0, [q_len] * B, seed=seed, causal=True, spare_blocks=1)
    kv = wl.bf16_bits_normal(seed + 1, (B, q_len, 2, d.num_kv_heads, d.head_dim))
    return c, np.ascontiguousarray(kv[:, :, 0]), np.ascontiguousarray(kv[:, :, 1])


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16)], ids=str)
@pytest.mark.parametrize("q_len", [2, 4])
def test_weights_of_drafts(d, q_len):
    """Multi-token decode steps of which some drafts are rejected: a batch with row offsets says what q's rows are, and a rejected
    draft, whose lse is set to minus infinity, has no vote."""
    ctx0 = np.array([300, 5, 64], np.int32)
    c, k_new, v_new = drafts(d, ctx0, q_len, 170)
    B, h, pool = 3, make_handle(d), to_dev_bf16(c.pool)
    layer, q = hb.Layer(pool, False), to_dev_bf16(c.q.reshape(B, q_len, d.num_q_heads, d.head_dim))
    ctx, head = dev_i32(ctx0), torch.zeros((B,), dtype=torch.int32, device="cuda")
    ring = torch.zeros((B, d.ring_pages), dtype=torch.int32, device="cuda")
    b = hb.Batch(ctx, dev_i32(c.table), ring, head, None, max_ctx_len=300)
    out = torch.zeros((B, q_len, d.num_q_heads, d.head_dim), device="cuda")
    lse = torch.zeros((B, q_len, d.num_q_heads), device="cuda")
    ws = torch.empty((max(256, hb.hswa_workspace_bytes(h, B, B * q_len, 300)),), dtype=torch.uint8, device="cuda")
    hb.hswa_decode_attn_mtp(h, layer, b, q_len, q, to_dev_bf16(k_new), to_dev_bf16(v_new), out, lse, ws)
    accepted = np.array([q_len, 1, q_len - 1], np.int32)
    rejected = torch.arange(q_len)[None, :] >= torch.from_numpy(accepted)[:, None]
    lse[rejected.cuda()] = -float("inf")
    old = np.random.default_rng(171).random((B, d.num_kv_heads, 310)).astype(np.float32)
    w = torch.from_numpy(old).cuda()
    with pytest.raises(AssertionError):  # one row per request is not what this q holds
        hb.hswa_attn_weights(h, layer, b, True, q, lse, 0.75, w)
    with pytest.raises(AssertionError):
        hb.hswa_cross_attn(h, layer, b, q, out, lse, ws)
    rows = hb.Batch(ctx, dev_i32(c.table), ring, head, dev_i32(c.indptr), max_q_len=q_len, total_q=B * q_len, max_ctx_len=300)
    hb.hswa_attn_weights(h, layer, rows, True, q, lse, 0.75, w)
    no_error(h)
    c.pool = to_host_bits(pool)
    check_weights(c, 0.75, lse.cpu().numpy().reshape(B * q_len, -1), old, w.cpu().numpy())
    # the next step begins at the accepted tokens; what a rejected draft's position held counts as 0
    indptr = np.zeros(B + 1, np.int32)
    indptr[1:] = np.cumsum(accepted)
    hb.hswa_step_advance(h, B, ctx, head, dev_i32(indptr))
    before = w.cpu().numpy().copy()
    c.ctx = ctx0 + accepted
    c.cached = c.ctx + 1
    c.n[:] = 1
    c.indptr, c.q = np.arange(B + 1, dtype=np.int32), wl.bf16_bits_normal(175, (B, d.num_q_heads, d.head_dim))
    for r in range(B):  # room for one more token
        if c.table[r, c.ctx[r] // d.page_size] < 0:
            c.table[r, c.ctx[r] // d.page_size] = c.free.pop()
    nk, nv = wl.bf16_bits_normal(176, (B, d.num_kv_heads, d.head_dim)), wl.bf16_bits_normal(177, (B, d.num_kv_heads, d.head_dim))
    b = hb.Batch(ctx, dev_i32(c.table), ring, head, None, max_ctx_len=304)
    out, lse = torch.zeros((B, d.num_q_heads, d.head_dim), device="cuda"), torch.zeros((B, d.num_q_heads), device="cuda")
    hb.hswa_decode_attn(h, layer, b, to_dev_bf16(c.q), to_dev_bf16(nk), to_dev_bf16(nv), out, lse, ws)
    hb.hswa_attn_weights(h, layer, b, True, to_dev_bf16(c.q), lse, 1.0, w)
    no_error(h)
    c.pool = to_host_bits(pool)
    check_weights(c, 1.0, lse.cpu().numpy(), before, w.cpu().numpy())


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16)], ids=str)
@pytest.mark.parametrize("kept", [[127, 200], [128, 127]])
def test_swa_layers_of_a_hybrid_stack_after_an_eviction(d, kept):
    """ctx_len cut to what the Full layers keep, at least W - 1: an SWA layer's ring, head and results stay what they were, and so does
    its bookkeeping once swa_valid_from has moved by as many positions."""
    B, ctx0 = 2, np.array([300, 1000], np.int32)
    h, kept = make_handle(d), np.asarray(kept, np.int32)
    C = d.ring_slots
    pool = torch.full((B * d.ring_pages, 2, d.num_kv_heads, d.page_size, d.head_dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    ring = dev_i32(np.random.default_rng(180).permutation(B * d.ring_pages).reshape(B, -1))
    ctx, head = dev_i32([0, 0]), dev_i32([0, 0])
    indptr = dev_i32([0, 300, 1300])
    kv = [to_dev_bf16(wl.bf16_bits_normal(181 + i, (1300, d.num_kv_heads, d.head_dim))) for i in range(2)]
    table = torch.zeros((B, 1), dtype=torch.int32, device="cuda")
    layer = hb.Layer(pool, True)
    hb.hswa_kv_append(h, layer, hb.Batch(ctx, table, ring, head, indptr, max_q_len=1000, total_q=1300, max_ctx_len=0), *kv)
    hb.hswa_step_advance(h, B, ctx, head, indptr)
    valid_from = dev_i32([0, 0])
    hb.hswa_swa_release(h, B, ctx, None, valid_from)
    assert valid_from.tolist() == [173, 873]
    state = pool.clone(), head.clone()
    results = []
    for lens in (ctx0, kept):
        pool.copy_(state[0])
        head.copy_(state[1])
        ctx.copy_(torch.from_numpy(lens))
        for k in range(3):
            q, kn, vn = (to_dev_bf16(wl.bf16_bits_normal(190 + 3 * k + i, (B, m, d.head_dim))) for i, m in
                         enumerate((d.num_q_heads, d.num_kv_heads, d.num_kv_heads)))
            out, lse = torch.zeros((B, d.num_q_heads, d.head_dim), device="cuda"), torch.zeros((B, d.num_q_heads), device="cuda")
            hb.hswa_decode_attn(h, layer, hb.Batch(ctx, table, ring, head, None, max_ctx_len=int(lens.max()) + k), q, kn, vn, out, lse)
            hb.hswa_step_advance(h, B, ctx, head)
            results.append((out, lse))
    no_error(h)
    for a, e in zip(results[3:], results[:3]):
        assert torch.isfinite(e[0]).all() and torch.equal(a[0], e[0]) and torch.equal(a[1], e[1])
    # the bookkeeping, moved by the positions that went
    ctx.copy_(torch.from_numpy(kept))
    valid_from = (valid_from - dev_i32(ctx0 - kept)).clamp_(min=0)
    mask = torch.zeros((B, 400), dtype=torch.uint8, device="cuda")
    hb.hswa_swa_valid_mask(h, B, ctx, valid_from, mask)
    assert mask.sum(dim=1).tolist() == [127, 127]
    for r in range(B):
        assert hb.hswa_window_safe_len(int(kept[r]), 128, mask[r].cpu().numpy()) == kept[r]
    hb.hswa_swa_release(h, B, ctx, None, valid_from)
    assert valid_from.tolist() == [int(k) - 127 for k in kept] and C >= 129
    no_error(h)


def scale_err(scale):
    """Relative error of a probability where the score's error bound of 2^-10 (before the scale) is multiplied by `scale`."""
    return scale * 2.0 ** -10 + S_ERR


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(5, 64, 16), dims(1, 128, 32)], ids=str)
@pytest.mark.parametrize("n", [1, 3, 200])
@pytest.mark.parametrize("sm_scale", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("ctx", [[3000, 500], [9000, 70, 0, 1200] * 12])
def test_cross_of_growing_maxima(d, n, sm_scale, ctx):
    """Scores so far apart that row maxima grow by more than the lazy rescale's slack (8 in log2 units) from tile to tile; every
    form, with and without slices."""
    ctx = ctx if n < 200 else ctx[:4]
    c = Case(d, ctx, [n] * len(ctx), seed=200)
    c.scale = sm_scale
    S = scale_err(sm_scale)
    K, Q = ref.rows(c.pool, c.table, 0, ctx[0], 0), wl.bits_to_f64(c.q[:n])
    s = np.einsum("ihd,jd->ihj", Q[:, : d.group], K[:, 0]) * sm_scale * 1.4427
    assert sm_scale < 1 or (s.max(axis=-1) - s[..., :128].max(axis=-1) > 8).any(), "no row's maximum grows enough"
    h, b, T = make_handle(d, sm_scale=sm_scale), c.batch(), int(c.indptr[-1])
    out, lse = torch.zeros((T, d.num_q_heads, d.head_dim), device="cuda"), torch.zeros((T, d.num_q_heads), device="cuda")
    hb.hswa_cross_attn(h, hb.Layer(to_dev_bf16(c.pool), False), b, to_dev_bf16(c.q), out, lse, workspace(h, b))
    no_error(h)
    want, want_lse, mag = ref.cross_attention(c.pool, c.table, c.ctx, c.indptr, c.q, sm_scale)
    assert (np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -8 + 2 * S) * mag + 1e-7).all()
    some = np.isfinite(want_lse)
    got_lse = lse.double().cpu().numpy()
    assert (np.abs(got_lse - want_lse)[some] <= S).all() and (got_lse[~some] == -np.inf).all()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(5, 64, 16)], ids=str)
@pytest.mark.parametrize("n", [1, 3, 60])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sm_scale", [0.03125, 1.0])
def test_weights_at_other_scales(d, n, causal, sm_scale):
    c = Case(d, [900, 40, 0], [n, n, n], seed=210, causal=causal)
    c.scale = sm_scale
    lse, old = weights_inputs(c, 211)
    h, w = make_handle(d, sm_scale=sm_scale), torch.from_numpy(old).cuda()
    hb.hswa_attn_weights(h, hb.Layer(to_dev_bf16(c.pool), False), c.batch(), causal, to_dev_bf16(c.q), torch.from_numpy(lse).cuda(), 0.5, w)
    no_error(h)
    want = ref.attn_weights(c.pool, c.table, c.ctx, c.indptr, c.q, lse, sm_scale, causal, 0.5, old)
    # (|lse| < 256 here: x = s log2(e) - lse log2(e) is rounded to 2^-24 of that, 2^-15 relative to 2^x, within S_ERR)
    assert (np.abs(w.cpu().numpy() - want) <= (scale_err(sm_scale) + (n * d.group + 2) * 2.0 ** -24) * want + 1e-30).all()


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16)], ids=str)
@pytest.mark.parametrize("n", [1, 5])
def test_cross_join_of_many_slices_in_bf16(d, n):
    c = Case(d, [9000], [n], seed=220)
    check_cross(c, *run_cross(c, torch.bfloat16), torch.bfloat16)


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(5, 64, 16), dims(8, 128, 32)], ids=str)
def test_weights_with_the_lse_of_a_prefill(d):
    """A prompt's prefill, whose lse goes into the weights; a second call lets the last tokens alone vote."""
    ctx0, n = np.array([130, 0, 77], np.int32), np.array([200, 40, 3], np.int32)
    c = Case(d, ctx0, n, seed=230, causal=True)
    h, pool, b, T = make_handle(d), to_dev_bf16(c.pool), c.batch(), int(c.indptr[-1])
    layer, q = hb.Layer(pool, False), to_dev_bf16(c.q)
    kn, vn = (to_dev_bf16(wl.bf16_bits_normal(231 + i, (T, d.num_kv_heads, d.head_dim))) for i in range(2))
    out, lse = torch.zeros((T, d.num_q_heads, d.head_dim), device="cuda"), torch.zeros((T, d.num_q_heads), device="cuda")
    hb.hswa_prefill_attn(h, layer, b, q, kn, vn, True, out, lse)
    old = np.zeros((3, d.num_kv_heads, 340), np.float32)
    w = torch.from_numpy(old.copy()).cuda()
    hb.hswa_attn_weights(h, layer, b, True, q, lse, 0.0, w)
    no_error(h)
    c.pool = to_host_bits(pool)
    check_weights(c, 0.0, lse.cpu().numpy(), old, w.cpu().numpy())
    total = w.double().sum(dim=-1).cpu().numpy()
    # every row's probabilities sum to one (the prefill's lse sums rounded ones where it sums them so: 2^-8)
    assert np.allclose(total, (n * d.group)[:, None], rtol=2.0 ** -8 + 2 * S_ERR, atol=0)
    last = 2  # the last two tokens of each prompt, the context that much longer
    keep = np.concatenate([np.arange(int(e) - last, int(e)) for e in c.indptr[1:]])
    c.ctx, c.n, c.indptr, c.q = ctx0 + n - last, np.full(3, last, np.int32), np.arange(4, dtype=np.int32) * last, c.q[keep]
    w = torch.from_numpy(old.copy()).cuda()
    hb.hswa_attn_weights(h, layer, c.batch(), True, to_dev_bf16(c.q), lse[torch.from_numpy(keep).cuda()].contiguous(), 0.0, w)
    no_error(h)
    check_weights(c, 0.0, lse.cpu().numpy()[keep], old, w.cpu().numpy())


@pytest.mark.parametrize("d", [dims(5, 128, 32), dims(8, 64, 64)], ids=str)
def test_encoder_states_appended_then_attended(d):
    """The states enter the pages by hswa_kv_append, in two chunks; tokens attend to all of them."""
    c = Case(d, [150, 0, 77], [20, 3, 1], seed=240)
    blank = np.full_like(c.pool, NAN_BITS)
    h, pool = make_handle(d), to_dev_bf16(blank)
    layer, table = hb.Layer(pool, False), dev_i32(c.table)
    ctx, head = dev_i32([0, 0, 0]), dev_i32([0, 0, 0])
    ring = torch.zeros((3, d.ring_pages), dtype=torch.int32, device="cuda")
    done = np.zeros(3, np.int64)
    for part in ([100, 0, 77], [50, 0, 0]):
        kv = []
        for which in (0, 1):
            rows = [c.pool[c.table[r, p // d.page_size], which, :, p % d.page_size] for r in range(3) for p in range(done[r], done[r] + part[r])]
            kv.append(to_dev_bf16(np.stack(rows)))
        indptr = dev_i32(np.concatenate([[0], np.cumsum(part)]))
        hb.hswa_kv_append(h, layer, hb.Batch(ctx, table, ring, head, indptr, max_q_len=max(part), total_q=sum(part), max_ctx_len=int(done.max())), *kv)
        hb.hswa_step_advance(h, 3, ctx, head, indptr)
        done += part
    assert ctx.tolist() == [150, 0, 77]
    b = hb.Batch(ctx, table, ring, head, dev_i32(c.indptr), max_q_len=20, total_q=24, max_ctx_len=150)
    out, lse = torch.zeros((24, d.num_q_heads, d.head_dim), device="cuda"), torch.zeros((24, d.num_q_heads), device="cuda")
    hb.hswa_cross_attn(h, layer, b, to_dev_bf16(c.q), out, lse, workspace(h, b))
    no_error(h)
    check_cross(c, out.double().cpu().numpy(), lse.double().cpu().numpy())


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16, 1)], ids=str)
def test_compact_of_positions_in_any_order_and_twice(d):
    """keep_idx by the caller: descending, and one position many times."""
    c = Case(d, [300, 70], [1, 1], seed=250)
    kept = np.array([90, 70], np.int32)
    idx = np.full((2, d.num_kv_heads, 90), -1, np.int32)
    idx[0], idx[1, :, :70] = np.arange(299, 209, -1), 69
    blocks = -(-90 // d.page_size)
    dst = (len(c.pool) + np.arange(2 * blocks)).reshape(2, blocks)
    c.pool = np.concatenate([c.pool, np.full((2 * blocks, *c.pool.shape[1:]), NAN_BITS, np.uint16)])
    h, pool = make_handle(d), to_dev_bf16(c.pool)
    hb.hswa_evict_compact(h, hb.Layer(pool, False), c.batch(), dev_i32(idx), dev_i32(kept), dev_i32(dst))
    no_error(h)
    assert np.array_equal(to_host_bits(pool), ref.evict_compact(c.pool, c.table, idx, kept, dst))


def test_several_streams_at_once():
    """Cross attention, weights and a choice of positions on several streams at a time, each with its own handle and workspace: every
    result is that of the call by itself."""
    jobs = []
    for i, (d, n) in enumerate([(dims(8, 128, 64, 4), 64), (dims(8, 64, 16, 4), 5), (dims(5, 128, 32, 4), 13), (dims(8, 128, 64, 4), 1)]):
        rng = np.random.default_rng(260 + i)
        c = Case(d, rng.integers(1, 900, 24), [n] * 24, seed=261 + i)
        h, b, T = make_handle(d), c.batch(), int(c.indptr[-1])
        j = dict(h=h, b=b, layer=hb.Layer(to_dev_bf16(c.pool), False), q=to_dev_bf16(c.q), ws=workspace(h, b), keep=dev_i32([40] * 24))
        j["out"], j["lse"] = torch.zeros((T, d.num_q_heads, d.head_dim), device="cuda"), torch.zeros((T, d.num_q_heads), device="cuda")
        j["w"] = torch.zeros((24, 4, 900), device="cuda")
        j["idx"], j["kept"] = torch.zeros((24, 4, 40), dtype=torch.int32, device="cuda"), torch.zeros((24,), dtype=torch.int32, device="cuda")
        jobs.append(j)

    def run(j):
        hb.hswa_cross_attn(j["h"], j["layer"], j["b"], j["q"], j["out"], j["lse"], j["ws"])
        hb.hswa_attn_weights(j["h"], j["layer"], j["b"], False, j["q"], j["lse"], 0.0, j["w"])
        hb.hswa_evict_select(j["h"], 24, j["b"].ctx_len, 900, j["w"], j["keep"], j["idx"], j["kept"], protect_last=4)

    names = ("out", "lse", "w", "idx", "kept")
    for j in jobs:
        run(j)
    torch.cuda.synchronize()
    want = [[j[k].clone() for k in names] for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        for j in jobs:
            for k in names:
                j[k].zero_()
        torch.cuda.synchronize()
        for j, s in zip(jobs, streams):
            with torch.cuda.stream(s):
                run(j)
        torch.cuda.synchronize()
        for j, e in zip(jobs, want):
            assert all(torch.equal(j[k], x) for k, x in zip(names, e))
    for j in jobs:
        no_error(j["h"])
