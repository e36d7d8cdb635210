"""Forking, compacting and copying pages on the GPU, against their statement page by page: equal, entry for entry."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl
from test_gpu_packed import S_ERR, dims, no_error, no_rings, workspace

pytestmark = pytest.mark.gpu
FILL = -7


def state(rng, P, rows, hi, pages, cache=0.1):
    """Counts, a table and the pages that each row holds; a prefix cache holds some pages too, of the rows' and of others."""
    lens = rng.integers(0, hi + 1, rows) if rows else np.zeros(0, int)
    held = (-(-lens // P)).astype(np.int32)
    if rows:
        held += rng.integers(0, 2, rows).astype(np.int32)  # a page in reserve
    blocks = max(1, int(held.max(initial=0)))
    perm = rng.permutation(pages)
    table = np.full((rows, blocks), -1, np.int32)
    counts = np.zeros(pages, np.int32)
    at = 0
    for r in range(rows):
        table[r, : held[r]] = perm[at:at + held[r]]
        at += held[r]
    counts[perm[:at]] = 1
    counts += rng.random(pages) < cache
    return counts, table, held, lens


def fork(h, counts, table, held, parent, length, need, out_blocks, sub=None):
    n, pages = len(parent), len(counts)
    dev = [dev_i32(x) for x in (counts, table, held, parent, length, need)]
    ref_out = torch.full((pages,), FILL, dtype=torch.int32, device="cuda")
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((n, out_blocks), (n,), (n,), (n,))]
    ws = torch.full((hb.hswa_pages_workspace_need(h, pages),), 255, dtype=torch.uint8, device="cuda")
    hb.hswa_pages_fork(h, dev[0], ref_out, dev[1], dev[2], dev[3], dev[4], dev[5], *outs, ws)
    return [x.cpu().numpy() for x in (ref_out, *outs)]


def check_fork(h, P, counts, table, held, parent, length, need, out_blocks):
    got = fork(h, counts, table, held, parent, length, need, out_blocks)
    want = ref.fork(counts, table, held, parent, length, need, P, out_blocks, FILL)
    no_error(h)
    for g, w, name in zip(got, want, ("ref", "table", "held", "src", "dst")):
        assert np.array_equal(g, w), (name, np.argwhere(g != w)[:5])
    return got


def children(rng, P, rows_out, held, lens, extra):
    rows_in = len(held)
    parent = rng.integers(-1, rows_in, rows_out).astype(np.int32)
    length = np.array([0 if p < 0 else max(0, int(lens[p]) - int(rng.integers(0, 2 * P) * rng.integers(0, 2))) for p in parent], np.int32)
    need = (length + rng.integers(0, extra + 1, rows_out)).astype(np.int32)
    return parent, length, need


@pytest.mark.parametrize("P", [16, 32, 64])
@pytest.mark.parametrize("rows_in,rows_out,hi,pages", [(1, 1, 1, 7), (3, 5, 100, 100), (8, 8, 300, 2048), (40, 64, 700, 5001), (0, 3, 0, 33),
                                                       (5, 0, 90, 64), (300, 1100, 40, 40000)])
def test_fork(P, rows_in, rows_out, hi, pages):
    rng = np.random.default_rng(P + rows_in)
    h = make_handle(dims(1, 64, P, 1))
    for _ in range(3):
        counts, table, held, lens = state(rng, P, rows_in, hi * P // 16, pages)
        parent, length, need = children(rng, P, rows_out, held, lens, 3 * P)
        blocks = max(1, int((-(-need.astype(int) // P)).max(initial=0)))
        check_fork(h, P, counts, table, held, parent, length, need, blocks)


def test_fork_of_one_row_into_many_and_shorter_and_longer_children():
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts, table, held = np.zeros(500, np.int32), np.arange(40, dtype=np.int32)[None] * 3, np.array([40], np.int32)
    counts[table[0]] = 1
    n = 33
    length = np.array([(i * 37) % 640 for i in range(n)], np.int32)
    check_fork(h, P, counts, table, held, np.zeros(n, np.int32), length, length + 5, 42)


def test_fork_of_long_rows():
    """Rows of thousands of pages, most of which go on unchanged: shared places in many chunks, long reserves."""
    rng = np.random.default_rng(3)
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts, table, held, lens = state(rng, P, 6, 40000, 30011)
    parent, length, need = np.array([0, 1, 1, 3, 4, 4], np.int32), lens[[0, 1, 1, 3, 4, 4]].astype(np.int32), np.full(6, 48000, np.int32)
    length[5] //= 2
    check_fork(h, P, counts, table, held, parent, length, need, 3000)


def test_fork_at_the_limits():
    rng = np.random.default_rng(4)
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts, table, held, lens = state(rng, P, 4096, 30, 1 << 23, cache=0.0)
    parent = rng.permutation(4096).astype(np.int32)
    got = fork(h, counts, table, held, parent, lens[parent].astype(np.int32), np.full(4096, 64, np.int32), 4)
    no_error(h)
    assert (got[2] == 4).all() and got[0].sum() == 4 * 4096 and got[0].max() == 1
    assert len(np.unique(got[1])) == 4 * 4096
    assert (got[3] == -1).all()


def test_fork_without_enough_pages_does_nothing():
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts = np.ones(64, np.int32)
    counts[[7, 9]] = 0
    table, held = np.array([[1, 2]], np.int32), np.array([2], np.int32)
    got = fork(h, counts, table, held, [0, 0], [20, 20], [40, 40], 4)
    assert hb.hswa_get_async_error(h) == (hb.HSWA_ERR_BOUNDS, -1, 3, 2)
    assert np.array_equal(got[0], counts) and all((g == FILL).all() for g in got[1:])
    got = fork(h, counts, table, held, [0, 0], [20, 20], [32, 32], 4)  # one page: the second child's copy
    no_error(h)
    assert got[1][:, :2].tolist() == [[1, 2], [1, 7]]


@pytest.mark.parametrize("bad", [dict(parent=[1]), dict(parent=[-2]), dict(length=[33]), dict(length=[-1]), dict(need=[65]), dict(held=[3]),
                                 dict(held=[-1]), dict(parent=[-1])])
def test_fork_records_arguments_out_of_range_and_does_nothing(bad):
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts, table = np.array([1, 1] + [0] * 30, np.int32), np.array([[0, 1]], np.int32)
    a = dict(held=[2], parent=[0], length=[20], need=[20])
    a.update(bad)
    got = fork(h, counts, table, a["held"], a["parent"], a["length"], a["need"], 4)
    st = hb.hswa_get_async_error(h)
    assert st[:3] == (hb.HSWA_ERR_BOUNDS, 0, -1 if "held" in bad else -2), st
    assert np.array_equal(got[0], counts) and all((g == FILL).all() for g in got[1:])


def test_fork_records_page_ids_out_of_range():
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts = np.array([1, 1] + [0] * 30, np.int32)
    for table in ([[-3, 1]], [[0, 32]]):
        got = fork(h, counts, np.array(table, np.int32), [2], [0, 0], [20, 20], [20, 20], 2)
        st = hb.hswa_get_async_error(h)
        assert st[0] == hb.HSWA_ERR_BOUNDS and got[0].min() >= 0 and (got[3] < 32).all(), st


@pytest.mark.parametrize("moves", [1, 5, 40, 4000])
@pytest.mark.parametrize("rows,hi,pages,cache", [(1, 5, 7, 0.3), (6, 300, 500, 0.2), (20, 900, 4099, 0.6), (0, 0, 1000, 0.5), (3, 100, 64, 1.0),
                                                 (3, 100, 70000, 0.01), (4, 60, 31, 0.0)])
def test_compact(rows, hi, pages, cache, moves):
    rng = np.random.default_rng(pages + moves)
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts, table, held, _ = state(rng, P, rows, hi, pages, cache)
    dev = [dev_i32(x) for x in (counts, table, held)]
    blocks = dev[1].shape[1]
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((pages,), (rows, blocks), (pages,), (moves,), (moves,))]
    hb.hswa_pages_compact(h, dev[0], outs[0], dev[1], dev[2], outs[1], outs[2], outs[3], outs[4])
    no_error(h)
    want = ref.compact(counts, table, held, moves, FILL)
    for g, w in zip(outs, want):
        assert np.array_equal(g.cpu().numpy(), w)
    # in place
    hb.hswa_pages_compact(h, dev[0], outs[0], dev[1], dev[2], dev[1], outs[2], outs[3], outs[4])
    no_error(h)
    assert np.array_equal(dev[1].cpu().numpy()[want[1] != FILL], want[1][want[1] != FILL])


def test_compact_at_the_limit_of_pages():
    pages = 1 << 23
    h = make_handle(dims(1, 64, 16, 1))
    live = torch.rand((pages,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)) < 0.4
    counts = live.to(torch.int32) * 3
    table, held = torch.nonzero(live)[-2000:].to(torch.int32).reshape(2, 1000).contiguous(), dev_i32([1000, 999])
    ref_out, page_map = torch.empty_like(counts), torch.empty_like(counts)
    src, dst = (torch.empty((pages,), dtype=torch.int32, device="cuda") for _ in range(2))
    table_out = torch.full_like(table, FILL)
    hb.hswa_pages_compact(h, counts, ref_out, table, held, table_out, page_map, src, dst)
    no_error(h)
    total = int(live.sum())
    n = total - int(live[:total].sum())
    assert (ref_out[:total] == 3).all() and (ref_out[total:] == 0).all()
    assert torch.equal(dst[:n].long(), torch.nonzero(~live[:total])[:, 0]) and (dst[n:] == -1).all()
    assert torch.equal(src[:n].long(), torch.nonzero(live[total:])[:, 0].flip(0) + total) and (src[n:] == -1).all()
    assert torch.equal(table_out[0], page_map[table[0].long()]) and table_out[1, 999] == FILL


def test_compact_records_values_out_of_range():
    h = make_handle(dims(1, 64, 16, 1))
    counts = dev_i32([0, 1, 1])
    for table, held, index in (([[5, 1]], [2], 0), ([[1, 2]], [3], -1)):
        o = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((3,), (1, 2), (3,), (2,), (2,))]
        hb.hswa_pages_compact(h, counts, o[0], dev_i32(table), dev_i32(held), o[1], o[2], o[3], o[4])
        st = hb.hswa_get_async_error(h)
        assert st[:3] == (hb.HSWA_ERR_BOUNDS, 0, index), st
        assert o[0].tolist() == [1, 1, 0] and o[2].tolist() == [0, 1, 0]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("d", [dims(1, 64, 16, 1), dims(1, 128, 32, 3), dims(8, 128, 64, 8)])
@pytest.mark.parametrize("layers", [1, 3, 70])
def test_copy(d, packed, layers):
    P, D, H, pages = d.page_size, d.head_dim, d.num_kv_heads, 11
    if layers == 70 and H == 8:
        pages = 5
    shape = (pages, 2, H, P * (D // 2 + D // 16)) if packed else (pages, 2, H, P, D)
    h = make_handle(d)
    g = torch.Generator(device="cuda").manual_seed(6)
    raw = [torch.randint(-2 ** 15, 2 ** 15, (pages, *((2, H, P * (D // 2 + D // 16) // 2) if packed else (2, H, P, D))), generator=g, device="cuda",
                         dtype=torch.int16) for _ in range(layers)]
    pools = [x.view(torch.uint8).reshape(shape) if packed else x.view(torch.bfloat16) for x in raw]
    want = [x.clone() for x in raw]
    src, dst = [3, -1, 3, 0], [1, -1, 4, 2]
    for w in want:
        w[[1, 4, 2]] = w[[3, 3, 0]]
    hb.hswa_pages_copy(h, [hb.PackedLayer(p) if packed else hb.Layer(p, False) for p in pools], dev_i32(src), dev_i32(dst))
    no_error(h)
    assert all(torch.equal(a, b) for a, b in zip(raw, want))


def test_copy_records_ids_out_of_range_and_takes_empty_lists():
    d = dims(1, 64, 16, 1)
    h = make_handle(d)
    pool = torch.randn((4, 2, 1, 16, 64), device="cuda").bfloat16()
    want = pool.clone()
    want[3] = want[0]
    for src, dst in (([4, 0], [1, 3]), ([1, 0], [-1, 3]), ([-1, 0], [1, 3]), ([0, 0], [3, 1 << 30])):
        hb.hswa_pages_copy(h, [hb.Layer(pool, False)], dev_i32(src), dev_i32(dst))
        st = hb.hswa_get_async_error(h)
        assert st[0] == hb.HSWA_ERR_BOUNDS and torch.equal(pool, want), st
    hb.hswa_pages_copy(h, [hb.Layer(pool, False)], dev_i32([]), dev_i32([]))
    hb.hswa_pages_copy(h, [], dev_i32([0]), dev_i32([1]))
    no_error(h)
    assert torch.equal(pool, want)


def test_copy_of_pages_far_into_a_large_pool():
    d = dims(8, 128, 64, 8)
    h = make_handle(d)
    pool = torch.zeros((20000, 2, 8, 64, 128), dtype=torch.bfloat16, device="cuda")  # 5.2 GB
    pool[19999] = 3.0
    hb.hswa_pages_copy(h, [hb.Layer(pool, False)], dev_i32([19999, 0]), dev_i32([19998, 1]))
    no_error(h)
    assert (pool[19998] == 3).all() and (pool[19997] == 0).all() and (pool[1] == 0).all()


def test_refusals():
    h = make_handle(dims(1, 64, 16, 1))
    lib, bad, uns = hb.load(), hb.HSWA_ERR_INVALID_ARG, hb.HSWA_ERR_UNSUPPORTED
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    counts, other, table, rows = z(8), z(8), z(2, 3), [z(2) for _ in range(7)]
    ws = torch.empty((256,), dtype=torch.uint8, device="cuda")

    def status(call, *a):
        with pytest.raises(hb.HswaError) as e:
            call(h, *a)
        return e.value.status

    fork_args = [counts, other, table, *rows[:4], z(2, 3), *rows[4:], ws]
    # ref_out = ref, table_out = table, held_out = held, copy_dst = copy_src, held_out = need, copy_src = length, copy_dst = held_out
    for i, same in ((1, 0), (7, 2), (8, 3), (10, 9), (8, 6), (9, 5), (10, 8)):
        a = list(fork_args)
        a[i] = a[same]
        assert status(hb.hswa_pages_fork, *a) == bad
    assert status(hb.hswa_pages_fork, *fork_args[:-1], ws[:128]) == hb.HSWA_ERR_WORKSPACE
    assert status(hb.hswa_pages_fork, *fork_args[:-1], torch.empty((512,), dtype=torch.uint8, device="cuda")[16:]) == hb.HSWA_ERR_WORKSPACE
    many = z(4097)
    assert status(hb.hswa_pages_fork, counts, other, z(4097, 1), many, *rows[:3], z(2, 3), *rows[3:6], ws) == uns
    wide = torch.empty((2, (1 << 29) + 1), dtype=torch.int32, device="cuda")
    assert status(hb.hswa_pages_fork, counts, other, wide, *rows[:4], z(2, 3), *rows[4:], ws) == uns
    assert status(hb.hswa_pages_fork, counts, other, table, *rows[:4], wide, *rows[4:], ws) == uns
    assert status(hb.hswa_pages_compact, counts, other, wide, rows[0], wide, z(8), rows[1], rows[2]) == uns
    del wide
    assert status(hb.hswa_pages_compact, counts, counts, table, rows[0], table, z(8), rows[1], rows[2]) == bad
    assert status(hb.hswa_pages_compact, counts, other, table, rows[0], table, counts, rows[1], rows[2]) == bad
    assert status(hb.hswa_pages_compact, counts, other, table, rows[0], table, z(8), rows[1], rows[1]) == bad
    assert status(hb.hswa_pages_compact, counts, other, table, rows[0], table, z(8), rows[0], rows[1]) == bad  # move_src = held
    big = torch.zeros(((1 << 23) + 1,), dtype=torch.int32, device="cuda")
    assert status(hb.hswa_pages_compact, big, torch.empty_like(big), table, rows[0], table, torch.empty_like(big), rows[1], rows[2]) == uns
    assert hb.hswa_pages_workspace_need(h, (1 << 23) + 1) == 0
    pool = torch.zeros((4, 2, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(AssertionError):
        hb.hswa_pages_copy(h, [hb.Layer(pool, False), hb.Layer(pool[:3].contiguous(), False)], rows[0], rows[1])
    at = (hb.C.c_void_p * 1)(pool.data_ptr() + 8)
    assert lib.hswa_pages_copy(h.ptr, 1, at, 4, 4096, 2, rows[0].data_ptr(), rows[1].data_ptr(), None) == bad
    at = (hb.C.c_void_p * 1)(pool.data_ptr())
    assert lib.hswa_pages_copy(h.ptr, 1, at, 4, 4090, 2, rows[0].data_ptr(), rows[1].data_ptr(), None) == bad
    assert lib.hswa_pages_copy(h.ptr, 1, at, 4, 4096, -1, rows[0].data_ptr(), rows[1].data_ptr(), None) == bad
    no_error(h)


@pytest.mark.parametrize("d", [dims(8, 128, 64), dims(4, 64, 16, 1)])
def test_a_run_of_beams_over_a_4_bit_cache(d):
    """Steps of forking, copying, appending and attending over two 4-bit layers, with a compaction in between: every row's
    attention is that over its own history."""
    P, D, H, layers = d.page_size, d.head_dim, d.num_kv_heads, 2
    h = make_handle(d, torch.float32)
    rng = np.random.default_rng(8)
    pages, blocks = 150, 150 // P + 20
    counts = dev_i32(np.zeros(pages, np.int32))
    pools = [hb.PackedLayer(torch.full((pages, 2, H, P * (D // 2 + D // 16)), 0x7f, dtype=torch.uint8, device="cuda"), 1.0, 0.5) for _ in range(layers)]
    table, held = torch.zeros((0, blocks), dtype=torch.int32, device="cuda"), dev_i32([])
    ws = torch.empty((hb.hswa_pages_workspace_need(h, pages),), dtype=torch.uint8, device="cuda")
    past = []  # of each row: per layer K and V, float64 [L][H][D]
    steps = [([-1, -1, -1], [70, 5, 33]), ([0, 0, 1, 2], [1] * 4), ([0, 1, 1, 3, 2], [2] * 5), ([1, 1, 1, 4, -1], [3, 3, 3, 3, 40]),
             ([0, 1, 2, 3, 4], [1] * 5), ([2, 4], [17, 1]), ([1, 0, 0], [1, 1, 1])]
    for step, (parent, n) in enumerate(steps):
        B, T = len(parent), sum(n)
        drop = [0 if p < 0 else int(rng.integers(0, 2)) for p in parent]  # some rows take a token back
        length = [0 if p < 0 else len(past[p][0][0]) - x for p, x in zip(parent, drop)]
        table_out = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda")
        held_out, src, dst = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(3))
        new = torch.empty_like(counts)
        hb.hswa_pages_fork(h, counts, new, table, held, dev_i32(parent), dev_i32(length), dev_i32([a + b for a, b in zip(length, n)]), table_out,
                           held_out, src, dst, ws)
        hb.hswa_pages_copy(h, pools, src, dst)
        counts, table, held = new, table_out, held_out
        if step in (2, 5):
            new, page_map, out = torch.empty_like(counts), torch.empty_like(counts), torch.full_like(table, -1)
            src, dst = (torch.empty((100,), dtype=torch.int32, device="cuda") for _ in range(2))
            hb.hswa_pages_compact(h, counts, new, table, held, out, page_map, src, dst)
            hb.hswa_pages_copy(h, pools, src, dst)
            counts, table = new, out
            live = int((counts > 0).sum())
            assert (counts[live:] == 0).all()
        indptr = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        b = hb.Batch(dev_i32(length), table, *no_rings(d, B), dev_i32(indptr), max_q_len=max(n), total_q=T, max_ctx_len=max(length))
        past = [[[x[:keep] for x in kv] for kv in past[p]] if p >= 0 else [[np.zeros((0, H, D))] * 2 for _ in range(layers)]
                for p, keep in zip(parent, length)]
        for layer in range(layers):
            bits = [wl.bf16_bits_normal(1000 * step + 10 * layer + i, (T, heads, D)) for i, heads in ((0, H), (1, H), (2, d.num_q_heads))]
            out, lse = torch.empty((T, d.num_q_heads, D), device="cuda"), torch.empty((T, d.num_q_heads), device="cuda")
            hb.hswa_packed_append(h, pools[layer], b, to_dev_bf16(bits[0]), to_dev_bf16(bits[1]))
            hb.hswa_packed_attn(h, pools[layer], b, True, to_dev_bf16(bits[2]), out, lse, workspace(h, b, True))
            no_error(h)
            q, o = wl.bits_to_f64(bits[2]), out.double().cpu().numpy()
            for r in range(B):
                a, e = indptr[r], indptr[r + 1]
                for which, scale in ((0, 1.0), (1, 0.5)):
                    x = wl.bits_to_f64(bits[which][a:e])
                    past[r][layer][which] = np.concatenate([past[r][layer][which], ref.values(*ref.round_rows(x, scale), scale)])
                K, V = past[r][layer]
                want, _, mag = ref.attention(K, V, q[a:e], [length[r] + i + 1 for i in range(n[r])], 1.0 / np.sqrt(D))
                tol = (2.0 ** -11 + 2 * S_ERR + len(K) * 2.0 ** -24) * mag + len(K) * 2.0 ** -25 * np.abs(V).max()
                assert (np.abs(o[a:e] - want) <= tol + 1e-7).all(), (step, r)
        # counts are the rows' holdings
        t, hd = table.cpu().numpy(), held.cpu().numpy()
        assert np.array_equal(np.bincount(np.concatenate([t[r, : hd[r]] for r in range(B)]), minlength=pages), counts.cpu().numpy())


def test_calls_captured_into_a_graph_replay_on_new_counts():
    rng = np.random.default_rng(9)
    P, h, pages = 16, make_handle(dims(1, 64, 16, 1)), 600
    first = state(rng, P, 5, 200, pages)
    dev = [dev_i32(x) for x in (first[0], np.zeros((5, 15), np.int32), first[2])]
    parent, length, need = (dev_i32([0] * 4) for _ in range(3))
    outs = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((4, 16), (4,), (4,), (4,))]
    ref_out = torch.empty_like(dev[0])
    ws = torch.empty((hb.hswa_pages_workspace_need(h, pages),), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.hswa_pages_fork(h, dev[0], ref_out, dev[1], dev[2], parent, length, need, *outs, ws)
    for _ in range(3):
        counts, table, held, lens = state(rng, P, 5, 200, pages)
        wide = np.full((5, 15), -1, np.int32)
        wide[:, : table.shape[1]] = table
        pa, le, ne = children(rng, P, 4, held, lens, 20)
        for x, y in zip((*dev, parent, length, need), (counts, wide, held, pa, le, ne)):
            x.copy_(dev_i32(y))
        outs[0].fill_(FILL)
        graph.replay()
        no_error(h)
        for g, w in zip((ref_out, *outs), ref.fork(counts, wide, held, pa, le, ne, P, 16, FILL)):
            assert np.array_equal(g.cpu().numpy(), w)


def test_tables_of_many_entries():
    """Rows times places past what the first launch rewrites itself: forked, then compacted, against the statement."""
    rng = np.random.default_rng(11)
    P, h, pages = 16, make_handle(dims(1, 64, 16, 1)), 50021
    counts, table, held, lens = state(rng, P, 60, 14000, pages)
    parent, length, need = children(rng, P, 70, held, lens, 50)
    blocks = 880
    assert table.size + 70 * blocks > 32768 * 2
    ref_out, table_out, held_out, _, _ = check_fork(h, P, counts, table, held, parent, length, need, blocks)
    dev = [dev_i32(x) for x in (ref_out, table_out, held_out)]
    moves = 20000
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((pages,), (70, blocks), (pages,), (moves,), (moves,))]
    hb.hswa_pages_compact(h, dev[0], outs[0], dev[1], dev[2], outs[1], outs[2], outs[3], outs[4])
    no_error(h)
    for g, w in zip(outs, ref.compact(ref_out, table_out, held_out, moves, FILL)):
        assert np.array_equal(g.cpu().numpy(), w)
    # without enough pages the second launch does nothing either
    counts[counts == 0] = 1
    got = fork(h, counts, table, held, parent, length, need, blocks)
    assert hb.hswa_get_async_error(h)[:2] == (hb.HSWA_ERR_BOUNDS, -1)
    assert np.array_equal(got[0], counts) and all((g == FILL).all() for g in got[1:])
