"""Page calls where they can go wrong: arguments out of range anywhere among many rows, tables without places, the launches of large pools and
large tables together, arrays off 16 bytes, handles side by side."""
import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_utils import dev_i32, make_handle, to_dev_bf16
from paper_2607_13095_b200 import binding as hb
from paper_2607_13095_b200 import workloads as wl
from test_gpu_packed import S_ERR, dims, no_error, no_rings
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


# ---- large pools and large tables together: counts copied by a launch before the cluster's, tables rewritten by one behind it ----
PAGES, BLOCKS = 70001, 900


def large(seed, rows_in=66, rows_out=70):
    rng = np.random.default_rng(seed)
    P = 16
    counts, table, held, lens = state(rng, P, rows_in, 14000, PAGES)
    parent, length, need = children(rng, P, rows_out, held, lens, 50)
    parent[3], parent[4], parent[5] = parent[2], parent[2], -1  # several children of one row, a new request of many pages
    length[2:5] = np.minimum([int(lens[max(parent[2], 0)])] * 3, [14000, 9999, 14000]) if parent[2] >= 0 else 0
    need[2:5] = length[2:5] + 20
    length[5], need[5] = 0, 13900
    assert rows_in * table.shape[1] + rows_out * BLOCKS > 32768 and PAGES > 65536
    return P, make_handle(dims(1, 64, P, 1)), counts, table, held, parent, length, need


@pytest.mark.parametrize("seed", [21, 22, 23])
def test_large_pools_with_large_tables(seed):
    """Forked, then compacted, entry for entry: shared, passed on, copied, fresh and freed pages, some of a prefix cache."""
    P, h, counts, table, held, parent, length, need = large(seed)
    ref_out, table_out, held_out, src, _ = check_fork(h, P, counts, table, held, parent, length, need, BLOCKS)
    assert (src >= 0).any() and (counts == 2).any()
    for moves in (7, 30000):
        dev = [dev_i32(x) for x in (ref_out, table_out, held_out)]
        rows = len(held_out)
        outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((PAGES,), (rows, BLOCKS), (PAGES,), (moves,), (moves,))]
        want = ref.compact(ref_out, table_out, held_out, moves, FILL)
        hb.hswa_pages_compact(h, dev[0], outs[0], dev[1], dev[2], outs[1], outs[2], outs[3], outs[4])
        no_error(h)
        for g, w in zip(outs, want):
            assert np.array_equal(g.cpu().numpy(), w)
        hb.hswa_pages_compact(h, dev[0], outs[0], dev[1], dev[2], dev[1], outs[2], outs[3], outs[4])  # in place
        no_error(h)
        assert np.array_equal(dev[1].cpu().numpy()[want[1] != FILL], want[1][want[1] != FILL])


def test_large_forks_that_are_refused_do_nothing():
    P, h, counts, table, held, parent, length, need = large(24)

    def refused(*what, **change):
        a = dict(counts=counts, held=held, parent=parent, length=length, need=need)
        a.update(change)
        got = fork(h, a["counts"], table, a["held"], a["parent"], a["length"], a["need"], BLOCKS)
        st = hb.hswa_get_async_error(h)
        assert st[: len(what)] == what, st
        assert np.array_equal(got[0], a["counts"]) and all((g == FILL).all() for g in got[1:])

    def at(x, i, v):
        y = np.array(x)
        y[i] = v
        return y

    few = np.where(counts == 0, 1, counts)
    few[[5, 69998]] = 0
    refused(hb.HSWA_ERR_BOUNDS, -1, counts=few)
    refused(hb.HSWA_ERR_BOUNDS, 50, -1, held=at(held, 50, table.shape[1] + 1))
    refused(hb.HSWA_ERR_BOUNDS, 61, -2, parent=at(parent, 61, 66))
    refused(hb.HSWA_ERR_BOUNDS, 62, -2, length=at(length, 62, -1))
    refused(hb.HSWA_ERR_BOUNDS, 63, -2, need=at(need, 63, BLOCKS * P + 1))
    # as many as there are: enough
    check_fork(h, P, counts, table, held, parent, length, need, BLOCKS)


def test_large_fork_replayed_from_a_graph():
    P, h, counts, table, held, parent, length, need = large(25)
    dev = [dev_i32(x) for x in (np.zeros_like(counts), table, held, parent, length, need)]
    n = len(parent)
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((PAGES,), (n, BLOCKS), (n,), (n,), (n,))]
    ws = torch.empty((hb.hswa_pages_workspace_need(h, PAGES),), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hb.hswa_pages_fork(h, dev[0], outs[0], dev[1], dev[2], dev[3], dev[4], dev[5], *outs[1:], ws)
    dev[0].copy_(dev_i32(counts))
    want = ref.fork(counts, table, held, parent, length, need, P, BLOCKS, FILL)
    for _ in range(3):
        for o in outs:
            o.fill_(FILL)
        ws.fill_(255)
        graph.replay()
        no_error(h)
        for g, w in zip(outs, want):
            assert np.array_equal(g.cpu().numpy(), w)


def off_by(x, places):
    """The same values in memory that starts `places` entries behind a 16-byte border."""
    buf = torch.full((x.numel() + 8,), FILL, dtype=torch.int32, device="cuda")
    view = buf[places:places + x.numel()].reshape(x.shape)
    view.copy_(x)
    return view


@pytest.mark.parametrize("pages", [1, 31, 5003, 70001])
@pytest.mark.parametrize("shift", [(1, 1, 1), (0, 3, 0), (2, 0, 1), (0, 0, 3)])
def test_arrays_off_16_bytes(pages, shift):
    """Counts, their copy and the map anywhere on 4 bytes, next to memory that stays as it was."""
    rng = np.random.default_rng(pages)
    P, h = 16, make_handle(dims(1, 64, 16, 1))
    counts, table, held, lens = state(rng, P, 3 if pages > 1000 else 0, 300, pages)
    parent, length, need = children(rng, P, 4 if pages > 1000 else 0, held, lens, 40)
    a, b, c = (off_by(dev_i32(x), s) for x, s in zip((counts, np.full(pages, FILL), np.full(pages, FILL)), shift))
    n, blocks = len(parent), 25
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((n, blocks), (n,), (n,), (n,))]
    ws = torch.empty((hb.hswa_pages_workspace_need(h, pages),), dtype=torch.uint8, device="cuda")
    dev = [off_by(dev_i32(x), 1) for x in (table, held, parent, length, need)]
    hb.hswa_pages_fork(h, a, b, *dev, *outs, ws)
    no_error(h)
    want = ref.fork(counts, table, held, parent, length, need, P, blocks, FILL)
    for g, w in zip((b, *outs), want):
        assert np.array_equal(g.cpu().numpy(), w)
    moves = 50
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in (tuple(table.shape), (moves,), (moves,))]
    hb.hswa_pages_compact(h, a, b, dev[0], dev[1], outs[0], c, outs[1], outs[2])
    no_error(h)
    for g, w in zip((b, outs[0], c, outs[1], outs[2]), ref.compact(counts, table, held, moves, FILL)):
        assert np.array_equal(g.cpu().numpy(), w)
    for x, s in ((b, shift[1]), (c, shift[2])):
        whole = torch.as_strided(x, (pages + 8,), (1,), 0)
        assert (whole[:s] == FILL).all() and (whole[s + pages:] == FILL).all()


def test_fresh_pages_at_the_limits_are_the_lowest():
    """8388608 pages, 4096 rows: fresh pages in the order of rows and places are the lowest free ones in order, whoever lists them."""
    P, pages, n = 16, 1 << 23, 4096
    h = make_handle(dims(1, 64, P, 1))
    counts = (torch.rand((pages,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(7)) < 0.7).to(torch.int32)
    places = torch.arange(n, device="cuda") % 9  # pages of each new request
    need = (places * P).to(torch.int32)
    ref_out = torch.empty_like(counts)
    outs = [torch.full(s, FILL, dtype=torch.int32, device="cuda") for s in ((n, 8), (n,), (n,), (n,))]
    ws = torch.empty((hb.hswa_pages_workspace_need(h, pages),), dtype=torch.uint8, device="cuda")
    hb.hswa_pages_fork(h, counts, ref_out, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), dev_i32([]), dev_i32([-1] * n), dev_i32([0] * n), need,
                       *outs, ws)
    no_error(h)
    inside = torch.arange(8, device="cuda")[None] < places[:, None]
    total = int(places.sum())
    fresh = torch.nonzero(counts == 0)[:total, 0]
    assert torch.equal(outs[0][inside].long(), fresh) and (outs[0][~inside] == FILL).all()
    counts[fresh] = 1
    assert torch.equal(ref_out, counts) and torch.equal(outs[1].long(), places)


@pytest.mark.parametrize("d", [dims(4, 64, 16, 1), dims(8, 128, 64, 2)])
def test_beams_on_a_hybrid_stack(d):
    """Steps of forking over a Full and an SWA layer: tables by the fork, rings taken over by one child and copied for the others, heads moved back
    by the tokens that a child takes back, as many as the ring still covers.  Every row's attention is that over its own history."""
    P, D, H, W, R, C = d.page_size, d.head_dim, d.num_kv_heads, d.window, d.ring_pages, d.ring_slots
    h = make_handle(d, torch.float32)
    pages, blocks, rings = 400, 700 // P + 3, 40
    pools = [hb.Layer(torch.full((n, 2, H, P, D), float("nan"), dtype=torch.bfloat16, device="cuda"), swa) for n, swa in ((pages, False), (rings * R, True))]
    counts = torch.zeros((pages,), dtype=torch.int32, device="cuda")
    table, held = torch.zeros((0, blocks), dtype=torch.int32, device="cuda"), dev_i32([])
    ws_pages = torch.empty((hb.hswa_pages_workspace_need(h, pages),), dtype=torch.uint8, device="cuda")
    past, ring_of, head_of, free = [], [], [], list(range(rings))  # of each row: per layer K and V; its ring; its head
    since = []  # of each row: the first position that its ring still holds
    most = C - W + 1
    steps = [([-1, -1], [300, 40], [0, 0]), ([0, 0, 1], [1] * 3, [0, most, 5]), ([0, 1, 1, 2], [1] * 4, [0, 0, 1, 0]), ([1, 1, 3], [30, 150, 7], [most, 1, 0]),
             ([0, 0, 1, 2, -1], [1] * 5, [0, 1, most, 3, 0]), ([4, 0, 2], [1] * 3, [0, 0, 1])]
    for step, (parent, n, back) in enumerate(steps):
        B, T = len(parent), sum(n)
        back = [x if p < 0 else min(x, len(past[p][0][0]) - (W - 1) - since[p] if since[p] else x) for p, x in zip(parent, back)]
        assert min(back) >= 0 and (step != 1 or back[1] == most)
        length = [0 if p < 0 else len(past[p][0][0]) - x for p, x in zip(parent, back)]
        since = [max(0 if p < 0 else since[p], a + b - C) for p, a, b in zip(parent, length, n)]
        table_out = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda")
        held_out, src, dst = (torch.empty((B,), dtype=torch.int32, device="cuda") for _ in range(3))
        new = torch.empty_like(counts)
        hb.hswa_pages_fork(h, counts, new, table, held, dev_i32(parent), dev_i32(length), dev_i32([a + b for a, b in zip(length, n)]), table_out,
                           held_out, src, dst, ws_pages)
        hb.hswa_pages_copy(h, pools[:1], src, dst)
        counts, table, held = new, table_out, held_out
        # rings: fresh ones from those that no row of the step before holds
        spare = [x for x in free if x not in ring_of]
        mine, pairs, heads, taken = [], [], [], set()
        for p, x in zip(parent, back):
            if p >= 0 and p not in taken:
                mine.append(ring_of[p])
                taken.add(p)
            else:
                mine.append(spare.pop())
                if p >= 0:
                    pairs += [(ring_of[p] * R + i, mine[-1] * R + i) for i in range(R)]
            heads.append(0 if p < 0 else (head_of[p] - x) % C)
        if pairs:
            hb.hswa_pages_copy(h, pools[1:], dev_i32([a for a, _ in pairs]), dev_i32([b for _, b in pairs]))
        ring_of, head_of = mine, heads
        past = [[[x[:keep] for x in kv] for kv in past[p]] if p >= 0 else [[np.zeros((0, H, D))] * 2 for _ in range(2)] for p, keep in zip(parent, length)]
        indptr = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        ring_table = dev_i32([[x * R + i for i in range(R)] for x in ring_of])
        ctx, head = dev_i32(length), dev_i32(head_of)
        single = max(n) == 1
        b = hb.Batch(ctx, table, ring_table, head, None if single else dev_i32(indptr), max_q_len=max(n), total_q=T, max_ctx_len=max(length))
        for layer in range(2):
            bits = [wl.bf16_bits_normal(3000 + 100 * step + 10 * layer + i, (T, heads_, D)) for i, heads_ in ((0, H), (1, H), (2, d.num_q_heads))]
            k, v, q = (to_dev_bf16(x) for x in bits)
            for r in range(B):
                for which in (0, 1):
                    past[r][layer][which] = np.concatenate([past[r][layer][which], wl.bits_to_f64(bits[which][indptr[r]:indptr[r + 1]])])
            if not single:  # (prompts: their rows are cached, and read by the steps behind)
                hb.hswa_kv_append(h, pools[layer], b, k, v)
                no_error(h)
                continue
            out = torch.empty((T, d.num_q_heads, D), device="cuda")
            ws = torch.empty((max(256, hb.hswa_workspace_bytes(h, B, T, max(length))),), dtype=torch.uint8, device="cuda")
            hb.hswa_decode_attn(h, pools[layer], b, q, k, v, out, None, ws)
            no_error(h)
            o = out.double().cpu().numpy()
            for r in range(B):
                K, V = (x[-W:] if layer else x for x in past[r][layer])
                want, _, mag = ref.attention(K, V, wl.bits_to_f64(bits[2][r:r + 1]), [len(K)], 1.0 / np.sqrt(D))
                # probabilities in bf16, 2^-8 of their value; scores as in test_gpu_packed.py
                tol = (2.0 ** -8 + 2 * S_ERR + len(K) * 2.0 ** -24) * mag
                assert (np.abs(o[r:r + 1] - want) <= tol + 1e-7).all(), (step, layer, r, np.abs(o[r:r + 1] - want).max())
        hb.hswa_step_advance(h, B, ctx, head, b.q_indptr)
        head_of = head.tolist()


def test_copy_refuses_what_its_grid_cannot_hold():
    d = dims(1, 64, 16, 1)
    h, lib = make_handle(d), hb.load()
    pool, ids = torch.zeros((4, 2, 1, 16, 64), dtype=torch.bfloat16, device="cuda"), dev_i32([0, 1])
    at = (hb.C.c_void_p * 1)(pool.data_ptr())
    for pages, size, pairs in ((1 << 31, 4096, 2), (4, (1 << 30) + 16, 2), (4, 1 << 30, 1 << 13)):
        assert lib.hswa_pages_copy(h.ptr, 1, at, pages, size, pairs, ids.data_ptr(), ids.data_ptr(), None) == hb.HSWA_ERR_UNSUPPORTED
    no_error(h)
