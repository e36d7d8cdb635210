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
