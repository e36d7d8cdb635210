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
