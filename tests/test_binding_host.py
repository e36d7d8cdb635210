"""The binding's checks of arguments, which need no GPU: they raise before a pointer is passed on."""
import subprocess
import sys

import pytest

from conftest import ROOT

CHECKS = """
from types import SimpleNamespace as N
import torch
from paper_2607_13095_b200 import binding as hb
h = N(ptr=None, out_dtype=torch.float32, cfg=N(num_q_heads=4, num_kv_heads=1, head_dim=64))
b = N(batch=2, total_q=2, q_indptr=None, c=None)
layer = N(c=None)
q, out, lse = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 4, 64)), torch.zeros((2, 4))
w, idx, n = torch.zeros((2, 1, 9)), torch.zeros((2, 1, 4), dtype=torch.int32), torch.zeros((2,), dtype=torch.int32)
calls = [
    lambda: hb._ptr(torch.zeros(2)),
    lambda: hb.Layer(torch.zeros(2), False),
    lambda: hb.hswa_cross_attn(h, layer, b, q[:1], out, lse),
    lambda: hb.hswa_cross_attn(h, layer, b, q, out[:1], lse),
    lambda: hb.hswa_cross_attn(h, layer, b, q, out, lse[:1]),
    lambda: hb.hswa_cross_attn(h, layer, b, q.float(), out, lse),
    lambda: hb.hswa_cross_attn(h, layer, b, q.view(1, 2, 4, 64), out, lse),
    lambda: hb.hswa_attn_weights(h, layer, b, False, q[:1], lse, 1.0, w),
    lambda: hb.hswa_attn_weights(h, layer, b, False, q, lse[:1], 1.0, w),
    lambda: hb.hswa_attn_weights(h, layer, b, False, q, lse, 1.0, w[:1]),
    lambda: hb.hswa_attn_weights(h, layer, b, False, q.view(1, 2, 4, 64), lse, 1.0, w),
    lambda: hb.hswa_evict_select(h, 2, n[:1], 9, w, n, idx, n.clone()),
    lambda: hb.hswa_evict_select(h, 2, n, 9, w[:1], n, idx, n.clone()),
    lambda: hb.hswa_evict_select(h, 2, n.long(), 9, w, n, idx, n.clone()),
    lambda: hb.hswa_evict_compact(h, layer, b, idx[:1], n, idx[:, 0]),
    lambda: hb.hswa_evict_compact(h, layer, b, idx, n[:1], idx[:, 0]),
    lambda: hb.hswa_evict_compact(h, layer, b, idx, n, idx[:, 0], w[:1], w),
]
for i, call in enumerate(calls):
    try:
        call()
    except AssertionError:
        continue
    raise SystemExit(f"call {i} was not refused")
print("refused", len(calls))
"""


@pytest.mark.parametrize("flags", [[], ["-O"]], ids=["plain", "optimised"])
def test_wrong_tensors_are_refused(flags):
    """Also where python drops assert statements."""
    run = subprocess.run([sys.executable, *flags, "-c", CHECKS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "refused 17" in run.stdout, run.stderr[-2000:] + run.stdout
