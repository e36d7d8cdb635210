"""The binding's checks of arguments, which need no GPU: they raise before a pointer is passed on."""
import subprocess
import sys

import pytest
import torch

from conftest import ROOT
from paper_2607_13095_b200 import binding as hb

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


class OnDevice:
    """A stand-in for a contiguous CUDA tensor of a device."""

    def __init__(self, t, device):
        self.t, self.device = t, device
        self.is_cuda, self.dtype, self.shape = True, t.dtype, t.shape
        self.is_contiguous, self.dim, self.numel, self.element_size = t.is_contiguous, t.dim, t.numel, t.element_size

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 4096


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(hb, "_device", lambda: 0)
    assert hb._ptrs(0, OnDevice(torch.zeros(4), 0), None) == [4096, None]
    for bad in (OnDevice(torch.zeros(4), 1), OnDevice(torch.zeros(4, 4).t(), 0), torch.zeros(4)):
        with pytest.raises(AssertionError, match="current device"):
            hb._ptrs(0, OnDevice(torch.zeros(4), 0), bad)
    i32 = torch.int32
    ints = lambda *shape, device=0: OnDevice(torch.zeros(shape, dtype=i32), device)  # noqa: E731
    pool = lambda device=0: hb.Layer(OnDevice(torch.zeros((1, 2, 1, 16, 64), dtype=torch.bfloat16), device), False)  # noqa: E731
    batch = lambda device=0, table=(2, 3), indptr=None: hb.Batch(  # noqa: E731
        ints(2, device=device), ints(*table, device=device), ints(2, 9), ints(2), indptr, max_ctx_len=9)
    hb._device_of(pool(), batch())
    hb._device_of(pool(), batch(indptr=ints(3)))
    hb._device_of(pool(), batch(table=(4, 3), indptr=ints(7)))
    for layer, b in ((pool(1), batch()), (pool(), batch(1)), (pool(), batch(table=(1, 3))), (pool(), batch(indptr=ints(2))),
                     (pool(), batch(indptr=OnDevice(torch.zeros(3, dtype=torch.int64), 0)))):
        with pytest.raises(AssertionError):
            hb._device_of(layer, b)
