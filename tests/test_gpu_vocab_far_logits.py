"""Rows whose logits lie far from those at the row's beginning, from which the listing pass takes what its sums are relative to:
the log-sum-exp against the oracle (tolerance of the sums in test_gpu_vocab)."""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import E, _back, _dt, _place, _sum_error

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu
INF = math.inf


def _lse(z, dtype, k, temperature):
    """Checks the call's record of the rows z; the rows as the call has them, and the log-sum-exps."""
    import torch

    dev = _place(z.astype(np.float32), dtype)
    n, V = z.shape
    values, lse = torch.full((n, k), math.nan, device="cuda"), torch.full((n,), math.nan, device="cuda")
    at = torch.full((n, k), -9, dtype=torch.int32, device="cuda")
    b.collm_top_logits(dev, values, at, lse, temperature=temperature)
    host, got = _back(dev), _back(lse)
    for i in range(n):
        want_v, want_at, want = ov.top(host[i], k, temperature)
        assert np.array_equal(_back(values[i]), want_v) and np.array_equal(at[i].cpu().numpy(), want_at), i
        assert got[i] == want or abs(got[i] - want) <= _sum_error(V) + 2 * E * abs(want), (i, got[i], want)
    return host, got


@pytest.mark.parametrize("temperature", [1.0, 0.05, 3.0])
@pytest.mark.parametrize("dtype,V,k", [("f32", 32000, 20), ("f32", 50257, 64), ("bf16", 50257, 20), ("bf16", 128256, 200), ("f32", 160001, 256)])
def test_a_logit_far_above_the_first_ones(dtype, V, k, temperature):
    rng = np.random.default_rng(V + k)
    z = rng.normal(size=(6, V))
    z[0, V - 1] = 1000.0
    z[1, V - 300:] += 1000.0                             # hundreds of them
    z[2, V // 2 + 7000] = 40.0
    z[3] = -1e4                                          # a mask of a finite value, fewer words left than are listed
    z[3, V - 1 - 40 * np.arange(150)] = rng.normal(size=150)
    z[4] -= 1e4
    z[4, V - 2] = 5.0
    z[5] *= 100.0
    _lse(z, dtype, k, temperature)
