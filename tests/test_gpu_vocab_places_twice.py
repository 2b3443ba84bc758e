"""Records that name places several times, by threads of different waves: against the oracle (tolerances of test_gpu_vocab), and the same bits on
every run."""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import _back, _check_distill, _place, _up, _workspace

from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["loss", "two", "step", "shared"])
@pytest.mark.parametrize("dtype,V,tau", [("bf16", 50003, 2.0), ("f32", 50257, 1.0), ("f32", 30001, 1.5), ("bf16", 70001, 1.0)])
def test_places_named_up_to_five_times(dtype, V, tau, how):
    import torch

    rng = np.random.default_rng(V)
    n, k = 6, 700
    dev = _place(rng.normal(size=(n, V)).astype(np.float32) * 3, dtype)
    host = _back(dev)
    at = rng.choice(rng.choice(V, 140, replace=False), (n, k)).astype(np.int32)
    at[1] = 77  # one place alone
    at[2, ::2] = -1
    values = rng.normal(size=(n, k)).astype(np.float32)
    lse = (np.log(np.exp(values.astype(np.float64) / tau).sum(1)) + 0.2).astype(np.float32)
    lab, dloss = at[:, 3].clip(0, V - 1).astype(np.int32), np.ones(n, np.float32)
    t, kw = (_up(values), _up(at, torch.int32)), dict(t_lse=_up(lse), labels=_up(lab, torch.int32), temperature=tau, kd_weight=0.7, ce_weight=0.3)
    runs = []
    for _ in range(4):
        loss, stats, grad = torch.full((n,), math.nan, device="cuda"), torch.zeros((n, b.DISTILL_STATS), device="cuda"), torch.zeros_like(dev)
        if how in ("loss", "two"):
            b.collm_distill_fwd(dev, *t, loss, None if how == "loss" else stats, **kw)
            if how == "two":
                b.collm_distill_bwd(dev, *t, stats, _up(dloss), grad, **kw)
        else:
            b.collm_distill_fwd_bwd(dev, *t, _up(dloss), loss, grad, workspace=_workspace(how == "shared"), **kw)
        runs.append((loss, stats, grad))
    loss, _, grad = runs[0]
    _check_distill(_back(loss), None if how == "loss" else _back(grad), host, values, at, lse, lab, dloss, V, dtype, tau, np.float32(0.7), np.float32(0.3))
    for other in runs[1:]:
        for x, y in zip(runs[0], other):
            assert torch.equal(x, y)
