"""Vocabulary operators at the least and the largest temperatures that they take."""
from __future__ import annotations

import numpy as np
import pytest
from test_gpu_vocab import E, _back, _check_distill, _place, _up

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [2.0**-127, 2.0**-126, 1e-30, 1e30, 3e38])
def test_temperatures_at_the_limits(temperature, dtype):
    import torch

    V, n, k = 5003, 3, 8
    z = np.random.default_rng(1).normal(size=(n, V)).astype(np.float32)
    z = _back(_place(z, dtype))
    z -= z.max(1, keepdims=True)  # (largest logit 0: the log-sum-exp is a number at any temperature)
    dev = _place(z, dtype)
    host = _back(dev)
    values, at, lse = torch.zeros((n, k), device="cuda"), torch.zeros((n, k), dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    b.collm_top_logits(dev, values, at, lse, temperature=temperature)
    for i in range(n):
        want_v, want_at, want = ov.top(host[i], k, temperature)
        assert np.array_equal(_back(values[i]), want_v) and np.array_equal(at[i].cpu().numpy(), want_at)
        assert abs(float(lse[i]) - want) <= 64 * E * max(1.0, abs(want))
    loss, grad, lab = torch.zeros(n, device="cuda"), torch.zeros_like(dev), at[:, 1].contiguous()
    if temperature > 1:  # (tau^2 times the divergence is no fp32 number there)
        return
    b.collm_distill_fwd_bwd(dev, values, at, torch.ones(n, device="cuda"), loss, grad, labels=lab, temperature=temperature, ce_weight=0.5)
    _check_distill(_back(loss), _back(grad), host, _back(values), at.cpu().numpy(), None, lab.cpu().numpy(), np.ones(n), V, dtype, temperature, 1.0, 0.5)
