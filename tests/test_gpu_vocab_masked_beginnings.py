"""Rows whose first columns, more than the listing pass reads before it takes what its sums are relative to, are all -inf, and whose other
logits are far from 0."""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import E, _back, _place, _up
from test_gpu_vocab_far_logits import _lse

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu
INF = math.inf


def _rows(V, rng, masked):
    """Flat rows (nearly all of the mass is beside any list) at several offsets; `masked` columns in front, and some behind, are -inf."""
    z = rng.normal(size=(8, V)) * 0.3 + np.array([-2000.0, -300.0, -130.0, -60.0, -8.0, 0.0, 130.0, 2000.0])[:, None]
    z[:, :masked] = -INF
    z[::2, V - 100:] = -INF
    return z


@pytest.mark.parametrize("temperature", [1.0, 0.05, 2.0])
@pytest.mark.parametrize("dtype,V,masked", [("f32", 50257, 17000), ("f32", 50257, 30000), ("bf16", 128256, 60000), ("f32", 50257, 40000), ("bf16", 128256, 33000), ("bf16", 128256, 120000), ("f32", 70000, 69990)])
def test_log_sum_exp(dtype, V, masked, temperature):
    _lse(_rows(V, np.random.default_rng(masked), masked), dtype, 64, temperature)


@pytest.mark.parametrize("masked", [17000, 30000, 32700, 33000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature,top_k,top_p,min_p", [(1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.05, 0, 0.5, 0.0), (0.7, 0, 1.0, 0.2), (1.0, 0, 0.001, 0.0),
                                                           (1.0, 50, 0.9, 0.0), (0.0, 0, 1.0, 0.0)])
def test_tokens(temperature, top_k, top_p, min_p, dtype, masked):
    import torch

    V = 50257
    rng = np.random.default_rng(7)
    dev = _place(_rows(V, rng, masked).astype(np.float32), dtype)
    n = dev.shape[0]
    host = _back(dev)
    for u in rng.random((4, n)).astype(np.float32):
        token, logprob = torch.full((n,), -9, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
        b.collm_sample(dev, _up(u), token, logprob, temperature=_up([temperature] * n), top_k=_up([top_k] * n, torch.int32), top_p=_up([top_p] * n),
                       min_p=_up([min_p] * n))
        for i in range(n):
            want, want_lp = ov.sample_whole(host[i], u[i], temperature, top_k, top_p, min_p)
            assert int(token[i]) == want, (i, u[i], int(token[i]), want)
            assert abs(float(logprob[i]) - want_lp) <= E * abs(want_lp) + 2.0**-17
