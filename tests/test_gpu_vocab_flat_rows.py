"""Sums over rows of nearly equal logits, where the roundings of a long sum in 32 bits all go one way, and the gradient's error in norm.

Tolerances, fixed beforehand; E = 2^-24 is half a step of fp32.
  sums      the terms of a 16-byte chunk (8 at most) are added in 32 bits (7 E), chunks in 64.  A term: an exp2 of one step (2 E) of an argument t
            that is rounded, as is what multiplies it (2 |t| E together; |t|: mean size of log2 of a term's share, by the terms' weights); of bf16 logits
            the argument is rounded near 32, to 2^-19.  S = (9 + 2 |t|) E, for bf16 2^-19 ln 2 more.
  loss      a tau^2 S from log sum, as much from the rest's, b S from the labels', and its rounding: 2 E of it
  gradient  of fp32 logits, in norm: every term's size times S (its sum) + (2 + 2 |t_v|) E (itself) + 3 E (coefficient, product, rounding)"""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import E, _back, _dt, _record, _up, _workspace

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu
A, B = np.float32(0.7), np.float32(0.3)


def _mean_log2(z, tau):
    """Mean |log2 of a term relative to the largest|, by the terms' shares."""
    y = (z - z.max()) / tau
    w = np.exp(y)
    return float((w * -y).sum() / w.sum()) / math.log(2)


def _sum_error(z, tau, dtype):
    t = max(_mean_log2(z, tau), _mean_log2(z, 1.0))
    return (9 + 2 * t) * E + (2.0**-19 * math.log(2) if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [128256, 262144, 1 << 20])
@pytest.mark.parametrize("n", [3, 1100, 2100])
def test_loss_of_many_reads_of_flat_rows(n, V, dtype):
    """Few rows and many (blocks of other sizes), all of them readings of the same twelve rows."""
    import torch

    rng = np.random.default_rng(V)
    k, tau, held = 5, 1.0, 12
    level = -0.4 - rng.random((held, 1))
    z = np.broadcast_to(level, (held, V)).copy()
    at = np.tile(np.array([3, 70000, 1000, V - 1, 50001], np.int32), (held, 1))
    z[np.arange(held)[:, None], at] = rng.random((held, k)) - 0.2
    z[:, at[0, 0]] = 0.0  # (the sums are relative to this one)
    dev = _up(z, _dt(dtype))
    host = _back(dev)
    values, lse = np.zeros((held, k), np.float32), np.full(held, np.log(k / 0.6), np.float32)
    lab = np.full(held, 17, np.int32)
    pick = np.arange(n) % held
    big = lambda x, dt=None: _up(x[pick], dt)
    loss = torch.full((n,), math.nan, device="cuda")
    b.collm_distill_fwd(dev, big(values), big(at, torch.int32), loss, t_lse=big(lse), labels=big(lab, torch.int32), temperature=tau, kd_weight=A,
                        ce_weight=B, rows=_up(pick, torch.int32))
    got = _back(loss)
    assert np.array_equal(got, got[:held][pick[:held].argsort()][pick] if n >= held else got)
    for i in range(min(n, held)):
        want = ov.distill(host[i], values[i], at[i], lse[i], lab[i], tau, A, B)[0]
        tol = (2 * A * tau * tau + B) * _sum_error(host[i], tau, dtype) + 2 * E * abs(want)
        assert abs(got[i] - want) <= tol, (i, got[i] - want, tol)


@pytest.mark.parametrize("how", ["step", "two", "shared"])
@pytest.mark.parametrize("V,tau", [(30000, 2.0), (50257, 1.0), (100001, 1.5), (160001, 2.0), (1 << 20, 2.0)])
def test_gradient_of_fp32_logits_in_norm(V, tau, how):
    import torch

    rng = np.random.default_rng(V)
    n, k = 4, 48
    z = (rng.normal(size=(n, V)) * np.array([0.01, 1.0, 2.0, 4.0])[:, None] - 0.6 * np.log(np.arange(V) + 2.0)).astype(np.float32)
    values, at, lse = _record(z, k, tau, rng)
    lab = at[:, 0].clip(0, V - 1).astype(np.int32)
    dev, host = _up(z), z.astype(np.float64)
    t, kw = (_up(values), _up(at, torch.int32)), dict(t_lse=_up(lse), labels=_up(lab, torch.int32), temperature=tau, kd_weight=A, ce_weight=B)
    loss, stats, grad, ones = torch.zeros(n, device="cuda"), torch.zeros((n, b.DISTILL_STATS), device="cuda"), torch.zeros_like(dev), torch.ones(n, device="cuda")
    if how == "two":
        b.collm_distill_fwd(dev, *t, loss, stats, **kw)
        b.collm_distill_bwd(dev, *t, stats, ones, grad, **kw)
    else:
        b.collm_distill_fwd_bwd(dev, *t, ones, loss, grad, workspace=_workspace(how == "shared"), **kw)
    got, g = _back(loss), _back(grad)
    for i in range(n):
        want, exact, size = ov.distill(host[i], values[i], at[i], lse[i], lab[i], tau, A, B)
        S = _sum_error(host[i], tau, "f32")
        assert abs(got[i] - want) <= (2 * A * tau * tau + B) * S + 2 * E * abs(want), (i, got[i], want)
        t_v = (host[i].max() - host[i]) / min(tau, 1.0) / math.log(2)
        tol = np.linalg.norm(size * (S + (5 + 2 * t_v) * E))
        assert np.linalg.norm(g[i] - exact) <= tol, (i, np.linalg.norm(g[i] - exact), tol)
