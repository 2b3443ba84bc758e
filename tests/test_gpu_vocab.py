"""Vocabulary operators on the GPU against the oracle in 64 bits.

Tolerances, fixed beforehand.  Tokens, places and the logits themselves are equal.  E = 2^-24 is half a step of fp32.
  sums     a thread adds at most ceil(V / 256) positive terms in fp32 (relative error up to that many E), each an exp2 of one
           step (2 E) whose argument of size |t| is rounded once (|t| E in the result).  Weighted with the terms' shares the mean
           |t| is at most log2(V) + 2 < 22 for V <= 2^20: S = (ceil(V / 256) + 24) E relative for any sum of exponentials.
  lse      S plus the rounding of the result.
  loss     weight * tau^2 * (its P + r = 1) * S from log sum, twice with the rest's, b S from the labels' sum, plus its rounding.
  gradient every term's size times (2 S + (|t| + 8) E), |t| <= 150 where the term is not zero, plus half a step of the result's type.
"""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu
E = 2.0**-24
INF, NAN = math.inf, math.nan


def _torch():
    import torch

    return torch


def _dt(dtype):
    torch = _torch()
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _place(rows, dtype, ld=None, offset=0):
    """rows [n, V] (numpy) as a GPU tensor with `ld` elements from row to row, `offset` elements into its memory; what lies
    between the rows is NaN."""
    torch = _torch()
    n, V = rows.shape
    ld = V if ld is None else ld
    flat = torch.full((offset + n * ld + 8,), NAN, dtype=_dt(dtype), device="cuda")
    z = flat[offset:].as_strided((n, V), (ld, 1))
    z.copy_(torch.from_numpy(rows.astype(np.float32)))
    return z


def _back(t):
    return t.float().cpu().numpy().astype(np.float64)


def _up(values, dtype=None):
    torch = _torch()
    return torch.tensor(np.asarray(values), dtype=dtype or torch.float32, device="cuda")


def _workspace(on):
    return _torch().empty(b.VOCAB_WORKSPACE, dtype=_torch().uint8, device="cuda").fill_(0xA5) if on else None


def _rows(V, rng):
    """One row of each kind that matters."""
    z = rng.normal(size=V) * 2
    kinds = [z, rng.normal(size=V) * 0.1, rng.normal(size=V) * 12]
    kinds.append(np.full(V, -INF))                                          # nothing left
    kinds.append(np.where(np.arange(V) == V // 2, 1.5, -INF))               # one left
    kinds.append(np.full(V, 3.25))                                          # all alike
    kinds.append(z + 100.0)                                                 # many alike in bf16
    kinds.append(np.where(rng.random(V) < 0.5, 1.0, 2.0))                   # two values
    kinds.append(np.where(rng.random(V) < 0.9, -3.3e38, z))                 # masked by the lowest value (of bf16)
    kinds.append(np.where(rng.random(V) < 0.99, -INF, z))                   # masked by -inf
    kinds.append(np.where(rng.random(V) < 0.3, NAN, z))
    kinds.append(np.where(np.arange(V) % max(1, V // 3) == 0, INF, z))
    kinds.append(np.where(rng.random(V) < 0.5, 0.0, -0.0))                  # zeros of both signs
    kinds.append(np.where(rng.random(V) < 0.5, 1e-39, -1e-38))              # below the normal numbers
    kinds.append(np.where(np.arange(V) == V - 1, 40.0, z))                  # one far above all others
    kinds.append(-np.log(np.arange(V) + 2.0) + rng.normal(size=V))
    return np.stack(kinds).astype(np.float32)


PARAMS = [  # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (0.0, 0, 1.0, 0.0), (1.3, 40, 1.0, 0.0), (0.8, 50, 0.95, 0.0), (1.0, 0, 0.5, 0.05), (1.0, 3, 0.99, 0.3),
    (1.0, 1, 0.5, 0.0), (2.0, 0, 0.0, 0.0), (1.0, 1 << 30, 0.999, 1.0), (1e-3, 0, 0.9, 0.0), (1e30, 0, 0.25, 0.0), (NAN, -5, NAN, NAN),
    (INF, 7, 1.0, 0.0), (1.0, 300, 0.7, 1e-6), (0.05, 0, 1.0, 2.0)]
VOCABS = [1, 2, 7, 64, 1000, 4097, 32000, 50257]


def _sample_case(V, dtype, seed, ld=None, offset=0, workspace=False, rows=None, n=None):
    torch = _torch()
    rng = np.random.default_rng(seed)
    kinds = _rows(V, rng)
    z = np.repeat(kinds, len(PARAMS), axis=0)
    par = np.array(PARAMS * len(kinds), dtype=np.float64)
    if n is not None:
        keep = rng.choice(len(z), size=n, replace=False)
        z, par = z[keep], par[keep]
    u = rng.random(len(z)).astype(np.float32)
    u[::7] = 0.0
    u[3::7] = np.float32(1.0 - 2.0**-24)
    dev = _place(z, dtype, ld, offset)
    t, k, p, m = (par[:, 0], par[:, 1], par[:, 2], par[:, 3])
    token = torch.full((len(z),), -9, dtype=torch.int32, device="cuda")
    logprob = torch.full((len(z),), NAN, device="cuda")
    b.collm_sample(dev, _up(u), token, logprob, temperature=_up(t), top_k=_up(k, torch.int32), top_p=_up(p), min_p=_up(m),
                   workspace=_workspace(workspace))
    host, got, lp = _back(dev), token.cpu().numpy(), _back(logprob)
    for i in range(len(z)):
        want, want_lp = ov.sample(host[i], u[i], t[i], int(k[i]), p[i], m[i])
        assert got[i] == want, (i // len(PARAMS), par[i], u[i], got[i], want)
        assert lp[i] == want_lp or abs(lp[i] - want_lp) <= E * abs(want_lp) + 1e-9, (i, lp[i], want_lp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", VOCABS)
def test_sample_every_kind_of_row(V, dtype):
    _sample_case(V, dtype, 100 + V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,n", [(1, 1), (3001, 2), (32000, 1), (50257, 3), (128256, 5), (151937, 8)])
def test_sample_few_rows_with_a_workspace(V, n, dtype):
    for seed in range(4):
        _sample_case(V, dtype, 200 + seed, workspace=True, n=n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ld,offset", [(1003, 0), (1008, 1), (1111, 3), (2000, 5)])
def test_sample_rows_of_any_alignment(ld, offset, dtype):
    _sample_case(1003, dtype, ld, ld, offset)


@pytest.mark.parametrize("dtype,V", [("bf16", 131072), ("bf16", 163841), ("bf16", 262147), ("f32", 65537), ("f32", 140001)])
def test_sample_long_rows(V, dtype):
    _sample_case(V, dtype, V, n=24)


def test_sample_defaults_and_rows_of_a_batch():
    torch = _torch()
    rng = np.random.default_rng(3)
    z = _place(rng.normal(size=(40, 777)).astype(np.float32) * 3, "bf16", 800)
    pick = np.array([5, 39, 0, 40, 17, -1, 2], np.int32)
    u = rng.random(len(pick)).astype(np.float32)
    token = torch.full((len(pick),), -9, dtype=torch.int32, device="cuda")
    b.collm_sample(z, _up(u), token, rows=_up(pick, torch.int32))
    host = _back(z)
    want = [ov.sample(host[r], x)[0] if 0 <= r < 40 else -1 for r, x in zip(pick, u)]
    assert token.cpu().tolist() == want


# ---- top logits ------------------------------------------------------------------------------------------------------
def _sum_error(V):
    return (math.ceil(V / 256) + 24) * E


def _top_case(V, dtype, k, tau, seed, ld=None, offset=0, workspace=False, n=None, rows=None):
    torch = _torch()
    rng = np.random.default_rng(seed)
    z = _rows(V, rng)
    if n is not None:
        z = z[rng.choice(len(z), size=n, replace=False)]
    dev = _place(z, dtype, ld, offset)
    n = len(z)
    values, lse = torch.full((n, k), NAN, device="cuda"), torch.full((n,), NAN, device="cuda")
    indices = torch.full((n, k), -9, dtype=torch.int32, device="cuda")
    b.collm_top_logits(dev, values, indices, lse, temperature=tau, workspace=_workspace(workspace))
    host, v, at, s = _back(dev), _back(values), indices.cpu().numpy(), _back(lse)
    for i in range(n):
        with np.errstate(all="ignore"):
            want_v, want_at, want_s = ov.top(host[i], k, tau)
        assert np.array_equal(v[i], want_v) and np.array_equal(at[i], want_at), i
        if np.isfinite(want_s):
            assert abs(s[i] - want_s) <= _sum_error(V) + 2 * E * abs(want_s), (i, s[i], want_s)
        elif want_s == -INF:
            assert s[i] == -INF
        else:
            assert not np.isfinite(s[i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k,tau", [(1, 1, 1.0), (5, 9, 1.0), (64, 64, 2.0), (1000, 1, 1.0), (4097, 250, 0.5), (32000, 64, 2.0), (50257, 1024, 1.0)])
def test_top_logits_every_kind_of_row(V, k, tau, dtype):
    _top_case(V, dtype, k, tau, 7 * V + k)


@pytest.mark.parametrize("dtype,V,k", [("bf16", 131072, 64), ("bf16", 163841, 255), ("bf16", 262147, 20), ("f32", 65537, 100), ("f32", 140001, 256)])
def test_top_logits_of_long_rows(V, k, dtype):
    _top_case(V, dtype, k, 1.5, V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k,ld,offset,n", [(1, 3, None, 0, 1), (3001, 20, 3003, 1, 2), (50257, 200, None, 3, 3), (128256, 64, None, 0, 4)])
def test_top_logits_few_rows_with_a_workspace(V, k, ld, offset, n, dtype):
    for seed in range(4):
        _top_case(V, dtype, k, 1.0, seed, ld, offset, workspace=True, n=n)


# ---- distillation ----------------------------------------------------------------------------------------------------
def _record(z, k, tau, rng):
    """A teacher that agrees with the rows up to noise: its k best, its log-sum-exp; some entries are none."""
    n, V = z.shape
    values, at, lse = np.full((n, k), -INF, np.float32), np.full((n, k), -1, np.int32), np.zeros(n, np.float32)
    for i in range(n):
        t = np.where(np.isfinite(z[i]), z[i], rng.normal()) + 0.5 * rng.normal(size=V)
        t = np.where(np.abs(t) > 1e30, 0.0, t).astype(np.float32)
        o = np.argsort(-t)[:k]
        values[i, :len(o)], at[i, :len(o)] = t[o], o
        lse[i] = ov.log_sum_exp(t.astype(np.float64) / tau)
    at[1::5, k // 2:] = -1
    at[3::7, 0] = V
    values[4::7, -1] = -INF
    if n > 6:
        at[6] = -1
        if k > 1:
            at[2, 1], values[2, 1] = at[2, 0], values[2, 0] - 1
    return values, at, lse


def _distill_rows(V, rng):
    z = _rows(V, rng)
    z[10] = np.where(rng.random(V) < 0.3, -INF, z[0])  # (in place of the NaN; those have a test of their own)
    z[11] = z[0] * 20                                   # (in place of the infinities)
    return z


def _check_distill(got_loss, got_grad, host, values, at, lse, labels, dloss, V, dtype, tau, a, w, rows=None):
    S = _sum_error(V)
    half = 2.0**-8 if dtype == "bf16" else E
    for i in range(len(got_loss)):
        r = i if rows is None else rows[i]
        if not 0 <= r < len(host):
            assert got_loss[i] == 0
            continue
        with np.errstate(all="ignore"):
            loss, grad, size = ov.distill(host[r], values[i], at[i], None if lse is None else lse[i], -1 if labels is None else labels[i], tau, a, w)
        if np.isfinite(loss):
            assert abs(got_loss[i] - loss) <= (2 * abs(a) * tau * tau + abs(w)) * S + 2 * E * abs(loss), (i, got_loss[i], loss)
        else:
            assert got_loss[i] == loss, (i, got_loss[i], loss)
        if got_grad is not None:
            d = abs(float(dloss[i]))
            off = np.abs(got_grad[r] - grad * float(dloss[i]))
            tol = size * d * (2 * S + 158 * E) * (1 + half) + half * np.abs(grad) * d + 1e-37
            assert (off <= tol).all(), (i, int(np.argmax(off - tol)), float((off - tol).max()))


def _distill_case(V, dtype, k, tau, tail, labels, seed, how="step", ld=None, offset=0, ld_grad=None, grad_offset=0, workspace=False, n=None, pick=None):
    torch = _torch()
    rng = np.random.default_rng(seed)
    z = _distill_rows(V, rng)
    if n is not None:
        z = z[rng.choice(len(z), size=n, replace=False)]
    dev = _place(z, dtype, ld, offset)
    host = _back(dev)
    rows = None if pick is None else np.array(pick, np.int32)
    of = z if rows is None else z[np.clip(rows, 0, len(z) - 1)]
    m = len(of)
    values, at, lse = _record(of, k, tau, rng)
    lab = np.where(rng.random(m) < 0.2, -100, at[:, 0]).astype(np.int32)
    lab[1::4] = rng.integers(0, V, size=len(lab[1::4]))
    dloss = (rng.random(m) + 0.5).astype(np.float32)
    a, w = 0.7, 0.3
    kw = dict(t_lse=_up(lse) if tail else None, labels=_up(lab, torch.int32) if labels else None, temperature=tau, kd_weight=a, ce_weight=w,
              rows=None if rows is None else _up(rows, torch.int32), workspace=_workspace(workspace))
    loss = torch.full((m,), NAN, device="cuda")
    stats = torch.full((m, b.DISTILL_STATS), NAN, device="cuda")
    t = (_up(values), _up(at, torch.int32))
    grad = None
    if how == "loss":
        b.collm_distill_fwd(dev, *t, loss, **kw)
    else:
        grad = dev if how == "in place" else _place(np.full((len(z), V), 7.5), dtype, ld_grad, grad_offset)
        if how == "two":
            b.collm_distill_fwd(dev, *t, loss, stats, **kw)
            b.collm_distill_bwd(dev, *t, stats, _up(dloss), grad, **kw)
        else:
            b.collm_distill_fwd_bwd(dev, *t, _up(dloss), loss, grad, **kw)
    got = None if grad is None else _back(grad)
    _check_distill(_back(loss), got, host, values, at, lse if tail else None, lab if labels else None, dloss, V, dtype, tau, np.float32(a), np.float32(w),
                   rows)
    if grad is not None and rows is not None:
        others = np.setdiff1d(np.arange(len(z)), rows)
        assert np.array_equal(got[others], host[others] if how == "in place" else np.full((len(others), V), 7.5), equal_nan=True)
    if grad is not None and how != "in place":  # what lies between the rows stays
        flat = grad.as_strided((grad.untyped_storage().nbytes() // grad.element_size(),), (1,), 0)
        kept = _torch().ones_like(flat, dtype=torch.bool)
        kept.as_strided(grad.shape, grad.stride(), grad.storage_offset()).fill_(False)
        assert bool(flat[kept].isnan().all())


@pytest.mark.parametrize("how", ["loss", "two", "step"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k,tau,tail,labels", [
    (1, 1, 1.0, True, True), (2, 3, 2.0, False, True), (7, 2, 1.0, True, False), (64, 64, 1.0, True, True), (1000, 16, 2.0, True, True),
    (4097, 250, 4.0, False, True), (32000, 32, 2.0, False, False), (50257, 48, 1.0, True, True)])
def test_distill_every_kind_of_row(V, k, tau, tail, labels, dtype, how):
    _distill_case(V, dtype, k, tau, tail, labels, 11 * V + k, how)


@pytest.mark.parametrize("how", ["two", "step"])
@pytest.mark.parametrize("dtype,V,k", [("bf16", 131072, 64), ("bf16", 163841, 33), ("bf16", 262147, 20), ("f32", 65537, 100), ("f32", 140001, 1024)])
def test_distill_long_rows(V, k, dtype, how):
    _distill_case(V, dtype, k, 2.0, True, True, V, how, n=6)


@pytest.mark.parametrize("how", ["two", "step", "in place"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ld,offset,ld_grad,grad_offset", [(1003, 0, 1003, 0), (1111, 3, 1003, 5), (1008, 1, 1008, 1), (1200, 2, 1016, 2)])
def test_distill_rows_of_any_alignment(ld, offset, ld_grad, grad_offset, dtype, how):
    _distill_case(1003, dtype, 20, 2.0, True, True, ld, how, ld, offset, ld_grad, grad_offset)


@pytest.mark.parametrize("how", ["loss", "two", "step"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k,n", [(1, 1, 1), (3001, 20, 2), (50257, 64, 3), (128256, 16, 4)])
def test_distill_few_rows_with_a_workspace(V, k, n, dtype, how):
    for seed in range(3):
        _distill_case(V, dtype, k, 2.0, seed != 1, seed != 2, seed, how, workspace=True, n=n)


@pytest.mark.parametrize("how", ["two", "step", "in place"])
def test_distill_rows_of_a_batch(how):
    _distill_case(777, "bf16", 12, 1.0, True, True, 5, how, ld=784, ld_grad=784, pick=[3, 0, 16, 9, -1, 7, 12, 15])


@pytest.mark.parametrize("how", ["loss", "two", "step", "in place"])
@pytest.mark.parametrize("dtype,V,n,copies", [("bf16", 257, 16, 130), ("bf16", 40000, 7, 90), ("bf16", 70001, 7, 50), ("f32", 30001, 5, 120)])
def test_distill_more_rows_than_blocks(dtype, V, n, copies, how):
    """Blocks that take several rows: copies of a few rows in another order, each row's results those of its first (all rows begin
    on 16 bytes: a row's sums are taken chunk by chunk)."""
    torch = _torch()
    rng = np.random.default_rng(V)
    k, tau = 20, 2.0
    z = _distill_rows(V, rng)[:n]
    values, at, lse = _record(z, k, tau, rng)
    lab = rng.integers(-1, V, size=n).astype(np.int32)
    dloss = (rng.random(n) + 0.5).astype(np.float32)
    order = np.concatenate([np.arange(n)] + [rng.permutation(n) for _ in range(copies - 1)])
    pick = _up(order, torch.int64)
    ld = (V + 7) // 8 * 8
    few = _place(z, dtype, ld)
    dev = torch.empty((len(order), ld), dtype=few.dtype, device="cuda")[:, :V]
    dev.copy_(few[pick])
    host = _back(few)
    big = lambda x, dt=None: _up(x, dt)[pick].contiguous()
    m = len(order)
    loss = torch.full((m,), NAN, device="cuda")
    stats = torch.full((m, b.DISTILL_STATS), NAN, device="cuda")
    t = (big(values), big(at, torch.int32))
    kw = dict(t_lse=big(lse), labels=big(lab, torch.int32), temperature=tau, kd_weight=0.7, ce_weight=0.3)
    grad = None if how == "loss" else dev if how == "in place" else torch.full((m, ld), 7.5, dtype=dev.dtype, device="cuda")[:, :V]
    if how == "loss":
        b.collm_distill_fwd(dev, *t, loss, **kw)
    elif how == "two":
        b.collm_distill_fwd(dev, *t, loss, stats, **kw)
        b.collm_distill_bwd(dev, *t, stats, big(dloss), grad, **kw)
    else:
        b.collm_distill_fwd_bwd(dev, *t, big(dloss), loss, grad, **kw)
    _check_distill(_back(loss[:n]), None if grad is None else _back(grad[:n]), host, values, at, lse, lab, dloss, V, dtype, tau, np.float32(0.7),
                   np.float32(0.3))
    assert torch.equal(loss, loss[:n][pick])
    if grad is not None:
        assert torch.equal(grad, grad[:n][pick])


def test_distill_mass_far_outside_the_record():
    """The rest of the row is so far below the record that 1 - sum q is nothing in 64 bits: its own sum keeps it."""
    torch = _torch()
    V, k = 5000, 4
    rng = np.random.default_rng(2)
    z = rng.normal(size=(2, V)).astype(np.float32)
    at = np.array([[5, 100, 2000, 4999]] * 2, np.int32)
    z[:, at[0]] += 60.0
    values = np.zeros((2, k), np.float32)
    lse = np.full(2, np.log(4 / 0.75), np.float32)  # a quarter outside
    dev, loss = _place(z, "f32"), torch.zeros(2, device="cuda")
    grad = torch.zeros_like(dev)
    ones = torch.ones(2, device="cuda")
    b.collm_distill_fwd_bwd(dev, _up(values), _up(at, torch.int32), ones, loss, grad, t_lse=_up(lse))
    _check_distill(_back(loss), _back(grad), _back(dev), values, at, lse, None, np.ones(2), V, "f32", 1.0, 1.0, 0.0)
    assert float(loss[0]) > 10


def test_distill_nan_reaches_the_loss_and_the_gradient():
    torch = _torch()
    z = torch.randn(3, 600, device="cuda")
    z[1, 77] = NAN
    z[2] = NAN
    loss, grad = torch.zeros(3, device="cuda"), torch.zeros_like(z)
    v, at = torch.zeros(3, 2, device="cuda"), torch.tensor([[1, 2]] * 3, dtype=torch.int32, device="cuda")
    for lse in (None, torch.ones(3, device="cuda")):
        b.collm_distill_fwd_bwd(z, v, at, torch.ones(3, device="cuda"), loss, grad, t_lse=lse)
        assert loss.isnan().tolist() == [False, True, True] and bool(grad[1:].isnan().all()) and not bool(grad[0].isnan().any())


def test_distill_gradient_against_differences_of_the_oracle_s_loss():
    torch = _torch()
    rng = np.random.default_rng(8)
    V, k, tau = 501, 9, 2.0
    z = rng.normal(size=(4, V)).astype(np.float32) * 2
    values, at, lse = _record(z, k, tau, rng)
    lab = rng.integers(0, V, size=4).astype(np.int32)
    dev, loss = _place(z, "f32"), torch.zeros(4, device="cuda")
    grad = torch.zeros_like(dev)
    b.collm_distill_fwd_bwd(dev, _up(values), _up(at, torch.int32), torch.ones(4, device="cuda"), loss, grad, t_lse=_up(lse),
                            labels=_up(lab, torch.int32), temperature=tau, kd_weight=0.5, ce_weight=0.5)
    host, g, h = _back(dev), _back(grad), 1e-4
    for i in range(4):
        along = rng.normal(size=V)
        f = lambda s: ov.distill(host[i] + s * along, values[i], at[i], lse[i], lab[i], tau, 0.5, 0.5)[0]
        diff = (f(h) - f(-h)) / (2 * h)
        # differences are good to h^2 times a third derivative of order |along|^3 / 6, below 1e-6 here
        assert abs(diff - float(g[i] @ along)) <= 1e-6 + (2 * _sum_error(V) + 158 * E) * float(np.abs(along).max()) * 4


# ---- runs, streams, graphs -------------------------------------------------------------------------------------------
def _all_ops(n, V, dtype, seed, workspace):
    """A closure that runs every operator on its own buffers, those buffers, and a function that draws new inputs into them."""
    torch = _torch()
    z = torch.empty((n, V), dtype=_dt(dtype), device="cuda")
    u, temp, top_p = (torch.empty(n, device="cuda") for _ in range(3))
    k = 12
    tv, ti, lse = torch.empty((n, k), device="cuda"), torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    token, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    loss, loss2, stats = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, 8), device="cuda")
    grad, grad2, dloss = torch.empty_like(z), torch.empty_like(z), torch.ones(n, device="cuda")
    teacher = torch.empty_like(z)
    ws = _workspace(workspace)

    def draw(s):
        g = torch.Generator(device="cuda").manual_seed(s)
        z.copy_(torch.randn(z.shape, generator=g, device="cuda") * 3)
        teacher.copy_(torch.randn(z.shape, generator=g, device="cuda") * 2)
        u.copy_(torch.rand(n, generator=g, device="cuda"))
        temp.copy_(0.5 + torch.rand(n, generator=g, device="cuda"))
        top_p.copy_(0.5 + 0.5 * torch.rand(n, generator=g, device="cuda"))

    def run(stream=None):
        kw = dict(workspace=ws, stream=stream)
        b.collm_sample(z, u, token, lp, temperature=temp, top_p=top_p, **kw)
        b.collm_top_logits(teacher, tv, ti, lse, temperature=2.0, **kw)
        kw.update(t_lse=lse, temperature=2.0)
        b.collm_distill_fwd(z, tv, ti, loss, stats, **kw)
        b.collm_distill_bwd(z, tv, ti, stats, dloss, grad, **kw)
        b.collm_distill_fwd_bwd(z, tv, ti, dloss, loss2, grad2, **kw)

    draw(seed)
    return run, (token, lp, tv, ti, lse, loss, grad, loss2, grad2), draw


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("n,V,dtype", [(3, 50257, "bf16"), (70, 8001, "f32")])
def test_runs_give_the_same_bits_also_on_another_stream(n, V, dtype, workspace):
    torch = _torch()
    run, outs, draw = _all_ops(n, V, dtype, 1, workspace)
    run()
    torch.cuda.synchronize()
    first = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for stream in (None, side):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        run(stream)
        torch.cuda.synchronize()
        for x, y in zip(first, outs):
            assert torch.equal(x, y)


@pytest.mark.parametrize("n,V,dtype", [(2, 32000, "bf16"), (300, 5003, "bf16"), (5, 40001, "f32")])
def test_recorded_calls_follow_their_inputs(n, V, dtype):
    torch = _torch()
    run, outs, draw = _all_ops(n, V, dtype, 1, True)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for seed in (2, 3, 4):
        draw(seed)
        run()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, outs):
            assert torch.equal(x, y)


def test_rows_beyond_32_bit_offsets():
    """Rows that begin more than 2^31 elements into the logits and their gradient."""
    torch = _torch()
    V, ld, n = 1000, 1 << 28, 12
    z = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda").as_strided((n, V), (ld, 1))
    z.copy_(torch.randn(n, V, device="cuda"))
    near = z.contiguous()
    k = 5
    outs = []
    for x in (z, near):
        values, at, lse = torch.empty((n, k), device="cuda"), torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        token, loss = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        grad = x if x is z else torch.empty_like(x)
        b.collm_top_logits(x, values, at, lse)
        b.collm_sample(x, torch.full((n,), 0.4, device="cuda"), token)
        b.collm_distill_fwd_bwd(x, values + 1, at, torch.ones(n, device="cuda"), loss, grad, t_lse=lse + 2)
        outs.append((values, at, lse, token, loss, grad.contiguous()))
    for x, y in zip(*outs):
        assert torch.equal(x, y)
