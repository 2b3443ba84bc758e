"""CPU oracle of the vocabulary operators -- TEST INFRASTRUCTURE ONLY.  Plain numpy in 64 bits, one row at a time; shares
nothing with the GPU library.

Pins (tests/test_vocab_host.py): hand-worked rows, central finite differences of the loss, brute-force sums.
"""
from __future__ import annotations

import numpy as np


def order(z):
    """Indices of the logits above -inf (NaN counts as -inf), falling, the lowest index first among equals."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    o = np.argsort(-z, kind="stable")
    return o[z[o] > -np.inf]


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log of its probability among those kept); (-1, -inf) where nothing is above -inf."""
    z, (u, temperature, top_p, min_p) = np.asarray(z, np.float64), (float(np.float32(v)) for v in (u, temperature, top_p, min_p))
    o = order(z)
    if not len(o):
        return -1, -np.inf
    if not temperature > 0:
        return int(o[0]), 0.0
    m = z[o[0]]
    with np.errstate(over="ignore", invalid="ignore"):
        y = np.where(z[o] == m, 0.0, (z[o] - m) / temperature if np.isfinite(m) else -np.inf)
        w = np.exp(y)
    if top_k > 0:
        w = w[:top_k]
    total = w.sum()
    n = len(w)
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int(np.count_nonzero(before < top_p * total)))
    if min_p > 0:
        n = min(n, int(np.count_nonzero(y >= np.log(min(min_p, 1.0)))))  # (in logarithms: exp(-1e-38) rounds to 1)
    run = np.cumsum(w[:n])
    at = min(int(np.count_nonzero(run <= u * run[-1])), int(np.count_nonzero(w[:n])) - 1)
    return int(o[at]), float(np.log(w[at] / run[-1]))


def sample_whole(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The same by weights rounded to whole multiples of 2^-45 (2^(log2 rows - 62) for long rows), which settle ties at a border beside a tail that weighs
    next to nothing.  Finite logits, -inf and NaN; temperature 0 or above 0 and finite.  (Weights next to half a unit, of which an exponential's last
    bits decide, are the caller's to keep away.)"""
    z, (u, temperature, top_p, min_p) = np.asarray(z, np.float64), (float(np.float32(v)) for v in (u, temperature, top_p, min_p))
    o = order(z)
    if not len(o):
        return -1, -np.inf
    if not temperature > 0:
        return int(o[0]), 0.0
    y = (z[o] - z[o[0]]) / temperature
    scale = min(45, 62 - int(len(z)).bit_length())
    w = np.rint(np.ldexp(np.exp(y), scale)).astype(np.int64)
    if top_k > 0:
        w = w[:top_k]
    run, n = np.cumsum(w), len(w)
    if top_p < 1:
        n = max(1, int(np.searchsorted(run - w, int(np.ceil(top_p * float(run[-1]))))))
    if min_p > 0:
        n = min(n, int(np.count_nonzero(y >= np.log(min(min_p, 1.0)))))
    kept = int(run[n - 1])
    at = int(np.searchsorted(run, min(int(u * float(kept)), kept - 1), side="right"))
    return int(o[at]), float(y[at] - np.log(np.ldexp(float(kept), -scale)))


def top(z, k, temperature=1.0):
    """(values [k], indices [k], log-sum-exp of z / temperature); -inf and -1 behind the last logit above -inf."""
    z = np.asarray(z, np.float64)
    o = order(z)[:k]
    values, indices = np.full(k, -np.inf), np.full(k, -1, np.int64)
    values[:len(o)], indices[:len(o)] = z[o], o
    return values, indices, log_sum_exp(z / np.float64(np.float32(temperature)))


def log_sum_exp(x):
    if np.isnan(x).any():
        return np.nan
    m = x.max(initial=-np.inf)
    return -np.inf if m == -np.inf else float(m + np.log(np.exp(x - m).sum()))


def distill(z, t, at, t_lse=None, label=-1, temperature=1.0, kd_weight=1.0, ce_weight=0.0):
    """(loss, gradient [V], sum of the magnitudes of the gradient's terms [V]) of one row."""
    z, t, at = np.asarray(z, np.float64), np.asarray(t, np.float64), np.asarray(at, np.int64)
    tau, a, b = (float(np.float32(v)) for v in (temperature, kd_weight, ce_weight))
    V = len(z)
    loss, grad, size = 0.0, np.zeros(V), np.zeros(V)
    if np.isnan(z).any():
        return np.nan, np.full(V, np.nan), np.full(V, np.nan)
    if not (z > -np.inf).any():
        return loss, grad, size
    z = z - z.max()  # (a logarithm of a sum beside -1e38 would be lost)
    valid = (at >= 0) & (at < V) & (t > -np.inf)
    if valid.any():
        t, at = t[valid] / tau, at[valid]
        p = np.exp(t - (log_sum_exp(t) if t_lse is None else float(t_lse)))
        lse = log_sum_exp(z / tau)
        q = np.exp(z / tau - lse)
        outside = np.ones(V, bool)
        outside[at] = False
        lse_out = log_sum_exp(z[outside] / tau) if outside.any() else -np.inf
        r = max(0.0, 1.0 - p.sum()) if t_lse is not None and lse_out > -np.inf else 0.0
        kd = sum(x * (np.log(x) - (z[v] / tau - lse)) for x, v in zip(p, at) if x > 0)
        teacher = np.zeros(V)
        np.add.at(teacher, at, p)
        rest = np.zeros(V)
        if lse_out > -np.inf:  # (from the rest's largest: beside 1e38 the logarithm of their number would be lost)
            rest[outside] = np.exp((z[outside] - z[outside].max()) / tau)
            rest /= rest.sum()
        if r > 0:
            kd += r * (np.log(r) - (lse_out - lse))
        P = p.sum() + r
        loss += a * tau * tau * kd
        grad += a * tau * (P * q - teacher - r * rest)
        size += abs(a) * tau * (P * q + teacher + r * rest)
    if 0 <= label < V:
        lse = log_sum_exp(z)
        hot = np.zeros(V)
        hot[label] = 1.0
        loss += b * (lse - z[label])
        grad += b * (np.exp(z - lse) - hot)
        size += abs(b) * (np.exp(z - lse) + hot)
    return loss, grad, size
