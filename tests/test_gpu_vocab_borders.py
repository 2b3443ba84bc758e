"""Vocabulary operators at values where formulas lose their meaning, against what the definitions say there."""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import _distill_case, _sample_case, _top_case

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


def _torch():
    import torch

    return torch


def _up(x, dtype=None):
    torch = _torch()
    return torch.tensor(np.asarray(x), dtype=dtype or torch.float32, device="cuda")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("V,k", [(1, 1), (7, 3), (5000, 64), (50257, 20), (50257, 300)])
def test_log_sum_exp_beside_infinities(V, k, dtype):
    """+inf anywhere in the row (among the first logits that are read, the last ones, all): +inf, but NaN where there is a NaN."""
    torch = _torch()
    rng = np.random.default_rng(V + k)
    z = rng.normal(size=(7, V)).astype(np.float32)
    z[0, 0], z[1, V - 1], z[2], z[3, V // 2] = INF, INF, INF, INF
    z[3, 0], z[4, V - 1], z[5] = NAN, NAN, -INF
    values, at, lse = torch.zeros((7, k), device="cuda"), torch.zeros((7, k), dtype=torch.int32, device="cuda"), torch.zeros(7, device="cuda")
    b.collm_top_logits(_up(z, getattr(torch, dtype)), values, at, lse, temperature=2.0)
    got = lse.cpu().numpy()
    assert np.array_equal(got[:3], [INF] * 3) and np.isnan(got[4]) and got[5] == -INF and np.isfinite(got[6])
    assert np.isnan(got[3])
    assert at[2].cpu().tolist() == [v if v < V else -1 for v in range(k)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("V", [5, 3000, 40001])
def test_sample_at_infinite_temperature(V, dtype):
    """All weights are alike, so min-p keeps all of them, at 1 too."""
    torch = _torch()
    rng = np.random.default_rng(V)
    par = [(0, 1.0, 0.0), (0, 1.0, 0.5), (0, 1.0, 1.0), (0, 1.0, 2.0), (3, 1.0, 1.0), (300, 0.5, 1.0), (0, 0.25, 1.0)]
    z = _up(rng.normal(size=(len(par), V)).astype(np.float32), getattr(torch, dtype))
    u = rng.random(len(par)).astype(np.float32)
    k, p, m = zip(*par)
    token, logprob = torch.zeros(len(par), dtype=torch.int32, device="cuda"), torch.zeros(len(par), device="cuda")
    b.collm_sample(z, _up(u), token, logprob, temperature=_up([INF] * len(par)), top_k=_up(k, torch.int32), top_p=_up(p), min_p=_up(m))
    host = z.float().cpu().numpy()
    for i in range(len(par)):
        want, want_lp = ov.sample(host[i], u[i], INF, k[i], p[i], m[i])
        assert int(token[i]) == want, (par[i], u[i], int(token[i]), want)
        assert abs(float(logprob[i]) - want_lp) <= 2.0**-24 * abs(want_lp) + 1e-9


def test_both_marshalling_routes_give_the_same_call(monkeypatch):
    """Compiled marshalling against the general path: the same results of plain arguments, the same refusals of others."""
    torch = _torch()
    rng = np.random.default_rng(4)
    n, held, V, k, ld = 9, 12, 1003, 7, 1040
    z = torch.zeros((held, ld), dtype=torch.bfloat16, device="cuda")[:, :V]
    z.copy_(_up(rng.normal(size=(held, V))))
    rows = _up(rng.permutation(held)[:n], torch.int32)
    ws = torch.zeros(b.VOCAB_WORKSPACE, dtype=torch.uint8, device="cuda")
    f = lambda lo=0.0: _up(lo + rng.random(n))
    u, temp, top_p, min_p, dloss, top_k = f(), f(0.5), f(), f(-0.9), f(), _up(rng.integers(0, 30, n), torch.int32)
    labels = _up(rng.integers(-1, V, n), torch.int32)
    new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")

    def everything():
        out = [new(n, dtype=torch.int32), new(n), new(n, k), new(n, k, dtype=torch.int32), new(n), new(n), new(n, b.DISTILL_STATS), torch.zeros_like(z),
               new(n), torch.zeros((held, V + 5), dtype=z.dtype, device="cuda")[:, :V]]
        token, lp, tv, ti, lse, loss, stats, grad, loss2, grad2 = out
        kw = dict(rows=rows, workspace=ws)
        assert b.collm_sample(z, u, token, lp, temp, top_k, top_p, min_p, **kw) is token
        assert b.collm_top_logits(z, tv, ti, lse, 2.0, **kw)[0] is tv
        t = dict(t_lse=lse, labels=labels, temperature=2.0, kd_weight=0.25, ce_weight=0.5, **kw)
        assert b.collm_distill_fwd(z, tv + 0.5, ti, loss, stats, **t) is loss
        assert b.collm_distill_bwd(z, tv + 0.5, ti, stats, dloss, grad, **t) is grad
        assert b.collm_distill_fwd_bwd(z, tv + 0.5, ti, dloss, loss2, grad2, **t) is loss2
        for bad in (dict(u=u.double()), dict(u=u[:4]), dict(token=token.long()), dict(rows=rows[::2]), dict(top_k=temp), dict(temperature=temp.cpu()),
                    dict(logits=z.half()), dict(logits=z.t()), dict(logits=z.cpu()), dict(workspace=ws.cpu())):
            with pytest.raises((ValueError, TypeError)):
                b.collm_sample(**{**dict(logits=z, u=u, token=token, rows=rows), **bad})
        for bad in (dict(dlogits=grad[:3]), dict(dlogits=grad.float()), dict(t_indices=ti[:, :3]), dict(loss=loss[:2]), dict(labels=labels.long())):
            with pytest.raises(ValueError):
                b.collm_distill_fwd_bwd(**{**dict(logits=z, t_values=tv, t_indices=ti, dloss=dloss, loss=loss2, dlogits=grad, rows=rows), **bad})
        with pytest.raises(RuntimeError):
            b.collm_top_logits(z, tv, ti, temperature=-1.0, **kw)
        return out

    assert b._marshal is not None
    first = everything()
    monkeypatch.setattr(b, "_marshal", None)
    for x, y in zip(first, everything()):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_vocabulary(dtype):
    """2^20 words and a record of 1024: the most shared memory a call asks for, the fewest bits of a weight."""
    V = 1 << 20
    _sample_case(V, dtype, 1, n=6)
    _top_case(V, dtype, 1024, 1.0, 2, n=3)
    for how, workspace in (("loss", False), ("step", False), ("step", True), ("two", False)):
        _distill_case(V, dtype, 1024, 2.0, True, True, 3, how, workspace=workspace, n=3)
