"""Distillation of few long rows, a row shared by several blocks: against the oracle, with the tolerances of the rows that one block takes
(a thread adds fewer terms here)."""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import _back, _distill_case, _distill_rows, _record, _up

from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ["two", "step", "in place"])
@pytest.mark.parametrize("dtype,V,offset,ld", [("bf16", 40000, 0, 40000), ("bf16", 65543, 3, 65600), ("bf16", 128256, 0, 128256), ("f32", 50257, 1, 50261),
                                               ("f32", 20003, 0, 20003), ("f32", 160001, 2, 160004)])
def test_every_kind_of_row(dtype, V, offset, ld, how):
    for k, tau, tail, labels in ((64, 2.0, True, True), (7, 1.0, False, True), (300, 1.5, True, False)):
        _distill_case(V, dtype, k, tau, tail, labels, V + k, how, ld, offset, ld, offset, workspace=True)


@pytest.mark.parametrize("n", [1, 2, 5, 31, 64, 127, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_of_rows(n, dtype):
    """Copies of a few rows: each has the results of its first, whatever the number of shares, also in the place of the logits, and near those
    of the call without a workspace."""
    import torch

    rng = np.random.default_rng(n)
    V, k, m = 70000, 40, min(n, 5)
    z = _distill_rows(V, rng)[:m]
    values, at, lse = _record(z, k, 2.0, rng)
    at[0, 3], at[0, 4], at[m - 1, 0] = 0, V - 1, V - 1  # the row's ends
    pick = torch.arange(n, device="cuda") % m
    big = lambda x, dtype=None: _up(x, dtype)[pick].contiguous()
    dev = big(z).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    kw = dict(t_lse=big(lse), labels=big(rng.integers(-1, V, m), torch.int32), temperature=2.0, kd_weight=0.7, ce_weight=0.3)
    t, dloss = (big(values), big(at, torch.int32)), big(rng.random(m) + 0.5)
    ws = torch.full((b.VOCAB_WORKSPACE,), 0xFF, dtype=torch.uint8, device="cuda")
    loss, loss0 = torch.full((n,), math.nan, device="cuda"), torch.full((n,), math.nan, device="cuda")
    grad, grad0 = torch.full_like(dev, math.nan), torch.full_like(dev, math.nan)
    b.collm_distill_fwd_bwd(dev, *t, dloss, loss0, grad0, **kw)
    b.collm_distill_fwd_bwd(dev, *t, dloss, loss, grad, workspace=ws, **kw)
    assert torch.equal(loss, loss[:m][pick]) and torch.equal(grad, grad[:m][pick])
    step = 2.0**-8 if dtype == "bf16" else 2.0**-18  # (fp32: 274 terms a thread and exponents of a few octaves, both ways)
    for x, y in ((loss, loss0), (grad, grad0)):
        x, y = _back(x), _back(y)
        same = np.isclose(x, y, rtol=2 * step, atol=1e-7 if x.ndim == 1 else 1e-9, equal_nan=True)
        assert same.all(), (np.argwhere(~same)[:4], x[~same][:4], y[~same][:4])
    b.collm_distill_fwd_bwd(dev, *t, dloss, loss0, dev, workspace=ws, **kw)
    assert torch.equal(loss, loss0) and torch.equal(grad, dev)


@pytest.mark.parametrize("nbytes", [0, 16, 4096])
def test_a_short_workspace_will_do(nbytes):
    import torch

    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(6, 100000, generator=g, device="cuda")
    values, at = z.topk(30, dim=1)
    ws = torch.full((nbytes + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    out = []
    for w in (None, ws[:nbytes] if nbytes else None):
        loss, grad = torch.zeros(6, device="cuda"), torch.zeros_like(z)
        b.collm_distill_fwd_bwd(z, values + 0.1, at.to(torch.int32), torch.ones(6, device="cuda"), loss, grad, workspace=w, ce_weight=0.0)
        out.append((loss, grad))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and bool((ws == 0x5A).all())
