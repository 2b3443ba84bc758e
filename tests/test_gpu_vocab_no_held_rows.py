"""Logits without a row (a batch that has none yet), and index lists into them: rows that are not there."""
from __future__ import annotations

import math

import pytest

from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("compiled", [True, False])
@pytest.mark.parametrize("V", [1, 5003])
def test_rows_of_no_logits_are_not_there(V, compiled, monkeypatch):
    import torch

    if not compiled:
        b.load_library()
        monkeypatch.setattr(b, "_marshal", None)
    n, k = 3, 4
    z = torch.empty((0, V), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, -1, 7], dtype=torch.int32, device="cuda")
    f = lambda *s: torch.full(s, 5.0, device="cuda")
    i32 = lambda *s: torch.full(s, 5, dtype=torch.int32, device="cuda")
    token, logprob, values, at, lse, loss, loss2, stats = i32(n), f(n), f(n, k), i32(n, k), f(n), f(n), f(n), f(n, b.DISTILL_STATS)
    b.collm_sample(z, f(n) / 10, token, logprob, rows=rows)
    b.collm_top_logits(z, values, at, lse, rows=rows)
    b.collm_distill_fwd(z, f(n, k), i32(n, k), loss, stats, rows=rows)
    b.collm_distill_bwd(z, f(n, k), i32(n, k), stats, f(n), torch.empty_like(z), rows=rows)
    b.collm_distill_fwd_bwd(z, f(n, k), i32(n, k), f(n), loss2, torch.empty_like(z), rows=rows)
    assert token.tolist() == [-1] * n and logprob.tolist() == [-math.inf] * n
    assert bool((values == -math.inf).all()) and bool((at == -1).all()) and loss.tolist() == loss2.tolist() == [0.0] * n
    # and no rows of them
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    b.collm_sample(z, torch.empty(0, device="cuda"), none)
    b.collm_sample(z, torch.empty(0, device="cuda"), none, rows=none)
