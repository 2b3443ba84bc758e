"""More rows than one launch takes blocks of: the results of a call are those of calls over parts of it."""
from __future__ import annotations

import pytest

from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("listed", [False, True])
def test_four_million_short_rows(listed):
    import torch

    n, V, k = (1 << 22) + 5, 8, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((n, V), generator=g, device="cuda").to(torch.bfloat16)
    rows = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda") if listed else None
    u, ones = torch.rand(n, generator=g, device="cuda"), torch.ones(n, device="cuda")
    f = lambda *s: torch.full(s, -7.0, device="cuda")
    i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")

    def run(z, u, ones, rows):
        n = len(u)
        token, lp, v, at, lse, loss, stats, loss2 = i32(n), f(n), f(n, k), i32(n, k), f(n), f(n), f(n, b.DISTILL_STATS), f(n)
        grad, grad2 = torch.zeros_like(z), torch.zeros_like(z)
        b.collm_sample(z, u, token, lp, rows=rows)
        b.collm_top_logits(z, v, at, lse, rows=rows)
        b.collm_distill_fwd(z, v + 0.5, at, loss, stats, t_lse=lse, rows=rows)
        b.collm_distill_bwd(z, v + 0.5, at, stats, ones, grad, t_lse=lse, rows=rows)
        b.collm_distill_fwd_bwd(z, v + 0.5, at, ones, loss2, grad2, t_lse=lse, rows=rows)
        return (token, lp, v, at, lse, loss, loss2), (grad, grad2)

    whole, grads = run(z, u, ones, rows)
    for lo in range(0, n, 1 << 20):
        hi = min(n, lo + (1 << 20))
        held = slice(lo, hi) if not listed else slice(n - hi, n - lo)
        part = torch.arange(hi - lo - 1, -1, -1, dtype=torch.int32, device="cuda") if listed else None
        outs, part_grads = run(z[held], u[lo:hi], ones[lo:hi], part)
        for x, y in zip(whole, outs):
            assert torch.equal(x[lo:hi], y)
        for x, y in zip(grads, part_grads):
            assert torch.equal(x[held], y)
