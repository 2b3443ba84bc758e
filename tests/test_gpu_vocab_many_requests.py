"""More requests than compute units, two to a unit by a kernel of their own: the results of a call for those that have one each."""
from __future__ import annotations

import numpy as np
import pytest
from test_gpu_vocab import PARAMS, _dt, _place, _rows, _up

from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ld,offset", [(7, 7, 0), (1000, 1003, 1), (32000, 32000, 0), (50257, 50260, 3), (131073, 131073, 0)])
def test_every_kind_of_row(V, ld, offset, dtype):
    import torch

    rng = np.random.default_rng(V)
    kinds = _rows(V, rng)
    z = np.tile(np.repeat(kinds, len(PARAMS), axis=0), (3, 1))
    par = np.array(PARAMS * (3 * len(kinds)), dtype=np.float64)
    n = len(z)
    order = rng.permutation(n)
    dev = _place(z[order], dtype, ld, offset)
    t, k, p, m = (_up(par[order, 0]), _up(par[order, 1], torch.int32), _up(par[order, 2]), _up(par[order, 3]))
    u = _up(rng.random(n))

    def run(at):
        token, logprob = torch.full((len(at),), -9, dtype=torch.int32, device="cuda"), torch.zeros(len(at), device="cuda")
        pick = at.long()
        b.collm_sample(dev, u[pick], token, logprob, temperature=t[pick], top_k=k[pick], top_p=p[pick], min_p=m[pick], rows=at)
        return token, logprob

    everything = torch.arange(n, dtype=torch.int32, device="cuda")
    token, logprob = run(everything)
    for part in everything.split(128):
        few, few_lp = run(part)
        assert torch.equal(token[part.long()], few) and torch.equal(logprob[part.long()], few_lp)
