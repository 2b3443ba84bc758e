"""One definition, three ways: the same row has the same token whichever way it is done.  Which way that is follows from the row:
    bf16 without top-k          by value
    fp32                        off a list; by steps if the list cannot decide
    fp32 with a NaN, uncut      by steps (the list's sum is no number); a NaN counts as -inf, so the row is the same row
The definition is in whole multiples of 2^-45 (2^-scale from vocabularies of 2^17 on): the oracle here adds whole numbers."""
from __future__ import annotations

import math

import numpy as np
import pytest
from test_gpu_vocab import _dt, _up

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


def _tokens(z, u, temperature, top_p, min_p, dtype):
    import torch

    n = len(z)
    token = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    b.collm_sample(_up(z, _dt(dtype)), _up(u), token, temperature=_up([temperature] * n), top_p=_up([top_p] * n), min_p=_up([min_p] * n))
    return token.cpu().tolist()


def _rows(V, rng):
    """A few logits alike at the top, whose share of the weights is a border, and a tail that weighs nothing: in whole numbers nothing at all, a unit
    each, or some units each.  The last logit is -inf."""
    rows = []
    for n_top in (2, 4, 5, 8):
        for tail in (-36.0, -33.0, -32.0, -31.0, -30.0, -28.0):
            z = tail - 8.0 * rng.random(V)
            z[rng.choice(V - 1, n_top, replace=False)] = 0.0
            rows.append(z)
    z = np.stack(rows)
    z[:, V - 1] = -INF
    z, scale = z.astype(np.float32).astype(np.float64), min(45, 62 - int(V).bit_length())
    for _ in range(20):  # (no weight near half a unit)
        units = np.ldexp(np.exp(z), scale)
        z[(np.abs(units - np.floor(units) - 0.5) < 1e-3) & (units < 1e6)] -= 1.0 / 64
    assert (np.abs(units - np.floor(units) - 0.5)[units < 1e6] >= 1e-3).all()
    return z.astype(np.float32)


@pytest.mark.parametrize("V", [1003, 50257, 131072])
@pytest.mark.parametrize("top_p,min_p", [(0.5, 0.0), (0.25, 0.0), (0.2, 0.0), (1.0, 0.0), (0.75, 0.0), (0.5, 0.1), (1.0, 1e-13)])
def test_ties_at_the_borders(V, top_p, min_p):
    z = _rows(V, np.random.default_rng(V))
    nan = z.copy()
    nan[:, V - 1] = NAN
    for u in (0.0, 0.25, 0.5, 0.75, 0.2, 0.9, 1.0 - 2.0**-24):
        u = np.full(len(z), u, np.float32)
        want = [ov.sample_whole(row, x, 1.0, 0, top_p, min_p)[0] for row, x in zip(z, u)]
        assert _tokens(nan, u, 1.0, top_p, min_p, "f32") == want, (u[0], "by steps")
        assert _tokens(z, u, 1.0, top_p, min_p, "f32") == want, (u[0], "off a list")


@pytest.mark.parametrize("temperature,top_p,min_p", [(1.0, 0.9, 0.0), (0.7, 1.0, 0.0), (1.0, 0.5, 0.01), (0.2, 0.95, 0.0), (1.3, 1.0, 0.05), (1.0, 0.0, 0.0)])
@pytest.mark.parametrize("V", [7, 1000, 32000, 50257])
def test_every_way_gives_the_same_token(V, temperature, top_p, min_p):
    """Rows of bf16 values, as bf16 and as fp32, with and without a NaN, at many random numbers."""
    import torch

    rng = np.random.default_rng(V)
    z = rng.normal(size=(5, V)) * np.array([0.1, 1.0, 2.0, 4.0, 12.0])[:, None] - np.log(np.arange(V) + 2.0)
    z = np.repeat(torch.tensor(z).to(torch.bfloat16).float().numpy(), 40, axis=0)
    z[:, V - 1] = -INF
    nan = z.copy()
    nan[:, V - 1] = NAN
    u = rng.random(len(z)).astype(np.float32)
    want = _tokens(z, u, temperature, top_p, min_p, "bf16")
    assert _tokens(z, u, temperature, top_p, min_p, "f32") == want
    assert _tokens(nan, u, temperature, top_p, min_p, "f32") == want


@pytest.mark.parametrize("rise", [5.0, 21.0, 23.0, 40.0, 60.0, 90.0])
def test_rows_that_rise_behind_their_beginning(rise):
    """What the listing pass's sum is relative to lies far below the rest of the row: at some distance the row goes by steps."""
    V = 50257
    rng = np.random.default_rng(int(rise))
    z = np.repeat((rng.normal(size=(2, V)) * np.array([0.001, 1.0])[:, None]).astype(np.float32), 60, axis=0)
    z[:, 16400:] += np.float32(rise)
    z[:, 30000] = rise + 9.0
    z[:, V - 1] = -INF
    nan = z.copy()
    nan[:, V - 1] = NAN
    u = rng.random(len(z)).astype(np.float32)
    for top_p, min_p in ((1.0, 0.0), (0.1, 0.0), (0.9, 0.0), (1.0, 0.5)):
        want = [ov.sample_whole(row, x, 1.0, 0, top_p, min_p)[0] for row, x in zip(z, u)]
        assert _tokens(nan, u, 1.0, top_p, min_p, "f32") == want
        assert _tokens(z, u, 1.0, top_p, min_p, "f32") == want
