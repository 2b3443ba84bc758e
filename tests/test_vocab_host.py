"""Vocabulary operators without a GPU: the oracle's pins and every refusal of the C entry points."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

from oracle import vocab as ov
from paper_2604_16400_amd import binding as b

INF, NAN = np.inf, np.nan


# ---- the oracle ------------------------------------------------------------------------------------------------------
def test_sample_by_hand():
    # weights 1, 1/2, 1/4, 1/4 in the order 2, 0, 1, 3: running sums 1, 1.5, 1.75, 2
    z = np.log([0.5, 0.25, 1.0, 0.25])
    draw = lambda u, **kw: ov.sample(z, u, **kw)[0]
    assert [draw(u) for u in (0.0, 0.49, 0.51, 0.74, 0.76, 0.87, 0.88)] == [2, 2, 0, 0, 1, 1, 3]
    assert [draw(u, top_k=2) for u in (0.0, 0.66, 0.67, 0.99)] == [2, 2, 0, 0]
    assert [draw(u, top_p=0.74) for u in (0.66, 0.67, 0.99)] == [2, 0, 0]
    assert [draw(u, min_p=0.3) for u in (0.66, 0.67, 0.99)] == [2, 0, 0]
    assert draw(0.99, temperature=0.0) == 2 and draw(0.99, top_p=0.0) == 2
    # at half the temperature the weights are squares: 1, 1/4, 1/16, 1/16
    assert [draw(u, temperature=0.5) for u in (0.72, 0.73)] == [2, 0]
    assert ov.sample(z, 0.6)[1] == pytest.approx(np.log(0.25))


def test_sample_ties_masks_and_infinities():
    assert ov.sample([1, 1, 1, 1], 0.5)[0] == 2 and ov.sample([1, 1, 1, 1], 0.9, top_k=2)[0] == 1
    assert ov.sample([1, 1, 1, 1], 0.9, top_p=0.5)[0] == 1
    assert ov.sample([-INF, NAN, -INF], 0.3) == (-1, -INF)
    assert ov.sample([-INF, 3.0, NAN, -INF], 0.999)[0] == 1
    assert ov.sample([0.0, INF, 5.0, INF], 0.6)[0] == 3


def test_top_by_hand():
    v, i, lse = ov.top([1.0, 3.0, -INF, 3.0], 4)
    assert list(v) == [3, 3, 1, -INF] and list(i) == [1, 3, 0, -1] and lse == pytest.approx(np.log(2 * np.e**3 + np.e))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distill_gradient_against_differences(tail, tau):
    rng = np.random.default_rng(5)
    z, at = rng.normal(size=23) * 2, np.array([3, 17, -1, 4, 17])
    t = rng.normal(size=5)
    kw = dict(t_lse=3.5 if tail else None, label=7, temperature=tau, kd_weight=0.5, ce_weight=0.25)
    _, grad, size = ov.distill(z, t, at, **kw)
    h = 1e-5
    for v in range(23):
        e = np.zeros(23)
        e[v] = h
        diff = (ov.distill(z + e, t, at, **kw)[0] - ov.distill(z - e, t, at, **kw)[0]) / (2 * h)
        assert abs(diff - grad[v]) < 1e-8
    assert abs(grad.sum()) < 1e-12 and (np.abs(grad) <= size + 1e-15).all()


def test_distill_is_the_divergence_of_the_whole_distribution():
    # a record of everything, with or without the log-sum-exp, is the plain KL; by hand for two words
    z, t = np.array([0.0, np.log(3.0)]), np.array([np.log(0.5), np.log(0.5)])
    want = 0.5 * np.log(0.5 / 0.25) + 0.5 * np.log(0.5 / 0.75)
    for lse in (None, 0.0):
        assert ov.distill(z, t, [0, 1], t_lse=lse)[0] == pytest.approx(want)
    # a record of one word and the rest as one: the divergence of the two-way split
    z = np.log([0.25, 0.25, 0.5])
    got = ov.distill(z, [np.log(0.75)], [2], t_lse=0.0)[0]
    assert got == pytest.approx(0.75 * np.log(0.75 / 0.5) + 0.25 * np.log(0.25 / 0.5))


def test_distill_rows_without_a_term():
    z = np.array([0.5, -1.0, 2.0])
    for at in ([-1], [3]):
        loss, grad, _ = ov.distill(z, [1.0], at)
        assert loss == 0 and not grad.any()
    assert ov.distill(z, [-INF], [1])[0] == 0
    assert ov.distill(np.full(3, -INF), [1.0], [1], label=0, ce_weight=1.0)[0] == 0


# ---- refusals: nothing below reaches a GPU ----------------------------------------------------------------------------
P = 0x10000  # stands for device memory


def _calls(sh, logits=P, names=None, **over):
    """The status of each entry point (of `names`) for these rows; `over` replaces arguments by name."""
    lib = b.load_library()
    g = lambda name, default: over.get(name, default)
    d = b.collm_distill(g("k", 4), g("values", P), g("indices", P), g("lse", P), g("labels", P), g("temperature", 1.0), g("kd_weight", 1.0),
                        g("ce_weight", 0.0))
    pr = b.collm_sampling(g("row_temperature", P), P, P, g("min_p", P))
    shp = None if sh is None else ctypes.byref(sh)
    ws = (g("workspace", None), g("workspace_bytes", 0))
    dp = None if g("teacher", True) is None else ctypes.byref(d)
    grad = (g("dlogits", P + (1 << 30)), g("ld_grad", 100))
    calls = {
        "sample": lambda: lib.collm_sample(0, shp, logits, g("u", P), ctypes.byref(pr), g("token", P), g("logprob", P), *ws, None),
        "top": lambda: lib.collm_top_logits(0, shp, logits, g("k", 4), g("temperature", 1.0), g("values", P), g("indices", P), g("lse", P), *ws,
                                            None),
        "fwd": lambda: lib.collm_distill_fwd(0, shp, logits, dp, g("loss", P), g("stats", P), *ws, None),
        "bwd": lambda: lib.collm_distill_bwd(0, shp, logits, dp, g("stats", P), g("dloss", P), *grad, None),
        "fwd_bwd": lambda: lib.collm_distill_fwd_bwd(0, shp, logits, dp, g("dloss", P), g("loss", P), *grad, *ws, None),
    }
    return {name: calls[name]() for name in names or ALL}


def _shape(n=3, held=3, vocab=100, dtype=b.COLLM_BF16, ld=100, rows=None):
    return b.collm_logits(n, held, vocab, dtype, ld, rows)


ALL = {"sample", "top", "fwd", "bwd", "fwd_bwd"}
DISTILL = {"fwd", "bwd", "fwd_bwd"}
NULL, SHAPE, DTYPE, ALIGN = -1, -2, -6, -7


@pytest.mark.parametrize("shape,logits,status", [
    (None, P, NULL), (_shape(), None, NULL), (_shape(dtype=2), P, DTYPE), (_shape(n=-1), P, SHAPE), (_shape(held=-1), P, SHAPE),
    (_shape(n=4), P, SHAPE), (_shape(vocab=0, ld=0), P, SHAPE), (_shape(vocab=(1 << 20) + 1, ld=1 << 21), P, SHAPE), (_shape(ld=99), P, SHAPE),
    (_shape(ld=1 << 61), P, SHAPE), (_shape(), P + 1, ALIGN), (_shape(dtype=b.COLLM_F32), P + 2, ALIGN), (_shape(rows=P + 2), P, ALIGN)])
def test_rows_are_refused(shape, logits, status):
    assert _calls(shape, logits) == {name: status for name in ALL}


@pytest.mark.parametrize("over,names,status", [
    ({"k": 0}, ALL - {"sample"}, SHAPE), ({"k": 1025}, ALL - {"sample"}, SHAPE),
    ({"temperature": 0.0}, ALL - {"sample"}, SHAPE), ({"temperature": -1.0}, ALL - {"sample"}, SHAPE),
    ({"temperature": NAN}, ALL - {"sample"}, SHAPE), ({"temperature": INF}, ALL - {"sample"}, SHAPE),
    ({"kd_weight": NAN}, DISTILL, SHAPE), ({"ce_weight": INF}, DISTILL, SHAPE), ({"teacher": None}, DISTILL, NULL),
    ({"values": None}, ALL - {"sample"}, NULL), ({"indices": None}, ALL - {"sample"}, NULL), ({"values": P + 2}, ALL - {"sample"}, ALIGN),
    ({"lse": P + 1}, ALL - {"sample"}, ALIGN), ({"labels": P + 2}, DISTILL, ALIGN),
    ({"u": None}, {"sample"}, NULL), ({"token": None}, {"sample"}, NULL), ({"logprob": P + 2}, {"sample"}, ALIGN), ({"min_p": P + 2}, {"sample"}, ALIGN),
    ({"row_temperature": P + 1}, {"sample"}, ALIGN),
    ({"loss": None}, {"fwd", "fwd_bwd"}, NULL), ({"stats": None}, {"bwd"}, NULL), ({"stats": P + 2}, {"fwd", "bwd"}, ALIGN),
    ({"dloss": None}, {"bwd", "fwd_bwd"}, NULL), ({"dlogits": None}, {"bwd", "fwd_bwd"}, NULL), ({"dlogits": P + (1 << 30) + 1}, {"bwd", "fwd_bwd"}, ALIGN),
    ({"ld_grad": 99}, {"bwd", "fwd_bwd"}, SHAPE), ({"ld_grad": 1 << 61}, {"bwd", "fwd_bwd"}, SHAPE),
    ({"dlogits": P + 16}, {"bwd", "fwd_bwd"}, SHAPE),                  # half over the logits
    ({"dlogits": P, "ld_grad": 108}, {"bwd", "fwd_bwd"}, SHAPE),       # in their place, rows elsewhere
    ({"workspace_bytes": -1}, ALL - {"bwd"}, SHAPE), ({"workspace_bytes": 64}, ALL - {"bwd"}, NULL),
    ({"workspace": P + 8, "workspace_bytes": 64}, ALL - {"bwd"}, ALIGN)])
def test_arguments_are_refused(over, names, status):
    assert _calls(_shape(), names=names, **over) == {n: status for n in names}


def test_no_rows_is_no_work():
    assert _calls(_shape(n=0, held=0), None, workspace=None) == {name: 0 for name in ALL}


def test_the_binding_refuses_other_tensors():
    torch = pytest.importorskip("torch")
    z = torch.zeros(3, 100, dtype=torch.bfloat16)
    f, i = torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    for bad in (dict(u=f.double()), dict(token=i.long()), dict(logits=z.t().contiguous().t()), dict(logits=z.half()), dict(top_k=f),
                dict(temperature=torch.zeros(6)[::2]), dict(rows=torch.zeros(2, dtype=torch.int32))):
        kw = dict(logits=z, u=f, token=i)
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            b.collm_sample(**kw)
    v, at = torch.zeros(3, 4), torch.zeros(3, 4, dtype=torch.int32)
    for bad in (dict(t_indices=at[:, :3]), dict(loss=f[:2]), dict(dlogits=z.float()), dict(dlogits=z[:2]), dict(labels=i.long())):
        kw = dict(logits=z, t_values=v, t_indices=at, dloss=f, loss=f, dlogits=torch.zeros_like(z))
        kw.update(bad)
        with pytest.raises(ValueError):
            b.collm_distill_fwd_bwd(**kw)
