"""The head's step over a mixed batch: its logits, tokens, record, loss and gradients against the oracles, and that it learns."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import vocab as ov

pytestmark = pytest.mark.gpu


def _head(torch, **kw):
    from paper_2604_16400_amd.mixed_step import MixedHead

    head = MixedHead(**kw)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = head.n_infer
    params = {"temperature": torch.full((n,), 0.8, device="cuda"), "top_p": torch.full((n,), 0.9, device="cuda")}
    draw = lambda: (torch.randn(n, head.d, generator=g, device="cuda"), torch.randn(head.n_train, head.d, generator=g, device="cuda"),
                    torch.rand(n, generator=g, device="cuda"))
    return head, params, draw


def test_one_step_against_the_oracles():
    import torch

    head, params, draw = _head(torch, d=128, vocab=5056, n_infer=7, n_train=40, top=30)
    # an adapter that has begun to learn, so that dA is not zero
    head.B[0].copy_(torch.randn(head.B[0].shape, device="cuda") * 0.1)
    A, B = (head.A[0].double(), head.B[0].double())
    requests, train, u = draw()
    head.step(requests, train, u, params)
    z = head.logits.double().cpu().numpy()
    x = head.x.double()
    for rows, a, b in ((slice(0, 7), A, B), (slice(7, 47), head.A[1].double(), head.B[1].double()), (slice(47, 87), A, B)):
        want = (x[rows] @ head.W.double() + 2.0 * (x[rows] @ a) @ b).cpu().numpy()
        assert np.abs(z[rows] - want).max() <= 1e-2 * np.abs(want).max()
    for i in range(7):
        assert int(head.token[i]) == ov.sample(z[i], float(u[i]), 0.8, 0, float(np.float32(0.9)))[0]
    d = np.zeros((40, 5056))
    for i in range(40):
        values, at, lse = ov.top(z[7 + i], 30, 2.0)
        assert np.array_equal(values, head.values[i].cpu().numpy()) and np.array_equal(at, head.indices[i].cpu().numpy())
        loss, grad, _ = ov.distill(z[47 + i], values, at, float(np.float32(lse)), -1, 2.0, 1.0, 0.0)
        # 20 sums' terms a thread and two logarithms: 40 roundings of fp32 on temperature^2 = 4
        assert abs(float(head.loss[i]) - loss) <= 4 * 80 * 2.0**-24 + 2.0**-23 * abs(loss)
        d[i] = grad / 40
    d = torch.from_numpy(d).cuda()
    # rounded to bf16: dlogits, the products' operands; the framework's own bound for a bf16 layer is 1e-2 of the maximum
    t = x[47:87]
    for got, want in ((head.grads[1][0], 2.0 * (t @ A).T @ d), (head.grads[0][0], 2.0 * t.T @ (d @ B.T))):
        assert float((got.double() - want).abs().max()) <= 1e-2 * float(want.abs().max())


def test_the_adapter_learns_the_teacher_s_answers():
    import torch

    head, params, draw = _head(torch, d=256, vocab=4096, n_infer=9, n_train=100)
    losses = []
    train = draw()[1]
    for _ in range(40):
        requests, _, u = draw()
        head.step(requests, train, u, params)
        losses.append(float(head.loss.mean()))
    assert losses[-1] < 0.7 * losses[0] and all(np.isfinite(losses))
    assert bool((head.token >= 0).all()) and bool((head.logprob <= 0).all())
