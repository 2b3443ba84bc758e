"""How much of a workspace the call that shares rows uses: all it needs, or nothing."""
from __future__ import annotations

import ctypes

import pytest

from paper_2604_16400_amd import binding as b

pytestmark = pytest.mark.gpu


class _Call:
    def __init__(self, n, V, k):
        import torch

        g = torch.Generator(device="cuda").manual_seed(n)
        self.z = torch.randn(n, V, generator=g, device="cuda")
        values, at = self.z.topk(k, dim=1)
        self.t = (values + 0.1, at.to(torch.int32))
        self.ones, self.guard = torch.ones(n, device="cuda"), torch.empty(b.VOCAB_WORKSPACE + 4096, dtype=torch.uint8, device="cuda")

    def __call__(self, nbytes):
        """(loss, gradient, whether the workspace of that many bytes was written to); nothing behind it may be."""
        import torch

        self.guard.fill_(0x5A)
        loss, grad = torch.zeros(len(self.z), device="cuda"), torch.zeros_like(self.z)
        sh = b.collm_logits(len(self.z), len(self.z), self.z.shape[1], b.COLLM_F32, self.z.shape[1], None)
        d = b.collm_distill(self.t[0].shape[1], self.t[0].data_ptr(), self.t[1].data_ptr(), None, None, 1.0, 1.0, 0.0)
        rc = b.load_library().collm_distill_fwd_bwd(0, ctypes.byref(sh), self.z.data_ptr(), ctypes.byref(d), self.ones.data_ptr(), loss.data_ptr(),
                                                    grad.data_ptr(), self.z.shape[1], self.guard.data_ptr(), nbytes,
                                                    torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        assert bool((self.guard[nbytes:] == 0x5A).all())
        return loss, grad, not bool((self.guard[:nbytes] == 0x5A).all())


@pytest.mark.parametrize("n,V,k", [(1, 100000, 30), (6, 100000, 30), (31, 70000, 1), (64, 1 << 17, 1024), (2, 1 << 20, 7)])
def test_a_workspace_is_used_from_the_size_that_suffices_on(n, V, k):
    import torch

    call = _Call(n, V, k)
    without = call(0)
    assert not without[2]
    low, high = 0, b.VOCAB_WORKSPACE // 16  # in steps of 16 bytes
    shared = call(16 * high)
    assert shared[2]
    while high - low > 1:
        middle = (low + high) // 2
        if call(16 * middle)[2]:
            high = middle
        else:
            low = middle
    for nbytes, want in ((16 * low, without), (16 * high - 1, without), (16 * high, shared), (16 * high + 1, shared)):
        got = call(nbytes)
        assert got[2] == want[2] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), nbytes
