"""A model's output head in a mixed batch, from hidden states to tokens and updated adapters:

    python -m paper_2604_16400_amd.mixed_step [--steps N]

One forward call takes three kinds of rows: requests that are answered (adapter 0), a teacher's view of the training tokens (adapter 1) and the training tokens themselves (adapter 0).  Behind it, on the logits as they lie: requests become tokens
(collm_sample), the teacher's rows a record of their top logits (collm_top_logits), the training rows a loss against that record and
the gradient of their logits (collm_distill_fwd_bwd), which enters the head's backward call; AdamW updates adapter 0.  The weight is
random and stays; over steps on the same training tokens the distance between the adapters' answers falls.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding


class MixedHead:
    """Buffers and adapters of the head.  n_infer requests, n_train training tokens; d: width of the hidden states; vocab and ranks: multiples
    of 8."""

    def __init__(self, d=1024, vocab=32000, n_infer=24, n_train=200, rank=32, teacher_rank=16, top=64, temperature=2.0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda std, *shape: (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)
        self.d, self.vocab, self.n_infer, self.n_train, self.temperature = d, vocab, n_infer, n_train, temperature
        T = n_infer + 2 * n_train
        self.rank = np.array([rank, teacher_rank], np.int32)
        self.W = normal(4.0 / d**0.5, d, vocab)
        self.A = [normal(1.0 / d**0.5, d, rank), normal(1.0 / d**0.5, d, teacher_rank)]
        self.B = [torch.zeros((rank, vocab), dtype=torch.bfloat16, device="cuda"), normal(0.3, teacher_rank, vocab)]
        # requests, a sequence each; the teacher's rows; the training rows
        self.seg_start = np.array(list(range(n_infer + 1)) + [n_infer + n_train, T], np.int32)
        self.seg_adapter = np.array([0] * n_infer + [1, 0], np.int32)
        self.seg_is_train = np.array([0] * n_infer + [0, 1], np.uint8)
        at = torch.arange(T, dtype=torch.int32, device="cuda")
        self.infer_rows, self.teacher_rows, self.train_rows = at[:n_infer], at[n_infer:n_infer + n_train].contiguous(), at[n_infer + n_train:].contiguous()
        self.ctx = binding.Context(T, n_infer + 2, 2, max(rank, teacher_rank), max(d, vocab))
        new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")
        self.x, self.logits, self.dlogits = (new(T, n, dtype=torch.bfloat16) for n in (d, vocab, vocab))
        self.h = new(T, max(rank, teacher_rank))
        self.token, self.logprob = new(n_infer, dtype=torch.int32), new(n_infer)
        self.values, self.indices, self.lse = new(n_train, top), new(n_train, top, dtype=torch.int32), new(n_train)
        self.loss, self.dloss = new(n_train), torch.full((n_train,), 1.0 / n_train, device="cuda")
        # (the teacher's adapter has no training rows: no gradient)
        self.grads = [[torch.zeros(t.shape, device="cuda") for t in tables] for tables in (self.A, self.B)]
        self.moments = [[(torch.zeros_like(t), torch.zeros_like(t)) for t in tables] for tables in self.grads]
        self.masters = [tables[0].float() for tables in (self.A, self.B)]
        self.workspace = new(binding.VOCAB_WORKSPACE, dtype=torch.uint8)
        self.steps = 0

    def step(self, requests, train, u, params, lr=1e-2):
        """requests [n_infer, d], train [n_train, d]: hidden states; u [n_infer]: random numbers; params: collm_sample's temperature, top_k,
        top_p and min_p.  Fills `token`, `logprob` and `loss` and updates adapter 0."""
        n, m = self.n_infer, self.n_train
        self.x[:n].copy_(requests)
        self.x[n:n + m].copy_(train)
        self.x[n + m:].copy_(train)
        head = (self.x, self.W, self.A, self.B, self.rank, self.seg_start, self.seg_adapter, self.seg_is_train, 2.0)
        self.ctx.collm_lora_linear_fwd(*head, self.logits, self.h)
        ws = self.workspace
        binding.collm_sample(self.logits, u, self.token, self.logprob, rows=self.infer_rows, workspace=ws, **params)
        binding.collm_top_logits(self.logits, self.values, self.indices, self.lse, self.temperature, rows=self.teacher_rows, workspace=ws)
        binding.collm_distill_fwd_bwd(self.logits, self.values, self.indices, self.dloss, self.loss, self.dlogits, t_lse=self.lse,
                                      temperature=self.temperature, rows=self.train_rows, workspace=ws)
        self.ctx.collm_lora_linear_bwd(*head, self.dlogits, self.h, None, self.grads[0], self.grads[1])
        self.steps += 1
        for tables, grads, moments, master in zip((self.A, self.B), self.grads, self.moments, self.masters):
            binding.collm_adapter_adamw(tables[0], grads[0], *moments[0], lr, 0.9, 0.99, 1e-8, 0.0, self.steps, master=master)


def main():
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=20)
    args = parser.parse_args()
    head = MixedHead()
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    n = head.n_infer
    params = {"temperature": torch.full((n,), 0.8, device="cuda"), "top_k": torch.full((n,), 50, dtype=torch.int32, device="cuda"),
              "top_p": torch.full((n,), 0.95, device="cuda")}
    train = rand(head.n_train, head.d)
    for i in range(args.steps):
        head.step(rand(n, head.d), train, torch.rand(n, generator=g, device="cuda"), params)
        if i % 5 == 0 or i + 1 == args.steps:
            print(f"step {i}: loss {float(head.loss.mean()):.4f}, first tokens {head.token[:4].tolist()}")


if __name__ == "__main__":
    main()
