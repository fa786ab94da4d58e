"""A small language model trained by N workers through the sparse step: python -m paper_2011_06495_b200.lm_example

Each worker holds its own token pairs (a bigram model: embedding, output matrix, softmax).  One step is what a user of
the library writes around `mv_sparse_step`:

    embedding lookup -> logits (a plain matrix product) -> log probabilities -> gradient of the logits
    -> gradient of the embedding by sorted tokens and of the output matrix -> one row per worker, clipped by its own
    norm -> majority-vote sparse step -> update of the K agreed coordinates
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B


class BigramWorkers:
    """N workers, a vocabulary of V, width D, T token pairs per worker and step; dtype: of the activations and logits."""

    def __init__(self, N=4, V=2000, D=128, T=4096, sparsity=0.01, lr=2.0, max_norm=1.0, seed=0, device="cuda",
                 dtype=torch.bfloat16):
        g = torch.Generator(device=device).manual_seed(seed)
        self.N, self.V, self.D, self.T, self.lr, self.max_norm = N, V, D, T, lr, max_norm
        self.d = 2 * V * D
        self.K = max(1, int(self.d * sparsity))
        self.theta = torch.empty(self.d, device=device).normal_(0.0, 0.1, generator=g)
        # every token has four likely successors; frequent tokens have low ids
        self.next = torch.randint(0, V, (V, 4), generator=g, device=device)
        self.g = g
        self.err = torch.zeros((N, self.d), device=device)
        self.rows = torch.empty((N, self.d), device=device)
        self.norms = torch.empty(N, device=device)
        # what a worker's backward pass writes: the embedding's gradient in 32 bits, the output matrix's in the activations' type
        self.d_embed = [torch.empty((V, D), device=device) for _ in range(N)]
        self.d_out = [torch.empty((V, D), dtype=dtype, device=device) for _ in range(N)]
        tensors = [t for n in range(N) for t in (self.d_embed[n], self.d_out[n])]
        self.clip = B.MvClip(tensors, [n for n in range(N) for _ in range(2)])
        self.ctx = B.MvContext(N, self.d, self.K, device=device)
        self.out_idx = torch.empty(self.K, dtype=torch.int32, device=device)
        self.out_val = torch.empty(self.K, device=device)
        self.ws = torch.empty(B.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device=device)
        self.h = torch.empty((T, D), dtype=dtype, device=device)
        self.lp, self.ent, self.lse = (torch.empty(T, device=device) for _ in range(3))
        self.weight = torch.full((T,), -1.0 / T, device=device)          # d(mean negative log probability) / d(log probability)

    def batch(self):
        u = torch.rand(self.T, generator=self.g, device=self.theta.device)
        x = (self.V ** u - 1.0).long().clamp_(0, self.V - 1)
        y = self.next[x, torch.randint(0, 4, (self.T,), generator=self.g, device=x.device)]
        return x, y

    def worker(self, n: int, x, y):
        """Loss of worker n on its pairs; leaves the gradients in d_embed[n] and d_out[n]."""
        E, W = self.theta[: self.V * self.D].view(self.V, self.D), self.theta[self.V * self.D:].view(self.V, self.D)
        Wb = W.to(self.h.dtype)
        B.mv_embed(E, x, self.h)
        logits = self.h @ Wb.t()
        B.mv_token_logprob(logits, y, logprob=self.lp, entropy=self.ent, lse=self.lse)
        loss = -self.lp.mean()
        B.mv_token_logprob_grad(logits, y, self.lse, self.weight, logits)            # in place
        torch.mm(logits.t(), self.h, out=self.d_out[n])
        B.mv_embed_grad(logits @ Wb, x, self.d_embed[n], self.ws)
        return loss

    def step(self) -> float:
        self.last = [self.batch() for _ in range(self.N)]
        loss = torch.stack([self.worker(n, *self.last[n]) for n in range(self.N)]).mean()
        self.clip.mv_clip_pack(self.max_norm, self.rows, self.norms)
        self.ctx.mv_sparse_step(self.rows, self.err, self.out_idx, self.out_val)
        self.theta.index_add_(0, self.out_idx.long(), self.out_val, alpha=-self.lr)
        return float(loss)

    def check_gradients(self):
        """Compares one worker's row with the same quantities in 64 bits, for 32-bit activations: a logit is off by at most
        D 2^-24 |h| |W|, which p shows as a relative error, and the products of the backward pass add T or V terms; all of it
        stays below 1e-4 of the norm while D |h| |W|, in sum, stays below 1000."""
        assert self.h.dtype == torch.float32
        x, y = self.batch()
        self.worker(0, x, y)
        V, D = self.V, self.D
        E, W = (p.view(V, D).double().requires_grad_(True) for p in self.theta.split(V * D))
        torch.nn.functional.cross_entropy(E[x] @ W.t(), y).backward()
        for got, want in ((self.d_embed[0], E.grad), (self.d_out[0], W.grad)):
            off = float((got.double() - want).norm() / want.norm())
            assert off < 1e-4, off
        norm = float(torch.sqrt(self.d_embed[0].double().pow(2).sum() + self.d_out[0].double().pow(2).sum()))
        self.clip.mv_clip_pack(self.max_norm, self.rows, self.norms)
        want = torch.cat([self.d_embed[0].reshape(-1), self.d_out[0].float().reshape(-1)]).double() * min(1.0, self.max_norm / norm)
        assert float((self.rows[0].double() - want).norm()) <= 1e-6 * float(want.norm())


def main():
    ap = argparse.ArgumentParser(description="a bigram model trained by N workers through the majority-vote sparse step")
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--sparsity", type=float, default=0.01)
    a = ap.parse_args()
    m = BigramWorkers(N=a.workers, sparsity=a.sparsity)
    for i in range(a.steps):
        loss = m.step()
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {loss:.4f}  norms {', '.join('%.3f' % v for v in m.norms.tolist())}  "
                  f"entropy {float(m.ent.mean()):.3f}  K = {m.K} of {m.d}")


if __name__ == "__main__":
    main()
