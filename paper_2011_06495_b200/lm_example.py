"""A small language model trained by N workers through the sparse step: python -m paper_2011_06495_b200.lm_example

Each worker holds its own token pairs (a bigram model: embedding, layer norm if asked for, output matrix, softmax).  One step is
what a user of the library writes around `mv_sparse_step`:

    embedding lookup -> layer norm -> logits (a plain matrix product) -> log probabilities, or the divergence from a teacher's
    alternatives -> gradient of the logits -> gradients of the norm, of the embedding by sorted tokens and of the output matrix
    -> one row per worker, clipped by its own norm -> majority-vote sparse step -> update of the K agreed coordinates

`generate` draws tokens from the model.  --distill trains a second model from the first one's alternatives.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B


class BigramWorkers:
    """N workers, a vocabulary of V, width D, T token pairs per worker and step; dtype: of the activations and logits; norm: a layer
    norm in front of the output matrix; teacher: a model of the same vocabulary whose k best tokens take the targets' place."""

    def __init__(self, N=4, V=2000, D=128, T=4096, sparsity=0.01, lr=2.0, max_norm=1.0, seed=0, device="cuda",
                 dtype=torch.bfloat16, norm=False, teacher=None, k=16):
        g = torch.Generator(device=device).manual_seed(seed)
        self.N, self.V, self.D, self.T, self.lr, self.max_norm = N, V, D, T, lr, max_norm
        self.norm, self.teacher = norm, teacher
        self.d = 2 * V * D + (2 * D if norm else 0)
        self.K = max(1, int(self.d * sparsity))
        self.theta = torch.empty(self.d, device=device).normal_(0.0, 0.1, generator=g)
        if norm:
            self.theta[2 * V * D:] = torch.cat([torch.ones(D, device=device), torch.zeros(D, device=device)])
        # every token has four likely successors; frequent tokens have low ids
        self.next = torch.randint(0, V, (V, 4), generator=g, device=device) if teacher is None else teacher.next
        self.g = g
        self.err = torch.zeros((N, self.d), device=device)
        self.rows = torch.empty((N, self.d), device=device)
        self.norms = torch.empty(N, device=device)
        # what a worker's backward pass writes: the embedding's and the norm's gradients in 32 bits, the output matrix's in the activations' type
        self.d_embed = [torch.empty((V, D), device=device) for _ in range(N)]
        self.d_out = [torch.empty((V, D), dtype=dtype, device=device) for _ in range(N)]
        self.d_norm = [torch.empty((2, D), device=device) for _ in range(N)] if norm else None
        tensors = [[self.d_embed[n], self.d_out[n]] + ([self.d_norm[n]] if norm else []) for n in range(N)]
        self.clip = B.MvClip([t for ts in tensors for t in ts], [n for n in range(N) for _ in tensors[n]])
        self.ctx = B.MvContext(N, self.d, self.K, device=device)
        self.out_idx = torch.empty(self.K, dtype=torch.int32, device=device)
        self.out_val = torch.empty(self.K, device=device)
        self.ws = torch.empty(B.embed_grad_workspace_bytes(T, V, D), dtype=torch.uint8, device=device)
        self.ws_norm = torch.empty(B.layer_norm_grad_workspace_bytes(T, D), dtype=torch.uint8, device=device)
        self.h = torch.empty((T, D), dtype=dtype, device=device)
        self.y = torch.empty_like(self.h) if norm else self.h               # what the output matrix sees
        self.lp, self.ent, self.lse, self.kl, self.log_rest, self.mean, self.rstd = (torch.empty(T, device=device) for _ in range(7))
        self.top = torch.empty((T, k), device=device)
        self.top_id = torch.empty((T, k), dtype=torch.int32, device=device)
        self.weight = torch.full((T,), -1.0 / T, device=device)          # d(mean negative log probability) / d(log probability)

    def batch(self):
        u = torch.rand(self.T, generator=self.g, device=self.theta.device)
        x = (self.V ** u - 1.0).long().clamp_(0, self.V - 1)
        y = self.next[x, torch.randint(0, 4, (self.T,), generator=self.g, device=x.device)]
        return x, y

    def parameters(self):
        """Embedding, output matrix, gain and bias of the norm (None without one)."""
        n = self.V * self.D
        E, W = self.theta[:n].view(self.V, self.D), self.theta[n:2 * n].view(self.V, self.D)
        return E, W, *((self.theta[2 * n:2 * n + self.D], self.theta[2 * n + self.D:]) if self.norm else (None, None))

    def logits(self, x):
        """Logits of the tokens x (as many as T or fewer) in the activations' type; leaves what the backward pass needs."""
        E, W, gain, bias = self.parameters()
        n = len(x)
        B.mv_embed(E, x, self.h[:n])
        if self.norm:
            B.mv_layer_norm(self.h[:n], gain, bias, self.y[:n], mean=self.mean[:n], rstd=self.rstd[:n])
        return self.y[:n] @ W.to(self.h.dtype).t()

    def worker(self, n: int, x, y):
        """Loss of worker n on its pairs; leaves the gradients in d_embed[n], d_out[n] and d_norm[n]."""
        W, gain = self.parameters()[1:3]
        logits = self.logits(x)
        if self.teacher is None:
            B.mv_token_logprob(logits, y, logprob=self.lp, entropy=self.ent, lse=self.lse)
            loss = -self.lp.mean()
            B.mv_token_logprob_grad(logits, y, self.lse, self.weight, logits)            # in place
        else:
            B.mv_token_logprob(self.teacher.logits(x), top_logprob=self.top, top_id=self.top_id)
            B.mv_distill(logits, self.top, self.top_id, kl=self.kl, lse=self.lse, log_rest=self.log_rest)
            loss = self.kl.mean()
            B.mv_distill_grad(logits, self.top, self.top_id, self.lse, -self.weight, logits, log_rest=self.log_rest)
        torch.mm(logits.t(), self.y, out=self.d_out[n])
        dh = logits @ W.to(self.h.dtype)
        if self.norm:
            B.mv_layer_norm_grad(dh, self.h, gain, self.mean, self.rstd, dh, self.d_norm[n][0], self.d_norm[n][1], self.ws_norm)
        B.mv_embed_grad(dh, x, self.d_embed[n], self.ws)
        return loss

    def step(self) -> float:
        self.last = [self.batch() for _ in range(self.N)]
        loss = torch.stack([self.worker(n, *self.last[n]) for n in range(self.N)]).mean()
        self.clip.mv_clip_pack(self.max_norm, self.rows, self.norms)
        self.ctx.mv_sparse_step(self.rows, self.err, self.out_idx, self.out_val)
        self.theta.index_add_(0, self.out_idx.long(), self.out_val, alpha=-self.lr)
        return float(loss)

    def generate(self, start, length: int, scale: float = 1.0, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
        """`length` tokens after each of `start` (at most T of them): int64 [length, len(start)]."""
        n, dev = len(start), start.device
        row = lambda v, dtype=torch.float32: torch.full((n,), v, dtype=dtype, device=dev)
        settings = dict(scale=row(scale), top_k=row(top_k, torch.int32), top_p=row(top_p), min_p=row(min_p))
        u = torch.rand((length, n), generator=self.g, device=dev)
        out = torch.empty((length, n), dtype=torch.int64, device=dev)
        for i in range(length):
            B.mv_sample(self.logits(out[i - 1] if i else start), u[i], out[i], **settings)
        return out

    def check_gradients(self):
        """Compares one worker's row with the same quantities in 64 bits, for 32-bit activations: a logit is off by at most
        D 2^-24 |h| |W|, which p shows as a relative error, and the products of the backward pass add T or V terms; all of it
        stays below 1e-4 of the norm while D |h| |W|, in sum, stays below 1000."""
        assert self.h.dtype == torch.float32
        x, y = self.batch()
        self.worker(0, x, y)
        E, W, gain, bias = (p.double().requires_grad_(True) if p is not None else None for p in self.parameters())
        h = E[x]
        if self.norm:
            h = torch.nn.functional.layer_norm(h, (self.D,), gain, bias)
        if self.teacher is None:
            torch.nn.functional.cross_entropy(h @ W.t(), y).backward()
        else:
            logp, ids, q = torch.log_softmax(h @ W.t(), 1), self.top_id.long(), self.top.double().exp()
            rest = 1.0 - q.sum(1)
            log_rest = torch.logsumexp(logp.scatter(1, ids, float("-inf")), 1)
            (-((q * logp.gather(1, ids)).sum(1) + rest * log_rest).mean()).backward()
        pairs = [(self.d_embed[0], E.grad), (self.d_out[0], W.grad)] + ([(self.d_norm[0], torch.stack([gain.grad, bias.grad]))] if self.norm else [])
        for got, want in pairs:
            off = float((got.double() - want).norm() / want.norm())
            assert off < 1e-4, off
        row = torch.cat([got.reshape(-1).double() for got, _ in pairs])
        self.clip.mv_clip_pack(self.max_norm, self.rows, self.norms)
        want = row * min(1.0, self.max_norm / float(row.norm()))
        assert float((self.rows[0].double() - want).norm()) <= 1e-6 * float(want.norm())


def train(m, steps):
    for i in range(steps):
        loss = m.step()
        if i % 10 == 0 or i == steps - 1:
            entropy = f"entropy {float(m.ent.mean()):.3f}  " if m.teacher is None else ""
            print(f"step {i:4d}  loss {loss:.4f}  norms {', '.join('%.3f' % v for v in m.norms.tolist())}  {entropy}K = {m.K} of {m.d}")


def main():
    ap = argparse.ArgumentParser(description="a bigram model trained by N workers through the majority-vote sparse step")
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--sparsity", type=float, default=0.01)
    ap.add_argument("--norm", action="store_true", help="a layer norm in front of the output matrix")
    ap.add_argument("--distill", action="store_true", help="train a second model from the first one's alternatives")
    ap.add_argument("--generate", type=int, default=0, help="tokens to draw after each of 1024 starts")
    a = ap.parse_args()
    m = BigramWorkers(N=a.workers, sparsity=a.sparsity, norm=a.norm)
    train(m, a.steps)
    if a.distill:
        m = BigramWorkers(N=a.workers, sparsity=a.sparsity, norm=a.norm, teacher=m, seed=1)
        train(m, a.steps)
    if a.generate:
        start = m.batch()[0][:1024]
        out = m.generate(start, a.generate, top_k=50, top_p=0.9)
        before = torch.cat([start[None], out[:-1]])
        print(f"drawn tokens that follow in the data: {float((m.next[before] == out[..., None]).any(-1).float().mean()):.3f}")


if __name__ == "__main__":
    main()
