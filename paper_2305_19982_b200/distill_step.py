"""A distillation step end to end: from tokens and a teacher's top logits to updated weights.

    python -m paper_2305_19982_b200.distill_step [--steps 150] [--vocab 1003] [--top 16] [--micro 2]

A small student (embedding, norm, one hidden layer, norm, output layer) learns what a larger frozen teacher answers,
of which it sees the `top` largest logits of each token and their log-sum-exp, as they would be read from a file.
The gradients of every layer go straight into its moments, micro-batch after micro-batch, and none is ever held
in memory; only library matrix products and the relu come between the calls:

    embedding                  the inputs' rows of the table (negative inputs are padding: rows of zeros)
    layer_norm                 and what its backward pass reads, mean and rstd
    distill_loss               divergence from the teacher, and its gradient dlogits in bf16 (over the logits)
    linear_wgrad_fold          the two linear layers' weight gradients into their moments
    layer_norm_backward_fold   the gradient of the norm's input; its weight's and bias's into their moments
    embedding_grad_fold        the table's gradient into its moments, touching the rows that occur
    apply_multi                the update of all layers

A micro-batch's loss weighs a token 1/tokens, and the optimizer takes the mean over the micro-batches.  A gradient
that is not finite stays in the moments, as with every fold.  Nothing waits for the host inside a step.  This module
only sequences library calls and owns memory.
"""
from __future__ import annotations

import argparse

import torch

from .binding import AdamA, TensorList


class DistillStep:
    def __init__(self, vocab: int = 1003, dim: int = 128, hidden: int = 256, top: int = 16, lr: float = 3e-3, seed: int = 0,
                 device: int = 0):
        self.vocab, self.top, self.lr = vocab, top, lr
        self.opt = AdamA(device=device)
        self.device = self.opt.device
        self.gen = torch.Generator(device=self.device).manual_seed(seed)
        self.pitch = -(-vocab // 8) * 8     # rows of logits and of the output layer's moments start aligned

        def weights(rows, cols, std, pitch=0):
            w = torch.randn(rows, cols, generator=self.gen, device=self.device).mul_(std)
            return torch.nn.functional.pad(w, (0, pitch - cols)) if pitch else w

        def norm(n):
            return torch.ones(n, device=self.device), torch.zeros(n, device=self.device)

        self.teacher = (weights(vocab, 2 * dim, 1.0).bfloat16(),
                        weights(2 * dim, vocab, 4.0 * (2 * dim) ** -0.5, self.pitch).bfloat16())
        # table, norm, hidden layer, norm, output layer
        self.w = [weights(vocab, dim, 1.0), *norm(dim), weights(dim, hidden, dim ** -0.5), *norm(hidden),
                  weights(hidden, vocab, hidden ** -0.5, self.pitch)]
        self.m, self.v = [torch.zeros_like(w) for w in self.w], [torch.zeros_like(w) for w in self.w]
        self._lists = [TensorList(t) for t in (self.w, self.m, self.v)]
        self.copies = {i: self.w[i].bfloat16() for i in (0, 3, 6)}      # what the matrix products read
        self.stats = torch.zeros(4, device=self.device)

    def batch(self, tokens: int, padding: float = 0.0):
        """Inputs, the teacher's top logits and their indices, and the log-sum-exp of all its logits."""
        x = torch.randint(0, self.vocab, (tokens,), generator=self.gen, device=self.device)
        out, table = self.teacher[1], self.teacher[0]
        e = torch.empty(tokens, table.shape[1], dtype=torch.bfloat16, device=self.device)
        self.opt.embedding(x, table, e)
        logits = (e @ out)[:, :self.vocab]
        logp, lse = torch.empty(2, tokens, device=self.device)
        self.opt.token_logprobs(logits, x, logp, lse=lse)
        values, ids = torch.topk(logits, self.top, dim=1)
        if padding:
            x = torch.where(torch.rand(tokens, generator=self.gen, device=self.device) < padding, -1, x)
        return x, values, ids, lse

    def micro_batch(self, x, values, ids, lse) -> None:
        """Forward and backward pass of one micro-batch; its gradients are folded, its loss terms left in self.stats."""
        opt, tokens = self.opt, x.numel()
        table, w1, b1, inner, w2, b2, head = self.w
        table, inner, head = self.copies[0], self.copies[3], self.copies[6]
        like = dict(dtype=torch.bfloat16, device=self.device)
        e = torch.empty(tokens, table.shape[1], **like)
        opt.embedding(x, table, e)
        (n1, mean1, rstd1), (n2, mean2, rstd2) = [
            (torch.empty(tokens, w.numel(), **like), *torch.empty(2, tokens, device=self.device)) for w in (w1, w2)]
        opt.layer_norm(e, w1, b1, n1, mean1, rstd1)
        h = torch.relu(n1 @ inner)
        opt.layer_norm(h, w2, b2, n2, mean2, rstd2)
        logits = n2 @ head      # zeros in the padding columns, where the gradient stays 0
        weights = torch.where(x < 0, 0.0, 1.0 / tokens)
        d = logits[:, :self.vocab]
        opt.distill_loss(d, values, ids, weights, d, self.stats, teacher_lse=lse)
        m, v = self.m, self.v
        dh = logits @ head.t()
        opt.linear_wgrad_fold(n2, d, m[6][:, :self.vocab], v[6][:, :self.vocab])
        opt.layer_norm_backward_fold(dh, h, w2, mean2, rstd2, dh, m[4], v[4], m[5], v[5])
        dh *= h > 0
        opt.linear_wgrad_fold(n1, dh, m[3], v[3])
        de = dh @ inner.t()
        opt.layer_norm_backward_fold(de, e, w1, mean1, rstd1, de, m[1], v[1], m[2], v[2])
        opt.embedding_grad_fold(x, de, m[0], v[0])

    def step(self, batches) -> None:
        """One update from the micro-batches of `batches`."""
        self.opt.begin_minibatch(len(batches))
        for batch in batches:
            self.micro_batch(*batch)
        self.opt.apply_multi(*self._lists, self.lr)
        for i, copy in self.copies.items():
            copy.copy_(self.w[i])

    def train(self, steps: int, tokens: int = 4096, micro: int = 2, every: int = 0):
        """`steps` updates; returns the last micro-batch's divergence of each."""
        losses = []
        for i in range(steps):
            self.step([self.batch(tokens) for _ in range(micro)])
            losses.append(self.stats[0].clone())
            if every and (i + 1) % every == 0:
                loss, ce, mass, teacher = self.stats.tolist()
                print(f"step {i + 1}: divergence {loss:.4f}  cross entropy {ce:.4f}  mass on the teacher's top {self.top} "
                      f"{mass:.3f} (its own {teacher:.3f})", flush=True)
        self.opt.sync_status()
        return torch.stack(losses).tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--micro", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=1003)
    ap.add_argument("--top", type=int, default=16)
    args = ap.parse_args()
    DistillStep(vocab=args.vocab, top=args.top).train(args.steps, args.tokens, args.micro, every=max(1, args.steps // 10))


if __name__ == "__main__":
    main()
