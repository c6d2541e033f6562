"""A policy fine-tuning step end to end: from sampled tokens to updated weights.

    python -m paper_2305_19982_b200.policy_step [--steps 150] [--vocab 1003] [--states 8|32]

A small next-token policy (embedding, one hidden layer, output layer) is trained on a synthetic task
in which the answer to token x is (7*x + 3) mod vocab.  It stands for the last part of a language model's
step; only library matrix products come between the calls:

    embedding             the inputs' rows of the table, and in the backward pass
    embedding_grad        the table's gradient: rows of equal tokens summed in fp32, in one fixed order
    token_logprobs        log-probabilities of the sampled answers, under the sampling policy (old)
                          and the frozen one that the KL term holds on to (ref)
    policy_loss           clipped loss with KL term, and its gradient dlogits in bf16
    grad_norm_multi       norm and clip factor of the gradients of the layers in front, left on the device
    linear_wgrad_fold     dlogits is the output layer's dY: its weight gradient goes straight into
                          m, v and is never written, so it is neither in that norm nor clipped
    fold_apply8_multi     (or fold_apply_multi) the update in one pass, the layers in front clipped,
                          with the bf16 copies that the next forward pass reads

A step whose gradients are not finite, or too large for v, leaves the whole model as it was: its factor is
NaN, and nothing is folded into the output layer's moments.  Nothing waits for the host inside a step.
This module only sequences library calls and owns memory.
"""
from __future__ import annotations

import argparse
import math

import torch

from .binding import AdamA, State8, State8List, TensorList


class PolicyStep:
    def __init__(self, vocab: int = 1003, dim: int = 128, hidden: int = 256, lr: float = 3e-3,
                 max_norm: float = 1.0, kl_coef: float = 0.01, states: int = 8, seed: int = 0, device: int = 0):
        if states not in (8, 32):
            raise ValueError("states must be 8 or 32 (bits)")
        self.vocab, self.lr, self.max_norm, self.kl_coef, self.states = vocab, lr, max_norm, kl_coef, states
        self.opt = AdamA(device=device)
        self.device = self.opt.device
        self.gen = torch.Generator(device=self.device).manual_seed(seed)
        self.pitch = -(-vocab // 8) * 8     # rows of logits and of the output layer's moments start aligned

        def weights(rows, cols, std):
            return torch.randn(rows, cols, generator=self.gen, device=self.device).mul_(std)

        self.embed, self.inner = weights(vocab, dim, 1.0), weights(dim, hidden, dim ** -0.5)
        self.head = torch.zeros(hidden, self.pitch, device=self.device)
        self.head[:, :vocab] = weights(hidden, vocab, hidden ** -0.5)
        self.head_m, self.head_v = torch.zeros_like(self.head), torch.zeros_like(self.head)
        self.embed_bf, self.inner_bf, self.head_bf = (w.bfloat16() for w in (self.embed, self.inner, self.head))
        self.ref = tuple(w.clone() for w in (self.embed_bf, self.inner_bf, self.head_bf))
        # the two layers in front: gradients in bf16, one-pass update
        self.grads = [torch.zeros_like(self.embed_bf), torch.zeros_like(self.inner_bf)]
        self._g = TensorList(self.grads)
        self._w = TensorList([self.embed, self.inner])
        self._copy = TensorList([self.embed_bf, self.inner_bf])
        if states == 8:
            self.moments = State8List([State8.zeros(w.numel(), self.device) for w in (self.embed, self.inner)])
        else:
            self._m, self._v = (TensorList([torch.zeros_like(w) for w in (self.embed, self.inner)]) for _ in range(2))
        # the output layer's last gradient is folded before its update, which then adds nothing
        self._head = [TensorList([t]) for t in (self.head, torch.zeros_like(self.head_bf), self.head_m, self.head_v)]
        self._head_copy = TensorList([self.head_bf])
        self.norm = torch.zeros(4, device=self.device)
        self.sizes = torch.zeros(4, device=self.device)
        self.stats = torch.zeros(4, device=self.device)

    def forward(self, x: torch.Tensor, weights=None):
        """Activations and logits [tokens, vocab] (bf16, aligned rows) of the inputs x."""
        embed, inner, head = weights if weights is not None else (self.embed_bf, self.inner_bf, self.head_bf)
        e = torch.empty(x.numel(), embed.shape[1], dtype=embed.dtype, device=self.device)
        self.opt.embedding(x, embed, e)
        pre = e @ inner
        h = torch.relu(pre)
        return e, pre, h, (h @ head)[:, :self.vocab]

    def rollout(self, tokens: int):
        """Samples inputs and answers; returns what a step needs."""
        x = torch.randint(0, self.vocab, (tokens,), generator=self.gen, device=self.device)
        logits = self.forward(x)[3]
        y = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=self.gen)[:, 0]
        old, ref = torch.empty(2, tokens, device=self.device)
        self.opt.token_logprobs(logits, y, old)
        self.opt.token_logprobs(self.forward(x, self.ref)[3], y, ref)
        reward = (y == (7 * x + 3) % self.vocab).float()
        return x, y, old, ref, reward

    def step(self, x, y, old, ref, advantages, weights) -> None:
        """One update from a rollout; the loss terms are left in self.stats."""
        opt = self.opt
        e, pre, h, logits = self.forward(x)
        dlogits = torch.zeros(x.numel(), self.pitch, dtype=torch.bfloat16, device=self.device)
        dl = dlogits[:, :self.vocab]
        opt.policy_loss(logits, y, old, advantages, weights, dl, self.stats, ref_logp=ref, kl_coef=self.kl_coef)
        dpre = (dlogits @ self.head_bf.t()) * (pre > 0)
        torch.mm(e.t(), dpre, out=self.grads[1])
        opt.embedding_grad(x, dpre @ self.inner_bf.t(), self.grads[0])
        opt.grad_norm_multi(self._g, self.max_norm, self.norm)
        # No entry of the output layer's gradient h' dlogits exceeds |h| |dlogits|, and so the square of the norm of
        # both; v holds the entry's square.  Where that overflows, or the factor is NaN, the step is skipped.
        opt.grad_norm_multi(TensorList([h, dlogits]), math.inf, self.sizes)
        taken = torch.isfinite(self.sizes[0] ** 4) & torch.isfinite(self.norm[1])
        self.norm[1].masked_fill_(~taken, math.nan)
        head_factor = torch.where(taken, 1.0, math.nan)
        h, dlogits = (torch.where(taken, t, 0.0) for t in (h, dlogits))
        opt.begin_minibatch(1)
        opt.linear_wgrad_fold(h, dlogits[:, :self.vocab], self.head_m[:, :self.vocab], self.head_v[:, :self.vocab])
        factor = self.norm[1:2]
        if self.states == 8:
            opt.fold_apply8_multi(self._w, self._g, self.moments, self.lr, w_bf16=self._copy, grad_factor=factor)
        else:
            opt.fold_apply_multi(self._w, self._g, self._m, self._v, self.lr, w_bf16=self._copy, grad_factor=factor)
        opt.fold_apply_multi(*self._head, self.lr, w_bf16=self._head_copy, grad_factor=head_factor)

    def train(self, steps: int, tokens: int = 4096, every: int = 0):
        """`steps` rollouts with one update each; returns the mean reward of every rollout."""
        rewards = []
        for i in range(steps):
            x, y, old, ref, reward = self.rollout(tokens)
            spread = reward.std() + 1e-4
            advantages = (reward - reward.mean()) / spread
            self.step(x, y, old, ref, advantages, torch.full_like(old, 1.0 / tokens))
            rewards.append(reward.mean())
            if every and (i + 1) % every == 0:
                loss, _, kl, cut = self.stats.tolist()
                print(f"step {i + 1}: reward {float(rewards[-1]):.3f}  loss {loss:+.4f}  kl {kl:.4f}  "
                      f"clipped {cut:.3f}  |g| {float(self.norm[0]):.3f}", flush=True)
        self.opt.sync_status()
        return torch.stack(rewards).tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=1003)
    ap.add_argument("--states", type=int, default=8, choices=(8, 32))
    args = ap.parse_args()
    PolicyStep(vocab=args.vocab, states=args.states).train(args.steps, args.tokens, every=max(1, args.steps // 10))


if __name__ == "__main__":
    main()
