"""A cascade as a policy: preferences first, then a clipped policy loss.

    python -m paper_1511_05946_amd.policy [--N 256] [--classes 200] [--K 4]

A small example of a whole training step around the cascade: the forward pass,
a loss on the first ``classes`` columns of its rows, the backward pass from the
gradient of that loss, the clipped norm of the parameters' gradients, and an
AdamW step (moments in 8 bits).

Problem.  Contexts x ~ N(0, 1) of width N; a teacher, itself a cascade of two
layers with diagonals ~ N(1, 0.5^2), scores the actions of a context; the
reward of an action is the share of the actions that score below it.  The
policy is the softmax over the outputs of a cascade of K layers with biases,
initialised as identity plus a small perturbation (Sec. 6.1), without
permutations and ReLU.

1. Preferences: pairs of short sequences (one context and action per row), the
   preferred one with the higher reward in every row, against the initial
   policy as the reference (``losses.preference_loss``).
2. Policy: actions drawn from the current policy, their log-probabilities and
   those of the reference (``losses.token_logprobs``), then a few steps of the
   clipped loss with a KL term on them (``losses.policy_loss``).

Prints one JSON line per phase: the mean reward of drawn actions and the loss.
"""

from __future__ import annotations

import argparse
import json

import torch

from . import acdc, losses, optim


class CascadePolicy:
    """A cascade's diagonals and biases, their moments, and their step."""

    def __init__(self, N: int, K: int, classes: int, device, seed: int = 0, lr: float = 2e-3, bits: int = 8):
        g = torch.Generator(device="cpu").manual_seed(seed)
        draw = lambda mean, std: (mean + std * torch.randn(K, N, generator=g)).to(device)  # noqa: E731
        self.params = [draw(1.0, 0.05), draw(1.0, 0.05), draw(0.0, 0.01)]
        self.moments = [optim.moments(p, bits) for p in self.params]
        self.classes, self.lr, self.steps = classes, lr, 0

    def logits(self, x):
        """Rows of logits (a view of the cascade's rows) and what the backward pass needs."""
        A, D, bias = self.params
        y, saved = acdc.forward(x, A, D, save=True, bias=bias)
        return y[:, :self.classes], saved

    def update(self, x, saved, grad_y):
        """Backward pass from the gradient of the rows, and one step. The norm of
        the gradients stays on the device."""
        A, D, bias = self.params
        _, *grads = acdc.backward(x, grad_y, A, D, saved=saved, bias=bias)
        clip = optim.grad_norm(grads, max_norm=1.0)
        self.steps += 1
        # diagonals near 1 are not to be drawn to 0
        optim.adamw_step(self.params, grads, self.moments, self.steps, lr=self.lr, weight_decay=0.0, grad_scale=clip[1:])
        return clip

    def step(self, x, loss):
        """One training step: ``loss(logits, out)`` writes dL/dlogits into ``out``.
        Columns past the classes have no part in the loss: their gradient is 0."""
        logits, saved = self.logits(x)
        grad_y = torch.zeros_like(x)
        r = loss(logits, grad_y[:, :self.classes])
        self.update(x, saved, grad_y)
        return r


def teacher(N: int, classes: int, device, seed: int = 1):
    """rewards(x): [rows, classes] in [0, 1), an action's rank among its context's."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    A, D = ((1.0 + 0.5 * torch.randn(2, N, generator=g)).to(device) for _ in range(2))

    def rewards(x):
        scores = acdc.forward(x, A, D)[0][:, :classes]
        return scores.argsort(1).argsort(1).float() / classes

    return rewards


def mean_reward(policy, rewards, x, gen):
    with torch.no_grad():
        logits, _ = policy.logits(x)
        a = torch.multinomial(logits.softmax(1), 1, generator=gen)
        return float(rewards(x).gather(1, a).mean())


def train(N: int = 256, classes: int = 200, K: int = 4, pairs: int = 64, length: int = 16, preference_steps: int = 60,
          rounds: int = 20, inner: int = 4, rows: int = 2048, bits: int = 8, seed: int = 0, device=None):
    """Both phases; returns [(phase, mean reward of drawn actions, last loss), ...]."""
    device = torch.device(device if device is not None else "cuda:0")
    gen = torch.Generator(device=device).manual_seed(seed)
    policy = CascadePolicy(N, K, classes, device, seed, bits=bits)
    reference = CascadePolicy(N, K, classes, device, seed, bits=bits)   # the same start
    rewards = teacher(N, classes, device)
    test = torch.randn(4096, N, generator=gen, device=device)
    history = [("start", mean_reward(policy, rewards, test, gen), None)]

    # sequences of `length` rows, preferred ones and others in turn
    offsets = torch.arange(0, 2 * pairs * length + 1, length, dtype=torch.int32, device=device)
    for _ in range(preference_steps):
        x = torch.randn(pairs, 1, length, N, generator=gen, device=device).expand(pairs, 2, length, N).reshape(-1, N)
        score = rewards(x).view(pairs, 2, length, classes)
        two = torch.randint(0, classes, (pairs, 2, length), generator=gen, device=device)
        r = score.gather(3, two.unsqueeze(3)).squeeze(3)
        two = torch.where((r[:, :1] >= r[:, 1:]), two, two.flip(1)).reshape(-1)
        ref = losses.token_logprobs(reference.logits(x)[0], two).logp
        out = policy.step(x, lambda y, g: losses.preference_loss(y, two, offsets, ref, beta=0.2, out=g))
    history.append(("preference", mean_reward(policy, rewards, test, gen), float(out.stats[0])))

    for _ in range(rounds):
        x = torch.randn(rows, N, generator=gen, device=device)
        logits, _ = policy.logits(x)
        a = torch.multinomial(logits.softmax(1), 1, generator=gen)
        r = rewards(x).gather(1, a).squeeze(1)
        adv = (r - r.mean()) / (r.std() + 1e-6)
        a = a.squeeze(1)
        old = losses.token_logprobs(logits, a).logp
        ref = losses.token_logprobs(reference.logits(x)[0], a).logp
        for _ in range(inner):
            out = policy.step(x, lambda y, g: losses.policy_loss(y, a, old, adv, logp_ref=ref, clip=(0.2, 0.28),
                                                                 kl_coef=1e-3, entropy_coef=1e-3, out=g))
    history.append(("policy", mean_reward(policy, rewards, test, gen), float(out.stats[0])))
    return history


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--N", type=int, default=256)
    ap.add_argument("--classes", type=int, default=200)
    ap.add_argument("--K", type=int, default=4)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    for phase, reward, loss in train(a.N, a.classes, a.K, bits=a.bits, seed=a.seed):
        print(json.dumps({"phase": phase, "mean_reward": reward, "loss": loss}), flush=True)


if __name__ == "__main__":
    main()
