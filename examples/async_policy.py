"""Asynchronous policy training of a small language model on one GPU, with every operator of include/softsync_learn.h in its place.

The task: read two tokens a, b and answer with (a + b) mod vocab.  Simulated learners take turns in random order, as in an asynchronous
training.  A learner samples answers with the weights it holds, pulls newer ones, computes the clipped policy loss of those answers under
them (with a KL term against the initial model), and at its next turn pushes the gradient with the timestamp it pulled, by then
stale.  The server scales every gradient by its staleness, sums c of them, clips the sum's norm and makes one AdamW step with 8-bit
moments.  A second phase shows the learners pairs of answers, a right and a wrong one, and trains with the preference loss through
the same server.

    python examples/async_policy.py
"""
from __future__ import annotations

import os
import random
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1511_05950_b200 as P  # noqa: E402

VOCAB, WIDTH, BATCH = 32, 256, 512
SHAPES = [(2 * VOCAB, WIDTH), (WIDTH,), (WIDTH, WIDTH), (WIDTH,), (WIDTH, VOCAB), (VOCAB,)]


def initial(seed: int, device) -> list:
    g = torch.Generator(device).manual_seed(seed)
    return [torch.randn(s, generator=g, device=device) * (s[0] ** -0.5) if len(s) == 2 else torch.zeros(s, device=device) for s in SHAPES]


def model(params, ab):
    """Logits of the answers to the questions ab (rows x 2)."""
    e, b0, w1, b1, w2, b2 = params
    h = torch.relu(e[ab[:, 0]] + e[VOCAB + ab[:, 1]] + b0)
    return torch.relu(h @ w1 + b1) @ w2 + b2


def questions(g, device):
    return torch.randint(0, VOCAB, (BATCH, 2), generator=g, device=device)


def accuracy(params, device) -> float:
    ab = torch.cartesian_prod(torch.arange(VOCAB, device=device), torch.arange(VOCAB, device=device))
    return float((model(params, ab).argmax(1) == ab.sum(1) % VOCAB).float().mean())


class Learner:
    """Holds a copy of the weights and the timestamp that belongs to it."""

    def __init__(self, server, params, reference, device, seed):
        self.server, self.shared, self.reference, self.device = server, params, reference, device
        self.g = torch.Generator(device).manual_seed(seed)
        self.pull()

    def pull(self):
        self.ts = self.server.pull()
        self.params = [p.clone().requires_grad_(True) for p in self.shared]

    def policy_gradient(self):
        with torch.no_grad():                                       # answers and their log probabilities under the weights at hand
            ab = questions(self.g, self.device)
            logits = model(self.params, ab)
            answers = torch.multinomial(torch.softmax(logits, 1), 1, generator=self.g).squeeze(1)
            old = P.token_logprob(logits, answers).logp
            ref = P.token_logprob(model(self.reference, ab), answers).logp
            reward = (answers == ab.sum(1) % VOCAB).float()
            advantages = (reward - reward.mean()) / (reward.std() + 1e-3)
        self.pull()                                                 # the server has moved on: the ratios are no longer one
        logits = model(self.params, ab)
        loss = P.policy_loss(logits, answers, old, advantages, ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=1e-3, entropy_coef=3e-3)
        logits.backward(loss.dlogits)
        return loss.stats

    def preference_gradient(self):
        self.pull()
        ab = questions(self.g, self.device)
        right = ab.sum(1) % VOCAB
        wrong = (right + torch.randint(1, VOCAB, right.shape, generator=self.g, device=self.device)) % VOCAB
        tokens = torch.stack([right, wrong], 1).view(-1)            # sequences of one token: answer, counter-answer, answer, ...
        rows = ab.repeat_interleave(2, 0)
        with torch.no_grad():
            ref = P.token_logprob(model(self.reference, rows), tokens).logp
        logits = model(self.params, rows)
        offsets = torch.arange(2 * BATCH + 1, device=self.device)
        loss = P.preference_loss(logits, tokens, offsets, ref, beta=0.5, label_smoothing=0.01)
        logits.backward(loss.dlogits)
        return loss.stats

    def push(self, learner: int):
        """What the last turn computed, if anything."""
        if self.params[0].grad is not None and self.server.push(learner, [p.grad for p in self.params], self.ts):
            self.server.apply_update()


def train(policy_turns: int = 4000, preference_turns: int = 1200, learners: int = 8, n: int = 4, seed: int = 0, log=print) -> dict:
    device = torch.device("cuda", 0)
    params = initial(seed, device)
    reference = [p.clone() for p in params]
    server = P.AdamWServer(params, learners, n, max_norm=1.0, lr=3e-3, betas=(0.9, 0.98), weight_decay=0.0, state_bits=8, seed=seed)
    crew = [Learner(server, params, reference, device, 100 + k) for k in range(learners)]
    order = random.Random(seed)
    seen = {"start": accuracy(params, device)}
    for phase, turns in (("policy", policy_turns), ("preference", preference_turns)):
        for k in range(turns):
            who = order.randrange(learners)
            crew[who].push(who)
            stats = crew[who].policy_gradient() if phase == "policy" else crew[who].preference_gradient()
            if log and k % 500 == 0:
                log("%s %5d: loss %.4f, updates %d, accuracy %.3f" % (phase, k, float(stats[0]), server.timestamps()[0], accuracy(params, device)))
        seen[phase] = accuracy(params, device)
    seen["staleness"] = server.staleness_histogram().tolist()
    if log:
        log("accuracy %.3f -> %.3f -> %.3f; gradients by staleness: %s" % (seen["start"], seen["policy"], seen["preference"], seen["staleness"]))
    return seen


if __name__ == "__main__":
    train()
