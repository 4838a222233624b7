#!/usr/bin/env python3
"""Learning with the message passing from rewards alone: no gradient of the reward is asked for, only its value.

A network's scores for every pixel (here: made up, noisy and badly scaled, in 16 bits) become unaries by a layer
norm, a few learned values per label distance become the pairwise function, ISGMR passes messages, and labels are
drawn from the SoftMin of the final costs.  A pixel whose label is right earns 1, others nothing; the policy loss
turns that into a gradient of the costs, which the backward pass carries to the weight and bias of the norm and to
the pairwise values.  Three updates per set of drawn labels: hence the old log-probabilities and the clipping; the KL
term holds the policy near the first one.

    python examples/learn_by_reward.py [--steps 20]
"""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_1910_10892_amd as mrf  # noqa: E402
from paper_1910_10892_amd.autograd import bucket_pairwise, layer_norm, message_passing, policy_loss, softmin_logp  # noqa: E402


def make_scores(B, H, W, L, generator, device):
    """A piecewise constant labelling, and scores that favour it: half of the pixels point elsewhere."""
    truth = torch.randint(0, L, (B, H // 8, W // 8), generator=generator, device=device)
    truth = truth.repeat_interleave(8, 1).repeat_interleave(8, 2)
    seen = torch.where(torch.rand(truth.shape, generator=generator, device=device) < 0.5, truth,
                       torch.randint(0, L, truth.shape, generator=generator, device=device))
    scores = 3.0 + 0.5 * torch.randn((B, H, W, L), generator=generator, device=device)
    scores.scatter_add_(3, seen[..., None], torch.full((B, H, W, 1), -2.0, device=device))
    return truth, scores.to(torch.bfloat16)


def learn(steps=20, B=4, H=32, W=48, L=16, n_buckets=9, updates=3, seed=0, device="cuda:0"):
    """Mean reward of every step's labels, the learned pairwise values and the last loss."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    truth, scores = make_scores(B, H, W, L, gen, device)
    weight = torch.ones(L, device=device, requires_grad=True)
    bias = torch.zeros(L, device=device, requires_grad=True)
    values = torch.zeros(n_buckets, device=device, requires_grad=True)
    # a symmetric function: buckets of distances, whatever their sign, so that every value has one
    lower = mrf.mrf_distance_buckets(n_buckets, L - 1, -(L - 1), L, two_sided=False)
    bucket_of = torch.from_numpy(np.concatenate([lower, lower[-2::-1]])).to(device)
    optimizer = torch.optim.Adam([weight, bias, values], lr=0.05)

    def costs():
        unary = layer_norm(scores, weight, bias, dtype=torch.float32)
        V = bucket_pairwise(values, bucket_of, -(L - 1), L, L)
        return message_passing(unary, V, algo="isgmr", K=2)[0]

    rewards, loss = [], None
    first = costs().detach()
    for _ in range(steps):
        drawn = costs().detach()
        noise = -torch.log(-torch.log(torch.rand(drawn.shape, generator=gen, device=device).clamp_(1e-9, 1.0 - 1e-7)))
        labels = (noise - drawn).argmax(3).to(torch.uint8)
        reward = (labels == truth).float()
        advantage = reward - reward.mean()
        old, reference = softmin_logp(drawn, labels), softmin_logp(first, labels)
        for _ in range(updates):
            optimizer.zero_grad()
            loss, _, _ = policy_loss(costs(), labels, advantage.reshape(-1), old, reference, kl_weight=0.001)
            loss.backward()
            optimizer.step()
        rewards.append(float(reward.mean()))
    return rewards, values.detach().cpu(), float(loss.detach())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    rewards, values, _ = learn(args.steps)
    for i, r in enumerate(rewards):
        print("step %2d  mean reward %.3f" % (i, r))
    print("pairwise values by bucket:", [round(float(v), 3) for v in values])
