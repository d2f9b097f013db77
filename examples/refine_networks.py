"""Refines the weights of discovered networks by gradient, and draws the next generation's parents.

A population's networks are discovered and built as usual; each network then answers a two-choice task (one
output per choice: which of its two inputs is the larger) and learns from its own answers: activation that keeps its
states in 8 bits, an answer drawn for every pattern, the loss of that answer weighted by whether it was
right, the gradient of the weights, a step along it. At the end parents are drawn by fitness, from the fittest
fifth.

    python examples/refine_networks.py [--genomes 200] [--updates 100] [--seed 0]
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2608_27612_amd import emr, workloads as W  # noqa: E402

STEPS = 4
TEMPERATURE = 0.1


def substrate():
    """Two inputs and a bias input below, one output for each of the two choices above."""
    return W.sources_array([(-1.0, -1.0, 0), (1.0, -1.0, 0), (0.0, -1.0, 0), (-0.5, 1.0, 1), (0.5, 1.0, 1)])


def task(patterns, generator):
    """Patterns [patterns, 3] and each one's right choice."""
    ab = torch.rand((patterns, 2), generator=generator, device="cuda") * 2 - 1
    return torch.cat([ab, torch.ones_like(ab[:, :1])], 1), (ab[:, 1] > ab[:, 0]).int()


def fitness(outputs, right):
    """Mean probability of the right choice, [genomes]."""
    p = torch.softmax(outputs / TEMPERATURE, 2)
    return p.gather(2, right.long()[None, :, None].expand(len(p), -1, 1)).mean((1, 2))


def refine(net, x, right, updates, rate, generator):
    """Policy-gradient steps on every network's weights; the weights after the last one."""
    G, P = net.info().n_genomes, len(x)
    w = torch.from_numpy(net.weights()).cuda()
    truth = right.repeat(G)
    for _ in range(updates):
        outputs, kept = net.activate_keep(x, STEPS)
        scores = outputs.view(G * P, -1)
        u = torch.rand((G * P, 1), generator=generator, device="cuda")
        answer, _ = emr.emr_sample(scores, u, temperature=TEMPERATURE, logp=False)
        answer = answer.view(-1)
        # +1 for a right answer, -1 for a wrong one, averaged over the patterns
        reward = torch.where(answer == truth, 1.0, -1.0) / P
        _, grad = emr.emr_answer_loss(scores, answer, scale=reward, temperature=TEMPERATURE)
        grad_w, _ = net.activate_backward(x, STEPS, outputs, kept, grad.view_as(outputs))
        w -= rate * grad_w
        net.set_weights(w)
    return w


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--genomes", type=int, default=200)
    a.add_argument("--updates", type=int, default=100)
    a.add_argument("--patterns", type=int, default=64)
    a.add_argument("--rate", type=float, default=2.0)
    a.add_argument("--depth", type=int, default=4)
    a.add_argument("--seed", type=int, default=0)
    a = a.parse_args(argv)
    g = torch.Generator(device="cuda")
    g.manual_seed(a.seed)
    pop = emr.emr_pack_population(W.population(a.seed, a.genomes, 20, 60))
    net = emr.emr_build_networks(pop, substrate(), a.depth, 0.03, emr.EMR_CONN_ALL, 0.1, 0)
    x, right = task(a.patterns, g)
    before = fitness(net.activate_keep(x, STEPS)[0], right)
    refine(net, x, right, a.updates, a.rate, g)
    after = fitness(net.activate_keep(x, STEPS)[0], right)
    u = torch.rand((1, a.genomes), generator=g, device="cuda")
    parents, _ = emr.emr_sample(after[None], u, temperature=0.05, top_k=max(1, a.genomes // 5))
    i = net.info()
    print("%d networks, %d nodes, %d edges" % (i.n_genomes, i.nodes, i.edges))
    print("probability of the right choice: mean %.3f -> %.3f, best %.3f -> %.3f"
          % (before.mean(), after.mean(), before.max(), after.max()))
    print("%d parents drawn, %d different ones, their mean %.3f"
          % (parents.numel(), parents.unique().numel(), after[parents[0].long()].mean()))
    return before, after, parents


if __name__ == "__main__":
    main()
