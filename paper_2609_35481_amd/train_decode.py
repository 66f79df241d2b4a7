"""One rank of a small mixture-of-experts model, from training to decoding,
with the framework's operators as a model calls them:

  training   router logits -> moe.route -> the layer's plan (topoep.Planner, on the
             ids as they come) -> experts in torch -> loss -> backward through
             the router's gradient -> moe.clip_grads over router, main experts
             and the replicas' copies -> update
  decoding   a few tokens through moe.moe_few with the trained weights

python -m paper_2609_35481_amd.train_decode [--steps N]

The experts of every rank sit on this one GPU; a replica's gradient is a copy
of its expert's share, as its rank would hold it before the push home.
"""
from __future__ import annotations

import argparse

import torch

import workload

from . import moe, topoep


def _experts(x, ids, weights, up, down):
    """sum_j w_j down_j (silu(gate_j x) * up_j x), expert by expert."""
    inter = down.shape[2]
    out = torch.zeros_like(x)
    for e in range(up.shape[0]):
        share = (weights * (ids == e)).sum(1, keepdim=True)
        h = x @ up[e].t()
        out = out + share * ((torch.nn.functional.silu(h[:, :inter]) * h[:, inter:]) @ down[e].t())
    return out


def run(steps=4, tokens=256, hidden=256, inter=128, decode=3, seed=0, log=print):
    """Trains for `steps` steps and decodes; returns the losses, the norms and
    the largest difference of the decoded tokens, relative to the largest output."""
    cfg = workload.get("tiny")
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std):
        return torch.randn(shape, generator=gen, device=dev).mul_(std)

    gate = normal(cfg.E, hidden, std=hidden ** -0.5).requires_grad_()
    up = normal(cfg.E, 2 * inter, hidden, std=hidden ** -0.5).requires_grad_()
    down = normal(cfg.E, hidden, inter, std=inter ** -0.5).requires_grad_()
    topo = topoep.topology(cfg.R, cfg.G, cfg.E, 0, cfg.c_intra, cfg.c_inter, cfg.S, cfg.W)
    planner = topoep.Planner(topo, tokens, cfg.k, cfg.N, device=dev)
    # the token batches of all ranks, fixed: the loss then has to fall
    batches = normal(cfg.R, tokens, hidden, std=1.0)
    target = normal(tokens, hidden, std=0.5)
    losses, norms = [], []
    for step in range(steps):
        with torch.no_grad():   # every rank's row of the routing matrix, as the all-gather brings it
            rows = [torch.bincount(moe.route(b @ gate.t(), cfg.k)[0].view(-1).long(), minlength=cfg.E) for b in batches]
        omega = torch.stack(rows).to(torch.int32)
        x = batches[0]
        ids, weights = moe.route(x @ gate.t(), cfg.k)
        slots, dest, send, status = planner.plan(omega, ids)
        loss = (_experts(x, ids, weights, up, down) - target).square().mean()
        loss.backward()
        replicas = [e for e in slots[0].tolist() if e >= 0]
        grads = [gate.grad] + [t.grad[e] for e in range(cfg.E) for t in (up, down)]
        copies = [t.grad[e].clone() for e in replicas for t in (up, down)]
        norm = moe.grad_norm(grads)                       # a replica's copy counts once, with its expert
        moe.clip_grads(grads + copies, 0.1, norm=norm)    # but is scaled with it
        with torch.no_grad():
            for p in (gate, up, down):
                p -= p.grad
                p.grad = None
        losses.append(float(loss.detach()))
        norms.append(float(norm))
        log("step %d: loss %.4f, gradient norm %.4f, plan status %d, assignments sent per rank %s" %
            (step, losses[-1], norms[-1], int(status[0]), send.tolist()))
    with torch.no_grad():
        half = [t.detach().to(torch.bfloat16) for t in (gate, up, down)]
        x = batches[0][:decode].to(torch.bfloat16)
        out, ids, weights = moe.moe_few(x, half[0], half[1], half[2], cfg.k)
        want = _experts(x.float(), ids, weights, half[1].float(), half[2].float())
        off = float((out.float() - want).abs().max() / want.abs().max())
    log("decoded %d tokens, largest difference %.4f of the largest output" % (decode, off))
    return losses, norms, off


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=4)
    run(steps=parser.parse_args().steps)
