"""One rank of a small mixture-of-experts model, from training to decoding,
with the framework's operators as a model calls them:

  training   router logits -> moe.route -> the layer's plan (topoep.Planner, on the
             ids as they come) -> experts in torch -> loss -> backward through
             the router's gradient -> moe.clip_grads over router, main experts
             and the replicas' copies -> update
  decoding   a few tokens through moe.moe_few with the trained weights

With --half the experts train in bfloat16 through ffn.experts, whose gradients reach
the router and 32-bit weights, and decoding goes through their 8-bit
integers too (ffn.expert_rows, ffn.quantize, ffn.matmul_int8).

python -m paper_2609_35481_amd.train_decode [--steps N] [--half]

The experts of every rank sit on this one GPU; a replica's gradient is a copy
of its expert's share, as its rank would hold it before the push home.
"""
from __future__ import annotations

import argparse

import torch

import workload

from . import ffn, moe, topoep


def _experts(x, ids, weights, up, down):
    """sum_j w_j down_j (silu(gate_j x) * up_j x), expert by expert."""
    inter = down.shape[2]
    out = torch.zeros_like(x)
    for e in range(up.shape[0]):
        share = (weights * (ids == e)).sum(1, keepdim=True)
        h = x @ up[e].t()
        out = out + share * ((torch.nn.functional.silu(h[:, :inter]) * h[:, inter:]) @ down[e].t())
    return out


def _experts_half(x, ids, weights, up, down):
    """The same by the framework's kernels, in bfloat16."""
    half = torch.bfloat16
    return ffn.experts(x.to(half), ids, weights, up.to(half), down.to(half)).float()


def _experts_int8(x, ids, weights, up, down):
    """The same in 8-bit integers: weights quantised by channel, as at loading, and rows by token."""
    E = up.shape[0]
    (qu, su), (qd, sd) = (ffn.quantize(w.flatten(0, 1)) for w in (up, down))
    offsets, pairs, places = ffn.expert_rows(ids, E)
    rows = x[pairs.long() // ids.shape[1]]
    h = ffn.matmul_int8(rows, qu.view(up.shape), su.view(E, -1), offsets, gated=True, dtype=torch.float32)
    y = ffn.matmul_int8(h, qd.view(down.shape), sd.view(E, -1), offsets, dtype=torch.float32)
    return (y[places.long()] * weights[:, :, None]).sum(1)


def run(steps=4, tokens=256, hidden=256, inter=128, decode=3, seed=0, log=print, half=False):
    """Trains for `steps` steps and decodes; returns the losses, the norms and
    the largest difference of the decoded tokens, relative to the largest output (with
    half, also that of the tokens decoded in 8-bit integers)."""
    block = _experts_half if half else _experts
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
        loss = (block(x, ids, weights, up, down) - target).square().mean()
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
        trained = [t.detach().to(torch.bfloat16) for t in (gate, up, down)]
        x = batches[0][:decode].to(torch.bfloat16)
        out, ids, weights = moe.moe_few(x, trained[0], trained[1], trained[2], cfg.k)
        want = _experts(x.float(), ids, weights, trained[1].float(), trained[2].float())
        off = [float((v.float() - want).abs().max() / want.abs().max()) for v in
               ([out, _experts_int8(x, ids, weights, trained[1], trained[2])] if half else [out])]
    log("decoded %d tokens, largest difference %.4f of the largest output" % (decode, off[0]))
    if half:
        log("in 8-bit integers %.4f of the largest output" % off[1])
    return (losses, norms, *off)


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=4)
    parser.add_argument("--half", action="store_true", help="experts in bfloat16, decoding in 8-bit integers too")
    args = parser.parse_args()
    run(steps=args.steps, half=args.half)
