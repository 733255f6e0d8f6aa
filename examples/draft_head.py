"""Trains a draft head by the library's supervised losses, as before the EM step.

A synthetic target model (its own LM head over random hidden states) stands in
for the model to be drafted for.  The draft head, an LM-head weight and a shift
of its hidden states, learns in three stages:

  labels    cross entropy of the target's greedy tokens (lmhead_cross_entropy),
            prompt positions ignored;
  teacher   the target's stored top logits (lmhead_distill), rows weighted by
            their depth; logits are never kept in either stage;
  logits    the same loss on the draft logits that the EM step reads
            (lmhead_logits, then topk_distill), written over with their gradient.

Run: python examples/draft_head.py [--rows R --vocab V --hidden H --steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_05774_gb300 import vsd  # noqa: E402


def train(rows=512, vocab=4096, hidden=256, topk=16, steps=30, temperature=2.0, seed=0,
          device="cuda", log=print):
    """Returns the first and last loss of each stage, by name."""
    g = torch.Generator(device=device).manual_seed(seed)
    f = dict(generator=g, device=device)
    h = torch.randn(rows, hidden, **f).to(torch.bfloat16)
    target = (torch.randn(vocab, hidden, **f) * (2.0 / hidden ** 0.5)).to(torch.bfloat16)
    top = vsd.lmhead_logits(h, target).float().topk(topk, dim=1)
    ids, teacher = top.indices.to(torch.int32), top.values.to(torch.bfloat16)
    labels = ids[:, 0].clone()
    labels[: rows // 4] = -100  # the prompt
    depth_weight = 1.05 ** (1.0 + torch.arange(rows, device=device) % 8).float()

    weight = (0.02 * torch.randn(vocab, hidden, **f)).to(torch.bfloat16)
    master = weight.float()                      # the optimizer's copy
    shift = torch.zeros(rows, hidden, device=device)  # the draft's own part of the hidden states
    ws = torch.empty(vsd.lmhead_loss_workspace_bytes(rows, vocab, hidden, topk),
                     dtype=torch.uint8, device=device)
    result = {}

    def stage(name, lr, step):
        losses = []
        for _ in range(steps):
            x = (h.float() + shift).to(torch.bfloat16)
            out = step(x)
            losses.append(out["loss"])
            master.add_(out["d_weight"].float(), alpha=-lr * rows)
            shift.add_(out["d_hidden"].float(), alpha=-lr * rows)
            weight.copy_(master)
        losses = torch.cat(losses).tolist()
        result[name] = (losses[0], losses[-1])
        log("%-8s loss %.4f -> %.4f" % (name, *result[name]))

    stage("labels", 0.02, lambda x: vsd.lmhead_cross_entropy(x, weight, labels, workspace=ws))
    stage("teacher", 0.02, lambda x: vsd.lmhead_distill(
        x, weight, ids, teacher, T=temperature, row_weight=depth_weight,
        grad_scale=temperature ** 2, workspace=ws))
    code, bits = vsd.device_status(ws)
    if code != 0:
        raise RuntimeError("device status %d bits %d" % (code, bits))

    def on_logits(x):
        logits = vsd.lmhead_logits(x, weight)
        out = vsd.topk_distill(logits, ids, teacher, T=temperature, row_weight=depth_weight,
                               grad_scale=temperature ** 2, grad=logits)
        out["d_hidden"] = out["grad"] @ weight
        out["d_weight"] = out["grad"].t() @ x
        return out

    stage("logits", 0.02, on_logits)
    return result


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    train(a.rows, a.vocab, a.hidden, steps=a.steps)


if __name__ == "__main__":
    main()
