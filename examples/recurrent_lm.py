"""A recurrent language model trained with compressed gradients on one GPU.

The model (``paper_2108_06004_amd.lm.RecurrentLM``) runs the gated linear recurrence, dropout and the
cross-entropy of this library; the gradients of P simulated workers, each on its own sequences, go through one
compression step per iteration (``GlobalSketchOptimizer``): momentum and error accumulation, sketches, their merge,
the top k coordinates, their exact values, the weight update. Afterwards the model continues a
prompt token by token, with the recurrence's state carried from call to call.

The text is synthetic: a fixed random successor for each token, followed nine times in ten.

    python examples/recurrent_lm.py [--steps 60] [--vocab 500] [--width 128] [--layers 2]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synth  # noqa: E402
from paper_2108_06004_amd.lm import RecurrentLM  # noqa: E402
from paper_2108_06004_amd.train import DensitySchedule, GlobalSketchOptimizer  # noqa: E402


def text(successor, batch: int, length: int, gen):
    """[batch][length] tokens: the successor of the token before, or one time in ten any token."""
    vocab = successor.numel()
    out = torch.empty((batch, length), dtype=torch.int64, device=successor.device)
    out[:, 0] = torch.randint(vocab, (batch,), generator=gen, device=successor.device)
    for t in range(1, length):
        any_token = torch.randint(vocab, (batch,), generator=gen, device=successor.device)
        stray = torch.rand(batch, generator=gen, device=successor.device) < 0.1
        out[:, t] = torch.where(stray, any_token, successor[out[:, t - 1]])
    return out


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--vocab", type=int, default=500)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=16, help="sequences of each worker")
    ap.add_argument("--length", type=int, default=48, help="tokens of a sequence")
    ap.add_argument("--lr", type=float, default=4.0)
    ap.add_argument("--density", type=float, default=0.05, help="share of the coordinates updated each step")
    ap.add_argument("--dtype", choices=("float32", "bfloat16"), default="float32")
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    torch.manual_seed(1)
    gen = torch.Generator(device=dev).manual_seed(2)
    successor = torch.randperm(a.vocab, generator=gen, device=dev)
    model = RecurrentLM(a.vocab, a.width, a.layers, p=0.1, seed=3, dtype=getattr(torch, a.dtype)).to(dev)
    d = sum(p.numel() for p in model.parameters())
    opt = GlobalSketchOptimizer(model.parameters(), a.workers, 5, max(64, d // 10), synth.hash_params(4, 5),
                                DensitySchedule(a.density, a.lr), rho=0.5)
    losses = []
    for step in range(a.steps):
        model.step.fill_(step)  # this step's dropout masks
        total = torch.zeros((), device=dev)
        for worker in range(a.workers):
            model.worker = worker
            tokens = text(successor, a.batch, a.length + 1, gen)
            total += model.loss_backward(tokens[:, :-1], tokens[:, 1:])
            opt.collect(worker)
        opt.step()
        losses.append(total / a.workers)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {float(losses[-1]):.4f}, {opt.last_k} of {d} coordinates updated", flush=True)
    prompt = text(successor, 4, 8, gen)
    said = model.generate(prompt, 12)
    want = [prompt[:, -1]]
    for _ in range(12):
        want.append(successor[want[-1]])
    right = float((said == torch.stack(want[1:], 1)).float().mean())
    print(f"continued 4 prompts by 12 tokens: {100 * right:.0f}% of them the successors", flush=True)
    opt.close()
    return {"first": float(losses[0]), "last": float(losses[-1]), "right": right}


if __name__ == "__main__":
    main()
