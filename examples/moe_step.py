"""Trains a small mixture-of-experts block under the controller, on a HIP device:

    python examples/moe_step.py [steps]

Tokens go to their two best experts of eight; each expert is W2 silu(W1 x).  Both
matrices of every expert are recoverable units: experts in A_t run in bf16, the others
in INT8; backward writes their gradients and the sums of squares that the controller
steps from; their update is the orthogonalised momentum.  The target is another
block's output, and one expert's data turn noisy halfway, which its unit's norm shows.
Synthetic data, random weights.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_00539_amd.torch_experts import ExpertUnits, OrthogonalMomentum  # noqa: E402

DIM, HIDDEN, EXPERTS, TOP, TOKENS = 256, 688, 8, 2, 1021


def route(x, router):
    """(rows, gate, offsets): the token of each row, sorted by expert, its weight, and the
    experts' boundaries, all on the device."""
    gate, expert = torch.topk(torch.softmax(x.float() @ router, -1), TOP)
    order = torch.argsort(expert.flatten(), stable=True)
    ends = torch.cumsum(torch.bincount(expert.flatten(), minlength=EXPERTS), 0)
    offsets = torch.zeros(EXPERTS + 1, dtype=torch.int32, device=x.device)
    offsets[1:] = ends
    return order // TOP, gate.flatten()[order], offsets


def block(x, router, up, down):
    """The block's output; up and down take (rows, offsets)."""
    rows, gate, offsets = route(x, router)
    h = torch.nn.functional.silu(up(x[rows], offsets))
    y = down(h, offsets).float() * gate[:, None]
    return torch.zeros(x.shape, dtype=torch.float32, device=x.device).index_add(0, rows, y)


def weights(g, scale):
    def make(o, i):
        return (torch.randn(EXPERTS, o, i, generator=g, device="cuda") * scale * i ** -0.5
                ).to(torch.bfloat16)
    return make(HIDDEN, DIM), make(DIM, HIDDEN)


def train(steps=40, seed=0, log=print):
    """Runs `steps` steps; returns the losses and each step's recovery set."""
    from paper_2606_00539_amd.torch_ops import grouped_linear

    g = torch.Generator(device="cuda").manual_seed(seed)
    router = torch.randn(DIM, EXPERTS, generator=g, device="cuda") * DIM ** -0.5
    teacher = weights(g, 1.0)
    student = [torch.nn.Parameter(w) for w in weights(g, 0.3)]
    units = ExpertUnits(zip(("up", "down"), student), max_o=3, lock_len=2)
    opt = OrthogonalMomentum(units, lr=0.02, momentum=0.9)
    losses, sets = [], []
    for t in range(1, steps + 1):
        units_step = 0.0
        for _ in range(2):      # two micro-batches
            x = torch.randn(TOKENS, DIM, generator=g, device="cuda").to(torch.bfloat16)
            with torch.no_grad():
                want = block(x, router, *(lambda r, o, w=w: grouped_linear(r, w, o)
                                          for w in teacher))
                if t == steps // 2:
                    noisy = torch.topk(x.float() @ router, 1).indices[:, 0] == 0
                    want = want + 20.0 * noisy[:, None] * torch.randn(
                        want.shape, generator=g, device="cuda")
            out = block(x, router, lambda r, o: units.linear("up", r, o),
                        lambda r, o: units.linear("down", r, o))
            loss = (out - want).square().mean()
            loss.backward()
            units_step += float(loss.detach()) / 2
        units.step(1.5 if t == 1 else 1.1, 1.5)
        opt.step()
        losses.append(units_step)
        sets.append(units.recovery_set())
        if log is not None:
            log(f"step {t:3d}  loss {losses[-1]:8.4f}  recovering {', '.join(sets[-1]) or '-'}")
    units.close()
    return losses, sets


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
