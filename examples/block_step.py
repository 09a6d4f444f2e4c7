"""Trains a small pre-norm block of gated experts under the controller, on a HIP device:

    python examples/block_step.py [steps]

x + sum over a token's two best of eight experts of  gate * V_e (silu(G_e z) * (U_e z)),  z the
layer norm of x.  The experts' gate and up projections are one matrix, and so one recoverable unit, the
down projections another; experts in A_t run in bf16, the others in INT8.  The controller steps from
the sums of squares that backward leaves, all gradients are clipped by the global norm that its norms
and those of the router and the layer norm make, the experts' update is the orthogonalised
momentum, that of the rest plain momentum.  Synthetic data, random weights.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_00539_amd.torch_experts import ExpertUnits, OrthogonalMomentum  # noqa: E402
from paper_2606_00539_amd.torch_layers import LayerNorm  # noqa: E402

DIM, HIDDEN, EXPERTS, TOP, TOKENS = 256, 344, 8, 2, 1021


def block(x, norm, router, experts):
    """The block's output in fp32; experts(rows, offsets) is the feed-forward of rows sorted by
    expert."""
    z = norm(x)
    gate, expert = torch.topk(torch.softmax(z.float() @ router, -1), TOP)
    order = torch.argsort(expert.flatten(), stable=True)
    offsets = torch.zeros(EXPERTS + 1, dtype=torch.int32, device=x.device)
    offsets[1:] = torch.cumsum(torch.bincount(expert.flatten(), minlength=EXPERTS), 0)
    rows = order // TOP
    y = experts(z[rows], offsets).float() * gate.flatten()[order][:, None]
    return x.float().index_add(0, rows, y)


def train(steps=30, seed=0, log=print):
    """Runs `steps` steps; returns the losses, the global norms and each step's recovery set."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    def weights(scale):
        return (normal(EXPERTS, 2 * HIDDEN, DIM, scale=scale * DIM ** -0.5).to(torch.bfloat16),
                normal(EXPERTS, DIM, HIDDEN, scale=scale * HIDDEN ** -0.5).to(torch.bfloat16))
    target = ExpertUnits(zip(("up", "down"), weights(2.0)), low_cost=False)
    units = ExpertUnits(zip(("up", "down"), map(torch.nn.Parameter, weights(0.5))), max_o=3,
                        lock_len=2)
    norm, router = LayerNorm(DIM), torch.nn.Parameter(normal(DIM, EXPERTS, scale=DIM ** -0.5))
    fixed_norm, fixed_router = LayerNorm(DIM), router.detach().clone()
    rest = [*norm.parameters(), router]
    opt = OrthogonalMomentum(units, lr=0.02, momentum=0.9)
    other = torch.optim.SGD(rest, lr=0.05, momentum=0.9)
    losses, norms, sets = [], [], []
    for t in range(1, steps + 1):
        x = normal(TOKENS, DIM, scale=1.0).to(torch.bfloat16)
        with torch.no_grad():
            want = block(x, fixed_norm, fixed_router,
                         lambda r, o: target.feed_forward("up", "down", r, o))
        out = block(x, norm, router, lambda r, o: units.feed_forward("up", "down", r, o))
        loss = (out - want).square().mean()
        loss.backward()
        n = units.step_clipped(1.5 if t == 1 else 1.1, 1.5, max_norm=0.5,
                               others=[p.grad for p in rest])
        opt.step()
        other.step()
        other.zero_grad()
        losses.append(float(loss.detach()))
        norms.append(float(n))
        sets.append(units.recovery_set())
        if log is not None:
            log(f"step {t:3d}  loss {losses[-1]:8.4f}  norm {norms[-1]:8.4f}  recovering "
                f"{', '.join(sets[-1]) or '-'}")
    units.close()
    target.close()
    return losses, norms, sets


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 30)
