"""Data reweighting of a residual expert block by the finite-difference hypergradient (arXiv 2207.02849, Sec. 3.2).

Lower problem: the block's parameters theta, trained on groups of rows with the cost
    C(theta, lambda) = sum_g w_g C_g(theta),   w = softmax(lambda),   C_g = mean square error of x' on group g;
half of the groups have corrupted targets.  Upper problem: lambda, on a clean batch.  The hypergradient is
    -alpha * [dC/dlambda(theta + eps v) - dC/dlambda(theta - eps v)] / (2 eps),   v = dC_clean/dtheta,  eps = eps0 / |v|,
so every iteration takes one gradient for the step, one gradient v on the clean batch, and two forward passes.

    python examples/reweight_expert_block.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2207_02849_b200 as bt  # noqa: E402
from paper_2207_02849_b200.expert_block import ExpertBlock  # noqa: E402

MATRICES = ("up", "down")


def parameters(g, n_experts, d, hidden, device="cuda"):
    """fp32 master parameters: norms near one, matrices of the usual size."""
    r = lambda *s, scale: torch.randn(*s, generator=g, device=device) * scale  # noqa: E731
    p = {"entry": 1.0 + r(3, d, scale=0.02), "exit": 1.0 + r(3, d, scale=0.02), "up": r(n_experts, 2 * hidden, d, scale=d ** -0.5),
         "down": r(n_experts, d, hidden, scale=hidden ** -0.5)}
    p["exit"][2] *= 0.5
    return p


def operands(p, dtype):
    return {k: v.to(dtype) if k in MATRICES else v for k, v in p.items()}


def batch(g, teacher, block, d, dtype, device="cuda"):
    """Rows sorted by expert, the teacher's outputs, and the experts' offsets."""
    n = block.rows
    expert = torch.randint(0, block.up.n_groups, (n,), generator=g, device=device).sort()[0]
    offsets = torch.searchsorted(expert, torch.arange(block.up.n_groups + 1, device=device)).to(torch.int32)
    x = torch.randn(n, d, generator=g, device=device)
    target, _, _ = block.forward(operands(teacher, dtype), offsets, x, next_norm=False)
    return offsets, x, target.clone()


def main(steps=60, n_experts=4, d=256, hidden=256, rows=1024, groups=8, lr=1.0, lr_upper=200.0, eps0=0.05, alpha=1.0, seed=0, out=print):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16
    block = ExpertBlock(n_experts, d, hidden, rows, dtype)
    teacher, theta = parameters(g, n_experts, d, hidden), parameters(g, n_experts, d, hidden)
    train, clean = batch(g, teacher, block, d, dtype), batch(g, teacher, block, d, dtype)
    group = torch.randint(0, groups, (rows,), generator=g, device="cuda")
    corrupted = group < groups // 2
    train = (train[0], train[1], torch.where(corrupted[:, None], torch.randn(rows, d, generator=g, device="cuda") * 2.0, train[2]))
    lam = torch.zeros(groups, device="cuda")
    per_group = torch.zeros(groups, device="cuda").index_add_(0, group, torch.ones(rows, device="cuda"))

    def residual(theta, data):
        x_out, _, kept = block.forward(operands(theta, dtype), data[0], data[1], next_norm=False)
        return x_out - data[2], kept

    def group_costs(theta):
        r, _ = residual(theta, train)
        return torch.zeros(groups, device="cuda").index_add_(0, group, r.square().mean(1)) / per_group

    def gradient(theta, data, row_weight):
        """dC/dtheta of sum_i row_weight_i mean_j r_ij^2."""
        r, kept = residual(theta, data)
        return block.backward(operands(theta, dtype), data[0], kept, r * (2.0 / d) * row_weight[:, None], None), r

    keys = ("entry", "exit", "up", "down")
    for step in range(steps):
        w = torch.softmax(lam, 0)
        grads, _ = gradient(theta, train, (w / per_group)[group])
        for k in keys:
            theta[k] -= lr * grads[k]
        v, r = gradient(theta, clean, torch.full((rows,), 1.0 / rows, device="cuda"))
        norm = torch.sqrt(sum(v[k].square().sum() for k in keys))
        eps = eps0 / norm
        moved = [{k: theta[k] + s * eps * v[k] for k in keys} for s in (1.0, -1.0)]
        costs = [group_costs(t) for t in moved]
        d_lam = [w * (c - (w * c).sum()) for c in costs]             # dC/dlambda of a softmax-weighted sum
        lam -= lr_upper * (-alpha * (d_lam[0] - d_lam[1]) / (2.0 * eps))
        if step % 20 == 0 or step == steps - 1:
            out(f"step {step:3d}  clean cost {float(r.square().mean()):.4f}  weight of corrupted groups {float(torch.softmax(lam, 0)[: groups // 2].sum()):.3f}")
    st, _ = bt.betty_poll_status(block.ws)
    assert st == bt.BETTY_OK
    return float(r.square().mean()), float(torch.softmax(lam, 0)[: groups // 2].sum())


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    main(ap.parse_args().steps)
