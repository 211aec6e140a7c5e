"""Which sources of a teacher's logits to trust: distillation of a small language model (a residual expert block and its head) whose rows
are weighed by the finite-difference hypergradient (arXiv 2207.02849, Sec. 3.2).

Lower problem: the student's parameters theta, trained against a teacher's top logits with the cost
    C(theta, lambda) = sum_g w_g C_g(theta),   w = softmax(lambda),   C_g = mean divergence of the rows of source g;
the teacher's logits of half of the sources belong to other rows.  Upper problem: lambda, by the cross entropy of rows with known
tokens.  The hypergradient is
    -alpha * [dC/dlambda(theta + eps v) - dC/dlambda(theta - eps v)] / (2 eps),   v = dC_upper/dtheta,  eps = eps0 / |v|,
so every iteration takes one gradient for the step, one gradient v, and two forward passes for their row losses.

    python examples/distill_expert_block.py [--steps 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2207_02849_b200 as bt  # noqa: E402
from paper_2207_02849_b200.expert_block import ExpertBlock  # noqa: E402
from paper_2207_02849_b200.language_head import LanguageHead  # noqa: E402

MATRICES = ("up", "down", "head")


def parameters(g, n_experts, d, hidden, vocab, device="cuda"):
    """fp32 master parameters: norms near one, matrices of the usual size."""
    r = lambda *s, scale: torch.randn(*s, generator=g, device=device) * scale  # noqa: E731
    return {"entry": 1.0 + r(3, d, scale=0.02), "exit": 1.0 + r(3, d, scale=0.02), "up": r(n_experts, 2 * hidden, d, scale=d ** -0.5),
            "down": r(n_experts, d, hidden, scale=hidden ** -0.5), "head": r(vocab, d, scale=2.0 * d ** -0.5)}


def operands(p, dtype):
    return {k: v.to(dtype) if k in MATRICES else v for k, v in p.items()}


class Student:
    """A block and a head: row losses, and gradients of their weighted sum."""

    def __init__(self, n_experts, d, hidden, vocab, rows, top, dtype):
        self.block, self.head, self.dtype = ExpertBlock(n_experts, d, hidden, rows, dtype), LanguageHead(vocab, d, rows, top, dtype), dtype

    def losses(self, theta, data):
        """(row losses, what `gradient` needs); data: offsets, x, and the tokens or the teacher's ids and logits."""
        p = operands(theta, self.dtype)
        _, u, kept = self.block.forward(p, data[0], data[1])
        loss, kept_head = self.head.forward(p["head"], u, data[2]) if len(data) == 3 else self.head.forward_teacher(p["head"], u, data[2], data[3])
        return loss, (p, kept, kept_head)

    def gradient(self, data, kept, weights):
        p, block, head = kept
        top = self.head.backward(p["head"], head, weights)
        grads = self.block.backward(p, data[0], block, None, top["u"])
        grads["head"] = top["w"]
        return grads


def per_source_means(values, source, rows_of):
    return torch.zeros_like(rows_of).index_add_(0, source, values) / rows_of


def hypergradient(student, theta, v, train, source, rows_of, w, eps0, alpha):
    """Of the upper cost by lambda, from the row losses at theta displaced along v, the upper cost's gradient: eps0 is the length of the
    step.  source: the rows' sources; rows_of: how many rows each has; w = softmax(lambda)."""
    eps = eps0 / torch.sqrt(sum(v[k].square().sum() for k in theta))
    moved = [{k: theta[k] + s * eps * v[k] for k in theta} for s in (1.0, -1.0)]
    costs = [per_source_means(student.losses(t, train)[0], source, rows_of) for t in moved]
    d_lam = [w * (c - (w * c).sum()) for c in costs]             # dC/dlambda of a softmax-weighted sum
    return -alpha * (d_lam[0] - d_lam[1]) / (2.0 * eps)


def main(steps=40, n_experts=4, d=256, hidden=256, vocab=2000, rows=1024, top=16, sources=8, far=0.4, lr=2.0, lr_upper=200.0, eps0=0.02, alpha=1.0,
         seed=0, out=print):
    g = torch.Generator(device="cuda").manual_seed(seed)
    student = Student(n_experts, d, hidden, vocab, rows, top, torch.bfloat16)
    teacher, theta = parameters(g, n_experts, d, hidden, vocab), parameters(g, n_experts, d, hidden, vocab)
    theta = {k: teacher[k] + far * (theta[k] - teacher[k]) for k in theta}           # a student that has seen some of what its teacher has

    def batch():
        expert = torch.randint(0, n_experts, (rows,), generator=g, device="cuda").sort()[0]
        offsets = torch.searchsorted(expert, torch.arange(n_experts + 1, device="cuda")).to(torch.int32)
        x = torch.randn(rows, d, generator=g, device="cuda")
        p = operands(teacher, student.dtype)
        _, u, _ = student.block.forward(p, offsets, x)
        return offsets, x, u.float() @ p["head"].float().t()

    offsets, x, z = batch()
    source = torch.randint(0, sources, (rows,), generator=g, device="cuda")
    mixed = source < sources // 2
    z = torch.where(mixed[:, None], z.roll(rows // 2, 0), z)
    logits, ids = z.topk(top, 1)
    train = (offsets, x, ids.to(torch.int32), logits)
    offsets, x, z = batch()
    known = (offsets, x, z.argmax(1))
    lam = torch.zeros(sources, device="cuda")
    per_source = torch.zeros(sources, device="cuda").index_add_(0, source, torch.ones(rows, device="cuda"))

    for step in range(steps):
        w = torch.softmax(lam, 0)
        _, kept = student.losses(theta, train)
        grads = student.gradient(train, kept, (w / per_source)[source])
        for k in theta:
            theta[k] -= lr * grads[k]
        loss, kept = student.losses(theta, known)
        v = student.gradient(known, kept, torch.full((rows,), 1.0 / rows, device="cuda"))
        lam -= lr_upper * hypergradient(student, theta, v, train, source, per_source, w, eps0, alpha)
        if step % 10 == 0 or step == steps - 1:
            out(f"step {step:3d}  cross entropy of known rows {float(loss.mean()):.4f}  weight of mixed-up sources {float(torch.softmax(lam, 0)[: sources // 2].sum()):.3f}")
    for ws in (student.block.ws, student.head.ws):
        assert bt.betty_poll_status(ws)[0] == bt.BETTY_OK
    return float(loss.mean()), float(torch.softmax(lam, 0)[: sources // 2].sum())


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    main(ap.parse_args().steps)
