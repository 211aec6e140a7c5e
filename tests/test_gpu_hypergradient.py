"""The finite-difference hypergradient of the distillation example against a 64-bit restatement of the same differences."""
import importlib.util
import os

import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOL = 2e-2          # relative L2 of the row losses of a block and a head in bf16, as in the tests of their gradients
E, D, HIDDEN, VOCAB, ROWS, TOP, SOURCES = 2, 64, 48, 200, 300, 8, 4


def _example():
    spec = importlib.util.spec_from_file_location("distill_expert_block", os.path.join(ROOT, "examples", "distill_expert_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _row_losses(p, offsets, x, ids, logits):
    """Divergence of each row from the teacher's logits, in 64 bits at the operands p."""
    p, x = {k: ref.d64(v) for k, v in p.items()}, ref.d64(x)
    spans = list(zip(offsets, offsets[1:]))
    _, h = ref.block_norm(p["entry"], x, None, None, pre="rms", post="none", act="none", per_gate=1, eps=1e-6)
    a = ref.hidden(torch.cat([h[i:j] @ p["up"][e].t() for e, (i, j) in enumerate(spans)]), HIDDEN, "silu", True)
    y = torch.cat([a[i:j] @ p["down"][e].t() for e, (i, j) in enumerate(spans)])
    _, u = ref.block_norm(p["exit"], x, y, None, pre="rms", post="rms", act="none", per_gate=1, eps=1e-6)
    logp = torch.log_softmax(ref.d64(logits), 1)
    return (logp.exp() * (logp - torch.log_softmax(u @ p["head"].t(), 1).gather(1, ids.cpu().long()))).sum(1)


@pytest.mark.parametrize("own", [0, 2])
@pytest.mark.parametrize("eps0", [0.5, 2.0])
def test_the_hypergradient_of_the_sources(own, eps0):
    """v is the gradient of one source's cost, so that this source's weight gets a gradient far below the others'.  Row losses that are TOL
    off in relative L2 put a mean over n of them off by TOL |l| / sqrt(n), a softmax-weighted difference by twice that, times its
    weight, at each of the two points."""
    m = _example()
    g = torch.Generator(device="cuda").manual_seed(own)
    student = m.Student(E, D, HIDDEN, VOCAB, ROWS, TOP, torch.bfloat16)
    theta = m.parameters(g, E, D, HIDDEN, VOCAB)
    o = [0, 130, ROWS]
    offsets = torch.tensor(o, dtype=torch.int32, device="cuda")
    x, logits = torch.randn(ROWS, D, generator=g, device="cuda"), 2 * torch.randn(ROWS, TOP, generator=g, device="cuda")
    ids = torch.randint(VOCAB, (ROWS, TOP), generator=g, device="cuda", dtype=torch.int32)
    source = torch.arange(ROWS, device="cuda") % SOURCES
    rows_of = torch.full((SOURCES,), ROWS / SOURCES, device="cuda")
    w = torch.softmax(torch.randn(SOURCES, generator=g, device="cuda"), 0)
    train = (offsets, x, ids, logits)
    _, kept = student.losses(theta, train)
    v = student.gradient(train, kept, (source == own).float() * SOURCES / ROWS)
    alpha = 0.7
    got = m.hypergradient(student, theta, v, train, source, rows_of, w, eps0, alpha).double().cpu()

    norm = float(torch.sqrt(sum(v[k].double().square().sum() for k in theta)))
    eps, w = eps0 / norm, w.double().cpu()
    d_lam, off = [], torch.zeros(SOURCES, dtype=torch.float64)
    for s in (1.0, -1.0):
        loss = _row_losses(m.operands({k: (theta[k].double() + s * eps * v[k].double()).float() for k in theta}, student.dtype), o, x, ids, logits)
        c = torch.zeros(SOURCES, dtype=torch.float64).index_add_(0, source.cpu(), loss) * SOURCES / ROWS
        d_lam.append(w * (c - (w * c).sum()))
        off += 2 * w * TOL * loss.norm() / (ROWS / SOURCES) ** 0.5
    want, off = -alpha * (d_lam[0] - d_lam[1]) / (2 * eps), alpha * off / (2 * eps)
    assert float(want[own]) < 0.0 and bool((want[torch.arange(SOURCES) != own] > 0).all())
    assert bool(((got - want).abs() <= off).all()), (got, want, off)
    # the longer step leaves the tolerance less than half of the values: a wrong sign, source or a factor of two shows
    assert eps0 < 1.0 or float(off[own]) < 0.5 * abs(float(want[own]))
