"""The residual expert block built from the operators: gradients against 64-bit autograd of the same block, and the
reweighting example.  Tolerance 2e-2 in relative L2, as for the other bf16 paths: u, z, a, y and the gradients between
the products are rounded to bf16 (2^-8 each, about eight in a chain), the hidden layer to 8 bits per group of 128."""
import importlib.util
import os

import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOL = 2e-2


def _rel(got, want):
    got, want = got.double().cpu(), want.double().cpu()
    return float((got - want).norm() / want.norm())


@pytest.mark.parametrize("gated,act,kind,gate,per_gate", [(True, "silu", "rms", "sigmoid", 1), (False, "gelu", "layer", "linear", 5)])
def test_block_gradients(gated, act, kind, gate, per_gate):
    import paper_2207_02849_b200 as bt
    from paper_2207_02849_b200.expert_block import ExpertBlock
    E, d, hidden, counts = 4, 136, 200, [50, 0, 131, 19]
    rows = sum(counts)
    g = torch.Generator().manual_seed(3)
    bias = kind == "layer"
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).cuda()  # noqa: E731
    p = {"entry": 1 + r(5 if bias else 3, d, scale=0.1), "exit": 1 + r(5 if bias else 3, d, scale=0.1),
         "up": r(E, hidden * (2 if gated else 1), d, scale=d ** -0.5).bfloat16(), "down": r(E, d, hidden, scale=hidden ** -0.5).bfloat16()}
    block = ExpertBlock(E, d, hidden, rows, act=("relu", "gelu", "silu").index(act), gated=gated, norm=ref.KINDS.index(kind),
                        gate=("none", "linear", "sigmoid").index(gate), rows_per_gate=per_gate, bias=bias)
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    offsets = torch.tensor(o, dtype=torch.int32, device="cuda")
    x, gt = r(rows, d), r(-(-rows // per_gate), d).bfloat16()
    dx_out, du_out = r(rows, d), r(rows, d).bfloat16()
    x_out, u_out, kept = block.forward(p, offsets, x, gt)
    grads = block.backward(p, offsets, kept, dx_out, du_out)
    assert bt.betty_poll_status(block.ws)[0] == bt.BETTY_OK

    leaves = {k: ref.d64(v).requires_grad_(True) for k, v in {**p, "x": x, "gate": gt}.items()}
    _, u = ref.block_norm(leaves["entry"], leaves["x"], None, None, pre=kind, post="none", act="none", per_gate=1, eps=1e-6)
    z = torch.cat([u[a:b] @ leaves["up"][e].t() for e, (a, b) in enumerate(zip(o, o[1:]))])
    h = ref.hidden(z, hidden, act, gated)
    y = torch.cat([h[a:b] @ leaves["down"][e].t() for e, (a, b) in enumerate(zip(o, o[1:]))])
    want_x, want_u = ref.block_norm(leaves["exit"], leaves["x"], y, leaves["gate"], pre=kind, post=kind, act=gate, per_gate=per_gate, eps=1e-6)
    assert _rel(x_out, want_x.detach()) < TOL and _rel(u_out, want_u.detach()) < TOL
    want = torch.autograd.grad((want_x * ref.d64(dx_out)).sum() + (want_u * ref.d64(du_out)).sum(), list(leaves.values()))
    for k, w in zip(leaves, want):
        if float(w.norm()) == 0.0:
            continue
        assert _rel(grads[k], w) < TOL, (k, _rel(grads[k], w))


def test_block_replays_from_a_graph():
    """A captured forward and backward pass gives the bits of the direct calls."""
    from paper_2207_02849_b200.expert_block import ExpertBlock
    E, d, hidden, rows = 3, 128, 192, 90
    g = torch.Generator().manual_seed(7)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).cuda()  # noqa: E731
    p = {"entry": 1 + r(3, d, scale=0.1), "exit": 1 + r(3, d, scale=0.1), "up": r(E, 2 * hidden, d, scale=0.1).bfloat16(),
         "down": r(E, d, hidden, scale=0.1).bfloat16()}
    block = ExpertBlock(E, d, hidden, rows)
    offsets = torch.tensor([0, 31, 31, 85], dtype=torch.int32, device="cuda")
    x, dx_out = r(rows, d), r(rows, d)

    def step():
        x_out, u_out, kept = block.forward(p, offsets, x)
        return [x_out, u_out] + [v for v in block.backward(p, offsets, kept, dx_out, None).values() if v is not None]

    direct = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for t in captured:
        t.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(direct, captured):
        assert torch.equal(a, b)


def test_reweighting_example_separates_the_groups():
    spec = importlib.util.spec_from_file_location("example", os.path.join(ROOT, "examples", "reweight_expert_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    lines = []
    cost, weight = m.main(steps=60, out=lines.append)
    assert weight < 0.3, lines
