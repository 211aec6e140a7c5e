"""A residual expert block and its head as they are trained together: gradients of weighted row losses against 64-bit autograd of the same
network, captured steps, and the example.  Tolerance 2e-2 in relative L2, as for the block alone: about nine roundings to bf16 (2^-8)
in a chain, the hidden layer to 8 bits per group of 128."""
import importlib.util
import os

import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOL = 2e-2
E, D, HIDDEN, VOCAB, COUNTS = 3, 136, 200, 1003, [70, 0, 113]
ROWS = sum(COUNTS)
EPS = 1e-6


def _rel(got, want):
    got, want = got.double().cpu(), want.double().cpu()
    return float((got - want).norm() / want.norm())


def _setup():
    from paper_2207_02849_b200.expert_block import ExpertBlock
    from paper_2207_02849_b200.language_head import LanguageHead
    g = torch.Generator().manual_seed(3)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).cuda()  # noqa: E731
    p = {"entry": 1 + r(3, D, scale=0.1), "exit": 1 + r(3, D, scale=0.1), "up": r(E, 2 * HIDDEN, D, scale=D ** -0.5).bfloat16(),
         "down": r(E, D, HIDDEN, scale=HIDDEN ** -0.5).bfloat16()}
    w = r(VOCAB, D, scale=2 * D ** -0.5).bfloat16()
    o = [0]
    for c in COUNTS:
        o.append(o[-1] + c)
    target = torch.randint(VOCAB, (ROWS,), generator=g)
    target[::7] = -100
    ids = torch.randint(VOCAB, (ROWS, 12), generator=g)
    ids[::5, 3:] = -1
    return (ExpertBlock(E, D, HIDDEN, ROWS), LanguageHead(VOCAB, D, ROWS, 12, temperature=2.0, smoothing=0.1, z_loss=1e-3), p, w, o,
            torch.tensor(o, dtype=torch.int32, device="cuda"), r(ROWS, D), target.cuda(), ids.cuda(), r(ROWS, 12, scale=3.0), torch.rand(ROWS, generator=g).cuda())


@pytest.mark.parametrize("distill", [False, True])
def test_gradients_through_block_and_head(distill):
    import paper_2207_02849_b200 as bt
    block, head, p, w, o, offsets, x, target, ids, logits, weights = _setup()
    _, u, kept = block.forward(p, offsets, x)
    loss, kept_head = head.forward_teacher(w, u, ids, logits) if distill else head.forward(w, u, target)
    top = head.backward(w, kept_head, weights)
    grads = block.backward(p, offsets, kept, None, top["u"])
    assert bt.betty_poll_status(block.ws)[0] == bt.betty_poll_status(head.ws)[0] == bt.BETTY_OK

    leaves = {k: ref.d64(v).requires_grad_(True) for k, v in {**p, "x": x, "head": w}.items()}
    _, h = ref.block_norm(leaves["entry"], leaves["x"], None, None, pre="rms", post="none", act="none", per_gate=1, eps=EPS)
    z = torch.cat([h[a:b] @ leaves["up"][e].t() for e, (a, b) in enumerate(zip(o, o[1:]))])
    a_ = ref.hidden(z, HIDDEN, "silu", True)
    y = torch.cat([a_[a:b] @ leaves["down"][e].t() for e, (a, b) in enumerate(zip(o, o[1:]))])
    _, v = ref.block_norm(leaves["exit"], leaves["x"], y, None, pre="rms", post="rms", act="none", per_gate=1, eps=EPS)
    z = v @ leaves["head"].t()
    if distill:
        i, held = ids.cpu().clamp(min=0), ids.cpu() >= 0
        logp = torch.log_softmax(torch.where(held, logits.double().cpu() / 2.0, -1e300), 1)
        want = torch.where(held, logp.exp() * (logp - torch.log_softmax(z / 2.0, 1).gather(1, i)), 0.0).sum(1)
    else:
        want = torch.nn.functional.cross_entropy(z, target.cpu(), ignore_index=-100, reduction="none", label_smoothing=0.1)
        want = want + 1e-3 * torch.logsumexp(z, 1) ** 2 * (target.cpu() >= 0)
    assert _rel(loss, want.detach()) < TOL
    gs = torch.autograd.grad((want * ref.d64(weights)).sum(), list(leaves.values()))
    got = {**grads, "head": top["w"]}
    for k, g in zip(leaves, gs):
        assert _rel(got[k], g) < TOL, (k, _rel(got[k], g))


def test_a_training_step_replays_from_a_graph():
    block, head, p, w, o, offsets, x, target, ids, logits, weights = _setup()

    def step():
        _, u, kept = block.forward(p, offsets, x)
        loss, a = head.forward(w, u, target)
        kd, b = head.forward_teacher(w, u, ids, logits)
        g1, g2 = head.backward(w, a, weights), head.backward(w, b, weights, wants=("u",))
        return [loss, kd, g1["w"], *[v for v in block.backward(p, offsets, kept, None, g1["u"] + g2["u"]).values() if v is not None]]

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_too_many_entries_are_refused():
    _, head, _, w, _, _, x, _, _, _, _ = _setup()
    ids = torch.zeros(ROWS, 13, dtype=torch.long, device="cuda")
    with pytest.raises(ValueError, match="12 entries"):
        head.forward_teacher(w, x.bfloat16(), ids, ids.float())


def test_example_runs():
    spec = importlib.util.spec_from_file_location("distill_expert_block", os.path.join(ROOT, "examples", "distill_expert_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lines = []
    loss, share = example.main(steps=4, rows=300, vocab=501, out=lines.append)
    assert len(lines) == 2 and 0.0 <= share <= 1.0 and loss == loss
