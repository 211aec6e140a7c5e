"""Two expert blocks in a row: the second takes the normed input that the first has made."""
import pytest
import torch

from tests import block_reference as ref
from tests.test_gpu_expert_block import TOL, _rel

pytestmark = pytest.mark.gpu


def _chain(kind, gate):
    from paper_2207_02849_b200.expert_block import ExpertBlock
    E, d, hidden, counts = 3, 136, 120, [40, 0, 77]
    rows, bias = sum(counts), kind == "layer"
    g = torch.Generator().manual_seed(8)
    r = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).cuda()  # noqa: E731
    n = 5 if bias else 3
    p = [{"entry": 1 + r(n, d, scale=0.1), "exit": 1 + r(n, d, scale=0.1), "up": r(E, 2 * hidden, d, scale=d ** -0.5).bfloat16(),
          "down": r(E, d, hidden, scale=hidden ** -0.5).bfloat16()} for _ in range(2)]
    p[1]["entry"] = p[0]["exit"].clone()              # the second block's entry norm is the first one's exit w_pre (and b_pre)
    block = ExpertBlock(E, d, hidden, rows, norm=ref.KINDS.index(kind), gate=("none", "linear", "sigmoid").index(gate), rows_per_gate=4, bias=bias)
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    x, gt, dx_out = r(rows, d), r(-(-rows // 4), d).bfloat16(), r(rows, d)
    return block, p, o, torch.tensor(o, dtype=torch.int32, device="cuda"), x, gt if gate != "none" else None, dx_out


@pytest.mark.parametrize("kind,gate", [("rms", "none"), ("layer", "sigmoid")])
def test_the_second_block_takes_the_first_ones_norm(kind, gate):
    import paper_2207_02849_b200 as bt
    block, p, o, offsets, x, gt, dx_out = _chain(kind, gate)
    x1, u1, kept1 = block.forward(p[0], offsets, x, gt)
    before = bt.betty_kernel_launches()
    x2, u2, kept2 = block.forward(p[1], offsets, x1, gt, u=u1, next_norm=False)
    launches = bt.betty_kernel_launches() - before
    before = bt.betty_kernel_launches()
    own, _, _ = block.forward(p[1], offsets, x1, gt)
    assert bt.betty_kernel_launches() - before == launches + 1 and u2 is None
    assert torch.equal(own, x2)                       # an fp32 stream is not rounded: the same u, bit for bit
    g2 = block.backward(p[1], offsets, kept2, dx_out, None)
    assert "entry" not in g2
    g1 = block.backward(p[0], offsets, kept1, g2["x"], g2["u"])
    assert bt.betty_poll_status(block.ws)[0] == bt.BETTY_OK

    leaf = lambda t: ref.d64(t).requires_grad_(True)  # noqa: E731
    w = [{k: leaf(v) for k, v in q.items()} for q in p]
    lx, lg = leaf(x), leaf(gt) if gt is not None else None
    stream, u = lx, ref.block_norm(w[0]["entry"], lx, None, None, pre=kind, post="none", act="none", per_gate=1, eps=1e-6)[1]
    for q in w:
        z = torch.cat([u[a:b] @ q["up"][e].t() for e, (a, b) in enumerate(zip(o, o[1:]))])
        h = ref.hidden(z, block.hidden, "silu", True)
        y = torch.cat([h[a:b] @ q["down"][e].t() for e, (a, b) in enumerate(zip(o, o[1:]))])
        stream, u = ref.block_norm(q["exit"], stream, y, lg, pre=kind, post=kind, act=gate, per_gate=4, eps=1e-6)
    assert _rel(x2, stream.detach()) < TOL
    names = [(g1, 0, k) for k in ("entry", "exit", "up", "down")] + [(g2, 1, k) for k in ("exit", "up", "down")]
    want = torch.autograd.grad((stream * ref.d64(dx_out)).sum(), [lx] + [w[i][k] for _, i, k in names])
    # twice the single block's roundings lie between the ends of the chain
    assert _rel(g1["x"], want[0]) < 2 * TOL
    for (g, i, k), v in zip(names, want[1:]):
        assert _rel(g[k], v) < 2 * TOL, (i, k, _rel(g[k], v))
