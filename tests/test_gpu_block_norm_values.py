"""Block norm at the ends of its ranges: calls without rows, rows of very large and very small values, gates where they saturate."""
import pytest
import torch

from tests import block_reference as ref
from tests.test_gpu_block_norm import SLACK, _cfg, _check_backward, _check_forward, _gradients, _problem, _wide

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def test_no_rows_and_no_gate_rows():
    """A call without rows has gates without rows, whatever addresses come with them: none is read, and the parameter gradients
    are zeros."""
    import paper_2207_02849_b200 as bt
    cfg = bt.BlockNorm(256, gate=bt.GATE_SIGMOID, rows_per_gate=4)
    params, dparams = torch.ones(3, 256, device="cuda"), torch.full((3, 256), float("nan"), device="cuda")
    y = torch.ones(1, 256, dtype=BF, device="cuda")                  # an address for the block's output; its gate has none
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 0))
    args = [y.data_ptr(), 256, None, 0] + [y.data_ptr(), 256] * 4 + [None, 0]
    status = bt.lib().betty_block_norm_backward(cfg._ref(BF, BF), params.data_ptr(), 0, y.data_ptr(), 256, *args, dparams.data_ptr(), ws.ptr, ws.nbytes,
                                                torch.cuda.current_stream().cuda_stream)
    assert status == bt.BETTY_OK and bt.betty_poll_status(ws)[0] == bt.BETTY_OK
    assert float(dparams.abs().max()) == 0.0 and float((y - 1).abs().max()) == 0.0


@pytest.mark.parametrize("size", [1e-17, 1e-13, 1e13, 1e17])
@pytest.mark.parametrize("which", ["x", "y"])
@pytest.mark.parametrize("kind,act", [("rms", "none"), ("rms", "linear"), ("layer", "none")])
@pytest.mark.parametrize("d", [256, 515])
def test_rows_of_any_size(size, which, kind, act, d):
    """A norm takes out its row's size: with eps = 0 the gradients of rows scaled by c are those of the rows divided by c.  What
    is added to them from elsewhere has the same size here, so that the same tolerances hold: every intermediate result is in
    range as long as the squares of the row are (1e-19 to 1e19)."""
    import paper_2207_02849_b200 as bt
    q = _problem(17, 12, d, F, F, act, 1, False)
    q[which] *= size
    if which == "x":
        q["dxo"] *= 1.0 / size
        q["y"] *= size                                # keeps u's own input at one size; eps is 0
    args = (d, kind, kind, act, 1, False, 0.0)
    cfg = _cfg(bt, *args)
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 12))
    dx, dy, dp = torch.empty_like(q["x"]), torch.empty_like(q["y"]), torch.empty_like(q["params"])
    dg = torch.empty_like(q["gate"]) if act != "none" else None
    bt.betty_block_norm_backward(cfg, q["params"], q["x"], q["y"], q["gate"], q["du"], q["dxo"], dx, dy, dg, dp, ws)
    want = _gradients(q, args)
    rms = lambda t: t.pow(2).mean(-1, keepdim=True).sqrt()  # noqa: E731
    n = rms(ref.d64(q["x"]) - (ref.d64(q["x"]).mean(1, keepdim=True) if kind == "layer" else 0.0))
    m = rms(ref.d64(q["y"]) - (ref.d64(q["y"]).mean(1, keepdim=True) if kind == "layer" else 0.0))
    p = ref.d64(q["params"]).abs().amax(1)
    big = rms(want["dx"]) + rms(ref.d64(q["dxo"])) + p[0] * rms(ref.d64(q["du"])) / n      # the terms that make dX
    amp = float(p[1] * p[2]) * (4.0 if act == "linear" else 1.0)
    assert float(((dx.double().cpu() - want["dx"]).abs() / big).max()) <= SLACK
    assert float(((dy.double().cpu() - want["dy"]).abs() / (rms(want["dy"]) + amp * big / m)).max()) <= SLACK
    if dg is not None:
        assert float(((dg.double().cpu() - want["dgate"]).abs() / (4.0 * amp * big)).max()) <= SLACK


@pytest.mark.parametrize("rows", [1, 9, 300, 3000])
@pytest.mark.parametrize("d,per_gate", [(96, 3), (515, 2), (515, 40), (1538, 3), (1540, 2), (2048, 2), (2048, 11), (2048, 700)])
def test_gate_sums_stay_in_the_workspace(rows, d, per_gate):
    """A workspace of exactly the size that contiguous matrices need: the gradients of the call with room for every layout, bit
    for bit, and nothing written behind it."""
    import paper_2207_02849_b200 as bt
    args = (d, "rms", "rms", "sigmoid", per_gate, False, 1e-5)
    q, cfg = _problem(rows + d, rows, d, F, BF, "sigmoid", per_gate, False), _cfg(bt, *args)
    need = bt.betty_block_norm_workspace_size(cfg, rows, any_layout=False)
    exact, room = bt.Workspace.of_bytes(need + 4096), bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, rows))
    exact.nbytes = need
    behind = exact.buf[need + exact.ptr - exact.buf.data_ptr():]
    behind.fill_(77)
    runs = []
    for ws in (exact, room):
        outs = [torch.full_like(q[k], float("nan")) for k in ("x", "y", "gate", "params")]
        bt.betty_block_norm_backward(cfg, q["params"], q["x"], q["y"], q["gate"], q["du"], q["dxo"], *outs, ws)
        runs.append(outs)
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    assert bool((behind == 77).all())
    want = _gradients(q, args)
    for got, k, t in zip(runs[0][:3], ("dx", "dy", "dgate"), (F, BF, BF)):
        scale = want[k].pow(2).mean(-1, keepdim=True).sqrt() + 30.0 * min(rows, per_gate)
        assert ref.close(got, want[k], t, SLACK, scale=scale) <= 0, k


@pytest.mark.parametrize("tx,ty", [(F, F), (F, BF)])
def test_sigmoid_gate_of_fp32_results_is_exact_in_relative_terms(tx, ty):
    """x' = a(g) with x = 0, y = 1, s = w_post = 1 and no norm.  From e = exp(-|g|): ex2 within 2^-22, the reciprocal and three
    roundings: below 8e-7 of the result; infinite gates are shut or open."""
    import paper_2207_02849_b200 as bt
    d = 512
    gate = torch.linspace(-80, 80, 40 * d).view(40, d).to(ty).cuda()
    gate[0, 0], gate[0, 1] = -float("inf"), float("inf")
    params = torch.ones(3, d, device="cuda")
    x, y = torch.zeros(40, d, dtype=tx, device="cuda"), torch.ones(40, d, dtype=ty, device="cuda")
    cfg = bt.BlockNorm(d, pre=bt.NORM_NONE, post=bt.NORM_NONE, gate=bt.GATE_SIGMOID)
    x_out = torch.empty_like(x)
    bt.betty_block_norm(cfg, params, x, y, gate, x_out, None)
    g = gate.double().cpu()
    want = 1.0 / (1.0 + torch.exp(-g))
    assert float(((x_out.double().cpu() - want).abs() - 8e-7 * want).max()) <= 0
    # dg = dx' s z a'(g), a' = a (1 - a): both factors to 8e-7
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 40))
    one, dx, dy, dg, dp = torch.ones_like(x), torch.empty_like(x), torch.empty_like(y), torch.empty_like(gate), torch.empty_like(params)
    bt.betty_block_norm_backward(cfg, params, None, y, gate, None, one, dx, dy, dg, dp, ws)
    slope = want / (1.0 + torch.exp(g))
    unit = 0.0 if ty == F else ref.UNIT[ty] * 1.001
    assert float(((dy.double().cpu() - want).abs() - (8e-7 + unit) * want).max()) <= 0
    assert float(((dg.double().cpu() - slope).abs() - (1.6e-6 + unit) * slope).max()) <= 0


@pytest.mark.parametrize("d", [257, 264, 384, 500, 512, 7200, 8192])
@pytest.mark.parametrize("per_gate", [1, 5])
@pytest.mark.parametrize("kind,bias", [("layer", True), ("layer", False), ("rms", True)])
def test_fp32_layer_norms_with_a_gate(d, per_gate, kind, bias):
    """Widths whose two rows and coefficients do not fit a block's share of the shared memory."""
    import paper_2207_02849_b200 as bt
    for rows in (3, 5000 if d < 600 else 330):
        q = _problem(rows + d, rows, d, F, F, "sigmoid", per_gate, bias)
        args = (d, kind, kind, "sigmoid", per_gate, bias, 1e-5)
        x_out, u = torch.full_like(q["x"], float("nan")), torch.full_like(q["y"], float("nan"))
        bt.betty_block_norm(_cfg(bt, *args), q["params"], q["x"], q["y"], q["gate"], x_out, u)
        _check_forward(q, args, x_out, u)
        _check_backward(bt, q, args)


@pytest.mark.parametrize("pad,shift", [(8, 8), (3, 0), (0, 1), (5, 2)])
@pytest.mark.parametrize("d,per_gate", [(264, 1), (264, 4), (1030, 1), (2304, 3)])
def test_layer_norms_with_biases_of_wider_buffers(pad, shift, d, per_gate):
    import paper_2207_02849_b200 as bt
    for tx, ty in ((F, F), (F, BF)):
        q = _problem(9, 21, d, tx, ty, "sigmoid", per_gate, True)
        args = (d, "layer", "layer", "sigmoid", per_gate, True, 1e-6)
        wide = lambda t: _wide(t, pad, shift)  # noqa: E731
        x_out, u = wide(torch.zeros_like(q["x"])), wide(torch.zeros_like(q["y"]))
        bt.betty_block_norm(_cfg(bt, *args), q["params"], wide(q["x"]), wide(q["y"]), wide(q["gate"]), x_out, u)
        _check_forward(q, args, x_out, u)
        _check_backward(bt, q, args, tensors=wide)


@pytest.mark.parametrize("rows,d", [(5000, 96), (2500, 1002), (700, 2051), (320, 4096)])
@pytest.mark.parametrize("kind,act,bias", [("rms", "linear", False), ("layer", "sigmoid", True)])
def test_parameter_gradients_element_by_element(rows, d, kind, act, bias):
    """Each is a sum over the rows, taken by walkers of at most 34 rows, at most eight warps of a block and 32 slices of at most ten
    blocks: no more than 34 + 8 + 10 + 32 roundings of a running sum whose size is at most the sum of the magnitudes: 84 * 2^-24 =
    5e-6 of it (roundings that all fall to one side, which they do not).  Each term besides carries the error of its own factors:
    SLACK of du n, and for the others SLACK of the row's size of dX (the tolerance that dx itself is held to) times the
    other factor."""
    import paper_2207_02849_b200 as bt
    q = _problem(rows, rows, d, F, F, act, 1, bias)
    args = (d, kind, kind, act, 1, bias, 1e-5)
    got = _check_backward(bt, q, args)[3].double().cpu()
    p, x, y, du = (ref.d64(q[k]) for k in ("params", "x", "y", "du"))
    g = ref.d64(q["gate"])
    a = g if act == "linear" else torch.sigmoid(g)
    want = _gradients(q, args)
    n, m, dX = ref.unit(x, kind, 1e-5), ref.unit(y, kind, 1e-5), want["dx"]
    rms = lambda t: t.pow(2).mean(-1, keepdim=True).sqrt()  # noqa: E731
    big = rms(dX) + rms(ref.d64(q["dxo"])) + rms(du)
    sums = lambda term, other: 5e-6 * term.abs().sum(0) + SLACK * (term.abs() + big * other.abs()).sum(0)  # noqa: E731
    post, flat = sums(dX * a * m, a * (m.abs() + 1.0)), sums(dX * a, a)
    bound = [5e-6 * (du * n).abs().sum(0) + SLACK * (du.abs() * (n.abs() + 1.0)).sum(0), p[2].abs() * post, p[1].abs() * post]
    if bias:
        bound[2] = bound[2] + p[4].abs() * flat
        bound += [5e-6 * du.abs().sum(0), p[2].abs() * flat]
    excess = (got - want["dparams"]).abs() / torch.stack(bound)
    assert float(excess.max()) <= 1.0, excess.amax(1)
