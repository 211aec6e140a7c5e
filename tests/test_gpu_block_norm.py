"""Norms before and after a block fused with its gate and residual scale, forward and backward, against the 64-bit
restatement.

Tolerances.  Every fp32 value on the way to an output goes through at most ~30 roundings and two approximate functions of
2 ulp (reciprocal square root, exp), so an element's error is below 40 * 2^-24 = 2.4e-6 of the row's size (the sums over
a row are trees of at most 8 + 4 + 15 additions per value); SLACK is 4e-6.  One rounding to a 16-bit type is added to
that.  Column sums over at most 400 rows add up to ~20 roundings of the running sum: 2e-6 of the sum of magnitudes."""
import itertools

import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
SLACK = 4e-6
BF, HF, F = torch.bfloat16, torch.float16, torch.float32
ACTS = ("none", "linear", "sigmoid")


def _rand(g, *shape, dtype=F, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def _wide(t, pad, shift):
    """The same values as rows of a wider buffer that starts `shift` values into it."""
    if t is None:
        return None
    buf = torch.full((t.shape[0], t.shape[1] + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[:, shift:shift + t.shape[1]]
    v.copy_(t)
    return v


def _problem(seed, rows, d, tx, ty, act, per_gate, bias):
    g = torch.Generator().manual_seed(seed)
    p = _rand(g, 5 if bias else 3, d, scale=0.3)
    p[:3] += 0.8
    gates = -(-rows // per_gate)
    return dict(params=p, x=_rand(g, rows, d, dtype=tx, scale=1.5), y=_rand(g, rows, d, dtype=ty) + 0.25,
                gate=_rand(g, gates, d, dtype=ty) if act != "none" else None,
                du=_rand(g, rows, d, dtype=ty), dxo=_rand(g, rows, d, dtype=tx))


def _cfg(bt, d, pre, post, act, per_gate, bias, eps):
    return bt.BlockNorm(d, pre=ref.KINDS.index(pre), post=ref.KINDS.index(post), gate=ACTS.index(act), rows_per_gate=per_gate, eps=eps,
                        bias=bias)


def _check_forward(q, cfg_args, x_out, u, with_y=True):
    d, pre, post, act, per_gate, bias, eps = cfg_args
    want_x, want_u = ref.block_norm(ref.d64(q["params"]), ref.d64(q["x"]), ref.d64(q["y"]) if with_y else None, ref.d64(q["gate"]),
                                    pre=pre, post=post, act=act, per_gate=per_gate, eps=eps)
    if x_out is not None:
        assert ref.close(x_out, want_x, x_out.dtype, SLACK) <= 0
    if u is not None:
        assert ref.close(u, want_u, u.dtype, SLACK, scale=_terms(want_u, q, bias)) <= 0


def _terms(want, q, bias):
    """Row scale of u: the norm's output is of size max |w_pre|, and 1 / rms amplifies nothing beyond the row's own size."""
    return want.pow(2).mean(1, keepdim=True).sqrt() + float(ref.d64(q["params"]).abs().max())


def _gradients(q, cfg_args, with_y=True, with_u=True, with_dxo=True):
    """64-bit gradients and, for the column sums, the sums of magnitudes."""
    d, pre, post, act, per_gate, bias, eps = cfg_args
    rows = q["x"].shape[0]
    params = ref.d64(q["params"]).requires_grad_(True)
    xo = ref.d64(q["x"]).requires_grad_(True)
    dX = ref.d64(q["dxo"]) if with_dxo else torch.zeros(rows, d, dtype=torch.float64)
    dparams = torch.zeros_like(params)
    if with_u:
        _, u = ref.block_norm(params, xo, None, None, pre=pre, post=post, act=act, per_gate=per_gate, eps=eps)
        gx, gp = torch.autograd.grad(u, (xo, params), ref.d64(q["du"]))
        dX, dparams = dX + gx, dparams + gp
    out = {"dx": dX}
    if with_y:
        y = ref.d64(q["y"]).requires_grad_(True)
        gate = ref.d64(q["gate"])
        ins = [y, params]
        if gate is not None:
            gate.requires_grad_(True)
            ins.append(gate)
        change, _ = ref.block_norm(params, torch.zeros(rows, d, dtype=torch.float64), y, gate, pre="none", post=post, act=act,
                                   per_gate=per_gate, eps=eps)
        got = torch.autograd.grad(change, ins, dX)
        out["dy"], dparams = got[0], dparams + got[1]
        if gate is not None:
            out["dgate"] = got[2]
    out["dparams"] = dparams
    return out


def _check_backward(bt, q, cfg_args, tensors=lambda t: t, with_y=True, with_u=True, with_dxo=True):
    d, pre, post, act, per_gate, bias, eps = cfg_args
    rows, tx, ty = q["x"].shape[0], q["x"].dtype, q["y"].dtype
    cfg = _cfg(bt, *cfg_args)
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, rows))
    x, y, gate, du, dxo = (tensors(q[k]) for k in ("x", "y", "gate", "du", "dxo"))
    nan = lambda t: tensors(torch.full_like(t.contiguous(), float("nan")))  # noqa: E731
    dx, dy = nan(q["x"]), nan(q["y"]) if with_y else None
    dgate = nan(q["gate"]) if act != "none" and with_y else None
    dparams = torch.full_like(q["params"], float("nan"))
    bt.betty_block_norm_backward(cfg, q["params"], x if with_u else None, y if with_y else None, gate if with_y else None,
                                 du if with_u else None, dxo if with_dxo else None, dx, dy, dgate, dparams, ws)
    assert bt.betty_poll_status(ws)[0] == bt.BETTY_OK
    want = _gradients(q, cfg_args, with_y, with_u, with_dxo)
    size = lambda t: t.pow(2).mean(-1, keepdim=True).sqrt()  # noqa: E731
    big = size(want["dx"]) + (size(ref.d64(q["dxo"])) + size(ref.d64(q["du"])) if rows else 0)
    assert ref.close(dx, want["dx"], tx, SLACK, scale=big) <= 0
    if with_y:
        q_norm = 1.0 / (ref.d64(q["y"]).var(1, keepdim=True, unbiased=False) + eps).sqrt() if post == "layer" else 1.0
        p = ref.d64(q["params"]).abs().amax(1)
        amp = float(p[1] * p[2]) * (4.0 if act == "linear" else 1.0)
        assert ref.close(dy, want["dy"], ty, SLACK, scale=size(want["dy"]) + amp * big * q_norm) <= 0
        if dgate is not None:
            n = min(rows, per_gate)
            assert ref.close(dgate, want["dgate"], ty, SLACK, scale=size(want["dgate"]) + 4.0 * n * amp * float(big.max())) <= 0
    # column sums: against the sum over rows of the magnitudes of what is added
    magnitude = rows * (float(ref.d64(q["du"]).abs().mean()) + float(want["dx"].abs().mean())) * 4.0 * float(q["params"].abs().max())
    assert float((dparams.double().cpu() - want["dparams"]).abs().max()) <= 2e-6 * magnitude + 1e-12
    return dx, dy, dgate, dparams


SIZES = [(1, 1), (1, 64), (3, 7), (5, 256), (9, 257), (2, 1000), (33, 1024), (400, 96), (4, 4096), (3, 5000), (2, 8192), (2, 16384),
         (3, 16383), (17, 1537)]
TYPES = [(F, F), (BF, BF), (HF, HF), (F, BF), (F, HF)]


@pytest.mark.parametrize("rows,d", SIZES)
@pytest.mark.parametrize("kind,act,per_gate,bias", [("rms", "linear", 1, False), ("layer", "sigmoid", 3, True), ("rms", "sigmoid", 128, False),
                                                    ("layer", "none", 1, False), ("rms", "linear", 7, True)])
def test_forward_and_backward_over_sizes(rows, d, kind, act, per_gate, bias):
    import paper_2207_02849_b200 as bt
    seed = rows * 31 + d
    tx, ty = TYPES[(rows + d + per_gate) % len(TYPES)]
    q = _problem(seed, rows, d, tx, ty, act, per_gate, bias)
    args = (d, kind, kind, act, per_gate, bias, 1e-5)
    x_out, u = torch.full_like(q["x"], float("nan")), torch.full_like(q["y"], float("nan"))
    bt.betty_block_norm(_cfg(bt, *args), q["params"], q["x"], q["y"], q["gate"], x_out, u)
    _check_forward(q, args, x_out, u)
    _check_backward(bt, q, args)


@pytest.mark.parametrize("rows,d", [(5000, 96), (5000, 130), (4800, 77), (2500, 1000), (2500, 1002), (700, 4096), (700, 2050), (700, 2051),
                                    (320, 5000), (320, 5002), (320, 8191)])
@pytest.mark.parametrize("kind,act,per_gate,bias", [("rms", "linear", 1, False), ("layer", "sigmoid", 1, True), ("rms", "sigmoid", 90, False),
                                                    ("layer", "linear", 33, True)])
def test_many_rows(rows, d, kind, act, per_gate, bias):
    """Enough rows for every thread group to walk several.  (Column sums of 5000 rows: each walker adds at most 34 of them, the
    walkers' sums are added over at most 2 x 148: 2e-6 of the sum of magnitudes holds as for fewer rows.)"""
    import paper_2207_02849_b200 as bt
    for tx, ty in ((F, F), (BF, BF), (F, HF)):
        q = _problem(rows + d, rows, d, tx, ty, act, per_gate, bias)
        args = (d, kind, kind, act, per_gate, bias, 1e-5)
        x_out, u = torch.full_like(q["x"], float("nan")), torch.full_like(q["y"], float("nan"))
        bt.betty_block_norm(_cfg(bt, *args), q["params"], q["x"], q["y"], q["gate"], x_out, u)
        _check_forward(q, args, x_out, u)
        _check_backward(bt, q, args)


def test_a_nan_row_among_many_stays_by_itself():
    import paper_2207_02849_b200 as bt
    for d in (2000, 2002, 2051):
        q = _problem(1, 900, d, F, F, "linear", 1, False)
        q["x"][450, 3] = float("nan")
        q["y"][300, d - 1] = float("inf")
        cfg = _cfg(bt, d, "rms", "rms", "linear", 1, False, 1e-6)
        ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 900))
        outs = [torch.full_like(q[k], float("nan")) for k in ("x", "y", "gate", "params")]
        bt.betty_block_norm_backward(cfg, q["params"], q["x"], q["y"], q["gate"], q["du"], q["dxo"], *outs, ws)
        keep = [i for i in range(900) if i not in (300, 450)]
        for t in outs[:3]:
            assert bool(torch.isfinite(t[keep]).all())
        assert bool(torch.isnan(outs[0][450]).all())


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("pre,post", list(itertools.product(ref.KINDS, ref.KINDS)))
def test_every_pair_of_norms_and_types(tx, ty, pre, post):
    import paper_2207_02849_b200 as bt
    q = _problem(5, 37, 520, tx, ty, "sigmoid", 5, True)
    args = (520, pre, post, "sigmoid", 5, True, 1e-6)
    x_out, u = torch.empty_like(q["x"]), torch.empty_like(q["y"])
    bt.betty_block_norm(_cfg(bt, *args), q["params"], q["x"], q["y"], q["gate"], x_out, u)
    _check_forward(q, args, x_out, u)
    _check_backward(bt, q, args)


@pytest.mark.parametrize("pad,shift", [(8, 8), (3, 0), (0, 1), (5, 2)])
@pytest.mark.parametrize("tx,ty", [(BF, BF), (F, HF)])
def test_rows_of_wider_buffers(pad, shift, tx, ty):
    import paper_2207_02849_b200 as bt
    q = _problem(9, 21, 264, tx, ty, "linear", 4, False)
    args = (264, "rms", "rms", "linear", 4, False, 1e-6)
    wide = lambda t: _wide(t, pad, shift)  # noqa: E731
    x_out, u = wide(torch.zeros_like(q["x"])), wide(torch.zeros_like(q["y"]))
    bt.betty_block_norm(_cfg(bt, *args), q["params"], wide(q["x"]), wide(q["y"]), wide(q["gate"]), x_out, u)
    _check_forward(q, args, x_out, u)
    base = x_out._base
    untouched = torch.ones(base.shape[1], dtype=torch.bool)
    untouched[shift:shift + 264] = False
    assert bool(torch.isnan(base[:, untouched.cuda()]).all())       # nothing is written beside the rows
    _check_backward(bt, q, args, tensors=wide)


def test_parts_left_out():
    import paper_2207_02849_b200 as bt
    q = _problem(3, 40, 384, F, BF, "linear", 1, False)
    args = (384, "rms", "rms", "linear", 1, False, 1e-6)
    cfg = _cfg(bt, *args)
    u = torch.empty_like(q["y"])
    bt.betty_block_norm(cfg, q["params"], q["x"], None, None, None, u)                  # entry norm alone
    _check_forward(q, args, None, u, with_y=False)
    x_out = torch.empty_like(q["x"])
    bt.betty_block_norm(cfg, q["params"], q["x"], q["y"], q["gate"], x_out, None)        # no block after
    _check_forward(q, args, x_out, None)
    for with_y, with_u, with_dxo in ((False, True, True), (False, True, False), (True, False, True), (True, True, False)):
        _check_backward(bt, q, args, with_y=with_y, with_u=with_u, with_dxo=with_dxo)


def test_in_place():
    import paper_2207_02849_b200 as bt
    q = _problem(4, 50, 640, BF, BF, "sigmoid", 1, False)
    cfg = _cfg(bt, 640, "rms", "rms", "sigmoid", 1, False, 1e-6)
    x_out, u, u2, x = torch.empty_like(q["x"]), torch.empty_like(q["y"]), torch.empty_like(q["y"]), q["x"].clone()
    bt.betty_block_norm(cfg, q["params"], q["x"], q["y"], q["gate"], x_out, u)
    bt.betty_block_norm(cfg, q["params"], x, q["y"], q["gate"], x, u2)
    assert torch.equal(x, x_out) and torch.equal(u, u2)
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 50))
    outs = [torch.empty_like(q["x"]), torch.empty_like(q["y"]), torch.empty_like(q["gate"]), torch.empty_like(q["params"])]
    bt.betty_block_norm_backward(cfg, q["params"], x_out, q["y"], q["gate"], q["du"], q["dxo"], *outs, ws)
    dx, dy, dg, dp = q["dxo"].clone(), q["y"].clone(), q["gate"].clone(), torch.empty_like(q["params"])
    bt.betty_block_norm_backward(cfg, q["params"], x_out, dy, dg, q["du"], dx, dx, dy, dg, dp, ws)
    for a, b in zip(outs, (dx, dy, dg, dp)):
        assert torch.equal(a, b)


def test_a_row_of_zeros_and_a_row_with_nan_stay_by_themselves():
    import paper_2207_02849_b200 as bt
    q = _problem(6, 12, 512, F, F, "linear", 1, False)
    q["x"][3].zero_()
    q["y"][3].zero_()
    args = (512, "rms", "rms", "linear", 1, False, 1e-6)
    cfg = _cfg(bt, *args)
    x_out, u = torch.empty_like(q["x"]), torch.empty_like(q["y"])
    bt.betty_block_norm(cfg, q["params"], q["x"], q["y"], q["gate"], x_out, u)
    assert float(x_out[3].abs().max()) == 0.0 and float(u[3].abs().max()) == 0.0
    _check_backward(bt, q, args)
    x = q["x"].clone()
    x[7, 100] = float("nan")
    x2, u2 = torch.empty_like(x), torch.empty_like(u)
    bt.betty_block_norm(cfg, q["params"], x, q["y"], q["gate"], x2, u2)
    assert bool(torch.isnan(u2[7]).all())
    keep = [i for i in range(12) if i != 7]
    assert torch.equal(u2[keep], u[keep]) and torch.equal(x2[keep], x_out[keep])


def test_no_rows():
    import paper_2207_02849_b200 as bt
    cfg = bt.BlockNorm(256, gate=bt.GATE_LINEAR)
    e = torch.empty(0, 256, dtype=BF, device="cuda")
    p = torch.ones(3, 256, device="cuda")
    bt.betty_block_norm(cfg, p, e, e, e, e, e)
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, 0))
    dp = torch.full_like(p, float("nan"))
    bt.betty_block_norm_backward(cfg, p, e, e, e, e, e, e, e, e, dp, ws)
    assert float(dp.abs().max()) == 0.0


@pytest.mark.parametrize("rows,per_gate", [(700, 64), (3000, 7), (3000, 1000)])
def test_gates_of_several_rows_and_repeatability(rows, per_gate):
    """Shares of the rows that cut through gates; the same call gives the same bits, on another stream too."""
    import paper_2207_02849_b200 as bt
    q = _problem(8, rows, 1024 if rows > 1000 else 96, F, BF, "linear", per_gate, False)
    d = q["x"].shape[1]
    args = (d, "rms", "rms", "linear", per_gate, False, 1e-6)
    cfg = _cfg(bt, *args)
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, rows))
    runs = []
    for stream in (None, torch.cuda.Stream()):
        outs = [torch.full_like(q[k], float("nan")) for k in ("x", "y", "gate", "params")]
        torch.cuda.synchronize()
        bt.betty_block_norm_backward(cfg, q["params"], q["x"], q["y"], q["gate"], q["du"], q["dxo"], *outs, ws, stream=stream)
        torch.cuda.synchronize()
        runs.append(outs)
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    want = _gradients(q, args)
    n = min(rows, per_gate)
    assert ref.close(runs[0][2], want["dgate"], BF, SLACK * n, scale=torch.full((1, 1), 8.0, dtype=torch.float64)) <= 0
    terms = rows * 8.0
    assert float((runs[0][3].double().cpu() - want["dparams"]).abs().max()) <= 2e-6 * terms


@pytest.mark.parametrize("kind,act,per_gate,bias", [("rms", "linear", 1, False), ("layer", "sigmoid", 4, True)])
def test_gradients_against_differences(kind, act, per_gate, bias):
    """Central differences of sum(c1 x') + sum(c2 u) along random directions of every input.  Step h = 2^-6: the
    difference's own error is h^2 / 6 times a third derivative of order one plus 2^-24 * |L| / h: below 2e-3 of the
    directions' size."""
    import paper_2207_02849_b200 as bt
    rows, d = 11, 200
    q = _problem(21, rows, d, F, F, act, per_gate, bias)
    cfg = _cfg(bt, d, kind, kind, act, per_gate, bias, 1e-3)
    c1, c2 = q["dxo"].double(), q["du"].double()

    def value(x, y, gate, params):
        x_out, u = torch.empty_like(x), torch.empty_like(y)
        bt.betty_block_norm(cfg, params, x, y, gate, x_out, u)
        return float((x_out.double() * c1).sum() + (u.double() * c2).sum()), x_out

    base = [q["x"], q["y"], q["gate"], q["params"]]
    _, x_out = value(*base)
    ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, rows))
    grads = [torch.empty_like(t) for t in base]
    bt.betty_block_norm_backward(cfg, q["params"], x_out, q["y"], q["gate"], q["du"], q["dxo"], *grads, ws)
    g = torch.Generator().manual_seed(2)
    h = 2.0 ** -6
    for i in range(4):
        dirn = _rand(g, *base[i].shape)
        moved = lambda s: [t + s * dirn if j == i else t for j, t in enumerate(base)]  # noqa: E731
        diff = (value(*moved(h))[0] - value(*moved(-h))[0]) / (2 * h)
        want = float((grads[i].double() * dirn.double()).sum())
        size = float(grads[i].double().norm() * dirn.double().norm()) / dirn.numel() ** 0.5
        assert abs(diff - want) <= 5e-3 * size, (i, diff, want, size)


def test_refusals_of_the_binding():
    import paper_2207_02849_b200 as bt
    cfg = bt.BlockNorm(64, gate=bt.GATE_LINEAR, rows_per_gate=2)
    p = torch.ones(3, 64, device="cuda")
    t = torch.zeros(4, 64, dtype=BF, device="cuda")
    gate = torch.zeros(2, 64, dtype=BF, device="cuda")
    o = torch.empty_like(t)
    with pytest.raises(ValueError):
        bt.betty_block_norm(cfg, p, t, t, t, o, o)                      # four gate rows where two are wanted
    with pytest.raises(ValueError):
        bt.betty_block_norm(cfg, p, t, t.float(), gate, o, o)
    with pytest.raises(ValueError):
        bt.betty_block_norm(cfg, p, t, t[:, :32], gate, o, o)
    with pytest.raises(ValueError):
        bt.betty_block_norm(cfg, p[:2], t, t, gate, o, o)
    with pytest.raises(ValueError):
        bt.betty_block_norm(cfg, p, torch.zeros(64, 4, dtype=BF, device="cuda").t(), t, gate, o, o)
    with pytest.raises(bt.BettyError) as e:
        bt.betty_block_norm(cfg, p, t, t, None, o, o)
    assert e.value.status == bt.BETTY_ERR_INVALID_ARG
    with pytest.raises(bt.BettyError) as e:                             # rows that overlap: a broadcast row
        bt.betty_block_norm(cfg, p, t[:1].expand(4, 64), t, gate, o, o)
    assert e.value.status == bt.BETTY_ERR_SHAPE
    with pytest.raises(bt.BettyError) as e:
        bt.betty_block_norm(cfg, p, t.half(), t, gate, t.half(), o)
    assert e.value.status == bt.BETTY_ERR_DTYPE
    small = bt.Workspace.of_bytes(256)
    with pytest.raises(bt.BettyError) as e:
        bt.betty_block_norm_backward(cfg, p, t, t, gate, t, t, o, o.clone(), gate.clone(), p.clone(), small)
    assert e.value.status == bt.BETTY_ERR_WORKSPACE


@pytest.mark.parametrize("rows", [1, 7, 8, 9, 15, 17, 85, 150, 1300])
@pytest.mark.parametrize("d,per_gate", [(515, 7), (515, 20), (1538, 7), (1540, 5), (4101, 9)])
def test_gates_shared_by_a_few_rows_of_an_odd_width(rows, d, per_gate):
    """Rows whose starts repeat every 2, 4 or 8 rows are walked by class, so a gate's rows lie in several walkers' shares; with
    few rows the classes differ in length and a share can be empty."""
    import paper_2207_02849_b200 as bt
    q = _problem(rows + d, rows, d, F, F, "sigmoid", per_gate, False)
    _check_backward(bt, q, (d, "rms", "rms", "sigmoid", per_gate, False, 1e-5))


@pytest.mark.parametrize("d", [5200, 8192])
@pytest.mark.parametrize("kind,bias", [("rms", False), ("layer", True)])
@pytest.mark.parametrize("rows", [3, 500])
def test_rows_too_wide_for_two_to_be_fetched(rows, d, kind, bias):
    import paper_2207_02849_b200 as bt
    for tx, ty in ((F, F), (BF, BF), (F, BF)):
        q = _problem(rows + d, rows, d, tx, ty, "sigmoid", 1, bias)
        _check_backward(bt, q, (d, kind, kind, "sigmoid", 1, bias, 1e-5))
