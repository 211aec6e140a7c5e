"""Losses over a vocabulary against 64-bit restatements (tests/vocab_reference.py says how far they may be off)."""
import pytest
import torch

from tests import vocab_reference as ref

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32
SIZES = [(1, 8), (2, 64), (100, 1), (257, 72), (1000, 200), (4099, 515), (513, 1025), (20000, 64)]
ROWS = [1, 7, 16, 17, 33, 128, 129, 300, 700]


def _problem(seed, rows, vocab, d, dtype, ignored=0.2, boost=6.0):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(vocab, d, generator=g) / d ** 0.5).to(dtype)
    target = torch.randint(vocab, (rows,), generator=g)
    x = (torch.randn(rows, d, generator=g) + boost * torch.rand(rows, 1, generator=g) * w[target].float()).to(dtype)
    target[torch.rand(rows, generator=g) < ignored] = -100
    dloss = torch.rand(rows, generator=g) * 2 - 0.5
    return x.cuda(), w.cuda(), target.cuda(), dloss.cuda()


def _cfg(bt, vocab, d, dtype, **k):
    return bt.VocabLoss(vocab, d, bt.BETTY_BF16 if dtype == BF else bt.BETTY_F16, **k)


def _nan(*shape, dtype=F):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def _ok(bt, ws):
    assert bt.betty_poll_status(ws, raise_on_error=False)[0] == bt.BETTY_OK


def _check_ce(bt, x, w, target, dloss, out=None, ws=None, any_layout=None, wants="xw", wrap=lambda t: t, **k):
    rows, (vocab, d), dtype = x.shape[0], w.shape, x.dtype
    cfg = _cfg(bt, vocab, d, dtype, **k)
    ws = ws or bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows, any_layout=any_layout))
    loss, lse = _nan(rows), _nan(rows)
    bt.betty_vocab_ce(cfg, wrap(x), wrap(w), target, loss, lse, ws)
    _ok(bt, ws)
    e = ref.Expected(x, w, ref.entries_ce(target, vocab, k.get("smoothing", 0.0)), k.get("temperature", 1.0), k.get("smoothing", 0.0), k.get("z_loss", 0.0))
    e.check_forward(loss, lse)
    dx = wrap(_nan(rows, d, dtype=out or dtype)) if "x" in wants else None
    dw = wrap(_nan(vocab, d, dtype=out or dtype)) if "w" in wants else None
    bt.betty_vocab_ce_backward(cfg, wrap(x), wrap(w), target, lse, dloss, dx, dw, ws)
    _ok(bt, ws)
    for got, want in zip((dx, dw), e.gradients(dloss)):
        assert got is None or ref.near(got, *want)
    if dx is not None:
        assert bool((dx[~e.live] == 0).all())
    return loss, lse, dx, dw


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("vocab,d", SIZES)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_cross_entropy(rows, vocab, d, dtype):
    import paper_2207_02849_b200 as bt
    _check_ce(bt, *_problem(rows + vocab, rows, vocab, d, dtype))


@pytest.mark.parametrize("rows,vocab,d", [(40, 300, 96), (300, 1111, 130), (129, 4000, 64)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("k", [dict(smoothing=0.1), dict(z_loss=1e-3), dict(temperature=0.5), dict(temperature=3.0), dict(smoothing=1.0), dict(smoothing=0.3, z_loss=0.02, temperature=1.7)],
                         ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()))
def test_smoothing_z_loss_temperature(rows, vocab, d, dtype, k):
    import paper_2207_02849_b200 as bt
    _check_ce(bt, *_problem(rows, rows, vocab, d, dtype), **k)


@pytest.mark.parametrize("wants", ["x", "w", "xw"])
@pytest.mark.parametrize("out", [F, None])
@pytest.mark.parametrize("rows,vocab,d", [(9, 2000, 520), (1000, 700, 264), (150, 9000, 1000)])
def test_either_gradient_and_fp32_results(wants, out, rows, vocab, d):
    import paper_2207_02849_b200 as bt
    for dtype in (BF, HF):
        _check_ce(bt, *_problem(7, rows, vocab, d, dtype), out=out, wants=wants)


@pytest.mark.parametrize("rows,vocab,d", [(16384, 20000, 64), (5000, 33000, 72), (20000, 9001, 40)])
def test_several_pieces_of_the_vocabulary(rows, vocab, d):
    import paper_2207_02849_b200 as bt
    _check_ce(bt, *_problem(3, rows, vocab, d, BF))


@pytest.mark.parametrize("rows", [1, 100, 128, 500])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_rows_left_out(rows, dtype):
    """Rows with a target outside the vocabulary or with no weight: NaN and infinities in them reach nothing."""
    import paper_2207_02849_b200 as bt
    vocab, d = 700, 136
    x, w, target, dloss = _problem(11, rows, vocab, d, dtype, ignored=0.0)
    for kind in range(3):
        t, g, x2 = target.clone(), dloss.clone(), x.clone()
        out = torch.arange(rows, device="cuda") % 3 != 1 if kind < 2 else torch.ones(rows, dtype=torch.bool, device="cuda")
        t[out] = torch.tensor([-1, vocab, -(1 << 40), 1 << 40], device="cuda")[torch.arange(rows, device="cuda") % 4][out]
        g[out] = float("nan")
        if kind == 1:                                   # those that count by their target have no weight, or one
            t, g = target.clone(), dloss.clone()
            g[out] = 0.0
        x2[out] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda", dtype=dtype)[torch.arange(rows, device="cuda") % 3][out][:, None]
        cfg = _cfg(bt, vocab, d, dtype)
        ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows))
        e = ref.Expected(x, w, ref.entries_ce(torch.where(out, -1, target), vocab, 0.0))
        loss, lse = _nan(rows), _nan(rows)
        if kind != 1:
            bt.betty_vocab_ce(cfg, x2, w, t, loss, lse, ws)
            e.check_forward(loss, lse)
        else:
            lse = torch.where(out, float("nan"), e.lse.float())
        dx, dw = _nan(rows, d, dtype=dtype), _nan(vocab, d, dtype=dtype)
        ws.buf[256 + (-ws.buf.data_ptr()) % 256:] = 255          # what a workspace holds before reaches nothing either: all NaN
        bt.betty_vocab_ce_backward(cfg, x2, w, t, lse, g, dx, dw, ws)
        (wx, ex), (ww, ew) = e.gradients(torch.where(out, 0.0, dloss))
        assert ref.near(dx, wx, ex) and ref.near(dw, ww, ew)
        assert bool((dx[out] == 0).all())
        if kind == 2:
            assert bool((dw == 0).all())


def test_int32_targets_and_more_rows_than_are_counted_in_one_round():
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(2, 9000, 515, 24, BF, ignored=0.5)
    a = _check_ce(bt, x, w, target, dloss)
    b = _check_ce(bt, x, w, target.int(), dloss)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_a_row_that_is_not_a_number_stays_alone():
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(5, 140, 900, 64, BF, ignored=0.0)
    clean = _check_ce(bt, x, w, target, dloss, wants="x")
    x[77] = float("nan")
    cfg = _cfg(bt, 900, 64, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 140))
    loss, lse, dx = _nan(140), _nan(140), torch.zeros_like(x)
    bt.betty_vocab_ce(cfg, x, w, target, loss, lse, ws)
    bt.betty_vocab_ce_backward(cfg, x, w, target, lse, dloss, dx, None, ws)
    others = torch.arange(140, device="cuda") != 77
    assert bool(loss[77].isnan()) and bool(lse[77].isnan()) and bool(dx[77].isnan().all())
    assert torch.equal(loss[others], clean[0][others]) and torch.equal(lse[others], clean[1][others]) and torch.equal(dx[others], clean[2][others])


def test_columns_of_minus_infinity_and_large_logits():
    """A row of W that makes a logit -inf has no part in the sums; logits of some thousands keep their differences."""
    import paper_2207_02849_b200 as bt
    g = torch.Generator().manual_seed(0)
    rows, vocab, d = 70, 600, 64
    x, w = torch.randn(rows, d, generator=g), torch.randn(vocab, d, generator=g)
    x[:, 0], w[:, 0] = 1.0, 0.0
    w[5:400:3, 0] = -float("inf")
    x, w = (x * 40).to(BF).cuda(), w.to(BF).cuda()
    target = torch.randint(400, 600, (rows,), generator=g).cuda()
    cfg = _cfg(bt, vocab, d, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows))
    loss, lse = _nan(rows), _nan(rows)
    bt.betty_vocab_ce(cfg, x, w, target, loss, lse, ws)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    finite = torch.where(w.isinf(), 0.0, w.double())
    slack = (d / 16 + 8) * 2.0 ** -23 * (x.double().abs() @ finite.abs().t()).amax(1) + ref.SUMS + 2.0 ** -21 * z[z.isfinite()].abs().max()
    assert bool(((lse.double() - want).abs() <= slack).all())
    assert bool(((loss.double() - (want - z.gather(1, target[:, None])[:, 0])).abs() <= 2 * slack).all())


def test_half_precision_keeps_rows_of_small_weight():
    """Weights from 1 to 2^-30 and to 2^20: each row's gradient is as near, relative to itself, as that of the others."""
    import paper_2207_02849_b200 as bt
    x, w, target, _ = _problem(9, 200, 3000, 96, HF, ignored=0.0)
    for low, high in ((-30, 0), (-12, 20), (-100, -60)):
        dloss = torch.logspace(low, high, 200, base=2.0, device="cuda") * torch.where(torch.arange(200, device="cuda") % 2 == 0, 1.0, -1.0)
        e = ref.Expected(x, w, ref.entries_ce(target, 3000, 0.0))
        cfg = _cfg(bt, 3000, 96, HF)
        ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 200))
        dx, dw = _nan(200, 96), _nan(3000, 96)
        bt.betty_vocab_ce_backward(cfg, x, w, target, e.lse.float(), dloss, dx, dw, ws)
        (wx, ex), (ww, ew) = e.gradients(dloss)
        assert ref.near(dx, wx, ex)
        # dW: rows below 2^-7 of the largest weight are scaled in x, whose smallest steps are 2^-24: 2^-25 2^14 / 2^13 of the largest weight
        assert ref.near(dw, ww, ew + 200 * 2.0 ** -24 * dloss.abs().max())


@pytest.mark.parametrize("rows,vocab,d", [(1, 700, 64), (5, 20000, 200), (24, 3000, 1025), (32, 999, 130)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_few_rows_keep_what_their_coefficients_lose(rows, vocab, d, dtype):
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(rows, rows, vocab, d, dtype, ignored=0.2 if rows > 1 else 0.0)
    cfg = _cfg(bt, vocab, d, dtype)
    e = ref.Expected(x, w, ref.entries_ce(target, vocab, 0.0))
    for room in (rows, 300):                       # a workspace for more rows changes nothing
        ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, room))
        ws.buf[256 + (-ws.buf.data_ptr()) % 256:] = 255
        dx, dw = _nan(rows, d), _nan(vocab, d)
        bt.betty_vocab_ce_backward(cfg, x, w, target, e.lse.float(), dloss, dx, dw, ws)
        (wx, ex), (ww, ew) = e.gradients(dloss, roundings=2)
        assert ref.near(dx, wx, ex) and ref.near(dw, ww, ew)
        for a, b in (((dx, None), (None, dw)) if rows > 1 else ()):
            one = [None if t is None else torch.full_like(t, float("nan")) for t in (a, b)]
            bt.betty_vocab_ce_backward(cfg, x, w, target, e.lse.float(), dloss, *one, ws)
            assert all(t is None or ref.near(t, *v) for t, v in zip(one, ((wx, ex), (ww, ew))))


def _wide(pad, shift):
    def wrap(t):
        buf = torch.full((*t.shape[:-1], t.shape[-1] + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
        v = buf[..., shift:shift + t.shape[-1]]
        v.copy_(t)
        return v
    return wrap


@pytest.mark.parametrize("pad,shift,d", [(8, 8, 128), (3, 0, 128), (0, 1, 136), (7, 2, 65), (1, 3, 64), (4, 4, 200), (5, 0, 67), (7, 0, 129), (14, 8, 66)])
@pytest.mark.parametrize("rows,vocab", [(20, 333), (260, 700)])
def test_rows_of_wider_buffers(pad, shift, d, rows, vocab):
    """What lies beside the rows is NaN: nothing of it may reach a sum."""
    import paper_2207_02849_b200 as bt
    for dtype, out in ((BF, None), (HF, F)):
        _check_ce(bt, *_problem(4, rows, vocab, d, dtype), out=out, wrap=_wide(pad, shift), any_layout=True)


def test_results_leave_their_neighbours():
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(6, 150, 401, 72, BF)
    cfg = _cfg(bt, 401, 72, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 150))
    lse = torch.logsumexp(x.float() @ w.float().t(), 1)
    for pad in (8, 5):
        bx, bw = torch.full((152, 72 + pad), 7.0, dtype=BF, device="cuda"), torch.full((403, 72 + pad), 7.0, dtype=BF, device="cuda")
        bt.betty_vocab_ce_backward(cfg, x, w, target, lse, dloss, bx[1:151, :72], bw[1:402, :72], ws)
        for b in (bx, bw):
            assert bool((b[0] == 7).all()) and bool((b[-1] == 7).all()) and bool((b[:, 72:] == 7).all())


# ---- distillation ----
def _entries(seed, rows, vocab, top, dtype, kind):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(vocab, (rows, top), generator=g) if kind != "top" else torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(rows)])
    t = torch.randn(rows, top, generator=g) * 3
    if kind == "dense":                                  # neighbouring ids, many of them twice
        ids = (ids % max(1, min(vocab, top)) + vocab // 3) % vocab
    if kind == "holes":
        bad = torch.rand(rows, top, generator=g) < 0.4
        bad[::5] = True
        ids[bad] = torch.tensor([-1, vocab, -(1 << 31), (1 << 31) - 1])[torch.randint(4, (int(bad.sum()),), generator=g)]
        t[bad] = float("nan")
        t[torch.rand(rows, top, generator=g) < 0.2] = -float("inf")
    return ids, t.to(dtype)


def _check_distill(bt, x, w, ids, teacher, dloss, temperature=1.0, wrap=lambda t: t, top_of_ws=None, any_layout=None, out=None):
    rows, (vocab, d), dtype = x.shape[0], w.shape, x.dtype
    cfg = _cfg(bt, vocab, d, dtype, temperature=temperature)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows, top_of_ws or ids.shape[1], any_layout))
    loss, lse = _nan(rows), _nan(rows)
    bt.betty_vocab_distill(cfg, wrap(x), wrap(w), ids, teacher, loss, lse, ws)
    _ok(bt, ws)
    e = ref.Expected(x, w, ref.entries_distill(ids, teacher, vocab, temperature), temperature, distill=True)
    e.check_forward(loss, lse)
    dx, dw = wrap(_nan(rows, d, dtype=out or dtype)), wrap(_nan(vocab, d, dtype=out or dtype))
    bt.betty_vocab_distill_backward(cfg, wrap(x), wrap(w), ids, teacher, lse, dloss, dx, dw, ws)
    _ok(bt, ws)
    (wx, ex), (ww, ew) = e.gradients(dloss)
    assert ref.near(dx, wx, ex) and ref.near(dw, ww, ew)
    assert bool((dx[~e.live] == 0).all())
    return loss, lse, dx, dw


@pytest.mark.parametrize("top", [1, 2, 5, 31, 32, 33, 64, 100, 200, 513, 1024])
@pytest.mark.parametrize("kind", ["any", "dense", "holes"])
@pytest.mark.parametrize("rows,vocab,d", [(40, 2000, 64), (200, 1030, 72)])
def test_distillation(top, kind, rows, vocab, d):
    import paper_2207_02849_b200 as bt
    for dtype, teacher, t in ((BF, F, 1.0), (HF, BF, 2.5), (BF, HF, 0.5)):
        x, w, _, dloss = _problem(top, rows, vocab, d, dtype, boost=0.0)
        ids, logits = _entries(top + rows, rows, vocab, top, teacher, kind)
        _check_distill(bt, x, w, ids.cuda() if teacher == F else ids.int().cuda(), logits.cuda(), dloss, t)


@pytest.mark.parametrize("rows", [1, 33, 129, 600])
@pytest.mark.parametrize("vocab,d", [(5, 16), (257, 100), (4099, 515)])
def test_distillation_sizes(rows, vocab, d):
    import paper_2207_02849_b200 as bt
    for top in (1, min(vocab, 7), min(vocab, 60)):
        x, w, _, dloss = _problem(rows, rows, vocab, d, BF, boost=0.0)
        ids, logits = _entries(rows, rows, vocab, top, F, "top")
        _check_distill(bt, x, w, ids.cuda(), logits.cuda(), dloss, top_of_ws=64)


def test_distillation_of_wider_buffers():
    import paper_2207_02849_b200 as bt
    x, w, _, dloss = _problem(8, 150, 900, 66, HF, boost=0.0)
    ids, logits = _entries(1, 150, 900, 9, F, "holes")
    b_ids, b_t = torch.full((150, 14), 3, device="cuda"), torch.full((150, 14), float("nan"), device="cuda")
    b_ids[:, 2:11], b_t[:, 2:11] = ids.cuda(), logits.cuda()
    a = _check_distill(bt, x, w, ids.cuda(), logits.cuda(), dloss)
    b = _check_distill(bt, x, w, b_ids[:, 2:11], b_t[:, 2:11], dloss, wrap=_wide(3, 1), any_layout=True, out=None)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_a_student_that_has_learnt_its_teacher():
    """All of a small vocabulary are entries, with the student's own logits: the loss and the gradients are nothing but roundings."""
    import paper_2207_02849_b200 as bt
    x, w, _, dloss = _problem(12, 130, 96, 64, BF, boost=0.0)
    z = (x.double() @ w.double().t()).float()
    ids = torch.stack([torch.randperm(96, generator=torch.Generator().manual_seed(i)) for i in range(130)]).cuda()
    loss, _, dx, _ = _check_distill(bt, x, w, ids, z.gather(1, ids), dloss, out=F)
    assert float(loss.abs().max()) < 1e-5 and float(dx.abs().max()) < 1e-4


def test_one_entry_is_a_cross_entropy():
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(13, 200, 1500, 80, BF)
    a = _check_ce(bt, x, w, target, dloss)
    b = _check_distill(bt, x, w, target[:, None], torch.full((200, 1), 5.0, device="cuda"), dloss)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


# ---- gradients against differences ----
@pytest.mark.parametrize("distill", [False, True])
def test_gradients_against_differences(distill):
    """Along a direction of x and one of W, with fp32 losses at points that are exact in half precision.  z(t) is a quadratic of the step
    t, so that the central difference of a loss is off by t^2 / 6 of its third derivative: |dz|^3 and less here, below 2e-3 at 1/64."""
    import paper_2207_02849_b200 as bt
    rows, vocab, d = 150, 400, 48
    g = torch.Generator().manual_seed(21)
    grid = lambda *s: (torch.randint(-8, 9, s, generator=g) / 16).to(HF).cuda()  # noqa: E731
    x, w, vx, vw = grid(rows, d), grid(vocab, d), grid(rows, d), grid(vocab, d)
    target = torch.randint(vocab, (rows,), generator=g).cuda()
    ids, logits = (t.cuda() for t in _entries(3, rows, vocab, 20, F, "holes"))
    cfg = _cfg(bt, vocab, d, HF, **({} if distill else dict(smoothing=0.2, z_loss=0.01)))
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows, 20))
    dloss = torch.rand(rows, generator=g).cuda()

    def loss_at(t):
        loss, lse = _nan(rows), _nan(rows)
        a, b = (x + t * vx), (w + t * vw)
        (bt.betty_vocab_distill(cfg, a, b, ids, logits, loss, lse, ws) if distill else bt.betty_vocab_ce(cfg, a, b, target, loss, lse, ws))
        return loss.double(), lse

    t = 1.0 / 64
    per_row = (loss_at(t)[0] - loss_at(-t)[0]) / (2 * t)
    _, lse = loss_at(0.0)
    dx, dw = _nan(rows, d), _nan(vocab, d)
    if distill:
        bt.betty_vocab_distill_backward(cfg, x, w, ids, logits, lse, dloss, dx, dw, ws)
    else:
        bt.betty_vocab_ce_backward(cfg, x, w, target, lse, dloss, dx, dw, ws)
    along = float((dx.double() * vx.double()).sum() + (dw.double() * vw.double()).sum())
    want = float((dloss.double() * per_row).sum())
    size = float(((dx.double() * vx.double()).sum(1).abs()).sum())
    assert abs(along - want) <= 2e-3 * rows + 2.0 ** -11 * size


# ---- calls ----
@pytest.mark.parametrize("rows,vocab,d", [(400, 5000, 200), (8, 5000, 200), (16, 30000, 64), (17, 30000, 64)])
def test_repeated_and_captured_calls_give_the_same_bits(rows, vocab, d):
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(14, rows, vocab, d, BF)
    ids, logits = (t.cuda() for t in _entries(5, rows, vocab, 40, F, "dense"))
    cfg = _cfg(bt, vocab, d, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows, 40))
    out = [_nan(rows), _nan(rows), _nan(rows, d, dtype=BF), _nan(vocab, d, dtype=BF), _nan(rows), _nan(rows), _nan(rows, d, dtype=BF), _nan(vocab, d, dtype=BF)]

    def step():
        bt.betty_vocab_ce(cfg, x, w, target, out[0], out[1], ws)
        bt.betty_vocab_ce_backward(cfg, x, w, target, out[1], dloss, out[2], out[3], ws)
        bt.betty_vocab_distill(cfg, x, w, ids, logits, out[4], out[5], ws)
        bt.betty_vocab_distill_backward(cfg, x, w, ids, logits, out[5], dloss, out[6], out[7], ws)

    step()
    first = [t.clone() for t in out]
    step()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for t in out:
        t.fill_(float("nan"))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))
    # other inputs in the same places, and fewer rows that count
    target[::2] = -1
    x.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in out]
    step()
    assert all(torch.equal(a, b) for a, b in zip(replayed, out)) and not torch.equal(first[0], out[0])


def test_two_streams_with_a_workspace_each():
    import paper_2207_02849_b200 as bt
    problems = [_problem(s, 300, 3000, 128, BF) for s in (1, 2)]
    cfg = _cfg(bt, 3000, 128, BF)
    want = [_check_ce(bt, *p) for p in problems]
    spaces = [bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 300)) for _ in problems]
    streams = [torch.cuda.Stream() for _ in problems]
    got = [[torch.empty_like(t) for t in w] for w in want]
    torch.cuda.synchronize()
    for _ in range(10):
        for (x, w, target, dloss), ws, s, o in zip(problems, spaces, streams, got):
            bt.betty_vocab_ce(cfg, x, w, target, o[0], o[1], ws, stream=s)
            bt.betty_vocab_ce_backward(cfg, x, w, target, o[1], dloss, o[2], o[3], ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for p, q in zip(want, got) for a, b in zip(p, q))


def test_no_rows():
    import paper_2207_02849_b200 as bt
    cfg = _cfg(bt, 300, 65, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 0, 4))
    e = lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    w = torch.ones(300, 65, dtype=BF, device="cuda")
    bt.betty_vocab_ce(cfg, e(0, 65), w, e(0, dtype=torch.long), e(0, dtype=F), e(0, dtype=F), ws)
    for out in (BF, F):
        dw = _nan(300, 65, dtype=out)
        bt.betty_vocab_ce_backward(cfg, e(0, 65), w, e(0, dtype=torch.long), e(0, dtype=F), e(0, dtype=F), e(0, 65), dw, ws)
        assert bool((dw == 0).all())
        dw = _nan(300, 65, dtype=out)
        bt.betty_vocab_distill_backward(cfg, e(0, 65), w, e(0, 4, dtype=torch.long), e(0, 4), e(0, dtype=F), e(0, dtype=F), None, dw, ws)
        assert bool((dw == 0).all())


@pytest.mark.parametrize("rows", [5, 100, 128, 200, 1000, 3000])
def test_a_workspace_of_the_stated_size_is_enough(rows):
    """The size for some rows serves any fewer, and nothing behind it is written."""
    import paper_2207_02849_b200 as bt
    vocab, d, top = 2500, 72, 6
    cfg = _cfg(bt, vocab, d, HF)
    need = bt.betty_vocab_workspace_size(cfg, 3000, top)
    ws = bt.Workspace.of_bytes(need)
    x, w, target, dloss = _problem(rows, rows, vocab, d, HF)
    end = (-ws.buf.data_ptr()) % 256 + need
    ws.buf[end:] = 77
    ids, logits = (t.cuda() for t in _entries(5, rows, vocab, top, F, "any"))
    loss, lse, dx, dw = _nan(rows), _nan(rows), _nan(rows, d, dtype=HF), _nan(vocab, d, dtype=HF)
    bt.betty_vocab_distill(cfg, x, w, ids, logits, loss, lse, ws)
    for a, b in ((dx, dw), (dx, None), (None, dw)):
        bt.betty_vocab_distill_backward(cfg, x, w, ids, logits, lse, dloss, a, b, ws)
    torch.cuda.synchronize()
    assert bool((ws.buf[end:] == 77).all())
    _check_ce(bt, x, w, target, dloss, ws=ws)


# ---- the ends of the ranges ----
@pytest.mark.parametrize("rows,vocab,d", [(3, 40, 65536), (200, 300, 20000), (4, (1 << 22) - 1, 8), (150, 1 << 21, 8), (100000, 50, 16)])
def test_largest_sizes(rows, vocab, d):
    import paper_2207_02849_b200 as bt
    _check_ce(bt, *_problem(1, rows, vocab, d, BF))


def test_ids_at_the_end_of_the_largest_vocabulary():
    import paper_2207_02849_b200 as bt
    vocab = (1 << 22) - 1
    x, w, _, dloss = _problem(1, 5, vocab, 8, HF, boost=0.0)
    ids = torch.full((5, 1024), -1, device="cuda")
    ids[:, -3:] = torch.tensor([vocab - 1, 0, vocab - 2], device="cuda")
    ids[0, :] = vocab - 1
    _check_distill(bt, x, w, ids, torch.randn(5, 1024, device="cuda"), dloss)


def test_offsets_beyond_32_bits():
    """Leading dimensions of 2^20: the last of 2500 rows begin behind 2^31 values."""
    import paper_2207_02849_b200 as bt

    def far(t):
        v = torch.empty(t.shape[0], 1 << 20, dtype=t.dtype, device="cuda")[:, :t.shape[1]]
        v.copy_(t)
        return v
    _check_ce(bt, *_problem(1, 2500, 2300, 64, BF), wrap=far)


@pytest.mark.parametrize("d,pad", [(67, 5), (65, 7), (130, 6), (3, 5)])
@pytest.mark.parametrize("out", [BF, F])
def test_aligned_results_of_odd_widths_leave_their_neighbours(d, pad, out):
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(6, 150, 401, d, BF)
    cfg = _cfg(bt, 401, d, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 150))
    lse = torch.logsumexp(x.float() @ w.float().t(), 1)
    bx, bw = torch.full((150, d + pad), 7.0, dtype=out, device="cuda"), torch.full((401, d + pad), 7.0, dtype=out, device="cuda")
    dx, dw = _nan(150, d, dtype=out), _nan(401, d, dtype=out)
    bt.betty_vocab_ce_backward(cfg, x, w, target, lse, dloss, bx[:, :d], bw[:, :d], ws)
    bt.betty_vocab_ce_backward(cfg, x, w, target, lse, dloss, dx, dw, ws)
    for b, t in ((bx, dx), (bw, dw)):
        assert bool((b[:, d:] == 7).all()) and torch.equal(b[:, :d], t)


def test_a_matrix_that_cannot_be_read_in_place_needs_room():
    """The refusal comes before anything is launched.  (Both gradients against a teacher take all of a workspace of the stated size;
    other calls may find room in what they do not need themselves.)"""
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(6, 30, 401, 64, BF)
    w1 = _wide(3, 0)(w)
    ids, logits = (t.cuda() for t in _entries(5, 30, 401, 7, F, "any"))
    cfg = _cfg(bt, 401, 64, BF)
    lse, dx, dw = torch.zeros(30, device="cuda"), _nan(30, 64, dtype=BF), _nan(401, 64, dtype=BF)
    torch.cuda.synchronize()
    for top, call in ((0, lambda ws: bt.betty_vocab_ce_backward(cfg, x, w1, target, lse, dloss, dx, dw, ws)),
                      (7, lambda ws: bt.betty_vocab_distill_backward(cfg, x, w1, ids, logits, lse, dloss, dx, dw, ws))):
        small = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 30, top, any_layout=False))
        before = bt.betty_kernel_launches()
        with pytest.raises(bt.BettyError) as e:
            call(small)
        assert e.value.status == bt.BETTY_ERR_WORKSPACE and bt.betty_kernel_launches() == before
        call(bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 30, top, any_layout=True)))


def test_a_matrix_changed_just_before_the_call():
    """W is asked for while its rows are counted: what the stream has written to it before is what counts."""
    import paper_2207_02849_b200 as bt
    x, w, target, dloss = _problem(16, 16, 40000, 512, BF)
    cfg = _cfg(bt, 40000, 512, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 16))
    loss, lse = _nan(16), _nan(16)
    for k in range(6):
        other = torch.randn_like(w)
        w.copy_(other * 0.05)
        bt.betty_vocab_ce(cfg, x, w, target, loss, lse, ws)
        w2 = w.clone()
        w.zero_()
        e = ref.Expected(x, w2, ref.entries_ce(target, 40000, 0.0))
        e.check_forward(loss, lse)
