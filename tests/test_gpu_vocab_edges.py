"""Losses over a vocabulary at the ends of their ranges."""
import pytest
import torch

from tests import vocab_reference as ref
from tests.test_gpu_vocab_loss import BF, F, HF, _cfg, _check_ce, _check_distill, _entries, _nan, _ok, _problem

pytestmark = pytest.mark.gpu


def test_an_empty_batch_without_a_weight_gradient():
    import paper_2207_02849_b200 as bt
    from paper_2207_02849_b200.language_head import LanguageHead
    cfg = _cfg(bt, 300, 64, BF)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, 0, 4))
    e = lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    w, rows = torch.ones(300, 64, dtype=BF, device="cuda"), (e(0, dtype=F), e(0, dtype=F))
    for out in (BF, F):
        bt.betty_vocab_ce_backward(cfg, e(0, 64), w, e(0, dtype=torch.long), *rows, e(0, 64, dtype=out), None, ws)
        bt.betty_vocab_distill_backward(cfg, e(0, 64), w, e(0, 4, dtype=torch.long), e(0, 4), *rows, e(0, 64, dtype=out), None, ws)
    head = LanguageHead(300, 64, 8, 4)
    for _, kept in (head.forward(w, e(0, 64), e(0, dtype=torch.long)), head.forward_teacher(w, e(0, 64), e(0, 4, dtype=torch.long), e(0, 4))):
        for wants in (("u",), ("w",), ("u", "w")):
            got = head.backward(w, kept, rows[0], wants)
            assert sorted(got) == sorted(wants) and ("u" not in got or got["u"].shape == (0, 64)) and ("w" not in got or bool((got["w"] == 0).all()))
    _ok(bt, head.ws)


@pytest.mark.parametrize("teacher", [F, BF, HF])
@pytest.mark.parametrize("temperature", [1e-3, 0.5, 1.0, 3.0])
def test_teachers_with_logits_at_the_ends_of_their_type(teacher, temperature):
    """Finite logits are entries however large they are: a mask of the type's lowest value beside others has no share, alone it is a uniform
    distribution; the quotient by a temperature below one need not be a number of fp32.
    A q below 2^-126 is subnormal and may count as zero: beside the reference's tolerances a coefficient may be off by 2^-126 |g| / T."""
    import paper_2207_02849_b200 as bt
    rows, vocab, d, top = 60, 500, 64, 8
    x, w, _, dloss = _problem(5, rows, vocab, d, BF, boost=0.0)
    g = torch.Generator().manual_seed(1)
    ids = torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(rows)]).cuda()
    t = torch.randn(rows, top, generator=g)
    low, high = torch.finfo(teacher).min, torch.finfo(teacher).max
    t[0::6] = low
    t[1::6, 2:] = low
    t[2::6, 3] = high
    t[3::6] = high
    t[4::6, :4], t[4::6, 4:] = low, high
    t = t.to(teacher).cuda()
    cfg = _cfg(bt, vocab, d, BF, temperature=temperature)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows, top))
    loss, lse, dx, dw = _nan(rows), _nan(rows), _nan(rows, d, dtype=BF), _nan(vocab, d, dtype=BF)
    bt.betty_vocab_distill(cfg, x, w, ids, t, loss, lse, ws)
    bt.betty_vocab_distill_backward(cfg, x, w, ids, t, lse, dloss, dx, dw, ws)
    _ok(bt, ws)
    e = ref.Expected(x, w, ref.entries_distill(ids, t, vocab, temperature), temperature, distill=True)
    assert bool(e.live.all())
    e.check_forward(loss, lse)
    (wx, ex), (ww, ew) = e.gradients(dloss)
    tiny = 2.0 ** -126 * dloss.double().abs()[:, None] / temperature
    assert ref.near(dx, wx, ex + tiny * w.double().abs().sum(0))
    assert ref.near(dw, ww, ew + (tiny * x.double().abs()).sum(0))


@pytest.mark.parametrize("rows", [20, 200])
@pytest.mark.parametrize("dtype,low,high,temperature", [(HF, 114, 118, 1.0), (BF, 114, 118, 1.0), (HF, -116, -112, 1.0), (HF, -14, -10, 1e30), (HF, 14, 18, 1e-30), (BF, 14, 18, 1e-30)])
def test_weights_at_the_ends_of_the_range(rows, dtype, low, high, temperature):
    """Gradients are as near, relative to their rows' weights over the temperature, as those of weights near one; results below the normal
    numbers of fp32 may be zero."""
    import paper_2207_02849_b200 as bt
    vocab, d = 700, 72
    x, w, target, _ = _problem(3, rows, vocab, d, dtype)
    dloss = torch.logspace(low, high, rows, base=2.0, device="cuda") * torch.where(torch.arange(rows, device="cuda") % 2 == 0, 1.0, -1.0)
    if temperature < 1.0:
        w.zero_()                                  # logits that are zero whatever they are divided by
    cfg = _cfg(bt, vocab, d, dtype, temperature=temperature)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows))
    e = ref.Expected(x, w, ref.entries_ce(target, vocab, 0.0), temperature)
    dx, dw = _nan(rows, d), _nan(vocab, d)
    bt.betty_vocab_ce_backward(cfg, x, w, target, e.lse.float(), dloss, dx, dw, ws)
    for got, (want, off) in zip((dx, dw), e.gradients(dloss)):
        small = torch.where(want.abs() <= 2.0 ** -125, 2.0 ** -125, 0.0)
        assert bool(((got.double() - want).abs() <= off + small).all())


@pytest.mark.parametrize("rows", [40, 600])
@pytest.mark.parametrize("smoothing", [0.0, 1.0])
def test_sums_over_the_largest_vocabulary(rows, smoothing):
    """Half tiles that all have the same sum, 1 + 127 exp(-0.65625): added one after the other, 2048 of them a thread, every addition rounds
    the same way, and the logarithm ends 3.0e-5 off, where 1.2e-5 is allowed."""
    import paper_2207_02849_b200 as bt
    vocab, d = (1 << 22) - 128, 8
    w = torch.zeros(vocab, d, dtype=BF, device="cuda")
    w[:, 0] = -0.65625
    w[::128, 0] = 0.0
    x = torch.zeros(rows, d, dtype=BF, device="cuda")
    x[:, 0] = 1.0
    target = torch.full((rows,), 5, device="cuda")
    cfg = _cfg(bt, vocab, d, BF, smoothing=smoothing)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows))
    loss, lse = _nan(rows), _nan(rows)
    bt.betty_vocab_ce(cfg, x, w, target, loss, lse, ws)
    _ok(bt, ws)
    one = ref.Expected(x[:1], w, ref.entries_ce(target[:1], vocab, smoothing), smoothing=smoothing)
    assert float((lse.double() - one.lse).abs().max()) <= float(one.e_lse)
    assert float((loss.double() - one.loss).abs().max()) <= float(one.e_loss)


@pytest.mark.parametrize("size", [1.0, 0.03])
@pytest.mark.parametrize("low", [-16, -22, -30])
def test_half_precision_matrix_gradient_of_small_weights(size, low):
    """Rows whose bound |dloss| (1 + 2 zeta |lse|) / T is 2^-6 of the largest or less, B: their coefficients are stored with bounds in
    [2^7, 2^8), and x times a power of two, off by half of the type's smallest step, 2^-25, where it leaves the normal numbers.  Brought
    back by at most B 2^-13, that is 2^-30 B of a row, times its |dz| over its bound."""
    import paper_2207_02849_b200 as bt
    rows, vocab, d = 300, 1200, 96
    x, w, target, _ = _problem(21, rows, vocab, d, HF, ignored=0.0, boost=0.0)
    x = (x.float() * size).to(HF)
    dloss = torch.ones(rows, device="cuda")
    dloss[2:] = torch.logspace(low, low + 3, rows - 2, base=2.0, device="cuda")
    z_loss = 0.01
    cfg = _cfg(bt, vocab, d, HF, z_loss=z_loss)
    ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, rows))
    e = ref.Expected(x, w, ref.entries_ce(target, vocab, 0.0), z_loss=z_loss)
    dw = _nan(vocab, d)
    bt.betty_vocab_ce_backward(cfg, x, w, target, e.lse.float(), dloss, None, dw, ws)
    _, (ww, ew) = e.gradients(dloss)
    factor = 1 + 2 * z_loss * e.lse.abs()
    q = torch.exp(x.double() @ w.double().t() - e.lse[:, None])
    dz = (q * factor[:, None]).scatter_add(1, target[:, None], -torch.ones(rows, 1, dtype=torch.float64, device="cuda"))
    lost = 2.0 ** -30 * float((dloss.double() * factor).max()) * (dz[2:].abs() / factor[2:, None]).sum(0)[:, None] * 1.01
    assert bool(((dw.double() - ww).abs() <= ew + lost).all()), float(((dw.double() - ww).abs() - ew - lost).max())


def _pieces(rows, vocab):
    """Columns of the vocabulary that are taken at a time: 2^27 coefficients, rows to multiples of 256, in pieces of about the same size."""
    fits = (1 << 27) // (-(-rows // 256) * 256) // 256 * 256
    return -(-(-(-vocab // -(-vocab // fits))) // 256) * 256


@pytest.mark.parametrize("dtype,d,out", [(BF, 72, None), (HF, 72, F), (HF, 65, None), (BF, 67, F)])
def test_distillation_over_several_pieces_of_the_vocabulary(dtype, d, out):
    """Entries in each piece, on both sides of their borders, twice the same, and none."""
    import paper_2207_02849_b200 as bt
    rows, vocab, top = 16384, 20000, 9
    piece = _pieces(rows, vocab)
    assert piece < vocab
    x, w, _, dloss = _problem(9, rows, vocab, d, dtype, boost=0.0)
    ids, logits = _entries(2, rows, vocab, top, F, "any")
    border = torch.tensor([0, piece - 1, piece, piece, 2 * piece - 1, 2 * piece, vocab - 1, vocab, -1])
    ids[::3] = border
    ids[1::7] = -1
    _check_distill(bt, x, w, ids.cuda(), logits.cuda(), dloss, 1.5, out=out)


@pytest.mark.parametrize("dtype,d,out", [(HF, 64, None), (HF, 67, None), (BF, 65, F)])
def test_cross_entropy_over_several_pieces_of_the_vocabulary(dtype, d, out):
    """Smoothed labels and z-loss, rows of all weights, results that are stored with and without TMA."""
    import paper_2207_02849_b200 as bt
    rows, vocab = 16384, 20000
    x, w, target, dloss = _problem(10, rows, vocab, d, dtype)
    piece = _pieces(rows, vocab)
    target[:6] = torch.tensor([0, piece - 1, piece, 2 * piece - 1, 2 * piece, vocab - 1], device="cuda")
    _check_ce(bt, x, w, target, dloss, out=out, smoothing=0.1, z_loss=1e-3)
