"""Losses over a vocabulary against 64-bit restatements (tests/vocab_reference.py says how far they may be off)."""
import pytest
import torch

from tests import vocab_reference as ref

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32
SIZES = [(1, 8), (2, 64), (100, 1), (257, 72), (1000, 200), (4099, 515), (513, 1025), (20000, 64)]
ROWS = [1, 7, 33, 128, 129, 300, 700]


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
