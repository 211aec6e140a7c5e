"""Losses over a vocabulary at the ends of their ranges."""
import pytest
import torch

from tests.test_gpu_vocab_loss import BF, F, _cfg, _ok

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
