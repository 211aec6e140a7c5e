"""Calls of the vocabulary losses that are decided before anything touches a device."""
import ctypes as C

import pytest

P = 1 << 20          # an aligned address that no call here reads


@pytest.fixture(scope="module")
def bt():
    from paper_2207_02849_b200 import build
    build.build()
    import paper_2207_02849_b200 as bt
    return bt


def test_an_empty_batch_without_a_weight_gradient(bt):
    """The gradient of no rows has no values and so no address: a call that wants it alone has nothing to do."""
    from paper_2207_02849_b200 import binding
    c = C.byref(binding._VocabCfg(300, 64, bt.BETTY_BF16, 1.0, 0.0, 0.0))
    ce = lambda rows, dx: bt.lib().betty_vocab_ce_backward(c, rows, P, 64, P, 64, P, 4, P, P, dx, 64, 1, None, 64, 1, P, 1 << 30, None)  # noqa: E731
    kd = lambda rows, dx: bt.lib().betty_vocab_distill_backward(c, rows, P, 64, P, 64, 5, P, 5, 4, P, 5, 0, P, P, dx, 64, 1, None, 64, 1, P, 1 << 30, None)  # noqa: E731
    for call in (ce, kd):
        assert call(0, None) == bt.BETTY_OK and call(0, P) == bt.BETTY_OK
        assert call(3, None) == bt.BETTY_ERR_INVALID_ARG


class _Fake:
    """As much of a tensor as is looked at before a call is made."""

    def __init__(self, device):
        self.device, self.shape = f"cuda:{device}", (4, 64)
        self.get_device = lambda: device


@pytest.mark.parametrize("call,n", [("betty_vocab_ce", 5), ("betty_vocab_ce_backward", 7), ("betty_vocab_distill", 6), ("betty_vocab_distill_backward", 8)])
def test_tensors_and_workspaces_of_another_device(bt, monkeypatch, call, n):
    """The current device is 1: whatever lies on 0 is refused, the workspace too, before the library is called."""
    from paper_2207_02849_b200 import binding
    monkeypatch.setattr(binding, "_raw_device", lambda: 1)
    monkeypatch.setattr(binding.torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    cfg = bt.VocabLoss(100, 64)
    for odd in range(n + 1):
        ws = binding.Workspace.__new__(binding.Workspace)
        ws.ptr, ws.nbytes, ws.buf = P, 1 << 30, _Fake(0 if odd == n else 1)
        with pytest.raises(ValueError, match="on cuda:0, the current device is cuda:1"):
            getattr(bt, call)(cfg, *[_Fake(0 if i == odd else 1) for i in range(n)], ws)
