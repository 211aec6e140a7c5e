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
