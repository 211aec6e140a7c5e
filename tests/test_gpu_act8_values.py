"""8-bit checkpoints over the whole range of finite values, against the 64-bit restatement."""
import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("cols,gated", [(256, False), (131, False), (128, True)])
def test_groups_with_very_large_finite_values(dtype, cols, gated):
    """The format's single fp32 operations hold up to the largest finite value: 1 / top is subnormal from top = 2^126 on, and
    127 * (1 / top) is an ordinary number again.  Numbers and scales are equal to the restatement's; a restored value is its
    exact product rounded once (2^-24, then the type), infinite where that is beyond the largest finite value."""
    import paper_2207_02849_b200 as bt
    most = torch.finfo(dtype).max
    tops = [2.0 ** 125, 2.0 ** 126, 1.0e38, 2.0 ** 127, 3.0e38, most, -most, 8.4e37]
    rows, width = len(tops), cols * (2 if gated else 1)
    g = torch.Generator().manual_seed(11)
    z = torch.randn(rows, width, generator=g)
    z[:, 0::3] *= 1e37
    for i, t in enumerate(tops):
        z[i, 5] = t
        z[i, width - 2] = -0.4 * t
        z[i, 17] = 0.99 * t
    z = z.to(dtype).cuda()
    cfg = bt.Act8(cols, act=bt.ACT_RELU, gated=gated)
    q, scales = cfg.empty(rows)
    back = torch.empty_like(z)
    bt.betty_act8_store(cfg, z, None, q, scales)
    bt.betty_act8_restore(cfg, q, scales, back)
    want_q, want_s = ref.checkpoint(z, cols)
    assert int(want_q[:, 5].abs().min()) == 127
    assert torch.equal(q.cpu(), want_q) and torch.equal(scales.cpu(), want_s)
    want = ref.restored(want_q, want_s, cols).float().to(dtype)      # the product of two fp32 values is exact in 64 bits
    assert torch.equal(back.cpu(), want)


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("dtype", [F, BF, HF])
def test_activations_at_the_ends_of_the_range(kind, dtype):
    """GELU and SiLU of the largest finite values and of +inf are the value itself, of the lowest finite value 0; NaN stays."""
    import paper_2207_02849_b200 as bt
    most = torch.finfo(dtype).max
    z = torch.tensor([most, -most, float("inf"), float("nan"), 0.0, -0.0], dtype=dtype, device="cuda")[:, None]
    cfg = bt.Act8(1, act=kind)
    q, scales = cfg.empty(6)
    a = torch.empty_like(z)
    bt.betty_act8_store(cfg, z, a, q, scales)
    a = a[:, 0].float().cpu()
    assert float(a[0]) == most and float(a[1]) == 0.0 and float(a[2]) == float("inf") and bool(torch.isnan(a[3]))
    assert float(a[4]) == 0.0 and float(a[5]) == 0.0
