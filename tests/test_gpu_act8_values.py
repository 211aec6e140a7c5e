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


def _every_value(dtype, low, high):
    """All numbers of a 16-bit type in [low, high]."""
    v = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32).to(torch.int16).view(dtype)
    v = v[torch.isfinite(v)]
    return v[(v.float() >= low) & (v.float() <= high)]


@pytest.mark.parametrize("dtype,low", [(HF, -9.0), (BF, -13.0)])
def test_gelu_of_16_bit_types_is_exact_in_relative_terms(dtype, low):
    """Every number of the type.  The distribution function is within 5e-6 of itself by its approximation and, its exponential
    being taken of v^2 / 2 as fp32 has it, within 7.5e-8 v^2 more (two and a half roundings) and ~1e-6 by ex2, the Horner steps and the
    reciprocal: 2e-5 for |v| <= 13.  The activation is that and one rounding, the slope (store and backward agree on v where the
    checkpoint holds v itself) that much of the sum of its two terms' magnitudes."""
    import paper_2207_02849_b200 as bt
    v = _every_value(dtype, low, 40.0)
    z = v[:, None].cuda()                                  # a group of one value: q = +-127, restored to itself within 2^-22
    cfg = bt.Act8(1, act=bt.ACT_GELU)
    q, scales = cfg.empty(len(v))
    a = torch.empty_like(z)
    bt.betty_act8_store(cfg, z, a, q, scales)
    v64 = v.double()[:, None]
    cdf = 0.5 * torch.special.erfc(-v64 / 2.0 ** 0.5)
    tiny = 2.0 ** -25 if dtype == HF else 2.0 ** -126
    bound = lambda want, size: (ref.UNIT[dtype] * want.abs() + 2e-5 * size) * 1.001 + tiny  # noqa: E731
    want = v64 * cdf
    assert float(((a.double().cpu() - want).abs() - bound(want, want.abs())).max()) <= 0
    dz, a8 = torch.empty_like(z), torch.empty_like(z)
    bt.betty_act8_backward(cfg, q, scales, torch.ones_like(z), dz, a8)
    r = ref.restored(q.cpu(), scales.cpu(), 1)
    cdf, pdf = 0.5 * torch.special.erfc(-r / 2.0 ** 0.5), torch.exp(-0.5 * r * r) / (2.0 * torch.pi) ** 0.5
    # q * scale is rounded to fp32 before its use: v^2 2^-23 more
    assert float(((a8.double().cpu() - r * cdf).abs() - bound(r * cdf, 2.0 * (r * cdf).abs())).max()) <= 0
    want = cdf + r * pdf
    assert float(((dz.double().cpu() - want).abs() - bound(want, 2.0 * (cdf + r.abs() * pdf))).max()) <= 0


def test_silu_of_fp32_values_is_exact_in_relative_terms():
    """sigmoid(v) from e = exp(-|v|): ex2 within 2^-22, its argument's rounding made good, the reciprocal and three roundings
    2^-24 to 2^-23 each: below 8e-7 of the result; the slope s (1 + v (1 - s)) below 1e-6 of the sum of its terms' magnitudes."""
    import paper_2207_02849_b200 as bt
    g = torch.Generator().manual_seed(2)
    z = torch.cat((torch.linspace(-80, 80, 20001), torch.randn(20000, generator=g) * 5.0))[:, None].cuda()
    cfg = bt.Act8(1, act=bt.ACT_SILU)
    q, scales = cfg.empty(z.shape[0])
    a = torch.empty_like(z)
    bt.betty_act8_store(cfg, z, a, q, scales)
    v = z.double().cpu()
    want = v / (1.0 + torch.exp(-v))
    assert float(((a.double().cpu() - want).abs() - 8e-7 * want.abs()).max()) <= 0
    back = torch.empty_like(z)
    bt.betty_act8_restore(cfg, q, scales, back)            # the fp32 numbers that the backward pass takes
    dz, a8 = torch.empty_like(z), torch.empty_like(z)
    bt.betty_act8_backward(cfg, q, scales, torch.ones_like(z), dz, a8)
    v = back.double().cpu()
    s, n = 1.0 / (1.0 + torch.exp(-v)), 1.0 / (1.0 + torch.exp(v))
    assert float(((a8.double().cpu() - v * s).abs() - 8e-7 * (v * s).abs()).max()) <= 0
    assert float(((dz.double().cpu() - s * (1.0 + v * n)).abs() - 1e-6 * s * (1.0 + v.abs() * n)).max()) <= 0
