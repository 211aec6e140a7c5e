"""8-bit checkpoints of a hidden layer and the backward pass from them, against the 64-bit restatement.

The whole numbers and scales are defined by single fp32 operations and have to be equal.  Activations and gradients are
products of at most three fp32 factors, each within 4 ulp or 3e-7 absolute (the 16-bit types' distribution function): 1e-6
of the element's own inputs, plus one rounding to the type."""
import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32
ACTS = ("relu", "gelu", "silu")
SLACK = 2e-6
SIZES = [(1, 1), (1, 8), (3, 7), (2, 127), (4, 128), (5, 129), (17, 1000), (9, 1001), (300, 96), (2, 4096), (3, 20000), (40, 2053)]


def _z(seed, rows, width, dtype):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, width, generator=g)
    z[:, ::17] *= 6.0
    return z.to(dtype).cuda()


def _wide(t, pad, shift):
    buf = torch.zeros(t.shape[0], t.shape[1] + pad + shift, dtype=t.dtype, device="cuda")
    v = buf[:, shift:shift + t.shape[1]]
    v.copy_(t)
    return v


def _check(bt, z, cols, kind, gated, wrap=lambda t: t):
    rows, t = z.shape[0], z.dtype
    cfg = bt.Act8(cols, act=ACTS.index(kind), gated=gated)
    q, scales = cfg.empty(rows)
    q.fill_(99)
    scales.fill_(-1.0)
    q, scales = wrap(q), wrap(scales)
    a = wrap(torch.full((rows, cols), float("nan"), dtype=t, device="cuda"))
    bt.betty_act8_store(cfg, wrap(z), a, q, scales)
    want_q, want_s = ref.checkpoint(z, cols)
    assert torch.equal(q.cpu(), want_q)
    assert torch.equal(scales.cpu(), want_s)
    z64 = ref.d64(z)
    scale = z64.abs().clamp(min=1e-3)
    scale = scale[:, :cols] * scale[:, cols:] if gated else scale
    assert ref.close(a, ref.hidden(z64, cols, kind, gated), t, SLACK, scale=scale) <= 0
    back = wrap(torch.full_like(z, float("nan")))
    bt.betty_act8_restore(cfg, q, scales, back)
    z8 = ref.restored(want_q, want_s, cols)
    assert ref.close(back, z8, t, 1e-7, scale=z8.abs()) <= 0
    # the checkpoint is within half a step of what it was made of
    step = ref.restored(torch.ones_like(want_q), want_s, cols)
    assert float(((z8 - z64).abs() - 0.5001 * step).max()) <= 0
    g = torch.Generator().manual_seed(5)
    da = torch.randn(rows, cols, generator=g).to(t).cuda()
    dz, a8 = wrap(torch.full_like(z, float("nan"))), wrap(torch.full((rows, cols), float("nan"), dtype=t, device="cuda"))
    bt.betty_act8_backward(cfg, q, scales, wrap(da), dz, a8)
    leaf = z8.clone().requires_grad_(True)
    out = ref.hidden(leaf, cols, kind, gated)
    (want,) = torch.autograd.grad(out, leaf, ref.d64(da))
    if kind == "relu":
        want = torch.where(torch.cat([z8[:, :cols] == 0] * (2 if gated else 1), 1), torch.zeros_like(want), want)   # slope 0 at 0
    z_abs = z8.abs() + 1.0
    scale = ref.d64(da).abs() * (z_abs[:, :cols] * z_abs[:, cols:] if gated else z_abs)
    scale = torch.cat((scale, scale), 1) if gated else scale
    assert ref.close(dz, want, t, SLACK, scale=scale) <= 0
    scale = z_abs[:, :cols] * z_abs[:, cols:] if gated else z_abs
    assert ref.close(a8, out.detach(), t, SLACK, scale=scale) <= 0
    return cfg, q, scales, da, dz, a8


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("kind,gated", [("gelu", False), ("silu", True), ("relu", False)])
def test_store_restore_backward(rows, cols, dtype, kind, gated):
    import paper_2207_02849_b200 as bt
    _check(bt, _z(rows + cols, rows, cols * (2 if gated else 1), dtype), cols, kind, gated)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("gated", [False, True])
def test_every_activation(kind, gated):
    import paper_2207_02849_b200 as bt
    _check(bt, _z(1, 33, 272 * (2 if gated else 1), BF), 272, kind, gated)


@pytest.mark.parametrize("pad,shift", [(8, 8), (16, 0), (3, 0), (0, 1), (5, 2)])
@pytest.mark.parametrize("gated", [False, True])
def test_rows_of_wider_buffers(pad, shift, gated):
    import paper_2207_02849_b200 as bt
    _check(bt, _z(2, 19, 264 * (2 if gated else 1), HF), 264, "silu", gated, wrap=lambda t: _wide(t, pad, shift))


def test_groups_of_zeros_of_tiny_and_of_non_finite_values():
    import paper_2207_02849_b200 as bt
    z = _z(3, 6, 384, F)
    z[0, :128] = 0.0
    z[1, 128:256] = 1e-33
    z[2, 5] = float("inf")
    z[3, 300] = float("nan")
    z[4, 130] = -float("inf")
    cfg = bt.Act8(384, act=bt.ACT_GELU)
    q, scales = cfg.empty(6)
    back = torch.empty_like(z)
    bt.betty_act8_store(cfg, z, None, q, scales)
    bt.betty_act8_restore(cfg, q, scales, back)
    want_q, want_s = ref.checkpoint(z, 384)
    assert torch.equal(q.cpu(), want_q)
    assert torch.equal(torch.nan_to_num(scales.cpu(), nan=-1.0), torch.nan_to_num(want_s, nan=-1.0))
    assert float(back[0, :128].abs().max()) == 0.0 and float(back[1, 128:256].abs().max()) == 0.0
    bad = torch.isnan(back)
    assert bool(bad[2, :128].all()) and bool(bad[3, 256:].all()) and bool(bad[4, 128:256].all())
    assert int(bad.sum()) == 3 * 128                               # and nothing else


def test_parts_left_out_and_no_rows():
    import paper_2207_02849_b200 as bt
    z = _z(4, 30, 512, BF)
    cfg, q, scales, da, dz, a8 = _check(bt, z, 256, "silu", True)
    only = torch.empty_like(dz)
    bt.betty_act8_backward(cfg, q, scales, da, only, None)
    assert torch.equal(only, dz)
    only = torch.empty_like(a8)
    bt.betty_act8_backward(cfg, q, scales, None, None, only)
    assert torch.equal(only, a8)
    e, (q0, s0) = torch.empty(0, 512, dtype=BF, device="cuda"), cfg.empty(0)
    bt.betty_act8_store(cfg, e, None, q0, s0)
    bt.betty_act8_restore(cfg, q0, s0, e)
    bt.betty_act8_backward(cfg, q0, s0, e[:, :256].contiguous(), e, None)


def test_gradient_against_differences():
    """dz against central differences of sum(da * a) along a direction, a from the checkpoint's values moved by +-h:
    h = 2^-7, smooth activations, fp32: error h^2 / 6 + 2^-24 |L| / h, below 1e-3 of the gradient's size."""
    import paper_2207_02849_b200 as bt
    for kind, gated in (("gelu", False), ("silu", True)):
        z = _z(6, 7, 200 * (2 if gated else 1), F)
        cfg, q, scales, da, dz, _ = _check(bt, z, 200, kind, gated)
        z8 = torch.empty_like(z)
        bt.betty_act8_restore(cfg, q, scales, z8)
        g = torch.Generator().manual_seed(1)
        dirn = torch.randn(z.shape, generator=g).cuda()
        h = 2.0 ** -7

        def value(v):
            a = torch.empty(7, 200, device="cuda")
            bt.betty_act8_store(cfg, v, a, q.clone(), scales.clone())
            return float((a.double() * da.double()).sum())

        diff = (value(z8 + h * dirn) - value(z8 - h * dirn)) / (2 * h)
        want = float((dz.double() * dirn.double()).sum())
        assert abs(diff - want) <= 2e-3 * float(dz.double().norm())


def test_rows_beyond_32_bits_of_values():
    """A checkpoint whose rows start beyond 2^32 values: int8, 70000 rows of 65536 (4.6 GB)."""
    import paper_2207_02849_b200 as bt
    rows, cols = 70000, 65536
    cfg = bt.Act8(cols, act=bt.ACT_RELU)
    q, scales = cfg.empty(rows)
    q.fill_(3)
    scales.fill_(0.5)
    z = torch.empty(rows, cols, dtype=BF, device="cuda")
    q[-1, -7:] = -2
    bt.betty_act8_restore(cfg, q, scales, z)
    assert float(z[-1, -7:].float().max()) == -1.0 and float(z[-1, :-7].float().min()) == 1.5
    assert float(z[rows - 200:].double().sum()) == 1.5 * (200 * cols - 7) - 7.0


def test_refusals_of_the_binding():
    import paper_2207_02849_b200 as bt
    cfg = bt.Act8(64)
    q, s = cfg.empty(4)
    z = torch.zeros(4, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        bt.betty_act8_store(cfg, z, None, q[:3], s)
    with pytest.raises(ValueError):
        bt.betty_act8_store(cfg, z, z.float(), q, s)
    with pytest.raises(ValueError):
        bt.betty_act8_store(cfg, z.to(torch.int32), None, q, s)
    with pytest.raises(ValueError):
        bt.betty_act8_restore(cfg, q.float(), s, z)
    with pytest.raises(bt.BettyError) as e:
        bt.betty_act8_backward(cfg, q, s, None, z, None)
    assert e.value.status == bt.BETTY_ERR_INVALID_ARG
    with pytest.raises(bt.BettyError) as e:
        bt.betty_act8_restore(cfg, q[:1].expand(4, 64), s, z)
    assert e.value.status == bt.BETTY_ERR_SHAPE
    with pytest.raises(bt.BettyError) as e:
        bt.betty_act8_store(bt.Act8(64, act=7), z, None, q, s)
    assert e.value.status == bt.BETTY_ERR_INVALID_ARG
