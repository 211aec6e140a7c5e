"""Matrix products grouped by expert against 64-bit products of the same values.

Tolerance.  Products of 16-bit values are exact in fp32; the tensor cores add 16 of them at a time to an fp32 sum, each
addition off by at most one unit of the last place (2^-23) of the magnitudes added: an element is within
(depth / 16 + 8) * 2^-23 of the sum of magnitudes, plus one rounding to the result's type."""
import pytest
import torch

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def _rand(g, *shape, dtype):
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def _offsets(counts):
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    return o, torch.tensor(o, dtype=torch.int32, device="cuda")


def _problem(seed, counts, spare, n_in, n_out, dtype):
    g = torch.Generator().manual_seed(seed)
    o, offsets = _offsets(counts)
    rows = o[-1] + spare
    return o, offsets, _rand(g, rows, n_in, dtype=dtype), _rand(g, len(counts), n_out, n_in, dtype=dtype), _rand(g, rows, n_out, dtype=dtype)


def _product(a, b):
    """64-bit product and the product of the magnitudes."""
    a, b = a.double(), b.double()
    return a @ b, a.abs() @ b.abs()


def _near(got, want, size, depth, dtype):
    unit = 0.0 if dtype == F else ref.UNIT[dtype]
    tiny = 2.0 ** -25 if dtype == HF else 0.0
    bound = unit * want.abs() * 1.001 + tiny + (depth / 16 + 8) * 2.0 ** -23 * size
    return bool(((got.double() - want).abs() <= bound).all())


def _check(bt, counts, spare, n_in, n_out, dtype, out=None, wrap=lambda t: t, any_layout=None, seed=0, ws=None):
    out = out or dtype
    o, offsets, x, w, dy = _problem(seed, counts, spare, n_in, n_out, dtype)
    rows, e = x.shape[0], len(counts)
    cfg = bt.Grouped(e, n_in, n_out, bt.BETTY_BF16 if dtype == BF else bt.BETTY_F16)
    ws = ws or bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, rows, any_layout))
    nan = lambda *s: wrap(torch.full(s, float("nan"), dtype=out, device="cuda"))  # noqa: E731
    y, dx, dw = nan(rows, n_out), nan(rows, n_in), nan(e, n_out, n_in)
    xs, w_, dys = wrap(x), wrap(w), wrap(dy)
    bt.betty_grouped_forward(cfg, offsets, xs, w_, y, ws)
    bt.betty_grouped_backward_data(cfg, offsets, dys, w_, dx, ws)
    bt.betty_grouped_backward_weight(cfg, offsets, dys, xs, dw, ws)
    assert bt.betty_poll_status(ws, raise_on_error=False)[0] == bt.BETTY_OK
    for i in range(e):
        a, b = o[i], o[i + 1]
        assert _near(y[a:b], *_product(x[a:b], w[i].t()), n_in, out), ("y", i)
        assert _near(dx[a:b], *_product(dy[a:b], w[i]), n_out, out), ("dx", i)
        assert _near(dw[i], *_product(dy[a:b].t(), x[a:b]), b - a, out), ("dw", i)
    assert not torch.isnan(y).any() and not torch.isnan(dx).any()
    if spare:
        assert float(y[o[-1]:].abs().max()) == 0.0 and float(dx[o[-1]:].abs().max()) == 0.0
    return y, dx, dw


COUNTS = [[1], [0, 1, 0], [5, 0, 17, 64, 3], [128, 128], [129, 300, 31, 0, 513], [700, 20], [0, 0], [33] * 9, [256, 257, 255]]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("n_in,n_out", [(64, 64), (128, 256), (200, 136), (320, 520), (8, 8), (1000, 72)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_products(counts, n_in, n_out, dtype):
    import paper_2207_02849_b200 as bt
    _check(bt, counts, 3 if sum(counts) % 2 else 0, n_in, n_out, dtype, seed=sum(counts) + n_in) if sum(counts) else \
        _check(bt, counts, 4, n_in, n_out, dtype)


@pytest.mark.parametrize("counts", [[1], [5, 0, 30], [64], [40, 55, 0, 61], [100, 90]], ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("n_in,n_out", [(4096, 200), (2056, 1032), (520, 130)])
def test_few_rows_and_long_contractions(counts, n_in, n_out):
    """Tiles whose contraction is shared by several CTAs."""
    import paper_2207_02849_b200 as bt
    for dtype in (BF, HF):
        _check(bt, counts, 1, n_in, n_out, dtype, seed=n_in + sum(counts))
        _check(bt, counts, 0, n_out, n_in, dtype, out=F, seed=n_in + sum(counts))


@pytest.mark.parametrize("n_in,n_out", [(1, 1), (7, 64), (64, 7), (129, 257), (1001, 33)])
@pytest.mark.parametrize("counts", [[3, 0, 70], [300, 161]])
def test_odd_widths(counts, n_in, n_out):
    import paper_2207_02849_b200 as bt
    _check(bt, counts, 5, n_in, n_out, BF, seed=3)


@pytest.mark.parametrize("out", [F, BF])
@pytest.mark.parametrize("counts", [[7, 9], [400, 100, 250]])
def test_fp32_results(out, counts):
    import paper_2207_02849_b200 as bt
    _check(bt, counts, 0, 512, 384, BF, out=out, seed=9)


def _wide(pad, shift):
    def wrap(t):
        buf = torch.full((*t.shape[:-1], t.shape[-1] + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
        v = buf[..., shift:shift + t.shape[-1]]
        v.copy_(t)
        return v
    return wrap


@pytest.mark.parametrize("pad,shift,n_in,n_out", [(8, 8, 128, 72), (3, 0, 128, 72), (0, 1, 136, 264), (7, 2, 65, 130)])
@pytest.mark.parametrize("counts", [[20, 0, 45], [260, 190]])
def test_rows_of_wider_buffers(pad, shift, n_in, n_out, counts):
    """What lies beside the rows is NaN: nothing of it may reach a sum."""
    import paper_2207_02849_b200 as bt
    _check(bt, counts, 2, n_in, n_out, BF, wrap=_wide(pad, shift), any_layout=True, seed=5)


def test_non_finite_rows_stay_with_their_expert():
    import paper_2207_02849_b200 as bt
    for counts in ([37, 100, 59], [300, 277, 333]):
        o, offsets, x, w, dy = _problem(1, counts, 6, 256, 320, BF)
        cfg = bt.Grouped(3, 256, 320)
        ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, x.shape[0]))
        clean = [torch.empty_like(dy), torch.empty_like(x), torch.empty_like(w)]
        dirty = [torch.empty_like(t) for t in clean]
        for outs in (clean, dirty):
            bt.betty_grouped_forward(cfg, offsets, x, w, outs[0], ws)
            bt.betty_grouped_backward_data(cfg, offsets, dy, w, outs[1], ws)
            bt.betty_grouped_backward_weight(cfg, offsets, dy, x, outs[2], ws)
            torch.cuda.synchronize()
            x[o[1]:o[2]] = float("nan")
            dy[o[1]:o[2]] = float("inf")
            x[o[3]:] = float("nan")
            dy[o[3]:] = float("nan")
            w[1] = float("nan")
        for c, d in zip(clean[:2], dirty[:2]):
            assert torch.equal(c[:o[1]], d[:o[1]]) and torch.equal(c[o[2]:], d[o[2]:])
            assert float(d[o[3]:].abs().max()) == 0.0
        assert torch.equal(clean[2][0], dirty[2][0]) and torch.equal(clean[2][2], dirty[2][2])


def test_no_rows_many_groups_and_repeatability():
    import paper_2207_02849_b200 as bt
    cfg = bt.Grouped(3, 64, 72)
    ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, 0))
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    e = lambda n: torch.empty(0, n, dtype=BF, device="cuda")  # noqa: E731
    dw = torch.full((3, 72, 64), float("nan"), dtype=BF, device="cuda")
    bt.betty_grouped_forward(cfg, offsets, e(64), dw, e(72), ws)
    bt.betty_grouped_backward_data(cfg, offsets, e(72), dw, e(64), ws)
    bt.betty_grouped_backward_weight(cfg, offsets, e(72), e(64), dw, ws)
    assert bt.betty_poll_status(ws)[0] == bt.BETTY_OK and float(dw.abs().max()) == 0.0
    counts = [(i * 7) % 5 for i in range(1000)]
    first = _check(bt, counts, 1, 72, 64, HF, seed=4)
    again = _check(bt, counts, 1, 72, 64, HF, seed=4)
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_offsets_out_of_order_or_range_are_clamped_and_reported():
    import paper_2207_02849_b200 as bt
    for bad in ([0, 50, 20, 100], [0, 50, 400, 100], [-7, 10, 20, 100], [0, -5, 60, 1 << 30], [3, 10, 20, 100]):
        _, _, x, w, dy = _problem(2, [40, 30, 30], 0, 128, 192, BF)
        cfg = bt.Grouped(3, 128, 192)
        ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, 100))
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        guard = torch.full((102, 192), 7.0, dtype=BF, device="cuda")
        y = guard[1:101]
        bt.betty_grouped_forward(cfg, offsets, x, w, y, ws)
        assert bt.betty_poll_status(ws, raise_on_error=False)[0] == bt.BETTY_ERR_INVALID_ARG
        bt.betty_reset_status(ws)
        bt.betty_grouped_backward_weight(cfg, offsets, dy, x, torch.empty_like(w), ws)
        assert bt.betty_poll_status(ws, raise_on_error=False)[0] == bt.BETTY_ERR_INVALID_ARG
        assert bool((guard[0] == 7).all()) and bool((guard[101] == 7).all())


def test_gradients_against_differences():
    """Central differences of sum(dy * y) along directions of x and w: y is linear in each, so the difference is exact up to
    the roundings of fp32 sums and of the moved 16-bit inputs (moved by whole steps of their own type)."""
    import paper_2207_02849_b200 as bt
    o, offsets, x, w, dy = _problem(11, [30, 0, 90, 11], 0, 96, 80, HF)
    cfg = bt.Grouped(4, 96, 80, bt.BETTY_F16)
    ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, 131))
    dx, dw = torch.empty(131, 96, device="cuda"), torch.empty(4, 80, 96, device="cuda")
    bt.betty_grouped_backward_data(cfg, offsets, dy, w, dx, ws)
    bt.betty_grouped_backward_weight(cfg, offsets, dy, x, dw, ws)

    def value(x, w):
        y = torch.empty(131, 80, device="cuda")
        bt.betty_grouped_forward(cfg, offsets, x, w, y, ws)
        return float((y.double() * dy.double()).sum())

    g = torch.Generator().manual_seed(3)
    for base, grad, move in ((x, dx, lambda t: (t, w)), (w, dw, lambda t: (x, t))):
        dirn = torch.randn(base.shape, generator=g).half().cuda()
        up, down = base + dirn, base - dirn
        step = up.double() - down.double()
        diff = value(*move(up)) - value(*move(down))
        want = float((grad.double() * step).sum())
        assert abs(diff - want) <= 1e-4 * float(grad.double().norm() * step.norm()) / step.numel() ** 0.5


def test_refusals_of_the_binding():
    import paper_2207_02849_b200 as bt
    cfg = bt.Grouped(2, 64, 32)
    ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, 10))
    offsets = torch.tensor([0, 4, 10], dtype=torch.int32, device="cuda")
    x, w, y = (torch.zeros(*s, dtype=BF, device="cuda") for s in ((10, 64), (2, 32, 64), (10, 32)))
    with pytest.raises(ValueError):
        bt.betty_grouped_forward(cfg, offsets.long(), x, w, y, ws)
    with pytest.raises(ValueError):
        bt.betty_grouped_forward(cfg, offsets[:2], x, w, y, ws)
    with pytest.raises(ValueError):
        bt.betty_grouped_forward(cfg, offsets, x.half(), w, y, ws)
    with pytest.raises(ValueError):
        bt.betty_grouped_forward(cfg, offsets, x, w.transpose(1, 2), y, ws)
    with pytest.raises(ValueError):
        bt.betty_grouped_forward(cfg, offsets, x, w, y[:9], ws)
    for status, call in (
            (bt.BETTY_ERR_DTYPE, lambda: bt.betty_grouped_forward(cfg, offsets, x, w, y.half(), ws)),
            (bt.BETTY_ERR_SHAPE, lambda: bt.betty_grouped_forward(cfg, offsets, x[:1].expand(10, 64), w, y, ws)),
            (bt.BETTY_ERR_SHAPE, lambda: bt.betty_grouped_forward(cfg, offsets, x, w[:1].expand(2, 32, 64), y, ws)),
            (bt.BETTY_ERR_WORKSPACE, lambda: bt.betty_grouped_forward(cfg, offsets, _wide(1, 0)(x), w, y, ws)),
            (bt.BETTY_ERR_DTYPE, lambda: bt.betty_grouped_workspace_size(bt.Grouped(2, 64, 32, bt.BETTY_F32), 4)),
            (bt.BETTY_ERR_SHAPE, lambda: bt.betty_grouped_workspace_size(bt.Grouped(0, 64, 32), 4)),
            (bt.BETTY_ERR_UNSUPPORTED, lambda: bt.betty_grouped_workspace_size(bt.Grouped(1025, 64, 32), 4))):
        with pytest.raises(bt.BettyError) as e:
            call()
        assert e.value.status == status
