"""Gradients of the vocabulary losses against differences of the losses, row by row.

x and W are multiples of 1/16, directions too, and the steps are 1/8 and 1/16, so that the displaced points are exact in both operand types
and z is linear in the step.  The differences over both steps are extrapolated, (4 D(t / 2) - D(t)) / 3, which leaves t^4 / 480 of the fifth
derivative; how far that is from the derivative is taken from the 64-bit losses at the same points.  A loss off by e at each point puts the
extrapolated difference (4 * 2e / t + e / t) / 3 = 3 e / t off."""
import pytest
import torch

from tests import vocab_reference as ref
from tests.test_gpu_vocab_loss import BF, F, HF, _cfg, _entries, _nan

pytestmark = pytest.mark.gpu
V, D, T = 400, 48, 1.0 / 8


def _grid(seed, dtype, *shape):
    return (torch.randint(-8, 9, shape, generator=torch.Generator().manual_seed(seed)) / 16).to(dtype).cuda()


class _Loss:
    """One of the losses: the library's calls and the 64-bit statement."""

    def __init__(self, rows, dtype, distill, temperature, smoothing=0.2, z_loss=0.05):
        import paper_2207_02849_b200 as bt
        self.bt, self.rows, self.dtype, self.distill = bt, rows, dtype, distill
        self.k = dict(temperature=temperature) if distill else dict(temperature=temperature, smoothing=smoothing, z_loss=z_loss)
        self.cfg = _cfg(bt, V, D, dtype, **self.k)
        self.ws = bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(self.cfg, rows, 20))
        self.target = torch.randint(V, (rows,), generator=torch.Generator().manual_seed(rows)).cuda()
        self.ids, self.logits = (t.cuda() for t in _entries(3, rows, V, 20, F, "holes"))
        self.entries = ref.entries_distill(self.ids, self.logits, V, temperature) if distill else ref.entries_ce(self.target, V, smoothing)

    def forward(self, x, w):
        loss, lse = _nan(self.rows), _nan(self.rows)
        if self.distill:
            self.bt.betty_vocab_distill(self.cfg, x, w, self.ids, self.logits, loss, lse, self.ws)
        else:
            self.bt.betty_vocab_ce(self.cfg, x, w, self.target, loss, lse, self.ws)
        return loss.double(), lse

    def backward(self, x, w, dloss, want):
        _, lse = self.forward(x, w)
        dx, dw = (_nan(self.rows, D) if want == "x" else None), (_nan(V, D) if want == "w" else None)
        if self.distill:
            self.bt.betty_vocab_distill_backward(self.cfg, x, w, self.ids, self.logits, lse, dloss, dx, dw, self.ws)
        else:
            self.bt.betty_vocab_ce_backward(self.cfg, x, w, self.target, lse, dloss, dx, dw, self.ws)
        return (dx if want == "x" else dw).double()

    def expected(self, x, w, **other):
        return ref.Expected(x, w, self.entries, distill=self.distill, **{**self.k, **other})

    def differences(self, x, w, vx, vw):
        """Per row: the extrapolated difference of the library's losses, how far it may be from the derivative, and the same difference in 64
        bits with each term of the loss left out in turn."""
        got, want, e = {}, {}, torch.zeros(self.rows, dtype=torch.float64, device="cuda")
        without = {k: {} for k in self.k if k != "temperature"}
        for t in (T, T / 2):
            for s in (t, -t):
                a, b = x + s * vx, w + s * vw
                got[s] = self.forward(a, b)[0]
                exact = self.expected(a, b)
                want[s] = exact.loss
                e = torch.maximum(e, exact.e_loss)
                for k in without:
                    without[k][s] = self.expected(a, b, **{k: 0.0}).loss
        join = lambda l: (4 * (l[T / 2] - l[-T / 2]) / T - (l[T] - l[-T]) / (2 * T)) / 3  # noqa: E731
        return join(got), join(want), 3 * e / T, {k: join(l) for k, l in without.items()}


CASES = [(False, 1.0), (False, 2.0), (True, 1.0), (True, 0.5)]


@pytest.mark.parametrize("rows,dtype", [(24, BF), (24, HF), (150, HF)])
@pytest.mark.parametrize("distill,temperature", CASES)
def test_rows_of_x(rows, dtype, distill, temperature):
    loss = _Loss(rows, dtype, distill, temperature)
    x, w, vx, none = _grid(1, dtype, rows, D), _grid(2, dtype, V, D), _grid(3, dtype, rows, D), torch.zeros(V, D, dtype=dtype, device="cuda")
    dloss = torch.rand(rows, generator=torch.Generator().manual_seed(4)).cuda() + 0.5
    along, exact, noise, without = loss.differences(x, w, vx, none)
    e = loss.expected(x, w)
    (wx, ex), _ = e.gradients(dloss, roundings=2 if rows <= 32 else 1)
    g = dloss.double()
    derivative = (wx * vx.double()).sum(1) / g
    left = (exact - derivative).abs()                                   # of the extrapolation, in 64 bits
    assert float(left.max()) < 1e-4
    off = noise + left + (ex * vx.double().abs()).sum(1) / g + 2.0 ** -22 * derivative.abs()
    got = (loss.backward(x, w, dloss, "x") * vx.double()).sum(1) / g
    assert bool(((got - along).abs() <= off).all()), float(((got - along).abs() - off).max())
    assert bool((got[~e.live] == 0).all()) and bool((along[~e.live] == 0).all())
    for k, l in without.items():                                        # a term that is missing shows
        assert float(((l - exact).abs() / off).max()) > 3.0, k


@pytest.mark.parametrize("rows", [24, 40])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("distill,temperature", CASES)
def test_the_matrix_by_one_row_at_a_time(rows, dtype, distill, temperature):
    loss = _Loss(rows, dtype, distill, temperature)
    x, w, none, vw = _grid(5, dtype, rows, D), _grid(6, dtype, V, D), torch.zeros(rows, D, dtype=dtype, device="cuda"), _grid(7, dtype, V, D)
    along, exact, noise, without = loss.differences(x, w, none, vw)
    e = loss.expected(x, w)
    shown = {k: 0.0 for k in without}
    for i in range(0, rows, 3):
        dloss = torch.zeros(rows, device="cuda")
        dloss[i] = 0.75
        _, (ww, ew) = e.gradients(dloss, roundings=2 if rows <= 32 else 1)
        derivative = float((ww * vw.double()).sum()) / 0.75
        left = abs(float(exact[i]) - derivative)
        assert left < 1e-4
        off = float(noise[i]) + left + float((ew * vw.double().abs()).sum()) / 0.75 + 2.0 ** -22 * abs(derivative)
        got = float((loss.backward(x, w, dloss, "w") * vw.double()).sum()) / 0.75
        assert abs(got - float(along[i])) <= off, (i, got, float(along[i]), off)
        if not bool(e.live[i]):
            assert got == 0.0
        shown = {k: max(shown[k], abs(float(without[k][i] - exact[i])) / off) for k in shown}
    # a term that is missing shows, where the coefficients' first rounding does not hide it (smoothing, lse less the mean logit, moves as little
    # as the differences' noise at temperature 2)
    assert rows > 32 or all(v > 3.0 for k, v in shown.items() if k != "smoothing" or temperature == 1.0), shown
