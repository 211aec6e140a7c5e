"""Plain 64-bit restatements of the losses over a vocabulary and of their gradients, and how far the kernels may be from them.

Tolerance of a logit.  Products of 16-bit values are exact in fp32; the tensor cores add 16 of them at a time to an fp32 sum, each
addition off by at most one unit of the last place (2^-23) of the magnitudes added: z is within (d / 16 + 8) 2^-23 of the sum of
magnitudes, over T.  Taking it to the base 2, away from the maximum and to a power adds 4 2^-24 of |z| and of |lse| and 2^-21
(the power's own error); a sum of powers is a chain of fewer than 128 additions, and the logarithm of at most 2^22 is
within 2^-21 of 24.  So lse is within the largest of its logits' errors and 2^-17, a relative error of q of the same size, and a loss
within the errors of its logits and of lse, weighted as they are.
A coefficient dz is rounded to the operands' type once (UNIT); sums over rows and over the vocabulary add as above.  In half precision
it is stored times a power of two that brings its row's bound |g| (1 + 2 zeta |lse|) to 2^7 or more (2^13 or more for rows of
nearly the largest bound), where half of the type's smallest step, 2^-25, is 2^-32 of the bound."""
import math

import torch

from tests.block_reference import UNIT

SUMS = 2.0 ** -17


def entries_ce(target, vocab, smoothing):
    """(ids, shares, live) of a cross entropy: one entry per row."""
    t = target.long().cpu()
    live = (t >= 0) & (t < vocab)
    return torch.where(live, t, 0)[:, None], torch.full((t.shape[0], 1), 1.0 - smoothing, dtype=torch.float64) * live[:, None], live


def entries_distill(ids, teacher, vocab, temperature):
    ids, t = ids.long().cpu(), teacher.double().cpu() / temperature
    held = (ids >= 0) & (ids < vocab) & (t != -math.inf)
    p = torch.zeros_like(t)
    for i in range(ids.shape[0]):
        if held[i].any():
            p[i][held[i]] = torch.softmax(t[i][held[i]], 0)
    return torch.where(held, ids, 0), p, held.any(1)


class Expected:
    """What a loss and its gradients have to be (64 bits) and by how much they may be off, for entries (ids, shares, live)."""

    def __init__(self, x, w, entries, temperature=1.0, smoothing=0.0, z_loss=0.0, distill=False):
        dev = x.device
        ids, p, live = (t.to(dev) for t in entries)
        self.live, self.dtype, self.rows, self.vocab, self.d = live, x.dtype, x.shape[0], w.shape[0], x.shape[1]
        xd = torch.where(live[:, None], x.double(), 0.0)
        wd = w.double()
        z = xd @ wd.t() / temperature
        ez = (self.d / 16 + 8) * 2.0 ** -23 * (xd.abs() @ wd.abs().t()) / temperature
        lse = torch.logsumexp(z, 1)
        self.e_lse = ez.amax(1) + SUMS + 2.0 ** -22 * (z.abs().amax(1) + lse.abs())
        at = lambda t: t.gather(1, ids)  # noqa: E731
        logp = torch.where(p > 0, torch.log(p.clamp(min=1e-300)), 0.0) if distill else torch.zeros_like(p)
        loss = (p * (logp - at(z) + lse[:, None])).sum(1) + smoothing * (lse - z.mean(1)) + z_loss * lse ** 2
        e_loss = (p * (at(ez) + 2.0 ** -22 * (at(z).abs() + logp.abs()) + 2.0 ** -20 * (at(z) - lse[:, None]).abs() + 2.0 ** -20)).sum(1) + self.e_lse * (1 + 2 * z_loss * lse.abs())
        e_loss = e_loss + smoothing * (ez.mean(1) + 2.0 ** -20 * z.abs().mean(1)) + 2.0 ** -21 * loss.abs() + z_loss * 2.0 ** -22 * lse ** 2
        self.lse, self.loss, self.e_loss = torch.where(live, lse, 0.0), torch.where(live, loss, 0.0), torch.where(live, e_loss, 0.0)
        self.e_lse = torch.where(live, self.e_lse, 0.0)
        self._grad = (xd, wd, z, ez, ids, p, temperature, smoothing, z_loss)

    def check_forward(self, loss, lse):
        assert bool(((lse.double() - self.lse).abs() <= self.e_lse).all()), float(((lse.double() - self.lse).abs() - self.e_lse).max())
        assert bool(((loss.double() - self.loss).abs() <= self.e_loss).all()), float(((loss.double() - self.loss).abs() - self.e_loss).max())
        assert bool((loss[~self.live] == 0).all()) and bool((lse[~self.live] == 0).all())

    def gradients(self, dloss, roundings=1):
        """(dx, how far it may be off before it is rounded), (dw, the same); roundings 2: what the first one takes away from dz is rounded
        itself and taken along."""
        xd, wd, z, ez, ids, p, temperature, smoothing, z_loss = self._grad
        g = torch.where(self.live, dloss.double(), 0.0)[:, None] / temperature
        q = torch.exp(z - self.lse[:, None]) * (1 + 2 * z_loss * self.lse[:, None])
        share = torch.zeros_like(z).scatter_add_(1, ids, p)
        dz = g * (q - smoothing / self.vocab - share)
        # q from the logit and lse that are given in fp32, p to 2^-20 of itself, one rounding to the operands' type
        size = g.abs() * (q.abs() + smoothing / self.vocab + share)
        e = g.abs() * q.abs() * (ez + 2.0 ** -18 + 2.0 ** -22 * (z.abs() + self.lse[:, None].abs())) + size * 2.0 ** -20
        step = 2.0 ** -32 * g.abs() * (1 + 2 * z_loss * self.lse[:, None].abs()) if self.dtype == torch.float16 else 0.0
        e = torch.where(g != 0, e + (UNIT[self.dtype] * 1.001) ** roundings * (dz.abs() + e) + step, 0.0)
        m = dz.abs() + e
        ex = e @ wd.abs() + (self.vocab / 16 + 64) * 2.0 ** -23 * (m @ wd.abs())
        ew = e.t() @ xd.abs() + (self.rows / 16 + 8) * 2.0 ** -23 * (m.t() @ xd.abs())
        return (dz @ wd, ex), (dz.t() @ xd, ew)


def near(got, want, off):
    unit = 0.0 if got.dtype == torch.float32 else UNIT[got.dtype]
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 0.0          # half the spacing of the smallest half-precision numbers
    excess = (got.double() - want).abs() - off - unit * 1.001 * (want.abs() + off) - tiny - 1e-37
    return bool((excess <= 0).all())
