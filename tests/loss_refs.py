"""Plain 64-bit forms of the losses from hidden states and the output matrix, and
bounds of the kernels' errors from their formats. u = 2^-24 is half a step of fp32;
dz is held in F16 as 2^14 dz / 2^E, off by 2^-11 of a value, or 2^-25 in those units.

A logit is a sum of D products in fp32, 32 at a time: D / 32 additions of a whole
step (2 u) each, and 32 inside the instruction, of magnitudes up to sum |x w|."""
from __future__ import annotations

import math

import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr

F64 = torch.float64
U = lr.U
DEV = "cuda"


def true(x):
    """True values of a ScaledArray in 64 bits, where its data is."""
    t = x.data.contiguous().view(lr.TORCH[x.fmt]).to(F64)
    return t * x.scale.to(F64) if x.scale is not None else t


class Loss:
    """x, w: ScaledArrays; row: row scales or None; labels, or (teacher, index, T)."""

    def __init__(self, x, w, row=None, labels=None, teacher=None, index=None, T=1.0):
        self.X, self.W = true(x), true(w)
        if row is not None:
            self.X = self.X * row.to(F64)[:, None]
        R, V, D = self.X.shape[0], self.W.shape[0], self.X.shape[1]
        self.T, self.V, self.D = T, V, D
        if labels is not None:
            self.on = (labels >= 0) & (labels < V)
            self.q = torch.zeros((R, V), dtype=F64, device=self.X.device)
            self.q[self.on, labels[self.on]] = 1.0
        else:
            t = true(teacher) / T
            self.there = (index >= 0) & (index < V)
            t = t.masked_fill(~self.there, -math.inf)
            self.on = (t > -math.inf).any(1)
            self.qe = torch.nan_to_num(torch.softmax(t, 1)) * self.on[:, None]
            self.at = torch.where(self.there, index, 0)
            self.q = torch.zeros((R, V), dtype=F64, device=self.X.device).scatter_add_(1, self.at, self.qe)
        self.X = torch.where(self.on[:, None], self.X, torch.zeros_like(self.X))
        self.z = self.X @ self.W.t() / T
        self.mag = (self.X.abs() @ self.W.abs().t() / T)
        # error of each logit: its sum's, and the factor's and product's roundings
        self.ez = (D / 32 + 40) * 2 * U * self.mag + 6 * U * self.z.abs()
        self.lse = torch.where(self.on, torch.logsumexp(self.z, 1), torch.zeros(R, dtype=F64, device=self.X.device))

    def lse_error(self):
        """A sum's 32 terms of a lane, its joins, exp2 and log2 (a step each), the
        arguments' roundings (at most log2 V bits of weight), and the logits' own."""
        V = self.V
        return self.ez.amax(1) + (96 + V / 32 + 16 * math.log2(V + 1)) * U + 6 * U * self.lse.abs()

    def check_forward(self, loss, lse, picked=None):
        loss, lse = loss.to(F64), lse.to(F64)
        el = self.lse_error()
        assert (lse[~self.on] == 0).all() and (loss[~self.on] == 0).all()
        assert ((lse - self.lse).abs() <= el)[self.on].all(), (lse - self.lse).abs().max()
        zero = torch.zeros_like(self.lse)
        if picked is None:
            zy = (self.q * self.z).sum(1)
            want, err = self.lse - zy, el + (self.q * self.ez).sum(1) + 6 * U * (zy.abs() + self.lse.abs())
        else:
            z, ez = self.z.gather(1, self.at), self.ez.gather(1, self.at)
            on = self.there & self.on[:, None]
            p = picked.to(F64)
            assert (p[~on] == 0).all()
            assert ((p - z).abs() <= ez + 6 * U * z.abs())[on].all()
            logq = torch.where(self.qe > 0, self.qe, torch.ones_like(self.qe)).log()
            terms = self.qe * (logq - z + self.lse[:, None])
            want = self.T ** 2 * terms.sum(1)
            # each term: log q of a softmax over at most 256 (its exp, sum and logarithm), its factors
            big = self.qe * (logq.abs() + z.abs() + self.lse.abs()[:, None] + 4)
            err = self.T ** 2 * (el + (self.qe * ez).sum(1) + 400 * U * big.sum(1))
        want = torch.where(self.on, want, zero)
        assert ((loss - want).abs() <= torch.where(self.on, err, zero)).all(), (loss - want).abs().max()

    def gradients(self, g, lse):
        """dx and dw (true values) for the true upstream gradient g, from a stored lse,
        with the bounds of their errors before the output's rounding."""
        g = torch.where(self.on, g.to(F64), torch.zeros_like(self.lse)) * self.T
        act = g != 0
        lse = torch.where(act, lse.to(F64), torch.zeros_like(self.lse))
        X = torch.where(act[:, None], self.X, torch.zeros_like(self.X))
        p = torch.exp(self.z - lse[:, None])
        dz = torch.where(act[:, None], g[:, None] * (p - self.q), torch.zeros_like(p))
        top = g.abs().max().item()
        E = math.frexp(top)[1] - 1 if top > 0 else 0
        log_err = self.ez + 8 * U * (self.z.abs() + lse.abs()[:, None] + 1)
        # (the teacher's probabilities: 400 u, as in the loss)
        ed = g.abs()[:, None] * (p * log_err + 400 * U * self.q) + 2.0 ** -11 * dz.abs() + 2.0 ** (E - 14 - 25)
        ed = torch.where(act[:, None], ed, torch.zeros_like(ed))
        R, V = dz.shape
        aw, ax = self.W.abs(), X.abs()
        ex = ed @ aw + (V / 32 + 128) * 2 * U * (dz.abs() @ aw)
        ew = ed.t() @ ax + (R / 32 + 128) * 2 * U * (dz.abs().t() @ ax)
        return dz @ self.W, dz.t() @ X, ex, ew


def check_gradient(got, want, err, base, mode, target=0, amax=None):
    """A gradient's scale (base: the propagated one) and data."""
    e = lr.log2_of(got)
    top = want.abs().max().item() / 2.0 ** base if want.numel() else 0.0
    if amax is not None:
        a = amax.item()
        tol = (err.max().item() / 2.0 ** base if err.numel() else 0.0)
        assert abs(a - top) <= tol, (a, top, tol)
    if mode == sc.RESCALE_NONE:
        assert e == base
    elif amax is not None:
        assert e == base + ((math.frexp(a)[1] - 1 - target) if a > 0 else 0)
    rel, sub = lr.HALF[got.fmt]
    d = (true(got) - want).abs()
    bound = err + (want.abs() + err) * rel + sub * 2.0 ** e
    assert (d <= bound).all(), ((d / bound.clamp(min=1e-300)).max(), d.max())
