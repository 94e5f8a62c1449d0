"""GPU parity of the losses' gradients where rows differ by many powers of two: their
upstream gradients, and their row scales.

Bounds, beside those of loss_refs: dz of a row is held in F16 with a power of two of its
own, off by 2^-11 of a value or by 2^-31 of the row's |g T|; x of a row comes into dw off
by what 2^-33 of the largest |g T| row_scale makes of it."""
import math

import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests import loss_refs as ref
from tests.helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3 = sc.F16, sc.E4M3
U, F64 = lr.U, torch.float64


def floor_log2(t):
    return torch.frexp(t.to(F64))[1].to(F64) - 1


def bounds(r, g, row, lse, ex):
    """Gradients of r (a ref.Loss, all of whose rows count, x of scale 2^ex) for the upstream
    gradient g (no 0 among it), and the bounds of their errors before the output's rounding."""
    gt = g.to(F64) * r.T
    e = floor_log2(gt.abs())
    w = e + (floor_log2(row) if row is not None else 0.0)
    s = w.max() - w                                            # how far a row's weight in dw lies below the largest
    p = torch.exp(r.z - lse.to(F64)[:, None])
    dz = gt[:, None] * (p - r.q)
    log_err = r.ez + 8 * U * (r.z.abs() + lse.to(F64).abs()[:, None] + 1)
    ed = gt.abs()[:, None] * (p * log_err + 400 * U * r.q) + 2.0 ** -11 * dz.abs() + torch.exp2(e - 31)[:, None]
    R, V = dz.shape
    aw, ax = r.W.abs(), r.X.abs()
    # (a row 2^8 or less below the largest keeps x as it is)
    xe = torch.where(s > 8, torch.exp2(w.max() - e - 33 + ex), torch.zeros_like(e))[:, None]
    edx = ed @ aw + (V / 32 + 128) * 2 * U * (dz.abs() @ aw)
    edw = ed.t() @ (ax + xe) + dz.abs().t() @ xe.expand_as(ax) + (R / 32 + 128) * 2 * U * (dz.abs().t() @ ax)
    return dz @ r.W, dz.t() @ r.X, edx, edw


def inputs(R, V, top, seed):
    g = torch.Generator().manual_seed(seed)
    if not top:
        return torch.randint(0, V, (R,), generator=g).to(DEV), None, None
    return None, lr.scaled(lr.values(R, top, F16, seed + 1, 2.0), F16, 0), torch.randint(0, V, (R, top), generator=g).to(DEV)


def run(X, W, row, labels, teacher, index, g, target, T=1.0):
    R, V, D = X.shape[0], W.shape[0], X.shape[1]
    loss, lse = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    dx, dw = lr.empty(R, D, F16), lr.empty(V, D, F16)
    kw = dict(dx=dx, dw=dw, dloss=g, row_scale=row, rescale=sc.RESCALE_AMAX, target_log2=target)
    if labels is not None:
        sc.scalify_cross_entropy_fwd(X, W, labels, loss, lse=lse, row_scale=row)
        sc.scalify_cross_entropy_bwd(X, W, labels, lse, **kw)
    else:
        picked = torch.empty(index.shape, device=DEV)
        sc.scalify_distillation_fwd(X, W, teacher, index, loss, temperature=T, lse=lse, picked=picked, row_scale=row)
        sc.scalify_distillation_bwd(X, W, teacher, index, lse, picked, temperature=T, **kw)
    torch.cuda.synchronize()
    return lse, dx, dw


@pytest.mark.parametrize("fx", [F16, E4M3])
@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("R", [20, 90, 150])
def test_upstream_gradients_of_many_magnitudes(R, top, fx):
    """Rows whose upstream gradient lies far below the largest keep their digits of dx: here the
    mean of an output matrix that is not centred, spread over 32768 small probabilities."""
    say(f"loss upstream magnitudes {R} {top} {fx}")
    V, D = 32768, 64
    W = lr.scaled((1.0 + 0.25 * lr.values(V, D, sc.F32, 2)).half(), F16, 0)
    X = lr.scaled(lr.values(R, D, fx, 3), fx, -5)
    g = torch.exp2(-4.0 * (torch.arange(R) % 8)).to(DEV) * 1.25
    case = inputs(R, V, top, 4)
    lse, dx, dw = run(X, W, None, *case, g, 14)
    want = bounds(ref.Loss(X, W, None, *case), g, None, lse, -5)
    ref.check_gradient(dx, want[0], want[2], 0, sc.RESCALE_AMAX, 14)
    ref.check_gradient(dw, want[1], want[3], -5, sc.RESCALE_AMAX, 14)


@pytest.mark.parametrize("fx", [F16, E4M3])
@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("R", [24, 90, 160])
def test_row_scales_of_many_magnitudes(R, top, fx):
    """Rows of small scales, alone with their tokens: the others, sure of a token of their own
    (and wrong), leave those no gradient."""
    say(f"loss row scales {R} {top} {fx}")
    V, D = 300, 64
    e = torch.tensor([0.0, -10.0, -20.0, -26.0])[torch.arange(R) % 4]
    w = lr.values(V, D, F16, 5)
    x = lr.values(R, D, F16, 6).float()
    sure = e == 0
    x[sure] = w[:R][sure].float()            # (z of about D, where the others' are of about 8)
    labels, teacher, index = inputs(R, 100, top, 7)
    what = labels if labels is not None else index
    what += 200                              # (no row is sure of these)
    what[sure.to(DEV)] = (torch.arange(R) % 100 + 100).to(DEV)[sure.to(DEV)].reshape(-1, *([1] * (what.dim() - 1)))
    X, W, row = lr.scaled(x.to(lr.TORCH[fx]), fx, 0), lr.scaled(w, F16, 0), torch.exp2(e).to(DEV)
    g = torch.ones(R, device=DEV)
    lse, dx, dw = run(X, W, row, labels, teacher, index, g, 14)
    want = bounds(ref.Loss(X, W, row, labels, teacher, index), g, row, lse, 0)
    ref.check_gradient(dx, want[0], want[2], 0, sc.RESCALE_AMAX, 14)
    ref.check_gradient(dw, want[1], want[3], 0, sc.RESCALE_AMAX, 14)
