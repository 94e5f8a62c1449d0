"""GPU tests of the losses where logits are so large that fp32 no longer holds their
differences: their statistics stay finite and right to fp32, and no probability of the
gradients passes 1."""
import math

import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests import loss_refs as ref
from tests.helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16 = sc.F16
U = lr.U


@pytest.mark.parametrize("top", [0, 4])
@pytest.mark.parametrize("R", [12, 40, 150])
@pytest.mark.parametrize("e", [18, 24, 28, 31, 36, 50])
def test_large_logits(R, top, e):
    """Logits of some 2^(e + 5), of whole numbers times 2^e: the loss and the log-sum-exp are right
    to some steps of the largest of them."""
    say(f"loss large {R} {top} {e}")
    V, D = 150, 32
    g = torch.Generator().manual_seed(8)
    X = lr.scaled(torch.randint(-2, 3, (R, D), generator=g).half(), F16, e)
    W = lr.scaled(torch.randint(-2, 3, (V, D), generator=g).half(), F16, 0)
    loss, lse = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    labels = teacher = index = None
    if top:
        teacher, index = lr.scaled(lr.values(R, top, F16, 9), F16, 0), torch.randint(0, V, (R, top), generator=g).to(DEV)
        sc.scalify_distillation_fwd(X, W, teacher, index, loss, lse=lse)
    else:
        labels = torch.randint(0, V, (R,), generator=g).to(DEV)
        sc.scalify_cross_entropy_fwd(X, W, labels, loss, lse=lse)
    torch.cuda.synchronize()
    r = ref.Loss(X, W, None, labels, teacher, index)
    # the products are exact; the factor's, the logit's and the results' roundings, a step each of the largest
    # magnitude, and what a sum of V terms and the teacher's entries add
    most = r.z.abs().amax(1)
    step = (8 + 4 * top) * U * most + (400 + V / 32) * U * (1 + math.log(V))
    assert ((lse.double() - r.lse).abs() <= step).all(), (lse.double() - r.lse).abs().max()
    if top:
        entropy = (r.qe * torch.where(r.qe > 0, r.qe, torch.ones_like(r.qe)).log()).sum(1)
        want = entropy - (r.q * r.z).sum(1) + r.lse
    else:
        want = r.lse - r.z.gather(1, labels[:, None])[:, 0]
    assert ((loss.double() - want).abs() <= 2 * step).all(), (loss.double() - want).abs().max()


@pytest.mark.parametrize("top", [0, 4])
@pytest.mark.parametrize("R", [12, 40, 150])
def test_gradients_of_large_logits(R, top):
    """A third of the rows have logits whose log-sum-exp fp32 holds to a whole number or worse. Their
    probabilities are at most 1 all the same; the other rows' gradients are as ever."""
    say(f"loss gradients of large logits {R} {top}")
    V, D = 150, 32
    g = torch.Generator().manual_seed(10)
    X = lr.scaled(torch.randint(-2, 3, (R, D), generator=g).half(), F16, -2)
    W = lr.scaled(torch.randint(-2, 3, (V, D), generator=g).half(), F16, -2)
    huge = torch.arange(R) % 3 == 0
    row = torch.where(huge, torch.exp2(24.0 + torch.arange(R) % 7), torch.ones(R)).to(DEV)
    huge = huge.to(DEV)
    loss, lse = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    dx, dw = lr.empty(R, D, F16), lr.empty(V, D, F16)
    kw = dict(dx=dx, dw=dw, row_scale=row, rescale=sc.RESCALE_NONE)
    labels = teacher = index = None
    if top:
        teacher, index = lr.scaled(lr.values(R, top, F16, 9), F16, 0), torch.randint(0, V, (R, top), generator=g).to(DEV)
        picked = torch.empty((R, top), device=DEV)
        sc.scalify_distillation_fwd(X, W, teacher, index, loss, lse=lse, picked=picked, row_scale=row)
        sc.scalify_distillation_bwd(X, W, teacher, index, lse, picked, **kw)
    else:
        labels = torch.randint(0, V, (R,), generator=g).to(DEV)
        sc.scalify_cross_entropy_fwd(X, W, labels, loss, lse=lse, row_scale=row)
        sc.scalify_cross_entropy_bwd(X, W, labels, lse, **kw)
    torch.cuda.synchronize()
    r = ref.Loss(X, W, row, labels, teacher, index)
    assert torch.isfinite(ref.true(dx)).all() and torch.isfinite(ref.true(dw)).all()
    # a row's probabilities, at most 1 for each token whose logit fp32 takes for the largest, less the targets; F16
    near = (r.z >= r.z.amax(1, keepdim=True) - 64 * U * r.z.abs().amax(1, keepdim=True)).sum(1)
    d = ref.true(dx).abs().amax(1)
    assert (d <= (near + 1) * r.W.abs().max() * (1 + 2.0 ** -9))[huge].all()
    want, _, err, _ = r.gradients(torch.ones(R, device=DEV), lse)
    rel, sub = lr.HALF[F16]
    off = (ref.true(dx) - want).abs() - (err + (want.abs() + err) * rel + sub * 2.0 ** -2)
    assert (off <= 0)[~huge].all(), off[~huge].max()
