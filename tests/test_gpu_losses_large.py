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
