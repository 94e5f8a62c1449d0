"""GPU tests of the losses' calls at their edges: no rows, outputs left out, operands
without scales, the ends of the temperature's range."""
import math

import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests import loss_refs as ref
from tests.helpers import say
from tests.test_gpu_losses import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3, E5M2 = sc.F16, sc.E4M3, sc.E5M2


@pytest.mark.parametrize("which", ["both", "dx", "dw"])
@pytest.mark.parametrize("mode", [sc.RESCALE_NONE, sc.RESCALE_AMAX])
@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("V", [50, (1 << 22) + 3])
def test_no_rows_have_scales(V, top, mode, which):
    """Gradients of no rows: dw is 0, and each gradient's scale and statistic is written."""
    say(f"loss no rows {V} {top} {mode} {which}")
    D = 24
    c = Case(1, V, D, top=top)
    c.R, c.loss, c.lse, c.g = 0, c.loss[:0], c.lse[:0], c.g[:0]
    c.x = sc.ScaledArray(c.x.data[:0], F16, c.x.scale)
    if top:
        c.teacher, c.index, c.picked = sc.ScaledArray(c.teacher.data[:0], F16, c.teacher.scale), c.index[:0], c.picked[:0]
    else:
        c.labels = c.labels[:0]
    c.forward()
    dx = lr.empty(1, D, F16)
    dx = sc.ScaledArray(dx.data[:0], F16, dx.scale) if which != "dw" else None
    dw = lr.empty(V, D, F16) if which != "dx" else None
    amax = torch.full((2,), -1.0, device=DEV)
    c.backward(dx, dw, rescale=mode, amax_out=amax)
    torch.cuda.synchronize()
    if dx is not None:
        assert lr.log2_of(dx) == c.ew - 3 and amax[0] == 0
    if dw is not None:
        assert (dw.data == 0).all() and lr.log2_of(dw) == c.ex - 3 and amax[1] == 0


@pytest.mark.parametrize("R", [20, 150])
@pytest.mark.parametrize("top", [0, 6])
def test_outputs_left_out(top, R):
    """The loss is the same without the outputs that are optional."""
    c = Case(R, 400, 72, E4M3, E4M3, True, top, 1.5 if top else 1.0)
    c.forward()
    want = c.loss.clone()
    for lse, picked in ((True, False), (False, True), (False, False)):
        c.loss.fill_(7.0)
        lse2, picked2 = torch.full_like(c.lse, 7.0), torch.full_like(c.picked, 7.0) if top else None
        kw = dict(lse=lse2 if lse else None, row_scale=c.row)
        if top:
            sc.scalify_distillation_fwd(c.x, c.w, c.teacher, c.index, c.loss, temperature=c.T, picked=picked2 if picked else None, **kw)
        else:
            sc.scalify_cross_entropy_fwd(c.x, c.w, c.labels, c.loss, **kw)
        torch.cuda.synchronize()
        assert torch.equal(c.loss, want) and (not lse or torch.equal(lse2, c.lse))
        assert not (top and picked) or torch.equal(picked2, c.picked)


@pytest.mark.parametrize("R", [20, 150])
@pytest.mark.parametrize("top", [0, 6])
def test_operands_without_scales(top, R):
    c = Case(R, 400, 72, top=top, seed=31)
    c.w.scale.fill_(1.0)
    c.x.data = (c.x.data.view(torch.float16) * 2.0 ** -4).view(torch.int16)
    c.x = sc.ScaledArray(c.x.data, F16, None)
    c.w = sc.ScaledArray(c.w.data, F16, None)
    c.ex = c.ew = 0
    c.check(mode=sc.RESCALE_AMAX)


@pytest.mark.parametrize("R", [20, 150])
@pytest.mark.parametrize("T", [2.0 ** -20, 2.0 ** -8, 2.0 ** 10])
def test_temperatures(T, R):
    """A temperature scales all logits: small ones leave the largest token alone, and all results
    finite; large ones even probabilities."""
    say(f"loss temperature {T} {R}")
    c = Case(R, 300, 64, E4M3, E4M3, top=7, T=T, seed=32)
    if T > 1:
        c.check()
        return
    c.forward()
    torch.cuda.synchronize()
    r = c.reference()
    on = r.on
    step = 64 * lr.U * r.z.abs().amax(1) + 1e-4
    assert ((c.lse.double() - r.lse).abs() <= step)[on].all()
    dx, dw = lr.empty(R, 64, F16), lr.empty(300, 64, F16)
    c.backward(dx, dw, rescale=sc.RESCALE_AMAX)
    torch.cuda.synchronize()
    for t in (ref.true(dx), ref.true(dw), c.loss, c.lse, c.picked):
        assert torch.isfinite(t).all()
