"""GPU tests of what is not a number in the losses' gradients, of few rows on the path of
many, and of captured calls of few rows."""
import math

import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests.helpers import say
from tests.test_gpu_losses import NAMES, Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3, E5M2 = sc.F16, sc.E4M3, sc.E5M2


def backward(c, fg, mode):
    dx, dw = lr.empty(c.R, c.D, fg), lr.empty(c.V, c.D, fg)
    c.backward(dx, dw, eg=0, rescale=mode)
    torch.cuda.synchronize()
    return dx, dw


@pytest.mark.parametrize("what", ["x", "logit", "dloss", "inf_dloss"])
@pytest.mark.parametrize("mode", [sc.RESCALE_NONE, sc.RESCALE_AMAX])
@pytest.mark.parametrize("fg", [F16, E4M3, E5M2])
@pytest.mark.parametrize("R,top", [(7, 0), (40, 0), (150, 0), (40, 5), (150, 5)])
def test_counted_nan_backward(R, top, fg, mode, what):
    """A counted row whose state is not a number, or infinite, or whose upstream gradient is: NaN
    in that row of dx and, as every token has a share of it, all over dw; the other rows of dx as
    if it did not count."""
    say(f"loss nan backward {R} {top} {NAMES[fg]} {mode} {what}")
    V, D, i = 300, 72, 3
    c = Case(R, V, D, top=top, skip=0, seed=21)
    c.g = (1.0 + 0.5 * torch.rand(R, generator=torch.Generator().manual_seed(2))).to(DEV)
    c.forward()
    if top:
        assert c.reference().on[i]
    c.g[i] = 0.0
    want, _ = backward(c, fg, mode)
    c.g[i] = {"x": 1.0, "logit": 1.0, "dloss": math.nan, "inf_dloss": math.inf}[what]
    if what == "x":
        c.x.data.view(torch.float16)[i, 5] = math.nan
    elif what == "logit":
        c.x.data.view(torch.float16)[i, 5] = math.inf
    c.forward()
    dx, dw = backward(c, fg, mode)
    others = torch.arange(R, device=DEV) != i
    assert torch.equal(dx.data[others], want.data[others]) and torch.equal(dx.scale, want.scale)
    if what == "inf_dloss":
        # infinite times probabilities: sums of infinities of either sign (saturated where they agree)
        largest = {E4M3: 448.0, E5M2: 57344.0, F16: 65504.0}[fg]
        for t in (lr.data(dx)[i], lr.data(dw)):
            assert (torch.isnan(t) | (t.abs() == largest)).all()
    else:
        assert torch.isnan(lr.data(dx)[i]).all() and torch.isnan(lr.data(dw)).all()
    assert lr.log2_of(dw) == c.ex


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("D", [8, 9])
def test_few_rows_of_a_vocabulary_in_pieces(D, top):
    """Few rows against more tokens than their own kernels take."""
    say(f"loss few rows in pieces {D} {top}")
    Case(3, (1 << 22) + 77, D, F16, E4M3, top=top, skip=0, seed=22).check()


@pytest.mark.parametrize("top", [0, 12])
@pytest.mark.parametrize("R", [9, 100])
def test_capture_of_few_rows(R, top):
    """Captured and replayed with other inputs, eager calls between: equal to the eager results."""
    say(f"loss capture of few rows {R} {top}")
    c = Case(R, 900, 136, E4M3, E4M3, True, top, seed=23)
    n = max(sc.scalify_distillation_bwd_workspace_size(R, 900, 136, max(top, 1), E4M3),
            sc.scalify_distillation_fwd_workspace_size(R, 900, 136, max(top, 1), E4M3))
    ws, scale = torch.empty(n, dtype=torch.uint8, device=DEV), sc.scale_tensor(-3, DEV)
    outs = lr.empty(R, 136, F16), lr.empty(900, 136, F16)

    def step(dx, dw, **kw):
        c.forward(**kw)
        kw = dict(dx=dx, dw=dw, dloss=c.g, dloss_scale=scale, row_scale=c.row, **kw)
        if top:
            sc.scalify_distillation_bwd(c.x, c.w, c.teacher, c.index, c.lse, c.picked, temperature=c.T, **kw)
        else:
            sc.scalify_cross_entropy_bwd(c.x, c.w, c.labels, c.lse, **kw)

    step(*outs, ws=ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(*outs, ws=ws)
    what = c.index if top else c.labels
    for _ in range(3):
        what.copy_(torch.roll(what, 1, 0))
        eager = lr.empty(R, 136, F16), lr.empty(900, 136, F16)
        step(*eager)
        want = [t.clone() for t in (c.loss, c.lse)]
        torch.cuda.synchronize()
        ws.fill_(0xFF)
        c.loss.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.loss, want[0]) and torch.equal(c.lse, want[1])
        for a, b in zip(outs, eager):
            assert torch.equal(a.data, b.data) and torch.equal(a.scale, b.scale)
