"""Host-side refusals of the losses' gradients over what the call still reads (no GPU; the
pointers are never dereferenced): a piece of the vocabulary writes its rows of dw before the
next one reads the teacher's tokens, logits and what the forward stored."""
import pytest

from tests import test_losses_host as h
from tests.test_losses_host import DW, DX, FAKE, GB, S

LAYOUT = 4
KD = {
    "dw_over_teacher": dict(dw=DW(at=4, scale=S + 768)), "dx_over_teacher": dict(dx=DX(at=4, scale=S + 512)),
    "dx_scale_of_teacher": dict(dx=DX(scale=S + 1024)), "dw_scale_of_teacher": dict(dw=DW(scale=S + 1024)),
}
VECTORS = ("lse", "g", "row")
# a vector of n elements of a size, the last of which lies on the first of dw, or the first on the last of dx
NEAR = {"into_dw": lambda n, size: h.DW().data - (n - 1) * size, "behind_dx": lambda n, size: h.DX().data + h.R * h.D * 2 - size}


@pytest.mark.parametrize("name", KD)
def test_distillation_gradients_over_the_teacher(name):
    assert h.kd_bwd(**KD[name]) == LAYOUT


@pytest.mark.parametrize("where", NEAR)
@pytest.mark.parametrize("which", VECTORS)
def test_gradients_over_rows_numbers(which, where):
    at = NEAR[where](h.R, 4)
    assert h.ce_bwd(**{which: at}) == LAYOUT
    assert h.kd_bwd(**{which: at}) == LAYOUT


@pytest.mark.parametrize("where", NEAR)
def test_gradients_over_labels_tokens_and_logits(where):
    assert h.ce_bwd(labels=NEAR[where](h.R, 8)) == LAYOUT
    assert h.kd_bwd(index=NEAR[where](h.R * h.TOP, 8)) == LAYOUT
    assert h.kd_bwd(picked=NEAR[where](h.R * h.TOP, 4)) == LAYOUT
