"""Host-side checks of the losses' entry points (no GPU): sizes of their workspaces
and the refusal of bad arguments before any launch (the pointers are never
dereferenced; every case differs in one point from a call whose other arguments are
valid, and the valid call itself is never made)."""
import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests.test_layers_host import FAKE, GB, arr, ref

R, V, D, TOP = 20, 300, 64, 8
LABELS, LOSS, LSE, ROW, PICKED, INDEX, G, GS = (FAKE + (40 + i) * GB for i in range(8))
WS = FAKE + 96 * GB
X, W = (lambda **k: arr(R, D, **{"at": 0, **k})), (lambda **k: arr(V, D, **{"at": 1, **k}))
DX, DW = (lambda **k: arr(R, D, **{"at": 2, **k})), (lambda **k: arr(V, D, **{"at": 3, **k}))
TEACHER = lambda **k: arr(R, TOP, **{"at": 4, **k})


def ce_fwd(x=X(), w=W(), labels=LABELS, row=None, loss=LOSS, lse=LSE, ws=WS, nws=1 << 40):
    return sc.load_library().scalify_cross_entropy_fwd(ref(x), ref(w), labels, row, loss, lse, ws, nws, None)


def ce_bwd(g=G, gs=GS, x=X(), w=W(), labels=LABELS, row=None, lse=LSE, dx=DX(), dw=DW(), mode=1, target=0, amax=None, ws=WS,
           nws=1 << 40):
    return sc.load_library().scalify_cross_entropy_bwd(g, gs, ref(x), ref(w), labels, row, lse, ref(dx), ref(dw), mode, target, 1,
                                                       amax, ws, nws, None)


def kd_fwd(x=X(), w=W(), t=TEACHER(), index=INDEX, T=1.0, row=None, loss=LOSS, lse=LSE, picked=PICKED, ws=WS, nws=1 << 40):
    return sc.load_library().scalify_distillation_fwd(ref(x), ref(w), ref(t), index, T, row, loss, lse, picked, ws, nws, None)


def kd_bwd(g=G, gs=GS, x=X(), w=W(), t=TEACHER(), index=INDEX, T=1.0, row=None, lse=LSE, picked=PICKED, dx=DX(), dw=DW(), mode=1,
           target=0, amax=None, ws=WS, nws=1 << 40):
    return sc.load_library().scalify_distillation_bwd(g, gs, ref(x), ref(w), ref(t), index, T, row, lse, picked, ref(dx), ref(dw),
                                                      mode, target, 1, amax, ws, nws, None)


BOTH = {
    "no_x": (1, dict(x=None)), "no_w": (1, dict(w=None)), "no_data": (1, dict(w=W(data=False))),
    "x_f32": (2, dict(x=X(dtype=sc.F32))), "w_f32": (2, dict(w=W(dtype=sc.F32))), "w_type": (2, dict(w=W(dtype=-1))),
    "columns": (3, dict(w=arr(V, D + 16, at=1))), "negative": (3, dict(x=arr(-1, D))), "no_vocabulary": (3, dict(w=arr(0, D, at=1))),
    "too_wide": (3, dict(x=arr(R, (1 << 20) + 16), w=arr(V, (1 << 20) + 16, at=1))), "small_ld": (3, dict(x=X(ld=48))),
    "huge_ld": (3, dict(w=W(ld=1 << 22))), "tiles": (3, dict(x=arr(1 << 29, D), w=arr(1 << 29, D, at=1))),
    "x_trans": (4, dict(x=X(trans=1))), "w_trans": (4, dict(w=W(trans=1))),
    "ld": (5, dict(x=X(ld=68))), "row_scale": (5, dict(row=ROW + 2)), "lse_align": (5, dict(lse=LSE + 1)),
    "no_ws": (6, dict(ws=None)), "small_ws": (6, dict(nws=256)), "ws_align": (6, dict(ws=WS + 128)),
}
FWD = {"no_loss": (1, dict(loss=None)), "loss_align": (5, dict(loss=LOSS + 2))}
LABELLED = {"no_labels": (1, dict(labels=None)), "labels_align": (5, dict(labels=LABELS + 4))}
TAUGHT = {
    "no_teacher": (1, dict(t=None)), "no_index": (1, dict(index=None)), "no_teacher_data": (1, dict(t=TEACHER(data=False))),
    "teacher_type": (2, dict(t=TEACHER(dtype=4))), "teacher_rows": (3, dict(t=arr(R + 1, TOP, at=4))),
    "no_entries": (3, dict(t=arr(R, 0, at=4))), "entries": (3, dict(t=arr(R, 257, at=4))), "teacher_trans": (4, dict(t=TEACHER(trans=1))),
    "teacher_ld": (5, dict(t=TEACHER(ld=12))), "index_align": (5, dict(index=INDEX + 4)), "T_0": (7, dict(T=0.0)),
    "T_negative": (7, dict(T=-1.0)), "T_nan": (7, dict(T=float("nan"))), "T_inf": (7, dict(T=float("inf"))),
    "picked_align": (5, dict(picked=PICKED + 2)),
}
S = FAKE + 64 * GB  # (matrix i's scale lies at S + 256 i)
BWD = {
    "no_lse": (1, dict(lse=None)), "no_gradient": (1, dict(dx=None, dw=None)), "no_dx_scale": (1, dict(dx=DX(scale=0))),
    "no_dw_scale": (1, dict(dw=DW(scale=0))), "dx_f32": (2, dict(dx=DX(dtype=sc.F32))), "dw_f32": (2, dict(dw=DW(dtype=sc.F32))),
    "rows_of_dx": (3, dict(dx=arr(R + 1, D, at=2))), "rows_of_dw": (3, dict(dw=arr(V - 1, D, at=3))),
    "dx_trans": (4, dict(dx=DX(trans=1))), "dw_ld": (5, dict(dw=DW(ld=68))), "dx_over_x": (4, dict(dx=DX(at=0, scale=S + 512))),
    "dw_over_w": (4, dict(dw=DW(at=1, scale=S + 768))), "dw_over_dx": (4, dict(dw=DW(at=2, scale=S + 768))),
    "scale_of_x": (4, dict(dx=DX(scale=S))), "scale_of_w": (4, dict(dw=DW(scale=S + 256))), "scales_shared": (4, dict(dw=DW(scale=S + 512))),
    "scale_of_dloss": (4, dict(dx=DX(scale=GS))), "dloss_align": (5, dict(g=G + 2)), "amax_align": (5, dict(amax=G + 1)),
    "delayed": (7, dict(mode=2)), "target": (7, dict(target=-1001)),
}


@pytest.mark.parametrize("name", {**BOTH, **FWD, **LABELLED})
def test_cross_entropy_fwd_refusals(name):
    status, kw = {**BOTH, **FWD, **LABELLED}[name]
    assert ce_fwd(**kw) == status


@pytest.mark.parametrize("name", {**BOTH, **BWD, **LABELLED})
def test_cross_entropy_bwd_refusals(name):
    status, kw = {**BOTH, **BWD, **LABELLED}[name]
    assert ce_bwd(**kw) == status


@pytest.mark.parametrize("name", {**BOTH, **FWD, **TAUGHT})
def test_distillation_fwd_refusals(name):
    status, kw = {**BOTH, **FWD, **TAUGHT}[name]
    assert kd_fwd(**kw) == status


@pytest.mark.parametrize("name", {**BOTH, **BWD, **TAUGHT, "no_picked": 0})
def test_distillation_bwd_refusals(name):
    status, kw = {**BOTH, **BWD, **TAUGHT, "no_picked": (1, dict(picked=None))}[name]
    assert kd_bwd(**kw) == status


def test_workspaces():
    f, b = sc.scalify_cross_entropy_fwd_workspace_size, sc.scalify_cross_entropy_bwd_workspace_size
    kf, kb = sc.scalify_distillation_fwd_workspace_size, sc.scalify_distillation_bwd_workspace_size
    assert f(-1, V, D, sc.F16) == 0 and f(R, 0, D, sc.F16) == 0 and f(R, V, 0, sc.F16) == 0 and f(R, V, D, sc.F32) == 0
    assert b(R, V, D, sc.F16, 2) == 0 and b(R, V, (1 << 20) + 1, sc.F16, 1) == 0
    assert kf(R, V, D, 0, sc.F16) == 0 and kf(R, V, D, 257, sc.F16) == 0 and kb(R, V, D, 8, sc.F16, 5) == 0
    # a matrix whose rows are no whole groups of 16 bytes is copied as F16, at most 512 MiB at a time
    assert f(4096, 32000, 2048, sc.E4M3) == f(4096, 32000, 2048, sc.F16) == f(4096, 32000, 2048, sc.E5M2)
    assert f(4096, 32000, 2056, sc.E4M3) > f(4096, 32000, 2056, sc.F16) + 32000 * 2056 * 2
    assert f(4096, 32000, 2049, sc.F16) == f(4096, 32000, 2049, sc.E4M3)
    assert f(300, 1 << 20, 4100, sc.E4M3) < 700 << 20
    # the logits are not kept: 8 bytes for 128 of them forward, at most 512 MiB (of their gradient) backward
    assert f(16384, 131072, 64, sc.F16) < 16384 * 131072 * 4 / 50
    assert b(16384, 1 << 20, 64, sc.F16, 0) < 900 << 20
    # the dynamic rescale keeps dw in fp32, but for few rows
    assert b(300, V, D, sc.F16, 1) - b(300, V, D, sc.F16, 0) == 4 * V * D
    assert b(R, V, D, sc.F16, 1) == b(R, V, D, sc.F16, 0)
    # sums of byte counts past 32 bits
    assert b(1 << 20, 1 << 20, 8192, sc.F16, 1) > 1 << 35


def test_binding_checks():
    x = sc.ScaledArray(torch.zeros((4, 64), dtype=torch.int16), sc.F16)
    w = sc.ScaledArray(torch.zeros((9, 64), dtype=torch.int16), sc.F16)
    loss = torch.zeros(4)
    with pytest.raises(ValueError):
        sc.scalify_cross_entropy_fwd(x, w, torch.zeros(4, dtype=torch.int32), loss)
    with pytest.raises(ValueError):
        sc.scalify_cross_entropy_fwd(x, w, torch.zeros(5, dtype=torch.int64), loss)
    t = sc.ScaledArray(torch.zeros((4, 8), dtype=torch.int16), sc.F16)
    with pytest.raises(ValueError):
        sc.scalify_distillation_fwd(x, w, t, torch.zeros((4, 7), dtype=torch.int64), loss)
    with pytest.raises(ValueError):
        sc.scalify_distillation_fwd(x, w, t, torch.zeros((8, 4), dtype=torch.int64).t(), loss)
