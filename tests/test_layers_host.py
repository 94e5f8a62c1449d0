"""Host-side checks of the RMS norm and attention entry points (no GPU): sizes
of their workspaces and the refusal of bad arguments before any launch (the
pointers are never dereferenced; every case differs in one point from a call
whose other arguments are valid, and the valid call itself is never made)."""
import ctypes

import pytest

from paper_2407_17353_amd import binding as sc

FAKE = 0x10000000
GB = 1 << 30


def arr(rows, cols, dtype=sc.F16, ld=None, trans=0, at=0, scale=None, data=True):
    """Matrix number `at` of a call, in memory of its own."""
    ld = ld if ld is not None else max(16, (cols + 15) // 16 * 16)
    return sc.CScaledArray(FAKE + at * GB if data else None, FAKE + 64 * GB + 256 * at if scale is None else scale or None,
                           dtype, trans, rows, cols, ld)


def ref(x):
    return ctypes.byref(x) if x is not None else None


# ---------------------------------------------------------------- RMS norm

def rms_fwd(x, res, s, out, row=None, blk=None, target=0, eps=1e-5, gamma=None, pre=None):
    return sc.load_library().scalify_rmsnorm_fwd(ref(x), ref(res), gamma, eps, ref(s), ref(out), row, blk, target, 1, pre, None)


R, D = 20, 64
X, RES, SUM, OUT = (lambda **k: arr(R, D, **{"at": 0, **k})), (lambda **k: arr(R, D, **{"at": 1, **k})), \
    (lambda **k: arr(R, D, **{"at": 2, **k})), (lambda **k: arr(R, D, sc.E4M3, **{"at": 3, **k}))

RMS_FWD = {
    "no_x": (1, dict(x=None)), "no_out": (1, dict(out=None)), "no_out_scale": (1, dict(out=OUT(scale=0))),
    "sum_without_residual": (1, dict(res=None)), "no_sum_scale": (1, dict(s=SUM(scale=0))),
    "no_data": (1, dict(x=X(data=False))), "no_residual_data": (1, dict(res=RES(data=False))),
    "x_type": (2, dict(x=X(dtype=7))), "out_f32": (2, dict(out=arr(R, D, sc.F32, at=3))),
    "residual_f32": (2, dict(res=RES(dtype=sc.F32))), "sum_f32": (2, dict(s=SUM(dtype=sc.F32))),
    "blocks_of_f16": (2, dict(out=arr(R, D, sc.F16, at=3), blk=FAKE + 32 * GB)),
    "both_scales": (7, dict(row=FAKE + 33 * GB, blk=FAKE + 32 * GB)), "target": (7, dict(target=2000)),
    "eps_negative": (7, dict(eps=-1.0)), "eps_nan": (7, dict(eps=float("nan"))),
    "rows": (3, dict(out=arr(R + 1, D, sc.E4M3, at=3))), "residual_columns": (3, dict(res=arr(R, D - 1, at=1))),
    "negative": (3, dict(x=arr(-1, D))), "too_wide": (3, dict(x=arr(R, 8193), res=None, s=None, out=arr(R, 8193, sc.E4M3, at=3))),
    "no_columns": (3, dict(x=arr(R, 0), res=None, s=None, out=arr(R, 0, sc.E4M3, at=3))), "small_ld": (3, dict(x=X(ld=48))),
    "trans": (4, dict(x=X(trans=1))), "sum_trans": (4, dict(s=SUM(trans=1))),
    "ld": (5, dict(x=X(ld=68))), "gamma": (5, dict(gamma=FAKE + 4)), "row_scale": (5, dict(row=FAKE + 33 * GB + 2)),
    "block_scale": (5, dict(blk=FAKE + 32 * GB + 1)), "pre_out": (5, dict(pre=FAKE + 8)),
    "out_over_x": (4, dict(out=arr(R, D, sc.E4M3, at=0))), "sum_in_residual": (4, dict(s=SUM(at=1, ld=96))),
    "sum_over_out": (4, dict(s=SUM(at=3))), "out_scale_of_x": (4, dict(out=OUT(scale=FAKE + 64 * GB))),
    "sum_scale_of_residual": (4, dict(s=SUM(scale=FAKE + 64 * GB + 256))),
    "sum_scale_of_out": (4, dict(s=SUM(scale=FAKE + 64 * GB + 768))),
}


@pytest.mark.parametrize("name", RMS_FWD)
def test_rmsnorm_fwd_refusals(name):
    status, kw = RMS_FWD[name]
    assert rms_fwd(**{"x": X(), "res": RES(), "s": SUM(), "out": OUT(), **kw}) == status


def rms_bwd(dy, x, ds, dx, mode=1, target=0, eps=1e-5, dg=None, ws=FAKE + 96 * GB, nws=1 << 40):
    return sc.load_library().scalify_rmsnorm_bwd(ref(dy), ref(x), ref(ds), None, eps, ref(dx), dg, mode, target, 1, None, None, ws,
                                                 nws, None)


RMS_BWD = {
    "no_dy": (1, dict(dy=None)), "no_dx_scale": (1, dict(dx=SUM(scale=0))), "dx_f32": (2, dict(dx=SUM(dtype=sc.F32))),
    "dsum_f32": (2, dict(ds=arr(R, D, sc.F32, at=3))), "delayed": (7, dict(mode=2)),
    "target": (7, dict(target=-2000)), "eps": (7, dict(eps=float("inf"))), "rows": (3, dict(dy=arr(R - 1, D))),
    "wide": (3, dict(x=arr(0, 9000, at=1), dy=arr(0, 9000), ds=None, dx=arr(0, 9000, at=2))),
    "trans": (4, dict(ds=arr(R, D, at=3, trans=1))), "dx_in_dy": (4, dict(dx=SUM(at=0, ld=80))),
    "dx_over_dsum": (4, dict(dx=arr(R, D, sc.E4M3, at=3))), "dgamma": (5, dict(dg=FAKE + 4)), "ld": (5, dict(dy=arr(R, D, ld=68))),
    "no_ws": (6, dict(ws=None)), "small_ws": (6, dict(nws=256)), "ws_align": (6, dict(ws=FAKE + 96 * GB + 128)),
}


@pytest.mark.parametrize("name", RMS_BWD)
def test_rmsnorm_bwd_refusals(name):
    status, kw = RMS_BWD[name]
    assert rms_bwd(**{"dy": X(), "x": RES(), "ds": arr(R, D, at=3), "dx": SUM(), **kw}) == status


def test_rmsnorm_workspace():
    f = sc.scalify_rmsnorm_bwd_workspace_size
    assert f(0, 64) == 256 and f(1, 64) == 256 + 16 + 256 and f(-1, 64) == 0 and f(4, 8193) == 0
    # 4 numbers a row, a partial row of dgamma for each group of rows up to 1024
    assert f(100000, 4096) == 256 + 16 * 100000 + 4 * 1024 * 4096
    assert f(8, 1024) == 256 + 16 * 8 + 4 * 2 * 1024


# ---------------------------------------------------------------- attention

H, HKV, HD, B, T = 4, 2, 64, 2, 40


def opts(**kw):
    o = dict(heads=H, kv_heads=HKV, head_dim=HD, causal=1, batch=B, softmax_scale=0.125, q_start=None, k_start=None, k_len=None,
             max_q=0, max_k=0)
    o.update(kw)
    return sc.CAttentionOpts(*o.values())


def q_like(at, **kw):
    return arr(T, H * HD, **{"at": at, **kw})


def k_like(at, **kw):
    return arr(T, HKV * HD, **{"at": at, **kw})


def attn_fwd(q, k, v, out, o, lse=None, ws=FAKE + 96 * GB, nws=1 << 40):
    return sc.load_library().scalify_attention_fwd(ref(q), ref(k), ref(v), ref(out), lse, ref(o), 1, ws, nws, None)


LONG = dict(q=arr(B, H * HD, at=0), k=arr(B * 100000, HKV * HD, at=1), v=arr(B * 100000, HKV * HD, at=2), out=arr(B, H * HD, at=3))

ATTN = {
    "no_q": (1, dict(q=None)), "no_opts": (1, dict(o=None)), "no_out_scale": (1, dict(out=q_like(3, scale=0))),
    "no_data": (1, dict(k=k_like(1, data=False))), "q_f32": (2, dict(q=q_like(0, dtype=sc.F32))),
    "out_f32": (2, dict(out=q_like(3, dtype=sc.F32))), "v_type": (2, dict(v=k_like(2, dtype=9))),
    "heads": (3, dict(o=opts(heads=3))), "no_heads": (3, dict(o=opts(heads=0))), "no_kv_heads": (3, dict(o=opts(kv_heads=0))),
    "head_dim_8": (3, dict(o=opts(head_dim=8))), "head_dim_72": (3, dict(o=opts(head_dim=72))),
    "head_dim_256": (3, dict(o=opts(head_dim=256))), "columns": (3, dict(k=arr(T, HKV * HD + 16, at=1))),
    "rows_of_v": (3, dict(v=arr(T + 2, HKV * HD, at=2))), "rows_of_out": (3, dict(out=arr(T + 2, H * HD, at=3))),
    "batch": (3, dict(o=opts(batch=0))), "uneven": (3, dict(o=opts(batch=3))), "max_q": (3, dict(o=opts(max_q=-1))),
    "small_ld": (3, dict(q=q_like(0, ld=128))), "huge_ld": (3, dict(q=q_like(0, ld=1 << 23))),
    "too_many": (3, dict(o=opts(batch=1, q_start=FAKE + 40 * GB), q=arr(1 << 30, H * HD, at=0), out=arr(1 << 30, H * HD, at=3))),
    "grid": (3, dict(o=opts(batch=1 << 30, q_start=FAKE + 40 * GB, k_start=FAKE + 41 * GB))),
    "trans": (4, dict(q=q_like(0, trans=1))), "out_over_q": (4, dict(out=q_like(0))), "out_in_k": (4, dict(out=q_like(1, ld=320))),
    "columns_that_meet": (4, dict(q=q_like(0, ld=512), out=sc.CScaledArray(FAKE + 2 * 240, FAKE, sc.F16, 0, T, H * HD, 512))),
    "scale_of_q": (4, dict(out=q_like(3, scale=FAKE + 64 * GB))), "scale_of_k": (4, dict(out=q_like(3, scale=FAKE + 64 * GB + 256))),
    "ld": (5, dict(k=k_like(1, ld=132))), "lse": (5, dict(lse=FAKE + 2)), "starts": (5, dict(o=opts(q_start=FAKE + 4))),
    "lengths": (5, dict(o=opts(k_len=FAKE + 4))), "causal": (7, dict(o=opts(causal=2))), "scale_0": (7, dict(o=opts(softmax_scale=0.0))),
    "scale_nan": (7, dict(o=opts(softmax_scale=float("nan")))), "scale_inf": (7, dict(o=opts(softmax_scale=float("inf")))),
    "no_ws": (6, dict(LONG, ws=None)), "small_ws": (6, dict(LONG, nws=4096)), "ws_align": (6, dict(LONG, ws=FAKE + 96 * GB + 16)),
}


@pytest.mark.parametrize("name", ATTN)
def test_attention_fwd_refusals(name):
    status, kw = ATTN[name]
    assert attn_fwd(**{"q": q_like(0), "k": k_like(1), "v": k_like(2), "out": q_like(3), "o": opts(), **kw}) == status


def attn_bwd(do, q, k, v, out, dq, dk, dv, o, lse=FAKE + 48 * GB, mode=1, target=0, ws=FAKE + 96 * GB, nws=1 << 40):
    return sc.load_library().scalify_attention_bwd(ref(do), ref(q), ref(k), ref(v), ref(out), lse, ref(dq), ref(dk), ref(dv), ref(o),
                                                   mode, target, 1, None, ws, nws, None)


ATTN_BWD = {
    "no_dout": (1, dict(do=None)), "no_lse": (1, dict(lse=None)), "no_dk_scale": (1, dict(dk=k_like(6, scale=0))),
    "out_8_bit": (2, dict(out=q_like(4, dtype=sc.E4M3))), "dq_f32": (2, dict(dq=q_like(5, dtype=sc.F32))),
    "dout_f32": (2, dict(do=q_like(0, dtype=sc.F32))), "rows_of_dk": (3, dict(dk=arr(T - 2, HKV * HD, at=6))),
    "heads": (3, dict(o=opts(heads=5))), "head_dim": (3, dict(o=opts(head_dim=40))), "dv_trans": (4, dict(dv=k_like(7, trans=1))),
    "dq_over_q": (4, dict(dq=q_like(1))), "dk_over_dv": (4, dict(dk=k_like(7))), "dk_in_dout": (4, dict(dk=k_like(0, ld=512))),
    "scale_shared": (4, dict(dk=k_like(6, scale=FAKE + 64 * GB + 5 * 256))), "scale_of_v": (4, dict(dv=k_like(7, scale=FAKE + 64 * GB + 3 * 256))),
    "ld": (5, dict(dq=q_like(5, ld=260))), "lse_align": (5, dict(lse=FAKE + 1)), "delayed": (7, dict(mode=2)),
    "target": (7, dict(target=1001)), "causal": (7, dict(o=opts(causal=-1))), "no_ws": (6, dict(ws=None)), "small_ws": (6, dict(nws=1000)),
}


@pytest.mark.parametrize("name", ATTN_BWD)
def test_attention_bwd_refusals(name):
    status, kw = ATTN_BWD[name]
    base = {"do": q_like(0), "q": q_like(1), "k": k_like(2), "v": k_like(3), "out": q_like(4), "dq": q_like(5), "dk": k_like(6),
            "dv": k_like(7), "o": opts()}
    assert attn_bwd(**{**base, **kw}) == status


def test_attention_workspaces():
    f, b = sc.scalify_attention_fwd_workspace_size, sc.scalify_attention_bwd_workspace_size
    assert f(4 * 4096, 4 * 4096, opts(batch=4, heads=32, kv_heads=32)) == 0          # the grid is full without splits
    assert f(1, 100, opts(batch=1)) == 0                                            # too few keys
    n = f(1, 100000, opts(batch=1))
    assert n > 0 and n % ((HD + 2) * 4 * H) == 0                                    # a partial result a split
    assert f(3, 100, opts(batch=2)) == 0 and f(1, 100, opts(batch=1, head_dim=24)) == 0
    assert b(T, T, opts(), 0) == 256 + 4 * (2 * T * H + T * HKV)
    assert b(T, T, opts(), 1) == b(T, T, opts(), 0) + 4 * HD * T * (H + 2 * HKV)
    assert b(T, T, opts(), 2) == 0 and b(T, T, opts(heads=3), 0) == 0


def test_binding_checks():
    import torch
    q = sc.ScaledArray(torch.zeros((4, 64), dtype=torch.int16), sc.F16)
    with pytest.raises(ValueError):
        sc.attention_opts(q, 1, batch=2, q_start=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        sc.attention_opts(q, 1, batch=2, k_len=torch.zeros(2, dtype=torch.int32))
    o = sc.attention_opts(q, 2, causal=True)
    assert (o.heads, o.kv_heads, o.head_dim, o.causal, o.batch) == (2, 2, 32, 1, 1) and abs(o.softmax_scale - 32 ** -0.5) < 1e-7
