"""GPU parity of the scaled RMS norm, forward and backward, through the C ABI,
against plain 64-bit forms. The kernels export the values they cast (`pre_out`):
  N1  those values against 64 bits: the row's sum of squares adds 16 terms in a
      lane, then 64 lanes, then up to 8 waves (29 additions at most on the way
      of a term), its root halves that; with the divisions, the root and the
      products under 24 u, u = 2^-24;
  N2  codes, scales and statistics exactly: the oracle's cast, and the power of
      two of the largest magnitude, of the kernel's own values;
  N3  dgamma within its additions' bound.
"""
import numpy as np
import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests.helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3, E5M2, F32 = sc.F16, sc.E4M3, sc.E5M2, sc.F32
NAMES = {F16: "f16", E4M3: "e4m3", E5M2: "e5m2", F32: "f32", None: "none"}


def _gamma(D, seed=3):
    return 1.0 + 0.2 * torch.randn(D, generator=torch.Generator().manual_seed(seed))


def stored_sum(x, ex, r, er, fmt):
    """The scaled add, one rounding of the sum, cast: data (64 bits), exponent, codes."""
    e = max(ex, er)
    h = (x.to(lr.F64) * 2.0 ** (ex - e) + r.to(lr.F64) * 2.0 ** (er - e)).float()
    c = lr.cast(h.numpy(), fmt)
    t = torch.from_numpy(c.view(np.int16) if fmt == F16 else c).view(lr.TORCH[fmt])
    return t.to(lr.F64), e, c


def run_fwd(x, fx, gamma=None, r=None, fr=F16, fs=F16, fo=E4M3, ex=-2, er=1, scales="one", target=0, eps=1e-5, sat=True,
            ld=None):
    R, D = x.shape
    X = lr.scaled(x, fx, ex, ld=ld)
    res = lr.scaled(r, fr, er) if r is not None else None
    s = lr.empty(R, D, fs) if r is not None else None
    out = lr.empty(R, D, fo, ld=(D + 48) // 16 * 16)
    pre = torch.full((R, D), 9.0, device=DEV)
    row = torch.full((R,), 7.0, device=DEV) if scales == "row" else None
    blk = torch.full((sc.scalify_mx_packed_bytes(R, D),), 0xEE, dtype=torch.uint8, device=DEV) if scales == "mx" else None
    sc.scalify_rmsnorm_fwd(X, out, residual=res, sum_out=s, gamma=gamma.to(DEV) if gamma is not None else None, eps=eps,
                           row_scale=row, block_scale=blk, target_log2=target, saturate=sat, pre_out=pre)
    torch.cuda.synchronize()
    return out, s, pre.cpu(), row, blk


def exponents(a, target):
    """Per-entry exponent of largest magnitudes (numpy fp32)."""
    e = np.zeros(a.shape, dtype=np.int64)
    m = np.isfinite(a) & (a > 0)
    e[m] = np.frexp(a[m].astype(np.float64))[1] - 1 - target
    return np.clip(e, -127, 127)


def check_fwd(x, fx, gamma, r, fr, fs, fo, scales, target, eps, got, ex=-2, er=1, sat=True):
    out, s, pre, row, blk = got
    R, D = x.shape
    if r is not None:
        h, e, c = stored_sum(x, ex, r, er, fs)
        assert np.array_equal(lr.codes(s), c) and lr.log2_of(s) == e
    else:
        h = x.to(lr.F64)
    g = gamma.to(lr.F64) if gamma is not None else torch.ones(D, dtype=lr.F64)
    m = h.square().mean(1, keepdim=True) + np.float64(np.float32(eps))
    y = torch.where(m > 0, h / torch.where(m > 0, m, torch.ones_like(m)).sqrt() * g, torch.zeros_like(h))
    assert ((pre.to(lr.F64) - y).abs() <= 24 * lr.U * y.abs() + 2.0 ** -140).all()
    p = pre.numpy()
    sh = np.zeros((R, D), dtype=np.int64)
    if scales == "row":
        e = exponents(np.abs(p).max(1), target)
        assert np.array_equal(row.cpu().numpy(), np.ldexp(np.float32(1), e.astype(np.int32)))
        sh += e[:, None]
    if scales == "mx":
        nb = -(-D // 32)
        pad = np.zeros((R, nb * 32), dtype=np.float32)
        pad[:, :D] = np.abs(p)
        e = exponents(pad.reshape(R, nb, 32).max(2), target)
        nat = torch.from_numpy((e + 127).astype(np.uint8)).to(DEV)
        assert torch.equal(blk, sc.scalify_mx_pack_block_scales(nat, D))
        sh += np.repeat(e, 32, axis=1)[:, :D]
    assert float(out.scale.item()) == 1.0
    want = lr.cast(np.ldexp(p.astype(np.float64), -sh), fo, 0, sat)
    assert np.array_equal(lr.codes(out), want)
    # the padding of the rows is as it was
    full = out.data.as_strided((R, out.data.stride(0)), (out.data.stride(0), 1))[:, D:].cpu().numpy()
    assert (full.view(np.uint8) == 0x5A).all()


FWD = [
    # R, D, x, residual, sum, out, scales, target
    (1, 1, F16, None, F16, E4M3, "row", 0), (3, 17, F16, F16, F16, E4M3, "mx", 8), (5, 32, E4M3, None, F16, E5M2, "one", 0),
    (70, 100, F16, E4M3, F16, E4M3, "mx", 7), (9, 1000, F16, F16, F16, F16, "one", 0), (6, 1024, F16, F16, F16, E4M3, "row", 7),
    (7, 1025, F32, F16, F16, E4M3, "row", 7), (65, 2048, F16, E5M2, E5M2, E5M2, "mx", 14), (33, 2049, E5M2, F16, F16, F16, "row", 3),
    (8, 4096, F16, F16, F16, E4M3, "row", 7), (128, 4096, F16, F16, F16, E4M3, "mx", 7), (10, 4100, E4M3, E4M3, E4M3, E4M3, "one", 0),
    (5, 8192, F16, F16, F16, E4M3, "mx", 7), (4, 8191, F32, None, F16, E4M3, "row", 7), (2000, 256, F16, F16, F16, E4M3, "mx", 7),
    (1300, 2048, F32, F16, F16, E4M3, "one", 0), (3000, 64, F16, None, F16, F16, "row", 0), (257, 8192, E4M3, F16, F16, E4M3, "row", 7),
]


@pytest.mark.parametrize("R,D,fx,fr,fs,fo,scales,target", FWD, ids=lambda v: str(v))
def test_forward(R, D, fx, fr, fs, fo, scales, target):
    say(f"rmsnorm fwd {R}x{D} {NAMES[fx]} + {NAMES[fr]} -> {NAMES[fo]} {scales}")
    x = lr.values(R, D, fx, R + D)
    r = lr.values(R, D, fr, R + D + 1) if fr is not None else None
    gamma = _gamma(D) if D % 3 else None
    got = run_fwd(x, fx, gamma, r, fr, fs, fo, scales=scales, target=target)
    check_fwd(x, fx, gamma, r, fr, fs, fo, scales, target, 1e-5, got)
    again = run_fwd(x, fx, gamma, r, fr, fs, fo, scales=scales, target=target)
    assert np.array_equal(lr.codes(got[0]), lr.codes(again[0]))


@pytest.mark.parametrize("eps", [0.0, 1e-6, 0.5])
@pytest.mark.parametrize("fx", [F16, F32])
def test_rows_of_any_magnitude(fx, eps):
    """Zero rows, tiny and huge ones (F32: squares far outside the range)."""
    x = lr.values(12, 300, F32, 4).float()
    span = [0, 1, -1, 10, -13, 14] if fx == F16 else [0, 60, -60, 120, -120, 126]
    for i, e in enumerate(span):
        x[i] = torch.ldexp(x[i].clamp(-1.9, 1.9), torch.tensor(e))
    x[6] = 0
    x[7] = -0.0
    x = x.to(lr.TORCH[fx])
    for scales in ("row", "mx"):
        got = run_fwd(x, fx, None, None, scales=scales, target=7, eps=eps)
        check_fwd(x, fx, None, None, F16, F16, E4M3, scales, 7, eps, got)


def test_values_that_are_not_finite():
    """A NaN or infinity spoils its own row only; the statistic of a scale skips NaN."""
    x = lr.values(70, 200, F16, 5)
    clean = run_fwd(x, F16, None, None, scales="mx", target=7)
    y = x.clone()
    y[3, 7], y[66, 0] = float("nan"), float("inf")
    for scales in ("mx", "row", "one"):
        a, b = run_fwd(x, F16, None, None, scales=scales, target=7), run_fwd(y, F16, None, None, scales=scales, target=7)
        keep = [i for i in range(70) if i not in (3, 66)]
        assert np.array_equal(lr.codes(a[0])[keep], lr.codes(b[0])[keep])
        assert lr.data(b[0])[3].isnan().all()
        assert lr.data(b[0])[66, 0].isnan() and (lr.data(b[0])[66, 1:] == 0).all()
    assert clean[0].shape == (70, 200)


def test_in_place():
    """The sum over the residual stream and the output over the branch."""
    R, D = 40, 513
    x, r = lr.values(R, D, F16, 1), lr.values(R, D, F16, 2)
    X, S = lr.scaled(x, F16, -2), lr.scaled(r, F16, 1)
    one = torch.zeros(1, device=DEV)
    out, s = sc.ScaledArray(X.data, F16, one), sc.ScaledArray(S.data, F16, one.clone())
    want = run_fwd(x, F16, None, r, fo=F16)
    sc.scalify_rmsnorm_fwd(X, out, residual=S, sum_out=s)
    torch.cuda.synchronize()
    assert np.array_equal(lr.codes(s), lr.codes(want[1])) and np.array_equal(lr.codes(out), lr.codes(want[0]))


@pytest.mark.parametrize("dx", [(-100, 27), (100, -100), (-127, 127), (127, -120)])
def test_scales_far_apart(dx):
    x, r = lr.values(9, 64, F16, 1), lr.values(9, 64, F16, 2)
    got = run_fwd(x, F16, None, r, ex=dx[0], er=dx[1])
    check_fwd(x, F16, None, r, F16, F16, E4M3, "one", 0, 1e-5, got, ex=dx[0], er=dx[1])


# ---------------------------------------------------------------- backward

def run_bwd(dy, fdy, x, fx, gamma=None, ds=None, fds=F16, fo=F16, mode=sc.RESCALE_AMAX, target=0, eps=1e-5, edy=-7, ex=1, eds=-5,
            ws=None):
    R, D = x.shape
    DY, X = lr.scaled(dy, fdy, edy), lr.scaled(x, fx, ex)
    DS = lr.scaled(ds, fds, eds) if ds is not None else None
    out = lr.empty(R, D, fo, ld=(D + 48) // 16 * 16)
    pre, dg = torch.full((R, D), 9.0, device=DEV), torch.full((D,), 9.0, device=DEV)
    amax = torch.full((1,), -1.0, device=DEV)
    if ws is None:
        ws = sc.workspace(sc.scalify_rmsnorm_bwd_workspace_size(R, D), DEV)
        ws.fill_(0xFF)
    sc.scalify_rmsnorm_bwd(DY, X, out, dsum=DS, gamma=gamma.to(DEV) if gamma is not None else None, eps=eps, rescale=mode,
                           target_log2=target, dgamma=dg, amax_out=amax, pre_out=pre, ws=ws)
    torch.cuda.synchronize()
    return out, pre.cpu(), dg.cpu(), float(amax.item())


def check_bwd(dy, x, gamma, ds, fo, mode, target, got, eps=1e-5, edy=-7, ex=1, eds=-5):
    out, pre, dg, amax = got
    R, D = x.shape
    h, d = x.to(lr.F64), dy.to(lr.F64)
    g = d * (gamma.to(lr.F64) if gamma is not None else 1.0)
    m = h.square().mean(1, keepdim=True) + np.float64(np.float32(eps))
    inv = torch.where(m > 0, 1 / torch.where(m > 0, m, torch.ones_like(m)).sqrt(), torch.zeros_like(m))
    dn = inv * (g - h * inv ** 2 * (g * h).mean(1, keepdim=True))
    mag = inv * (g.abs() + h.abs() * inv ** 2 * (g * h).abs().mean(1, keepdim=True))
    e, q = edy - ex, 0.0
    if ds is not None:
        e = max(e, eds)
        dn, mag = dn * 2.0 ** (edy - ex - e), mag * 2.0 ** (edy - ex - e)
        q = ds.to(lr.F64) * 2.0 ** (eds - e)
    want = dn + q
    # (the row's two sums, 29 additions on a term's way at most, and inv cubed: under 110 u of the terms)
    assert ((pre.to(lr.F64) - want).abs() <= 110 * lr.U * mag + 2 * lr.U * want.abs() + 2.0 ** -140).all()
    p = pre.numpy()
    a = np.abs(p[~np.isnan(p)]).max() if p.size else 0.0
    assert amax == a
    er = ((lr.floor_log2(a) or 0) - target if a > 0 else 0) if mode == sc.RESCALE_AMAX else 0
    eo = max(-127, min(127, e + er))
    assert lr.log2_of(out) == eo
    assert np.array_equal(lr.codes(out), lr.cast(p, fo, eo - e))
    t = (d * h * inv).abs().sum(0)
    assert ((dg.to(lr.F64) - (d * h * inv).sum(0)).abs() <= (30 + R / 256 + 100) * lr.U * t + 2.0 ** -140).all()
    full = out.data.as_strided((R, out.data.stride(0)), (out.data.stride(0), 1))[:, D:].cpu().numpy()
    assert (full.view(np.uint8) == 0x5A).all()


BWD = [
    # R, D, dy, x, dsum, out, mode, target
    (1, 1, F16, F16, None, F16, 1, 0), (3, 17, E5M2, F16, F16, E5M2, 1, 0), (70, 100, F16, E4M3, None, F16, 0, 0),
    (9, 1000, E5M2, F16, E5M2, E5M2, 1, 15), (6, 1024, F32, F16, F16, F16, 0, 0), (7, 1025, E5M2, F32, F16, E5M2, 1, 0),
    (65, 2048, F16, F16, F16, F16, 1, 4), (33, 2049, F16, E5M2, E4M3, E4M3, 0, 0), (8, 4096, E5M2, F16, F16, E5M2, 1, 0),
    (10, 4100, E4M3, F16, F16, E4M3, 1, 7), (5, 8192, F16, F16, F16, F16, 0, 0), (4, 8191, F32, F32, None, F16, 1, 0),
    (5000, 64, F16, F16, F16, F16, 0, 0), (2100, 2048, E5M2, F16, E5M2, E5M2, 1, 0), (1500, 4096, F16, F16, None, F16, 1, 0),
]


@pytest.mark.parametrize("R,D,fdy,fx,fds,fo,mode,target", BWD, ids=lambda v: str(v))
def test_backward(R, D, fdy, fx, fds, fo, mode, target):
    say(f"rmsnorm bwd {R}x{D} {NAMES[fdy]} {NAMES[fx]} {NAMES[fds]} -> {NAMES[fo]} mode {mode}")
    rows = -10 * torch.rand(R, generator=torch.Generator().manual_seed(1))
    dy, x = lr.values(R, D, fdy, R + D, rows=rows), lr.values(R, D, fx, R + D + 1)
    ds = lr.values(R, D, fds, R + D + 2, rows=rows) if fds is not None else None
    gamma = _gamma(D) if D % 3 else None
    got = run_bwd(dy, fdy, x, fx, gamma, ds, fds, fo, mode, target)
    check_bwd(dy, x, gamma, ds, fo, mode, target, got)
    again = run_bwd(dy, fdy, x, fx, gamma, ds, fds, fo, mode, target)
    assert np.array_equal(lr.codes(got[0]), lr.codes(again[0])) and torch.equal(got[2], again[2])


def test_backward_rows_of_any_magnitude():
    x = lr.values(8, 300, F32, 4).float()
    for i, e in enumerate([0, 60, -60, 100, -100]):
        x[i] = torch.ldexp(x[i].clamp(-1.9, 1.9), torch.tensor(e))
    x[6] = 0
    dy = lr.values(8, 300, F16, 5)
    for mode in (0, 1):
        got = run_bwd(dy, F16, x, F32, None, None, fo=F16, mode=mode, eps=1e-6)
        check_bwd(dy, x, None, None, F16, mode, 0, got, eps=1e-6)


def test_backward_differences():
    """dx and dgamma against central differences of the 64-bit forward."""
    R, D, eps = 4, 40, 1e-3
    x, dy, gamma = lr.values(R, D, F16, 1), lr.values(R, D, F16, 2), _gamma(D)
    out, pre, dg, _ = run_bwd(dy, F16, x, F16, gamma, mode=0, eps=eps)

    def loss(h, g):
        return float((dy.to(lr.F64) * h / (h.square().mean(1, keepdim=True) + eps).sqrt() * g).sum())
    h0, g0, step = x.to(lr.F64), gamma.to(lr.F64), 1e-5
    for i in range(R):
        for j in range(0, D, 7):
            d = torch.zeros_like(h0)
            d[i, j] = step
            num = (loss(h0 + d, g0) - loss(h0 - d, g0)) / (2 * step)
            assert abs(float(pre[i, j]) - num) <= 1e-5 * (1 + abs(num))
    for j in range(0, D, 5):
        d = torch.zeros_like(g0)
        d[j] = step
        num = (loss(h0, g0 + d) - loss(h0, g0 - d)) / (2 * step)
        assert abs(float(dg[j]) - num) <= 1e-5 * (1 + abs(num))


def test_backward_in_place_and_shared_scale():
    """dx over dy, its scale in the memory of dy's scale, in both modes."""
    R, D = 300, 700
    dy, x, ds = lr.values(R, D, F16, 1), lr.values(R, D, F16, 2), lr.values(R, D, F16, 3)
    for mode in (0, 1):
        want = run_bwd(dy, F16, x, F16, None, ds, mode=mode)
        DY, X, DS = lr.scaled(dy, F16, -7), lr.scaled(x, F16, 1), lr.scaled(ds, F16, -5)
        sc.scalify_rmsnorm_bwd(DY, X, DY, dsum=DS, rescale=mode)
        torch.cuda.synchronize()
        assert np.array_equal(lr.codes(DY), lr.codes(want[0])) and lr.log2_of(DY) == lr.log2_of(want[0])


def test_no_rows():
    for fx in (F16, F32):
        x = sc.ScaledArray(torch.empty((0, 64), dtype=sc.STORAGE_DTYPE[fx], device=DEV), fx, sc.scale_tensor(3, DEV))
        out = sc.ScaledArray(torch.empty((0, 64), dtype=torch.int16, device=DEV), F16, torch.zeros(1, device=DEV))
        dg, amax = torch.full((64,), 5.0, device=DEV), torch.full((1,), 5.0, device=DEV)
        sc.scalify_rmsnorm_fwd(x, out)
        torch.cuda.synchronize()
        assert out.scale.item() == 1.0
        sc.scalify_rmsnorm_bwd(x, x, out, dgamma=dg, amax_out=amax)
        torch.cuda.synchronize()
        assert out.scale.item() == 1.0 and amax.item() == 0.0 and (dg == 0).all()


def test_capture():
    R, D = 90, 1500
    dy, x, ds = lr.values(R, D, E5M2, 1), lr.values(R, D, F16, 2), lr.values(R, D, F16, 3)
    want = run_bwd(dy, E5M2, x, F16, None, ds, fo=E5M2)
    DY, X, DS = lr.scaled(dy, E5M2, -7), lr.scaled(x, F16, 1), lr.scaled(ds, F16, -5)
    ws = sc.workspace(sc.scalify_rmsnorm_bwd_workspace_size(R, D), DEV)
    outs = [lr.empty(R, D, E5M2) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    for o in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            sc.scalify_rmsnorm_bwd(DY, X, o, dsum=DS, ws=ws)
        graphs.append(g)
    for _ in range(3):
        ws.fill_(0xFF)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert np.array_equal(lr.codes(o), lr.codes(want[0])) and o.scale.item() == want[0].scale.item()
        run_bwd(dy, E5M2, x, F16, None, ds, fo=E5M2, ws=ws)


def test_offsets_past_32_bits():
    """Rows of matrices of 5 GB: the results of the same rows side by side."""
    R, D, ld = 70000, 64, 37000 // 8 * 8
    inputs = torch.empty((R, ld), dtype=torch.int16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    def pair(i, t=None):
        near = sc.ScaledArray(t if t is not None else torch.zeros((R, D), dtype=torch.int16, device=DEV), F16, sc.scale_tensor(i, DEV))
        st = inputs if t is not None else torch.empty_like(inputs)
        far = sc.ScaledArray(st[:, 64 * i:64 * i + 64], F16, sc.scale_tensor(i, DEV))
        far.data.copy_(near.data)
        return near, far
    x, r, d = (pair(i, torch.randn((R, D), generator=g, device=DEV).half().view(torch.int16)) for i in range(3))
    s, y, dx = (pair(i) for i in range(3, 6))
    ends = []
    for i in range(2):
        dg = torch.empty(D, device=DEV)
        sc.scalify_rmsnorm_fwd(x[i], y[i], residual=r[i], sum_out=s[i])
        sc.scalify_rmsnorm_bwd(d[i], s[i], dx[i], dsum=r[i], dgamma=dg)
        ends.append(dg)
    torch.cuda.synchronize()
    for a, b in (s, y, dx):
        assert torch.equal(a.data, b.data) and a.scale.item() == b.scale.item()
    assert torch.equal(*ends)
