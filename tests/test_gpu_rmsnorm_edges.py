"""GPU parity of the RMS norm where its arguments meet their edges."""
import numpy as np
import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests import test_gpu_rmsnorm as rms
from tests.helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3, E5M2, F32 = sc.F16, sc.E4M3, sc.E5M2, sc.F32


@pytest.mark.parametrize("ex,er", [(0, -80), (-80, 0), (0, -126), (1, -2), (-70, -127), (127, 10)])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
@pytest.mark.parametrize("fx,fr", [(F16, F16), (E4M3, F16), (F16, E5M2), (F32, F16)])
@pytest.mark.parametrize("D,scales", [(64, "row"), (1024, "mx"), (2000, "one"), (4096, "row"), (5000, "mx")])
def test_residual_without_a_stored_sum(D, scales, fx, fr, eps, ex, er):
    """The fp32 sum of both is normalized, of any magnitude that their scales give it:
    rows where either is zero lie on the other's scale alone."""
    say(f"rmsnorm fwd no sum {D} {scales} {rms.NAMES[fx]} {rms.NAMES[fr]} {eps} {ex} {er}")
    R, target = 9, 7
    x, r = lr.values(R, D, fx, 1), lr.values(R, D, fr, 2)
    for i in (1, 4):
        x[i] = torch.zeros_like(x[i])
    for i in (2, 4, 8):
        r[i] = torch.zeros_like(r[i])
    X, S, out = lr.scaled(x, fx, ex), lr.scaled(r, fr, er), lr.empty(R, D, E4M3)
    pre = torch.full((R, D), 9.0, device=DEV)
    row = torch.full((R,), 7.0, device=DEV) if scales == "row" else None
    blk = torch.full((sc.scalify_mx_packed_bytes(R, D),), 0xEE, dtype=torch.uint8, device=DEV) if scales == "mx" else None
    sc.scalify_rmsnorm_fwd(X, out, residual=S, eps=eps, row_scale=row, block_scale=blk, target_log2=target, pre_out=pre)
    torch.cuda.synchronize()
    e = max(ex, er)
    # (each part on the larger scale, then their sum, in fp32)
    h = (x.to(lr.F64) * 2.0 ** (ex - e)).float() + (r.to(lr.F64) * 2.0 ** (er - e)).float()
    h = h.to(lr.F64)
    m = h.square().mean(1, keepdim=True) + np.float64(np.float32(eps))
    y = torch.where(m > 0, h / torch.where(m > 0, m, torch.ones_like(m)).sqrt(), torch.zeros_like(h))
    pre = pre.cpu()
    assert ((pre.to(lr.F64) - y).abs() <= 24 * lr.U * y.abs() + 2.0 ** -140).all()
    p = pre.numpy()
    sh = np.zeros((R, D), dtype=np.int64)
    if scales == "row":
        ee = rms.exponents(np.abs(p).max(1), target)
        assert np.array_equal(row.cpu().numpy(), np.ldexp(np.float32(1), ee.astype(np.int32)))
        sh += ee[:, None]
    if scales == "mx":
        pad = np.zeros((R, -(-D // 32) * 32), dtype=np.float32)
        pad[:, :D] = np.abs(p)
        ee = rms.exponents(pad.reshape(R, -1, 32).max(2), target)
        assert torch.equal(blk, sc.scalify_mx_pack_block_scales(torch.from_numpy((ee + 127).astype(np.uint8)).to(DEV), D))
        sh += np.repeat(ee, 32, axis=1)[:, :D]
    assert np.array_equal(lr.codes(out), lr.cast(np.ldexp(p.astype(np.float64), -sh), E4M3))


@pytest.mark.parametrize("eps", [1e-5, 3e-9, 1e-30])
@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("D", [300, 2048, 5000])
def test_backward_rows_of_subnormal_numbers(D, mode, eps):
    """F32 rows whose largest number is 2^-126 to 2^-149: eps alone is their mean square."""
    say(f"rmsnorm bwd subnormal {D} {mode} {eps}")
    x = lr.values(9, D, F32, 4)
    for i, e in enumerate([0, -126, -130, -134, -138, -142, -146, -149]):
        x[i] = torch.ldexp(x[i].clamp(-1.9, 1.9), torch.tensor(e))
    assert (x[7] != 0).any()
    dy = lr.values(9, D, F16, 5)
    got = rms.run_bwd(dy, F16, x, F32, None, None, fo=F16, mode=mode, eps=eps)
    rms.check_bwd(dy, x, None, None, F16, mode, 0, got, eps=eps)


@pytest.mark.parametrize("eps", [0.0, 1e-5, 1e-30])
def test_rows_of_subnormal_numbers(eps):
    x = lr.values(9, 300, F32, 4)
    for i, e in enumerate([0, -126, -130, -134, -138, -142, -146, -149]):
        x[i] = torch.ldexp(x[i].clamp(-1.9, 1.9), torch.tensor(e))
    for scales in ("row", "mx"):
        got = rms.run_fwd(x, F32, None, None, scales=scales, target=7, eps=eps)
        rms.check_fwd(x, F32, None, None, F16, F16, E4M3, scales, 7, eps, got)
