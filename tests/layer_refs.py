"""Plain 64-bit forms of the RMS norm and of attention on ScaledArray data, and
bounds of the kernels' errors from their formats (CPU, torch float64). u = 2^-24
is half a step of fp32; F16 is off by at most 2^-11 of a value (2^-25 below its
normal range), E4M3 by 2^-4 (2^-10), E5M2 by 2^-3 (2^-17)."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import oracle as orc
from paper_2407_17353_amd import binding as sc

F64 = torch.float64
U = 2.0 ** -24
TORCH = {sc.E4M3: torch.float8_e4m3fn, sc.E5M2: torch.float8_e5m2, sc.F16: torch.float16, sc.F32: torch.float32}
HALF = {sc.E4M3: (2.0 ** -4, 2.0 ** -10), sc.E5M2: (2.0 ** -3, 2.0 ** -17), sc.F16: (2.0 ** -11, 2.0 ** -25)}
ELEMS16 = {sc.E4M3: 16, sc.E5M2: 16, sc.F16: 8, sc.F32: 4}


def values(R, C, fmt, seed, scale=1.0, rows=None):
    """N(0, scale^2) values (rows multiplied by 2^rows where given) in a format: a CPU tensor of that type."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((R, C), generator=g) * scale
    if rows is not None:
        x = x * torch.exp2(rows.float())[:, None]
    return x.to(TORCH[fmt])


def scaled(t, fmt, e=None, device="cuda", ld=None, fill=float("nan")):
    """ScaledArray of a CPU tensor in device rows ld elements apart whose padding holds `fill`."""
    R, C = t.shape
    ld = ld or -(-C // ELEMS16[fmt]) * ELEMS16[fmt]
    st = torch.full((max(R, 1), max(ld, 1)), fill, dtype=torch.float32).to(TORCH[fmt])
    st[:R, :C] = t
    st = st.view(sc.STORAGE_DTYPE[fmt]).to(device)[:R, :C]
    return sc.ScaledArray(st, fmt, sc.scale_tensor(e, device) if e is not None else None)


def empty(R, C, fmt, device="cuda", ld=None):
    """Output ScaledArray whose rows and padding hold the byte 0x5A and whose scale holds 3."""
    ld = ld or -(-C // ELEMS16[fmt]) * ELEMS16[fmt]
    st = torch.full((max(R, 1), max(ld, 1) * (2 if fmt == sc.F16 else 1)), 0x5A, dtype=torch.uint8, device=device)
    st = st.view(sc.STORAGE_DTYPE[fmt])
    return sc.ScaledArray(st[:R, :C], fmt, torch.full((1,), 3.0, device=device))


def codes(x):
    """Raw codes of a ScaledArray, as numpy."""
    a = x.data.cpu().numpy()
    return a.view(np.uint16) if x.fmt == sc.F16 else a


def data(x):
    """Data component of a ScaledArray in 64 bits."""
    return x.data.cpu().contiguous().view(TORCH[x.fmt]).to(F64)


def log2_of(x):
    return math.frexp(float(x.scale.item()))[1] - 1


def cast(y, fmt, shift=0, sat=True):
    """The oracle's cast of fp32 values times 2^-shift."""
    return orc.cast(fmt, np.ldexp(np.asarray(y, dtype=np.float64), -shift), sat)


def floor_log2(a):
    return math.frexp(float(a))[1] - 1 if a > 0 and math.isfinite(a) else None


# ---------------------------------------------------------------- attention

def spans(B, rows_q, rows_k, q_start=None, k_start=None, k_len=None):
    """(first query row, queries, first key row, keys) of every sequence."""
    out = []
    for b in range(B):
        q0, q1 = (q_start[b], q_start[b + 1]) if q_start is not None else (b * (rows_q // B), (b + 1) * (rows_q // B))
        k0, k1 = (k_start[b], k_start[b + 1]) if k_start is not None else (b * (rows_k // B), (b + 1) * (rows_k // B))
        out.append((q0, q1 - q0, k0, min(k1 - k0, k_len[b]) if k_len is not None else k1 - k0))
    return out


def admitted(a, b, causal):
    i, j = torch.arange(a)[:, None], torch.arange(b)[None, :]
    return (j <= i + b - a) if causal else torch.ones((a, b), dtype=torch.bool)


def attention(q, k, v, H, Hkv, alpha, seqs, causal, out_fmt):
    """out (data in units of v's) and lse of the data tensors q, k, v (alpha holds
    the scales), with bounds of the kernel's errors."""
    D = q.shape[1] // H
    Tq = q.shape[0]
    o, eo = torch.zeros((Tq, H * D), dtype=F64), torch.zeros((Tq, H * D), dtype=F64)
    lse, el = torch.full((H, Tq), -math.inf, dtype=F64), torch.zeros((H, Tq), dtype=F64)
    rel, sub = HALF[out_fmt]
    for q0, a, k0, b in seqs:
        see = admitted(a, b, causal)
        for h in range(H):
            u = h // (H // Hkv)
            x, y, z = q[q0:q0 + a, h * D:(h + 1) * D], k[k0:k0 + b, u * D:(u + 1) * D], v[k0:k0 + b, u * D:(u + 1) * D]
            if a == 0 or b == 0:
                continue
            s = (alpha * (x @ y.t())).masked_fill(~see, -math.inf)
            # a score: fp32 sums of D products, its factor and the maximum's subtraction
            es = torch.where(see, (D + 8) * 2 * U * alpha * (x.abs() @ y.abs().t()) + 8 * U * s.abs().nan_to_num(posinf=0.0), 0.0)
            es = es.amax(1, keepdim=True) + 16 * U
            p = torch.softmax(s, 1).nan_to_num(0.0)
            av = p @ z.abs()
            n = b / 16 + 80  # (additions of a result)
            at, cols = slice(q0, q0 + a), slice(h * D, (h + 1) * D)
            o[at, cols] = p @ z
            # P in F16 as 2^10 P relative to a score's exponential: half a step is 2^-11 of
            # it, and 2^-25 / 2^10 below the normal range (the row's sum is at least 1)
            err = av * (2 * es + 2.0 ** -11 + 2 * n * U) + 2.0 ** -35 * see.to(F64) @ z.abs()
            eo[at, cols] = err + (o[at, cols].abs() + err) * rel + sub
            lse[h, at] = torch.logsumexp(s, 1)
            el[h, at] = (2 * es[:, 0] + 2 * n * U + 8 * U * (lse[h, at].abs().nan_to_num(posinf=0.0) + s.abs().nan_to_num(posinf=0.0).amax(1) + 30))
    return o, eo, lse, el


def attention_grads(do, q, k, v, out, lse, H, Hkv, alpha, e_vo, seqs, causal):
    """dq, dk, dv in the units of their propagated scales, and bounds of the
    kernel's errors before their cast. out: data in units of 2^e_vo of v's;
    alpha holds the scales in the scores, and `lone` alone is the factor of dq, dk."""
    alpha, lone = alpha
    D = q.shape[1] // H
    g = [torch.zeros(t.shape, dtype=F64) for t in (q, k, v)]
    e = [torch.zeros(t.shape, dtype=F64) for t in (q, k, v)]
    for q0, a, k0, b in seqs:
        see = admitted(a, b, causal)
        if a == 0 or b == 0:
            continue
        rows_d = do[q0:q0 + a]
        for h in range(H):
            u = h // (H // Hkv)
            ch, cu = slice(h * D, (h + 1) * D), slice(u * D, (u + 1) * D)
            at, to = slice(q0, q0 + a), slice(k0, k0 + b)
            x, d, w = q[at, ch], rows_d[:, ch], out[at, ch] * 2.0 ** e_vo
            y, z = k[to, cu], v[to, cu]
            s = alpha * (x @ y.t())
            L = lse[h, at].to(F64)[:, None]
            p = torch.where(see, torch.exp(s - L), 0.0).nan_to_num(0.0)
            es = (D + 8) * 2 * U * alpha * (x.abs() @ y.abs().t()) + 8 * U * (s.abs() + L.abs().nan_to_num(posinf=0.0) + 20)
            dp = d @ z.t()
            dl = (d * w).sum(1, keepdim=True)
            ds = p * (dp - dl)
            edp = (D + 8) * 2 * U * (d.abs() @ z.abs().t() + (d * w).abs().sum(1, keepdim=True))
            # the power of two of dS: its bound over the head's sequence (any of the
            # kernels' bounds is at most this one)
            top = 2 * d.norm(dim=1).max() * z.norm(dim=1).max()
            for g2 in range(H // Hkv):
                dd = rows_d[:, (u * (H // Hkv) + g2) * D:(u * (H // Hkv) + g2 + 1) * D]
                top = torch.maximum(top, 2 * dd.norm(dim=1).max() * z.norm(dim=1).max())
            flush = see.to(F64) * (top * 2.0 ** -14 * 2.0 ** -24)
            eds = ds.abs() * (2.0 ** -11 + 2 * es + 8 * U) + p * edp + flush
            ep = p * (2.0 ** -11 + 2 * es) + see.to(F64) * 2.0 ** -38
            nk, nq = 2 * (b / 16 + 80) * U, 2 * (a / 16 + 80) * (H // Hkv) * U
            g[0][at, ch] += lone * (ds @ y)
            e[0][at, ch] += lone * (eds @ y.abs() + nk * (ds.abs() @ y.abs()))
            g[1][to, cu] += lone * (ds.t() @ x)
            e[1][to, cu] += lone * (eds.t() @ x.abs() + nq * (ds.abs().t() @ x.abs()))
            g[2][to, cu] += p.t() @ d
            e[2][to, cu] += ep.t() @ d.abs() + nq * (p.t() @ d.abs())
    return g, e
