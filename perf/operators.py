"""Operators of a transformer layer beside the scaled matmul, measured against
their plain forms: the RMS norm with the residual's addition and an output in
8 bits with its scales, its gradient, and attention over ScaledArrays forward
(prompts, packed batches, single tokens against a cache) and backward.

The sizes are those of the layer GEMMs in paper_2407_17353_amd/workloads.py
(d_model 2048 at 4096 tokens; d 4096 with 32 heads of 128 at 16384 tokens)
with ragged token counts where batches are packed, and of a cache that a
server keeps in 8 bits.

  listed()            the named cases
  draw(rng)           one more case of the same ranges
  prepare(case, seed) inputs, outputs on the GPU
  run(state)          one call (own: the library's; else the plain form)
  work(case)          bytes and operations that the call cannot do without
  exact(case, seed)   the outputs in 64 bits, from the definition
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "f16": torch.float16}
BYTES = {"e4m3": 1, "e5m2": 1, "f16": 2, "none": 0}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0, "f16": 65504.0}
FMT = {"e4m3": 0, "e5m2": 1, "f16": 2}            # scalify_dtype
MOST_PAIRS = 4 * 32 * 4096 * 4096                 # scores of the largest listed case
MOST_ELEMS = 16384 * 4096


def listed():
    return [
        # serving: eight sequences' tokens enter a layer of d 4096; one E4M3 row each with a scale of its own
        {"name": "rms_decode", "op": "rms_fwd", "R": 8, "D": 4096, "x": "f16", "res": "f16", "sum": "f16",
         "out": "e4m3", "scales": "row"},
        # a packed batch of 1777 tokens, E4M3 branch added to the F16 stream, a ragged width
        {"name": "rms_ragged", "op": "rms_fwd", "R": 1777, "D": 5000, "x": "e4m3", "res": "f16", "sum": "f16",
         "out": "e4m3", "scales": "row"},
        # training, forward: d 4096 at 16384 tokens, the operand of a block-scaled matmul
        {"name": "rms_train_mx", "op": "rms_fwd", "R": 16384, "D": 4096, "x": "f16", "res": "f16", "sum": "f16",
         "out": "e4m3", "scales": "mx"},
        # training, backward: d_model 2048 at 4096 tokens, E5M2 gradients, dynamic rescale
        {"name": "rms_bwd_2048", "op": "rms_bwd", "R": 4096, "D": 2048, "x": "f16", "dy": "e5m2", "dsum": "e5m2",
         "out": "e5m2", "rescale": "amax"},
        # training, backward: d 4096 at 16384 tokens, F16 gradient stream
        {"name": "rms_bwd_4096", "op": "rms_bwd", "R": 16384, "D": 4096, "x": "f16", "dy": "f16", "dsum": "f16",
         "out": "f16", "rescale": "none"},
        # serving, the smallest: one sequence's next token over a short F16 cache
        _attn(name="attn_token", B=1, Lq=1, Lk=513, H=16, Hkv=16, D=64, layout="cache"),
        # serving: 32 sequences' next tokens over E4M3 caches of up to 4096 keys, 8 heads shared by 32
        _attn(name="attn_decode_8bit", B=32, Lq=1, Lk=4096, H=32, Hkv=8, D=128, kv="e4m3", layout="cache"),
        # serving: the next token of one long document
        _attn(name="attn_decode_long", B=1, Lq=1, Lk=131072, H=32, Hkv=8, D=128, layout="cache"),
        # serving: five prompts packed into 3001 rows of an E4M3 QKV projection of d_model 2048
        _attn(name="attn_packed_8bit", B=5, T=3001, H=16, Hkv=16, D=128, q="e4m3", kv="e4m3", causal=True,
              layout="packed"),
        # training, forward: d 4096 at 16384 tokens
        _attn(name="attn_train", B=4, Lq=4096, Lk=4096, H=32, Hkv=32, D=128, causal=True, lse=True),
        # training, backward: packed documents, shared heads, E5M2 gradients in and out
        _attn(name="attn_bwd_packed", op="attn_bwd", B=3, T=1777, H=16, Hkv=4, D=128, causal=True, layout="packed",
              dout="e5m2", grad="e5m2", rescale="amax"),
        # training, backward: d 4096 at 16384 tokens, the largest
        _attn(name="attn_bwd_train", op="attn_bwd", B=4, Lq=4096, Lk=4096, H=32, Hkv=32, D=128, causal=True,
              dout="f16", grad="f16", rescale="none"),
    ]


def _attn(**kw):
    case = {"op": "attn_fwd", "T": 0, "Lq": 0, "Lk": 0, "q": "f16", "kv": "f16", "out": "f16", "causal": False,
            "layout": "dense", "lse": kw.get("op") == "attn_bwd", "dout": "none", "grad": "none", "rescale": "none"}
    case.update(kw)
    return case


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rms_fwd", "rms_bwd", "attn_fwd", "attn_fwd", "attn_token", "attn_bwd"])
    if op in ("rms_fwd", "rms_bwd"):
        D = _log_int(rng, 64, 8192)
        D = D // 64 * 64 if rng.random() < 0.6 else D
        R = min(_log_int(rng, 1, 16384), MOST_ELEMS // D)
        case = {"op": op, "R": R, "D": D, "x": rng.choice(["f16", "f16", "e4m3"])}
        if op == "rms_fwd":
            case["res"] = rng.choice(["f16", "f16", "e4m3", "none"])
            case["sum"] = "f16" if case["res"] != "none" else "none"
            case["scales"] = rng.choice(["mx", "row", "one"])
            case["out"] = rng.choice(["e4m3", "e4m3", "e5m2"] if case["scales"] == "mx" else ["e4m3", "f16"])
        else:
            case["x"] = "f16"
            case["dy"] = rng.choice(["e5m2", "f16"])
            case["dsum"] = rng.choice(["f16", "e5m2", "none"])
            case["out"] = rng.choice(["e5m2", "f16"])
            case["rescale"] = "amax" if case["out"] == "e5m2" else rng.choice(["amax", "none"])
        return case
    D = rng.choice([64, 128, 128, 48, 80, 96])
    Hkv = rng.choice([1, 2, 4, 8, 16, 32])
    H = Hkv * rng.choice([1, 1, 2, 4, 8])
    H, Hkv = (H, Hkv) if H <= 64 else (Hkv, Hkv)
    fmt = rng.choice(["f16", "f16", "e4m3"])
    if op == "attn_token":
        Lk = _log_int(rng, 1, 65536)
        B = max(1, min(_log_int(rng, 1, 64), (1 << 20) // Lk, 2 * MOST_ELEMS // (Lk * Hkv * D)))
        return _attn(B=B, Lq=rng.choice([1, 1, 1, 2, 5]), Lk=max(8, Lk), H=H, Hkv=Hkv, D=D, kv=fmt,
                     causal=rng.random() < 0.5, layout="cache")
    T = min(_log_int(rng, 16, 16384), MOST_ELEMS // (H * D))
    B = rng.choice([1, 2, 3, 5, 8])
    L = max(1, min(T // B, 4096, int(math.sqrt(MOST_PAIRS / (B * H)))))
    kw = {"B": B, "H": H, "Hkv": Hkv, "D": D, "q": fmt, "kv": fmt, "causal": rng.random() < 0.75}
    layout = rng.choice(["dense", "packed", "cross"])
    if layout == "packed":
        kw.update(T=max(B, B * L - rng.randrange(0, B)), layout="packed")
        # (a packed sequence is at most twice the mean length)
        if 4 * L * L * B * H > MOST_PAIRS:
            kw["T"] = max(B, kw["T"] // 2)
    elif layout == "cross":
        kw.update(Lq=max(1, L // rng.choice([1, 2, 4])), Lk=L, layout="dense")
    else:
        kw.update(Lq=L, Lk=L, layout="dense")
    if op == "attn_fwd":
        return _attn(lse=rng.random() < 0.5, out=rng.choice(["f16", "f16", "e4m3"]), **kw)
    grad = rng.choice(["f16", "f16", "e5m2"])
    return _attn(op="attn_bwd", dout=rng.choice(["f16", "e5m2"]), grad=grad,
                 rescale="amax" if grad == "e5m2" else "none", **kw)


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Lengths of a case's sequences, from the case alone: (queries, keys)."""
    B = case["B"]
    r = random.Random(1000003 * B + 7919 * case["T"] + case["Lk"])
    if case["layout"] == "packed":
        T = case["T"]
        w = [1.0 + r.random() for _ in range(B)]
        at = [0] + [int(round(T * sum(w[:i + 1]) / sum(w))) for i in range(B)]
        n = [at[i + 1] - at[i] for i in range(B)]
        return n, n
    if case["layout"] == "cache":
        return [case["Lq"]] * B, [case["Lk"] if B == 1 else r.randint((case["Lk"] + 1) // 2, case["Lk"]) for _ in range(B)]
    return [case["Lq"]] * B, [case["Lk"]] * B


def _pairs(case):
    """Admitted (query, key) pairs of one head."""
    n = 0
    for q, k in zip(*_lengths(case)):
        n += sum(max(0, min(k, i + k - q + 1)) for i in range(q)) if case["causal"] else q * k
    return n


def _normal(g, rows, cols, fmt, ld=None):
    """Values of N(0, 1) in a format, rows 16-byte aligned."""
    per = 16 // BYTES[fmt]
    ld = ld or -(-cols // per) * per
    t = torch.randn((rows, ld), generator=g, device=DEV, dtype=torch.float32).to(TORCH[fmt])
    return t[:, :cols]


def _empty(rows, cols, fmt):
    per = 16 // BYTES[fmt]
    return torch.empty((rows, -(-cols // per) * per), device=DEV, dtype=TORCH[fmt])[:, :cols]


def _scale(e):
    return torch.full((1,), 2.0 ** e, device=DEV, dtype=torch.float32)


def _one():
    return torch.empty(1, device=DEV, dtype=torch.float32)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(240717353 + seed)
    r = random.Random(seed)
    s = {"case": case}
    if case["op"] == "rms_fwd":
        R, D = case["R"], case["D"]
        s["x"], s["x_scale"] = _normal(g, R, D, case["x"]), _scale(r.randint(-2, 1))
        if case["res"] != "none":
            s["res"], s["res_scale"] = _normal(g, R, D, case["res"]), _scale(r.randint(0, 2))
            s["sum"], s["sum_scale"] = _empty(R, D, case["sum"]), _one()
        s["gamma"] = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEV)
        s["out"], s["out_scale"] = _empty(R, D, case["out"]), _one()
        if case["scales"] == "row":
            s["row_scale"] = torch.empty(R, device=DEV, dtype=torch.float32)
        if case["scales"] == "mx":
            n = 256 * -(-D // 128) * -(-R // 64)
            s["block_scale"] = torch.empty(n, device=DEV, dtype=torch.uint8)
        return s
    if case["op"] == "rms_bwd":
        R, D = case["R"], case["D"]
        # gradient rows of many magnitudes, as a loss over a packed batch gives
        rows = torch.exp2(-10 * torch.rand((R, 1), generator=g, device=DEV))
        for n in ("dy", "dsum"):
            if case[n] != "none":
                t = _normal(g, R, D, case[n])
                s[n], s[n + "_scale"] = t.copy_(t.float() * rows), _scale(r.randint(-9, -6))
        s["x"], s["x_scale"] = _normal(g, R, D, case["x"]), _scale(r.randint(0, 2))
        s["gamma"] = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEV)
        s["dx"], s["dx_scale"] = _empty(R, D, case["out"]), _one()
        s["dgamma"] = torch.empty(D, device=DEV, dtype=torch.float32)
        return s
    B, H, Hkv, D = case["B"], case["H"], case["Hkv"], case["D"]
    nq, nk = _lengths(case)
    Tq = sum(nq)
    Tk = B * case["Lk"] if case["layout"] == "cache" else sum(nk)
    e = r.randint(-2, 2)
    s["q"], s["q_scale"] = _normal(g, Tq, H * D, case["q"]), _scale(e)
    s["k"], s["k_scale"] = _normal(g, Tk, Hkv * D, case["kv"]), _scale(-e)
    s["v"], s["v_scale"] = _normal(g, Tk, Hkv * D, case["kv"]), _scale(r.randint(-3, 0))
    s["alpha"] = 1.0 / math.sqrt(D)
    s["q_start"] = s["k_start"] = s["k_len"] = None
    s["max_q"], s["max_k"] = max(nq), max(nk)
    if case["layout"] == "packed":
        at = torch.tensor([0] + nq, device=DEV, dtype=torch.int64).cumsum(0)
        s["q_start"] = s["k_start"] = at
    if case["layout"] == "cache":
        s["k_len"] = torch.tensor(nk, device=DEV, dtype=torch.int64)
    if case["op"] == "attn_fwd":
        s["out"], s["out_scale"] = _empty(Tq, H * D, case["out"]), _one()
        s["lse"] = torch.empty((H, Tq), device=DEV, dtype=torch.float32) if case["lse"] else None
        return s
    t = _normal(g, Tq, H * D, case["dout"])
    s["dout"], s["dout_scale"] = t, _scale(r.randint(-9, -6))
    # what the forward pass left
    o, s["lse"] = _attention(s, torch.float32)
    s["out"], s["out_scale"] = (o / s["v_scale"]).to(torch.float16), s["v_scale"].clone()
    for n, of in (("dq", "q"), ("dk", "k"), ("dv", "v")):
        s[n], s[n + "_scale"] = _empty(s[of].shape[0], s[of].shape[1], case["grad"]), _one()
    return s


# ------------------------------------------------------------------ plain forms (32 bits)

def _value(s, name, dtype=torch.float32):
    return s[name].to(dtype) * s[name + "_scale"].to(dtype)


def _cast(y, fmt):
    """Saturating cast of a data component."""
    return y.clamp(-LARGEST[fmt], LARGEST[fmt]).to(TORCH[fmt])


def _exponent(amax, target=0):
    """floor(log2 amax) - target, 0 where amax is 0."""
    e = torch.frexp(amax)[1].to(torch.int32) - 1 - target
    return torch.where(amax == 0, torch.zeros_like(e), e).clamp(-127, 127)


TARGET = {"e4m3": 7, "e5m2": 14, "f16": 0}  # rescaled amax in [2^t, 2^(t+1)), inside the format's range


def _rms_fwd(s):
    c = s["case"]
    out = {}
    h = s["x"].float()
    if c["res"] != "none":
        e = torch.maximum(s["x_scale"], s["res_scale"])
        h = _cast(h * (s["x_scale"] / e) + s["res"].float() * (s["res_scale"] / e), c["sum"])
        out["sum"], out["sum_scale"] = h, e
        h = h.float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["gamma"]
    t = TARGET[c["out"]]
    if c["scales"] == "row":
        e = _exponent(y.abs().amax(1), t)
        out["row_scale"] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
        y = torch.ldexp(y, -e[:, None])
    elif c["scales"] == "mx":
        R, D = y.shape
        K, P = -(-D // 128) * 128, -(-R // 64) * 64
        b = torch.nn.functional.pad(y, (0, K - D, 0, P - R)).view(P, K // 32, 32)
        e = _exponent(b.abs().amax(2), t)
        y = torch.ldexp(b, -e[:, :, None]).view(P, K)[:R, :D]
        out["block_scale"] = _packed((e + 127).to(torch.uint8)).view(torch.float8_e8m0fnu)
    out["out"], out["out_scale"] = _cast(y, c["out"]), torch.ones(1, device=DEV)
    return out


def _packed(b):
    """Block-scale bytes [rows, blocks] (whole groups of 64 rows and 4 blocks)
    in the order a block-scaled matmul reads: step of 4 blocks, group of 64
    rows, block of the step, row of 16, row block."""
    P, K = b.shape
    return b.view(P // 64, 4, 16, K // 4, 4).permute(3, 0, 4, 2, 1).reshape(-1)


def _rescaled(d, e, c, fmt):
    """A gradient d (data, true value d * 2^e) cast to fmt with its rescale."""
    if c["rescale"] == "amax":
        er = _exponent(d.abs().amax().reshape(1), 0)
        return _cast(torch.ldexp(d, -er), fmt), torch.ldexp(torch.ones(1, device=DEV), e + er)
    return _cast(d, fmt), torch.ldexp(torch.ones(1, device=DEV), e)


def _log2(t):
    return torch.frexp(t)[1].to(torch.int32) - 1


def _rms_bwd(s):
    c = s["case"]
    h, dy = s["x"].float(), s["dy"].float()
    inv = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    n = h * inv
    g = dy * s["gamma"]
    d = inv * (g - n * (g * n).mean(1, keepdim=True))
    e = _log2(s["dy_scale"]) - _log2(s["x_scale"])
    if c["dsum"] != "none":
        es = _log2(s["dsum_scale"])
        eo = torch.maximum(e, es)
        d = torch.ldexp(d, e - eo) + torch.ldexp(s["dsum"].float(), es - eo)
        e = eo
    dx, scale = _rescaled(d, e, c, c["out"])
    return {"dx": dx, "dx_scale": scale, "dgamma": (dy * n).sum(0)}


def _plan(s):
    """Rows of every sequence's queries and keys (padded to the longest), which
    of them are there, and which pairs are admitted."""
    c = s["case"]
    B, nq, nk = c["B"], s["max_q"], s["max_k"]
    i, j = torch.arange(nq, device=DEV), torch.arange(nk, device=DEV)
    if s["q_start"] is not None:
        q0, lq = s["q_start"][:-1], s["q_start"].diff()
        k0, lk = s["k_start"][:-1], s["k_start"].diff()
    else:
        Lq, Lk = s["q"].shape[0] // B, s["k"].shape[0] // B
        q0, k0 = torch.arange(B, device=DEV) * Lq, torch.arange(B, device=DEV) * Lk
        lq = torch.full_like(q0, Lq)
        lk = s["k_len"] if s["k_len"] is not None else torch.full_like(q0, Lk)
    hasq, hask = i < lq[:, None], j < lk[:, None]
    see = hask[:, None, :] & hasq[:, :, None]
    if c["causal"]:
        see = see & (j <= i[:, None] + (lk - lq)[:, None, None])
    qi = torch.where(hasq, q0[:, None] + i, 0)
    ki = torch.where(hask, k0[:, None] + j, 0)
    return qi, ki, hasq, see


def _heads(x, rows, n, D):
    """[B, n heads, rows, D] of the rows of x, contiguous."""
    return x[rows.reshape(-1)].view(rows.shape[0], rows.shape[1], n, D).transpose(1, 2).contiguous()


def _scores(s, dtype, qi, ki, see):
    """Scores with the heads that share a key head beside each other:
    [B, kv heads, heads of one, queries, keys], what is not admitted -inf."""
    c = s["case"]
    B, H, Hkv, D = c["B"], c["H"], c["Hkv"], c["D"]
    q = _heads(_value(s, "q", dtype), qi, H, D).view(B, Hkv, H // Hkv * qi.shape[1], D)
    k = _heads(_value(s, "k", dtype), ki, Hkv, D)
    z = torch.matmul(q, k.transpose(2, 3)).mul_(s["alpha"]).view(B, Hkv, H // Hkv, qi.shape[1], ki.shape[1])
    return q, k, z.masked_fill_(~see[:, None, None], -math.inf)


def _to_rows(o, rows, has, like):
    """[B, heads, rows, D] back to the rows of a packed matrix."""
    B, H, L, D = o.shape
    out = torch.zeros(like.shape, device=DEV, dtype=o.dtype)
    out[rows[has]] = o.transpose(1, 2).reshape(B, L, H * D)[has]
    return out


def _attention(s, dtype):
    c = s["case"]
    B, H, Hkv, D = c["B"], c["H"], c["Hkv"], c["D"]
    qi, ki, hasq, see = _plan(s)
    z = _scores(s, dtype, qi, ki, see)[2]
    m = z.amax(4, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    z = z.sub_(m).exp_()
    n = z.sum(4, keepdim=True)
    v = _heads(_value(s, "v", dtype), ki, Hkv, D)
    o = torch.matmul(z.view(B, Hkv, -1, ki.shape[1]), v).view(B, Hkv, H // Hkv, -1, D)
    o = torch.where(n > 0, o / torch.where(n > 0, n, torch.ones_like(n)), torch.zeros_like(o))
    lse = (m + n.log()).reshape(B, H, -1)
    rows = torch.zeros((H, s["q"].shape[0]), device=DEV, dtype=dtype)
    rows[:, qi[hasq]] = lse.transpose(1, 2)[hasq].t()
    return _to_rows(o.reshape(B, H, -1, D), qi, hasq, s["q"]), rows


def _attn_fwd(s):
    c = s["case"]
    o, lse = _attention(s, torch.float32)
    out = {"out": _cast(o / s["v_scale"], c["out"]), "out_scale": s["v_scale"]}
    if c["lse"]:
        out["lse"] = lse
    return out


def _gradients(s, dtype):
    """dq, dk, dv (true values) of the stored output and log-sum-exp."""
    c = s["case"]
    B, H, Hkv, D = c["B"], c["H"], c["Hkv"], c["D"]
    qi, ki, hasq, see = _plan(s)
    q, k, p = _scores(s, dtype, qi, ki, see)
    nq, nk = qi.shape[1], ki.shape[1]
    lse = s["lse"].to(dtype)[:, qi.reshape(-1)].view(H, B, nq).transpose(0, 1).reshape(B, Hkv, H // Hkv, nq, 1)
    p = p.sub_(torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_().view(B, Hkv, -1, nk)
    do = _heads(_value(s, "dout", dtype), qi, H, D).mul_(hasq[:, None, :, None]).view(B, Hkv, -1, D)
    o = _heads(_value(s, "out", dtype), qi, H, D).view(B, Hkv, -1, D)
    v = _heads(_value(s, "v", dtype), ki, Hkv, D)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * o).sum(3, keepdim=True)).mul_(p)
    dq = torch.matmul(ds, k) * s["alpha"]
    dk = torch.matmul(ds.transpose(2, 3), q) * s["alpha"]
    hask = see.any(1) if not c["causal"] else torch.arange(nk, device=DEV) < _key_counts(s)[:, None]
    return (_to_rows(dq.reshape(B, H, nq, D), qi, hasq, s["q"]), _to_rows(dk, ki, hask, s["k"]),
            _to_rows(dv, ki, hask, s["v"]))


def _key_counts(s):
    c = s["case"]
    if s["k_start"] is not None:
        return s["k_start"].diff()
    if s["k_len"] is not None:
        return s["k_len"]
    return torch.full((c["B"],), s["k"].shape[0] // c["B"], device=DEV)


def _attn_bwd(s):
    c = s["case"]
    eq, ek, ev, eo = (_log2(s[n + "_scale"]) for n in ("q", "k", "v", "dout"))
    out = {}
    grads = _gradients(s, torch.float32)
    out["dq"], out["dq_scale"] = _rescaled(torch.ldexp(grads[0], -(eo + ev + ek)), eo + ev + ek, c, c["grad"])
    out["dk"], out["dk_scale"] = _rescaled(torch.ldexp(grads[1], -(eo + ev + eq)), eo + ev + eq, c, c["grad"])
    out["dv"], out["dv_scale"] = _rescaled(torch.ldexp(grads[2], -eo), eo, c, c["grad"])
    return out


PLAIN = {"rms_fwd": _rms_fwd, "rms_bwd": _rms_bwd, "attn_fwd": _attn_fwd, "attn_bwd": _attn_bwd}


# ------------------------------------------------------------------ the library's calls

def _scaled(sc, s, name, fmt):
    t = s[name]
    return sc.ScaledArray(t.view(torch.int16 if fmt == "f16" else torch.uint8), FMT[fmt], s[name + "_scale"])


def _own(s):
    from paper_2407_17353_amd import binding as sc
    c = s["case"]
    if c["op"] == "rms_fwd":
        res = c["res"] != "none"
        sc.scalify_rmsnorm_fwd(_scaled(sc, s, "x", c["x"]), _scaled(sc, s, "out", c["out"]),
                               residual=_scaled(sc, s, "res", c["res"]) if res else None,
                               sum_out=_scaled(sc, s, "sum", c["sum"]) if res else None, gamma=s["gamma"], eps=EPS,
                               row_scale=s.get("row_scale"), block_scale=s.get("block_scale"),
                               target_log2=TARGET[c["out"]])
        out = {"out": s["out"], "out_scale": s["out_scale"]}
        if res:
            out["sum"], out["sum_scale"] = s["sum"], s["sum_scale"]
        if c["scales"] == "row":
            out["row_scale"] = s["row_scale"]
        if c["scales"] == "mx":
            out["block_scale"] = s["block_scale"].view(torch.float8_e8m0fnu)
        return out
    mode = sc.RESCALE_AMAX if c.get("rescale") == "amax" else sc.RESCALE_NONE
    if c["op"] == "rms_bwd":
        sc.scalify_rmsnorm_bwd(_scaled(sc, s, "dy", c["dy"]), _scaled(sc, s, "x", c["x"]), _scaled(sc, s, "dx", c["out"]),
                               dsum=_scaled(sc, s, "dsum", c["dsum"]) if c["dsum"] != "none" else None,
                               gamma=s["gamma"], eps=EPS, rescale=mode, dgamma=s["dgamma"])
        return {"dx": s["dx"], "dx_scale": s["dx_scale"], "dgamma": s["dgamma"]}
    kw = {"heads": c["H"], "kv_heads": c["Hkv"], "batch": c["B"], "causal": c["causal"], "softmax_scale": s["alpha"],
          "q_start": s["q_start"], "k_start": s["k_start"], "k_len": s["k_len"], "max_q": s["max_q"], "max_k": s["max_k"]}
    q, k, v = _scaled(sc, s, "q", c["q"]), _scaled(sc, s, "k", c["kv"]), _scaled(sc, s, "v", c["kv"])
    if c["op"] == "attn_fwd":
        sc.scalify_attention_fwd(q, k, v, _scaled(sc, s, "out", c["out"]), lse=s["lse"], **kw)
        out = {"out": s["out"], "out_scale": s["out_scale"]}
        if c["lse"]:
            out["lse"] = s["lse"]
        return out
    sc.scalify_attention_bwd(_scaled(sc, s, "dout", c["dout"]), q, k, v, _scaled(sc, s, "out", "f16"), s["lse"],
                             _scaled(sc, s, "dq", c["grad"]), _scaled(sc, s, "dk", c["grad"]),
                             _scaled(sc, s, "dv", c["grad"]), rescale=mode, **kw)
    return {n: s[n] for n in ("dq", "dq_scale", "dk", "dk_scale", "dv", "dv_scale")}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ cost, and the values in 64 bits

def work(case):
    if case["op"] == "rms_fwd":
        n = case["R"] * case["D"]
        per = BYTES[case["x"]] + BYTES[case["res"]] + BYTES[case["sum"]] + BYTES[case["out"]]
        extra = {"row": 4 * case["R"], "mx": n // 32, "one": 4}[case["scales"]]
        return {"bytes": n * per + extra + 4 * case["D"], "flops": 5 * n}
    if case["op"] == "rms_bwd":
        n = case["R"] * case["D"]
        return {"bytes": n * sum(BYTES[case[k]] for k in ("x", "dy", "dsum", "out")) + 8 * case["D"], "flops": 12 * n}
    nq, nk = _lengths(case)
    q, kv = sum(nq) * case["H"] * case["D"], sum(nk) * case["Hkv"] * case["D"]
    pairs = _pairs(case) * case["H"]
    rows = 4 * sum(nq) * case["H"] if case["lse"] else 0
    if case["op"] == "attn_fwd":
        return {"bytes": q * (BYTES[case["q"]] + BYTES[case["out"]]) + 2 * kv * BYTES[case["kv"]] + rows,
                "flops": 4 * case["D"] * pairs}
    return {"bytes": q * (BYTES[case["q"]] + 2 + BYTES[case["dout"]] + BYTES[case["grad"]]) + rows
            + 2 * kv * (BYTES[case["kv"]] + BYTES[case["grad"]]), "flops": 10 * case["D"] * pairs}


def _held(y, fmt):
    """What an 8-bit format holds of a value (the rounding is part of what the
    operator is defined to give); 16-bit outputs are left unrounded."""
    if fmt == "f16":
        return y
    return y.clamp(-LARGEST[fmt], LARGEST[fmt]).to(TORCH[fmt]).to(torch.float64)


def _exact_rms_fwd(s):
    """Row by row definition: the stored sum, its root mean square, the powers
    of two from the logarithm of the largest magnitudes."""
    c, f = s["case"], torch.float64
    got = {}
    if c["res"] == "none":
        h = s["x"].to(f)
    else:
        top = max(s["x_scale"].item(), s["res_scale"].item())
        h = (s["x"].to(f) * s["x_scale"].item() + s["res"].to(f) * s["res_scale"].item()) / top
        got["sum"], got["sum_scale"] = h, torch.tensor([top], dtype=f, device=DEV)
        h = h.to(torch.float32).to(TORCH[c["sum"]]).to(f)  # what the norm sees is the stored sum
    y = h / torch.sqrt((h * h).sum(1, keepdim=True) / c["D"] + EPS) * s["gamma"].to(f)
    t = TARGET[c["out"]]

    def power(a):
        return torch.where(a == 0, torch.ones_like(a), torch.exp2(torch.floor(torch.log2(torch.where(a == 0, torch.ones_like(a), a))) - t))
    if c["scales"] == "row":
        got["row_scale"] = power(y.abs().amax(1))
        y = y / got["row_scale"][:, None]
    if c["scales"] == "mx":
        R, D = y.shape
        full = torch.zeros((-(-R // 64) * 64, -(-D // 128) * 128), dtype=f, device=DEV)
        full[:R, :D] = y
        p = power(full.unflatten(1, (-1, 32)).abs().amax(2))
        y = (full / p.repeat_interleave(32, 1))[:R, :D]
        # 128-column step t, 64-row group u, block g, row r of 16, row block m
        p = p.unflatten(0, (-1, 4, 16)).unflatten(3, (-1, 4))          # u, m, r, t, g
        got["block_scale"] = torch.einsum("umrtg->tugrm", p).reshape(-1)
    got["out"], got["out_scale"] = _held(y, c["out"]), torch.ones(1, dtype=f, device=DEV)
    return got


def _exact_rescaled(true, base, mode, fmt):
    a = true.abs().max().item()
    p = 2.0 ** math.floor(math.log2(a)) if a and mode == "amax" else base
    return _held(true / p, fmt), torch.tensor([p], dtype=torch.float64, device=DEV)


def _exact_rms_bwd(s):
    c, f = s["case"], torch.float64
    sx, sdy = s["x_scale"].item(), s["dy_scale"].item()
    h, dy = s["x"].to(f), s["dy"].to(f)
    rms = torch.sqrt((h * h).sum(1, keepdim=True) / c["D"] + EPS)
    g = dy * s["gamma"].to(f)
    true = (g / rms - h * (g * h).sum(1, keepdim=True) / (c["D"] * rms ** 3)) * (sdy / sx)
    base = sdy / sx
    if c["dsum"] != "none":
        true = true + s["dsum"].to(f) * s["dsum_scale"].item()
        base = max(base, s["dsum_scale"].item())
    dx, p = _exact_rescaled(true, base, c["rescale"], c["out"])
    return {"dx": dx, "dx_scale": p, "dgamma": (dy * h / rms).sum(0)}


def _exact_spans(s):
    c = s["case"]
    nq, nk = _lengths(c)
    q0 = k0 = 0
    for a, b in zip(nq, nk):
        yield q0, a, k0, b
        q0, k0 = q0 + a, k0 + (c["Lk"] if c["layout"] == "cache" else b)


def _exact_head(s, h, q0, a, k0, b):
    """One sequence's head: queries, keys, values and probabilities."""
    c, f = s["case"], torch.float64
    D, u = c["D"], h // (c["H"] // c["Hkv"])
    q = s["q"][q0:q0 + a, h * D:(h + 1) * D].to(f) * s["q_scale"].item()
    k = s["k"][k0:k0 + b, u * D:(u + 1) * D].to(f) * s["k_scale"].item()
    v = s["v"][k0:k0 + b, u * D:(u + 1) * D].to(f) * s["v_scale"].item()
    z = (q @ k.t()) / math.sqrt(D)
    if c["causal"]:
        hidden = torch.ones((a, b), device=DEV, dtype=torch.bool).triu(b - a + 1)
        z[hidden] = -math.inf
    return q, k, v, z


def _exact_attn(s):
    c, f = s["case"], torch.float64
    D, Tq = c["D"], s["q"].shape[0]
    o = torch.zeros((Tq, c["H"] * D), dtype=f, device=DEV)
    lse = torch.zeros((c["H"], Tq), dtype=f, device=DEV)
    gq = torch.zeros_like(o)
    gk, gv = (torch.zeros(s["k"].shape, dtype=f, device=DEV) for _ in range(2))
    back = c["op"] == "attn_bwd"
    for q0, a, k0, b in _exact_spans(s):
        for h in range(c["H"]):
            q, k, v, z = _exact_head(s, h, q0, a, k0, b)
            at, cols = slice(q0, q0 + a), slice(h * D, (h + 1) * D)
            if not back:
                lse[h, at] = torch.logsumexp(z, 1)
                o[at, cols] = torch.nan_to_num(torch.softmax(z, 1)) @ v
                continue
            u = h // (c["H"] // c["Hkv"])
            to, kv = slice(k0, k0 + b), slice(u * D, (u + 1) * D)
            p = torch.nan_to_num(torch.exp(z - s["lse"][h, at].to(f)[:, None]))
            d = s["dout"][at, cols].to(f) * s["dout_scale"].item()
            y = s["out"][at, cols].to(f) * s["out_scale"].item()
            w = p * (d @ v.t() - (d * y).sum(1, keepdim=True)) / math.sqrt(D)
            gv[to, kv] += p.t() @ d
            gq[at, cols] = w @ k
            gk[to, kv] += w.t() @ q
    return o, lse, gq, gk, gv


def exact(case, seed):
    if case["op"].startswith("attn") and case["B"] * case["H"] > 2048:
        return None  # (too many products of one head for the time)
    s = prepare(case, seed)
    if case["op"] == "rms_fwd":
        return _exact_rms_fwd(s)
    if case["op"] == "rms_bwd":
        return _exact_rms_bwd(s)
    o, lse, gq, gk, gv = _exact_attn(s)
    sv = s["v_scale"].item()
    if case["op"] == "attn_fwd":
        got = {"out": _held(o / sv, case["out"]), "out_scale": torch.tensor([sv], dtype=torch.float64, device=DEV)}
        return {**got, "lse": lse} if case["lse"] else got
    base = s["dout_scale"].item()
    got = {}
    for n, g, b in (("dq", gq, base * sv * s["k_scale"].item()), ("dk", gk, base * sv * s["q_scale"].item()), ("dv", gv, base)):
        got[n], got[n + "_scale"] = _exact_rescaled(g, b, case["rescale"], case["grad"])
    return got
