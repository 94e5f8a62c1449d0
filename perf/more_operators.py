"""The losses behind a transformer's last layer, measured against their plain
forms: softmax cross entropy over a vocabulary and distillation from a
teacher's top logits, both from the hidden states and the output matrix (the
logits are not kept), forward and backward.

The sizes are those of the layer GEMMs in paper_2407_17353_amd/workloads.py
(d_model 2048 at 4096 tokens; d 4096 at 16384 tokens), ragged ones, and the
few rows of a scored answer, with vocabularies of 30 to 130 thousand tokens.

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
IGNORED = -100                                    # the label of a row that is not counted
TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "f16": torch.float16}
BYTES = {"e4m3": 1, "e5m2": 1, "f16": 2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0, "f16": 65504.0}
FMT = {"e4m3": 0, "e5m2": 1, "f16": 2}            # scalify_dtype
MOST_PRODUCTS = 16384 * 32000 * 4096              # of the largest listed case
MOST_LOGITS = 16384 * 32000
MOST_WEIGHTS = 131072 * 4096


def listed():
    return [
        # serving, the smallest: the log-probability of one sampled token, 8-bit output matrix
        _case("ce_token", "ce_fwd", R=1, D=2048, V=32000, w="e4m3"),
        # serving: an answer of 48 tokens scored, both operands in 8 bits
        _case("ce_score", "ce_fwd", R=48, D=4096, V=32000, x="e4m3", w="e4m3", rows=True),
        # a packed batch of 1777 tokens, of which the prompts' (a third) are not counted; ragged width and vocabulary
        _case("ce_ragged", "ce_fwd", R=1777, D=5000, V=50021, x="e4m3", rows=True, ignored=0.33),
        # training, forward: d 4096 at 16384 tokens, the norm's E4M3 rows with their scales
        _case("ce_train", "ce_fwd", R=16384, D=4096, V=32000, x="e4m3", w="e4m3", rows=True),
        # fine-tuning, backward: 300 tokens of a short batch, half of them prompts
        _case("ce_bwd_few", "ce_bwd", R=300, D=2048, V=32000, ignored=0.5),
        # training, backward: d_model 2048 at 4096 tokens, 8-bit operands and gradients, dynamic rescale
        _case("ce_bwd_2048", "ce_bwd", R=4096, D=2048, V=32000, x="e4m3", w="e4m3", rows=True, grad="e5m2",
              rescale="amax"),
        # training, backward: a large vocabulary, a tenth of the rows padding
        _case("ce_bwd_vocab", "ce_bwd", R=2048, D=4096, V=131072, ignored=0.1),
        # training, backward: d 4096 at 16384 tokens, the largest
        _case("ce_bwd_train", "ce_bwd", R=16384, D=4096, V=32000, x="e4m3", w="e4m3", rows=True, rescale="amax"),
        # speculative serving: a draft model's 16 tokens against the target's top 8
        _case("kd_few", "kd_fwd", R=16, D=2048, V=32000, k=8, temp=1.0),
        # training a student, forward: d_model 2048 at 4096 tokens, 64 stored logits a token
        _case("kd_train", "kd_fwd", R=4096, D=2048, V=32000, w="e4m3", k=64, temp=2.0),
        # training a student, backward: ragged everything, a fifth of the rows without a teacher
        _case("kd_bwd_ragged", "kd_bwd", R=777, D=1000, V=50021, k=20, temp=1.5, ignored=0.2),
        # training a student, backward: 8192 tokens of d 4096, 128 stored logits a token
        _case("kd_bwd_train", "kd_bwd", R=8192, D=4096, V=32000, x="e4m3", w="e4m3", rows=True, k=128, temp=2.0,
              grad="e5m2", rescale="amax"),
    ]


def _case(name, op, **kw):
    case = {"op": op, "x": "f16", "w": "f16", "rows": False, "ignored": 0.0, "k": 0, "temp": 1.0, "grad": "f16",
            "rescale": "none"}
    case.update(kw)
    return {"name": name, **case} if name else case


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["ce_fwd", "ce_bwd", "kd_fwd", "kd_bwd"])
    D = _log_int(rng, 64, 8192)
    D = D // 64 * 64 if rng.random() < 0.7 else D
    V = min(_log_int(rng, 500, 131072), MOST_WEIGHTS // D)
    V = V // 128 * 128 if V >= 128 and rng.random() < 0.5 else V
    R = min(_log_int(rng, 1, 16384), MOST_LOGITS // V, MOST_PRODUCTS // (V * D))
    x = rng.choice(["f16", "e4m3", "e5m2"])
    kw = {"R": max(1, R), "D": D, "V": V, "x": x, "w": rng.choice(["f16", "e4m3", "e4m3", "e5m2"]),
          "rows": x != "f16" and rng.random() < 0.6, "ignored": rng.choice([0.0, 0.0, 0.1, 0.4, 0.8])}
    if op.startswith("kd"):
        kw.update(k=_log_int(rng, 1, 128), temp=rng.choice([1.0, 2.0, 1.5, 4.0]))
    if op.endswith("bwd"):
        kw["grad"] = rng.choice(["f16", "f16", "e5m2"])
        kw["rescale"] = "amax" if kw["grad"] == "e5m2" else rng.choice(["amax", "none"])
    return _case(None, op, **kw)


# ------------------------------------------------------------------ inputs

def _normal(g, rows, cols, fmt):
    """Values of N(0, 1) in a format, rows 16-byte aligned."""
    t = torch.empty((rows, _pitch(cols, fmt)), device=DEV, dtype=TORCH[fmt])
    for at in range(0, rows, 8192):
        part = t[at:at + 8192]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV, dtype=torch.float32))
    return t[:, :cols]


def _pitch(cols, fmt):
    per = 16 // BYTES[fmt]
    return -(-cols // per) * per


def _empty(rows, cols, fmt):
    return torch.empty((rows, _pitch(cols, fmt)), device=DEV, dtype=TORCH[fmt])[:, :cols]


def _scale(e):
    return torch.full((1,), 2.0 ** e, device=DEV, dtype=torch.float32)


def _one():
    return torch.empty(1, device=DEV, dtype=torch.float32)


def _uncounted(case):
    """Rows that are not counted: how many."""
    return min(int(round(case["ignored"] * case["R"])), case["R"] - 1)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(240717353 + seed)
    r = random.Random(seed)
    R, D, V, k = case["R"], case["D"], case["V"], case["k"]
    s = {"case": case, "w": _normal(g, V, D, case["w"])}
    # logits of about N(0, 1) but for the tokens that the hidden state points to
    s["w_scale"] = _scale(-round(math.log2(D) / 2) + r.randint(-1, 1))
    s["x_scale"] = _scale(0)
    token = torch.randint(0, V, (R,), generator=g, device=DEV)
    x = torch.randn((R, D), generator=g, device=DEV, dtype=torch.float32)
    for at in range(0, R, 4096):
        part = token[at:at + 4096]
        # (from rows that know their token to rows that do not)
        a = 12.0 * torch.rand((len(part), 1), generator=g, device=DEV) / math.sqrt(D)
        x[at:at + 4096] += a * s["w"][part].float()
    s["x"] = _empty(R, D, case["x"])
    if case["rows"]:
        # rows of magnitudes within a few powers of two, each with its scale
        e = torch.randint(-2, 2, (R, 1), generator=g, device=DEV).float()
        s["row_scale"] = torch.exp2(e)[:, 0].contiguous()
        x = x * torch.exp2(3 - e)
        s["x_scale"] = _scale(-3)
    s["x"].copy_(x)
    del x
    left_out = torch.randperm(R, generator=g, device=DEV)[:_uncounted(case)]
    if k:
        # the teacher's tokens: the one the state points to and k - 1 others, all different
        step = torch.randint(1, max(2, V // max(k, 1)), (R, 1), generator=g, device=DEV)
        s["index"] = ((token[:, None] + step * torch.arange(k, device=DEV)) % V).contiguous()
        s["index"][left_out] = IGNORED
        t = torch.randn((R, k), generator=g, device=DEV).abs().cumsum(1) * (8.0 / max(k, 8))
        s["teacher"] = _empty(R, k, "f16")
        s["teacher"].copy_(10.0 - t)
        s["teacher_scale"] = _scale(r.randint(0, 1))
    else:
        s["labels"] = token
        s["labels"][left_out] = IGNORED
    s["lse"] = torch.empty(R, device=DEV, dtype=torch.float32)
    s["picked"] = torch.empty((R, k), device=DEV, dtype=torch.float32) if k else None
    if case["op"].endswith("fwd"):
        s["loss"] = torch.empty(R, device=DEV, dtype=torch.float32)
        return s
    # the mean over the rows that count, some of them weighted
    s["dloss"] = 0.5 + torch.rand(R, generator=g, device=DEV)
    s["dloss_scale"] = _scale(-round(math.log2(R)))
    s["dx"], s["dx_scale"] = _empty(R, D, case["grad"]), _one()
    s["dw"], s["dw_scale"] = _empty(V, D, case["grad"]), _one()
    got = PLAIN["kd_fwd" if k else "ce_fwd"](s)      # what the forward pass left
    s["lse"].copy_(got["lse"])
    if k:
        s["picked"].copy_(got["picked"])
    return s


# ------------------------------------------------------------------ plain forms (32 bits)

def _logits(s):
    c = s["case"]
    x = s["x"].float() * s["x_scale"]
    if c["rows"]:
        x = x * s["row_scale"][:, None]
    return torch.matmul(x, (s["w"].float() * s["w_scale"]).t())


def _log_sum_exp(z):
    m = z.amax(1, keepdim=True)
    return (m + (z - m).exp().sum(1, keepdim=True).log())[:, 0]


def _ce_fwd(s):
    V = s["case"]["V"]
    counts = (s["labels"] >= 0) & (s["labels"] < V)
    z = _logits(s)
    lse = _log_sum_exp(z)
    at = torch.where(counts, s["labels"], 0)
    loss = lse - z.gather(1, at[:, None])[:, 0]
    zero = torch.zeros_like(lse)
    return {"loss": torch.where(counts, loss, zero), "lse": torch.where(counts, lse, zero)}


def _targets(s):
    """The teacher's tokens, which of them are there, their probabilities (of
    the ones that are there) and the logarithms of these."""
    there = (s["index"] >= 0) & (s["index"] < s["case"]["V"])
    t = (s["teacher"].float() * s["teacher_scale"] / s["case"]["temp"]).masked_fill(~there, -math.inf)
    m = t.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = (t - m).exp()
    n = e.sum(1, keepdim=True)
    counts = n[:, 0] > 0
    n = torch.where(n > 0, n, torch.ones_like(n))
    return torch.where(there, s["index"], 0), there, e / n, t - m - n.log(), counts


def _kd_fwd(s):
    temp = s["case"]["temp"]
    z = _logits(s) / temp
    lse = _log_sum_exp(z)
    at, there, q, logq, counts = _targets(s)
    picked = z.gather(1, at)
    terms = q * (logq - (picked - lse[:, None]))
    loss = temp * temp * torch.where(q > 0, terms, torch.zeros_like(terms)).sum(1)
    zero = torch.zeros_like(lse)
    return {"loss": torch.where(counts, loss, zero), "lse": torch.where(counts, lse, zero),
            "picked": torch.where(there & counts[:, None], picked, torch.zeros_like(picked))}


def _exponent(amax):
    """floor(log2 amax), 0 where amax is 0."""
    e = torch.frexp(amax)[1].to(torch.int32) - 1
    return torch.where(amax == 0, torch.zeros_like(e), e)


def _rescaled(s, true, base, name):
    """A gradient (true values) as data and scale."""
    c = s["case"]
    scale = base
    if c["rescale"] == "amax":
        scale = torch.ldexp(base, _exponent((true / base).abs().amax().reshape(1)))
    y = true / scale
    return {name: y.clamp(-LARGEST[c["grad"]], LARGEST[c["grad"]]).to(TORCH[c["grad"]]), name + "_scale": scale}


def _gradients(s, dz):
    """dx and dw of the logits' gradient dz (which is consumed)."""
    c = s["case"]
    g = s["dloss_scale"]
    w = s["w"].float() * s["w_scale"]
    out = _rescaled(s, torch.matmul(dz, w), g * s["w_scale"], "dx")
    del w
    x = s["x"].float() * s["x_scale"]
    if c["rows"]:
        x = x * s["row_scale"][:, None]
    out.update(_rescaled(s, torch.matmul(dz.t(), x), g * s["x_scale"], "dw"))
    return out


def _ce_bwd(s):
    V = s["case"]["V"]
    counts = (s["labels"] >= 0) & (s["labels"] < V)
    dz = _logits(s).sub_(s["lse"][:, None]).exp_()
    at = torch.where(counts, s["labels"], 0)
    dz.scatter_add_(1, at[:, None], -torch.ones_like(dz[:, :1]))
    dz.mul_(torch.where(counts, s["dloss"] * s["dloss_scale"], torch.zeros_like(s["dloss"]))[:, None])
    return _gradients(s, dz)


def _kd_bwd(s):
    temp = s["case"]["temp"]
    at, _, q, _, counts = _targets(s)
    dz = _logits(s).div_(temp).sub_(s["lse"][:, None]).exp_()
    dz.scatter_add_(1, at, -q)
    dz.mul_(torch.where(counts, s["dloss"] * s["dloss_scale"] * temp, torch.zeros_like(s["dloss"]))[:, None])
    return _gradients(s, dz)


PLAIN = {"ce_fwd": _ce_fwd, "ce_bwd": _ce_bwd, "kd_fwd": _kd_fwd, "kd_bwd": _kd_bwd}


# ------------------------------------------------------------------ the library's calls

def _scaled(sc, s, name, fmt):
    return sc.ScaledArray(s[name].view(torch.int16 if fmt == "f16" else torch.uint8), FMT[fmt], s[name + "_scale"])


def _own(s):
    from paper_2407_17353_amd import binding as sc
    c = s["case"]
    x, w = _scaled(sc, s, "x", c["x"]), _scaled(sc, s, "w", c["w"])
    kw = {"row_scale": s.get("row_scale")}
    if c["k"]:
        kw["temperature"] = c["temp"]
        teacher = _scaled(sc, s, "teacher", "f16")
    if c["op"] == "ce_fwd":
        sc.scalify_cross_entropy_fwd(x, w, s["labels"], s["loss"], lse=s["lse"], **kw)
        return {"loss": s["loss"], "lse": s["lse"]}
    if c["op"] == "kd_fwd":
        sc.scalify_distillation_fwd(x, w, teacher, s["index"], s["loss"], lse=s["lse"], picked=s["picked"], **kw)
        return {"loss": s["loss"], "lse": s["lse"], "picked": s["picked"]}
    kw.update(dloss=s["dloss"], dloss_scale=s["dloss_scale"], dx=_scaled(sc, s, "dx", c["grad"]),
              dw=_scaled(sc, s, "dw", c["grad"]),
              rescale=sc.RESCALE_AMAX if c["rescale"] == "amax" else sc.RESCALE_NONE)
    if c["op"] == "ce_bwd":
        sc.scalify_cross_entropy_bwd(x, w, s["labels"], s["lse"], **kw)
    else:
        sc.scalify_distillation_bwd(x, w, teacher, s["index"], s["lse"], s["picked"], **kw)
    return {n: s[n] for n in ("dx", "dx_scale", "dw", "dw_scale")}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ cost, and the values in 64 bits

def work(case):
    """Rows that are not counted need nothing: only the others are read and multiplied."""
    V, D, k = case["V"], case["D"], case["k"]
    R, n = case["R"], case["R"] - _uncounted(case)
    size = n * D * BYTES[case["x"]] + V * D * BYTES[case["w"]] + (4 * n if case["rows"] else 0)
    size += R * 10 * k if k else R * 8
    if case["op"].endswith("fwd"):
        return {"bytes": size + 8 * R + 4 * R * k, "flops": 2 * n * V * D}
    size += 8 * n + 4 * n * k
    return {"bytes": size + (R + V) * D * BYTES[case["grad"]], "flops": 6 * n * V * D}


def _held(y, fmt):
    """What an 8-bit format holds of a value (the rounding is part of what the
    operator is defined to give); 16-bit outputs are left unrounded."""
    if fmt == "f16":
        return y
    return y.clamp(-LARGEST[fmt], LARGEST[fmt]).to(TORCH[fmt]).to(torch.float64)


def _exact_gradient(true, base, case):
    a = true.abs().max().item()
    p = 2.0 ** math.floor(math.log2(a)) if a and case["rescale"] == "amax" else base
    return _held(true / p, case["grad"]), torch.tensor([p], dtype=torch.float64, device=DEV)


def exact(case, seed):
    """Some rows at a time: their probabilities, their loss and their part of
    the gradients, each from its formula."""
    if case["R"] * case["V"] * case["D"] > MOST_PRODUCTS:
        return None  # (too many products of 64 bits for the time)
    s, f = prepare(case, seed), torch.float64
    c, R, V, D, k, T = case, case["R"], case["V"], case["D"], case["k"], case["temp"]
    W = s["w"].to(f)
    sw, sx = s["w_scale"].item(), s["x_scale"].item()
    back = c["op"].endswith("bwd")
    loss, lse = torch.zeros(R, dtype=f, device=DEV), torch.zeros(R, dtype=f, device=DEV)
    picked = torch.zeros((R, k), dtype=f, device=DEV)
    dx = torch.zeros((R, D), dtype=f, device=DEV) if back else None
    dw = torch.zeros((V, D), dtype=f, device=DEV) if back else None
    for at in range(0, R, 2048):
        rows = slice(at, min(R, at + 2048))
        X = s["x"][rows].to(f) * sx
        if c["rows"]:
            X = X * s["row_scale"][rows].to(f)[:, None]
        n = X.shape[0]
        Z = (X @ W.t()) * (sw / T)
        want = torch.zeros((n, V), dtype=f, device=DEV)   # the probabilities that the rows are to have
        if k:
            idx = s["index"][rows]
            has = (idx >= 0) & (idx < V)
            t = s["teacher"][rows].to(f) * s["teacher_scale"].item() / T
            q = torch.nan_to_num(torch.softmax(t.masked_fill(~has, -math.inf), 1))
            want.scatter_add_(1, idx.clamp(0, V - 1), q)
            on = q.sum(1) > 0
        else:
            y = s["labels"][rows]
            on = (y >= 0) & (y < V)
            want[on, y[on]] = 1.0
        L = torch.logsumexp(Z, 1)
        if not back:
            lse[rows] = torch.where(on, L, 0.0)
            if k:
                z = Z.gather(1, idx.clamp(0, V - 1))
                picked[rows] = torch.where(has & on[:, None], z, 0.0)
                ent = torch.special.entr(q).sum(1)
                loss[rows] = torch.where(on, T * T * ((L - (q * z).sum(1)) - ent), 0.0)
            else:
                loss[rows] = torch.where(on, -(want * (Z - L[:, None])).sum(1), 0.0)
            continue
        P = torch.exp(Z - s["lse"][rows].to(f)[:, None])  # (from the stored log-sum-exp)
        G = (P - want) * (on * s["dloss"][rows].to(f) * s["dloss_scale"].item() * T)[:, None]
        dx[rows] = (G @ W) * sw
        dw += G.t() @ X
    if not back:
        return {"loss": loss, "lse": lse, "picked": picked} if k else {"loss": loss, "lse": lse}
    g = s["dloss_scale"].item()
    got = {}
    got["dx"], got["dx_scale"] = _exact_gradient(dx, g * sw, c)
    got["dw"], got["dw_scale"] = _exact_gradient(dw, g * sx, c)
    return got
