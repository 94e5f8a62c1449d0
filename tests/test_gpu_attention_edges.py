"""GPU parity of attention where its sizes, masks and magnitudes meet their
edges, against the plain 64-bit forms and bounds of tests/layer_refs.py."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests import test_gpu_attention as attn
from tests.helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3, E5M2 = sc.F16, sc.E4M3, sc.E5M2


# ---------------------------------------------------------------- magnitudes of v along a sequence

def _lone_last_key(D, small, H=1, Lq=64, n=128, causal=False):
    """n keys of equal scores and values along one direction, and a last key of about
    half of every query's weight whose value is `small` of theirs: dS of the last
    key, -P delta, is far beyond what its own value gives."""
    case = attn._case("lone", H=H, Hkv=1, D=D, Lq=Lq, Lk=n + 1, causal=causal)
    g = torch.Generator().manual_seed(D)
    w = torch.randn(D, generator=g)
    factor = case["alpha"] * 2.0 ** (case["eq"] + case["ek"])
    q = 1.0 + 0.01 * torch.randn((Lq, H * D), generator=g)
    k = 0.01 * torch.randn((n + 1, D), generator=g)
    k[n] += math.log(n) / (factor * D)
    v = w + 0.05 * torch.randn((n + 1, D), generator=g)
    v[n] *= small
    do = w.repeat(H) + 0.05 * torch.randn((Lq, H * D), generator=g)
    return case, [t.half() for t in (q, k, v, do)]


@pytest.mark.parametrize("small", [2.0 ** -6, 2.0 ** -8, 2.0 ** -12])
@pytest.mark.parametrize("D,H", [(64, 1), (128, 1), (80, 4)])
def test_backward_small_value_of_a_heavy_key(D, H, small):
    say(f"attention bwd lone key {D} {H} {small}")
    case, t = _lone_last_key(D, small, H)
    res = attn.run_bwd(case, *t)
    attn.check_bwd(case, *t, res)
    assert all(lr.data(x).isfinite().all() for x in res[0])


@pytest.mark.parametrize("causal,sq,e", [(False, 1.0, -13), (False, 4.0, -10), (True, 4.0, -13)])
@pytest.mark.parametrize("D,H,Lq", [(64, 2, 160), (128, 2, 160), (64, 8, 1000)])
def test_backward_small_values_of_the_last_keys(D, H, Lq, causal, sq, e):
    """The last of 160 keys' values times 2^e (with 1000 queries of 8 heads a key head: in parts)."""
    say(f"attention bwd small values {D} {H} {Lq} {causal} {e}")
    case = attn._case("small", H=H, Hkv=1 if H == 8 else 2, D=D, Lq=Lq, Lk=160, sq=sq, causal=causal)
    q, k, v, do = attn._bwd_inputs(case)
    v[128:] *= 2.0 ** e
    for mode in (sc.RESCALE_NONE, sc.RESCALE_AMAX):
        attn.check_bwd(case, q, k, v, do, attn.run_bwd(case, q, k, v, do, mode=mode))


@pytest.mark.parametrize("scale", [2.0 ** -8, 2.0 ** -12])
@pytest.mark.parametrize("D,causal", [(64, False), (128, True)])
def test_backward_keys_without_values(D, causal, scale):
    """Keys 128 ... 255 of 300 with zeros for values: their dS is -P delta."""
    say(f"attention bwd no values {D} {scale}")
    case = attn._case("zeros", H=2, Hkv=1, D=D, Lq=300, Lk=300, causal=causal)
    q, k, v, do = attn._bwd_inputs(case)
    v[128:256] = 0
    do = (do.float() * scale).half()
    res = attn.run_bwd(case, q, k, v, do, mode=sc.RESCALE_AMAX)
    attn.check_bwd(case, q, k, v, do, res)
    assert (res[0][1].data[128:256] != 0).any()


# ---------------------------------------------------------------- rows without keys

@pytest.mark.parametrize("D,H", [(64, 2), (128, 2), (64, 1)])
@pytest.mark.parametrize("mode", [sc.RESCALE_NONE, sc.RESCALE_AMAX])
def test_backward_query_without_keys_of_any_value(D, H, mode):
    """A query that sees no key has no gradient and gives none, whatever q, dO and
    the rows beside it hold (rows 0 to 9 of 150 queries over 140 keys)."""
    say(f"attention bwd no keys {D} {H} {mode}")
    case = attn._case("empty_rows", H=H, Hkv=1, D=D, Lq=150, Lk=140)
    q, k, v, do = attn._bwd_inputs(case)
    clean = attn.run_bwd(case, q, k, v, do, mode=mode)
    q2, d2 = q.clone(), do.clone()
    q2[0], q2[5, 3], q2[9] = float("nan"), float("inf"), float("nan")
    d2[1, 2], d2[2], d2[3, 4], d2[9] = float("inf"), float("nan"), float("-inf"), float("nan")
    got = attn.run_bwd(case, q2, k, v, d2, mode=mode)
    assert (got[0][0].data[:10] == 0).all()
    for a, b in zip(got[0], clean[0]):
        assert np.array_equal(lr.codes(a), lr.codes(b)) and a.scale.item() == b.scale.item()
    assert torch.equal(got[1], clean[1])


@pytest.mark.parametrize("Lq,max_q,Lk", [(100, 40, 130), (70, 8, 300), (90, 1, 60), (300, 140, 300)])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_past_max_q(D, Lq, max_q, Lk):
    """Rows of a sequence past max_q are left out; the others see the keys that
    their place in the whole sequence gives them."""
    say(f"attention past max_q {D} {Lq} {max_q} {Lk}")
    case = attn._case("past", H=2, Hkv=1, D=D, B=2, Tq=2 * Lq, Tk=2 * Lk, q_start=[0, Lq, 2 * Lq], max_q=max_q)
    q, k, v, do = attn._bwd_inputs(case)
    res = attn.run_bwd(case, q, k, v, do)
    out, lse = res[2], res[3]
    live = torch.zeros(2 * Lq, dtype=torch.bool)
    live[:max_q] = live[Lq:Lq + max_q] = True
    o, eo, l, el = lr.attention(q.to(lr.F64), k.to(lr.F64), v.to(lr.F64), 2, 1, case["alpha"] * 2.0 ** (case["eq"] + case["ek"]),
                                attn._seqs(case), True, F16)
    assert ((lr.data(out) - o).abs() <= eo)[live].all() and (lr.codes(out)[~live.numpy()] == 0x5A5A).all()
    m = lse.cpu().to(lr.F64)
    assert torch.equal(m[:, live].isinf(), l[:, live].isinf()) and (m[:, ~live] == 7.0).all()
    f = l.isfinite() & live
    assert ((m - l).abs() <= el)[f].all()
    do[~live] = 0  # (what a query that is left out gives)
    want, err = attn._reference(case, q, k, v, do, out, lse)
    rel, sub = lr.HALF[F16]
    for x, w, e, rows in zip(res[0], want, err, (live, slice(None), slice(None))):
        assert ((lr.data(x) - w).abs() <= e + (w.abs() + e) * rel + sub)[rows].all()
    assert (lr.codes(res[0][0])[~live.numpy()] == 0x5A5A).all()


# ---------------------------------------------------------------- grids

MANY = dict(B=2048, H=32, Hkv=32, D=16, Tq=32768, Tk=32768)


def _many(seed=1):
    """2048 short sequences packed into 32768 rows of 32 heads, with the bounds that
    the options give by default (any number of rows each)."""
    case = attn._case("many", fk=F16, **MANY)
    r = np.random.RandomState(seed)
    at = np.sort(r.randint(0, case["Tq"] + 1, case["B"] - 1))
    case["q_start"] = case["k_start"] = [0, *at.tolist(), case["Tq"]]
    return case


def _bounded(case):
    n = int(np.diff(case["q_start"]).max())
    return dict(case, max_q=n, max_k=n)


@pytest.mark.parametrize("mode", [sc.RESCALE_NONE, sc.RESCALE_AMAX])
def test_packed_sequences_without_bounds(mode):
    """More than 2^24 workgroups: what a call with the bounds gives, to the bit."""
    say(f"attention many workgroups {mode}")
    case = _many()
    q, k, v, do = attn._bwd_inputs(case)
    want = attn.run_bwd(_bounded(case), q, k, v, do, mode=mode)
    got = attn.run_bwd(case, q, k, v, do, mode=mode)
    assert np.array_equal(lr.codes(got[2]), lr.codes(want[2])) and torch.equal(got[3], want[3])
    for a, b in zip(got[0], want[0]):
        assert np.array_equal(lr.codes(a), lr.codes(b)) and a.scale.item() == b.scale.item()
    assert torch.equal(got[1], want[1])
    assert lr.data(want[2]).isfinite().all() and (lr.data(want[2]) != 0).any()


def test_more_rows_and_heads_than_threads_of_a_launch():
    """The last 64 of 2^20 + 64 rows of 256 heads (25 GB in all): their numbers lie past
    2^32 threads of the kernel that forms them. What the same rows give by themselves."""
    say("attention bwd 2^28 rows and heads")
    n, H, D, before = 64, 256, 16, 1 << 20
    case = attn._case("rows", H=H, D=D, Lq=n, Lk=n, fq=E4M3, fk=E4M3)
    q, k, v = attn._inputs(case)
    do = lr.values(n, H * D, E4M3, 9)
    want = attn.run_bwd(case, q, k, v, do, fdo=E4M3, fg=E4M3)
    T = before + n

    def tall(fmt, e, t=None):
        x = torch.zeros((T, H * D), dtype=sc.STORAGE_DTYPE[fmt], device=DEV)
        if t is not None:
            x[before:] = t
        return sc.ScaledArray(x, fmt, sc.scale_tensor(e, DEV))
    K, V = lr.scaled(k, E4M3, case["ek"]), lr.scaled(v, E4M3, case["ev"])
    Q, DO = (tall(E4M3, e, t.view(torch.uint8).to(DEV)) for t, e in ((q, case["eq"]), (do, -6)))
    out, dq = tall(F16, 0), tall(E4M3, 0)
    dk, dv = lr.empty(n, H * D, E4M3), lr.empty(n, H * D, E4M3)
    lse = torch.zeros((H, T), device=DEV)
    opts = dict(attn._opts(case), q_start=attn._i64([before, T]), max_q=n)
    sc.scalify_attention_fwd(Q, K, V, out, lse=lse, **opts)
    sc.scalify_attention_bwd(DO, Q, K, V, out, lse, dq, dk, dv, rescale=sc.RESCALE_NONE, **opts)
    torch.cuda.synchronize()
    assert torch.equal(out.data[before:], want[2].data) and torch.equal(lse[:, before:], want[3])
    for x, y in ((sc.ScaledArray(dq.data[before:], E4M3, dq.scale), want[0][0]), (dk, want[0][1]), (dv, want[0][2])):
        assert np.array_equal(lr.codes(x), lr.codes(y)) and x.scale.item() == y.scale.item()
    assert (dq.data[:before] == 0).all() and (out.data[:before] == 0).all()


# ---------------------------------------------------------------- placement over the XCDs

@pytest.mark.parametrize("B,H,Hkv,D,L,causal", [(5, 16, 8, 64, 150, True), (10, 8, 8, 64, 140, True), (5, 8, 8, 128, 131, False),
                                                (3, 16, 16, 64, 129, True), (7, 8, 8, 64, 65, True)])
def test_heads_in_groups(B, H, Hkv, D, L, causal):
    """Key heads a multiple of 8: 5, 6, 7 or 10 of them on an XCD, the last group of
    one, two or three, with several tiles each."""
    say(f"attention placement {B} {H} {Hkv} {D}")
    case = attn._case("placed", B=B, H=H, Hkv=Hkv, D=D, Lq=L, Lk=L, causal=causal)
    t = attn._bwd_inputs(case)
    res = attn.run_bwd(case, *t)
    attn.check_fwd(case, *t[:3], res[2], res[3])
    attn.check_bwd(case, *t, res)


@pytest.mark.parametrize("B,Hkv", [(5, 8), (10, 8), (1, 40), (2, 4)])
@pytest.mark.parametrize("Lq,fk", [(1, F16), (1, E4M3), (9, F16)])
def test_heads_in_groups_split_keys(B, Hkv, Lq, fk):
    """The same for few queries, whose keys are split over workgroups and joined."""
    say(f"attention placement split {B} {Hkv} {Lq}")
    case = attn._case("placed_split", B=B, H=4 * Hkv, Hkv=Hkv, D=64, Lq=Lq, Lk=1100, fk=fk, k_len=[1100 - 37 * b for b in range(B)])
    q, k, v = attn._inputs(case)
    Q = lr.scaled(q, F16, case["eq"])
    assert sc.scalify_attention_fwd_workspace_size(B * Lq, B * 1100, sc.attention_opts(Q, **attn._opts(case))) > 0
    out, lse = attn.run_fwd(case, q, k, v)
    attn.check_fwd(case, q, k, v, out, lse)


@pytest.mark.parametrize("B,Hkv", [(5, 8), (3, 16)])
def test_heads_in_groups_parts(B, Hkv):
    """The same for the backward whose queries are shared by several workgroups."""
    say(f"attention placement parts {B} {Hkv}")
    case = attn._case("placed_parts", B=B, H=2 * Hkv, Hkv=Hkv, D=64, Lq=500, Lk=100)
    t = attn._bwd_inputs(case)
    Q = lr.scaled(t[0], F16, case["eq"])
    n = sc.scalify_attention_bwd_workspace_size(500 * B, 100 * B, sc.attention_opts(Q, **attn._opts(case)), sc.RESCALE_NONE)
    assert n > 256 + 4 * (2 * 500 * B * 2 * Hkv + 100 * B * Hkv) + 16
    attn.check_bwd(case, *t, attn.run_bwd(case, *t))


def test_an_error_of_an_earlier_call_stops_nothing():
    """The HIP runtime keeps the last error of any call; a call's launches go by their own."""
    case = attn._case("stale", Lq=70, Lk=90)
    t = attn._bwd_inputs(case)
    want = attn.run_bwd(case, *t)
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64" in line)
    hip = ctypes.CDLL(path)
    Q, K, V, DO = (lr.scaled(x, F16, e) for x, e in zip((*t[:3], t[3]), (case["eq"], case["ek"], case["ev"], -6)))
    out, lse = lr.empty(70, 128, F16), torch.zeros((2, 70), device=DEV)
    grads = [lr.empty(*x.shape, F16) for x in t[:3]]
    o = attn._opts(case)
    ws = sc.workspace(sc.scalify_attention_bwd_workspace_size(70, 90, sc.attention_opts(Q, **o), sc.RESCALE_NONE), DEV)
    torch.cuda.synchronize()
    assert hip.hipSetDevice(1 << 20) != 0
    sc.scalify_attention_fwd(Q, K, V, out, lse=lse, **o)
    hip.hipSetDevice(1 << 20)
    sc.scalify_attention_bwd(DO, Q, K, V, out, lse, *grads, rescale=sc.RESCALE_NONE, ws=ws, **o)
    hip.hipGetLastError()
    torch.cuda.synchronize()
    assert np.array_equal(lr.codes(out), lr.codes(want[2]))
    assert all(np.array_equal(lr.codes(a), lr.codes(b)) for a, b in zip(grads, want[0]))
