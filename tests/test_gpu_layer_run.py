"""A layer's first half on the GPU, as it would be run: the residual's addition
and RMS norm with 8-bit scales, the scaled matmul that takes those scales, attention
over column ranges of its result, and the way back; and a token's step over an 8-bit
cache. Each stage is checked against its plain 64-bit form on the arrays that it
was given, and the whole, captured, against the eager run."""
import numpy as np
import pytest
import torch

from paper_2407_17353_amd import binding as sc
from tests import layer_refs as lr
from tests import test_gpu_attention as attn
from tests import test_gpu_rmsnorm as rms
from tests.helpers import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, E4M3, E5M2 = sc.F16, sc.E4M3, sc.E5M2
H, HKV, D, C, EPS = 4, 2, 64, 320, 1e-5
NQ, NK = H * D, HKV * D
STARTS = [0, 41, 42, 42, 160]  # packed prompts: one of a single token, one empty
T = STARTS[-1]


def columns(x, a, b):
    return sc.ScaledArray(x.data[:, a:b], x.fmt, x.scale)


def check_product(a, b, extra, out):
    """out against a b + extra (64-bit true values): fp32 sums of K products, the
    scaled add's rounding, and the cast (2^-11 of the value, 2^-25 below the normal range)."""
    want = a @ b + extra
    e = lr.log2_of(out)
    err = 2 * (a.shape[1] + 4) * lr.U * (a.abs() @ b.abs()) + 4 * lr.U * want.abs()
    rel, sub = lr.HALF[out.fmt]
    got = lr.data(out) * 2.0 ** e
    assert ((got - want).abs() <= err + (want.abs() + err) * rel + sub * 2.0 ** e).all()


def true(x):
    return lr.data(x) * 2.0 ** lr.log2_of(x)


class Block:
    def __init__(self, scales):
        self.scales = scales
        self.x, self.r = lr.values(T, C, F16, 1), lr.values(T, C, F16, 2)
        self.gamma = 1.0 + 0.2 * torch.randn(C, generator=torch.Generator().manual_seed(3))
        w = lr.values(C, NQ + 2 * NK, E4M3, 4)
        self.do, self.dsum = lr.values(T, NQ, F16, 5), lr.values(T, C, F16, 6)
        self.X, self.R, self.W = lr.scaled(self.x, F16, -2), lr.scaled(self.r, F16, 1), lr.scaled(w, E4M3, -6)
        self.wt = w.to(lr.F64) * 2.0 ** -6
        self.DO, self.DSUM = lr.scaled(self.do, F16, -6), lr.scaled(self.dsum, F16, -7)
        self.g = self.gamma.to(DEV)
        self.row = torch.full((T,), 7.0, device=DEV) if scales == "row" else None
        self.blk = self.wblk = None
        if scales == "mx":
            self.blk = torch.full((sc.scalify_mx_packed_bytes(T, C),), 0xEE, dtype=torch.uint8, device=DEV)
            nat = torch.randint(126, 129, (NQ + 2 * NK, C // 32), generator=torch.Generator().manual_seed(7), dtype=torch.uint8)
            self.wblk = sc.scalify_mx_pack_block_scales(nat.to(DEV), C)
            self.wscaled = self.wt * torch.exp2(nat.double() - 127).t().repeat_interleave(32, 0)
        else:
            self.wscaled = self.wt
        self.S, self.N = lr.empty(T, C, F16), lr.empty(T, C, E4M3, ld=(C + 48) // 16 * 16)
        self.pre = torch.full((T, C), 9.0, device=DEV)
        self.QKV, self.O = lr.empty(T, NQ + 2 * NK, F16), lr.empty(T, NQ, F16)
        self.lse = torch.full((H, T), 7.0, device=DEV)
        self.grads = [lr.empty(T, n, E5M2) for n in (NQ, NK, NK)]
        self.amax = torch.full((3,), -1.0, device=DEV)
        self.dn = [lr.empty(T, C, F16) for _ in range(3)]
        self.DX = lr.empty(T, C, E5M2, ld=(C + 48) // 16 * 16)
        self.pre_dx, self.dgamma = torch.full((T, C), 9.0, device=DEV), torch.full((C,), 9.0, device=DEV)
        self.amax_dx = torch.full((1,), -1.0, device=DEV)
        start = torch.tensor(STARTS, dtype=torch.int64, device=DEV)
        self.opts = dict(heads=H, kv_heads=HKV, batch=len(STARTS) - 1, causal=True, q_start=start, k_start=start)

    def outputs(self):
        arrays = [self.S, self.N, self.QKV, self.O, *self.grads, *self.dn, self.DX]
        plain = [self.pre, self.lse, self.amax, self.pre_dx, self.dgamma, self.amax_dx, self.row, self.blk]
        return [t for a in arrays for t in (a.data, a.scale)] + [t for t in plain if t is not None]

    def run(self):
        sc.scalify_rmsnorm_fwd(self.X, self.N, residual=self.R, sum_out=self.S, gamma=self.g, eps=EPS, row_scale=self.row,
                               block_scale=self.blk, target_log2=7, pre_out=self.pre)
        sc.scalify_matmul(self.N, self.W, self.QKV, rescale=sc.RESCALE_NONE, a_channel_scale=self.row,
                          a_block_scale=self.blk, b_block_scale=self.wblk)
        q, k, v = (columns(self.QKV, a, b) for a, b in ((0, NQ), (NQ, NQ + NK), (NQ + NK, NQ + 2 * NK)))
        sc.scalify_attention_fwd(q, k, v, self.O, lse=self.lse, **self.opts)
        sc.scalify_attention_bwd(self.DO, q, k, v, self.O, self.lse, *self.grads, target_log2=0, amax_out=self.amax, **self.opts)
        at = 0
        for i, x in enumerate(self.grads):
            n = x.shape[1]
            w = sc.ScaledArray(self.W.data[:, at:at + n], E4M3, self.W.scale, trans=True)
            sc.scalify_matmul(x, w, self.dn[i], residual=self.dn[i - 1] if i else None)
            at += n
        sc.scalify_rmsnorm_bwd(self.dn[2], self.S, self.DX, dsum=self.DSUM, gamma=self.g, eps=EPS, dgamma=self.dgamma,
                               amax_out=self.amax_dx, pre_out=self.pre_dx)


@pytest.mark.parametrize("scales", ["row", "mx"])
def test_layer(scales):
    say(f"layer {scales}")
    b = Block(scales)
    b.run()
    torch.cuda.synchronize()
    rms.check_fwd(b.x, F16, b.gamma, b.r, F16, F16, E4M3, scales, 7, EPS, (b.N, b.S, b.pre.cpu(), b.row, b.blk))
    # the norm's true values, from the exponents that check_fwd has checked
    p = np.abs(b.pre.cpu().numpy())
    if scales == "row":
        e = np.repeat(rms.exponents(p.max(1), 7)[:, None], C, 1)
    else:
        e = np.repeat(rms.exponents(p.reshape(T, C // 32, 32).max(2), 7), 32, 1)
    n = lr.data(b.N) * torch.exp2(torch.from_numpy(e).double())
    check_product(n, b.wscaled, 0.0, b.QKV)
    eq = lr.log2_of(b.QKV)
    q, k, v = (lr.data(columns(b.QKV, a, c)) for a, c in ((0, NQ), (NQ, NQ + NK), (NQ + NK, NQ + 2 * NK)))
    case = attn._case("layer", H=H, Hkv=HKV, D=D, B=len(STARTS) - 1, Tq=T, Tk=T, q_start=STARTS, k_start=STARTS)
    case.update(eq=eq, ek=eq, ev=eq, alpha=D ** -0.5)
    attn.check_fwd(case, q, k, v, b.O, b.lse)
    attn.check_bwd(case, q, k, v, b.do, (b.grads, b.amax.cpu(), b.O, b.lse, None), E5M2)
    at, before = 0, 0.0
    for x, y in zip(b.grads, b.dn):
        m = x.shape[1]
        check_product(true(x), b.wt[:, at:at + m].t(), before, y)
        before, at = true(y), at + m
    rms.check_bwd(lr.data(b.dn[2]), lr.data(b.S), b.gamma, b.dsum, E5M2, sc.RESCALE_AMAX, 0,
                  (b.DX, b.pre_dx.cpu(), b.dgamma.cpu(), float(b.amax_dx.item())), eps=EPS, edy=lr.log2_of(b.dn[2]),
                  ex=lr.log2_of(b.S), eds=-7)


@pytest.mark.parametrize("scales", ["row", "mx"])
def test_layer_captured(scales):
    """The whole run as one graph, replayed over dirtied outputs with eager runs between."""
    b, eager = Block(scales), Block(scales)
    eager.run()
    torch.cuda.synchronize()
    want = [t.clone() for t in eager.outputs()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        b.run()
    for _ in range(3):
        for t in b.outputs():
            t.fill_(1)
        g.replay()
        eager.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(b.outputs(), want))
        assert all(torch.equal(x, y) for x, y in zip(eager.outputs(), want))


def test_tokens_over_an_8_bit_cache():
    """Four steps of three sequences: norm, product, the new key and value cast into the
    cache, and attention over what each sequence holds by then."""
    say("tokens over a cache")
    B, room, lens = 3, 70, [0, 31, 64]
    w = lr.values(C, NQ + 2 * NK, E4M3, 4)
    W, gamma = lr.scaled(w, E4M3, -6), rms._gamma(C)
    cache = [lr.scaled(torch.full((B * room, NK), float("nan")).to(lr.TORCH[E4M3]), E4M3, e) for e in (-1, 0)]
    for c in cache:
        old = lr.values(B * room, NK, E4M3, 11)
        for i, n in enumerate(lens):
            c.data[i * room:i * room + n] = old[i * room:i * room + n].view(torch.uint8).to(DEV)
    k_len = torch.tensor(lens, dtype=torch.int64, device=DEV)
    first = torch.arange(0, B * room, room, device=DEV)
    for step in range(4):
        x, r = lr.values(B, C, F16, 20 + step), lr.values(B, C, F16, 30 + step)
        out, s, pre, row, _ = rms.run_fwd(x, F16, gamma, r, scales="row", target=7)
        rms.check_fwd(x, F16, gamma, r, F16, F16, E4M3, "row", 7, 1e-5, (out, s, pre, row, None))
        qkv, o = lr.empty(B, NQ + 2 * NK, F16), lr.empty(B, NQ, F16)
        sc.scalify_matmul(out, W, qkv, rescale=sc.RESCALE_NONE, a_channel_scale=row)
        for c, e, a in ((cache[0], -1, NQ), (cache[1], 0, NQ + NK)):
            new = lr.empty(B, NK, E4M3)
            sc.scalify_set_scaling(sc.ScaledArray(qkv.data[:, a:a + NK].contiguous(), F16, qkv.scale), new, e)
            c.data[first + k_len] = new.data
        k_len += 1
        sc.scalify_attention_fwd(columns(qkv, 0, NQ), *cache, o, heads=H, kv_heads=HKV, batch=B, causal=True, k_len=k_len)
        torch.cuda.synchronize()
        check_product(lr.data(out) * row.cpu().double()[:, None], w.to(lr.F64) * 2.0 ** -6, 0.0, qkv)
        held = [n + step + 1 for n in lens]
        case = attn._case("tokens", H=H, Hkv=HKV, D=D, B=B, Lq=1, Lk=room, fk=E4M3, k_len=held)
        case.update(eq=lr.log2_of(qkv), ek=-1, ev=0, alpha=D ** -0.5)
        k, v = (lr.data(c).clone() for c in cache)
        for t in (k, v):
            for i in range(B):
                assert t[i * room:i * room + held[i]].isfinite().all()
                t[i * room + held[i]:(i + 1) * room] = 0.0  # (NaN, which no row may see)
        attn.check_fwd(case, lr.data(columns(qkv, 0, NQ)), k, v, o, None)


def test_calls_side_by_side():
    """Calls of each kind on two streams at once, each with a workspace of its own."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    blocks = [Block("row"), Block("mx")]
    serial = [Block("row"), Block("mx")]
    long = next(c for c in attn.CASES if c["name"] == "token_long")
    q, k, v = attn._inputs(long)
    A = [lr.scaled(t, F16, e) for t, e in ((q, 1), (k, -2), (v, 3))]
    want, _ = attn.run_fwd(long, q, k, v)
    for b in serial:
        b.run()
    torch.cuda.synchronize()
    for _ in range(3):
        outs = [[lr.empty(1, q.shape[1], F16) for _ in range(4)] for _ in streams]
        torch.cuda.synchronize()
        for i in range(4):
            for s, b, o in zip(streams, blocks, outs):
                with torch.cuda.stream(s):
                    sc.scalify_attention_fwd(*A, o[i], **attn._opts(long))
                    b.run()
        torch.cuda.synchronize()
        for b, c in zip(blocks, serial):
            assert all(torch.equal(x, y) for x, y in zip(b.outputs(), c.outputs()))
        assert all(np.array_equal(lr.codes(x), lr.codes(want)) for o in outs for x in o)
