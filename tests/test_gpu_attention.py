"""The attention block (include/small_attn.h of the package) through the C ABI: group normalization with an activation, attention and their
gradients, against plain implementations in 64 bits on the CPU, at sizes, layouts and masks where they can go wrong.

Tolerances, in units of u = 2^-24 (derived, before the first run, from how many roundings reach a value):
 - a sum of K products in any order is off by at most K u sum |a b|; for values without a common sign the errors add like a random walk, sqrt(K).
   Results are compared with 64 bits at (32 + 4 sqrt(K)) u times their tensor's largest magnitude, where K is the longest sum on the
   way (channels and keys; values of a group). The 32 is for what does not grow with K: exp2 and its argument (scores up to 16 in size
   have a spacing of 2^-20, 16 u, and so does the probability's relative error), divisions, tanh.
 - a gradient passes a second chain of such sums over differences of the first one's results, P (dP - delta) with |dP| and |delta| up to ten times the result:
   ten times as much.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2303_04769_amd as S
from gpu_util import CANARY, DEV, GUARD

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def bound(K, ref, grad=False):
    return (32 + 4 * math.sqrt(K)) * U * (10 if grad else 1) * max(float(ref[torch.isfinite(ref)].abs().max()) if torch.isfinite(ref).any() else 0.0, 1e-3)


def assert_near(got, ref, K, what, grad=False):
    got = got.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.equal(torch.isfinite(got), torch.isfinite(ref)), f"{what}: infinities or NaN elsewhere"
    assert torch.equal(got[torch.isinf(got)], ref[torch.isinf(ref)]), what
    fin = torch.isfinite(ref)
    err = float((got - ref)[fin].abs().max()) if fin.any() else 0.0
    assert err <= bound(K, ref, grad), f"{what}: off by {err:.3e}, {bound(K, ref, grad):.3e} allowed"


def guarded(shape):
    """A tensor inside a larger one whose margins hold canaries, NaN inside: (tensor, check)."""
    n = int(np.prod(shape))
    full = torch.full((n + 2 * GUARD,), CANARY, dtype=torch.float32, device=DEV)
    t = full[GUARD:GUARD + n].view(*shape)
    t.fill_(float("nan"))

    def check():
        torch.cuda.synchronize()
        assert bool((full[:GUARD] == CANARY).all()) and bool((full[GUARD + n:] == CANARY).all()), "written outside the output"
    return t, check


def blocked(x, Cb):
    """[N][C][S] -> [N][C/Cb][S][Cb]"""
    N, Cc, P = x.shape
    return x.reshape(N, Cc // Cb, Cb, P).transpose(2, 3).contiguous()


def plain(x):
    """[N][C/Cb][S][Cb] -> [N][C][S]"""
    return x.transpose(2, 3).reshape(x.shape[0], -1, x.shape[2])


# ---------------------------------------------------------------------------------------------------- group normalization

def norm_ref(x, gamma, beta, G, eps, act):
    """64 bits, plain [N][C][S]."""
    N, Cc, P = x.shape
    g = x.reshape(N, G, -1)
    mean, var = g.mean(2, keepdim=True), g.var(2, unbiased=False, keepdim=True)
    rstd = (var + eps).rsqrt()
    z = ((g - mean) * rstd).reshape(N, Cc, P) * gamma[:, None] + beta[:, None]
    out = z if act == "none" else torch.where(z > 0, z, torch.zeros_like(z)) if act == "relu" else z * torch.sigmoid(z)
    return out, torch.cat((mean, rstd), 2)


def norm_case(N, Cc, H, W, seed, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, Cc, H * W, generator=g) * (1 + torch.rand(Cc, 1, generator=g)) + torch.randn(Cc, 1, generator=g) + shift
    return x, 1 + 0.3 * torch.randn(Cc, generator=g), 0.5 * torch.randn(Cc, generator=g), torch.randn(N, Cc, H * W, generator=g)


NORMS = [
    # N, C, H, W, G, Cb
    (1, 16, 1, 1, 1, 16), (1, 16, 1, 1, 16, 16), (2, 16, 1, 2, 4, 16),       # one pixel, one value a group
    (1, 64, 8, 8, 8, 16), (3, 64, 8, 8, 8, 64), (5, 48, 5, 7, 3, 16),        # groups as long as blocks, channels last
    (2, 96, 13, 9, 8, 16), (2, 96, 57, 43, 8, 16), (2, 48, 7, 5, 2, 16),     # groups that end inside blocks; one launch, two launches
    (3, 10, 6, 5, 2, 10), (3, 10, 6, 5, 5, 5), (1, 7, 9, 11, 7, 7), (2, 6, 120, 110, 3, 3),   # blocks that four does not divide
    (2, 256, 5, 5, 1, 16), (2, 512, 3, 3, 32, 512), (1, 2048, 2, 2, 2, 1024), (1, 4096, 1, 3, 4, 4096), (1, 1536, 40, 3, 3, 512),
    (1, 16, 56, 56, 2, 16), (300, 32, 4, 4, 4, 16), (600, 16, 16, 16, 4, 16), (1, 32, 200, 190, 4, 16), (2, 64, 128, 128, 1, 16),
]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("N,Cc,H,W,G,Cb", NORMS)
def test_groupnorm_and_its_gradient(N, Cc, H, W, G, Cb, act):
    x, gamma, beta, dout = norm_case(N, Cc, H, W, 11)
    eps = 1e-5
    xd, gd, bd = (t.double().requires_grad_() for t in (x, gamma, beta))
    out, stats = norm_ref(xd, gd, bd, G, eps, act)
    out.backward(dout.double())
    plan = S.GroupNorm(N, Cc, H, W, G, eps=eps, act=act, Cb=Cb)
    shape = (N, Cc // Cb, H * W, Cb)
    xb, gb, bb, db = blocked(x, Cb).to(DEV), gamma.to(DEV), beta.to(DEV), blocked(dout, Cb).to(DEV)
    (o, ok), (st, sk) = guarded(shape), guarded((N, G, 2))
    plan.run(xb, gb, bb, o, st)
    ok(), sk()
    n = Cc // G * H * W
    # (xhat is as far off as the mean is against the deviation; with a value or two in a group rstd grows up to 316 and carries that)
    K = n + (1e4 if n < 16 else 0)
    assert_near(plain(o), out.detach(), K, "out")
    assert_near(st, stats.detach(), K, "stats")
    (dx, xk), (dg, gk), (db2, bk) = guarded(shape), guarded((Cc,)), guarded((Cc,))
    plan.grad(xb, gb, bb, st, db, dx, dg, db2)
    xk(), gk(), bk()
    assert_near(db2, bd.grad, N * H * W, "dbeta", grad=True)
    assert_near(dg, gd.grad, max(K, N * H * W), "dgamma", grad=True)
    if n >= 16:        # (a few values: the gradient is the difference of nearly equal ones, all rounding)
        assert_near(plain(dx), xd.grad, n, "din", grad=True)
    # the same without parameters' gradients, in place of dout; and the forward call in place, without statistics
    again = db.clone()
    plan.grad(xb, gb, bb, st, again, again)
    assert torch.equal(again, dx)
    inplace = xb.clone()
    plan.run(inplace, gb, bb, inplace)
    assert torch.equal(inplace, o)


@pytest.mark.parametrize("H,W,Cb", [(8, 8, 16), (90, 90, 16), (9, 7, 48)])
def test_groupnorm_of_values_far_from_zero(H, W, Cb):
    """Values near 1000 with deviations near one: their squares' sums would leave two digits of the variance."""
    x, gamma, beta, _ = norm_case(2, 48, H, W, 3, shift=1000.0)
    out, stats = norm_ref(x.double(), gamma.double(), beta.double(), 4, 1e-5, "none")
    o, st = torch.empty(2, 48 // Cb, H * W, Cb, device=DEV), torch.empty(2, 4, 2, device=DEV)
    S.GroupNorm(2, 48, H, W, 4, Cb=Cb).run(blocked(x, Cb).to(DEV), gamma.to(DEV), beta.to(DEV), o, st)
    # a mean near 1000 is a multiple of 2^-14: half of that spacing, and as much for sums on the way, over a deviation of one or more
    assert float((plain(o).double().cpu() - out).abs().max()) <= 2 * 2.0 ** -14 * float(gamma.abs().max())
    assert float((st[..., 1].double().cpu() / stats[..., 1] - 1).abs().max()) <= 1e-6


def test_groupnorm_gradient_against_differences():
    """din, dgamma and dbeta against central differences of the forward formula, a few places each."""
    N, Cc, H, W, G, Cb, eps = 2, 32, 4, 5, 4, 16, 1e-3
    x, gamma, beta, dout = norm_case(N, Cc, H, W, 21)
    st, o = torch.empty(N, G, 2, device=DEV), torch.empty(N, Cc // Cb, H * W, Cb, device=DEV)
    plan = S.GroupNorm(N, Cc, H, W, G, eps=eps, act="silu", Cb=Cb)
    xb, gb, bb = blocked(x, Cb).to(DEV), gamma.to(DEV), beta.to(DEV)
    plan.run(xb, gb, bb, o, st)
    dx, dg, db = torch.empty_like(o), torch.empty(Cc, device=DEV), torch.empty(Cc, device=DEV)
    plan.grad(xb, gb, bb, st, blocked(dout, Cb).to(DEV), dx, dg, db)
    value = lambda *t: float((norm_ref(*t, G, eps, "silu")[0] * dout.double()).sum())  # noqa: E731
    args, h = [x.double(), gamma.double(), beta.double()], 1e-5
    for k, got in enumerate((plain(dx), dg, db)):
        flat = got.double().cpu().reshape(-1)
        for at in range(0, flat.numel(), max(1, flat.numel() // 9)):
            hi, lo = ([t.clone() for t in args] for _ in range(2))
            hi[k].reshape(-1)[at] += h
            lo[k].reshape(-1)[at] -= h
            diff = (value(*hi) - value(*lo)) / (2 * h)      # (off by h^2 times the third derivative, and by 2^-53 * 640 / h)
            assert abs(float(flat[at]) - diff) <= 1e-5 * max(1.0, abs(diff)), (k, at)


def test_groupnorm_infinities_and_nan_stay_in_their_group():
    x, gamma, beta, _ = norm_case(2, 32, 6, 6, 5)
    x[0, 3, 7], x[1, 20, 2] = float("inf"), float("nan")
    o = torch.empty(2, 2, 36, 16, device=DEV)
    S.GroupNorm(2, 32, 6, 6, 4, Cb=16, act="silu").run(blocked(x, 16).to(DEV), gamma.to(DEV), beta.to(DEV), o)
    bad = ~torch.isfinite(plain(o)).cpu().reshape(2, 4, -1).all(2)
    assert bad.tolist() == [[True, False, False, False], [False, False, True, False]]


# ---------------------------------------------------------------------------------------------------- attention

def attention_ref(q, k, v, heads, scale, cap=0.0, causal=False, lengths=None, first=None, prefix=None, docs=None, slopes=None, table=None,
                  bucket=None, reach=0, width=1):
    """64 bits, plain [N][C][S] tensors: (out [N][C][Sq], lse [N][heads][Sq])."""
    N, Cq, Sq = q.shape
    D, Sk = Cq // heads, k.shape[2]
    kv = k.shape[1] // D
    outs, lses = [], []
    j = torch.arange(Sk)
    for n in range(N):
        p = (Sk - Sq if first is None else int(first[n])) + torch.arange(Sq)
        seen = torch.ones(Sq, Sk, dtype=torch.bool)
        if lengths is not None:
            seen &= (j < int(lengths[n]))[None]
        if causal:
            seen &= (j[None] <= p[:, None]) | (j < (0 if prefix is None else int(prefix[n])))[None]
        if docs is not None:
            inside = (p >= 0) & (p < Sk)
            mine = torch.where(inside, docs[n][p.clamp(0, Sk - 1)], torch.tensor(-1))
            seen &= (docs[n][None] == mine[:, None]) & (mine >= 0)[:, None]
        for h in range(heads):
            kh, vh = k[n].reshape(kv, D, Sk)[h * kv // heads], v[n].reshape(kv, D, Sk)[h * kv // heads]
            s = scale * q[n].reshape(heads, D, Sq)[h].t() @ kh
            if cap:
                s = cap * torch.tanh(s / cap)
            if slopes is not None:
                s = s - slopes[h] * (p[:, None] - j[None]).abs()
            if table is not None:
                code = lambda x: torch.div(x, width, rounding_mode="floor") * (2 * width - 1) + x % width  # noqa: E731
                at = (code(j)[None] - code(p)[:, None]).clamp(-reach, reach) + reach
                s = s + table[h][bucket[at].long()]
            s = torch.where(seen, s, torch.tensor(-math.inf, dtype=s.dtype))
            empty = ~(s > -math.inf).any(1)
            s = torch.where(empty[:, None], torch.zeros_like(s), s)
            lse = torch.logsumexp(s, 1)
            # (keys that a row does not see count for nothing, whatever they hold)
            w = torch.where(seen & ~empty[:, None], torch.exp(s - lse[:, None]), torch.zeros_like(s))
            outs.append((w @ torch.where(torch.isfinite(vh), vh, torch.zeros_like(vh)).t()).t())
            lses.append(torch.where(empty, torch.tensor(-math.inf, dtype=s.dtype), lse))
    return torch.cat(outs).reshape(N, Cq, Sq), torch.stack(lses).reshape(N, heads, Sq)


class Case:
    def __init__(self, N=1, Sq=17, Sk=None, heads=2, kv=None, D=16, Cb=16, seed=1, cap=0.0, causal=False, lengths=None, first=None, prefix=None,
                 docs=None, slopes=False, bias=None, scale=None, size=1.0, table=None):
        g = torch.Generator().manual_seed(seed)
        self.N, self.Sq, self.Sk, self.heads, self.kv, self.D, self.Cb = N, Sq, Sk or Sq, heads, kv or heads, D, Cb
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.q, self.k, self.v = r(N, heads * D, Sq) * size, r(N, self.kv * D, self.Sk) * size, r(N, self.kv * D, self.Sk)
        self.dout = r(N, heads * D, Sq)
        self.scale, self.cap, self.causal = scale or D ** -0.5, cap, causal
        ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32)  # noqa: E731
        self.lengths, self.first, self.prefix, self.docs = ints(lengths), ints(first), ints(prefix), ints(docs)
        self.slopes = torch.tensor([2.0 ** -(h + 1) for h in range(heads)]) if slopes else None
        self.table = self.bucket = None
        self.reach, self.width, self.buckets = 0, 1, 0
        if bias == "log":
            self.bucket, self.buckets, self.reach = S.log_buckets(24, 12)
        elif bias == "wide":
            self.bucket, self.buckets, self.reach = S.log_buckets(9000, 16)
        elif bias is not None:
            self.bucket, self.buckets, self.reach, self.width = S.pixel_buckets(*bias)
        if bias is not None:
            self.table = r(heads, self.buckets) if table is None else table(heads, self.buckets)
        self.masks = {n: getattr(self, n) for n in ("lengths", "first", "prefix", "docs", "slopes", "table", "bucket")}

    def plan(self):
        return S.Attention(self.N, self.Sq, self.Sk, self.heads, self.kv, self.D, Cb=self.Cb, scale=self.scale, cap=self.cap, causal=self.causal,
                           width=self.width, reach=self.reach, buckets=self.buckets)

    def ref(self, q=None, k=None, v=None, table=None):
        m = {n: t.double() if t is not None and t.is_floating_point() else t for n, t in self.masks.items()}
        if table is not None:
            m["table"] = table
        return attention_ref(*((t if u is None else u).double() for t, u in ((self.q, q), (self.k, k), (self.v, v))), self.heads, self.scale,
                             cap=self.cap, causal=self.causal, reach=self.reach, width=self.width, **m)

    def dev(self):
        return [blocked(t, self.Cb).to(DEV) for t in (self.q, self.k, self.v)], {n: None if t is None else t.to(DEV) for n, t in self.masks.items()}

    def forward(self, plan=None, stats=True):
        (q, k, v), m = self.dev()
        (o, ok), (l, lk) = guarded((self.N, self.heads * self.D // self.Cb, self.Sq, self.Cb)), guarded((self.N, self.heads, self.Sq))
        (plan or self.plan()).run(q, k, v, o, l if stats else None, **m)
        ok(), lk()
        return o, l

    def check(self, grad=True):
        if not grad:
            ref, lse = self.ref()
        else:
            leaves = [t.double().requires_grad_() for t in (self.q, self.k, self.v)]
            table = None if self.table is None else self.table.double().requires_grad_()
            ref, lse = self.ref(*leaves, table=table)
            ref.backward(self.dout.double())
        K = self.D + self.Sk
        o, l = self.forward()
        assert_near(plain(o), ref.detach(), K, "out")
        assert_near(l, lse.detach(), K, "lse")
        if not grad:
            return
        (q, k, v), m = self.dev()
        (dq, c1), (dk, c2), (dv, c3) = (guarded(t.shape) for t in (q, k, v))
        dt, c4 = guarded(self.table.shape) if table is not None else (None, lambda: None)
        p = self.plan()
        p.grad(q, k, v, o, l, blocked(self.dout, self.Cb).to(DEV), dq, dk, dv, dt, **m)
        c1(), c2(), c3(), c4()
        rows = self.Sq * self.heads // self.kv
        zero = torch.zeros_like
        for name, got, leaf, n in (("dq", dq, leaves[0], K), ("dk", dk, leaves[1], rows + self.D), ("dv", dv, leaves[2], rows + self.D)):
            want = leaf.grad if leaf.grad is not None else zero(leaf)
            # (an absolute part where a softmax over a key or two leaves next to nothing of the differences it is taken from)
            scale = torch.cat((want.reshape(-1), torch.tensor([1.0], dtype=torch.float64)))
            err = float((plain(got).double().cpu() - want).abs().max())
            assert err <= bound(n, scale, True), f"{name}: off by {err:.3e}, {bound(n, scale, True):.3e} allowed"
        if dt is not None:
            want = table.grad if table.grad is not None else zero(table)
            K = self.N * self.Sq * self.Sk / max(1, min(self.buckets, 8))
            scale = torch.cat((want.reshape(-1), torch.tensor([1.0], dtype=torch.float64)))
            err = float((dt.double().cpu() - want).abs().max())
            assert err <= bound(K, scale, True), f"dtable: off by {err:.3e}, {bound(K, scale, True):.3e} allowed"


def _docs(N, S, sizes):
    rows = []
    for n in range(N):
        row = [d for d, s in enumerate(sizes[n % len(sizes)]) for _ in range(s)]
        rows.append((row + [-1] * S)[:S])
    return rows


CASES = {
    "one token, one key": dict(Sq=1),
    "one key, many rows": dict(Sq=70, Sk=1, N=2),
    "two keys": dict(Sq=2, N=3),
    "64 keys": dict(Sq=64, D=32), "65 keys": dict(Sq=65, D=64, heads=1), "63 rows on 129 keys": dict(Sq=63, Sk=129, D=48),
    "heads of 8": dict(Sq=40, D=8), "heads of 4 in blocks of 8": dict(Sq=40, D=4, Cb=8), "heads of 40 across blocks": dict(Sq=50, D=40),
    "heads of 5": dict(Sq=33, D=5, heads=3, Cb=5), "heads of 7 in one block": dict(Sq=33, D=7, heads=2, Cb=14),
    "heads of 80": dict(Sq=90, D=80, heads=2), "heads of 96": dict(Sq=70, D=96), "heads of 128": dict(Sq=100, D=128), "heads of 200": dict(Sq=40, D=200, Cb=8),
    "heads of 256": dict(Sq=70, D=256, heads=1), "heads of 131, odd": dict(Sq=30, D=131, heads=1, Cb=131),
    "channels last": dict(Sq=77, D=32, heads=4, Cb=128), "channels last, odd heads": dict(Sq=50, D=12, heads=3, kv=1, Cb=12),
    "shared key heads": dict(Sq=100, heads=6, kv=2, D=32), "shared key heads, few rows": dict(Sq=5, Sk=150, heads=8, kv=1, D=64),
    "shared key heads, rows of several heads in a tile": dict(Sq=23, heads=8, kv=2, D=16, bias="log", causal=True),
    "causal": dict(Sq=150, causal=True, D=64, heads=1), "causal, fewer rows than keys": dict(Sq=20, Sk=90, causal=True, heads=4, kv=2),
    "causal, more rows than keys": dict(Sq=90, Sk=20, causal=True),
    "prefix": dict(N=4, Sq=80, causal=True, prefix=[0, 1, 64, 200]), "prefix on a causal tile's edge": dict(N=2, Sq=130, causal=True, prefix=[65, 129]),
    "lengths with none": dict(N=4, Sq=70, lengths=[0, 1, 64, 70]), "lengths over and under": dict(N=3, Sq=66, lengths=[-3, 1000, 65], causal=True),
    "positions of their own": dict(N=5, Sq=10, Sk=100, causal=True, first=[0, 90, -4, -40, 300], slopes=True),
    "documents": dict(N=3, Sq=140, docs=_docs(3, 140, [[3, 60, 70], [140], [64, 64]])),
    "documents, causal": dict(N=2, Sq=100, causal=True, docs=_docs(2, 100, [[1, 1, 97], [30, 40]])),
    "documents out of order": dict(N=1, Sq=90, docs=[[(7 * i) % 4 - (i % 9 == 0) for i in range(90)]]),
    "no document at all": dict(N=2, Sq=70, docs=[[-1] * 70, [5] * 70]),
    "documents and positions outside": dict(N=2, Sq=30, Sk=60, docs=_docs(2, 60, [[20, 40]]), first=[-10, 45]),
    "distances": dict(N=2, Sq=100, slopes=True), "distances, causal, lengths": dict(N=2, Sq=90, slopes=True, causal=True, lengths=[90, 33]),
    "buckets": dict(N=2, Sq=150, bias="log", heads=3), "buckets, causal, shared": dict(Sq=140, bias="log", causal=True, heads=4, kv=2, D=32),
    "buckets too many for LDS": dict(N=1, Sq=80, bias="wide", heads=2), "buckets and distances": dict(Sq=90, bias="log", slopes=True),
    "pixels": dict(N=2, Sq=64, bias=(8, 8), heads=4), "pixels, odd": dict(N=2, Sq=91, bias=(7, 13), D=32), "pixels, one row": dict(Sq=70, bias=(1, 70)),
    "pixels, wide rows": dict(Sq=210, bias=(3, 70), heads=1), "pixels, some lines only": dict(N=1, Sq=30, Sk=60, bias=(10, 6)),
    "pixels with positions outside": dict(N=2, Sq=24, Sk=24, bias=(4, 6), first=[-7, 9]),
    "capped": dict(Sq=90, cap=5.0, size=2.0), "capped hard": dict(Sq=60, cap=0.5, size=4.0, causal=True),
    "capped, buckets, prefix": dict(N=2, Sq=90, cap=20.0, bias="log", causal=True, prefix=[10, 80], heads=4, kv=2, D=64),
    "everything": dict(N=3, Sq=100, cap=10.0, bias="log", slopes=True, causal=True, prefix=[5, 0, 77], lengths=[100, 64, 80],
                       docs=_docs(3, 100, [[50, 45], [100], [10, 10, 70]]), heads=6, kv=3, D=24, Cb=8),
}


@pytest.mark.parametrize("name", CASES)
def test_attention_and_its_gradient(name):
    Case(**CASES[name]).check()


# Larger sizes: all gradients but one (a table too large for LDS) and most forward calls are computed with values in two parts (which, test_gpu_attention_forms.py says).
LARGE = {
    "plain": dict(Sq=640, heads=4, D=64), "odd": dict(Sq=651, heads=4, D=64, Cb=8), "rows and keys of unlike number": dict(Sq=130, Sk=3100, heads=4, D=64),
    "causal, shared": dict(Sq=660, heads=8, kv=2, D=32, causal=True), "causal, distances": dict(Sq=700, heads=4, D=64, causal=True, slopes=True),
    "prefix, capped, buckets": dict(N=2, Sq=460, heads=4, kv=2, D=64, causal=True, prefix=[100, 321], cap=4.0, bias="log"),
    "lengths": dict(N=4, Sq=333, heads=4, D=64, lengths=[0, 1, 64, 333]), "documents": dict(N=2, Sq=500, heads=4, D=64, docs=_docs(2, 500, [[3, 60, 70, 300], [250, 250]])),
    "documents out of order": dict(N=1, Sq=700, heads=4, D=64, docs=[[(7 * i) % 4 - (i % 9 == 0) for i in range(700)]]),
    "positions of their own": dict(N=3, Sq=400, heads=4, D=64, causal=True, first=[-100, 50, 390], bias="log"),
    "pixels": dict(N=1, Sq=660, heads=4, D=64, bias=(20, 33)), "pixels, wide rows": dict(N=1, Sq=640, heads=4, D=64, bias=(2, 320)), "buckets": dict(Sq=651, heads=4, D=64, bias="log"),
    "buckets too many for LDS": dict(Sq=640, heads=4, D=64, bias="wide"), "heads of 16": dict(Sq=1300, heads=4, D=16, bias="log"), "heads of 8": dict(Sq=1300, heads=8, D=8),
    "heads of 40": dict(Sq=800, heads=4, D=40, Cb=8, bias="log", causal=True), "heads of 37": dict(Sq=850, heads=4, D=37, Cb=37), "heads of 80": dict(Sq=600, heads=4, D=80),
    "heads of 96": dict(Sq=540, heads=4, D=96, bias="log"), "heads of 128": dict(Sq=480, heads=4, D=128, causal=True, slopes=True, cap=9.0), "channels last": dict(Sq=640, heads=4, D=64, Cb=256),
    "causal, sixty-four heads": dict(N=4, Sq=600, heads=16, kv=4, D=16, causal=True, bias="log"),
    "causal, twenty-seven heads": dict(Sq=1220, heads=27, kv=9, D=8, Cb=8, causal=True), "small images": dict(N=40, Sq=196, heads=4, D=32, bias=(14, 14)),
    "few rows": dict(Sq=70, Sk=12000, heads=2, D=64, bias="log"), "everything": dict(N=3, Sq=400, cap=10.0, bias="log", slopes=True, causal=True, prefix=[50, 0, 300],
        lengths=[400, 64, 290], docs=_docs(3, 400, [[150, 235], [400], [10, 10, 370]]), heads=6, kv=3, D=48),
}


@pytest.mark.parametrize("name", LARGE)
def test_attention_and_its_gradient_in_parts(name):
    Case(**LARGE[name]).check()


@pytest.mark.parametrize("shape", [dict(Sq=300, heads=2, D=16), dict(Sq=1000, heads=4, D=48)], ids=["small", "in parts"])
def test_rows_far_behind_the_keys_they_see(shape):
    """Scores of several hundred by distance alone, whose lse is rounded to some 2^-15: weights and gradients are not. A weight is the power of a sum of
    at most four numbers below 16 with three roundings, 16 * 3 * 2^-24 = 2.9e-6 at most and a third of that in the mean square over hundreds of rows."""
    c = Case(N=2, lengths=[1, 7], slopes=True, **shape)
    leaves = [t.double().requires_grad_() for t in (c.q, c.k, c.v)]
    ref, _ = c.ref(*leaves)
    ref.backward(c.dout.double())
    plan = c.plan()
    (q, k, v), m = c.dev()
    o, lse = c.forward(plan)
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    plan.grad(q, k, v, o, lse, blocked(c.dout, c.Cb).to(DEV), dq, dk, dv, **m)
    for got, leaf, name in zip((dq, dk, dv), leaves, ("dq", "dk", "dv")):
        off = plain(got).double().cpu() - leaf.grad
        assert float(off.norm()) <= 2e-6 * float(leaf.grad.norm()), name


@pytest.mark.parametrize("N,Sk", [(16, 1500), (16, 6000), (2, 40000)])
def test_single_tokens_with_steep_distances(N, Sk):
    """Distances of thousands of keys at a slope of a half: what the far ones round must not reach the near ones, which alone count. Weights that do are
    powers of numbers below 16, rounded three times by 2^-21 at most, 1.4e-6, and a third of that in the mean square."""
    c = Case(N=N, Sq=1, Sk=Sk, heads=4, kv=2, D=32, slopes=True, cap=20.0)
    ref, _ = c.ref()
    o, _ = c.forward()
    off, want = ((t.double().cpu()).reshape(c.N, 4, 32) for t in (plain(o) - ref.to(DEV), ref))
    assert float((off.norm(dim=2) / want.norm(dim=2)).max()) <= 1e-6


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 30])
def test_parts_carry_any_magnitude(size):
    """Tensors far from one in size, and tokens of very different sizes beside each other: fp16 alone holds neither."""
    c = Case(Sq=640, heads=4, D=64)
    c.k, c.v, c.dout, c.scale = c.k * size, c.v * size, c.dout / size, c.scale / size
    c.check()
    c = Case(Sq=640, heads=4, D=64)
    steps = 2.0 ** (torch.arange(640) // 40 - 8)
    c.v, c.dout = c.v * steps, c.dout * steps.flip(0)
    c.check()


def test_parts_leave_what_masked_places_hold():
    """As for small sizes: NaN and infinities past lengths, in other documents, behind a causal row."""
    shape = dict(Sq=640, heads=4, D=64)
    c = Case(lengths=[600], **shape)
    want, lse = c.ref()
    c.k[0, :, 600:], c.v[0, :, 600:] = float("nan"), float("inf")
    o, l = c.forward()
    assert_near(plain(o), want, 704, "out past the length")
    assert_near(l, lse, 704, "lse past the length")
    for masks in (dict(causal=True), dict(docs=_docs(1, 640, [[500, 140]]))):
        want, lse = Case(**shape, **masks).ref()
        c = Case(**shape, **masks)
        c.v[0, 5, 510], c.k[0, :, 511] = float("inf"), float("nan")
        o, l = c.forward()
        assert_near(plain(o)[:, :, :500], want[:, :, :500], 704, "out in front")
        assert_near(l[:, :, :500], lse[:, :, :500], 704, "lse in front")
        assert not torch.isfinite(plain(o)[0, 5, 512:]).any()


TOKENS = {
    "one stream": dict(Sk=777, heads=8, D=32), "one key": dict(N=2, Sk=1), "a tile and a key": dict(N=2, Sk=33, D=64),
    "long": dict(N=1, Sk=5000, heads=2, D=64, bias="log"), "long, shared heads": dict(N=2, Sk=3001, heads=16, kv=1, D=128),
    "sixteen heads of 256": dict(N=1, Sk=600, heads=16, kv=1, D=256), "heads of 40": dict(N=3, Sk=500, heads=4, kv=2, D=40, Cb=8),
    "heads of 5": dict(N=2, Sk=300, heads=3, D=5, Cb=5), "heads of 16": dict(N=2, Sk=1500, heads=4, D=16), "heads of 80": dict(N=1, Sk=700, heads=2, D=80),
    "heads of 96": dict(N=1, Sk=1100, heads=2, D=96, slopes=True), "heads of 48": dict(N=1, Sk=1100, heads=2, D=48, cap=8.0),
    "ragged": dict(N=5, Sk=900, lengths=[0, 1, 31, 512, 900], first=[-1, 0, 30, 511, 899], causal=True, bias="log", heads=4, kv=2, D=64),
    "documents": dict(N=2, Sk=200, docs=_docs(2, 200, [[90, 110], [150]])), "pixels": dict(N=2, Sk=60, bias=(10, 6), causal=True),
    "four tokens": dict(N=2, Sq=4, Sk=700, heads=4, kv=1, causal=True, D=64), "wide bias": dict(N=1, Sk=1200, heads=4, kv=2, bias="wide"),
    "everything": dict(N=3, Sk=1200, cap=10.0, bias="log", slopes=True, causal=True, prefix=[5, 0, 77], lengths=[1100, 64, 1200],
                       docs=_docs(3, 1200, [[700, 500], [1200], [10, 1100]]), heads=8, kv=2, D=64, first=[1099, 63, 1000]),
}


@pytest.mark.parametrize("name", TOKENS)
def test_single_tokens_against_a_cache(name):
    Case(**{"Sq": 1, **TOKENS[name]}).check(grad=False)


@pytest.mark.parametrize("Sq,Sk", [(64, 2000), (20, 3000), (1, 4000)])
def test_rows_are_the_same_however_the_keys_are_split(Sq, Sk):
    """Few rows on many keys go over several workgroups and are joined: against 64 bits, and rows that see nothing."""
    Case(N=2, Sq=Sq, Sk=Sk, heads=2, D=32, lengths=[Sk, 0], bias="log", causal=True).check(grad=False)


def test_parts_of_one_tensor_longer_caches_and_unaligned_tensors():
    """q, k, v as slices of one projection's output; gradients into slices of one; a cache of which the first tokens are used; bases that
    are not 16-byte aligned: the same results as contiguous tensors give."""
    c = Case(N=3, Sq=50, heads=4, kv=2, D=32, bias="log", causal=True)
    (q, k, v), m = c.dev()
    o, l = c.forward()
    qkv = torch.cat((q, k, v), 1)
    nq, nk = q.shape[1], k.shape[1]
    parts = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
    o2, l2 = torch.empty_like(o), torch.empty_like(l)
    c.plan().run(*parts, o2, l2, **m)
    assert torch.equal(o, o2) and torch.equal(l, l2)
    dout = blocked(c.dout, 16).to(DEV)
    want = [torch.empty_like(t) for t in (q, k, v)]
    dt, dt2 = torch.empty_like(m["table"]), torch.empty_like(m["table"])
    c.plan().grad(q, k, v, o, l, dout, *want, dt, **m)
    grads = torch.full_like(qkv, float("nan"))
    c.plan().grad(*parts, o, l, dout, grads[:, :nq], grads[:, nq:nq + nk], grads[:, nq + nk:], dt2, **m)
    assert torch.equal(grads, torch.cat(want, 1)) and torch.equal(dt, dt2)
    # a cache with room for more
    room = [torch.full((3, nk, 90, 16), float("nan"), device=DEV) for _ in range(2)]
    for r, t in zip(room, (k, v)):
        r[:, :, :50] = t
    c.plan().run(q, room[0][:, :, :50], room[1][:, :, :50], o2, l2, **m)
    assert torch.equal(o, o2)
    # one float further on
    shifted = []
    for t in (q, k, v):
        s = torch.empty(t.numel() + 1, device=DEV)[1:].view(t.shape)
        shifted.append(s.copy_(t))
    c.plan().run(*shifted, o2, l2, **m)
    assert torch.equal(o, o2) and torch.equal(l, l2)


@pytest.mark.parametrize("shape", [dict(Sq=100, heads=2, D=32), dict(Sq=1, Sk=300, heads=4, kv=2, D=64), dict(Sq=30, Sk=1500, heads=1, D=16)])
def test_what_masked_places_hold_reaches_no_row(shape):
    """Keys past the length hold NaN and infinities; so do keys of other documents and keys behind a causal row."""
    N, Sk = 2, shape.get("Sk", shape["Sq"])
    c = Case(N=N, lengths=[Sk - 7, Sk // 2], **shape)
    want, lse = c.ref()
    for n, length in enumerate((Sk - 7, Sk // 2)):
        c.k[n, :, length:], c.v[n, :, length:] = float("nan"), float("inf")
    o, l = c.forward()
    assert_near(plain(o), want, Sk + c.D, "out past lengths")
    assert_near(l, lse, Sk + c.D, "lse past lengths")
    c = Case(N=1, docs=_docs(1, Sk, [[Sk // 3, Sk - Sk // 3]]), **shape)
    bad = Sk // 3 - 5
    c.k[0, :, bad], c.v[0, 3, bad] = float("inf"), float("nan")
    rows = (Sk - shape["Sq"] + torch.arange(shape["Sq"])) >= Sk // 3
    good = Case(N=1, docs=_docs(1, Sk, [[Sk // 3, Sk - Sk // 3]]), **shape)
    want, lse = good.ref()
    o, l = c.forward()
    assert_near(plain(o)[:, :, rows.to(DEV)], want[:, :, rows], Sk + c.D, "out of another document")
    assert_near(l[:, :, rows.to(DEV)], lse[:, :, rows], Sk + c.D, "lse of another document")
    if shape["Sq"] == 100:
        c = Case(N=1, causal=True, **shape)
        c.v[0, 5, 70], c.k[0, :, 71] = float("inf"), float("nan")
        want, lse = Case(N=1, causal=True, **shape).ref()
        o, l = c.forward()
        assert_near(plain(o)[:, :, :70], want[:, :, :70], Sk + c.D, "out in front of a causal key")
        assert not torch.isfinite(plain(o)[0, 5, 70:]).any() and not torch.isfinite(l[0, :, 71:]).any()


@pytest.mark.parametrize("value", [-math.inf, torch.finfo(torch.float32).min, -2e30])
def test_biases_of_the_lowest_value_and_of_minus_infinity(value):
    """A table entry of minus infinity hides its offsets, and so does one of the type's lowest value; rows left with nothing give zeros."""
    hide = lambda share: lambda heads, n: torch.where(torch.arange(n)[None] < share * n, torch.tensor(value), torch.zeros(heads, n))  # noqa: E731
    for Sq, Sk in ((70, 70), (1, 300)):
        c = Case(N=1, Sq=Sq, Sk=Sk, bias="log", causal=True, table=hide(0.25))
        low = Case(N=1, Sq=Sq, Sk=Sk, bias="log", causal=True, table=hide(0.25))
        low.masks["table"] = torch.where(low.table < -1e30, torch.tensor(-math.inf), low.table)
        want, lse = low.ref()
        o, l = c.forward()
        assert_near(plain(o), want, Sk + c.D, "out")
        assert_near(l, lse, Sk + c.D, "lse")
        c = Case(N=1, Sq=Sq, Sk=Sk, bias="log", table=hide(2))
        o, l = c.forward()
        assert bool((o == 0).all()) and bool((l == -math.inf).all())
        (q, k, v), m = c.dev()
        grads = [torch.empty_like(t) for t in (q, k, v)] + [torch.empty_like(m["table"])]
        c.plan().grad(q, k, v, o, l, blocked(c.dout, 16).to(DEV), *grads, **m)
        assert all(bool((t == 0).all()) for t in grads)


def test_attention_gradient_against_differences():
    """dq, dk, dv, dtable against central differences of the formula in 64 bits, a few places each."""
    c = Case(N=1, Sq=20, heads=2, kv=1, D=8, Cb=8, bias="log", causal=True, cap=3.0, prefix=[4])
    (q, k, v), m = c.dev()
    o, l = c.forward()
    grads = [torch.empty_like(t) for t in (q, k, v)] + [torch.empty_like(m["table"])]
    c.plan().grad(q, k, v, o, l, blocked(c.dout, 8).to(DEV), *grads, **m)
    args, h = [c.q.double(), c.k.double(), c.v.double(), c.table.double()], 1e-5
    value = lambda a: float((c.ref(*a[:3], table=a[3])[0] * c.dout.double()).sum())  # noqa: E731
    for i, got in enumerate(grads):
        flat = (got if i == 3 else plain(got)).double().cpu().reshape(-1)
        for at in range(0, flat.numel(), max(1, flat.numel() // 7)):
            hi, lo = ([t.clone() for t in args] for _ in range(2))
            hi[i].reshape(-1)[at] += h
            lo[i].reshape(-1)[at] -= h
            diff = (value(hi) - value(lo)) / (2 * h)
            assert abs(float(flat[at]) - diff) <= 2e-5 * max(1.0, abs(diff)), (i, at)


def test_calls_repeat_bit_for_bit_and_in_a_graph_and_on_another_stream():
    c = Case(N=4, Sq=130, heads=4, kv=2, D=32, bias="log", causal=True, cap=10.0)
    (q, k, v), m = c.dev()
    dout = blocked(c.dout, 16).to(DEV)
    norm = S.GroupNorm(4, 128, 10, 13, 8, act="silu")
    gamma, beta = torch.rand(128, device=DEV), torch.rand(128, device=DEV)
    plan = c.plan()

    def step(x):
        y, st, o, l = torch.empty_like(x), torch.empty(4, 8, 2, device=DEV), torch.empty_like(x), torch.empty(4, 4, 130, device=DEV)
        norm.run(x, gamma, beta, y, st)
        plan.run(y, k, v, o, l, **m)
        dq, dk, dv, dt = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(m["table"])
        plan.grad(y, k, v, o, l, dout, dq, dk, dv, dt, **m)
        dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
        norm.grad(x, gamma, beta, st, dq, dx, dg, db)
        return o, dk, dv, dt, dx, dg, db
    want = step(q)
    assert all(torch.equal(a, b) for a, b in zip(want, step(q)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step(q)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    static = q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(static)
    for scale in (1.0, 0.5, 1.0, 2.0):
        static.copy_(q * scale)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(q * scale), held))


def test_a_cache_of_more_than_2_31_values():
    """A cache whose offsets pass 32 bits: the last image's last tokens, against 64 bits of those alone."""
    N, Sk, heads, D = 5, 4_200_000, 2, 64
    k = torch.zeros(N, heads * D // 16, Sk, 16, device=DEV)
    v = torch.zeros_like(k)
    g = torch.Generator().manual_seed(9)
    last = 40
    kk, vv, q = (torch.randn(1, heads * D, s, generator=g) for s in (last, last, 1))
    k[-1:, :, -last:], v[-1:, :, -last:] = blocked(kk, 16).to(DEV), blocked(vv, 16).to(DEV)
    docs = torch.zeros(N, Sk, dtype=torch.int32, device=DEV)
    docs[:, -last:] = 1
    out = torch.empty(N, heads * D // 16, 1, 16, device=DEV)
    S.Attention(N, 1, Sk, heads, heads, D).run(blocked(q, 16).to(DEV).expand(N, -1, -1, -1), k, v, out, docs=docs)
    ref, _ = attention_ref(q.double(), kk.double(), vv.double(), heads, D ** -0.5)
    assert_near(plain(out)[-1:], ref, last + D, "out")
    assert bool((out[:-1] == 0).all())
