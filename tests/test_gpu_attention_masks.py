"""Attention and its gradient where masks leave little or nothing, and what hidden places hold: against the 64-bit implementation of
test_gpu_attention.py, with its tolerances unless a test derives its own.
"""
import pytest
import torch

from gpu_util import DEV
from test_gpu_attention import Case, _docs, blocked, guarded, plain

pytestmark = pytest.mark.gpu


def gradients(c, dout=None):
    """(out, lse, dq, dk, dv, dtable) of a case, the gradients in plain layout; every tensor NaN before."""
    (q, k, v), m = c.dev()
    o, l = c.forward()
    (dq, c1), (dk, c2), (dv, c3) = (guarded(t.shape) for t in (q, k, v))
    dt, c4 = guarded(c.table.shape) if c.table is not None else (None, lambda: None)
    c.plan().grad(q, k, v, o, l, blocked(c.dout if dout is None else dout, c.Cb).to(DEV), dq, dk, dv, dt, **m)
    c1(), c2(), c3(), c4()
    return plain(o), l, plain(dq), plain(dk), plain(dv), dt


@pytest.mark.parametrize("bias", [None, "log", "wide"])
@pytest.mark.parametrize("causal", [False, True])
def test_documents_and_positions_wholly_outside(causal, bias):
    """Images whose rows all lie in front of the tokens or behind them, beside others: they see nothing and nothing sees them."""
    first = [300, -1000003, -37, 100, 45, 2 ** 28, -30, 70]
    c = Case(N=8, Sq=30, Sk=100, docs=_docs(8, 100, [[100], [40, 60], [64, 36]]), first=first, heads=4, kv=2, causal=causal, bias=bias)
    c.check()
    out, lse, dq, dk, dv, _ = gradients(c)
    outside = [n for n, f in enumerate(first) if f >= 100 or f + 30 <= 0]
    assert len(outside) == 6
    for t in (out, dq, dk, dv):
        assert bool((t[outside] == 0).all())
    assert bool((lse[outside] == -float("inf")).all())


# ---------------------------------------------------------------------------------------------------- value by value

U = 2.0 ** -24


def exact(c):
    """Results and gradients in 64 bits, each with the sum of the magnitudes that it is made of: {name: (value, magnitudes)}, plain layouts.

    Rounding errors of a sum are in proportion to its terms' magnitudes, so a result is held to (32 + 4 sqrt(K)) u times the sum of these
    (the rule of test_gpu_attention.py, there with the tensor's largest value in their place): what is far larger than a row's own
    terms and hidden from it must not be seen in it. Gradients pass two such chains, so twice that. A weight is off by what its score is: the 32
    holds for scores up to 16 and for those so large that their weights are 0 or 1."""
    N, heads, kv, D, Sq, Sk = c.N, c.heads, c.kv, c.D, c.Sq, c.Sk
    group = heads // kv
    split = lambda t, h: t.double().reshape(N, h, D, -1).transpose(2, 3)  # noqa: E731  [N][h][S][D]
    q, k, v, do = split(c.q, heads), split(c.k, kv), split(c.v, kv), split(c.dout, heads)
    k, v = (t.repeat_interleave(group, 1) for t in (k, v))
    j = torch.arange(Sk)
    first = torch.full((N,), Sk - Sq) if c.first is None else c.first.long()
    p_at = first[:, None] + torch.arange(Sq)
    seen = torch.ones(N, Sq, Sk, dtype=torch.bool)
    if c.lengths is not None:
        seen &= (j < c.lengths[:, None])[:, None]
    if c.causal:
        seen &= (j <= p_at[..., None]) | (j < (torch.zeros(N, 1) if c.prefix is None else c.prefix[:, None]))[:, None]
    if c.docs is not None:
        mine = torch.where((p_at >= 0) & (p_at < Sk), c.docs.long().gather(1, p_at.clamp(0, Sk - 1)), torch.tensor(-1))
        seen &= (c.docs[:, None] == mine[..., None]) & (mine >= 0)[..., None]
    x = c.scale * q @ k.transpose(2, 3)
    size = c.scale * q.abs() @ k.abs().transpose(2, 3)
    slope = 1.0
    if c.cap:
        t = torch.tanh(x / c.cap)
        x, slope = c.cap * t, 1 - t * t
        size = size.clamp(max=c.cap)
    if c.slopes is not None:
        x = x - c.slopes.double()[:, None, None] * (p_at[:, None, :, None] - j).abs()
    at = None
    if c.table is not None:
        code = lambda y: torch.div(y, c.width, rounding_mode="floor") * (2 * c.width - 1) + y % c.width  # noqa: E731
        at = c.bucket.long()[(code(j) - code(p_at)[..., None]).clamp(-c.reach, c.reach) + c.reach]            # [N][Sq][Sk]
        x = x + torch.stack([c.table.double()[:, at[n]] for n in range(N)])
    x = x.masked_fill(~seen[:, None], -float("inf"))
    lse = torch.logsumexp(x, 3)
    p = torch.exp(x - torch.where(lse == -float("inf"), torch.zeros_like(lse), lse)[..., None])
    out, out_size = p @ v, p @ v.abs()
    delta = (do * out).sum(3, keepdim=True)
    ds = p * (do @ v.transpose(2, 3) - delta)
    ds_size = p * (do.abs() @ v.abs().transpose(2, 3) + (do.abs() * out_size).sum(3, keepdim=True))
    fold = lambda t: t.reshape(N, kv, group, Sk, D).sum(2)  # noqa: E731
    join = lambda t: t.transpose(2, 3).reshape(N, -1, t.shape[2])  # noqa: E731
    db = None
    if at is not None:
        db = [torch.zeros_like(c.table, dtype=torch.float64) for _ in range(2)]
        for n in range(N):
            for to, d in zip(db, (ds, ds_size)):
                to.index_add_(1, at[n].reshape(-1), d[n].reshape(heads, -1))
    # (1 - tanh^2 is off by some 4 u whatever it is)
    dx, dx_size = c.scale * ds * slope, c.scale * ds_size * (slope + 0.2 if c.cap else 1.0)
    r = {"out": (join(out), join(out_size)), "lse": (lse, (p * size).sum(3) + lse.abs().nan_to_num(posinf=0.0) + 1),
         "dq": (join(dx @ k), join(dx_size @ k.abs())),
         "dk": (join(fold(dx.transpose(2, 3) @ q)), join(fold(dx_size.transpose(2, 3) @ q.abs()))),
         "dv": (join(fold(p.transpose(2, 3) @ do)), join(fold(p.transpose(2, 3) @ do.abs())))}
    if db:
        r["dtable"] = tuple(db)
    return r


def terms(c, name):
    rows = c.Sq * c.heads // c.kv
    return {"out": c.D + c.Sk, "lse": c.D + c.Sk, "dq": c.D + c.Sk, "dk": c.D + rows, "dv": c.D + rows, "dtable": c.D + c.N * c.Sq}[name]


def compare(c, got, ref, where=None):
    """Value by value; where: {name: mask of what is to be right} (all of it)."""
    for name, t in got.items():
        want, size = ref[name]
        t = t.double().cpu()
        allowed = (32 + 4 * terms(c, name) ** 0.5) * U * (1 if name in ("out", "lse") else 2) * size
        off = (t - want).abs()
        off[(t == want)] = 0.0
        bad = ~(off <= allowed)
        if where is not None and name in where:
            bad &= where[name]
        if bool(bad.any()):
            worst = torch.where(bad, off / allowed.clamp(min=1e-300), torch.zeros_like(off)).nan_to_num(nan=float("inf"))
            i = int(worst.argmax())
            raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} values off, the worst by {float(worst.max()):.2e} of what is allowed: "
                                 f"{float(t.reshape(-1)[i])} for {float(want.reshape(-1)[i])}, place {i}")


def everything(c):
    return dict(zip(("out", "lse", "dq", "dk", "dv") + (("dtable",) if c.table is not None else ()), gradients(c)))


# Shapes of each kernel: fp16 parts (with one workgroup a row tile, with keys split over several, with the forms of their biases), fp32 (gradients: heads of
# more than 128 channels or a reach past 2047), few rows.
SHAPES = {
    "parts": dict(Sq=640, heads=4, D=64), "parts, many rows": dict(Sq=640, heads=24, kv=8, D=32), "parts, odd heads": dict(Sq=700, heads=4, D=37, Cb=37),
    "parts, 128 channels": dict(Sq=500, heads=4, D=128), "parts, distances": dict(Sq=640, heads=4, D=64, slopes=True),
    "parts, capped, buckets": dict(Sq=640, heads=4, kv=2, D=64, cap=10.0, bias="log"), "parts, everything": dict(Sq=640, heads=4, D=48, cap=10.0, bias="log", slopes=True),
    "fp32": dict(Sq=200, heads=2, D=32, bias="wide"), "fp32, wide heads": dict(Sq=150, heads=2, D=200, Cb=8), "small": dict(Sq=100, heads=2, D=16),
}


def causal(S):
    return dict(causal=True)


def documents(S):
    return dict(docs=_docs(1, S, [[S // 3 + 5, S - S // 3 - 5]]))


@pytest.mark.parametrize("big", [1e6, 1e20])
@pytest.mark.parametrize("mask", [causal, documents], ids=["causal", "documents"])
@pytest.mark.parametrize("shape", SHAPES)
def test_large_values_in_hidden_places(shape, mask, big):
    """Finite values far larger than the others, in places that a part of the rows does not see (for queries and dout: whose row does not see a part of
    the keys): in no tensor do they change what does not depend on them. One tensor after another; the others keep their size. (What does depend on a large key or query
    has scores of its size, and is left out.)"""
    S = SHAPES[shape]["Sq"]
    edge = S // 3 + 5                                            # the first row of the second document
    rows = torch.arange(S)
    for name in ("v", "k", "dout", "q"):
        c = Case(**SHAPES[shape], **mask(S))
        # (keys: late tokens of the first document, and of the sequence; rows: early ones of both)
        places = [edge - 2, S - 40] if name in "kv" else [edge - 15, edge + 7]
        if mask is documents and name in "kq":
            places = places[:1]                                  # (one document keeps its size)
        getattr(c, name)[0, :, places] *= big
        where = None
        if name == "k":
            good_rows = rows < places[0] if mask is causal else rows >= edge
            good_keys = torch.zeros(S, dtype=torch.bool) if mask is causal else rows >= edge
            where = {"out": good_rows, "lse": good_rows, "dq": good_rows, "dk": good_keys, "dv": good_keys, "dtable": torch.tensor(False)}
        elif name == "q":
            good_rows = torch.ones(S, dtype=torch.bool)
            good_rows[places] = False
            good_keys = rows > places[-1] if mask is causal else rows >= edge
            where = {"out": good_rows, "lse": good_rows, "dq": good_rows, "dk": good_keys, "dv": good_keys, "dtable": torch.tensor(False)}
        try:
            compare(c, everything(c), exact(c), where)
        except AssertionError as e:
            raise AssertionError(f"{name}: {e}") from None


@pytest.mark.parametrize("whole", [False, True], ids=["some", "tile"])
@pytest.mark.parametrize("mask", [causal, documents], ids=["causal", "documents"])
@pytest.mark.parametrize("shape", SHAPES)
def test_zeros_beside_large_values_in_hidden_places(shape, mask, whole):
    """Tokens of nothing but zeros, which rows see, beside large ones that these rows do not see, a few of each or a whole tile of 64: zeros have no size of their own to
    go by."""
    S = SHAPES[shape]["Sq"]
    edge = S // 3 + 5
    begin = edge // 64 * 64
    low, high = list(range(begin, edge)), list(range(edge, min(begin + 64, S)))
    rows = torch.arange(S)
    for name in ("v", "k", "dout", "q"):
        c = Case(**SHAPES[shape], **mask(S))
        t = getattr(c, name)
        # (of a causal mask's keys the late ones are hidden; of rows, and of documents here, the early ones)
        large, zeros = (high, low) if mask is causal and name in "kv" else (low, high)
        if not whole:
            large, zeros = large[-1:], zeros[::7]
        t[0, :, large] *= 1e20
        t[0, :, zeros] = 0.0
        where = None
        if name in "kq":
            good = rows >= edge if mask is documents else rows < large[0] if name == "k" else rows > large[-1]
            none = torch.zeros(S, dtype=torch.bool)
            out = good if name == "k" else torch.tensor([int(i) not in large for i in rows])
            keys = good if mask is documents else none if name == "k" else good
            where = {"out": out, "lse": out, "dq": out, "dk": keys, "dv": keys, "dtable": torch.tensor(False)}
        try:
            compare(c, everything(c), exact(c), where)
        except AssertionError as e:
            raise AssertionError(f"{name}: {e}") from None


@pytest.mark.parametrize("step", [1.0, 20.0])
@pytest.mark.parametrize("shape", ["parts", "parts, many rows", "parts, capped, buckets", "fp32"])
def test_magnitudes_that_rise_along_a_sequence(shape, step):
    """Values and dout that double every `step` tokens: early rows see small values only, late keys only small rows."""
    S = SHAPES[shape]["Sq"]
    c = Case(**SHAPES[shape], causal=True)
    rise = 2.0 ** (torch.arange(S) / step).floor().clamp(max=60)
    c.v, c.dout = c.v * rise, c.dout * rise.flip(0)
    compare(c, everything(c), exact(c))


@pytest.mark.parametrize("Sq,Sk", [(300, 3100), (64, 4000), (1, 3000)])
def test_large_values_in_hidden_places_of_long_caches(Sq, Sk):
    """Rows whose keys are split over workgroups, and single tokens."""
    for name in ("v", "k"):
        c = Case(N=2, Sq=Sq, Sk=Sk, heads=4, D=64, docs=_docs(2, Sk, [[1500, Sk - 1500], [Sk - 5, 5]]))
        getattr(c, name)[:, :, [10, 1499, Sk - 7]] *= 1e20
        got = c.forward()
        where = None
        if name == "k":                                          # (rows that see none of these)
            at = Sk - Sq + torch.arange(Sq)
            good = torch.stack([torch.zeros(Sq, dtype=torch.bool), at >= Sk - 5])[:, None].expand(2, 1, Sq)
            where = {"out": good, "lse": good}
        compare(c, {"out": plain(got[0]), "lse": got[1]}, exact(c), where)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_nan_and_infinities_in_hidden_places(shape, value):
    """Tokens and rows that hold NaN or infinities: results and gradients of rows that do not see such a token are what they are without it, and so are the gradients of
    keys that no such row sees; those that do see it are not finite."""
    S = SHAPES[shape]["Sq"]
    at = S // 3 + 12                                             # the second document's; rows of the first do not see it, nor does that row see its keys
    for mask in (causal, documents):
        ref = exact(Case(**SHAPES[shape], **mask(S)))
        for name in ("k", "v", "q", "dout"):
            c = Case(**SHAPES[shape], **mask(S))
            getattr(c, name)[0, 3, at] = value
            got = everything(c)
            got.pop("dtable", None)
            keys = name in "kv"
            rows_ok, keys_ok = (torch.zeros(S, dtype=torch.bool) for _ in range(2))
            if mask is causal:
                rows_ok[:at if keys else S] = True
                if not keys:
                    rows_ok[at] = False
                keys_ok[at + 1:] = not keys                      # (keys up to `at` are seen by a row that sees it, or by the row that holds it)
            else:
                keys_ok[:S // 3 + 5] = True
                rows_ok[:S // 3 + 5 if keys else S] = True
                if not keys:
                    rows_ok[at] = False
            forward = rows_ok if name != "dout" else torch.ones_like(rows_ok)
            where = {"out": forward, "lse": forward, "dq": rows_ok, "dk": keys_ok, "dv": keys_ok}
            try:
                compare(c, got, ref, where)
            except AssertionError as e:
                raise AssertionError(f"{name}, {mask.__name__}: {e}") from None
            if name != "v":
                assert not bool(torch.isfinite(got["dk"][0, :c.D, at if keys else at - 1]).any()), name
            if name in "kv":
                assert not bool(torch.isfinite(got["dq"][0, :c.D, at + 1]).any()), name
            if name == "dout":
                assert not bool(torch.isfinite(got["dv"][0, 3, at - 1])), name


@pytest.mark.parametrize("shape", SHAPES)
def test_what_stands_past_lengths_reaches_no_gradient(shape):
    S = SHAPES[shape]["Sq"]
    for length in (S - 7, S // 2, 1):
        c = Case(**SHAPES[shape], lengths=[length])
        ref = exact(c)
        c.k[0, :, length:], c.v[0, :, length:] = float("nan"), float("inf")
        got = everything(c)
        compare(c, got, ref)
        assert bool((got["dk"][:, :, length:] == 0).all()) and bool((got["dv"][:, :, length:] == 0).all())


# ---------------------------------------------------------------------------------------------------- biases

def with_offsets(c, reach, buckets=None):
    """The case with a table over offsets -reach .. reach: each its own bucket, or `buckets` in turn."""
    size = 2 * reach + 1
    c.reach, c.width, c.buckets = reach, 1, buckets or size
    c.bucket = (torch.arange(size) % c.buckets).int()
    c.table = torch.randn(c.heads, c.buckets, generator=torch.Generator().manual_seed(3))
    c.masks.update(table=c.table, bucket=c.bucket)
    return c


@pytest.mark.parametrize("D", [96, 97, 100, 128])
@pytest.mark.parametrize("reach", [1599, 1612, 1640, 2047])
def test_wide_tables_of_wide_heads(D, reach):
    """Tables whose sums by offset are about all that a workgroup's LDS holds beside tiles of as many channels, and more than that."""
    c = with_offsets(Case(Sq=130, heads=2, D=D, Cb=D, causal=True), reach, 64)
    compare(c, everything(c), exact(c))


@pytest.mark.parametrize("side", [29, 32])
def test_pixels_of_wide_heads(side):
    c = Case(Sq=side * side, heads=1, D=128, bias=(side, side))
    compare(c, everything(c), exact(c))


@pytest.mark.parametrize("D", [16, 48, 160])
def test_table_gradient_of_rows_far_behind_the_keys_they_see(D):
    """As test_rows_far_behind_the_keys_they_see (whose bound this is), the table's gradient beside distances: a bucket for every offset, so that what rounding
    leaves of a row's lse does not cancel within one."""
    S = 400
    c = with_offsets(Case(N=2, Sq=S, heads=2, D=D, lengths=[2, 7], slopes=True), S - 1)
    want = exact(c)["dtable"][0]
    off = gradients(c)[5].double().cpu() - want
    assert float(off.norm()) <= 2e-6 * float(want.norm())


@pytest.mark.parametrize("big", [1e9, 1e20])
@pytest.mark.parametrize("shape", ["parts", "parts, many rows", "parts, distances", "parts, everything", "fp32", "fp32, wide heads", "small"])
def test_large_scores_that_are_seen(shape, big):
    """A few keys far larger than the others, which rows do see: their scores are so far apart that a row's weights are 0 or 1 (or theirs are 0 and the
    others' what they are without them). Forward calls; a score's rounding, which is that of its size, must not become a weight."""
    S = SHAPES[shape]["Sq"]
    c = Case(**SHAPES[shape], causal=True)
    c.k[0, :, [5, S // 2, S // 2 + 1, S - 40]] *= torch.tensor([1.0, 3.0, 0.5, 2.0]) * big
    o, l = c.forward()
    compare(c, {"out": plain(o), "lse": l}, exact(c))


@pytest.mark.parametrize("Sk", [33, 900, 5000])
def test_large_scores_that_single_tokens_see(Sk):
    c = Case(N=3, Sq=1, Sk=Sk, heads=8, kv=2, D=32)
    c.k[:, :, [3, 17, Sk - 2]] *= torch.tensor([1.0, 3.0, 0.5]) * 1e20
    o, l = c.forward()
    compare(c, {"out": plain(o), "lse": l}, exact(c))
