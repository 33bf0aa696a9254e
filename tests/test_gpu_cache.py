"""The paged cache on the GPU: what it stores bit for bit against its definition, what it reads back, what stays untouched, and attention over it in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2303_04769_amd as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["float32", "bfloat16", "int8"]


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def tokens_of(t, heads):
    """[N][C/Cb][S][Cb] -> [N][S][heads][D] on the host"""
    t = t.detach().cpu()
    return t.permute(0, 2, 1, 3).reshape(t.shape[0], t.shape[2], heads, -1)


def codes_of(x):
    """Codes and scales of float32 tokens [..][D], by the definition, each operation rounded to fp32."""
    x = x.numpy()
    top = np.abs(x).max(-1)
    with np.errstate(all="ignore"):
        scale, by = (top / np.float32(127)).astype(np.float32), (np.float32(127) / top).astype(np.float32)
        code = np.rint((x * by[..., None]).astype(np.float32))
    none = ~np.isfinite(top)
    scale = np.where(none, np.float32(np.nan), np.where(top < np.float32(2.0 ** -100), np.float32(0), scale))
    code = np.where((none | (top < np.float32(2.0 ** -100)))[..., None], 0, code)
    return torch.from_numpy(code.astype(np.int8)), torch.from_numpy(scale.astype(np.float32))


def stored(x, kind):
    """What a cache has of float32 tokens: (elements, scales or None)."""
    return codes_of(x) if kind == "int8" else (x.to(torch.bfloat16 if kind == "bfloat16" else torch.float32), None)


def held(x, kind):
    """What it gives back for them."""
    e, s = stored(x, kind)
    return e.float() * s[..., None] if kind == "int8" else e.float()


def table_for(N, per, pages, seed=0):
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:N * per]
    return order.reshape(N, per).to(torch.int32).to(DEV)


def garbage(cache):
    """Fills a cache's memory with what nothing may depend on (keys behind D stay zero)."""
    for t in (cache.keys[..., :cache.D], cache.values):
        t.fill_(77 if t.dtype == torch.int8 else math.nan)
    for t in (cache.key_scales, cache.value_scales):
        if t is not None:
            t.fill_(math.nan)


FORMS = [
    # N, S, kv, D, Cb, page, per_stream, first, counts
    (1, 1, 1, 4, 4, 16, 1, None, None),
    (3, 1, 2, 64, 64, 32, 4, [0, 31, 127], None),
    (3, 2, 2, 64, 16, 16, 3, [15, 0, 46], [2, 0, 1]),
    (2, 5, 1, 40, 8, 16, 2, [3, 14], None),
    (2, 48, 3, 16, 48, 16, 4, None, None),
    (3, 61, 2, 32, 16, 64, 2, [0, 7, 70], [61, 13, 58]),
    (2, 100, 1, 10, 5, 32, 5, [1, 60], [100, 1]),
    (2, 33, 2, 7, 7, 16, 4, [5, 0], None),
    (1, 300, 2, 128, 16, 128, 3, [40], None),
    (2, 40, 1, 256, 256, 256, 1, [200, 3], [40, 99]),
    (4, 17, 5, 80, 400, 16, 3, [-3, 44, 16, 1 << 29], [17, 17, -5, 17]),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
def test_write_and_read(form, kind):
    N, T, kv, D, Cb, page, per, first, counts = form
    nk = kv * D // Cb
    pages = N * per + 2
    cache = S.PagedCache(pages, page, kv, D, kind=kind)
    garbage(cache)
    before = [t if t is None else t.cpu().clone() for t in (cache.keys, cache.values, cache.key_scales, cache.value_scales)]
    k, v = rand(1, N, nk, T, Cb) * 3, rand(2, N, nk, T, Cb)
    k[0, :, 0] *= 1e-33                                       # (whose codes are zero)
    table = table_for(N, per, pages)
    starts = [0] * N if first is None else first
    many = [T] * N if counts is None else [max(0, min(c, T)) for c in counts]
    first, counts = (x if x is None else ints(x) for x in (first, counts))
    cache.write(k.to(DEV), v.to(DEV), table, first, counts=counts)
    rows = [t if t is None else t.cpu() for t in (cache.keys, cache.values, cache.key_scales, cache.value_scales)]
    kt, vt = tokens_of(k, kv), tokens_of(v, kv)
    (ke, ks), (ve, vs) = stored(kt, kind), stored(vt, kind)
    want = [t if t is None else t.clone() for t in before]
    ko, vo = torch.full((N, T, kv, D), 5.0), torch.full((N, T, kv, D), 5.0)
    for n in range(N):
        for i in range(many[n]):
            p = starts[n] + i
            if not 0 <= p < per * page:
                continue
            at, place = int(table[n, p // page]), p % page
            want[0][at, :, place] = 0
            want[0][at, :, place, :D], want[1][at, :, :, place] = ke[n, i], ve[n, i]
            if kind == "int8":
                want[2][at, :, place], want[3][at, :, place] = ks[n, i], vs[n, i]
            ko[n, i], vo[n, i] = held(kt[n, i], kind), held(vt[n, i], kind)
    bits = {torch.float32: torch.int32, torch.bfloat16: torch.int16, torch.int8: torch.int8}
    for name, x, y in zip(("keys", "values", "key_scales", "value_scales"), rows, want):
        if x is not None:
            nan = torch.isnan(y.float())
            assert torch.equal(torch.isnan(x.float()), nan), name
            assert torch.equal(x.view(bits[x.dtype])[~nan], y.view(bits[y.dtype])[~nan]), name
    back = [torch.full((N, nk, T, Cb), 5.0, device=DEV) for _ in range(2)]
    cache.read(*back, table, first, counts=counts)
    assert torch.equal(tokens_of(back[0], kv), ko) and torch.equal(tokens_of(back[1], kv), vo)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,halves,F,D,Cb,pairs", [(1, True, 1, 64, 64, 32), (1, False, 2, 16, 16, 4), (40, True, 2, 40, 8, 20), (40, True, 1, 64, 16, 10), (35, False, 1, 32, 16, 16),
                                                   (20, False, 2, 10, 10, 3), (20, True, 1, 6, 3, 3)])
def test_turned_on_the_way(T, halves, F, D, Cb, pairs, kind):
    """Keys that a write turns have the bits of keys that were turned before it, queries too."""
    N, heads, kv, page, per = 3, 4, 2, 16, 8
    q, k, v = rand(1, N, heads * D // Cb, T, Cb).to(DEV), rand(2, N, kv * D // Cb, T, Cb).to(DEV), rand(3, N, kv * D // Cb, T, Cb).to(DEV)
    freq, first, counts = rand(4, F, 1, pairs).to(DEV), ints([0, 9, 70]), ints([T, T, max(0, T - 7)])
    table = table_for(N, per, N * per)
    plan = S.Rotary(N, T, heads, kv, D, pairs=pairs, halves=halves, freq_heads=F, Cb=Cb)
    a, b = (S.PagedCache(N * per, page, kv, D, kind=kind) for _ in range(2))
    q1, q2, k2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(k)
    a.write(k, v, table, first, counts=counts, rotary=plan, freq=freq, q=q, q_out=q1)
    plan.run(q, k, freq, q2, k2, first=first)
    b.write(k2, v, table, first, counts=counts)
    assert torch.equal(q1, q2)
    for x, y in zip((a.keys, a.values, a.key_scales, a.value_scales), (b.keys, b.values, b.key_scales, b.value_scales)):
        assert x is None or torch.equal(x, y)
    again = q.clone()
    a.write(k, v, table, first, counts=counts, rotary=plan, freq=freq, q=again)                 # in place
    assert torch.equal(again, q1)
    a.write(k, v, table, first, counts=counts, rotary=plan, freq=freq)                          # keys alone
    assert torch.equal(a.keys, b.keys)
    places = (first[:, None] + torch.arange(T, device=DEV))[..., None].int().contiguous()       # places of the program's own
    c = S.PagedCache(N * per, page, kv, D, kind=kind)
    c.write(k, v, table, first, counts=counts, rotary=plan, freq=freq, positions=places, q=q, q_out=again)
    assert torch.equal(c.keys, b.keys) and torch.equal(again, q1)


@pytest.mark.parametrize("T", [1, 20])
def test_non_finite_tokens_and_extreme_scales(T):
    N, kv, D, page = 1, 2, 16, 16
    cache = S.PagedCache(4, page, kv, D)
    k = rand(0, N, kv, T, D)
    v = k.clone()
    k[0, 0, 0, 3], k[0, 1, T - 1, 2] = math.nan, -math.inf
    v[0, 0, 0] = 3.4e38
    v[0, 1, 0] = 0.0
    v[0, 1, 0, 5] = 2.0 ** -100
    table = ints([[2, 0]])
    cache.write(k.to(DEV), v.to(DEV), table)
    ko, vo = (torch.empty(N, kv, T, D, device=DEV) for _ in range(2))
    cache.read(ko, vo, table)
    for x, y in ((k, ko), (v, vo)):
        want = held(tokens_of(x, kv), "int8")
        assert torch.equal(torch.isnan(tokens_of(y, kv)), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(tokens_of(y, kv)), torch.nan_to_num(want))
    assert torch.isnan(ko[0, 0, 0]).all() and torch.isnan(ko[0, 1, T - 1]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1, 40])
def test_pages_that_are_none(kind, T):
    """Numbers outside the pool: nothing is written, nothing read."""
    N, kv, D, page = 2, 2, 32, 16
    cache = S.PagedCache(5, page, kv, D, kind=kind)
    k = rand(0, N, kv, T, D).to(DEV)
    for bad in (-1, 5, 1 << 30, -(1 << 31)):
        cache.keys.zero_()
        cache.values.zero_()
        table = ints([[1, bad, 2], [bad, bad, bad]])
        cache.write(k, k, table)
        out = torch.full_like(k, 9.0)
        cache.read(out, torch.empty_like(k), table)
        want = tokens_of(out, kv)
        seen = torch.zeros(N, T, dtype=torch.bool)
        seen[0, :16] = True
        seen[0, 32:] = True
        assert bool((want[~seen] == 9.0).all()) and torch.equal(want[seen], held(tokens_of(k, kv)[seen], kind))
        assert not cache.keys[[0, 3, 4]].any() and not cache.values[[0, 3, 4]].any()


# ---------------------------------------------------------------------------------------------------- attention

def attend(q, k, v, lengths, first, scale, cap=0.0, slopes=None, table=None, bucket=None, reach=0):
    """In 64 bits: q [N][Sq][heads][D], k, v [N][room][kv][D] -> out, lse [N][heads][Sq], and the largest sum of absolute products of a score that counts."""
    N, Sq, heads, D = q.shape
    kv = k.shape[2]
    group = heads // kv
    out, lse, size = torch.zeros(N, Sq, heads, D, dtype=torch.float64), torch.full((N, heads, Sq), -math.inf, dtype=torch.float64), 0.0
    for n in range(N):
        L = max(0, min(int(lengths[n]), k.shape[1]))
        at = (L - Sq if first is None else int(first[n])) + torch.arange(Sq)
        j = torch.arange(L)
        for h in range(heads):
            kk, vv = k[n, :L, h // group].double(), v[n, :L, h // group].double()
            for i in range(Sq):
                seen = j <= at[i]
                qq = q[n, i, h].double()
                s = scale * (kk @ qq)
                if cap:
                    s = cap * torch.tanh(s / cap)
                if slopes is not None:
                    s = s - float(slopes[h]) * (at[i] - j).abs()
                if table is not None:
                    b = table[h].double()[bucket.long()[(j - at[i]).clamp(-reach, reach) + reach]]
                    s = s + torch.where(b < -1e30, -math.inf, b)
                seen = seen & (s != -math.inf)
                if not bool(seen.any()):
                    continue
                s, vs = s[seen], vv[seen]
                l = torch.logsumexp(s, 0)
                lse[n, h, i] = l
                out[n, i, h] = torch.exp(s - l) @ vs
                size = max(size, float(scale * (kk[seen].abs() @ qq.abs()).max()), float(s.abs().max()))
    return out, lse, size


def check_attention(got, lse, ref, ref_lse, size, D, room, v):
    """A score is a sum of D products and a few terms, each rounded to 24 bits: off by (D + 16) 2^-24 of its products' sum. Weights are off by that, twice with their sum's,
    and sums over keys by 2^-24 for every addition one after the other -- a lane's of each eighth key at most, and joins."""
    ds = (D + 16) * 2.0 ** -24 * size
    sums = (room / 8 + 64) * 2.0 ** -24
    assert torch.isfinite(got).all()
    assert float((got.double() - ref).abs().max()) <= (2 * ds + 2 * sums) * float(v.abs().max()), float((got.double() - ref).abs().max())
    fine = torch.isfinite(ref_lse)
    assert torch.equal(lse.cpu()[~fine].double(), ref_lse[~fine])
    assert float((lse.cpu().double() - ref_lse)[fine].abs().max()) <= ds + sums + 2.0 ** -22 * (1 + float(ref_lse[fine].abs().max()))


def buckets_of(reach, buckets):
    bucket, buckets, reach = S.log_buckets(reach, buckets, both=False)
    return bucket.to(DEV), buckets, reach


ATTENTION = [
    # N, Sq, heads, kv, D, Cb, page, per, lengths, first, bias, cap
    (1, 1, 1, 1, 4, 4, 16, 1, [1], None, "none", 0.0),
    (4, 1, 8, 8, 32, 32, 16, 5, [0, 1, 16, 80], None, "none", 0.0),
    (4, 1, 8, 2, 64, 16, 32, 8, [255, 256, 17, 64], None, "slopes", 30.0),
    (3, 1, 4, 2, 16, 16, 64, 3, [63, 64, 65], None, "buckets", 0.0),
    (2, 5, 4, 1, 40, 8, 16, 9, [144, 3], None, "none", 0.0),
    (2, 3, 8, 8, 80, 16, 128, 3, [384, 130], None, "slopes", 0.0),
    (2, 7, 10, 2, 48, 480, 16, 20, [320, 99], None, "buckets", 15.0),         # 35 rows: three tiles of them
    (2, 2, 6, 3, 96, 96, 32, 6, [100, 192], [40, 190], "none", 0.0),           # places of the program's own
    (1, 1, 32, 1, 128, 128, 256, 2, [500], None, "none", 50.0),
    (2, 1, 4, 2, 256, 16, 16, 30, [479, 100], None, "buckets", 0.0),
    (2, 1, 3, 1, 7, 21, 16, 4, [64, 33], None, "none", 0.0),                   # nothing aligned
    (1, 1, 4, 4, 64, 64, 64, 80, [5000], None, "slopes", 0.0),                 # split over workgroups
    (2, 2, 5, 5, 10, 5, 32, 40, [1280, 1111], [5, 1200], "buckets", 0.0),
]


def attention_setup(form, kind, seed=0):
    N, Sq, heads, kv, D, Cb, page, per, lengths, first, bias, cap = form
    pages = N * per + 1
    cache = S.PagedCache(pages, page, kv, D, kind=kind)
    garbage(cache)
    room = per * page
    k, v = rand(seed + 1, N, kv, room, D), rand(seed + 2, N, kv, room, D)
    table = table_for(N, per, pages, seed)
    cache.write(k.to(DEV), v.to(DEV), table, counts=ints(lengths))              # (behind the lengths: garbage)
    for n, held_ in enumerate(lengths):
        table[n, -(-held_ // page):] = -7
    q = rand(seed + 3, N, -(-heads * D // Cb), Sq, Cb)
    more = {}
    reach = buckets = 0
    if bias == "slopes":
        more["slopes"] = torch.tensor([2.0 ** (-8 * (h + 1) / heads) for h in range(heads)], device=DEV)
    elif bias == "buckets":
        more["bucket"], buckets, reach = buckets_of(64, 12)
        more["table"] = rand(seed + 4, heads, buckets).to(DEV)
    plan = S.CacheAttention(cache, N, Sq, heads, per, Cb=Cb, cap=cap, reach=reach, buckets=buckets)
    return cache, table, q, held(tokens_of(k, kv), kind), held(tokens_of(v, kv), kind), more, reach, plan


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", ATTENTION)
def test_attention(form, kind):
    N, Sq, heads, kv, D, Cb, page, per, lengths, first, bias, cap = form
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    out, lse = torch.full(q.shape, math.nan, device=DEV), torch.full((N, heads, Sq), math.nan, device=DEV)
    plan.run(q.to(DEV), out, table, ints(lengths), lse=lse, first=None if first is None else ints(first), **more)
    host = {n: t.cpu() for n, t in more.items()}
    ref, ref_lse, size = attend(tokens_of(q, heads), k, v, lengths, first, D ** -0.5, cap, host.get("slopes"), host.get("table"), host.get("bucket"), reach)
    check_attention(tokens_of(out, heads), lse, ref, ref_lse, size, D, per * page, v)
    again = torch.empty_like(out)
    plan.run(q.to(DEV), again, table, ints(lengths), first=None if first is None else ints(first), **more)       # without lse: the same bits
    assert torch.equal(out, again)


MANY_ROWS = [
    # N, Sq, heads, kv, D, Cb, page, per, lengths, first, bias, cap: 17 rows of a key head and more
    (2, 17, 1, 1, 16, 16, 16, 9, [144, 11], None, "none", 0.0),
    (2, 5, 8, 2, 64, 16, 32, 8, [250, 3], None, "slopes", 30.0),
    (1, 33, 1, 1, 32, 32, 16, 6, [90], None, "buckets", 0.0),
    (2, 11, 6, 2, 64, 384, 64, 5, [320, 7], None, "buckets", 0.0),
    (2, 9, 8, 2, 80, 16, 16, 13, [208, 100], [150, 40], "slopes", 0.0),
    (1, 16, 8, 2, 96, 96, 64, 9, [576], None, "none", 15.0),
    (2, 40, 3, 3, 128, 128, 32, 8, [256, 50], None, "slopes", 0.0),
    (1, 7, 8, 1, 120, 8, 16, 60, [951], None, "buckets", 20.0),
    (1, 50, 1, 1, 256, 256, 16, 5, [75], None, "none", 0.0),
    (3, 7, 16, 2, 40, 8, 64, 90, [5760, 0, 4001], None, "slopes", 0.0),
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", MANY_ROWS)
def test_many_rows(form, kind):
    test_attention(form, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_many_rows_around_an_infinite_value(kind, D):
    """The third token from the end holds an infinite value: rows that do not see it, in both tiles of a unit, have the results of a cache without it."""
    form = (2, 9, 8, 2, D, 16, 16, 8, [128, 61], None, "none", 0.0)
    N, Sq, heads, kv, D, Cb, page, per, lengths, *_ = form
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    out = torch.empty(q.shape, device=DEV)
    plan.run(q.to(DEV), out, table, ints(lengths))
    clean = tokens_of(out, heads)
    one_k, one_v = rand(8, N, kv, 1, D), torch.full((N, kv, 1, D), math.inf)
    cache.write(one_k.to(DEV), one_v.to(DEV), table, first=ints([x - 3 for x in lengths]))
    plan.run(q.to(DEV), out, table, ints(lengths))
    got = tokens_of(out, heads)
    assert not torch.isfinite(got[:, Sq - 3:]).any()
    # (in another order: sums of up to 128 weights below 1 and their products, each rounded to 24 bits, on both sides)
    assert float((got - clean)[:, : Sq - 3].abs().max()) <= 2 * (D + 16 + 2 * 128) * 2.0 ** -24 * max(1.0, D ** 0.5) * float(v.abs().max())


@pytest.mark.parametrize("kind", KINDS)
def test_hidden_tokens_reach_no_row(kind):
    """A token that holds NaN and infinities, seen by the later of three new tokens only; pages of another stream's that hold them too."""
    form = (2, 3, 4, 2, 32, 32, 16, 6, [90, 70], None, "none", 0.0)
    N, Sq, heads, kv, D, Cb, page, per, lengths, *_ = form
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    out = torch.empty(q.shape, device=DEV)
    plan.run(q.to(DEV), out, table, ints(lengths))
    clean = out.clone()
    at, place = int(table[0, 89 // 16]), 89 % 16
    if kind == "int8":
        cache.value_scales[at, :, place], cache.key_scales[at, :, place] = math.inf, math.nan
    else:
        cache.values[at, :, 3:9, place], cache.values[at, :, 1, place], cache.keys[at, :, place, 0] = math.nan, math.inf, math.inf
    plan.run(q.to(DEV), out, table, ints(lengths))
    got, want = tokens_of(out, heads), tokens_of(clean, heads)
    assert torch.equal(got[1], want[1])                        # the other stream
    assert float((got[0, :2] - want[0, :2]).abs().max()) <= 2.0 ** -18 * float(v.abs().max())      # (key by key: another order of 90 sums)
    assert torch.isnan(got[0, 2]).any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Sq,heads,D,page,bias", [(1, 4, 32, 16, "none"), (1, 16, 64, 64, "slopes"), (5, 8, 32, 64, "none"), (9, 8, 64, 32, "buckets")])
def test_capped_scores_beside_memory_of_no_token(Sq, heads, D, page, bias, kind):
    """With a cap the same bits, whatever stands behind a stream's length in its last page and in the page that stands in for one that is none: nothing, or keys whose scores are far
    larger than any that count, where another way to compute the cap would be chosen."""
    N, kv, per = 3, 2, 9
    lengths = [Sq + 3, 5 * page + 7, 9 * page - 2]
    form = (N, Sq, heads, kv, D, D, page, per, lengths, None, bias, 30.0)
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    table[1, 3] = -1
    free = next(p for p in range(1, cache.pages) if not bool((table == p).any()))
    for t in (cache.keys, cache.values, cache.key_scales, cache.value_scales):
        if t is not None:
            t[free] = t[0]
    table[table == 0] = free                                   # (page 0 is nobody's: it is read where there is no page)
    rows, outs = table.cpu(), []
    for fill in (0, 100):
        for n, held_ in enumerate(lengths):
            at, place = int(rows[n, held_ // page]), held_ % page
            cache.keys[at, :, place:, :D], cache.values[at, :, :, place:] = fill, fill
            if kind == "int8":
                cache.key_scales[at, :, place:], cache.value_scales[at, :, place:] = 1.0, 1.0
        cache.keys[0, ..., :D], cache.values[0] = fill, fill
        if kind == "int8":
            cache.key_scales[0], cache.value_scales[0] = 1.0, 1.0
        out, lse = torch.empty(q.shape, device=DEV), torch.empty(N, heads, Sq, device=DEV)
        plan.run(q.to(DEV), out, table, ints(lengths), lse=lse, **more)
        outs.append((out, lse))
    assert torch.isfinite(outs[0][0]).all()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@pytest.mark.parametrize("kind", KINDS)
def test_biases_that_hide(kind):
    """A learned bias of the type's lowest value hides its offsets, all of them a whole row."""
    form = (2, 1, 4, 2, 16, 16, 16, 8, [100, 128], None, "buckets", 0.0)
    N, Sq, heads, kv, D, Cb, page, per, lengths, *_ = form
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    more["table"][0] = -math.inf
    more["table"][1, :6] = torch.finfo(torch.float32).min
    out, lse = torch.empty(q.shape, device=DEV), torch.empty(N, heads, Sq, device=DEV)
    plan.run(q.to(DEV), out, table, ints(lengths), lse=lse, **more)
    ref, ref_lse, size = attend(tokens_of(q, heads), k, v, lengths, None, D ** -0.5, 0.0, None, more["table"].cpu(), more["bucket"].cpu(), reach)
    assert bool((ref_lse[:, 0] == -math.inf).all())
    check_attention(tokens_of(out, heads), lse, ref, ref_lse, size, D, per * page, v)


@pytest.mark.parametrize("kind", KINDS)
def test_pages_that_are_none_are_not_seen(kind):
    form = (2, 1, 4, 2, 64, 64, 16, 12, [180, 192], None, "none", 0.0)
    N, Sq, heads, kv, D, Cb, page, per, lengths, *_ = form
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    cache.values[0], cache.keys[0] = (77, 77) if kind == "int8" else (math.nan, math.nan)
    if kind == "int8":
        cache.value_scales[0] = math.nan
    table[table == 0] = -1
    gone = [[5], [0, 11]]
    for n, which in enumerate(gone):
        for p in which:
            table[n, p] = (-1, 1 << 30)[n]
    rows = table.cpu()
    out, lse = torch.empty(q.shape, device=DEV), torch.empty(N, heads, Sq, device=DEV)
    plan.run(q.to(DEV), out, table, ints(lengths), lse=lse)
    # the same as a bias of minus infinity on those tokens
    ref = torch.zeros(N, Sq, heads, D, dtype=torch.float64)
    for n in range(N):
        there = torch.tensor([0 <= int(rows[n, j // page]) < cache.pages for j in range(lengths[n])])
        for h in range(heads):
            s = D ** -0.5 * (k[n, :lengths[n], h // 2].double() @ tokens_of(q, heads)[n, 0, h].double())
            ref[n, 0, h] = torch.softmax(s[there], 0) @ v[n, :lengths[n], h // 2].double()[there]
    assert float((tokens_of(out, heads).double() - ref).abs().max()) <= 2 * (D + 100) * 2.0 ** -24 * 20 * float(v.abs().max())


@pytest.mark.parametrize("kind", KINDS)
def test_large_and_small_tokens_beside_each_other(kind):
    """Values of one token 2^40 times its neighbours', weights that make up for it: what counts keeps its precision."""
    N, kv, D, page, per = 1, 1, 32, 16, 4
    cache = S.PagedCache(per, page, kv, D, kind=kind)
    k, v = rand(0, N, kv, 64, D), rand(1, N, kv, 64, D)
    k[0, 0, :, 0] = 0
    k[0, 0, 20, 0] = -50.0                                     # a weight near 2^-72 with q[0] = 1 and scale 1 ...
    v[0, 0, 20] *= 2.0 ** 60                                   # ... of values as large
    q = torch.zeros(N, 1, 1, D)
    q[..., 0] = 1.0
    table = ints([[3, 1, 0, 2]])
    cache.write(k.to(DEV), v.to(DEV), table)
    out = torch.empty(N, 1, 1, D, device=DEV)
    S.CacheAttention(cache, N, 1, 1, per, Cb=D, scale=1.0).run(q.to(DEV), out, table, ints([64]))
    ref, _, size = attend(tokens_of(q, 1), held(tokens_of(k, kv), kind), held(tokens_of(v, kv), kind), [64], None, 1.0)
    others = float(v[0, 0, :16].abs().max())
    assert float((tokens_of(out, 1).double() - ref).abs().max()) <= 2.0 ** -17 * max(others, float(ref.abs().max()))


@pytest.mark.parametrize("kind,N,D", [("float32", 300, 8), ("int8", 700, 16), ("bfloat16", 150, 136), ("int8", 257, 256)])
def test_many_streams(kind, N, D):
    """More streams than a workgroup has threads, of all lengths from none on."""
    heads, kv, page, per = 2, 1, 16, 10
    lengths = [(37 * n) % 161 for n in range(N)]
    pages = sum(-(-x // page) for x in lengths) + 1
    cache = S.PagedCache(pages, page, kv, D, kind=kind)
    garbage(cache)
    k, v, q = rand(1, N, kv, per * page, D), rand(2, N, kv, per * page, D), rand(3, N, heads, 1, D)
    table, at = torch.full((N, per), -1, dtype=torch.int32), 0
    for n, x in enumerate(lengths):
        table[n, :-(-x // page)] = torch.arange(at, at + -(-x // page))
        at += -(-x // page)
    table = table.to(DEV)
    cache.write(k.to(DEV), v.to(DEV), table, counts=ints(lengths))
    out, lse = torch.full((N, heads, 1, D), math.nan, device=DEV), torch.full((N, heads, 1), math.nan, device=DEV)
    S.CacheAttention(cache, N, 1, heads, per, Cb=D).run(q.to(DEV), out, table, ints(lengths), lse=lse)
    kh, vh = held(tokens_of(k, kv), kind), held(tokens_of(v, kv), kind)
    ref, ref_lse, size = attend(tokens_of(q, heads), kh, vh, lengths, None, D ** -0.5)
    check_attention(tokens_of(out, heads), lse, ref, ref_lse, size, D, per * page, v)


@pytest.mark.parametrize("kind,rounds,keys", [("float32", 100, 64), ("float32", 160, 64), ("bfloat16", 70, 128), ("bfloat16", 140, 128), ("int8", 70, 256)])
def test_shares_of_a_few_rounds(kind, rounds, keys):
    """Streams whose tokens are two to four times what all workgroups take at once: shared out in pieces that end with a stream's, or -- 140 -- in equal shares that do not."""
    N, Sq, heads, kv, D, page = 12, 3, 2, 2, 128, 64
    per = rounds * keys // page
    lengths = [min(rounds * keys, x) for x in [0, 1, rounds * keys, keys + 1] + [rounds * keys * (n + 2) // 10 - 7 * n for n in range(8)]]
    pages = sum(-(-x // page) for x in lengths) + 1
    cache = S.PagedCache(pages, page, kv, D, kind=kind)
    garbage(cache)
    k, v, q = rand(1, N, kv, per * page, D), rand(2, N, kv, per * page, D), rand(3, N, heads, Sq, D)
    table, at = torch.full((N, per), -1, dtype=torch.int32), 0
    for n, x in enumerate(lengths):
        table[n, :-(-x // page)] = torch.arange(at, at + -(-x // page)).flip(0)
        at += -(-x // page)
    table = table.to(DEV)
    cache.write(k.to(DEV), v.to(DEV), table, counts=ints(lengths))
    out, lse = torch.full((N, heads, Sq, D), math.nan, device=DEV), torch.full((N, heads, Sq), math.nan, device=DEV)
    plan = S.CacheAttention(cache, N, Sq, heads, per, Cb=D)
    plan.run(q.to(DEV), out, table, ints(lengths), lse=lse)
    ref, ref_lse, size = attend(tokens_of(q, heads), held(tokens_of(k, kv), kind), held(tokens_of(v, kv), kind), lengths, None, D ** -0.5)
    check_attention(tokens_of(out, heads), lse, ref, ref_lse, size, D, per * page, v)
    again = torch.empty_like(out)
    plan.run(q.to(DEV), again, table, ints(lengths))
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", KINDS)
def test_queries_that_are_not_finite(kind):
    """... have no result but NaN, and the rows beside them theirs."""
    form = (2, 2, 4, 2, 32, 32, 16, 6, [90, 70], None, "none", 0.0)
    N, Sq, heads, kv, D, Cb, page, per, lengths, *_ = form
    cache, table, q, k, v, more, reach, plan = attention_setup(form, kind)
    out = torch.empty(q.shape, device=DEV)
    plan.run(q.to(DEV), out, table, ints(lengths))
    clean = tokens_of(out, heads)
    q[0, 1, 0, 3], q[1, 2, 1, 0] = math.nan, math.inf
    plan.run(q.to(DEV), out, table, ints(lengths))
    got = tokens_of(out, heads)
    hit = torch.zeros(N, Sq, heads, dtype=torch.bool)
    hit[0, 0, 1] = hit[1, 1, 2] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], clean[~hit])


def test_captured_beside_eager_calls_and_another_stream():
    """A step of serving -- turn, write, attend -- captured once and replayed with new tokens, lengths and tables; every replay against the eager calls on another cache."""
    N, heads, kv, D, page, per = 3, 4, 2, 32, 16, 8
    caches = [S.PagedCache(N * per, page, kv, D) for _ in range(2)]
    plans = [S.CacheAttention(c, N, 1, heads, per, Cb=D) for c in caches]
    turns = S.Rotary(N, 1, heads, kv, D, halves=True, Cb=D)
    freq = S.axis_frequencies(D // 2).to(DEV)
    q, k, v = rand(0, N, heads, 1, D).to(DEV), rand(1, N, kv, 1, D).to(DEV), rand(2, N, kv, 1, D).to(DEV)
    table, first, lengths = table_for(N, per, N * per), ints([0, 0, 0]), ints([1, 1, 1])
    outs = [torch.empty_like(q) for _ in range(2)]
    turned = [torch.empty_like(q) for _ in range(2)]

    def step(x):
        caches[x].write(k, v, table, first, rotary=turns, freq=freq, q=q, q_out=turned[x])
        plans[x].run(turned[x], outs[x], table, lengths)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(0)
        step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for at in range(40):
        for n, t in enumerate((q, k, v)):
            t.copy_(rand(10 * at + n, *t.shape))
        first.fill_(at)
        lengths.fill_(at + 1)
        graph.replay()
        torch.cuda.synchronize()
        if at % 2:
            step(1)
        else:
            with torch.cuda.stream(side):
                step(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(caches[0].keys, caches[1].keys) and torch.equal(caches[0].values, caches[1].values)


@pytest.mark.parametrize("T", [1, 17])
def test_very_many_heads(T):
    """More heads than fit 31 bits with the workgroups that share them."""
    kv = 1100000
    cache = S.PagedCache(1, 32, kv, 1, kind="float32")
    k, v = rand(0, 1, kv // 16, T, 16).to(DEV), rand(1, 1, kv // 16, T, 16).to(DEV)
    cache.write(k, v, ints([[0]]), ints([3]))
    back = [torch.full_like(k, math.nan) for _ in range(2)]
    cache.read(*back, ints([[0]]), ints([3]))
    assert torch.equal(back[0], k) and torch.equal(back[1], v)


@pytest.mark.parametrize("kind", KINDS)
def test_calls_with_a_stream(kind):
    """A stream that is given, which goes through ctypes: the same bits as on the current stream."""
    N, heads, kv, D, page, per, T = 2, 4, 2, 32, 16, 6, 20
    q, k, v = rand(0, N, heads, T, D).to(DEV), rand(1, N, kv, T, D).to(DEV), rand(2, N, kv, T, D).to(DEV)
    freq, first, lengths, table, side = rand(3, 1, 1, 16).to(DEV), ints([0, 37]), ints([T, 37 + T]), table_for(N, per, N * per), torch.cuda.Stream()
    found = []
    for stream in (None, side):
        cache, turns = S.PagedCache(N * per, page, kv, D, kind=kind), S.Rotary(N, T, heads, kv, D, Cb=D)
        turned, out, back = torch.empty_like(q), torch.empty_like(q), [torch.zeros_like(k) for _ in range(2)]
        plan, lse = S.CacheAttention(cache, N, T, heads, per, Cb=D), torch.empty(N, heads, T, device=DEV)
        torch.cuda.synchronize()
        cache.write(k, v, table, first, rotary=turns, freq=freq, q=q, q_out=turned, stream=stream)
        cache.read(*back, table, first, stream=stream)
        plan.run(turned, out, table, lengths, lse=lse, first=first, stream=stream)
        torch.cuda.synchronize()
        found.append([turned, out, lse, *back])
        assert cache.record.N == 0 and not cache.record.table and not turns.record.freq
    assert all(torch.equal(a, b) for a, b in zip(*found))


def test_a_cache_past_two_gigabytes():
    """Offsets of pages and channels past 32 bits: the last pages of a pool of 2.3 GB."""
    kv, D, page = 4, 256, 256
    pages = 4300
    cache = S.PagedCache(pages, page, kv, D, kind="bfloat16")
    assert cache.keys.numel() * 2 > 1 << 31
    k, v, q = rand(0, 1, kv, 300, D), rand(1, 1, kv, 300, D), rand(2, 1, kv, 1, D)
    table = ints([[pages - 1, pages - 2]])
    cache.write(k.to(DEV), v.to(DEV), table)
    back = [torch.empty(1, kv, 300, D, device=DEV) for _ in range(2)]
    cache.read(*back, table)
    assert torch.equal(back[0].cpu(), k.bfloat16().float()) and torch.equal(back[1].cpu(), v.bfloat16().float())
    out, lse = torch.empty(1, kv, 1, D, device=DEV), torch.empty(1, kv, 1, device=DEV)
    S.CacheAttention(cache, 1, 1, kv, 2, Cb=D).run(q.to(DEV), out, table, ints([300]), lse=lse)
    ref, ref_lse, size = attend(tokens_of(q, kv), held(tokens_of(k, kv), "bfloat16"), held(tokens_of(v, kv), "bfloat16"), [300], None, D ** -0.5)
    check_attention(tokens_of(out, kv), lse, ref, ref_lse, size, D, 512, v)
