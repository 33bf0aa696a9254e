"""The measured work of serving and training with rotary positions and a paged cache, next to the attention block.

Rotary positions over one axis (frames), two (pixels) or three (pixels of a clip's images), their gradient with that of learned frequencies;
keys and values written into the pages of a cache as 32-bit, bfloat16 or 8-bit numbers, and read back into activations; attention of
one or a few new tokens a stream over such a cache. Activations are channel-blocked, [N][C/Cb][tokens][Cb], as the convolutions write
them. Sizes are those of the stand-in networks of `workloads/`, of the layer sweep and of the attention block, generic sequence lengths, and ragged
ones between them. `listed()` names the cases, `draw(rng)` gives further ones of the same ranges. Where `own` is false, `run`
computes the operators from elementary torch operations: products and softmax in fp32, angles and rotations in 64 bits (a position in the
hundred thousands times a frequency, and codes whose values stand next to a border), each result rounded once.

A cache of `kind` "float32", "bfloat16" or "int8" has `pages` pages of `page` tokens:
    keys [pages][kv_heads][page][D, filled up to 16 bytes], values [pages][kv_heads][D][page], and for int8 two [pages][kv_heads][page] of scales.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "int8": torch.int8}


def listed():
    return [
        # ---- rotary positions
        # Feature maps of 14 x 14 pixels at the layer sweep's batch: rows turn one half of a head's pairs, columns the other.
        {"name": "rotary_pixels_14x14_b64", "kind": "rotary", "N": 64, "T": 1, "H": 14, "W": 14, "heads": 8, "kv_heads": 8, "D": 32, "Cb": 16,
         "axes": 2, "pairs": 16, "halves": False, "learned": "no", "given": False, "far": 0},
        # Clips of 16 images, three axes, heads as blocks, a pair's channels half a head apart: memory traffic and little else.
        {"name": "rotary_clip_16x28x28_b2", "kind": "rotary", "N": 2, "T": 16, "H": 28, "W": 28, "heads": 8, "kv_heads": 2, "D": 64, "Cb": 64,
         "axes": 3, "pairs": 32, "halves": True, "learned": "no", "given": False, "far": 0},
        # A training step on small images whose every head has learned directions and frequencies.
        {"name": "rotary_grad_8x8_b256", "kind": "rotary_grad", "N": 256, "T": 1, "H": 8, "W": 8, "heads": 4, "kv_heads": 4, "D": 16, "Cb": 16,
         "axes": 2, "pairs": 8, "halves": False, "learned": "heads", "given": False, "far": 0},
        # Odd everything: pieces cut from long recordings, heads of 40 channels of which 24 turn, learned frequencies that all heads share.
        {"name": "rotary_grad_frames_999_b6", "kind": "rotary_grad", "N": 6, "T": 999, "H": 1, "W": 1, "heads": 6, "kv_heads": 3, "D": 40, "Cb": 8,
         "axes": 1, "pairs": 12, "halves": True, "learned": "shared", "given": True, "far": 4000},
        # ---- into the cache, and back
        # One new frame of each of many streams, its queries and keys turned on the way: latency is what counts.
        {"name": "write_frame_b32", "kind": "write", "N": 32, "S": 1, "heads": 8, "kv_heads": 2, "D": 64, "Cb": 64, "type": "int8", "page": 32,
         "room": 16384, "rotary": True, "pairs": 32, "halves": True, "ragged": False, "far": 16000},
        # The first frames of four streams, of unequal numbers, in one padded batch.
        {"name": "write_frames_4096_b4", "kind": "write", "N": 4, "S": 4096, "heads": 16, "kv_heads": 4, "D": 64, "Cb": 16, "type": "int8", "page": 64,
         "room": 4096, "rotary": True, "pairs": 32, "halves": False, "ragged": True, "far": 0},
        # A further piece of some recordings that ends and begins inside pages, heads of 40 channels that begin inside channel blocks.
        {"name": "write_frames_999_b6", "kind": "write", "N": 6, "S": 999, "heads": 6, "kv_heads": 3, "D": 40, "Cb": 8, "type": "bfloat16", "page": 16,
         "room": 2048, "rotary": False, "pairs": 0, "halves": False, "ragged": True, "far": 1000},
        # What a further piece of a stream attends to by the whole-sequence call: all that is in the cache.
        {"name": "read_frames_8192_b8", "kind": "read", "N": 8, "S": 8192, "heads": 8, "kv_heads": 8, "D": 64, "Cb": 16, "type": "int8", "page": 64,
         "room": 8192, "ragged": False, "far": 0},
        # A few short streams with heads of 80 channels, whole numbers of nothing.
        {"name": "read_frames_301_b3", "kind": "read", "N": 3, "S": 301, "heads": 5, "kv_heads": 5, "D": 80, "Cb": 400, "type": "float32", "page": 16,
         "room": 512, "ragged": True, "far": 77},
        # ---- new tokens against the cache
        # One stream, one new frame: latency.
        {"name": "token_777_b1", "kind": "token", "N": 1, "Sq": 1, "Sk": 777, "heads": 8, "kv_heads": 8, "D": 32, "Cb": 32, "type": "float32", "page": 16,
         "bias": "buckets", "cap": 0.0, "ragged": False},
        # Many streams of different ages on 8-bit keys and values, key heads shared by four: the cache's bytes. The largest one.
        {"name": "token_16384_b64", "kind": "token", "N": 64, "Sq": 1, "Sk": 16384, "heads": 16, "kv_heads": 4, "D": 64, "Cb": 16, "type": "int8", "page": 64,
         "bias": "slopes", "cap": 50.0, "ragged": True},
        # Five frames that were guessed ahead, checked at once.
        {"name": "tokens_5_of_3001_b16", "kind": "token", "N": 16, "Sq": 5, "Sk": 3001, "heads": 8, "kv_heads": 2, "D": 128, "Cb": 128, "type": "bfloat16",
         "page": 128, "bias": "none", "cap": 0.0, "ragged": True},
    ]


# ---------------------------------------------------------------------------------------------------- drawn cases

MAX_TURN = 12e6        # values that a drawn rotation turns; the largest listed one has 16e6
MAX_STORE = 24e6       # values of keys and values written and read back, or read; the largest listed one has 67e6
MAX_CACHE = 240e6      # bytes of a drawn cache that tokens attend to; the largest listed one has 571e6


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _heads(rng):
    D = rng.choice([16, 16, 32, 32, 40, 64, 64, 64, 80, 96, 128, 256])
    kv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 4, 8])
    Cb = rng.choice([16, 16, D, kv * D, 8]) if D % 16 == 0 else rng.choice([8, D, kv * D])
    return {"heads": kv * group, "kv_heads": kv, "D": D, "Cb": Cb}


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "rotary_grad", "rotary_grad", "write", "write", "read", "token", "token", "token"])
    c = {"kind": kind, **_heads(rng)}
    D, heads, kv = c["D"], c["heads"], c["kv_heads"]
    if kind.startswith("rotary"):
        axes = rng.choice([1, 2, 2, 3])
        T = 1 if axes == 2 else _log(rng, 1, 4096) if axes == 1 else _log(rng, 1, 24)
        H, W = (1, 1) if axes == 1 else (_log(rng, 2, 40), _log(rng, 2, 40))
        if kind == "rotary_grad" and axes == 1:              # (a position of zero has no gradient by the frequencies)
            T = max(T, 2)
        while T * H * W * (heads + kv) * D > MAX_TURN:
            T, H, W = (T // 2 + 1, H, W) if T > 2 else (T, H // 2 + 1, W // 2 + 1)
        most = int(MAX_TURN // (T * H * W * (heads + kv) * D))
        return {**c, "N": max(1, min(_log(rng, 1, 256), most)), "T": T, "H": H, "W": W, "axes": axes, "pairs": rng.choice([D // 2, D // 2, D // 4, 3]),
                "halves": rng.random() < 0.5, "learned": rng.choice(["no", "shared", "heads"]), "given": rng.random() < 0.3,
                "far": rng.choice([0, 0, 100000]) if axes == 1 and kind == "rotary" else 0}
    c |= {"type": rng.choice(["float32", "bfloat16", "int8", "int8"]), "page": rng.choice([16, 32, 64, 128])}
    if kind == "token":
        token = 2 * kv * D * TYPES[c["type"]].itemsize
        Sq, Sk = rng.choice([1, 1, 1, 1, 2, 7]), min(_log(rng, 1, 32768), int(MAX_CACHE // token))
        most = int(MAX_CACHE // (Sk * token))
        return {**c, "N": max(1, min(_log(rng, 1, 256), most)), "Sq": min(Sq, Sk), "Sk": Sk, "bias": rng.choice(["none", "slopes", "buckets"]),
                "cap": rng.choice([0.0, 0.0, 15.0, 50.0]), "ragged": rng.random() < 0.7}
    S, far = rng.choice([1, _log(rng, 1, 4096), _log(rng, 1, 4096)]), rng.choice([0, 0, 333, 3000])
    S = min(S, int(MAX_STORE // ((2 * kv + heads) * D)))
    most = int(MAX_STORE // (S * (2 * kv + heads) * D))
    N = max(1, min(_log(rng, 1, 256), most))
    c |= {"N": N, "S": S, "room": max(S + far, 16), "ragged": rng.random() < 0.5, "far": far}
    if kind == "write":
        rotary = rng.random() < 0.6
        c |= {"rotary": rotary, "pairs": rng.choice([D // 2, D // 2, D // 4]) if rotary else 0, "halves": rng.random() < 0.5}
    return c


# ---------------------------------------------------------------------------------------------------- inputs

REACH, BUCKETS = 512, 32       # of the biases by buckets: frames further back are in the last bucket


def log_buckets(reach, buckets):
    """The bucket of each offset -reach .. reach of a key against its query, for keys at or before it: one half of the buckets for
    single offsets, the other for offsets that grow by a constant factor."""
    single = buckets // 2
    edges = [single * (reach / single) ** (k / (buckets - single)) for k in range(buckets - single)]
    found = []
    for r in range(-reach, reach + 1):
        d = max(0, -r)
        found.append(d if d < single else single - 1 + sum(d >= e for e in edges))
    return found


def _lengths(case):
    """Streams of ages spread evenly over the range; with many, one place without a stream."""
    N, S = case["N"], case["Sk"]
    if not case["ragged"]:
        return [S] * N
    low = max(1, S // 8)
    lengths = [S - (S - low) * n // max(1, N) for n in range(N)]
    if N >= 16:
        lengths[1] = 0
    return lengths


def _counts(case):
    """New frames of each stream: all of the padded batch's, or unequal numbers down to a quarter."""
    N, S = case["N"], case["S"]
    return [S - (S - (S + 3) // 4) * n // N if case["ragged"] else S for n in range(N)]


def _tokens(case):
    return case["T"] * case["H"] * case["W"]


def _frequencies(case, rand):
    """[1 or kv_heads][axes][pairs]: a section of the pairs for each axis, falling from 1 to 1/10000 (frames) or 1/100 (pixels) radians a step;
    learned ones turn by all axes."""
    axes, pairs = case.get("axes", 1), case["pairs"]
    learned = case.get("learned", "no")
    base = 10000.0 if axes == 1 else 100.0
    if learned != "no":
        fall = torch.tensor([base ** (-k / pairs) for k in range(pairs)], device=DEV)
        return (rand(case["kv_heads"] if learned == "heads" else 1, axes, pairs) * fall).contiguous()
    freq = torch.zeros(1, axes, pairs)
    for a in range(axes):
        lo, hi = pairs * a // axes, pairs * (a + 1) // axes
        for k in range(lo, hi):
            freq[0, a, k] = base ** (-(k - lo) / (hi - lo))
    return freq.to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    order = random.Random(int(seed))
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    N, heads, kv, D, Cb = (case[n] for n in ("N", "heads", "kv_heads", "D", "Cb"))
    nq, nk = heads * D // Cb, kv * D // Cb
    state = {**case, "first": None, "positions": None, "freq": None, "q": None}
    if case["kind"].startswith("rotary"):
        S = _tokens(case)
        # the parts of one projection's output
        qkv = rand(N, nq + 2 * nk, S, Cb)
        state["q"], state["k"] = qkv[:, :nq], qkv[:, nq:nq + nk]
        state["freq"] = _frequencies(case, rand)
        state["extent"] = (case["H"], case["W"])[3 - case["axes"]:] if case["axes"] > 1 else ()
        starts = [order.randint(0, case["far"]) for _ in range(N)]
        if case["far"]:
            state["first"] = ints(starts)
        if case["given"]:
            # positions that the program keeps itself: pixels and frames as they stand in a larger whole
            t = torch.arange(S, device=DEV) + ints(starts)[:, None]
            columns = [t // (case["H"] * case["W"]), t // case["W"] % case["H"], t % case["W"]]
            columns = columns[:1] if case["axes"] == 1 else columns[3 - case["axes"]:]
            state["positions"], state["first"] = torch.stack([c + 3 * a for a, c in enumerate(columns)], 2).int().contiguous(), None
        if case["kind"] == "rotary_grad":
            state["dq"], state["dk"] = rand(N, nq, S, Cb), rand(N, nk, S, Cb)
        return state
    # a cache that other streams have used before: pages in any order, all of them full
    page, kind = case["page"], TYPES[case["type"]]
    room = case["Sk"] if case["kind"] == "token" else case["room"]
    each = -(-room // page)
    pages = N * each + 3
    Dk = -(-D * kind.itemsize // 16) * 16 // kind.itemsize

    def fill(*shape):
        if kind is not torch.int8:
            return rand(*shape).to(kind)
        return torch.cat([rand(-(-shape[0] // 8), *shape[1:]).mul_(40).round_().clamp_(-127, 127).to(torch.int8) for _ in range(8)])[:shape[0]].contiguous()
    state["keys"], state["values"] = fill(pages, kv, page, Dk), fill(pages, kv, D, page)
    state["keys"][..., D:] = 0
    state["key_scales"] = state["value_scales"] = None
    if kind is torch.int8:
        state["key_scales"], state["value_scales"] = ((0.02 + 0.02 * rand(pages, kv, page).abs()) for _ in range(2))
    numbers = list(range(pages))
    order.shuffle(numbers)
    state["pages"] = ints(numbers[:N * each]).reshape(N, each)
    if case["kind"] == "token":
        Sq, lengths = case["Sq"], _lengths(case)
        order.shuffle(lengths)
        state["lengths"] = ints(lengths)
        for n, held in enumerate(lengths):                   # (what a table holds behind a stream's last page)
            state["pages"][n, -(-held // page):] = -1
        state["q"] = rand(N, nq, Sq, Cb)
        state["scale"], state["slopes"], state["table"], state["bucket"] = 1 / math.sqrt(D), None, None, None
        if case["bias"] == "slopes":
            state["slopes"] = torch.tensor([2.0 ** (-8 * (h + 1) / heads) for h in range(heads)], device=DEV)
        elif case["bias"] == "buckets":
            state["table"], state["bucket"] = 0.5 * rand(heads, BUCKETS), ints(log_buckets(REACH, BUCKETS))
        return state
    counts = _counts(case)
    order.shuffle(counts)
    state["counts"] = ints(counts) if case["ragged"] else None
    state["first"] = ints([order.randint(0, case["far"]) if case["far"] else 0 for _ in range(N)])
    S = case["S"]
    if case["kind"] == "write":
        qkv = rand(N, nq + 2 * nk, S, Cb)
        state["q"], state["k"], state["v"] = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
        if case["rotary"]:
            state["freq"] = _frequencies(case, rand)
    # where read values go, and what stood there before
    state["k_out"], state["v_out"] = torch.zeros(N, nk, S, Cb, device=DEV), torch.zeros(N, nk, S, Cb, device=DEV)
    return state


# ---------------------------------------------------------------------------------------------------- the operators

def run(state):
    kind = state["kind"]
    if own:
        return {"rotary": _own_rotary, "rotary_grad": _own_rotary_grad, "write": _own_write, "read": _own_read, "token": _own_token}[kind](state)
    return {"rotary": _plain_rotary, "rotary_grad": _plain_rotary_grad, "write": _plain_write, "read": _plain_read, "token": _plain_token}[kind](state)


def _own_plan(s, S):
    import paper_2303_04769_amd as A
    if "plan" not in s:
        s["plan"] = A.Rotary(s["N"], S, s["heads"], s["kv_heads"], s["D"], axes=s.get("axes", 1), pairs=s["pairs"], halves=s["halves"],
                             extent=s.get("extent", ()), freq_heads=s["freq"].shape[0], Cb=s["Cb"])
    return s["plan"]


def _own_cache(s):
    import paper_2303_04769_amd as A
    if "cache" not in s:
        tensors = (s["keys"], s["values"], s["key_scales"], s["value_scales"])
        s["cache"] = A.PagedCache(s["keys"].shape[0], s["page"], s["kv_heads"], s["D"], kind=s["type"], tensors=tensors)
    return s["cache"]


def _own_rotary(s):
    q, k = torch.empty(s["q"].shape, device=DEV), torch.empty(s["k"].shape, device=DEV)
    _own_plan(s, _tokens(s)).run(s["q"], s["k"], s["freq"], q, k, first=s["first"], positions=s["positions"])
    return {"q": q, "k": k}


def _own_rotary_grad(s):
    dq, dk = torch.empty_like(s["dq"]), torch.empty_like(s["dk"])
    dfreq = None if s["learned"] == "no" else torch.empty_like(s["freq"])
    _own_plan(s, _tokens(s)).grad(s["dq"], s["dk"], s["freq"], dq, dk, q=s["q"], k=s["k"], dfreq=dfreq, first=s["first"], positions=s["positions"])
    return {"dq": dq, "dk": dk, **({} if dfreq is None else {"dfreq": dfreq})}


def _own_write(s):
    cache, turned = _own_cache(s), {}
    if s["rotary"]:
        q = torch.empty(s["q"].shape, device=DEV)
        cache.write(s["k"], s["v"], s["pages"], s["first"], counts=s["counts"], rotary=_own_plan(s, s["S"]), freq=s["freq"], q=s["q"], q_out=q)
        turned = {"q": q}
    else:
        cache.write(s["k"], s["v"], s["pages"], s["first"], counts=s["counts"])
    return {**turned, **_own_read(s)}


def _own_read(s):
    _own_cache(s).read(s["k_out"], s["v_out"], s["pages"], s["first"], counts=s["counts"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_token(s):
    import paper_2303_04769_amd as A
    if "attention" not in s:
        s["attention"] = A.CacheAttention(_own_cache(s), s["N"], s["Sq"], s["heads"], s["pages"].shape[1], Cb=s["Cb"], scale=s["scale"], cap=s["cap"],
                                          reach=REACH if s["table"] is not None else 0, buckets=BUCKETS if s["table"] is not None else 0)
    out, lse = torch.empty(s["q"].shape, device=DEV), torch.empty(s["N"], s["heads"], s["Sq"], device=DEV)
    s["attention"].run(s["q"], out, s["pages"], s["lengths"], lse=lse, slopes=s["slopes"], table=s["table"], bucket=s["bucket"])
    return {"out": out, "lse": lse}


def _split(t, heads):
    """[N][C/Cb][S][Cb] -> [N][heads][S][D]"""
    return t.permute(0, 1, 3, 2).reshape(t.shape[0], heads, -1, t.shape[2]).transpose(2, 3)


def _merge(t, Cb):
    return t.transpose(2, 3).reshape(t.shape[0], -1, Cb, t.shape[2]).permute(0, 1, 3, 2).contiguous()


def _angles(s, S):
    """Positions [N or 1][S][axes] and angles [N or 1][heads of the frequencies][S][pairs], in 64 bits."""
    if s["positions"] is not None:
        p = s["positions"].double()
    else:
        t = torch.arange(S, device=DEV)[None]
        if s["first"] is not None:
            t = t + s["first"][:, None]
        axes = s.get("axes", 1)
        columns = [t] if axes == 1 else [t // s["W"], t % s["W"]] if axes == 2 else [t // (s["H"] * s["W"]), t // s["W"] % s["H"], t % s["W"]]
        p = torch.stack(columns, 2).double()
    return p, (p[:, None, :, :, None] * s["freq"].double()[None, :, None]).sum(3)


def _pairs(t, s):
    """The two channels of every pair, and where they stand: [N][heads][S][pairs] each."""
    n = s["pairs"]
    return (t[..., :n], t[..., n:2 * n]) if s["halves"] else (t[..., 0:2 * n:2], t[..., 1:2 * n:2])


def _turn(t, heads, s, angles, sign=1.0):
    """Turned heads [N][heads][S][D] in 64 bits, of an activation."""
    x = _split(t, heads).double()
    by = angles if angles.shape[1] == 1 else angles.repeat_interleave(heads // angles.shape[1], 1)
    c, d = torch.cos(by), sign * torch.sin(by)
    out = x.clone()
    x0, x1 = _pairs(x, s)
    y0, y1 = _pairs(out, s)
    y0.copy_(x0 * c - x1 * d)
    y1.copy_(x0 * d + x1 * c)
    return out


def _plain_rotary(s):
    angles = _angles(s, _tokens(s))[1]
    return {n: _merge(_turn(s[n], h, s, angles), s["Cb"]).float() for n, h in (("q", s["heads"]), ("k", s["kv_heads"]))}


def _plain_rotary_grad(s):
    p, angles = _angles(s, _tokens(s))
    result = {n: _merge(_turn(s[n], h, s, angles, -1.0), s["Cb"]).float() for n, h in (("dq", s["heads"]), ("dk", s["kv_heads"]))}
    if s["learned"] == "no":
        return result
    by_angle = 0.0
    for x, d, heads in (("q", "dq", s["heads"]), ("k", "dk", s["kv_heads"])):
        (x0, x1), (d0, d1) = (_pairs(_split(s[n], heads).double(), s) for n in (x, d))
        g = d1 * x0 - d0 * x1                                # (of the turned channels: q and k are what the forward call gave)
        by_angle = by_angle + g.reshape(g.shape[0], s["freq"].shape[0], -1, *g.shape[2:]).sum(2)
    return {**result, "dfreq": torch.einsum("nfsk,nsa->fak", by_angle, p.expand(s["N"], -1, -1)).float()}


def _codes(x):
    """8-bit codes and scales of [N][heads][S][D]: a scale for each token of a head."""
    most = x.abs().amax(3)
    fine, top = most >= 2.0 ** -100, torch.full_like(most, 127)          # (a tensor: by a number torch multiplies with its reciprocal)
    scale = torch.where(fine, most / top, 0.0)
    by = torch.where(fine, top / torch.where(fine, most, 1.0), 0.0)
    return torch.round(x * by[..., None]).to(torch.int8), scale


def _places(s):
    """Page and place in it of every token [N][S], and whether there is such a token."""
    t = torch.arange(s["S"], device=DEV)[None]
    p = t + s["first"][:, None]
    there = (t < s["counts"][:, None]) if s["counts"] is not None else torch.ones_like(p, dtype=torch.bool)
    at = torch.where(there, p, 0)
    return s["pages"].gather(1, (at // s["page"]).long()).long(), (at % s["page"]).long(), there


def _plain_write(s):
    k, v = _split(s["k"], s["kv_heads"]), _split(s["v"], s["kv_heads"])
    result = {}
    if s["rotary"]:
        angles = _angles(s, s["S"])[1]
        k = _turn(s["k"], s["kv_heads"], s, angles).float()
        result["q"] = _merge(_turn(s["q"], s["heads"], s, angles), s["Cb"]).float()
    page, place, there = _places(s)
    if s["type"] == "int8":
        (k, k_scale), (v, v_scale) = _codes(k), _codes(v)
        for to, scale in ((s["key_scales"], k_scale), (s["value_scales"], v_scale)):
            to[page[there], :, place[there]] = scale.permute(0, 2, 1)[there]
    kind = TYPES[s["type"]]
    s["keys"][page[there], :, place[there], :s["D"]] = k.permute(0, 2, 1, 3)[there].to(kind)
    s["values"][page[there], :, :, place[there]] = v.permute(0, 2, 1, 3)[there].to(kind)
    return {**result, **_plain_read(s)}


def _plain_read(s):
    page, place, there = _places(s)
    k, v = s["keys"][page, :, place, :s["D"]].float(), s["values"][page, :, :, place].float()        # [N][S][kv][D]
    if s["type"] == "int8":
        k, v = (x * scale[page, :, place][..., None] for x, scale in ((k, s["key_scales"]), (v, s["value_scales"])))
    for x, to in ((k, s["k_out"]), (v, s["v_out"])):
        to.copy_(torch.where(there[:, None, :, None], _merge(x.permute(0, 2, 1, 3), s["Cb"]), to))
    return {"k": s["k_out"], "v": s["v_out"]}


def _held(s):
    """All keys and values of the streams, [N][kv][Sk][D], in fp32."""
    at = s["pages"].clamp(min=0).long()
    N, each = at.shape
    k, v = s["keys"][at][..., :s["D"]].float(), s["values"][at].float()              # [N][each][kv][page][D], [..][D][page]
    if s["type"] == "int8":
        k, v = k * s["key_scales"][at][..., None], v * s["value_scales"][at][..., None, :]
    whole = lambda t: t.permute(0, 2, 1, 3, 4).reshape(N, s["kv_heads"], each * s["page"], s["D"])  # noqa: E731
    return whole(k), whole(v.transpose(3, 4))


def _plain_token(s):
    N, heads, kv, Sq, D = s["N"], s["heads"], s["kv_heads"], s["Sq"], s["D"]
    k, v = _held(s)
    Sk, group = k.shape[2], heads // kv
    q = _split(s["q"], heads).reshape(N, kv, group * Sq, D)
    x = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).reshape(N, heads, Sq, Sk)
    if s["cap"]:
        x = torch.tanh(x / s["cap"]) * s["cap"]
    j = torch.arange(Sk, device=DEV)
    pos = (s["lengths"] - Sq)[:, None] + torch.arange(Sq, device=DEV)                  # [N][Sq]
    if s["slopes"] is not None:
        x = x - s["slopes"].reshape(heads, 1, 1) * (pos[:, None, :, None] - j).abs()
    if s["table"] is not None:
        index = s["bucket"][(j - pos[:, :, None]).clamp(-REACH, REACH) + REACH].long()
        x = x + s["table"][:, index].transpose(0, 1)
    x = torch.where((j <= pos[:, :, None])[:, None], x, -math.inf)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = torch.matmul(p.reshape(N, kv, group * Sq, Sk), v).reshape(N, heads, Sq, D)
    return {"out": _merge(out, s["Cb"]), "lse": (top + torch.log(total)).squeeze(3)}


# ---------------------------------------------------------------------------------------------------- work

def work(case):
    N, heads, kv, D = (case[n] for n in ("N", "heads", "kv_heads", "D"))
    if case["kind"].startswith("rotary"):
        values, turns = N * _tokens(case) * (heads + kv) * D, N * _tokens(case) * (heads + kv) * case["pairs"]
        freq = (kv if case["learned"] == "heads" else 1) * case["axes"] * case["pairs"]
        given = N * _tokens(case) * case["axes"] if case["given"] else 0
        if case["kind"] == "rotary":
            return {"bytes": 4 * (2 * values + freq + given), "flops": 6 * turns}
        learned = case["learned"] != "no"
        # the rotated channels are read where frequencies are learned: only those that turn
        return {"bytes": 4 * (2 * values + freq + given + (2 * turns + freq if learned else 0)), "flops": (11 if learned else 6) * turns}
    size = TYPES[case["type"]].itemsize
    token = 2 * kv * (D * size + (4 if size == 1 else 0))      # bytes that a token has in the cache
    if case["kind"] == "token":
        seen = sum(_lengths(case))
        return {"bytes": seen * token + 4 * N * case["Sq"] * heads * (2 * D + 1), "flops": 4 * seen * case["Sq"] * heads * D}
    there = sum(_counts(case))
    plain = 4 * there * 2 * kv * D
    if case["kind"] == "read":
        return {"bytes": there * token + plain, "flops": there * 2 * kv * D}
    # written into the cache, and read back from it
    queries = 2 * 4 * N * case["S"] * heads * D if case["rotary"] else 0
    turns = N * case["S"] * heads * case["pairs"] + there * kv * case["pairs"]
    return {"bytes": 2 * plain + 2 * there * token + queries, "flops": there * 8 * kv * D + 6 * turns}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "rotary_grad": _exact_rotary, "write": _exact_write, "read": _exact_read, "token": _exact_token}[case["kind"]](s)


def _channels(t):
    """[N][C][S] in 64 bits, channels in order."""
    return t.double().transpose(2, 3).reshape(t.shape[0], -1, t.shape[2])


def _blocks(t, Cb):
    return t.view(t.shape[0], -1, Cb, t.shape[2]).transpose(2, 3).contiguous()


def _exact_coordinates(s, n, S):
    """[S][axes] of image n."""
    if s["positions"] is not None:
        return s["positions"][n].double()
    t = torch.arange(S, device=DEV, dtype=torch.float64) + (0 if s["first"] is None else int(s["first"][n]))
    found = []
    for size in reversed(s.get("extent", ())):
        found.insert(0, torch.remainder(t, size))
        t = torch.floor(t / size)
    return torch.stack([t] + found, 1)


def _exact_turned(x, s, n, freq, heads):
    """Image n's [heads * D][S], turned as complex numbers."""
    S, D, P = x.shape[1], s["D"], s["pairs"]
    at = _exact_coordinates(s, n, S)
    x = x.view(heads, D, S)
    first, second = (slice(0, P), slice(P, 2 * P)) if s["halves"] else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    turned = torch.empty_like(x)
    turned[:, 2 * P:] = x[:, 2 * P:]
    per = heads // freq.shape[0]
    pieces = []
    for h in range(heads):
        angle = torch.matmul(at, freq[h // per]).t()
        pieces.append(torch.complex(x[h, first], x[h, second]) * torch.polar(torch.ones_like(angle), angle))
    z = torch.stack(pieces)
    turned = turned.index_copy(1, torch.arange(D, device=DEV)[first], z.real).index_copy(1, torch.arange(D, device=DEV)[second], z.imag)
    return turned.reshape(heads * D, S)


def _exact_rotary(s):
    """Image by image; gradients by automatic differentiation at the channels that were turned back."""
    grad = s["kind"] == "rotary_grad"
    parts = (("q", s["heads"]), ("k", s["kv_heads"]))
    found = {n: [] for n, _ in parts}
    freq = s["freq"].double()
    dfreq = torch.zeros_like(freq)
    for n in range(s["N"]):
        for name, heads in parts:
            x = _channels(s[name][n:n + 1])[0]
            if not grad:
                found[name].append(_exact_turned(x, s, n, freq, heads))
                continue
            before = _exact_turned(x, s, n, -freq, heads).requires_grad_()
            f = freq.clone().requires_grad_()
            after = _exact_turned(before, s, n, f, heads)
            a, b = torch.autograd.grad(after, (before, f), _channels(s["d" + name][n:n + 1])[0])
            found[name].append(a)
            dfreq += b
    result = {("d" if grad else "") + name: _blocks(torch.stack(found[name]), s["Cb"]) for name, _ in parts}
    return {**result, "dfreq": dfreq} if grad and s["learned"] != "no" else result


def _held_as(x, kind, D):
    """What a cache of this type gives back for [kv * D][S]: the type's rounding, by its definition."""
    if kind == "float32":
        return x.float().double()
    if kind == "bfloat16":
        return x.float().bfloat16().double()
    x = x.float().double().view(-1, D, x.shape[1])
    most = x.abs().max(1, keepdim=True).values
    small = most < 2.0 ** -100
    most = most.masked_fill(small, math.inf)
    scale, by = (most / 127).float().double().masked_fill(small, 0.0), (127 / most).float().double()
    return ((x * by).float().round().double() * scale).float().double().reshape(-1, x.shape[2])


def _exact_write(s):
    k, v = [], []
    freq = s["freq"].double() if s["rotary"] else None
    for n in range(s["N"]):
        a, b = _channels(s["k"][n:n + 1])[0], _channels(s["v"][n:n + 1])[0]
        if s["rotary"]:
            a = _exact_turned(a, s, n, freq, s["kv_heads"])
        count = s["S"] if s["counts"] is None else int(s["counts"][n])
        for x, to in ((a, k), (b, v)):
            held = _held_as(x, s["type"], s["D"])
            held[:, count:] = 0
            to.append(held)
    result = {"k": _blocks(torch.stack(k), s["Cb"]), "v": _blocks(torch.stack(v), s["Cb"])}
    if s["rotary"]:
        q = [_exact_turned(_channels(s["q"][n:n + 1])[0], s, n, freq, s["heads"]) for n in range(s["N"])]
        result["q"] = _blocks(torch.stack(q), s["Cb"])
    return result


def _exact_stream(s, n, held):
    """Keys and values [kv][held][D] of stream n."""
    numbers = s["pages"][n, :-(-held // s["page"])].long()
    k, v = s["keys"][numbers, :, :, :s["D"]].double(), s["values"][numbers].double().transpose(2, 3)
    if s["type"] == "int8":
        k, v = k * s["key_scales"][numbers].double()[..., None], v * s["value_scales"][numbers].double()[..., None]
    return (t.transpose(0, 1).reshape(s["kv_heads"], -1, s["D"])[:, :held] for t in (k, v))


def _exact_read(s):
    outs = []
    for n in range(s["N"]):
        first, count = int(s["first"][n]), s["S"] if s["counts"] is None else int(s["counts"][n])
        pair = []
        for t in _exact_stream(s, n, first + count):
            x = torch.zeros(s["kv_heads"] * s["D"], s["S"], dtype=torch.float64, device=DEV)
            x[:, :count] = t[:, first:].transpose(1, 2).reshape(-1, count)
            pair.append(x)
        outs.append(pair)
    return {name: _blocks(torch.stack([o[i] for o in outs]), s["Cb"]) for i, name in enumerate(("k", "v"))}


def _exact_token(s):
    heads, kv, Sq, D = s["heads"], s["kv_heads"], s["Sq"], s["D"]
    group = heads // kv
    outs, lses = [], []
    for n in range(s["N"]):
        held = int(s["lengths"][n])
        if not held:
            outs.append(torch.zeros(heads * D, Sq, dtype=torch.float64, device=DEV))
            lses.append(torch.full((heads, Sq), -math.inf, dtype=torch.float64, device=DEV))
            continue
        k, v = _exact_stream(s, n, held)
        q = _channels(s["q"][n:n + 1])[0].view(kv, group, D, Sq)
        x = torch.matmul(k[:, None], q) * s["scale"]                                   # [kv][group][held][Sq]
        if s["cap"]:
            x = s["cap"] * torch.tanh(x / s["cap"])
        behind = torch.arange(held - Sq, held, device=DEV)[None] - torch.arange(held, device=DEV)[:, None]
        if s["slopes"] is not None:
            x = x - s["slopes"].double().view(kv, group, 1, 1) * behind.abs()
        if s["table"] is not None:
            x = x + s["table"].double()[:, s["bucket"].long()[REACH - behind.clamp(-REACH, REACH)]].view(kv, group, held, Sq)
        hidden = behind < 0
        x = x.masked_fill(hidden, -math.inf)
        empty = hidden.all(0)
        l = torch.logsumexp(x.masked_fill(empty, 0.0), 2)
        p = torch.exp(x - l[:, :, None])
        outs.append(torch.matmul(p.transpose(2, 3), v[:, None]).transpose(2, 3).reshape(heads * D, Sq))
        lses.append(l.masked_fill(empty, -math.inf).view(heads, Sq))
    return {"out": _blocks(torch.stack(outs), s["Cb"]), "lse": torch.stack(lses)}
