"""The measured work of the attention block: what programs that put normalization and attention between convolutions have it do.

Group normalization with an activation, attention over the pixels of feature maps or the frames of a clip (scores capped by a
tanh, learned relative position biases by buckets, biases that fall with the distance, causal, prefix and document masks, ragged
lengths), its form for single tokens against a cache, and the gradients of all of them, on the channel-blocked layout
[N][C/Cb][pixels][Cb] that the convolutions read and write. Sizes are those of the stand-in networks of `workloads/` and of the layer
sweep, generic sequence lengths, and ragged ones between them. `listed()` names the cases, `draw(rng)` gives further ones of the
same ranges. Where `own` is false, `run` computes the operators from elementary torch operations in fp32.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # ---- group normalization with an activation
        # One image through the last stage of a small residual network: latency is what counts.
        {"name": "norm_64x8_b1", "kind": "norm", "N": 1, "C": 64, "H": 8, "W": 8, "G": 8, "act": "silu", "Cb": 16},
        # The audio network's feature maps at its large batch, channels last (one block of all channels).
        {"name": "norm_64x25x5_b1024_last", "kind": "norm", "N": 1024, "C": 64, "H": 25, "W": 5, "G": 4, "act": "relu", "Cb": 64},
        # The largest row of the layer sweep: memory traffic and little else.
        {"name": "norm_256x56_b64", "kind": "norm", "N": 64, "C": 256, "H": 56, "W": 56, "G": 32, "act": "silu", "Cb": 16},
        # A training step on ragged sizes: odd image, groups of twelve channels that begin and end inside channel blocks.
        {"name": "norm_grad_96x57x43_b32", "kind": "norm_grad", "N": 32, "C": 96, "H": 57, "W": 43, "G": 8, "act": "silu", "Cb": 16},
        # ---- attention over whole images and clips
        # The last stage of the residual network on its benchmark's batch: 64 pixels, heads of 16 channels, a learned bias for every
        # offset of two pixels.
        {"name": "pixels_8x8_b256", "kind": "attn", "N": 256, "H": 8, "W": 8, "heads": 4, "kv_heads": 4, "D": 16, "Cb": 16,
         "mask": "none", "bias": "pixels", "cap": 0.0},
        # A recording as one sequence of frames: causal, scores capped, a learned bias by logarithmic buckets, shared key heads.
        {"name": "frames_4096_causal_b2", "kind": "attn", "N": 2, "H": 4096, "W": 1, "heads": 8, "kv_heads": 2, "D": 64, "Cb": 16,
         "mask": "causal", "bias": "buckets", "cap": 30.0},
        # Many clips packed into one long sequence, each attending to itself, a bias that falls with the distance; the last
        # frames are padding. The longest one.
        {"name": "frames_8192_documents_b1", "kind": "attn", "N": 1, "H": 8192, "W": 1, "heads": 8, "kv_heads": 8, "D": 64, "Cb": 16,
         "mask": "documents", "documents": 5, "bias": "slopes", "cap": 0.0},
        # ---- single tokens against a cache
        # One stream, one new frame: latency.
        {"name": "token_777_b1", "kind": "token", "N": 1, "Sk": 777, "heads": 8, "kv_heads": 8, "D": 32, "Cb": 16, "bias": "buckets",
         "cap": 0.0, "ragged": False},
        # Many streams of different ages with key heads shared by four: the cache's bytes.
        {"name": "token_16384_b64", "kind": "token", "N": 64, "Sk": 16384, "heads": 16, "kv_heads": 4, "D": 64, "Cb": 16, "bias": "slopes",
         "cap": 50.0, "ragged": True},
        # ---- training steps
        # Feature maps of 14 x 14 pixels at the sweep's batch, with the gradient of the learned bias.
        {"name": "grad_pixels_14x14_b64", "kind": "attn_grad", "N": 64, "H": 14, "W": 14, "heads": 8, "kv_heads": 8, "D": 32, "Cb": 16,
         "mask": "none", "bias": "pixels", "cap": 0.0},
        # A sequence with a prompt that every frame sees, capped scores, shared key heads, tokens-major tensors.
        {"name": "grad_frames_2048_prefix_b4", "kind": "attn_grad", "N": 4, "H": 2048, "W": 1, "heads": 8, "kv_heads": 2, "D": 64,
         "Cb": 64, "mask": "prefix", "bias": "buckets", "cap": 20.0},
        # Odd everything: clips of unequal lengths, heads of 40 channels that begin inside channel blocks.
        {"name": "grad_frames_999_ragged_b6", "kind": "attn_grad", "N": 6, "H": 999, "W": 1, "heads": 6, "kv_heads": 3, "D": 40, "Cb": 8,
         "mask": "lengths", "bias": "buckets", "cap": 0.0},
    ]


# ---------------------------------------------------------------------------------------------------- drawn cases

MAX_NORM = 16e6        # values of a drawn norm's tensor; the largest listed one has 51e6
MAX_PAIRS = 200e6      # query-key pairs times heads of a drawn attention; the largest listed one has 537e6
MAX_MACS = 12e9        # multiply-adds of one of its products; the largest listed one has 34e9
MAX_CACHE = 100e6      # values of a drawn cache; the largest listed one has 537e6


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _heads(rng):
    D = rng.choice([16, 16, 32, 32, 40, 64, 64, 64, 80, 128])
    kv, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 4])
    Cb = rng.choice([16, 16, kv * D, 8]) if D % 16 == 0 else rng.choice([8, kv * D])
    return {"heads": kv * group, "kv_heads": kv, "D": D, "Cb": Cb}


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "attn", "attn", "token", "token", "attn_grad", "attn_grad"])
    if kind.startswith("norm"):
        C = rng.choice([4, 10, 16, 32, 48, 64, 96, 128, 160, 256, 320, 512])
        H, W, N = _log(rng, 1, 120), _log(rng, 1, 120), _log(rng, 1, 1024)
        N = max(1, min(N, int(MAX_NORM // (C * H * W))))
        if kind == "norm_grad":                              # (with a few values in a group every gradient is nearly zero: rounding alone)
            H, W = max(H, 4), max(W, 4)
            N = max(1, min(N, int(MAX_NORM // (C * H * W))))
        G = rng.choice([g for g in range(1, C + 1) if C % g == 0])
        return {"kind": kind, "N": N, "C": C, "H": H, "W": W, "G": G, "act": rng.choice(["none", "relu", "silu", "silu"]),
                "Cb": rng.choice([min(16, C), min(16, C), C])}
    c = {"kind": kind, **_heads(rng)}
    c["cap"] = rng.choice([0.0, 0.0, 15.0, 50.0])
    if kind == "token":
        Sk = _log(rng, 1, 32768)
        most = int(MAX_CACHE // (2 * Sk * c["kv_heads"] * c["D"]))
        N = max(1, min(_log(rng, 1, 256), most))
        return {**c, "N": N, "Sk": Sk, "bias": rng.choice(["none", "slopes", "buckets"]), "ragged": rng.random() < 0.7}
    least = 4 if kind == "attn_grad" else 1                  # (likewise with a key or two)
    if rng.random() < 0.4:                                   # an image
        H, W = _log(rng, least, 40), _log(rng, least, 40)
        mask, bias = "none", rng.choice(["none", "pixels", "pixels"])
    else:                                                    # a sequence
        H, W = _log(rng, least * least, 4096), 1
        mask, bias = rng.choice(["none", "causal", "prefix", "documents", "lengths"]), rng.choice(["none", "slopes", "buckets", "buckets"])
    S = H * W
    most = min(MAX_PAIRS / (S * S * c["heads"]), MAX_MACS / (S * S * c["heads"] * c["D"]))
    c = {**c, "N": max(1, min(_log(rng, 1, 256), int(most))), "H": H, "W": W, "mask": mask, "bias": bias}
    if mask == "documents":
        c["documents"] = rng.randint(1, max(1, min(9, S // 8)))
    return c


# ---------------------------------------------------------------------------------------------------- inputs

REACH, BUCKETS = 512, 32       # of the biases by buckets: offsets beyond the reach are in its last bucket


def log_buckets(reach, buckets):
    """The bucket of each offset -reach .. reach of a key against its query: half of the buckets for keys behind the query, half for
    those at or before it; of each half one half for single offsets, the other for offsets that grow by a constant factor."""
    half = buckets // 2
    single = half // 2
    edges = [single * (reach / single) ** (k / (half - single)) for k in range(half - single)]
    found = []
    for r in range(-reach, reach + 1):
        d = abs(r)
        b = d if d < single else single - 1 + sum(d >= e for e in edges)
        found.append(b + (half if r > 0 else 0))
    return found


def _lengths(case):
    """Lengths spread evenly from a short one to all of it; the seed says which image has which."""
    N, S = case["N"], case["Sk"] if case["kind"] == "token" else case["H"] * case["W"]
    if case["kind"] == "token" and not case["ragged"]:
        return [S] * N
    low = max(1, S // 8)
    return [S - (S - low) * n // max(1, N) for n in range(N)]


def _documents(case):
    """Uneven document lengths that leave a sixteenth of the sequence as padding; the seed says in which order they stand."""
    S, n = case["H"] * case["W"], case["documents"]
    used = S - S // 16
    weights = [1 + k for k in range(n)]
    sizes = [used * w // sum(weights) for w in weights]
    sizes[-1] += used - sum(sizes)
    return sizes


def _prefixes(case):
    S = case["H"] * case["W"]
    return [1 + (S // 3) * (n + 1) // case["N"] for n in range(case["N"])]


def _bias_size(case):
    """(buckets, reach, width) of the learned bias."""
    if case["bias"] == "pixels":
        H, W = case["H"], case["W"]
        reach = (H - 1) * (2 * W - 1) + W - 1
        return 2 * reach + 1, reach, W
    return BUCKETS, REACH, 1


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    order = random.Random(int(seed))
    rand = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    N = case["N"]
    if case["kind"].startswith("norm"):
        C, Cb, S = case["C"], case["Cb"], case["H"] * case["W"]
        # feature maps behind a convolution: channels with means and sizes of their own
        x = rand(N, C // Cb, S, Cb).mul_(1 + rand(C // Cb, 1, Cb).abs()).add_(rand(C // Cb, 1, Cb))
        return {**case, "x": x, "gamma": 1 + 0.2 * rand(C), "beta": 0.3 * rand(C), "eps": 1e-5,
                "dout": rand(N, C // Cb, S, Cb) if case["kind"] == "norm_grad" else None}
    heads, kv, D, Cb = case["heads"], case["kv_heads"], case["D"], case["Cb"]
    state = {**case, "scale": 1 / math.sqrt(D), "lengths": None, "first": None, "prefix": None, "docs": None,
             "slopes": None, "table": None, "bucket": None, "reach": 0, "width": 1, "dout": None}
    nq, nk = heads * D // Cb, kv * D // Cb
    if case["kind"] == "token":
        # a cache as it stands: as many tokens as each stream has come to, and what earlier streams left behind them
        Sq, Sk = 1, case["Sk"]
        state["q"], state["k"], state["v"] = rand(N, nq, 1, Cb), rand(N, nk, Sk, Cb), rand(N, nk, Sk, Cb)
        lengths = _lengths(case)
        order.shuffle(lengths)
        state["lengths"] = ints(lengths)
        state["first"] = state["lengths"] - 1
        state["causal"] = True
    else:
        # the three parts of one projection's output
        Sq = Sk = case["H"] * case["W"]
        qkv = rand(N, nq + 2 * nk, Sk, Cb)
        state["q"], state["k"], state["v"] = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
        state["causal"] = case["mask"] in ("causal", "prefix")
        if case["mask"] == "lengths":
            lengths = _lengths(case)
            order.shuffle(lengths)
            state["lengths"] = ints(lengths)
        if case["mask"] == "prefix":
            prefix = _prefixes(case)
            order.shuffle(prefix)
            state["prefix"] = ints(prefix)
        if case["mask"] == "documents":
            rows = []
            for _ in range(N):
                sizes = _documents(case)
                order.shuffle(sizes)
                rows.append([k for k, n in enumerate(sizes) for _ in range(n)] + [-1] * (Sk - sum(sizes)))
            state["docs"] = ints(rows)
    if case["bias"] == "slopes":
        state["slopes"] = torch.tensor([2.0 ** (-8 * (h + 1) / heads) for h in range(heads)], device=DEV)
    elif case["bias"] != "none":
        buckets, state["reach"], state["width"] = _bias_size(case)
        state["table"] = 0.5 * rand(heads, buckets)
        state["bucket"] = ints(list(range(buckets)) if case["bias"] == "pixels" else log_buckets(REACH, BUCKETS))
    if case["kind"] == "attn_grad":
        state["dout"] = rand(N, nq, Sq, Cb)
    return state


# ---------------------------------------------------------------------------------------------------- the operators

def run(state):
    if own:
        return _own_norm(state) if state["kind"].startswith("norm") else _own_attention(state)
    return _plain_norm(state) if state["kind"].startswith("norm") else _plain_attention(state)


def _own_norm(s):
    import paper_2303_04769_amd as S
    if "plan" not in s:
        s["plan"] = S.GroupNorm(s["N"], s["C"], s["H"], s["W"], s["G"], eps=s["eps"], act=s["act"], Cb=s["Cb"])
    x, out, stats = s["x"], torch.empty_like(s["x"]), torch.empty(s["N"], s["G"], 2, device=DEV)
    s["plan"].run(x, s["gamma"], s["beta"], out, stats)
    if s["dout"] is None:
        return {"out": out, "stats": stats}
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    s["plan"].grad(x, s["gamma"], s["beta"], stats, s["dout"], dx, dgamma, dbeta)
    return {"out": out, "stats": stats, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _own_attention(s):
    import paper_2303_04769_amd as S
    q, k, v = s["q"], s["k"], s["v"]
    if "plan" not in s:
        s["plan"] = S.Attention(s["N"], q.shape[2], k.shape[2], s["heads"], s["kv_heads"], s["D"], Cb=s["Cb"], scale=s["scale"],
                                cap=s["cap"], causal=s["causal"], reach=s["reach"], width=s["width"],
                                buckets=0 if s["table"] is None else s["table"].shape[1])
    masks = {n: s[n] for n in ("lengths", "first", "prefix", "docs", "slopes", "table", "bucket")}
    out = torch.empty(q.shape, device=DEV)
    if s["kind"] == "token":
        s["plan"].run(q, k, v, out, **masks)
        return {"out": out}
    lse = torch.empty(s["N"], s["heads"], q.shape[2], device=DEV)
    s["plan"].run(q, k, v, out, lse, **masks)
    if s["dout"] is None:
        return {"out": out, "lse": lse}
    dq, dk, dv = torch.empty(q.shape, device=DEV), torch.empty(k.shape, device=DEV), torch.empty(v.shape, device=DEV)
    dtable = None if s["table"] is None else torch.empty_like(s["table"])
    s["plan"].grad(q, k, v, out, lse, s["dout"], dq, dk, dv, dtable, **masks)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv, **({} if dtable is None else {"dtable": dtable})}


def _sigmoid(z):
    return 1 / (1 + torch.exp(-z))


def _plain_norm(s):
    N, C, G, Cb, S = s["N"], s["C"], s["G"], s["Cb"], s["H"] * s["W"]
    groups = lambda t: t.permute(0, 1, 3, 2).reshape(N, G, C // G, S)  # noqa: E731
    blocked = lambda t: t.reshape(N, C // Cb, Cb, S).permute(0, 1, 3, 2).contiguous()  # noqa: E731
    x, gamma, beta = groups(s["x"]), s["gamma"].reshape(G, C // G, 1), s["beta"].reshape(G, C // G, 1)
    mean = x.mean((2, 3), keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean((2, 3), keepdim=True) + s["eps"])
    xhat = d * rstd
    z = xhat * gamma + beta
    out = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0), "silu": lambda: z * _sigmoid(z)}[s["act"]]()
    result = {"out": blocked(out), "stats": torch.stack((mean.reshape(N, G), rstd.reshape(N, G)), 2)}
    if s["dout"] is None:
        return result
    dz = groups(s["dout"])
    if s["act"] == "relu":
        dz = torch.where(z > 0, dz, 0.0)
    elif s["act"] == "silu":
        y = _sigmoid(z)
        dz = dz * (y * (1 + z * (1 - y)))
    dxhat = dz * gamma
    a, b = dxhat.mean((2, 3), keepdim=True), (dxhat * xhat).mean((2, 3), keepdim=True)
    return {**result, "dx": blocked(rstd * (dxhat - a - xhat * b)), "dgamma": (dz * xhat).sum((0, 3)).reshape(C), "dbeta": dz.sum((0, 3)).reshape(C)}


def _plain_attention(s):
    N, heads, kv, D, Cb = s["N"], s["heads"], s["kv_heads"], s["D"], s["Cb"]
    group = heads // kv
    # [N][C/Cb][S][Cb] -> [N][heads][S][D] and back
    split = lambda t, h: t.permute(0, 1, 3, 2).reshape(N, h, D, t.shape[2]).transpose(2, 3).contiguous()  # noqa: E731
    merge = lambda t: t.transpose(2, 3).reshape(N, -1, Cb, t.shape[2]).permute(0, 1, 3, 2).contiguous()  # noqa: E731
    q, k, v = split(s["q"], heads), split(s["k"], kv), split(s["v"], kv)
    Sq, Sk = q.shape[2], k.shape[2]
    kg, vg = k, v
    if group > 1:
        kg, vg = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = torch.matmul(q, kg.transpose(2, 3)) * s["scale"]
    if s["cap"]:
        t = torch.tanh(x / s["cap"])
        x = t * s["cap"]
    j = torch.arange(Sk, device=DEV)
    first = s["first"] if s["first"] is not None else torch.full((N,), Sk - Sq, device=DEV)
    pos = first.reshape(N, 1) + torch.arange(Sq, device=DEV)                        # [N][Sq]
    if s["slopes"] is not None:
        x = x - s["slopes"].reshape(heads, 1, 1) * (pos[:, None, :, None] - j).abs()
    index = None
    if s["table"] is not None:
        W = s["width"]
        code = lambda p: torch.div(p, W, rounding_mode="floor") * (2 * W - 1) + p % W  # noqa: E731
        rows = pos if s["first"] is not None else pos[:1]
        index = s["bucket"][(code(j) - code(rows)[:, :, None]).clamp(-s["reach"], s["reach"]) + s["reach"]].long()   # [N or 1][Sq][Sk]
        x = x + s["table"][:, index].transpose(0, 1)
    seen = None
    if s["causal"]:
        seen = j <= pos[:, :, None]
        if s["prefix"] is not None:
            seen = seen | (j < s["prefix"].reshape(N, 1, 1))
    if s["lengths"] is not None:
        there = (j < s["lengths"].reshape(N, 1))[:, None]
        seen = there if seen is None else seen & there
    if s["docs"] is not None:
        same = (s["docs"][:, :, None] == s["docs"][:, None, :]) & (s["docs"][:, None, :] >= 0)
        seen = same if seen is None else seen & same
    if seen is not None:
        x = torch.where(seen[:, None], x, -math.inf)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = torch.matmul(p, vg)
    if s["kind"] == "token":
        return {"out": merge(out)}
    result = {"out": merge(out), "lse": (top + torch.log(total)).squeeze(3)}
    if s["dout"] is None:
        return result
    dout = split(s["dout"], heads)
    fold = lambda t: t.reshape(N, kv, group, Sk, D).sum(2) if group > 1 else t  # noqa: E731
    dv = fold(torch.matmul(p.transpose(2, 3), dout))
    ds = p * (torch.matmul(dout, vg.transpose(2, 3)) - (dout * out).sum(3, keepdim=True))
    if index is not None:
        by = ds.sum(0).reshape(heads, -1)                    # (one index for all images: no case here has positions of its own)
        result["dtable"] = torch.zeros_like(s["table"]).index_add_(1, index.reshape(-1), by)
    if s["cap"]:
        ds = ds * (1 - t * t)
    ds = ds * s["scale"]
    return {**result, "dq": merge(torch.matmul(ds, kg)), "dk": merge(fold(torch.matmul(ds.transpose(2, 3), q))), "dv": merge(dv)}


# ---------------------------------------------------------------------------------------------------- work

def _pairs(case):
    """Query-key pairs that see each other, over all images, for one head."""
    N = case["N"]
    if case["kind"] == "token":
        return sum(_lengths(case))
    S = case["H"] * case["W"]
    if case["mask"] == "causal":
        return N * S * (S + 1) // 2
    if case["mask"] == "prefix":
        return sum(p * p + (S * (S + 1) - p * (p + 1)) // 2 for p in _prefixes(case))
    if case["mask"] == "documents":
        return N * sum(n * n for n in _documents(case))
    if case["mask"] == "lengths":
        return sum(n * S for n in _lengths(case))
    return N * S * S


def work(case):
    N = case["N"]
    if case["kind"].startswith("norm"):
        n = N * case["C"] * case["H"] * case["W"]
        if case["kind"] == "norm":
            return {"bytes": 4 * (2 * n + 2 * case["C"] + 2 * N * case["G"]), "flops": 10 * n}
        return {"bytes": 4 * (4 * n + 4 * case["C"] + 2 * N * case["G"]), "flops": 30 * n}
    Sq, Sk = (1, case["Sk"]) if case["kind"] == "token" else (case["H"] * case["W"],) * 2
    rows, pairs = case["heads"] * case["D"], _pairs(case)
    keys = sum(_lengths(case)) if case["kind"] == "token" or case["mask"] == "lengths" else N * Sk
    table = 0 if case["bias"] in ("none", "slopes") else case["heads"] * _bias_size(case)[0]
    forward = {"bytes": 4 * (2 * N * Sq * rows + 2 * keys * case["kv_heads"] * case["D"] + table), "flops": 4 * pairs * rows}
    if case["kind"] != "attn_grad":
        return forward
    # q, k, v, dout in; out, lse, dq, dk, dv and the table's gradient out; two products forward, five backward
    return {"bytes": 4 * (4 * N * Sq * rows + N * Sq * case["heads"] + 4 * N * Sk * case["kv_heads"] * case["D"] + 2 * table), "flops": 14 * pairs * rows}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(s) if case["kind"].startswith("norm") else _exact_attention(s)


def _exact_norm(s):
    """Image by image, the gradients by automatic differentiation."""
    N, C, G, Cb, S = s["N"], s["C"], s["G"], s["Cb"], s["H"] * s["W"]
    grad = s["dout"] is not None
    if N > 300 and grad:
        return None                                          # (an image at a time takes too long)
    per = max(1, min(N, 64) if not grad else 8)
    gamma, beta = (s[n].double().requires_grad_(grad) for n in ("gamma", "beta"))
    outs, stats, dxs = [], [], []
    for n in range(0, N, per):
        x = s["x"][n:n + per].double().requires_grad_(grad)
        B = x.shape[0]
        c = x.transpose(2, 3).reshape(B, G, -1)
        var, mean = torch.var_mean(c, 2, unbiased=False)
        rstd = (var + s["eps"]) ** -0.5
        z = ((c - mean[..., None]) * rstd[..., None]).reshape(B, C, S) * gamma[:, None] + beta[:, None]
        y = z if s["act"] == "none" else z.clamp(min=0) if s["act"] == "relu" else z * torch.special.expit(z)
        y = y.reshape(B, C // Cb, Cb, S).transpose(2, 3)
        if grad:
            y.backward(s["dout"][n:n + per].double())
            dxs.append(x.grad)
        outs.append(y.detach().contiguous())
        stats.append(torch.stack((mean.detach(), rstd.detach()), 2))
    result = {"out": torch.cat(outs), "stats": torch.cat(stats)}
    return {**result, "dx": torch.cat(dxs), "dgamma": gamma.grad, "dbeta": beta.grad} if grad else result


def _exact_attention(s):
    """Key head by key head of every image (query heads and their table rows beside it), the gradients by automatic differentiation."""
    N, heads, kv, D = s["N"], s["heads"], s["kv_heads"], s["D"]
    group, Sq, Sk = heads // kv, s["q"].shape[2], s["k"].shape[2]
    grad = s["dout"] is not None
    if N * kv > 1100:
        return None                                          # (takes too long)
    plain = lambda t: t.double().transpose(2, 3).reshape(N, -1, t.shape[2])  # noqa: E731  [N][C][S]
    q, k, v = plain(s["q"]), plain(s["k"]), plain(s["v"])
    dout = plain(s["dout"]) if grad else None
    out = torch.empty_like(q)
    lse = torch.empty(N, heads, Sq, dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    dtable = None if s["table"] is None else torch.zeros_like(s["table"], dtype=torch.float64)
    key = torch.arange(Sk, device=DEV)[None, :]
    W, R = s["width"], s["reach"]
    for n in range(N):
        start = Sk - Sq if s["first"] is None else int(s["first"][n])
        at = start + torch.arange(Sq, device=DEV)[:, None]
        hidden = torch.zeros(Sq, Sk, dtype=torch.bool, device=DEV)
        if s["causal"]:
            hidden |= (key > at) & (key >= (0 if s["prefix"] is None else int(s["prefix"][n])))
        if s["lengths"] is not None:
            hidden |= key >= int(s["lengths"][n])
        if s["docs"] is not None:
            hidden |= (s["docs"][n][None, :] != s["docs"][n][at]) | (s["docs"][n][None, :] < 0)
        if s["table"] is not None:
            # rows and columns between the two pixels
            r = (key // W - at // W) * (2 * W - 1) + key % W - at % W
            bucket = s["bucket"].long()[r.clamp(-R, R) + R]
        for h in range(kv):
            rows = slice(h * group, (h + 1) * group)
            qh = q[n].view(heads, D, Sq)[rows].requires_grad_(grad)
            kh, vh = (t[n].view(kv, D, Sk)[h].clone().requires_grad_(grad) for t in (k, v))
            x = s["scale"] * torch.matmul(qh.transpose(1, 2).reshape(group * Sq, D), kh).view(group, Sq, Sk)
            if s["cap"]:
                x = s["cap"] * torch.tanh(x / s["cap"])
            if s["slopes"] is not None:
                x = x - s["slopes"].double()[rows].view(group, 1, 1) * (key - at).abs()
            if s["table"] is not None:
                th = s["table"].double()[rows].clone().requires_grad_(grad)
                x = x + th[:, bucket]
            x = x.masked_fill(hidden, -math.inf)
            empty = hidden.all(1)
            l = torch.logsumexp(x.masked_fill(empty[None, :, None], 0.0), 2)
            p = torch.exp(x - l[..., None])
            o = torch.matmul(p.reshape(group * Sq, Sk), vh.t()).view(group, Sq, D).transpose(1, 2)
            if grad:
                o.backward(dout[n].view(heads, D, Sq)[rows])
                dq[n].view(heads, D, Sq)[rows] = qh.grad
                dk[n].view(kv, D, Sk)[h], dv[n].view(kv, D, Sk)[h] = kh.grad, vh.grad
                if s["table"] is not None:
                    dtable[rows] += th.grad
            out[n].view(heads, D, Sq)[rows] = o.detach()
            lse[n, rows] = l.detach().masked_fill(empty, -math.inf)
    blocked = lambda t: t.view(N, -1, s["Cb"], t.shape[2]).transpose(2, 3).contiguous()  # noqa: E731
    result = {"out": blocked(out)}
    if s["kind"] != "token":
        result["lse"] = lse
    if grad:
        result |= {"dq": blocked(dq), "dk": blocked(dk), "dv": blocked(dv), **({} if dtable is None else {"dtable": dtable})}
    return result
