"""The attention block of a convolutional network put together from the library's layers:

    out = in + conv1x1(attention(q, k, v)),   (q, k, v) = conv1x1(silu(groupnorm(in)))

ImageBlock runs it over the pixels of feature maps with a learned bias for every offset of rows and columns, or rotary positions of rows and columns, or both, and takes
the gradients of its input, gamma, beta, the bias table and the rotary frequencies through frozen filters (the data gradient of a 1x1 convolution is a 1x1 convolution
with the transposed filter).
FrameBlock runs it over the frames of sequences, causally and with a bias over distances: a whole sequence at once, or frame by frame
on a cache of the keys and values that were seen.
StreamBlock runs it over streams that come and go, each of an age of its own, with rotary positions, on a paged cache that they share: the next frames of each, one or many.

    python -m paper_2303_04769_amd.attention_block        trains the first for a few steps, compares both ways through the second and the third

Everything is enqueued on torch's current stream; tensors are float32, activations channel-blocked. No arithmetic of the layers happens here.
"""
import time

import torch

from . import attn as A
from . import binding as B
from . import cache as K


def _packed(weight, Cib, Cob):
    """Filter [Co][Ci] of a 1x1 convolution, laid out once."""
    Co, Ci = weight.shape
    out = torch.empty(weight.numel(), device=weight.device)
    B.small_pack_filter(weight.contiguous(), out, Co, Ci, 1, 1, Cob, Cib)
    return out


def _shaped(t, shape):
    if tuple(t.shape) != shape:
        raise ValueError(f"expected a tensor {list(shape)}, got {list(t.shape)}")


def _conv1x1(inp, filt, out, N, Ci, Co, H, W, Cib, Cob):
    B.small_conv2d(inp, filt, out, N, Ci, Co, H, W, 1, 1, 1, (0, 0, 0, 0), Cib, Cob)


class ImageBlock:
    """The block over N images of H x W pixels and Cc channels. w_in: [(heads + 2 kv_heads) D][Cc], w_out: [Cc][heads D], frozen. halves: how rotary
    positions pair channels (cache.Rotary)."""

    def __init__(self, w_in, w_out, N, Cc, H, W, G, heads, kv_heads, D, cap=0.0, Cb=16, halves=False):
        self.N, self.C, self.H, self.W, self.Cb = N, Cc, H, W, Cb
        self.Cq, self.Ck = heads * D, kv_heads * D
        self.Cqkv = self.Cq + 2 * self.Ck
        if tuple(w_in.shape) != (self.Cqkv, Cc) or tuple(w_out.shape) != (Cc, self.Cq):
            raise ValueError(f"filters of shapes {tuple(w_in.shape)} and {tuple(w_out.shape)} do not fit {heads} and {kv_heads} heads of {D} and {Cc} channels")
        dev = w_in.device
        self.w_in, self.w_out = _packed(w_in, Cb, Cb), _packed(w_out, Cb, Cb)
        self.w_in_t, self.w_out_t = _packed(w_in.t(), Cb, Cb), _packed(w_out.t(), Cb, Cb)
        bucket, buckets, reach, width = A.pixel_buckets(H, W)
        self.bucket, self.buckets = bucket.to(dev), buckets
        self.norm = A.GroupNorm(N, Cc, H, W, G, act="silu", Cb=Cb, device=dev)
        self.attention = A.Attention(N, H * W, H * W, heads, kv_heads, D, Cb=Cb, cap=cap, width=width, reach=reach, buckets=buckets, device=dev)
        self._turns, self._turn_sizes = {}, (N, H * W, heads, kv_heads, D)
        self.halves = halves
        self.stats = torch.empty(N, G, 2, device=dev)
        self.lse = torch.empty(N, heads, H * W, device=dev)
        self.h, self.qkv, self.ctx = self._empty(Cc), self._empty(self.Cqkv), self._empty(self.Cq)
        self.dh, self.dqkv, self.dctx = self._empty(Cc), self._empty(self.Cqkv), self._empty(self.Cq)

    def _empty(self, Cc):
        return torch.empty(self.N, Cc // self.Cb, self.H * self.W, self.Cb, device=self.w_in.device)

    def _parts(self, t):
        """The queries, keys and values in one projection's output (or in its gradient)."""
        q, k = self.Cq // self.Cb, self.Ck // self.Cb
        return t[:, :q], t[:, q:q + k], t[:, q + k:]

    def _conv(self, inp, filt, out):
        _conv1x1(inp, filt, out, self.N, inp.shape[1] * self.Cb, out.shape[1] * self.Cb, self.H, self.W, self.Cb, self.Cb)

    def _turn(self, freq):
        """The plan of rotary positions with frequencies of this shape."""
        F, axes, pairs = freq.shape
        if (F, axes, pairs) not in self._turns:
            if axes != 2:
                raise ValueError(f"expected frequencies [1 or key heads][2][pairs] for rows and columns, got {list(freq.shape)}")
            self._turns[F, axes, pairs] = K.Rotary(*self._turn_sizes, axes=2, pairs=pairs, halves=self.halves, extent=(self.W,), freq_heads=F, Cb=self.Cb, device=self.w_in.device)
        return self._turns[F, axes, pairs]

    def forward(self, inp, gamma, beta, table=None, freq=None):
        """inp: [N][C/Cb][H*W][Cb]; table: [heads][buckets]; freq: [1 or kv_heads][2][pairs], rotary positions of rows and columns. Returns the output; what grad
        needs stays in the block."""
        _shaped(inp, (self.N, self.C // self.Cb, self.H * self.W, self.Cb))
        out = torch.empty_like(inp)
        self.norm.run(inp, gamma, beta, self.h, self.stats)
        self._conv(self.h, self.w_in, self.qkv)
        if freq is not None:
            self._turn(freq).run(*self._parts(self.qkv)[:2], freq)
        self.attention.run(*self._parts(self.qkv), self.ctx, lse=self.lse, table=table, bucket=None if table is None else self.bucket)
        self._conv(self.ctx, self.w_out, out)
        B.small_add(out, inp, out, out.numel())
        return out

    def grad(self, inp, gamma, beta, table, dout, freq=None):
        """Gradients (inp, gamma, beta, table) of the last forward call, which had the same arguments, and that of freq behind them if there is one (None for a table of None)."""
        _shaped(dout, (self.N, self.C // self.Cb, self.H * self.W, self.Cb))
        din, dgamma, dbeta, dtable, dfreq = (None if t is None else torch.empty_like(t) for t in (inp, gamma, beta, table, freq))
        self._conv(dout, self.w_out_t, self.dctx)
        self.attention.grad(*self._parts(self.qkv), self.ctx, self.lse, self.dctx, *self._parts(self.dqkv), dtable=dtable, table=table,
                            bucket=None if table is None else self.bucket)
        if freq is not None:
            q, k, _ = self._parts(self.qkv)
            dq, dk, _ = self._parts(self.dqkv)
            self._turn(freq).grad(dq, dk, freq, q=q, k=k, dfreq=dfreq)
        self._conv(self.dqkv, self.w_in_t, self.dh)
        self.norm.grad(inp, gamma, beta, self.stats, self.dh, din, dgamma, dbeta)
        B.small_add(din, dout, din, din.numel())
        return (din, dgamma, dbeta, dtable) if freq is None else (din, dgamma, dbeta, dtable, dfreq)


KEPT_PLANS = 4


class FrameBlock:
    """The block over sequences of up to `room` frames, channels last: [N][S][Cc]. Each frame is normalized by itself and sees itself and
    the frames before it. gamma, beta: [Cc]; table, bucket: a bias over distances (log_buckets). To the convolutions the frames are images
    of one pixel, whose channels stand in order whatever their block Cb."""

    def __init__(self, w_in, w_out, gamma, beta, table, bucket, N, room, Cc, G, heads, kv_heads, D, cap=0.0, Cb=16):
        dev = w_in.device
        self.N, self.room, self.C, self.G = N, room, Cc, G
        self.heads, self.kv_heads, self.D, self.cap, self.Cb = heads, kv_heads, D, cap, Cb
        self.Cq, self.Ck = heads * D, kv_heads * D
        _shaped(w_in, (self.Cq + 2 * self.Ck, Cc))
        _shaped(w_out, (Cc, self.Cq))
        self.w_q, self.w_kv = _packed(w_in[:self.Cq], Cb, Cb), _packed(w_in[self.Cq:], Cb, Cb)
        self.w_out = _packed(w_out, Cb, Cb)
        self.gamma, self.beta, self.table, self.bucket = gamma, beta, table, bucket
        self.cache = torch.zeros(N, 1, room, 2 * self.Ck, device=dev)       # keys then values of a frame
        self.length, self._plans = 0, {}

    def _plan(self, S, Sk):
        """What calls of S new frames on Sk in all need (for a single frame: on the whole cache, up to lengths). The last few are kept: a sequence in pieces comes to
        ever new sizes."""
        plan = self._plans.pop((S, Sk), None)
        if plan is None:
            dev, tokens = self.cache.device, self.N * S
            plan = (
                A.GroupNorm(tokens, self.C, 1, 1, self.G, act="silu", Cb=self.C, device=dev),
                A.Attention(self.N, S, Sk, self.heads, self.kv_heads, self.D, Cb=self.D, cap=self.cap, causal=True, reach=self.bucket.numel() // 2,
                            buckets=self.table.shape[1], device=dev),
                torch.empty(tokens, self.C, device=dev), torch.empty(tokens, self.Cq, device=dev), torch.empty(tokens, 2 * self.Ck, device=dev),
                torch.empty(tokens, self.Cq, device=dev),
                torch.empty(self.N, dtype=torch.int32, device=dev), torch.empty(self.N, dtype=torch.int32, device=dev))
            while len(self._plans) >= KEPT_PLANS:
                del self._plans[next(iter(self._plans))]                   # (the one that was not used for longest)
        self._plans[S, Sk] = plan
        return plan

    def _heads(self, t, first, heads):
        """View of `heads` heads from channel `first` on of frames [N][S][channels], each head a block of its own."""
        N, S, ch = t.shape[0], t.shape[1], t.shape[2]
        return t.as_strided((N, heads, S, self.D), (t.stride(0), self.D, t.stride(1), 1), t.storage_offset() + first)

    def forward(self, frames):
        """The next frames [N][S][Cc] of every sequence: their outputs; their keys and values go into the cache."""
        S, start = frames.shape[1], self.length
        _shaped(frames, (self.N, S, self.C))
        if start + S > self.room:
            raise ValueError(f"{start} frames and {S} more do not fit {self.room}")
        Sk = self.room if S == 1 else start + S                            # (one plan for every single frame)
        norm, attention, h, q, kv, ctx, lengths, first = self._plan(S, Sk)
        out = torch.empty_like(frames)
        norm.run(frames, self.gamma, self.beta, h)
        for w, to, channels in ((self.w_q, q, self.Cq), (self.w_kv, kv, 2 * self.Ck)):
            _conv1x1(h, w, to, self.N * S, self.C, channels, 1, 1, self.Cb, self.Cb)
        self.cache[:, 0, start:start + S] = kv.view(self.N, S, -1)
        cache = self.cache[:, 0, :Sk]
        lengths.fill_(start + S)
        first.fill_(start)
        attention.run(self._heads(q.view(self.N, S, -1), 0, self.heads), self._heads(cache, 0, self.kv_heads),
                      self._heads(cache, self.Ck, self.kv_heads), self._heads(ctx.view(self.N, S, -1), 0, self.heads), lengths=lengths, first=first,
                      table=self.table, bucket=self.bucket)
        _conv1x1(ctx, self.w_out, out, self.N * S, self.Cq, self.C, 1, 1, self.Cb, self.Cb)
        B.small_add(out, frames, out, out.numel())
        self.length = start + S
        return out


# Rows of a key head (new frames times the query heads that share it) up to which frames attend to the cache itself. Up to there that is ahead of reading it back for the sequence kernels
# for every kind and head width measured, the further the wider the heads (64 rows on 8 streams of 4096: floats of 32 channels 25 us and 31, of 96 37 and 59, of 256 76 and 130; bfloat16
# of 96 26 and 57; codes 24 and 55). They draw level further on: floats at 256 rows (51 and 50, 92 and 93, 245 and 246), fewer bits beyond (codes of 96 53 and 87).
ROWS_ON_CACHE = 64


class StreamBlock:
    """The block over up to N streams, channels last, with rotary positions (freq: [1 or kv_heads][1][pairs]) and a paged cache of `pages` pages of `page` tokens for all of them,
    `per_stream` of them at most for one; kind: what the cache holds (cache.PagedCache), 8-bit codes unless another is named. Each call brings the next frames of some or all streams; a stream that ends gives its
    pages back. Few new frames attend to the cache itself, many to what is read back from it: the same keys and values, whichever way a stream's frames come in."""

    def __init__(self, w_in, w_out, gamma, beta, freq, N, pages, page, per_stream, Cc, G, heads, kv_heads, D, kind="int8", cap=0.0, halves=True, Cb=16):
        dev = w_in.device
        self.N, self.C, self.G, self.heads, self.kv_heads, self.D, self.cap, self.halves, self.Cb = N, Cc, G, heads, kv_heads, D, cap, halves, Cb
        self.Cq, self.Ck = heads * D, kv_heads * D
        _shaped(w_in, (self.Cq + 2 * self.Ck, Cc))
        _shaped(w_out, (Cc, self.Cq))
        _shaped(gamma, (Cc,))
        _shaped(beta, (Cc,))
        if freq.dim() != 3 or freq.shape[1] != 1:
            raise ValueError(f"expected frequencies [1 or key heads][1][pairs], got {list(freq.shape)}")
        self.w_in, self.w_out = _packed(w_in, Cb, Cb), _packed(w_out, Cb, Cb)
        self.gamma, self.beta, self.freq = gamma, beta, freq
        self.cache = K.PagedCache(pages, page, kv_heads, D, kind=kind, device=dev)
        self.page, self.per_stream = page, per_stream
        self.free, self.held = list(range(pages))[::-1], [[] for _ in range(N)]
        self.lengths = [0] * N
        self.table = torch.full((N, per_stream), -1, dtype=torch.int32, device=dev)
        self._length, self._after = (torch.zeros(N, dtype=torch.int32, device=dev) for _ in range(2))        # before and after the frames of a call
        self._plans = {}

    def _plan(self, S, Sk):
        """What calls of S new frames need; Sk: tokens that are read back (a page of them at least), 0 where the cache is attended to. The last few are kept."""
        plan = self._plans.pop((S, Sk), None)
        if plan is None:
            dev, tokens = self.w_in.device, self.N * S
            e = lambda *shape: torch.empty(*shape, device=dev)  # noqa: E731
            F, _, pairs = self.freq.shape
            attention = A.Attention(self.N, S, Sk, self.heads, self.kv_heads, self.D, Cb=self.D, cap=self.cap, causal=True, device=dev) if Sk else \
                K.CacheAttention(self.cache, self.N, S, self.heads, self.per_stream, Cb=self.D, cap=self.cap, device=dev)
            plan = (A.GroupNorm(tokens, self.C, 1, 1, self.G, act="silu", Cb=self.C, device=dev),
                    K.Rotary(self.N, S, self.heads, self.kv_heads, self.D, pairs=pairs, halves=self.halves, freq_heads=F, Cb=self.D, device=dev), attention,
                    e(tokens, self.C), e(tokens, self.Cq + 2 * self.Ck), e(tokens, self.Cq),
                    (e(self.N, self.kv_heads, Sk, self.D), e(self.N, self.kv_heads, Sk, self.D)) if Sk else None)
            while len(self._plans) >= KEPT_PLANS:
                del self._plans[next(iter(self._plans))]                   # (the one that was not used for longest)
        self._plans[S, Sk] = plan
        return plan

    def _new_pages(self, counts):
        """Pages for so many more frames of each stream, all or none. They are still free."""
        need = [-(-(held + more) // self.page) - len(pages) for held, more, pages in zip(self.lengths, counts, self.held)]
        for n, (held, more) in enumerate(zip(self.lengths, counts)):
            if held + more > self.per_stream * self.page:
                raise ValueError(f"stream {n}: {held} frames and {more} more do not fit {self.per_stream} pages of {self.page}")
        if sum(need) > len(self.free):
            raise ValueError(f"{sum(need)} pages are needed and {len(self.free)} free")
        last_first = iter(self.free[::-1])
        return [[next(last_first) for _ in range(more)] for more in need]

    def release(self, n):
        """Stream n ends: its pages are free, its place is empty for another."""
        self.free += self.held[n][::-1]
        self.held[n] = []
        self.lengths[n] = 0
        self._length[n] = 0
        self.table[n] = -1

    def forward(self, frames, counts=None):
        """The next frames [N][S][Cc], of which stream n has counts[n] (a list; None: S each): their outputs. What stands behind a stream's frames, in and out, is of no
        meaning. A call that raises leaves all streams as they were."""
        S = frames.shape[1]
        _shaped(frames, (self.N, S, self.C))
        if counts is not None and (len(counts) != self.N or not all(0 <= c <= S for c in counts)):
            raise ValueError(f"expected {self.N} numbers of frames in 0 .. {S}, got {counts}")
        more = [S] * self.N if counts is None else [int(c) for c in counts]
        pages, lengths = self._new_pages(more), [a + b for a, b in zip(self.lengths, more)]
        few = S * (self.heads // self.kv_heads) <= ROWS_ON_CACHE
        plan = self._plan(S, 0 if few else max(1, -(-max(lengths) // self.page)) * self.page)
        here = None if counts is None else torch.tensor(more, dtype=torch.int32).to(self._length.device)
        torch.add(self._length, S if here is None else here, out=self._after)
        try:
            for n, new in enumerate(pages):
                if new:
                    at = len(self.held[n])
                    self.table[n, at:at + len(new)] = torch.tensor(new, dtype=torch.int32)
            out = self._layers(frames, here, few, *plan)
        except BaseException:
            for n, new in enumerate(pages):
                if new:
                    self.table[n, len(self.held[n]):] = -1
            raise
        self._length, self._after, self.lengths = self._after, self._length, lengths
        self.held = [held + new for held, new in zip(self.held, pages)]
        del self.free[len(self.free) - sum(map(len, pages)):]
        return out

    def _layers(self, frames, here, few, norm, rotary, attention, h, qkv, ctx, read):
        S, out = frames.shape[1], torch.empty_like(frames)
        norm.run(frames, self.gamma, self.beta, h)
        _conv1x1(h, self.w_in, qkv, self.N * S, self.C, self.Cq + 2 * self.Ck, 1, 1, self.Cb, self.Cb)
        heads = lambda t, first, n: t.as_strided((self.N, n, S, self.D), (S * t.shape[1], self.D, t.shape[1], 1), first)  # noqa: E731
        q, k, v = heads(qkv, 0, self.heads), heads(qkv, self.Cq, self.kv_heads), heads(qkv, self.Cq + self.Ck, self.kv_heads)
        self.cache.write(k, v, self.table, self._length, counts=here, rotary=rotary, freq=self.freq, q=q)
        if few:
            attention.run(q, heads(ctx, 0, self.heads), self.table, self._after, first=self._length)
        else:
            self.cache.read(*read, self.table, counts=self._after)
            attention.run(q, *read, heads(ctx, 0, self.heads), lengths=self._after, first=self._length)
        _conv1x1(ctx, self.w_out, out, self.N * S, self.Cq, self.C, 1, 1, self.Cb, self.Cb)
        B.small_add(out, frames, out, out.numel())
        return out


def _uniform(gen, *shape, of=1.0):
    return (torch.rand(*shape, generator=gen) * (2 * of) - of).cuda()


def main(steps=20):
    gen = torch.Generator().manual_seed(0)
    N, Cc, H, W, G, heads, kv_heads, D = 16, 64, 14, 14, 8, 4, 2, 32
    w_in, w_out = _uniform(gen, (heads + 2 * kv_heads) * D, Cc, of=Cc ** -0.5), _uniform(gen, Cc, heads * D, of=(heads * D) ** -0.5)
    block = ImageBlock(w_in, w_out, N, Cc, H, W, G, heads, kv_heads, D)
    x = _uniform(gen, N, Cc // 16, H * W, 16)
    target = block.forward(x, 1 + _uniform(gen, Cc, of=0.5), _uniform(gen, Cc, of=0.5), _uniform(gen, heads, block.buckets, of=2.0))
    params = [torch.ones(Cc, device="cuda"), torch.zeros(Cc, device="cuda"), torch.zeros(heads, block.buckets, device="cuda")]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for step in range(steps):
        off = block.forward(x, *params) - target
        if step % 5 == 0 or step == steps - 1:
            print(f"step {step:2d}: half the mean squared error {0.5 * float((off * off).mean()):.6f}")
        for p, g in zip(params, block.grad(x, *params, off)[1:]):
            p.sub_(g, alpha=1e-3)
    torch.cuda.synchronize()
    print(f"{steps} steps of {N} images {H} x {W} x {Cc} in {1e3 * (time.perf_counter() - t0):.1f} ms")

    S, room = 100, 160
    bucket, buckets, _ = A.log_buckets(64, 16, both=False)
    table = _uniform(gen, heads, buckets)
    frames = _uniform(gen, 2, room, Cc)
    whole, single = (FrameBlock(w_in, w_out, params[0], params[1], table, bucket.cuda(), 2, room, Cc, G, heads, kv_heads, D, cap=20.0) for _ in range(2))
    at_once = whole.forward(frames)
    in_turn = torch.cat([single.forward(frames[:, :S].contiguous())] + [single.forward(frames[:, i:i + 1].contiguous()) for i in range(S, room)], 1)
    print(f"{room} frames at once, and {S} and then one by one: outputs differ by {float((at_once - in_turn).abs().max()):.1e} at most")

    freq = K.axis_frequencies(D // 2).cuda()
    whole, single = (StreamBlock(w_in, w_out, params[0], params[1], freq, 2, 24, 16, 12, Cc, G, heads, kv_heads, D, cap=20.0) for _ in range(2))
    at_once = whole.forward(frames)
    in_turn = torch.cat([single.forward(frames[:, :S].contiguous())] + [single.forward(frames[:, i:i + 1].contiguous()) for i in range(S, room)], 1)
    print(f"the same on 8-bit pages: outputs differ by {float((at_once - in_turn).abs().max()):.1e} at most")


if __name__ == "__main__":
    main()
