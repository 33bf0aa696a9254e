"""The attention block of a convolutional network put together from the library's layers:

    out = in + conv1x1(attention(q, k, v)),   (q, k, v) = conv1x1(silu(groupnorm(in)))

ImageBlock runs it over the pixels of feature maps with a learned bias for every offset of rows and columns, and takes the gradients of its input,
gamma, beta and the bias table through frozen filters (the data gradient of a 1x1 convolution is a 1x1 convolution with the transposed filter).
FrameBlock runs it over the frames of sequences, causally and with a bias over distances: a whole sequence at once, or frame by frame
on a cache of the keys and values that were seen.

    python -m paper_2303_04769_amd.attention_block        trains the first for a few steps, compares both ways through the second

Everything is enqueued on torch's current stream; tensors are float32, activations channel-blocked. No arithmetic of the layers happens here.
"""
import time

import torch

from . import attn as A
from . import binding as B


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
    """The block over N images of H x W pixels and Cc channels. w_in: [(heads + 2 kv_heads) D][Cc], w_out: [Cc][heads D], frozen."""

    def __init__(self, w_in, w_out, N, Cc, H, W, G, heads, kv_heads, D, cap=0.0, Cb=16):
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

    def forward(self, inp, gamma, beta, table):
        """inp: [N][C/Cb][H*W][Cb]; table: [heads][buckets]. Returns the output; what grad needs stays in the block."""
        _shaped(inp, (self.N, self.C // self.Cb, self.H * self.W, self.Cb))
        out = torch.empty_like(inp)
        self.norm.run(inp, gamma, beta, self.h, self.stats)
        self._conv(self.h, self.w_in, self.qkv)
        self.attention.run(*self._parts(self.qkv), self.ctx, lse=self.lse, table=table, bucket=self.bucket)
        self._conv(self.ctx, self.w_out, out)
        B.small_add(out, inp, out, out.numel())
        return out

    def grad(self, inp, gamma, beta, table, dout):
        """Gradients (inp, gamma, beta, table) of the last forward call, which had the same arguments."""
        _shaped(dout, (self.N, self.C // self.Cb, self.H * self.W, self.Cb))
        din, dgamma, dbeta, dtable = (torch.empty_like(t) for t in (inp, gamma, beta, table))
        self._conv(dout, self.w_out_t, self.dctx)
        self.attention.grad(*self._parts(self.qkv), self.ctx, self.lse, self.dctx, *self._parts(self.dqkv), dtable=dtable, table=table,
                            bucket=self.bucket)
        self._conv(self.dqkv, self.w_in_t, self.dh)
        self.norm.grad(inp, gamma, beta, self.stats, self.dh, din, dgamma, dbeta)
        B.small_add(din, dout, din, din.numel())
        return din, dgamma, dbeta, dtable


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


if __name__ == "__main__":
    main()
