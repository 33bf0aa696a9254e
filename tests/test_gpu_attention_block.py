"""The attention block put together from the library's layers: outputs against 64 bits, gradients against differences of them, a sequence in
pieces and frame by frame against the whole.

Tolerances: a 1x1 convolution over K channels is within 1e-4 (sqrt(K) max + 1) by the rule of the other layers' tests; the block chains
two of them (K <= 96 here), a normalization and a softmax, whose errors are below 1e-5, so 2e-4 (sqrt(96) + 1) = 2.2e-3 of the largest value
bounds it. Central differences of step 1e-4 in 64 bits are exact to 1e-7 of the loss' third derivative, far below that.
"""
import pytest
import torch

from paper_2303_04769_amd import attn as A
from paper_2303_04769_amd import attention_block as AB

pytestmark = pytest.mark.gpu
TOL = 2.2e-3


def uniform(gen, *shape, of=1.0):
    return torch.rand(*shape, generator=gen, dtype=torch.float64) * (2 * of) - of


def norm64(x, gamma, beta, G, eps=1e-5):
    """x: [N][S][C], one group's statistics over all S."""
    N, S, Cc = x.shape
    g = x.view(N, S, G, Cc // G)
    mean = g.mean((1, 3), keepdim=True)
    var = ((g - mean) ** 2).mean((1, 3), keepdim=True)
    z = ((g - mean) / torch.sqrt(var + eps)).view(N, S, Cc) * gamma + beta
    return z * torch.sigmoid(z)


def attention64(qkv, heads, kv_heads, D, bias, cap, seen=None):
    N, S, _ = qkv.shape
    q, k, v = qkv.split([heads * D, kv_heads * D, kv_heads * D], 2)
    q = q.view(N, S, heads, D).transpose(1, 2)
    k, v = (t.view(N, S, kv_heads, D).transpose(1, 2).repeat_interleave(heads // kv_heads, 1) for t in (k, v))
    s = q @ k.transpose(2, 3) * D ** -0.5
    if cap:
        s = cap * torch.tanh(s / cap)
    s = s + bias
    if seen is not None:
        s = s.masked_fill(~seen, float("-inf"))
    return (torch.softmax(s, -1) @ v).transpose(1, 2).reshape(N, S, heads * D)


def blocked(x, Cb):
    N, S, Cc = x.shape
    return x.view(N, S, Cc // Cb, Cb).transpose(1, 2).float().contiguous().cuda()


def plain(x):
    N, b, S, Cb = x.shape
    return x.cpu().double().transpose(1, 2).reshape(N, S, b * Cb)


def close(got, want, what):
    assert float((got.cpu().double() - want).abs().max()) <= TOL * (1 + float(want.abs().max())), what


@pytest.mark.parametrize("N,Cc,H,W,G,heads,kv_heads,D,cap,Cb", [(2, 32, 5, 3, 4, 2, 1, 16, 0.0, 16), (3, 48, 1, 1, 3, 3, 3, 16, 5.0, 16),
                                                               (1, 96, 9, 7, 8, 4, 2, 24, 2.0, 8)])
def test_image_block(N, Cc, H, W, G, heads, kv_heads, D, cap, Cb):
    gen = torch.Generator().manual_seed(N * Cc + H)
    Cqkv = (heads + 2 * kv_heads) * D
    w_in, w_out = uniform(gen, Cqkv, Cc, of=Cc ** -0.5).float().double(), uniform(gen, Cc, heads * D, of=(heads * D) ** -0.5).float().double()
    block = AB.ImageBlock(w_in.float().cuda(), w_out.float().cuda(), N, Cc, H, W, G, heads, kv_heads, D, cap=cap, Cb=Cb)
    x, gamma, beta, table, dout = (t.float().double() for t in (uniform(gen, N, H * W, Cc), 1 + uniform(gen, Cc, of=0.3), uniform(gen, Cc, of=0.3),
                                                                uniform(gen, heads, block.buckets), uniform(gen, N, H * W, Cc)))
    rows, cols = torch.arange(H * W) // W, torch.arange(H * W) % W
    at = (rows[None] - rows[:, None]) * (2 * W - 1) + cols[None] - cols[:, None] + block.attention.record.reach

    def run(x, gamma, beta, table):
        h = norm64(x, gamma, beta, G)
        return x + attention64(h @ w_in.t(), heads, kv_heads, D, table[:, at], cap) @ w_out.t()

    args = [x, gamma, beta, table]
    on = [blocked(x, Cb)] + [t.float().cuda() for t in args[1:]]
    close(plain(block.forward(*on)), run(*args), "out")
    grads = block.grad(*on, blocked(dout, Cb))
    grads = [plain(grads[0])] + [g.cpu().double() for g in grads[1:]]
    for i, g in enumerate(grads):
        way = uniform(gen, *args[i].shape)
        ends = [float((run(*[a + t * way if j == i else a for j, a in enumerate(args)]) * dout).sum()) for t in (1e-4, -1e-4)]
        want = (ends[0] - ends[1]) / 2e-4
        assert abs(float((g * way).sum()) - want) <= TOL * (1 + float((g * way).abs().sum())), ("inp", "gamma", "beta", "table")[i]


@pytest.mark.parametrize("pieces", [[37], [20, 17], [36, 1], [1] * 5 + [31, 1]])
def test_frame_block(pieces):
    N, Cc, G, heads, kv_heads, D, cap, room = 3, 48, 4, 4, 2, 16, 6.0, 40
    S = sum(pieces)
    gen = torch.Generator().manual_seed(S + len(pieces))
    Cqkv = (heads + 2 * kv_heads) * D
    w_in, w_out = uniform(gen, Cqkv, Cc, of=Cc ** -0.5).float().double(), uniform(gen, Cc, heads * D, of=(heads * D) ** -0.5).float().double()
    bucket, buckets, reach = A.log_buckets(12, 8, both=False)
    x, gamma, beta, table = (t.float().double() for t in (uniform(gen, N, S, Cc), 1 + uniform(gen, Cc, of=0.3), uniform(gen, Cc, of=0.3),
                                                          uniform(gen, heads, buckets)))
    block = AB.FrameBlock(w_in.float().cuda(), w_out.float().cuda(), gamma.float().cuda(), beta.float().cuda(), table.float().cuda(), bucket.cuda(),
                          N, room, Cc, G, heads, kv_heads, D, cap=cap)
    got, at = [], 0
    for n in pieces:
        got.append(block.forward(x[:, at:at + n].float().contiguous().cuda()))
        at += n
    off = torch.arange(S)[None] - torch.arange(S)[:, None]
    bias = table[:, bucket.long()[off.clamp(-reach, reach) + reach]]
    h = norm64(x.view(N * S, 1, Cc), gamma, beta, G).view(N, S, Cc)
    want = x + attention64(h @ w_in.t(), heads, kv_heads, D, bias, cap, seen=off <= 0) @ w_out.t()
    close(torch.cat(got, 1), want, pieces)
    with pytest.raises(ValueError):
        block.forward(torch.zeros(N, room, Cc, device="cuda"))


def test_image_block_refuses_filters():
    w = torch.zeros(8, 8, device="cuda")
    with pytest.raises(ValueError):
        AB.ImageBlock(w, w, 1, 16, 2, 2, 4, 1, 1, 16)
