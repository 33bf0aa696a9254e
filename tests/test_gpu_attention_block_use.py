"""The attention block in use: what it keeps, and what it refuses."""
import pytest
import torch

from paper_2303_04769_amd import attn as A
from paper_2303_04769_amd import attention_block as AB

pytestmark = pytest.mark.gpu


def frame_block(room, N=2, Cc=32, heads=2, kv_heads=1, D=16):
    gen = torch.Generator().manual_seed(7)
    r = lambda *s: (torch.rand(*s, generator=gen) - 0.5).cuda()  # noqa: E731
    bucket, buckets, _ = A.log_buckets(12, 8, both=False)
    return AB.FrameBlock(r((heads + 2 * kv_heads) * D, Cc), r(Cc, heads * D), 1 + r(Cc), r(Cc), r(heads, buckets), bucket.cuda(), N, room, Cc, 4, heads, kv_heads, D)


def test_a_sequence_in_many_pieces_keeps_few_plans():
    """Pieces of different sizes, each at a length of its own, and single frames between them: the same as at once (its tolerance: two runs of the same layers, each within
    1.1e-3 of 64 bits by the rule of test_gpu_attention_block.py), and no more is kept than the last few plans."""
    frames = torch.rand(2, 60, 32, generator=torch.Generator().manual_seed(8)).cuda()
    want = frame_block(60).forward(frames)
    block, got, at = frame_block(60), [], 0
    for n in [2, 3, 1, 4, 5, 1, 6, 7, 1, 8, 9, 1, 12]:
        got.append(block.forward(frames[:, at:at + n].contiguous()))
        at += n
        assert len(block._plans) <= AB.KEPT_PLANS
    assert at == 60 and float((torch.cat(got, 1) - want).abs().max()) <= 2.2e-3 * (1 + float(want.abs().max()))


def test_tensors_of_other_sizes_are_refused():
    """Group normalization reads as many values as its plan says, the blocks as many images, frames and channels: a tensor that has others is refused before anything
    is enqueued, by the extension's calls and by those with a stream."""
    import paper_2303_04769_amd as S
    plan = S.GroupNorm(2, 32, 4, 4, 4)
    e = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    x, c, st = e(2, 2, 16, 16), e(32), e(2, 4, 2)
    for stream in (None, torch.cuda.current_stream()):
        plan.run(x, c, c, e(2, 2, 16, 16), st, stream=stream)
        plan.grad(x, c, c, st, x, e(2, 2, 16, 16), e(32), e(32), stream=stream)
        for at in range(5):
            args = [x, c, c, e(2, 2, 16, 16), st]
            args[at] = args[at][:1].contiguous()
            with pytest.raises(TypeError):
                plan.run(*args, stream=stream)
        for at in range(8):
            args = [x, c, c, st, x, e(2, 2, 16, 16), e(32), e(32)]
            args[at] = args[at][:1].contiguous()
            with pytest.raises(TypeError):
                plan.grad(*args, stream=stream)
    block = frame_block(8)
    for shape in ((1, 3, 32), (2, 3, 16), (3, 3, 32)):
        with pytest.raises(ValueError):
            block.forward(e(*shape))
    with pytest.raises(ValueError):
        AB.FrameBlock(e(48, 32), e(32, 32), c, c, e(2, 8), e(25).int(), 2, 8, 32, 4, 2, 1, 16)
    with pytest.raises(ValueError):
        AB.FrameBlock(e(64, 32), e(32, 48), c, c, e(2, 8), e(25).int(), 2, 8, 32, 4, 2, 1, 16)
    image = AB.ImageBlock(e(64, 32), e(32, 32), 2, 32, 3, 4, 4, 2, 1, 16)
    with pytest.raises(ValueError):
        image.forward(e(1, 2, 12, 16), c, c, e(2, image.buckets))
    out = image.forward(e(2, 2, 12, 16), c, c, e(2, image.buckets))
    with pytest.raises(ValueError):
        image.grad(e(2, 2, 12, 16), c, c, e(2, image.buckets), out[:1].contiguous())
