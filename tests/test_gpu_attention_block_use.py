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
