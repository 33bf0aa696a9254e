"""Every form of the attention kernels by its rule, with what tells that it runs: whole sequences on fp16 parts lay keys and values out in the workspace, the others need one
only for split rows. Value by value against 64 bits (test_gpu_attention_masks.py)."""
import pytest
import torch

import paper_2303_04769_amd as S
from test_gpu_attention import Case, _docs, plain
from test_gpu_attention_masks import compare, everything, exact

pytestmark = pytest.mark.gpu


def up(n):
    return (n + 255) // 256 * 256


def workspace(c, grad):
    r = c.plan().record
    if c.table is not None:
        r.table = r.bucket = 256
    return S.small_attention_workspace(r, grad)


def unsplit(c):
    """Enough tiles of 64 rows for two workgroups a compute unit: keys are not split, so only parts need a workspace."""
    return c.N * c.heads * -(-c.Sq // 64) >= 2 * torch.cuda.get_device_properties(0).multi_processor_count


def plain_grad_bytes(c):
    """What a gradient call on fp32 products needs."""
    n = up(8 * c.N * c.heads * c.Sq)
    if c.table is not None:
        size = 2 * c.reach + 1
        n += up(4 * c.N * c.heads * -(-c.Sq // 64) * size) + up(4 * c.heads * size)
    return n


UNSPLIT = {
    "plain": dict(N=16, Sq=260, heads=8, D=32), "odd": dict(N=20, Sq=331, heads=5, D=37, Cb=37), "128 channels": dict(N=16, Sq=270, heads=8, D=128),
    "shared heads": dict(N=16, Sq=260, heads=8, kv=2, D=32), "lengths": dict(N=18, Sq=300, heads=6, D=32, lengths=[0, 1, 64, 65, 299, 300] * 3),
    "documents": dict(N=18, Sq=300, heads=6, D=32, docs=_docs(18, 300, [[3, 60, 70, 100], [150, 150], [300]])),
    "documents out of order": dict(N=18, Sq=300, heads=6, D=32, docs=[[(7 * i) % 4 - (i % 9 == 0) for i in range(300)]] * 18),
    "pixels": dict(N=13, Sq=17 * 16, heads=8, D=32, bias=(17, 16)), "pixels of wide heads": dict(N=13, Sq=17 * 16, heads=8, D=80, bias=(17, 16)),
    "small images": dict(N=80, Sq=196, heads=4, D=32, bias=(14, 14)), "buckets": dict(N=16, Sq=260, heads=8, D=64, bias="log"),
    "buckets, capped": dict(N=16, Sq=260, heads=8, D=64, bias="log", cap=5.0, size=2.0), "distances": dict(N=16, Sq=260, heads=8, D=32, slopes=True),
    "distances, capped": dict(N=16, Sq=260, heads=8, D=16, slopes=True, cap=5.0), "capped": dict(N=16, Sq=260, heads=8, D=16, cap=0.5, size=4.0),
    "causal": dict(N=16, Sq=260, heads=8, D=16, causal=True), "prefix, 96 channels": dict(N=16, Sq=260, heads=8, D=96, causal=True, prefix=[0, 64, 65, 260] * 4),
    "longer keys": dict(N=16, Sq=260, Sk=400, heads=8, D=32, causal=True), "positions of their own": dict(N=16, Sq=260, Sk=300, heads=8, D=32, causal=True, first=[-100, 50, 290, 7] * 4),
}


@pytest.mark.parametrize("name", UNSPLIT)
def test_whole_rows_on_parts(name):
    c = Case(**UNSPLIT[name])
    assert unsplit(c) and workspace(c, 0) > 0
    o, l = c.forward()
    compare(c, {"out": plain(o), "lse": l}, exact(c))


SPLIT = {"rows and keys of unlike number": dict(Sq=300, Sk=3100, heads=4, D=64), "lengths": dict(N=2, Sq=400, heads=4, D=64, lengths=[400, 129], bias="log"),
         "documents": dict(N=1, Sq=900, heads=4, D=64, docs=_docs(1, 900, [[100, 700, 80]])), "pixels": dict(N=1, Sq=660, heads=4, D=64, bias=(20, 33))}


@pytest.mark.parametrize("name", SPLIT)
def test_split_rows_on_parts(name):
    c = Case(**SPLIT[name])
    rows = c.N * c.heads * c.Sq
    parts = min(-(-c.Sk // 256), -(-512 // (c.N * c.heads * -(-c.Sq // 64))))
    assert not unsplit(c) and workspace(c, 0) > up(up(4 * rows * parts * c.D) + 8 * rows * parts)      # (more than the parts of split rows)
    o, l = c.forward()
    compare(c, {"out": plain(o), "lse": l}, exact(c))


# A reach past 2047, or heads of more than 128 channels.
FP32 = {
    "odd heads": dict(Sq=150, heads=3, D=37, Cb=37, bias="wide"), "shared heads, causal": dict(Sq=150, heads=6, kv=2, D=24, Cb=8, bias="wide", causal=True),
    "capped": dict(Sq=130, heads=2, D=64, bias="wide", cap=5.0, size=2.0), "distances": dict(Sq=130, heads=2, D=80, bias="wide", slopes=True),
    "prefix": dict(N=3, Sq=140, heads=2, D=96, bias="wide", causal=True, prefix=[0, 65, 140]), "documents": dict(N=2, Sq=140, heads=2, D=128, bias="wide", docs=_docs(2, 140, [[3, 60, 70], [140]])),
    "lengths": dict(N=4, Sq=100, heads=2, D=48, bias="wide", lengths=[0, 1, 64, 99]), "positions of their own": dict(N=3, Sq=40, Sk=100, heads=2, D=32, bias="wide", causal=True, first=[-20, 30, 90]),
    "wide heads, capped": dict(Sq=100, heads=2, D=192, cap=5.0, causal=True), "wide heads, distances": dict(Sq=100, heads=2, D=160, slopes=True, bias="log"),
    "wide heads, odd, shared": dict(N=2, Sq=90, heads=4, kv=2, D=131, Cb=131, docs=_docs(2, 90, [[40, 50], [10, 60]])),
    "everything": dict(N=3, Sq=100, cap=10.0, bias="wide", slopes=True, causal=True, prefix=[5, 0, 77], lengths=[100, 64, 80], docs=_docs(3, 100, [[50, 45], [100], [10, 10, 70]]), heads=6, kv=3, D=24, Cb=8),
}


@pytest.mark.parametrize("name", FP32)
def test_gradients_on_fp32_products(name):
    c = Case(**FP32[name])
    assert workspace(c, 1) == plain_grad_bytes(c)
    compare(c, everything(c), exact(c))


@pytest.mark.parametrize("name", ["plain", "odd", "128 channels", "shared heads", "lengths", "documents", "pixels", "buckets, capped", "distances, capped", "capped", "prefix, 96 channels"])
def test_gradients_on_parts(name):
    c = Case(**{**UNSPLIT[name], "N": 2, **({"lengths": [65, 299]} if "lengths" in UNSPLIT[name] else {}), **({"docs": UNSPLIT[name]["docs"][:2]} if "docs" in UNSPLIT[name] else {}),
                **({"prefix": [64, 260]} if "prefix" in UNSPLIT[name] else {})})
    assert workspace(c, 1) > plain_grad_bytes(c)
    compare(c, everything(c), exact(c))
