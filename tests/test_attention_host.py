"""Host side of the attention block (include/small_attn.h of the package): exports, refusals, workspace sizes, bucket maps. No GPU needed: every
call here fails its checks before anything is enqueued."""
import ctypes as C
import os
import re

import pytest

import paper_2303_04769_amd as S
from paper_2303_04769_amd import attn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [C.c_void_p(0x10000000 * (k + 1)) for k in range(16)]          # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return attn.load()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "paper_2303_04769_amd", "include", "small_attn.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(small_[a-z0-9_]+)\s*\(", text))) == sorted(attn.ATTN_EXPORTS)
    for name in attn.ATTN_EXPORTS:
        assert getattr(lib, name) is not None and hasattr(S, name)


def test_groupnorm_refusals(lib):
    ws = 1 << 20
    ok = dict(N=2, Cc=32, H=4, W=4, G=4, eps=1e-5, act=1, Cb=16)

    def forward(x=P[0], gamma=P[1], beta=P[2], out=P[3], stats=P[4], work=P[5], size=ws, **kw):
        k = {**ok, **kw}
        return lib.small_groupnorm(x, gamma, beta, out, stats, k["N"], k["Cc"], k["H"], k["W"], k["G"], k["eps"], k["act"], k["Cb"], work, size, None)
    assert forward(x=None) == forward(gamma=None) == forward(beta=None) == forward(out=None) == 1
    for bad in (dict(N=0), dict(Cc=0), dict(H=-1), dict(W=0), dict(G=0), dict(G=5), dict(G=64), dict(Cb=0), dict(Cb=24), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(act=3), dict(act=-1), dict(H=65536, W=65536), dict(N=1 << 30, Cc=1 << 10, Cb=16)):
        assert forward(**bad) == 2, bad
    assert forward(Cc=8192, Cb=8192) == 3 and forward(Cc=1030, G=1, Cb=1030) == 3
    assert forward(Cc=2048, Cb=2048, x=C.c_void_p(0x10000004)) == 3
    assert forward(size=8) == 6 and forward(work=None) == 6 and forward(work=C.c_void_p(0x60000010)) == 6
    assert forward(out=C.c_void_p(0x10000004)) == 4 and forward(stats=P[3]) == 4 and forward(work=P[0]) == 4 and forward(gamma=P[3]) == 4
    assert forward(stats=P[5]) == 4 and forward(beta=P[4]) == 4

    def grad(x=P[0], gamma=P[1], beta=P[2], stats=P[3], dout=P[4], din=P[5], dgamma=P[6], dbeta=P[7], work=P[8], size=ws, **kw):
        k = {**ok, **kw}
        return lib.small_groupnorm_grad(x, gamma, beta, stats, dout, din, dgamma, dbeta, k["N"], k["Cc"], k["H"], k["W"], k["G"], k["act"], k["Cb"], work, size, None)
    assert all(grad(**{n: None}) == 1 for n in ("x", "gamma", "beta", "stats", "dout", "din", "dgamma", "dbeta"))
    assert grad(G=3) == 2 and grad(act=7) == 2 and grad(Cc=8192, Cb=8192) == 3 and grad(size=0) == 6
    assert grad(din=P[0]) == 4 and grad(dgamma=P[7]) == 4 and grad(dgamma=P[1]) == 4 and grad(work=P[4]) == 4 and grad(din=C.c_void_p(0x50000004)) == 4
    n = C.c_size_t(0)
    assert lib.small_groupnorm_workspace(2, 32, 4, 4, 4, 16, None) == 1 and lib.small_groupnorm_workspace(2, 32, 4, 4, 3, 16, C.byref(n)) == 2
    assert lib.small_groupnorm_workspace(2, 32, 4, 4, 4, 16, C.byref(n)) == 0 and n.value >= 2 * 32 * 8


def record(**kw):
    k = dict(N=2, Sq=8, Sk=8, heads=4, kv_heads=2, D=16, Cb=16, scale=0.25, cap=0.0, causal=0, width=1, reach=0, buckets=0)
    k.update(kw)
    r = attn.small_attn(**{n: v for n, v in k.items() if n in dict(attn.small_attn._fields_)})
    for name, heads, tokens in (("q", k["heads"], k["Sq"]), ("k", k["kv_heads"], k["Sk"]), ("v", k["kv_heads"], k["Sk"]), ("out", k["heads"], k["Sq"]),
                                ("dout", k["heads"], k["Sq"]), ("dq", k["heads"], k["Sq"]), ("dk", k["kv_heads"], k["Sk"]), ("dv", k["kv_heads"], k["Sk"])):
        if name not in kw:
            setattr(r, name, attn.small_tokens(max(0, heads * k["D"] * tokens), max(0, tokens * k["Cb"]), max(0, k["Cb"])))
    return r


def test_attention_refusals(lib):
    def forward(r, q=P[0], k=P[1], v=P[2], out=P[3], lse=P[4], work=P[5], size=1 << 26):
        return lib.small_attention(C.byref(r) if r is not None else None, q, k, v, out, lse, work, size, None)
    assert forward(None) == 1
    assert all(forward(record(), **{n: None}) == 1 for n in ("q", "k", "v", "out"))
    for bad in (dict(N=0), dict(Sq=0), dict(Sk=0), dict(heads=0), dict(kv_heads=3), dict(kv_heads=8), dict(D=0), dict(D=257), dict(Cb=0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("inf")), dict(cap=float("nan")), dict(width=0),
                dict(Sk=1 << 29), dict(N=1 << 20, Sq=1 << 12)):
        assert forward(record(**bad)) == 2, bad
    assert forward(record(table=0x90000000, buckets=4)) == 1 and forward(record(bucket=0x90000000)) == 1
    both = dict(table=0x90000000, bucket=0xa0000000)
    assert forward(record(**both, buckets=0)) == 2 and forward(record(**both, buckets=4, reach=-1)) == 2
    # overlaps: whole ranges, masks, parts of one tensor that do or do not interleave
    assert forward(record(), out=P[0]) == 4 and forward(record(), lse=P[1]) == 4 and forward(record(), lse=P[3]) == 4
    assert forward(record(lengths=0x40000000)) == 4 and forward(record(docs=0x50000000)) == 4
    qkv = attn.small_tokens(128 * 8, 8 * 16, 16)
    part = lambda blocks: C.c_void_p(0x10000000 + blocks * 8 * 16 * 4)  # noqa: E731
    assert forward(record(q=qkv, k=qkv, out=qkv), q=part(0), k=part(4), out=part(2)) == 4
    # an output whose own values share places
    assert forward(record(out=attn.small_tokens(0, 128, 16))) == 2 and forward(record(out=attn.small_tokens(512, 128, 8))) == 2
    # few rows on many keys need a workspace
    n = C.c_size_t(0)
    r = record(N=1, Sq=1, Sk=50000)
    assert lib.small_attention_workspace(C.byref(r), 0, C.byref(n)) == 0 and n.value > 0
    assert forward(r, size=n.value - 1) == 6 and forward(r, work=None) == 6 and forward(r, work=C.c_void_p(0x60000010)) == 6 and forward(r, work=P[1]) == 4
    assert lib.small_attention_workspace(C.byref(record(D=300)), 0, C.byref(n)) == 2 and lib.small_attention_workspace(None, 0, C.byref(n)) == 1

    def grad(r, q=P[0], k=P[1], v=P[2], out=P[3], lse=P[4], dout=P[5], dq=P[6], dk=P[7], dv=P[8], dtable=None, work=P[9], size=1 << 26):
        return lib.small_attention_grad(C.byref(r) if r is not None else None, q, k, v, out, lse, dout, dq, dk, dv, dtable, work, size, None)
    assert grad(None) == 1 and all(grad(record(), **{n: None}) == 1 for n in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"))
    assert grad(record(D=300)) == 2 and grad(record(), dtable=P[10]) == 1 and grad(record(), size=0) == 6
    assert grad(record(), dq=P[0]) == 4 and grad(record(), dk=P[8]) == 4 and grad(record(), dv=P[9]) == 4 and grad(record(), work=P[4]) == 4
    assert grad(record(**both, buckets=3, reach=1), dtable=C.c_void_p(0x90000000)) == 4
    assert grad(record(dk=attn.small_tokens(256, 128, 8))) == 2


def test_python_checks(lib):
    import torch
    plan = object.__new__(S.Attention)
    plan.record = record()
    with pytest.raises(TypeError):
        plan._blocks(torch.zeros(2, 4, 8, 16), 4, 8)                 # not on the GPU
    with pytest.raises(TypeError):
        attn._ints(torch.zeros(3, dtype=torch.int32), (2,))
    with pytest.raises(TypeError):
        attn._floats(torch.zeros(3), (2,))
    with pytest.raises(KeyError):
        S.GroupNorm(1, 16, 1, 1, 1, act="gelu")


def test_bucket_maps():
    m, buckets, reach = S.log_buckets(128, 32)
    assert len(m) == 257 and buckets == 32 and reach == 128 and int(m.min()) == 0 and int(m.max()) == 31
    assert int(m[128]) == 0 and [int(m[128 - d]) for d in range(8)] == list(range(8)) and [int(m[128 + d]) for d in range(1, 8)] == [16 + d for d in range(1, 8)]
    back = [int(m[128 - d]) for d in range(129)]
    assert back == sorted(back) and back[-1] == 15 and len(set(back)) == 16
    m, _, _ = S.log_buckets(128, 32, both=False)
    assert set(int(x) for x in m[128:]) == {0} and int(m[0]) == 31
    m, buckets, reach, width = S.pixel_buckets(3, 5)
    code = [(p // 5) * 9 + p % 5 for p in range(15)]
    offsets = {}
    for i in range(15):
        for j in range(15):
            at = code[j] - code[i] + reach
            assert 0 <= at < buckets
            offsets.setdefault(int(m[at]), set()).add((j // 5 - i // 5, j % 5 - i % 5))
    assert width == 5 and all(len(v) == 1 for v in offsets.values()) and len(offsets) == 5 * 9
