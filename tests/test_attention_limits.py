"""Sizes at which a launch of an attention call would have more threads than a launch can: refused before anything is enqueued. No GPU needed."""
import ctypes as C

import pytest

from paper_2303_04769_amd import attn
from test_attention_host import P, record


@pytest.fixture(scope="module")
def lib():
    return attn.load()


def answers(lib, r):
    n = C.c_size_t(0)
    query = [lib.small_attention_workspace(C.byref(r), grad, C.byref(n)) for grad in (0, 1)]
    room = 1 << 60
    return query, [lib.small_attention(C.byref(r), P[0], P[1], P[2], P[3], None, P[5], room, None),
                   lib.small_attention_grad(C.byref(r), P[0], P[1], P[2], P[3], P[4], P[5], P[6], P[7], P[8], None, P[9], room, None)]


def test_more_tiles_than_a_launch_has_workgroups(lib):
    # 2^24 tiles of rows: the call that lays keys and values out could be launched, the next one not
    for kw in (dict(N=1 << 20, Sq=256, Sk=256, heads=4, kv_heads=1, D=4, Cb=4), dict(N=1 << 18, Sq=4096, Sk=64, heads=1, kv_heads=1, D=4, Cb=4)):
        assert answers(lib, record(**kw)) == ([2, 2], [2, 2])
    # half as many: the forward call's launches are fine, of the gradient's, which lays out four tensors, one is not
    n = C.c_size_t(0)
    r = record(N=1 << 19, Sq=192, Sk=192, heads=4, kv_heads=4, D=4, Cb=4)
    assert [lib.small_attention_workspace(C.byref(r), grad, C.byref(n)) for grad in (0, 1)] == [0, 2]
    r = record(N=1 << 17, Sq=192, Sk=192, heads=4, kv_heads=4, D=4, Cb=4)
    assert [lib.small_attention_workspace(C.byref(r), grad, C.byref(n)) for grad in (0, 1)] == [0, 0]


def test_more_offsets_than_a_launch_sums(lib):
    both = dict(table=0x90000000, bucket=0xa0000000, buckets=4)
    n = C.c_size_t(0)
    for reach, want in ((1 << 23, 2), (1 << 22, 0)):
        r = record(N=1, Sq=64, Sk=64, heads=8, kv_heads=8, reach=reach, **both)
        assert lib.small_attention_workspace(C.byref(r), 1, C.byref(n)) == want and lib.small_attention_workspace(C.byref(r), 0, C.byref(n)) == 0
