"""Host side of rotary positions and the paged cache (include/small_cache.h of the package): exports, refusals, workspace sizes. No GPU needed: every
call here fails its checks before anything is enqueued."""
import ctypes as C
import os
import re

import pytest

import paper_2303_04769_amd as S
from paper_2303_04769_amd import cache as K

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [C.c_void_p(0x100000000 * (k + 1)) for k in range(20)]         # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return K.load()


def at(p, off=0):
    return C.c_void_p(p.value + off)


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "paper_2303_04769_amd", "include", "small_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(small_[a-z0-9_]+)\s*\(", text))) == sorted(S.CACHE_EXPORTS)
    for name in S.CACHE_EXPORTS:
        assert getattr(lib, name) is not None and hasattr(S, name)


def tokens(channels, S_, Cb):
    return S.small_tokens(channels * S_, S_ * Cb, Cb)


def rotation(**kw):
    k = dict(N=2, S=8, heads=4, kv_heads=2, D=16, Cb=16, axes=2, pairs=8, halves=0, freq_heads=1)
    k.update({n: v for n, v in kw.items() if n in k})
    r = S.small_rotation(**k)
    r.extent = (C.c_int * 4)(*kw.get("extent", (0, 4, 4, 4)))
    for n in ("q", "q_out", "dq"):
        setattr(r, n, kw.get(n, tokens(k["heads"] * k["D"], k["S"], k["Cb"])))
    for n in ("k", "k_out", "dk"):
        setattr(r, n, kw.get(n, tokens(k["kv_heads"] * k["D"], k["S"], k["Cb"])))
    r.freq, r.first, r.positions = kw.get("freq", P[10]), kw.get("first", P[11]), kw.get("positions")
    return r


def test_rotary_refusals(lib):
    def forward(q=P[0], k=P[1], qo=P[2], ko=P[3], **kw):
        return lib.small_rotary(C.byref(rotation(**kw)), q, k, qo, ko, None)
    assert lib.small_rotary(None, P[0], P[1], P[2], P[3], None) == 1
    assert forward(q=None) == forward(ko=None) == forward(q=None, qo=None, k=None, ko=None) == forward(freq=None) == 1
    for bad in (dict(N=0), dict(S=0), dict(heads=3), dict(kv_heads=0), dict(D=0), dict(D=257), dict(Cb=0), dict(axes=0), dict(axes=5), dict(pairs=0), dict(pairs=9),
                dict(freq_heads=3), dict(freq_heads=0), dict(extent=(0, 0, 4, 4)), dict(S=(1 << 28) + 1), dict(N=1 << 20, S=1 << 20), dict(N=1 << 12, S=1 << 14, heads=8)):
        assert forward(**bad) == 2, bad
    assert forward(q_out=S.small_tokens(512, 0, 16)) == 2                           # blocks on one another
    assert forward(qo=at(P[0], 16)) == 4 and forward(qo=P[0], q_out=S.small_tokens(1024, 128, 16)) == 4       # neither in place nor apart
    assert forward(qo=P[1]) == 4 and forward(ko=P[0]) == 4 and forward(ko=P[2]) == 4
    assert forward(qo=P[10]) == 4 and forward(ko=P[11]) == 4 and forward(positions=P[2]) == 4
    assert forward(extent=(0, 0, 0, 0), positions=P[12], qo=P[1]) == 4              # extents are not looked at beside positions

    def grad(dqo=P[0], dko=P[1], q=P[2], k=P[3], dq=P[4], dk=P[5], df=P[6], ws=P[7], size=1 << 20, **kw):
        return lib.small_rotary_grad(C.byref(rotation(**kw)), dqo, dko, q, k, dq, dk, df, ws, size, None)
    assert all(grad(**{n: None}) == 1 for n in ("dqo", "dko", "q", "k", "dq", "dk"))
    assert grad(ws=None) == 6 and grad(size=8) == 6 and grad(ws=at(P[7], 16)) == 6
    assert grad(axes=0) == 2 and grad(dq=P[1]) == 4 and grad(dq=P[2]) == 4 and grad(df=P[0]) == 4 and grad(df=P[4]) == 4 and grad(df=P[10]) == 4 and grad(ws=P[3]) == 4
    assert grad(df=P[7]) == 4 and grad(dk=P[4]) == 4 and grad(dk=P[7]) == 4
    n = C.c_size_t(0)
    assert lib.small_rotary_workspace(None, C.byref(n)) == 1 and lib.small_rotary_workspace(C.byref(rotation(pairs=0)), C.byref(n)) == 2
    assert lib.small_rotary_workspace(C.byref(rotation()), C.byref(n)) == 0 and n.value >= 8 * 2 * 8 and n.value % 256 == 0


def cache(**kw):
    k = dict(kind=2, pages=8, page=16, kv_heads=2, D=16, N=2, per_stream=4)
    k.update({n: v for n, v in kw.items() if n in k})
    c = S.small_cache(**k)
    c.keys, c.values, c.key_scales, c.value_scales, c.table = (kw.get(n, P[12 + i]) for i, n in enumerate(("keys", "values", "key_scales", "value_scales", "table")))
    return c


def span(**kw):
    k = dict(S=8, Cb=16)
    k.update({n: v for n, v in kw.items() if n in k})
    s = S.small_span(**k)
    s.k = s.v = kw.get("strides", tokens(32, k["S"], k["Cb"]))
    s.first, s.counts = kw.get("first", P[17]), kw.get("counts", P[18])
    return s


def test_write_and_read_refusals(lib):
    def write(k=P[0], v=P[1], q=None, qo=None, turn=None, **kw):
        return lib.small_cache_write(C.byref(cache(**kw)), C.byref(span(**kw)), k, v, None if turn is None else C.byref(turn), q, qo, None)

    def read(k=P[0], v=P[1], **kw):
        return lib.small_cache_read(C.byref(cache(**kw)), C.byref(span(**kw)), k, v, None)
    for call in (write, read):
        assert call(k=None) == call(v=None) == call(keys=None) == call(values=None) == call(key_scales=None) == call(value_scales=None) == call(table=None) == 1
        for bad in (dict(kind=3), dict(kind=-1), dict(pages=0), dict(page=8), dict(page=24), dict(page=512), dict(kv_heads=0), dict(D=0), dict(D=257), dict(N=0),
                    dict(per_stream=0), dict(per_stream=1 << 25), dict(S=0), dict(Cb=0), dict(S=(1 << 28) + 1)):
            assert call(**bad) == 2, bad
        assert call(keys=at(P[12], 4)) == 2 and call(value_scales=at(P[15], 8)) == 2
        assert call(k=P[12]) == 4 and call(v=P[13]) == 4 and call(k=P[14]) == 4
    assert write(values=P[12]) == 4 and write(key_scales=P[15]) == 4 and write(table=P[13]) == 4 and write(first=P[14]) == 4 and write(counts=P[12]) == 4
    assert read(k=P[1]) == 4 and read(k=P[16]) == 4 and read(v=P[17]) == 4 and read(strides=S.small_tokens(256, 128, 0)) == 2
    # with turns
    turn = rotation(axes=1, first=None)
    assert write(q=P[2], qo=P[3]) == 1 and write(q=P[2], turn=turn) == 1 and write(qo=P[2], turn=turn) == 1
    for bad in (dict(N=1), dict(S=7), dict(kv_heads=1), dict(D=32), dict(Cb=8), dict(pairs=9)):
        assert write(turn=rotation(axes=1, **bad)) == 2, bad
    assert write(q=P[2], qo=at(P[2], 64), turn=turn) == 4 and write(q=P[2], qo=P[0], turn=turn) == 4 and write(q=P[2], qo=P[13], turn=turn) == 4
    assert write(q=P[12], qo=P[3], turn=turn) == 4 and write(q=P[2], qo=P[10], turn=turn) == 4 and write(q=P[2], qo=P[17], turn=turn) == 4 and write(keys=P[10], turn=turn) == 4


def record(**kw):
    k = dict(N=2, Sq=1, Sk=0, heads=4, kv_heads=2, D=16, Cb=16, scale=0.25, cap=0.0, causal=0, width=1, reach=0, buckets=0)
    k.update({n: v for n, v in kw.items() if n in k})
    r = S.small_attn(**k)
    r.q = kw.get("q", tokens(k["heads"] * k["D"], k["Sq"], k["Cb"]))
    r.out = kw.get("out", tokens(k["heads"] * k["D"], k["Sq"], k["Cb"]))
    r.lengths, r.first, r.prefix, r.docs = kw.get("lengths", P[4]), kw.get("first"), kw.get("prefix"), kw.get("docs")
    r.slopes, r.table, r.bucket = kw.get("slopes"), kw.get("bias"), kw.get("bucket")
    return r


def test_attention_refusals(lib):
    def call(q=P[0], out=P[1], lse=P[2], ws=P[3], size=1 << 30, per=64, **kw):
        c = {n: v for n, v in kw.items() if n in ("kind", "keys", "values", "key_scales", "pages", "page")}
        a = {n: v for n, v in kw.items() if n not in c}
        return lib.small_cache_attention(C.byref(cache(per_stream=per, **c)), C.byref(record(**a)), q if not isinstance(q, S.small_tokens) else P[0], out, lse, ws, size, None)
    assert call(q=None) == call(out=None) == call(lengths=None) == call(keys=None) == 1
    assert call(bias=P[5]) == 1 and call(bucket=P[5]) == 1
    for bad in (dict(N=3), dict(Sq=0), dict(heads=5), dict(kv_heads=4), dict(D=32), dict(Cb=0), dict(width=2), dict(prefix=P[5]), dict(docs=P[5]), dict(scale=float("nan")),
                dict(cap=-1.0), dict(cap=float("inf")), dict(bias=P[5], bucket=P[6], buckets=0), dict(bias=P[5], bucket=P[6], buckets=2, reach=-1), dict(kind=5), dict(page=48)):
        assert call(**bad) == 2, bad
    assert call(size=8) == 6 and call(ws=None) == 6 and call(ws=at(P[3], 64)) == 6
    assert call(out=P[0]) == 4 and call(lse=P[0]) == 4 and call(lse=P[1]) == 4 and call(ws=P[0]) == 4 and call(out=P[12]) == 4 and call(ws=P[13]) == 4 and call(out=P[4]) == 4
    assert call(lse=P[4]) == 4 and call(out=P[16]) == 4 and call(slopes=P[1]) == 4 and call(first=P[3]) == 4
    n = C.c_size_t(0)
    sizes = lambda **kw: lib.small_cache_attention_workspace(C.byref(cache(per_stream=kw.pop("per", 64))), C.byref(record(**kw)), C.byref(n))  # noqa: E731
    assert sizes() == 0 and n.value % 256 == 0 and n.value >= 2 * 4 * 2 * 16 * 4       # split in two at least
    assert sizes(per=1) == 0 and n.value == 0
    assert sizes(N=1) == 2 and sizes(lengths=None) == 0
    assert lib.small_cache_attention_workspace(C.byref(cache()), C.byref(record()), None) == 1


def test_frequencies():
    f = S.axis_frequencies(8, 100.0, 2)
    assert tuple(f.shape) == (1, 2, 8) and not f[0, 0, 4:].any() and not f[0, 1, :4].any()
    assert f[0, 0, :4].tolist() == f[0, 1, 4:].tolist() == pytest.approx([1.0, 100 ** -0.25, 0.1, 100 ** -0.75])
    assert tuple(S.axis_frequencies(5).shape) == (1, 1, 5)
    with pytest.raises(ValueError):
        S.Rotary(1, 4, 1, 1, 8, axes=3, extent=(4,))


def test_tensors_are_checked_before_the_library():
    import torch
    with pytest.raises(TypeError):
        S.PagedCache(4, 16, 1, 8, tensors=[torch.zeros(1)] * 4)
    with pytest.raises(KeyError):
        S.PagedCache(4, 16, 1, 8, kind="float16")


@pytest.fixture
def on_ctypes(monkeypatch):
    """Calls through ctypes with tensors on the host, and the library's functions replaced: what(record, ...) runs in the place of each."""
    import torch
    from paper_2303_04769_amd import attn, binding
    what = {}
    monkeypatch.setattr(attn, "_tokens", lambda t, N, S_, Cb: (t.data_ptr(), S.small_tokens(*t.stride()[:3])))
    for name in ("_ptr", "_ptr32i"):
        monkeypatch.setattr(binding, name, lambda t: None if t is None else t.data_ptr())
    for name in ("small_rotary", "small_rotary_grad", "small_cache_write", "small_cache_read", "small_cache_attention"):
        monkeypatch.setattr(K, name, lambda *args, name=name, **kw: what[name](*args, **kw))
    return what


def bits(record):
    return bytes(C.string_at(C.addressof(record), C.sizeof(record)))


def test_calls_at_the_same_time_have_records_of_their_own(on_ctypes):
    """Two threads that serve different streams on one cache, and turn with one plan: while one is in the library the other fills its arguments. Neither sees the other's."""
    import torch
    pool = object.__new__(S.PagedCache)
    pool.kind, pool.pages, pool.page, pool.kv_heads, pool.D = 0, 8, 16, 1, 4
    pool.record = S.small_cache(kind=0, pages=8, page=16, kv_heads=1, D=4, keys=0x1000, values=0x2000)
    turn = S.Rotary(1, 3, 2, 1, 4, Cb=4, device="cpu")
    turn._workspace = torch.zeros(256, dtype=torch.uint8)
    plans = []
    for N, per in ((1, 2), (1, 3)):
        plan = object.__new__(S.CacheAttention)
        plan.cache, plan.per_stream, plan.workspace = pool, per, None
        plan.record = S.small_attn(N=N, Sq=3, Sk=per * 16, heads=2, kv_heads=1, D=4, Cb=4, width=1)
        plans.append(plan)
    q, k, freq = torch.zeros(1, 2, 3, 4), torch.zeros(1, 1, 3, 4), [torch.zeros(1, 1, 2) for _ in range(2)]
    tables, lengths = [torch.zeros(1, n, dtype=torch.int32) for n in (2, 3)], torch.zeros(1, dtype=torch.int32)
    calls = {
        "small_cache_write": lambda x: pool.write(k, k, tables[x], rotary=turn, freq=freq[x], q=q, stream="one"),
        "small_cache_read": lambda x: pool.read(k, k, tables[x], stream="one"),
        "small_cache_attention": lambda x: plans[x].run(q, q, tables[x], lengths, stream="one"),
        "small_rotary": lambda x: turn.run(q, k, freq[x], stream="one"),
        "small_rotary_grad": lambda x: turn.grad(q, k, freq[x], q=q, k=k, dfreq=torch.zeros(1, 1, 2), from_inputs=bool(x), stream="one"),
    }
    for name, call in calls.items():
        seen = []

        def inside(*args, **kw):
            records = [a for a in args if isinstance(a, (S.small_cache, S.small_rotation))]
            before = [bits(r) for r in records]
            for r in records:
                if isinstance(r, S.small_cache):
                    assert (r.per_stream, r.table) == (tables[len(seen)].shape[1], tables[len(seen)].data_ptr()), name
                else:
                    assert r.freq == freq[len(seen)].data_ptr(), name
            seen.append(records)
            if len(seen) == 1:
                call(1)                                        # (the other thread, meanwhile)
            assert [bits(r) for r in records] == before, name
        on_ctypes.clear()
        on_ctypes[name] = inside
        call(0)
        assert len(seen) == 2
