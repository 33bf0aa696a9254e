"""StreamBlock's own state -- pages, lengths, tables -- without a GPU: the layers are stand-ins that record what they are given and compute nothing."""
import pytest
import torch

from paper_2303_04769_amd import attention_block as AB

N, PAGE, PER, CC, HEADS, KV, D = 3, 16, 8, 8, 4, 2, 4


class Layers:
    """What the stand-ins were called with; `refuse`: the one that raises."""

    def __init__(self):
        self.calls, self.refuse = [], None

    def of(self, name):
        def layer(*args, **kw):
            if self.refuse == name:
                raise TypeError(name)
            self.calls.append((name, [a.clone() if isinstance(a, torch.Tensor) else a for a in args], {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}))
        return layer

    def plan(self, name, **methods):
        def make(*args, **kw):
            if self.refuse == name:
                raise MemoryError(name)
            self.calls.append((name, args, kw))
            return type(name, (), {m: staticmethod(self.of(of)) for m, of in methods.items()})()
        return make

    def last(self, name):
        return next(c for c in reversed(self.calls) if c[0] == name)


@pytest.fixture
def layers(monkeypatch):
    l = Layers()
    monkeypatch.setattr(AB, "_packed", lambda w, *a: w)
    monkeypatch.setattr(AB, "_conv1x1", l.of("conv"))
    monkeypatch.setattr(AB.B, "small_add", l.of("add"))
    monkeypatch.setattr(AB.A, "GroupNorm", l.plan("GroupNorm", run="norm"))
    monkeypatch.setattr(AB.A, "Attention", l.plan("Attention", run="attend"))
    monkeypatch.setattr(AB.K, "Rotary", l.plan("Rotary"))
    monkeypatch.setattr(AB.K, "CacheAttention", l.plan("CacheAttention", run="attend"))
    monkeypatch.setattr(AB.K, "PagedCache", l.plan("PagedCache", write="write", read="read"))
    return l


def block(pages=12):
    w = torch.zeros
    return AB.StreamBlock(w((HEADS + 2 * KV) * D, CC), w(CC, HEADS * D), w(CC), w(CC), w(1, 1, D // 2), N, pages, PAGE, PER, CC, 2, HEADS, KV, D, Cb=4)


def state(b):
    return b.lengths[:], b.free[:], [h[:] for h in b.held], b.table.clone().tolist(), b._length.tolist()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("refuse", ["GroupNorm", "Rotary", "plan", "norm", "conv", "write", "read", "attend", "add"])
def test_a_refused_call_leaves_the_streams_as_they_were(layers, refuse, wide):
    b = block()
    b.forward(torch.zeros(N, 3, CC), [3, 1, 0])
    before = state(b)
    layers.refuse = ("Attention" if wide else "CacheAttention") if refuse == "plan" else refuse
    frames, counts = torch.zeros(N, 40 if wide else 20, CC), [20, 17, 0]
    if refuse == "read" and not wide:
        layers.refuse = "attend"                               # (few frames read nothing back)
    with pytest.raises((TypeError, MemoryError)):
        b.forward(frames, counts)
    assert state(b) == before
    # and the next call goes on from there
    layers.refuse = None
    b.forward(frames, counts)
    _, args, kw = layers.last("write")
    assert args[3].tolist() == before[0] and kw["counts"].tolist() == counts
    assert layers.last("attend")[2]["first"].tolist() == before[0] and b.lengths == [l + c for l, c in zip(before[0], counts)] == b._length.tolist()
    for n in range(N):
        assert b.table[n].tolist() == b.held[n] + [-1] * (PER - len(b.held[n])) and len(b.held[n]) == -(-b.lengths[n] // PAGE)
    assert sorted(b.free + sum(b.held, [])) == list(range(12))


def test_frames_are_counted_from_call_to_call(layers):
    b = block()
    at = [0] * N
    for counts in ([2, 0, 5], None, [0, 0, 0], [1, 5, 5], None):
        b.forward(torch.zeros(N, 5, CC), counts)
        more = counts or [5] * N
        assert layers.last("write")[1][3].tolist() == at and layers.last("attend")[2]["first"].tolist() == at
        at = [a + m for a, m in zip(at, more)]
        assert layers.last("attend")[1][3].tolist() == at == b.lengths
    b.release(2)
    b.forward(torch.zeros(N, 5, CC))
    assert b.lengths == [at[0] + 5, at[1] + 5, 5] and layers.last("write")[1][3].tolist() == [at[0], at[1], 0]


def test_wide_call_on_empty_streams(layers):
    """An idle batch, more rows than are attended on the cache, in streams without a frame so far: a plan of the wide form, of a page at least."""
    b = block()
    b.forward(torch.zeros(N, 40, CC), [0, 0, 0])
    assert layers.last("Attention")[1][2] >= 1 and layers.last("read")[2]["counts"].tolist() == [0, 0, 0]
    name, args, kw = layers.last("attend")
    assert kw["lengths"].tolist() == [0, 0, 0] and b.lengths == [0, 0, 0] and not sum(b.held, []) and len(b.free) == 12
    b.forward(torch.zeros(N, 40, CC), [40, 0, 1])
    assert b.lengths == [40, 0, 1]
