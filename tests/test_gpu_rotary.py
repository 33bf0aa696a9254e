"""Rotary positions on the GPU against their definition in 64 bits: forms, layouts, places, far angles, in place, gradients by the definition and by differences."""
import math

import pytest
import torch

import paper_2303_04769_amd as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def heads_of(t, heads):
    """[N][C/Cb][S][Cb] on the device -> [N][heads][S][D] in 64 bits on the host"""
    t = t.detach().cpu().double()
    return t.permute(0, 1, 3, 2).reshape(t.shape[0], -1, t.shape[2])[:, :].reshape(t.shape[0], heads, -1, t.shape[2]).transpose(2, 3)


def places(N, S_, axes, extent, first, positions):
    if positions is not None:
        return positions.cpu().double()
    out = torch.zeros(N, S_, axes, dtype=torch.float64)
    for n in range(N):
        for i in range(S_):
            t = i + (0 if first is None else int(first[n]))
            for a in range(axes - 1, 0, -1):
                out[n, i, a] = t % extent[a - 1]
                t = t // extent[a - 1]
            out[n, i, 0] = t
    return out


def turned(x, place, freq, pairs, halves, sign=1.0):
    """x [N][heads][S][D] in 64 bits -> the turned one, and the angles [N][heads][S][pairs]"""
    heads = x.shape[1]
    angle = torch.einsum("nsa,fak->nfsk", place, freq.double()).repeat_interleave(heads // freq.shape[0], 1)
    a, b = (slice(0, pairs), slice(pairs, 2 * pairs)) if halves else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    y = x.clone()
    c, s = torch.cos(angle), sign * torch.sin(angle)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y, angle


def check(got, x, place, freq, pairs, halves, sign=1.0):
    """Results are rounded once: half a step of the value. Before that an angle is off by the rounding of its sum over axes, 2^-53 of it for each, and the sines, the
    products and their sum by less than 2^-50 of the pair's channels."""
    ref, angle = turned(x, place, freq, pairs, halves, sign)
    far = float(angle.abs().max())
    tol = 2.0 ** -24 * ref.abs() + (2.0 ** -50 + 4 * 2.0 ** -53 * far) * 2 * float(x.abs().max()) + 2.0 ** -149
    off = (got - ref).abs() - tol
    assert bool((off <= 0).all()), f"off by {float(off.max())} more than a rounding"


FORMS = [
    # N, S, heads, kv, D, Cb, axes, pairs, halves, extent, freq_heads, first, positions
    (1, 1, 1, 1, 2, 2, 1, 1, False, (), 1, None, False),
    (1, 1, 8, 8, 32, 32, 1, 16, True, (), 1, [123456], False),
    (3, 7, 4, 2, 16, 16, 1, 8, False, (), 1, [0, 5, 1000000], False),
    (2, 33, 6, 3, 40, 8, 1, 12, True, (), 3, [3, -9], False),
    (2, 35, 4, 4, 16, 16, 2, 8, False, (5,), 1, None, False),
    (2, 35, 4, 4, 16, 64, 2, 8, True, (7,), 4, None, False),
    (2, 60, 4, 1, 32, 16, 3, 16, False, (4, 5), 1, [0, 11], False),
    (1, 60, 2, 2, 80, 160, 3, 40, True, (4, 5), 2, None, False),
    (2, 24, 2, 1, 24, 24, 4, 12, False, (2, 3, 2), 1, None, False),
    (2, 13, 3, 1, 10, 5, 1, 5, False, (), 1, None, False),              # pairs that cross blocks, nothing aligned
    (2, 13, 3, 3, 6, 1, 2, 2, True, (3,), 3, None, False),              # a channel a block
    (2, 19, 5, 5, 7, 35, 1, 3, False, (), 5, None, True),               # a channel that stays
    (2, 19, 2, 2, 64, 16, 3, 10, True, (), 1, None, True),
    (5, 130, 8, 2, 256, 16, 2, 64, True, (13,), 2, None, False),
    (1, 1000, 16, 4, 128, 512, 1, 32, False, (), 1, [70000], False),
]


def setup(form, seed=0):
    N, S_, heads, kv, D, Cb, axes, pairs, halves, extent, F, first, given = form
    nq, nk = -(-heads * D // Cb), -(-kv * D // Cb)
    q, k = rand(seed, N, nq, S_, Cb).to(DEV), rand(seed + 1, N, nk, S_, Cb).to(DEV)
    freq = rand(seed + 2, F, axes, pairs).to(DEV)
    first = None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV)
    positions = torch.randint(-50, 5000, (N, S_, axes), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).to(DEV) if given else None
    plan = S.Rotary(N, S_, heads, kv, D, axes=axes, pairs=pairs, halves=halves, extent=extent, freq_heads=F, Cb=Cb)
    return plan, q, k, freq, first, positions, places(N, S_, axes, extent, first, positions)


@pytest.mark.parametrize("form", FORMS)
def test_turns(form):
    N, S_, heads, kv, D, Cb, axes, pairs, halves, extent, F, _, _ = form
    plan, q, k, freq, first, positions, place = setup(form)
    qo, ko = torch.full_like(q, math.nan), torch.full_like(k, math.nan)
    plan.run(q, k, freq, qo, ko, first=first, positions=positions)
    check(heads_of(qo, heads), heads_of(q, heads), place, freq.cpu(), pairs, halves)
    check(heads_of(ko, kv), heads_of(k, kv), place, freq.cpu(), pairs, halves)
    # in place, one at a time: the same bits
    q2, k2 = q.clone(), k.clone()
    plan.run(q2, None, freq, first=first, positions=positions)
    plan.run(None, k2, freq, first=first, positions=positions)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("form", FORMS)
def test_gradients(form):
    N, S_, heads, kv, D, Cb, axes, pairs, halves, extent, F, _, _ = form
    plan, q, k, freq, first, positions, place = setup(form)
    dq, dk = rand(7, *q.shape).to(DEV), rand(8, *k.shape).to(DEV)
    plan.run(q, k, freq, first=first, positions=positions)              # (in place: q and k are the turned ones from here on)
    outs = [torch.full_like(t, math.nan) for t in (dq, dk)]
    dfreq = torch.full_like(freq, math.nan)
    plan.grad(dq, dk, freq, *outs, q=q, k=k, dfreq=dfreq, first=first, positions=positions)
    a, b = (slice(0, pairs), slice(pairs, 2 * pairs)) if halves else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    total, size = 0.0, 0.0
    for out, d, y, h in ((outs[0], dq, q, heads), (outs[1], dk, k, kv)):
        d, y = heads_of(d, h), heads_of(y, h)
        check(heads_of(out, h), d, place, freq.cpu(), pairs, halves, -1.0)
        cross = d[..., b] * y[..., a] - d[..., a] * y[..., b]
        by = cross.reshape(N, F, h // F, S_, pairs)
        total = total + torch.einsum("nfhsk,nsa->fak", by, place)
        size = size + torch.einsum("nfhsk,nsa->fak", by.abs(), place.abs())
    # sums in 64 bits, of fewer than 2^13 terms here, rounded once
    off = (dfreq.cpu().double() - total).abs() - 2.0 ** -24 * total.abs() - 2.0 ** -39 * size
    assert bool((off <= 0).all()), float(off.max())
    # without the frequencies' gradient, and in place: the same
    other = [torch.empty_like(t) for t in (dq, dk)]
    plan.grad(dq, dk, freq, *other, first=first, positions=positions)
    assert all(torch.equal(x, y) for x, y in zip(outs, other))
    again = torch.empty_like(dfreq)
    plan.grad(dq, dk, freq, q=q, k=k, dfreq=again, first=first, positions=positions)
    assert torch.equal(dq, outs[0]) and torch.equal(dk, outs[1]) and torch.equal(again, dfreq)


@pytest.mark.parametrize("halves", [False, True])
def test_frequency_gradient_by_differences(halves):
    """A step of 2^-8 in one frequency: the loss's symmetric difference, in 64 bits, is off its derivative by h^2 / 6 of the third derivative, the tokens' places cubed
    times their channels."""
    N, S_, heads, kv, D = 2, 6, 4, 2, 8
    plan = S.Rotary(N, S_, heads, kv, D, axes=2, halves=halves, extent=(3,), freq_heads=kv, Cb=8)
    q, k = rand(1, N, heads, S_, D).to(DEV), rand(2, N, kv, S_, D).to(DEV)
    wq, wk = rand(3, *q.shape).to(DEV), rand(4, *k.shape).to(DEV)
    freq = rand(5, kv, 2, D // 2).to(DEV)
    dfreq = torch.empty_like(freq)
    plan.grad(wq, wk, freq, torch.empty_like(q), torch.empty_like(k), q=_run(plan, q, k, freq)[0], k=_run(plan, q, k, freq)[1], dfreq=dfreq)
    place = places(N, S_, 2, (3,), None, None)
    h = 2.0 ** -8
    worst = float(sum((t.abs().double().sum() for t in (q * wq, k * wk)))) * 2
    for f in range(kv):
        for a in range(2):
            for p in range(D // 2):
                loss = []
                for sign in (1, -1):
                    moved = freq.clone().cpu().double()
                    moved[f, a, p] += sign * h
                    loss.append(sum(float((turned(heads_of(x, n), place, moved, D // 2, halves)[0] * heads_of(w, n)).sum()) for x, w, n in ((q, wq, heads), (k, wk, kv))))
                slope = (loss[0] - loss[1]) / (2 * h)
                assert abs(slope - float(dfreq[f, a, p])) <= h * h / 6 * 8 * worst + 1e-5 * abs(slope)


@pytest.mark.parametrize("form", FORMS)
def test_frequency_gradient_from_inputs(form):
    """From what was turned instead of what that gave, against automatic differentiation in 64 bits. A term is off by half a step of the turned back gradient's two channels, by 2^-50 of
    the pairs' sizes and by the angle's rounding (check); sums of fewer than 2^13 terms in 64 bits, rounded once. Gradients in place, through ctypes: the same bits."""
    N, S_, heads, kv, D, Cb, axes, pairs, halves, extent, F, _, _ = form
    plan, q, k, freq, first, positions, place = setup(form)
    dq, dk = rand(7, *q.shape).to(DEV), rand(8, *k.shape).to(DEV)
    outs = [torch.full_like(t, math.nan) for t in (dq, dk)]
    dfreq = torch.full_like(freq, math.nan)
    plan.grad(dq, dk, freq, *outs, q=q, k=k, dfreq=dfreq, first=first, positions=positions, from_inputs=True)
    leaf = freq.cpu().double().requires_grad_()
    loss, size, far = 0.0, 0.0, 0.0
    a, b = (slice(0, pairs), slice(pairs, 2 * pairs)) if halves else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    for d, x, h in ((dq, q, heads), (dk, k, kv)):
        d, x = heads_of(d, h), heads_of(x, h)
        y, angle = turned(x, place, leaf, pairs, halves)
        far = max(far, float(angle.detach().abs().max()))
        loss = loss + (y * d).sum()
        both = ((d[..., a].abs() + d[..., b].abs()) * (x[..., a].abs() + x[..., b].abs())).reshape(N, F, h // F, S_, pairs)
        size = size + torch.einsum("nfhsk,nsa->fak", both, place.abs())
    total, = torch.autograd.grad(loss, leaf)
    off = (dfreq.cpu().double() - total).abs() - 2.0 ** -24 * total.abs() - (2.0 ** -24 + 2.0 ** -39 + 2 * (2.0 ** -50 + 4 * 2.0 ** -53 * far)) * size
    assert bool((off <= 0).all()), float(off.max())
    again, other, copies = torch.empty_like(dfreq), torch.cuda.Stream(), (dq.clone(), dk.clone())
    torch.cuda.synchronize()
    plan.grad(*copies, freq, q=q, k=k, dfreq=again, first=first, positions=positions, from_inputs=True, stream=other)
    other.synchronize()
    assert torch.equal(again, dfreq)
    # from outputs: the same but for the rounding of one or the other
    plan.run(q, k, freq, first=first, positions=positions)
    plan.grad(dq, dk, freq, *outs, q=q, k=k, dfreq=again, first=first, positions=positions)
    assert bool(((again - dfreq).abs().cpu().double() <= 2.0 ** -23 * total.abs() + (2.0 ** -23 + 2.0 ** -38 + 4 * (2.0 ** -50 + 4 * 2.0 ** -53 * far)) * size).all())


def _run(plan, q, k, freq):
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    plan.run(q, k, freq, qo, ko)
    return qo, ko


def test_parts_of_one_projection():
    """Queries and keys as slices of one tensor, turned in place: the values beside them stay."""
    N, S_, heads, kv, D, Cb = 2, 30, 4, 2, 32, 16
    qkv = rand(0, N, (heads + 2 * kv) * D // Cb, S_, Cb).to(DEV)
    before = qkv.clone()
    nq, nk = heads * D // Cb, kv * D // Cb
    freq = S.axis_frequencies(16, 100.0, 2).to(DEV)
    plan = S.Rotary(N, S_, heads, kv, D, axes=2, extent=(6,), Cb=Cb)
    plan.run(qkv[:, :nq], qkv[:, nq:nq + nk], freq)
    place = places(N, S_, 2, (6,), None, None)
    check(heads_of(qkv[:, :nq], heads), heads_of(before[:, :nq], heads), place, freq.cpu(), 16, False)
    check(heads_of(qkv[:, nq:nq + nk], kv), heads_of(before[:, nq:nq + nk], kv), place, freq.cpu(), 16, False)
    assert torch.equal(qkv[:, nq + nk:], before[:, nq + nk:])


@pytest.mark.parametrize("heads,kv,halves", [(65536, 65536, False), (1 << 21, 1, True)])
def test_very_many_heads_of_one_token(heads, kv, halves):
    """More heads than their square fits 31 bits, shared out over workgroups."""
    q, k = rand(0, 1, heads, 1, 2).to(DEV), rand(1, 1, kv, 1, 2).to(DEV)
    freq, first = rand(2, 1, 1, 1).to(DEV), torch.tensor([12345], dtype=torch.int32, device=DEV)
    plan = S.Rotary(1, 1, heads, kv, 2, halves=halves, Cb=2)
    qo, ko, dfreq = torch.full_like(q, math.nan), torch.full_like(k, math.nan), torch.empty_like(freq)
    plan.run(q, k, freq, qo, ko, first=first)
    place = places(1, 1, 1, (), first, None)
    check(heads_of(qo, heads), heads_of(q, heads), place, freq.cpu(), 1, halves)
    check(heads_of(ko, kv), heads_of(k, kv), place, freq.cpu(), 1, halves)
    dq, dk = (torch.full_like(t, math.nan) for t in (q, k))
    plan.grad(q, k, freq, dq, dk, q=qo, k=ko, dfreq=dfreq, first=first)
    check(heads_of(dq, heads), heads_of(q, heads), place, freq.cpu(), 1, halves, -1.0)
    terms = torch.cat([12345.0 * (d[..., 1] * y[..., 0] - d[..., 0] * y[..., 1]).flatten() for d, y in ((q.double(), qo.double()), (k.double(), ko.double()))])
    assert abs(float(dfreq) - float(terms.sum())) <= 2.0 ** -24 * abs(float(terms.sum())) + 2.0 ** -31 * float(terms.abs().sum())      # (2^22 terms at most, in 64 bits)


def test_unaligned_views_have_the_same_bits():
    N, S_, heads, D = 2, 21, 3, 16
    base = rand(0, N * heads * S_ * D + 1).to(DEV)
    odd = base[1:].view(N, heads, S_, D)
    even = odd.clone()
    freq = rand(1, 1, 1, 8).to(DEV)
    plan = S.Rotary(N, S_, heads, heads, D, Cb=D)
    out = [torch.empty_like(even) for _ in range(2)]
    plan.run(odd, None, freq, out[0])
    plan.run(even, None, freq, out[1])
    assert torch.equal(out[0], out[1])


def test_non_finite_channels_stay_in_their_pairs():
    N, S_, D = 1, 4, 8
    x = rand(0, N, 1, S_, D).to(DEV)
    clean = x.clone()
    x[0, 0, 1, 2] = math.nan
    x[0, 0, 2, 5] = math.inf
    freq = rand(1, 1, 1, 4).to(DEV)
    plan = S.Rotary(N, S_, 1, 1, D, Cb=D)
    a, b = torch.empty_like(x), torch.empty_like(x)
    plan.run(x, None, freq, a)
    plan.run(clean, None, freq, b)
    touched = torch.zeros_like(x, dtype=torch.bool)
    touched[0, 0, 1, 2:4] = touched[0, 0, 2, 4:6] = True
    assert torch.equal(a[~touched], b[~touched]) and not torch.isfinite(a[touched]).any()


def test_captured_and_replayed():
    form = FORMS[6]
    N, S_, heads, kv, D, Cb, axes, pairs, halves, extent, F, _, _ = form
    plan, q, k, freq, first, positions, _ = setup(form)
    dq, dk, dfreq = torch.empty_like(q), torch.empty_like(k), torch.empty_like(freq)
    qo, ko = torch.empty_like(q), torch.empty_like(k)

    def step():
        plan.run(q, k, freq, qo, ko, first=first)
        plan.grad(qo, ko, freq, dq, dk, q=qo, k=ko, dfreq=dfreq, first=first)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        q.copy_(rand(10 + turn, *q.shape))
        k.copy_(rand(20 + turn, *k.shape))
        first.fill_(17 * turn)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (qo, ko, dq, dk, dfreq)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (qo, ko, dq, dk, dfreq)))
