"""Attention and its gradient where masks leave little or nothing, and what hidden places hold: against the 64-bit implementation of
test_gpu_attention.py, with its tolerances unless a test derives its own.
"""
import pytest
import torch

from gpu_util import DEV
from test_gpu_attention import Case, _docs, blocked, guarded, plain

pytestmark = pytest.mark.gpu


def gradients(c, dout=None):
    """(out, lse, dq, dk, dv, dtable) of a case, the gradients in plain layout; every tensor NaN before."""
    (q, k, v), m = c.dev()
    o, l = c.forward()
    (dq, c1), (dk, c2), (dv, c3) = (guarded(t.shape) for t in (q, k, v))
    dt, c4 = guarded(c.table.shape) if c.table is not None else (None, lambda: None)
    c.plan().grad(q, k, v, o, l, blocked(c.dout if dout is None else dout, c.Cb).to(DEV), dq, dk, dv, dt, **m)
    c1(), c2(), c3(), c4()
    return plain(o), l, plain(dq), plain(dk), plain(dv), dt


@pytest.mark.parametrize("bias", [None, "log", "wide"])
@pytest.mark.parametrize("causal", [False, True])
def test_documents_and_positions_wholly_outside(causal, bias):
    """Images whose rows all lie in front of the tokens or behind them, beside others: they see nothing and nothing sees them."""
    first = [300, -1000003, -37, 100, 45, 2 ** 28, -30, 70]
    c = Case(N=8, Sq=30, Sk=100, docs=_docs(8, 100, [[100], [40, 60], [64, 36]]), first=first, heads=4, kv=2, causal=causal, bias=bias)
    c.check()
    out, lse, dq, dk, dv, _ = gradients(c)
    outside = [n for n, f in enumerate(first) if f >= 100 or f + 30 <= 0]
    assert len(outside) == 6
    for t in (out, dq, dk, dv):
        assert bool((t[outside] == 0).all())
    assert bool((lse[outside] == -float("inf")).all())
