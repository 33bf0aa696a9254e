"""Binding of the attention block in libsmall_hip.so (include/small_attn.h): group normalization with an activation, attention over
pixels, frames and caches, and their gradients. Same names and arguments as the header (small_groupnorm, small_attention, ...), and two plans that
keep sizes and workspace between calls: GroupNorm and Attention. No arithmetic happens here.

Tensors are torch CUDA tensors, float32, masks and buckets int32. Activations of attention may be views: a tensor [N][C/Cb][S][Cb] is taken with the
strides that it has, so the parts of one projection's output, or the first Sk tokens of a longer cache, are passed as slices.
"""
import ctypes as C

import torch

from . import binding as B
from .binding import SmallError  # noqa: F401

__all__ = ["ACT_NONE", "ACT_RELU", "ACT_SILU", "ATTN_EXPORTS", "Attention", "GroupNorm", "log_buckets", "pixel_buckets", "small_attention",
           "small_attention_grad", "small_attention_workspace", "small_attn", "small_groupnorm", "small_groupnorm_grad",
           "small_groupnorm_workspace", "small_tokens"]

ACT_NONE, ACT_RELU, ACT_SILU = 0, 1, 2
_ACTS = {"none": ACT_NONE, "relu": ACT_RELU, "silu": ACT_SILU}

ATTN_EXPORTS = ["small_groupnorm_workspace", "small_groupnorm", "small_groupnorm_grad", "small_attention_workspace", "small_attention",
                "small_attention_grad"]


class small_tokens(C.Structure):
    """Strides in floats of a tensor [N][C/Cb][S][Cb]."""
    _fields_ = [("image", C.c_size_t), ("block", C.c_size_t), ("token", C.c_size_t)]


class small_attn(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("N", "Sq", "Sk", "heads", "kv_heads", "D", "Cb")] + \
               [(n, small_tokens) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")] + [("scale", C.c_float), ("cap", C.c_float)] + \
               [(n, C.c_int) for n in ("causal", "width", "reach", "buckets")] + \
               [(n, C.c_void_p) for n in ("lengths", "first", "prefix", "docs", "slopes", "table", "bucket")]


_lib = None


def load():
    global _lib
    if _lib is None:
        lib = B.load()
        i, p, sz, f = C.c_int, C.c_void_p, C.c_size_t, C.c_float
        a = C.POINTER(small_attn)
        sig = {
            "small_groupnorm_workspace": [i] * 6 + [C.POINTER(sz)],
            "small_groupnorm": [p] * 5 + [i] * 5 + [f, i, i, p, sz, p],
            "small_groupnorm_grad": [p] * 8 + [i] * 7 + [p, sz, p],
            "small_attention_workspace": [a, i, C.POINTER(sz)],
            "small_attention": [a] + [p] * 6 + [sz, p],
            "small_attention_grad": [a] + [p] * 11 + [sz, p],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = i, args
        _lib = lib
    return _lib


_fastcall = None


def _fast():
    """The extension's calls (binding._fast), told once what an attention plan's record is."""
    global _fastcall
    if _fastcall is None:
        fast = B._fast()
        fast.bind_attention(small_attn)
        _fastcall = fast
    return _fastcall


def _bytes(t):
    """Device pointer and size of a workspace tensor."""
    return (None, 0) if t is None else (t.data_ptr(), t.numel() * t.element_size())


def small_groupnorm_workspace(N, Cc, H, W, G, Cb):
    n = C.c_size_t(0)
    B._check(load().small_groupnorm_workspace(N, Cc, H, W, G, Cb, C.byref(n)), "small_groupnorm_workspace")
    return n.value


def _holds(*tensors):
    """Each tensor that there is has as many values as are written behind it (sizes that the library refuses are its to refuse)."""
    for t, values in zip(tensors[::2], tensors[1::2]):
        if t is not None and values > 0 and t.numel() != values:
            raise TypeError(f"expected {values} values, got {tuple(t.shape)}")


def small_groupnorm(inp, gamma, beta, out, stats, N, Cc, H, W, G, eps, act, Cb, workspace, stream=None):
    rc = _fast().groupnorm(inp, gamma, beta, out, stats, N, Cc, H, W, G, eps, act, Cb, workspace, None) if stream is None else None
    if rc is not None:
        return B._check(rc, "small_groupnorm")
    values = N * Cc * H * W
    _holds(inp, values, gamma, Cc, beta, Cc, out, values, stats, 2 * N * G)
    ws, size = _bytes(workspace)
    B._check(load().small_groupnorm(B._ptr(inp), B._ptr(gamma), B._ptr(beta), B._ptr(out), B._ptr(stats), N, Cc, H, W, G, eps, act, Cb,
                                    ws, size, B._stream(stream)), "small_groupnorm")


def small_groupnorm_grad(inp, gamma, beta, stats, dout, din, dgamma, dbeta, N, Cc, H, W, G, act, Cb, workspace, stream=None):
    rc = _fast().groupnorm_grad(inp, gamma, beta, stats, dout, din, dgamma, dbeta, N, Cc, H, W, G, act, Cb, workspace, None) if stream is None else None
    if rc is not None:
        return B._check(rc, "small_groupnorm_grad")
    values = N * Cc * H * W
    _holds(inp, values, gamma, Cc, beta, Cc, stats, 2 * N * G, dout, values, din, values, dgamma, Cc, dbeta, Cc)
    ws, size = _bytes(workspace)
    B._check(load().small_groupnorm_grad(B._ptr(inp), B._ptr(gamma), B._ptr(beta), B._ptr(stats), B._ptr(dout), B._ptr(din),
                                         B._ptr(dgamma), B._ptr(dbeta), N, Cc, H, W, G, act, Cb, ws, size, B._stream(stream)),
             "small_groupnorm_grad")


def _tokens(t, N, S, Cb):
    """(pointer, strides) of a float32 activation [N][blocks][S][Cb] that may be a view."""
    if not (t.is_cuda and t.dtype == torch.float32 and t.dim() == 4 and t.shape[0] == N and t.shape[2] == S and t.shape[3] == Cb and
            (Cb == 1 or t.stride(3) == 1)):
        raise TypeError(f"expected a float32 CUDA tensor [{N}][blocks][{S}][{Cb}] with neighbouring channels, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr(), small_tokens(t.stride(0), t.stride(1), t.stride(2))


def _ints(t, shape):
    if t is None:
        return None
    if tuple(t.shape) != shape:
        raise TypeError(f"expected an int32 tensor of shape {shape}, got {tuple(t.shape)}")
    return B._ptr32i(t)


def _floats(t, shape):
    if t is None:
        return None
    if tuple(t.shape) != shape:
        raise TypeError(f"expected a float32 tensor of shape {shape}, got {tuple(t.shape)}")
    return B._ptr(t)


def small_attention_workspace(record, grad):
    n = C.c_size_t(0)
    B._check(load().small_attention_workspace(C.byref(record), int(grad), C.byref(n)), "small_attention_workspace")
    return n.value


def small_attention(record, q, k, v, out, lse, workspace, stream=None):
    """q, k, v, out: device pointers that record's strides describe."""
    ws, size = _bytes(workspace)
    B._check(load().small_attention(C.byref(record), q, k, v, out, B._ptr(lse), ws, size, B._stream(stream)), "small_attention")


def small_attention_grad(record, q, k, v, out, lse, dout, dq, dk, dv, dtable, workspace, stream=None):
    ws, size = _bytes(workspace)
    B._check(load().small_attention_grad(C.byref(record), q, k, v, out, B._ptr(lse), dout, dq, dk, dv, B._ptr(dtable), ws, size,
                                         B._stream(stream)), "small_attention_grad")


class GroupNorm:
    """Group normalization of [N][C/Cb][H][W][Cb] in G groups, then `act` ("none", "relu", "silu"). The workspace belongs to the plan: its calls
    must not overlap in time on different streams."""

    def __init__(self, N, Cc, H, W, G, eps=1e-5, act="none", Cb=16, device="cuda:0"):
        self.sizes, self.eps, self.act, self.Cb = (N, Cc, H, W, G), eps, _ACTS[act], Cb
        n = small_groupnorm_workspace(N, Cc, H, W, G, Cb)
        self.workspace = torch.empty(max(n, 256), dtype=torch.uint8, device=device)

    def run(self, inp, gamma, beta, out, stats=None, stream=None):
        small_groupnorm(inp, gamma, beta, out, stats, *self.sizes, self.eps, self.act, self.Cb, self.workspace, stream)

    def grad(self, inp, gamma, beta, stats, dout, din, dgamma=None, dbeta=None, stream=None):
        small_groupnorm_grad(inp, gamma, beta, stats, dout, din, dgamma, dbeta, *self.sizes, self.act, self.Cb, self.workspace, stream)


class Attention:
    """Attention of N images, Sq queries on Sk keys, `heads` query heads on `kv_heads` key heads of D channels. The workspaces belong to
    the plan: its calls must not overlap in time on different streams.

    Every call takes the masks and biases as device tensors: lengths, first, prefix int32 [N]; docs int32 [N][Sk]; slopes [heads];
    table [heads][buckets] with bucket int32 [2 * reach + 1] (log_buckets, pixel_buckets)."""

    def __init__(self, N, Sq, Sk, heads, kv_heads, D, Cb=16, scale=None, cap=0.0, causal=False, width=1, reach=0, buckets=0, device="cuda:0"):
        self.device = torch.device(device)
        self.record = small_attn(N=N, Sq=Sq, Sk=Sk, heads=heads, kv_heads=kv_heads, D=D, Cb=Cb, scale=D ** -0.5 if scale is None else scale, cap=cap,
                                 causal=bool(causal), width=width, reach=reach, buckets=buckets)
        self._workspace = {}

    def _fill(self, lengths, first, prefix, docs, slopes, table, bucket):
        r = self.record
        r.lengths, r.first, r.prefix = _ints(lengths, (r.N,)), _ints(first, (r.N,)), _ints(prefix, (r.N,))
        r.docs = _ints(docs, (r.N, r.Sk))
        r.slopes = _floats(slopes, (r.heads,))
        r.table, r.bucket = _floats(table, (r.heads, r.buckets)), _ints(bucket, (2 * r.reach + 1,))

    def _space(self, grad):
        """Workspace of the forward or the gradient call, enough for calls with a table and without."""
        if grad not in self._workspace:
            r = small_attn.from_buffer_copy(self.record)
            sizes = []
            for there in (None, 256)[:2 if r.buckets else 1]:         # (a table is only looked at for being there)
                r.table = r.bucket = there
                sizes.append(small_attention_workspace(r, grad))
            self._workspace[grad] = torch.empty(max(sizes), dtype=torch.uint8, device=self.device) if max(sizes) else None
        return self._workspace[grad]

    def _blocks(self, t, heads, S):
        r = self.record
        p, s = _tokens(t, r.N, S, r.Cb)
        if t.shape[1] * r.Cb < heads * r.D:
            raise TypeError(f"{t.shape[1]} blocks of {r.Cb} channels hold no {heads} heads of {r.D}")
        return p, s

    def run(self, q, k, v, out, lse=None, lengths=None, first=None, prefix=None, docs=None, slopes=None, table=None, bucket=None, stream=None):
        r = self.record
        if stream is None:
            rc = _fast().attention(r, q, k, v, out, lse, self._space(0), lengths, first, prefix, docs, slopes, table, bucket, None)
            if rc is not None:
                return B._check(rc, "small_attention")
        self._fill(lengths, first, prefix, docs, slopes, table, bucket)
        pq, r.q = self._blocks(q, r.heads, r.Sq)
        pk, r.k = self._blocks(k, r.kv_heads, r.Sk)
        pv, r.v = self._blocks(v, r.kv_heads, r.Sk)
        po, r.out = self._blocks(out, r.heads, r.Sq)
        if lse is not None:
            _floats(lse, (r.N, r.heads, r.Sq))
        small_attention(r, pq, pk, pv, po, lse, self._space(0), stream)

    def grad(self, q, k, v, out, lse, dout, dq, dk, dv, dtable=None, lengths=None, first=None, prefix=None, docs=None, slopes=None,
             table=None, bucket=None, stream=None):
        r = self.record
        if stream is None:
            rc = _fast().attention_grad(r, q, k, v, out, lse, dout, dq, dk, dv, dtable, self._space(1), lengths, first, prefix, docs, slopes,
                                        table, bucket, None)
            if rc is not None:
                return B._check(rc, "small_attention_grad")
        self._fill(lengths, first, prefix, docs, slopes, table, bucket)
        _floats(lse, (r.N, r.heads, r.Sq))
        if dtable is not None:
            _floats(dtable, (r.heads, r.buckets))
        pq, r.q = self._blocks(q, r.heads, r.Sq)
        pk, r.k = self._blocks(k, r.kv_heads, r.Sk)
        pv, r.v = self._blocks(v, r.kv_heads, r.Sk)
        po, r.out = self._blocks(out, r.heads, r.Sq)
        pdo, r.dout = self._blocks(dout, r.heads, r.Sq)
        pdq, r.dq = self._blocks(dq, r.heads, r.Sq)
        pdk, r.dk = self._blocks(dk, r.kv_heads, r.Sk)
        pdv, r.dv = self._blocks(dv, r.kv_heads, r.Sk)
        small_attention_grad(r, pq, pk, pv, po, lse, pdo, pdq, pdk, pdv, dtable, self._space(1), stream)


def pixel_buckets(H, W):
    """(bucket map, buckets, reach, width) that give every offset of rows and columns of an H x W image a bucket of its own."""
    reach = (H - 1) * (2 * W - 1) + W - 1
    return torch.arange(2 * reach + 1, dtype=torch.int32), 2 * reach + 1, reach, W


def log_buckets(reach, buckets, both=True):
    """(bucket map, buckets, reach) of a bias over distances in a sequence. Offsets -reach .. reach of a key against its query, those
    beyond are taken into the last bucket of their side. Half of the buckets (all of them, for causal attention: both=False) are for
    keys at or before the query: one half of these for single distances, the other for distances that grow by a constant
    factor up to the reach. The other half is for keys behind the query likewise."""
    side = buckets // 2 if both else buckets
    single = max(1, side // 2)
    grow = side - single
    edges = [single * (reach / single) ** (k / grow) for k in range(grow)]
    found = []
    for r in range(-reach, reach + 1):
        d = abs(r) if both or r < 0 else 0
        b = d if d < single else max(0, single - 1 + sum(d >= e for e in edges))
        found.append(min(b, side - 1) + (side if both and r > 0 else 0))
    return torch.tensor(found, dtype=torch.int32), buckets, reach
