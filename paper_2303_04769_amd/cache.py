"""Binding of rotary positions and the paged cache in libsmall_hip.so (include/small_cache.h): turns of queries and keys and their gradient, keys and values
into the pages of a cache and back, and attention of new tokens over it. Same names and arguments as the header (small_rotary, small_cache_write, ...), and
three objects that keep sizes, memory and workspace between calls: Rotary, PagedCache and CacheAttention. No arithmetic happens here.

Activations are torch CUDA tensors, float32, and may be views [N][C/Cb][S][Cb] as in attn; first positions, counts, lengths and page tables are int32.
"""
import ctypes as C

import torch

from . import attn as A
from . import binding as B
from .attn import small_attn, small_tokens

__all__ = ["CACHE_EXPORTS", "CACHE_BF16", "CACHE_F32", "CACHE_I8", "CacheAttention", "PagedCache", "Rotary", "axis_frequencies", "small_cache", "small_cache_attention",
           "small_cache_attention_workspace", "small_cache_read", "small_cache_write", "small_rotary", "small_rotary_grad", "small_rotary_workspace", "small_rotation",
           "small_span"]

CACHE_EXPORTS = ["small_rotary_workspace", "small_rotary", "small_rotary_grad", "small_cache_write", "small_cache_read", "small_cache_attention_workspace",
                 "small_cache_attention"]
CACHE_F32, CACHE_BF16, CACHE_I8 = 0, 1, 2
_KINDS = {"float32": (CACHE_F32, torch.float32), "bfloat16": (CACHE_BF16, torch.bfloat16), "int8": (CACHE_I8, torch.int8)}


class small_rotation(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("N", "S", "heads", "kv_heads", "D", "Cb", "axes", "pairs", "halves", "freq_heads")] + [("extent", C.c_int * 4), ("from_inputs", C.c_int)] + \
               [(n, small_tokens) for n in ("q", "k", "q_out", "k_out", "dq", "dk")] + [(n, C.c_void_p) for n in ("freq", "first", "positions")]


class small_cache(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("kind", "pages", "page", "kv_heads", "D")] + [(n, C.c_void_p) for n in ("keys", "values", "key_scales", "value_scales")] + \
               [("N", C.c_int), ("per_stream", C.c_int), ("table", C.c_void_p)]


class small_span(C.Structure):
    _fields_ = [("S", C.c_int), ("Cb", C.c_int), ("k", small_tokens), ("v", small_tokens), ("first", C.c_void_p), ("counts", C.c_void_p)]


_lib = None


def load():
    global _lib
    if _lib is None:
        lib = B.load()
        i, p, sz = C.c_int, C.c_void_p, C.c_size_t
        r, c, s, a = (C.POINTER(t) for t in (small_rotation, small_cache, small_span, small_attn))
        sig = {
            "small_rotary_workspace": [r, C.POINTER(sz)],
            "small_rotary": [r] + [p] * 5,
            "small_rotary_grad": [r] + [p] * 8 + [sz, p],
            "small_cache_write": [c, s, p, p, r, p, p, p],
            "small_cache_read": [c, s, p, p, p],
            "small_cache_attention_workspace": [c, a, C.POINTER(sz)],
            "small_cache_attention": [c, a, p, p, p, p, sz, p],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = i, args
        _lib = lib
    return _lib


_fastcall = None


def _fast():
    """The extension's calls (binding._fast), told once what the plans' records are."""
    global _fastcall
    if _fastcall is None:
        fast = A._fast()
        fast.bind_cache(small_rotation, small_cache)
        _fastcall = fast
    return _fastcall


def small_rotary_workspace(record):
    n = C.c_size_t(0)
    B._check(load().small_rotary_workspace(C.byref(record), C.byref(n)), "small_rotary_workspace")
    return n.value


def small_rotary(record, q, k, q_out, k_out, stream=None):
    """q, k, q_out, k_out (here and below): device pointers that record's strides describe, or None."""
    B._check(load().small_rotary(C.byref(record), q, k, q_out, k_out, B._stream(stream)), "small_rotary")


def small_rotary_grad(record, dq_out, dk_out, q, k, dq, dk, dfreq, workspace, stream=None):
    ws, size = A._bytes(workspace)
    B._check(load().small_rotary_grad(C.byref(record), dq_out, dk_out, q, k, dq, dk, B._ptr(dfreq), ws, size, B._stream(stream)), "small_rotary_grad")


def small_cache_write(cache, span, k, v, rotation=None, q=None, q_out=None, stream=None):
    B._check(load().small_cache_write(C.byref(cache), C.byref(span), k, v, None if rotation is None else C.byref(rotation), q, q_out, B._stream(stream)),
             "small_cache_write")


def small_cache_read(cache, span, k, v, stream=None):
    B._check(load().small_cache_read(C.byref(cache), C.byref(span), k, v, B._stream(stream)), "small_cache_read")


def small_cache_attention_workspace(cache, record):
    n = C.c_size_t(0)
    B._check(load().small_cache_attention_workspace(C.byref(cache), C.byref(record), C.byref(n)), "small_cache_attention_workspace")
    return n.value


def small_cache_attention(cache, record, q, out, lse, workspace, stream=None):
    ws, size = A._bytes(workspace)
    B._check(load().small_cache_attention(C.byref(cache), C.byref(record), q, out, B._ptr(lse), ws, size, B._stream(stream)), "small_cache_attention")


def _blocks(t, N, S, Cb, channels):
    """(pointer, strides) of an activation that has so many channels at least."""
    p, s = A._tokens(t, N, S, Cb)
    if t.shape[1] * Cb < channels:
        raise TypeError(f"{t.shape[1]} blocks of {Cb} channels hold no {channels}")
    return p, s


class Rotary:
    """Turns of pairs of channels by the place of their token on `axes` axes: of N images of S tokens, `heads` query heads and `kv_heads` key heads of D
    channels. The first 2 * pairs channels of a head turn (all of them, unless `pairs` says how many pairs), as neighbours or, with halves, `pairs` apart. extent:
    the sizes of all axes but the first, from which a token's number gives its place -- (W,) for images, (H, W) for clips; calls may give places instead.
    freq: [freq_heads][axes][pairs], radians a step (axis_frequencies); freq_heads 1 or kv_heads.

    The gradient's workspace belongs to the plan, which makes it at the first call with dfreq: such calls must not overlap in time on different streams."""

    def __init__(self, N, S, heads, kv_heads, D, axes=1, pairs=None, halves=False, extent=(), freq_heads=1, Cb=16, device="cuda:0"):
        extent = tuple(extent)
        if len(extent) not in (0, axes - 1):
            raise ValueError(f"{axes} axes have {axes - 1} extents behind the first, got {extent}")
        self.device = torch.device(device)
        self.record = small_rotation(N=N, S=S, heads=heads, kv_heads=kv_heads, D=D, Cb=Cb, axes=axes, pairs=D // 2 if pairs is None else pairs, halves=bool(halves),
                                     freq_heads=freq_heads, extent=(C.c_int * 4)(0, *extent))
        self._extents, self._workspace = len(extent) == axes - 1, None

    def _filled(self, freq, first, positions):
        """A call's own record: two threads may turn by one plan."""
        r = small_rotation.from_buffer_copy(self.record)
        if positions is None and not self._extents:
            raise ValueError(f"places on {r.axes} axes need extents or positions")
        r.freq = A._floats(freq, (r.freq_heads, r.axes, r.pairs))
        r.first, r.positions = A._ints(first, (r.N,)), A._ints(positions, (r.N, r.S, r.axes))
        return r

    @staticmethod
    def _pair(r, q, k, names):
        """Pointers of a tensor of queries and one of keys, either of which may be None, with their strides in the record."""
        found = []
        for t, heads, name in ((q, r.heads, names[0]), (k, r.kv_heads, names[1])):
            p, s = (None, small_tokens()) if t is None else _blocks(t, r.N, r.S, r.Cb, heads * r.D)
            setattr(r, name, s)
            found.append(p)
        return found

    def run(self, q, k, freq, q_out=None, k_out=None, first=None, positions=None, stream=None):
        """Turns q and k (either may be None) into q_out and k_out, or in place where these are None."""
        if stream is None:
            rc = _fast().rotary(self.record, q, k, freq, positions, first, q_out, k_out, None)
            if rc is not None:
                return B._check(rc, "small_rotary")
        r = self._filled(freq, first, positions)
        pq, pk = self._pair(r, q, k, ("q", "k"))
        po, pko = self._pair(r, q if q_out is None else q_out, k if k_out is None else k_out, ("q_out", "k_out"))
        small_rotary(r, pq, pk, po, pko, stream)

    def grad(self, dq_out, dk_out, freq, dq=None, dk=None, q=None, k=None, dfreq=None, first=None, positions=None, stream=None, from_inputs=False):
        """Turns the gradients of run's outputs back into those of its inputs (in place where dq and dk are None). With dfreq, [freq_heads][axes][pairs], the frequencies'
        gradient too, from q and k: run's outputs, or with from_inputs its inputs."""
        if dfreq is not None and self._workspace is None:
            self._workspace = torch.empty(small_rotary_workspace(self._filled(freq, first, positions)), dtype=torch.uint8, device=self.device)
        if stream is None:
            rc = _fast().rotary_grad(self.record, dq_out, dk_out, freq, positions, first, dq, dk, q, k, dfreq, None if dfreq is None else self._workspace, int(from_inputs), None)
            if rc is not None:
                return B._check(rc, "small_rotary_grad")
        r = self._filled(freq, first, positions)
        r.from_inputs = bool(from_inputs)
        if dfreq is not None:
            A._floats(dfreq, (r.freq_heads, r.axes, r.pairs))
        pq, pk = self._pair(r, q, k, ("q", "k"))
        pdo, pdko = self._pair(r, dq_out, dk_out, ("q_out", "k_out"))
        pd, pdk = self._pair(r, dq_out if dq is None else dq, dk_out if dk is None else dk, ("dq", "dk"))
        small_rotary_grad(r, pdo, pdko, pq, pk, pd, pdk, dfreq, None if dfreq is None else self._workspace, stream)


class PagedCache:
    """`pages` pages of `page` tokens (16, 32, 64, 128 or 256) for the keys and values of kv_heads heads of D channels, as "float32", "bfloat16" or "int8" (codes and a
    scale for each token of a head), the last unless another is named. Its memory is four tensors, keys, values, key_scales, value_scales (the last two None but for int8); tensors: these, instead of new
    ones. Which pages a stream has is the program's affair: every call takes a table, int32 [N][pages of a stream at most]."""

    def __init__(self, pages, page, kv_heads, D, kind="int8", device="cuda:0", tensors=None):
        self.kind, dtype = _KINDS[kind]
        self.pages, self.page, self.kv_heads, self.D = pages, page, kv_heads, D
        fill = 16 // dtype.itemsize
        shapes = (pages, kv_heads, page, -(-D // fill) * fill), (pages, kv_heads, D, page), (pages, kv_heads, page), (pages, kv_heads, page)
        dtypes = dtype, dtype, torch.float32, torch.float32
        if tensors is None:
            tensors = [torch.zeros(s, dtype=t, device=device) if n < 2 or kind == "int8" else None for n, (s, t) in enumerate(zip(shapes, dtypes))]
        for n, (t, shape, dtype) in enumerate(zip(tensors, shapes, dtypes)):
            if n >= 2 and kind != "int8":
                if t is not None:
                    raise TypeError(f"a cache of {kind} has no scales")
            elif not (t.is_cuda and t.dtype == dtype and tuple(t.shape) == shape and t.is_contiguous()):
                raise TypeError(f"expected a contiguous {dtype} CUDA tensor {list(shape)}, got {t.dtype} {list(t.shape)}")
        self.keys, self.values, self.key_scales, self.value_scales = tensors
        self.record = small_cache(kind=self.kind, pages=pages, page=page, kv_heads=kv_heads, D=D, keys=self.keys.data_ptr(), values=self.values.data_ptr(),
                                  key_scales=self.key_scales.data_ptr() if kind == "int8" else None,
                                  value_scales=self.value_scales.data_ptr() if kind == "int8" else None)

    def _with(self, pages, N):
        """The cache's record with a call's table: threads that serve different streams share the cache."""
        if pages.dim() != 2 or pages.shape[0] != N:
            raise TypeError(f"expected a table of pages of {N} streams, got {list(pages.shape)}")
        c = small_cache.from_buffer_copy(self.record)
        c.N, c.per_stream, c.table = N, pages.shape[1], B._ptr32i(pages)
        return c

    def _span(self, k, v, pages, first, counts):
        N, S, Cb = k.shape[0], k.shape[2], k.shape[3]
        c = self._with(pages, N)
        pk, sk = _blocks(k, N, S, Cb, self.kv_heads * self.D)
        pv, sv = _blocks(v, N, S, Cb, self.kv_heads * self.D)
        return c, small_span(S=S, Cb=Cb, k=sk, v=sv, first=A._ints(first, (N,)), counts=A._ints(counts, (N,))), pk, pv

    def write(self, k, v, pages, first=None, counts=None, rotary=None, freq=None, positions=None, q=None, q_out=None, stream=None):
        """Tokens i < counts[n] of k and v into the cache at positions first[n] + i of stream n. With a Rotary plan of these sizes (and its freq) keys are turned on the way,
        and queries q into q_out (in place where it is None). No two tokens of a call may have one place: it would hold parts of both."""
        if stream is None:
            rc = _fast().cache_write(self.record, k, v, pages, first, counts, None if rotary is None else rotary.record, freq, positions, q, q_out, None)
            if rc is not None:
                return B._check(rc, "small_cache_write")
        c, span, pk, pv = self._span(k, v, pages, first, counts)
        if rotary is None:
            if q is not None:
                raise TypeError("queries are turned by a Rotary plan: none was given")
            return small_cache_write(c, span, pk, pv, stream=stream)
        r = rotary._filled(freq, None, positions)
        pq, _ = rotary._pair(r, q, None, ("q", "k"))
        po, _ = rotary._pair(r, q if q_out is None else q_out, None, ("q_out", "k_out"))
        small_cache_write(c, span, pk, pv, r, pq, po, stream)

    def read(self, k, v, pages, first=None, counts=None, stream=None):
        """The same tokens from the cache into k and v; what is no token of a stream's is left as it was."""
        if stream is None:
            rc = _fast().cache_read(self.record, k, v, pages, first, counts, None)
            if rc is not None:
                return B._check(rc, "small_cache_read")
        c, span, pk, pv = self._span(k, v, pages, first, counts)
        small_cache_read(c, span, pk, pv, stream)


class CacheAttention:
    """Attention of Sq new tokens (one, or a few) of each of N streams over a PagedCache, `heads` query heads, tables of per_stream pages. Scores as in Attention:
    scale, cap, distances (slopes), learned biases (table and bucket, with reach and buckets); each token sees itself and those before it.
    The workspace belongs to the plan: its calls must not overlap in time on different streams."""

    def __init__(self, cache, N, Sq, heads, per_stream, Cb=16, scale=None, cap=0.0, reach=0, buckets=0, device="cuda:0"):
        self.cache, self.per_stream = cache, per_stream
        self.record = small_attn(N=N, Sq=Sq, Sk=per_stream * cache.page, heads=heads, kv_heads=cache.kv_heads, D=cache.D, Cb=Cb, scale=cache.D ** -0.5 if scale is None else scale,
                                 cap=cap, causal=1, width=1, reach=reach, buckets=buckets)
        sizes = small_cache.from_buffer_copy(cache.record)
        sizes.N, sizes.per_stream = N, per_stream
        n = small_cache_attention_workspace(sizes, self.record)
        self.workspace = torch.empty(n, dtype=torch.uint8, device=torch.device(device)) if n else None

    def run(self, q, out, pages, lengths, lse=None, first=None, slopes=None, table=None, bucket=None, stream=None):
        """q, out: [N][blocks][Sq][Cb]; pages: the streams' table; lengths: tokens that each stream has in the cache, with the new ones; first: position of the first new one
        (None: the last Sq)."""
        r = self.record
        if stream is None:
            rc = _fast().cache_attention(self.cache.record, r, q, out, lse, self.workspace, pages, lengths, first, slopes, table, bucket, None)
            if rc is not None:
                return B._check(rc, "small_cache_attention")
        if pages.shape[1] != self.per_stream:
            raise TypeError(f"expected a table of {self.per_stream} pages a stream, got {list(pages.shape)}")
        c, r = self.cache._with(pages, r.N), small_attn.from_buffer_copy(r)
        r.lengths, r.first = A._ints(lengths, (r.N,)), A._ints(first, (r.N,))
        r.slopes = A._floats(slopes, (r.heads,))
        r.table, r.bucket = A._floats(table, (r.heads, r.buckets)), A._ints(bucket, (2 * r.reach + 1,))
        pq, r.q = _blocks(q, r.N, r.Sq, r.Cb, r.heads * r.D)
        po, r.out = _blocks(out, r.N, r.Sq, r.Cb, r.heads * r.D)
        if lse is not None:
            A._floats(lse, (r.N, r.heads, r.Sq))
        small_cache_attention(c, r, pq, po, lse, self.workspace, stream)


def axis_frequencies(pairs, base=10000.0, axes=1):
    """Frequencies [1][axes][pairs] of which each axis turns a section of the pairs: of n pairs the k-th by base ** (-k / n) radians a step."""
    freq = torch.zeros(1, axes, pairs)
    for a in range(axes):
        lo, hi = pairs * a // axes, pairs * (a + 1) // axes
        for k in range(lo, hi):
            freq[0, a, k] = base ** (-(k - lo) / (hi - lo))
    return freq
