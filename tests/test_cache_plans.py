"""How calls of rotary positions and the paged cache are laid over workgroups, for any sizes that are not refused: cache_api.hip built for the host alone, with launches that look at
what the kernels would do. No GPU needed, nothing is launched."""
import ctypes as C
import os
import random
import subprocess

import pytest

import paper_2303_04769_amd as S
from paper_2303_04769_amd import build

SOURCE = r'''
#include "cache_api.hip"

namespace small {
int device_cus() { return 256; }
namespace {
char said[256];
int launched;
// The shares of `all` heads that `parts` workgroups take, in the kernels' 32-bit arithmetic: one behind the other, all of them.
bool shares(const FastDiv &by_parts, int parts, int all)
{
    int at = 0;
    for (int part = 0; part < parts; ++part) {
        const int lo = by_parts.div((int)((unsigned)part * (unsigned)all)), hi = by_parts.div((int)((unsigned)(part + 1) * (unsigned)all));
        if (lo != at || hi < lo) return snprintf(said, sizeof said, "part %d of %d: heads %d .. %d of %d behind %d", part, parts, lo, hi, all, at), false;
        at = hi;
    }
    return at == all || (snprintf(said, sizeof said, "%d parts have %d heads of %d", parts, at, all), false);
}
void threads(double n)
{
    if (n >= 4294967296.0) snprintf(said, sizeof said, "%.0f threads", n);
}
void turns(const RotaryArgs &a)
{
    const int all = (a.q ? a.heads / a.freq_heads : 0) + (a.k ? a.kv_heads / a.freq_heads : 0);
    shares(a.by_parts, a.parts, all);
    if ((double)a.freq_heads * a.parts >= 2147483648.0) snprintf(said, sizeof said, "sets");
    ++launched;
}
void stores(const StoreArgs &a)
{
    shares(a.by_parts, a.parts, a.items);
    threads((double)a.N * a.tiles * a.parts * (((a.tile << a.lanes_log2) + 63) / 64 * 64));
    ++launched;
}
}  // namespace
hipError_t launch_rotary(const RotaryArgs &a, bool, bool, hipStream_t)
{
    turns(a);
    threads(256.0 * ((a.turn_threads + 255.0) / 256.0 + 1) * a.freq_heads * a.parts + 256.0 * (a.copy_threads / 256 + 1));
    return hipSuccess;
}
hipError_t launch_rotary_grad(const RotaryArgs &a, bool, bool, bool, float *, hipStream_t)
{
    turns(a);
    threads(256.0 * a.freq_heads * a.parts * a.runs * a.chunks + 256.0 * (a.copy_threads / 256 + 1));
    if ((double)a.chunks * a.per_chunk < (double)a.N * a.S || (double)a.chunks * a.per_chunk > 2147483647.0) snprintf(said, sizeof said, "chunks");
    return hipSuccess;
}
hipError_t launch_cache_write(const StoreArgs &a, bool, bool, hipStream_t) { stores(a); return hipSuccess; }
hipError_t launch_cache_read(const StoreArgs &a, bool, hipStream_t) { stores(a); return hipSuccess; }
TokenShape token_shape(int, int, int) { return TokenShape{16, 64, 2}; }
hipError_t launch_cache_token(const AttnArgs &, const CacheArgs &, bool, hipStream_t) { return hipSuccess; }
}  // namespace small

extern "C" const char *said_of_calls(int *calls)
{
    static char out[256];
    snprintf(out, sizeof out, "%s", small::said);
    small::said[0] = 0;
    *calls = small::launched;
    small::launched = 0;
    return out;
}
'''


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    at = tmp_path_factory.mktemp("plans")
    src, lib = at / "plans.hip", at / "plans.so"
    src.write_text(SOURCE)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "-std=c++17", "--offload-host-only", "--offload-arch=gfx950", "-fPIC", "-shared", "-I" + build.CSRC, str(src), "-o",
                    str(lib)], check=True, capture_output=True)
    lib = C.CDLL(str(lib))
    lib.said_of_calls.restype = C.c_char_p
    for f in ("small_rotary", "small_rotary_grad", "small_cache_write", "small_cache_read"):
        getattr(lib, f).argtypes = None
    return lib


def at(n):
    return C.c_void_p(n << 44)                                 # (never dereferenced, and far apart)


def tokens(channels, S_, Cb):
    blocks = -(-channels // Cb)
    return S.small_tokens(blocks * S_ * Cb, S_ * Cb, Cb)


def call(plans, fn, *args):
    """The call's result, and what is wrong with its launch (nothing: empty)."""
    rc, calls = getattr(plans, fn)(*args), C.c_int(0)
    said = plans.said_of_calls(C.byref(calls)).decode()
    assert calls.value == (rc == 0), (rc, calls.value)
    return rc, said


def rotary(plans, N, S_, heads, kv, D, Cb, pairs, halves, freq_heads, grad, which=3):
    r = S.small_rotation(N=N, S=S_, heads=heads, kv_heads=kv, D=D, Cb=Cb, axes=1, pairs=pairs, halves=halves, freq_heads=freq_heads)
    r.q = r.q_out = r.dq = tokens(heads * D, S_, Cb)
    r.k = r.k_out = r.dk = tokens(kv * D, S_, Cb)
    r.freq = at(1)
    q, k, qo, ko, dq, dk = (at(n) if which & (1 + n % 2) else None for n in range(2, 8))
    if not grad:
        return call(plans, "small_rotary", C.byref(r), q, k, qo, ko, None)
    n = C.c_size_t(0)
    if plans.small_rotary_workspace(C.byref(r), C.byref(n)):
        return 2, ""
    return call(plans, "small_rotary_grad", C.byref(r), q, k, qo, ko, dq, dk, at(8), at(9), n, None)


def store(plans, read, N, S_, kv, D, Cb, kind, with_first, heads=0):
    c = S.small_cache(kind=kind, pages=1, page=16, kv_heads=kv, D=D, keys=at(1), values=at(2), key_scales=at(3), value_scales=at(4), N=N, per_stream=4, table=at(5))
    s = S.small_span(S=S_, Cb=Cb, k=tokens(kv * D, S_, Cb), v=tokens(kv * D, S_, Cb), first=at(6) if with_first else None, counts=None)
    if read:
        return call(plans, "small_cache_read", C.byref(c), C.byref(s), at(7), at(8), None)
    if not heads:
        return call(plans, "small_cache_write", C.byref(c), C.byref(s), at(7), at(8), None, None, None, None)
    r = S.small_rotation(N=N, S=S_, heads=heads, kv_heads=kv, D=D, Cb=Cb, axes=1, pairs=max(1, D // 2), freq_heads=1)
    r.q = r.q_out = tokens(heads * D, S_, Cb)
    r.freq = at(9)
    return call(plans, "small_cache_write", C.byref(c), C.byref(s), at(7), at(8), C.byref(r), at(10), at(11), None)


def test_many_heads_of_few_tokens(plans):
    """As many heads as a call may have, shared out over as many workgroups as it asks for: part times heads stays below 2^31."""
    for heads in (46341, 65536, 1 << 20, 1 << 23):
        for kv in (1, heads):
            assert rotary(plans, 1, 1, heads, kv, 2, 2, 1, 0, 1, False) == (0, ""), heads
            assert rotary(plans, 1, 1, heads, kv, 2, 2, 1, 0, 1, True) == (0, ""), heads
    for kv in (1 << 20, (1 << 21) + 3, 1 << 24):
        for read in (False, True):
            assert store(plans, read, 1, 1, kv, 1, 1, 0, False) == (0, ""), kv
            assert store(plans, read, 1, 20, kv, 1, 1, 2, True) == (0, ""), kv
    assert store(plans, False, 1, 1, 1 << 22, 2, 2, 0, True, heads=1 << 23) == (0, "")


def test_any_sizes(plans):
    """Whatever is not refused has a launch of fewer than 2^32 threads whose shares are whole."""
    rng, ran = random.Random(5), 0
    log = lambda hi: max(1, min(hi, int(2 ** rng.uniform(0, hi.bit_length()))))  # noqa: E731
    for _ in range(3000):
        D, N, S_ = rng.choice([1, 2, 3, 4, 7, 8, 16, 64, 100, 256]), log(1 << 16), log(1 << 22)
        most = int(min((1 << 24) // D, max(1, (1 << 33) // (N * S_ * D))))
        kv = log(most)
        heads = kv * log(max(1, most // kv))
        Cb = rng.choice([1, D, 16, 4])
        kind = rng.choice(["rotary", "grad", "write", "read"])
        if kind in ("rotary", "grad"):
            if D < 2:
                continue
            rc, said = rotary(plans, N, S_, heads, kv, D, Cb, rng.randint(1, D // 2), rng.randint(0, 1), rng.choice([1, kv]), kind == "grad", rng.choice([1, 2, 3]))
        else:
            turned = kind == "write" and D > 1 and rng.random() < 0.5
            rc, said = store(plans, kind == "read", N, S_, kv, D, Cb, rng.randint(0, 2), rng.random() < 0.5, heads if turned else 0)
        assert rc in (0, 2) and said == "", (kind, N, S_, heads, kv, D, Cb, rc, said)
        ran += rc == 0
    assert ran > 1000


WILD = S.small_tokens(1 << 50, 1 << 50, 1 << 50)


def test_what_a_write_does_not_read_is_not_looked_at(plans):
    """Of a write's rotation: first, k, k_out, dq and dk, and without queries q and q_out. Nor the strides of queries or keys that a turn does not have."""
    c = S.small_cache(kind=0, pages=2, page=16, kv_heads=2, D=8, keys=at(1), values=at(2), N=1, per_stream=2, table=at(5))
    s = S.small_span(S=5, Cb=8, k=tokens(16, 5, 8), v=tokens(16, 5, 8))
    r = S.small_rotation(N=1, S=5, heads=4, kv_heads=2, D=8, Cb=8, axes=1, pairs=4, freq_heads=1)
    r.freq, r.first = at(9), at(1)                             # (first: in the cache's keys)
    r.k = r.k_out = r.dq = r.dk = WILD
    r.q = r.q_out = tokens(32, 5, 8)
    assert call(plans, "small_cache_write", C.byref(c), C.byref(s), at(7), at(8), C.byref(r), at(10), at(11), None) == (0, "")
    r.first = at(11)                                           # (in the queries' result)
    assert call(plans, "small_cache_write", C.byref(c), C.byref(s), at(7), at(8), C.byref(r), at(10), at(11), None) == (0, "")
    r.q = r.q_out = WILD
    assert call(plans, "small_cache_write", C.byref(c), C.byref(s), at(7), at(8), C.byref(r), None, None, None) == (0, "")
    assert call(plans, "small_cache_write", C.byref(c), C.byref(s), at(7), at(8), C.byref(r), at(10), at(11), None)[0] == 2
    r.first = None
    for q, k in ((at(10), None), (None, at(10))):
        r.q = r.q_out = tokens(32, 5, 8) if q else WILD
        r.k = r.k_out = tokens(16, 5, 8) if k else WILD
        assert call(plans, "small_rotary", C.byref(r), q, k, q and at(11), k and at(11), None) == (0, "")
        r.dq, r.dk = r.q, r.k
        assert call(plans, "small_rotary_grad", C.byref(r), q, k, None, None, q and at(11), k and at(11), None, None, 0, None) == (0, "")
    r.dq = WILD
    assert call(plans, "small_rotary_grad", C.byref(r), None, at(10), None, None, None, at(11), None, None, 0, None) == (0, "")
    n = C.c_size_t(0)
    assert plans.small_rotary_workspace(C.byref(r), C.byref(n)) == 0        # sizes alone
