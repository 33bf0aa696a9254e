// C-ABI layer of rotary positions and the paged cache (include/small_cache.h has the contract of every entry point): argument checks and sizes, host only.
#include "attn_laid.h"
#include "cache.h"

#include <initializer_list>

#include <limits.h>
#include <math.h>

using namespace small;

namespace {

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }
int power_of_two_of(int x) { return x & -x; }

Laid laid(int N, int S, int heads, int D, int Cb, const float *p, const small_tokens &s)
{
    return Laid{p, s, (size_t)N, ((size_t)heads * D + Cb - 1) / Cb, (size_t)S, (size_t)Cb};
}
Range bytes_of(const void *p, size_t bytes) { return Range(p, p ? (bytes + 3) / 4 : 0); }
bool meets_any(const Range &w, std::initializer_list<Range> reads)
{
    for (const Range &r : reads)
        if (w.meets(r)) return true;
    return false;
}
bool same(const small_tokens &a, const small_tokens &b) { return a.image == b.image && a.block == b.block && a.token == b.token; }

const size_t kMostStride = (size_t)1 << 40;
int strides_check(std::initializer_list<const small_tokens *> strides)
{
    for (const small_tokens *s : strides)
        if (s->image > kMostStride || s->block > kMostStride || s->token > kMostStride) return SMALL_ERR_SHAPE;
    return SMALL_OK;
}
int sizes_check(int N, int S, int heads, int kv_heads, int D, int Cb, std::initializer_list<const small_tokens *> strides)
{
    if (N <= 0 || S <= 0 || heads <= 0 || kv_heads <= 0 || D <= 0 || Cb <= 0 || heads % kv_heads || D > 256 || S > kFar || Cb > 1 << 20) return SMALL_ERR_SHAPE;
    if ((double)heads * D > 1 << 24 || (double)N * S > INT_MAX) return SMALL_ERR_SHAPE;
    return strides_check(strides);
}
// Four channels of a head stand together and aligned in all of these.
bool quads(int D, int Cb, std::initializer_list<const small_tokens *> strides, std::initializer_list<const void *> tensors)
{
    size_t bits = 0;
    for (const small_tokens *s : strides) bits |= s->image | s->block | s->token;
    uintptr_t at = 0;
    for (const void *t : tensors) at |= (uintptr_t)t;
    return D % 4 == 0 && Cb % 4 == 0 && bits % 4 == 0 && at % 16 == 0;
}

// Shares of so many heads: as many as are wanted, no more than there are heads, and so that a share's number times the heads, which the kernels divide, fits an int.
int shares_of(int heads, double wanted) { return (int)fmin(fmin(heads, wanted), INT_MAX / heads); }

// ---- rotary positions

// (but for the strides, which are those of the tensors that a call has)
int rotation_check(const small_rotation &r)
{
    if (const int rc = sizes_check(r.N, r.S, r.heads, r.kv_heads, r.D, r.Cb, {})) return rc;
    if (r.axes < 1 || r.axes > 4 || r.pairs < 1 || 2 * r.pairs > r.D || (r.freq_heads != 1 && r.freq_heads != r.kv_heads)) return SMALL_ERR_SHAPE;
    if (!r.freq) return SMALL_ERR_NULL;
    if (!r.positions)
        for (int x = 1; x < r.axes; ++x)
            if (r.extent[x] < 1 || r.extent[x] > kFar) return SMALL_ERR_SHAPE;
    return SMALL_OK;
}

// How a call's work is laid over threads (rotary.hip): units of neighbouring pairs, runs of units that stand together in a block.
struct TurnPlan {
    int unit, units, run, parts, chunks, per_chunk, copies, copy_run;
    size_t bytes;
};
bool turn_vec(const small_rotation &r, bool quad) { return quad && r.pairs % (r.halves ? 4 : 2) == 0; }
TurnPlan plan_turn(const small_rotation &r, bool vec, bool q, bool k, bool grad)
{
    TurnPlan p{};
    p.unit = vec ? (r.halves ? 4 : 2) : 1;
    p.units = r.pairs / p.unit;
    const int block = vec ? r.Cb / 4 : r.halves ? r.Cb : r.Cb % 2 ? 1 : r.Cb / 2;
    p.run = gcd(block, p.units);
    p.copies = (r.D - 2 * r.pairs) / (vec ? 4 : 1);
    p.copy_run = p.copies ? gcd(vec ? r.Cb / 4 : r.Cb, p.copies) : 1;
    const int items = (q ? r.heads : 0) / r.freq_heads + (k ? r.kv_heads : 0) / r.freq_heads;
    const double tokens = (double)r.N * r.S;
    p.parts = p.chunks = 1;
    if (!grad) {
        // two waves a SIMD at least, if there are heads enough to share out
        const double threads = tokens * p.units * r.freq_heads, want = 131072.0;
        if (threads < want) p.parts = shares_of(items, ceil(want / threads));
        return p;
    }
    p.run = power_of_two_of(p.run);
    if (p.run > 64) p.run = 64;
    const int at_once = 256 / p.run, wanted = 1024;
    const long rounds = ((long)r.N * r.S + at_once - 1) / at_once, sets = (long)r.freq_heads * (p.units / p.run);
    if (rounds * sets < wanted) p.parts = shares_of(items, (double)((wanted + rounds * sets - 1) / (rounds * sets)));
    long chunks = wanted / (sets * p.parts);
    if (chunks < 1) chunks = 1;
    if (chunks > rounds) chunks = rounds;
    p.per_chunk = (int)((rounds + chunks - 1) / chunks * at_once);
    p.chunks = (int)(((long)r.N * r.S + p.per_chunk - 1) / p.per_chunk);
    p.bytes = ((size_t)r.freq_heads * p.chunks * p.parts * r.axes * r.pairs * sizeof(double) + 255) / 256 * 256;
    return p;
}
size_t grad_bytes(const small_rotation &r)
{
    size_t most = 0;
    for (int vec = 0; vec < 2; ++vec) {
        if (vec && !turn_vec(r, r.D % 4 == 0 && r.Cb % 4 == 0)) continue;
        for (int parts = 1; parts < 4; ++parts) {
            const size_t b = plan_turn(r, vec, parts & 1, parts & 2, true).bytes;
            if (b > most) most = b;
        }
    }
    return most;
}
// (threads for pairs that turn and channels that do not, numbered in 31 bits each)
bool turn_launches(const small_rotation &r, bool vec) { return (double)r.N * r.S * (r.heads + r.kv_heads) * r.D / (vec ? 4 : 1) <= INT_MAX - 512.0; }

RotaryArgs rotary_args(const small_rotation &r)
{
    RotaryArgs x{};
    x.N = r.N; x.S = r.S; x.heads = r.heads; x.kv_heads = r.kv_heads; x.D = r.D; x.Cb = r.Cb;
    x.axes = r.axes; x.pairs = r.pairs; x.freq_heads = r.freq_heads; x.sign = 1.f;
    x.freq = r.freq; x.first = r.first; x.positions = r.positions;
    x.by_Cb = make_fastdiv(r.Cb); x.by_S = make_fastdiv(r.S); x.by_freq_heads = make_fastdiv(r.freq_heads);
    for (int e = 0; e < 4; ++e) {
        const bool used = e > 0 && e < r.axes && !r.positions;
        x.extent[e] = used ? r.extent[e] : 1;
        x.by_extent[e] = make_fastdiv(x.extent[e]);
    }
    return x;
}
void place(RotaryArgs &x, const TurnPlan &p, bool grad)
{
    x.run = p.run; x.runs = p.units / p.run; x.parts = p.parts; x.chunks = p.chunks; x.per_chunk = p.per_chunk;
    x.by_run = make_fastdiv(p.run); x.by_runs = make_fastdiv(x.runs); x.by_parts = make_fastdiv(p.parts); x.by_chunks = make_fastdiv(p.chunks);
    x.turn_threads = grad ? 0u : (unsigned)((double)x.N * x.S * p.units);          // (for every set of heads)
    x.by_sets = make_fastdiv(x.freq_heads * p.parts);
    const int copied = (x.q && x.q != x.qo ? x.heads : 0) + (x.k && x.k != x.ko ? x.kv_heads : 0);
    x.copy_run = p.copy_run; x.copy_runs = p.copies ? p.copies / p.copy_run : 1;
    x.by_copy_run = make_fastdiv(p.copy_run); x.by_copy_runs = make_fastdiv(x.copy_runs); x.by_copy_heads = make_fastdiv(copied ? copied : 1);
    x.copy_threads = (unsigned)((double)x.N * x.S * p.copies * copied);
}

// Floats from a head to the next, if they are the same from each to the next and the tensor is small enough for offsets of 32 bits in bytes; else 0.
long long head_step(const Laid &t, int heads, int D)
{
    if (t.floats() >= (size_t)1 << 30) return 0;
    return D % t.Cb == 0 ? (long long)(D / t.Cb * t.s.block) : (size_t)heads * D <= t.Cb ? D : 0;
}

// The rotation's own inputs, which nothing that is written may meet.
bool meets_rotation(const small_rotation &r, const Range &w)
{
    return meets_any(w, {bytes_of(r.freq, (size_t)r.freq_heads * r.axes * r.pairs * 4), bytes_of(r.first, (size_t)r.N * 4),
                         bytes_of(r.positions, (size_t)r.N * r.S * r.axes * 4)});
}

int rotary(const small_rotation &r, const float *q, const float *k, float *q_out, float *k_out, const small_tokens &qs, const small_tokens &ks,
           const small_tokens &qos, const small_tokens &kos, const float *yq, const float *yk, float *dfreq, bool back, void *workspace, size_t workspace_bytes, hipStream_t stream)
{
    if ((!q && !k) || !q != !q_out || !k != !k_out) return SMALL_ERR_NULL;
    if (const int rc = rotation_check(r)) return rc;
    if (const int rc = strides_check({q ? &qs : &ks, q ? &qos : &kos, k ? &ks : &qs, k ? &kos : &qos})) return rc;
    if (dfreq)
        if (const int rc = strides_check({q ? &r.q : &r.k, k ? &r.k : &r.q})) return rc;
    if (dfreq && ((q && !yq) || (k && !yk))) return SMALL_ERR_NULL;
    const Laid none{nullptr, {}, 1, 0, 1, 0};
    const Laid in[] = {q ? laid(r.N, r.S, r.heads, r.D, r.Cb, q, qs) : none, k ? laid(r.N, r.S, r.kv_heads, r.D, r.Cb, k, ks) : none};
    const Laid out[] = {q ? laid(r.N, r.S, r.heads, r.D, r.Cb, q_out, qos) : none, k ? laid(r.N, r.S, r.kv_heads, r.D, r.Cb, k_out, kos) : none};
    const Laid saved[] = {dfreq && q ? laid(r.N, r.S, r.heads, r.D, r.Cb, yq, r.q) : none, dfreq && k ? laid(r.N, r.S, r.kv_heads, r.D, r.Cb, yk, r.k) : none};
    bool vec = quads(r.D, r.Cb, {q ? &qs : &ks, q ? &qos : &kos, k ? &ks : &qs, k ? &kos : &qos}, {q, k, q_out, k_out});
    if (dfreq) vec = vec && quads(r.D, r.Cb, {q ? &r.q : &r.k, k ? &r.k : &r.q}, {q ? yq : nullptr, k ? yk : nullptr});
    vec = turn_vec(r, vec);
    if (!turn_launches(r, vec)) return SMALL_ERR_SHAPE;
    const TurnPlan p = plan_turn(r, vec, q, k, dfreq != nullptr);
    if (dfreq && !workspace_ok(workspace, workspace_bytes, p.bytes)) return SMALL_ERR_WORKSPACE;
    const Range flat[] = {bytes_of(dfreq, (size_t)r.freq_heads * r.axes * r.pairs * 4), dfreq ? bytes_of(workspace, p.bytes) : Range(nullptr, 0)};
    if (flat[0].meets(flat[1])) return SMALL_ERR_ALIAS;
    for (int t = 0; t < 2; ++t) {
        if (meets_rotation(r, flat[t])) return SMALL_ERR_ALIAS;
        if (!out[t].p) continue;
        if (!out[t].distinct()) return SMALL_ERR_SHAPE;
        if (meets_rotation(r, out[t].range())) return SMALL_ERR_ALIAS;
        for (int u = 0; u < 2; ++u) {
            const bool in_place = t == u && in[u].p == out[t].p && same(in[u].s, out[t].s);
            if (in[u].p && !in_place && !out[t].apart(in[u])) return SMALL_ERR_ALIAS;
            if (u != t && out[u].p && !out[t].apart(out[u])) return SMALL_ERR_ALIAS;
            if (saved[u].p && !out[t].apart(saved[u])) return SMALL_ERR_ALIAS;
            if (!out[t].apart(flat[u])) return SMALL_ERR_ALIAS;
        }
    }
    for (const Range &f : flat)
        for (int u = 0; u < 2; ++u)
            if ((in[u].p && !in[u].apart(f)) || (saved[u].p && !saved[u].apart(f))) return SMALL_ERR_ALIAS;
    RotaryArgs x = rotary_args(r);
    x.q = q; x.k = k; x.qo = q_out; x.ko = k_out;
    x.qs = strides(qs); x.ks = strides(ks); x.qos = strides(qos); x.kos = strides(kos);
    x.yq = yq; x.yk = yk; x.yqs = strides(r.q); x.yks = strides(r.k);
    x.partial = (double *)workspace;
    x.fast = vec;
    const auto step = [&](const Laid &t, int heads) {
        const long long floats = t.p ? head_step(t, heads, r.D) : 0;
        if (t.p && !floats) x.fast = 0;
        return floats;
    };
    x.q_step = step(in[0], r.heads); x.k_step = step(in[1], r.kv_heads);
    x.qo_step = step(out[0], r.heads); x.ko_step = step(out[1], r.kv_heads);
    x.yq_step = step(saved[0], r.heads); x.yk_step = step(saved[1], r.kv_heads);
    if (back) x.sign = -1.f;
    place(x, p, dfreq != nullptr);
    return from_hip(dfreq ? launch_rotary_grad(x, vec, r.halves != 0, r.from_inputs != 0, dfreq, stream) : launch_rotary(x, vec, r.halves != 0, stream));
}

// ---- the cache

int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

int cache_check(const small_cache &c)
{
    if (c.kind != SMALL_CACHE_F32 && c.kind != SMALL_CACHE_BF16 && c.kind != SMALL_CACHE_I8) return SMALL_ERR_SHAPE;
    if (c.pages <= 0 || c.page < 16 || c.page > 256 || (c.page & (c.page - 1)) || c.kv_heads <= 0 || c.D <= 0 || c.D > 256 || c.N <= 0 || c.per_stream <= 0) return SMALL_ERR_SHAPE;
    if ((double)c.per_stream * c.page > kFar || (double)c.N * c.per_stream > INT_MAX || (double)c.kv_heads * c.D > 1 << 24) return SMALL_ERR_SHAPE;
    return SMALL_OK;
}
int cache_memory(const small_cache &c)
{
    if (!c.keys || !c.values || !c.table || (c.kind == SMALL_CACHE_I8 && (!c.key_scales || !c.value_scales))) return SMALL_ERR_NULL;
    uintptr_t at = (uintptr_t)c.keys | (uintptr_t)c.values;
    if (c.kind == SMALL_CACHE_I8) at |= (uintptr_t)c.key_scales | (uintptr_t)c.value_scales;
    return at % 16 ? SMALL_ERR_SHAPE : SMALL_OK;
}
CacheArgs cache_args(const small_cache &c)
{
    const int size = cache_bytes(c.kind), fill = 16 / size;
    return CacheArgs{(char *)c.keys, (char *)c.values, c.key_scales, c.value_scales, c.kind, c.pages, log2_of(c.page), c.kv_heads, c.D, (c.D + fill - 1) / fill * fill,
                     c.per_stream, c.table, 0, nullptr, {}};
}
struct CacheRanges { Range r[4]; };
CacheRanges cache_ranges(const small_cache &c)
{
    const CacheArgs x = cache_args(c);
    const size_t rows = (size_t)c.pages * c.kv_heads * c.page, size = cache_bytes(c.kind), scales = c.kind == SMALL_CACHE_I8 ? rows * 4 : 0;
    return CacheRanges{{bytes_of(c.keys, rows * x.Dk * size), bytes_of(c.values, rows * c.D * size), bytes_of(scales ? c.key_scales : nullptr, scales),
                        bytes_of(scales ? c.value_scales : nullptr, scales)}};
}
Range table_range(const small_cache &c) { return bytes_of(c.table, (size_t)c.N * c.per_stream * 4); }

// A call that writes or reads spans: its arguments but for the tensors.
int plan_store(StoreArgs &x, const small_cache &c, const small_span &s, int heads, bool reads)
{
    x.c = cache_args(c);
    x.N = c.N; x.S = s.S;
    x.first = s.first; x.counts = s.counts;
    x.lanes_log2 = 2;
    while ((4 << x.lanes_log2) < c.D) ++x.lanes_log2;
    x.tile = !reads && s.S <= 4 ? 1 : 16;
    x.tiles = x.tile == 1 ? s.S : (s.S + 15) / 16 + (s.first != nullptr);       // (a span may begin inside a tile)
    x.items = heads + 2 * c.kv_heads;
    // four workgroups a compute unit, if there are heads enough to share out
    const double base = (double)c.N * x.tiles;
    x.parts = base < 1024 ? shares_of(x.items, ceil(1024 / base)) : 1;
    x.by_parts = make_fastdiv(x.parts); x.by_tiles = make_fastdiv(x.tiles);
    x.r.by_Cb = make_fastdiv(s.Cb);
    const double threads = ((x.tile << x.lanes_log2) + 63) / 64 * 64;
    return launches(base * x.parts, threads) && base * x.parts < INT_MAX ? SMALL_OK : SMALL_ERR_SHAPE;
}

// ---- attention over the cache

int token_check(const small_cache &c, const small_attn &a)
{
    if (const int rc = cache_check(c)) return rc;
    if (const int rc = sizes_check(a.N, a.Sq, a.heads, a.kv_heads, a.D, a.Cb, {&a.q, &a.out})) return rc;
    if (a.N != c.N || a.kv_heads != c.kv_heads || a.D != c.D || a.width != 1 || a.prefix || a.docs) return SMALL_ERR_SHAPE;
    if ((double)a.N * a.heads * a.Sq > INT_MAX || !isfinite(a.scale) || !(a.cap >= 0.f) || isinf(a.cap)) return SMALL_ERR_SHAPE;
    if (!a.table != !a.bucket) return SMALL_ERR_NULL;
    if (a.table && (a.reach < 0 || a.reach > kFar || a.buckets < 1 || (double)a.heads * a.buckets > 1 << 30)) return SMALL_ERR_SHAPE;
    return SMALL_OK;
}
// How the calls of these sizes share out their work (cache_token.hip): units' rows (one or two tiles), workgroups, and places of parts: one for each pair of a workgroup and a
// unit (such rows of a key head of a stream) that it has a part of, of which there are fewer than workgroups and units together.
struct TokenPlan {
    int rows, row_tiles, workgroups;
    bool joined;
    double rounds;
    size_t ml_at, units_at, bytes;
};
TokenPlan plan_token(const small_cache &c, const small_attn &a)
{
    TokenPlan p{};
    p.rows = a.heads / a.kv_heads * a.Sq;
    const TokenShape shape = token_shape(c.kind, c.D, p.rows);
    p.row_tiles = (p.rows + shape.rows - 1) / shape.rows;
    const long of_unit = ((long)c.per_stream * c.page + shape.keys - 1) / shape.keys;
    const double units = (double)a.N * a.kv_heads * p.row_tiles;
    p.rounds = units * of_unit;
    p.workgroups = (int)fmin(p.rounds, (double)shape.per_cu * device_cus());
    p.joined = of_unit > 1;
    const auto up = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    if (p.joined) {
        const size_t pieces = (size_t)(units + p.workgroups) * shape.rows;
        p.ml_at = up(pieces * a.D * sizeof(float));
        p.units_at = up(p.ml_at + pieces * sizeof(float2));
        p.bytes = up(p.units_at + (size_t)units * sizeof(int2));
    }
    return p;
}
bool token_launches(const small_attn &a, const TokenPlan &p)
{
    return p.rounds < 1 << 30 && launches((double)a.N * a.kv_heads * p.rows, 256);
}

}  // namespace

extern "C" {

int small_rotary_workspace(const small_rotation *r, size_t *bytes)
{
    if (!r || !bytes) return SMALL_ERR_NULL;
    if (const int rc = rotation_check(*r)) return rc;
    *bytes = grad_bytes(*r);
    return SMALL_OK;
}

int small_rotary(const small_rotation *r, const float *q, const float *k, float *q_out, float *k_out, void *stream)
{
    if (!r) return SMALL_ERR_NULL;
    return rotary(*r, q, k, q_out, k_out, r->q, r->k, r->q_out, r->k_out, nullptr, nullptr, nullptr, false, nullptr, 0, (hipStream_t)stream);
}

int small_rotary_grad(const small_rotation *r, const float *dq_out, const float *dk_out, const float *q, const float *k, float *dq, float *dk,
                      float *dfreq, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!r) return SMALL_ERR_NULL;
    return rotary(*r, dq_out, dk_out, dq, dk, r->q_out, r->k_out, r->dq, r->dk, q, k, dfreq, true, workspace, workspace_bytes, (hipStream_t)stream);
}

int small_cache_write(const small_cache *c, const small_span *s, const float *k, const float *v, const small_rotation *r, const float *q,
                      float *q_out, void *stream)
{
    if (!c || !s || !k || !v || !q != !q_out || (q && !r)) return SMALL_ERR_NULL;
    if (const int rc = cache_check(*c)) return rc;
    if (const int rc = cache_memory(*c)) return rc;
    if (const int rc = sizes_check(c->N, s->S, c->kv_heads, c->kv_heads, c->D, s->Cb, {&s->k, &s->v})) return rc;
    small_rotation turn{};
    if (r) {
        turn = *r;
        turn.first = nullptr;                                  // (the span's takes its place)
        if (const int rc = rotation_check(turn)) return rc;
        if (q)
            if (const int rc = strides_check({&r->q, &r->q_out})) return rc;
        if (r->N != c->N || r->S != s->S || r->kv_heads != c->kv_heads || r->D != c->D || r->Cb != s->Cb) return SMALL_ERR_SHAPE;
    }
    const Laid in[] = {laid(c->N, s->S, c->kv_heads, c->D, s->Cb, k, s->k), laid(c->N, s->S, c->kv_heads, c->D, s->Cb, v, s->v)};
    const CacheRanges held = cache_ranges(*c);
    const Range ints[] = {table_range(*c), bytes_of(s->first, (size_t)c->N * 4), bytes_of(s->counts, (size_t)c->N * 4)};
    for (int w = 0; w < 4; ++w) {
        for (const Laid &t : in)
            if (!t.apart(held.r[w])) return SMALL_ERR_ALIAS;
        for (const Range &t : ints)
            if (t.meets(held.r[w])) return SMALL_ERR_ALIAS;
        for (int o = 0; o < w; ++o)
            if (held.r[o].meets(held.r[w])) return SMALL_ERR_ALIAS;
        if (r && meets_rotation(turn, held.r[w])) return SMALL_ERR_ALIAS;
    }
    if (q) {
        const Laid queries = laid(c->N, s->S, r->heads, c->D, s->Cb, q, r->q), out = laid(c->N, s->S, r->heads, c->D, s->Cb, q_out, r->q_out);
        if (!out.distinct()) return SMALL_ERR_SHAPE;
        if (!(q == q_out && same(r->q, r->q_out)) && !out.apart(queries)) return SMALL_ERR_ALIAS;
        for (const Laid &t : in)
            if (!out.apart(t)) return SMALL_ERR_ALIAS;
        for (const Range &t : ints)
            if (!out.apart(t)) return SMALL_ERR_ALIAS;
        for (const Range &t : held.r)
            if (!out.apart(t) || !queries.apart(t)) return SMALL_ERR_ALIAS;
        if (meets_rotation(turn, out.range())) return SMALL_ERR_ALIAS;
    }
    StoreArgs x{};
    if (r) x.r = rotary_args(turn);
    if (const int rc = plan_store(x, *c, *s, q ? r->heads : 0, false)) return rc;
    x.k = k; x.v = v;
    x.ks = strides(s->k); x.vs = strides(s->v);
    x.turns = r != nullptr;
    bool vec = quads(c->D, s->Cb, {&s->k, &s->v}, {k, v});
    if (r) {
        x.r.q = q; x.r.qo = q_out;
        x.r.qs = strides(r->q); x.r.qos = strides(r->q_out);
        if (q) vec = vec && quads(c->D, s->Cb, {&r->q, &r->q_out}, {q, q_out});
        x.by_per_q = make_fastdiv(r->heads / r->freq_heads);
    }
    x.k_step = head_step(in[0], c->kv_heads, c->D); x.v_step = head_step(in[1], c->kv_heads, c->D);
    x.fast = vec && x.k_step && x.v_step;
    if (q) {
        x.q_step = head_step(laid(c->N, s->S, r->heads, c->D, s->Cb, q, r->q), r->heads, c->D);
        x.qo_step = head_step(laid(c->N, s->S, r->heads, c->D, s->Cb, q_out, r->q_out), r->heads, c->D);
        x.fast = x.fast && x.q_step && x.qo_step;
    }
    return from_hip(launch_cache_write(x, vec, r && r->halves, (hipStream_t)stream));
}

int small_cache_read(const small_cache *c, const small_span *s, float *k, float *v, void *stream)
{
    if (!c || !s || !k || !v) return SMALL_ERR_NULL;
    if (const int rc = cache_check(*c)) return rc;
    if (const int rc = cache_memory(*c)) return rc;
    if (const int rc = sizes_check(c->N, s->S, c->kv_heads, c->kv_heads, c->D, s->Cb, {&s->k, &s->v})) return rc;
    const Laid out[] = {laid(c->N, s->S, c->kv_heads, c->D, s->Cb, k, s->k), laid(c->N, s->S, c->kv_heads, c->D, s->Cb, v, s->v)};
    const CacheRanges held = cache_ranges(*c);
    for (const Laid &o : out) {
        if (!o.distinct()) return SMALL_ERR_SHAPE;
        for (const Range &t : held.r)
            if (!o.apart(t)) return SMALL_ERR_ALIAS;
        if (!o.apart(table_range(*c)) || !o.apart(bytes_of(s->first, (size_t)c->N * 4)) || !o.apart(bytes_of(s->counts, (size_t)c->N * 4))) return SMALL_ERR_ALIAS;
    }
    if (!out[0].apart(out[1])) return SMALL_ERR_ALIAS;
    StoreArgs x{};
    if (const int rc = plan_store(x, *c, *s, 0, true)) return rc;
    x.k_out = k; x.v_out = v;
    x.ks = strides(s->k); x.vs = strides(s->v);
    const bool vec = quads(c->D, s->Cb, {&s->k, &s->v}, {k, v});
    x.k_step = head_step(out[0], c->kv_heads, c->D); x.v_step = head_step(out[1], c->kv_heads, c->D);
    x.fast = vec && x.k_step && x.v_step;
    return from_hip(launch_cache_read(x, vec, (hipStream_t)stream));
}

int small_cache_attention_workspace(const small_cache *c, const small_attn *a, size_t *bytes)
{
    if (!c || !a || !bytes) return SMALL_ERR_NULL;
    if (const int rc = token_check(*c, *a)) return rc;
    const TokenPlan p = plan_token(*c, *a);
    if (!token_launches(*a, p)) return SMALL_ERR_SHAPE;
    *bytes = p.bytes;
    return SMALL_OK;
}

int small_cache_attention(const small_cache *c, const small_attn *a, const float *q, float *out, float *lse, void *workspace,
                          size_t workspace_bytes, void *stream)
{
    if (!c || !a || !q || !out || !a->lengths) return SMALL_ERR_NULL;
    if (const int rc = token_check(*c, *a)) return rc;
    if (const int rc = cache_memory(*c)) return rc;
    const TokenPlan p = plan_token(*c, *a);
    if (!token_launches(*a, p)) return SMALL_ERR_SHAPE;
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return SMALL_ERR_WORKSPACE;
    const Laid queries = laid(a->N, a->Sq, a->heads, a->D, a->Cb, q, a->q), o = laid(a->N, a->Sq, a->heads, a->D, a->Cb, out, a->out);
    if (!o.distinct()) return SMALL_ERR_SHAPE;
    const Range l = bytes_of(lse, (size_t)a->N * a->heads * a->Sq * 4), ws = bytes_of(workspace, p.bytes);
    const CacheRanges held = cache_ranges(*c);
    const size_t N = a->N;
    const Range reads[] = {held.r[0], held.r[1], held.r[2], held.r[3], table_range(*c), bytes_of(a->lengths, N * 4), bytes_of(a->first, N * 4),
                           bytes_of(a->slopes, (size_t)a->heads * 4), bytes_of(a->table, a->table ? (size_t)a->heads * a->buckets * 4 : 0),
                           bytes_of(a->bucket, a->bucket ? (2 * (size_t)a->reach + 1) * 4 : 0)};
    if (!o.apart(queries) || !o.apart(l) || !o.apart(ws) || l.meets(ws) || !queries.apart(l) || !queries.apart(ws)) return SMALL_ERR_ALIAS;
    for (const Range &r : reads)
        if (!o.apart(r) || l.meets(r) || ws.meets(r)) return SMALL_ERR_ALIAS;
    AttnArgs x{};
    x.q = q; x.o = out; x.lse = lse;
    x.qs = strides(a->q); x.os = strides(a->out);
    x.N = a->N; x.Sq = a->Sq; x.Sk = c->per_stream * c->page; x.heads = a->heads; x.group = a->heads / a->kv_heads; x.D = a->D; x.Cb = a->Cb;
    x.scale = a->scale; x.cap = a->cap;
    x.causal = 1; x.width = 1; x.reach = a->reach; x.buckets = a->buckets;
    x.lengths = a->lengths; x.first = a->first; x.slopes = a->slopes; x.table = a->table; x.bucket = a->bucket;
    x.pack = 1; x.head_sets = a->kv_heads; x.rows = p.rows; x.row_tiles = p.row_tiles;
    x.by_Cb = make_fastdiv(a->Cb); x.by_Sq = make_fastdiv(a->Sq); x.by_width = make_fastdiv(1); x.by_group = make_fastdiv(x.group);
    x.by_sets = make_fastdiv(a->kv_heads);
    x.part_o = (float *)workspace;
    x.part_ml = (float2 *)((char *)workspace + p.ml_at);
    x.vec = quads(a->D, a->Cb, {&a->q, &a->out}, {q, out});
    CacheArgs held_args = cache_args(*c);
    held_args.workgroups = p.workgroups;
    held_args.units = p.joined ? (int2 *)((char *)workspace + p.units_at) : nullptr;
    held_args.by_rows = make_fastdiv(p.rows);
    return from_hip(launch_cache_token(x, held_args, p.joined, (hipStream_t)stream));
}

}  // extern "C"
