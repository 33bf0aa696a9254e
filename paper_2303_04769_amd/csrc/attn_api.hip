// C-ABI layer of the attention block (include/small_attn.h has the contract of every entry point): argument checks and sizes, host only.
#include "../../include/small.h"
#include "../include/small_attn.h"
#include "attn_parts.h"

#include <initializer_list>

#include <limits.h>
#include <math.h>

using namespace small;

namespace {

constexpr size_t kWorkspaceAlign = 256;

inline int from_hip(hipError_t e) { return e == hipSuccess ? SMALL_OK : SMALL_ERR_LAUNCH; }

// A range of device memory, in bytes.
struct Range {
    uintptr_t at, end;
    Range(const void *p, size_t floats) : at((uintptr_t)p), end((uintptr_t)p + floats * sizeof(float)) {}
    bool meets(const Range &o) const { return at < o.end && o.at < end; }
};

bool workspace_ok(const void *ws, size_t have, size_t need)
{
    return need == 0 || (ws && have >= need && (uintptr_t)ws % kWorkspaceAlign == 0);
}

// Sizes of a group normalization: values of the tensor, or 0 and the error.
size_t norm_elems(int N, int C, int H, int W, int G, int Cb, int *rc)
{
    *rc = SMALL_ERR_SHAPE;
    if (N <= 0 || C <= 0 || H <= 0 || W <= 0 || G <= 0 || Cb <= 0 || C % G || C % Cb) return 0;
    if (Cb > 4096 || (Cb % 4 && Cb > 1024)) { *rc = SMALL_ERR_BLOCK; return 0; }
    // a plane and a group within 32-bit offsets, the tensor's size within 2^40 values, a workgroup's number in 31 bits
    const double n = (double)N * C * H * W;
    if ((double)H * W * Cb > INT_MAX || (double)H * W * (C / G) > INT_MAX || n > 1e12 || (double)N * C > INT_MAX) return 0;
    if ((double)groupnorm_workspace(N, C, H * W, G, Cb) / (sizeof(float) * 2 * Cb) > INT_MAX) return 0;
    *rc = SMALL_OK;
    return (size_t)N * C * H * W;
}

int act_ok(int act) { return act == SMALL_ACT_NONE || act == SMALL_ACT_RELU || act == SMALL_ACT_SILU; }

// Blocks beyond 1024 channels need four-channel accesses.
bool block_ok(int Cb, uintptr_t bits) { return Cb <= 1024 || bits % 16 == 0; }

// ---- attention

// A tensor of `heads` heads over `tokens` tokens, as the strides lay it out.
struct Laid {
    const float *p;
    small_tokens s;
    size_t n, blocks, tokens, Cb;
    size_t floats() const { return (n - 1) * s.image + (blocks - 1) * s.block + (tokens - 1) * s.token + Cb; }
    Range range() const { return Range(p, floats()); }
    // (stride, size) by falling stride
    void levels(size_t (&stride)[3], size_t (&size)[3]) const
    {
        const size_t st[3] = {s.image, s.block, s.token}, sz[3] = {n, blocks, tokens};
        int order[3] = {0, 1, 2};
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2 - i; ++j)
                if (st[order[j]] < st[order[j + 1]]) { const int t = order[j]; order[j] = order[j + 1]; order[j + 1] = t; }
        for (int i = 0; i < 3; ++i) { stride[i] = st[order[i]]; size[i] = sz[order[i]]; }
    }
    // Whether no two of its values share a place: every stride passes all that lies below it.
    bool distinct() const
    {
        size_t stride[3], size[3], below = Cb;
        levels(stride, size);
        for (int i = 2; i >= 0; --i) {
            if (size[i] == 1) continue;
            if (stride[i] < below) return false;
            below += (size[i] - 1) * stride[i];
        }
        return true;
    }
    // Whether it shares no place with o, as far as ranges, or equal strides that interleave them, show.
    bool apart(const Laid &o) const
    {
        if (!range().meets(o.range())) return true;
        if (((uintptr_t)p - (uintptr_t)o.p) % sizeof(float)) return false;
        size_t sa[3], na[3], sb[3], nb[3];
        levels(sa, na);
        o.levels(sb, nb);
        long long rel = ((long long)(uintptr_t)o.p - (long long)(uintptr_t)p) / (long long)sizeof(float);
        for (int i = 0; i < 3; ++i) {
            if (sa[i] != sb[i] || sa[i] == 0) return false;
            size_t ea = Cb, eb = o.Cb;
            for (int k = i + 1; k < 3; ++k) { ea += (na[k] - 1) * sa[k]; eb += (nb[k] - 1) * sb[k]; }
            const long long st = (long long)sa[i];
            rel = (rel % st + st) % st;
            if ((size_t)rel >= ea && (size_t)rel + eb <= sa[i]) return true;
        }
        return false;
    }
    bool apart(const Range &r) const { return !range().meets(r); }
};

Laid laid(const small_attn &a, const float *p, const small_tokens &s, int heads, int tokens)
{
    return Laid{p, s, (size_t)a.N, ((size_t)heads * a.D + a.Cb - 1) / a.Cb, (size_t)tokens, (size_t)a.Cb};
}

int attn_check(const small_attn &a)
{
    if (a.N <= 0 || a.Sq <= 0 || a.Sk <= 0 || a.heads <= 0 || a.kv_heads <= 0 || a.D <= 0 || a.Cb <= 0) return SMALL_ERR_SHAPE;
    if (a.heads % a.kv_heads || a.D > 256 || a.Sq > kFar || a.Sk > kFar || a.Cb > 1 << 20) return SMALL_ERR_SHAPE;
    if ((double)a.heads * a.D > 1 << 24 || (double)a.N * a.heads * a.Sq > INT_MAX || (double)a.N * a.kv_heads * a.Sk > 1e12) return SMALL_ERR_SHAPE;
    if ((double)a.N * a.heads * ((a.Sk + 63) / 64) > INT_MAX) return SMALL_ERR_SHAPE;
    if (!isfinite(a.scale) || !(a.cap >= 0.f) || isinf(a.cap)) return SMALL_ERR_SHAPE;
    const size_t most = (size_t)1 << 40;
    for (const small_tokens *s : {&a.q, &a.k, &a.v, &a.out, &a.dout, &a.dq, &a.dk, &a.dv})
        if (s->image > most || s->block > most || s->token > most) return SMALL_ERR_SHAPE;
    if (!a.table != !a.bucket) return SMALL_ERR_NULL;
    if (a.width < 1 || a.width > kFar || (a.table && (a.reach < 0 || a.reach > kFar || a.buckets < 1))) return SMALL_ERR_SHAPE;
    return SMALL_OK;
}

// Words for the powers of two of so many tiles: their tokens', 16-byte aligned, then their own.
size_t parts_words(size_t tiles) { return (65 * tiles + 3) / 4 * 4; }

// What a call of these sizes runs: few rows against the cache, or tiles of rows, these with fp32 products or with values in two parts; and over
// how many workgroups a row's keys are split.
struct AttnPlan {
    bool token, parts;
    int pack, head_sets, rows, row_tiles, splits;
    size_t ml_at, k_at, v_at, exps_at, bytes;          // places in the workspace, in bytes
};
// Where values in two parts take a forward call: keys and values are laid out for it once, which rows of their heads and products have to pay for. fp32 -> parts:
// 8 x 8 pixels, 512 images, 18 -> 35 us; 10 x 10, 200 images, 30 -> 33; 14 x 14, 16 images, 21 -> 24, 64 images 61 -> 53; 400 frames, 4 heads of 64, 23 -> 22;
// 150 frames, 4 heads a key head, 16 sequences, 31 -> 20.
bool forward_in_parts(const small_attn &a)
{
    const double rows = (double)(a.heads / a.kv_heads) * a.Sq, work = (double)a.N * a.heads * a.Sq * a.Sk * a.D;
    return a.D <= 128 && (rows >= 256 ? work >= 4e7 : rows >= 128 && work >= 3e8);
}
AttnPlan plan_attn(const small_attn &a)
{
    AttnPlan p{};
    const int group = a.heads / a.kv_heads;
    const long packed = (long)group * a.Sq, cus = device_cus();
    p.token = packed <= 16;
    p.pack = group > 1 && (p.token || a.Sq < 64);
    p.head_sets = p.pack ? a.kv_heads : a.heads;
    p.rows = (int)(p.pack ? packed : a.Sq);
    p.parts = !p.token && !p.pack && forward_in_parts(a);
    const long sets = (long)a.N * p.head_sets;
    p.row_tiles = p.token ? 1 : (p.rows + 63) / 64;
    const long base = sets * p.row_tiles;
    // Parts of 256 keys at least. Tiles of rows: two workgroups a compute unit. Single tokens: one round of workgroups, or, where there is about one without
    // parts, four, whose lengths may differ (64 streams of 2048 to 16384 keys: 302 us with two rounds, 250 with four, 262 with eight).
    const long most = (a.Sk + 255) / 256;
    const long want = p.token ? (base < cus / 2 ? cus / base : (4 * cus + base - 1) / base) : base < 2 * cus ? (2 * cus + base - 1) / base : 1;
    p.splits = (int)(want < most ? want : most);
    if (p.splits < 1) p.splits = 1;
    const auto up = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    if (p.splits > 1) {
        const size_t pieces = (size_t)sets * p.rows * p.splits;
        p.ml_at = up(pieces * a.D * sizeof(float));
        p.bytes = up(p.ml_at + pieces * sizeof(float2));
    }
    if (p.parts) {
        const size_t tiles = (size_t)a.N * a.kv_heads * ((a.Sk + 63) / 64), image = tiles * parts_tile_bytes(parts_steps(a.D));
        p.k_at = p.bytes;
        p.v_at = p.k_at + image;
        p.exps_at = p.v_at + image;
        p.bytes = up(p.exps_at + 2 * parts_words(tiles) * sizeof(int));
    }
    return p;
}

TokenStrides strides(const small_tokens &s) { return TokenStrides{(long long)s.image, (long long)s.block, (long long)s.token}; }

AttnArgs attn_args(const small_attn &a, const float *q, const float *k, const float *v, const float *o)
{
    AttnArgs x{};
    x.q = q; x.k = k; x.v = v; x.o = const_cast<float *>(o);
    x.qs = strides(a.q); x.ks = strides(a.k); x.vs = strides(a.v); x.os = strides(a.out);
    x.N = a.N; x.Sq = a.Sq; x.Sk = a.Sk; x.heads = a.heads; x.group = a.heads / a.kv_heads; x.D = a.D; x.Cb = a.Cb;
    x.scale = a.scale; x.cap = a.cap;
    x.causal = a.causal; x.width = a.width; x.reach = a.reach; x.buckets = a.buckets;
    x.lengths = a.lengths; x.first = a.first; x.prefix = a.prefix; x.docs = a.docs;
    x.slopes = a.slopes; x.table = a.table; x.bucket = a.bucket;
    x.by_Cb = make_fastdiv(a.Cb); x.by_Sq = make_fastdiv(a.Sq); x.by_width = make_fastdiv(a.width); x.by_group = make_fastdiv(x.group);
    return x;
}

void place(AttnArgs &x, const AttnPlan &p, void *ws)
{
    x.pack = p.pack; x.head_sets = p.head_sets; x.rows = p.rows; x.row_tiles = p.row_tiles; x.splits = p.splits;
    x.by_tiles = make_fastdiv(p.row_tiles); x.by_sets = make_fastdiv(p.head_sets); x.by_splits = make_fastdiv(p.splits);
    x.part_o = (float *)ws;
    x.part_ml = (float2 *)((char *)ws + p.ml_at);
}

// The images of keys and values in the workspace, and the launch that makes them.
hipError_t make_parts(AttnArgs &x, const AttnPlan &p, const small_attn &a, void *ws, bool vec, hipStream_t s)
{
    const int tiles = (a.Sk + 63) / 64;
    const size_t all = (size_t)a.N * a.kv_heads * tiles;
    int *const k_words = (int *)((char *)ws + p.exps_at), *const v_words = k_words + parts_words(all);
    PartsArgs args{};
    args.count = 2;
    args.t[0] = PartsTensor{x.k, x.ks, a.kv_heads, a.Sk, tiles, 0, (char *)ws + p.k_at, k_words + 64 * all, k_words, 0};
    args.t[1] = PartsTensor{x.v, x.vs, a.kv_heads, a.Sk, tiles, 0, (char *)ws + p.v_at, v_words + 64 * all, v_words, 0};
    x.k_tok = args.t[0].image; x.k_exps = args.t[0].exps; x.k_each = args.t[0].each;
    x.v_tok = args.t[1].image; x.v_exps = args.t[1].exps; x.v_each = args.t[1].each;
    return launch_make_parts(x, args, vec, s);
}

// Four channels of a head at a time: they stand together in every tensor.
bool attn_vec(const small_attn &a, std::initializer_list<const void *> tensors)
{
    size_t bits = 0;
    for (const small_tokens *s : {&a.q, &a.k, &a.v, &a.out}) bits |= s->image | s->block | s->token;
    uintptr_t at = 0;
    for (const void *t : tensors) at |= (uintptr_t)t;
    return a.D % 4 == 0 && a.Cb % 4 == 0 && bits % 4 == 0 && at % 16 == 0;
}

// Bytes of the expanded bias of the heads that a tile of rows has, if it goes into LDS.
size_t bias_bytes(const small_attn &a, const AttnPlan &p)
{
    if (!a.table) return 0;
    const int span = 64 / a.Sq + 2, group = a.heads / a.kv_heads, heads = p.pack ? (span < group ? span : group) : 1;
    const double offsets = (double)heads * (2.0 * a.reach + 1);
    return offsets <= kBiasLds ? (size_t)offsets * sizeof(float) : 0;
}

// Bytes of LDS that the rows' gradient in parts has for its tiles, the expanded bias and `copies` sets of the sums by offset (attn_parts_grad.hip).
size_t grad_lds(const small_attn &a, int copies)
{
    const size_t size = a.table ? 2 * (size_t)a.reach + 1 : 0;
    return 3 * parts_tile_bytes(parts_steps(a.D)) + sizeof(float) * (size + (size ? copies * (size + 1) : 0));
}
// Where values in two parts take a gradient call: with a bias, one whose sums by offset fit LDS, four sets of them at least (wanted or not: the workspace must do for both).
// fp32 -> parts: 20 frames, 4 heads of 16, a bias by buckets, 48 -> 43 us;
// 100 frames, 4 heads of 32, 37 -> 33, with a bias 76 -> 53; 14 x 14 pixels, 8 images, 126 -> 76; 10 x 10, 24 images, no bias, 37 -> 38, 200 images 142 -> 109.
bool grad_in_parts(const small_attn &a)
{
    return a.D <= 128 && (!a.table || (a.reach < 2048 && grad_lds(a, 4) <= kGradLds));
}

// The gradient's workspace: delta and share [N][heads][Sq]; with a table its sums by offset, of every tile of rows and of every head; in parts the images of keys, values,
// queries and dout, their powers of two, and dk's and dv's parts where a key tile's rows are shared out. Places in bytes.
struct GradPlan {
    bool parts;
    int row_tiles, key_tiles, splits, row_parts;
    size_t part_at, sums_at, images[4], exps[4], dkv_at, bytes;
};
GradPlan plan_grad(const small_attn &a)
{
    GradPlan p{};
    p.row_tiles = (a.Sq + 63) / 64;
    p.key_tiles = (a.Sk + 63) / 64;
    p.splits = p.row_parts = 1;
    size_t end = 0;
    const auto take = [&](size_t bytes) { const size_t at = end; end += (bytes + 255) / 256 * 256; return at; };
    take(2 * (size_t)a.N * a.heads * a.Sq * sizeof(float));
    if (a.table) {
        const size_t size = 2 * (size_t)a.reach + 1;
        p.part_at = take((size_t)a.N * a.heads * p.row_tiles * size * sizeof(float));
        p.sums_at = take((size_t)a.heads * size * sizeof(float));
    }
    p.parts = grad_in_parts(a);
    if (p.parts) {
        const size_t tile = parts_tile_bytes(parts_steps(a.D)), keys = (size_t)a.N * a.kv_heads * p.key_tiles, rows = (size_t)a.N * a.heads * p.row_tiles;
        for (int x = 0; x < 4; ++x) p.images[x] = take((x < 2 ? keys : rows) * tile);      // k, v; q, dout
        for (int x = 0; x < 4; ++x) p.exps[x] = take(parts_words(x < 2 ? keys : rows) * sizeof(int));
        // six workgroups a compute unit: by heads that share a key head, then by rows of 256 at least
        const long want = (6L * device_cus() + (long)keys - 1) / (long)keys;
        const int group = a.heads / a.kv_heads;
        int heads = 1;
        while (heads < group && (heads < want || group % heads)) ++heads;
        long rows_of = (want + heads - 1) / heads;
        if (rows_of > (a.Sq + 255) / 256) rows_of = (a.Sq + 255) / 256;
        p.row_parts = (int)(rows_of < 1 ? 1 : rows_of);
        p.splits = heads * p.row_parts;
        if (p.splits > 1) p.dkv_at = take((size_t)p.splits * a.N * a.kv_heads * a.Sk * 2 * a.D * sizeof(float));
    }
    p.bytes = end;
    return p;
}
// Whether every launch of a call is one: a grid has fewer than 2^32 threads. (Asked for before the first, so that a call is enqueued whole or not at all.)
bool launches(double workgroups, double threads) { return workgroups * threads < 4294967296.0; }
bool attn_launches(const small_attn &a, const AttnPlan &p)
{
    return p.token || (launches((double)a.N * p.head_sets * p.row_tiles * p.splits, 256) && (!p.parts || launches(2.0 * a.N * a.kv_heads * ((a.Sk + 63) / 64), 256)));
}
bool grad_launches(const small_attn &a, const GradPlan &p)
{
    const double keys = (double)a.N * a.kv_heads * p.key_tiles, rows = (double)a.N * a.heads * p.row_tiles;
    const double sums = a.table ? (double)a.heads * ((2.0 * a.reach + 1) / 32 + 1) : 0, buckets = a.table ? (double)a.heads * (a.buckets / 32.0 + 1) : 0;
    return launches(2 * (keys + rows), 256) && launches(sums, 1024) && launches(buckets, 1024);
}
bool grad_vec(const small_attn &a)
{
    size_t bits = 0;
    for (const small_tokens *s : {&a.dout, &a.dq, &a.dk, &a.dv}) bits |= s->image | s->block | s->token;
    return bits % 4 == 0;
}

// Whether what a call writes meets the masks and biases that it reads.
bool meets_masks(const small_attn &a, const Range &w)
{
    const size_t N = a.N, table = a.table ? (size_t)a.heads * a.buckets : 0, map = a.bucket ? 2 * (size_t)a.reach + 1 : 0;
    const Range reads[] = {Range(a.lengths, a.lengths ? N : 0), Range(a.first, a.first ? N : 0), Range(a.prefix, a.prefix ? N : 0),
                           Range(a.docs, a.docs ? N * a.Sk : 0), Range(a.slopes, a.slopes ? a.heads : 0), Range(a.table, table), Range(a.bucket, map)};
    for (const Range &r : reads)
        if (w.meets(r)) return true;
    return false;
}

}  // namespace

extern "C" {

int small_attention_workspace(const small_attn *a, int grad, size_t *bytes)
{
    if (!a || !bytes) return SMALL_ERR_NULL;
    if (const int rc = attn_check(*a)) return rc;
    const AttnPlan forward = plan_attn(*a);
    const GradPlan gradient = plan_grad(*a);
    if (!(grad ? grad_launches(*a, gradient) : attn_launches(*a, forward))) return SMALL_ERR_SHAPE;
    *bytes = grad ? gradient.bytes : forward.bytes;
    return SMALL_OK;
}

int small_attention(const small_attn *a, const float *q, const float *k, const float *v, float *out, float *lse, void *workspace,
                    size_t workspace_bytes, void *stream)
{
    if (!a || !q || !k || !v || !out) return SMALL_ERR_NULL;
    if (const int rc = attn_check(*a)) return rc;
    const AttnPlan p = plan_attn(*a);
    if (!attn_launches(*a, p)) return SMALL_ERR_SHAPE;
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return SMALL_ERR_WORKSPACE;
    const Laid o = laid(*a, out, a->out, a->heads, a->Sq);
    const Laid in[] = {laid(*a, q, a->q, a->heads, a->Sq), laid(*a, k, a->k, a->kv_heads, a->Sk), laid(*a, v, a->v, a->kv_heads, a->Sk)};
    if (!o.distinct()) return SMALL_ERR_SHAPE;
    const Range l(lse, lse ? (size_t)a->N * a->heads * a->Sq : 0), ws(workspace, p.bytes / sizeof(float));
    if (!o.apart(l) || !o.apart(ws) || l.meets(ws) || meets_masks(*a, o.range()) || meets_masks(*a, l) || meets_masks(*a, ws)) return SMALL_ERR_ALIAS;
    for (const Laid &t : in)
        if (!o.apart(t) || !t.apart(l) || !t.apart(ws)) return SMALL_ERR_ALIAS;
    AttnArgs x = attn_args(*a, q, k, v, out);
    x.lse = lse;
    place(x, p, workspace);
    const bool vec = attn_vec(*a, {q, k, v, out});
    x.vec = vec;
    const size_t bias = p.token ? 0 : bias_bytes(*a, p);
    x.bias_lds = bias != 0;
    hipError_t e = p.parts ? make_parts(x, p, *a, workspace, vec, (hipStream_t)stream) : hipSuccess;
    if (e == hipSuccess)
        e = p.token ? launch_attn_token(x, vec, (hipStream_t)stream)
            : p.parts ? launch_attn_rows_parts(x, bias, (hipStream_t)stream) : launch_attn_rows(x, vec, bias, (hipStream_t)stream);
    if (e == hipSuccess && p.splits > 1) e = launch_attn_join(x, (hipStream_t)stream);
    return from_hip(e);
}

int small_attention_grad(const small_attn *a, const float *q, const float *k, const float *v, const float *out, const float *lse,
                         const float *dout, float *dq, float *dk, float *dv, float *dtable, void *workspace, size_t workspace_bytes,
                         void *stream)
{
    if (!a || !q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv) return SMALL_ERR_NULL;
    if (const int rc = attn_check(*a)) return rc;
    if (dtable && !a->table) return SMALL_ERR_NULL;
    const GradPlan p = plan_grad(*a);
    if (!grad_launches(*a, p)) return SMALL_ERR_SHAPE;
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return SMALL_ERR_WORKSPACE;
    const Laid in[] = {laid(*a, q, a->q, a->heads, a->Sq), laid(*a, k, a->k, a->kv_heads, a->Sk), laid(*a, v, a->v, a->kv_heads, a->Sk),
                       laid(*a, out, a->out, a->heads, a->Sq), laid(*a, dout, a->dout, a->heads, a->Sq)};
    const Laid made[] = {laid(*a, dq, a->dq, a->heads, a->Sq), laid(*a, dk, a->dk, a->kv_heads, a->Sk), laid(*a, dv, a->dv, a->kv_heads, a->Sk)};
    const Range flat[] = {Range(workspace, p.bytes / sizeof(float)), Range(dtable, dtable ? (size_t)a->heads * a->buckets : 0)};
    const Range l(lse, (size_t)a->N * a->heads * a->Sq);
    if (flat[0].meets(flat[1])) return SMALL_ERR_ALIAS;
    for (const Range &f : flat) {
        if (f.meets(l) || meets_masks(*a, f)) return SMALL_ERR_ALIAS;
        for (const Laid &t : in)
            if (!t.apart(f)) return SMALL_ERR_ALIAS;
    }
    for (const Laid &m : made) {
        if (!m.distinct()) return SMALL_ERR_SHAPE;
        if (!m.apart(l) || !m.apart(flat[0]) || !m.apart(flat[1]) || meets_masks(*a, m.range())) return SMALL_ERR_ALIAS;
        for (const Laid &t : in)
            if (!m.apart(t)) return SMALL_ERR_ALIAS;
        for (const Laid &o : made)
            if (&o != &m && !m.apart(o)) return SMALL_ERR_ALIAS;
    }
    AttnArgs x = attn_args(*a, q, k, v, out);
    x.lse_in = lse; x.dout = dout; x.dq = dq; x.dk = dk; x.dv = dv;
    x.dos = strides(a->dout); x.dqs = strides(a->dq); x.dks = strides(a->dk); x.dvs = strides(a->dv);
    x.row_tiles = p.row_tiles; x.key_tiles = p.key_tiles; x.splits = p.splits; x.row_parts = p.row_parts;
    x.by_tiles = make_fastdiv(p.row_tiles); x.by_key_tiles = make_fastdiv(p.key_tiles); x.by_heads = make_fastdiv(a->heads);
    x.by_sets = make_fastdiv(a->kv_heads); x.by_splits = make_fastdiv(p.splits);
    x.by_code = make_fastdiv(2 * a->width - 1);
    char *const at = (char *)workspace;
    x.delta = (float *)at;
    x.share = x.delta + (size_t)a->N * a->heads * a->Sq;
    x.part_bias = dtable ? (float *)(at + p.part_at) : nullptr;
    x.vec = attn_vec(*a, {q, k, v, out, dout, dq, dk, dv}) && grad_vec(*a);
    const double size = 2.0 * a->reach + 1;
    x.bias_lds = a->table && size <= kBiasLds;
    x.bias_acc_lds = dtable && size <= kBiasLds;
    // sets of sums by offset, 16, 8 or 4: as many as leave the three workgroups a compute unit (two from 65 channels on) that registers allow
    // (14 x 14 pixels, 8 heads, 64 images, all of the gradient: 16 sets 261 us, 8 sets 246, 4 sets 259)
    x.bias_copies = 16;
    while (x.bias_copies > 4 && grad_lds(*a, x.bias_copies) > (a->D <= 64 ? 53000 : 79000)) x.bias_copies /= 2;
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    x.share_known = a->slopes && dtable;
    if (x.share_known) e = launch_attn_grad_shares(x, x.vec, s);
    if (e != hipSuccess) return from_hip(e);
    if (p.parts) {
        PartsArgs args{};
        args.count = 4;
        const size_t keys = (size_t)a->N * a->kv_heads * p.key_tiles, rows = (size_t)a->N * a->heads * p.row_tiles;
        int *const each[] = {(int *)(at + p.exps[0]), (int *)(at + p.exps[1]), (int *)(at + p.exps[2]), (int *)(at + p.exps[3])};
        args.t[0] = PartsTensor{k, x.ks, a->kv_heads, a->Sk, p.key_tiles, 0, at + p.images[0], each[0] + 64 * keys, each[0], 0};
        args.t[1] = PartsTensor{v, x.vs, a->kv_heads, a->Sk, p.key_tiles, 0, at + p.images[1], each[1] + 64 * keys, each[1], 0};
        args.t[2] = PartsTensor{q, x.qs, a->heads, a->Sq, p.row_tiles, 1, at + p.images[2], each[2] + 64 * rows, each[2], 0};
        args.t[3] = PartsTensor{dout, x.dos, a->heads, a->Sq, p.row_tiles, 1, at + p.images[3], each[3] + 64 * rows, each[3], 0};
        x.k_tok = args.t[0].image; x.v_tok = args.t[1].image; x.q_tok = args.t[2].image; x.do_tok = args.t[3].image;
        x.k_exps = args.t[0].exps; x.v_exps = args.t[1].exps; x.q_exps = args.t[2].exps; x.do_exps = args.t[3].exps;
        x.k_each = each[0]; x.v_each = each[1]; x.q_each = each[2]; x.do_each = each[3];
        x.part_o = (float *)(at + p.dkv_at);
        e = launch_make_parts(x, args, x.vec, s);
        if (e == hipSuccess) e = launch_attn_grad_rows_parts(x, s);
        if (e == hipSuccess) e = launch_attn_grad_keys_parts(x, s);
    } else {
        e = launch_attn_grad_rows(x, x.vec, s);
        if (e == hipSuccess) e = launch_attn_grad_keys(x, x.vec, s);
    }
    if (e == hipSuccess && dtable) e = launch_attn_grad_bias(x, (float *)(at + p.sums_at), dtable, s);
    return from_hip(e);
}

int small_groupnorm_workspace(int N, int C, int H, int W, int G, int Cb, size_t *bytes)
{
    if (!bytes) return SMALL_ERR_NULL;
    int rc;
    if (!norm_elems(N, C, H, W, G, Cb, &rc)) return rc;
    *bytes = groupnorm_workspace(N, C, H * W, G, Cb);
    return SMALL_OK;
}

int small_groupnorm(const float *in, const float *gamma, const float *beta, float *out, float *stats, int N, int C, int H, int W,
                    int G, float eps, int act, int Cb, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!in || !gamma || !beta || !out) return SMALL_ERR_NULL;
    int rc;
    const size_t n = norm_elems(N, C, H, W, G, Cb, &rc);
    if (!n) return rc;
    if (!(eps >= 0.f) || isinf(eps) || !act_ok(act)) return SMALL_ERR_SHAPE;
    if (!block_ok(Cb, (uintptr_t)in | (uintptr_t)out)) return SMALL_ERR_BLOCK;
    const size_t need = groupnorm_workspace(N, C, H * W, G, Cb);
    if (!workspace_ok(workspace, workspace_bytes, need)) return SMALL_ERR_WORKSPACE;
    const Range o(out, n), st(stats, stats ? 2 * (size_t)N * G : 0), ws(workspace, need / sizeof(float));
    const Range reads[] = {Range(gamma, C), Range(beta, C)};
    if ((in != out && Range(in, n).meets(o)) || st.meets(o) || ws.meets(o) || st.meets(ws)) return SMALL_ERR_ALIAS;
    if (st.meets(Range(in, n)) || ws.meets(Range(in, n))) return SMALL_ERR_ALIAS;
    for (const Range &r : reads)
        if (r.meets(o) || r.meets(st) || r.meets(ws)) return SMALL_ERR_ALIAS;
    return from_hip(launch_groupnorm(in, gamma, beta, nullptr, nullptr, out, stats, nullptr, nullptr, N, C, H * W, G, eps, act, Cb,
                                     workspace, (hipStream_t)stream));
}

int small_groupnorm_grad(const float *in, const float *gamma, const float *beta, const float *stats, const float *dout, float *din,
                         float *dgamma, float *dbeta, int N, int C, int H, int W, int G, int act, int Cb, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    if (!in || !gamma || !beta || !stats || !dout || !din || !dgamma != !dbeta) return SMALL_ERR_NULL;
    int rc;
    const size_t n = norm_elems(N, C, H, W, G, Cb, &rc);
    if (!n) return rc;
    if (!act_ok(act)) return SMALL_ERR_SHAPE;
    if (!block_ok(Cb, (uintptr_t)in | (uintptr_t)dout | (uintptr_t)din)) return SMALL_ERR_BLOCK;
    const size_t need = groupnorm_workspace(N, C, H * W, G, Cb);
    if (!workspace_ok(workspace, workspace_bytes, need)) return SMALL_ERR_WORKSPACE;
    const size_t np = dgamma ? C : 0;
    const Range writes[] = {Range(din, n), Range(dgamma, np), Range(dbeta, np), Range(workspace, need / sizeof(float))};
    const Range reads[] = {Range(in, n), Range(gamma, C), Range(beta, C), Range(stats, 2 * (size_t)N * G), Range(dout, n)};
    for (const Range &w : writes) {
        for (const Range &r : reads)
            if (w.meets(r) && !(w.at == (uintptr_t)din && r.at == (uintptr_t)dout && din == dout)) return SMALL_ERR_ALIAS;
        for (const Range &o : writes)
            if (&w != &o && w.meets(o)) return SMALL_ERR_ALIAS;
    }
    return from_hip(launch_groupnorm(in, gamma, beta, stats, dout, din, nullptr, dgamma, dbeta, N, C, H * W, G, 0.f, act, Cb,
                                     workspace, (hipStream_t)stream));
}

}  // extern "C"
