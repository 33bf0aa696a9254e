// What the attention kernels share (attn.hip, attn_token.hip, attn_grad.hip): arguments, addresses, scores, tiles in LDS (gfx950).
//
// All products run on v_mfma_f32_16x16x4_f32: lane l = 16 g + m gives row m of the left operand (column m of the right one) at
// reduction index g, and holds rows 4g .. 4g+3 of column m of the result. Reduction indices may be permuted as long as both
// operands agree, and two permutations make every operand come straight from where it lies:
//   - over channels, index g of step (c, e) is channel 16c + 4g + e: a lane's four steps are one 16-byte load;
//   - over the tokens of a tile, index g of step (b, r) is token 16b + 4g + r: exactly the rows that a lane already holds of the product
//     before. So scores are taken transposed (rows: keys, columns: queries), and their exponentials are the next product's right
//     operand in the registers where they were computed; softmax statistics are per lane and column, joined over four lanes.
// The left operand of that second product wants channels in lanes: channel 16 VD grp + VD m + v for result tile grp * VD + v, so
// that a lane reads VD neighbouring channels of a token at once and ends up with 4 VD neighbouring ones of the result.
#pragma once
#include "small_internal.h"

namespace small {

struct TokenStrides { long long image, block, token; };      // floats

struct AttnArgs {
    const float *q, *k, *v;
    float *o, *lse;
    TokenStrides qs, ks, vs, os;
    int N, Sq, Sk, heads, group, D, Cb;
    float scale, cap;                                        // scale of the dot products; cap = 0: none
    int causal, width, reach, buckets;
    const int *lengths, *first, *prefix, *docs;
    const float *slopes, *table;
    const int *bucket;
    // derived
    int pack;                     // a workgroup's rows run over the query heads of one key head (few queries, shared heads)
    int head_sets, rows;          // heads / group sets of group * Sq rows, or heads of Sq
    int splits, bias_lds;         // bias_lds: heads whose expanded bias fits LDS (0: gathered from memory)
    int row_tiles, vec;           // vec: four channels of a head stand together and aligned in every tensor
    FastDiv by_Cb, by_Sq, by_width, by_tiles, by_sets, by_splits, by_group;
    float *part_o;
    float2 *part_ml;              // splits > 1: results before joining, and their (maximum, sum)
    // values in two parts (attn_parts.h): images of keys and values, their powers of two by tile and by token
    const char *k_tok, *v_tok, *q_tok, *do_tok;
    const int *k_exps, *v_exps, *q_exps, *do_exps;
    const int *k_each, *v_each, *q_each, *do_each;
    // gradient
    const float *dout, *lse_in;
    float *share;                                            // [N * heads][Sq]: what a row's weights, taken from its lse, are to be multiplied by (with slopes)
    int share_known;                                         // by attn_grad_shares, before the rows' gradient
    float *dq, *dk, *dv, *delta, *part_bias;                 // part_bias: null, or [N * heads * row_tiles][2 reach + 1]
    TokenStrides dos, dqs, dks, dvs;
    int key_tiles, bias_acc_lds, bias_copies, row_parts;
    FastDiv by_key_tiles, by_code, by_heads;                 // by_code: 2 width - 1
};

// The kernel's arguments read anew from where they are passed: what only a kernel's end needs would otherwise be kept in scalar registers, and spilled from
// them, all the way through its loop.
__device__ __forceinline__ AttnArgs late_args()
{
    auto at = (const __attribute__((address_space(4))) unsigned *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    unsigned words[sizeof(AttnArgs) / 4];
#pragma unroll
    for (unsigned i = 0; i < sizeof(AttnArgs) / 4; ++i) words[i] = at[i];
    return __builtin_bit_cast(AttnArgs, words);
}

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr int kFar = 1 << 28;     // first positions are taken into -kFar .. kFar: differences of positions' numbers fit an int
constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ const float *token_at(const float *p, const TokenStrides &s, int n, long long t)
{
    return p + n * s.image + t * s.token;
}
// Offset of a channel from its token's place.
__device__ __forceinline__ long long channel_at(const AttnArgs &a, const TokenStrides &s, int ch)
{
    const int b = a.by_Cb.div(ch);
    return b * s.block + (ch - b * a.Cb);
}

// Channels d .. d + 3 of a head whose first channel is c0, zeros from channel D on. VEC: D, Cb and all strides are multiples of four
// and the tensors 16-byte aligned, so that the four stand together.
template <bool VEC>
__device__ __forceinline__ floatx4 load_quad(const AttnArgs &a, const TokenStrides &s, const float *token, int c0, int d)
{
    if constexpr (VEC) {
        if (d >= a.D) return floatx4{0.f, 0.f, 0.f, 0.f};
        return *reinterpret_cast<const floatx4 *>(token + channel_at(a, s, c0 + d));
    } else {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = d + i < a.D ? token[channel_at(a, s, c0 + d + i)] : 0.f;
        return floatx4{x[0], x[1], x[2], x[3]};
    }
}
template <bool VEC>
__device__ __forceinline__ void store_quad(const AttnArgs &a, const TokenStrides &s, float *token, int c0, int d, floatx4 x)
{
    if constexpr (VEC) {
        if (d < a.D) *reinterpret_cast<floatx4 *>(token + channel_at(a, s, c0 + d)) = x;
    } else {
        const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < a.D) token[channel_at(a, s, c0 + d + i)] = y[i];
    }
}

__device__ __forceinline__ floatx4 mfma(float a, float b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// VD of the second product's left operand.
template <int DT> constexpr int kVD = DT % 4 == 0 ? 4 : DT % 2 == 0 ? 2 : 1;

// Number of a position: differs by a number of its own for every offset of rows and columns of images `width` pixels wide.
__device__ __forceinline__ int code_of(const AttnArgs &a, int p)
{
    const int w = a.width;
    if (w == 1) return p;
    const int row = p >= 0 ? a.by_width.div(p) : -a.by_width.div(w - 1 - p);
    return row * (2 * w - 1) + (p - row * w);
}

// What masks an image's keys: length, prefix.
struct ImageMask {
    int len, prefix, first;
    __device__ __forceinline__ ImageMask(const AttnArgs &a, int n)
    {
        len = a.lengths ? max(0, min(a.lengths[n], a.Sk)) : a.Sk;
        prefix = a.prefix ? min(a.prefix[n], a.Sk) : 0;
        first = a.first ? max(-kFar, min(a.first[n], kFar)) : a.Sk - a.Sq;
    }
    __device__ __forceinline__ int position(int i) const { return first + i; }
};

// What a query needs besides its channels. It sees the keys in front of `bound` -- of its document, if there are documents.
struct RowState {
    int p, code, bound, doc, head;
    float slope;                  // times log2(e)
    RowState() = default;
    __device__ __forceinline__ RowState(const AttnArgs &a, const ImageMask &im, int n, int i, int h)
    {
        p = im.position(i);
        code = a.table ? code_of(a, p) : 0;
        bound = a.causal ? min(im.len, max(p + 1, im.prefix)) : im.len;
        doc = a.docs && p >= 0 && p < a.Sk ? a.docs[(size_t)n * a.Sk + p] : -2;
        if (doc < 0) doc = -2;
        head = h;
        slope = a.slopes ? a.slopes[h] * kLog2e : 0.f;
    }
    // (no branches: a choice among vector elements behind lane-dependent branches has been compiled wrongly here)
    __device__ __forceinline__ bool sees(int j, int key_doc, bool docs) const { return (j < bound) & (!docs | (key_doc == doc)); }
};
__device__ __forceinline__ int key_document(const AttnArgs &a, int n, int j)       // -1: none (no query has that)
{
    return max(-1, a.docs[(size_t)n * a.Sk + min(j, a.Sk - 1)]);
}

// tanh as the seventh convergent of Lambert's continued fraction x / (1 + x^2 / (3 + x^2 / (5 + ...))), all of whose terms are positive:
// within 2^-23 of its value up to |x| = 2; beyond, 1 - 2 / (exp(2x) + 1), where nothing cancels any more.
__device__ __forceinline__ float tanh_of(float x)
{
    const float y = x * x;
    const float n = fmaf(y, fmaf(y, y + 378.f, 17325.f), 135135.f), d = fmaf(y, fmaf(y, fmaf(y, 28.f, 3150.f), 62370.f), 135135.f);
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * (2.f * kLog2e));
    const float r = fabsf(x) > 2.f ? copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f), x) : x * n * __builtin_amdgcn_rcpf(d);
    return r;
}

// The same for |x| <= 0.6, a polynomial fitted at Chebyshev points (relative error 2.5e-9 before rounding): capped scores are mostly small against
// their cap, and this takes no reciprocal.
__device__ __forceinline__ float tanh_small(float x)
{
    const float y = x * x;
    return x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -0.00585642783f, 0.0207574759f), -0.05376992f), 0.133317053f), -0.333332837f), 1.f);
}
template <int NB>
__device__ __forceinline__ void tanh_all(floatx4 (&s)[NB])
{
    float most = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) most = fmaxf(most, fmaxf(fmaxf(fabsf(s[b].x), fabsf(s[b].y)), fmaxf(fabsf(s[b].z), fabsf(s[b].w))));
    if (__any(most > 0.6f)) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][e] = tanh_of(s[b][e]);
    } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][e] = tanh_small(s[b][e]);
    }
}

// A bias in units of log2. One of about the type's lowest value hides its offsets as minus infinity does: a sum of weights of scores of that size
// could not be written next to them in a row's lse, from which the gradient takes the weights.
__device__ __forceinline__ float bias_log2(float b) { return b < -1e30f ? -kInf : b * kLog2e; }
__device__ __forceinline__ float bias_gather(const AttnArgs &a, int head, int at)       // at: offset's place in 0 .. 2 reach
{
    const int b = max(0, min(a.bucket[at], a.buckets - 1));
    return bias_log2(a.table[(size_t)head * a.buckets + b]);
}
// A head's biases by offset into LDS, by the whole workgroup (of 256).
__device__ __forceinline__ void expand_bias(const AttnArgs &a, int head, float *lds)
{
#pragma unroll 4
    for (int x = threadIdx.x; x <= 2 * a.reach; x += 256) lds[x] = bias_gather(a, head, x);
}
__device__ __forceinline__ int offset_at(const AttnArgs &a, int key_code, int code) { return max(-a.reach, min(key_code - code, a.reach)) + a.reach; }

// The scores of a lane's four neighbouring keys j0 .. j0 + 3 for its row, in units of log2, from their dot products. bias: the row's head's
// expanded bias in LDS, or null. far: every offset of the tile is at one end of the reach, whose bias is far_bias.
struct Scorer {
    const AttnArgs &a;
    float scale2, cap_in, cap2;
    __device__ __forceinline__ Scorer(const AttnArgs &args) : a(args)
    {
        scale2 = a.scale * kLog2e;
        cap_in = a.cap > 0.f ? a.scale / a.cap : 0.f;
        cap2 = a.cap * kLog2e;
    }
    __device__ __forceinline__ float capped(float dot) const { return a.cap > 0.f ? cap2 * tanh_of(dot * cap_in) : dot * scale2; }
    __device__ __forceinline__ float biased(float t, const RowState &row, int j, int key_code, const float *bias) const
    {
        if (a.slopes) t = fmaf(-row.slope, fabsf((float)(row.p - j)), t);
        if (a.table) {
            const int at = offset_at(a, key_code, row.code);
            t += bias ? bias[at] : bias_gather(a, row.head, at);
        }
        return t;
    }
};

// A lane's scores from its dot products (which stand for 2^-dot_exp of what they are), in units of log2 and relative to `ref`, of the keys j0 + 16b + 4g + e
// of a tile whose numbers and documents are in LDS (key_doc[16 NB]: the document of all of them, or -3); hidden keys get minus infinity. bias: the head's expanded
// bias in LDS, or null; far_lo, far_hi: its ends. A score is one operation where there is neither cap nor bias, so `ref` costs nothing.
// MODE: which of cap (1), distances (2) and table (4) there may be at all; what a kernel is compiled without costs it no registers.
template <int MODE, int NB>
__device__ __forceinline__ void finish_scores(const AttnArgs &a, floatx4 (&s)[NB], const RowState &row, int dot_exp, float ref, int j0, const int *key_code, const int *key_doc,
                                              int g, const float *bias, float far_lo, float far_hi, floatx4 *core = nullptr)       // core: gets tanh, where there is a cap
{
    const bool capped = (MODE & 1) && a.cap > 0.f, slopes = (MODE & 2) && a.slopes, table = (MODE & 4) && a.table;
    float in = ldexpf(capped ? a.scale / a.cap : a.scale * kLog2e, dot_exp), base = -ref;
    if (capped) {
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] *= in;
        tanh_all(s);
        if (core)
#pragma unroll
            for (int b = 0; b < NB; ++b) core[b] = s[b];
        in = a.cap * kLog2e;
    }
    bool near = false;
    if (table) {
        const bool all_lo = __all(key_code[16 * NB - 1] - row.code <= -a.reach), all_hi = __all(key_code[0] - row.code >= a.reach);
        near = !all_lo && !all_hi;
        base += all_lo ? far_lo : all_hi ? far_hi : 0.f;
    }
    if (slopes) {
        const float from = (float)(j0 + 4 * g - row.p);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][e] = fmaf(s[b][e], in, fmaf(-row.slope, fabsf(from + (float)(16 * b + e)), base));
    } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][e] = fmaf(s[b][e], in, base);
    }
    if (near) {
        // Where the whole tile is inside the reach nothing is clamped, and in a sequence the biases of a lane's keys stand one behind the other.
        const int first = key_code[0] + 4 * g - row.code + a.reach;
        if (bias && a.width == 1 && __all((first >= 0) & (first + 16 * NB - 13 <= 2 * a.reach))) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] += bias[first + 16 * b + e];
        } else if (bias && __all((key_code[0] - row.code >= -a.reach) & (key_code[16 * NB - 1] - row.code <= a.reach))) {
            const int here = a.reach - row.code;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int4 kc = *reinterpret_cast<const int4 *>(key_code + 16 * b + 4 * g);
                s[b].x += bias[kc.x + here];
                s[b].y += bias[kc.y + here];
                s[b].z += bias[kc.z + here];
                s[b].w += bias[kc.w + here];
            }
        } else if (bias) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int4 kc = *reinterpret_cast<const int4 *>(key_code + 16 * b + 4 * g);
                s[b].x += bias[offset_at(a, kc.x, row.code)];
                s[b].y += bias[offset_at(a, kc.y, row.code)];
                s[b].z += bias[offset_at(a, kc.z, row.code)];
                s[b].w += bias[offset_at(a, kc.w, row.code)];
            }
        } else {
#pragma unroll 1
            for (int x = 0; x < 4 * NB; ++x) {
                const float y = bias_gather(a, row.head, offset_at(a, key_code[16 * (x >> 2) + 4 * g + (x & 3)], row.code));
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][e] += x == 4 * b + e ? y : 0.f;
            }
        }
    }
    if (!__all(j0 + 16 * NB <= row.bound)) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][e] = j0 + 16 * b + 4 * g + e < row.bound ? s[b][e] : -kInf;
    }
    if (a.docs && !__all(key_doc[16 * NB] == row.doc)) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int4 kd = *reinterpret_cast<const int4 *>(key_doc + 16 * b + 4 * g);
            s[b].x = kd.x == row.doc ? s[b].x : -kInf;
            s[b].y = kd.y == row.doc ? s[b].y : -kInf;
            s[b].z = kd.z == row.doc ? s[b].z : -kInf;
            s[b].w = kd.w == row.doc ? s[b].w : -kInf;
        }
    }
}

// Numbers (keys past the end: the last one's) and documents of a tile's KT keys into LDS, by the first KT threads of the workgroup; key_doc[KT]: the document of all of them, or -3.
template <int KT>
__device__ __forceinline__ void stage_keys(const AttnArgs &a, int n, int j0, int *key_code, int *key_doc)
{
    if (threadIdx.x >= KT) return;
    const int j = j0 + threadIdx.x;
    if (a.table) key_code[threadIdx.x] = code_of(a, min(j, a.Sk - 1));
    if (a.docs) {
        const int doc = key_document(a, n, j), first = __builtin_amdgcn_readfirstlane(doc);
        key_doc[threadIdx.x] = doc;
        if (threadIdx.x == 0) key_doc[KT] = -3;
        if (__all(doc == first)) key_doc[KT] = first;
    }
}

// A tile of KT tokens in LDS: [channels / 16][token][16], chunks 16 floats further apart than they are long, so that the four chunks that a
// wave reads of one token are in different banks.
template <int DT, int KT>
struct Tile {
    static constexpr int kChunk = KT * 16 + 16, kFloats = DT * kChunk, kAll = KT * DT * 4, kQuads = (kAll + 255) / 256;
    // Thread t's quads of the tile, tokens from j0 on; on(token) says which are read, others are zeros.
    template <bool VEC, typename On>
    static __device__ __forceinline__ void fetch(floatx4 (&x)[kQuads], const AttnArgs &a, const TokenStrides &s, const float *base, int n, int c0, int j0, On on)
    {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int e = threadIdx.x + i * 256, q = e & 3, j = (e >> 2) % KT, c = (e >> 2) / KT;
            x[i] = floatx4{0.f, 0.f, 0.f, 0.f};
            if ((kAll % 256 == 0 || e < kAll) && on(j)) x[i] = load_quad<VEC>(a, s, token_at(base, s, n, j0 + j), c0, c * 16 + q * 4);
        }
    }
    static __device__ __forceinline__ void put(float *lds, const floatx4 (&x)[kQuads])
    {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int e = threadIdx.x + i * 256, q = e & 3, j = (e >> 2) % KT, c = (e >> 2) / KT;
            if (kAll % 256 == 0 || e < kAll) *reinterpret_cast<floatx4 *>(lds + c * kChunk + j * 16 + q * 4) = x[i];
        }
    }
    // The same for what sums with weights are taken of, where 0 times a hidden token's infinity or NaN would not be 0: such values become zeros, and
    // their tokens' words, and `any`, get the stamp.
    static __device__ __forceinline__ void put_finite(float *lds, floatx4 (&x)[kQuads], int *bad, int *any, int stamp)
    {
#pragma unroll
        for (int i = 0; i < kQuads; ++i) {
            const int e = threadIdx.x + i * 256, j = (e >> 2) % KT;
            bool off = false;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const bool here = !(fabsf(x[i][d]) < kInf);
                x[i][d] = here ? 0.f : x[i][d];
                off |= here;
            }
            if (off && (kAll % 256 == 0 || e < kAll)) { bad[j] = stamp; *any = stamp; }
        }
        put(lds, x);
    }
    // Left operand with tokens in lanes: channels 16c + 4g .. +3 of token 16b + m.
    static __device__ __forceinline__ floatx4 tokens(const float *lds, int b, int c, int m, int g)
    {
        return *reinterpret_cast<const floatx4 *>(lds + c * kChunk + (16 * b + m) * 16 + 4 * g);
    }
    // Left operand with channels in lanes: channels VD m .. of group grp of token j.
    template <int VD>
    static __device__ __forceinline__ void channels(float (&x)[VD], const float *lds, int j, int grp, int m)
    {
        const float *p = lds + (grp * VD + m * VD / 16) * kChunk + j * 16 + (m * VD & 15);
        if constexpr (VD == 4) {
            const floatx4 f = *reinterpret_cast<const floatx4 *>(p);
            x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
        } else if constexpr (VD == 2) {
            const float2 f = *reinterpret_cast<const float2 *>(p);
            x[0] = f.x; x[1] = f.y;
        } else {
            x[0] = *p;
        }
    }
};

// The largest of a lane's value over the four lanes of its column, and the sum, by swaps of lanes (a shuffle is a trip through LDS).
template <typename F>
__device__ __forceinline__ float over_column(float v, F f)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const unsigned w = __float_as_uint(f(__uint_as_float(h[0]), __uint_as_float(h[1])));
    const auto r = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float column_max(float v) { return over_column(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ __forceinline__ float column_sum(float v) { return over_column(v, [](float x, float y) { return x + y; }); }

// A row's weights as its lse gives them sum to one but for the rounding of lse itself, which is a part of 2^-24 of its size: where distances make scores large
// -- a row whose nearest key is far away, behind a length, say -- that is more than all other errors. What makes them sum to one, for a lane's row; total: of this lane's keys.
__device__ __forceinline__ float share_of(const AttnArgs &a, float total)
{
    if (!a.slopes) return 1.f;
    total = column_sum(total);
    return total > 0.f ? 1.f / total : 0.f;
}

// A row's reference, against which its weights are taken (the same in the four lanes of its column): a score that it had, or minus infinity so far. It is
// taken anew only where a score passes it by more than kSlack: weights are then at most 2^kSlack, and most tiles need no exchange between lanes and rescale
// nothing. Scores s come relative to `top.at` and leave relative to the new one.
constexpr float kSlack = 6.f;
struct Reference {
    float at;
    bool seen;                    // a score was; until then `at` is what distances alone make of the nearest key, so that large ones cancel unrounded
    Reference() = default;
    __device__ __forceinline__ Reference(const AttnArgs &a, const RowState &row, int begin, int end) : at(0.f), seen(false)
    {
        if (a.slopes) at = -row.slope * fabsf((float)(row.p - max(begin, min(row.p, end - 1))));
    }
    __device__ __forceinline__ float maximum() const { return seen ? at : -kInf; }
};
template <int NB, int DT>
__device__ __forceinline__ void raise_top(floatx4 (&s)[NB], Reference &top, float &sum, floatx4 (&o)[DT], float lift = 0.f)      // (s: `lift` more than that)
{
    float mx = -kInf;
#pragma unroll
    for (int b = 0; b < NB; ++b) mx = fmaxf(mx, fmaxf(fmaxf(s[b].x, s[b].y), fmaxf(s[b].z, s[b].w)));
    if (!__any(mx > (top.seen ? kSlack + lift : -kInf))) return;
    mx = column_max(mx) - lift;
    // (a lower reference is never taken; what is taken off is what the reference gains after rounding, or old sums and new ones would stand for different ones)
    const float gain = top.seen ? fmaxf(mx, 0.f) : (mx == -kInf ? 0.f : mx), now = top.at + gain, by = now - top.at;
    // (from 2^23 on a reference's rounding is a whole power of two or more: there the largest score is the reference by decree, or its weight could be 0 or infinite)
    const float off = fabsf(now) < 8388608.f ? by : gain;
    const float w = top.seen ? __builtin_amdgcn_exp2f(-by) : 1.f;                    // (nothing was summed so far)
    top.at = now;
    top.seen |= mx != -kInf;
    sum *= w;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] *= w;
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] -= off;
}

// 4 VD neighbouring channels of a lane's column from result tiles grp * VD .. : quad x of them.
template <int DT>
__device__ __forceinline__ floatx4 result_quad(const floatx4 (&o)[DT], int grp, int x)
{
    constexpr int VD = kVD<DT>;
    floatx4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 4 * x + i;
        r[i] = o[grp * VD + e % VD][e / VD];
    }
    return r;
}

// The keys of documents that a tile of rows belongs to: the smallest and one past the largest key whose document lies within lo .. hi
// (whole workgroup; `words`: two ints of LDS, free afterwards for another call behind a barrier).
__device__ __forceinline__ void document_hull(const int *docs, int from, int to, int lo, int hi, int *words, int *begin, int *end)
{
    if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
    __syncthreads();
    int first = 0x7fffffff, last = -1;
    for (int j = from + threadIdx.x; j < to; j += blockDim.x) {
        const int d = docs[j];
        if (d >= 0 && d >= lo && d <= hi) { first = min(first, j); last = j; }
    }
    if (last >= 0) { atomicMin(&words[0], first); atomicMax(&words[1], last); }
    __syncthreads();
    *begin = words[0] == 0x7fffffff ? to : words[0];
    *end = words[1] + 1;
    if (*end < *begin) *end = *begin;
}

// Expanded biases and their gradients' sums go into LDS up to so many offsets.
constexpr int kBiasLds = 8192;

// A launch whose dynamic LDS may pass the 64 KB that a kernel has without asking (160 KB a compute unit).
template <typename K>
hipError_t launch_lds(K *kernel, unsigned grid, size_t lds, const AttnArgs &a, hipStream_t s)
{
    if (lds > 8192)
        if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds); e != hipSuccess) {
            (void)hipGetLastError();                     // (or the next call of somebody else would report it)
            return e;
        }
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), lds, s, a);
    return hipGetLastError();
}

// attn.hip, attn_token.hip, attn_grad.hip
inline int attn_mode(const AttnArgs &a) { return (a.cap > 0.f ? 1 : 0) | (a.slopes ? 2 : 0) | (a.table ? 4 : 0); }
hipError_t launch_attn_rows(const AttnArgs &a, bool vec, size_t bias_bytes, hipStream_t s);
hipError_t launch_attn_join(const AttnArgs &a, hipStream_t s);
hipError_t launch_attn_grad_shares(const AttnArgs &a, bool vec, hipStream_t s);
hipError_t launch_attn_grad_rows(const AttnArgs &a, bool vec, hipStream_t s);
hipError_t launch_attn_grad_keys(const AttnArgs &a, bool vec, hipStream_t s);
hipError_t launch_attn_grad_bias(const AttnArgs &a, float *sums, float *dtable, hipStream_t s);
hipError_t launch_attn_token(const AttnArgs &a, bool vec, hipStream_t s);

}  // namespace small
