// Attention over whole sequences, forward, on the fp16 matrix instructions with values in two parts (gfx950); attn_parts.h has the arithmetic and the
// layouts. Tiles of 64 rows (16 a wave) walk over tiles of 64 keys in LDS, four workgroups a compute unit up to 64 channels: sixteen rows a wave leave
// registers for that (32 rows a wave, half the LDS reads but half the waves: 311 against 208 us in an early form).
//
// Bound by vector instructions, not by the matrix instructions that they feed, and by waits at the two barriers of a tile: a score is scaled, capped, biased, masked, made a weight and split in two,
// some thirty instructions, 1900 cycles for a wave's tile of 16 x 64, where the matrix instructions take 768 at 64 channels. Counters for 4096 causal frames,
// 8 heads of 64, capped, a bias by buckets, 2 sequences: vector ALU busy some 57 % of the time, matrix pipe 30 %. Measured: that case 140 to 151 us (4 D operations
// a pair that is seen: 235 TFLOP/s; fp32 instructions 494 us), 8192 frames of packed documents with distances 138 to 147 us, 14 x 14 pixels, 8 heads of 32, 64 images,
// 36 us and 18 for laying keys and values out. Uneven tiles (below): 212 us, 152 us.
#include "attn_parts.h"

#include <type_traits>

namespace small {

namespace {

extern __shared__ __attribute__((aligned(1024))) char parts_lds[];

// Tiles of 64 tokens of up to four tensors, one workgroup each: the largest magnitudes, then the image. A thread takes 4 tokens x 4 channels.
template <int STEPS, bool VEC>
__global__ void __launch_bounds__(256) attn_make_parts(AttnArgs a, PartsArgs args)
{
    constexpr int DQ = STEPS * 8, PER = (16 * DQ + 255) / 256;      // quads of channels, micro tiles a thread
    __shared__ alignas(16) float most_of[4][64];           // of the tokens, by wave
    int which = 0;
    while (which + 1 < args.count && blockIdx.x >= args.t[which + 1].first_block) ++which;
    const PartsTensor &t = args.t[which];
    const int id = (int)(blockIdx.x - t.first_block), by_tile = id / t.tiles, tile = id - by_tile * t.tiles, n = by_tile / t.heads, head = by_tile - n * t.heads;
    const int len = !t.rows && a.lengths ? max(0, min(a.lengths[n], t.tokens)) : t.tokens;
    floatx4 x[PER][4];
    const int tq = threadIdx.x >> 2 & 15;
    floatx4 most{0.f, 0.f, 0.f, 0.f};
    int there = 0;                                         // of the four tokens: those that anything may see
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int e = threadIdx.x + p * 256, dq = (e & 3) | (e >> 6) << 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = tile * 64 + tq * 4 + i;
            bool on = dq < DQ && j < len;
            if (on && t.rows) on = a.lse_in[((size_t)n * t.heads + head) * t.tokens + j] != -kInf;
            if (on && !t.rows && a.docs) on = a.docs[(size_t)n * a.Sk + j] >= 0;
            x[p][i] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (on) x[p][i] = load_quad<VEC>(a, t.s, token_at(t.p, t.s, n, j), head * a.D, dq * 4);
            there |= on << i;
#pragma unroll
            for (int d = 0; d < 4; ++d) most[i] = fmaxf(most[i], any_magnitude(x[p][i][d]));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        most[i] = fmaxf(most[i], lane_shift1<0xb1>(most[i]));      // quad_perm: the neighbour's, the other pair's
        most[i] = fmaxf(most[i], lane_shift1<0x4e>(most[i]));
    }
    if ((threadIdx.x & 3) == 0) *reinterpret_cast<floatx4 *>(&most_of[threadIdx.x >> 6][tq * 4]) = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const floatx4 y = *reinterpret_cast<const floatx4 *>(&most_of[w][tq * 4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) most[i] = fmaxf(most[i], y[i]);
    }
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) all = fmaxf(all, finite_magnitude(most[i]));
    all = fmaxf(all, lane_shift1<0x124>(all));                         // row_ror
    all = fmaxf(all, lane_shift1<0x128>(all));
    all = column_max(all);
    // (nothing but zeros: any power does for them)
    const int ex = parts_exponent(all);
    int own[4];
    bool mixed = false, zeros = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int y = parts_exponent(most[i]);
        own[i] = most[i] == kInf ? kBad : most[i] == 0.f ? y : y >= ex - kSpread ? ex : y;
        mixed |= most[i] != 0.f && own[i] != ex;
        zeros |= most[i] == 0.f && (there >> i & 1);
    }
    mixed = __any(mixed);
    zeros = __any(zeros);
    if ((mixed | zeros) && threadIdx.x < 64 && (threadIdx.x & 3) == 0) *reinterpret_cast<int4 *>(t.each + (size_t)id * 64 + tq * 4) = int4{own[0], own[1], own[2], own[3]};
    if (threadIdx.x == 0) t.exps[id] = tile_word(all == 0.f ? kNone : ex, zeros, mixed);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int e = threadIdx.x + p * 256, dq = (e & 3) | (e >> 6) << 2;
        if (dq >= DQ) continue;
        half4 hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const float y = own[i] == kBad ? 0.f : ldexpf(x[p][i][d], -own[i]);
                hi[i][d] = (_Float16)y;
                lo[i][d] = (_Float16)(y - (float)hi[i][d]);
            }
        // token 4 tq + i of block tq / 4, channels 4 dq .. : half of lane (token, dq / 2)'s eight of step dq / 8
        char *to = t.image + (size_t)id * parts_tile_bytes(STEPS) + ((tq >> 2) * STEPS + (dq >> 3)) * 2048 + token_place((tq & 3) * 4, dq >> 1 & 3) + (dq & 1) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<half4 *>(to + i * 16) = hi[i];
            *reinterpret_cast<half4 *>(to + i * 16 + 1024) = lo[i];
        }
    }
}

template <int STEPS, int MODE>
// (waves a SIMD: what the walk over even tiles has registers for)
__global__ void __launch_bounds__(256, STEPS == 1 && MODE <= 2 ? 5 : STEPS <= 2 ? 4 : STEPS == 3 || MODE <= 4 ? 3 : 2) attn_rows_parts(AttnArgs a)
{
    constexpr int DT = 2 * STEPS, IMAGE = (int)parts_tile_bytes(STEPS);
    __shared__ alignas(16) int key_code[64];
    __shared__ alignas(16) int key_doc[65];
    __shared__ int words[2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const RowTile here = row_tile_of<true>(a, (unsigned)a.N * a.head_sets);
    const int split = here.split, tile = here.tile, n = a.by_sets.div(here.group), head = here.group - n * a.head_sets, key_head = a.by_group.div(head), kv = a.head_sets / a.group;
    const int row0 = tile * 64, i_raw = row0 + wave * 16 + m, i = min(i_raw, a.Sq - 1);      // rows past the end repeat the last one
    const ImageMask im(a, n);
    const RowState row(a, im, n, i, head);
    half8 q_hi[STEPS], q_lo[STEPS];
    int q_exp;
    {
        const float *token = token_at(a.q, a.qs, n, i);
        floatx4 x[STEPS][2];
        float most = 0.f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int d = 32 * s + 8 * g + 4 * h;
                x[s][h] = a.vec ? load_quad<true>(a, a.qs, token, head * a.D, d) : load_quad<false>(a, a.qs, token, head * a.D, d);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, finite_magnitude(x[s][h][e]));
            }
        q_exp = parts_exponent(column_max(most));
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[s][h][e] = ldexpf(x[s][h][e], -q_exp);
            split_results(x[s][0], x[s][1], q_hi[s], q_lo[s]);
        }
    }

    int lo = 0, hi = im.len;
    if (a.causal) hi = max(0, min(hi, max(im.position(min(row0 + 63, a.Sq - 1)) + 1, im.prefix)));
    if (a.docs) {
        if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
        __syncthreads();
        if (row.doc >= 0) { atomicMin(&words[0], row.doc); atomicMax(&words[1], row.doc); }
        __syncthreads();
        const int d0 = words[0], d1 = words[1];
        __syncthreads();
        document_hull(a.docs + (size_t)n * a.Sk, 0, hi, d0, d1, words, &lo, &hi);
    }
    int begin = __builtin_amdgcn_readfirstlane(lo) & ~63, end = __builtin_amdgcn_readfirstlane(hi);
    if (a.splits > 1) {
        const int per = ((end - begin + 63) / 64 + a.splits - 1) / a.splits * 64;
        begin = min(end, begin + split * per);
        end = min(end, begin + per);
    }
    // The largest power of two that the values of these keys carry: all weighted sums are kept at it, where no tile's is less than a quarter of it and no tile is mixed
    // (even). Where not, each row's at its own.
    const int tiles = (a.Sk + 63) / 64;
    const size_t first_tile = ((size_t)n * kv + key_head) * tiles;
    const int *k_exps = a.k_exps + first_tile, *v_exps = a.v_exps + first_tile;
    Powers powers;
    for (int x = begin / 64 + lane; x * 64 < end; x += 64) {
        powers.add(v_exps[x]);
        powers.add_mixed(k_exps[x]);
    }
    const bool even = powers.even(kFall);
    const int v_exp = powers.most;

    const char *k_image = a.k_tok + first_tile * IMAGE, *v_image = a.v_tok + first_tile * IMAGE;
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)parts_lds;
    const auto copy = [&](const char *image, int j0, unsigned to) {
#pragma unroll
        for (int x = 0; x < IMAGE / 4096; ++x) {
            const unsigned part = (unsigned)(wave * (IMAGE / 4096) + x) * 1024u;
            dma16(image + (size_t)(j0 / 64) * IMAGE, part + lane * 16, lds + to + part);
        }
    };
    if (begin < end) copy(k_image, begin, 0);

    const float *bias = nullptr;
    float far_lo = 0.f, far_hi = 0.f;
    if ((MODE & 4) && a.table) {
        if (a.bias_lds) {
            float *const e = reinterpret_cast<float *>(parts_lds + 2 * IMAGE);
            expand_bias(a, head, e);
            bias = e;
        }
        far_lo = bias_gather(a, head, 0);
        far_hi = bias_gather(a, head, 2 * a.reach);
    }

    floatx4 o[DT] = {};
    Reference top(a, row, begin, end);
    float sum = 0.f;
    ColumnScale vs;
    // Values are on their way while scores are computed, the next keys while values are summed; a barrier in front of either, behind which the
    // other's buffer is free.
    const auto walk = [&](auto is_even) {
        constexpr bool EVEN = decltype(is_even)::value;
        for (int j0 = begin; j0 < end; j0 += 64) {
            const int k_word = exponents_at(k_exps, j0 / 64), v_word = exponents_at(v_exps, j0 / 64), v_now = tile_exponent(v_word);
            int dot_exp = q_exp + tile_exponent(k_word);
            stage_keys<64>(a, n, j0, key_code, key_doc);
            wait_vmcnt<0>();
            __syncthreads();
            copy(v_image, j0, IMAGE);
            const char *kt = parts_lds + token_place(m, g), *vt = parts_lds + IMAGE + across_place(m, g);

            // (products of a step part by part over all results: one that adds to the one before it would wait for it)
            floatx4 s[4] = {};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                half8 k_hi[4], k_lo[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) k_lo[b] = *reinterpret_cast<const half8 *>(kt + (b * STEPS + st) * 2048 + 1024);
#pragma unroll
                for (int b = 0; b < 4; ++b) k_hi[b] = *reinterpret_cast<const half8 *>(kt + (b * STEPS + st) * 2048);
#pragma unroll
                for (int part = 0; part < 3; ++part)
#pragma unroll
                    for (int b = 0; b < 4; ++b) s[b] = mfma16(part == 0 ? k_lo[b] : k_hi[b], part == 1 ? q_lo[st] : q_hi[st], s[b]);
            }
            if (!EVEN && tile_mixed(k_word)) {
                by_token(s, a.k_each + first_tile * 64 + j0 + 4 * g, q_exp);
                bad_tokens<false>(s, a.k_each + first_tile * 64 + j0 + 4 * g);
                dot_exp = 0;
            }
            if (!EVEN && tile_mixed(v_word)) bad_tokens<false>(s, a.v_each + first_tile * 64 + j0 + 4 * g);
            // weights near fp16's top, and at the power of two that the sums carry
            const int lift = !EVEN ? 0 : kLift + max(v_now - v_exp, -kFall);
            const float in_exponent = (float)lift, was = top.at;
            finish_scores<MODE>(a, s, row, dot_exp, top.at - in_exponent, j0, key_code, key_doc, g, bias, far_lo, far_hi);
            raise_top(s, top, sum, o, in_exponent);
            if (!EVEN) vs.follow(top.at - was, o);
            floatx4 part = {};
#pragma unroll
            for (int b = 0; b < 4; ++b) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] = __builtin_amdgcn_exp2f(s[b][e]);
                part += s[b];
            }
            sum = fmaf((part.x + part.y) + (part.z + part.w), ldexpf(1.f, -lift), sum);
            if (!EVEN) {
                if (tile_by_tokens(v_word)) by_token(s, a.v_each + first_tile * 64 + j0 + 4 * g);
                vs.apply(s, tile_by_tokens(v_word) ? 0 : v_now, o);
            }
            half8 p_hi[2], p_lo[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) split_results(s[2 * b], s[2 * b + 1], p_hi[b], p_lo[b]);
            wait_vmcnt<0>();
            __syncthreads();
            if (j0 + 64 < end) copy(k_image, j0 + 64, 0);
#pragma unroll
            for (int b = 0; b < 2; ++b) products_across<STEPS>(o, vt, b, p_hi[b], p_lo[b]);
        }
    };
    // (uneven tiles are rare, and their walk must not cost this one registers: it is the one that spills)
    if (__builtin_expect(even, 1)) walk(std::true_type{});
    else walk(std::false_type{});

    const AttnArgs z = late_args();
    const float all = column_sum(sum);
    bool nan = false;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) nan |= !(fabsf(o[d][e]) < kInf);
    const unsigned long long lanes = __ballot(nan);
    const unsigned columns = (unsigned)((lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffffu);
    if (i_raw < z.Sq && !(columns >> m & 1)) {
        const size_t part = (((size_t)n * z.heads + head) * z.Sq + i) * z.splits + split;
        const float inv = z.splits > 1 ? 1.f : all == 0.f ? 0.f : 1.f / all;
        const int back = even ? v_exp - kLift : vs.back();
        float *token = const_cast<float *>(token_at(z.o, z.os, n, i));
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            floatx4 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = ldexpf(o[d][e] * inv, back);
            if (z.splits > 1 && z.D % 4 == 0) {
                if (16 * d + 4 * g < z.D) *reinterpret_cast<floatx4 *>(z.part_o + part * z.D + 16 * d + 4 * g) = y;
            } else if (z.splits > 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (16 * d + 4 * g + e < z.D) z.part_o[part * z.D + 16 * d + 4 * g + e] = y[e];
            } else if (z.vec) {
                store_quad<true>(z, z.os, token, head * z.D, 16 * d + 4 * g, y);
            } else {
                store_quad<false>(z, z.os, token, head * z.D, 16 * d + 4 * g, y);
            }
        }
        if (g == 0 && z.splits > 1) z.part_ml[part] = float2{top.maximum(), all};
        if (g == 0 && z.splits == 1 && z.lse) z.lse[((size_t)n * z.heads + head) * z.Sq + i] = all == 0.f ? -kInf : (top.at + __builtin_amdgcn_logf(all)) * kLn2;
    }
    for (unsigned left = columns; left; left &= left - 1) {
        const int rr = row0 + wave * 16 + __ffs((int)left) - 1;
        if (rr < z.Sq) attend_row_and_store(z, ImageMask(z, n), n, head, rr, split, begin, end);
    }
}

}  // namespace

hipError_t launch_make_parts(const AttnArgs &a, PartsArgs &args, bool vec, hipStream_t s)
{
    unsigned blocks = 0;
    for (int t = 0; t < args.count; ++t) {
        args.t[t].first_block = blocks;
        blocks += (unsigned)((long)a.N * args.t[t].heads * args.t[t].tiles);
    }
#define PARTS(st) \
    if (a.D <= 32 * st) { \
        if (vec) hipLaunchKernelGGL((attn_make_parts<st, true>), dim3(blocks), dim3(256), 0, s, a, args); \
        else hipLaunchKernelGGL((attn_make_parts<st, false>), dim3(blocks), dim3(256), 0, s, a, args); \
        return hipGetLastError(); \
    }
    PARTS(1) PARTS(2) PARTS(3) PARTS(4)
#undef PARTS
    return hipErrorInvalidValue;
}

hipError_t launch_attn_rows_parts(const AttnArgs &a, size_t bias_bytes, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.heads * a.row_tiles * a.splits);
    const int mode = attn_mode(a);
#define ROWS(st) \
    if (a.D <= 32 * st) { \
        const size_t lds = 2 * parts_tile_bytes(st) + bias_bytes; \
        switch (mode) { \
            case 0: return launch_lds(attn_rows_parts<st, 0>, grid, lds, a, s); \
            case 2: return launch_lds(attn_rows_parts<st, 2>, grid, lds, a, s); \
            case 4: return launch_lds(attn_rows_parts<st, 4>, grid, lds, a, s); \
            case 5: return launch_lds(attn_rows_parts<st, 5>, grid, lds, a, s); \
            default: return launch_lds(attn_rows_parts<st, 7>, grid, lds, a, s); \
        } \
    }
    ROWS(1) ROWS(2) ROWS(3) ROWS(4)
#undef ROWS
    return hipErrorInvalidValue;
}

}  // namespace small
