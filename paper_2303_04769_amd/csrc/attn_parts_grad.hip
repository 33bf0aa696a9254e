// Gradients of attention on the fp16 matrix instructions with values in two parts (gfx950); attn_grad.hip has the mathematics, attn_parts.h
// the arithmetic and the layouts. attn_grad_rows_parts keeps 64 rows and walks over tiles of 64 keys, attn_grad_keys_parts keeps 64 keys and walks over
// tiles of 32 rows of its query heads; where there are few key tiles, its rows are shared out over several workgroups, whose sums attn_grad_join adds.
//
// The tile that a wave holds comes straight from the images (a lane's operand is what the image has at its place), what it walks over through LDS.
// P and dS have no size of their own -- a long row's weights are small, and so are their gradients, and a key may have small ones only -- so they carry
// a power of two for each column, set by the first tile and raised where a value would pass fp16's range.
//
// Bound as the forward kernel is, by some forty vector instructions a pair in either walk, and by waits that three workgroups a compute unit (registers; two from 65
// channels on) do not cover: vector ALU busy 46 % and 41 %, matrix pipe 19 % and 22 % for 2048 frames with a prefix, 8 heads of 64 on 2, capped, a bias by
// buckets, 4 sequences. Measured there: rows 175 to 182 us, keys 191 to 200, and with the forward call and all else 446 to 463 (fp32
// instructions: 2123); 14 x 14 pixels, 8 heads of 32, a bias by offsets, 64 images: rows 67, keys 53.
#include "attn_parts.h"

#include <type_traits>

namespace small {

namespace {

extern __shared__ __attribute__((aligned(1024))) char parts_lds[];

// Two or four operands in two parts against one right operand in two parts, part by part.
template <int NB>
__device__ __forceinline__ void products(floatx4 (&c)[NB], const char *lds, int stride, half8 b_hi, half8 b_lo)
{
    half8 hi[NB], lo[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) lo[b] = *reinterpret_cast<const half8 *>(lds + b * stride + 1024);
#pragma unroll
    for (int b = 0; b < NB; ++b) hi[b] = *reinterpret_cast<const half8 *>(lds + b * stride);
#pragma unroll
    for (int part = 0; part < 3; ++part)
#pragma unroll
        for (int b = 0; b < NB; ++b) c[b] = mfma16(part == 0 ? lo[b] : hi[b], part == 1 ? b_lo : b_hi, c[b]);
}

// The bias gradient's sums by offset, in LDS: places of one wave, `copies` (4, 2 or 1) sets of them for its four groups of lanes, which have keys of their own; the
// groups that share a set take turns. mine: the place of offset 0 in the lane's set; offsets at the ends of the reach are summed in registers, and what has no place
// goes to one behind the upper end that nobody reads. No atomic operations (LDS does those of floats lane by lane): what adds at once has
// offsets of its own, and a wave's accesses to LDS are done in order.
//
// In a sequence key and row that both move on by one have the same offset: lane m takes what lane m + e has of the key e further on, from the lanes it
// runs over into that of the next sixteen keys, and five places remain of sixteen keys and rows, which differ. offset: of the lane's row and first key.
__device__ __forceinline__ void sums_in_line(const floatx4 (&s)[4], int reach, int offset, int m, int g, int copies, float *mine, float &lo, float &hi)
{
    floatx4 x[4];
    const bool inside = __all((offset + 51 < reach) & (offset > -reach));
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        x[b] = s[b];
        if (!inside)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int off = offset + 16 * b + e;
                const bool below = off <= -reach, above = (off >= reach) & !below;
                lo += below ? x[b][e] : 0.f;
                hi += above ? x[b][e] : 0.f;
                x[b][e] = (below | above) ? 0.f : x[b][e];
            }
    }
    float t[5] = {x[0].x, x[1].x, x[2].x, x[3].x, 0.f};
    const auto along = [&](int b, float from, bool over) {
        t[b] += over ? 0.f : from;
        t[b + 1] += over ? from : 0.f;
    };
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        along(b, lane_shift1<0x12f>(x[b].y), m + 1 > 15);        // row_ror: 15, 14, 13: from one, two, three lanes on
        along(b, lane_shift1<0x12e>(x[b].z), m + 2 > 15);
        along(b, lane_shift1<0x12d>(x[b].w), m + 3 > 15);
    }
    for (int turn = 0; turn < 4; turn += copies) {
        if ((unsigned)(g - turn) >= (unsigned)copies) continue;
        float *at[5], was[5];
#pragma unroll
        for (int b = 0; b < 5; ++b) {
            const int off = offset + 16 * b;
            at[b] = mine + (((off > -reach) & (off < reach)) ? off : reach + 1);
            was[b] = *at[b];
        }
#pragma unroll
        for (int b = 0; b < 5; ++b) *at[b] = was[b] + t[b];
    }
}
// In an image of several columns: one key of each lane after another, whose rows, and so offsets, differ (there: the lane has a row of its own; keys: how many
// of the tile's there are).
__device__ __forceinline__ void sums_in_image(const floatx4 (&s)[4], int reach, const int *key_code, int row_code, bool there, int keys, int g, int copies, float *mine, float &lo, float &hi)
{
    int at[4][4];
    const bool inside = keys >= 64 && __all(there & (key_code[0] - row_code > -reach) & (key_code[63] - row_code < reach));
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int4 kc = *reinterpret_cast<const int4 *>(key_code + 16 * b + 4 * g);
        const int off[4] = {kc.x - row_code, kc.y - row_code, kc.z - row_code, kc.w - row_code};
#pragma unroll
        for (int e = 0; e < 4; ++e) at[b][e] = off[e];
    }
    if (!inside)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int off = at[b][e];
                const bool below = off <= -reach, above = (off >= reach) & !below;
                lo += below ? s[b][e] : 0.f;
                hi += above ? s[b][e] : 0.f;
                at[b][e] = (below | above | !there | (16 * b + 4 * g + e >= keys)) ? reach + 1 : off;
            }
    // (Two lanes that share a place have keys as far apart as their rows, at most 15: of the keys 16 apart all places differ.)
    for (int turn = 0; turn < 4; turn += copies) {
        if ((unsigned)(g - turn) >= (unsigned)copies) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float was[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) was[b] = mine[at[b][e]];
#pragma unroll
            for (int b = 0; b < 4; ++b) mine[at[b][e]] = was[b] + s[b][e];
            asm volatile("" ::: "memory");
        }
    }
}

__device__ __forceinline__ void copy_image(const char *image, int bytes, unsigned lds_at)       // (whole workgroup; bytes a multiple of 4096)
{
    const unsigned wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int x = 0; x < bytes / 4096; ++x) {
        const unsigned part = (wave * (bytes / 4096) + x) * 1024u;
        dma16(image, part + lane * 16, lds_at + part);
    }
}
__device__ __forceinline__ unsigned lds_address(const void *p) { return (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void *)p; }

template <int STEPS, int MODE>
__global__ void __launch_bounds__(256, STEPS <= 2 ? 3 : 2) attn_grad_rows_parts(AttnArgs a)
{
    constexpr int DT = 2 * STEPS, IMAGE = (int)parts_tile_bytes(STEPS);
    __shared__ alignas(16) int key_code[64];
    __shared__ alignas(16) int key_doc[65];
    __shared__ int words[2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const RowTile here = row_tile_of<false>(a, (unsigned)a.N * a.heads);
    const int tile = here.tile, n = a.by_heads.div(here.group), head = here.group - n * a.heads, key_head = a.by_group.div(head), kv = a.by_group.div(a.heads);
    const int row0 = tile * 64, i_raw = row0 + wave * 16 + m, i = min(i_raw, a.Sq - 1);
    const ImageMask im(a, n);
    const RowState row(a, im, n, i, head);
    const size_t at_row = ((size_t)n * a.heads + head) * a.Sq + i, at_tile = ((size_t)n * a.heads + head) * a.row_tiles + tile;
    // a row that saw nothing has no gradient, and neither has one past the end: weights exp2(-inf)
    const float lse = a.lse_in[at_row];
    const bool dead = lse == -kInf || i_raw >= a.Sq;
    float lse2 = dead ? kInf : lse * kLog2e;
    float delta = 0.f;
    {
        const float *td = token_at(a.dout, a.dos, n, i), *to = token_at(a.o, a.os, n, i);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const int d = 16 * c + 4 * g;
            const floatx4 x = a.vec ? load_quad<true>(a, a.dos, td, head * a.D, d) : load_quad<false>(a, a.dos, td, head * a.D, d);
            const floatx4 y = a.vec ? load_quad<true>(a, a.os, to, head * a.D, d) : load_quad<false>(a, a.os, to, head * a.D, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) delta = fmaf(dead ? 0.f : x[e], dead ? 0.f : y[e], delta);
        }
        delta = column_sum(delta);
        if (g == 0 && i_raw < a.Sq) a.delta[at_row] = delta;
    }
    half8 q_hi[STEPS], q_lo[STEPS], d_hi[STEPS], d_lo[STEPS];
    {
        const size_t at = at_tile * IMAGE + wave * STEPS * 2048 + token_place(m, g);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            q_hi[s] = *reinterpret_cast<const half8 *>(a.q_tok + at + s * 2048);
            q_lo[s] = *reinterpret_cast<const half8 *>(a.q_tok + at + s * 2048 + 1024);
            d_hi[s] = *reinterpret_cast<const half8 *>(a.do_tok + at + s * 2048);
            d_lo[s] = *reinterpret_cast<const half8 *>(a.do_tok + at + s * 2048 + 1024);
        }
    }
    const int q_word = exponents_at(a.q_exps, at_tile), d_word = exponents_at(a.do_exps, at_tile);

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
    const int begin = __builtin_amdgcn_readfirstlane(lo) & ~63, end = __builtin_amdgcn_readfirstlane(hi);

    const int tiles = (a.Sk + 63) / 64;
    const size_t first_tile = ((size_t)n * kv + key_head) * tiles;
    const int *k_exps = a.k_exps + first_tile, *v_exps = a.v_exps + first_tile;
    Powers powers;
    powers.add_mixed(q_word | d_word);
    for (int x = begin / 64 + lane; x * 64 < end; x += 64) {
        powers.add(k_exps[x]);
        powers.add_mixed(v_exps[x]);
    }
    const bool even = powers.even_terms();
    const unsigned lds = lds_address(parts_lds);
    if (begin < end) {
        copy_image(a.k_tok + (first_tile + begin / 64) * IMAGE, IMAGE, lds);
        copy_image(a.v_tok + (first_tile + begin / 64) * IMAGE, IMAGE, lds + 2 * IMAGE);
    }
    // The next tile's keys are copied into the other of two buffers all the while, its values behind the barrier that ends the products with these.
    unsigned now = 0;
    const auto next_keys = [&](int j0) {
        now ^= IMAGE;
        if (j0 + 64 < end) copy_image(a.k_tok + (first_tile + j0 / 64 + 1) * IMAGE, IMAGE, lds + now);
    };
    const auto next_values = [&](int j0) {
        if (j0 + 64 < end) copy_image(a.v_tok + (first_tile + j0 / 64 + 1) * IMAGE, IMAGE, lds + 2 * IMAGE);
    };

    // LDS behind the three tiles: the expanded bias; its gradient's sums by offset, as often as there are waves times 4, 2 or 1 (bias_copies)
    const int size = 2 * a.reach + 1;
    float *at_lds = reinterpret_cast<float *>(parts_lds + 3 * IMAGE);
    const float *bias = nullptr;
    float far_lo = 0.f, far_hi = 0.f;
    if ((MODE & 4) && a.table) {
        if (a.bias_lds) {
            expand_bias(a, head, at_lds);
            bias = at_lds;
            at_lds += size;
        }
        far_lo = bias_gather(a, head, 0);
        far_hi = bias_gather(a, head, 2 * a.reach);
    }
    const bool sums = (MODE & 4) && a.part_bias;
    const int stride = size + 1, per_wave = a.bias_copies >> 2;
    float *const acc = at_lds, *const mine = acc + (wave * per_wave + (g & (per_wave - 1))) * stride + a.reach;
    if (sums)
        for (int x = threadIdx.x; x < a.bias_copies * stride; x += 256) acc[x] = 0.f;
    float sum_lo = 0.f, sum_hi = 0.f, total = 0.f;
    const float known = (MODE & 2) && a.share_known ? a.share[at_row] : 1.f;

    ColumnScale cs;
    floatx4 dq[DT] = {};
    // (where tiles are mixed: tokens with powers of two of their own)
    const auto walk = [&](auto is_mixed) {
        constexpr bool MIXED = decltype(is_mixed)::value;
        int q_exp = tile_exponent(q_word), d_exp = tile_exponent(d_word);
        if (MIXED) {
            if (tile_mixed(q_word)) q_exp = a.q_each[at_tile * 64 + wave * 16 + m];
            if (tile_mixed(d_word)) d_exp = a.do_each[at_tile * 64 + wave * 16 + m];
            if ((q_exp == kBad) | (d_exp == kBad)) lse2 = __builtin_nanf("");       // (in every score that is not hidden)
            q_exp = q_exp == kBad ? 0 : q_exp;
            d_exp = d_exp == kBad ? 0 : d_exp;
        }
        for (int j0 = begin; j0 < end; j0 += 64) {
            const int k_word = exponents_at(k_exps, j0 / 64), v_word = exponents_at(v_exps, j0 / 64);
            int dot_exp = q_exp + tile_exponent(k_word), dp_exp = d_exp + tile_exponent(v_word);
            stage_keys<64>(a, n, j0, key_code, key_doc);
            wait_vmcnt<0>();
            __syncthreads();
            const char *kt = parts_lds + now, *vt = parts_lds + 2 * IMAGE + token_place(m, g);
            next_keys(j0);
            floatx4 s[4] = {}, dp_half[2] = {}, dp_turned[2] = {};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                products(s, kt + token_place(m, g) + st * 2048, STEPS * 2048, q_hi[st], q_lo[st]);
                products(dp_half, vt + st * 2048, STEPS * 2048, d_hi[st], d_lo[st]);
                // half of the keys with dO's sign turned: the matrix instructions round their sums to one side, by a tenth of a spacing, and over a row
                // that would add up in the bias's gradient, which is what is left of sums that cancel
                products(dp_turned, vt + (2 * STEPS + st) * 2048, STEPS * 2048, -d_hi[st], -d_lo[st]);
            }
            floatx4 dp[4] = {dp_half[0], dp_half[1], -dp_turned[0], -dp_turned[1]};
            if (MIXED && tile_mixed(v_word)) {
                by_token(dp, a.v_each + first_tile * 64 + j0 + 4 * g, d_exp);
                dp_exp = 0;
            }
            if (MIXED && tile_mixed(k_word)) {
                by_token(s, a.k_each + first_tile * 64 + j0 + 4 * g, q_exp);
                dot_exp = 0;
            }
            const float dp_in = ldexpf(1.f, dp_exp);
            floatx4 core[4];
            finish_scores<MODE>(a, s, row, dot_exp, lse2, j0, key_code, key_doc, g, bias, far_lo, far_hi, (MODE & 1) ? core : nullptr);
            if (MIXED && tile_mixed(k_word)) bad_tokens<true>(s, a.k_each + first_tile * 64 + j0 + 4 * g);      // (of V: delta is NaN)
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(s[b][e]);
                    if (MODE & 2) total += p;
                    s[b][e] = p == 0.f ? 0.f : p * fmaf(dp[b][e], dp_in, -delta);
                }
            if ((MODE & 2) && a.share_known)
#pragma unroll
                for (int b = 0; b < 4; ++b) s[b] *= known;
            if (sums) {
                const bool all_lo = __all(key_code[63] - row.code <= -a.reach), all_hi = __all(key_code[0] - row.code >= a.reach);
                if (all_lo || all_hi) {
                    float x = 0.f;
#pragma unroll
                    for (int b = 0; b < 4; ++b) x += (s[b].x + s[b].y) + (s[b].z + s[b].w);
                    sum_lo += all_lo ? x : 0.f;
                    sum_hi += all_lo ? 0.f : x;
                } else {
                    if (a.width == 1) sums_in_line(s, a.reach, j0 + 4 * g - (im.first + i_raw), m, g, per_wave, mine, sum_lo, sum_hi);
                    else sums_in_image(s, a.reach, key_code, row.code, i_raw < a.Sq, a.Sk - j0, g, per_wave, mine, sum_lo, sum_hi);
                }
            }
            if ((MODE & 1) && a.cap > 0.f)
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][e] *= fmaf(-core[b][e], core[b][e], 1.f);
            if (MIXED && tile_by_tokens(k_word)) by_token(s, a.k_each + first_tile * 64 + j0 + 4 * g);
            cs.apply(s, MIXED && tile_by_tokens(k_word) ? 0 : tile_exponent(k_word), dq);
            half8 hi_[2], lo_[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) split_results(s[2 * b], s[2 * b + 1], hi_[b], lo_[b]);
            __syncthreads();
            next_values(j0);
#pragma unroll
            for (int b = 0; b < 2; ++b) products_across<STEPS>(dq, kt + across_place(m, g), b, hi_[b], lo_[b]);
        }
    };
    // (a wave whose rows are all past the end does its share of the copies only)
    if (__builtin_amdgcn_readfirstlane(row0 + wave * 16) >= a.Sq)
        for (int j0 = begin; j0 < end; j0 += 64) {
            wait_vmcnt<0>();
            __syncthreads();
            next_keys(j0);
            __syncthreads();
            next_values(j0);
        }
    else if (__builtin_expect(even, 1)) walk(std::false_type{});
    else walk(std::true_type{});
    const AttnArgs z = late_args();
    if (sums) {
        __shared__ float ends[8];
        sum_lo = wave_sum(sum_lo);
        sum_hi = wave_sum(sum_hi);
        if (lane == 0) { ends[wave] = sum_lo; ends[4 + wave] = sum_hi; }
        __syncthreads();
        float *const part = z.part_bias + at_tile * size;
        for (int x = threadIdx.x; x < size; x += 256) {
            float y = 0.f;
            for (int c = 0; c < z.bias_copies; ++c) y += acc[c * stride + x];
            if (x == 0) y += (ends[0] + ends[1]) + (ends[2] + ends[3]);
            if (x == size - 1) y += (ends[4] + ends[5]) + (ends[6] + ends[7]);
            part[x] = y;
        }
    }
    const float share = (MODE & 2) && !z.share_known ? share_of(z, total) : 1.f;
    if (i_raw < z.Sq) {
        if ((MODE & 2) && z.slopes && !z.share_known && g == 0) z.share[at_row] = share;
        const float back = cs.back(z.scale) * share;
        float *token = const_cast<float *>(token_at(z.dq, z.dqs, n, i));
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            if (z.vec) store_quad<true>(z, z.dqs, token, head * z.D, 16 * d + 4 * g, dq[d] * back);
            else store_quad<false>(z, z.dqs, token, head * z.D, 16 * d + 4 * g, dq[d] * back);
        }
    }
}

template <int STEPS, int MODE>
// (waves a SIMD: what the walk over even tiles has registers for)
__global__ void __launch_bounds__(256, STEPS == 1 ? 4 : STEPS == 2 || (STEPS == 3 && MODE == 0) ? 3 : 2) attn_grad_keys_parts(AttnArgs a)
{
    constexpr int DT = 2 * STEPS, IMAGE = (int)parts_tile_bytes(STEPS), HALF = IMAGE / 2;
    struct Rows {
        float lse[32], delta[32], share[32];
        int p[32], code[32], bound[36], doc[36];       // bound[32]: the smallest; doc[32]: of all rows, or -3
    };
    __shared__ alignas(16) Rows rows_of[2];
    __shared__ int words[2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_part = a.by_splits.div((int)id), part = (int)id - by_part * a.splits;
    const int by_tile = a.by_key_tiles.div(by_part), tile = by_part - by_tile * a.key_tiles;      // (causal: the first keys have the most rows)
    const int kv = a.by_group.div(a.heads), n = a.by_sets.div(by_tile), key_head = by_tile - n * kv;
    const ImageMask im(a, n);
    const int j0 = tile * 64, j_raw = j0 + wave * 16 + m, j = min(j_raw, a.Sk - 1);
    const int code = (MODE & 4) && a.table ? code_of(a, j) : 0, doc = a.docs ? key_document(a, n, j) : -1;
    const size_t at_tile = ((size_t)n * kv + key_head) * a.key_tiles + tile;
    half8 k_hi[STEPS], k_lo[STEPS], v_hi[STEPS], v_lo[STEPS];
    {
        const size_t at = at_tile * IMAGE + wave * STEPS * 2048 + token_place(m, g);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            k_hi[s] = *reinterpret_cast<const half8 *>(a.k_tok + at + s * 2048);
            k_lo[s] = *reinterpret_cast<const half8 *>(a.k_tok + at + s * 2048 + 1024);
            v_hi[s] = *reinterpret_cast<const half8 *>(a.v_tok + at + s * 2048);
            v_lo[s] = *reinterpret_cast<const half8 *>(a.v_tok + at + s * 2048 + 1024);
        }
    }
    const int k_word = exponents_at(a.k_exps, at_tile), v_word = exponents_at(a.v_exps, at_tile);
    // rows that can see any of the keys; this part's heads, and of their rows its share
    int lo = 0, hi = j0 < im.len ? a.Sq : 0;
    if (a.causal && im.prefix <= j0) lo = max(0, min(a.Sq, j0 - im.first));
    if (a.docs) {
        if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
        __syncthreads();
        if (j_raw < im.len && doc >= 0) { atomicMin(&words[0], doc); atomicMax(&words[1], doc); }
        __syncthreads();
        const int d0 = words[0], d1 = words[1];
        __syncthreads();
        int first, last;
        const int p0 = max(0, min(im.first + lo, a.Sk)), p1 = max(p0, min(im.first + hi, a.Sk));
        document_hull(a.docs + (size_t)n * a.Sk, p0, p1, d0, d1, words, &first, &last);
        lo = first - im.first;
        hi = last - im.first;
    }
    // (no such row: an empty hull may lie at any distance from the rows there are, and rounding its begin down would make a tile of it)
    if (lo >= hi) lo = hi = 0;
    int begin = __builtin_amdgcn_readfirstlane(lo) & ~31, end = __builtin_amdgcn_readfirstlane(hi);
    const int head_part = part / a.row_parts, row_part = part - head_part * a.row_parts, head_parts = a.splits / a.row_parts;
    const int h0 = key_head * a.group + a.group * head_part / head_parts, h1 = key_head * a.group + a.group * (head_part + 1) / head_parts;
    if (a.row_parts > 1) {
        const int per = ((end - begin + 31) / 32 + a.row_parts - 1) / a.row_parts * 32;
        begin = min(end, begin + row_part * per);
        end = min(end, begin + per);
    }
    // Whether neither these keys nor the rows' queries and dO have powers of two by token that count.
    Powers of_q, of_d;
    of_q.add_mixed(k_word | v_word);
    for (int h = h0; h < h1; ++h)
        for (int x = begin / 64 + lane; x * 64 < end; x += 64) {
            const size_t at = ((size_t)n * a.heads + h) * a.row_tiles + x;
            of_q.add(a.q_exps[at]);
            of_d.add(a.do_exps[at]);
        }
    const bool even = of_q.even_terms() & of_d.even_terms();

    float *const bias_lds = reinterpret_cast<float *>(parts_lds + 4 * HALF);
    const unsigned lds = lds_address(parts_lds);
    // (a wave whose keys are all past the end, of the image or of its length, does its share of the copies only)
    const bool idle = __builtin_amdgcn_readfirstlane(j0 + wave * 16) >= im.len;
    ColumnScale cs, vs;
    floatx4 dk[DT] = {}, dv[DT] = {};
    const auto walk = [&](auto is_even) {
        constexpr bool EVEN = decltype(is_even)::value;
        int k_exp = tile_exponent(k_word), v_exp = tile_exponent(v_word);
        bool k_bad = false;
        if (!EVEN) {
            if (tile_mixed(k_word)) k_exp = a.k_each[at_tile * 64 + wave * 16 + m];
            if (tile_mixed(v_word)) v_exp = a.v_each[at_tile * 64 + wave * 16 + m];
            k_bad = k_exp == kBad;
            k_exp = k_bad ? 0 : k_exp;
            v_exp = v_exp == kBad ? 0 : v_exp;                              // (delta is NaN in the rows that see it)
        }
        for (int head = h0; head < h1 && begin < end; ++head) {
            const float slope = (MODE & 2) && a.slopes ? a.slopes[head] * kLog2e : 0.f;
            const float *bias = nullptr;
            float far_lo = 0.f, far_hi = 0.f;
            __syncthreads();                                                        // (the last head's tiles and bias are still read)
            if ((MODE & 4) && a.table) {
                if (a.bias_lds) {
                    expand_bias(a, head, bias_lds);
                    bias = bias_lds;
                }
                far_lo = bias_gather(a, head, 0);
                far_hi = bias_gather(a, head, 2 * a.reach);
            }
            const size_t first_row = ((size_t)n * a.heads + head) * a.Sq, first_tile = ((size_t)n * a.heads + head) * a.row_tiles;
            const auto at = [&](int i0) { return (first_tile + i0 / 64) * IMAGE + (i0 & 32 ? HALF : 0); };
            // While a tile is worked on, the next one is copied into the other of two buffers; one barrier a tile.
            unsigned now = 0;
            const auto copy_rows = [&](int i0, unsigned to) {
                copy_image(a.q_tok + at(i0), HALF, lds + to);
                copy_image(a.do_tok + at(i0), HALF, lds + to + HALF);
            };
            copy_rows(begin, 0);
            if (idle)
                for (int i0 = begin; i0 < end; i0 += 32, now ^= 2 * HALF) {
                    wait_vmcnt<0>();
                    __syncthreads();
                    if (i0 + 32 < end) copy_rows(i0 + 32, now ^ 2 * HALF);
                }
            else
            for (int i0 = begin; i0 < end; i0 += 32, now ^= 2 * HALF) {
                Rows &rows = rows_of[now != 0];
                const int q_word = exponents_at(a.q_exps, first_tile + i0 / 64), d_word = exponents_at(a.do_exps, first_tile + i0 / 64);
                const int q_exp = tile_exponent(q_word), d_exp = tile_exponent(d_word);
                int dot_exp = q_exp + k_exp, dp_exp = v_exp + d_exp;
                if (threadIdx.x < 32) {
                    const int i = i0 + threadIdx.x, ii = min(i, a.Sq - 1);
                    const RowState row(a, im, n, i, head);
                    const float lse = i < a.Sq ? a.lse_in[first_row + ii] : -kInf;
                    const bool dead = lse == -kInf;
                    rows.lse[threadIdx.x] = dead ? kInf : lse * kLog2e;
                    rows.delta[threadIdx.x] = dead ? 0.f : a.delta[first_row + ii];
                    if ((MODE & 2) && a.slopes) rows.share[threadIdx.x] = a.share[first_row + ii];
                    rows.p[threadIdx.x] = row.p;
                    rows.code[threadIdx.x] = i < a.Sq ? row.code : RowState(a, im, n, ii, head).code;
                    rows.bound[threadIdx.x] = row.bound;
                    rows.doc[threadIdx.x] = row.doc;
                    int least = row.bound;
                    for (int d = 16; d; d >>= 1) least = min(least, __shfl_xor(least, d));
                    rows.bound[32] = least;
                    rows.doc[32] = -3;
                    const int first = __builtin_amdgcn_readfirstlane(row.doc);
                    if (__all(row.doc == first)) rows.doc[32] = first;
                }
                wait_vmcnt<0>();
                __syncthreads();
                if (i0 + 32 < end) copy_rows(i0 + 32, now ^ 2 * HALF);
                const char *tile_at = parts_lds + now, *qt = tile_at + token_place(m, g);
                floatx4 s[2] = {}, dp[2] = {};
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    products(s, qt + st * 2048, STEPS * 2048, k_hi[st], k_lo[st]);
                    products(dp, qt + HALF + st * 2048, STEPS * 2048, v_hi[st], v_lo[st]);
                }
                if (!EVEN && tile_mixed(q_word)) {
                    by_token(s, a.q_each + first_tile * 64 + i0 + 4 * g, k_exp);
                    dot_exp = 0;
                }
                if (!EVEN && tile_mixed(d_word)) {
                    by_token(dp, a.do_each + first_tile * 64 + i0 + 4 * g, v_exp);
                    dp_exp = 0;
                }
                const float dp_in = ldexpf(1.f, dp_exp);
                const bool capped = (MODE & 1) && a.cap > 0.f;
                float in = ldexpf(capped ? a.scale / a.cap : a.scale * kLog2e, dot_exp);
                floatx4 core[2];
                if (capped) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) s[b] *= in;
                    tanh_all(s);
#pragma unroll
                    for (int b = 0; b < 2; ++b) core[b] = s[b];
                    in = a.cap * kLog2e;
                }
                bool near = false;
                float base = 0.f;
                if ((MODE & 4) && a.table) {
                    const bool all_lo = __all(code - rows.code[0] <= -a.reach), all_hi = __all(code - rows.code[31] >= a.reach);
                    near = !all_lo && !all_hi;
                    base = all_lo ? far_lo : all_hi ? far_hi : 0.f;
                }
                if (!EVEN && k_bad) base = __builtin_nanf("");
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const floatx4 l4 = *reinterpret_cast<const floatx4 *>(rows.lse + 16 * b + 4 * g);
                    floatx4 u = base - l4;
                    if ((MODE & 2) && a.slopes) {
                        const int4 p4 = *reinterpret_cast<const int4 *>(rows.p + 16 * b + 4 * g);
                        u.x = fmaf(-slope, fabsf((float)(p4.x - j)), u.x);
                        u.y = fmaf(-slope, fabsf((float)(p4.y - j)), u.y);
                        u.z = fmaf(-slope, fabsf((float)(p4.z - j)), u.z);
                        u.w = fmaf(-slope, fabsf((float)(p4.w - j)), u.w);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][e] = fmaf(s[b][e], in, u[e]);
                }
                const int first = code - rows.code[0] - 4 * g + a.reach;
                if (near && bias && a.width == 1 && __all((first <= 2 * a.reach) & (first >= 19))) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][e] += bias[first - 16 * b - e];
                } else if (near && bias && __all((code - rows.code[31] >= -a.reach) & (code - rows.code[0] <= a.reach))) {
                    const int here = a.reach + code;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int4 c4 = *reinterpret_cast<const int4 *>(rows.code + 16 * b + 4 * g);
                        s[b].x += bias[here - c4.x];
                        s[b].y += bias[here - c4.y];
                        s[b].z += bias[here - c4.z];
                        s[b].w += bias[here - c4.w];
                    }
                } else if (near) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int4 c4 = *reinterpret_cast<const int4 *>(rows.code + 16 * b + 4 * g);
                        const int codes[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int x = offset_at(a, code, codes[e]);
                            s[b][e] += bias ? bias[x] : bias_gather(a, head, x);
                        }
                    }
                }
                if (!__all(j_raw < rows.bound[32])) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int4 x = *reinterpret_cast<const int4 *>(rows.bound + 16 * b + 4 * g);
                        s[b].x = j_raw < x.x ? s[b].x : -kInf;
                        s[b].y = j_raw < x.y ? s[b].y : -kInf;
                        s[b].z = j_raw < x.z ? s[b].z : -kInf;
                        s[b].w = j_raw < x.w ? s[b].w : -kInf;
                    }
                }
                if (a.docs && !__all(rows.doc[32] == doc)) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int4 x = *reinterpret_cast<const int4 *>(rows.doc + 16 * b + 4 * g);
                        s[b].x = x.x == doc ? s[b].x : -kInf;
                        s[b].y = x.y == doc ? s[b].y : -kInf;
                        s[b].z = x.z == doc ? s[b].z : -kInf;
                        s[b].w = x.w == doc ? s[b].w : -kInf;
                    }
                }
                if (!EVEN && tile_mixed(q_word)) bad_tokens<true>(s, a.q_each + first_tile * 64 + i0 + 4 * g);
                if (!EVEN && tile_mixed(d_word)) bad_tokens<true>(s, a.do_each + first_tile * 64 + i0 + 4 * g);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const floatx4 d4 = *reinterpret_cast<const floatx4 *>(rows.delta + 16 * b + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][e] = __builtin_amdgcn_exp2f(s[b][e]);
                    if ((MODE & 2) && a.slopes) s[b] *= *reinterpret_cast<const floatx4 *>(rows.share + 16 * b + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = s[b][e];
                        dp[b][e] = p == 0.f ? 0.f : p * fmaf(dp[b][e], dp_in, -d4[e]);
                    }
                }
                if (capped)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) dp[b][e] *= fmaf(-core[b][e], core[b][e], 1.f);
                const bool q_by_tokens = !EVEN && tile_by_tokens(q_word);
                if (q_by_tokens) by_token(dp, a.q_each + first_tile * 64 + i0 + 4 * g);
                cs.apply(dp, q_by_tokens ? 0 : q_exp, dk);
                const bool d_by_tokens = !EVEN && tile_by_tokens(d_word);
                if (d_by_tokens) by_token(s, a.do_each + first_tile * 64 + i0 + 4 * g);
                vs.apply(s, d_by_tokens ? 0 : d_exp, dv);
                half8 p_hi, p_lo, s_hi, s_lo;
                split_results(s[0], s[1], p_hi, p_lo);
                split_results(dp[0], dp[1], s_hi, s_lo);
                products_across<STEPS>(dv, tile_at + HALF + across_place(m, g), 0, p_hi, p_lo);
                products_across<STEPS>(dk, tile_at + across_place(m, g), 0, s_hi, s_lo);
            }
        }
    };
    if (__builtin_expect(even, 1)) walk(std::true_type{});
    else walk(std::false_type{});
    const AttnArgs z = late_args();
    if (j_raw >= z.Sk) return;
    const float dk_back = cs.back(z.scale), dv_back = vs.back(1.f);
    if (z.splits > 1) {
        // [part][image, key head][key][dk, dv][D]
        float *to = z.part_o + ((((size_t)part * z.N + n) * kv + key_head) * z.Sk + j) * 2 * z.D;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int c = 16 * d + 4 * g;
            if (z.vec) {
                if (c < z.D) {
                    *reinterpret_cast<floatx4 *>(to + c) = dk[d] * dk_back;
                    *reinterpret_cast<floatx4 *>(to + z.D + c) = dv[d] * dv_back;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < z.D) { to[c + e] = dk[d][e] * dk_back; to[z.D + c + e] = dv[d][e] * dv_back; }
            }
        }
        return;
    }
    float *tk = const_cast<float *>(token_at(z.dk, z.dks, n, j)), *tv = const_cast<float *>(token_at(z.dv, z.dvs, n, j));
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        const int c = 16 * d + 4 * g;
        if (z.vec) {
            store_quad<true>(z, z.dks, tk, key_head * z.D, c, dk[d] * dk_back);
            store_quad<true>(z, z.dvs, tv, key_head * z.D, c, dv[d] * dv_back);
        } else {
            store_quad<false>(z, z.dks, tk, key_head * z.D, c, dk[d] * dk_back);
            store_quad<false>(z, z.dvs, tv, key_head * z.D, c, dv[d] * dv_back);
        }
    }
}

// Adds the parts of dk and dv, in their order. A thread VEC neighbouring channels; units: how many of those there are.
template <int VEC>
__global__ void __launch_bounds__(256) attn_grad_join(AttnArgs a, size_t units)
{
    const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= units) return;
    float x[VEC] = {};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const float *from = a.part_o + ((size_t)s * units + e) * VEC;
        if constexpr (VEC == 4) {
            const floatx4 y = *reinterpret_cast<const floatx4 *>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] += y[i];
        } else {
            x[0] += *from;
        }
    }
    const int kv = a.by_group.div(a.heads), two = 2 * a.D / VEC;
    const size_t token = e / (unsigned)two;
    int c = (int)(e - token * two) * VEC;
    const size_t by_head = token / (unsigned)a.Sk;
    const int j = (int)(token - by_head * a.Sk), n = (int)(by_head / (unsigned)kv), key_head = (int)(by_head - (size_t)n * kv);
    const bool is_v = c >= a.D;
    c -= is_v ? a.D : 0;
    const TokenStrides &s = is_v ? a.dvs : a.dks;
    float *const to = const_cast<float *>(token_at(is_v ? a.dv : a.dk, s, n, j)) + channel_at(a, s, key_head * a.D + c);
    if constexpr (VEC == 4) *reinterpret_cast<floatx4 *>(to) = floatx4{x[0], x[1], x[2], x[3]};
    else *to = x[0];
}

}  // namespace

hipError_t launch_attn_grad_rows_parts(const AttnArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.heads * a.row_tiles);
    const size_t size = 2 * (size_t)a.reach + 1;
    const size_t more = ((a.bias_lds ? size : 0) + (a.part_bias ? a.bias_copies * (size + 1) : 0)) * sizeof(float);
    // (a cap and a table without distances have a form of their own: the walk over mixed tiles beside the other one leaves registers for no more. 2048 frames
    // with a prefix, 4 sequences, 190 us by the form for everything, 178 by this one)
    const int mode = attn_mode(a);
#define ROWS(st) \
    if (a.D <= 32 * st) { \
        const size_t lds = 3 * parts_tile_bytes(st) + more; \
        return mode == 0 ? launch_lds(attn_grad_rows_parts<st, 0>, grid, lds, a, s) \
             : mode == 4 ? launch_lds(attn_grad_rows_parts<st, 4>, grid, lds, a, s) \
             : mode == 5 ? launch_lds(attn_grad_rows_parts<st, 5>, grid, lds, a, s) : launch_lds(attn_grad_rows_parts<st, 7>, grid, lds, a, s); \
    }
    ROWS(1) ROWS(2) ROWS(3) ROWS(4)
#undef ROWS
    return hipErrorInvalidValue;
}

hipError_t launch_attn_grad_keys_parts(const AttnArgs &a, hipStream_t s)
{
    const int kv = a.heads / a.group;
    const unsigned grid = (unsigned)((long)a.N * kv * a.key_tiles * a.splits);
    const size_t more = a.bias_lds ? (2 * (size_t)a.reach + 1) * sizeof(float) : 0;
    const int mode = attn_mode(a);
    hipError_t e = hipErrorInvalidValue;
#define KEYS(st) \
    if (a.D <= 32 * st && a.D > 32 * (st - 1)) { \
        const size_t lds = 2 * parts_tile_bytes(st) + more; \
        e = mode == 0 ? launch_lds(attn_grad_keys_parts<st, 0>, grid, lds, a, s) \
          : mode == 4 ? launch_lds(attn_grad_keys_parts<st, 4>, grid, lds, a, s) : launch_lds(attn_grad_keys_parts<st, 7>, grid, lds, a, s); \
    }
    KEYS(1) KEYS(2) KEYS(3) KEYS(4)
#undef KEYS
    if (e != hipSuccess || a.splits == 1) return e;
    const size_t units = (size_t)a.N * kv * a.Sk * 2 * a.D / (a.vec ? 4 : 1);
    if (a.vec) hipLaunchKernelGGL(attn_grad_join<4>, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, s, a, units);
    else hipLaunchKernelGGL(attn_grad_join<1>, dim3((unsigned)((units + 255) / 256)), dim3(256), 0, s, a, units);
    return hipGetLastError();
}

}  // namespace small
