// Attention over whole sequences, forward (gfx950): tiles of 64 rows (16 a wave) walk over tiles of keys in LDS with the running maximum and
// sum of their softmax; see attn_tile.h for how the operands lie.
//
// Bound by the fp32 matrix instructions: a pair of a query and a key costs 4 D of their 64 flops a cycle and SIMD, 4 cycles at D = 64, against
// some twelve vector operations of which other waves' hide behind them, and 8 D / 64 bytes of LDS reads. It has what is too small for values in two parts (8 x 8
// pixels, 4 heads of 16, 256 images: 10 us, 4 of them the launch), heads of more than 128 channels, and rows of key heads packed together.
#include "attn_row.h"

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) float bias_lds_mem[];

template <int DT, int KT, bool VEC>
__global__ void __launch_bounds__(256, 2) attn_rows(AttnArgs a)
{
    constexpr int VD = kVD<DT>, GR = DT / VD, NB = KT / 16;
    using T = Tile<DT, KT>;
    __shared__ float kt[T::kFloats], vt[T::kFloats];
    __shared__ alignas(16) int key_code[KT];
    __shared__ alignas(16) int key_doc[KT + 1];
    __shared__ int words[2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    // (image, set of heads, tile of rows, split), the rows with the most keys first; neighbours share an XCD's cache
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_split = a.by_splits.div((int)id), split = (int)id - by_split * a.splits;
    const int by_tile = a.by_tiles.div(by_split), tile = a.row_tiles - 1 - (by_split - by_tile * a.row_tiles);
    const int n = a.by_sets.div(by_tile), set = by_tile - n * a.head_sets;

    const int row0 = tile * 64, r_raw = row0 + wave * 16 + m, r = min(r_raw, a.rows - 1);     // rows past the end repeat the last one
    const int hh = a.pack ? a.by_Sq.div(r) : 0, i = r - hh * a.Sq;
    const int head = a.pack ? set * a.group + hh : set, key_head = a.pack ? set : a.by_group.div(set);
    const ImageMask im(a, n);
    const RowState row(a, im, n, i, head);
    float q[DT * 4];
    {
        const float *token = token_at(a.q, a.qs, n, i);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const floatx4 x = load_quad<VEC>(a, a.qs, token, head * a.D, 16 * c + 4 * g);
            q[4 * c] = x.x; q[4 * c + 1] = x.y; q[4 * c + 2] = x.z; q[4 * c + 3] = x.w;
        }
    }

    // keys that any of the rows can see
    int lo = 0, hi = im.len;
    if (a.causal) {
        const int last = min(row0 + 63, a.rows - 1);
        const int h0 = a.pack ? a.by_Sq.div(row0) : 0, h1 = a.pack ? a.by_Sq.div(last) : 0;
        const int p_max = im.position(h0 == h1 ? last - h1 * a.Sq : a.Sq - 1);
        hi = max(0, min(hi, max(p_max + 1, im.prefix)));
    }
    if (a.docs) {
        if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
        __syncthreads();
        if (row.doc >= 0) { atomicMin(&words[0], row.doc); atomicMax(&words[1], row.doc); }
        __syncthreads();
        const int d0 = words[0], d1 = words[1];
        __syncthreads();
        document_hull(a.docs + (size_t)n * a.Sk, 0, hi, d0, d1, words, &lo, &hi);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    int begin = lo, end = hi;
    if (a.splits > 1) {
        const int per = ((hi - lo + KT - 1) / KT + a.splits - 1) / a.splits * KT;
        begin = min(hi, lo + split * per);
        end = min(hi, begin + per);
    }

    const float *bias = nullptr;
    float far_lo = 0.f, far_hi = 0.f;
    if (a.table) {
        if (a.bias_lds) {
            const int h0 = a.pack ? a.by_Sq.div(row0) : 0, h1 = a.pack ? a.by_Sq.div(min(row0 + 63, a.rows - 1)) : 0, size = 2 * a.reach + 1;
            for (int h = h0; h <= h1; ++h)
                for (int x = threadIdx.x; x < size; x += 256) bias_lds_mem[(h - h0) * size + x] = bias_gather(a, a.pack ? set * a.group + h : set, x);
            bias = bias_lds_mem + (hh - h0) * size;
        }
        far_lo = bias_gather(a, head, 0);
        far_hi = bias_gather(a, head, 2 * a.reach);
    }

    floatx4 o[DT] = {};
    Reference top(a, row, begin, end);
    float sum = 0.f;
    floatx4 kx[T::kQuads], vx[T::kQuads];
    const auto fetch = [&](int j0) {
        const auto on = [&](int j) { return j0 + j < im.len; };
        T::template fetch<VEC>(kx, a, a.ks, a.k, n, key_head * a.D, j0, on);
        T::template fetch<VEC>(vx, a, a.vs, a.v, n, key_head * a.D, j0, on);
    };
    if (begin < end) fetch(begin);
    for (int j0 = begin; j0 < end; j0 += KT) {
        __syncthreads();
        T::put(kt, kx);
        T::put(vt, vx);
        stage_keys<KT>(a, n, j0, key_code, key_doc);
        __syncthreads();
        if (j0 + KT < end) fetch(j0 + KT);

        floatx4 s[NB] = {};
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const floatx4 x = T::tokens(kt, b, c, m, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b] = mfma(x[e], q[4 * c + e], s[b]);
            }

        finish_scores<7>(a, s, row, 0, top.at, j0, key_code, key_doc, g, bias, far_lo, far_hi);

        raise_top(s, top, sum, o);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[b][e] = __builtin_amdgcn_exp2f(s[b][e]);
                sum += s[b][e];
            }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int grp = 0; grp < GR; ++grp) {
                    float x[VD];
                    T::template channels<VD>(x, vt, 16 * b + 4 * g + e, grp, m);
#pragma unroll
                    for (int v = 0; v < VD; ++v) o[grp * VD + v] = mfma(x[v], s[b][e], o[grp * VD + v]);
                }
    }
    sum = column_sum(sum);

    bool nan = false;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) nan |= o[d][e] != o[d][e];
    const unsigned long long lanes = __ballot(nan);
    const unsigned columns = (unsigned)((lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xffffu);
    if (r_raw < a.rows && !(columns >> m & 1)) {
        if (a.splits > 1) {
            const size_t part = (((size_t)n * a.head_sets + set) * a.rows + r) * a.splits + split;
            float *to = a.part_o + part * a.D;
#pragma unroll
            for (int grp = 0; grp < GR; ++grp)
#pragma unroll
                for (int x = 0; x < VD; ++x) {
                    const int d = grp * 16 * VD + 4 * g * VD + 4 * x;
                    const floatx4 y = result_quad<DT>(o, grp, x);
                    if (a.D % 4 == 0) {
                        if (d < a.D) *reinterpret_cast<floatx4 *>(to + d) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (d + e < a.D) to[d + e] = y[e];
                    }
                }
            if (g == 0) a.part_ml[part] = float2{top.maximum(), sum};
        } else {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;      // a row that saw nothing: zeros
            float *token = const_cast<float *>(token_at(a.o, a.os, n, i));
#pragma unroll
            for (int grp = 0; grp < GR; ++grp)
#pragma unroll
                for (int x = 0; x < VD; ++x)
                    store_quad<VEC>(a, a.os, token, head * a.D, grp * 16 * VD + 4 * g * VD + 4 * x, result_quad<DT>(o, grp, x) * inv);
            if (a.lse && g == 0) a.lse[((size_t)n * a.heads + head) * a.Sq + i] = sum == 0.f ? -kInf : (top.at + __builtin_amdgcn_logf(sum)) * kLn2;
        }
    }
    for (unsigned left = columns; left; left &= left - 1) {
        const int rr = row0 + wave * 16 + __ffs((int)left) - 1;
        if (rr < a.rows) attend_row_and_store(a, im, n, set, rr, split, begin, end);
    }
}

// Joins a row's parts: each is an unnormalized sum of values with the reference that its weights were taken against. WAVES waves a row (1: four rows a
// workgroup; 4: one row, for many parts), which take the parts in turn.
template <int WAVES>
__global__ void __launch_bounds__(256) attn_join(AttnArgs a, size_t rows)
{
    __shared__ float sums[4][256], all[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first = WAVES == 1 ? 0 : wave;
    const size_t at = WAVES == 1 ? (size_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (at >= rows) return;                                     // (WAVES 4: never)
    const float2 *ml = a.part_ml + at * a.splits;
    const float *parts = a.part_o + at * a.splits * a.D;
    float top = -kInf, sum = 0.f, o[4] = {};
#pragma unroll 4
    for (int s = lane; s < a.splits; s += 64) top = fmaxf(top, ml[s].x);
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float ref = top == -kInf ? 0.f : top;
#pragma unroll 4
    for (int s = first; s < a.splits; s += WAVES) {
        const float2 w = ml[s];
        const float x = w.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(w.x - ref);      // (a part that saw no key)
        sum = fmaf(x, w.y, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (lane + 64 * k < a.D) {
                const float y = parts[(size_t)s * a.D + lane + 64 * k];
                o[k] += w.y == 0.f ? 0.f : x * y;
            }
    }
    if constexpr (WAVES == 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[wave][lane + 64 * k] = o[k];
        if (lane == 0) all[wave] = sum;
        __syncthreads();
        if (wave) return;
        sum = (all[0] + all[1]) + (all[2] + all[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = (sums[0][lane + 64 * k] + sums[1][lane + 64 * k]) + (sums[2][lane + 64 * k] + sums[3][lane + 64 * k]);
    }
    const int by_set = (int)(at / (unsigned)a.rows), r = (int)(at - (size_t)by_set * a.rows), n = a.by_sets.div(by_set), set = by_set - n * a.head_sets;
    const int hh = a.pack ? a.by_Sq.div(r) : 0, i = r - hh * a.Sq, head = a.pack ? set * a.group + hh : set;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    float *token = const_cast<float *>(token_at(a.o, a.os, n, i));
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (lane + 64 * k < a.D) token[channel_at(a, a.os, head * a.D + lane + 64 * k)] = sum == 0.f ? 0.f : o[k] * inv;
    if (a.lse && lane == 0) a.lse[((size_t)n * a.heads + head) * a.Sq + i] = sum == 0.f ? -kInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

hipError_t launch_attn_rows(const AttnArgs &a, bool vec, size_t bias_bytes, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.head_sets * a.row_tiles * a.splits);
#define ROWS(dt, kt) \
    if (a.D <= 16 * dt) { \
        return vec ? launch_lds(attn_rows<dt, kt, true>, grid, bias_bytes, a, s) : launch_lds(attn_rows<dt, kt, false>, grid, bias_bytes, a, s); \
    }
    ROWS(1, 64) ROWS(2, 64) ROWS(3, 64) ROWS(4, 64) ROWS(5, 64) ROWS(6, 64) ROWS(8, 32) ROWS(16, 16)
#undef ROWS
    return hipErrorInvalidValue;
}

hipError_t launch_attn_join(const AttnArgs &a, hipStream_t s)
{
    const size_t rows = (size_t)a.N * a.head_sets * a.rows;
    if (a.splits >= 16 && rows < (1u << 30)) hipLaunchKernelGGL((attn_join<4>), dim3((unsigned)rows), dim3(256), 0, s, a, rows);
    else hipLaunchKernelGGL((attn_join<1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a, rows);
    return hipGetLastError();
}

}  // namespace small
