// Attention of few rows (at most 16: single tokens, and the query heads that share a key head) against a long cache, forward (gfx950).
//
// Bound by the cache's bytes: every key and value is read once, straight into the registers where the matrix instructions want it (no
// LDS: nothing is shared between waves). A key head's rows are the 16 columns of a wave's products -- mostly empty for single tokens, which the
// matrix pipe can afford: 256 bytes of cache are 32 of its cycles, 19 TB/s over the chip. The waves of a workgroup take the
// tiles of its keys in turn and join through LDS; long caches are split over workgroups too and joined by attn_join.
//
// Measured: 64 streams of 2048 to 16384 keys, 16 heads of 64 on 4, 250 us, 4.9 TB/s; one stream of 777 keys, 8 heads of 32, a bias by buckets, 13.4 us, two
// launches of some 4 us and the time that a chain of dependent loads takes (bucket, bias, keys, values).
#include "attn_row.h"

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) float token_lds[];

// The key that row 4g + e of result b stands for: keys in turn over the lane groups, so that the four that a wave's load of values takes are neighbours.
__device__ __forceinline__ int key_of(int j0, int b, int e, int g) { return j0 + 16 * b + 4 * e + g; }

template <int DT, int KT, int WAVES, int LAYOUT>
__global__ void __launch_bounds__(64 * WAVES) attn_token(AttnArgs a)
{
    constexpr int VD = kVD<DT>, GR = DT / VD, NB = KT / 16, DP = DT * 16;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_split = a.by_splits.div((int)id), split = (int)id - by_split * a.splits;
    const int n = a.by_sets.div(by_split), set = by_split - n * a.head_sets;
    const int r = min(m, a.rows - 1), hh = a.pack ? a.by_Sq.div(r) : 0, i = r - hh * a.Sq;
    const int head = a.pack ? set * a.group + hh : set, key_head = a.pack ? set : a.by_group.div(set), key_base = key_head * a.D;
    constexpr bool VEC = LAYOUT > 0;
    const float *kbase = token_at(a.k, a.ks, n, 0), *vbase = token_at(a.v, a.vs, n, 0);
    floatx4 kx[NB][DT];
    float vx[NB * 4][GR][VD];
    // Loads without conditions: tokens past the cache are its last one (its score is hidden, its value set to zero), channels past the head's are its last
    // ones (they meet zeros of q, and belong to results that nobody stores).
    // LAYOUT 2: sixteen channels stand together, so their block is the same for a wave, and a token is within 32 bits of the first.
    const auto fetch_k = [&](int j0) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int j = min(key_of(j0, b, m & 3, m >> 2), a.Sk - 1);
            const float *token = kbase + (long long)j * a.ks.token;
            const unsigned off = (unsigned)j * (unsigned)a.ks.token + 4u * g;
#pragma unroll
            for (int c = 0; c < DT; ++c) {
                const int d = 16 * c + 4 * g;
                if constexpr (LAYOUT == 2) kx[b][c] = *reinterpret_cast<const floatx4 *>(kbase + channel_at(a, a.ks, key_base + min(16 * c, a.D - 16)) + off);
                else if constexpr (VEC) kx[b][c] = *reinterpret_cast<const floatx4 *>(token + channel_at(a, a.ks, key_head * a.D + min(d, a.D - 4)));
                else
#pragma unroll
                    for (int x = 0; x < 4; ++x) kx[b][c][x] = token[channel_at(a, a.ks, key_head * a.D + min(d + x, a.D - 1))];
            }
        }
    };
    // (a lane's channels of a group: VD m .. of 16 VD, a block of 16 for each 16 / VD lanes)
    const unsigned v_in = (unsigned)(m * VD & 15);
    const auto fetch_v = [&](int j0) {
#pragma unroll
        for (int grp = 0; grp < GR; ++grp) {
            const int d = (grp * 16 + m) * VD;
            const float *lane_base = vbase + channel_at(a, a.vs, key_base + min(d & ~15, a.D - 16)) + v_in;      // (LAYOUT 2)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = min(key_of(j0, b, e, g), a.Sk - 1);
                    const float *token = vbase + (long long)j * a.vs.token;
                    float(&x)[VD] = vx[4 * b + e][grp];
                    const float *from = LAYOUT == 2 ? lane_base + (unsigned)j * (unsigned)a.vs.token : token + channel_at(a, a.vs, key_head * a.D + min(d, a.D - VD));
                    if constexpr (VEC && VD == 4) {
                        const floatx4 f = *reinterpret_cast<const floatx4 *>(from);
                        x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
                    } else if constexpr (VEC && VD == 2) {
                        const float2 f = *reinterpret_cast<const float2 *>(from);
                        x[0] = f.x; x[1] = f.y;
                    } else if constexpr (VEC) {
                        x[0] = *from;
                    } else {
#pragma unroll
                        for (int v = 0; v < VD; ++v) x[v] = token[channel_at(a, a.vs, key_head * a.D + min(d + v, a.D - 1))];
                    }
                }
        }
    };
    // Where keys are not split, a wave's first tile does not depend on the image's length: it is on its way before that is known.
    const int first = wave * KT;
    const bool early = a.splits == 1 && first < a.Sk && !a.slopes;
    if (early) { fetch_k(first); fetch_v(first); }
    floatx4 q[DT];
    {
        const float *token = token_at(a.q, a.qs, n, i);
#pragma unroll
        for (int c = 0; c < DT; ++c) q[c] = load_quad<VEC>(a, a.qs, token, head * a.D, 16 * c + 4 * g);
    }
    const ImageMask im(a, n);
    const RowState row(a, im, n, i, head);
    // keys up to the last one that a row can see, this workgroup's share of them in whole tiles
    int hi = im.len;
    if (a.causal) hi = max(0, min(hi, max(im.position(a.Sq - 1) + 1, im.prefix)));
    const int per = ((hi + KT - 1) / KT + a.splits - 1) / a.splits * KT, begin = min(hi, split * per), end = min(hi, begin + per);

    const float far_lo = a.table ? bias_gather(a, head, 0) : 0.f, far_hi = a.table ? bias_gather(a, head, 2 * a.reach) : 0.f;
    floatx4 o[DT] = {};
    Reference top(a, row, begin, end);
    float sum = 0.f;
    const int step = waves * KT;
    // With distances from the last tile to the first: the nearest keys set the reference, and no score that counts is rounded far above it (a step of
    // 256 keys at a slope of 0.7 against it: errors of 3e-6).
    int left = begin + first < end ? (end - begin - first + step - 1) / step : 0;
    const int stride = a.slopes ? -step : step;
    int j0 = begin + first + (a.slopes ? (left - 1) * step : 0);
    if (!early && left) { fetch_k(j0); fetch_v(j0); }
    for (; left; --left, j0 += stride) {
        // a learned bias: all buckets are asked for, then all biases -- unless the tile's keys are all at one end of the reach, as most of a long cache is
        bool near = false;
        float far = 0.f, bias[NB][4];
        if (a.table) {
            const bool all_lo = __all(code_of(a, j0 + KT - 1) - row.code <= -a.reach), all_hi = __all(code_of(a, j0) - row.code >= a.reach);
            near = !all_lo && !all_hi;
            far = all_lo ? far_lo : all_hi ? far_hi : 0.f;
            if (near) {
                int bucket[NB][4];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bucket[b][e] = a.bucket[offset_at(a, code_of(a, key_of(j0, b, e, g)), row.code)];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bias[b][e] = a.table[(size_t)head * a.buckets + max(0, min(bucket[b][e], a.buckets - 1))];
            }
        }
        floatx4 s[NB] = {};
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b] = mfma(kx[b][c][e], q[c][e], s[b]);
        if (left > 1) fetch_k(j0 + stride);
        const float base = far - top.at;
        float in = a.scale * kLog2e;
        if (a.cap > 0.f) {
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] *= a.scale / a.cap;
            tanh_all(s);
            in = a.cap * kLog2e;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][e] = fmaf(s[b][e], in, a.slopes ? fmaf(-row.slope, fabsf((float)(row.p - key_of(j0, b, e, g))), base) : base);
        if (near)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] += bias_log2(bias[b][e]);
        if (!__all(j0 + KT <= min(row.bound, end))) {
            const int bound = min(row.bound, end);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] = key_of(j0, b, e, g) < bound ? s[b][e] : -kInf;
        }
        if (a.docs) {
            int doc[NB][4];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) doc[b][e] = key_document(a, n, key_of(j0, b, e, g));
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] = doc[b][e] == row.doc ? s[b][e] : -kInf;
        }
        if (j0 + KT > end)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int grp = 0; grp < GR; ++grp)
#pragma unroll
                        for (int v = 0; v < VD; ++v) vx[4 * b + e][grp][v] = key_of(j0, b, e, g) < end ? vx[4 * b + e][grp][v] : 0.f;
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
                for (int grp = 0; grp < GR; ++grp)
#pragma unroll
                    for (int v = 0; v < VD; ++v) o[grp * VD + v] = mfma(vx[4 * b + e][grp][v], s[b][e], o[grp * VD + v]);
        if (left > 1) fetch_v(j0 + stride);
    }
    sum = column_sum(sum);

    // join the waves: [wave][row][DP] and [wave][row] (maximum, sum)
    float *const lo_ = token_lds;
    float2 *const ml = reinterpret_cast<float2 *>(token_lds + waves * a.rows * DP);
    int *const flags = reinterpret_cast<int *>(ml + waves * a.rows);
    if (m < a.rows) {
#pragma unroll
        for (int grp = 0; grp < GR; ++grp)
#pragma unroll
            for (int x = 0; x < VD; ++x)
                *reinterpret_cast<floatx4 *>(lo_ + (wave * a.rows + m) * DP + grp * 16 * VD + 4 * g * VD + 4 * x) = result_quad<DT>(o, grp, x);
        if (g == 0) ml[wave * a.rows + m] = float2{top.maximum(), sum};
    }
    if (threadIdx.x < 16) flags[threadIdx.x] = 0;
    __syncthreads();
    constexpr int QD = DP / 4;
    for (int e = threadIdx.x; e < a.rows * QD; e += blockDim.x) {
        const int rr = e / QD, d = (e - rr * QD) * 4;
        // (in steps of four, whose reads are on their way together)
        float all = -kInf, total = 0.f;
#pragma unroll 4
        for (int w = 0; w < waves; ++w) all = fmaxf(all, ml[w * a.rows + rr].x);
        const float ref = all == -kInf ? 0.f : all;
        floatx4 y = {};
#pragma unroll 4
        for (int w = 0; w < waves; ++w) {
            const float2 p = ml[w * a.rows + rr];
            const floatx4 z = *reinterpret_cast<const floatx4 *>(lo_ + (w * a.rows + rr) * DP + d);
            const float f = __builtin_amdgcn_exp2f(p.x - ref);
            total += p.y == 0.f ? 0.f : f * p.y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] += p.y == 0.f ? 0.f : f * z[x];       // (a wave that saw no key)
        }
        if (y.x != y.x || y.y != y.y || y.z != y.z || y.w != y.w) flags[rr] = 1;
        const int h2 = a.pack ? a.by_Sq.div(rr) : 0, i2 = rr - h2 * a.Sq, head2 = a.pack ? set * a.group + h2 : set;
        const size_t part = (((size_t)n * a.head_sets + set) * a.rows + rr) * a.splits + split;
        if (a.splits > 1) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (d + x < a.D) a.part_o[part * a.D + d + x] = y[x];
            if (d == 0) a.part_ml[part] = float2{all, total};
        } else {
            store_quad<VEC>(a, a.os, const_cast<float *>(token_at(a.o, a.os, n, i2)), head2 * a.D, d, total == 0.f ? floatx4{} : y * (1.f / total));
            if (a.lse && d == 0) a.lse[((size_t)n * a.heads + head2) * a.Sq + i2] = total == 0.f ? -kInf : (all + __builtin_amdgcn_logf(total)) * kLn2;
        }
    }
    __syncthreads();
    for (int rr = wave; rr < a.rows; rr += waves)
        if (flags[rr]) attend_row_and_store(a, im, n, set, rr, split, begin, end);
}

}  // namespace

hipError_t launch_attn_token(const AttnArgs &a, bool vec, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.head_sets * a.splits);
    const int layout = !vec ? 0 : a.D % 16 == 0 && a.Cb % 16 == 0 && (double)a.Sk * a.ks.token < 1e9 && (double)a.Sk * a.vs.token < 1e9 ? 2 : 1;
    // waves of a workgroup: as many as have a tile to do each, as far as their results fit 64 KB of LDS together
#define TOKEN(dt, kt, most) \
    if (a.D <= 16 * dt) { \
        const int need = ((a.Sk + kt - 1) / kt + a.splits - 1) / a.splits; \
        int w = 1; \
        while (w < most && w < need && 2 * w * a.rows * (16 * dt + 2) * 4 + 64 <= 65536) w *= 2; \
        const size_t lds = (size_t)w * a.rows * (16 * dt + 2) * 4 + 64; \
        if (layout == 2) hipLaunchKernelGGL((attn_token<dt, kt, most, 2>), dim3(grid), dim3(64 * w), lds, s, a); \
        else if (layout == 1) hipLaunchKernelGGL((attn_token<dt, kt, most, 1>), dim3(grid), dim3(64 * w), lds, s, a); \
        else hipLaunchKernelGGL((attn_token<dt, kt, most, 0>), dim3(grid), dim3(64 * w), lds, s, a); \
        return hipGetLastError(); \
    }
    TOKEN(1, 32, 8) TOKEN(2, 32, 8) TOKEN(3, 32, 8) TOKEN(4, 32, 8) TOKEN(5, 16, 8) TOKEN(6, 16, 8) TOKEN(8, 16, 8) TOKEN(16, 16, 4)
#undef TOKEN
    return hipErrorInvalidValue;
}

}  // namespace small
