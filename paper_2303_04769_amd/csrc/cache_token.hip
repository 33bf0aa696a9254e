// Attention of new tokens over a paged cache (gfx950).
//
// Bound by the cache's bytes: every key and value is read once, straight into the registers where the matrix instructions want it. A tile is as many keys as make 64
// bytes of one channel: 16 floats, 32 bfloat16, 64 codes. Lane 16 g + m loads 16 bytes at a time: of keys E (m / 4) + 4 b + m % 4 (E elements a load, b a
// result's number) the channels E g .. of a chunk of 4 E, and of channels 16 c + m the values of keys E g .. E g + E - 1. So a lane's scores, rows 4 g .. 4 g + 3 of every
// result b, are of the keys whose values it holds, E neighbours that stand in one page, and become the next product's right operand where they are.
// Sixteen rows -- new tokens times the query heads of a key head -- are the columns of the products, mostly empty ones for single tokens.
//
// Codes are whole numbers below 128 and so bfloat16 numbers; queries and weights go in three bfloat16 parts of eight bits, which hold all of a float's 24 at its own
// range, so the products are those of floats: no power of two that a token's neighbours set, whatever the scales. A key's scale multiplies its score, a value's its weight.
#include "attn_tile.h"
#include "cache.h"

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) float token_lds[];

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ floatx4 mfma_bf16(uintx4 a, uintx4 b, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// The upper halves of two words.
__device__ __forceinline__ unsigned upper(unsigned lo, unsigned hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
// Eight codes as bfloat16 numbers.
__device__ __forceinline__ uintx4 widened(unsigned lo, unsigned hi)
{
    uintx4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = i < 2 ? lo : hi, at = 16 * (i & 1);
        r[i] = upper(__float_as_uint((float)(signed char)(w >> at)), __float_as_uint((float)(signed char)(w >> (at + 8))));
    }
    return r;
}
// Eight floats in three parts of eight bits each, cut off, not rounded: their sum is the float.
struct Parts3 { uintx4 p[3]; };
__device__ __forceinline__ Parts3 parts_of(const float (&x)[8])
{
    Parts3 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned h[2], m[2], l[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float v = x[2 * i + e];
            h[e] = __float_as_uint(v);
            const float rest = v - __uint_as_float(h[e] & 0xffff0000u);
            m[e] = __float_as_uint(rest);
            l[e] = __float_as_uint(rest - __uint_as_float(m[e] & 0xffff0000u));
        }
        r.p[0][i] = upper(h[0], h[1]);
        r.p[1][i] = upper(m[0], m[1]);
        r.p[2][i] = upper(l[0], l[1]);
    }
    return r;
}

// One row by one wave, key by key, for rows whose sums came out as NaN: in a product of tiles a key of weight zero contributes 0 * v, which is NaN where a token that
// the row does not see holds an infinite or NaN value. Slow, and reached only by caches that hold such values.
template <int KIND>
__device__ void attend_cached_row(const AttnArgs &a, const CacheArgs &c, const RowState &row, int n, int i, int key_head, int begin, int end, float (&o)[4], float &maximum, float &sum)
{
    const Scorer sc(a);
    const int lane = threadIdx.x & 63;
    const float *q = token_at(a.q, a.qs, n, i);
    const auto key = [&](size_t at, int d) -> float {
        if constexpr (KIND == SMALL_CACHE_F32) return reinterpret_cast<const float *>(c.keys)[at * c.Dk + d];
        else if constexpr (KIND == SMALL_CACHE_BF16) return (float)reinterpret_cast<const __bf16 *>(c.keys)[at * c.Dk + d];
        else return (float)reinterpret_cast<const signed char *>(c.keys)[at * c.Dk + d];
    };
    const auto value = [&](size_t page_row, int place, int d) -> float {
        const size_t at = page_row * c.D + ((size_t)d << c.shift) + place;
        if constexpr (KIND == SMALL_CACHE_F32) return reinterpret_cast<const float *>(c.values)[at];
        else if constexpr (KIND == SMALL_CACHE_BF16) return (float)reinterpret_cast<const __bf16 *>(c.values)[at];
        else return (float)reinterpret_cast<const signed char *>(c.values)[at];
    };
    const int inside = (1 << c.shift) - 1;
    const auto score = [&](int j) {
        const int page = j < end ? page_of(c, n, j) : -1;
        if (page < 0 || j >= row.bound) return -kInf;
        const size_t at = place_at(c, page, key_head, j & inside);
        float dot = 0.f;
        for (int d = 0; d < a.D; ++d) dot = fmaf(q[channel_at(a, a.qs, row.head * a.D + d)], key(at, d), dot);
        if constexpr (KIND == SMALL_CACHE_I8) dot *= c.key_scales[at];
        return sc.biased(sc.capped(dot), row, j, a.table ? j : 0, nullptr);
    };
    float top = -kInf;
    for (int j = begin + lane; j < end; j += 64) top = fmaxf(top, score(j));
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float ref = top == -kInf ? 0.f : top;
    float total = 0.f;
    o[0] = o[1] = o[2] = o[3] = 0.f;
    for (int j0 = begin; j0 < end; j0 += 64) {
        const float s = score(j0 + lane);
        const float p = s == -kInf ? 0.f : __builtin_amdgcn_exp2f(s - ref);
        total += p;
        for (unsigned long long left = __ballot(s != -kInf); left; left &= left - 1) {
            const int b = __ffsll((long long)left) - 1, j = j0 + b;
            float w = __shfl(p, b);
            const size_t page_row = place_at(c, page_of(c, n, j), key_head, 0);
            if constexpr (KIND == SMALL_CACHE_I8) w *= c.value_scales[page_row + (j & inside)];
            for (int x = 0; x < 4; ++x)
                if (lane + 64 * x < a.D) o[x] = fmaf(w, value(page_row, j & inside, lane + 64 * x), o[x]);
        }
    }
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    maximum = top;
    sum = total;
}

template <int KIND, int DT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) cache_token(AttnArgs a, CacheArgs c)
{
    constexpr int B = cache_bytes(KIND), E = 16 / B, NB = E / 4, KT = 4 * E, NS = (16 * DT + KT - 1) / KT, DP = 16 * DT, H = E / 8 > 0 ? E / 8 : 1;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_split = a.by_splits.div((int)id), split = (int)id - by_split * a.splits;
    const int by_tile = a.by_tiles.div(by_split), r0 = 16 * (by_split - by_tile * a.row_tiles);
    const int n = a.by_sets.div(by_tile), key_head = by_tile - n * a.head_sets, rows = min(16, a.rows - r0);
    const int r = r0 + min(m, rows - 1), hh = a.by_Sq.div(r), i = r - hh * a.Sq, head = key_head * a.group + hh;
    ImageMask im(a, n);
    if (!a.first) im.first = im.len - a.Sq;
    const RowState row(a, im, n, i, head);
    // keys up to the last one that a row of the tile can see, this workgroup's share of them in whole tiles
    const int last = a.by_Sq.div(r0) == a.by_Sq.div(r0 + rows - 1) ? r0 + rows - 1 - a.by_Sq.div(r0) * a.Sq : a.Sq - 1;
    const int hi = max(0, min(im.len, im.position(last) + 1));
    const int per = ((hi + KT - 1) / KT + a.splits - 1) / a.splits * KT, begin = min(hi, split * per), end = min(hi, begin + per);

    const int step = waves * KT, first = begin + wave * KT;
    int left = first < end ? (end - first + step - 1) / step : 0;
    const int stride = a.slopes ? -step : step;
    int j0 = first + (a.slopes ? (left - 1) * step : 0);

    uintx4 kx[NB][NS], vx[DT];
    floatx4 ksc[NB], vsc[NB];                                  // scales of codes
    // Pages of a lane's keys and of its values' keys: of tile j0, -1 where there is none.
    int k_page, v_page, k_next = -1, v_next = -1;
    const auto pages_at = [&](int j, int &kp, int &vp) {
        kp = page_of(c, n, min(j + E * (m >> 2), end - 1));    // (a chunk behind the last key: its page; its keys are hidden)
        vp = page_of(c, n, min(j + E * g, end - 1));
    };
    const auto fetch_k = [&](int j) {
        const int chunk = min(j + E * (m >> 2), (end - 1) & -E), place = chunk & ((1 << c.shift) - 1);
        const size_t at = place_at(c, max(0, k_page), key_head, place + (m & 3));
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int s = 0; s < NS; ++s) kx[b][s] = *reinterpret_cast<const uintx4 *>(c.keys + ((at + 4 * b) * c.Dk + min(E * g + KT * s, c.Dk - E)) * B);
        if constexpr (KIND == SMALL_CACHE_I8) {
            const int vplace = min(j + E * g, (end - 1) & -E) & ((1 << c.shift) - 1);
            const float *from = c.key_scales + place_at(c, max(0, v_page), key_head, vplace);
#pragma unroll
            for (int b = 0; b < NB; ++b) ksc[b] = *reinterpret_cast<const floatx4 *>(from + 4 * b);
        }
    };
    const auto fetch_v = [&](int j) {
        const int place = min(j + E * g, (end - 1) & -E) & ((1 << c.shift) - 1);
        const size_t page_row = place_at(c, max(0, v_page), key_head, 0);
        const char *from = c.values + (page_row * c.D + place) * B;
#pragma unroll
        for (int d = 0; d < DT; ++d) vx[d] = *reinterpret_cast<const uintx4 *>(from + ((size_t)min(16 * d + m, c.D - 1) << c.shift) * B);
        if constexpr (KIND == SMALL_CACHE_I8) {
#pragma unroll
            for (int b = 0; b < NB; ++b) vsc[b] = *reinterpret_cast<const floatx4 *>(c.value_scales + page_row + place + 4 * b);
        }
    };
    if (left) {
        pages_at(j0, k_page, v_page);
        fetch_k(j0);
        fetch_v(j0);
    }
    // queries: floats, or their parts
    floatx4 qf[KIND == SMALL_CACHE_F32 ? DT : 1];
    Parts3 qp[KIND == SMALL_CACHE_F32 ? 1 : NS * H];
    {
        const float *token = token_at(a.q, a.qs, n, i);
        const auto quad = [&](int d) { return a.vec ? load_quad<true>(a, a.qs, token, head * a.D, d) : load_quad<false>(a, a.qs, token, head * a.D, d); };
        if constexpr (KIND == SMALL_CACHE_F32) {
#pragma unroll
            for (int s = 0; s < DT; ++s) qf[s] = quad(16 * s + 4 * g);
        } else {
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const floatx4 f = quad(KT * s + E * g + 8 * h + 4 * e);
#pragma unroll
                        for (int y = 0; y < 4; ++y) x[4 * e + y] = f[y];
                    }
                    qp[s * H + h] = parts_of(x);
                }
        }
    }
    const float far_lo = a.table ? bias_gather(a, head, 0) : 0.f, far_hi = a.table ? bias_gather(a, head, 2 * a.reach) : 0.f;
    floatx4 o[DT] = {};
    Reference top(a, row, begin, end);
    float sum = 0.f;
    if (left > 1) pages_at(j0 + stride, k_next, v_next);
    for (; left; --left, j0 += stride) {
        const int key0 = j0 + E * g;                           // of this lane's scores: key0 + 4 b + e
        const bool no_page = v_page < 0;
        // a learned bias: all buckets are asked for, then all biases -- unless the tile's keys are all at one end of the reach, as most of a long cache is
        bool near = false;
        float far = 0.f, bias[NB][4];
        if (a.table) {
            const bool all_lo = __all(j0 + KT - 1 - row.code <= -a.reach), all_hi = __all(j0 - row.code >= a.reach);
            near = !all_lo && !all_hi;
            far = all_lo ? far_lo : all_hi ? far_hi : 0.f;
            if (near) {
                int bucket[NB][4];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bucket[b][e] = a.bucket[offset_at(a, key0 + 4 * b + e, row.code)];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bias[b][e] = a.table[(size_t)head * a.buckets + max(0, min(bucket[b][e], a.buckets - 1))];
            }
        }
        floatx4 s[NB] = {};
#pragma unroll
        for (int x = 0; x < NS; ++x)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if constexpr (KIND == SMALL_CACHE_F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b] = mfma(__uint_as_float(kx[b][x][e]), qf[x][e], s[b]);
                } else if constexpr (KIND == SMALL_CACHE_BF16) {
#pragma unroll
                    for (int p = 2; p >= 0; --p) s[b] = mfma_bf16(kx[b][x], qp[x].p[p], s[b]);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uintx4 k = widened(kx[b][x][2 * h], kx[b][x][2 * h + 1]);
#pragma unroll
                        for (int p = 2; p >= 0; --p) s[b] = mfma_bf16(k, qp[2 * x + h].p[p], s[b]);
                    }
                }
            }
        if constexpr (KIND == SMALL_CACHE_I8) {
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] *= ksc[b];
        }
        if (left > 1) {
            const int v_now = v_page;
            k_page = k_next; v_page = v_next;                  // (v_page too: key scales stand at the values' keys)
            fetch_k(j0 + stride);
            v_page = v_now;
        }
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
            for (int e = 0; e < 4; ++e) s[b][e] = fmaf(s[b][e], in, a.slopes ? fmaf(-row.slope, fabsf((float)(row.p - (key0 + 4 * b + e))), base) : base);
        if (near)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] += bias_log2(bias[b][e]);
        const int bound = min(row.bound, end);
        if (!__all((j0 + KT <= bound) & !no_page)) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b][e] = ((key0 + 4 * b + e < bound) & !no_page) ? s[b][e] : -kInf;
        }
        if (KIND != SMALL_CACHE_I8 && (j0 + KT > end || __any(no_page))) {       // what stands behind the last key, or in no page of the stream's, becomes zeros
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (KIND == SMALL_CACHE_F32) vx[d][x] = ((key0 + x < end) & !no_page) ? vx[d][x] : 0u;
                    else vx[d][x] &= no_page ? 0u : key0 + 2 * x + 1 < end ? 0xffffffffu : key0 + 2 * x < end ? 0xffffu : 0u;
                }
        }
        raise_top(s, top, sum, o);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[b][e] = __builtin_amdgcn_exp2f(s[b][e]);
                sum += s[b][e];
            }
        if constexpr (KIND == SMALL_CACHE_F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] = mfma(__uint_as_float(vx[d][e]), s[0][e], o[d]);
        } else {
#pragma unroll
            for (int h = 0; h < H; ++h) {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = s[2 * h + e / 4][e & 3];
                    if constexpr (KIND == SMALL_CACHE_I8) w[e] = p == 0.f ? 0.f : p * vsc[2 * h + e / 4][e & 3];      // (the scale of a hidden token may be anything)
                    else w[e] = p;
                }
                const Parts3 p = parts_of(w);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    uintx4 v;
                    if constexpr (KIND == SMALL_CACHE_I8) v = widened(vx[d][2 * h], vx[d][2 * h + 1]);
                    else v = vx[d];
#pragma unroll
                    for (int x = 2; x >= 0; --x) o[d] = mfma_bf16(v, p.p[x], o[d]);
                }
            }
        }
        if (left > 1) {
            v_page = v_next;
            fetch_v(j0 + stride);
            if (left > 2) pages_at(j0 + 2 * stride, k_next, v_next);
        }
    }
    sum = column_sum(sum);

    // join the waves: [wave][row][DP] and [wave][row] (maximum, sum)
    float *const lo_ = token_lds;
    float2 *const ml = reinterpret_cast<float2 *>(token_lds + waves * rows * DP);
    int *const flags = reinterpret_cast<int *>(ml + waves * rows);
    if (m < rows) {
#pragma unroll
        for (int d = 0; d < DT; ++d) *reinterpret_cast<floatx4 *>(lo_ + (wave * rows + m) * DP + 16 * d + 4 * g) = o[d];
        if (g == 0) ml[wave * rows + m] = float2{top.maximum(), sum};
    }
    if (threadIdx.x < 16) flags[threadIdx.x] = 0;
    __syncthreads();
    constexpr int QD = DP / 4;
    for (int e = threadIdx.x; e < rows * QD; e += blockDim.x) {
        const int rr = e / QD, d = (e - rr * QD) * 4;
        float all = -kInf, total = 0.f;
#pragma unroll 4
        for (int w = 0; w < waves; ++w) all = fmaxf(all, ml[w * rows + rr].x);
        const float ref = all == -kInf ? 0.f : all;
        floatx4 y = {};
#pragma unroll 4
        for (int w = 0; w < waves; ++w) {
            const float2 p = ml[w * rows + rr];
            const floatx4 z = *reinterpret_cast<const floatx4 *>(lo_ + (w * rows + rr) * DP + d);
            const float f = __builtin_amdgcn_exp2f(p.x - ref);
            total += p.y == 0.f ? 0.f : f * p.y;
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] += p.y == 0.f ? 0.f : f * z[x];       // (a wave that saw no key)
        }
        if (d < a.D && (y.x != y.x || y.y != y.y || y.z != y.z || y.w != y.w)) flags[rr] = 1;
        const int h2 = a.by_Sq.div(r0 + rr), i2 = r0 + rr - h2 * a.Sq, head2 = key_head * a.group + h2;
        const size_t part = (((size_t)n * a.head_sets + key_head) * a.rows + r0 + rr) * a.splits + split;
        if (a.splits > 1) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (d + x < a.D) a.part_o[part * a.D + d + x] = y[x];
            if (d == 0) a.part_ml[part] = float2{all, total};
        } else {
            const floatx4 z = total == 0.f ? floatx4{} : y * (1.f / total);
            float *token = const_cast<float *>(token_at(a.o, a.os, n, i2));
            if (a.vec) store_quad<true>(a, a.os, token, head2 * a.D, d, z);
            else store_quad<false>(a, a.os, token, head2 * a.D, d, z);
            if (a.lse && d == 0) a.lse[((size_t)n * a.heads + head2) * a.Sq + i2] = total == 0.f ? -kInf : (all + __builtin_amdgcn_logf(total)) * kLn2;
        }
    }
    __syncthreads();
    for (int rr = wave; rr < rows; rr += waves) {
        if (!flags[rr]) continue;
        const int h2 = a.by_Sq.div(r0 + rr), i2 = r0 + rr - h2 * a.Sq, head2 = key_head * a.group + h2;
        const RowState again(a, im, n, i2, head2);
        float y[4], most, total;
        attend_cached_row<KIND>(a, c, again, n, i2, key_head, begin, end, y, most, total);
        const size_t part = (((size_t)n * a.head_sets + key_head) * a.rows + r0 + rr) * a.splits + split;
        const float inv = total == 0.f ? 0.f : 1.f / total;
        for (int x = 0; x < 4; ++x) {
            const int d = lane + 64 * x;
            if (d >= a.D) continue;
            if (a.splits > 1) a.part_o[part * a.D + d] = y[x];
            else const_cast<float *>(token_at(a.o, a.os, n, i2))[channel_at(a, a.os, head2 * a.D + d)] = total == 0.f ? 0.f : y[x] * inv;
        }
        if (lane) continue;
        if (a.splits > 1) a.part_ml[part] = float2{most, total};
        else if (a.lse) a.lse[((size_t)n * a.heads + head2) * a.Sq + i2] = total == 0.f ? -kInf : (most + __builtin_amdgcn_logf(total)) * kLn2;
    }
}

template <int KIND>
hipError_t token_kind(const AttnArgs &a, const CacheArgs &c, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.head_sets * a.row_tiles * a.splits);
    const int rows = a.rows < 16 ? a.rows : 16, keys = 64 / cache_bytes(KIND);
    // waves of a workgroup: as many as have a tile to do each, as far as their results fit 64 KB of LDS together
#define TOKEN(dt, most) \
    if (a.D <= 16 * dt) { \
        const int need = ((a.Sk + keys - 1) / keys + a.splits - 1) / a.splits; \
        int w = 1; \
        while (w < most && w < need && 2 * w * rows * (16 * dt + 2) * 4 + 64 <= 65536) w *= 2; \
        hipLaunchKernelGGL((cache_token<KIND, dt, most>), dim3(grid), dim3(64 * w), (size_t)w * rows * (16 * dt + 2) * 4 + 64, s, a, c); \
        return hipGetLastError(); \
    }
    TOKEN(1, 8) TOKEN(2, 8) TOKEN(3, 8) TOKEN(4, 8) TOKEN(5, 8) TOKEN(6, 8) TOKEN(8, 8) TOKEN(16, 4)
#undef TOKEN
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_token(const AttnArgs &a, const CacheArgs &c, bool vec, hipStream_t s)
{
    AttnArgs x = a;
    x.vec = vec;
    switch (c.kind) {
    case SMALL_CACHE_F32: return token_kind<SMALL_CACHE_F32>(x, c, s);
    case SMALL_CACHE_BF16: return token_kind<SMALL_CACHE_BF16>(x, c, s);
    default: return token_kind<SMALL_CACHE_I8>(x, c, s);
    }
}

}  // namespace small
