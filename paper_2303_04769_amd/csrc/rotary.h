// Turns of pairs of channels by the place of their token, as rotary.hip and cache_store.hip compute them (gfx950).
//
// Angles and turns are in 64 bits: the vector units multiply and add doubles as fast as floats, a token's sines serve all heads, and what remains is
// bound by memory. So a key that is turned on its way into a cache has the bits of one that was turned by itself, and codes that are rounded from it are the same.
#pragma once
#include "attn_tile.h"

namespace small {

struct RotaryArgs {
    const float *q, *k;
    float *qo, *ko;
    TokenStrides qs, ks, qos, kos;
    int N, S, heads, kv_heads, D, Cb, axes, pairs, freq_heads;
    float sign;                              // -1: back
    const float *freq;
    const int *first, *positions;
    FastDiv by_Cb, by_extent[4], by_S;
    int extent[4];
    // FAST: a head stands a fixed number of floats behind the one before in every tensor, and no tensor has 2^30 or more. Then what differs between lanes is an offset of 32
    // bits that all heads share, and a head's place is scalar: no vector operation is spent on addresses (14 x 14 pixels, 64 images, 8 heads of 32: 12.8 -> 11.2 us).
    int fast;
    long long q_step, k_step, qo_step, ko_step, yq_step, yk_step;
    // gradient by the frequencies: y (the turned q and k, or those before the turn) beside them
    const float *yq, *yk;
    TokenStrides yqs, yks;
    double *partial;                         // [freq_heads][chunks * parts][axes][pairs]
    // mapping (rotary.hip)
    int run, runs, parts, copy_run, copy_runs, chunks, per_chunk;
    unsigned turn_threads, copy_threads;
    FastDiv by_run, by_runs, by_parts, by_freq_heads, by_copy_run, by_copy_runs, by_copy_heads, by_chunks, by_sets;      // by_sets: freq_heads * parts
};

__device__ __forceinline__ long long channel_of(const FastDiv &by_Cb, const TokenStrides &s, int ch)
{
    const int b = by_Cb.div(ch);
    return b * s.block + (ch - b * (int)by_Cb.d);
}

__device__ __forceinline__ floatx4 quad_at(const float *base, unsigned bytes) { return *reinterpret_cast<const floatx4 *>(reinterpret_cast<const char *>(base) + bytes); }
// (results stream past the caches: 8 x 8192 tokens of 8 heads of 64 read from a cache of 8-bit codes 86 -> 68 us, clips of 16 x 28 x 28 pixels turned 26 -> 23)
__device__ __forceinline__ void put_quad_at(float *base, unsigned bytes, floatx4 x)
{
    __builtin_nontemporal_store(x, reinterpret_cast<floatx4 *>(reinterpret_cast<char *>(base) + bytes));
}
// A barrier that waits for what was written to LDS, and not for stores to memory, as __syncthreads does.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The place of a token on every axis.
__device__ __forceinline__ void place_of(const RotaryArgs &a, int n, int i, int first, int (&place)[4])
{
    if (a.positions) {
        const int *at = a.positions + ((size_t)n * a.S + i) * a.axes;
#pragma unroll
        for (int x = 0; x < 4; ++x) place[x] = x < a.axes ? at[x] : 0;
        return;
    }
    int t = max(-kFar, min(first, kFar)) + i;
#pragma unroll
    for (int x = 3; x >= 0; --x) {
        if (x >= a.axes) { place[x] = 0; continue; }
        if (x == 0) { place[0] = t; continue; }
        const int e = a.extent[x], up = t >= 0 ? a.by_extent[x].div(t) : -1 - a.by_extent[x].div(-1 - t);
        place[x] = t - up * e;
        t = up;
    }
}

struct Turn { double c, s; };

// Cosine and sine by their Taylor series on -pi/4 .. pi/4 (remainders below 2^-53), after the nearest multiple of pi/2 is taken off in two parts.
__device__ __forceinline__ Turn turn_by(double angle)
{
    constexpr double hi = 1.5707963267948966, lo = 6.123233995736766e-17, per = 0.6366197723675814;      // pi/2 = hi + lo, 2/pi
    const double n = __builtin_rint(angle * per);
    const double r = __builtin_fma(-n, lo, __builtin_fma(-n, hi, angle)), z = r * r;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;                                       // -1/15!, 1/16!
    s = __builtin_fma(s, z, 1.0 / 6227020800.0);
    c = __builtin_fma(c, z, -1.0 / 87178291200.0);
    s = __builtin_fma(s, z, -1.0 / 39916800.0);
    c = __builtin_fma(c, z, 1.0 / 479001600.0);
    s = __builtin_fma(s, z, 1.0 / 362880.0);
    c = __builtin_fma(c, z, -1.0 / 3628800.0);
    s = __builtin_fma(s, z, -1.0 / 5040.0);
    c = __builtin_fma(c, z, 1.0 / 40320.0);
    s = __builtin_fma(s, z, 1.0 / 120.0);
    c = __builtin_fma(c, z, -1.0 / 720.0);
    s = __builtin_fma(s, z, -1.0 / 6.0);
    c = __builtin_fma(c, z, 1.0 / 24.0);
    s = __builtin_fma(s * z, r, r);
    c = __builtin_fma(__builtin_fma(c, z, -0.5), z, 1.0);
    const int quarter = (int)__builtin_fma(-4.0, __builtin_floor(n * 0.25), n);
    const double x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
    return Turn{quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y};
}

// The turn of pair k of the heads of frequencies f, at a place; sign -1: back.
__device__ __forceinline__ Turn turn_of(const RotaryArgs &a, const int (&place)[4], int f, int k)
{
    const float *freq = a.freq + (size_t)f * a.axes * a.pairs + k;
    double angle = 0.0;
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (x < a.axes) angle = __builtin_fma((double)place[x], (double)freq[(size_t)x * a.pairs], angle);
    Turn t = turn_by(angle);
    t.s *= (double)a.sign;
    return t;
}
__device__ __forceinline__ float first_of(const Turn &t, float x0, float x1) { return (float)__builtin_fma((double)x0, t.c, -((double)x1 * t.s)); }
__device__ __forceinline__ float second_of(const Turn &t, float x0, float x1) { return (float)__builtin_fma((double)x0, t.s, (double)x1 * t.c); }

}  // namespace small
