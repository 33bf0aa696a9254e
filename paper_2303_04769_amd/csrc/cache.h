// What the kernels of the paged cache share (cache_store.hip, cache_token.hip): its layout and codes (gfx950).
#pragma once
#include "rotary.h"
#include "../include/small_cache.h"

namespace small {

struct CacheArgs {
    char *keys, *values;
    float *key_scales, *value_scales;
    int kind, pages, shift, kv_heads, D, Dk, per_stream;      // shift: log2 of a page's tokens
    const int *table;
    int workgroups;                                           // attention: at most so many
    int2 *units;                                              // the first and last workgroup that has a part of a unit; null: none is split
    FastDiv by_rows;
};

__host__ __device__ constexpr int cache_bytes(int kind) { return kind == SMALL_CACHE_F32 ? 4 : kind == SMALL_CACHE_BF16 ? 2 : 1; }

// Number of the page that holds token p of stream n, or -1.
__device__ __forceinline__ int page_of(const CacheArgs &c, int n, int p)
{
    if (p < 0 || (p >> c.shift) >= c.per_stream) return -1;
    const int page = c.table[(size_t)n * c.per_stream + (p >> c.shift)];
    return (unsigned)page < (unsigned)c.pages ? page : -1;
}
// Elements in front of place `at` of a head's page: of the scales; times D of the values, times Dk of the keys at place 0.
__device__ __forceinline__ size_t place_at(const CacheArgs &c, int page, int head, int at) { return (((size_t)page * c.kv_heads + head) << c.shift) + at; }

// 8-bit codes: scale and factor of a token whose largest channel has these bits.
struct Scale { float scale, by; };
__device__ __forceinline__ Scale scale_of(unsigned top_bits)
{
    const float top = __uint_as_float(top_bits);
    if (top_bits >= 0x7f800000u) return Scale{__uint_as_float(0x7fc00000u), 0.f};        // infinite or NaN
    if (top < 0x1p-100f) return Scale{0.f, 0.f};
    return Scale{top / 127.f, 127.f / top};
}
__device__ __forceinline__ int code_of_value(float x, float by) { return by == 0.f ? 0 : (int)__builtin_rintf(x * by); }

hipError_t launch_rotary(const RotaryArgs &a, bool vec, bool halves, hipStream_t s);                       // rotary.hip
hipError_t launch_rotary_grad(const RotaryArgs &a, bool vec, bool halves, bool from_inputs, float *dfreq, hipStream_t s);

struct StoreArgs {
    CacheArgs c;
    RotaryArgs r;                            // turns, where `turns`; its N, S, D, Cb, by_Cb are the call's anyway
    const float *k, *v;
    float *k_out, *v_out;                    // read
    TokenStrides ks, vs;
    int fast;                                // RotaryArgs' FAST, of these tensors
    long long q_step, qo_step, k_step, v_step;
    int turns, N, S, lanes_log2, tile, tiles, items, parts;      // tile: tokens of a workgroup, 16 or 1
    const int *first, *counts;
    FastDiv by_parts, by_tiles, by_per_q;                        // by_per_q: query heads of one set of frequencies
};
hipError_t launch_cache_write(const StoreArgs &a, bool vec, bool halves, hipStream_t s);                   // cache_store.hip
hipError_t launch_cache_read(const StoreArgs &a, bool vec, hipStream_t s);
struct TokenShape { int rows, keys, per_cu; };               // rows of a unit, keys of a round, workgroups that a compute unit runs at a time
TokenShape token_shape(int kind, int D, int rows);                                                          // cache_token.hip
hipError_t launch_cache_token(const AttnArgs &a, const CacheArgs &c, bool joined, hipStream_t s);

}  // namespace small
