// Keys and values into the pages of a cache and back (gfx950).
//
// Bound by memory: activations in, codes out, or the other way. A workgroup has sixteen tokens that are neighbours in one page (or one token, where a call brings one a
// stream), four channels of a token a thread, and goes through its share of the heads: queries that are only turned, keys, values. Sines are computed
// once for all heads that share them. Values go through LDS, since a channel's tokens stand together in the cache: sixteen of them are a store of 16 to 64 bytes.
#include "cache.h"

#include <type_traits>

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) char store_lds[];

template <int KIND> using Stored = std::conditional_t<KIND == SMALL_CACHE_F32, float, std::conditional_t<KIND == SMALL_CACHE_BF16, __bf16, signed char>>;
// Bytes from one channel to the next in LDS.
template <int KIND> constexpr int kPitch = 16 * cache_bytes(KIND) + 16;

// Channels d .. d + 3 of a head, zeros behind its last.
template <bool VEC>
__device__ __forceinline__ floatx4 quad_of(const FastDiv &by_Cb, int D, const TokenStrides &s, const float *token, int c0, int d)
{
    floatx4 x = {};
    if constexpr (VEC) {
        if (d < D) x = *reinterpret_cast<const floatx4 *>(token + channel_of(by_Cb, s, c0 + d));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < D) x[e] = token[channel_of(by_Cb, s, c0 + d + e)];
    }
    return x;
}
template <bool VEC>
__device__ __forceinline__ void put_quad(const FastDiv &by_Cb, int D, const TokenStrides &s, float *token, int c0, int d, floatx4 x)
{
    if constexpr (VEC) {
        if (d < D) *reinterpret_cast<floatx4 *>(token + channel_of(by_Cb, s, c0 + d)) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (d + e < D) token[channel_of(by_Cb, s, c0 + d + e)] = x[e];
    }
}

// The turns of channels d .. d + 3: of their four pairs with HALVES, else of their two.
template <bool HALVES>
struct QuadTurns {
    Turn t[HALVES ? 4 : 2];
    __device__ __forceinline__ void set(const RotaryArgs &r, const int (&place)[4], int f, int d)
    {
#pragma unroll
        for (int e = 0; e < (HALVES ? 4 : 2); ++e) {
            const int k = HALVES ? (d + e < r.pairs ? d + e : d + e - r.pairs) : d / 2 + e;
            t[e] = turn_of(r, place, f, min(k, r.pairs - 1));
        }
    }
    // x: the quad; the other channels of its pairs are fetched where they are not in it
    template <bool VEC>
    __device__ __forceinline__ floatx4 turned(const RotaryArgs &r, const TokenStrides &s, const float *token, int c0, int d, floatx4 x) const
    {
        const int P = r.pairs;
        if constexpr (HALVES) {
            if (d >= 2 * P) return x;
            floatx4 y = {};
            if (VEC && P % 4 == 0) {
                y = *reinterpret_cast<const floatx4 *>(token + channel_of(r.by_Cb, s, c0 + (d < P ? d + P : d - P)));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < 2 * P) y[e] = token[channel_of(r.by_Cb, s, c0 + (d + e < P ? d + e + P : d + e - P))];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < 2 * P) x[e] = d + e < P ? first_of(t[e], x[e], y[e]) : second_of(t[e], y[e], x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (d + 2 * e < 2 * P) {
                    const float p = x[2 * e], q = x[2 * e + 1];
                    x[2 * e] = first_of(t[e], p, q);
                    x[2 * e + 1] = second_of(t[e], p, q);
                }
        }
        return x;
    }
};

// What a workgroup's thread is at: stream, token, first channel, and the tile's places.
struct At {
    int n, part, tok, d, first, count, i, lo, hi, base;       // tokens lo .. hi - 1 of the tile are the call's to write or read; base: position of its first
    int page, place;                                          // of base, page -1: none
    __device__ __forceinline__ At(const StoreArgs &a)
    {
        const int by_part = a.by_parts.div((int)blockIdx.x);
        part = (int)blockIdx.x - by_part * a.parts;
        n = a.by_tiles.div(by_part);
        const int j = by_part - n * a.tiles;
        tok = (int)threadIdx.x >> a.lanes_log2;
        d = 4 * ((int)threadIdx.x & ((1 << a.lanes_log2) - 1));
        first = a.first ? max(-kFar, min(a.first[n], kFar)) : 0;
        count = a.counts ? max(0, min(a.counts[n], a.S)) : a.S;
        base = (first & -a.tile) + j * a.tile;
        i = base - first + tok;
        lo = max(0, first - base);
        hi = min(a.tile, first + count - base);
        page = page_of(a.c, n, base);
        place = base & ((1 << a.c.shift) - 1);
    }
};

template <int KIND, bool VEC, bool HALVES>
__global__ void __launch_bounds__(1024) cache_write(StoreArgs a)
{
    using T = Stored<KIND>;
    constexpr int B = cache_bytes(KIND);
    const At at(a);
    const bool token = at.tok < a.tile && at.i >= 0 && at.i < a.S;      // there is such a token (of the padded batch)
    const bool kept = at.tok >= at.lo && at.tok < at.hi && at.page >= 0;
    const int lo_item = a.by_parts.div(at.part * a.items), hi_item = a.by_parts.div((at.part + 1) * a.items);
    const int q_items = a.items - 2 * a.c.kv_heads, D = a.c.D;
    int place[4];
    if (a.turns) place_of(a.r, at.n, at.i, at.first, place);
    QuadTurns<HALVES> turns;
    int turns_of = -1;
    const int i = max(0, min(at.i, a.S - 1));
    // An item's tensor, by its values: a choice between the arguments' own places would put them all into scratch memory.
    struct Source { const float *token; TokenStrides s; int head; bool is_q, is_k; };
    const auto source = [&](int item) {
        Source x;
        x.is_q = item < q_items;
        x.is_k = !x.is_q && item < q_items + a.c.kv_heads;
        x.head = x.is_q ? item : x.is_k ? item - q_items : item - q_items - a.c.kv_heads;
        x.s.image = x.is_q ? a.r.qs.image : x.is_k ? a.ks.image : a.vs.image;
        x.s.block = x.is_q ? a.r.qs.block : x.is_k ? a.ks.block : a.vs.block;
        x.s.token = x.is_q ? a.r.qs.token : x.is_k ? a.ks.token : a.vs.token;
        x.token = token_at(x.is_q ? a.r.q : x.is_k ? a.k : a.v, x.s, at.n, i);
        return x;
    };
    const auto fetch = [&](const Source &x) { return quad_of<VEC>(a.r.by_Cb, D, x.s, x.token, x.head * D, at.d); };
    Source coming = source(lo_item);
    floatx4 next = fetch(coming);
    for (int item = lo_item; item < hi_item; ++item) {
        floatx4 x = next;
        const Source now = coming;
        if (item + 1 < hi_item) {
            coming = source(item + 1);
            next = fetch(coming);
        }
        const bool is_q = now.is_q, is_k = now.is_k;
        const int head = now.head;
        if (a.turns && (is_q || is_k) && at.d < 2 * a.r.pairs) {
            const int f = a.r.freq_heads == 1 ? 0 : is_q ? a.by_per_q.div(head) : head;
            if (f != turns_of) turns.set(a.r, place, f, at.d);
            turns_of = f;
            x = turns.template turned<VEC>(a.r, now.s, now.token, head * D, at.d, x);
        }
        if (is_q) {
            if (token) put_quad<VEC>(a.r.by_Cb, D, a.r.qos, const_cast<float *>(token_at(a.r.qo, a.r.qos, at.n, i)), head * D, at.d, x);
            continue;
        }
        const size_t page_row = at.page >= 0 ? place_at(a.c, at.page, head, 0) : 0, row = page_row + at.place + at.tok;
        T c[4];
        if constexpr (KIND == SMALL_CACHE_I8) {
            unsigned top = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            for (int l = 1 << (a.lanes_log2 - 1); l; l >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, l));
            const Scale scale = scale_of(top);
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = (T)code_of_value(x[e], scale.by);
            if (kept && at.d == 0) (is_k ? a.c.key_scales : a.c.value_scales)[row] = scale.scale;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = (T)x[e];
        }
        if (is_k) {
            typedef T Quad __attribute__((ext_vector_type(4)));
            if (kept && at.d < a.c.Dk) *reinterpret_cast<Quad *>(a.c.keys + (row * a.c.Dk + at.d) * B) = Quad{c[0], c[1], c[2], c[3]};
            continue;
        }
        T *const tile = reinterpret_cast<T *>(a.c.values) + page_row * D + at.place;              // channel 0 of the tile's first token
        const int P = 1 << a.c.shift;
        if (a.tile == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (kept && at.d + e < D) tile[(size_t)(at.d + e) * P] = c[e];
            continue;
        }
        __syncthreads();                                       // (what the item before put there has been read)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at.d + e < D) reinterpret_cast<T *>(store_lds + (at.d + e) * kPitch<KIND>)[at.tok] = c[e];
        __syncthreads();
        if (at.page < 0 || at.lo >= at.hi) continue;           // (the same in all threads)
        if (at.lo == 0 && at.hi == 16) {
            for (int e = threadIdx.x; e < D * B; e += blockDim.x) {
                const int ch = e / B, piece = e % B;
                *reinterpret_cast<int4 *>(reinterpret_cast<char *>(tile + (size_t)ch * P) + 16 * piece) = *reinterpret_cast<const int4 *>(store_lds + ch * kPitch<KIND> + 16 * piece);
            }
        } else {
            for (int e = threadIdx.x; e < D * 16; e += blockDim.x) {
                const int ch = e >> 4, t = e & 15;
                if (t >= at.lo && t < at.hi) tile[(size_t)ch * P + t] = reinterpret_cast<const T *>(store_lds + ch * kPitch<KIND>)[t];
            }
        }
    }
}

template <int KIND, bool VEC>
__global__ void __launch_bounds__(1024) cache_read(StoreArgs a)
{
    using T = Stored<KIND>;
    constexpr int B = cache_bytes(KIND);
    const At at(a);
    if (at.page < 0 || at.lo >= at.hi) return;                 // (the whole workgroup)
    const bool kept = at.tok >= at.lo && at.tok < at.hi;
    const int lo_item = a.by_parts.div(at.part * a.items), hi_item = a.by_parts.div((at.part + 1) * a.items);
    const int D = a.c.D, P = 1 << a.c.shift, i = max(0, min(at.i, a.S - 1));
    for (int item = lo_item; item < hi_item; ++item) {
        const bool is_k = item < a.c.kv_heads;
        const int head = is_k ? item : item - a.c.kv_heads;
        const size_t page_row = place_at(a.c, at.page, head, 0), row = page_row + at.place + at.tok;
        T c[4] = {};
        if (is_k) {
            typedef T Quad __attribute__((ext_vector_type(4)));
            if (kept && at.d < a.c.Dk) {
                const Quad q = *reinterpret_cast<const Quad *>(a.c.keys + (row * a.c.Dk + at.d) * B);
#pragma unroll
                for (int e = 0; e < 4; ++e) c[e] = q[e];
            }
        } else {
            const T *const tile = reinterpret_cast<const T *>(a.c.values) + page_row * D + at.place;
            __syncthreads();
            for (int e = threadIdx.x; e < D * B; e += blockDim.x) {
                const int ch = e / B, piece = e % B;
                *reinterpret_cast<int4 *>(store_lds + ch * kPitch<KIND> + 16 * piece) = *reinterpret_cast<const int4 *>(reinterpret_cast<const char *>(tile + (size_t)ch * P) + 16 * piece);
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at.d + e < D) c[e] = reinterpret_cast<const T *>(store_lds + (at.d + e) * kPitch<KIND>)[at.tok];
        }
        if (!kept) continue;
        floatx4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)c[e];
        if constexpr (KIND == SMALL_CACHE_I8) {
            const float scale = (is_k ? a.c.key_scales : a.c.value_scales)[row];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] *= scale;
        }
        put_quad<VEC>(a.r.by_Cb, D, is_k ? a.ks : a.vs, (is_k ? a.k_out : a.v_out) + (at.n * (is_k ? a.ks : a.vs).image + i * (is_k ? a.ks : a.vs).token), head * D, at.d, x);
    }
}

template <int KIND>
hipError_t write_kind(const StoreArgs &a, bool vec, bool halves, unsigned grid, unsigned threads, hipStream_t s)
{
    const size_t lds = a.tile == 1 ? 0 : (size_t)a.c.D * kPitch<KIND>;
    if (vec && halves) hipLaunchKernelGGL((cache_write<KIND, true, true>), dim3(grid), dim3(threads), lds, s, a);
    else if (vec) hipLaunchKernelGGL((cache_write<KIND, true, false>), dim3(grid), dim3(threads), lds, s, a);
    else if (halves) hipLaunchKernelGGL((cache_write<KIND, false, true>), dim3(grid), dim3(threads), lds, s, a);
    else hipLaunchKernelGGL((cache_write<KIND, false, false>), dim3(grid), dim3(threads), lds, s, a);
    return hipGetLastError();
}
template <int KIND>
hipError_t read_kind(const StoreArgs &a, bool vec, unsigned grid, unsigned threads, hipStream_t s)
{
    const size_t lds = (size_t)a.c.D * kPitch<KIND>;
    if (vec) hipLaunchKernelGGL((cache_read<KIND, true>), dim3(grid), dim3(threads), lds, s, a);
    else hipLaunchKernelGGL((cache_read<KIND, false>), dim3(grid), dim3(threads), lds, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const StoreArgs &a, bool vec, bool halves, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.tiles * a.parts), threads = (unsigned)((a.tile << a.lanes_log2) + 63) / 64 * 64;
    switch (a.c.kind) {
    case SMALL_CACHE_F32: return write_kind<SMALL_CACHE_F32>(a, vec, halves, grid, threads, s);
    case SMALL_CACHE_BF16: return write_kind<SMALL_CACHE_BF16>(a, vec, halves, grid, threads, s);
    default: return write_kind<SMALL_CACHE_I8>(a, vec, halves, grid, threads, s);
    }
}

hipError_t launch_cache_read(const StoreArgs &a, bool vec, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.tiles * a.parts), threads = (unsigned)(a.tile << a.lanes_log2);
    switch (a.c.kind) {
    case SMALL_CACHE_F32: return read_kind<SMALL_CACHE_F32>(a, vec, grid, threads, s);
    case SMALL_CACHE_BF16: return read_kind<SMALL_CACHE_BF16>(a, vec, grid, threads, s);
    default: return read_kind<SMALL_CACHE_I8>(a, vec, grid, threads, s);
    }
}

}  // namespace small
