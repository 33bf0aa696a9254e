// Keys and values into the pages of a cache and back (gfx950).
//
// Bound by memory: activations in, codes out, or the other way. A workgroup has sixteen tokens that are neighbours in one page (or one token, where a call brings one a
// stream), four channels of a token a thread, and goes through its share of the heads: queries that are only turned, keys, values. Sines are computed
// once for all heads that share them. Values go through LDS, since a channel's tokens stand together in the cache: sixteen of them are a store of 16 to 64 bytes.
// 8 x 8192 tokens of 8 heads of 64 read from 8-bit codes: 67 us, 5.0 TB/s; 4 x 4096 tokens turned and written: 36 us (a large copy: 4.9 TB/s).
// Written as they are, 8 x 8192 tokens: floats 127 us, 4.2 TB/s, bfloat16 103, 3.9, codes 83, 4.1; read: floats 102, 5.3, bfloat16 91, 4.4.
#include "cache.h"

#include <type_traits>

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) char store_lds[];

template <int KIND> using Stored = std::conditional_t<KIND == SMALL_CACHE_F32, float, std::conditional_t<KIND == SMALL_CACHE_BF16, __bf16, signed char>>;
// Bytes from one channel to the next in LDS: a word more than sixteen tokens, so that lanes with a token's channels, four apart, are in different banks.
template <int KIND> constexpr int kPitch = 16 * cache_bytes(KIND) + 4;
typedef int Words4 __attribute__((ext_vector_type(4), aligned(4)));

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
    // The other channels of a quad's pairs, where they are not in it.
    template <bool VEC>
    static __device__ __forceinline__ floatx4 others(const RotaryArgs &r, const TokenStrides &s, const float *token, int c0, int d)
    {
        const int P = r.pairs;
        floatx4 y = {};
        if (!HALVES || d >= 2 * P) return y;
        if (VEC && P % 4 == 0) {
            y = *reinterpret_cast<const floatx4 *>(token + channel_of(r.by_Cb, s, c0 + (d < P ? d + P : d - P)));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < 2 * P) y[e] = token[channel_of(r.by_Cb, s, c0 + (d + e < P ? d + e + P : d + e - P))];
        }
        return y;
    }
    __device__ __forceinline__ floatx4 turned(const RotaryArgs &r, int d, floatx4 x, floatx4 y) const
    {
        const int P = r.pairs;
        if constexpr (HALVES) {
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

// A lane's offset in the image of a tensor, in bytes, as FAST takes it (rotary.h).
__device__ __forceinline__ unsigned lane_offset(const FastDiv &by_Cb, const TokenStrides &s, int i, int ch) { return 4u * (unsigned)(i * s.token + channel_of(by_Cb, s, ch)); }

template <int KIND, bool VEC, bool HALVES, bool FAST>
__global__ void __launch_bounds__(1024) cache_write(StoreArgs a)
{
    using T = Stored<KIND>;
    constexpr int B = cache_bytes(KIND);
    const At at(a);
    const bool token = at.tok < a.tile && at.i >= 0 && at.i < a.S;      // there is such a token (of the padded batch)
    const bool kept = at.tok >= at.lo && at.tok < at.hi && at.page >= 0;
    const int lo_item = a.by_parts.div(at.part * a.items), hi_item = a.by_parts.div((at.part + 1) * a.items);
    const int q_items = a.items - 2 * a.c.kv_heads, D = a.c.D;
    QuadTurns<HALVES> turns;
    int turns_of = -1;
    const int i = max(0, min(at.i, a.S - 1)), other = max(0, at.d < a.r.pairs ? at.d + a.r.pairs : at.d - a.r.pairs), P = 1 << a.c.shift;
    const bool turning = a.turns && at.d < 2 * a.r.pairs;
    int place[4];
    if (a.turns) place_of(a.r, at.n, i, at.first, place);      // (of a token that there is: the tile's others have places, and positions, of none)
    // Heads of queries, of keys, of values, each kind with code of its own (a choice between the arguments' places, at run time, puts them all into scratch memory). The quads of
    // some heads, with HALVES with the other channels of their pairs, are on their way together.
    constexpr int G = 4;
    const auto heads = [&](auto kind) {
        constexpr int W = decltype(kind)::value;
        const int before = W == 0 ? 0 : W == 1 ? q_items : q_items + a.c.kv_heads, all = W == 0 ? q_items : a.c.kv_heads;
        const int lo = max(0, lo_item - before), hi = min(all, hi_item - before);
        if (lo >= hi) return;
        const TokenStrides s = W == 0 ? a.r.qs : W == 1 ? a.ks : a.vs;
        const float *const image = (W == 0 ? a.r.q : W == 1 ? a.k : a.v) + at.n * s.image;
        const long long step = W == 0 ? a.q_step : W == 1 ? a.k_step : a.v_step;
        const unsigned here = lane_offset(a.r.by_Cb, s, i, at.d), there = lane_offset(a.r.by_Cb, s, i, other);
        struct Source { floatx4 x, y; };
        const auto fetch = [&](int head) {
            Source r{};
            if constexpr (FAST) {
                if (at.d < D) r.x = quad_at(image + head * step, here);
                if (HALVES && W < 2 && turning) r.y = quad_at(image + head * step, there);
            } else {
                r.x = quad_of<VEC>(a.r.by_Cb, D, s, image + i * s.token, head * D, at.d);
                if (HALVES && W < 2 && turning) r.y = QuadTurns<HALVES>::template others<VEC>(a.r, s, image + i * s.token, head * D, at.d);
            }
            return r;
        };
        for (int first = lo; first < hi; first += G) {
        Source now[G];
#pragma unroll
        for (int b = 0; b < G; ++b) now[b] = fetch(min(first + b, hi - 1));
#pragma unroll
        for (int b = 0; b < G; ++b) {
            const int head = first + b;
            if (head >= hi) break;
            floatx4 x = now[b].x;
            if (W < 2 && turning) {
                const int f = a.r.freq_heads == 1 ? 0 : W == 0 ? a.by_per_q.div(head) : head;
                if (f != turns_of) turns.set(a.r, place, f, at.d);
                turns_of = f;
                x = turns.turned(a.r, at.d, x, now[b].y);
            }
            if constexpr (W == 0) {
                if constexpr (FAST) {
                    if (token && at.d < D) put_quad_at(a.r.qo + at.n * a.r.qos.image + head * a.qo_step, lane_offset(a.r.by_Cb, a.r.qos, i, at.d), x);
                } else if (token) {
                    put_quad<VEC>(a.r.by_Cb, D, a.r.qos, const_cast<float *>(token_at(a.r.qo, a.r.qos, at.n, i)), head * D, at.d, x);
                }
            } else {
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
                    if (kept && at.d == 0) (W == 1 ? a.c.key_scales : a.c.value_scales)[row] = scale.scale;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[e] = (T)x[e];
                }
                if constexpr (W == 1) {
                    typedef T Quad __attribute__((ext_vector_type(4)));
                    if (kept && at.d < a.c.Dk) *reinterpret_cast<Quad *>(a.c.keys + (row * a.c.Dk + at.d) * B) = Quad{c[0], c[1], c[2], c[3]};
                } else {
                    T *const tile = reinterpret_cast<T *>(a.c.values) + page_row * D + at.place;              // channel 0 of the tile's first token
                    if (a.tile == 1) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (kept && at.d + e < D) tile[(size_t)(at.d + e) * P] = c[e];
                        continue;
                    }
                    lds_barrier();                             // (what the head before put there has been read)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at.d + e < D) reinterpret_cast<T *>(store_lds + (at.d + e) * kPitch<KIND>)[at.tok] = c[e];
                    lds_barrier();
                    if (at.page < 0 || at.lo >= at.hi) continue;           // (the same in all threads)
                    if (at.lo == 0 && at.hi == 16) {
                        for (int e = threadIdx.x; e < D * B; e += blockDim.x) {
                            const int ch = e / B, piece = e % B;
                            *reinterpret_cast<int4 *>(reinterpret_cast<char *>(tile + (size_t)ch * P) + 16 * piece) =
                                __builtin_bit_cast(int4, *reinterpret_cast<const Words4 *>(store_lds + ch * kPitch<KIND> + 16 * piece));
                        }
                    } else {
                        for (int e = threadIdx.x; e < D * 16; e += blockDim.x) {
                            const int ch = e >> 4, t = e & 15;
                            if (t >= at.lo && t < at.hi) tile[(size_t)ch * P + t] = reinterpret_cast<const T *>(store_lds + ch * kPitch<KIND>)[t];
                        }
                    }
                }
            }
        }
        }
    };
    heads(std::integral_constant<int, 0>{});
    heads(std::integral_constant<int, 1>{});
    heads(std::integral_constant<int, 2>{});
}

// Heads at a time: their loads are on their way together, and for values there is one wait of the workgroup instead of one for each (8 x 8192 tokens of 8 heads of 64, 8 bits:
// one at a time 91 us, four 86, before results streamed past the caches).
template <int KIND, bool VEC, int G, bool FAST>
__global__ void __launch_bounds__(1024) cache_read(StoreArgs a)
{
    using T = Stored<KIND>;
    typedef T Quad __attribute__((ext_vector_type(4)));
    constexpr int B = cache_bytes(KIND);
    const At at(a);
    if (at.page < 0 || at.lo >= at.hi) return;                 // (the whole workgroup)
    const bool kept = at.tok >= at.lo && at.tok < at.hi;
    const int lo_item = a.by_parts.div(at.part * a.items), hi_item = a.by_parts.div((at.part + 1) * a.items);
    const int D = a.c.D, P = 1 << a.c.shift, i = max(0, min(at.i, a.S - 1)), pitch = D * kPitch<KIND>;
    const unsigned k_at = lane_offset(a.r.by_Cb, a.ks, i, at.d), v_at = lane_offset(a.r.by_Cb, a.vs, i, at.d);
    // items: heads of keys, then heads of values
    for (int item = lo_item; item < hi_item;) {
        const bool is_k = item < a.c.kv_heads;
        const int head = is_k ? item : item - a.c.kv_heads, count = min(G, (is_k ? min(hi_item, a.c.kv_heads) : hi_item) - item);
        Quad q[G] = {};
        if (is_k) {
#pragma unroll
            for (int u = 0; u < G; ++u)
                if (u < count && kept && at.d < a.c.Dk)
                    q[u] = *reinterpret_cast<const Quad *>(a.c.keys + ((place_at(a.c, at.page, head + u, at.place) + at.tok) * a.c.Dk + at.d) * B);
        } else {
            lds_barrier();                                     // (what the heads before put there has been read)
            for (int e = threadIdx.x; e < D * B; e += blockDim.x) {
                const int ch = e / B, piece = e % B;
                int4 x[G];
#pragma unroll
                for (int u = 0; u < G; ++u)
                    x[u] = *reinterpret_cast<const int4 *>(a.c.values + (place_at(a.c, at.page, head + min(u, count - 1), 0) * D + (size_t)ch * P + at.place) * B + 16 * piece);
#pragma unroll
                for (int u = 0; u < G; ++u)
                    if (u < count) *reinterpret_cast<Words4 *>(store_lds + u * pitch + ch * kPitch<KIND> + 16 * piece) = __builtin_bit_cast(Words4, x[u]);
            }
            lds_barrier();
#pragma unroll
            for (int u = 0; u < G; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (u < count && at.d + e < D) q[u][e] = reinterpret_cast<const T *>(store_lds + u * pitch + (at.d + e) * kPitch<KIND>)[at.tok];
        }
        float scale[G];
        if constexpr (KIND == SMALL_CACHE_I8) {
            const float *scales = is_k ? a.c.key_scales : a.c.value_scales;
#pragma unroll
            for (int u = 0; u < G; ++u) scale[u] = kept ? scales[place_at(a.c, at.page, head + min(u, count - 1), at.place) + at.tok] : 0.f;
        }
        TokenStrides s;
        s.image = is_k ? a.ks.image : a.vs.image; s.block = is_k ? a.ks.block : a.vs.block; s.token = is_k ? a.ks.token : a.vs.token;
        float *const image = (is_k ? a.k_out : a.v_out) + at.n * s.image;
#pragma unroll
        for (int u = 0; u < G; ++u) {
            if (u >= count) break;
            floatx4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (float)q[u][e];
            if constexpr (KIND == SMALL_CACHE_I8) x *= scale[u];
            if constexpr (FAST) {
                if (kept && at.d < D) put_quad_at(image + (head + u) * (is_k ? a.k_step : a.v_step), is_k ? k_at : v_at, x);
            } else if (kept) {
                put_quad<VEC>(a.r.by_Cb, D, s, image + i * s.token, (head + u) * D, at.d, x);
            }
        }
        item += count;
    }
}

template <int KIND>
hipError_t write_kind(const StoreArgs &a, bool vec, bool halves, unsigned grid, unsigned threads, hipStream_t s)
{
    const size_t lds = a.tile == 1 ? 0 : (size_t)a.c.D * kPitch<KIND>;
    const bool fast = a.fast && (!halves || a.r.pairs % 4 == 0);
    if (fast && halves) hipLaunchKernelGGL((cache_write<KIND, true, true, true>), dim3(grid), dim3(threads), lds, s, a);
    else if (fast) hipLaunchKernelGGL((cache_write<KIND, true, false, true>), dim3(grid), dim3(threads), lds, s, a);
    else if (vec && halves) hipLaunchKernelGGL((cache_write<KIND, true, true, false>), dim3(grid), dim3(threads), lds, s, a);
    else if (vec) hipLaunchKernelGGL((cache_write<KIND, true, false, false>), dim3(grid), dim3(threads), lds, s, a);
    else if (halves) hipLaunchKernelGGL((cache_write<KIND, false, true, false>), dim3(grid), dim3(threads), lds, s, a);
    else hipLaunchKernelGGL((cache_write<KIND, false, false, false>), dim3(grid), dim3(threads), lds, s, a);
    return hipGetLastError();
}
template <int KIND>
hipError_t read_kind(const StoreArgs &a, bool vec, unsigned grid, unsigned threads, hipStream_t s)
{
    const size_t lds = (size_t)a.c.D * kPitch<KIND>;
    const bool four = 4 * lds <= 65536;                        // (three of 256 floats)
    if (a.fast && four) hipLaunchKernelGGL((cache_read<KIND, true, 4, true>), dim3(grid), dim3(threads), 4 * lds, s, a);
    else if (a.fast) hipLaunchKernelGGL((cache_read<KIND, true, 3, true>), dim3(grid), dim3(threads), 3 * lds, s, a);
    else if (vec) hipLaunchKernelGGL((cache_read<KIND, true, 3, false>), dim3(grid), dim3(threads), 3 * lds, s, a);
    else hipLaunchKernelGGL((cache_read<KIND, false, 3, false>), dim3(grid), dim3(threads), 3 * lds, s, a);
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
