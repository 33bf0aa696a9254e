// Rotary positions: turns of queries and keys, forward and back, and the gradient of learned frequencies (gfx950).
//
// Bound by memory: every channel is read and written once. A thread computes the sines of a token's two or four neighbouring pairs (some 45 operations in 64 bits for
// each) and turns these in all heads that share them, four heads' loads on their way at a time; lanes go along a channel block first and then along
// tokens, so a wave's access is whole lines. Where tokens are few, heads are shared out over threads and sines computed again.
// 14 x 14 pixels of 64 images, 8 heads of 32: 10.8 us, 4.8 TB/s; clips of 16 x 28 x 28 pixels: 24 us, 5.4 TB/s (a large copy: 4.9, one of 64 MB 8.0).
//
// With y = R(t) x, t = sum over axes of place * frequency: dx = R(-t) dy, and dt of a pair is dy1 y0 - dy0 y1, which needs no sine -- or dx1 x0 - dx0 x1, where x is what there is:
// a turn of both leaves their cross product as it is (dx as it was rounded, as y is where that is read). Its sums times the places run in 64 bits
// over a chunk of tokens for each workgroup, whose results a second launch adds up in a fixed order (8 x 8 pixels of 256 images: 12 us and 4; 6 x 999 frames: 10.5 and 2.5).
#include "rotary.h"

namespace small {

namespace {

// Two or four neighbouring pairs of a head, or one where channels do not stand together: x[0] their first channels and x[1] their second ones with HALVES, else
// x[0] pairs one behind the other.
template <bool VEC, bool HALVES>
struct Pairs {
    static constexpr int kCount = VEC ? (HALVES ? 4 : 2) : 1;
    float x[2 * kCount];
    // unit u of the head whose first channel is c0
    __device__ __forceinline__ void load(const RotaryArgs &a, const TokenStrides &s, const float *token, int c0, int u)
    {
        if constexpr (VEC && HALVES) {
            const floatx4 p = *reinterpret_cast<const floatx4 *>(token + channel_of(a.by_Cb, s, c0 + 4 * u));
            const floatx4 q = *reinterpret_cast<const floatx4 *>(token + channel_of(a.by_Cb, s, c0 + a.pairs + 4 * u));
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = p[i]; x[2 * i + 1] = q[i]; }
        } else if constexpr (VEC) {
            const floatx4 p = *reinterpret_cast<const floatx4 *>(token + channel_of(a.by_Cb, s, c0 + 4 * u));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = p[i];
        } else {
            x[0] = token[channel_of(a.by_Cb, s, c0 + (HALVES ? u : 2 * u))];
            x[1] = token[channel_of(a.by_Cb, s, c0 + (HALVES ? a.pairs + u : 2 * u + 1))];
        }
    }
    __device__ __forceinline__ void store(const RotaryArgs &a, const TokenStrides &s, float *token, int c0, int u) const
    {
        if constexpr (VEC && HALVES) {
            *reinterpret_cast<floatx4 *>(token + channel_of(a.by_Cb, s, c0 + 4 * u)) = floatx4{x[0], x[2], x[4], x[6]};
            *reinterpret_cast<floatx4 *>(token + channel_of(a.by_Cb, s, c0 + a.pairs + 4 * u)) = floatx4{x[1], x[3], x[5], x[7]};
        } else if constexpr (VEC) {
            *reinterpret_cast<floatx4 *>(token + channel_of(a.by_Cb, s, c0 + 4 * u)) = floatx4{x[0], x[1], x[2], x[3]};
        } else {
            token[channel_of(a.by_Cb, s, c0 + (HALVES ? u : 2 * u))] = x[0];
            token[channel_of(a.by_Cb, s, c0 + (HALVES ? a.pairs + u : 2 * u + 1))] = x[1];
        }
    }
    // FAST: two offsets of a lane in a tensor (the second with HALVES), and quads at them from a head's place on
    struct Offsets {
        unsigned at[HALVES ? 2 : 1];
        __device__ __forceinline__ Offsets(const RotaryArgs &a, const TokenStrides &s, int n, int i, int u)
        {
            const long long token = n * s.image + i * s.token;
            at[0] = 4u * (unsigned)(token + channel_of(a.by_Cb, s, 4 * u));
            if constexpr (HALVES) at[1] = 4u * (unsigned)(token + channel_of(a.by_Cb, s, a.pairs + 4 * u));
        }
    };
    __device__ __forceinline__ void load_at(const float *head, const Offsets &o)
    {
        if constexpr (VEC && HALVES) {
            const floatx4 p = quad_at(head, o.at[0]), q = quad_at(head, o.at[1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = p[i]; x[2 * i + 1] = q[i]; }
        } else if constexpr (VEC) {
            const floatx4 p = quad_at(head, o.at[0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = p[i];
        }
    }
    __device__ __forceinline__ void store_at(float *head, const Offsets &o) const
    {
        if constexpr (VEC && HALVES) {
            put_quad_at(head, o.at[0], floatx4{x[0], x[2], x[4], x[6]});
            put_quad_at(head, o.at[1], floatx4{x[1], x[3], x[5], x[7]});
        } else if constexpr (VEC) {
            put_quad_at(head, o.at[0], floatx4{x[0], x[1], x[2], x[3]});
        }
    }
    __device__ __forceinline__ void turn(const Turn (&t)[kCount])
    {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const float p = x[2 * i], q = x[2 * i + 1];
            x[2 * i] = first_of(t[i], p, q);
            x[2 * i + 1] = second_of(t[i], p, q);
        }
    }
};

// Heads of frequencies f: first those of queries, then those of keys; part `part` of them.
struct Heads {
    int q0, k0, per_q, lo, hi;
    __device__ __forceinline__ Heads(const RotaryArgs &a, int f, int part)
    {
        per_q = a.q ? a.by_freq_heads.div(a.heads) : 0;
        const int per_k = a.k ? a.by_freq_heads.div(a.kv_heads) : 0;
        q0 = f * per_q;
        k0 = f * per_k;
        lo = a.by_parts.div(part * (per_q + per_k));
        hi = a.by_parts.div((part + 1) * (per_q + per_k));
    }
    __device__ __forceinline__ bool is_q(int j) const { return j < per_q; }
    __device__ __forceinline__ int head(int j) const { return j < per_q ? q0 + j : k0 + j - per_q; }
};

// Channels that do not turn, of tensors that are not turned in place.
template <bool VEC>
__device__ __forceinline__ void copy_rest(const RotaryArgs &a, unsigned idx)
{
    if (idx >= a.copy_threads) return;
    const int rest = a.by_copy_run.div((int)idx);
    const int uq = (int)idx - rest * a.copy_run, above = a.by_S.div(rest), i = rest - above * a.S;
    const int over = a.by_copy_runs.div(above), u = (above - over * a.copy_runs) * a.copy_run + uq;
    const int n = a.by_copy_heads.div(over), h = over - n * (int)a.by_copy_heads.d;
    const int q_heads = a.q && a.q != a.qo ? a.heads : 0;
    const bool is_q = h < q_heads;
    const int c = (is_q ? h : h - q_heads) * a.D + 2 * a.pairs + (VEC ? 4 : 1) * u;
    const float *from = token_at(is_q ? a.q : a.k, is_q ? a.qs : a.ks, n, i) + channel_of(a.by_Cb, is_q ? a.qs : a.ks, c);
    float *to = const_cast<float *>(token_at(is_q ? a.qo : a.ko, is_q ? a.qos : a.kos, n, i)) + channel_of(a.by_Cb, is_q ? a.qos : a.kos, c);
    if constexpr (VEC) *reinterpret_cast<floatx4 *>(to) = *reinterpret_cast<const floatx4 *>(from);
    else *to = *from;
}

// A workgroup has one set of heads (part of those of one set of frequencies), a thread a unit of a token.
template <bool VEC, bool HALVES, bool FAST>
__global__ void __launch_bounds__(256) rotary_turn(RotaryArgs a)
{
    using Unit = Pairs<VEC, HALVES>;
    constexpr int G = HALVES ? 4 : 8;                                // heads at a time
    const unsigned sets = (unsigned)(a.freq_heads * a.parts), turning = (a.turn_threads + 255u) / 256u * sets;
    if (blockIdx.x >= turning) return copy_rest<VEC>(a, (blockIdx.x - turning) * 256u + threadIdx.x);
    const int group = a.by_sets.div((int)blockIdx.x), set = (int)blockIdx.x - group * (int)sets, f = a.by_parts.div(set), part = set - f * a.parts;
    const unsigned idx = (unsigned)group * 256u + threadIdx.x;
    if (idx >= a.turn_threads) return;
    int rest = a.by_run.div((int)idx);
    const int uq = (int)idx - rest * a.run, above = a.by_S.div(rest), i = rest - above * a.S;
    const int n = a.by_runs.div(above), u = (above - n * a.runs) * a.run + uq;
    const Heads heads(a, f, part);
    int place[4];
    Turn t[Unit::kCount];
    const auto turns = [&] {
        place_of(a, n, i, a.first ? a.first[n] : 0, place);
#pragma unroll
        for (int p = 0; p < Unit::kCount; ++p) t[p] = turn_of(a, place, f, Unit::kCount * u + p);
    };
    bool turned = false;
    // queries, then keys
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
        const int lo = tensor ? max(heads.lo, heads.per_q) : heads.lo, hi = tensor ? heads.hi : min(heads.hi, heads.per_q);
        if (lo >= hi) continue;
        const float *const from = tensor ? a.k : a.q;
        float *const to = tensor ? a.ko : a.qo;
        const TokenStrides &fs = tensor ? a.ks : a.qs, &ts = tensor ? a.kos : a.qos;
        const typename Unit::Offsets fo(a, fs, n, i, u), so(a, ts, n, i, u);
        const float *const token = token_at(from, fs, n, i);
        float *const token_out = const_cast<float *>(token_at(to, ts, n, i));
        for (int j0 = lo; j0 < hi; j0 += G) {
            Unit x[G];
#pragma unroll
            for (int b = 0; b < G; ++b) {
                const int h = heads.head(min(j0 + b, hi - 1));
                if constexpr (FAST) x[b].load_at(from + h * (tensor ? a.k_step : a.q_step), fo);
                else x[b].load(a, fs, token, h * a.D, u);
            }
            if (!turned) turns();                                    // (the first loads are on their way)
            turned = true;
#pragma unroll
            for (int b = 0; b < G; ++b) {
                if (j0 + b >= hi) break;
                const int h = heads.head(j0 + b);
                x[b].turn(t);
                if constexpr (FAST) x[b].store_at(to + h * (tensor ? a.ko_step : a.qo_step), so);
                else x[b].store(a, ts, token_out, h * a.D, u);
            }
        }
    }
}

// The turn back, with the sums over a chunk of tokens for the frequencies' gradient. A workgroup has one run of units of one set of frequencies; run is a power of two.
// INPUTS: from_inputs, a form of its own: chosen at run time it takes 16 to 29 registers more, and with them a wave a SIMD.
template <bool VEC, bool HALVES, bool FAST, bool INPUTS>
__global__ void __launch_bounds__(256) rotary_grad(RotaryArgs a)
{
    using Unit = Pairs<VEC, HALVES>;
    constexpr int P = Unit::kCount, G = HALVES ? 2 : 4;
    __shared__ double sums[4][4 * P][64];
    const unsigned summing = (unsigned)(a.freq_heads * a.parts * a.runs * a.chunks);
    if (blockIdx.x >= summing) return copy_rest<VEC>(a, (blockIdx.x - summing) * 256u + threadIdx.x);
    const int rest = a.by_chunks.div((int)blockIdx.x);
    const int chunk = (int)blockIdx.x - rest * a.chunks;
    const int above = a.by_runs.div(rest), ub = rest - above * a.runs, f = a.by_parts.div(above), part = above - f * a.parts;
    const int uq = threadIdx.x & (a.run - 1), u = ub * a.run + uq, tokens = 256 / a.run;
    const Heads heads(a, f, part);
    double acc[P][4] = {};
    const int end = min(a.N * a.S, (chunk + 1) * a.per_chunk);
    for (int at = chunk * a.per_chunk + (int)threadIdx.x / a.run; at < end; at += tokens) {
        const int n = a.by_S.div(at), i = at - n * a.S;
        int place[4];
        Turn t[P];
        double g[P] = {};
        bool turned = false;
#pragma unroll
        for (int tensor = 0; tensor < 2; ++tensor) {
            const int lo = tensor ? max(heads.lo, heads.per_q) : heads.lo, hi = tensor ? heads.hi : min(heads.hi, heads.per_q);
            if (lo >= hi) continue;
            const float *const from = tensor ? a.k : a.q, *const saved = tensor ? a.yk : a.yq;
            float *const to = tensor ? a.ko : a.qo;
            const TokenStrides &fs = tensor ? a.ks : a.qs, &ts = tensor ? a.kos : a.qos, &ss = tensor ? a.yks : a.yqs;
            const typename Unit::Offsets fo(a, fs, n, i, u), to_at(a, ts, n, i, u), so(a, ss, n, i, u);
            const float *const token = token_at(from, fs, n, i), *const token_saved = token_at(saved, ss, n, i);
            float *const token_out = const_cast<float *>(token_at(to, ts, n, i));
            for (int j0 = lo; j0 < hi; j0 += G) {
                Unit x[G], y[G];
#pragma unroll
                for (int b = 0; b < G; ++b) {
                    const int h = heads.head(min(j0 + b, hi - 1));
                    if constexpr (FAST) {
                        x[b].load_at(from + h * (tensor ? a.k_step : a.q_step), fo);
                        y[b].load_at(saved + h * (tensor ? a.yk_step : a.yq_step), so);
                    } else {
                        x[b].load(a, fs, token, h * a.D, u);
                        y[b].load(a, ss, token_saved, h * a.D, u);
                    }
                }
                if (!turned) {
                    place_of(a, n, i, a.first ? a.first[n] : 0, place);
#pragma unroll
                    for (int p = 0; p < P; ++p) t[p] = turn_of(a, place, f, P * u + p);
                    turned = true;
                }
#pragma unroll
                for (int b = 0; b < G; ++b) {
                    if (j0 + b >= hi) break;
                    const int h = heads.head(j0 + b);
                    const auto cross = [&] {
#pragma unroll
                        for (int p = 0; p < P; ++p)
                            g[p] += __builtin_fma((double)x[b].x[2 * p + 1], (double)y[b].x[2 * p], -((double)x[b].x[2 * p] * (double)y[b].x[2 * p + 1]));
                    };
                    if constexpr (!INPUTS) cross();
                    x[b].turn(t);
                    if constexpr (INPUTS) cross();
                    if constexpr (FAST) x[b].store_at(to + h * (tensor ? a.ko_step : a.qo_step), to_at);
                    else x[b].store(a, ts, token_out, h * a.D, u);
                }
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int x4 = 0; x4 < 4; ++x4) acc[p][x4] = __builtin_fma((double)place[x4], g[p], acc[p][x4]);
    }
    // the lanes of a unit, the four waves
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (x >= a.axes) break;
            double v = acc[p][x];
            for (int d = 32; d >= a.run; d >>= 1) v += __shfl_xor(v, d);
            if (lane < a.run) sums[wave][p * 4 + x][lane] = v;
        }
    __syncthreads();
    const size_t row = ((size_t)f * a.chunks + chunk) * a.parts + part;
    for (int e = threadIdx.x; e < P * 4 * a.run; e += 256) {
        const int v = e / a.run, at = e - v * a.run, p = v >> 2, x = v & 3;
        if (x < a.axes)
            a.partial[(row * a.axes + x) * a.pairs + P * (ub * a.run + at) + p] = (sums[0][v][at] + sums[1][v][at]) + (sums[2][v][at] + sums[3][v][at]);
    }
}

// One wave for each frequency: its sums over all chunks.
__global__ void __launch_bounds__(256) rotary_grad_join(const double *partial, float *dfreq, int rows, int each, int all)
{
    const int at = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (at >= all) return;
    const int f = at / each, e = at - f * each;
    double v = 0.0;
    for (int r0 = lane; r0 < rows; r0 += 8 * 64) {            // (eight asked for at a time)
        double x[8];
#pragma unroll
        for (int b = 0; b < 8; ++b) x[b] = r0 + 64 * b < rows ? partial[((size_t)f * rows + r0 + 64 * b) * each + e] : 0.0;
#pragma unroll
        for (int b = 0; b < 8; ++b) v += x[b];
    }
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if (lane == 0) dfreq[at] = (float)v;
}

#define BY_FORM(kernel, grid, vec, halves, s, a, ...)                                                                                           \
    do {                                                                                                                                        \
        if (vec && halves && a.fast) hipLaunchKernelGGL((kernel<true, true, true __VA_OPT__(, ) __VA_ARGS__>), dim3(grid), dim3(256), 0, s, a); \
        else if (vec && a.fast) hipLaunchKernelGGL((kernel<true, false, true __VA_OPT__(, ) __VA_ARGS__>), dim3(grid), dim3(256), 0, s, a);     \
        else if (vec && halves) hipLaunchKernelGGL((kernel<true, true, false __VA_OPT__(, ) __VA_ARGS__>), dim3(grid), dim3(256), 0, s, a);     \
        else if (vec) hipLaunchKernelGGL((kernel<true, false, false __VA_OPT__(, ) __VA_ARGS__>), dim3(grid), dim3(256), 0, s, a);              \
        else if (halves) hipLaunchKernelGGL((kernel<false, true, false __VA_OPT__(, ) __VA_ARGS__>), dim3(grid), dim3(256), 0, s, a);           \
        else hipLaunchKernelGGL((kernel<false, false, false __VA_OPT__(, ) __VA_ARGS__>), dim3(grid), dim3(256), 0, s, a);                      \
    } while (0)

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, bool vec, bool halves, hipStream_t s)
{
    const unsigned grid = (a.turn_threads + 255u) / 256u * (unsigned)(a.freq_heads * a.parts) + (a.copy_threads + 255u) / 256u;
    BY_FORM(rotary_turn, grid, vec, halves, s, a);
    return hipGetLastError();
}

hipError_t launch_rotary_grad(const RotaryArgs &a, bool vec, bool halves, bool from_inputs, float *dfreq, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.freq_heads * a.parts * a.runs * a.chunks) + (a.copy_threads + 255u) / 256u;
    if (from_inputs) BY_FORM(rotary_grad, grid, vec, halves, s, a, true);
    else BY_FORM(rotary_grad, grid, vec, halves, s, a, false);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int each = a.axes * a.pairs, all = a.freq_heads * each;
    hipLaunchKernelGGL(rotary_grad_join, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a.partial, dfreq, a.chunks * a.parts, each, all);
    return hipGetLastError();
}

}  // namespace small
