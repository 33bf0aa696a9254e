// Rotary positions: turns of queries and keys, forward and back, and the gradient of learned frequencies (gfx950).
//
// Bound by memory: every channel is read and written once. A thread computes the sines of a token's two or four neighbouring pairs (some 45 operations in 64 bits for
// each) and turns these in all heads that share them, four heads' loads on their way at a time; lanes go along a channel block first and then along
// tokens, so a wave's access is whole lines. Where tokens are few, heads are shared out over threads and sines computed again.
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

template <bool VEC, bool HALVES>
__global__ void __launch_bounds__(256) rotary_turn(RotaryArgs a)
{
    using Unit = Pairs<VEC, HALVES>;
    const unsigned idx = blockIdx.x * 256u + threadIdx.x;
    const unsigned turning = (a.turn_threads + 255u) & ~255u;
    if (idx >= turning) return copy_rest<VEC>(a, idx - turning);
    if (idx >= a.turn_threads) return;
    int rest = a.by_run.div((int)idx);
    const int uq = (int)idx - rest * a.run, above = a.by_S.div(rest), i = rest - above * a.S;
    rest = a.by_runs.div(above);
    const int u = (above - rest * a.runs) * a.run + uq, by_part = a.by_parts.div(rest), part = rest - by_part * a.parts;
    const int n = a.by_freq_heads.div(by_part), f = by_part - n * a.freq_heads;
    int place[4];
    place_of(a, n, i, a.first ? a.first[n] : 0, place);
    Turn t[Unit::kCount];
#pragma unroll
    for (int p = 0; p < Unit::kCount; ++p) t[p] = turn_of(a, place, f, Unit::kCount * u + p);
    const Heads heads(a, f, part);
    for (int j0 = heads.lo; j0 < heads.hi; j0 += 4) {
        Unit x[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int j = min(j0 + b, heads.hi - 1);
            const bool is_q = heads.is_q(j);
            x[b].load(a, is_q ? a.qs : a.ks, token_at(is_q ? a.q : a.k, is_q ? a.qs : a.ks, n, i), heads.head(j) * a.D, u);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int j = j0 + b;
            if (j >= heads.hi) break;
            const bool is_q = heads.is_q(j);
            x[b].turn(t);
            x[b].store(a, is_q ? a.qos : a.kos, const_cast<float *>(token_at(is_q ? a.qo : a.ko, is_q ? a.qos : a.kos, n, i)), heads.head(j) * a.D, u);
        }
    }
}

// The turn back, with the sums over a chunk of tokens for the frequencies' gradient. A workgroup has one run of units of one set of frequencies; run is a power of two.
template <bool VEC, bool HALVES>
__global__ void __launch_bounds__(256) rotary_grad(RotaryArgs a)
{
    using Unit = Pairs<VEC, HALVES>;
    constexpr int P = Unit::kCount;
    __shared__ double sums[4][64];
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
        place_of(a, n, i, a.first ? a.first[n] : 0, place);
        Turn t[P];
#pragma unroll
        for (int p = 0; p < P; ++p) t[p] = turn_of(a, place, f, P * u + p);
        double g[P] = {};
        for (int j0 = heads.lo; j0 < heads.hi; j0 += 2) {
            Unit x[2], y[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int j = min(j0 + b, heads.hi - 1), c0 = heads.head(j) * a.D;
                const bool is_q = heads.is_q(j);
                x[b].load(a, is_q ? a.qs : a.ks, token_at(is_q ? a.q : a.k, is_q ? a.qs : a.ks, n, i), c0, u);
                y[b].load(a, is_q ? a.yqs : a.yks, token_at(is_q ? a.yq : a.yk, is_q ? a.yqs : a.yks, n, i), c0, u);
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int j = j0 + b;
                if (j >= heads.hi) break;
                const bool is_q = heads.is_q(j);
#pragma unroll
                for (int p = 0; p < P; ++p)
                    g[p] += __builtin_fma((double)x[b].x[2 * p + 1], (double)y[b].x[2 * p], -((double)x[b].x[2 * p] * (double)y[b].x[2 * p + 1]));
                x[b].turn(t);
                x[b].store(a, is_q ? a.qos : a.kos, const_cast<float *>(token_at(is_q ? a.qo : a.ko, is_q ? a.qos : a.kos, n, i)), heads.head(j) * a.D, u);
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[p][x] = __builtin_fma((double)place[x], g[p], acc[p][x]);
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const size_t row = ((size_t)f * a.chunks + chunk) * a.parts + part;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (x >= a.axes) break;
            double v = acc[p][x];
            for (int d = 32; d >= a.run; d >>= 1) v += __shfl_xor(v, d);
            __syncthreads();
            sums[wave][lane] = v;
            __syncthreads();
            if ((int)threadIdx.x < a.run) a.partial[(row * a.axes + x) * a.pairs + P * u + p] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
        }
}

// One wave for each frequency: its sums over all chunks.
__global__ void __launch_bounds__(256) rotary_grad_join(const double *partial, float *dfreq, int rows, int each, int all)
{
    const int at = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (at >= all) return;
    const int f = at / each, e = at - f * each;
    double v = 0.0;
#pragma unroll 4
    for (int r = lane; r < rows; r += 64) v += partial[((size_t)f * rows + r) * each + e];
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if (lane == 0) dfreq[at] = (float)v;
}

#define BY_FORM(kernel, grid, vec, halves, s, a)                                                       \
    do {                                                                                               \
        if (vec && halves) hipLaunchKernelGGL((kernel<true, true>), dim3(grid), dim3(256), 0, s, a);   \
        else if (vec) hipLaunchKernelGGL((kernel<true, false>), dim3(grid), dim3(256), 0, s, a);       \
        else if (halves) hipLaunchKernelGGL((kernel<false, true>), dim3(grid), dim3(256), 0, s, a);    \
        else hipLaunchKernelGGL((kernel<false, false>), dim3(grid), dim3(256), 0, s, a);               \
    } while (0)

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, bool vec, bool halves, hipStream_t s)
{
    const unsigned grid = (a.turn_threads + 255u) / 256u + (a.copy_threads + 255u) / 256u;
    BY_FORM(rotary_turn, grid, vec, halves, s, a);
    return hipGetLastError();
}

hipError_t launch_rotary_grad(const RotaryArgs &a, bool vec, bool halves, float *dfreq, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.freq_heads * a.parts * a.runs * a.chunks) + (a.copy_threads + 255u) / 256u;
    BY_FORM(rotary_grad, grid, vec, halves, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int each = a.axes * a.pairs, all = a.freq_heads * each;
    hipLaunchKernelGGL(rotary_grad_join, dim3((unsigned)((all + 3) / 4)), dim3(256), 0, s, a.partial, dfreq, a.chunks * a.parts, each, all);
    return hipGetLastError();
}

}  // namespace small
