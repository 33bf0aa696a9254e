// Group normalization with an activation on the channel-blocked layout, and its gradient (gfx950).
//
// Memory bounds all of it: a value is 8 bytes of traffic forward (12 in the gradient) and some ten operations. So what matters is
// how often a tensor is read. Whole groups lie in units of U = lcm(C/G, Cb) channels, U / Cb planes that stand one behind the other in
// memory. Where a unit fits the registers of one workgroup (65536 values forward, 32768 in the gradient, which holds two
// tensors), that workgroup reads it once, takes sum and squared differences from the registers and writes the result (norm_unit,
// norm_unit_grad: one launch, every value read once). Otherwise statistics of pieces of planes are taken by one launch
// (norm_stats, norm_sums) and joined and applied by the next (norm_apply, norm_apply_grad), which reads the tensors again; many pieces are
// joined by a launch in between (norm_groups).
//
// Measured: 56 x 56 pixels of 256 channels, 64 images, 94 us, 4.4 TB/s (norm_unit, values streamed in and out; a thread with 25 rows in two
// smaller workgroups a compute unit runs out of registers, 101 us); 25 x 5 of 64 channels, 1024 images, 13.5 us, 4.9 TB/s; gradient of
// 57 x 43 pixels of 96 channels, 32 images, with the forward that it needs 57 us; 120 x 120 of 128 channels, 4 images, in pieces 22 us.
//
// A thread holds the same VEC channels throughout and walks over pixels, so the sums of a channel are thread-local until the end.
#include "small_internal.h"
#include "../include/small_attn.h"

namespace small {

namespace {

struct NormArgs {
    const float *x, *gamma, *beta, *dy, *stats_in;
    float *y, *stats;
    float2 *fin;                  // [N][G]: what norm_groups made of them, or null (then every workgroup does that for its groups)
    float2 *part;                 // [N][C/Cb][chunks][Cb]: (mean, M2) or (sum dz, sum dz xhat) of a channel in a piece
    int S, Cb, nCb, C, G, cg, P, U, TP, RP, act, LG, LC, chunks, chunk_rows;
    float eps, inv_n;             // 1 / values of a group
    FastDiv by_cg, by_TP, by_quads, by_units, by_chunks, by_nCb, by_Cb;
};

// z / (1 + exp(-z)) and the logistic function itself. exp(-z) as a power of two whose exponent keeps the bits that the product
// with log2(e) rounds away, so that it is as exact for large |z| as for small ones. Past 2^126 and below 2^-126 there is nothing to keep, and where the product
// overflows nothing to keep it from (infinity less infinity).
__device__ __forceinline__ float logistic(float z)
{
    const float t = z * -1.44269504f, lo = fmaf(z, -1.44269504f, -t) + z * -1.92596303e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return __builtin_amdgcn_rcpf(1.f + (fabsf(t) < 126.f ? fmaf(e, lo * 0.693147181f, e) : e));
}
__device__ __forceinline__ float act_of(float z, int act)
{
    if (act == SMALL_ACT_RELU) return z > 0.f ? z : 0.f;
    if (act == SMALL_ACT_SILU) return z * logistic(z);
    return z;
}
// d act / d z, times dy
__device__ __forceinline__ float act_grad(float z, float dy, int act)
{
    if (act == SMALL_ACT_RELU) return z > 0.f ? dy : 0.f;
    if (act == SMALL_ACT_SILU) {
        const float s = logistic(z);
        return dy * (s * fmaf(z, 1.f - s, 1.f));
    }
    return dy;
}

template <int VEC> struct Vec { float v[VEC]; };
template <int VEC>
__device__ __forceinline__ Vec<VEC> load(const float *p)
{
    Vec<VEC> r;
    if constexpr (VEC == 4) {
        const floatx4 q = *reinterpret_cast<const floatx4 *>(p);
        r.v[0] = q.x; r.v[1] = q.y; r.v[2] = q.z; r.v[3] = q.w;
    } else {
        r.v[0] = *p;
    }
    return r;
}
// One that is read this once.
template <int VEC>
__device__ __forceinline__ Vec<VEC> load_once(const float *p)
{
    if constexpr (VEC == 4) {
        const floatx4 q = __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(p));
        return Vec<VEC>{{q.x, q.y, q.z, q.w}};
    } else {
        return Vec<VEC>{{*p}};
    }
}
// Results stream past the caches, which hold what is read again (57 x 43 pixels of 96 channels, 32 images, forward and gradient 60.7 -> 57.3 us).
template <int VEC>
__device__ __forceinline__ void store(float *p, const Vec<VEC> &r)
{
    if constexpr (VEC == 4)
        __builtin_nontemporal_store(floatx4{r.v[0], r.v[1], r.v[2], r.v[3]}, reinterpret_cast<floatx4 *>(p));
    else
        *p = r.v[0];
}

template <int VEC>
__device__ __forceinline__ void keep(float *lds, const Vec<VEC> &r)
{
#pragma unroll
    for (int i = 0; i < VEC; ++i) lds[i] = r.v[i];
}

// out(i, sum over e < count of f(i, e)) for i < n: `lanes` neighbouring lanes (a power of two, at most 64) for each i. The order of a
// sum depends on the sizes alone. Every lane of the workgroup calls it; the workgroup is a multiple of 64 lanes.
template <typename F, typename O>
__device__ __forceinline__ void segment_sums(int n, int count, int lanes, F f, O out)
{
    const int lane = threadIdx.x & (lanes - 1), per = blockDim.x / lanes;
    for (int i = threadIdx.x / lanes; i < n; i += per) {
        float s = 0.f;
        for (int e = lane; e < count; e += lanes) s += f(i, e);
        for (int d = lanes >> 1; d; d >>= 1) s += __shfl_xor(s, d);
        if (lane == 0) out(i, s);
    }
}

extern __shared__ __attribute__((aligned(16))) float norm_lds[];

// One workgroup, one unit of U channels of one image; K rows of VEC channels in a thread's registers.
// LDS: red[RP][U], then the groups' sums.
template <int VEC, int K>
__global__ void __launch_bounds__(1024) norm_unit(NormArgs a)
{
    float *const red = norm_lds, *const mean_g = red + a.RP * a.U, *const rstd_g = mean_g + a.U / a.cg;
    const int t = threadIdx.x, p = a.by_TP.div(t), u = t - p * a.TP, r0 = a.by_quads.div(u), c = (u - r0 * (int)a.by_quads.d) * VEC;
    const bool on = p < a.P;
    const size_t at = (size_t)blockIdx.x * a.U * a.S + (size_t)p * a.S * a.Cb + c;
    const int groups = a.U / a.cg, cu = p * a.Cb + c;
    Vec<VEC> v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + k * a.RP;
        v[k] = Vec<VEC>{};
        if (on && r < a.S) v[k] = load_once<VEC>(a.x + at + (size_t)r * a.Cb);
    }
    Vec<VEC> s{};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) s.v[i] += v[k].v[i];
    if (on) keep<VEC>(red + r0 * a.U + cu, s);
    __syncthreads();
    const auto of_group = [&](int g, int e) { const int r = a.by_cg.div(e); return red[r * a.U + g * a.cg + (e - r * a.cg)]; };
    segment_sums(groups, a.cg * a.RP, a.LG, of_group, [&](int g, float x) { mean_g[g] = x * a.inv_n; });
    __syncthreads();
    float m[VEC];
    int g[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        g[i] = on ? a.by_cg.div(cu + i) : 0;
        m[i] = mean_g[g[i]];
        s.v[i] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (r0 + k * a.RP < a.S)
#pragma unroll
            for (int i = 0; i < VEC; ++i) { const float d = v[k].v[i] - m[i]; s.v[i] = fmaf(d, d, s.v[i]); }
    if (on) keep<VEC>(red + r0 * a.U + cu, s);
    __syncthreads();
    const int n = a.by_units.div(blockIdx.x), g0 = (blockIdx.x - n * (int)a.by_units.d) * groups;
    segment_sums(groups, a.cg * a.RP, a.LG, of_group, [&](int g, float x) {
        const float rstd = 1.f / sqrtf(fmaf(x, a.inv_n, a.eps));
        rstd_g[g] = rstd;
        if (a.stats) reinterpret_cast<float2 *>(a.stats)[(size_t)n * a.G + g0 + g] = float2{mean_g[g], rstd};
    });
    __syncthreads();
    if (!on) return;
    float ga[VEC], be[VEC];
    const int c_img = g0 * a.cg + cu;
#pragma unroll
    for (int i = 0; i < VEC; ++i) { ga[i] = rstd_g[g[i]] * a.gamma[c_img + i]; be[i] = a.beta[c_img + i]; }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + k * a.RP;
        if (r < a.S) {
            Vec<VEC> y;
#pragma unroll
            for (int i = 0; i < VEC; ++i) y.v[i] = act_of(fmaf(v[k].v[i] - m[i], ga[i], be[i]), a.act);
            store<VEC>(a.y + at + (size_t)r * a.Cb, y);
        }
    }
}

// The gradient of the same unit. LDS: red[2][RP][U], the channels' sums [2][U], the groups' [2][U / cg].
template <int VEC, int K>
__global__ void __launch_bounds__(1024) norm_unit_grad(NormArgs a)
{
    float *const red1 = norm_lds, *const red2 = red1 + a.RP * a.U, *const ch1 = red2 + a.RP * a.U, *const ch2 = ch1 + a.U;
    float *const gr1 = ch2 + a.U, *const gr2 = gr1 + a.U / a.cg;
    const int t = threadIdx.x, p = a.by_TP.div(t), u = t - p * a.TP, r0 = a.by_quads.div(u), c = (u - r0 * (int)a.by_quads.d) * VEC;
    const bool on = p < a.P;
    const size_t at = (size_t)blockIdx.x * a.U * a.S + (size_t)p * a.S * a.Cb + c;
    const int groups = a.U / a.cg, cu = p * a.Cb + c;
    const int n = a.by_units.div(blockIdx.x), g0 = (blockIdx.x - n * (int)a.by_units.d) * groups, c_img = g0 * a.cg + cu;
    Vec<VEC> v[K], d[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + k * a.RP;
        v[k] = Vec<VEC>{};
        d[k] = Vec<VEC>{};
        if (on && r < a.S) {
            v[k] = load<VEC>(a.x + at + (size_t)r * a.Cb);
            d[k] = load<VEC>(a.dy + at + (size_t)r * a.Cb);
        }
    }
    float m[VEC], rs[VEC], ga[VEC], be[VEC];
    int g[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        g[i] = on ? a.by_cg.div(cu + i) : 0;
        const float2 st = reinterpret_cast<const float2 *>(a.stats_in)[(size_t)n * a.G + g0 + g[i]];
        m[i] = st.x; rs[i] = st.y;
        ga[i] = on ? a.gamma[c_img + i] : 0.f;
        be[i] = on ? a.beta[c_img + i] : 0.f;
    }
    Vec<VEC> s1{}, s2{};
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (on && r0 + k * a.RP < a.S)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xh = (v[k].v[i] - m[i]) * rs[i], dz = act_grad(fmaf(xh, ga[i], be[i]), d[k].v[i], a.act);
                v[k].v[i] = xh; d[k].v[i] = dz;
                s1.v[i] += dz;
                s2.v[i] = fmaf(dz, xh, s2.v[i]);
            }
    if (on) {
        keep<VEC>(red1 + r0 * a.U + cu, s1);
        keep<VEC>(red2 + r0 * a.U + cu, s2);
    }
    __syncthreads();
    // channels, for the parameters' gradients; then groups
    segment_sums(2 * a.U, a.RP, a.LC, [&](int i, int r) { return i < a.U ? red1[r * a.U + i] : red2[r * a.U + i - a.U]; },
                 [&](int i, float x) { ch1[i] = x; });
    __syncthreads();
    if (a.part)
        for (int i = t; i < a.U; i += blockDim.x) a.part[(size_t)blockIdx.x * a.U + i] = float2{ch1[i], ch2[i]};
    segment_sums(2 * groups, a.cg, a.LG, [&](int i, int e) {
        const int second = i >= groups, cc = (i - second * groups) * a.cg + e;
        return (second ? ch2 : ch1)[cc] * a.gamma[g0 * a.cg + cc]; }, [&](int i, float x) { gr1[i] = x * a.inv_n; });
    __syncthreads();
    if (!on) return;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int r = r0 + k * a.RP;
        if (r < a.S) {
            Vec<VEC> y;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                y.v[i] = rs[i] * (fmaf(-v[k].v[i], gr2[g[i]], fmaf(ga[i], d[k].v[i], -gr1[g[i]])));
            store<VEC>(a.y + at + (size_t)r * a.Cb, y);
        }
    }
}

// Which piece of which plane a workgroup of the two-launch form has, and what of it a thread.
struct Piece {
    int plane, chunk, row0, rows, b, r0, c, step;      // step: rows a pass of the workgroup covers
    bool on;
};
template <int VEC>
__device__ __forceinline__ Piece piece_of(const NormArgs &a, int block)
{
    Piece p;
    p.plane = a.by_chunks.div(block);
    p.chunk = block - p.plane * a.chunks;
    p.row0 = p.chunk * a.chunk_rows;
    p.rows = min(a.chunk_rows, a.S - p.row0);
    p.b = p.plane - a.by_nCb.div(p.plane) * a.nCb;
    const int quads = (int)a.by_quads.d;
    p.r0 = a.by_quads.div(threadIdx.x);
    p.c = (threadIdx.x - p.r0 * quads) * VEC;
    p.step = a.RP;
    p.on = p.r0 < a.RP;
    return p;
}

// Mean and sum of squared differences of each channel in a piece. Eight rows at a time are summed and their differences to their own
// mean squared; then the two halves so far are joined: mean of both, and the squares grow by the distance of the means.
template <int VEC>
__global__ void __launch_bounds__(1024) norm_stats(NormArgs a)
{
    const Piece p = piece_of<VEC>(a, blockIdx.x);
    float *const ms = norm_lds, *const sq = ms + a.RP * a.Cb, *const mc = sq + a.RP * a.Cb;
    const float *x = a.x + ((size_t)p.plane * a.S + p.row0) * a.Cb + p.c;
    float n = 0.f, mean[VEC] = {}, m2[VEC] = {};
    constexpr int K = 8;
    for (int r = p.r0; p.on && r < p.rows; r += K * p.step) {
        Vec<VEC> v[K];
        const int left = min(K, (p.rows - r + p.step - 1) / p.step);
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = load<VEC>(x + (size_t)(k < left ? r + k * p.step : r) * a.Cb);
        const float nb = (float)left, inv = 1.f / nb, share = nb / (n + nb);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) s += k < left ? v[k].v[i] : 0.f;
            const float mb = s * inv;
#pragma unroll
            for (int k = 0; k < K; ++k) { const float d = v[k].v[i] - mb; q += k < left ? d * d : 0.f; }
            const float d = mb - mean[i];
            mean[i] = fmaf(d, share, mean[i]);
            m2[i] += fmaf(d * d, n * share, q);
        }
        n += nb;
    }
    if (p.on)
#pragma unroll
        for (int i = 0; i < VEC; ++i) { ms[p.r0 * a.Cb + p.c + i] = mean[i]; sq[p.r0 * a.Cb + p.c + i] = m2[i]; }
    __syncthreads();
    const int rows = min(a.RP, p.rows);
    const float inv = 1.f / (float)p.rows;
    const auto count = [&](int r) { return (float)((p.rows - r + p.step - 1) / p.step); };
    segment_sums(a.Cb, rows, a.LC, [&](int c, int r) { return count(r) * ms[r * a.Cb + c]; }, [&](int c, float s) { mc[c] = s * inv; });
    __syncthreads();
    float2 *const out = a.part + (size_t)blockIdx.x * a.Cb;
    segment_sums(a.Cb, rows, a.LC, [&](int c, int r) { const float d = ms[r * a.Cb + c] - mc[c]; return fmaf(count(r) * d, d, sq[r * a.Cb + c]); },
                 [&](int c, float s) { out[c] = float2{mc[c], s}; });
}

// The entry e of a group's channels x pieces, for the groups g0 .. that a plane's channels belong to.
struct GroupEntry { size_t at; int chunk, c; };
__device__ __forceinline__ GroupEntry group_entry(const NormArgs &a, int image, int g, int e)
{
    const int k = a.by_cg.div(e), c = g * a.cg + (e - k * a.cg), b = a.by_Cb.div(c);
    return GroupEntry{(((size_t)image * a.nCb + b) * a.chunks + k) * a.Cb + (c - b * a.Cb), k, c};
}

// Mean and rstd of the groups g0 .. g0 + groups - 1 of an image from their channels' statistics in all pieces: the mean of means, then the squares around it.
// The entries are asked for once where a lane has four at most.
template <typename Out>
__device__ __forceinline__ void group_moments(const NormArgs &a, int image, int g0, int groups, Out out)
{
    const int lane = threadIdx.x & (a.LG - 1), per = blockDim.x / a.LG, entries = a.cg * a.chunks;
    const auto count = [&](int k) { return (float)min(a.chunk_rows, a.S - k * a.chunk_rows); };
    for (int g = threadIdx.x / a.LG; g < groups; g += per) {
        float2 w[4];
        float n[4], s = 0.f, q = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = lane + k * a.LG;
            const GroupEntry x = group_entry(a, image, g0 + g, min(e, entries - 1));
            w[k] = a.part[x.at];
            n[k] = e < entries ? count(x.chunk) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) s = fmaf(n[k], w[k].x, s);
        for (int e = lane + 4 * a.LG; e < entries; e += a.LG) {
            const GroupEntry x = group_entry(a, image, g0 + g, e);
            s = fmaf(count(x.chunk), a.part[x.at].x, s);
        }
        for (int d = a.LG >> 1; d; d >>= 1) s += __shfl_xor(s, d);
        const float mean = s * a.inv_n;
#pragma unroll
        for (int k = 0; k < 4; ++k) { const float d = w[k].x - mean; q += n[k] == 0.f ? 0.f : fmaf(n[k] * d, d, w[k].y); }
        for (int e = lane + 4 * a.LG; e < entries; e += a.LG) {
            const GroupEntry x = group_entry(a, image, g0 + g, e);
            const float d = a.part[x.at].x - mean;
            q += fmaf(count(x.chunk) * d, d, a.part[x.at].y);
        }
        for (int d = a.LG >> 1; d; d >>= 1) q += __shfl_xor(q, d);
        if (lane == 0) out(g, mean, 1.f / sqrtf(fmaf(q, a.inv_n, a.eps)));
    }
}

// The sums of gamma dz and gamma dz xhat over a group, divided by its values.
template <typename Out>
__device__ __forceinline__ void group_sums(const NormArgs &a, int image, int g0, int groups, Out out)
{
    const int lane = threadIdx.x & (a.LG - 1), per = blockDim.x / a.LG, entries = a.cg * a.chunks;
    for (int g = threadIdx.x / a.LG; g < groups; g += per) {
        float s = 0.f, q = 0.f;
#pragma unroll 4
        for (int e = lane; e < entries; e += a.LG) {
            const GroupEntry x = group_entry(a, image, g0 + g, e);
            const float2 w = a.part[x.at];
            const float ga = a.gamma[x.c];
            s = fmaf(w.x, ga, s);
            q = fmaf(w.y, ga, q);
        }
        for (int d = a.LG >> 1; d; d >>= 1) { s += __shfl_xor(s, d); q += __shfl_xor(q, d); }
        if (lane == 0) out(g, s * a.inv_n, q * a.inv_n);
    }
}

// Either of these once for every group, in a launch of its own, where the pieces' workgroups would read too much for theirs. A wave a group (LG = 64).
template <bool GRAD>
__global__ void __launch_bounds__(256) norm_groups(NormArgs a, unsigned count)
{
    const unsigned id = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= count) return;
    const int image = (int)(id / (unsigned)a.G), g0 = (int)(id - (unsigned)image * a.G) - (threadIdx.x >> 6);       // (group_*: group threadIdx.x / 64 from g0 on)
    if constexpr (GRAD) group_sums(a, image, g0, (threadIdx.x >> 6) + 1, [&](int, float s, float q) { a.fin[id] = float2{s, q}; });
    else
        group_moments(a, image, g0, (threadIdx.x >> 6) + 1, [&](int, float mean, float rstd) {
            a.fin[id] = float2{mean, rstd};
            if (a.stats) reinterpret_cast<float2 *>(a.stats)[id] = float2{mean, rstd};
        });
}

// Rows of a piece that a thread asks for before it knows the statistics.
constexpr int kEarly = 4;

template <int VEC>
__global__ void __launch_bounds__(1024) norm_apply(NormArgs a)
{
    const unsigned block = gridDim.x - 1 - blockIdx.x;       // the pieces that norm_stats read last may still be in a cache
    const Piece p = piece_of<VEC>(a, (int)block);
    const size_t at = ((size_t)p.plane * a.S + p.row0) * a.Cb + p.c;
    Vec<VEC> early[kEarly];
#pragma unroll
    for (int k = 0; k < kEarly; ++k)
        if (p.on && p.r0 + k * p.step < p.rows) early[k] = load<VEC>(a.x + at + (size_t)(p.r0 + k * p.step) * a.Cb);
    const int image = a.by_nCb.div(p.plane), g0 = a.by_cg.div(p.b * a.Cb), groups = a.by_cg.div(p.b * a.Cb + a.Cb - 1) - g0 + 1;
    float *const mean_g = norm_lds, *const rstd_g = mean_g + groups;
    if (a.fin) {
        for (int g = threadIdx.x; g < groups; g += blockDim.x) {
            const float2 w = a.fin[(size_t)image * a.G + g0 + g];
            mean_g[g] = w.x;
            rstd_g[g] = w.y;
        }
    } else group_moments(a, image, g0, groups, [&](int g, float mean, float rstd) {
        mean_g[g] = mean;
        rstd_g[g] = rstd;
        // the piece that holds the group's first channel writes its statistics
        if (a.stats && p.chunk == 0 && (g0 + g) * a.cg >= p.b * a.Cb)
            reinterpret_cast<float2 *>(a.stats)[(size_t)image * a.G + g0 + g] = float2{mean, rstd};
    });
    __syncthreads();
    if (!p.on) return;
    float m[VEC], ga[VEC], be[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int c = p.b * a.Cb + p.c + i, g = a.by_cg.div(c) - g0;
        m[i] = mean_g[g]; ga[i] = rstd_g[g] * a.gamma[c]; be[i] = a.beta[c];
    }
    const auto apply = [&](int r, const Vec<VEC> &v) {
        Vec<VEC> y;
#pragma unroll
        for (int i = 0; i < VEC; ++i) y.v[i] = act_of(fmaf(v.v[i] - m[i], ga[i], be[i]), a.act);
        store<VEC>(a.y + at + (size_t)r * a.Cb, y);
    };
#pragma unroll
    for (int k = 0; k < kEarly; ++k)
        if (p.r0 + k * p.step < p.rows) apply(p.r0 + k * p.step, early[k]);
#pragma unroll 4
    for (int r = p.r0 + kEarly * p.step; r < p.rows; r += p.step) apply(r, load<VEC>(a.x + at + (size_t)r * a.Cb));
}

// What both gradient kernels need of a channel.
template <int VEC>
struct ChannelParams {
    float m[VEC], rs[VEC], ga[VEC], be[VEC];
    __device__ __forceinline__ ChannelParams(const NormArgs &a, const Piece &p, int image)
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = p.b * a.Cb + p.c + i;
            const float2 st = reinterpret_cast<const float2 *>(a.stats_in)[(size_t)image * a.G + a.by_cg.div(c)];
            m[i] = st.x; rs[i] = st.y; ga[i] = a.gamma[c]; be[i] = a.beta[c];
        }
    }
};

template <int VEC>
__global__ void __launch_bounds__(1024) norm_sums(NormArgs a)
{
    const Piece p = piece_of<VEC>(a, blockIdx.x);
    float *const red1 = norm_lds, *const red2 = red1 + a.RP * a.Cb, *const ch1 = red2 + a.RP * a.Cb;
    if (p.on) {
        const ChannelParams<VEC> w(a, p, a.by_nCb.div(p.plane));
        const size_t at = ((size_t)p.plane * a.S + p.row0) * a.Cb + p.c;
        Vec<VEC> s1{}, s2{};
#pragma unroll 4
        for (int r = p.r0; r < p.rows; r += p.step) {
            const Vec<VEC> v = load<VEC>(a.x + at + (size_t)r * a.Cb), d = load<VEC>(a.dy + at + (size_t)r * a.Cb);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float xh = (v.v[i] - w.m[i]) * w.rs[i], dz = act_grad(fmaf(xh, w.ga[i], w.be[i]), d.v[i], a.act);
                s1.v[i] += dz;
                s2.v[i] = fmaf(dz, xh, s2.v[i]);
            }
        }
        keep<VEC>(red1 + p.r0 * a.Cb + p.c, s1);
        keep<VEC>(red2 + p.r0 * a.Cb + p.c, s2);
    }
    __syncthreads();
    segment_sums(2 * a.Cb, a.RP, a.LC, [&](int i, int r) { return i < a.Cb ? red1[r * a.Cb + i] : red2[r * a.Cb + i - a.Cb]; },
                 [&](int i, float s) { ch1[i] = s; });
    __syncthreads();
    for (int c = threadIdx.x; c < a.Cb; c += blockDim.x) a.part[(size_t)blockIdx.x * a.Cb + c] = float2{ch1[c], ch1[a.Cb + c]};
}

template <int VEC>
__global__ void __launch_bounds__(1024) norm_apply_grad(NormArgs a)
{
    const unsigned block = gridDim.x - 1 - blockIdx.x;
    const Piece p = piece_of<VEC>(a, (int)block);
    const size_t at = ((size_t)p.plane * a.S + p.row0) * a.Cb + p.c;
    Vec<VEC> early_x[kEarly], early_d[kEarly];
#pragma unroll
    for (int k = 0; k < kEarly; ++k)
        if (p.on && p.r0 + k * p.step < p.rows) {
            early_x[k] = load<VEC>(a.x + at + (size_t)(p.r0 + k * p.step) * a.Cb);
            early_d[k] = load<VEC>(a.dy + at + (size_t)(p.r0 + k * p.step) * a.Cb);
        }
    const int image = a.by_nCb.div(p.plane), g0 = a.by_cg.div(p.b * a.Cb), groups = a.by_cg.div(p.b * a.Cb + a.Cb - 1) - g0 + 1;
    float *const gr = norm_lds;
    if (a.fin) {
        for (int g = threadIdx.x; g < groups; g += blockDim.x) {
            const float2 w = a.fin[(size_t)image * a.G + g0 + g];
            gr[g] = w.x;
            gr[groups + g] = w.y;
        }
    } else group_sums(a, image, g0, groups, [&](int g, float s, float q) { gr[g] = s; gr[groups + g] = q; });
    __syncthreads();
    if (!p.on) return;
    const ChannelParams<VEC> w(a, p, image);
    float s1[VEC], s2[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int g = a.by_cg.div(p.b * a.Cb + p.c + i) - g0;
        s1[i] = gr[g]; s2[i] = gr[groups + g];
    }
    const auto apply = [&](int r, const Vec<VEC> &v, const Vec<VEC> &d) {
        Vec<VEC> y;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float xh = (v.v[i] - w.m[i]) * w.rs[i], dz = act_grad(fmaf(xh, w.ga[i], w.be[i]), d.v[i], a.act);
            y.v[i] = w.rs[i] * fmaf(-xh, s2[i], fmaf(w.ga[i], dz, -s1[i]));
        }
        store<VEC>(a.y + at + (size_t)r * a.Cb, y);
    };
#pragma unroll
    for (int k = 0; k < kEarly; ++k)
        if (p.r0 + k * p.step < p.rows) apply(p.r0 + k * p.step, early_x[k], early_d[k]);
#pragma unroll 4
    for (int r = p.r0 + kEarly * p.step; r < p.rows; r += p.step)
        apply(r, load<VEC>(a.x + at + (size_t)r * a.Cb), load<VEC>(a.dy + at + (size_t)r * a.Cb));
}

// dbeta, dgamma: the channels' sums over images and pieces. 16 channels a workgroup, 64 slices of the (image, piece) pairs.
__global__ void __launch_bounds__(1024) norm_params(const float2 *part, float *dgamma, float *dbeta, int N, int C, FastDiv by_Cb, int chunks, FastDiv by_chunks)
{
    __shared__ float2 red[64][16];
    const int lane = threadIdx.x & 15, slice = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
    float2 s{0.f, 0.f};
    if (c < C) {
        const int Cb = (int)by_Cb.d, b = by_Cb.div(c), col = c - b * Cb;
#pragma unroll 4
        for (int e = slice; e < N * chunks; e += 64) {
            const int n = by_chunks.div(e), k = e - n * chunks;
            const float2 w = part[(((size_t)n * (C / Cb) + b) * chunks + k) * Cb + col];
            s.x += w.x; s.y += w.y;
        }
    }
    red[slice][lane] = s;
    for (int d = 32; d; d >>= 1) {
        __syncthreads();
        if (slice < d) { red[slice][lane].x += red[slice + d][lane].x; red[slice][lane].y += red[slice + d][lane].y; }
    }
    if (slice == 0 && c < C) { dbeta[c] = red[0][lane].x; dgamma[c] = red[0][lane].y; }
}

int pow2_at_most(int v, int most)
{
    int p = 1;
    while (2 * p <= v && 2 * p <= most) p *= 2;
    return p;
}

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

int round_up(int v, int m) { return (v + m - 1) / m * m; }

void chunks_of(int N, int C, int S, int Cb, int *chunks, int *rows)
{
    // some 512 workgroups (two a compute unit), pieces of 16 KB at least. With 2048 the sums of the pieces cost more
    // than the fuller device gains: 384 x 384 pixels of 256 channels 234 us, 512 pieces 141, 256 pieces 157
    const long planes = (long)N * (C / Cb), want = (512 + planes - 1) / planes;
    const long least = (4096 + Cb - 1) / Cb, each = (S + want - 1) / want;
    *rows = (int)(each > least ? each : least < S ? least : S);
    *chunks = (S + *rows - 1) / *rows;
}

template <int VEC>
hipError_t unit_launch(const NormArgs &a, bool grad, int K, unsigned units, int T, size_t lds, hipStream_t s)
{
#define UNIT(k) \
    if (K <= k) { \
        if (grad) hipLaunchKernelGGL((norm_unit_grad<VEC, k>), dim3(units), dim3(T), lds, s, a); \
        else hipLaunchKernelGGL((norm_unit<VEC, k>), dim3(units), dim3(T), lds, s, a); \
        return hipGetLastError(); \
    }
    UNIT(1) UNIT(2) UNIT(4) UNIT(8)
#undef UNIT
    if (!grad && K <= 16) { hipLaunchKernelGGL((norm_unit<VEC, 16>), dim3(units), dim3(T), lds, s, a); return hipGetLastError(); }
    return hipErrorInvalidValue;
}

template <int VEC>
hipError_t norm(NormArgs a, bool grad, int N, float *dgamma, float *dbeta, float2 *ws, hipStream_t s)
{
    const int quads = a.Cb / VEC;
    a.by_cg = make_fastdiv(a.cg);
    a.by_quads = make_fastdiv(quads);
    a.by_nCb = make_fastdiv(a.nCb);
    a.by_Cb = make_fastdiv(a.Cb);
    a.inv_n = (float)(1.0 / ((double)a.cg * a.S));
    const long U = (long)a.cg / gcd(a.cg, a.Cb) * a.Cb;       // at most C
    a.U = (int)U;
    a.P = a.U / a.Cb;
    // ---- one launch, if the unit fits a workgroup's registers and its planes the workgroup's threads
    const int most = grad ? 8 : 16;
    const long vecs = U / VEC * a.S;
    const unsigned units = (unsigned)((long)N * (a.C / a.U));
    if (a.P * quads <= 1024 && U <= 2048 && vecs <= 1024L * most) {       // (2048 channels: 64 KB of LDS for their sums)
        // few units: as many threads as there are values, for latency; many: eight rows a thread, so that several workgroups share a unit
        long T = units < 2 * (unsigned)device_cus() ? vecs : (vecs + 7) / 8;
        T = T < 64 ? 64 : T > 1024 ? 1024 : T;
        const int least = a.P * quads;
        if (T < least) T = least;
        for (; T <= 1024; T = T < 512 ? T * 2 : T < 1024 ? 1024 : 1025) {
            a.TP = (int)T / a.P / quads * quads;
            a.RP = a.TP / quads;
            if (a.RP > a.S) { a.RP = a.S; a.TP = a.RP * quads; }
            const int K = (a.S + a.RP - 1) / a.RP;
            if (K > most) continue;
            const int threads = round_up(a.P * a.TP, 64);
            const int groups = a.U / a.cg;
            a.by_TP = make_fastdiv(a.TP);
            a.by_units = make_fastdiv(a.C / a.U);
            a.LC = pow2_at_most(threads / (2 * a.U) > 0 ? threads / (2 * a.U) : 1, 64);
            const int gr = grad ? 2 * groups : groups;
            a.LG = pow2_at_most(threads / gr > 0 ? threads / gr : 1, 64);
            const size_t lds = sizeof(float) * (grad ? 2 * ((size_t)a.RP * a.U + a.U + groups) : (size_t)a.RP * a.U + 2 * groups);
            a.part = grad && dgamma ? ws : nullptr;
            a.chunks = 1;
            hipError_t e = unit_launch<VEC>(a, grad, K, units, threads, lds, s);
            if (e != hipSuccess || !a.part) return e;
            hipLaunchKernelGGL(norm_params, dim3((a.C + 15) / 16), dim3(1024), 0, s, ws, dgamma, dbeta, N, a.C, a.by_Cb, 1, make_fastdiv(1));
            return hipGetLastError();
        }
    }
    // ---- two launches over pieces of planes
    chunks_of(N, a.C, a.S, a.Cb, &a.chunks, &a.chunk_rows);
    a.by_chunks = make_fastdiv(a.chunks);
    a.part = ws;
    const int T = quads <= 256 ? 256 : round_up(quads, 64);
    a.RP = T / quads;
    a.LC = pow2_at_most(T / a.Cb > 0 ? T / a.Cb : 1, 64);
    const unsigned grid = (unsigned)((long)N * a.nCb * a.chunks);
    const int touched = (a.Cb + a.cg - 2) / a.cg + 1 < a.Cb ? (a.Cb + a.cg - 2) / a.cg + 1 : a.Cb;   // groups in a plane, at most
    const size_t rows_lds = sizeof(float) * 2 * ((size_t)a.RP * a.Cb + a.Cb), group_lds = sizeof(float) * 2 * touched;
    a.LG = pow2_at_most(T / touched > 0 ? T / touched : 1, 64);
    // a workgroup that joins its groups' pieces itself reads them from the caches; past some 4 KB that takes longer than a launch for all groups
    const bool apart = (long)touched * a.cg * a.chunks > 512;
    if (apart) a.fin = ws + (size_t)N * a.C * a.chunks;
    const auto groups = [&]() -> hipError_t {
        if (!apart) return hipSuccess;
        NormArgs b = a;
        b.LG = 64;
        const unsigned count = (unsigned)((long)N * a.G);
        if (grad) hipLaunchKernelGGL((norm_groups<true>), dim3((count + 3) / 4), dim3(256), 0, s, b, count);
        else hipLaunchKernelGGL((norm_groups<false>), dim3((count + 3) / 4), dim3(256), 0, s, b, count);
        return hipGetLastError();
    };
    if (grad) {
        hipLaunchKernelGGL((norm_sums<VEC>), dim3(grid), dim3(T), rows_lds, s, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (hipError_t e = groups(); e != hipSuccess) return e;
        hipLaunchKernelGGL((norm_apply_grad<VEC>), dim3(grid), dim3(T), group_lds, s, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess || !dgamma) return e;
        hipLaunchKernelGGL(norm_params, dim3((a.C + 15) / 16), dim3(1024), 0, s, ws, dgamma, dbeta, N, a.C, a.by_Cb, a.chunks, a.by_chunks);
    } else {
        hipLaunchKernelGGL((norm_stats<VEC>), dim3(grid), dim3(T), rows_lds, s, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        if (hipError_t e = groups(); e != hipSuccess) return e;
        hipLaunchKernelGGL((norm_apply<VEC>), dim3(grid), dim3(T), group_lds, s, a);
    }
    return hipGetLastError();
}

}  // namespace

// Bytes for the sums of channels in pieces (the form of several launches has the most) and of groups.
size_t groupnorm_workspace(int N, int C, int S, int G, int Cb)
{
    int chunks, rows;
    chunks_of(N, C, S, Cb, &chunks, &rows);
    return ((size_t)N * C * chunks + (size_t)N * G) * sizeof(float2);
}

hipError_t launch_groupnorm(const float *x, const float *gamma, const float *beta, const float *stats_in, const float *dy, float *y, float *stats,
                            float *dgamma, float *dbeta, int N, int C, int S, int G, float eps, int act, int Cb, void *ws, hipStream_t s)
{
    NormArgs a{};
    a.x = x; a.gamma = gamma; a.beta = beta; a.stats_in = stats_in; a.dy = dy; a.y = y; a.stats = stats;
    a.S = S; a.Cb = Cb; a.nCb = C / Cb; a.C = C; a.G = G; a.cg = C / G; a.eps = eps; a.act = act;
    const bool vec = Cb % 4 == 0 && ((((uintptr_t)x | (uintptr_t)y | (uintptr_t)dy) & 15u) == 0);
    if (vec) return norm<4>(a, dy != nullptr, N, dgamma, dbeta, (float2 *)ws, s);
    return norm<1>(a, dy != nullptr, N, dgamma, dbeta, (float2 *)ws, s);
}

}  // namespace small
