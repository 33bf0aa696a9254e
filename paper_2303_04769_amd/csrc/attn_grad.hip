// Gradients of attention (gfx950). With P = exp(s - lse) taken anew from queries and keys,
//   dV = P^T dO,  dP = dO V^T,  dS = P (dP - delta),  delta = rowsum(dO o),  dbias = dS summed over its bucket,
//   dS *= 1 - tanh^2 (capped scores),  dQ = scale dS K,  dK = scale dS^T Q.
// attn_grad_rows keeps 64 rows and walks over the keys (scores, dP, dQ: three products), attn_grad_keys keeps 64 keys and walks over the
// rows of all query heads on them (scores, dP, dV, dK: four). Seven products instead of the five that one walk would take, but every
// gradient is summed where it stays, in a fixed order, with no atomic additions.
//
// Bound by the fp32 matrix instructions, as the forward kernel, whose tiles and operand layouts these are (attn_tile.h). These kernels have heads of more than 128
// channels and biases whose sums by offset do not fit LDS; attn_parts_grad.hip has all others (10 x 10 pixels, 4 heads of 32, 200 images: 142 us here, 109 there).
#include "attn_tile.h"

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) float grad_lds[];

// A score's way to its probability: capped (returned as tanh, or as the dot product where there is no cap), biased.
__device__ __forceinline__ float score_core(const AttnArgs &a, const Scorer &sc, float dot) { return a.cap > 0.f ? tanh_of(dot * sc.cap_in) : dot; }
__device__ __forceinline__ float score_of(const AttnArgs &a, const Scorer &sc, float core) { return core * (a.cap > 0.f ? sc.cap2 : sc.scale2); }

// What each row's weights are to be multiplied by (share_of), on its own: dq takes that at the end of its walk over the keys, when their sum is known, but the bias's gradient sums
// over rows all along. So with distances and a table's gradient this runs first: scores only, one product of seven (2048 frames with a prefix,
// capped, 8 heads of 64 on 2, 4 sequences: 190 us of some 650 with the forward call; 400 frames, 2 sequences: 21).
template <int DT, int KT, bool VEC>
__global__ void __launch_bounds__(256, 2) attn_grad_shares(AttnArgs a)
{
    constexpr int NB = KT / 16;
    using T = Tile<DT, KT>;
    __shared__ float kt[T::kFloats];
    __shared__ alignas(16) int key_code[KT];
    __shared__ alignas(16) int key_doc[KT + 1];
    __shared__ int words[2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_tile = a.by_tiles.div((int)id), tile = a.row_tiles - 1 - ((int)id - by_tile * a.row_tiles);
    const int n = a.by_heads.div(by_tile), head = by_tile - n * a.heads, key_head = a.by_group.div(head);
    const int row0 = tile * 64, i_raw = row0 + wave * 16 + m, i = min(i_raw, a.Sq - 1);
    const ImageMask im(a, n);
    const RowState row(a, im, n, i, head);
    const float lse = a.lse_in[((size_t)n * a.heads + head) * a.Sq + i];
    const float lse2 = lse == -kInf ? kInf : lse * kLog2e;
    float q[DT * 4];
    {
        const float *token = token_at(a.q, a.qs, n, i);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            const floatx4 x = load_quad<VEC>(a, a.qs, token, head * a.D, 16 * c + 4 * g);
            q[4 * c] = x.x; q[4 * c + 1] = x.y; q[4 * c + 2] = x.z; q[4 * c + 3] = x.w;
        }
    }
    int lo = 0, hi = im.len;
    if (a.causal) hi = max(0, min(hi, max(im.position(min(row0 + 63, a.Sq - 1)) + 1, im.prefix)));
    if (a.docs) {
        if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
        __syncthreads();
        if (row.doc >= 0) { atomicMin(&words[0], row.doc); atomicMax(&words[1], row.doc); }
        __syncthreads();
        const int d0 = words[0], d1 = words[1];
        __syncthreads();
        document_hull(a.docs + (size_t)n * a.Sk, 0, hi, d0, d1, words, &lo, &hi);
    }
    const float *bias = nullptr;
    if (a.bias_lds) {
        expand_bias(a, head, grad_lds);
        bias = grad_lds;
    }
    const float far_lo = bias_gather(a, head, 0), far_hi = bias_gather(a, head, 2 * a.reach);
    floatx4 kx[T::kQuads];
    const auto fetch = [&](int j0) { T::template fetch<VEC>(kx, a, a.ks, a.k, n, key_head * a.D, j0, [&](int j) { return j0 + j < im.len; }); };
    if (lo < hi) fetch(lo);
    float total = 0.f;
    for (int j0 = lo; j0 < hi; j0 += KT) {
        __syncthreads();
        T::put(kt, kx);
        stage_keys<KT>(a, n, j0, key_code, key_doc);
        __syncthreads();
        if (j0 + KT < hi) fetch(j0 + KT);
        floatx4 s[NB] = {};
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const floatx4 x = T::tokens(kt, b, c, m, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[b] = mfma(x[e], q[4 * c + e], s[b]);
            }
        finish_scores<7>(a, s, row, 0, lse2, j0, key_code, key_doc, g, bias, far_lo, far_hi);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) total += __builtin_amdgcn_exp2f(s[b][e]);
    }
    const float share = share_of(a, total);
    if (i_raw < a.Sq && g == 0) a.share[((size_t)n * a.heads + head) * a.Sq + i] = share;
}

template <int DT, int KT, bool VEC>
__global__ void __launch_bounds__(256, DT <= 6 ? 2 : 1) attn_grad_rows(AttnArgs a)
{
    constexpr int VD = kVD<DT>, GR = DT / VD, NB = KT / 16;
    using T = Tile<DT, KT>;
    __shared__ float kt[T::kFloats], vt[T::kFloats];
    __shared__ alignas(16) int key_code[KT];
    __shared__ alignas(16) int key_doc[KT];
    __shared__ int key_bad[KT], any_bad;                          // j0 of a tile in which the key, or any, is bad (put_finite)
    __shared__ int row_code[64], words[2];
    __shared__ float ends[8];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_tile = a.by_tiles.div((int)id), tile = a.row_tiles - 1 - ((int)id - by_tile * a.row_tiles);
    const int n = a.by_heads.div(by_tile), head = by_tile - n * a.heads, key_head = a.by_group.div(head);
    const int row0 = tile * 64, i_raw = row0 + wave * 16 + m, i = min(i_raw, a.Sq - 1);
    const ImageMask im(a, n);
    const RowState row(a, im, n, i, head);
    const size_t at_row = ((size_t)n * a.heads + head) * a.Sq + i;
    // a row that saw nothing has no gradient, and neither has one past the end: weights exp2(-inf)
    const float lse = a.lse_in[at_row];
    const bool dead = lse == -kInf || i_raw >= a.Sq;
    const float lse2 = dead ? kInf : lse * kLog2e;
    floatx4 q[DT], dout[DT];
    float delta = 0.f;
    {
        const float *tq = token_at(a.q, a.qs, n, i), *td = token_at(a.dout, a.dos, n, i), *to = token_at(a.o, a.os, n, i);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            q[c] = load_quad<VEC>(a, a.qs, tq, head * a.D, 16 * c + 4 * g);
            dout[c] = load_quad<VEC>(a, a.dos, td, head * a.D, 16 * c + 4 * g);
            const floatx4 x = load_quad<VEC>(a, a.os, to, head * a.D, 16 * c + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                dout[c][e] = dead ? 0.f : dout[c][e];
                q[c][e] = dead ? 0.f : q[c][e];
                delta = fmaf(dout[c][e], dead ? 0.f : x[e], delta);
            }
        }
        delta = column_sum(delta);
        if (g == 0 && i_raw < a.Sq) a.delta[at_row] = delta;
    }
    if (g == 0) row_code[wave * 16 + m] = row.code;
    if (threadIdx.x < KT) key_bad[threadIdx.x] = -1;              // (a barrier is in front of the first tile)
    if (threadIdx.x == 0) any_bad = -1;

    int lo = 0, hi = im.len;
    if (a.causal) hi = max(0, min(hi, max(im.position(min(row0 + 63, a.Sq - 1)) + 1, im.prefix)));
    if (a.docs) {
        if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
        __syncthreads();
        if (row.doc >= 0) { atomicMin(&words[0], row.doc); atomicMax(&words[1], row.doc); }
        __syncthreads();
        const int d0 = words[0], d1 = words[1];
        __syncthreads();
        document_hull(a.docs + (size_t)n * a.Sk, 0, hi, d0, d1, words, &lo, &hi);
    }

    // LDS behind the tiles: the expanded bias, the gradient's tile [64][KT + 1] and its sums by offset
    const int size = 2 * a.reach + 1;
    float *at_lds = grad_lds;
    const float *bias = nullptr;
    float far_lo = 0.f, far_hi = 0.f;
    if (a.table) {
        if (a.bias_lds) {
            for (int x = threadIdx.x; x < size; x += 256) at_lds[x] = bias_gather(a, head, x);
            bias = at_lds;
            at_lds += size;
        }
        far_lo = bias_gather(a, head, 0);
        far_hi = bias_gather(a, head, 2 * a.reach);
    }
    float *const ds_tile = at_lds;
    float *acc = nullptr, *const part = a.part_bias ? a.part_bias + (((size_t)n * a.heads + head) * a.row_tiles + tile) * size : nullptr;
    if (part) {
        acc = a.bias_acc_lds ? at_lds + 64 * (KT + 1) : part;
        for (int x = threadIdx.x; x < size; x += 256) acc[x] = 0.f;       // (behind the next barrier a place is one thread's until the loop's end)
    }
    float sum_lo = 0.f, sum_hi = 0.f, total = 0.f;
    const float known = a.share_known ? a.share[at_row] : 1.f;

    const Scorer sc(a);
    floatx4 dq[DT] = {};
    floatx4 kx[T::kQuads], vx[T::kQuads];
    const auto fetch = [&](int j0) {
        const auto on = [&](int j) { return j0 + j < im.len; };
        T::template fetch<VEC>(kx, a, a.ks, a.k, n, key_head * a.D, j0, on);
        T::template fetch<VEC>(vx, a, a.vs, a.v, n, key_head * a.D, j0, on);
    };
    if (lo < hi) fetch(lo);
    for (int j0 = lo; j0 < hi; j0 += KT) {
        __syncthreads();
        T::put_finite(kt, kx, key_bad, &any_bad, j0);
        T::put(vt, vx);
        if (threadIdx.x < KT) {
            const int j = j0 + threadIdx.x;
            if (a.table) key_code[threadIdx.x] = code_of(a, j);
            if (a.docs) key_doc[threadIdx.x] = key_document(a, n, j);
        }
        __syncthreads();
        if (j0 + KT < hi) fetch(j0 + KT);

        floatx4 s[NB] = {}, dp[NB] = {};
#pragma unroll
        for (int c = 0; c < DT; ++c)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const floatx4 x = T::tokens(kt, b, c, m, g), y = T::tokens(vt, b, c, m, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[b] = mfma(x[e], q[c][e], s[b]);
                    dp[b] = mfma(y[e], dout[c][e], dp[b]);
                }
            }
        const bool edge = a.docs || !__all(j0 + KT <= row.bound), bad = any_bad == j0;
        const bool all_lo = a.table && __all(key_code[KT - 1] - row.code <= -a.reach), all_hi = a.table && __all(key_code[0] - row.code >= a.reach);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            int docs[4] = {row.doc, row.doc, row.doc, row.doc}, codes[4] = {0, 0, 0, 0};
            if (a.docs) {
                const int4 x = *reinterpret_cast<const int4 *>(key_doc + 16 * b + 4 * g);
                docs[0] = x.x; docs[1] = x.y; docs[2] = x.z; docs[3] = x.w;
            }
            if (a.table) {
                const int4 x = *reinterpret_cast<const int4 *>(key_code + 16 * b + 4 * g);
                codes[0] = x.x; codes[1] = x.y; codes[2] = x.z; codes[3] = x.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = j0 + 16 * b + 4 * g + e;
                const float core = score_core(a, sc, s[b][e]);
                float t = score_of(a, sc, core);
                t += a.slopes ? fmaf(-row.slope, fabsf((float)(row.p - j)), -lse2) : -lse2;       // (large ones cancel unrounded)
                if (a.table) {
                    if (all_lo || all_hi) t += all_lo ? far_lo : far_hi;
                    else {
                        const int at = offset_at(a, codes[e], row.code);
                        t += bias ? bias[at] : bias_gather(a, head, at);
                    }
                }
                if (bad) t = key_bad[16 * b + 4 * g + e] == j0 ? __builtin_nanf("") : t;
                const float p = __builtin_amdgcn_exp2f(t);
                float ds = p * (dp[b][e] - delta) * known;
                const bool seen = !edge | row.sees(j, docs[e], true);
                ds = seen ? ds : 0.f;
                total += seen ? p : 0.f;
                if (part) {
                    const int off = codes[e] - row.code;
                    sum_lo += off <= -a.reach ? ds : 0.f;
                    sum_hi += off >= a.reach && off > -a.reach ? ds : 0.f;
                    if (!all_lo && !all_hi) ds_tile[(wave * 16 + m) * (KT + 1) + 16 * b + 4 * g + e] = ds;
                }
                dp[b][e] = a.cap > 0.f ? ds * fmaf(-core, core, 1.f) : ds;
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int grp = 0; grp < GR; ++grp) {
                    float x[VD];
                    T::template channels<VD>(x, kt, 16 * b + 4 * g + e, grp, m);
#pragma unroll
                    for (int v = 0; v < VD; ++v) dq[grp * VD + v] = mfma(x[v], dp[b][e], dq[grp * VD + v]);
                }
        if (part) {
            // sums by offset of what lies between the ends of the reach: a thread takes the offsets that are its number modulo 256,
            // and looks in every row for the key at that offset
            __syncthreads();
            const int c0 = key_code[0], c1 = key_code[KT - 1];
            const int r0 = max(c0 - row_code[63], -a.reach + 1), r1 = min(c1 - row_code[0], a.reach - 1);
            for (int r = r0 + (((int)threadIdx.x - r0) & 255); r <= r1; r += 256) {
                float x = 0.f;
#pragma unroll 4
                for (int y = 0; y < 64; ++y) {
                    const int o = row_code[y] + r, line = o < 0 ? 0 : a.by_code.div(o), col = o - line * (2 * a.width - 1), j = line * a.width + col - j0;
                    if (o >= 0 && col < a.width && j >= 0 && j < KT) x += ds_tile[y * (KT + 1) + j];
                }
                acc[r + a.reach] += x;
            }
        }
    }
    if (part) {
        sum_lo = wave_sum(sum_lo);
        sum_hi = wave_sum(sum_hi);
        __syncthreads();
        if (lane == 0) { ends[wave] = sum_lo; ends[4 + wave] = sum_hi; }
        __syncthreads();
        for (int x = threadIdx.x; x < size; x += 256) {
            float y = acc[x];
            if (x == 0) y += (ends[0] + ends[1]) + (ends[2] + ends[3]);
            if (x == size - 1) y += (ends[4] + ends[5]) + (ends[6] + ends[7]);
            part[x] = y;
        }
    }
    const float share = a.share_known ? 1.f : share_of(a, total);
    if (i_raw < a.Sq) {
        if (a.slopes && !a.share_known && g == 0) a.share[((size_t)n * a.heads + head) * a.Sq + i] = share;
        float *token = const_cast<float *>(token_at(a.dq, a.dqs, n, i));
#pragma unroll
        for (int grp = 0; grp < GR; ++grp)
#pragma unroll
            for (int x = 0; x < VD; ++x)
                store_quad<VEC>(a, a.dqs, token, head * a.D, grp * 16 * VD + 4 * g * VD + 4 * x, result_quad<DT>(dq, grp, x) * (a.scale * share));
    }
}

template <int DT, int KT, bool VEC>
__global__ void __launch_bounds__(256, DT <= 6 ? 2 : 1) attn_grad_keys(AttnArgs a)
{
    constexpr int VD = kVD<DT>, GR = DT / VD, NB = KT / 16;
    using T = Tile<DT, KT>;
    __shared__ float qt[T::kFloats], dt[T::kFloats];
    __shared__ alignas(16) float row_lse[KT];
    __shared__ alignas(16) float row_delta[KT];
    __shared__ alignas(16) float row_share[KT];
    __shared__ alignas(16) int row_p[KT];
    __shared__ alignas(16) int row_code[KT];
    __shared__ alignas(16) int row_bound[KT];
    __shared__ alignas(16) int row_doc[KT];
    __shared__ int row_bad[KT], any_bad;                          // number of a tile in which the row, or any, is bad (put_finite)
    __shared__ int words[2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const unsigned id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int by_tile = a.by_key_tiles.div((int)id), tile = (int)id - by_tile * a.key_tiles;      // (causal: the first keys have the most rows)
    const int kv = a.heads / a.group, n = by_tile / kv, key_head = by_tile - n * kv;
    const ImageMask im(a, n);
    const int j0 = tile * 64, j_raw = j0 + wave * 16 + m, j = min(j_raw, a.Sk - 1);
    const int code = a.table ? code_of(a, j) : 0, doc = a.docs ? key_document(a, n, j) : -1;
    // a key past the length is not read; nor is one that belongs to no document
    const bool dead = j_raw >= im.len || (a.docs && doc < 0);
    floatx4 k[DT], v[DT];
    {
        const float *tk = token_at(a.k, a.ks, n, j), *tv = token_at(a.v, a.vs, n, j);
#pragma unroll
        for (int c = 0; c < DT; ++c) {
            k[c] = floatx4{0.f, 0.f, 0.f, 0.f};
            v[c] = floatx4{0.f, 0.f, 0.f, 0.f};
            if (!dead) {
                k[c] = load_quad<VEC>(a, a.ks, tk, key_head * a.D, 16 * c + 4 * g);
                v[c] = load_quad<VEC>(a, a.vs, tv, key_head * a.D, 16 * c + 4 * g);
            }
        }
    }
    // rows that can see any of the keys
    int lo = 0, hi = j0 < im.len ? a.Sq : 0;
    if (a.causal && im.prefix <= j0) lo = max(0, min(a.Sq, j0 - im.first));
    if (a.docs) {
        if (threadIdx.x == 0) { words[0] = 0x7fffffff; words[1] = -1; }
        __syncthreads();
        if (!dead) { atomicMin(&words[0], doc); atomicMax(&words[1], doc); }
        __syncthreads();
        const int d0 = words[0], d1 = words[1];
        __syncthreads();
        int begin, end;
        const int p0 = max(0, min(im.first + lo, a.Sk)), p1 = max(p0, min(im.first + hi, a.Sk));
        document_hull(a.docs + (size_t)n * a.Sk, p0, p1, d0, d1, words, &begin, &end);
        lo = begin - im.first;
        hi = end - im.first;
    }
    const int size = 2 * a.reach + 1;
    const Scorer sc(a);
    if (threadIdx.x < KT) row_bad[threadIdx.x] = -1;              // (a barrier is in front of the first tile)
    if (threadIdx.x == 0) any_bad = -1;
    int number = 0;
    floatx4 dk[DT] = {}, dv[DT] = {};
    floatx4 qx[T::kQuads], dx[T::kQuads];
    for (int head = key_head * a.group; head < (key_head + 1) * a.group && lo < hi; ++head) {
        const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.f;
        const float *bias = nullptr;
        float far_lo = 0.f, far_hi = 0.f;
        if (a.table) {
            if (a.bias_lds) {
                __syncthreads();                                                    // (the last head's is still read)
                for (int x = threadIdx.x; x < size; x += 256) grad_lds[x] = bias_gather(a, head, x);
                bias = grad_lds;
            }
            far_lo = bias_gather(a, head, 0);
            far_hi = bias_gather(a, head, 2 * a.reach);
        }
        const float *lse_in = a.lse_in + ((size_t)n * a.heads + head) * a.Sq, *delta_in = a.delta + ((size_t)n * a.heads + head) * a.Sq,
                    *share_in = a.share + ((size_t)n * a.heads + head) * a.Sq;
        const auto fetch = [&](int i0) {
            // (rows that saw nothing are not read either)
            const auto on = [&](int i) { return i0 + i < a.Sq && lse_in[min(i0 + i, a.Sq - 1)] != -kInf; };
            T::template fetch<VEC>(qx, a, a.qs, a.q, n, head * a.D, i0, on);
            T::template fetch<VEC>(dx, a, a.dos, a.dout, n, head * a.D, i0, on);
        };
        fetch(lo);
        for (int i0 = lo; i0 < hi; i0 += KT, ++number) {
            __syncthreads();
            T::put_finite(qt, qx, row_bad, &any_bad, number);
            T::put_finite(dt, dx, row_bad, &any_bad, number);
            if (threadIdx.x < KT) {
                const int i = i0 + threadIdx.x, ii = min(i, a.Sq - 1);
                const RowState row(a, im, n, i, head);
                const float lse = i < a.Sq ? lse_in[ii] : -kInf;
                row_lse[threadIdx.x] = lse == -kInf ? kInf : lse * kLog2e;
                row_delta[threadIdx.x] = lse == -kInf ? 0.f : delta_in[ii];
                row_share[threadIdx.x] = a.slopes ? share_in[ii] : 1.f;
                row_p[threadIdx.x] = row.p;
                row_code[threadIdx.x] = row.code;
                row_bound[threadIdx.x] = row.bound;
                row_doc[threadIdx.x] = row.doc;
            }
            __syncthreads();
            if (i0 + KT < hi) fetch(i0 + KT);

            floatx4 s[NB] = {}, dp[NB] = {};
#pragma unroll
            for (int c = 0; c < DT; ++c)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const floatx4 x = T::tokens(qt, b, c, m, g), y = T::tokens(dt, b, c, m, g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[b] = mfma(x[e], k[c][e], s[b]);
                        dp[b] = mfma(y[e], v[c][e], dp[b]);
                    }
                }
            const bool all_lo = a.table && __all(code - row_code[0] <= -a.reach), all_hi = a.table && __all(code - row_code[KT - 1] >= a.reach), bad = any_bad == number;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const floatx4 l4 = *reinterpret_cast<const floatx4 *>(row_lse + 16 * b + 4 * g), d4 = *reinterpret_cast<const floatx4 *>(row_delta + 16 * b + 4 * g);
                const floatx4 h4 = *reinterpret_cast<const floatx4 *>(row_share + 16 * b + 4 * g);
                const int4 b4 = *reinterpret_cast<const int4 *>(row_bound + 16 * b + 4 * g);
                const int bounds[4] = {b4.x, b4.y, b4.z, b4.w};
                int ps[4] = {}, codes[4] = {}, docs[4] = {doc, doc, doc, doc};
                if (a.slopes) {
                    const int4 x = *reinterpret_cast<const int4 *>(row_p + 16 * b + 4 * g);
                    ps[0] = x.x; ps[1] = x.y; ps[2] = x.z; ps[3] = x.w;
                }
                if (a.table) {
                    const int4 x = *reinterpret_cast<const int4 *>(row_code + 16 * b + 4 * g);
                    codes[0] = x.x; codes[1] = x.y; codes[2] = x.z; codes[3] = x.w;
                }
                if (a.docs) {
                    const int4 x = *reinterpret_cast<const int4 *>(row_doc + 16 * b + 4 * g);
                    docs[0] = x.x; docs[1] = x.y; docs[2] = x.z; docs[3] = x.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float core = score_core(a, sc, s[b][e]);
                    float t = score_of(a, sc, core);
                    t += a.slopes ? fmaf(-slope, fabsf((float)(ps[e] - j)), -l4[e]) : -l4[e];
                    if (a.table) {
                        if (all_lo || all_hi) t += all_lo ? far_lo : far_hi;
                        else {
                            const int at = offset_at(a, code, codes[e]);
                            t += bias ? bias[at] : bias_gather(a, head, at);
                        }
                    }
                    if (bad) t = row_bad[16 * b + 4 * g + e] == number ? __builtin_nanf("") : t;
                    const bool seen = (j_raw < bounds[e]) & (docs[e] == doc);
                    const float p = seen ? __builtin_amdgcn_exp2f(t) * h4[e] : 0.f;
                    const float ds = seen ? p * (dp[b][e] - d4[e]) : 0.f;
                    s[b][e] = p;
                    dp[b][e] = a.cap > 0.f && ds != 0.f ? ds * fmaf(-core, core, 1.f) : ds;      // (of a hidden key core may be NaN)
                }
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int grp = 0; grp < GR; ++grp) {
                        float x[VD], y[VD];
                        T::template channels<VD>(x, dt, 16 * b + 4 * g + e, grp, m);
                        T::template channels<VD>(y, qt, 16 * b + 4 * g + e, grp, m);
#pragma unroll
                        for (int w = 0; w < VD; ++w) {
                            dv[grp * VD + w] = mfma(x[w], s[b][e], dv[grp * VD + w]);
                            dk[grp * VD + w] = mfma(y[w], dp[b][e], dk[grp * VD + w]);
                        }
                    }
        }
    }
    if (j_raw < a.Sk) {
        float *tk = const_cast<float *>(token_at(a.dk, a.dks, n, j)), *tv = const_cast<float *>(token_at(a.dv, a.dvs, n, j));
#pragma unroll
        for (int grp = 0; grp < GR; ++grp)
#pragma unroll
            for (int x = 0; x < VD; ++x) {
                const int d = grp * 16 * VD + 4 * g * VD + 4 * x;
                store_quad<VEC>(a, a.dks, tk, key_head * a.D, d, result_quad<DT>(dk, grp, x) * a.scale);
                store_quad<VEC>(a, a.dvs, tv, key_head * a.D, d, result_quad<DT>(dv, grp, x));
            }
    }
}

// The sum of 32 slices' values, for slice 0, in a fixed order.
__device__ __forceinline__ float sum_of_slices(float (*red)[32], float mine)
{
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    red[slice][lane] = mine;
    for (int d = 16; d; d >>= 1) {
        __syncthreads();
        if (slice < d) red[slice][lane] += red[slice + d][lane];
    }
    return red[slice][lane];
}

// The table's gradient from the workgroups' sums by offset: over images and tiles of rows of a head, 32 offsets a workgroup ...
__global__ void __launch_bounds__(1024) attn_bias_offsets(const float *part, float *sums, int N, int heads, int row_tiles, int size, int blocks)
{
    __shared__ float red[32][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, head = blockIdx.x / blocks, x = (blockIdx.x - head * blocks) * 32 + lane;
    float s[4] = {};
    if (x < size)
        for (int e0 = slice; e0 < N * row_tiles; e0 += 128)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e = e0 + 32 * k, n = e / row_tiles, tile = e - n * row_tiles;
                if (e < N * row_tiles) s[k] += part[(((size_t)n * heads + head) * row_tiles + tile) * size + x];
            }
    const float all = sum_of_slices(red, (s[0] + s[1]) + (s[2] + s[3]));
    if (slice == 0 && x < size) sums[(size_t)head * size + x] = all;
}
// ... and over the offsets of a bucket, 32 buckets a workgroup.
__global__ void __launch_bounds__(1024) attn_bias_buckets(const float *sums, const int *bucket, float *dtable, int size, int buckets, int blocks)
{
    __shared__ float red[32][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, head = blockIdx.x / blocks, b = (blockIdx.x - head * blocks) * 32 + lane;
    float s[4] = {};
    for (int x0 = slice; x0 < size; x0 += 128)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int x = min(x0 + 32 * k, size - 1), at = max(0, min(bucket[x], buckets - 1));
            const float y = sums[(size_t)head * size + x];
            s[k] += x == x0 + 32 * k && at == b ? y : 0.f;
        }
    const float all = sum_of_slices(red, (s[0] + s[1]) + (s[2] + s[3]));
    if (slice == 0 && b < buckets) dtable[(size_t)head * buckets + b] = all;
}

}  // namespace

// Tiles of the streamed side.
#define GRAD_FORMS(X) X(1, 64) X(2, 64) X(3, 64) X(4, 64) X(5, 32) X(6, 32) X(8, 32) X(16, 16)

hipError_t launch_attn_grad_shares(const AttnArgs &a, bool vec, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.heads * a.row_tiles);
    const size_t lds = a.bias_lds ? (2 * (size_t)a.reach + 1) * sizeof(float) : 0;
#define FORM(dt, kt) \
    if (a.D <= 16 * dt) { \
        return vec ? launch_lds(attn_grad_shares<dt, kt, true>, grid, lds, a, s) : launch_lds(attn_grad_shares<dt, kt, false>, grid, lds, a, s); \
    }
    GRAD_FORMS(FORM)
#undef FORM
    return hipErrorInvalidValue;
}

hipError_t launch_attn_grad_rows(const AttnArgs &a, bool vec, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * a.heads * a.row_tiles);
    const size_t size = 2 * (size_t)a.reach + 1;
#define FORM(dt, kt) \
    if (a.D <= 16 * dt) { \
        size_t lds = a.bias_lds ? size : 0; \
        if (a.part_bias) lds += 64 * (kt + 1) + (a.bias_acc_lds ? size : 0); \
        lds *= sizeof(float); \
        return vec ? launch_lds(attn_grad_rows<dt, kt, true>, grid, lds, a, s) : launch_lds(attn_grad_rows<dt, kt, false>, grid, lds, a, s); \
    }
    GRAD_FORMS(FORM)
#undef FORM
    return hipErrorInvalidValue;
}

hipError_t launch_attn_grad_keys(const AttnArgs &a, bool vec, hipStream_t s)
{
    const unsigned grid = (unsigned)((long)a.N * (a.heads / a.group) * a.key_tiles);
    const size_t lds = a.bias_lds ? (2 * (size_t)a.reach + 1) * sizeof(float) : 0;
#define FORM(dt, kt) \
    if (a.D <= 16 * dt) { \
        return vec ? launch_lds(attn_grad_keys<dt, kt, true>, grid, lds, a, s) : launch_lds(attn_grad_keys<dt, kt, false>, grid, lds, a, s); \
    }
    GRAD_FORMS(FORM)
#undef FORM
    return hipErrorInvalidValue;
}

hipError_t launch_attn_grad_bias(const AttnArgs &a, float *sums, float *dtable, hipStream_t s)
{
    const int size = 2 * a.reach + 1, by_offset = (size + 31) / 32, by_bucket = (a.buckets + 31) / 32;
    hipLaunchKernelGGL(attn_bias_offsets, dim3(a.heads * by_offset), dim3(1024), 0, s, a.part_bias, sums, a.N, a.heads, a.row_tiles, size, by_offset);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(attn_bias_buckets, dim3(a.heads * by_bucket), dim3(1024), 0, s, sums, a.bucket, dtable, size, a.buckets, by_bucket);
    return hipGetLastError();
}

}  // namespace small
