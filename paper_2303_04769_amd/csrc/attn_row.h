// One row of attention by one wave, key by key, for rows whose sums came out as NaN: in a product of tiles a key of weight zero
// contributes 0 * v, which is NaN where a hidden token's v is infinite or NaN. Here a key that the row does not see is left out. Slow, and
// reached only by inputs that hold such values.
#pragma once
#include "attn_tile.h"

namespace small {

// Keys begin .. end - 1 for the query (n, i) of `row`: o[k] is channel lane + 64 k of the unnormalized sum; maximum in units of log2.
__device__ __forceinline__ void attend_row(const AttnArgs &a, const RowState &row, int n, int i, int key_head, int begin, int end,
                                               float (&o)[4], float &maximum, float &sum)
{
    const Scorer sc(a);
    const int lane = threadIdx.x & 63;
    const float *q = token_at(a.q, a.qs, n, i), *k = token_at(a.k, a.ks, n, 0), *v = token_at(a.v, a.vs, n, 0);
    const auto score = [&](int j) {
        if (j >= end || !row.sees(j, a.docs ? key_document(a, n, j) : 0, a.docs)) return -kInf;
        float dot = 0.f;
        for (int d = 0; d < a.D; ++d)
            dot = fmaf(q[channel_at(a, a.qs, row.head * a.D + d)], k[(long long)j * a.ks.token + channel_at(a, a.ks, key_head * a.D + d)], dot);
        return sc.biased(sc.capped(dot), row, j, a.table ? code_of(a, j) : 0, nullptr);
    };
    float top = -kInf;
    for (int j = begin + lane; j < end; j += 64) top = fmaxf(top, score(j));
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float at = top == -kInf ? 0.f : top;
    float total = 0.f;
    o[0] = o[1] = o[2] = o[3] = 0.f;
    for (int j0 = begin; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < end && row.sees(j, a.docs ? key_document(a, n, j) : 0, a.docs);
        const float p = seen ? __builtin_amdgcn_exp2f(score(j) - at) : 0.f;
        total += p;
        for (unsigned long long left = __ballot(seen); left; left &= left - 1) {
            const int b = __ffsll((long long)left) - 1;
            const float w = __shfl(p, b);
            for (int x = 0; x < 4; ++x)
                if (lane + 64 * x < a.D) o[x] = fmaf(w, v[(long long)(j0 + b) * a.vs.token + channel_at(a, a.vs, key_head * a.D + lane + 64 * x)], o[x]);
        }
    }
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    maximum = top;
    sum = total;
}

// The same, written where the row belongs: the result, or its part of a split.
__device__ __forceinline__ void attend_row_and_store(const AttnArgs &a, const ImageMask &im, int n, int set, int r, int split, int begin, int end)
{
    const int hh = a.pack ? a.by_Sq.div(r) : 0, i = r - hh * a.Sq, head = a.pack ? set * a.group + hh : set, key_head = a.pack ? set : a.by_group.div(set);
    const RowState row(a, im, n, i, head);
    float o[4], top, sum;
    attend_row(a, row, n, i, key_head, begin, end, o, top, sum);
    const int lane = threadIdx.x & 63;
    const size_t part = (((size_t)n * a.head_sets + set) * a.rows + r) * a.splits + split;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int x = 0; x < 4; ++x) {
        const int d = lane + 64 * x;
        if (d >= a.D) continue;
        if (a.splits > 1) a.part_o[part * a.D + d] = o[x];
        else const_cast<float *>(token_at(a.o, a.os, n, i))[channel_at(a, a.os, head * a.D + d)] = sum == 0.f ? 0.f : o[x] * inv;
    }
    if (lane) return;
    if (a.splits > 1) a.part_ml[part] = float2{top, sum};
    else if (a.lse) a.lse[((size_t)n * a.heads + head) * a.Sq + i] = sum == 0.f ? -kInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace small
