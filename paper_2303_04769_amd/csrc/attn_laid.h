// Places of tensors in memory, as the checks of the attention block's calls look at them (attn_api.hip, cache_api.hip): host only.
#pragma once
#include "../../include/small.h"
#include "../include/small_attn.h"
#include "attn_tile.h"

#include <stdint.h>

namespace small {

constexpr size_t kWorkspaceAlign = 256;

inline int from_hip(hipError_t e) { return e == hipSuccess ? SMALL_OK : SMALL_ERR_LAUNCH; }

// A range of device memory, in bytes.
struct Range {
    uintptr_t at, end;
    Range(const void *p, size_t floats) : at((uintptr_t)p), end((uintptr_t)p + floats * sizeof(float)) {}
    bool meets(const Range &o) const { return at < o.end && o.at < end; }
};

inline bool workspace_ok(const void *ws, size_t have, size_t need)
{
    return need == 0 || (ws && have >= need && (uintptr_t)ws % kWorkspaceAlign == 0);
}

// A tensor of `heads` heads over `tokens` tokens, as the strides lay it out.
struct Laid {
    const float *p;
    small_tokens s;
    size_t n, blocks, tokens, Cb;
    size_t floats() const { return (n - 1) * s.image + (blocks - 1) * s.block + (tokens - 1) * s.token + Cb; }
    Range range() const { return Range(p, floats()); }
    // (stride, size) by falling stride
    void levels(size_t (&stride)[3], size_t (&size)[3]) const
    {
        const size_t st[3] = {s.image, s.block, s.token}, sz[3] = {n, blocks, tokens};
        int order[3] = {0, 1, 2};
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2 - i; ++j)
                if (st[order[j]] < st[order[j + 1]]) { const int t = order[j]; order[j] = order[j + 1]; order[j + 1] = t; }
        for (int i = 0; i < 3; ++i) { stride[i] = st[order[i]]; size[i] = sz[order[i]]; }
    }
    // Whether no two of its values share a place: every stride passes all that lies below it.
    bool distinct() const
    {
        size_t stride[3], size[3], below = Cb;
        levels(stride, size);
        for (int i = 2; i >= 0; --i) {
            if (size[i] == 1) continue;
            if (stride[i] < below) return false;
            below += (size[i] - 1) * stride[i];
        }
        return true;
    }
    // Whether it shares no place with o, as far as ranges, or equal strides that interleave them, show.
    bool apart(const Laid &o) const
    {
        if (!range().meets(o.range())) return true;
        if (((uintptr_t)p - (uintptr_t)o.p) % sizeof(float)) return false;
        size_t sa[3], na[3], sb[3], nb[3];
        levels(sa, na);
        o.levels(sb, nb);
        long long rel = ((long long)(uintptr_t)o.p - (long long)(uintptr_t)p) / (long long)sizeof(float);
        for (int i = 0; i < 3; ++i) {
            if (sa[i] != sb[i] || sa[i] == 0) return false;
            size_t ea = Cb, eb = o.Cb;
            for (int k = i + 1; k < 3; ++k) { ea += (na[k] - 1) * sa[k]; eb += (nb[k] - 1) * sb[k]; }
            const long long st = (long long)sa[i];
            rel = (rel % st + st) % st;
            if ((size_t)rel >= ea && (size_t)rel + eb <= sa[i]) return true;
        }
        return false;
    }
    bool apart(const Range &r) const { return !range().meets(r); }
};

// Whether every launch of a call is one: a grid has fewer than 2^32 threads. (Asked for before the first, so that a call is enqueued whole or not at all.)
inline bool launches(double workgroups, double threads) { return workgroups * threads < 4294967296.0; }

inline TokenStrides strides(const small_tokens &s) { return TokenStrides{(long long)s.image, (long long)s.block, (long long)s.token}; }

}  // namespace small
