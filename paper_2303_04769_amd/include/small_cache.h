/*
 * small_cache.h -- rotary positions and a paged cache for the attention block of libsmall_hip (gfx950): turns of queries and keys over one to four
 * axes and their gradient, keys and values written into pages as 32-bit, bfloat16 or 8-bit numbers and read back, and attention of new
 * tokens over such a cache.
 *
 * Activations, strides, conventions and error codes are those of small_attn.h: [N][C/Cb][S][Cb] fp32 views, device pointers owned by the
 * caller, nothing allocated, freed or synchronised, work enqueued on `stream`, nothing enqueued when an error is returned. Every result is a
 * function of the inputs alone: the order of each sum is fixed, there are no atomic additions.
 */
#ifndef SMALL_CACHE_H
#define SMALL_CACHE_H

#include "small_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions.
 * Of each head's D channels the first 2 * pairs turn in pairs by angles that depend on the token's place, the others stay as they are. Pair k is channels
 * 2k and 2k + 1, or with `halves` channels k and pairs + k:
 *     y0 = x0 cos t - x1 sin t,   y1 = x0 sin t + x1 cos t,   t = sum over axes of place[axis] * freq[f][axis][k]           (radians)
 * freq: [freq_heads][axes][pairs] floats; freq_heads is 1 (all heads turn alike) or kv_heads (f = h of key head h and of the query heads that read it). Pairs
 * of one axis have zeros for the others; learned frequencies may turn by all of them.
 * A token's place is positions[n][i][axis] (int32 [N][S][axes]), or, where positions is NULL, that of number first[n] + i (first NULL: i, of at most 2^28 either
 * way) in rows of extent[axes - 1] places, planes of extent[axes - 2] rows and so on: extent[0] is not read, the first axis has no end.
 * Angles and turns are computed in 64 bits and rounded once, so results are within half a step of fp32, and 2^-50 of the pair's larger channel times one and the size of the
 * angle.
 *
 * small_rotary turns q ([N] images of `heads` heads, to q_out) and k (`kv_heads` heads, to k_out); q and q_out, or k and k_out, may both be NULL. An output may equal
 * its input exactly (in place); then channels that do not turn are not touched. Other overlaps are refused.
 *
 * small_rotary_grad: given the gradients dq_out, dk_out of q_out, k_out, the gradients dq, dk of q, k -- the turn back; in place likewise -- and, where dfreq is not NULL,
 *     dfreq[f][axis][k] = sum over images, tokens, the heads that turn by f of place[axis] * (dy1 y0 - dy0 y1)                  (summed in 64 bits)
 * for which it reads q and k: what small_rotary gave (y above, and dy are dq_out, dk_out), or with r->from_inputs what it was given (y and dy are q and dq, k and dk: turned back by one
 * angle, both have the same cross product; neither has it with the other). They may be NULL without dfreq. Strides: r->q, r->k are those of
 * q and k, r->q_out, r->k_out of dq_out and dk_out, r->dq, r->dk of dq and dk. small_rotary_workspace (host only): bytes that the gradient call with dfreq needs,
 * 256-byte aligned; without dfreq none are needed.
 *
 * Limits: D <= 256, 1 <= axes <= 4, 2 * pairs <= D, and N * S * (heads + kv_heads) * D < 2^33 (2^31 where four channels of a head do not stand together and aligned). */
typedef struct {
    int N, S, heads, kv_heads, D, Cb;
    int axes, pairs, halves, freq_heads;
    int extent[4];
    int from_inputs;                    /* this, dq and dk are read by the gradient call only */
    small_tokens q, k, q_out, k_out;
    small_tokens dq, dk;
    const float *freq;
    const int *first, *positions;
} small_rotation;
int small_rotary_workspace(const small_rotation *r, size_t *bytes);
int small_rotary(const small_rotation *r, const float *q, const float *k, float *q_out, float *k_out, void *stream);
int small_rotary_grad(const small_rotation *r, const float *dq_out, const float *dk_out, const float *q, const float *k, float *dq, float *dk,
                      float *dfreq, void *workspace, size_t workspace_bytes, void *stream);

/* ---- a paged cache.
 * `pages` pages of `page` tokens (16, 32, 64, 128 or 256) hold the keys and values of kv_heads heads of D channels:
 *     keys    [pages][kv_heads][page][Dk]     Dk: D filled up to 16 bytes; what is behind D is zero
 *     values  [pages][kv_heads][D][page]      a channel's tokens stand together, as the product with weights reads them
 *     SMALL_CACHE_F32   floats as they are;   SMALL_CACHE_BF16   rounded to the nearest, ties to even
 *     SMALL_CACHE_I8    signed codes -127 .. 127 and a float for each token of a head, key_scales and value_scales [pages][kv_heads][page]:
 *                       scale = top / 127,  code = x * (127 / top) to the nearest whole number, ties to even (each operation rounded to fp32),
 *                       where top is the token's largest channel of that head; a top below 2^-100 gives scale 0 and codes 0, one that is infinite or NaN
 *                       the scale NaN and codes 0. What a code stands for is code * scale.
 * keys and values are 16-byte aligned; the scales are not read for the other kinds. Memory that was never written must hold zeros in keys behind D, anything elsewhere.
 * Token p of stream n (of N) is in place p % page of page table[n][p / page]; table: int32 [N][per_stream], device memory like all of these. A page number outside
 * 0 .. pages - 1 is none: what would be written there is dropped, what would be read from there is left as it was, attention does not see it. Tokens in front of 0
 * or at and beyond per_stream * page are none either.
 *
 * small_cache_write puts tokens i < counts[n] (NULL: all S; taken into 0 .. S) of k and v at first[n] + i (first NULL: i). With r (else NULL) keys are turned first, as small_rotary
 * turns them, bit for bit, and q, if it is not NULL, is turned into q_out: all its S tokens. r's N, S, kv_heads, D and Cb are the call's; its first is not read (the call's takes its place),
 * its k, k_out, dq, dk are not read. Streams may share pages that are read. No place may be written
 * twice by one call: it would hold parts of both tokens, codes of one with the scale of the other perhaps.
 * small_cache_read: the same tokens from the cache to k and v; tokens that are none and those from counts[n] on are left as they were.
 * k, v: [N][blocks][S][Cb] views as in small_attn.h. Limits: of the launch's threads -- a quarter of D, filled up to a power of two
 * and to 4 at least, for each of N * (S + 31) tokens; where S <= 4, at least 64 for each -- there are fewer than 2^32; per_stream * page <= 2^28. */
enum { SMALL_CACHE_F32 = 0, SMALL_CACHE_BF16 = 1, SMALL_CACHE_I8 = 2 };
typedef struct {
    int kind, pages, page, kv_heads, D;
    void *keys, *values;
    float *key_scales, *value_scales;
    int N, per_stream;
    const int *table;
} small_cache;
typedef struct {
    int S, Cb;
    small_tokens k, v;
    const int *first, *counts;
} small_span;
int small_cache_write(const small_cache *c, const small_span *s, const float *k, const float *v, const small_rotation *r, const float *q,
                      float *q_out, void *stream);
int small_cache_read(const small_cache *c, const small_span *s, float *k, float *v, void *stream);

/* ---- attention of new tokens over the cache: small_attention with the keys and values of each stream's first lengths[n] tokens, causal. Of *a are read
 * N, Sq, heads, D, Cb, q, out, scale, cap, reach, buckets, lengths (not NULL; at most per_stream * page count), first (NULL: lengths[n] - Sq, the last tokens),
 * slopes, table (the bias's) and bucket; width must be 1, prefix and docs NULL, kv_heads and D the cache's. A stream of length zero is an empty place: out = 0,
 * lse = -inf. Meant for one token, or a few, a stream: every sixteen rows (tokens times the query heads of a key head), or 32, read the cache once. The streams' work is shared out by all of
 * their lengths: where a row's sums are split, and so how they are rounded, depends on the other streams' too. heads * buckets <= 2^30, and of tiles of sixteen rows and at least
 * 32 keys there are fewer than 2^30.
 * What a row does not see, and what is behind a stream's length in its last page or in no page of its, does not reach it, however large, infinite or NaN. (What other rows of a call see
 * of the same stream may decide which of two ways a value of a row is rounded, no more; memory that holds no token of a stream's does not decide even that.)
 * small_cache_attention_workspace (host only) looks at sizes alone. */
int small_cache_attention_workspace(const small_cache *c, const small_attn *a, size_t *bytes);
int small_cache_attention(const small_cache *c, const small_attn *a, const float *q, float *out, float *lse, void *workspace,
                          size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SMALL_CACHE_H */
