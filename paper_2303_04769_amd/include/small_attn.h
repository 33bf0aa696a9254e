/*
 * small_attn.h -- the attention block of libsmall_hip (gfx950): group normalization with an activation, attention over the pixels
 * of feature maps or the frames of sequences, its form for single tokens, and the gradients of both.
 *
 * These layers stand between the convolutions of small.h and work on the same channel-blocked activations, so a 1x1
 * convolution writes the queries, keys and values that attention reads, and another reads what attention wrote:
 *
 *   activations  [N][C/Cb][S][Cb]       S = H * W pixels in row-major order (or S frames), Cb fastest
 *
 * All data are IEEE fp32; sums, softmax statistics and gradients are accumulated in fp32. Conventions and error codes are
 * those of small.h: device pointers owned by the caller, nothing allocated, freed or synchronised, work enqueued on `stream`,
 * nothing enqueued when an error is returned. Unlike there, a channel block may be any divisor of C (Cb = C is the channels-last
 * layout [N][S][C]), at most 4096, or 1024 where 4 does not divide it or a tensor is not 16-byte aligned: SMALL_ERR_BLOCK beyond.
 * Every result is a function of the inputs alone: the order of each sum is fixed, there are no atomic additions.
 */
#ifndef SMALL_ATTN_H
#define SMALL_ATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- group normalization with an activation.
 * The C channels are split into G groups of C / G consecutive ones; mean and var are those of a group's C/G * H*W values in one image:
 *   xhat = (x - mean) * rstd,  rstd = 1 / sqrt(var + eps),  z = gamma[c] * xhat + beta[c],  out = act(z)
 *   act: SMALL_ACT_NONE z;  SMALL_ACT_RELU z > 0 ? z : +0;  SMALL_ACT_SILU z / (1 + exp(-z)).
 * gamma, beta: C floats in plain channel order. stats: [N][G][2], mean then rstd of each group (NULL in the forward call: not
 * wanted). in / out: [N][C/Cb][H][W][Cb]; out may equal in exactly (in place), other overlaps are refused.
 * The variance is taken from differences to a mean, never as a difference of two large sums.
 *
 * small_groupnorm_grad: given dout and the forward call's stats (which it reads), with dz = dout * act'(z) (RELU: 0 for z <= 0) and
 * sums over the group's n = C/G * H*W values,
 *   dgamma[c] = sum_{images, pixels} dz * xhat,  dbeta[c] = sum dz,
 *   din = rstd * (gamma dz - sum(gamma dz) / n - xhat * sum(gamma dz xhat) / n).
 * din may equal dout exactly (in place). dgamma and dbeta may both be NULL (parameters that are not trained).
 *
 * small_groupnorm_workspace (host only): bytes of workspace that both calls need for these sizes, 256-byte aligned (0 is
 * possible: then it may be NULL). */
enum { SMALL_ACT_NONE = 0, SMALL_ACT_RELU = 1, SMALL_ACT_SILU = 2 };
int small_groupnorm_workspace(int N, int C, int H, int W, int G, int Cb, size_t *bytes);
int small_groupnorm(const float *in, const float *gamma, const float *beta, float *out, float *stats, int N, int C, int H, int W,
                    int G, float eps, int act, int Cb, void *workspace, size_t workspace_bytes, void *stream);
int small_groupnorm_grad(const float *in, const float *gamma, const float *beta, const float *stats, const float *dout, float *din,
                         float *dgamma, float *dbeta, int N, int C, int H, int W, int G, int act, int Cb, void *workspace,
                         size_t workspace_bytes, void *stream);

/* ---- attention.
 * heads query heads of D channels, kv_heads key heads (heads a multiple of kv_heads; query head h reads key head
 * h / (heads / kv_heads)); head h's channel d is channel h * D + d of its tensor. Channel c of token t of image n stands at
 *   base + n * image + (c / Cb) * block + t * token + c % Cb                                              (floats)
 * with the strides of small_tokens: of a contiguous tensor of Ct channels and S tokens image = Ct * S, block = S * Cb, token = Cb; the
 * parts of one projection's output and a cache of which the first Sk tokens are read have strides of their own.
 *
 * Query i of image n is the token at position p = first[n] + i (first NULL: Sk - Sq + i, the last Sq of the Sk tokens). Key j is seen by it when
 *     j < lengths[n]                                    (lengths NULL: Sk; values above Sk count as Sk)
 *     and (not causal or j <= p or j < prefix[n])       (prefix NULL: 0)
 *     and (docs NULL or docs[n][j] == docs[n][p] >= 0)  (docs: [N][Sk]; a position outside 0 .. Sk-1 sees nothing)
 * Scores over the keys that are seen, their softmax and the result:
 *     s = scale * (q . k);  if cap > 0: s = cap * tanh(s / cap)
 *     s += table[h][bucket[min(max(code(j) - code(p), -reach), reach) + reach]]      (table NULL: no such term)
 *     s -= slopes[h] * |p - j|                                                       (slopes NULL: no such term)
 *     out = sum softmax(s) * v,   lse[n][h][i] = log(sum exp(s))
 * with code(p) = (p div width) * (2 * width - 1) + p mod width, which differs by a number of its own for every offset of rows and
 * columns of images that are `width` pixels wide; width = 1 makes it the distance in a sequence. bucket: 2 * reach + 1 bucket indices
 * in 0 .. buckets - 1 (values outside are taken into that range); table: [heads][buckets]; a bias below -1e30, so also one of the
 * type's lowest value, hides its offsets as minus infinity does.
 * A row that sees no key, or only keys of score -inf, gives out = 0 and lse = -inf. Keys at and beyond an image's length may hold
 * anything (NaN among it), and neither does what a key hidden by another mask holds, however large, infinite or NaN, reach a row that does not see it. So it is
 * in the gradients: dq of rows that do not see such a key, dk and dv of keys that no row sees which is such itself or sees one. Gradients of those that do are not finite.
 *
 * Precision. Larger calls hold values as two fp16 numbers at a power of two of their token's largest channel: 22 bits of values down to 2^-12 of that, one less for every
 * halving below; their products are summed in fp32. So results are as near to 64 bits as those of fp32 products (which round every addition)
 * where the channels of a token are of like size, and a channel 2^-35 of its neighbours is lost. A row's weights are held to 2^-33 of its largest or better, and the
 * terms of a gradient to 2^-33 of its largest: what only smaller ones contribute may come out as zero. Distances past 2^24 are rounded as fp32 does. (What a mask hides may decide which of two ways a value is rounded, no
 * more.) The gradients take their weights from lse, and so have the error of lse's rounding, 2^-24 of its size; with slopes, which make lse large, weights are scaled to sum
 * to one. Past scores of some 2^20 lse does not hold them apart any more, and gradients of rows that see such may be infinite or NaN.
 *
 * All of lengths, first, prefix, docs, slopes, table and bucket are DEVICE pointers. Limits: D <= 256; Sq, Sk <= 2^28, first positions are
 * taken into -2^28 .. 2^28; heads / kv_heads * Sq and N * heads * Sq < 2^31, and of the launches none has 2^32 threads (tiles of
 * 64 tokens of all heads and images below 2^24 forward and 2^23 in the gradient; heads times offsets of a table below 2^27 there). Tensors may be larger than 2^31 values.
 * lse may be NULL in the forward call. small_attention_workspace (host only): bytes for a forward call (grad = 0) or a gradient call (grad = 1); of the pointers in *a it only matters whether table is NULL;
 * 256-byte aligned (0 is possible: then it may be NULL).
 *
 * small_attention_grad: given out and lse of the forward call and dout, the gradients dq, dk, dv (dk, dv summed over a key head's query heads) and dtable ([heads][buckets]; NULL when not wanted or table is NULL). Every value of
 * dq, dk, dv of the heads' channels is written: zero for tokens that saw nothing or were not seen.
 * What a call writes must overlap neither itself (SMALL_ERR_SHAPE where strides make it), nor anything else that the call uses
 * (SMALL_ERR_ALIAS). Parts of one tensor, whose ranges interleave, are told apart where their strides are equal. */
typedef struct { size_t image, block, token; } small_tokens;
typedef struct {
    int N, Sq, Sk, heads, kv_heads, D, Cb;
    small_tokens q, k, v, out;
    small_tokens dout, dq, dk, dv;      /* read by the gradient call only */
    float scale, cap;
    int causal, width, reach, buckets;
    const int *lengths, *first, *prefix, *docs;
    const float *slopes, *table;
    const int *bucket;
} small_attn;
int small_attention_workspace(const small_attn *a, int grad, size_t *bytes);
int small_attention(const small_attn *a, const float *q, const float *k, const float *v, float *out, float *lse, void *workspace,
                    size_t workspace_bytes, void *stream);
int small_attention_grad(const small_attn *a, const float *q, const float *k, const float *v, const float *out, const float *lse,
                         const float *dout, float *dq, float *dk, float *dv, float *dtable, void *workspace, size_t workspace_bytes,
                         void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SMALL_ATTN_H */
