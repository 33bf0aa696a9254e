// Attention on the fp16 matrix instructions with values in two parts (attn_parts.hip, attn_parts_grad.hip).
//
// x = hi + lo with hi = fp16(x), lo = fp16(x - hi) keeps x to 2^-22 of its size, and the products hi hi, hi lo, lo hi, summed in fp32, keep a
// product to some 2^-21.5: sums of D or more of them come out as near to 64 bits as those of fp32 instructions, whose every addition rounds (errors
// of both are in the tests and in the measured cases). Three v_mfma_f32_16x16x32_f16 of 16 cycles do what eight
// v_mfma_f32_16x16x4_f32 of 32 do: 5.3 times the rate.
//
// fp16 has little range, so values carry a power of two: one for each tile of 64 tokens of a head (its largest magnitude comes to lie in
// [2^10, 2^11)), one for each row that a wave holds in registers. A value 2^-12 times the tile's largest still has 22 bits, and below that the error is
// 2^-35 of the largest one; weighted sums over tiles, whose weights carry the difference of their powers, have an error of 2^-32 of the largest value that the
// row's range of keys holds. So no magnitude is out of reach, and what stands beside values 2^9 times its own still has fp32's precision; infinities and NaN become NaN.
//
// attn_make_parts lays tiles out once, as the matrix instructions want them: blocks of 1 KB, [16 tokens][32 channels][part], lane (m, g) with its eight
// values behind each other (channels 8g .. 8g+7 of token m), so a wave reads an operand with tokens in lanes as one linear kilobyte, and copies of tiles into LDS
// are linear too. The operand with channels in lanes is read from the same block by the transposing reads of LDS (across): lane (m, g) gets tokens
// 4g .. 4g+3 and 16+4g .. 16+4g+3 of channel m, the order in which two results of 16 tokens each lie in a lane's registers, which are the other operand of
// that product.
#pragma once
#include "attn_row.h"

namespace small {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));

constexpr int kTop = 10;                       // exponent of a tile's or row's largest value
constexpr int kLift = 8;                       // of weights: with kSlack below 2^15

__device__ __forceinline__ floatx4 mfma16(half8 a, half8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef unsigned uintx4v __attribute__((ext_vector_type(4)));

// Two values into half a register's worth of parts each. (The factor is hidden from the compiler, which would take a subtraction for the multiply-add and with it
// a conversion each way for the one instruction that reads and writes halves.)
__device__ __forceinline__ void split_pair(float x, float y, unsigned &hi, unsigned &lo)
{
    float minus = -1.f;
    asm("" : "+s"(minus));
    const half2v h = __builtin_convertvector((float2v{x, y}), half2v), l = {(_Float16)fmaf((float)h.x, minus, x), (_Float16)fmaf((float)h.y, minus, y)};
    hi = __builtin_bit_cast(unsigned, h);
    lo = __builtin_bit_cast(unsigned, l);
}
// Results of 32 tokens (two of 16) of a lane's column as a right operand in two parts.
__device__ __forceinline__ void split_results(const floatx4 &first, const floatx4 &second, half8 &hi, half8 &lo)
{
    uintx4v h, l;
    unsigned x, y;
    split_pair(first.x, first.y, x, y); h.x = x; l.x = y;
    split_pair(first.z, first.w, x, y); h.y = x; l.y = y;
    split_pair(second.x, second.y, x, y); h.z = x; l.z = y;
    split_pair(second.z, second.w, x, y); h.w = x; l.w = y;
    hi = __builtin_bit_cast(half8, h);
    lo = __builtin_bit_cast(half8, l);
}

// Power of two e such that a magnitude `most` times 2^-e lies in [2^kTop, 2^(kTop + 1)); nothing but zeros: a small one.
__device__ __forceinline__ int parts_exponent(float most)
{
    if (most == 0.f) return -100;
    const int e = (int)(__float_as_uint(most) >> 23) - 127 - kTop;
    return max(e, -100);
}
__device__ __forceinline__ float finite_magnitude(float x) { return fabsf(x) < kInf ? fabsf(x) : 0.f; }

// A workgroup's tile of rows, of which (image, head), and its split of the keys. Causal rows have ever more keys, so there the longest tiles come first; where the device's eight
// parts get whole heads, those of one head stay in one. Of the 32 workgroups that meet the 32 compute units of a part in turn, every other set comes in
// reverse order, so that the workgroups that begin together on a compute unit have about the same work everywhere.
struct RowTile { int group, tile, split; };
template <bool SPLITS>
__device__ __forceinline__ RowTile row_tile_of(const AttnArgs &a, unsigned groups)
{
    const unsigned tiles = (unsigned)a.row_tiles;
    if (!a.causal || (SPLITS && a.splits > 1)) {
        const int id = (int)xcd_contiguous(blockIdx.x, gridDim.x), by_split = SPLITS ? a.by_splits.div(id) : id, group = a.by_tiles.div(by_split);
        return {group, (int)tiles - 1 - (by_split - group * (int)tiles), SPLITS ? id - by_split * a.splits : 0};
    }
    const bool whole = (groups & 7) == 0;
    const unsigned part = whole ? blockIdx.x & 7 : 0, each = whole ? groups >> 3 : groups, at = whole ? blockIdx.x >> 3 : blockIdx.x;
    const unsigned units = whole ? 32 : 256, set = at / units;
    const unsigned r = (set & 1) && (set + 1) * units <= each * tiles ? (2 * set + 1) * units - 1 - at : at, by_tile = r / each;
    return {(int)(part * each + (r - by_tile * each)), (int)(tiles - 1 - by_tile), 0};
}

// An exponent, by a scalar load: it counts apart from the copies into LDS, which the compiler does not see and which a wait for a vector load would include.
__device__ __forceinline__ int exponent_at(const int *exps, size_t at) { return ((const __attribute__((address_space(4))) int *)exps)[at]; }

struct PartsTensor {
    const float *p;
    TokenStrides s;
    int heads, tokens, tiles, rows;            // rows: not keys but queries (their masks: rows of lse = -inf are left out)
    char *image;
    int *exps;                                 // [N * heads][tiles]
    unsigned first_block;
};
struct PartsArgs {
    PartsTensor t[4];
    int count;
};

// A lane's place in a block as the operand with tokens in lanes. The sixteen tokens of odd groups of channels stand in another order, their fours the other
// way round, for the transposing reads: thirty-two lanes take eight tokens of two groups there, which then are in different banks.
__device__ __forceinline__ int token_place(int m, int g) { return (16 * g + (m ^ (g & 1) * 12)) * 16; }
// Left operand with channels in lanes: of the 32 tokens of pair `pair`, the 16 channels of block d, one part. at: a tile in LDS, this lane's place in it.
__device__ __forceinline__ int across_place(int m, int g) { return ((m & 2) << 7) + ((4 * g + (m >> 2)) ^ (m >> 1 & 1) * 12) * 16 + (m & 1) * 8; }
template <int STEPS>
__device__ __forceinline__ half8 across(const char *at, int pair, int d, int part)
{
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v *lds4;
    const char *const from = at + (2 * pair * STEPS + d / 2) * 2048 + part * 1024 + (d & 1) * 512;
    const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)from), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(from + STEPS * 2048));
    return __builtin_bit_cast(half8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}
// acc += channels of 32 tokens times results in two parts, part by part over up to four blocks of channels.
template <int STEPS>
__device__ __forceinline__ void products_across(floatx4 (&acc)[2 * STEPS], const char *at, int pair, half8 b_hi, half8 b_lo)
{
    constexpr int DT = 2 * STEPS, ND = DT < 4 ? DT : 4;
#pragma unroll
    for (int d0 = 0; d0 < DT; d0 += ND) {
        half8 hi[ND], lo[ND];
#pragma unroll
        for (int d = 0; d < ND && d0 + d < DT; ++d) lo[d] = across<STEPS>(at, pair, d0 + d, 1);
#pragma unroll
        for (int d = 0; d < ND && d0 + d < DT; ++d) hi[d] = across<STEPS>(at, pair, d0 + d, 0);
#pragma unroll
        for (int part = 0; part < 3; ++part)
#pragma unroll
            for (int d = 0; d < ND && d0 + d < DT; ++d) acc[d0 + d] = mfma16(part == 0 ? lo[d] : hi[d], part == 1 ? b_lo : b_hi, acc[d0 + d]);
    }
}

constexpr size_t parts_tile_bytes(int steps) { return (size_t)64 * 32 * steps * 4; }
constexpr int parts_steps(int D) { return (D + 31) / 32; }
// What the rows' gradient may ask for behind the few hundred bytes that it has anyway: 160 KB a compute unit.
constexpr size_t kGradLds = 160 * 1024 - 2048;

// attn_parts.hip
hipError_t launch_make_parts(const AttnArgs &a, PartsArgs &args, bool vec, hipStream_t s);
hipError_t launch_attn_grad_rows_parts(const AttnArgs &a, hipStream_t s);        // attn_parts_grad.hip
hipError_t launch_attn_grad_keys_parts(const AttnArgs &a, hipStream_t s);
hipError_t launch_attn_rows_parts(const AttnArgs &a, size_t bias_bytes, hipStream_t s);

}  // namespace small
