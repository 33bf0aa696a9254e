// Attention on the fp16 matrix instructions with values in two parts (attn_parts.hip, attn_parts_grad.hip).
//
// x = hi + lo with hi = fp16(x), lo = fp16(x - hi) keeps x to 2^-22 of its size, and the products hi hi, hi lo, lo hi, summed in fp32, keep a
// product to some 2^-21.5: sums of D or more of them come out as near to 64 bits as those of fp32 instructions, whose every addition rounds (errors
// of both are in the tests and in the measured cases). Three v_mfma_f32_16x16x32_f16 of 16 cycles do what eight
// v_mfma_f32_16x16x4_f32 of 32 do: 5.3 times the rate.
//
// fp16 has little range, so values carry a power of two: one for each tile of 64 tokens of a head (its largest magnitude comes to lie in
// [2^10, 2^11)), one for each row that a wave holds in registers. A value 2^-12 times the tile's largest still has 22 bits, and below that the error is
// 2^-35 of the largest one. A mask may hide any token of a tile from a row, and what it hides must not cost the row precision: so a token whose largest value is
// less than 2^-kSpread of the tile's carries a power of its own, and the tile says so (mixed). Weighted sums over tiles are kept at a power of two for each row (column of
// a product), which follows the largest of the terms that the row sees (ColumnScale) -- those of values at one for all rows where all tiles of a walk have about the same
// and none is mixed (even). So no magnitude is out of reach, and a result's error is in proportion to the largest
// magnitude among the channels of the tokens that it is made of, not to anything else. A token that holds an infinity or NaN is laid out as zeros (0 times it would not
// be 0) and says so in place of its power of two (kBad); scores of those that see it become NaN.
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
constexpr int kLift = 9, kFall = 2;            // of weights: with kSlack 2^15 at most; tiles of values that may be 2^-kFall of the largest keep weights that much lower

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
constexpr int kSpread = 8;
__device__ __forceinline__ int parts_exponent(float most)
{
    if (most == 0.f) return -100;
    const int e = (int)(__float_as_uint(most) >> 23) - 127 - kTop;
    return max(e, -100);
}
__device__ __forceinline__ float finite_magnitude(float x) { return fabsf(x) < kInf ? fabsf(x) : 0.f; }
__device__ __forceinline__ float any_magnitude(float x) { return fabsf(x) < kInf ? fabsf(x) : kInf; }     // (NaN, too)

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

// What a tile's tokens carry, in a word: the power of two (kNone: nothing but zeros), whether tokens have some of their own (mixed), and whether there are zeros
// among them. A token of zeros has no size: where sums follow the largest term, one that carried its tile's power would raise them to the size of what may be hidden. So there its
// power is the smallest one, as if the tile were mixed (by_tokens); where sums are kept at one power of two anyway, it may carry any.
constexpr int kNone = -1000, kBad = 10000;
__device__ __forceinline__ int tile_word(int exponent, bool zeros, bool mixed) { return exponent * 4 + zeros * 2 + mixed; }
__device__ __forceinline__ int tile_exponent(int word) { return word >> 2; }
__device__ __forceinline__ bool tile_mixed(int word) { return word & 1; }
__device__ __forceinline__ bool tile_by_tokens(int word) { return word & 3; }

// Of the words that a wave's lanes go through one after another: the largest power of two and the smallest (of tiles that have one), and whether any tile is mixed.
struct Powers {
    int most = kNone, least = -kNone;
    bool mixed = false, zeros = false;
    __device__ __forceinline__ void add(int word)
    {
        const int e = tile_exponent(word);
        most = max(most, e);
        least = e == kNone ? least : min(least, e);
        mixed |= tile_mixed(word);
        zeros |= tile_by_tokens(word);
    }
    __device__ __forceinline__ void add_mixed(int word) { mixed |= tile_mixed(word); }
    // Over the wave: whether no tile is mixed and all are within 2^-spread of the largest. most: uniform from here on.
    __device__ __forceinline__ bool even(int spread)
    {
        // (as floats, by shifts of lanes: a shuffle is a trip through LDS)
        const auto over_wave = [](float v) {
            v = fmaxf(v, lane_shift1<0x128>(v));                 // row_ror: 8, 4, 2, 1
            v = fmaxf(v, lane_shift1<0x124>(v));
            v = fmaxf(v, lane_shift1<0x122>(v));
            v = fmaxf(v, lane_shift1<0x121>(v));
            return __builtin_amdgcn_readfirstlane((int)column_max(v));
        };
        const int low = -over_wave((float)-least);
        most = over_wave((float)most);
        return !__any(mixed) && most - low <= spread;
    }
    // For terms whose scale follows the largest: whether no tile is mixed, and none has zeros (tile_word) where tiles are of unlike size.
    __device__ __forceinline__ bool even_terms() { return __any(zeros) ? even(kSpread) : !__any(mixed); }
};

// A tile's word, by a scalar load: it counts apart from the copies into LDS, which the compiler does not see and which a wait for a vector load would include.
__device__ __forceinline__ int exponents_at(const int *exps, size_t at) { return ((const __attribute__((address_space(4))) int *)exps)[at]; }

struct PartsTensor {
    const float *p;
    TokenStrides s;
    int heads, tokens, tiles, rows;            // rows: not keys but queries (their masks: rows of lse = -inf are left out)
    char *image;
    int *exps, *each;                          // [N * heads][tiles], [N * heads][tiles][64] (written for mixed tiles and those with zeros)
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

// Values y, or results of a product with a mixed tile's tokens, of which a lane has the tokens 16b + 4g .. of the tile that `each` points to (by 4g): times their powers of
// two, and 2^more.
template <int NB>
__device__ __forceinline__ void by_token(floatx4 (&y)[NB], const int *each, int more = 0)
{
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int4 e = *reinterpret_cast<const int4 *>(each + 16 * b);
        y[b].x = ldexpf(y[b].x, e.x + more);
        y[b].y = ldexpf(y[b].y, e.y + more);
        y[b].z = ldexpf(y[b].z, e.z + more);
        y[b].w = ldexpf(y[b].w, e.w + more);
    }
}

// Scores, of tokens of a mixed tile: NaN where the token is bad. MASKED: behind their masks, minus infinity where the token is hidden, which stays so.
template <bool MASKED, int NB>
__device__ __forceinline__ void bad_tokens(floatx4 (&s)[NB], const int *each)
{
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int4 e = *reinterpret_cast<const int4 *>(each + 16 * b);
        s[b].x = (e.x == kBad) & (!MASKED | (s[b].x != -kInf)) ? __builtin_nanf("") : s[b].x;
        s[b].y = (e.y == kBad) & (!MASKED | (s[b].y != -kInf)) ? __builtin_nanf("") : s[b].y;
        s[b].z = (e.z == kBad) & (!MASKED | (s[b].z != -kInf)) ? __builtin_nanf("") : s[b].z;
        s[b].w = (e.w == kBad) & (!MASKED | (s[b].w != -kInf)) ? __builtin_nanf("") : s[b].w;
    }
}

// The power of two of a column's terms: they times `scale` stay within 2^14. Nothing but zeros so far: scale = 2^127, which any term passes.
struct ColumnScale {
    float scale = 0x1p127f;
    // Takes terms y that count 2^exp each to the column's scale, which is set anew, and the sums acc along, where one passes 2^14.
    template <int NB, int DT>
    __device__ __forceinline__ void apply(floatx4 (&y)[NB], int exp, floatx4 (&acc)[DT])
    {
        float mx = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b) mx = fmaxf(mx, fmaxf(fmaxf(fabsf(y[b].x), fabsf(y[b].y)), fmaxf(fabsf(y[b].z), fabsf(y[b].w))));
        float f = ldexpf(scale, exp);
        if (__any(!(mx * f <= 0x1p14f))) {
            mx = column_max(ldexpf(mx, exp));
            const bool more = mx * scale > 0x1p14f;
            const int e = max(-100, (int)(__float_as_uint(mx) >> 23) - 127);
            const float now = more ? ldexpf(1.f, 8 - e) : scale, by = ldexpf(now, back());
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= by;
            scale = now;
            f = ldexpf(scale, exp);
            if (__any(f == kInf)) {                              // (tokens 2^20 times and more as large as what the column has seen: it does not see these)
                const float first = ldexpf(1.f, exp);
#pragma unroll
                for (int b = 0; b < NB; ++b) y[b] *= first;
                f = scale;
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) y[b] *= f;
    }
    // All terms so far count 2^-by of what they did (the sums acc are that already): the scale follows, as far as floats go.
    template <int DT>
    __device__ __forceinline__ void follow(float by, floatx4 (&acc)[DT])
    {
        if (!__any(by >= 1.f)) return;
        const int k = max(0, min((int)fminf(by, 300.f), 108 + back()));
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[d][x] = ldexpf(acc[d][x], k);
        scale = ldexpf(scale, k);
    }
    __device__ __forceinline__ int back() const { return 127 - (int)(__float_as_uint(scale) >> 23); }      // scale = 2^-back
    __device__ __forceinline__ float back(float factor) const { return ldexpf(factor, back()); }
};

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
