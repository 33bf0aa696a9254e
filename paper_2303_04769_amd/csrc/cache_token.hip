// Attention of new tokens over a paged cache (gfx950).
//
// Bound by the cache's bytes: every key and value is read once, straight into the registers where the matrix instructions want it. A tile is as many keys as make 64
// bytes of one channel: 16 floats, 32 bfloat16, 64 codes. Lane 16 g + m loads 16 bytes at a time: of keys E (m / 4) + 4 b + m % 4 (E elements a load, b a
// result's number) the channels E g .. of a chunk of 4 E, and of channels 16 c + m the values of keys E g .. E g + E - 1. So a lane's scores, rows 4 g .. 4 g + 3 of every
// result b, are of the keys whose values it holds, E neighbours that stand in one page, and become the next product's right operand where they are.
// Sixteen rows -- new tokens times the query heads of a key head -- are the columns of the products; where there are fewer, keys share the columns out (SP).
//
// Codes are whole numbers below 128 and so bfloat16 numbers; queries and weights go in three bfloat16 parts of eight bits, which hold all of a float's 24 at its own
// range, so the products are those of floats: no power of two that a token's neighbours set, whatever the scales. A key's scale multiplies its score, a value's its weight.
//
// 64 streams of 2048 to 16384 tokens, 16 heads on 4 key heads of 64, 8 bits: 68 us for 316 MB, 4.6 TB/s (a large copy: 4.9), and 5 for the join. Where the cache is smaller, a
// workgroup's chain of dependent loads is what it takes: lengths, page numbers, keys and values, the waves' join (one round for each: 8 us).
#include "attn_tile.h"
#include "cache.h"

#include <climits>

namespace small {

namespace {

extern __shared__ __attribute__((aligned(16))) float token_lds[];

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ floatx4 mfma_bf16(uintx4 a, uintx4 b, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// The upper halves of two words.
__device__ __forceinline__ unsigned upper(unsigned lo, unsigned hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }
// Eight codes as bfloat16 numbers. (Taken apart here: behind the load, where the compiler would do it, it is a wait for the load, and four registers for every one.)
__device__ __forceinline__ uintx4 widened(unsigned lo, unsigned hi)
{
    uintx4 r;
    asm volatile("" : "+v"(lo), "+v"(hi));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = i < 2 ? lo : hi, at = 16 * (i & 1);
        r[i] = upper(__float_as_uint((float)(signed char)(w >> at)), __float_as_uint((float)(signed char)(w >> (at + 8))));
    }
    return r;
}
// Four floats in three parts of eight bits each, cut off, not rounded: their sum is the float.
struct Parts3 { unsigned p[3][2]; };
__device__ __forceinline__ Parts3 parts_of(floatx4 x)
{
    Parts3 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        unsigned h[2], m[2], l[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float v = x[2 * i + e];
            h[e] = __float_as_uint(v);
            const float rest = v - __uint_as_float(h[e] & 0xffff0000u);
            m[e] = __float_as_uint(rest);
            l[e] = __float_as_uint(rest - __uint_as_float(m[e] & 0xffff0000u));
        }
        r.p[0][i] = upper(h[0], h[1]);
        r.p[1][i] = upper(m[0], m[1]);
        r.p[2][i] = upper(l[0], l[1]);
    }
    return r;
}
__device__ __forceinline__ uintx4 words(const unsigned (&lo)[2], const unsigned (&hi)[2]) { return uintx4{lo[0], lo[1], hi[0], hi[1]}; }

// What stands so many bytes behind a place that all lanes share: below 2^32, so that an address takes one register.
template <typename T>
__device__ __forceinline__ T at_bytes(const T *base, unsigned bytes) { return *reinterpret_cast<const T *>(reinterpret_cast<const char *>(base) + bytes); }

// One row by one wave, key by key, for rows whose sums came out as NaN: in a product of tiles a key of weight zero contributes 0 * v, which is NaN where a token that
// the row does not see holds an infinite or NaN value. Slow, and reached only by caches that hold such values.
template <int KIND>
__device__ void attend_cached_row(const AttnArgs &a, const CacheArgs &c, const RowState &row, int n, int i, int key_head, int begin, int end, float (&o)[4], float &maximum, float &sum)
{
    const Scorer sc(a);
    const int lane = threadIdx.x & 63;
    const float *q = token_at(a.q, a.qs, n, i);
    const auto key = [&](size_t at, int d) -> float {
        if constexpr (KIND == SMALL_CACHE_F32) return reinterpret_cast<const float *>(c.keys)[at * c.Dk + d];
        else if constexpr (KIND == SMALL_CACHE_BF16) return (float)reinterpret_cast<const __bf16 *>(c.keys)[at * c.Dk + d];
        else return (float)reinterpret_cast<const signed char *>(c.keys)[at * c.Dk + d];
    };
    const auto value = [&](size_t page_row, int place, int d) -> float {
        const size_t at = page_row * c.D + ((size_t)d << c.shift) + place;
        if constexpr (KIND == SMALL_CACHE_F32) return reinterpret_cast<const float *>(c.values)[at];
        else if constexpr (KIND == SMALL_CACHE_BF16) return (float)reinterpret_cast<const __bf16 *>(c.values)[at];
        else return (float)reinterpret_cast<const signed char *>(c.values)[at];
    };
    const int inside = (1 << c.shift) - 1;
    const auto score = [&](int j) {
        const int page = j < end ? page_of(c, n, j) : -1;
        if (page < 0 || j >= row.bound) return -kInf;
        const size_t at = place_at(c, page, key_head, j & inside);
        float dot = 0.f;
        for (int d = 0; d < a.D; ++d) dot = fmaf(q[channel_at(a, a.qs, row.head * a.D + d)], key(at, d), dot);
        if constexpr (KIND == SMALL_CACHE_I8) dot *= c.key_scales[at];
        return sc.biased(sc.capped(dot), row, j, a.table ? j : 0, nullptr);
    };
    float top = -kInf;
    for (int j = begin + lane; j < end; j += 64) top = fmaxf(top, score(j));
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float ref = top == -kInf ? 0.f : top;
    float total = 0.f;
    o[0] = o[1] = o[2] = o[3] = 0.f;
    for (int j0 = begin; j0 < end; j0 += 64) {
        const float s = score(j0 + lane);
        const float p = s == -kInf ? 0.f : __builtin_amdgcn_exp2f(s - ref);
        total += p;
        for (unsigned long long left = __ballot(s != -kInf); left; left &= left - 1) {
            const int b = __ffsll((long long)left) - 1, j = j0 + b;
            float w = __shfl(p, b);
            const size_t page_row = place_at(c, page_of(c, n, j), key_head, 0);
            if constexpr (KIND == SMALL_CACHE_I8) w *= c.value_scales[page_row + (j & inside)];
            for (int x = 0; x < 4; ++x)
                if (lane + 64 * x < a.D) o[x] = fmaf(w, value(page_row, j & inside, lane + 64 * x), o[x]);
        }
    }
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    maximum = top;
    sum = total;
}

// The kernel's second argument likewise (late_args).
__device__ __forceinline__ CacheArgs late_cache_args()
{
    static_assert(sizeof(AttnArgs) % 8 == 0 && alignof(CacheArgs) <= 8, "one behind the other");
    auto at = (const __attribute__((address_space(4))) unsigned *)__builtin_amdgcn_kernarg_segment_ptr() + sizeof(AttnArgs) / 4;
    asm volatile("" : "+s"(at));
    unsigned words[sizeof(CacheArgs) / 4];
#pragma unroll
    for (unsigned i = 0; i < sizeof(CacheArgs) / 4; ++i) words[i] = at[i];
    return __builtin_bit_cast(CacheArgs, words);
}

// Waves a SIMD that the registers are to leave room for, and waves of a workgroup: as many workgroups run at a time.
constexpr int least_waves(int kind, int DT, int SP, int TR)
{
    if (TR == 2) return kind == SMALL_CACHE_F32 ? (DT <= 1 ? 4 : DT <= 3 ? 3 : 2) : DT <= 1 ? 3 : DT <= 4 ? 2 : 1;
    return kind == SMALL_CACHE_I8 ? (DT <= 4 && SP == 4 ? 3 : DT <= 5 || (DT <= 8 && SP > 1) ? 2 : 1) : DT <= 1 ? 5 : DT <= 3 ? 4 : DT == 4 ? 3 : DT <= 8 ? 2 : 1;
}
constexpr int group_waves(int DT) { return DT > 8 ? 2 : 4; }      // (their results fit 64 KB of LDS together)

// Who does what: a round is a tile for each wave of a workgroup, a stream's tokens are R rounds (one at least) of each tile of rows of each key head, and the rounds
// of all streams one behind the other are shared out evenly: streams differ in length, workgroups do not (64 streams of 2048 to 16384 tokens, 8 bits, in equal parts of each
// stream: 86 us; in pieces of equal length: 93; evenly: 73). Known only on the device, where each workgroup sums up the lengths.
struct Rounds {
    int *prefix;                  // LDS: rounds in front of each of the chunk's streams; their sum, [threads]; the waves' sums, 4; what was found
    int keys;                     // of a round, or of a piece of several
    int threads, units, all = 0, chunk = 0, before = 0, workgroups, each, more;
    __device__ __forceinline__ int of(const AttnArgs &a, int n) const { return max(1, (max(0, min(a.lengths[n], a.Sk)) + keys - 1) / keys); }
    // Sums of the streams from `first` on, a thread each.
    __device__ __forceinline__ int scan(const AttnArgs &a, int first)
    {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                         // (or what only this needs is computed once and kept in registers throughout)
        const int lane = tid & 63, wave = tid >> 6, n = first + tid;
        const int mine = n < a.N ? of(a, n) * units : 0;
        int sum = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const int below = __shfl_up(sum, d);
            sum += lane >= d ? below : 0;
        }
        lds_barrier();
        if (lane == 63) prefix[threads + 1 + wave] = sum;
        lds_barrier();
        int total = 0, under = 0;
        for (int w = 0; w < threads >> 6; ++w) {
            const int x = prefix[threads + 1 + w];
            under += w < wave ? x : 0;
            total += x;
        }
        prefix[tid] = under + sum - mine;
        if (tid == 0) prefix[threads] = total;
        lds_barrier();
        return __builtin_amdgcn_readfirstlane(total);
    }
    __device__ __forceinline__ Rounds(const AttnArgs &a, const CacheArgs &c, int round, int *lds) : prefix(lds), keys(round), threads(blockDim.x), units(a.head_sets * a.row_tiles)
    {
        for (int n = 0; n < a.N; n += threads) all += scan(a, n);
        int most = (all + c.workgroups - 1) / c.workgroups;      // rounds of the longest: no more workgroups than that takes, for the fewest parts
        // Few rounds each: in pieces of so many, if these are no more than the workgroups, so that none has to begin anew with another unit's queries and pages (16 streams of
        // two key heads, 3001 tokens at most: 24.0 us instead of 26.4). Looking for it costs the time of one more sum, 1 us, which for longer shares it does not bring in.
        if (most > 1 && most <= 4 && a.N <= threads && a.N * units <= c.workgroups) {
            keys = round * most;
            const int pieces = scan(a, 0);
            if (pieces <= c.workgroups) {
                all = pieces;
                most = 1;
            } else {
                keys = round;
                scan(a, 0);
            }
        }
        workgroups = (all + most - 1) / most;
        each = all / workgroups;
        more = all - each * workgroups;                       // the first so many have one more
    }
    __device__ __forceinline__ int begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int owner(int x) const
    {
        const int longer = more * (each + 1);
        return x < longer ? x / (each + 1) : more + (x - longer) / each;
    }
    // The stream that has round x, and the first round of its first unit.
    __device__ __forceinline__ int stream(const AttnArgs &a, int x, int *start)
    {
        if (a.N > threads) {
            if (x < before) { chunk = 0; before = 0; }
            int here = scan(a, chunk);
            while (x >= before + here) {
                before += here;
                chunk += threads;
                here = scan(a, chunk);
            }
        }
        const int y = x - before;
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        if (prefix[tid] <= y && y < prefix[tid + 1]) prefix[threads + 5] = tid;
        lds_barrier();
        const int found = __builtin_amdgcn_readfirstlane(prefix[threads + 5]);
        *start = before + __builtin_amdgcn_readfirstlane(prefix[found]);
        return chunk + found;
    }
};
constexpr int rounds_ints(int threads) { return threads + 6; }

// SP: into how many columns a row's keys of a tile are shared out, where there are at most 16 / SP rows. Column m then has row m mod (16 / SP), and of the tile's results only
// those of its share, m / (16 / SP): as if it were a row of its own, with a maximum, a sum and a result of its own, joined in the end. So the 16 columns
// of single tokens' products are not mostly empty lanes in all that lies between the products.
// TR: tiles of rows of a unit (two_tiles).
template <int KIND, int DT, int SP, bool ONE, int TR>
__global__ void __launch_bounds__(64 * group_waves(DT)) __attribute__((amdgpu_waves_per_eu(least_waves(KIND, DT, SP, TR)))) cache_token(AttnArgs args, CacheArgs cache_args)
{
    constexpr int B = cache_bytes(KIND), E = 16 / B, NB = E / 4, KT = 4 * E, NS = (16 * DT + KT - 1) / KT, DP = 16 * DT, H = E / 8 > 0 ? E / 8 : 1;
    constexpr int NV = NB / SP, R = 16 / SP, RU = R * TR;      // results of a lane that count, rows of a tile and of a unit
    constexpr int waves = group_waves(DT), KR = waves * KT;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    __shared__ int rounds_lds[rounds_ints(64 * waves)];
    Rounds rounds(args, cache_args, KR, rounds_lds);
    // (neighbours on one XCD: they have the tiles of rows that read the same keys)
    const int w_id = (int)xcd_contiguous(blockIdx.x, gridDim.x);
    if (w_id >= rounds.workgroups) return;
    int stream_start = 0, stream_rounds = 0, of_unit = 1, n = 0;
    for (int round = rounds.begin(w_id), stop = rounds.begin(w_id + 1); round < stop;) {
    const AttnArgs a = late_args();                            // (anew for every unit: what the compiler would compute of them once and keep does not fit the registers)
    const CacheArgs c = late_cache_args();
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int tid = 64 * wave + lane, m = lane & 15, g = lane >> 4;
    if (round >= stream_start + stream_rounds) {
        n = rounds.stream(a, round, &stream_start);
        of_unit = __builtin_amdgcn_readfirstlane(rounds.of(a, n));
        stream_rounds = of_unit * rounds.units;
    }
    const int unit = (round - stream_start) / of_unit, lo_round = round - stream_start - unit * of_unit, hi_round = min(of_unit, lo_round + stop - round);
    const int key_head = unit / a.row_tiles, tile = unit - key_head * a.row_tiles;
    const bool whole = lo_round == 0 && hi_round == of_unit;
    round += hi_round - lo_round;
    const int r0 = RU * tile, rows = min(RU, a.rows - r0), share = m / R;
    ImageMask im(a, n);
    im.len = __builtin_amdgcn_readfirstlane(im.len);           // (the same for all lanes, which only scalar loads would tell the compiler: what follows from them is scalar)
    im.prefix = 0;
    im.first = a.first ? __builtin_amdgcn_readfirstlane(im.first) : im.len - a.Sq;
    RowState row_of[TR];                                       // of this lane's column in each tile
    int place_of_row[TR];
#pragma unroll
    for (int t = 0; t < TR; ++t) {
        const int r = r0 + min(R * t + m % R, rows - 1), hh = a.by_Sq.div(r);
        place_of_row[t] = r - hh * a.Sq;
        row_of[t] = RowState(a, im, n, place_of_row[t], key_head * a.group + hh);
    }
    // keys up to the last one that a row of the unit can see, of these rounds
    const int last = a.by_Sq.div(r0) == a.by_Sq.div(r0 + rows - 1) ? r0 + rows - 1 - a.by_Sq.div(r0) * a.Sq : a.Sq - 1;
    const int hi = max(0, min(im.len, im.position(last) + 1));
    const int begin = min(hi, lo_round * rounds.keys), end = min(hi, hi_round * rounds.keys);
    const int step = waves * KT, first = begin + wave * KT;
    int left = first < end ? (end - first + step - 1) / step : 0;
    const int stride = a.slopes ? -step : step;
    int j0 = first + (a.slopes ? (left - 1) * step : 0);

    uintx4 kx[NB][NS], vx[DT];
    floatx4 ksc[NV], vsc[NV];                                  // scales of codes, of the keys of a lane's share
    // Pages of a lane's keys and of its values' keys: of tile j0, -1 where there is none. Their numbers come by scalar loads: these have a counter of their own, so that waiting
    // for them is not waiting for all keys and values asked for before. ONE: pages hold whole tiles, so that a tile's place is the same for all lanes, and a lane's offset
    // from it the same for all tiles; else a tile is in up to four pages.
    constexpr int NP = KT / 16;
    const auto *const table = (const __attribute__((address_space(4))) int *)(c.table + (size_t)n * c.per_stream);
    const int k_in = E * (m >> 2) >> c.shift, v_in = E * g >> c.shift, last_page = (end - 1) >> c.shift;
    int k_page = -1, v_page = -1, page0 = -1, page1 = -1, page2 = -1, page3 = -1;
    const auto ask_pages = [&](int j) {
        const int at = j >> c.shift;
        page0 = table[min(at, last_page)];
        if constexpr (!ONE && NP > 1) page1 = table[min(at + 1, last_page)];
        if constexpr (!ONE && NP > 2) {
            page2 = table[min(at + 2, last_page)];
            page3 = table[min(at + 3, last_page)];
        }
    };
    const auto page_in = [&](int in) {
        int page = page0;
        if constexpr (!ONE && NP > 1) page = in == 1 ? page1 : page;
        if constexpr (!ONE && NP > 2) page = in == 2 ? page2 : in == 3 ? page3 : page;
        return (unsigned)page < (unsigned)c.pages ? page : -1;
    };
    const auto at_lane = [](const void *base, unsigned bytes) { return *reinterpret_cast<const uintx4 *>(static_cast<const char *>(base) + bytes); };
    const auto fetch_k = [&](int j) {
        if constexpr (ONE) {
            const size_t at = place_at(c, max(0, v_page), key_head, j & ((1 << c.shift) - 1));
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int s = 0; s < NS; ++s)
                    kx[b][s] = at_lane(c.keys + (at + 4 * b) * (size_t)(c.Dk * B), (unsigned)(((E * (m >> 2) + (m & 3)) * c.Dk + min(E * g + KT * s, c.Dk - E)) * B));
            if constexpr (KIND == SMALL_CACHE_I8) {
#pragma unroll
                for (int b = 0; b < NV; ++b) ksc[b] = __builtin_bit_cast(floatx4, at_lane(c.key_scales + at, 4u * (unsigned)(E * g + 4 * (share * NV + b))));
            }
        } else {
            const int chunk = min(j + E * (m >> 2), (end - 1) & -E), place = chunk & ((1 << c.shift) - 1);
            const size_t at = place_at(c, max(0, k_page), key_head, place + (m & 3));
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int s = 0; s < NS; ++s) kx[b][s] = *reinterpret_cast<const uintx4 *>(c.keys + ((at + 4 * b) * c.Dk + min(E * g + KT * s, c.Dk - E)) * B);
            if constexpr (KIND == SMALL_CACHE_I8) {
                const int vplace = min(j + E * g, (end - 1) & -E) & ((1 << c.shift) - 1);
                const float *from = c.key_scales + place_at(c, max(0, v_page), key_head, vplace);
#pragma unroll
                for (int b = 0; b < NV; ++b) ksc[b] = *reinterpret_cast<const floatx4 *>(from + 4 * (share * NV + b));
            }
        }
    };
    const auto fetch_v = [&](int j) {
        const int place = (ONE ? j : min(j + E * g, (end - 1) & -E)) & ((1 << c.shift) - 1);
        const size_t page_row = place_at(c, max(0, v_page), key_head, 0);
        const char *from = c.values + (page_row * c.D + place) * B;
        if constexpr (ONE) {
#pragma unroll
            for (int d = 0; d < DT; ++d) vx[d] = at_lane(from, (unsigned)(((min(16 * d + m, c.D - 1) << c.shift) + E * g) * B));
        } else {
#pragma unroll
            for (int d = 0; d < DT; ++d) vx[d] = *reinterpret_cast<const uintx4 *>(from + ((size_t)min(16 * d + m, c.D - 1) << c.shift) * B);
        }
        if constexpr (KIND == SMALL_CACHE_I8) {
#pragma unroll
            for (int b = 0; b < NV; ++b)
                vsc[b] = ONE ? __builtin_bit_cast(floatx4, at_lane(c.value_scales + page_row + place, 4u * (unsigned)(E * g + 4 * (share * NV + b))))
                             : *reinterpret_cast<const floatx4 *>(c.value_scales + page_row + place + 4 * (share * NV + b));
        }
    };
    if (left) {
        ask_pages(j0);
        k_page = page_in(k_in);
        v_page = page_in(v_in);
        fetch_k(j0);
        fetch_v(j0);
    }
    // queries, times what makes their products scores (or, with a cap, what the tanh is taken of): floats, or their parts
    floatx4 qf[TR][KIND == SMALL_CACHE_F32 ? DT : 1];
    Parts3 qp[TR][KIND == SMALL_CACHE_F32 ? 1 : 2 * NS * H];
#pragma unroll
    for (int t = 0; t < TR; ++t) {
        const float *token = token_at(a.q, a.qs, n, place_of_row[t]);
        const float in = a.cap > 0.f ? a.scale / a.cap : a.scale * kLog2e;
        const auto quad = [&](int d) { return (a.vec ? load_quad<true>(a, a.qs, token, row_of[t].head * a.D, d) : load_quad<false>(a, a.qs, token, row_of[t].head * a.D, d)) * in; };
        if constexpr (KIND == SMALL_CACHE_F32) {
#pragma unroll
            for (int s = 0; s < DT; ++s) qf[t][s] = quad(16 * s + 4 * g);
        } else {
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int h = 0; h < 2 * H; ++h) qp[t][2 * H * s + h] = parts_of(quad(KT * s + E * g + 4 * h));
        }
    }
    float far_lo[TR], far_hi[TR], sum[TR] = {};
    floatx4 o[TR][DT] = {};
#pragma unroll
    for (int t = 0; t < TR; ++t) {
        far_lo[t] = a.table ? bias_gather(a, row_of[t].head, 0) : 0.f;
        far_hi[t] = a.table ? bias_gather(a, row_of[t].head, 2 * a.reach) : 0.f;
    }
    Reference top[TR];
#pragma unroll
    for (int t = 0; t < TR; ++t) top[t] = Reference(a, row_of[t], begin, end);
    if (left > 1) ask_pages(j0 + stride);
    for (; left; --left, j0 += stride) {
        const int value0 = j0 + E * g, key0 = value0 + 4 * NV * share;        // of this lane's values, and of its scores: key0 + 4 b + e
        const bool no_page = v_page < 0;
        // a learned bias: all buckets are asked for, then all biases -- unless the tile's keys are all at one end of the reach, as most of a long cache is
        bool near[TR];
        float far[TR], bias[TR][NV][4];
#pragma unroll
        for (int t = 0; t < TR; ++t) {
            const RowState &row = row_of[t];
            near[t] = false;
            far[t] = 0.f;
            if (!a.table) continue;
            const bool all_lo = __all(j0 + KT - 1 - row.code <= -a.reach), all_hi = __all(j0 - row.code >= a.reach);
            near[t] = !all_lo && !all_hi;
            far[t] = all_lo ? far_lo[t] : all_hi ? far_hi[t] : 0.f;
            if (near[t]) {
                int bucket[NV][4];
#pragma unroll
                for (int b = 0; b < NV; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bucket[b][e] = at_bytes(a.bucket, 4u * (unsigned)offset_at(a, key0 + 4 * b + e, row.code));
#pragma unroll
                for (int b = 0; b < NV; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bias[t][b][e] = at_bytes(a.table, 4u * (unsigned)(row.head * a.buckets + max(0, min(bucket[b][e], a.buckets - 1))));
            }
        }
        floatx4 all[TR][NB] = {};
#pragma unroll
        for (int x = 0; x < NS; ++x)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if constexpr (KIND == SMALL_CACHE_F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int t = 0; t < TR; ++t) all[t][b] = mfma(__uint_as_float(kx[b][x][e]), qf[t][x][e], all[t][b]);
                } else {
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        uintx4 k = kx[b][x];
                        if constexpr (KIND == SMALL_CACHE_I8) k = widened(kx[b][x][2 * h], kx[b][x][2 * h + 1]);
#pragma unroll
                        for (int p = 2; p >= 0; --p)
#pragma unroll
                            for (int t = 0; t < TR; ++t) all[t][b] = mfma_bf16(k, words(qp[t][2 * (H * x + h)].p[p], qp[t][2 * (H * x + h) + 1].p[p]), all[t][b]);
                    }
                }
            }
        floatx4 scores[TR][NV];
#pragma unroll
        for (int t = 0; t < TR; ++t)
#pragma unroll
            for (int b = 0; b < NV; ++b) {
                scores[t][b] = all[t][b];
#pragma unroll
                for (int x = 1; x < SP; ++x) scores[t][b] = share == x ? all[t][x * NV + b] : scores[t][b];
                if constexpr (KIND == SMALL_CACHE_I8) scores[t][b] *= ksc[b];
            }
        if (left > 1) {
            const int v_now = v_page;
            k_page = page_in(k_in);
            v_page = page_in(v_in);                            // (key scales stand at the values' keys)
            fetch_k(j0 + stride);
            v_page = v_now;
        }
        if (KIND != SMALL_CACHE_I8 && (j0 + KT > end || __any(no_page))) {       // what stands behind the last key, or in no page of the stream's, becomes zeros
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (KIND == SMALL_CACHE_F32) vx[d][x] = ((value0 + x < end) & !no_page) ? vx[d][x] : 0u;
                    else vx[d][x] &= no_page ? 0u : value0 + 2 * x + 1 < end ? 0xffffffffu : value0 + 2 * x < end ? 0xffffu : 0u;
                }
        }
#pragma unroll
        for (int t = 0; t < TR; ++t) {
            const RowState &row = row_of[t];
            floatx4(&s)[NV] = scores[t];
            floatx4 weight[NV];                                // of codes' values, zero where the row does not see them
            if constexpr (KIND == SMALL_CACHE_I8) {
#pragma unroll
                for (int b = 0; b < NV; ++b) weight[b] = vsc[b];
            }
            const float base = far[t] - top[t].at;
            const int bound = min(row.bound, end);
            const bool all_seen = __all((j0 + KT <= bound) & !no_page);
            const auto seen = [&](int b, int e) { return (key0 + 4 * b + e < bound) & !no_page; };
            if (a.cap > 0.f) {
                if (!all_seen)                                 // (the largest score chooses how the cap is computed, in other last bits: not one of a key that is not there)
#pragma unroll
                    for (int b = 0; b < NV; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][e] = seen(b, e) ? s[b][e] : 0.f;
                tanh_all(s);
                const float out = a.cap * kLog2e;
#pragma unroll
                for (int b = 0; b < NV; ++b) s[b] *= out;
            }
            if (a.slopes) {
                const float from = (float)(row.p - key0);
#pragma unroll
                for (int b = 0; b < NV; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][e] += fmaf(-row.slope, fabsf(from - (float)(4 * b + e)), base);
            } else {
#pragma unroll
                for (int b = 0; b < NV; ++b) s[b] += base;
            }
            if (near[t])
#pragma unroll
                for (int b = 0; b < NV; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][e] += bias_log2(bias[t][b][e]);
            if (!all_seen) {
#pragma unroll
                for (int b = 0; b < NV; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[b][e] = seen(b, e) ? s[b][e] : -kInf;
                        if constexpr (KIND == SMALL_CACHE_I8) weight[b][e] = seen(b, e) ? weight[b][e] : 0.f;        // (the scale of a hidden token may be anything)
                    }
            }
            raise_top(s, top[t], sum[t], o[t]);
#pragma unroll
            for (int b = 0; b < NV; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[b][e] = __builtin_amdgcn_exp2f(s[b][e]);
                    sum[t] += s[b][e];
                }
            if constexpr (KIND == SMALL_CACHE_F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[t][d] = mfma(__uint_as_float(vx[d][e]), s[0][e], o[t][d]);
            } else {
                Parts3 w[NV];
#pragma unroll
                for (int b = 0; b < NV; ++b) {
                    if constexpr (KIND == SMALL_CACHE_I8) s[b] *= weight[b];
                    w[b] = parts_of(s[b]);
                }
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    uintx4 p[3];                                   // (zeros at the other shares' keys)
#pragma unroll
                    for (int x = 0; x < 3; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int b = 2 * h + y / 2;
                            p[x][y] = SP == 1 || share == b / NV ? w[b % NV].p[x][y & 1] : 0u;
                        }
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        uintx4 v = vx[d];
                        if constexpr (KIND == SMALL_CACHE_I8) v = widened(vx[d][2 * h], vx[d][2 * h + 1]);
#pragma unroll
                        for (int x = 2; x >= 0; --x) o[t][d] = mfma_bf16(v, p[x], o[t][d]);
                    }
                }
            }
        }
        if (left > 1) {
            v_page = page_in(v_in);
            fetch_v(j0 + stride);
            if (left > 2) ask_pages(j0 + 2 * stride);
        }
    }
    float most[TR];
#pragma unroll
    for (int t = 0; t < TR; ++t) {
        sum[t] = column_sum(sum[t]);
        most[t] = top[t].maximum();
    }
    if constexpr (SP > 1) {                                    // a row's shares: columns 16 / SP apart, in the same sixteen lanes
        static_assert(TR == 1, "rows that fill the columns have no shares");
        float all = most[0];
        all = fmaxf(all, __int_as_float(dpp_of<0x128>(__float_as_int(all))));            // row_ror:8
        if constexpr (SP == 4) all = fmaxf(all, __int_as_float(dpp_of<0x124>(__float_as_int(all))));
        const float w = sum[0] == 0.f ? 0.f : __builtin_amdgcn_exp2f(most[0] - all);            // (a share that saw no key)
        const auto over = [&](float x) {
            x = sum[0] == 0.f ? 0.f : x * w;
            x += __int_as_float(dpp_of<0x128>(__float_as_int(x)));
            if constexpr (SP == 4) x += __int_as_float(dpp_of<0x124>(__float_as_int(x)));
            return x;
        };
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[0][d][e] = over(o[0][d][e]);
        sum[0] = over(sum[0]);
        most[0] = all;
    }

    // join the waves: [wave][row][DP] and [wave][row] (maximum, sum), a tile of rows at a time
    const AttnArgs z = late_args();
    const CacheArgs zc = late_cache_args();
    const size_t all_units = (size_t)n * rounds.units + unit, unit_part = (w_id + all_units) * RU;       // (workgroups and units both only grow: a place of its own for each pair)
    if (zc.units && lo_round == 0 && tid == 0) zc.units[all_units] = int2{w_id, rounds.owner(round - (hi_round - lo_round) + of_unit - 1)};      // who has parts of it, for the join
    constexpr int LP = DP + 4;                                 // (rows of lanes that write at a time in different banks)
#pragma clang loop unroll(disable)
    for (int t = 0; t < TR; ++t) {
        const int r0 = RU * tile + R * t, rows = min(R, z.rows - r0);
        if (rows <= 0) break;
        const size_t part = unit_part + R * t;
        float *const lo_ = token_lds;
        float2 *const ml = reinterpret_cast<float2 *>(token_lds + waves * rows * LP);
        int *const flags = reinterpret_cast<int *>(ml + waves * rows);
        const auto put = [&](const floatx4(&of)[DT], float maximum, float total) {
            const int mine = wave * rows + m;
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<floatx4 *>(lo_ + mine * LP + 16 * d + 4 * g) = of[d];
            if (g == 0) ml[mine] = float2{maximum, total};
        };
        if (m < rows) {
            if (t == 0) put(o[0], most[0], sum[0]);
            else put(o[TR - 1], most[TR - 1], sum[TR - 1]);
        }
        if (tid < 17) flags[tid] = 0;                             // of rows, and of any
        lds_barrier();
        constexpr int QD = DP / 4;
        for (int e = tid; e < rows * QD; e += 64 * waves) {
            const int rr = e / QD, d = (e - rr * QD) * 4;
            float all = -kInf, total = 0.f;
#pragma unroll 4
            for (int w = 0; w < waves; ++w) all = fmaxf(all, ml[w * rows + rr].x);
            const float ref = all == -kInf ? 0.f : all;
            floatx4 y = {};
#pragma unroll 4
            for (int w = 0; w < waves; ++w) {
                const float2 p = ml[w * rows + rr];
                const floatx4 w4 = *reinterpret_cast<const floatx4 *>(lo_ + (w * rows + rr) * LP + d);
                const float f = __builtin_amdgcn_exp2f(p.x - ref);
                total += p.y == 0.f ? 0.f : f * p.y;
#pragma unroll
                for (int x = 0; x < 4; ++x) y[x] += p.y == 0.f ? 0.f : f * w4[x];       // (a wave that saw no key)
            }
            if (d < z.D && (y.x != y.x || y.y != y.y || y.z != y.z || y.w != y.w)) flags[rr] = flags[16] = 1;
            const int h2 = z.by_Sq.div(r0 + rr), i2 = r0 + rr - h2 * z.Sq, head2 = key_head * z.group + h2;
            if (!whole && z.D % 4 == 0) {
                if (d < z.D) *reinterpret_cast<floatx4 *>(z.part_o + (part + rr) * z.D + d) = y;
                if (d == 0) z.part_ml[part + rr] = float2{all, total};
            } else if (!whole) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    if (d + x < z.D) z.part_o[(part + rr) * z.D + d + x] = y[x];
                if (d == 0) z.part_ml[part + rr] = float2{all, total};
            } else {
                const floatx4 all_of = total == 0.f ? floatx4{} : y * (1.f / total);
                float *token = const_cast<float *>(token_at(z.o, z.os, n, i2));
                if (z.vec) store_quad<true>(z, z.os, token, head2 * z.D, d, all_of);
                else store_quad<false>(z, z.os, token, head2 * z.D, d, all_of);
                if (z.lse && d == 0) z.lse[((size_t)n * z.heads + head2) * z.Sq + i2] = total == 0.f ? -kInf : (all + __builtin_amdgcn_logf(total)) * kLn2;
            }
        }
        lds_barrier();
        if (!__builtin_amdgcn_readfirstlane(flags[16])) {
            lds_barrier();                                         // (what the join read is free)
            continue;
        }
        __syncthreads();                                           // (stores of these rows have come to pass)
        for (int rr = wave; rr < rows; rr += waves) {
            if (!flags[rr]) continue;
            const int h2 = z.by_Sq.div(r0 + rr), i2 = r0 + rr - h2 * z.Sq, head2 = key_head * z.group + h2;
            // (a query that is not finite itself has no other result, and may be padding)
            const float *query = token_at(z.q, z.qs, n, i2);
            bool fine = true;
            for (int d = lane; d < z.D; d += 64) fine &= fabsf(query[channel_at(z, z.qs, head2 * z.D + d)]) < kInf;
            if (!__all(fine)) continue;
            const RowState again(z, im, n, i2, head2);
            float y[4], most, total;
            attend_cached_row<KIND>(z, zc, again, n, i2, key_head, begin, end, y, most, total);
            const float inv = total == 0.f ? 0.f : 1.f / total;
            for (int x = 0; x < 4; ++x) {
                const int d = lane + 64 * x;
                if (d >= z.D) continue;
                if (!whole) z.part_o[(part + rr) * z.D + d] = y[x];
                else const_cast<float *>(token_at(z.o, z.os, n, i2))[channel_at(z, z.os, head2 * z.D + d)] = total == 0.f ? 0.f : y[x] * inv;
            }
            if (lane) continue;
            if (!whole) z.part_ml[part + rr] = float2{most, total};
            else if (z.lse) z.lse[((size_t)n * z.heads + head2) * z.Sq + i2] = total == 0.f ? -kInf : (most + __builtin_amdgcn_logf(total)) * kLn2;
        }
        __syncthreads();                                           // (what the join read is free)
    }
    }
}

// Rows whose rounds more than one workgroup had: their parts joined, a workgroup for each row. (Who had them stands in the workspace: summing up the lengths again took it
// 7.0 us instead of 5.9, 64 streams of 16 heads.)
__global__ void __launch_bounds__(256) cache_token_join(AttnArgs a, CacheArgs c, int most_rows)
{
    __shared__ float sums[4][256], all[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int by_head = c.by_rows.div((int)blockIdx.x), r = (int)blockIdx.x - by_head * a.rows, n = a.by_sets.div(by_head), key_head = by_head - n * a.head_sets;
    const int tile = r / most_rows;
    const size_t unit = (size_t)by_head * a.row_tiles + tile;
    const int from = c.units[unit].x, to = c.units[unit].y;
    if (from == to) return;
    const size_t step = most_rows, first = (from + unit) * most_rows + (r - tile * most_rows);
    float top = -kInf, sum = 0.f, o[4] = {};
    // (a wave's first part is asked for before the largest maximum is known)
    float2 w = {};
    float y[4] = {};
    const auto fetch = [&](int s) {
        w = a.part_ml[first + s * step];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (lane + 64 * k < a.D) y[k] = a.part_o[(first + s * step) * a.D + lane + 64 * k];
    };
    const int parts = to - from + 1;
    if (wave < parts) fetch(wave);
#pragma unroll 4
    for (int s = lane; s < parts; s += 64) top = fmaxf(top, a.part_ml[first + s * step].x);
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float ref = top == -kInf ? 0.f : top;
#pragma unroll 4
    for (int s = wave; s < parts; s += 4) {
        if (s != wave) fetch(s);
        const float x = w.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(w.x - ref);      // (a part that saw no key)
        sum = fmaf(x, w.y, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] += w.y == 0.f ? 0.f : x * y[k];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[wave][lane + 64 * k] = o[k];
    if (lane == 0) all[wave] = sum;
    __syncthreads();
    const int d = threadIdx.x;
    sum = (all[0] + all[1]) + (all[2] + all[3]);
    const int hh = a.by_Sq.div(r), i = r - hh * a.Sq, head = key_head * a.group + hh;
    if (d < a.D) {
        const float y = (sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]);
        const_cast<float *>(token_at(a.o, a.os, n, i))[channel_at(a, a.os, head * a.D + d)] = sum == 0.f ? 0.f : y * (1.f / sum);
    }
    if (a.lse && d == 0) a.lse[((size_t)n * a.heads + head) * a.Sq + i] = sum == 0.f ? -kInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Rows of a tile: as many as leave each a column of its own, or fewer that share the columns out.
constexpr int token_shares(int kind, int rows)
{
    return kind == SMALL_CACHE_I8 ? (rows <= 4 ? 4 : rows <= 8 ? 2 : 1) : kind == SMALL_CACHE_BF16 && rows <= 8 ? 2 : 1;
}
int token_tiles(int D)
{
    for (const int dt : {1, 2, 3, 4, 5, 6, 8})
        if (D <= 16 * dt) return dt;
    return 16;
}

// Two tiles of rows in a unit: a tile of keys and values is loaded once for both. They halve the loads of calls with three tiles or more and leave room for fewer waves (8 streams
// of 4096 tokens, 56 rows: floats of 64 channels 50 -> 40 us, bfloat16 33 -> 26 and of 128 channels 43 -> 35). With two tiles the waves lost cost as much but for small heads of
// bfloat16 (32 streams, 20 rows: floats 36 -> 42, bfloat16 25.5 -> 24, of 128 channels 41 -> 47), and codes taken apart need the registers themselves (56 rows 25 -> 28.5).
constexpr bool two_tiles(int kind, int DT, int rows)
{
    return kind == SMALL_CACHE_F32 ? DT <= 6 && rows > 32 : kind == SMALL_CACHE_BF16 && (DT <= 4 ? rows > 16 : DT <= 8 && rows > 32);
}

template <int KIND, int SP, bool ONE, int TR>
hipError_t token_form(const AttnArgs &a, const CacheArgs &c, hipStream_t s)
{
    const int rows = a.rows < 16 / SP ? a.rows : 16 / SP;
    switch (token_tiles(a.D)) {
#define TOKEN(dt) \
    case dt: \
        hipLaunchKernelGGL((cache_token<KIND, dt, SP, ONE, (two_tiles(KIND, dt, INT_MAX) ? TR : 1)>), dim3((unsigned)c.workgroups), dim3(64 * group_waves(dt)), (size_t)group_waves(dt) * rows * (16 * dt + 6) * 4 + 80, s, a, c); \
        break;
        TOKEN(1) TOKEN(2) TOKEN(3) TOKEN(4) TOKEN(5) TOKEN(6) TOKEN(8) TOKEN(16)
#undef TOKEN
    }
    return hipGetLastError();
}
template <int KIND, int SP, int TR>
hipError_t token_pages(const AttnArgs &a, const CacheArgs &c, hipStream_t s)
{
    if constexpr (KIND != SMALL_CACHE_F32)
        if ((1 << c.shift) < 64 / cache_bytes(KIND)) return token_form<KIND, SP, false, TR>(a, c, s);
    return token_form<KIND, SP, true, TR>(a, c, s);
}

}  // namespace

TokenShape token_shape(int kind, int D, int rows)
{
    const int shares = token_shares(kind, rows), dt = token_tiles(D), waves = group_waves(dt), tiles = two_tiles(kind, dt, rows) ? 2 : 1;
    return TokenShape{16 / shares * tiles, waves * 64 / cache_bytes(kind), least_waves(kind, dt, shares, tiles) * 4 / waves};
}

hipError_t launch_cache_token(const AttnArgs &a, const CacheArgs &c, bool joined, hipStream_t s)
{
    const int shares = token_shares(c.kind, a.rows), two = two_tiles(c.kind, token_tiles(a.D), a.rows);
    hipError_t e;
    switch (c.kind) {
    case SMALL_CACHE_F32: e = two ? token_pages<SMALL_CACHE_F32, 1, 2>(a, c, s) : token_pages<SMALL_CACHE_F32, 1, 1>(a, c, s); break;
    case SMALL_CACHE_BF16:
        e = two ? token_pages<SMALL_CACHE_BF16, 1, 2>(a, c, s) : shares == 2 ? token_pages<SMALL_CACHE_BF16, 2, 1>(a, c, s) : token_pages<SMALL_CACHE_BF16, 1, 1>(a, c, s);
        break;
    default:
        e = shares == 4 ? token_pages<SMALL_CACHE_I8, 4, 1>(a, c, s) : shares == 2 ? token_pages<SMALL_CACHE_I8, 2, 1>(a, c, s) : token_pages<SMALL_CACHE_I8, 1, 1>(a, c, s);
    }
    if (e != hipSuccess || !joined) return e;
    const TokenShape shape = token_shape(c.kind, a.D, a.rows);
    hipLaunchKernelGGL(cache_token_join, dim3((unsigned)((long)a.N * a.head_sets * a.rows)), dim3(256), 0, s, a, c, shape.rows);
    return hipGetLastError();
}

}  // namespace small
