// Softmax attention over the pages of a key/value cache: tent_kv_attend, and with kTree tent_kv_attend_tree, whose rows see of each other what
// their masks name (struct Sight).
//
//   s_rt = scale q_r . k_t,  m_r = max_t s_rt,  l_r = sum_t exp(s_rt - m_r),  o_r = sum_t exp(s_rt - m_r) v_t / l_r
//
// in one pass over the tokens with the running maximum and sum.  The query heads that share a head of the cache and the rows
// of a sequence are one list of "lines" (line = row * group + head in the group), so the cache is read once for all of them.
// Both kernels compute the transposed products S^T = K Q^T and O^T = V^T P^T: a lane then holds scores, weights and sums of
// one line only, and the weights come out of the first product in the lanes where the second one wants them.  V is read
// from LDS with the transposing read; K's rows may enter the first product in any order, which is chosen so that a lane gets
// the tokens that its part of the second product sums over.
//
//   narrow_kernel  up to 64 lines: 16 lines to a matrix tile, each wave takes tokens of its own, the cache streams from HBM
//                  through registers; bound by its loads
//   wide_kernel    more lines: 128 to a workgroup, 32 to a wave, tiles of 64 tokens in LDS for all four waves; bound by the
//                  matrix units and the softmax's vector work beside them.  For trees of 33 to 64 lines 64 to a workgroup, of
//                  which two waves take 32, each half of a tile's tokens
//
// Measured, 32 heads on 8 of 128 dimensions: 32 rows over 2k-8k tokens each in 4 bits 44 us and 5 for the join (152 MB, 3.4 TB/s; no more
// than that is read from memory), over 16-bit pages 114 (573 MB, 5.0 TB/s); 8 rows over 100k-131k tokens in 4 bits 69 + 8 us (256 MB, 3.7
// TB/s); two prompts of 4k tokens 297 us, call and all (890 TFLOP/s, a large matrix product reaches 1251); 1128 rows in three chunks
// behind 6k-16k tokens in 4 bits 330 us, of it 17 for the join.
//
// Where lines are few and contexts long the tokens are split over workgroups; their parts (largest score, sum, output, all in
// 32 bits) go through the workspace and are joined by join_kernel.
//
// Scores, maxima, sums and outputs are in 32 bits.  Weights alone are rounded to the 16-bit type, as the second product takes such, and
// their sum takes them before that.  It costs a third more error (bf16, against 64 bits: 2.2e-3 of the outputs' norm, where rounding the
// outputs costs 1.65e-3 by itself).  A second product with what the rounding leaves ends it: at 52.2 us instead of 50.4 for the 32 rows in 4
// bits, 404 instead of 309 for the prompts, and 420 instead of 334 for the chunks, which is more than it is worth to a result of 16 bits.
#pragma once

#include "kv_elem.h"

namespace tent {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The maximum that weights are taken against may lag behind the true one by a factor of 2^8: sums and products are in 32 bits
// and lose nothing by it, and most tiles then need no rescaling.
constexpr float kLag = 8.f;
// The most that weights are taken against.  Scores of plus infinity stay infinite weights against it, and so the sum and the
// logsumexp are infinite and the outputs NaN; against infinity they would be NaN, and not told from a score that is.
constexpr float kMost = 3.402823466e38f;
// Joined parts are added up as 2^-11 each, and there are at most 1536: sums of finite parts are finite.
constexpr float kPart = 0x1p-11f;
constexpr int32_t kStep = 32;          // splits and the tokens that a workgroup begins with are multiples of it

struct AttendArgs {
    KvCache c;
    tent_kv_batch b;
    const uint8_t* q;
    uint8_t* out;
    float* lse;
    uint64_t q_stride, out_stride;     // bytes
    float* part_o;                     // [n_rows * q_heads][n_splits][D], or null: one split
    float* part_ml;                    // [n_rows * q_heads][n_splits][2]
    uint32_t q_heads, group, window, all;
    float to_log2;                     // scale * log2(e)
    uint32_t n_splits, split_tokens;   // tokens of a split: a multiple of 128
    uint32_t line_tiles;               // workgroups over the lines of a sequence and head
    uint32_t first;                    // of the launch's workgroups
    const uint64_t* masks;             // a tree's: [n_rows][mask_stride], bit j: the row sees row j of its sequence
    uint32_t mask_stride;
};

// The arguments of either kernel (each has this one structure), read anew: what hardly any call comes to should not keep them in
// registers all along.
__device__ __forceinline__ const AttendArgs& args_again()
{
    typedef const __attribute__((address_space(4))) AttendArgs* ArgsAt;
    ArgsAt at = (ArgsAt)__builtin_amdgcn_kernarg_segment_ptr();
    __asm__ volatile("" : "+s"(at));
    return *(const AttendArgs*)at;
}

// ---- what both kernels share ---------------------------------------------------------------------
// What a row sees.  In a tree (kTree) that is the context, from `lo` on, and of the rows those that its mask names; else a span.
template <bool kTree>
struct Sight : KvSpan {
    __device__ __forceinline__ bool sees(int32_t t) const { return t >= lo && t < hi; }
    __device__ __forceinline__ int32_t end() const { return hi; }
};
template <>
struct Sight<true> : KvTreeSpan {
    const uint64_t* mask;
    __device__ __forceinline__ uint64_t word(int32_t i) const { return i < words ? dev_load<uint64_t>(mask + i) : 0; }
    __device__ __forceinline__ bool sees(int32_t t) const { return t >= 0 && t < len && (t < base ? t >= lo : (word((t - base) >> 6) >> ((t - base) & 63) & 1u) != 0); }
    __device__ __forceinline__ int32_t end() const { return len; }
    // Which of the 64 tokens from t0 on it sees.
    __device__ __forceinline__ uint64_t bits(int32_t t0) const
    {
        return kv_tree_bits(*this, t0, [&](int32_t i) { return word(i); });
    }
};
template <bool kTree>
__device__ __forceinline__ Sight<kTree> sight(const AttendArgs& g, const KvSeq& q, int32_t row)
{
    if constexpr (kTree) {
        Sight<true> s;
        s.mask = g.masks + (uint64_t)(q.row0 + row) * g.mask_stride;
        s.words = (q.rows + 63) >> 6;
        int32_t deep = 0;                                                // rows that it sees
        if (g.window)
            for (int32_t i = 0; i < s.words; ++i) deep += __popcll(dev_load<uint64_t>(s.mask + i) & (i + 1 < s.words || !(q.rows & 63) ? ~0ull : ~(~0ull << (q.rows & 63))));
        (KvTreeSpan&)s = kv_tree_span(q.rows, q.len, g.window, deep);
        return s;
    } else {
        Sight<false> s;
        (KvSpan&)s = kv_span(row, q.rows, q.len, g.window, g.all);
        return s;
    }
}
// The tokens that rows `first` to `last` of a sequence all see one after the other: all of them from lo to hi.
template <bool kTree>
__device__ __forceinline__ KvSpan seen_by_rows(const AttendArgs& g, const KvSeq& q, int32_t first, int32_t last)
{
    if constexpr (kTree) {
        const KvTreeSpan s = kv_tree_span(q.rows, q.len, g.window, q.rows);
        return KvSpan{s.lo, s.base};
    } else {
        return KvSpan{kv_span(last, q.rows, q.len, g.window, g.all).lo, kv_span(first, q.rows, q.len, g.window, g.all).hi};
    }
}
// The tokens that any of the rows `first` to `last` sees: none in front of lo, none from hi on.
template <bool kTree>
__device__ __forceinline__ KvSpan seen_by_any(const AttendArgs& g, const KvSeq& q, int32_t first, int32_t last)
{
    if constexpr (kTree) return KvSpan{kv_tree_span(q.rows, q.len, g.window, 0).lo, q.len};
    else return KvSpan{kv_span(first, q.rows, q.len, g.window, g.all).lo, kv_span(last, q.rows, q.len, g.window, g.all).hi};
}

// A sequence's splits begin at the first token that its first row sees, rounded down to a whole step.
template <bool kTree>
__device__ __forceinline__ int32_t splits_from(const AttendArgs& g, const KvSeq& q)
{
    return seen_by_any<kTree>(g, q, 0, 0).lo & ~(kStep - 1);
}
template <bool kTree>
__device__ __forceinline__ uint32_t splits_of(const AttendArgs& g, const KvSeq& q)
{
    const uint32_t span = (uint32_t)(q.len - splits_from<kTree>(g, q));
    const uint32_t n = (span + g.split_tokens - 1) / g.split_tokens;
    return n < 1 ? 1 : n;
}

// The tokens that a workgroup goes through: those that its lines see, within its split.
struct Range { int32_t lo, hi; };
template <bool kTree>
__device__ __forceinline__ Range token_range(const AttendArgs& g, const KvSeq& q, int32_t first_line, int32_t last_line, uint32_t split)
{
    const KvSpan any = seen_by_any<kTree>(g, q, first_line / (int32_t)g.group, last_line / (int32_t)g.group);
    const int64_t lo = (int64_t)splits_from<kTree>(g, q) + (int64_t)split * g.split_tokens, hi = lo + g.split_tokens;
    const int32_t first = any.lo & ~(kStep - 1);
    return Range{first > lo ? first : (int32_t)lo, any.hi < hi ? any.hi : (int32_t)hi};
}

// Place of a token's row of this head in a pool: bytes to its values, or to its codes and its scales.
template <int kBits>
struct RowAt;
template <>
struct RowAt<16> { uint64_t row; };
template <>
struct RowAt<4> { uint64_t row, scale; };

template <int D, int kBits>
__device__ __forceinline__ RowAt<kBits> row_at(const KvCache& c, uint32_t page, uint32_t token, uint32_t head)
{
    const uint64_t at = page * c.page_stride;
    const uint32_t r = (token & ((1u << c.page_shift) - 1u)) * c.heads + head;
    if constexpr (kBits == 16) return RowAt<16>{at + (uint64_t)r * (D * 2)};
    else return RowAt<4>{at + (uint64_t)r * (D / 2), at + ((uint64_t)(c.heads * (D / 2)) << c.page_shift) + (uint64_t)r * (D / 32)};
}

// Largest value, and sum, over the lanes that hold one line: lane ^ 32 and, where 16 lines make a tile, lane ^ 16.
__device__ __forceinline__ float max_over32(float x)
{
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
__device__ __forceinline__ float max_over16(float x)
{
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
}
// A value that all lanes of a wave have, for branches that the wave takes as a whole.
__device__ __forceinline__ uint64_t same_in_wave(uint64_t x)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}
__device__ __forceinline__ float sum_over32(float x) { return x + __shfl_xor(x, 32, 64); }
__device__ __forceinline__ float sum_over16(float x) { return x + __shfl_xor(x, 16, 64); }

// The root of 2^(a - b), where a is what weights were taken against before and b what they are taken against now; nothing yet is
// 0.  Sums are multiplied by it twice: the power itself may be below the least normal number where the product is not.
__device__ __forceinline__ float rescale(float a, float b) { return a == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(0.5f * (a - b)); }

// Where a token's row has its 16-byte chunk `chunk` in LDS (as a chunk number): eight chunks cover all banks once, and eight
// lanes of a 16-byte access, or 32 of a transposing one, go at a time.  Blocks of 32 dimensions (chunk / 4) and, by the token,
// the chunks' lowest three bits are mixed so that each of these is spread evenly: rows written by lanes side by side (four
// chunks apart from 4-bit pages, one apart from 16-bit ones), K read by lanes of one token each, V's transposing reads of four
// tokens by 16 or 32 dimensions.
template <int D>
__device__ __forceinline__ constexpr uint32_t spread(uint32_t chunk)
{
    return D == 64 ? chunk : (chunk & 16u) | (chunk & 2u) << 2 | (chunk >> 1 & 6u) | (chunk & 1u);
}
template <int D>
__device__ __forceinline__ constexpr uint32_t gather(uint32_t place)     // the inverse
{
    return D == 64 ? place : (place & 16u) | (place & 6u) << 1 | (place >> 2 & 2u) | (place & 1u);
}
__device__ __forceinline__ uint32_t k_swap(uint32_t t) { return t & 7u; }
__device__ __forceinline__ uint32_t v_swap(uint32_t t) { return (t & 1u) * 5u | (t & 2u); }

// The lanes of 16 give the addresses of four values each, rows of 16 in the order of the lanes; lane i gets value i of each row.
__device__ __forceinline__ u32x2 read_transposed(const uint8_t* p)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}

// LDS written by some lanes of a wave is read by others: the wave's LDS operations keep their order, the compiler has to as well.
__device__ __forceinline__ void same_wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// In a tile where some lines do not see some tokens, a value that is infinite or NaN would reach lines that do not see it,
// by way of a weight of zero.  There zeros take the places of such values in LDS, and what lines see of them is added behind
// the loop, in a second walk over those tiles (add_unfinite) that hardly any call takes.
template <class E>
__device__ __forceinline__ u32x4 finite_only(u32x4 v, bool& other)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7FFFu) >= E::kInf) { v[i] &= 0xFFFF0000u; other = true; }
        if (((v[i] >> 16) & 0x7FFFu) >= E::kInf) { v[i] &= 0xFFFFu; other = true; }
    }
    return v;
}

// 16 bytes a lane from device memory to LDS, where lane i's go to `to` + 16 i; `to` is the same in the wave.
__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint8_t* to)
{
    __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(uintptr_t)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
__device__ __forceinline__ void loads_to_lds_done() { __builtin_amdgcn_s_waitcnt(0x0F70); }      // vmcnt(0)

// Waits for loaded values.  Without it the wait stands in front of their first use, in a loop, where it is a wait for the loop's own
// loads from the second time on.
__device__ __forceinline__ void arrived(u32x4& v) { __asm__ volatile("" : "+v"(v)); }

// Adds the values that are not finite among four of a row of V that a line sees: dims `dim` .. `dim` + 3.
template <class E, int D, int kBits>
__device__ __forceinline__ void add_unfinite(float* o, const uint8_t* pool, const RowAt<kBits>& at, uint32_t dim)
{
    if constexpr (kBits == 16) {
        const u32x2 v = dev_load<u32x2>(pool + at.row + dim * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = (v[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
            if ((x & 0x7FFFu) >= E::kInf) o[i] += E::to_float(x);
        }
    } else {
        if (dev_load<uint8_t>(pool + at.scale + dim / 32) != 255u) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = NAN;
    }
}

__device__ __forceinline__ float lse_of(float top, float sum, float shift)
{
    return sum > 0.f ? kLn2 * (top - shift + __builtin_amdgcn_logf(sum)) : sum == 0.f ? -INFINITY : sum;
}

// ---- sums that pass 32 bits ----------------------------------------------------------------------
// bfloat16 values go up to 2^128, as sums in 32 bits do, and weights of 2^16 and more times values pass it where outputs do not.  A line
// whose sum of weights is finite and some of whose sums of values are not, though it sees no value in those dimensions that is not, is
// gone through once more by one wave in plain steps, with each weight divided by the sum of all weights before it multiplies a value.
// Both walks take 64 tokens at a time: a lane finds one token's row (and its score), then has D / 64 dimensions of all 64 rows.
// The lane's number, counted anew rather than kept.
__device__ __forceinline__ uint32_t lane_again() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }
template <int D, int kBits>
struct Rows64 {
    RowAt<kBits> at;                                                     // of this lane's token
    uint64_t held;                                                       // which tokens are there
};
template <int D, int kBits>
__device__ __forceinline__ Rows64<D, kBits> rows_64(const AttendArgs& g, uint32_t seq, uint32_t head, int32_t t0, int32_t hi)
{
    const int32_t mine = t0 + (int32_t)lane_again(), t = mine < hi ? mine : hi - 1;
    const uint32_t page = dev_load<uint32_t>(g.b.page_table + (uint64_t)seq * g.b.table_stride + ((uint32_t)t >> g.c.page_shift));
    const bool there = mine < hi && page < g.c.n_pages;
    return Rows64<D, kBits>{row_at<D, kBits>(g.c, there ? page : 0u, (uint32_t)t, head), __ballot(there)};
}

// This lane's dimensions, D / 64 from D / 64 * lane on, of the row of V that lane i has found, in 16 bits each.
template <class E, int D, int kBits>
struct Dims {
    static constexpr int kPer = D / 64;
    uint32_t v[(kPer + 1) / 2];
    __device__ __forceinline__ float value(int k) const { return E::to_float(v[k / 2] >> (16 * (k & 1)) & 0xFFFFu); }
};
__device__ __forceinline__ uint64_t of_lane(uint64_t x, int i)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, i);
}
template <class E, int D, int kBits>
__device__ __forceinline__ Dims<E, D, kBits> dims_of(const uint8_t* pool, const Rows64<D, kBits>& rows, int i)
{
    constexpr int kPer = D / 64;
    const uint32_t lane = lane_again();
    const uint8_t* const p = pool + of_lane(rows.at.row, i);
    Dims<E, D, kBits> to;
    if constexpr (kBits == 16) {
        if constexpr (kPer == 1) to.v[0] = dev_load<uint16_t>(p + lane * 2);
        else
#pragma unroll
            for (int k = 0; k < kPer / 2; ++k) to.v[k] = dev_load<uint32_t>(p + (lane * kPer + 2 * k) * 2);
    } else {
        const float scale = scale_of(dev_load<uint8_t>(pool + of_lane(rows.at.scale, i) + lane * kPer / 32));
        if constexpr (kPer == 1) to.v[0] = E::template decode2<0>(dev_load<uint8_t>(p + lane / 2), scale) >> (16 * (lane & 1u)) & 0xFFFFu;
        else
#pragma unroll
            for (int k = 0; k < kPer / 2; ++k) to.v[k] = E::template decode2<0>(dev_load<uint8_t>(p + lane * (kPer / 2) + k), scale);
    }
    return to;
}

// The first and the last token from lo to hi with a value that is not finite, for each of this lane's dimensions.
template <int D>
struct Unfinite {
    int32_t first[D / 64], last[D / 64];
    // Whether a line that sees the tokens of `see` is known to see such a value of dimension `dim`, of which `k` is dim % (D / 64).
    // All lanes come here together.
    template <class S>
    __device__ __forceinline__ bool seen(const S& see, uint32_t dim, int k) const
    {
        const int32_t a = __shfl(first[k], (int)(dim / (D / 64)), 64), z = __shfl(last[k], (int)(dim / (D / 64)), 64);
        return see.sees(a) || see.sees(z);
    }
};
template <class E, int D, int kBits>
__device__ __forceinline__ Unfinite<D> find_unfinite(const AttendArgs& g, uint32_t seq, uint32_t head, const Range& range)
{
    Unfinite<D> u;
#pragma unroll
    for (int k = 0; k < D / 64; ++k) u.first[k] = u.last[k] = -1;
#pragma unroll 1
    for (int32_t t0 = range.lo; t0 < range.hi; t0 += 64) {
        const Rows64<D, kBits> rows = rows_64<D, kBits>(g, seq, head, t0, range.hi);
#pragma unroll 1
        for (int i = 0; i < 64; i += 16) {
            Dims<E, D, kBits> v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = dims_of<E, D, kBits>(g.c.v, rows, i + j);
#pragma unroll
            for (int j = 0; j < 16; ++j)
#pragma unroll
                for (int k = 0; k < D / 64; ++k)
                    if (!(fabsf(v[j].value(k)) < INFINITY) && (rows.held >> (i + j) & 1u)) {
                        u.first[k] = u.first[k] < 0 ? t0 + i + j : u.first[k];
                        u.last[k] = t0 + i + j;
                    }
        }
    }
    return u;
}

// `line_top`, `line_sum`: what the loops below have found, which stand for the logsumexp and for a part.  Scores are finite or minus
// infinity here; values that are not finite are added as they are, whatever their weight.
template <class E, int D, int kBits, bool kTree>
__device__ __forceinline__ void plain_line(const AttendArgs& g, const KvSeq& seq_of, uint32_t seq, uint32_t head, uint32_t split, int32_t line, const Range& range,
                                           float line_top, float line_sum)
{
    constexpr int kPer = D / 64;
    const uint32_t lane = lane_again();
    const int32_t row = line / (int32_t)g.group, h = line - row * (int32_t)g.group;
    const uint32_t q_head = head * g.group + (uint32_t)h;
    const uint64_t out_row = (uint64_t)(seq_of.row0 + row);
    const Sight<kTree> see = sight<kTree>(g, seq_of, row);
    const int32_t lo = see.lo > range.lo ? see.lo : range.lo, hi = see.end() < range.hi ? see.end() : range.hi;
    auto find = [&](int32_t t0) {
        Rows64<D, kBits> rows = rows_64<D, kBits>(g, seq, head, t0, hi);
        if constexpr (kTree) rows.held &= same_in_wave(see.bits(t0));
        return rows;
    };
    const uint8_t* const q = g.q + out_row * g.q_stride + (uint64_t)q_head * D * 2;
    float top = -INFINITY, sum = 0.f, y[kPer];
    auto score = [&](const Rows64<D, kBits>& rows) -> float {            // of this lane's token, times log2(e)
        float s = 0.f;
#pragma unroll 4
        for (uint32_t c = 0; c < D / 8; ++c) {
            const u32x4 a = dev_load<u32x4>(q + c * 16);
            u32x4 k;
            if constexpr (kBits == 16) k = dev_load<u32x4>(g.c.k + rows.at.row + c * 16);
            else k = decode8<E>(dev_load<uint32_t>(g.c.k + rows.at.row + c * 4), scale_of(dev_load<uint8_t>(g.c.k + rows.at.scale + c / 4)));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s = fmaf(E::to_float(a[i] & 0xFFFFu), E::to_float(k[i] & 0xFFFFu), s);
                s = fmaf(E::to_float(a[i] >> 16), E::to_float(k[i] >> 16), s);
            }
        }
        return rows.held >> lane & 1u ? s * g.to_log2 : -INFINITY;
    };
#pragma unroll 1
    for (int32_t t0 = lo; t0 < hi; t0 += 64) {
        const float x = score(find(t0));
        float now = x;
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) now = fmaxf(now, __shfl_xor(now, k, 64));
        now = fmaxf(now, top);
        float add = __builtin_amdgcn_exp2f(x - (now == -INFINITY ? 0.f : now));
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) add += __shfl_xor(add, k, 64);
        const float f = rescale(top, now);
        sum = sum * f * f + add;
        top = now;
    }
    const float share = 1.f / sum;
#pragma unroll
    for (int k = 0; k < kPer; ++k) y[k] = 0.f;
#pragma unroll 1
    for (int32_t t0 = lo; t0 < hi; t0 += 64) {
        const Rows64<D, kBits> rows = find(t0);
        const float w = __builtin_amdgcn_exp2f(score(rows) - top) * share;
#pragma unroll 1
        for (int i = 0; i < 64; i += 16) {
            Dims<E, D, kBits> v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = dims_of<E, D, kBits>(g.c.v, rows, i + j);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float wj = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(w), i + j));
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const float x = v[j].value(k);
                    if (rows.held >> (i + j) & 1u) y[k] = fabsf(x) < INFINITY ? fmaf(wj, x, y[k]) : y[k] + x;
                }
            }
        }
    }
    if (g.part_o) {                                                      // the sum brought to 1 at most, by a power of two whose root is one
        const uint64_t at = (out_row * g.q_heads + q_head) * g.n_splits + split;
        const int power = ((int)(__float_as_uint(line_sum) >> 23) - 127 + 2) & ~1;
        line_sum = ldexpf(line_sum, -power);
#pragma unroll
        for (int k = 0; k < kPer; ++k) dev_store(g.part_o + at * D + lane * kPer + k, y[k] * line_sum);
        if (lane == 0) dev_store(g.part_ml + at * 2, f32x2{line_top + (float)power, line_sum});
        return;
    }
    uint8_t* const to = g.out + out_row * g.out_stride + (uint64_t)q_head * D * 2;
    if constexpr (kPer == 1) {
        dev_store(to + lane * 2, (uint16_t)E::pack2(y[0], 0.f));
    } else {
#pragma unroll
        for (int k = 0; k < kPer; k += 2) dev_store(to + (lane * kPer + k) * 2, E::pack2(y[k], y[k + 1]));
    }
}

// ---- few lines -----------------------------------------------------------------------------------
constexpr int kWaves = 4;
constexpr int kTile = 32;              // tokens of a wave's step

// Scale bytes as the aligned word that holds them, and how far up they are in it.  A byte's load would be extended to a register
// where it is loaded, behind a wait for it; this is taken apart where it is used.
struct ScaleWord { uint32_t word, shift; };
__device__ __forceinline__ ScaleWord load_scale(const uint8_t* p)
{
    const uintptr_t at = (uintptr_t)p;
    return ScaleWord{dev_load<uint32_t>((const void*)(at & ~(uintptr_t)3)), (uint32_t)(at & 3u) * 8u};
}
__device__ __forceinline__ uint32_t byte_of(const ScaleWord& s, uint32_t i = 0) { return s.word >> (s.shift + 8 * i) & 0xFFu; }

// One tile of a wave in registers, as it is loaded: a token's row in lanes side by side, 16 bytes each.
template <int D, int kBits>
struct Tile {
    static constexpr int kPerRow = kBits == 16 ? D / 8 : D / 32;         // lanes to a row
    static constexpr int kPasses = kTile * kPerRow / 64;
    static constexpr int kTokens = 64 / kPerRow;                         // tokens of a pass
    static constexpr int kWords = D == 256 ? 2 : 1;                      // words that hold a row's scale bytes
    u32x4 k[kPasses], v[kPasses];
    uint32_t scale[kWords];                                              // of token lane % 32, K in the lower half of the lanes, V in the upper
    uint32_t shift;                                                      // where its bytes begin in the word: two of them need not at the first
};

// What the first product reads of K.  Lane (m = lane % 16, quad = lane / 16) takes token 8 (m / 4) + 4 half + m % 4 for half 0 and
// 1: after the product, quad holds tokens 8 quad .. 8 quad + 7.
__device__ __forceinline__ uint32_t k_token(uint32_t m, uint32_t half) { return 8 * (m >> 2) + 4 * half + (m & 3u); }
// Eight lanes side by side, each of a token of its own, are to read from all banks: rows of 16 bits as in `spread`, rows of codes
// are D / 32 chunks long.
template <int D, int kBits>
__device__ __forceinline__ uint32_t k_place(uint32_t t, uint32_t chunk)
{
    if constexpr (kBits == 16) return t * (D * 2) + ((spread<D>(chunk) ^ ((t & 3u) | (t >> 1 & 4u))) << 4);
    else return t * (D / 2) + ((chunk ^ (D == 64 ? t >> 3 & 1u : D == 128 ? (t >> 1 & 1u) | (t >> 2 & 2u) : (t & 3u) | (t >> 1 & 4u))) << 4);
}

// Four waves, a tile of 32 tokens each in turn, 16 lines (or two or four times that) in a wave's registers.  Waves share nothing until
// their parts are joined at the end, so no barrier holds the loads up: a tile's rows are loaded while the one before is worked on,
// its page numbers one tile earlier still.
template <class E, int D, int kBits, int kLineTiles, bool kTree>
__global__ void __launch_bounds__(256) narrow_kernel(const AttendArgs g)
{
    constexpr int kK = D / 32;                                           // steps of the first product
    constexpr int kDims = D / 16;                                        // tiles of 16 dimensions of the second
    using T = Tile<D, kBits>;
    constexpr uint32_t kVBytes = kWaves * kTile * D * 2, kOBytes = kWaves * 16 * (D + 4) * 4;
    __shared__ __align__(16) uint8_t lds[kVBytes > kOBytes ? kVBytes : kOBytes];
    __shared__ RowAt<kBits> rows_at[kWaves][kTile];
    __shared__ float line_top[kWaves][16 * kLineTiles], line_sum[kWaves][16 * kLineTiles];
    __shared__ uint64_t line_mask[kTree ? kWaves : 1][kTree ? 16 * kLineTiles : 1];      // a tree of up to 64 rows: a word each

    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t m = lane & 15u, quad = lane >> 4;
    // All heads of a (sequence, split) go to one XCD one after the other: the heads of a token share lines of its page.  The later
    // splits, which short sequences do not have, come last, and each of them begins with another sequence: otherwise the XCDs that
    // get them, or get the long sequences, would have more or less to do than the others.
    const uint32_t block = g.first + blockIdx.x, eight = block / (8 * g.c.heads), in_eight = block - eight * 8 * g.c.heads;
    const uint32_t unit = eight * 8 + in_eight % 8, head = in_eight / 8;
    if (unit >= g.b.n_seqs * g.n_splits) return;
    const uint32_t split = unit / g.b.n_seqs, seq = (unit + split) % g.b.n_seqs;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.bad && threadIdx.x == 0 && split == 0 && head == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    if (q.rows == 0 || split >= splits_of<kTree>(g, q)) return;
    const int32_t lines = q.rows * (int32_t)g.group;                     // at most 16 kLineTiles, by the host's choice
    const Range range = token_range<kTree>(g, q, 0, lines - 1, split);

    // This lane's line of every tile of 16: its queries as the second operand of S^T, and the tokens that it sees.
    u32x4 qf[kLineTiles][kK];
    KvSpan see[kLineTiles];                                              // of a tree the context only
#pragma unroll
    for (int rt = 0; rt < kLineTiles; ++rt) {
        const int32_t line = rt * 16 + (int32_t)m;
        const int32_t row = line < lines ? line / (int32_t)g.group : 0, h = line < lines ? line - row * (int32_t)g.group : 0;
        if constexpr (kTree) {
            const Sight<true> s = sight<true>(g, q, row);
            see[rt] = KvSpan{s.lo, s.base};
            if (quad == 0) line_mask[wave][rt * 16 + m] = s.word(0);
        } else {
            see[rt] = kv_span(row, q.rows, q.len, g.window, g.all);
        }
        // dims in the order of K's operand: a lane has every fourth eight of a 16-bit row, and D / 4 in a row of codes
        const uint8_t* p = g.q + (uint64_t)(q.row0 + row) * g.q_stride + ((uint64_t)(head * g.group + h) * D + quad * (kBits == 16 ? 8 : D / 4)) * 2;
#pragma unroll
        for (int k = 0; k < kK; ++k) qf[rt][k] = dev_load<u32x4>(p + k * (kBits == 16 ? 64 : 16));
    }
#pragma unroll
    for (int rt = 0; rt < kLineTiles; ++rt)
#pragma unroll
        for (int k = 0; k < kK; ++k) arrived(qf[rt][k]);
    // tokens that every line sees
    const KvSpan by_all = seen_by_rows<kTree>(g, q, 0, q.rows - 1);
    const int32_t all_lo = by_all.lo, all_hi = by_all.hi;

    f32x4 o[kLineTiles][kDims];
    float top[kLineTiles], sum[kLineTiles];
#pragma unroll
    for (int rt = 0; rt < kLineTiles; ++rt) {
        top[rt] = -INFINITY;
        sum[rt] = 0.f;
#pragma unroll
        for (int d = 0; d < kDims; ++d) o[rt][d] = f32x4{0, 0, 0, 0};
    }

    auto seen_by_all = [&](int32_t t0) -> bool { return t0 >= all_lo && t0 + kTile <= all_hi; };

    // Waves take tiles in turn.  Page numbers are loaded two of a wave's tiles ahead, rows one ahead.
    const int32_t tiles = (range.hi - range.lo + kTile - 1) / kTile;
    // Nothing of that stands behind a condition in the loop: the compiler then knows how many loads are behind the one that it
    // waits for, and does not wait for them.  Past the last tile they go to a row that is there.
    bool bad_page = false;
    auto load_page = [&](int32_t tile) -> uint32_t {
        const int32_t t = min(range.lo + tile * kTile + (int32_t)(lane & 31u), range.hi - 1);
        return dev_load<uint32_t>(g.b.page_table + (uint64_t)seq * g.b.table_stride + ((uint32_t)t >> g.c.page_shift));
    };
    // Puts the places of a tile's rows into LDS and says which of its tokens are there.
    auto place_rows = [&](int32_t tile, uint32_t page) -> uint32_t {
        const int32_t t = range.lo + tile * kTile + (int32_t)(lane & 31u);
        const bool inside = t < range.hi, there = inside && page < g.c.n_pages;
        bad_page |= inside && !there;
        uint32_t to = lane;
        __asm__ volatile("" : "+v"(to));                                 // its address is computed here, not kept in a register
        if (lane < 32) rows_at[wave][to] = row_at<D, kBits>(g.c, there ? page : 0u, (uint32_t)t, head);
        same_wave_order();
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)__ballot(there));
    };
    T now;
    auto load_rows = [&](u32x4* to, const uint8_t* pool) {
#pragma unroll
        for (int i = 0; i < T::kPasses; ++i) {
            const uint32_t part = lane % T::kPerRow;
            to[i] = dev_load<u32x4>(pool + rows_at[wave][i * T::kTokens + lane / T::kPerRow].row + (kBits == 16 ? gather<D>(part) : part) * 16);
        }
    };
    auto load_scales = [&]() {
        if constexpr (kBits == 4) {
            // whole words: a byte's load would be extended to a register where it is loaded, behind a wait for it
            const uintptr_t at = (uintptr_t)(lane < 32 ? g.c.k : g.c.v) + rows_at[wave][lane & 31u].scale;
            if constexpr (T::kWords == 2) {
                const u32x2 w = dev_load<u32x2>((const void*)at);
                now.scale[0] = w[0];
                now.scale[1] = w[1];
                now.shift = 0;
            } else {
                now.scale[0] = dev_load<uint32_t>((const void*)(at & ~(uintptr_t)3));
                now.shift = (uint32_t)(at & 3u) * 8;
            }
        }
    };
    // Scale byte `block` of token t of K (of V for t from 32 on), from the lane that has loaded it.
    auto scale_at = [&](uint32_t t, uint32_t block) -> uint32_t {
        uint32_t w = (uint32_t)__builtin_amdgcn_ds_bpermute((int)(t * 4), (int)(now.scale[0] >> now.shift));
        if constexpr (T::kWords == 2) {
            const uint32_t upper = (uint32_t)__builtin_amdgcn_ds_bpermute((int)(t * 4), (int)now.scale[1]);
            w = block >= 4 ? upper : w;
        }
        return w >> (8 * (block & 3u)) & 0xFFu;
    };
    // K's rows and V's take the same place one after the other.
    uint8_t* const v_lds = lds + wave * (kTile * D * 2);
    uint8_t* const k_lds = v_lds;
    uint32_t there = 0, next_page = 0;
    bool unfinite = false;                                               // this lane met a value that is infinite or NaN in a tile that is not whole
    if (tiles > 0) {
        there = place_rows((int32_t)wave, load_page((int32_t)wave));
        next_page = load_page((int32_t)wave + kWaves);                   // in front of the rows, as in the loop
        load_rows(now.k, g.c.k);
        load_scales();
        load_rows(now.v, g.c.v);
    }
    for (int32_t tile = (int32_t)wave; tile < tiles; tile += kWaves) {
        const int32_t t0 = range.lo + tile * kTile;
        same_wave_order();
        const uint32_t there_next = place_rows(tile + kWaves, next_page);
        next_page = load_page(tile + 2 * kWaves);
        // S^T
#pragma unroll
        for (int i = 0; i < T::kPasses; ++i) {
            const uint32_t t = i * T::kTokens + lane / T::kPerRow, part = lane % T::kPerRow;
            *(u32x4*)(k_lds + k_place<D, kBits>(t, kBits == 16 ? gather<D>(part) : part)) = now.k[i];
        }
        load_rows(now.k, g.c.k);
        __builtin_amdgcn_sched_barrier(0);                               // the next rows are on their way before anything waits for V's
        same_wave_order();
        f32x4 s[kLineTiles][2];
#pragma unroll
        for (int rt = 0; rt < kLineTiles; ++rt) s[rt][0] = s[rt][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const uint32_t t = k_token(m, a);
            u32x4 kf[kK];
            if constexpr (kBits == 16) {
#pragma unroll
                for (int k = 0; k < kK; ++k) kf[k] = *(const u32x4*)(k_lds + k_place<D, 16>(t, 4 * k + quad));
            } else if constexpr (D == 64) {
                const u32x2 c = *(const u32x2*)(k_lds + k_place<D, 4>(t, quad >> 1) + (quad & 1u) * 8);
                const float scale = scale_of(scale_at(t, quad >> 1));
                kf[0] = decode8<E>(c[0], scale);
                kf[1] = decode8<E>(c[1], scale);
            } else {
#pragma unroll
                for (int b = 0; b < D / 128; ++b) {
                    const u32x4 c = *(const u32x4*)(k_lds + k_place<D, 4>(t, quad * (D / 128) + b));
                    const float scale = scale_of(scale_at(t, quad * (D / 128) + b));
#pragma unroll
                    for (int k = 0; k < 4; ++k) kf[b * 4 + k] = decode8<E>(c[k], scale);
                }
            }
#pragma unroll
            for (int k = 0; k < kK; ++k)
#pragma unroll
                for (int rt = 0; rt < kLineTiles; ++rt) s[rt][a] = E::mfma16(kf[k], qf[rt][k], s[rt][a]);
        }
        same_wave_order();
        // V's rows to LDS, tokens that are not there as zeros
        const bool whole = there == 0xFFFFFFFFu && seen_by_all(t0);
#pragma unroll
        for (int i = 0; i < T::kPasses; ++i) {
            const uint32_t t = i * T::kTokens + lane / T::kPerRow, part = lane % T::kPerRow, x = v_swap(t);
            bool gone = !whole && !((there >> t) & 1u);
            if constexpr (kBits == 16) {
                u32x4 v = now.v[i];
                if (!whole) v = gone ? u32x4{0, 0, 0, 0} : finite_only<E>(v, unfinite);
                *(u32x4*)(v_lds + t * (D * 2) + ((part ^ x) << 4)) = v;
            } else {
                const uint32_t byte = scale_at(32 + t, part);
                if (!whole && !gone && byte == 255u) gone = unfinite = true;
                const float scale = scale_of(gone ? 0u : byte);
#pragma unroll
                for (int c = 0; c < 4; ++c) *(u32x4*)(v_lds + t * (D * 2) + ((spread<D>(part * 4 + c) ^ x) << 4)) = decode8<E>(gone ? 0u : now.v[i][c], scale);
            }
        }
        load_scales();
        load_rows(now.v, g.c.v);
        __builtin_amdgcn_sched_barrier(0);
        same_wave_order();
        // O^T's first operand: tokens 8 quad .. 8 quad + 7 of 16 dimensions
        const uint32_t vt = 8 * quad + (m >> 2);
        const uint8_t *row_a = v_lds + vt * (D * 2) + (m & 1u) * 8, *row_b = row_a + 4 * (D * 2);
        const uint32_t x = v_swap(vt) ^ ((m >> 1) & 1u);                  // the same four tokens on
        auto v_operand = [&](int d) -> u32x4 {
            const u32x2 a = read_transposed(row_a + ((spread<D>(2 * d) ^ x) << 4)), b = read_transposed(row_b + ((spread<D>(2 * d) ^ x) << 4));
            return u32x4{a[0], a[1], b[0], b[1]};
        };
        u32x4 p[kLineTiles];
#pragma unroll
        for (int rt = 0; rt < kLineTiles; ++rt) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = s[rt][j >> 2][j & 3];
            if (!whole) {                                                // this lane has tokens t0 + 8 quad + 0 .. 7 of its line
                uint32_t seen = there;
                if constexpr (kTree) {
                    const uint64_t mask = line_mask[wave][rt * 16 + m];
                    seen &= (uint32_t)kv_tree_bits(KvTreeSpan{see[rt].lo, see[rt].hi, q.len, 1}, t0, [&](int32_t i) { return i == 0 ? mask : 0; });
                } else {
                    if (see[rt].hi < t0 + kTile) seen = see[rt].hi > t0 ? seen & ~(~0u << (see[rt].hi - t0)) : 0u;
                    if (see[rt].lo > t0) seen = see[rt].lo < t0 + kTile ? seen & ~0u << (see[rt].lo - t0) : 0u;
                }
                seen >>= 8 * quad;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = seen & (1u << j) ? x[j] : -INFINITY;
            }
            float big = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            big = max_over32(max_over16(big)) * g.to_log2;
            if (__any(big > top[rt] + kLag)) {
                const float now = fminf(fmaxf(top[rt], big), kMost), f = rescale(top[rt], now);
                top[rt] = now;
                sum[rt] = sum[rt] * f * f;
#pragma unroll
                for (int d = 0; d < kDims; ++d) o[rt][d] = o[rt][d] * f * f;
            }
            const float against = E::kWeightShift - (top[rt] == -INFINITY ? 0.f : top[rt]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = __builtin_amdgcn_exp2f(fmaf(x[j], g.to_log2, against));
                sum[rt] += x[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) p[rt][j] = E::pack2(x[2 * j], x[2 * j + 1]);     // rounded to nearest: see the head of this file
        }
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            const u32x4 vf = v_operand(d);
#pragma unroll
            for (int rt = 0; rt < kLineTiles; ++rt) o[rt][d] = E::mfma16(vf, p[rt], o[rt][d]);
        }
        there = there_next;
    }

    if (bad_page) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
    if (__any(unfinite)) {
#pragma unroll 1
        for (int32_t tile = (int32_t)wave; tile < tiles; tile += kWaves) {
            const int32_t t0 = range.lo + tile * kTile;
            there = place_rows(tile, load_page(tile));
            if (there == 0xFFFFFFFFu && seen_by_all(t0)) continue;
#pragma unroll 1
            for (int32_t t = 0; t < kTile; ++t) {
                if (!((there >> t) & 1u)) continue;
                const RowAt<kBits> at = rows_at[wave][t];
#pragma unroll
                for (int rt = 0; rt < kLineTiles; ++rt) {
                    if constexpr (kTree) {
                        const int32_t j = t0 + t - see[rt].hi;           // among the rows
                        if (j >= 0 ? !(line_mask[wave][rt * 16 + m] >> j & 1u) : t0 + t < see[rt].lo) continue;
                    } else {
                        if (t0 + t < see[rt].lo || t0 + t >= see[rt].hi) continue;
                    }
#pragma unroll
                    for (int d = 0; d < kDims; ++d) {
                        float x[4] = {o[rt][d][0], o[rt][d][1], o[rt][d][2], o[rt][d][3]};
                        add_unfinite<E, D, kBits>(x, g.c.v, at, d * 16 + quad * 4);
                        o[rt][d] = f32x4{x[0], x[1], x[2], x[3]};
                    }
                }
            }
        }
    }

    // The waves' parts are joined over LDS, 16 lines at a time.
#pragma unroll
    for (int rt = 0; rt < kLineTiles; ++rt) {
        sum[rt] = sum_over32(sum_over16(sum[rt]));
        if (quad == 0) {
            line_top[wave][rt * 16 + m] = top[rt];
            line_sum[wave][rt * 16 + m] = sum[rt];
        }
    }
    float* const o_lds = (float*)lds;
    constexpr uint32_t kRow = D + 4, kSeg = D / 16;
    uint64_t large = 0;                                                  // lines of this wave whose sums passed 32 bits
#pragma unroll
    for (int rt = 0; rt < kLineTiles; ++rt) {
        __syncthreads();
        float now = line_top[0][rt * 16 + m];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) now = fmaxf(now, line_top[w][rt * 16 + m]);
        const float f = rescale(top[rt], now);
#pragma unroll
        for (int d = 0; d < kDims; ++d) *(f32x4*)(o_lds + (wave * 16 + m) * kRow + d * 16 + quad * 4) = o[rt][d] * f * f;
        __syncthreads();
        const uint32_t in_tile = threadIdx.x >> 4, seg = threadIdx.x & 15u;
        const int32_t line = rt * 16 + (int32_t)in_tile;
        float best = line_top[0][line], total = 0.f;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) best = fmaxf(best, line_top[w][line]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float r = rescale(line_top[w][line], best);
            total += line_sum[w][line] * r * r;
        }
        float y[kSeg];
#pragma unroll
        for (uint32_t i = 0; i < kSeg; ++i) {
            y[i] = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) y[i] += o_lds[(w * 16 + in_tile) * kRow + seg * kSeg + i];
        }
        if constexpr (E::kLarge) {                                       // a line is in 16 lanes side by side, four of them in a wave
            float x = 0.f;
#pragma unroll
            for (uint32_t i = 0; i < kSeg; ++i) x = fmaf(y[i], 0.f, x);
            bool odd = line < lines && total > 0.f && total < INFINITY && !(x == 0.f);
            if (__any(odd)) {
                const AttendArgs& a = args_again();
                const Unfinite<D> u = find_unfinite<E, D, kBits>(a, seq, head, range);
                const Sight<kTree> see_line = sight<kTree>(a, q, (line < lines ? line : 0) / (int32_t)a.group);
                bool more = false;
#pragma unroll
                for (uint32_t i = 0; i < kSeg; ++i) more |= !u.seen(see_line, seg * kSeg + i, i % (D / 64)) && !(fabsf(y[i]) < INFINITY);
                const uint64_t here = __ballot(odd && more);
#pragma unroll
                for (int i = 0; i < 4; ++i) large |= (uint64_t)((here >> (16 * i) & 0xFFFFu) != 0) << (rt * 16 + 4 * wave + i);
            }
        }
        if (line >= lines) continue;
        const bool stands = !(large >> line & 1u);                       // else plain_line stores it
        const int32_t row = line / (int32_t)g.group, h = line - row * (int32_t)g.group;
        const uint32_t q_head = head * g.group + (uint32_t)h;
        const uint64_t out_row = (uint64_t)(q.row0 + row);
        if (g.part_o) {
            const uint64_t at = (out_row * g.q_heads + q_head) * g.n_splits + split;
            if (!stands) continue;
#pragma unroll
            for (uint32_t i = 0; i < kSeg / 4; ++i) dev_store(g.part_o + at * D + seg * kSeg + i * 4, f32x4{y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]});
            if (seg == 0) dev_store(g.part_ml + at * 2, f32x2{best, total});
        } else {
            const float scale = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (uint32_t i = 0; i < kSeg; ++i) y[i] = total == 0.f ? 0.f : y[i];    // no weight: zeros, whatever the values
            uint8_t* to = g.out + out_row * g.out_stride + ((uint64_t)q_head * D + seg * kSeg) * 2;
            if (stands)
#pragma unroll
                for (uint32_t i = 0; i < kSeg / 4; ++i) dev_store(to + i * 8, u32x2{E::pack2(y[4 * i] * scale, y[4 * i + 1] * scale), E::pack2(y[4 * i + 2] * scale, y[4 * i + 3] * scale)});
            if (g.lse && seg == 0) g.lse[out_row * g.q_heads + q_head] = lse_of(best, total, E::kWeightShift);
        }
    }
    if constexpr (E::kLarge) {
        if (large) {
            const AttendArgs& a = args_again();
#pragma unroll 1
            for (; large; large &= large - 1) {
                const int32_t line = __builtin_ctzll(large);
                float best = line_top[0][line], total = 0.f;
#pragma unroll
                for (int w = 1; w < kWaves; ++w) best = fmaxf(best, line_top[w][line]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float r = rescale(line_top[w][line], best);
                    total += line_sum[w][line] * r * r;
                }
                plain_line<E, D, kBits, kTree>(a, q, seq, head, split, line, range, best, total);
            }
        }
    }
}

// ---- many lines ----------------------------------------------------------------------------------
constexpr int kWideTile = 64;          // tokens of a step
constexpr int kWideLines = 128;        // 32 a wave, where four waves have lines of their own

// What a workgroup is for.  Heads vary fastest, so a head stays on an XCD where there are eight, and its tokens in that XCD's cache;
// the rows that see the most tokens come first.
struct WideUnit { uint32_t head, seq, split, line_tile; };
__device__ __forceinline__ WideUnit wide_unit(const AttendArgs& g, uint32_t block)
{
    WideUnit u;
    u.head = block % g.c.heads;
    block /= g.c.heads;
    u.seq = block % g.b.n_seqs;
    block /= g.b.n_seqs;
    u.split = block % g.n_splits;
    u.line_tile = g.line_tiles - 1 - block / g.n_splits;
    return u;
}

// 32 lines a wave, so that scores, outputs and queries of two waves fit a SIMD's registers (one wave for 256 dimensions): a wave's
// vector work can run beside the other's products as well as beside its own.  Four waves share a tile because LDS, read by every wave
// in full, would otherwise be what is short: 128 bytes a cycle feed four SIMDs of these products exactly.
// kGroups: waves with lines of their own, 4 or 2.  Two lots of 32 lines have two waves each, which take half of a tile's tokens, 32, and whose
// sums are joined at the end.
template <class E, int D, int kBits, bool kTree, int kGroups>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) wide_kernel(const AttendArgs g)
{
    constexpr int kK = D / 16, kDims = D / 32;
    constexpr int kS = kGroups / 2, kLines = 32 * kGroups;               // lots of 32 tokens that a wave takes of a tile; lines of the workgroup
    constexpr int kPairs = 8 * kS;                                       // of a lane's weights
    constexpr int kPerRow = kBits == 16 ? D / 8 : D / 32;                // lanes to a row
    constexpr int kItems = 2 * kWideTile * kPerRow / 256;                // of a thread: K's rows, then V's
    constexpr uint32_t kPlane = kWideTile * D * 2;
    // Two places for a tile of K and two for one of V, [64 tokens][D] each.  They are variables of their own, and which of them a step
    // loads to is known when it is compiled: a read of LDS would otherwise wait for every load to LDS that is on its way.
    __shared__ __align__(16) uint8_t k_even[kPlane], k_odd[kPlane], v_even[kPlane], v_odd[kPlane];
    __shared__ RowAt<kBits> rows_at[4][kWideTile];
    __shared__ uint64_t there_lds[4];
    __shared__ uint32_t unfinite_lds;                                    // a value was infinite or NaN in a tile that is not whole
    __shared__ f32x2 joined[kGroups == 4 ? 1 : 2][kGroups == 4 ? 1 : 64]; // maxima and sums of the waves with the second tokens

    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t m = lane & 31u, upper = lane >> 5;
    const uint32_t lot = kGroups == 4 ? wave : wave & 1u, part = kGroups == 4 ? 0u : wave >> 1;      // of the lines; of a tile's tokens
    const WideUnit unit = wide_unit(g, g.first + blockIdx.x);
    const uint32_t head = unit.head, seq = unit.seq, split = unit.split, line_tile = unit.line_tile;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.bad && threadIdx.x == 0 && split == 0 && head == 0 && line_tile == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    const int32_t lines = q.rows * (int32_t)g.group, line0 = (int32_t)line_tile * kLines;
    if (line0 >= lines || split >= splits_of<kTree>(g, q)) return;
    const int32_t last_line = line0 + kLines < lines ? line0 + kLines - 1 : lines - 1;
    const Range range = token_range<kTree>(g, q, line0, last_line, split);

    const int32_t line = line0 + (int32_t)(lot * 32 + m);
    const bool mine = line < lines;
    const int32_t row = mine ? line / (int32_t)g.group : q.rows - 1, h = mine ? line - row * (int32_t)g.group : 0;
    const Sight<kTree> see = sight<kTree>(g, q, row);
    const uint32_t q_head = head * g.group + (uint32_t)h;
    // what the wave's first and last lines see
    const int32_t wave_first = line0 + (int32_t)lot * 32, wave_last = wave_first + 31 < lines ? wave_first + 31 : lines - 1;
    const bool idle = wave_first >= lines;
    const int32_t first_row = idle ? 0 : wave_first / (int32_t)g.group, last_row = idle ? 0 : wave_last / (int32_t)g.group;
    const KvSpan wave_any = seen_by_any<kTree>(g, q, first_row, last_row), wave_all = seen_by_rows<kTree>(g, q, first_row, last_row);

    // tokens that every line of the workgroup sees
    const KvSpan by_all = seen_by_rows<kTree>(g, q, line0 / (int32_t)g.group, last_line / (int32_t)g.group);
    const int32_t all_lo = by_all.lo, all_hi = by_all.hi;

    u32x4 qf[kK];
    {
        const uint8_t* p = g.q + (uint64_t)(q.row0 + row) * g.q_stride + ((uint64_t)q_head * D + upper * 8) * 2;
#pragma unroll
        for (int k = 0; k < kK; ++k) qf[k] = dev_load<u32x4>(p + k * 32);
    }
    f32x16 o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float top = -INFINITY, sum = 0.f;

    const int32_t tiles = range.hi > range.lo ? (range.hi - range.lo + kWideTile - 1) / kWideTile : 0;
    bool bad_page = false;
    // The first wave looks up where a tile's rows are, a step before they are loaded.  Past the last tile they are where some page is.
    auto load_page = [&](int32_t tile) -> uint32_t {
        const int32_t t = min(range.lo + tile * kWideTile + (int32_t)lane, range.hi - 1);
        return dev_load<uint32_t>(g.b.page_table + (uint64_t)seq * g.b.table_stride + ((uint32_t)t >> g.c.page_shift));
    };
    auto place_rows = [&](int32_t tile, uint32_t page) {
        const int32_t t = range.lo + tile * kWideTile + (int32_t)lane;
        const bool inside = t < range.hi, there = inside && page < g.c.n_pages;
        rows_at[tile & 3][lane] = row_at<D, kBits>(g.c, there ? page : 0u, (uint32_t)t, head);
        bad_page |= inside && !there;
        const uint64_t all = __ballot(there);
        if (lane == 0) there_lds[tile & 3] = all;
    };
    auto seen_by_all = [&](int32_t t0) -> bool { return t0 >= all_lo && t0 + kWideTile <= all_hi; };
    if (threadIdx.x == 0) unfinite_lds = 0;                              // before the barriers in front of the first rows
    // 16 bits: rows go straight to LDS, a wave's 64 chunks in the order of its lanes, so a lane picks the chunk that belongs in its
    // place.  4 bits: by way of registers, where they are decoded.
    u32x4 staged[kBits == 4 ? kItems : 1];
    ScaleWord staged_scale[kBits == 4 ? kItems : 1];
    // K's rows of one tile and V's of another, where there are such.
    auto load_rows = [&](int32_t k_tile, uint8_t* k_to, int32_t v_tile, uint8_t* v_to) {
        constexpr uint32_t kRows = 256 / kPerRow;                        // of an item; eight at least, so a lane's place in its row stays
        const uint32_t part = threadIdx.x % kPerRow, t_in = threadIdx.x / kPerRow % kWideTile;
        auto load = [&](int i) {
            const bool is_v = kItems == 1 ? threadIdx.x >= 128u : i >= kItems / 2;
            const RowAt<kBits> at = rows_at[(is_v ? v_tile : k_tile) & 3][t_in + i * kRows % kWideTile];
            const uint8_t* pool = is_v ? g.c.v : g.c.k;
            if constexpr (kBits == 16) {
                static_assert(kRows % 8 == 0, "places in a row repeat every eight rows");
                const uint32_t chunk = gather<D>(part ^ (is_v ? v_swap(t_in) : k_swap(t_in)));
                load_to_lds(pool + chunk * 16 + at.row, (is_v ? v_to : k_to) + (uint32_t)i % (kItems / 2) * 4096u + wave * 1024u);
            } else {
                staged[i] = dev_load<u32x4>(pool + at.row + part * 16);
                staged_scale[i] = load_scale(pool + at.scale + part);
            }
        };
        if constexpr (kItems == 1) {
            if ((threadIdx.x >= 128u ? v_tile : k_tile) < tiles) load(0);
        } else {
            if (k_tile < tiles)
#pragma unroll
                for (int i = 0; i < kItems / 2; ++i) load(i);
            if (v_tile < tiles)
#pragma unroll
                for (int i = kItems / 2; i < kItems; ++i) load(i);
        }
    };
    // What was loaded is in LDS when the barrier behind this is passed.  K's rows go as they are: scores of tokens that a line does
    // not see are replaced.  V's do where every line sees the whole tile.
    auto store_rows = [&](int32_t k_tile, uint8_t* k_to, int32_t v_tile, uint8_t* v_to, uint64_t there) {
        const bool whole = there == ~0ull && seen_by_all(range.lo + v_tile * kWideTile);
        bool unfinite = false;
        if constexpr (kBits == 16) {
            loads_to_lds_done();
            if (!whole && v_tile < tiles) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < kItems / 2; ++i) {
                    const uint32_t t = (i * 256 + threadIdx.x) / kPerRow;
                    u32x4* const v = (u32x4*)(v_to + (i * 256 + threadIdx.x) * 16);
                    *v = (there >> t) & 1u ? finite_only<E>(*v, unfinite) : u32x4{0, 0, 0, 0};
                }
            }
        } else {
            uint32_t thread = threadIdx.x;
            __asm__ volatile("" : "+v"(thread));                         // places are computed in every step, not kept in registers
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                const uint32_t item = i * 256 + thread, t = item / kPerRow % kWideTile, part = item % kPerRow;
                const bool is_v = item >= (uint32_t)(kWideTile * kPerRow);
                const int32_t tile = is_v ? v_tile : k_tile;
                if (tile >= tiles) continue;
                uint8_t* const to = (is_v ? v_to : k_to) + t * (D * 2);
                const uint32_t x = is_v ? v_swap(t) : k_swap(t);
                uint32_t byte = byte_of(staged_scale[i]);
                bool gone = false;
                if (!whole && is_v) {
                    gone = !((there >> t) & 1u);
                    if (!gone && byte == 255u) gone = unfinite = true;
                    byte = gone ? 0u : byte;
                }
                const float scale = scale_of(byte);
#pragma unroll
                for (int c = 0; c < 4; ++c) *(u32x4*)(to + ((spread<D>(part * 4 + c) ^ x) << 4)) = decode8<E>(gone ? 0u : staged[i][c], scale);
            }
        }
        if (unfinite) unfinite_lds = 1;
    };

    // S^T of a tile, in s[a][i] the score of token 32 (a + part) + 8 (i / 4) + 4 upper + i % 4.  Operands are read two steps ahead; `beside(k)`
    // is done beside step k, and nothing is moved from step to step.
    auto scores = [&](const uint8_t* from, f32x16 (&s)[kS], auto beside) {
        const uint32_t x = spread<D>(upper) ^ k_swap(m);                 // the same 32 tokens on
        const uint8_t* p = from + (kGroups == 4 ? m : part * 32 + m) * (D * 2);
        u32x4 kf[kK][kS];
        auto read = [&](int k) {
#pragma unroll
            for (int a = 0; a < kS; ++a) kf[k][a] = *(const u32x4*)(p + a * (32 * D * 2) + ((spread<D>(2 * k) ^ x) << 4));
        };
#pragma unroll
        for (int a = 0; a < kS; ++a)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[a][i] = 0.f;
        read(0);
        read(1);
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            if (k + 2 < kK) read(k + 2);
#pragma unroll
            for (int a = 0; a < kS; ++a) s[a] = E::mfma32(kf[k][a], qf[k], s[a]);
            beside(k);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto largest = [&](const f32x16 (&s)[kS]) -> float {
        float big = s[0][0];
#pragma unroll
        for (int i = 1; i < 16 * kS; ++i) big = fmaxf(big, s[i >> 4][i & 15]);
        return big;
    };

    // A step multiplies a tile's weights by its values, and beside their exponentials the next tile's keys by the queries.  Meanwhile
    // the keys of the tile behind that and the values of the next are loaded, to the places that the step before has read, and the
    // first wave writes where the tile after them is.
    uint32_t page = 0;
    uint64_t there = 0;
    float big_of = 0.f;                                                  // largest of a step's scores, of this lane's
    // `k_from` has the next tile's keys, `v_from` this tile's values.
    auto step = [&](int32_t tile, f32x16 (&s)[kS], f32x16 (&next)[kS], uint8_t* k_from, uint8_t* k_to, uint8_t* v_from, uint8_t* v_to) {
        const int32_t t0 = range.lo + tile * kWideTile;
        load_rows(tile + 2, k_to, tile + 1, v_to);
        const uint64_t there_next = same_in_wave(there_lds[(tile + 1) & 3]);
        if (!idle && t0 < wave_any.hi && t0 + kWideTile > wave_any.lo) {
            const bool masked = !(there == ~0ull && t0 >= wave_all.lo && t0 + kWideTile <= wave_all.hi);
            if (masked) {
                uint64_t seen = there;                                   // the tile's tokens that this line sees
                if constexpr (kTree) {
                    seen &= see.bits(t0);
                } else {
                    if (see.hi < t0 + kWideTile) seen = see.hi > t0 ? seen & ~(~0ull << (see.hi - t0)) : 0;
                    if (see.lo > t0) seen = see.lo < t0 + kWideTile ? seen & ~0ull << (see.lo - t0) : 0;
                }
                seen >>= 32 * part + 4 * upper;
#pragma unroll
                for (int a = 0; a < kS; ++a) {
                    const uint32_t half = (uint32_t)(seen >> (32 * a));
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[a][i] = half & (1u << (8 * (i >> 2) + (i & 3))) ? s[a][i] : -INFINITY;
                }
            }
            const float big = max_over32(masked ? largest(s) : big_of) * g.to_log2;
            if (__any(big > top + kLag)) {
                const float now = fminf(fmaxf(top, big), kMost), f = rescale(top, now);
                top = now;
                sum = sum * f * f;
#pragma unroll
                for (int d = 0; d < kDims; ++d) o[d] = o[d] * f * f;
            }
            const float against = E::kWeightShift - (top == -INFINITY ? 0.f : top);
            u32x4 p[kPairs / 4];
            float add[2] = {0.f, 0.f};
            auto weights = [&](int from, int to) {                       // pairs of them
#pragma unroll
                for (int j = from; j < to; ++j) {
                    const float x0 = __builtin_amdgcn_exp2f(fmaf(s[j >> 3][2 * (j & 7)], g.to_log2, against)),
                                x1 = __builtin_amdgcn_exp2f(fmaf(s[j >> 3][2 * (j & 7) + 1], g.to_log2, against));
                    add[0] += x0;
                    add[1] += x1;
                    p[j >> 2][j & 3] = E::pack2(x0, x1);                 // rounded to nearest: see the head of this file
                }
            };
            // O^T's first operand: step u takes tokens 16 u + {0, 8} + 4 upper + 0 .. 3
            const uint32_t i16 = lane & 15u, low = 2 * ((lane >> 4) & 1u) + ((i16 >> 1) & 1u);
            constexpr int kSteps = 2 * kS * kDims;
            u32x4 vf[kSteps];
            auto read = [&](int i) {
                const uint32_t ta = 32 * part + 16 * (i / kDims) + 4 * upper + (i16 >> 2);
                const uint8_t *row_a = v_from + ta * (D * 2) + (i16 & 1u) * 8, *row_b = row_a + 8 * (D * 2);
                const uint32_t at = (spread<D>(4 * (i % kDims)) ^ spread<D>(low) ^ v_swap(ta)) << 4;     // the same eight tokens on
                const u32x2 a = read_transposed(row_a + at), b = read_transposed(row_b + at);
                vf[i] = u32x4{a[0], a[1], b[0], b[1]};
            };
            __builtin_amdgcn_sched_barrier(0);
            scores(k_from, next, [&](int k) {
                weights(kPairs * 3 / 4 * k / kK, kPairs * 3 / 4 * (k + 1) / kK);
                if (k == kK - 1) { read(0); read(1); }
            });
            big_of = next[0][0];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (i + 2 < kSteps) read(i + 2);
                o[i % kDims] = E::mfma32(vf[i], p[i / kDims], o[i % kDims]);
                if (i < kSteps / 2) {
                    weights(kPairs * 3 / 4 + kPairs / 4 * i / (kSteps / 2), kPairs * 3 / 4 + kPairs / 4 * (i + 1) / (kSteps / 2));
                } else {
#pragma unroll
                    for (int j = 16 * kS * (i - kSteps / 2) / (kSteps / 2); j < 16 * kS * (i + 1 - kSteps / 2) / (kSteps / 2); ++j) big_of = fmaxf(big_of, next[j >> 4][j & 15]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            sum += add[0] + add[1];
        } else if (!idle) {
            scores(k_from, next, [](int) {});
            big_of = largest(next);
        }
        if (wave == 0) {
            place_rows(tile + 3, page);
            page = load_page(tile + 4);
        }
        store_rows(tile + 2, k_to, tile + 1, v_to, there_next);
        there = there_next;
        __syncthreads();
    };

    if (tiles > 0) {
        if (wave == 0) {
            const uint32_t page0 = load_page(0), page1 = load_page(1), page2 = load_page(2);
            page = load_page(3);
            place_rows(0, page0);
            place_rows(1, page1);
            place_rows(2, page2);
        }
        __syncthreads();
        there = same_in_wave(there_lds[0]);
        load_rows(0, k_even, 0, v_even);
        if constexpr (kBits == 4) store_rows(0, k_even, 0, v_even, there);
        load_rows(1, k_odd, tiles, v_odd);
        if constexpr (kBits == 4) store_rows(1, k_odd, tiles, v_odd, 0);
        else store_rows(0, k_even, 0, v_even, there);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kK; ++k) arrived(qf[k]);
        f32x16 s0[kS], s1[kS];
        scores(k_even, s0, [](int) {});
        big_of = largest(s0);
        __syncthreads();
        for (int32_t tile = 0; tile < tiles; tile += 2) {
            step(tile, s0, s1, k_odd, k_even, v_even, v_odd);
            if (tile + 1 < tiles) step(tile + 1, s1, s0, k_even, k_odd, v_odd, v_even);
        }
    }

    if (bad_page) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
    sum = sum_over32(sum);
    if constexpr (kGroups == 2) {
        // The waves with the second tokens hand theirs over: what takes a tile in the loop holds a wave's sums exactly.  The loop's last
        // barrier is behind its last read.
        float* const theirs = (float*)(lot ? v_even : k_even);
        if (part) {
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) theirs[(d * 16 + i) * 64 + lane] = o[d][i];
            joined[lot][lane] = f32x2{top, sum};
        }
        __syncthreads();
        if (part) return;
        const f32x2 other = joined[lot][lane];
        const float now = fmaxf(top, other[0]), mine_by = rescale(top, now), theirs_by = rescale(other[0], now);
        sum = sum * mine_by * mine_by + other[1] * theirs_by * theirs_by;
#pragma unroll
        for (int d = 0; d < kDims; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * mine_by * mine_by + theirs[(d * 16 + i) * 64 + lane] * theirs_by * theirs_by;
        top = now;
    }
    if (tiles > 0 && unfinite_lds && !idle) {                            // behind the loop's last barrier
#pragma unroll 1
        for (int32_t tile = 0; tile < tiles; ++tile) {
            // the tiles that store_rows took values from: those that are not whole
            const int32_t t0 = range.lo + tile * kWideTile;
            const uint32_t page_no = load_page(tile);
            const uint64_t held = __ballot(t0 + (int32_t)lane < range.hi && page_no < g.c.n_pages);
            if (held == ~0ull && seen_by_all(t0)) continue;
#pragma unroll 1
            for (int32_t i = 0; i < kWideTile; ++i) {
                if (!((held >> i) & 1u)) continue;
                const int32_t t = t0 + i;
                const uint32_t in = (uint32_t)__builtin_amdgcn_readlane((int)page_no, i);
                if (!see.sees(t)) continue;
                const RowAt<kBits> at = row_at<D, kBits>(g.c, in, (uint32_t)t, head);
#pragma unroll
                for (int d = 0; d < kDims; ++d)
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        float x[4] = {o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]};
                        add_unfinite<E, D, kBits>(x, g.c.v, at, d * 32 + b * 8 + upper * 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k) o[d][4 * b + k] = x[k];
                    }
            }
        }
    }
    bool large = false;                                                  // this line's sums passed 32 bits
    if constexpr (E::kLarge) {
        float x = 0.f;
#pragma unroll
        for (int d = 0; d < kDims; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) x = fmaf(o[d][i], 0.f, x);
        x = sum_over32(x);
        const bool odd = mine && sum > 0.f && sum < INFINITY && !(x == 0.f);
        if (__any(odd)) {
            const AttendArgs& a = args_again();
            const WideUnit u = wide_unit(a, a.first + blockIdx.x);
            const KvSeq q = kv_sequence(a.b, u.seq);
            const int32_t line0 = (int32_t)u.line_tile * kLines, lines = q.rows * (int32_t)a.group;
            const Range range = token_range<kTree>(a, q, line0, line0 + kLines < lines ? line0 + kLines - 1 : lines - 1, u.split);
            const Unfinite<D> unfinite = find_unfinite<E, D, kBits>(a, u.seq, u.head, range);
            const int32_t first_line = line0 + (int32_t)lot * 32, my_line = first_line + (int32_t)(lane_again() & 31u);
            const Sight<kTree> see = sight<kTree>(a, q, my_line < lines ? my_line / (int32_t)a.group : 0);
            bool more = false;
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    more |= !unfinite.seen(see, d * 32 + (i >> 2) * 8 + upper * 4 + (i & 3), i % (D / 64)) && !(fabsf(o[d][i]) < INFINITY);
            const uint64_t here = __ballot(odd && more);
            uint32_t lines_left = (uint32_t)here | (uint32_t)(here >> 32);
            large = lines_left >> m & 1u;
#pragma unroll 1
            for (; lines_left; lines_left &= lines_left - 1) {
                const int i = __builtin_ctz(lines_left);
                plain_line<E, D, kBits, kTree>(a, q, u.seq, u.head, u.split, first_line + i, range,
                                        __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(top), i)),
                                        __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(sum), i)));
            }
        }
    }
    if (!mine) return;                                                   // plain_line has stored lines that are large
    const uint64_t out_row = (uint64_t)(q.row0 + row);
    if (g.part_o) {
        const uint64_t at = (out_row * g.q_heads + q_head) * g.n_splits + split;
        if (large) return;
        if (upper == 0) dev_store(g.part_ml + at * 2, f32x2{top, sum});
        if (sum == 0.f) return;                                          // join_kernel does not read it
#pragma unroll
        for (int d = 0; d < kDims; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b) dev_store(g.part_o + at * D + d * 32 + b * 8 + upper * 4, f32x4{o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2], o[d][4 * b + 3]});
    } else {
        const float scale = sum == 0.f ? 0.f : 1.f / sum;
        if (sum == 0.f) {                                                // no weight: zeros, whatever the values
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        }
        uint8_t* to = g.out + out_row * g.out_stride + ((uint64_t)q_head * D + upper * 4) * 2;
        if (!large)
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    dev_store(to + (d * 32 + b * 8) * 2, u32x2{E::pack2(o[d][4 * b] * scale, o[d][4 * b + 1] * scale), E::pack2(o[d][4 * b + 2] * scale, o[d][4 * b + 3] * scale)});
        if (g.lse && upper == 0) g.lse[out_row * g.q_heads + q_head] = lse_of(top, sum, E::kWeightShift);
    }
}

// ---- the splits' parts ---------------------------------------------------------------------------
// o = sum_i o_i 2^(m_i - m) / sum_i l_i 2^(m_i - m).  A workgroup for each row and query head, whose waves take parts in turn, or,
// where a wave has few parts to go through anyway, a wave for each: kLines of them to a workgroup.
template <class E, int D, int kLines, bool kTree>
__global__ void __launch_bounds__(256) join_kernel(const AttendArgs g)
{
    constexpr int kPer = D / 64, kAhead = 4;                             // values of a lane; parts that a wave has in flight
    constexpr uint32_t kTurn = kWaves / kLines;                          // waves that share a line
    __shared__ float o_lds[kLines == 1 ? kWaves : 1][D], sum_lds[kWaves];
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t line = blockIdx.x * kLines + wave / kTurn, turn = wave % kTurn;
    const uint32_t row = line / g.q_heads, q_head = line - row * g.q_heads;
    const KvSeq q = kv_sequence(g.b, blockIdx.y);
    if ((int32_t)row >= q.rows) return;                                  // with kLines 1 the whole workgroup
    const uint64_t out_row = (uint64_t)q.row0 + row, first = (out_row * g.q_heads + q_head) * g.n_splits;
    const uint32_t n = splits_of<kTree>(g, q);
    float top = -INFINITY, sum = 0.f, y[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) y[k] = 0.f;
    for (uint32_t i = lane; i < n; i += 64) top = fmaxf(top, dev_load<f32x2>(g.part_ml + (first + i) * 2)[0]);
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
    for (uint32_t i = turn; i < n; i += kTurn * kAhead) {
        f32x2 ml[kAhead];
        float part[kAhead][kPer];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const uint64_t at = first + min(i + a * kTurn, n - 1);
            ml[a] = dev_load<f32x2>(g.part_ml + at * 2);
#pragma unroll
            for (int k = 0; k < kPer; ++k) part[a][k] = dev_load<float>(g.part_o + at * D + lane * kPer + k);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (i + a * kTurn >= n || ml[a][1] == 0.f) continue;         // an empty part has a sum of 0 and no output
            const float f = rescale(ml[a][0], top);
            sum += ml[a][1] * f * (f * kPart);
#pragma unroll
            for (int k = 0; k < kPer; ++k) y[k] += part[a][k] * f * (f * kPart);
        }
    }
    uint8_t* const to = g.out + out_row * g.out_stride + (uint64_t)q_head * D * 2;
    if constexpr (kLines > 1) {
        const float scale = sum == 0.f ? 0.f : 1.f / sum;
        if constexpr (kPer == 1) {
            dev_store(to + lane * 2, (uint16_t)E::pack2(y[0] * scale, 0.f));
        } else {
#pragma unroll
            for (int k = 0; k < kPer; k += 2) dev_store(to + (lane * kPer + k) * 2, E::pack2(y[k] * scale, y[k + 1] * scale));
        }
        if (g.lse && lane == 0) g.lse[out_row * g.q_heads + q_head] = lse_of(top, sum * (1.f / kPart), E::kWeightShift);
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) o_lds[wave][lane * kPer + k] = y[k];
        if (lane == 0) sum_lds[wave] = sum;
        __syncthreads();
        if (threadIdx.x >= D / 2) return;                                // two values a thread
        float total = 0.f, a = 0.f, b = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            total += sum_lds[w];
            a += o_lds[w][threadIdx.x * 2];
            b += o_lds[w][threadIdx.x * 2 + 1];
        }
        const float scale = total == 0.f ? 0.f : 1.f / total;
        dev_store(to + threadIdx.x * 4, E::pack2(a * scale, b * scale));
        if (g.lse && threadIdx.x == 0) g.lse[out_row * g.q_heads + q_head] = lse_of(top, total * (1.f / kPart), E::kWeightShift);
    }
}

// ---- host ----------------------------------------------------------------------------------------
struct Shape {
    uint32_t line_tiles;       // narrow: 16-line tiles of a workgroup (1, 2 or 4); wide: workgroups over the lines
    bool wide, half;           // half: 64 lines to a workgroup
    uint32_t n_splits, split_tokens;
    uint64_t workspace;
};

// Which kernel, and how many splits.  Few lines: enough workgroups to fill the 256 compute units several times over, while a split
// keeps enough tokens for its waves to have a tile in flight beside the one they work on; a context of up to 768 tokens stays
// whole, as a split of it saves less than its join takes, 3 to 4 us.  Whole and split, one row of 8 heads of 128 dimensions, 16 bits: 512
// tokens 9.3 and 10.0 us, 768 11.8 and 10.0; 4 bits: 640 8.9 and 9.1, 768 9.8 and 9.2; 64 dimensions: 768 8.4 and 8.5; 64 rows: 768
// 33.9 and 38.4.  Of 256 dimensions in 16 bits the two cross at 400 tokens already (768: 21.3 and 14.3), which the rule does not follow.
// Many lines: enough workgroups to fill the compute units, or, if they are filled already and contexts so long that joins cost
// little, to leave none with much more to do than others.  Three chunks of 511 rows, 384 workgroups, 4 bits, whole and in the rule's
// three: behind 8k tokens 265 and 275 us, 16k 527 and 511, 32k 1047 and 977; 1024 workgroups stay whole behind 16k (1116, and
// 1198 in two).
//
// Trees of 33 to 64 lines take the wide kernel with two waves to 32 lines; the narrow one has one wave to a SIMD then.  16 rows of 32 heads on
// 8 of 128 dimensions, narrow, wide and so: 32 of them over 5k tokens in 4 bits 160, 131 and 96 us, in 16 bits 222, 153 and 145; 4 over 32k
// 138, 86 and 83, 189, 125 and 122; 500 tokens 18.5, and 18.5 so, 20.7 and 16.8; of 64 dimensions 13 and 15, which the rule does not follow.  Of these workgroups 512 are
// enough: 32 trees over 2k to 8k tokens take 149 us with 512, with 256, 1024 and 1536 229, 152 and 168.
inline Shape shape_of(const tent_kv_cache& c, const tent_kv_batch& b, const tent_kv_attend_args& a, bool tree)
{
    Shape s{};
    const uint32_t group = a.q_heads / c.kv_heads;
    const uint64_t lines = (uint64_t)b.max_rows * group;
    s.wide = lines > (tree || c.head_dim == 256 ? 32u : 64u);
    s.half = tree && s.wide && lines <= 64;
    s.line_tiles = s.wide ? (uint32_t)((lines + kWideLines - 1) / kWideLines) : lines <= 16 ? 1 : lines <= 32 ? 2 : 4;
    uint64_t span = b.max_kv;                                            // most tokens that a sequence's rows see together
    if (a.window && !(a.flags & TENT_KV_ATTEND_ALL) && (uint64_t)a.window + b.max_rows < span) span = (uint64_t)a.window + b.max_rows;
    if (a.window && (a.flags & TENT_KV_ATTEND_ALL) && a.window < span) span = a.window;
    span += kStep;                                                       // the first token is rounded down
    const uint64_t units = (uint64_t)b.n_seqs * c.kv_heads * (s.wide ? s.line_tiles : 1);
    const bool filled = s.wide && !s.half && units >= 256;
    const uint64_t wanted = filled ? 1024 : s.wide ? 512 : 1536, least = filled ? 4096 : s.wide ? 512 : 256;
    uint64_t n = (wanted + units - 1) / units, most = filled ? span / least : (span + least - 1) / least;
    n = n > most ? most : n;
    n = n < 1 || (!s.wide && span <= 768) ? 1 : n;
    const uint64_t tokens = ((span + n - 1) / n + 127) / 128 * 128;
    s.split_tokens = (uint32_t)tokens;
    s.n_splits = (uint32_t)((span + tokens - 1) / tokens);
    if (s.n_splits > 1) s.workspace = (uint64_t)b.n_rows * a.q_heads * s.n_splits * (c.head_dim + 2) * 4;
    return s;
}

inline int check(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args)
{
    int rc = kv_check_cache(cache);
    if (rc == TENT_OK) rc = kv_check_batch(cache, batch);
    if (rc != TENT_OK) return rc;
    if (!args || (args->flags & ~(uint32_t)TENT_KV_ATTEND_ALL)) return TENT_ERR_INVALID;
    if (args->q_heads < 1 || args->q_heads > TENT_KV_MAX_HEADS || args->q_heads % cache->kv_heads) return TENT_ERR_RANGE;
    if (!(args->scale > 0.f) || args->scale > 3.4e38f || args->window > (1u << 30)) return TENT_ERR_RANGE;
    return TENT_OK;
}

inline uint64_t blocks_of(const Shape& s, const AttendArgs& g)
{
    if (s.wide) return (uint64_t)s.line_tiles * s.n_splits * g.b.n_seqs * g.c.heads;
    return ((uint64_t)g.b.n_seqs * s.n_splits + 7) / 8 * 8 * g.c.heads;
}

template <class E, int D, int kBits, bool kTree>
int launch(const Shape& s, AttendArgs g, hipStream_t stream)
{
    const dim3 threads(256);
    const int rc = launch_blocks(blocks_of(s, g), [&](uint32_t first, uint32_t blocks) {
        const dim3 grid(blocks);
        g.first = first;
        if (s.wide) {
            if constexpr (kTree) {
                if (s.half) hipLaunchKernelGGL((wide_kernel<E, D, kBits, kTree, 2>), grid, threads, 0, stream, g);
            }
            if (!s.half) hipLaunchKernelGGL((wide_kernel<E, D, kBits, kTree, 4>), grid, threads, 0, stream, g);
        } else if (s.line_tiles == 1) {
            hipLaunchKernelGGL((narrow_kernel<E, D, kBits, 1, kTree>), grid, threads, 0, stream, g);
        } else if (s.line_tiles == 2) {
            hipLaunchKernelGGL((narrow_kernel<E, D, kBits, 2, kTree>), grid, threads, 0, stream, g);
        } else {
            if constexpr (D != 256 && !kTree) hipLaunchKernelGGL((narrow_kernel<E, D, kBits, 4, kTree>), grid, threads, 0, stream, g);
        }
    });
    if (rc != TENT_OK) return rc;
    if (g.part_o) {
        // There are splits where fewer workgroups are wanted than the 1536 of shape_of, of 128 lines at most: a launch holds their joins.
        const uint64_t join = (uint64_t)g.b.max_rows * g.q_heads;
        // A wave to a line: up to four parts are all in flight at once.
        if (s.n_splits <= 4) hipLaunchKernelGGL((join_kernel<E, D, kWaves, kTree>), dim3((uint32_t)((join + kWaves - 1) / kWaves), g.b.n_seqs), threads, 0, stream, g);
        else hipLaunchKernelGGL((join_kernel<E, D, 1, kTree>), dim3((uint32_t)join, g.b.n_seqs), threads, 0, stream, g);
        if (hipGetLastError() != hipSuccess) return TENT_ERR_HIP;
    }
    return TENT_OK;
}

// The call behind its entry points; `args` has passed check, and `tree`, which is null without one, has too.
template <bool kTree>
int attend(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args, const tent_kv_tree* tree, void* stream)
{
    int rc;
    if (batch->n_seqs == 0 || batch->n_rows == 0) return TENT_OK;
    const uint32_t D = cache->head_dim;
    if ((rc = kv_check_rows(args->q, args->q_stride, args->q_heads, D, batch->n_rows)) != TENT_OK) return rc;
    if ((rc = kv_check_rows(args->out, args->out_stride, args->q_heads, D, batch->n_rows)) != TENT_OK) return rc;
    if ((uintptr_t)args->lse & 3u) return TENT_ERR_INVALID;
    const Shape s = shape_of(*cache, *batch, *args, kTree);
    if (s.workspace && (!args->workspace || !kv_aligned(args->workspace))) return TENT_ERR_INVALID;
    if (s.workspace > args->workspace_bytes) return TENT_ERR_RANGE;
    AttendArgs g{};
    g.c = kv_cache_dev(*cache);
    g.b = *batch;
    g.q = static_cast<const uint8_t*>(args->q);
    g.out = static_cast<uint8_t*>(args->out);
    g.lse = args->lse;
    g.q_stride = args->q_stride * 2;
    g.out_stride = args->out_stride * 2;
    g.q_heads = args->q_heads;
    g.group = args->q_heads / cache->kv_heads;
    g.window = args->window;
    g.all = args->flags & TENT_KV_ATTEND_ALL ? 1 : 0;
    g.to_log2 = args->scale * kLog2e;
    g.n_splits = s.n_splits;
    g.split_tokens = s.split_tokens;
    g.line_tiles = s.line_tiles;
    if (s.workspace) {
        g.part_o = static_cast<float*>(args->workspace);
        g.part_ml = g.part_o + (uint64_t)batch->n_rows * args->q_heads * s.n_splits * D;
    }
    if constexpr (kTree) {
        g.masks = tree->masks;
        g.mask_stride = tree->mask_stride;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
#define TENT_ATTEND(dim)                                                                                                            \
    (cache->type == TENT_BF16 ? (cache->bits == 16 ? launch<Bf16, dim, 16, kTree>(s, g, st) : launch<Bf16, dim, 4, kTree>(s, g, st)) \
                              : (cache->bits == 16 ? launch<Fp16, dim, 16, kTree>(s, g, st) : launch<Fp16, dim, 4, kTree>(s, g, st)))
    return D == 64 ? TENT_ATTEND(64) : D == 128 ? TENT_ATTEND(128) : TENT_ATTEND(256);
#undef TENT_ATTEND
}

}  // namespace
}  // namespace tent
