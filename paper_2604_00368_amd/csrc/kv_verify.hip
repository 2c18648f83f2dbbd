// Verification of drafted tokens: tent_kv_verify.
//
// From the row c that stands last the rows behind it are tried.  After k rows were refused the residual is
//   r(t) = max(p(t) - b q(t), 0) / z,   z = sum_t max(p(t) - b q(t), 0),   p = target[c], q = draft[c]
// (by induction: max(max(p - b q, 0) / z - q, 0) = max(p - (b + z) q, 0) / z), with b = 0, z = 1 before the first, then b = 1, b + z, ..
// So the way is decided by single values, and by one sum over the vocabulary for each row that is refused: the last of these sums is
// what the next token is drawn from, too.  Without `draft` a refused token is taken out of p, and a sum is needed at the end only.
//
// A workgroup does a sequence by itself: its first wave goes the way, and where a sum is needed its waves sum pieces of the vocabulary in
// turn.  Where the vocabulary is long and sequences are few the first sum, most often the only one, is made by a launch ahead of it, in
// which workgroups go the way as far as that sum and take some pieces each.
//
// Bound by the rate at which one compute unit reads (some 100 GB/s; 64-bit arithmetic beside it) where a workgroup is alone, by latencies
// (lengths, rows, their probabilities, a piece, barriers) where there is little to read.  Measured, fp32: 6 rows that were chosen, 32,000
// tokens, 11.6 us; 64 sequences of 4 to 8 drawn rows, 128,000 tokens, 14 us (65 MB, 4.6 TB/s) for the sums ahead and 9.6 behind them.
#include "kv_elem.h"

namespace tent {
namespace {

constexpr uint32_t kPiece = 2048;      // tokens of a piece, a wave's
constexpr uint32_t kMostPieces = TENT_KV_MAX_VOCAB / kPiece;

// Where a sequence's way has got to.
struct alignas(16) Way {
    double b, z;                       // of the residual (with draft); z: of what is left (without)
    int32_t at;                        // the row that stands last
    int32_t next;                      // rows from here on are still to be tried
    int32_t stand;                     // rows that stand
    int32_t refused;                   // rows behind `at` that do not
    int32_t known;                     // z is the sum, not only what stands in its place before the first refusal
    int32_t whole;                     // nothing was left: the target's probabilities as they are
    int32_t ended;                     // no row is left to try, and z is known to be the sum
    int32_t reserved;
};
static_assert(sizeof(Way) == 48, "three vectors");

struct VerifyArgs {
    tent_kv_verify_args a;
    tent_kv_batch b;
    Way* ways;                         // [n_seqs]: where the launch ahead needed its sum; null: there is no such launch
    double* sums;                      // [n_seqs][pieces]: that sum's
    uint32_t pieces;
    uint32_t first;                    // of the launch's workgroups
};

template <uint32_t kType>
struct Prob;
template <>
struct Prob<TENT_FP32> {
    using Raw = float;
    typedef float Vec __attribute__((ext_vector_type(4), aligned(4)));
    static constexpr uint32_t kPer = 4;
    static __device__ __forceinline__ float value(float x) { return x; }
    // Whether all of a vector are probabilities, or 0: by their patterns, as whole numbers.
    static __device__ __forceinline__ bool sound(const Vec& v)
    {
        uint32_t most = 0;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) most = max(most, __float_as_uint(v[i]));
        return most < 0x7F800000u;
    }
};
template <>
struct Prob<TENT_BF16> {
    using Raw = uint16_t;
    typedef uint16_t Vec __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr uint32_t kPer = 8;
    static __device__ __forceinline__ float value(uint16_t x) { return Bf16::to_float(x); }
    static __device__ __forceinline__ bool sound(const Vec& v)
    {
        uint32_t most = 0;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) most = max(most, (uint32_t)v[i]);
        return most < Bf16::kInf;
    }
};
template <>
struct Prob<TENT_FP16> {
    using Raw = uint16_t;
    typedef uint16_t Vec __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr uint32_t kPer = 8;
    static __device__ __forceinline__ float value(uint16_t x) { return Fp16::to_float(x); }
    static __device__ __forceinline__ bool sound(const Vec& v)
    {
        uint32_t most = 0;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) most = max(most, (uint32_t)v[i]);
        return most < Fp16::kInf;
    }
};
// What is no probability counts as 0.
__device__ __forceinline__ double sound(float x) { return x > 0.f && x < INFINITY ? (double)x : 0.0; }

__device__ __forceinline__ double from_lane(double x, int lane)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return __longlong_as_double((long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)u, lane)));
}
// A value of another lane of 16, by one of the patterns that need no LDS.
template <int kPattern>
__device__ __forceinline__ double of_row(double x)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)u, kPattern, 0xF, 0xF, true), hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(u >> 32), kPattern, 0xF, 0xF, true);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double wave_sum(double x)
{
    x += of_row<0xB1>(x);                                                // lane ^ 1
    x += of_row<0x4E>(x);                                                // lane ^ 2
    x += of_row<0x141>(x);                                               // the other four of eight, in reverse
    x += of_row<0x140>(x);                                               // the other eight of 16
    return (from_lane(x, 0) + from_lane(x, 16)) + (from_lane(x, 32) + from_lane(x, 48));
}

template <uint32_t kType>
__device__ __forceinline__ double value_at(const void* p, uint64_t row, uint64_t stride, uint32_t token, uint32_t vocab)
{
    using P = Prob<kType>;
    if (token >= vocab) return 0.0;
    return sound(P::value(dev_load<typename P::Raw>((const typename P::Raw*)p + row * stride + token)));
}

// 64 rows, one a lane, as far as they are behind a row of their sequence.
struct Rows {
    int32_t first;                     // of the 64, -1: none yet
    int32_t parent;                    // -1: behind none
    uint32_t token;
    double u, p, d;
};
template <uint32_t kType>
__device__ __forceinline__ Rows load_rows(const VerifyArgs& g, const KvSeq& q, int32_t first)
{
    const tent_kv_verify_args& a = g.a;
    const int32_t i = first + (int32_t)(threadIdx.x & 63u);
    Rows r{first, -1, 0u, 0.0, 0.0, 0.0};
    if (i >= 1 && i < q.rows) {
        const uint64_t row = (uint64_t)(q.row0 + i);
        const int32_t parent = a.parents ? a.parents[row] : i - 1;
        r.token = (uint32_t)a.tokens[row];
        r.u = (double)a.accept[row];
        if (parent >= 0 && parent < i) {
            r.parent = parent;
            r.p = value_at<kType>(a.target, (uint64_t)(q.row0 + parent), a.target_stride, r.token, a.vocab);
            if (a.draft) r.d = value_at<kType>(a.draft, (uint64_t)(q.row0 + parent), a.draft_stride, r.token, a.vocab);
        }
    }
    return r;
}

// The residual of one token, times z.
__device__ __forceinline__ double residual(double p, double q, double b)
{
    return fmax(fma(-b, q, p), 0.0);
}

// One wave goes on until a sum is needed that is not known, or to the end.  `path`, if given, gets the rows that stand.
template <uint32_t kType>
__device__ void go_on(const VerifyArgs& g, const KvSeq& q, Way& w, Rows& rows, int32_t* path)
{
    const tent_kv_verify_args& a = g.a;
    const int32_t lane = (int32_t)(threadIdx.x & 63u);
    while (w.next < q.rows) {
        const int32_t block = w.next & ~63, i = block + lane;
        if (rows.first != block) rows = load_rows<kType>(g, q, block);
        uint64_t left = __ballot(i >= w.next && rows.parent == w.at);
        while (left) {
            const int k = __builtin_ctzll(left);
            left &= left - 1;
            const double uk = from_lane(rows.u, k), pk = from_lane(rows.p, k), dk = from_lane(rows.d, k);
            double r = residual(pk, dk, w.b);
            if (!a.draft && w.refused) {                                 // a token that was taken out already
                const uint32_t x = (uint32_t)__builtin_amdgcn_readlane((int)rows.token, k);
                bool twice = false;
                for (int32_t j0 = 0; j0 <= block; j0 += 64) {
                    const int32_t j = j0 + lane;
                    const bool before = j < block + k && j < q.rows;
                    const uint64_t at = (uint64_t)(q.row0 + (before ? j : 0));
                    twice |= __any(before && (a.parents ? a.parents[at] : j - 1) == w.at && j > w.at && (uint32_t)a.tokens[at] == x);
                }
                if (twice) r = 0.0;
            }
            if (uk * (a.draft ? dk * w.z : w.z) < r) {
                w.at = block + k;
                if (path && lane == 0) path[w.stand] = w.at;
                ++w.stand;
                w.refused = 0;
                w.b = 0.0;
                w.z = 1.0;
                w.known = 0;
                left = __ballot(rows.parent == w.at);                    // all of them are later ones
                continue;
            }
            ++w.refused;
            if (a.draft) {
                w.next = block + k + 1;
                w.b += w.refused > 1 ? w.z : 1.0;
                w.known = 0;
                return;
            }
            w.z = w.z > r ? w.z - r : 0.0;
        }
        w.next = block + 64;
    }
    if (!w.known) return;
    if (w.z > 0.0 || w.whole) {
        w.ended = 1;
    } else {                                                             // nothing is left: the target's own probabilities
        w.whole = 1;
        w.known = 0;
        w.b = 0.0;
    }
}

// LDS written by some lanes of a wave is read by others: the wave's LDS operations keep their order, the compiler has to as well.
__device__ __forceinline__ void same_wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A piece's tokens in a wave's registers: kVecs vectors a lane, of lanes side by side or (kInOrder) of a lane side by side.
template <uint32_t kType, bool kInOrder>
struct Piece {
    using P = Prob<kType>;
    using Vec = typename P::Vec;
    using Raw = typename P::Raw;
    static constexpr uint32_t kPer = P::kPer, kVecs = kPiece / kPer / 64;
    Vec x[kVecs], y[kVecs];
    bool two, out;                     // there is something to take off; tokens were taken out
    double b;
    uint32_t* gone;                    // those, as bits: the wave's own words

    // The number in the piece of a vector's first token.
    static __device__ __forceinline__ uint32_t at(uint32_t j)
    {
        const uint32_t lane = threadIdx.x & 63u;
        return (kInOrder ? lane * kVecs + j : j * 64 + lane) * kPer;
    }
    __device__ __forceinline__ void load(const VerifyArgs& g, const KvSeq& q, const Way& w, uint32_t piece, uint32_t* wave_gone)
    {
        const tent_kv_verify_args& a = g.a;
        const uint32_t t0 = piece * kPiece, n = a.vocab - t0 < kPiece ? a.vocab - t0 : kPiece;
        two = a.draft && w.b != 0.0;
        out = !a.draft && w.refused && !w.whole;
        b = w.b;
        gone = wave_gone;
        const Raw* const p = (const Raw*)a.target + (uint64_t)(q.row0 + w.at) * a.target_stride + t0;
        const Raw* const d = two ? (const Raw*)a.draft + (uint64_t)(q.row0 + w.at) * a.draft_stride + t0 : p;
        if (n == kPiece) {
#pragma unroll
            for (uint32_t j = 0; j < kVecs; ++j) x[j] = dev_load<Vec>(p + at(j));
            if (two)
#pragma unroll
                for (uint32_t j = 0; j < kVecs; ++j) y[j] = dev_load<Vec>(d + at(j));
        } else {                                                         // the row's end is inside
#pragma unroll
            for (uint32_t j = 0; j < kVecs; ++j)
#pragma unroll
                for (uint32_t i = 0; i < kPer; ++i) {
                    x[j][i] = at(j) + i < n ? dev_load<Raw>(p + at(j) + i) : Raw(0);
                    if (two) y[j][i] = at(j) + i < n ? dev_load<Raw>(d + at(j) + i) : Raw(0);
                }
        }
        if (out) {                                                       // beside the loads
            const uint32_t lane = threadIdx.x & 63u;
            gone[lane] = 0;
            static_assert(kPiece == 32 * 64, "a word a lane");
            same_wave_order();
            for (int32_t i = w.at + 1 + (int32_t)lane; i < q.rows; i += 64) {
                const uint32_t t = (uint32_t)a.tokens[q.row0 + i] - t0;
                if ((a.parents ? a.parents[q.row0 + i] : i - 1) == w.at && t < n) atomicOr(&gone[t / 32], 1u << (t & 31u));
            }
            same_wave_order();
        }
    }
    // Calls f(i, r) for the tokens of vector j in their order, with their residuals times z.
    template <class F>
    __device__ __forceinline__ void each(uint32_t j, F f) const
    {
        const uint32_t bits = out ? gone[at(j) / 32] >> (at(j) & 31u) & ((1u << kPer) - 1) : 0u;
        if (__any(!P::sound(x[j]) || (two && !P::sound(y[j])) || bits)) {        // what is no probability, and tokens that were taken out
#pragma unroll
            for (uint32_t i = 0; i < kPer; ++i) {
                const double p = sound(P::value(x[j][i]));
                f(i, bits >> i & 1u ? 0.0 : two ? residual(p, sound(P::value(y[j][i])), b) : p);
            }
        } else if (two) {
#pragma unroll
            for (uint32_t i = 0; i < kPer; ++i) f(i, residual((double)P::value(x[j][i]), (double)P::value(y[j][i]), b));
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kPer; ++i) f(i, (double)P::value(x[j][i]));
        }
    }
};
template <uint32_t kType>
__device__ __forceinline__ double sum_of_piece(const VerifyArgs& g, const KvSeq& q, const Way& w, uint32_t piece, uint32_t* gone)
{
    Piece<kType, false> p;
    p.load(g, q, w, piece, gone);
    double sum[2] = {0.0, 0.0};
#pragma unroll
    for (uint32_t j = 0; j < p.kVecs; ++j) p.each(j, [&](uint32_t i, double r) { sum[i & 1] += r; });
    return wave_sum(sum[0] + sum[1]);
}

__device__ __forceinline__ Way start_of() { return Way{0.0, 1.0, 0, 1, 1, 0, 0, 0, 0, 0}; }

// Ahead: the first sum of every sequence, a wave to a piece.
constexpr uint32_t kAheadWaves = 4;
template <uint32_t kType>
__global__ void __launch_bounds__(64 * kAheadWaves) verify_ahead_kernel(const VerifyArgs g)
{
    __shared__ Way way;
    __shared__ uint32_t gone[kAheadWaves][kPiece / 32];
    const uint32_t parts = (g.pieces + kAheadWaves - 1) / kAheadWaves;
    const uint32_t block = g.first + blockIdx.x, seq = block / parts, part = block - seq * parts, wave = threadIdx.x >> 6;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.rows < 1) return;
    if (wave == 0) {
        Way w = start_of();
        Rows rows = load_rows<kType>(g, q, 0);
        go_on<kType>(g, q, w, rows, part == 0 ? g.a.path + (uint64_t)seq * g.a.path_stride : nullptr);
        if (threadIdx.x == 0) {
            way = w;
            if (part == 0) g.ways[seq] = w;
        }
    }
    __syncthreads();
    const uint32_t piece = part * kAheadWaves + wave;
    if (piece >= g.pieces) return;
    const double sum = sum_of_piece<kType>(g, q, way, piece, gone[wave]);
    if ((threadIdx.x & 63u) == 0) dev_store(g.sums + (uint64_t)seq * g.pieces + piece, sum);
}

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;
template <uint32_t kType>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyArgs g)
{
    __shared__ Way way;
    __shared__ uint32_t gone[kWaves][kPiece / 32];
    __shared__ double sums[kMostPieces];
    const tent_kv_verify_args& a = g.a;
    const uint32_t seq = g.first + blockIdx.x, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const KvSeq q = kv_sequence(g.b, seq);
    int32_t* const path = a.path + (uint64_t)seq * a.path_stride;
    if (q.bad && threadIdx.x == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    if (q.rows < 1) {
        for (uint32_t i = threadIdx.x; i < g.b.max_rows; i += kThreads) path[i] = -1;
        if (threadIdx.x == 0) {
            a.counts[seq] = 0;
            a.token[seq] = -1;
        }
        return;
    }
    Rows rows;                                                           // the first wave's
    double next = 0.0;
    if (wave == 0) {
        Way w = start_of();
        double z = 0.0;
        if (g.ways) {                                                    // beside the rows' loads
            w = g.ways[seq];
            for (uint32_t c = lane; c < g.pieces; c += 64) {
                const double part = dev_load<double>(g.sums + (uint64_t)seq * g.pieces + c);
                sums[c] = part;
                z += part;
            }
        }
        next = (double)a.next[seq];
        rows = load_rows<kType>(g, q, 0);
        if (g.ways) {
            w.z = wave_sum(z);
            w.known = 1;
        }
        if (lane == 0) path[0] = 0;
        go_on<kType>(g, q, w, rows, path);
        if (lane == 0) way = w;
    } else {
        for (int32_t i = 1 + (int32_t)threadIdx.x - 64; i < q.rows; i += (int32_t)kThreads - 64)
            if ((uint32_t)a.tokens[q.row0 + i] >= a.vocab) kv_note(g.b.errors, TENT_KV_BAD_TOKEN);
    }
    __syncthreads();
    while (!way.ended) {                                                 // a sum, of pieces in turn
        const Way w = way;
        for (uint32_t c = wave; c < g.pieces; c += kWaves) {
            const double sum = sum_of_piece<kType>(g, q, w, c, gone[wave]);
            if (lane == 0) sums[c] = sum;
        }
        __syncthreads();
        if (wave == 0) {
            double z = 0.0;
            for (uint32_t c = lane; c < g.pieces; c += 64) z += sums[c];
            Way v = w;
            v.z = wave_sum(z);
            v.known = 1;
            go_on<kType>(g, q, v, rows, path);
            if (lane == 0) way = v;
        }
        __syncthreads();
    }
    const Way w = way;
    if (wave != 0) {
        for (int32_t i = w.stand + (int32_t)threadIdx.x - 64; i < (int32_t)g.b.max_rows; i += (int32_t)kThreads - 64) path[i] = -1;
        return;
    }
    // The first wave draws: the piece in which the sum passes the number, then the lane's vector, then the token.
    int32_t token = -1;
    if (w.z > 0.0) {
        const double wanted = next * w.z;
        double before = 0.0;
        uint32_t piece;
        {                                                                // a few pieces side by side a lane
            const uint32_t per = (g.pieces + 63) / 64, c0 = lane * per, c1 = c0 + per < g.pieces ? c0 + per : g.pieces;
            double mine = 0.0;
            for (uint32_t c = c0; c < c1; ++c) mine += sums[c];
            double up_to = mine;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const double up = __shfl_up(up_to, m, 64);
                up_to += lane >= (uint32_t)m ? up : 0.0;
            }
            // the first lane in which the sum passes; by the roundings of sums it may be none, then the last that has anything
            const uint64_t passes = __ballot(mine > 0.0 && up_to > wanted), some = __ballot(mine > 0.0);
            double so_far = up_to - mine;
            uint32_t found = c0;
            for (uint32_t c = c0; c < c1; ++c) {
                const double s = sums[c];
                if (s > 0.0) {
                    found = c;
                    before = so_far;
                    if (so_far + s > wanted) break;
                }
                so_far += s;
            }
            const int from = passes ? __builtin_ctzll(passes) : 63 - __builtin_clzll(some);
            piece = (uint32_t)__builtin_amdgcn_readlane((int)found, from);
            before = from_lane(before, from);
        }
        // tokens in their order, some side by side a lane: their sum, and then, with the sum up to them, the token
        Piece<kType, true> p;
        p.load(g, q, w, piece, gone[0]);
        double mine = 0.0;
#pragma unroll
        for (uint32_t j = 0; j < p.kVecs; ++j) p.each(j, [&](uint32_t, double r) { mine += r; });
        double up_to = mine;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const double up = __shfl_up(up_to, m, 64);
            up_to += lane >= (uint32_t)m ? up : 0.0;
        }
        const uint64_t some = __ballot(mine > 0.0), passes = __ballot(mine > 0.0 && before + up_to > wanted);
        double so_far = before + (up_to - mine);
        uint32_t at = 0;
        bool over = false;
#pragma unroll
        for (uint32_t j = 0; j < p.kVecs; ++j)
            p.each(j, [&](uint32_t i, double r) {
                so_far += r;
                if (r > 0.0 && !over) {
                    at = p.at(j) + i;
                    over = so_far > wanted;
                }
            });
        token = (int32_t)(piece * kPiece) + __builtin_amdgcn_readlane((int)at, passes ? __builtin_ctzll(passes) : 63 - __builtin_clzll(some));
    }
    if (lane == 0) {
        a.counts[seq] = w.stand;
        a.token[seq] = token;
    }
}

// Whether a launch makes the first sums ahead: where a sequence's workgroup would take longer than a launch does, and the sequences are
// not enough to fill the card by themselves.  Four drafted tokens each, fp32, by itself and with a launch ahead: 64,000 tokens, 1 and 64
// sequences 16 and 20 us, 18 and 21; 128,000, 8, 64 and 128 sequences 23 and 21, 26 and 23, 30 and 29; 256,000, 1 and 64 sequences 32
// and 21, 38 and 30.  In bfloat16, half the bytes, the same way: 64,000 tokens, 1 and 128 sequences 15 and 19, 18 and 20; 128,000, 1, 64 and
// 128 sequences 21 and 19, 24 and 21, 25 and 25; 256,000, 8 and 128 sequences 29 and 19, 36 and 33.  Two and three launches ahead gain no
// more for trees than they cost others.
struct VerifyShape { uint32_t pieces; bool ahead; uint64_t workspace; };
VerifyShape shape_of(const tent_kv_batch& b, const tent_kv_verify_args& a)
{
    VerifyShape s{};
    s.pieces = (a.vocab + kPiece - 1) / kPiece;
    s.ahead = s.pieces > 48 && b.n_seqs <= 128;
    s.workspace = s.ahead ? (uint64_t)b.n_seqs * (sizeof(Way) + (uint64_t)s.pieces * 8) : 0;
    return s;
}

int check(const tent_kv_batch* batch, const tent_kv_verify_args* args)
{
    const int rc = kv_check_sequences(batch);
    if (rc != TENT_OK) return rc;
    if (!args || args->reserved || args->type > TENT_FP32) return TENT_ERR_INVALID;
    return args->vocab < 1 || args->vocab > TENT_KV_MAX_VOCAB ? TENT_ERR_RANGE : TENT_OK;
}

template <uint32_t kType>
int launch(const VerifyShape& s, VerifyArgs g, hipStream_t stream)
{
    if (s.ahead) {
        const int rc = launch_blocks((uint64_t)g.b.n_seqs * ((s.pieces + kAheadWaves - 1) / kAheadWaves), [&](uint32_t first, uint32_t blocks) {
            g.first = first;
            hipLaunchKernelGGL((verify_ahead_kernel<kType>), dim3(blocks), dim3(64 * kAheadWaves), 0, stream, g);
        });
        if (rc != TENT_OK) return rc;
    }
    return launch_blocks(g.b.n_seqs, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((verify_kernel<kType>), dim3(blocks), dim3(kThreads), 0, stream, g);
    });
}

}  // namespace
}  // namespace tent

using namespace tent;

extern "C" int tent_kv_verify_workspace(const tent_kv_batch* batch, const tent_kv_verify_args* args, uint64_t* bytes)
{
    const int rc = check(batch, args);
    if (rc != TENT_OK) return rc;
    if (!bytes) return TENT_ERR_INVALID;
    *bytes = batch->n_seqs == 0 || batch->n_rows == 0 ? 0 : shape_of(*batch, *args).workspace;
    return TENT_OK;
}

extern "C" int tent_kv_verify(const tent_kv_batch* batch, const tent_kv_verify_args* args, void* stream)
{
    const int rc = check(batch, args);
    if (rc != TENT_OK) return rc;
    if (batch->n_seqs == 0) return TENT_OK;
    if ((!args->path && batch->max_rows) || !args->counts || !args->token || (((uintptr_t)args->path | (uintptr_t)args->counts | (uintptr_t)args->token) & 3u)) return TENT_ERR_INVALID;
    if (args->path_stride < batch->max_rows) return TENT_ERR_RANGE;
    VerifyShape s{1, false, 0};
    if (batch->n_rows) {
        const uintptr_t odd = args->type == TENT_FP32 ? 3u : 1u;
        if (!args->target || !args->tokens || !args->accept || !args->next) return TENT_ERR_INVALID;
        if ((((uintptr_t)args->target | (uintptr_t)args->draft) & odd) ||
            (((uintptr_t)args->tokens | (uintptr_t)args->parents | (uintptr_t)args->accept | (uintptr_t)args->next) & 3u)) return TENT_ERR_INVALID;
        const uint64_t most = ((uint64_t)1 << 60) / batch->n_rows;
        if (args->target_stride < args->vocab || args->target_stride > most) return TENT_ERR_RANGE;
        if (args->draft && (args->draft_stride < args->vocab || args->draft_stride > most)) return TENT_ERR_RANGE;
        s = shape_of(*batch, *args);
        if (s.workspace && (!args->workspace || !kv_aligned(args->workspace))) return TENT_ERR_INVALID;
        if (s.workspace > args->workspace_bytes) return TENT_ERR_RANGE;
    }
    Way* const ways = s.ahead ? static_cast<Way*>(args->workspace) : nullptr;
    const VerifyArgs g{*args, *batch, ways, s.ahead ? reinterpret_cast<double*>(ways + batch->n_seqs) : nullptr, s.pieces, 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return args->type == TENT_FP32 ? launch<TENT_FP32>(s, g, st) : args->type == TENT_BF16 ? launch<TENT_BF16>(s, g, st) : launch<TENT_FP16>(s, g, st);
}
