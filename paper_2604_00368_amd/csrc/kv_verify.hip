// Verification of drafted tokens: tent_kv_verify.
//
// From the row c that stands last the rows behind it are tried.  After k rows were refused the residual is
//   r(t) = max(p(t) - b q(t), 0) / z,   z = sum_t max(p(t) - b q(t), 0),   p = target[c], q = draft[c]
// (by induction: max(max(p - b q, 0) / z - q, 0) = max(p - (b + z) q, 0) / z), with b = 0, z = 1 before the first, then b = 1, b + z, ..
// So the way is decided by single values, and by one sum over the vocabulary for each row that is refused: the last of these sums is
// what the next token is drawn from, too.  Without `draft` a refused token is taken out of p, and a sum is needed at the end only.
//
// A workgroup sums a piece of the vocabulary for its sequence, all pieces side by side, and every workgroup goes the way by itself
// as far as the sums known so far lead.  That makes a launch for each sum; as nobody knows how many there will be, some launches of
// pieces are followed by one in which a workgroup goes on alone and draws the token.
#include "kv_elem.h"

namespace tent {
namespace {

constexpr uint32_t kPiece = 8192;      // tokens of a piece
constexpr uint32_t kMostPieces = TENT_KV_MAX_VOCAB / kPiece;

struct VerifyArgs {
    tent_kv_verify_args a;
    tent_kv_batch b;
    double* sums;                      // [rounds][n_seqs][pieces]
    uint32_t pieces, rounds;           // launches of pieces ahead of the last
    uint32_t round;                    // this launch's
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
};
template <>
struct Prob<TENT_BF16> {
    using Raw = uint16_t;
    typedef uint16_t Vec __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr uint32_t kPer = 8;
    static __device__ __forceinline__ float value(uint16_t x) { return Bf16::to_float(x); }
};
template <>
struct Prob<TENT_FP16> {
    using Raw = uint16_t;
    typedef uint16_t Vec __attribute__((ext_vector_type(8), aligned(2)));
    static constexpr uint32_t kPer = 8;
    static __device__ __forceinline__ float value(uint16_t x) { return Fp16::to_float(x); }
};
// What is no probability counts as 0.
__device__ __forceinline__ double sound(float x) { return x > 0.f && x < INFINITY ? (double)x : 0.0; }

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m, 64);
    return x;
}
__device__ __forceinline__ double from_lane(double x, int lane)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return __longlong_as_double((long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)u, lane)));
}

// Where a sequence's way has got to.
struct Way {
    int32_t at;                        // the row that stands last
    int32_t next;                      // rows from here on are still to be tried
    int32_t stand;                     // rows that stand
    int32_t refused;                   // rows behind `at` that do not
    double b, z;                       // of the residual (with draft); z: of what is left (without)
    bool known;                        // z is the sum, not only what stands in its place before the first refusal
    bool whole;                        // nothing was left: the target's probabilities as they are
    bool ended;                        // no row is left to try, and z is known to be the sum
};

template <uint32_t kType>
__device__ __forceinline__ double value_at(const void* p, uint64_t row, uint64_t stride, uint32_t token, uint32_t vocab)
{
    using P = Prob<kType>;
    if (token >= vocab) return 0.0;
    return sound(P::value(dev_load<typename P::Raw>((const typename P::Raw*)p + row * stride + token)));
}

// One wave goes on until a sum is needed that is not known, or to the end.  `path`, if given, gets the rows that stand.
template <uint32_t kType>
__device__ void go_on(const VerifyArgs& g, const KvSeq& q, Way& w, int32_t* path)
{
    const tent_kv_verify_args& a = g.a;
    const int32_t lane = (int32_t)(threadIdx.x & 63u);
    while (w.next < q.rows) {
        const int32_t block = w.next & ~63, i = block + lane;
        const bool there = i < q.rows && i >= w.next;
        const uint64_t row = (uint64_t)(q.row0 + (i < q.rows ? i : 0));
        int32_t parent = i - 1;
        if (a.parents && there) parent = a.parents[row];
        const bool behind = there && parent >= 0 && parent < i;
        const uint32_t token = behind ? (uint32_t)a.tokens[row] : 0u;
        const double u = behind ? (double)a.accept[row] : 0.0;
        const double p = behind ? value_at<kType>(a.target, (uint64_t)(q.row0 + parent), a.target_stride, token, a.vocab) : 0.0;
        const double d = behind && a.draft ? value_at<kType>(a.draft, (uint64_t)(q.row0 + parent), a.draft_stride, token, a.vocab) : 0.0;
        uint64_t left = __ballot(behind && parent == w.at);
        while (left) {
            const int k = __builtin_ctzll(left);
            left &= left - 1;
            const double uk = from_lane(u, k), pk = from_lane(p, k), dk = from_lane(d, k);
            double r = a.draft ? pk - w.b * dk : pk;
            if (!(r > 0.0)) r = 0.0;
            if (!a.draft && w.refused) {                                 // a token that was taken out already
                const uint32_t x = (uint32_t)__builtin_amdgcn_readlane((int)token, k);
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
                w.known = false;
                left = __ballot(behind && parent == w.at);               // all of them are later ones
                continue;
            }
            ++w.refused;
            if (a.draft) {
                w.next = block + k + 1;
                w.b += w.refused > 1 ? w.z : 1.0;
                w.known = false;
                return;
            }
            w.z = w.z > r ? w.z - r : 0.0;
        }
        w.next = block + 64;
    }
    if (!w.known) return;
    if (w.z > 0.0 || w.whole) {
        w.ended = true;
    } else {                                                             // nothing is left: the target's own probabilities
        w.whole = true;
        w.known = false;
        w.b = 0.0;
    }
}

// The residual of one token, times z.
__device__ __forceinline__ double residual(double p, double q, double b)
{
    const double r = p - b * q;
    return r > 0.0 ? r : 0.0;
}

// Tokens that were taken out, of `n` from t0 on, as bits in LDS.  The whole workgroup comes here.
__device__ void mark_gone(const VerifyArgs& g, const KvSeq& q, const Way& w, uint32_t t0, uint32_t n, uint32_t* gone)
{
    for (uint32_t i = threadIdx.x; i < kPiece / 32; i += blockDim.x) gone[i] = 0;
    __syncthreads();
    if (!g.a.draft && w.refused && !w.whole)
        for (int32_t i = w.at + 1 + (int32_t)threadIdx.x; i < q.rows; i += (int32_t)blockDim.x) {
            const uint32_t x = (uint32_t)g.a.tokens[q.row0 + i] - t0;
            if ((g.a.parents ? g.a.parents[q.row0 + i] : i - 1) == w.at && x < n) atomicOr(&gone[x / 32], 1u << (x & 31u));
        }
    __syncthreads();
}

// Calls f(token in the piece, residual times z) for the tokens of a piece from t0 on that a lane of `lanes` has: whole vectors, one after the other.
template <uint32_t kType, bool kGone, class F>
__device__ __forceinline__ void over_piece(const VerifyArgs& g, const KvSeq& q, const Way& w, uint32_t t0, uint32_t n, uint32_t lane, uint32_t lanes, const uint32_t* gone, F f)
{
    using P = Prob<kType>;
    using Vec = typename P::Vec;
    const tent_kv_verify_args& a = g.a;
    const typename P::Raw* const p = (const typename P::Raw*)a.target + (uint64_t)(q.row0 + w.at) * a.target_stride + t0;
    const bool two = a.draft && w.b != 0.0;
    const typename P::Raw* const d = two ? (const typename P::Raw*)a.draft + (uint64_t)(q.row0 + w.at) * a.draft_stride + t0 : p;
    const double b = two ? w.b : 0.0;
    for (uint32_t v = lane; v * P::kPer < n; v += lanes) {
        const uint32_t t = v * P::kPer;
        if (t + P::kPer <= n) {
            const Vec x = dev_load<Vec>(p + t), y = two ? dev_load<Vec>(d + t) : x;
#pragma unroll
            for (uint32_t i = 0; i < P::kPer; ++i) {
                const double r = residual(sound(P::value(x[i])), sound(P::value(y[i])), b);
                f(t + i, kGone && gone[(t + i) / 32] >> ((t + i) & 31u) & 1u ? 0.0 : r);
            }
        } else {
            for (uint32_t i = t; i < n; ++i) {
                const double r = residual(sound(P::value(dev_load<typename P::Raw>(p + i))), sound(P::value(dev_load<typename P::Raw>(d + i))), b);
                f(i, kGone && gone[i / 32] >> (i & 31u) & 1u ? 0.0 : r);
            }
        }
    }
}

__device__ __forceinline__ Way start_of()
{
    return Way{0, 1, 1, 0, 0.0, 1.0, false, false, false};
}

// One wave goes the way as far as the sums of `rounds` launches lead; says the sums of how many it took.
template <uint32_t kType>
__device__ uint32_t replay(const VerifyArgs& g, const KvSeq& q, uint32_t seq, uint32_t rounds, Way& w, int32_t* path)
{
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t i = 0;; ++i) {
        go_on<kType>(g, q, w, path);
        if (w.ended || i == rounds) return i;
        const double* const s = g.sums + ((uint64_t)i * g.b.n_seqs + seq) * g.pieces;
        double z = 0.0;
        for (uint32_t c = lane; c < g.pieces; c += 64) z += dev_load<double>(s + c);
        w.z = wave_sum(z);
        w.known = true;
    }
}

template <uint32_t kType>
__global__ void __launch_bounds__(256) verify_pieces_kernel(const VerifyArgs g)
{
    __shared__ Way way;
    __shared__ uint32_t gone[kPiece / 32];
    __shared__ double part[4];
    const uint32_t block = g.first + blockIdx.x, seq = block / g.pieces, piece = block - seq * g.pieces;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.rows < 1) return;
    if (threadIdx.x < 64) {
        Way w = start_of();
        replay<kType>(g, q, seq, g.round, w, nullptr);
        if (threadIdx.x == 0) way = w;
    }
    __syncthreads();
    const Way w = way;
    if (w.ended) return;
    const uint32_t t0 = piece * kPiece, n = g.a.vocab - t0 < kPiece ? g.a.vocab - t0 : kPiece;
    double sum = 0.0;
    auto add = [&](uint32_t, double r) { sum += r; };
    if (!g.a.draft && w.refused && !w.whole) {
        mark_gone(g, q, w, t0, n, gone);
        over_piece<kType, true>(g, q, w, t0, n, threadIdx.x, 256, gone, add);
    } else {
        over_piece<kType, false>(g, q, w, t0, n, threadIdx.x, 256, gone, add);
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) dev_store(g.sums + ((uint64_t)g.round * g.b.n_seqs + seq) * g.pieces + piece, part[0] + part[1] + part[2] + part[3]);
}

constexpr uint32_t kLastThreads = 1024, kLastWaves = kLastThreads / 64;

template <uint32_t kType>
__global__ void __launch_bounds__(kLastThreads) verify_last_kernel(const VerifyArgs g)
{
    __shared__ Way way;
    __shared__ uint32_t gone[kPiece / 32];
    __shared__ double sums[kMostPieces], wave_part[kLastWaves];
    __shared__ uint32_t piece_lds, found_lds, last_lds;
    __shared__ double before_lds;
    const tent_kv_verify_args& a = g.a;
    const uint32_t seq = g.first + blockIdx.x, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const KvSeq q = kv_sequence(g.b, seq);
    int32_t* const path = a.path + (uint64_t)seq * a.path_stride;
    if (q.bad && threadIdx.x == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    for (int32_t i = 1 + (int32_t)threadIdx.x; i < q.rows; i += kLastThreads)
        if ((uint32_t)a.tokens[q.row0 + i] >= a.vocab) kv_note(g.b.errors, TENT_KV_BAD_TOKEN);
    if (q.rows < 1) {
        for (uint32_t i = threadIdx.x; i < g.b.max_rows; i += kLastThreads) path[i] = -1;
        if (threadIdx.x == 0) {
            a.counts[seq] = 0;
            a.token[seq] = -1;
        }
        return;
    }
    if (wave == 0) {
        if (lane == 0) path[0] = 0;
        Way w = start_of();
        const uint32_t taken = replay<kType>(g, q, seq, g.rounds, w, path);
        if (w.ended)
            for (uint32_t c = lane; c < g.pieces; c += 64) sums[c] = dev_load<double>(g.sums + ((uint64_t)(taken - 1) * g.b.n_seqs + seq) * g.pieces + c);
        if (lane == 0) way = w;
    }
    __syncthreads();
    while (!way.ended) {                                                 // alone: a wave for each piece in turn, tokens taken out by all
        const Way w = way;
        const bool out = !a.draft && w.refused && !w.whole;
        for (uint32_t c0 = 0; c0 < g.pieces; c0 += out ? 1 : kLastWaves) {
            const uint32_t c = out ? c0 : c0 + wave;
            const uint32_t t0 = c * kPiece, n = c < g.pieces ? (a.vocab - t0 < kPiece ? a.vocab - t0 : kPiece) : 0u;
            double sum = 0.0;
            auto add = [&](uint32_t, double r) { sum += r; };
            if (out) {
                mark_gone(g, q, w, t0, n, gone);
                over_piece<kType, true>(g, q, w, t0, n, threadIdx.x, kLastThreads, gone, add);
                sum = wave_sum(sum);
                if (lane == 0) wave_part[wave] = sum;
                __syncthreads();
                if (threadIdx.x == 0) {
                    sum = 0.0;
                    for (uint32_t i = 0; i < kLastWaves; ++i) sum += wave_part[i];
                    sums[c] = sum;
                }
            } else if (c < g.pieces) {
                over_piece<kType, false>(g, q, w, t0, n, lane, 64, gone, add);
                sum = wave_sum(sum);
                if (lane == 0) sums[c] = sum;
            }
        }
        __syncthreads();
        if (wave == 0) {
            double z = 0.0;
            for (uint32_t c = lane; c < g.pieces; c += 64) z += sums[c];
            Way v = w;
            v.z = wave_sum(z);
            v.known = true;
            go_on<kType>(g, q, v, path);
            if (lane == 0) way = v;
        }
        __syncthreads();
    }
    const Way w = way;
    for (int32_t i = w.stand + (int32_t)threadIdx.x; i < (int32_t)g.b.max_rows; i += kLastThreads) path[i] = -1;
    if (threadIdx.x == 0) a.counts[seq] = w.stand;
    if (!(w.z > 0.0)) {
        if (threadIdx.x == 0) a.token[seq] = -1;
        return;
    }
    // the piece in which the sum passes the number, then the vector, then the token
    const double wanted = (double)a.next[seq] * w.z;
    if (threadIdx.x == 0) {
        double before = 0.0;
        uint32_t c = 0, last = 0;
        double last_before = 0.0;
        for (;; ++c) {
            if (c == g.pieces) {                                         // by the roundings of sums only
                c = last;
                before = last_before;
                break;
            }
            if (sums[c] > 0.0) { last = c; last_before = before; }
            if (before + sums[c] > wanted) break;
            before += sums[c];
        }
        piece_lds = c;
        before_lds = before;
        found_lds = ~0u;
        last_lds = 0;
    }
    __syncthreads();
    const uint32_t t0 = piece_lds * kPiece, n = a.vocab - t0 < kPiece ? a.vocab - t0 : kPiece;
    mark_gone(g, q, w, t0, n, gone);
    constexpr uint32_t kMine = kPiece / kLastThreads;
    double r[kMine], sum = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) r[i] = 0.0;
    const uint32_t mine = threadIdx.x * kMine;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        const uint32_t t = mine + i;
        if (t < n) {
            const uint32_t token = t0 + t;
            const double p = value_at<kType>(a.target, (uint64_t)(q.row0 + w.at), a.target_stride, token, a.vocab);
            const double d = a.draft && w.b != 0.0 ? value_at<kType>(a.draft, (uint64_t)(q.row0 + w.at), a.draft_stride, token, a.vocab) : 0.0;
            r[i] = gone[t / 32] >> (t & 31u) & 1u ? 0.0 : residual(p, d, w.b);
        }
        sum += r[i];
    }
    double up_to = sum;                                                  // of this lane and those before it in its wave
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const double up = __shfl_up(up_to, m, 64);
        up_to += lane >= (uint32_t)m ? up : 0.0;
    }
    if (lane == 63) wave_part[wave] = up_to;
    __syncthreads();
    double before = before_lds;
    for (uint32_t i = 0; i < wave; ++i) before += wave_part[i];
    before += up_to - sum;
    uint32_t here = ~0u, last = 0;
    double so_far = before;
#pragma unroll
    for (uint32_t i = 0; i < kMine; ++i) {
        so_far += r[i];
        if (r[i] > 0.0) {
            last = mine + i + 1;
            if (so_far > wanted && here == ~0u) here = mine + i;
        }
    }
    if (here != ~0u) atomicMin(&found_lds, here);
    if (last) atomicMax(&last_lds, last);
    __syncthreads();
    if (threadIdx.x == 0) a.token[seq] = (int32_t)(t0 + (found_lds != ~0u ? found_lds : last_lds - 1));
}

// Launches of pieces: one where a sequence needs one sum at most, the end's, as rows one after the other and chosen ones do; trees of
// drawn tokens need one for each row that is refused.  None where the vocabulary is a single piece.
struct VerifyShape { uint32_t pieces, rounds; uint64_t workspace; };
VerifyShape shape_of(const tent_kv_batch& b, const tent_kv_verify_args& a)
{
    VerifyShape s{};
    s.pieces = (a.vocab + kPiece - 1) / kPiece;
    s.rounds = s.pieces == 1 ? 0 : a.draft && a.parents && b.max_rows > 2 ? 4 : 1;
    s.workspace = (uint64_t)s.rounds * b.n_seqs * s.pieces * 8;
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
    for (g.round = 0; g.round < s.rounds; ++g.round) {
        const int rc = launch_blocks((uint64_t)g.b.n_seqs * s.pieces, [&](uint32_t first, uint32_t blocks) {
            g.first = first;
            hipLaunchKernelGGL((verify_pieces_kernel<kType>), dim3(blocks), dim3(256), 0, stream, g);
        });
        if (rc != TENT_OK) return rc;
    }
    return launch_blocks(g.b.n_seqs, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((verify_last_kernel<kType>), dim3(blocks), dim3(kLastThreads), 0, stream, g);
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
    VerifyShape s{1, 0, 0};
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
    const VerifyArgs g{*args, *batch, static_cast<double*>(args->workspace), s.pieces, s.rounds, 0, 0};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return args->type == TENT_FP32 ? launch<TENT_FP32>(s, g, st) : args->type == TENT_BF16 ? launch<TENT_BF16>(s, g, st) : launch<TENT_FP16>(s, g, st);
}
