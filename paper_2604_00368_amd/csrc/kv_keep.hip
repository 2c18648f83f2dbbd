// What a sequence of a key/value cache keeps, and the move that makes it the sequence: tent_kv_choose and tent_kv_keep.
#include <type_traits>

#include "kv_elem.h"

namespace tent {
namespace {

// ---- choosing ------------------------------------------------------------------------------------
// A workgroup for each list.  The weight that the last chosen token has is found digit by digit: a histogram of the digits of those
// weights whose higher digits are the wanted ones, then the digit at which as many lie above as are wanted.  Where up to 128 weights have
// that digit they are put side by side and the one is found among them by its rank, most often after the second digit.  Up to 16,384 tokens
// are held in registers for all of it; more are read again for each digit, or, where lists are few, shared by several workgroups
// (choose_part_kernel).
//
// Barriers and latencies bound it.  Measured: one list of 6,000 tokens 12.6 us, 256 lists of 1,000 to 16,384 tokens, four fifths of whose
// weights are zero, 25.3 us (with four digits of 8 bits and no ranks 15.5 and 22.6: the digits are those of few lists, at a loss of an eighth
// for many); weights that differ in their last bits only, which take all three digits, 15.4 and, of 256 lists of 16,384, 26.3; one list of
// 131,072 tokens 43 us, by one workgroup 182.
struct ChooseArgs {
    tent_kv_choose_args a;
    tent_kv_batch b;
    uint32_t first;                    // of the launch's workgroups
};
struct ChoosePartArgs : ChooseArgs {
    uint32_t* counts;                  // [2][lists][parts][kDigits]: of the digits of two launches, in turn
    uint32_t* before;                  // [lists][parts]: weights above the digits found that lie in the parts before
    u32x2* found;                      // [2][lists]: the digits found, and how many weights are wanted of those that have them; in turn, too
    uint32_t parts, part_tokens;       // workgroups to a list, and their tokens: whole rounds of kChooseThreads, of kHeldTokens in lists that take several
};
constexpr uint32_t kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr uint32_t kHeld = 16, kHeldTokens = kHeld * kChooseThreads;     // tokens of a thread, and of the workgroup
// Weights are alike, often zero, and lanes side by side count the same digits: those that have the first lane's are counted at once, and four
// copies of the counters, in banks side by side, keep the others apart.
constexpr uint32_t kDigits = 2048, kCopies = 4;
constexpr uint32_t kRanked = 128;      // each is compared with each

// The digits of a key, from the highest one down: every bit is in one of them.
struct Digit {
    int shift, bits;
    __device__ __forceinline__ uint32_t of(uint32_t key) const { return key >> shift & ((1u << bits) - 1); }
};
constexpr int kDigitsOfKey = 3;
__host__ __device__ constexpr Digit digit_of_key(int i) { return i == 0 ? Digit{21, 11} : i == 1 ? Digit{10, 11} : Digit{0, 10}; }
constexpr bool digits_cover_keys(int i)
{
    return i == kDigitsOfKey ? digit_of_key(i - 1).shift == 0
                             : 1u << digit_of_key(i).bits <= kDigits && digit_of_key(i).shift + digit_of_key(i).bits == (i ? digit_of_key(i - 1).shift : 32) && digits_cover_keys(i + 1);
}
static_assert(digits_cover_keys(0), "a bit in two digits counts weights twice, one in none leaves them apart");

// Larger weights as larger whole numbers; zeros are alike, NaN is minus infinity.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t x = w != w ? 0xFF800000u : w == 0.f ? 0u : __float_as_uint(w);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// Calls f(i) for each of a thread's tokens, 1024 apart, where `n` are left.
template <class F>
__device__ __forceinline__ void each_held(uint32_t n, F f)
{
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i)
        if (i * kChooseThreads < n) f(i);                                // the whole workgroup
}

// The keys of kHeldTokens tokens from t0 on, of which `n` less t0 are there.
__device__ __forceinline__ void hold_keys(uint32_t (&key)[kHeld], const float* w, uint32_t t0, uint32_t n)
{
    float x[kHeld];
    each_held(n - t0, [&](uint32_t i) {
        const uint32_t t = t0 + i * kChooseThreads + threadIdx.x;
        x[i] = t < n ? dev_load<float>(w + t) : 0.f;
    });
    each_held(n - t0, [&](uint32_t i) { key[i] = weight_key(x[i]); });
}

__device__ __forceinline__ void clear_counts(uint32_t* count)
{
#pragma unroll
    for (uint32_t i = 0; i < kDigits * kCopies / 4 / kChooseThreads; ++i) *(u32x4*)&count[(i * kChooseThreads + threadIdx.x) * 4] = u32x4{0, 0, 0, 0};
}
// Counts a digit; lanes that do not count are not here.
__device__ __forceinline__ void count_digit(uint32_t* count, uint32_t digit, uint32_t lane, uint32_t wave)
{
    const uint32_t one = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
    const uint64_t alike = __ballot(digit == one);
    if (digit != one) atomicAdd(&count[digit * kCopies + (lane & (kCopies - 1))], 1u);
    else if (lane == (uint32_t)__builtin_ctzll(alike)) atomicAdd(&count[one * kCopies + (wave & (kCopies - 1))], (uint32_t)__popcll(alike));
}
__device__ __forceinline__ uint32_t counted(const uint32_t* count, uint32_t digit)
{
    const u32x4 c = *(const u32x4*)&count[digit * kCopies];
    return c[0] + c[1] + c[2] + c[3];
}
// Finds the digit that the weight has which is the wanted one from the largest on, of which there are mine[0] and mine[1] with the thread's two
// digits, the larger one first; says into digit_lds which, into wanted_lds the how manieth of them, and into all_lds how many there are.
__device__ __forceinline__ uint32_t first_digit() { return kDigits - 1 - 2 * threadIdx.x; }
__device__ __forceinline__ void find_digit(const uint32_t (&mine)[2], uint32_t wanted, uint32_t* before_lds, uint32_t& digit_lds, uint32_t& wanted_lds, uint32_t& all_lds)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, both = mine[0] + mine[1];
    uint32_t up_to = both;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t up = __shfl_up(up_to, m, 64);
        up_to += lane >= (uint32_t)m ? up : 0u;
    }
    if (lane == 63) before_lds[wave] = up_to;
    __syncthreads();
    uint32_t before = up_to - both;
    for (uint32_t i = 0; i < wave; ++i) before += before_lds[i];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        if (before < wanted && before + mine[i] >= wanted) {
            digit_lds = first_digit() - i;
            wanted_lds = wanted - before;
            all_lds = mine[i];
        }
        before += mine[i];
    }
    __syncthreads();
}
// Puts the tokens that are kept of kHeldTokens from t0 on into the list, in their order: how many there are before each, from counts of every
// wave's 64.  kind(i, more, same): whether the thread's token i is kept, or at the border, of which the first `equal` are.
// more_before and equal_before: of the list, in front of t0; then behind.
template <class Kind>
__device__ __forceinline__ void put_tokens(int32_t* to, uint32_t t0, uint32_t n, uint32_t equal, uint32_t& more_before, uint32_t& equal_before,
                                           uint32_t* before_lds, uint32_t& all_lds, Kind kind)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    each_held(n - t0, [&](uint32_t i) {
        bool more, same;
        kind(i, more, same);
        const uint32_t both = (uint32_t)__popcll(__ballot(more)) | (uint32_t)__popcll(__ballot(same)) << 16;    // at most 16,384 each
        if (lane == 0) before_lds[i * kChooseWaves + wave] = both;
    });
    __syncthreads();
    if (wave == 0) {
        uint32_t mine[4], sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t at = lane * 4 + i;
            sum += mine[i] = t0 + at / kChooseWaves * kChooseThreads < n ? before_lds[at] : 0u;
        }
        uint32_t up_to = sum;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t up = __shfl_up(up_to, m, 64);
            up_to += lane >= (uint32_t)m ? up : 0u;
        }
        if (lane == 63) all_lds = up_to;
        up_to -= sum;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            before_lds[lane * 4 + i] = up_to;
            up_to += mine[i];
        }
    }
    __syncthreads();
    each_held(n - t0, [&](uint32_t i) {
        bool more, same;
        kind(i, more, same);
        const uint64_t below = (1ull << lane) - 1, more_mask = __ballot(more), same_mask = __ballot(same);
        const uint32_t both = before_lds[i * kChooseWaves + wave];
        const uint32_t at = more_before + (both & 0xFFFFu) + (uint32_t)__popcll(more_mask & below);
        const uint32_t eq = equal_before + (both >> 16) + (uint32_t)__popcll(same_mask & below);
        if (more || (same && eq < equal)) to[at + (eq < equal ? eq : equal)] = (int32_t)(t0 + i * kChooseThreads + threadIdx.x);
    });
    more_before += all_lds & 0xFFFFu;
    equal_before += all_lds >> 16;
    __syncthreads();
}

__global__ void __launch_bounds__(kChooseThreads) choose_kernel(const ChooseArgs g)
{
    __shared__ __align__(16) uint32_t count[kDigits * kCopies];
    __shared__ uint32_t before_lds[kHeld * kChooseWaves], digit_lds, wanted_lds, there_lds, all_lds;
    const tent_kv_choose_args& a = g.a;
    const uint32_t block = g.first + blockIdx.x, seq = block / a.n_lists, list = block - seq * a.n_lists;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.bad && threadIdx.x == 0 && list == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    const uint32_t n = (uint32_t)q.len, kept = n < a.budget ? n : a.budget;      // 0 of a bad sequence
    int32_t* const to = a.lists + (uint64_t)block * a.list_stride;
    if (threadIdx.x == 0 && list == 0) a.counts[seq] = (int32_t)kept;
    for (uint32_t j = kept + threadIdx.x; j < a.budget; j += kChooseThreads) to[j] = -1;
    if (n <= a.budget) {
        for (uint32_t j = threadIdx.x; j < n; j += kChooseThreads) to[j] = (int32_t)j;
        return;
    }
    const float* const w = a.weights + (uint64_t)block * a.weights_stride;
    const uint32_t lo = a.first, hi = n - a.recent;                      // the tokens that weights decide on: more than are wanted of them
    const bool once = n <= kHeldTokens;
    uint32_t key[kHeld];
    auto hold = [&](uint32_t t0) { hold_keys(key, w, t0, n); };
    auto decided = [&](uint32_t t) -> bool { return t >= lo && t < hi; };
    if (once) hold(0);
    // Keys above `border` are kept, and the first `equal` of those at it; whatever is not decided on is.
    uint32_t wanted = a.budget - a.first - a.recent, border = 0xFFFFFFFFu, equal = 0;
    if (wanted) {
        uint32_t above = 0;                                              // the digits found, at their places
        for (int i_digit = 0; ; ++i_digit) {
            const Digit digit = digit_of_key(i_digit);
            const int found_shift = digit.shift + digit.bits;            // the bits from here on are found: 32 at first
            clear_counts(count);
            __syncthreads();
            for (uint32_t t0 = 0; t0 < n; t0 += kHeldTokens) {
                if (!once) hold(t0);
                each_held(n - t0, [&](uint32_t i) {
                    if (decided(t0 + i * kChooseThreads + threadIdx.x) && (i_digit == 0 || key[i] >> found_shift == above >> found_shift)) {
                        // as count_digit, but called it makes the kernel 3 % slower
                        const uint32_t mine = digit.of(key[i]), one = (uint32_t)__builtin_amdgcn_readfirstlane((int)mine);
                        const uint64_t alike = __ballot(mine == one);
                        if (mine != one) atomicAdd(&count[mine * kCopies + (lane & (kCopies - 1))], 1u);
                        else if (lane == (uint32_t)__builtin_ctzll(alike)) atomicAdd(&count[one * kCopies + (wave & (kCopies - 1))], (uint32_t)__popcll(alike));
                    }
                });
            }
            __syncthreads();
            if (threadIdx.x == 0) there_lds = 0;
            const uint32_t mine[2] = {counted(count, first_digit()), counted(count, first_digit() - 1)};
            find_digit(mine, wanted, before_lds, digit_lds, wanted_lds, all_lds);
            above |= digit_lds << digit.shift;
            wanted = wanted_lds;
            const uint32_t there = all_lds;
            if (i_digit == kDigitsOfKey - 1) break;
            if (there > kRanked) continue;
            // Those with the digit, in any order, and the rank of each: the greater ones and, of the same, the earlier ones come before it.
            for (uint32_t t0 = 0; t0 < n; t0 += kHeldTokens) {
                if (!once) hold(t0);
                each_held(n - t0, [&](uint32_t i) {
                    const uint32_t t = t0 + i * kChooseThreads + threadIdx.x;
                    if (decided(t) && key[i] >> digit.shift == above >> digit.shift) *(u32x2*)&count[2 * atomicAdd(&there_lds, 1u)] = u32x2{key[i], t};
                });
            }
            __syncthreads();
            if (threadIdx.x < there) {
                const u32x2 me = *(const u32x2*)&count[2 * threadIdx.x];
                uint32_t rank = 0, same = 0;
#pragma unroll 8
                for (uint32_t i = 0; i < there; ++i) {
                    const u32x2 other = *(const u32x2*)&count[2 * i];
                    const bool alike = other[0] == me[0] && other[1] < me[1];
                    rank += other[0] > me[0] || alike;
                    same += alike;
                }
                if (rank == wanted - 1) {
                    digit_lds = me[0];
                    wanted_lds = same + 1;
                }
            }
            __syncthreads();
            above = digit_lds;
            wanted = wanted_lds;
            break;
        }
        border = above;
        equal = wanted;                                                  // of those at the border the first so many
    }
    uint32_t more_before = 0, equal_before = 0;
    for (uint32_t t0 = 0; t0 < n; t0 += kHeldTokens) {
        if (!once) hold(t0);
        put_tokens(to, t0, n, equal, more_before, equal_before, before_lds, all_lds, [&](uint32_t i, bool& more, bool& same) {
            const uint32_t t = t0 + i * kChooseThreads + threadIdx.x;
            more = t < n && (!decided(t) || (equal && key[i] > border));
            same = t < n && decided(t) && equal && key[i] == border;
        });
    }
}

// Several workgroups to a list, each with tokens of its own, in four launches: kStage 0 to 2 count the digits of 11, 11 and 10 bits, each of
// the weights that have the digits found before, and 3 puts the tokens into the list.  Every workgroup finds the digit of the launch before
// it by itself, from all workgroups' counts of its list, and how many weights above it lie in front of its own tokens.
template <int kStage>
__global__ void __launch_bounds__(kChooseThreads) choose_part_kernel(const ChoosePartArgs g)
{
    __shared__ __align__(16) uint32_t count[kDigits * kCopies];
    __shared__ uint32_t before_lds[kHeld * kChooseWaves], digit_lds, wanted_lds, all_lds, above_lds[kChooseWaves], same_lds;
    constexpr Digit kDigit = digit_of_key(kStage);                       // this stage's (not of the last stage); how far down the one before it goes
    constexpr int kBefore = kStage == 0 ? 0 : digit_of_key(kStage - 1).shift;
    const tent_kv_choose_args& a = g.a;
    const uint32_t block = g.first + blockIdx.x, at = block / g.parts, part = block - at * g.parts, seq = at / a.n_lists, list = at - seq * a.n_lists;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const KvSeq q = kv_sequence(g.b, seq);
    const uint32_t n = (uint32_t)q.len, kept = n < a.budget ? n : a.budget;      // 0 of a bad sequence
    const uint32_t t_first = part * g.part_tokens, t_end = n - t_first < g.part_tokens ? n : t_first + g.part_tokens;     // where t_first < n
    int32_t* const to = a.lists + (uint64_t)at * a.list_stride;
    if constexpr (kStage == 3) {
        if (q.bad && threadIdx.x == 0 && list == 0 && part == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
        if (threadIdx.x == 0 && list == 0 && part == 0) a.counts[seq] = (int32_t)kept;
        for (uint64_t j = kept + part * kChooseThreads + threadIdx.x; j < a.budget; j += (uint64_t)g.parts * kChooseThreads) to[j] = -1;
        if (n <= a.budget) {
            for (uint64_t j = part * kChooseThreads + threadIdx.x; j < n; j += (uint64_t)g.parts * kChooseThreads) to[j] = (int32_t)j;
            return;
        }
    }
    uint32_t wanted = a.budget - a.first - a.recent;
    if (t_first >= n || n <= a.budget || (kStage < 3 && !wanted)) return;
    const float* const w = a.weights + (uint64_t)at * a.weights_stride;
    const uint32_t lo = a.first, hi = n - a.recent;
    auto decided = [&](uint32_t t) -> bool { return t >= lo && t < hi; };
    uint32_t key[kHeld];
    hold_keys(key, w, t_first, t_end);                                   // beside the counts
    const uint64_t lists = (uint64_t)g.b.n_seqs * a.n_lists, half = lists * g.parts * kDigits;
    uint32_t above = 0, more_before = 0, equal_before = 0;
    if (kStage > 0 && wanted) {
        const uint32_t* const counts = g.counts + (kStage & 1 ? 0 : half) + (uint64_t)at * g.parts * kDigits;
        const uint32_t used = (n - 1) / g.part_tokens + 1;
        uint32_t mine[2] = {0, 0}, in_front[2] = {0, 0};                 // of the thread's two digits: all, and those of the parts before
        for (uint32_t p = 0; p < used; ++p) {
            const u32x2 c = *(const u32x2*)(counts + (uint64_t)p * kDigits + first_digit() - 1);
            mine[0] += c[1];
            mine[1] += c[0];
            in_front[0] += p < part ? c[1] : 0u;
            in_front[1] += p < part ? c[0] : 0u;
        }
        if (kStage > 1) {
            const u32x2 found = g.found[(kStage & 1 ? 0 : lists) + at];
            above = found[0];
            wanted = found[1];
            more_before = g.before[(uint64_t)at * g.parts + part];
        }
        find_digit(mine, wanted, before_lds, digit_lds, wanted_lds, all_lds);
        const uint32_t digit = digit_lds;
        uint32_t sum = (first_digit() > digit ? in_front[0] : 0u) + (first_digit() - 1 > digit ? in_front[1] : 0u);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m, 64);
        if (lane == 0) above_lds[wave] = sum;
        if (first_digit() == digit) same_lds = in_front[0];
        if (first_digit() - 1 == digit) same_lds = in_front[1];
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kChooseWaves; ++i) more_before += above_lds[i];
        equal_before = same_lds;                                         // at the border itself after the last digit
        above |= digit << kBefore;
        wanted = wanted_lds;
    }
    if constexpr (kStage < 3) {
        if (kStage > 0 && threadIdx.x == 0) {
            g.before[(uint64_t)at * g.parts + part] = more_before;
            if (part == 0) g.found[(kStage & 1 ? lists : 0) + at] = u32x2{above, wanted};
        }
        clear_counts(count);
        __syncthreads();
        for (uint32_t t0 = t_first; t0 < t_end; t0 += kHeldTokens) {
            if (t0 != t_first) hold_keys(key, w, t0, t_end);
            each_held(t_end - t0, [&](uint32_t i) {
                const uint32_t t = t0 + i * kChooseThreads + threadIdx.x;
                if (t < t_end && decided(t) && (kStage == 0 || key[i] >> kBefore == above >> kBefore))
                    count_digit(count, kDigit.of(key[i]), lane, wave);
            });
        }
        __syncthreads();
        uint32_t* const counts = g.counts + (kStage & 1 ? half : 0) + ((uint64_t)at * g.parts + part) * kDigits;
        *(u32x2*)(counts + first_digit() - 1) = u32x2{counted(count, first_digit() - 1), counted(count, first_digit())};
    } else {
        const uint32_t border = wanted ? above : 0xFFFFFFFFu, equal = wanted;
        more_before += (t_first < lo ? t_first : lo) + (t_first > hi ? t_first - hi : 0u);      // tokens in front that are not decided on
        for (uint32_t t0 = t_first; t0 < t_end; t0 += kHeldTokens) {
            if (t0 != t_first) hold_keys(key, w, t0, t_end);
            put_tokens(to, t0, t_end, equal, more_before, equal_before, before_lds, all_lds, [&](uint32_t i, bool& more, bool& same) {
                const uint32_t t = t0 + i * kChooseThreads + threadIdx.x;
                more = t < t_end && (!decided(t) || (equal && key[i] > border));
                same = t < t_end && decided(t) && equal && key[i] == border;
            });
        }
    }
}

// ---- moving --------------------------------------------------------------------------------------
struct KeepArgs {
    KvCache c;
    tent_kv_batch b;
    tent_kv_keep_args a;
    uint32_t columns;                  // in place: workgroups that share a head's row
    uint32_t parts;                    // to other pages: workgroups that share a list
    uint32_t first;                    // of the launch's workgroups
};
constexpr uint64_t kNowhere = ~0ull;

__device__ __forceinline__ KvKept kept_of(const tent_kv_keep_args& a, const KvSeq& q, uint32_t seq)
{
    return kv_kept(q, a.flags & TENT_KV_KEEP_ROWS, a.to_table != nullptr, a.counts[seq], a.most);
}
// By one thread of the sequence's workgroups.
__device__ __forceinline__ void tell_length(const KeepArgs& g, const KvKept& k, uint32_t seq)
{
    if (k.bad) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    if (g.a.kv_len_out) g.a.kv_len_out[seq] = k.bad ? g.b.kv_len[seq] : k.length();
}
__device__ __forceinline__ bool entry_ok(const tent_kv_keep_args& a, const KvKept& k, int32_t entry, int32_t j)
{
    return entry < k.have && entry >= (a.to_table ? 0 : j);
}

// Where a token is: its page, and the number in it of its row of a head.  The page is kNowhere where the table names none.
struct Place { uint64_t page; uint32_t row; };
__device__ __forceinline__ Place place_of(const KvCache& c, const int32_t* table, uint32_t entries, uint32_t token, uint32_t head)
{
    const uint32_t at = token >> c.page_shift, page = at < entries ? (uint32_t)table[at] : ~0u;
    return Place{page < c.n_pages ? page * c.page_stride : kNowhere, (token & ((1u << c.page_shift) - 1u)) * c.heads + head};
}
template <int D>
__device__ __forceinline__ uint64_t scales_at(const KvCache& c, const Place& p)
{
    return p.page + ((uint64_t)(c.heads * (D / 2)) << c.page_shift) + (uint64_t)p.row * (D / 32);
}
template <int D>
using Scales = std::conditional_t<D == 64, uint16_t, std::conditional_t<D == 128, uint32_t, u32x2>>;     // of a row

// In place.  A workgroup has a column of a head's rows of K and V, and takes the list's entries in turn.  Every entry is at or behind its own
// place, so what a batch of entries writes no later one reads; within a batch all is read before anything is written.  Columns have
// nothing to do with each other.  The next batch's places are looked up while a batch's rows are on their way.
// Bound by latency: lengths, entries, pages, rows, one after the other.  Paths of 64 sequences of 9 to 16 rows, 8 heads of 128 dimensions, 16 bits:
// 4.4 us (11 with K and V one after the other and no places looked up ahead).
constexpr uint32_t kEntries = 64;      // of a batch
template <int D, int kBits>
__global__ void __launch_bounds__(256) keep_kernel(const KeepArgs g)
{
    constexpr uint32_t kChunks = kBits == 16 ? D / 8 : D / 32;           // vectors of a head's row, without the scales
    constexpr uint32_t kItems = (2 * kEntries * kChunks + 255) / 256;    // of a thread, of a whole row of K and V
    __shared__ Place from[3][kEntries], to[3][kEntries];                 // of this batch, of the next, and of the one that others may still be storing
    const tent_kv_keep_args& a = g.a;
    uint32_t x = g.first + blockIdx.x;
    const uint32_t column = x % g.columns; x /= g.columns;
    const uint32_t head = x % g.c.heads, seq = x / g.c.heads;
    const int32_t* const list = a.lists + ((uint64_t)seq * a.n_lists + (a.n_lists == 1 ? 0u : head)) * a.list_stride;
    int32_t entry_ahead = threadIdx.x < kEntries && threadIdx.x < a.most ? list[threadIdx.x] : -1;       // on its way beside the lengths
    const KvSeq q = kv_sequence(g.b, seq);
    const KvKept k = kept_of(a, q, seq);
    if (column == 0 && head == 0 && threadIdx.x == 0) tell_length(g, k, seq);
    if (k.bad) return;
    const int32_t* const table = g.b.page_table + (uint64_t)seq * g.b.table_stride;
    const uint32_t count = (uint32_t)k.count;
    const uint32_t wide = kChunks / g.columns, chunk0 = column * wide, wide_log = 31 - __builtin_clz(wide);      // vectors of the column, a power of two
    auto find = [&](uint32_t j0, int32_t entry, uint32_t buffer) {
        const uint32_t j = j0 + threadIdx.x;
        if (threadIdx.x >= kEntries || j >= count) return;
        Place read{kNowhere, 0}, write{kNowhere, 0};
        int32_t wrong = 0;
        if (!entry_ok(a, k, entry, (int32_t)j)) wrong = TENT_KV_BAD_POSITION;
        else if (entry != (int32_t)j) {
            read = place_of(g.c, table, g.b.table_stride, (uint32_t)(k.base + entry), head);
            write = place_of(g.c, table, g.b.table_stride, (uint32_t)k.base + j, head);
            if (read.page == kNowhere || write.page == kNowhere) {
                wrong = TENT_KV_BAD_PAGE;
                read.page = kNowhere;
            }
        }
        if (wrong && column == 0) kv_note(g.b.errors, wrong);
        from[buffer][threadIdx.x] = read;
        to[buffer][threadIdx.x] = write;
    };
    if (count == 0) return;
    find(0, entry_ahead, 0);
    __syncthreads();
    uint32_t buffer = 0;
    for (uint32_t j0 = 0; j0 < count; j0 += kEntries) {
        const uint32_t n = count - j0 < kEntries ? count - j0 : kEntries, next = buffer == 2 ? 0u : buffer + 1;
        const uint32_t half = n << wide_log;                             // vectors of K, then as many of V
        u32x4 v[kItems] = {};
        Scales<D> s = {};
        auto vector = [&](const Place& p, uint32_t item) -> uint8_t* {
            return (item >= half ? g.c.v : g.c.k) + p.page + (uint64_t)p.row * (kChunks * 16) + (chunk0 + ((item >= half ? item - half : item) & (wide - 1))) * 16;
        };
        auto entry_of = [&](uint32_t item) -> uint32_t { return (item >= half ? item - half : item) >> wide_log; };
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t item = i * 256 + threadIdx.x;
            if (item < 2 * half && from[buffer][entry_of(item)].page != kNowhere) v[i] = dev_load<u32x4>(vector(from[buffer][entry_of(item)], item));
        }
        const uint32_t e = threadIdx.x % kEntries;                       // a thread for the scales of each entry of K, then of V
        uint8_t* const scale_pool = threadIdx.x < kEntries ? g.c.k : g.c.v;
        const bool scales = kBits == 4 && column == 0 && threadIdx.x < 2 * kEntries && e < n && from[buffer][e].page != kNowhere;
        if (scales) s = dev_load<Scales<D>>(scale_pool + scales_at<D>(g.c, from[buffer][e]));
        if (j0 + kEntries < count) {
            const uint32_t j = j0 + kEntries + threadIdx.x;
            find(j0 + kEntries, threadIdx.x < kEntries && j < count ? list[j] : -1, next);
        }
        // all of it is here before any of it is written
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) __asm__ volatile("" : "+v"(v[i]));
        __asm__ volatile("" : "+v"(s));
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t item = i * 256 + threadIdx.x;
            if (item < 2 * half && from[buffer][entry_of(item)].page != kNowhere) dev_store(vector(to[buffer][entry_of(item)], item), v[i]);
        }
        if (scales) dev_store(scale_pool + scales_at<D>(g.c, to[buffer][e]), s);
        buffer = next;
    }
}

// To other pages, so nothing that is written is read.  A workgroup has some entries of a list: the rows of K and V of its head or, where one
// list is for all heads, of all of them, which lie side by side.
// Bound by memory: 24 x 2,048 tokens out of 4k to 8k, a list for each of 8 heads of 128 dimensions, 16 bits, 404 MB read and written in 90 us,
// 4.5 TB/s, as fast as a large copy (by the kernel for moves in place, a workgroup to a list, 228).
constexpr uint32_t kCopyEntries = 32;
template <int D, int kBits>
__global__ void __launch_bounds__(256) keep_copy_kernel(const KeepArgs g)
{
    constexpr uint32_t kChunks = kBits == 16 ? D / 8 : D / 32;
    constexpr uint32_t kAhead = 4;                                       // vectors of a lane in flight
    __shared__ Place from[kCopyEntries], to[kCopyEntries];
    const tent_kv_keep_args& a = g.a;
    // All heads of some entries go to one XCD one after the other: heads of a token share lines of its page.
    const uint32_t block = g.first + blockIdx.x, eight = block / (8 * a.n_lists), in_eight = block - eight * 8 * a.n_lists;
    const uint32_t unit = eight * 8 + in_eight % 8, head = in_eight / 8;
    if (unit >= g.b.n_seqs * g.parts) return;
    const uint32_t seq = unit % g.b.n_seqs, j0 = unit / g.b.n_seqs * kCopyEntries;
    const KvSeq q = kv_sequence(g.b, seq);
    const KvKept k = kept_of(a, q, seq);
    if (head == 0 && j0 == 0 && threadIdx.x == 0) tell_length(g, k, seq);
    if (k.bad || j0 >= (uint32_t)k.count) return;
    const uint32_t n = (uint32_t)k.count - j0 < kCopyEntries ? (uint32_t)k.count - j0 : kCopyEntries;
    if (threadIdx.x < n) {
        const int32_t j = (int32_t)(j0 + threadIdx.x), entry = a.lists[((uint64_t)seq * a.n_lists + head) * a.list_stride + j];
        Place read{kNowhere, 0}, write{kNowhere, 0};
        if (!entry_ok(a, k, entry, j)) {
            kv_note(g.b.errors, TENT_KV_BAD_POSITION);
        } else {
            read = place_of(g.c, g.b.page_table + (uint64_t)seq * g.b.table_stride, g.b.table_stride, (uint32_t)(k.base + entry), head);
            write = place_of(g.c, a.to_table + (uint64_t)seq * a.to_stride, a.to_entries, (uint32_t)(k.base + j), head);
            if (read.page == kNowhere || write.page == kNowhere) {
                kv_note(g.b.errors, TENT_KV_BAD_PAGE);
                read.page = kNowhere;
            }
        }
        from[threadIdx.x] = read;
        to[threadIdx.x] = write;
    }
    __syncthreads();
    const uint32_t heads = a.n_lists == 1 ? g.c.heads : 1u, wide = heads * kChunks, half = n * wide, items = 2 * half;      // vectors of K, and of both
    for (uint32_t first = threadIdx.x; first < items; first += kAhead * 256) {
        u32x4 v[kAhead];
        uint8_t* where[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
            const uint32_t item = first + i * 256 < items ? first + i * 256 : first;
            const bool is_v = item >= half;
            const uint32_t y = is_v ? item - half : item, e = y / wide, chunk = y - e * wide;
            const Place p = from[e], t = to[e];
            uint8_t* const pool = is_v ? g.c.v : g.c.k;
            where[i] = p.page == kNowhere ? nullptr : pool + t.page + (uint64_t)t.row * (kChunks * 16) + chunk * 16;
            v[i] = dev_load<u32x4>(p.page == kNowhere ? pool : pool + p.page + (uint64_t)p.row * (kChunks * 16) + chunk * 16);
        }
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i)
            if (first + i * 256 < items && where[i]) dev_store(where[i], v[i]);
    }
    if constexpr (kBits == 4) {
        for (uint32_t item = threadIdx.x; item < 2 * n * heads; item += 256) {
            const bool is_v = item >= n * heads;
            const uint32_t y = is_v ? item - n * heads : item, e = y / heads, h = y - e * heads;
            Place p = from[e], t = to[e];
            if (p.page == kNowhere) continue;
            p.row += h;
            t.row += h;
            uint8_t* const pool = is_v ? g.c.v : g.c.k;
            dev_store(pool + scales_at<D>(g.c, t), dev_load<Scales<D>>(pool + scales_at<D>(g.c, p)));
        }
    }
}

// The weights of kept tokens, a workgroup for each list of them: in their order, so that in place nothing is read that was written.
__global__ void __launch_bounds__(256) keep_weights_kernel(const KeepArgs g)
{
    const tent_kv_keep_args& a = g.a;
    const uint32_t block = g.first + blockIdx.x, seq = block / a.n_weights, l = block - seq * a.n_weights;
    const KvSeq q = kv_sequence(g.b, seq);
    const KvKept k = kept_of(a, q, seq);
    const int32_t* const list = a.lists + ((uint64_t)seq * a.n_lists + (a.n_lists == 1 ? 0u : l)) * a.list_stride;
    const float* const from = a.weights + (uint64_t)block * a.weights_stride;
    float* const to = a.weights_out + (uint64_t)block * a.weights_stride;
    const int32_t base = k.bad ? (int32_t)g.b.max_kv : k.base, count = k.bad ? 0 : k.count, most = (int32_t)g.b.max_kv;
    if (from != to)
        for (int32_t t = threadIdx.x; t < base; t += 256) to[t] = from[t];
    constexpr int32_t kAhead = 4;
    for (int32_t j0 = 0; j0 < count; j0 += 256 * kAhead) {
        float w[kAhead] = {};
#pragma unroll
        for (int32_t i = 0; i < kAhead; ++i) {
            const int32_t j = j0 + i * 256 + (int32_t)threadIdx.x;
            const int32_t entry = j < count ? list[j] : 0;
            if (j < count && base + j < most) w[i] = from[base + (entry_ok(a, k, entry, j) ? entry : j)];
        }
#pragma unroll
        for (int32_t i = 0; i < kAhead; ++i) __asm__ volatile("" : "+v"(w[i]));
        __syncthreads();
#pragma unroll
        for (int32_t i = 0; i < kAhead; ++i) {
            const int32_t j = j0 + i * 256 + (int32_t)threadIdx.x;
            if (j < count && base + j < most) to[base + j] = w[i];
        }
    }
    for (int32_t t = (k.bad ? most : k.length_up_to(most)) + (int32_t)threadIdx.x; t < most; t += 256) to[t] = 0.f;
}

// Whether several workgroups share a list, and how many: each finds the digits from the counts of all of them, so there are not many.
// Quarters of lists, with a workgroup to a list, to 16,384 and to 8,192 tokens: 1 list of 17,000 tokens 33, 31 and 29 us, 32,768 50, 39 and
// 32, 131,072 182, 45 and 43; 64 lists 34, 34 and 33, 51, 43 and 38, 185, 77 and 110; 128 lists 34, 36 and 46, 52, 46 and 49, 190, 140 and 204;
// 256 lists of 65,536 105, 129 and 188, as they fill the card by themselves.
struct ChooseShape { uint32_t parts, part_tokens; uint64_t workspace; };
constexpr uint32_t kMostParts = 64, kMostSplit = 128;
static_assert(kHeldTokens == TENT_KV_CHOOSE_WHOLE, "lists of up to that many tokens take no workspace");
ChooseShape choose_shape(const tent_kv_batch& b, const tent_kv_choose_args& a)
{
    ChooseShape s{1, kHeldTokens, 0};
    const uint64_t lists = (uint64_t)b.n_seqs * a.n_lists;
    if (b.max_kv <= kHeldTokens || lists > kMostSplit) return s;
    const uint32_t halves = (b.max_kv + kHeldTokens / 2 - 1) / (kHeldTokens / 2);
    uint32_t parts = lists * halves <= kMostSplit ? halves : (halves + 1) / 2;
    if (parts > kMostParts) parts = kMostParts;
    const uint32_t step = b.max_kv > kMostParts * kHeldTokens ? kHeldTokens : kChooseThreads;      // whole rounds of a workgroup
    s.part_tokens = ((b.max_kv + parts - 1) / parts + step - 1) / step * step;
    s.parts = (b.max_kv + s.part_tokens - 1) / s.part_tokens;
    s.workspace = lists * (s.parts * (2 * kDigits + 1) * 4ull + 2 * sizeof(u32x2));
    return s;
}
template <int kStage>
int launch_part(ChoosePartArgs g, hipStream_t stream)
{
    return launch_blocks((uint64_t)g.b.n_seqs * g.a.n_lists * g.parts, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((choose_part_kernel<kStage>), dim3(blocks), dim3(kChooseThreads), 0, stream, g);
    }, kMostBlocks / 4);
}

template <int D, int kBits>
int launch_keep(KeepArgs g, hipStream_t s)
{
    constexpr uint32_t kChunks = kBits == 16 ? D / 8 : D / 32;
    if (g.a.to_table) {
        g.parts = g.a.most ? (g.a.most + kCopyEntries - 1) / kCopyEntries : 1;
        return launch_blocks(((uint64_t)g.b.n_seqs * g.parts + 7) / 8 * 8 * g.a.n_lists, [&](uint32_t first, uint32_t blocks) {
            g.first = first;
            hipLaunchKernelGGL((keep_copy_kernel<D, kBits>), dim3(blocks), dim3(256), 0, s, g);
        });
    }
    const uint64_t lists = (uint64_t)g.b.n_seqs * g.c.heads;
    // Columns until the card is filled.  8 heads of 128 dimensions, 16 bits, 1,500 entries, 1 column, 2 and 4: 1 sequence 107, 72 and 57 us, 16 of them 142,
    // 97 and 71, 64 of them 254, 293 and 388; 16 entries take 8 to 9 whichever way.
    while (lists * g.columns < 512 && kChunks / g.columns > 4) g.columns *= 2;
    return launch_blocks(lists * g.columns, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((keep_kernel<D, kBits>), dim3(blocks), dim3(256), 0, s, g);
    });
}

}  // namespace
}  // namespace tent

using namespace tent;

extern "C" int tent_kv_choose_workspace(const tent_kv_batch* batch, const tent_kv_choose_args* args, uint64_t* bytes)
{
    const int rc = kv_check_sequences(batch);
    if (rc != TENT_OK) return rc;
    if (!args || !bytes) return TENT_ERR_INVALID;
    if (args->n_lists < 1 || args->n_lists > TENT_KV_MAX_HEADS) return TENT_ERR_RANGE;
    *bytes = batch->n_seqs == 0 ? 0 : choose_shape(*batch, *args).workspace;
    return TENT_OK;
}

extern "C" int tent_kv_choose(const tent_kv_batch* batch, const tent_kv_choose_args* args, void* stream)
{
    const int rc = kv_check_sequences(batch);
    if (rc != TENT_OK) return rc;
    if (!args) return TENT_ERR_INVALID;
    if (batch->n_seqs == 0) return TENT_OK;
    if ((!args->weights && batch->max_kv) || !args->lists || !args->counts) return TENT_ERR_INVALID;
    if (((uintptr_t)args->weights | (uintptr_t)args->lists | (uintptr_t)args->counts) & 3u) return TENT_ERR_INVALID;
    if (args->n_lists < 1 || args->n_lists > TENT_KV_MAX_HEADS || args->budget < 1 || args->budget > (1u << 30)) return TENT_ERR_RANGE;
    if ((uint64_t)args->first + args->recent > args->budget) return TENT_ERR_RANGE;
    if (kv_meet(args->counts, batch->n_seqs * 4ull, batch->kv_len, batch->n_seqs * 4ull)) return TENT_ERR_INVALID;     // read by workgroups of every list
    const uint64_t lists = (uint64_t)batch->n_seqs * args->n_lists, most = ((uint64_t)1 << 60) / lists;
    if (args->weights_stride < batch->max_kv || args->weights_stride > most || args->list_stride < args->budget || args->list_stride > most) return TENT_ERR_RANGE;
    const ChooseShape shape = choose_shape(*batch, *args);
    if (shape.workspace && (!args->workspace || !kv_aligned(args->workspace))) return TENT_ERR_INVALID;
    if (shape.workspace > args->workspace_bytes) return TENT_ERR_RANGE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (shape.parts > 1) {
        uint32_t* const counts = static_cast<uint32_t*>(args->workspace);
        u32x2* const found = reinterpret_cast<u32x2*>(counts + 2 * lists * shape.parts * kDigits);
        const ChoosePartArgs g{{*args, *batch, 0}, counts, reinterpret_cast<uint32_t*>(found + 2 * lists), found, shape.parts, shape.part_tokens};
        int status = launch_part<0>(g, s);
        if (status == TENT_OK) status = launch_part<1>(g, s);
        if (status == TENT_OK) status = launch_part<2>(g, s);
        return status == TENT_OK ? launch_part<3>(g, s) : status;
    }
    ChooseArgs g{*args, *batch, 0};
    return launch_blocks(lists, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL(choose_kernel, dim3(blocks), dim3(kChooseThreads), 0, s, g);
    }, kMostBlocks / 4);
}

extern "C" int tent_kv_keep(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_keep_args* args, void* stream)
{
    int rc = kv_check_cache(cache);
    if (rc == TENT_OK) rc = kv_check_sequences(batch);
    if (rc != TENT_OK) return rc;
    if (!args || args->reserved || (args->flags & ~(uint32_t)TENT_KV_KEEP_ROWS)) return TENT_ERR_INVALID;
    if (batch->n_seqs == 0) return TENT_OK;
    if ((rc = kv_check_table(cache, batch)) != TENT_OK) return rc;
    if ((!args->lists && args->most) || !args->counts) return TENT_ERR_INVALID;
    const uint64_t a_number_each = batch->n_seqs * 4ull;                 // other workgroups read lengths and counts
    if (kv_meet(args->kv_len_out, a_number_each, batch->kv_len, a_number_each) || kv_meet(args->kv_len_out, a_number_each, args->counts, a_number_each) ||
        kv_meet(args->kv_len_out, a_number_each, batch->row_start, a_number_each + 4)) return TENT_ERR_INVALID;
    if (((uintptr_t)args->lists | (uintptr_t)args->counts | (uintptr_t)args->to_table | (uintptr_t)args->kv_len_out | (uintptr_t)args->weights |
         (uintptr_t)args->weights_out) & 3u) return TENT_ERR_INVALID;
    if ((!args->weights) != (!args->weights_out) || (args->to_table && args->weights && args->weights == args->weights_out)) return TENT_ERR_INVALID;
    const uint64_t most = ((uint64_t)1 << 60) / ((uint64_t)batch->n_seqs * cache->kv_heads);
    if ((args->n_lists != 1 && args->n_lists != cache->kv_heads) || args->most > (1u << 30)) return TENT_ERR_RANGE;
    if (args->list_stride < args->most || args->list_stride > most || args->to_entries > args->to_stride) return TENT_ERR_RANGE;
    if (args->weights) {
        if ((args->n_weights != 1 && args->n_weights != cache->kv_heads) || args->n_weights < args->n_lists) return TENT_ERR_RANGE;
        if (args->weights_stride < batch->max_kv || args->weights_stride > most) return TENT_ERR_RANGE;
        if (kv_lists_meet(args->weights, args->weights_out, (uint64_t)batch->n_seqs * args->n_weights, batch->max_kv, args->weights_stride)) return TENT_ERR_INVALID;
    }
    KeepArgs g{kv_cache_dev(*cache), *batch, *args, 1, 1, 0};
    if (!g.a.to_entries) g.a.to_entries = g.a.to_stride;
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_KEEP(dim) (cache->bits == 16 ? launch_keep<dim, 16>(g, s) : launch_keep<dim, 4>(g, s))
    rc = cache->head_dim == 64 ? TENT_KEEP(64) : cache->head_dim == 128 ? TENT_KEEP(128) : TENT_KEEP(256);
    if (rc != TENT_OK || !args->weights) return rc;
    return launch_blocks((uint64_t)batch->n_seqs * args->n_weights, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL(keep_weights_kernel, dim3(blocks), dim3(256), 0, s, g);
    });
}
