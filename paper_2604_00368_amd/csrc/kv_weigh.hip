// Attention weights onto the tokens of a cache: tent_kv_weigh.
//
//   w_t += sum over the lines l (rows and query heads of a cache head) that see token t of exp(scale q_l . k_t - lse_l)
//
// Both kernels compute S = Q K^T, 32 lines by 32 tokens: a lane then has scores of one token, and adds its weights up in a register.
// (S^T, with a line to a lane, takes 31 exchanges between lanes for each tile of tokens: 82 us instead of 27 for 32 rows over 5,120 tokens
// each in 4 bits, 8 heads of 128 dimensions.)  Each weight is written by one workgroup, in an order that does not change.
//
//   few_kernel   up to 32 lines: the queries stay in registers, the keys stream through; bound by its loads: 32 rows over 2k to 8k tokens, 8 heads
//                of 128 dimensions, 16 bits, 85 us for 360 MB, 4.2 TB/s
//   many_kernel  more lines: the keys stay, the queries go through LDS for the four waves that share them; bound by the exponentials beside
//                the products: two prompts of 4k tokens, 32 heads on 8 of 128 dimensions, 154 us, 771 TFLOP/s
#include "kv_elem.h"

namespace tent {
namespace {

struct WeighArgs {
    KvCache c;
    tent_kv_batch b;
    const uint8_t* q;
    const float *lse, *weights;
    float* out;
    float* by_head;                    // [n_seqs][heads][max_kv]: what weigh_join_kernel adds up, where one list is for many lines
    uint64_t q_stride, weights_stride; // bytes; values
    uint32_t q_heads, group, n_lists, window, all;
    float to_log2;                     // scale * log2(e)
    uint32_t tiles;                    // workgroups over the tokens of a sequence
    uint32_t run;                      // tiles of a wave, one after the other
    uint32_t first;                    // of the launch's workgroups
};
constexpr float kLog2e = 1.4426950408889634f;

// A lane has the scores of one token; its 16 are of lines 8 (i / 4) + 4 upper + i % 4 of 32.  What sees the token are some rows one after
// the other, so some lines: from lo to hi - 1.
struct Lines { int32_t lo, hi; };
__device__ __forceinline__ Lines lines_of(const WeighArgs& g, const KvSeq& q, int32_t t)
{
    if (g.all) return t >= q.len - (g.window ? (int64_t)g.window : (int64_t)q.len) ? Lines{0, q.rows * (int32_t)g.group} : Lines{0, 0};
    const int32_t before = q.len - q.rows, first = t - before > 0 ? t - before : 0;      // the row of token t
    int64_t last = q.rows;
    if (g.window && (int64_t)t - before + g.window < last) last = (int64_t)t - before + g.window;
    return last > first ? Lines{first * (int32_t)g.group, (int32_t)last * (int32_t)g.group} : Lines{0, 0};
}
// Those of 32 lines from l0 on, as bits.
__device__ __forceinline__ uint32_t line_bits(const Lines& see, int32_t l0)
{
    const int32_t lo = see.lo - l0, hi = see.hi - l0;
    const uint32_t below = hi >= 32 ? ~0u : hi > 0 ? ~(~0u << hi) : 0u;
    return lo <= 0 ? below : lo < 32 ? below & ~0u << lo : 0u;
}
// Adds exp2(s to_log2 + against) of the lines whose bits are set.
__device__ __forceinline__ void add_weights(float (&sum)[2], const f32x16& s, float to_log2, const f32x4 (&against)[4], uint32_t seen, uint32_t upper)
{
    seen >>= 4 * upper;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[i], to_log2, against[i >> 2][i & 3]));
        sum[i & 1] += seen & (1u << (8 * (i >> 2) + (i & 3))) ? w : 0.f;
    }
}
// What is added to a line's scores, in powers of two; infinite where the line has no sum and adds nothing.
__device__ __forceinline__ float against_of(float lse) { return fabsf(lse) < INFINITY ? -lse * kLog2e : INFINITY; }

// The rows that see any of `n` tokens from t0 on: from first to last - 1.
struct Rows { int32_t first, last; };
__device__ __forceinline__ Rows rows_of(const WeighArgs& g, const KvSeq& q, int32_t t0, int32_t n)
{
    if (g.all) return Rows{0, q.rows};
    const int32_t before = q.len - q.rows;                               // tokens in front of the first row's
    int32_t first = t0 - before > 0 ? t0 - before : 0, last = q.rows;
    if (g.window) {
        const int64_t end = (int64_t)t0 + n - 1 + g.window - before;
        last = end < last ? (end > 0 ? (int32_t)end : 0) : last;
    }
    return Rows{first, last};
}

// A wave's LDS written by some of its lanes is read by others: its LDS operations keep their order, the compiler has to as well.
__device__ __forceinline__ void same_wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// ---- few lines -----------------------------------------------------------------------------------
// A wave goes through `run` tiles of 32 tokens of a head (or, with one list, of its heads' one tile: four waves share the heads, and their
// sums are joined over LDS).  Rows come as they lie, in lanes side by side, and by way of LDS into the operand's order; those of the next
// step are on their way while one is worked on.
template <class E, int D, int kBits, bool kOne>
__global__ void __launch_bounds__(256) few_kernel(const WeighArgs g)
{
    constexpr int kK = D / 16, kWaves = 4;
    constexpr int kRow = kBits == 16 ? D * 2 : D / 2, kPerRow = kRow / 16, kPasses = 32 * kPerRow / 64;
    constexpr int kWords = kBits == 4 && D == 256 ? 2 : 1;
    __shared__ __align__(16) uint8_t lds[kWaves][32 * kRow];
    __shared__ uint64_t rows_at[kWaves][32];
    __shared__ float joined[kOne ? kWaves : 1][32];
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t m = lane & 31u, upper = lane >> 5;
    // All heads of some tokens go to one XCD one after the other: heads of a token share lines of its page.
    const uint32_t block = g.first + blockIdx.x, eight = block / (8 * g.n_lists), in_eight = block - eight * 8 * g.n_lists;
    const uint32_t unit = eight * 8 + in_eight % 8, list = in_eight / 8;
    if (unit >= g.b.n_seqs * g.tiles) return;
    const uint32_t seq = unit % g.b.n_seqs, part = unit / g.b.n_seqs;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.bad && threadIdx.x == 0 && part == 0 && list == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    const int32_t most = (int32_t)g.b.max_kv;
    const uint64_t at = ((uint64_t)seq * g.n_lists + list) * g.weights_stride;
    // steps: a tile of one head each
    const int32_t tile0 = kOne ? (int32_t)part : (int32_t)((part * kWaves + wave) * g.run);
    const int32_t steps = kOne ? ((int32_t)g.c.heads - (int32_t)wave + kWaves - 1) / kWaves : (int32_t)g.run;
    auto head_of = [&](int32_t step) -> uint32_t { return kOne ? wave + (uint32_t)step * kWaves : list; };
    auto first_of = [&](int32_t step) -> int32_t { return (tile0 + (kOne ? 0 : step)) * 32; };
    const int32_t lines = q.rows * (int32_t)g.group;                     // at most 32, by the host's choice
    const int32_t line = (int32_t)m < lines ? (int32_t)m : 0, row = line / (int32_t)g.group, h = line - row * (int32_t)g.group;
    const uint64_t q_row = (uint64_t)(q.row0 + row);
    auto works = [&](int32_t step) -> bool { return step < steps && q.rows > 0 && first_of(step) < q.len; };

    u32x4 qf[kK], rows[kPasses];
    uint32_t scales[kWords] = {}, shift = 0;
    float lse = 0.f, before = 0.f;
    __shared__ __align__(16) float against_lds[kWaves][32];
    auto load_before = [&](int32_t step) {                               // the weight so far of this lane's token
        const int32_t t = first_of(step) + (int32_t)m;
        if (g.weights && t < most) before = dev_load<float>(g.weights + at + t);
    };
    auto load_queries = [&](int32_t step) {
        const uint32_t q_head = head_of(step) * g.group + (uint32_t)h;
        const uint8_t* const p = g.q + q_row * g.q_stride + ((uint64_t)q_head * D + upper * (kBits == 16 ? 8 : D / 2)) * 2;
#pragma unroll
        for (int k = 0; k < kK; ++k) qf[k] = dev_load<u32x4>(p + k * (kBits == 16 ? 32 : 16));
        lse = dev_load<float>(g.lse + q_row * g.q_heads + q_head);
    };
    auto load_page = [&](int32_t step) -> uint32_t {
        const int32_t t = min(first_of(step) + (int32_t)m, q.len - 1);
        return dev_load<uint32_t>(g.b.page_table + (uint64_t)seq * g.b.table_stride + ((uint32_t)t >> g.c.page_shift));
    };
    // Puts the places of a tile's rows into LDS, and says which of its tokens are there.
    auto place_rows = [&](int32_t step, uint32_t page) -> uint32_t {
        const int32_t t = first_of(step) + (int32_t)m;
        const bool inside = t < q.len, there = inside && page < g.c.n_pages;
        if (inside && !there && upper == 0) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
        const uint32_t r = ((uint32_t)t & ((1u << g.c.page_shift) - 1u)) * g.c.heads + head_of(step);
        if (upper == 0) rows_at[wave][m] = (there ? page * g.c.page_stride : 0) + (uint64_t)r * kRow;
        same_wave_order();
        return (uint32_t)__ballot(there);
    };
    auto load_rows = [&](int32_t step) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) rows[i] = dev_load<u32x4>(g.c.k + rows_at[wave][i * (64 / kPerRow) + lane / kPerRow] + lane % kPerRow * 16);
        if constexpr (kBits == 4) {                                      // the words that hold the scales of token m
            const uint32_t r = ((uint32_t)(first_of(step) + (int32_t)m) & ((1u << g.c.page_shift) - 1u)) * g.c.heads + head_of(step);
            const uintptr_t p = (uintptr_t)g.c.k + rows_at[wave][m] - (uint64_t)r * kRow + ((uint64_t)(g.c.heads * (D / 2)) << g.c.page_shift) + (uint64_t)r * (D / 32);
            if constexpr (kWords == 2) {
                const u32x2 w = dev_load<u32x2>((const void*)p);
                scales[0] = w[0];
                scales[1] = w[1];
            } else {
                scales[0] = dev_load<uint32_t>((const void*)(p & ~(uintptr_t)3));
                shift = (uint32_t)(p & 3u) * 8;
            }
        }
    };
    uint32_t there = 0, page = 0;
    if (works(0)) {
        page = load_page(0);
        load_queries(0);
        there = place_rows(0, page);
        if (!kOne) load_before(0);
        if (works(1)) page = load_page(1);
        load_rows(0);
    } else if (!kOne) {
        load_before(0);
    }
    float sum[2] = {0.f, 0.f};
    f32x4 against[4];
    uint32_t valid = 0;                                                  // lines that add anything
    auto spread_lse = [&](float x) {
        const float y = (int32_t)m < lines ? against_of(x) : INFINITY;
        valid = (uint32_t)__ballot(y < INFINITY);
        if (upper == 0) against_lds[wave][m] = y;
        same_wave_order();
#pragma unroll
        for (int i = 0; i < 4; ++i) against[i] = *(const f32x4*)&against_lds[wave][8 * i + 4 * upper];
    };
    for (int32_t step = 0; step < steps; ++step) {
        const int32_t t0 = first_of(step);
        float before_now = before;
        if (works(step)) {
            uint8_t* const mine = lds[wave];
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const uint32_t t = i * (64 / kPerRow) + lane / kPerRow, chunk = lane % kPerRow;
                *(u32x4*)(mine + t * kRow + ((kBits == 16 ? chunk ^ (t & 7u) : chunk) << 4)) = rows[i];
            }
            same_wave_order();
            // what comes next is on its way before this is worked on
            const uint32_t there_now = there;
            if (kOne || step == 0) spread_lse(lse);
            const uint32_t scales_now[2] = {scales[0] >> shift, scales[kWords - 1]};
            u32x4 now[kOne ? kK : 1];
            if constexpr (kOne)
#pragma unroll
                for (int k = 0; k < kK; ++k) now[k] = qf[k];
            if (works(step + 1)) {
                there = place_rows(step + 1, page);
                if (works(step + 2)) page = load_page(step + 2);
                if constexpr (kOne) load_queries(step + 1);
                else load_before(step + 1);
                load_rows(step + 1);
            } else if (!kOne && step + 1 < steps) {
                load_before(step + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
            u32x4 kf[kK];
            if constexpr (kBits == 16) {
#pragma unroll
                for (int k = 0; k < kK; ++k) kf[k] = *(const u32x4*)(mine + m * kRow + (((uint32_t)(2 * k) + upper) ^ (m & 7u)) * 16);
            } else {
#pragma unroll
                for (int b = 0; b < D / 64; ++b) {
                    const u32x4 codes = *(const u32x4*)(mine + m * kRow + (upper * (D / 64) + b) * 16);
                    const uint32_t at_byte = upper * (D / 64) + b;       // lane m and lane m + 32 both have token m's
                    const uint32_t w = kWords == 2 && at_byte >= 4 ? scales_now[1] : scales_now[0];
                    const float scale = scale_of(w >> (8 * (at_byte & 3u)) & 0xFFu);
#pragma unroll
                    for (int c = 0; c < 4; ++c) kf[4 * b + c] = decode8<E>(codes[c], scale);
                }
            }
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
            for (int k = 0; k < kK; ++k) s = E::mfma32(kOne ? now[kOne ? k : 0] : qf[k], kf[k], s);
            const uint32_t seen = there_now >> m & 1u ? line_bits(lines_of(g, q, t0 + (int32_t)m), 0) & valid : 0u;
            add_weights(sum, s, g.to_log2, against, seen, upper);
        } else if (!kOne && step + 1 < steps) {
            load_before(step + 1);
        }
        if constexpr (!kOne) {
            const float total = sum[0] + sum[1], both = total + __shfl_xor(total, 32, 64);
            const int32_t t = t0 + (int32_t)m;
            if (upper == 0 && t < most) dev_store(g.out + at + t, before_now + both);
            sum[0] = sum[1] = 0.f;
        }
    }
    if constexpr (kOne) {
        const float total = sum[0] + sum[1], both = total + __shfl_xor(total, 32, 64);
        if (upper == 0) joined[wave][m] = both;
        __syncthreads();
        const int32_t t = tile0 * 32 + (int32_t)threadIdx.x;
        if (threadIdx.x < 32 && t < most)
            g.out[at + t] = (g.weights ? g.weights[at + t] : 0.f) + ((joined[0][threadIdx.x] + joined[1][threadIdx.x]) + (joined[2][threadIdx.x] + joined[3][threadIdx.x]));
    }
}

// ---- many lines ----------------------------------------------------------------------------------
// Eight waves, two of a SIMD: 64 tokens for each four, which take 32 lines each of a step's 128 (256 dimensions: 32 tokens for each two, 64
// lines).  The lines' queries lie in LDS; those of the next step but one are on their way meanwhile, and a step's exponentials run beside
// the products of the next (154 us instead of 186; 12 waves, each by itself, 165; 32 tokens to a wave read LDS twice as often, 162; two
// prompts of 4k tokens, 4 bits).  A workgroup takes a tile of 128 tokens and then the one that is as far from the end: of a prompt
// the first tile is seen by all rows, the last by few.
constexpr int32_t kTileTokens = 128;
constexpr int kManyThreads = 512;
template <class E, int D, int kBits>
__global__ void __launch_bounds__(kManyThreads, 2) many_kernel(const WeighArgs g)
{
    constexpr int kBlocks = D == 256 ? 1 : 2, kSubs = 4 / kBlocks, kThreads = kManyThreads, kParts = kThreads / 64 / kSubs;  // blocks of 32 tokens of a wave; waves for the tokens; waves for the lines
    constexpr int32_t kStepLines = 32 * kParts;
    constexpr int kK = D / 16, kItems = (kStepLines * D / 8 + kThreads - 1) / kThreads;          // vectors of a step that a thread loads
    constexpr int kApart = kThreads * 8 / D;                             // lines between them, a multiple of 16
    static_assert(kApart % 16 == 0 && kStepLines % kApart == 0, "a thread has whole vectors of its own place in a line");
    // Lanes side by side read a vector of a line each: they are to read from all banks, which 16 vectors cover once.
    auto swap = [](uint32_t line) -> uint32_t { return D == 64 ? line >> 1 & 7u : line & 15u; };
    constexpr uint32_t kPlane = kStepLines * D * 2;
    __shared__ __align__(16) uint8_t q_even[kPlane], q_odd[kPlane];
    __shared__ __align__(16) float against_lds[4][kStepLines];           // of four steps
    __shared__ float joined[kParts - 1][kTileTokens];
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t m = lane & 31u, upper = lane >> 5, sub = wave % kSubs, part = wave / kSubs, my_line = part * 32 + m;
    uint32_t x = g.first + blockIdx.x;
    const uint32_t head = x % g.c.heads; x /= g.c.heads;
    const uint32_t seq = x % g.b.n_seqs, pair = x / g.b.n_seqs;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.bad && threadIdx.x == 0 && pair == 0 && head == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    const int32_t most = (int32_t)g.b.max_kv, tiles = q.rows > 0 ? (q.len + kTileTokens - 1) / kTileTokens : 0;
    const bool one = g.by_head != nullptr;
    float* const out = one ? g.by_head + ((uint64_t)seq * g.c.heads + head) * g.b.max_kv : g.out + ((uint64_t)seq * g.n_lists + head) * g.weights_stride;
    const float* const in = one || !g.weights ? nullptr : g.weights + ((uint64_t)seq * g.n_lists + head) * g.weights_stride;
    for (int32_t t = (tiles + (int32_t)pair) * kTileTokens + (int32_t)threadIdx.x; t < most; t += (int32_t)g.tiles * kTileTokens)
        if (threadIdx.x < kTileTokens) out[t] = in ? in[t] : 0.f;        // behind the last token
    const int32_t group = (int32_t)g.group, whole_rows = kStepLines / group, rest = kStepLines - whole_rows * group;
    const uint64_t further = (uint64_t)whole_rows * g.q_stride + (uint32_t)rest * (D * 2);
    for (int32_t turn = 0; turn < 2; ++turn) {
        const int32_t tile = turn ? tiles - 1 - (int32_t)pair : (int32_t)pair;
        if (turn ? tile <= (int32_t)pair : 2 * tile >= tiles) continue;
        const int32_t t0 = tile * kTileTokens + (int32_t)sub * (32 * kBlocks);
        u32x4 kf[kBlocks][kK];
        Lines see[kBlocks];                                              // of the tokens t0 + m, t0 + 32 + m
        int32_t any_lo = 0x7FFFFFFF, any_hi = 0, all_lo = 0, all_hi = 0x7FFFFFFF;      // lines that some and that all of them are seen by
#pragma unroll
        for (int a = 0; a < kBlocks; ++a) {
            const int32_t t = t0 + 32 * a + (int32_t)m;
            const int64_t page = t < q.len ? kv_page_of(g.c, g.b, seq, (uint32_t)t) : -1;
            if (page < 0 && t < q.len && upper == 0 && part == 0) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
            see[a] = page >= 0 ? lines_of(g, q, t) : Lines{0, 0};
            if (see[a].hi > see[a].lo) {
                any_lo = min(any_lo, see[a].lo);
                any_hi = max(any_hi, see[a].hi);
            }
            all_lo = max(all_lo, see[a].lo);
            all_hi = min(all_hi, see[a].hi);
            const uint64_t slot = (uint64_t)((uint32_t)t & ((1u << g.c.page_shift) - 1u)) * g.c.heads + head;
            if constexpr (kBits == 16) {
                const uint8_t* const p = g.c.k + (page >= 0 ? (uint64_t)page + slot * (D * 2) : 0) + upper * 16;
#pragma unroll
                for (int k = 0; k < kK; ++k) kf[a][k] = dev_load<u32x4>(p + k * 32);
            } else {                                                     // half a row of codes each, in the order of the row
                const uint8_t* const p = g.c.k + (page >= 0 ? (uint64_t)page + slot * (D / 2) : 0) + upper * (D / 4);
                const uint8_t* const scales = g.c.k + (page >= 0 ? (uint64_t)page + ((uint64_t)(g.c.heads * (D / 2)) << g.c.page_shift) + slot * (D / 32) : 0) + upper * (D / 64);
#pragma unroll
                for (int k = 0; k < kK; k += 4) {
                    const u32x4 codes = dev_load<u32x4>(p + k * 4);
                    const float scale = scale_of(dev_load<uint8_t>(scales + k / 4));
#pragma unroll
                    for (int i = 0; i < 4; ++i) kf[a][k + i] = decode8<E>(codes[i], scale);
                }
            }
        }
#pragma unroll
        for (int bit = 1; bit < 32; bit <<= 1) {
            any_lo = min(any_lo, __shfl_xor(any_lo, bit, 64));
            any_hi = max(any_hi, __shfl_xor(any_hi, bit, 64));
            all_lo = max(all_lo, __shfl_xor(all_lo, bit, 64));
            all_hi = min(all_hi, __shfl_xor(all_hi, bit, 64));
        }
        any_lo = __builtin_amdgcn_readfirstlane(any_lo), any_hi = __builtin_amdgcn_readfirstlane(any_hi);
        all_lo = __builtin_amdgcn_readfirstlane(all_lo), all_hi = __builtin_amdgcn_readfirstlane(all_hi);
        const Rows rows = rows_of(g, q, tile * kTileTokens, kTileTokens);
        const int32_t line0 = rows.first * group, lines = rows.last * group, steps = lines > line0 ? (lines - line0 + kStepLines - 1) / kStepLines : 0;
        // The last lines come first: workgroups of a head then read the same queries at about the same time, out of the cache.
        const int32_t last0 = line0 + (steps - 1) * kStepLines;          // first line of the last step
        // Places of the queries that this thread loads: they go a step's lines back each time.
        const uint8_t* from[kItems];
        int32_t from_h[kItems];
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int32_t line = last0 + (int32_t)(threadIdx.x / (D / 8)) + i * kApart, row = line / group;
            from_h[i] = line - row * group;
            const uint32_t place = threadIdx.x % (D / 8), chunk = place ^ swap(threadIdx.x / (D / 8));
            from[i] = g.q + (uint64_t)(q.row0 + row) * g.q_stride + ((uint64_t)(head * g.group + (uint32_t)from_h[i]) * D) * 2 + chunk * 16;
        }
        int32_t loaded = last0;                                          // first line of the next step to load
        auto load_step = [&](uint8_t* to) {
            const int32_t left = loaded >= line0 ? lines - loaded : 0;
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (left >= kStepLines || (int32_t)(threadIdx.x / (D / 8)) + i * kApart < left)
                    __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(uintptr_t)from[i],
                                                     (__attribute__((address_space(3))) void*)(to + i * kThreads * 16 + wave * 1024), 16, 0, 0);
                from[i] -= further;
                if (rest) {
                    from_h[i] -= rest;
                    if (from_h[i] < 0) {
                        from_h[i] += group;
                        from[i] -= g.q_stride - (uint64_t)g.group * (D * 2);
                    }
                }
            }
            loaded -= kStepLines;
        };
        // A thread for each line has its sum, a step ahead of the queries, and makes of it what is added to scores.
        const bool has_line = threadIdx.x < (uint32_t)kStepLines;        // whole waves
        int32_t line = last0 + (int32_t)(threadIdx.x % kStepLines), row = line / group, h = line - row * group;
        float lse = INFINITY;
        auto load_lse = [&]() {
            lse = line >= line0 && line < lines ? dev_load<float>(g.lse + (uint64_t)(q.row0 + row) * g.q_heads + head * g.group + (uint32_t)h) : INFINITY;
            line -= kStepLines;
            row -= whole_rows;
            h -= rest;
            if (h < 0) {
                h += group;
                --row;
            }
        };
        float sum[kBlocks][2] = {};
        // S of a step's 32 lines and the wave's tokens; operands are read two steps ahead, `beside` is done behind each product, and nothing is
        // moved from step to step.
        auto scores = [&](const uint8_t* from_lds, f32x16 (&s)[kBlocks], auto beside) {
            const uint8_t* const p = from_lds + my_line * (D * 2);
            u32x4 qf[kK];
            auto read = [&](int k) { qf[k] = *(const u32x4*)(p + (((kBits == 16 ? 2 * k + upper : upper * kK + k) ^ swap(m)) << 4)); };
#pragma unroll
            for (int j = 0; j < 16 * kBlocks; ++j) s[j >> 4][j & 15] = 0.f;
            read(0);
            read(1);
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                if (k + 2 < kK) read(k + 2);
#pragma unroll
                for (int a = 0; a < kBlocks; ++a) {
                    s[a] = E::mfma32(qf[k], kf[a][k], s[a]);
                    beside(kBlocks * k + a);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        auto first_line = [&](int32_t i) -> int32_t { return last0 - i * kStepLines + (int32_t)part * 32; };
        auto any_seen = [&](int32_t i) -> bool { return i < steps && first_line(i) < any_hi && first_line(i) + 32 > any_lo; };
        // Adds a step's weights, and beside them computes the next one's scores, whose queries are in `q_next`; to `q_load` go those behind.
        auto step = [&](int32_t i, f32x16 (&s)[kBlocks], f32x16 (&next)[kBlocks], const uint8_t* q_next, uint8_t* q_load) {
            load_step(q_load);
            if (has_line) {
                against_lds[(i + 2) & 3][threadIdx.x] = against_of(lse);
                load_lse();
            }
            const int32_t l0 = first_line(i);
            const float* const against = &against_lds[i & 3][part * 32];
            f32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *(const f32x4*)&against[8 * j + 4 * upper];
            const uint32_t valid = (uint32_t)__ballot(against[m] < INFINITY);        // lines that add anything
            const bool more = any_seen(i + 1);
            if (more && l0 >= all_lo && l0 + 32 <= all_hi && valid == ~0u) {
                __builtin_amdgcn_sched_barrier(0);
                scores(q_next, next, [&](int at) {                       // kBlocks kK times
                    constexpr int kPer = 16 / kK;
                    float w[kPer];
#pragma unroll
                    for (int j = 0; j < kPer; ++j) w[j] = fmaf(s[(kPer * at + j) % kBlocks][(kPer * at + j) / kBlocks], g.to_log2, x[(kPer * at + j) / kBlocks >> 2][(kPer * at + j) / kBlocks & 3]);
#pragma unroll
                    for (int j = 0; j < kPer; ++j) w[j] = __builtin_amdgcn_exp2f(w[j]);
#pragma unroll
                    for (int j = 0; j < kPer; ++j) sum[(kPer * at + j) % kBlocks][(kPer * at + j) / kBlocks & 1] += w[j];
                });
            } else {
                if (any_seen(i)) {
#pragma unroll
                    for (int a = 0; a < kBlocks; ++a) add_weights(sum[a], s[a], g.to_log2, x, line_bits(see[a], l0) & valid, upper);
                }
                if (more) scores(q_next, next, [](int) {});
            }
            __builtin_amdgcn_s_waitcnt(0x0F70);                          // vmcnt(0): the queries behind are in LDS
            __syncthreads();
        };
        if (steps > 0) {
            if (has_line) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    load_lse();
                    against_lds[i][threadIdx.x] = against_of(lse);
                }
                load_lse();
            }
            load_step(q_even);
            load_step(q_odd);
            __builtin_amdgcn_s_waitcnt(0x0F70);
            __syncthreads();
            f32x16 s0[kBlocks], s1[kBlocks];
            scores(q_even, s0, [](int) {});
            __syncthreads();
            for (int32_t i = 0; i < steps; i += 2) {
                step(i, s0, s1, q_odd, q_even);
                if (i + 1 < steps) step(i + 1, s1, s0, q_even, q_odd);
            }
        }
#pragma unroll
        for (int a = 0; a < kBlocks; ++a) {
            const float both = sum[a][0] + sum[a][1];
            sum[a][0] = both + __shfl_xor(both, 32, 64);
            if (part && upper == 0) joined[part - 1][sub * (32 * kBlocks) + 32 * a + m] = sum[a][0];
        }
        __syncthreads();
        if (part == 0 && (kBlocks == 2 || upper == 0)) {                 // with 64 tokens the upper lanes have the second 32
            const uint32_t t_in = sub * (32 * kBlocks) + (kBlocks == 2 ? lane : m);
            const int32_t t = tile * kTileTokens + (int32_t)t_in;
            float total = upper ? sum[kBlocks - 1][0] : sum[0][0];
#pragma unroll
            for (int i = 0; i < kParts - 1; ++i) total += joined[i][t_in];
            if (t < most) out[t] = (in ? in[t] : 0.f) + total;
        }
        __syncthreads();
    }
}

// One list for all heads: the heads' sums, one after the other.
__global__ void __launch_bounds__(256) weigh_join_kernel(const WeighArgs g)
{
    const uint32_t x = g.first + blockIdx.x, seq = x % g.b.n_seqs, t = x / g.b.n_seqs * 256 + threadIdx.x;
    if (t >= g.b.max_kv) return;
    const float* const from = g.by_head + (uint64_t)seq * g.c.heads * g.b.max_kv + t;
    float total = 0.f;
    for (uint32_t h = 0; h < g.c.heads; ++h) total += from[(uint64_t)h * g.b.max_kv];
    const uint64_t at = (uint64_t)seq * g.weights_stride + t;
    g.out[at] = (g.weights ? g.weights[at] : 0.f) + total;
}

// Lines that few_kernel holds; it has no form for more.  32 sequences of 5,120 tokens, 8 heads of 128 dimensions, few_kernel and many_kernel: 4 lines in
// 4 bits 27 and 244 us, in 16 bits 70 and 312; 32 lines 37 and 245, 74 and 312.  So a step over a cache is slow from 33 lines on: 33 to 64 lines 245
// and 310 us, 128 lines 257 and 325, the latencies of a tile with one step of products.
bool few_lines(const tent_kv_cache& c, const tent_kv_batch& b, const tent_kv_weigh_args& a)
{
    return (uint64_t)b.max_rows * (a.q_heads / c.kv_heads) <= 32;
}
uint64_t workspace_of(const tent_kv_cache& c, const tent_kv_batch& b, const tent_kv_weigh_args& a)
{
    return a.n_lists == 1 && c.kv_heads > 1 && !few_lines(c, b, a) ? (uint64_t)b.n_seqs * c.kv_heads * b.max_kv * 4 : 0;
}

template <class E, int D, int kBits>
int launch(bool few, WeighArgs g, hipStream_t s)
{
    const uint64_t max_kv = g.b.max_kv;
    if (few) {
        const bool one = g.n_lists == 1 && g.c.heads > 1;
        // A wave's run of tiles: as long as there are workgroups for all compute units eight times over.  8 heads of 128 dimensions, 1, 2 and 4 tiles: 4
        // sequences of 5,120 tokens in 4 bits 7.8, 8.5 and 8.5 us; 16 of them 19.2, 17.0 and 17.7; 64 of them 67.8, 53.1 and 50.2, in 16 bits 152, 138 and 138.
        const uint64_t units = (uint64_t)g.b.n_seqs * g.n_lists * ((max_kv + 127) / 128);
        g.run = one || units < 4096 ? 1 : units < 16384 ? 2 : 4;
        g.tiles = (uint32_t)((max_kv + (one ? 32 : 128 * g.run) - 1) / (one ? 32 : 128 * g.run));
        return launch_blocks(((uint64_t)g.tiles * g.b.n_seqs + 7) / 8 * 8 * g.n_lists, [&](uint32_t first, uint32_t blocks) {
            g.first = first;
            if (one) hipLaunchKernelGGL((few_kernel<E, D, kBits, true>), dim3(blocks), dim3(256), 0, s, g);
            else hipLaunchKernelGGL((few_kernel<E, D, kBits, false>), dim3(blocks), dim3(256), 0, s, g);
        });
    }
    g.tiles = (uint32_t)((max_kv + 2 * kTileTokens - 1) / (2 * kTileTokens));
    const int rc = launch_blocks((uint64_t)g.tiles * g.b.n_seqs * g.c.heads, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((many_kernel<E, D, kBits>), dim3(blocks), dim3(kManyThreads), 0, s, g);
    }, kMostBlocks / 4);
    if (rc != TENT_OK || !g.by_head) return rc;
    return launch_blocks((max_kv + 255) / 256 * g.b.n_seqs, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL(weigh_join_kernel, dim3(blocks), dim3(256), 0, s, g);
    });
}

// Lines of a sequence and head are numbered in 32 bits, those of a last step behind them as well.
constexpr uint64_t kMostLines = 0x7FFFFFFFull - 1024;

int check(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_weigh_args* args)
{
    int rc = kv_check_cache(cache);
    if (rc == TENT_OK) rc = kv_check_sequences(batch);
    if (rc != TENT_OK) return rc;
    if (!args || args->reserved || (args->flags & ~(uint32_t)TENT_KV_ATTEND_ALL)) return TENT_ERR_INVALID;
    if (args->q_heads < 1 || args->q_heads > TENT_KV_MAX_HEADS || args->q_heads % cache->kv_heads) return TENT_ERR_RANGE;
    if (!(args->scale > 0.f) || args->scale > 3.4e38f || args->window > (1u << 30)) return TENT_ERR_RANGE;
    if (batch->n_seqs && batch->n_rows && (uint64_t)batch->max_rows * (args->q_heads / cache->kv_heads) > kMostLines) return TENT_ERR_RANGE;
    return args->n_lists != 1 && args->n_lists != cache->kv_heads ? TENT_ERR_RANGE : TENT_OK;
}

}  // namespace
}  // namespace tent

using namespace tent;

extern "C" int tent_kv_weigh_workspace(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_weigh_args* args, uint64_t* bytes)
{
    const int rc = check(cache, batch, args);
    if (rc != TENT_OK) return rc;
    if (!bytes) return TENT_ERR_INVALID;
    *bytes = batch->n_seqs == 0 ? 0 : workspace_of(*cache, *batch, *args);
    return TENT_OK;
}

extern "C" int tent_kv_weigh(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_weigh_args* args, void* stream)
{
    int rc = check(cache, batch, args);
    if (rc != TENT_OK) return rc;
    if (batch->n_seqs == 0) return TENT_OK;
    if ((rc = kv_check_table(cache, batch)) != TENT_OK) return rc;
    if (batch->n_rows) {
        if ((rc = kv_check_rows(args->q, args->q_stride, args->q_heads, cache->head_dim, batch->n_rows)) != TENT_OK) return rc;
        if (!args->lse) return TENT_ERR_INVALID;
    }
    if ((!args->weights_out && batch->max_kv) || (((uintptr_t)args->lse | (uintptr_t)args->weights | (uintptr_t)args->weights_out) & 3u)) return TENT_ERR_INVALID;
    if (args->weights_stride < batch->max_kv || args->weights_stride > ((uint64_t)1 << 60) / ((uint64_t)batch->n_seqs * args->n_lists)) return TENT_ERR_RANGE;
    if (kv_lists_meet(args->weights, args->weights_out, (uint64_t)batch->n_seqs * args->n_lists, batch->max_kv, args->weights_stride)) return TENT_ERR_INVALID;
    const uint64_t need = workspace_of(*cache, *batch, *args);
    if (need && (!args->workspace || !kv_aligned(args->workspace))) return TENT_ERR_INVALID;
    if (need > args->workspace_bytes) return TENT_ERR_RANGE;
    const bool few = few_lines(*cache, *batch, *args);
    WeighArgs g{};
    g.c = kv_cache_dev(*cache);
    g.b = *batch;
    g.q = static_cast<const uint8_t*>(args->q);
    g.lse = args->lse;
    g.weights = args->weights;
    g.out = args->weights_out;
    g.by_head = need ? static_cast<float*>(args->workspace) : nullptr;
    g.q_stride = args->q_stride * 2;
    g.weights_stride = args->weights_stride;
    g.q_heads = args->q_heads;
    g.group = args->q_heads / cache->kv_heads;
    g.n_lists = args->n_lists;
    g.window = args->window;
    g.all = args->flags & TENT_KV_ATTEND_ALL ? 1 : 0;
    g.to_log2 = args->scale * kLog2e;
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_WEIGH(dim)                                                                                                  \
    (cache->type == TENT_BF16 ? (cache->bits == 16 ? launch<Bf16, dim, 16>(few, g, s) : launch<Bf16, dim, 4>(few, g, s)) \
                              : (cache->bits == 16 ? launch<Fp16, dim, 16>(few, g, s) : launch<Fp16, dim, 4>(few, g, s)))
    return cache->head_dim == 64 ? TENT_WEIGH(64) : cache->head_dim == 128 ? TENT_WEIGH(128) : TENT_WEIGH(256);
}
