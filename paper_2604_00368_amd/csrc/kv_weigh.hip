// Attention weights onto the tokens of a cache: tent_kv_weigh.
//
//   w_t += sum over the lines l (rows and query heads of a cache head) that see token t of exp(scale q_l . k_t - lse_l)
//
// A workgroup has a tile of tokens, whose keys stay in registers as the first operand of S^T = K Q^T, and goes through the lines that see
// any of them.  A lane holds scores of one line of 32; its sums by token are added over the lanes at the end.  Each weight is
// written by one workgroup, in an order that does not change.
#include "kv_elem.h"

namespace tent {
namespace {

struct WeighArgs {
    KvCache c;
    tent_kv_batch b;
    const uint8_t* q;
    const float *lse, *weights;
    float* out;
    uint64_t q_stride, weights_stride; // bytes; values
    uint32_t q_heads, group, n_lists, window, all;
    float to_log2;                     // scale * log2(e)
    uint32_t tiles;                    // workgroups over the tokens of a sequence
    uint32_t first;                    // of the launch's workgroups
};
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWeighTokens = 128;      // of a workgroup: 32 a wave

// Adds the 16 sums of a lane over the 32 lanes that hold the same tokens: half of the sums go to the other lane each time.
// Afterwards lane m of the 32 has the sum of token i = m / 2 (in the order of the sums).
__device__ __forceinline__ float sum_lines(float (&x)[16], uint32_t m)
{
#pragma unroll
    for (int half = 8, bit = 16; half >= 1; half >>= 1, bit >>= 1) {
        const bool upper = m & (uint32_t)bit;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float give = upper ? x[i] : x[i + half], keep = upper ? x[i + half] : x[i];
            x[i] = keep + __shfl_xor(give, bit, 64);
        }
    }
    return x[0] + __shfl_xor(x[0], 1, 64);
}

template <class E, int D, int kBits>
__global__ void __launch_bounds__(256) weigh_kernel(const WeighArgs g)
{
    constexpr int kK = D / 16;
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t m = lane & 31u, upper = lane >> 5;
    uint32_t x = g.first + blockIdx.x;
    const uint32_t list = x % g.n_lists; x /= g.n_lists;
    const uint32_t seq = x % g.b.n_seqs, tile = x / g.b.n_seqs;
    const KvSeq q = kv_sequence(g.b, seq);
    if (q.bad && threadIdx.x == 0 && tile == 0 && list == 0) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
    const int32_t t0 = (int32_t)tile * kWeighTokens + (int32_t)wave * 32, most = (int32_t)g.b.max_kv;
    const uint64_t at = ((uint64_t)seq * g.n_lists + list) * g.weights_stride;
    float sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;

    if (q.rows > 0 && t0 < q.len) {
        // lane (m, upper) has dims of token t0 + m
        const int32_t mine = t0 + (int32_t)m;
        const int64_t page = mine < q.len ? kv_page_of(g.c, g.b, seq, (uint32_t)mine) : -1;
        if (page < 0 && mine < q.len && list == 0 && upper == 0) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
        const uint32_t there = (uint32_t)__ballot(page >= 0);
        // the rows that see any of the tokens: those at positions from t0 on, up to a window later
        const int32_t before = q.len - q.rows;
        int32_t first = 0, last = q.rows;                                // rows
        if (!g.all) {
            first = t0 - before > 0 ? t0 - before : 0;
            if (g.window) {
                const int64_t end = (int64_t)t0 + 31 + g.window - before;
                last = end < last ? (end > 0 ? (int32_t)end : 0) : last;
            }
            if (first < -before) first = -before;
        }
        const uint32_t heads = g.n_lists == 1 ? g.c.heads : 1u;
        for (uint32_t h = 0; h < heads; ++h) {
            const uint32_t head = g.n_lists == 1 ? h : list;
            u32x4 kf[kK];
            const uint64_t slot = (uint64_t)((uint32_t)mine & ((1u << g.c.page_shift) - 1u)) * g.c.heads + head;
            if constexpr (kBits == 16) {
                const uint8_t* const row = g.c.k + (page >= 0 ? (uint64_t)page + slot * (D * 2) : 0) + upper * 16;
#pragma unroll
                for (int k = 0; k < kK; ++k) kf[k] = dev_load<u32x4>(row + k * 32);
            } else {                                                     // half a row of codes each, in the order of the row
                const uint8_t* const row = g.c.k + (page >= 0 ? (uint64_t)page + slot * (D / 2) : 0) + upper * (D / 4);
                const uint8_t* const scales = g.c.k + (page >= 0 ? (uint64_t)page + ((uint64_t)(g.c.heads * (D / 2)) << g.c.page_shift) + slot * (D / 32) : 0) + upper * (D / 64);
#pragma unroll
                for (int k = 0; k < kK; k += 4) {
                    const u32x4 codes = dev_load<u32x4>(row + k * 4);
                    const float scale = scale_of(dev_load<uint8_t>(scales + k / 4));
#pragma unroll
                    for (int i = 0; i < 4; ++i) kf[k + i] = decode8<E>(codes[i], scale);
                }
            }
            const int32_t line0 = first * (int32_t)g.group, lines = last * (int32_t)g.group;
            for (int32_t l0 = line0; l0 < lines; l0 += 32) {
                const int32_t line = l0 + (int32_t)m < lines ? l0 + (int32_t)m : lines - 1;
                const int32_t row = line / (int32_t)g.group;
                const uint32_t q_head = head * g.group + (uint32_t)(line - row * (int32_t)g.group);
                const uint64_t q_row = (uint64_t)(q.row0 + row);
                const uint8_t* const p = g.q + q_row * g.q_stride + ((uint64_t)q_head * D + upper * (kBits == 16 ? 8 : D / 2)) * 2;
                const float lse = dev_load<float>(g.lse + q_row * g.q_heads + q_head);
                f32x16 s;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
                for (int k = 0; k < kK; ++k) s = E::mfma32(kf[k], dev_load<u32x4>(p + k * (kBits == 16 ? 32 : 16)), s);
                // which of the 32 tokens the line sees
                const KvSpan see = kv_span(row, q.rows, q.len, g.window, g.all);
                uint32_t seen = there;
                if (see.hi < t0 + 32) seen = see.hi > t0 ? seen & ~(~0u << (see.hi - t0)) : 0u;
                if (see.lo > t0) seen = see.lo < t0 + 32 ? seen & ~0u << (see.lo - t0) : 0u;
                if (l0 + (int32_t)m >= lines || !(fabsf(lse) < INFINITY)) seen = 0u;
                seen >>= 4 * upper;
                const float shift = -lse * kLog2e;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(s[i], g.to_log2, shift));
                    sum[i] += seen & (1u << (8 * (i >> 2) + (i & 3))) ? w : 0.f;
                }
            }
        }
    }
    // token 8 (i / 4) + 4 upper + i % 4 of sum i
    const float total = sum_lines(sum, m);
    const uint32_t i = m >> 1;
    const int32_t t = t0 + (int32_t)(8 * (i >> 2) + 4 * upper + (i & 3u));
    if ((m & 1u) == 0 && t < most) g.out[at + t] = (g.weights ? g.weights[at + t] : 0.f) + total;
}

template <class E, int D, int kBits>
int launch(WeighArgs g, hipStream_t s)
{
    g.tiles = (g.b.max_kv + kWeighTokens - 1) / kWeighTokens;
    return launch_blocks((uint64_t)g.tiles * g.b.n_seqs * g.n_lists, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((weigh_kernel<E, D, kBits>), dim3(blocks), dim3(256), 0, s, g);
    });
}

}  // namespace
}  // namespace tent

using namespace tent;

extern "C" int tent_kv_weigh(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_weigh_args* args, void* stream)
{
    int rc = kv_check_cache(cache);
    if (rc == TENT_OK) rc = kv_check_sequences(batch);
    if (rc != TENT_OK) return rc;
    if (!args || args->reserved || (args->flags & ~(uint32_t)TENT_KV_ATTEND_ALL)) return TENT_ERR_INVALID;
    if (args->q_heads < 1 || args->q_heads > TENT_KV_MAX_HEADS || args->q_heads % cache->kv_heads) return TENT_ERR_RANGE;
    if (!(args->scale > 0.f) || args->scale > 3.4e38f || args->window > (1u << 30)) return TENT_ERR_RANGE;
    if (args->n_lists != 1 && args->n_lists != cache->kv_heads) return TENT_ERR_RANGE;
    if (batch->n_seqs == 0) return TENT_OK;
    if ((rc = kv_check_table(cache, batch)) != TENT_OK) return rc;
    if (batch->n_rows) {
        if ((rc = kv_check_rows(args->q, args->q_stride, args->q_heads, cache->head_dim, batch->n_rows)) != TENT_OK) return rc;
        if (!args->lse) return TENT_ERR_INVALID;
    }
    if ((!args->weights_out && batch->max_kv) || (((uintptr_t)args->lse | (uintptr_t)args->weights | (uintptr_t)args->weights_out) & 3u)) return TENT_ERR_INVALID;
    if (args->weights_stride < batch->max_kv || args->weights_stride > ((uint64_t)1 << 60) / ((uint64_t)batch->n_seqs * args->n_lists)) return TENT_ERR_RANGE;
    WeighArgs g{};
    g.c = kv_cache_dev(*cache);
    g.b = *batch;
    g.q = static_cast<const uint8_t*>(args->q);
    g.lse = args->lse;
    g.weights = args->weights;
    g.out = args->weights_out;
    g.q_stride = args->q_stride * 2;
    g.weights_stride = args->weights_stride;
    g.q_heads = args->q_heads;
    g.group = args->q_heads / cache->kv_heads;
    g.n_lists = args->n_lists;
    g.window = args->window;
    g.all = args->flags & TENT_KV_ATTEND_ALL ? 1 : 0;
    g.to_log2 = args->scale * kLog2e;
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_WEIGH(dim)                                                                                    \
    (cache->type == TENT_BF16 ? (cache->bits == 16 ? launch<Bf16, dim, 16>(g, s) : launch<Bf16, dim, 4>(g, s)) \
                              : (cache->bits == 16 ? launch<Fp16, dim, 16>(g, s) : launch<Fp16, dim, 4>(g, s)))
    return cache->head_dim == 64 ? TENT_WEIGH(64) : cache->head_dim == 128 ? TENT_WEIGH(128) : TENT_WEIGH(256);
}
