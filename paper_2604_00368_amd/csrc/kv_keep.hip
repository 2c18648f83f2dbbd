// What a sequence of a key/value cache keeps, and the move that makes it the sequence: tent_kv_choose and tent_kv_keep.
#include "kv_elem.h"

namespace tent {
namespace {

// ---- choosing ------------------------------------------------------------------------------------
// A workgroup for each list.  The weight that the last chosen token has is found digit by digit: a histogram of the digits of those
// weights whose higher digits are the wanted ones, then the digit at which as many lie above as are wanted.
struct ChooseArgs {
    tent_kv_choose_args a;
    tent_kv_batch b;
    uint32_t first;                    // of the launch's workgroups
};
constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr int kDigit = 256;

// Larger weights as larger whole numbers; zeros are alike, NaN is minus infinity.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t x = w != w ? 0xFF800000u : w == 0.f ? 0u : __float_as_uint(w);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

__global__ void __launch_bounds__(kChooseThreads) choose_kernel(const ChooseArgs g)
{
    __shared__ uint32_t count[kDigit], wave_above[kChooseWaves], wave_equal[kChooseWaves], digit_lds, wanted_lds;
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
    uint32_t wanted = a.budget - a.first - a.recent, border = 0xFFFFFFFFu, equal = 0;
    if (wanted) {
        uint32_t above = 0;                                              // the digits found, at their places
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < kDigit) count[threadIdx.x] = 0;
            __syncthreads();
            for (uint32_t t = lo + threadIdx.x; t < hi; t += kChooseThreads) {
                const uint32_t key = weight_key(w[t]);
                if (shift == 24 || key >> (shift + 8) == above >> (shift + 8)) atomicAdd(&count[key >> shift & 255u], 1u);
            }
            __syncthreads();
            if (wave == 0) {                                             // four digits a lane, the largest in lane 0
                uint32_t mine[4], sum = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += mine[i] = count[255 - (4 * lane + i)];
                uint32_t before = sum;
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) {
                    const uint32_t up = __shfl_up(before, m, 64);
                    before += lane >= (uint32_t)m ? up : 0u;
                }
                before -= sum;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (before < wanted && before + mine[i] >= wanted) {
                        digit_lds = 255 - (4 * lane + i);
                        wanted_lds = wanted - before;
                    }
                    before += mine[i];
                }
            }
            __syncthreads();
            above |= digit_lds << shift;
            wanted = wanted_lds;
        }
        border = above;
        equal = wanted;                                                  // of those at the border the first so many
    }
    // Tokens in their order: which are kept, and how many before them.
    uint32_t base = 0, equal_before = 0;
    for (uint32_t t0 = 0; t0 < n; t0 += kChooseThreads) {
        const uint32_t t = t0 + threadIdx.x;
        const bool there = t < n, decided = there && t >= lo && t < hi;
        const uint32_t key = decided ? weight_key(w[t]) : 0u;
        const bool always = there && !decided, more = always || (decided && equal && key > border), same = decided && equal && key == border;
        const uint64_t more_mask = __ballot(more), same_mask = __ballot(same), below = (1ull << lane) - 1;
        if (lane == 0) {
            wave_above[wave] = (uint32_t)__popcll(more_mask);
            wave_equal[wave] = (uint32_t)__popcll(same_mask);
        }
        __syncthreads();
        uint32_t at = base + (uint32_t)__popcll(more_mask & below), eq = equal_before + (uint32_t)__popcll(same_mask & below);
        for (uint32_t i = 0; i < kChooseWaves; ++i) {
            const uint32_t m = wave_above[i], s = wave_equal[i];
            if (i < wave) { at += m; eq += s; }
            base += m;
            equal_before += s;
        }
        if (more || (same && eq < equal)) to[at + (eq < equal ? eq : equal)] = (int32_t)t;
        __syncthreads();
    }
}

// ---- moving --------------------------------------------------------------------------------------
struct KeepArgs {
    KvCache c;
    tent_kv_batch b;
    tent_kv_keep_args a;
    uint32_t columns;                  // workgroups that share a head's row, in place
    uint32_t parts;                    // workgroups that share a list, to other pages
    uint32_t first;                    // of the launch's workgroups
};
constexpr uint32_t kEntries = 128;     // of a list at a time
constexpr uint64_t kNowhere = ~0ull;

// What a sequence's lists are about: tokens from `base` on, `have` of them, of which `count` entries are kept.
struct Kept { int32_t base, have, count; bool bad; };
__device__ __forceinline__ Kept kept_of(const tent_kv_keep_args& a, const KvSeq& q, uint32_t seq)
{
    const bool rows = a.flags & TENT_KV_KEEP_ROWS;
    Kept k{rows ? q.len - q.rows : 0, rows ? q.rows : q.len, a.counts[seq], false};
    k.bad = q.bad || k.base < 0 || k.count < 0 || (uint32_t)k.count > a.most || (!a.to_table && k.count > k.have);
    return k;
}
__device__ __forceinline__ bool entry_ok(const tent_kv_keep_args& a, const Kept& k, int32_t entry, int32_t j)
{
    return entry < k.have && entry >= (a.to_table ? 0 : j);
}

// A workgroup has a head's rows of K or V (in place a column of them), and of the list all entries in turn, or (to other pages) some.  In
// place every entry is at or behind its own place, so what a batch of entries writes no later one reads; within a batch all is
// read before anything is written.  Columns have nothing to do with each other.
template <int D, int kBits>
__global__ void __launch_bounds__(256) keep_kernel(const KeepArgs g)
{
    constexpr uint32_t kChunks = kBits == 16 ? D / 8 : D / 32;           // vectors of a head's row, without the scales
    constexpr uint32_t kItems = kEntries * kChunks / 256;                // of a thread, of a whole row
    constexpr uint32_t kScale = D / 32;                                  // bytes of scales
    __shared__ uint64_t from[kEntries], to[kEntries], from_scale[kBits == 4 ? kEntries : 1], to_scale[kBits == 4 ? kEntries : 1];
    const tent_kv_keep_args& a = g.a;
    uint32_t x = g.first + blockIdx.x;
    const uint32_t column = x % g.columns; x /= g.columns;
    const uint32_t is_v = x & 1u; x >>= 1;
    const uint32_t head = x % g.c.heads; x /= g.c.heads;
    const uint32_t part = x % g.parts, seq = x / g.parts;
    const KvSeq q = kv_sequence(g.b, seq);
    const Kept k = kept_of(a, q, seq);
    const bool tells = column == 0 && is_v == 0 && head == 0 && part == 0 && threadIdx.x == 0;
    if (tells) {
        if (k.bad) kv_note(g.b.errors, TENT_KV_BAD_SEQUENCE);
        if (a.kv_len_out) a.kv_len_out[seq] = k.bad ? g.b.kv_len[seq] : k.base + k.count;
    }
    if (k.bad) return;
    uint8_t* const pool = is_v ? g.c.v : g.c.k;
    const int32_t* const list = a.lists + ((uint64_t)seq * a.n_lists + (a.n_lists == 1 ? 0u : head)) * a.list_stride;
    const uint32_t wide = kChunks / g.columns, chunk0 = column * wide, wide_log = 31 - __builtin_clz(wide);      // vectors of the column, a power of two
    const bool in_place = !a.to_table;
    auto place = [&](uint32_t token, const int32_t* table, uint64_t stride, uint32_t entries, uint64_t& row, uint64_t& scale) {
        const uint32_t at = token >> g.c.page_shift;
        const uint32_t page = at < entries ? (uint32_t)table[seq * stride + at] : ~0u;
        if (page >= g.c.n_pages) return false;
        const uint32_t r = (token & ((1u << g.c.page_shift) - 1u)) * g.c.heads + head;
        row = page * g.c.page_stride + (uint64_t)r * (kBits == 16 ? D * 2 : D / 2);
        scale = page * g.c.page_stride + ((uint64_t)(g.c.heads * (D / 2)) << g.c.page_shift) + (uint64_t)r * kScale;
        return true;
    };
    const uint32_t first = part * kEntries, step = g.parts * kEntries;
    for (uint32_t j0 = first; j0 < (uint32_t)k.count; j0 += step) {
        const uint32_t n = (uint32_t)k.count - j0 < kEntries ? (uint32_t)k.count - j0 : kEntries;
        if (threadIdx.x < n) {
            const int32_t j = (int32_t)(j0 + threadIdx.x), entry = list[j];
            uint64_t row = kNowhere, scale = 0, to_row = 0, to_sc = 0;
            int32_t wrong = 0;
            if (!entry_ok(a, k, entry, j)) wrong = TENT_KV_BAD_POSITION;
            else if (!in_place || entry != j) {
                const bool read = place((uint32_t)(k.base + entry), g.b.page_table, g.b.table_stride, g.b.table_stride, row, scale);
                const bool write = place((uint32_t)(k.base + j), in_place ? g.b.page_table : a.to_table, in_place ? g.b.table_stride : a.to_stride,
                                         in_place ? g.b.table_stride : a.to_stride, to_row, to_sc);
                if (!read || !write) {
                    wrong = TENT_KV_BAD_PAGE;
                    row = kNowhere;
                }
            }
            if (wrong && column == 0 && is_v == 0) kv_note(g.b.errors, wrong);
            from[threadIdx.x] = row;
            to[threadIdx.x] = to_row;
            if constexpr (kBits == 4) {
                from_scale[threadIdx.x] = scale;
                to_scale[threadIdx.x] = to_sc;
            }
        }
        __syncthreads();
        u32x4 v[kItems] = {};
        u32x2 s = {0, 0};
        const uint32_t items = n * wide;
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t item = i * 256 + threadIdx.x;
            if (item < items && from[item >> wide_log] != kNowhere) v[i] = dev_load<u32x4>(pool + from[item >> wide_log] + (chunk0 + (item & (wide - 1))) * 16);
        }
        if constexpr (kBits == 4) {
            if (column == 0 && threadIdx.x < n && from[threadIdx.x] != kNowhere) {
                const uint8_t* const p = pool + from_scale[threadIdx.x];
                if constexpr (kScale == 2) s[0] = dev_load<uint16_t>(p);
                else if constexpr (kScale == 4) s[0] = dev_load<uint32_t>(p);
                else s = dev_load<u32x2>(p);
            }
        }
        // all of it is here before any of it is written
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) __asm__ volatile("" : "+v"(v[i]));
        __asm__ volatile("" : "+v"(s));
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t item = i * 256 + threadIdx.x;
            if (item < items && from[item >> wide_log] != kNowhere) dev_store(pool + to[item >> wide_log] + (chunk0 + (item & (wide - 1))) * 16, v[i]);
        }
        if constexpr (kBits == 4) {
            if (column == 0 && threadIdx.x < n && from[threadIdx.x] != kNowhere) {
                uint8_t* const p = pool + to_scale[threadIdx.x];
                if constexpr (kScale == 2) dev_store(p, (uint16_t)s[0]);
                else if constexpr (kScale == 4) dev_store(p, s[0]);
                else dev_store(p, s);
            }
        }
        __syncthreads();                                                 // the places are written anew
    }
}

// The weights of kept tokens, a workgroup for each list of them: in their order, so that in place nothing is read that was written.
__global__ void __launch_bounds__(256) keep_weights_kernel(const KeepArgs g)
{
    const tent_kv_keep_args& a = g.a;
    const uint32_t block = g.first + blockIdx.x, seq = block / a.n_weights, l = block - seq * a.n_weights;
    const KvSeq q = kv_sequence(g.b, seq);
    const Kept k = kept_of(a, q, seq);
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
    for (int32_t t = base + count + (int32_t)threadIdx.x; t < most; t += 256) to[t] = 0.f;
}

template <int D, int kBits>
int launch_keep(KeepArgs g, hipStream_t s)
{
    constexpr uint32_t kChunks = kBits == 16 ? D / 8 : D / 32;
    const uint64_t lists = (uint64_t)g.b.n_seqs * 2 * g.c.heads;
    g.columns = 1;
    g.parts = 1;
    if (g.a.to_table) {
        g.parts = (g.a.most + kEntries - 1) / kEntries;
        if (g.parts < 1) g.parts = 1;
    } else {
        while (lists * g.columns < 512 && kChunks / g.columns > 4) g.columns *= 2;
    }
    return launch_blocks(lists * g.columns * g.parts, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((keep_kernel<D, kBits>), dim3(blocks), dim3(256), 0, s, g);
    });
}

}  // namespace
}  // namespace tent

using namespace tent;

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
    const uint64_t lists = (uint64_t)batch->n_seqs * args->n_lists, most = ((uint64_t)1 << 60) / lists;
    if (args->weights_stride < batch->max_kv || args->weights_stride > most || args->list_stride < args->budget || args->list_stride > most) return TENT_ERR_RANGE;
    ChooseArgs g{*args, *batch, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
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
    if ((!args->lists && args->most) || !args->counts || args->kv_len_out == batch->kv_len) return TENT_ERR_INVALID;
    if (((uintptr_t)args->lists | (uintptr_t)args->counts | (uintptr_t)args->to_table | (uintptr_t)args->kv_len_out | (uintptr_t)args->weights |
         (uintptr_t)args->weights_out) & 3u) return TENT_ERR_INVALID;
    if ((!args->weights) != (!args->weights_out) || (args->to_table && args->weights && args->weights == args->weights_out)) return TENT_ERR_INVALID;
    const uint64_t most = ((uint64_t)1 << 60) / ((uint64_t)batch->n_seqs * cache->kv_heads);
    if ((args->n_lists != 1 && args->n_lists != cache->kv_heads) || args->most > (1u << 30)) return TENT_ERR_RANGE;
    if (args->list_stride < args->most || args->list_stride > most) return TENT_ERR_RANGE;
    if (args->weights) {
        if ((args->n_weights != 1 && args->n_weights != cache->kv_heads) || args->n_weights < args->n_lists) return TENT_ERR_RANGE;
        if (args->weights_stride < batch->max_kv || args->weights_stride > most) return TENT_ERR_RANGE;
    }
    KeepArgs g{kv_cache_dev(*cache), *batch, *args, 1, 1, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_KEEP(dim) (cache->bits == 16 ? launch_keep<dim, 16>(g, s) : launch_keep<dim, 4>(g, s))
    rc = cache->head_dim == 64 ? TENT_KEEP(64) : cache->head_dim == 128 ? TENT_KEEP(128) : TENT_KEEP(256);
    if (rc != TENT_OK || !args->weights) return rc;
    return launch_blocks((uint64_t)batch->n_seqs * args->n_weights, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL(keep_weights_kernel, dim3(blocks), dim3(256), 0, s, g);
    });
}
