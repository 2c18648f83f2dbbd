// Addressing and checks of the paged key/value caches, shared by the operators on them (tent.h, "Operators on paged
// key/value caches").  Everything here is plain arithmetic, so that it also compiles for the host alone.
#pragma once

#include <stdint.h>

#include "../../include/tent.h"

#ifdef __HIP__
#define TENT_KV_BOTH __host__ __device__ __forceinline__
#else
#define TENT_KV_BOTH inline
#endif

namespace tent {

// ---- host: what a call is refused for ----
inline bool kv_aligned(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline uint64_t kv_page_bytes(uint32_t page_tokens, uint32_t kv_heads, uint32_t head_dim, uint32_t bits)
{
    const uint64_t rows = (uint64_t)page_tokens * kv_heads;
    return bits == 16 ? rows * head_dim * 2 : rows * (head_dim / 2 + head_dim / 32);
}

inline bool kv_sizes_ok(uint32_t page_tokens, uint32_t kv_heads, uint32_t head_dim)
{
    return page_tokens >= 1 && page_tokens <= TENT_KV_MAX_PAGE_TOKENS && (page_tokens & (page_tokens - 1)) == 0 &&
           kv_heads >= 1 && kv_heads <= TENT_KV_MAX_HEADS && (head_dim == 64 || head_dim == 128 || head_dim == 256);
}

inline int kv_check_cache(const tent_kv_cache* c)
{
    if (!c || !c->k || !c->v || !kv_aligned(c->k) || !kv_aligned(c->v) || (c->page_stride & 15u)) return TENT_ERR_INVALID;
    if ((c->type != TENT_BF16 && c->type != TENT_FP16) || (c->bits != 16 && c->bits != 4) || c->reserved) return TENT_ERR_INVALID;
    if (!kv_sizes_ok(c->page_tokens, c->kv_heads, c->head_dim)) return TENT_ERR_RANGE;
    if (c->n_pages < 1 || c->n_pages > 0x7FFFFFFFull) return TENT_ERR_RANGE;
    if (c->page_stride < kv_page_bytes(c->page_tokens, c->kv_heads, c->head_dim, c->bits)) return TENT_ERR_RANGE;
    if (c->page_stride > ((uint64_t)1 << 62) / c->n_pages) return TENT_ERR_RANGE;
    return TENT_OK;
}

// A batch of no rows or no sequences passes: the caller has nothing to do for it.
inline int kv_check_batch(const tent_kv_cache* c, const tent_kv_batch* b)
{
    if (!b || b->reserved) return TENT_ERR_INVALID;
    if (b->n_seqs == 0 || b->n_rows == 0) return TENT_OK;
    if (!b->page_table || !b->kv_len || !b->row_start) return TENT_ERR_INVALID;
    if (((uintptr_t)b->page_table | (uintptr_t)b->kv_len | (uintptr_t)b->row_start | (uintptr_t)b->errors) & 3u) return TENT_ERR_INVALID;
    if (b->n_seqs > 65535 || b->n_rows > 0x7FFFFFFFu || b->max_rows < 1 || b->max_rows > b->n_rows) return TENT_ERR_RANGE;
    if (b->max_kv > (1u << 30) || b->max_kv > (uint64_t)b->table_stride * c->page_tokens) return TENT_ERR_RANGE;
    return TENT_OK;
}

// Rows of `heads` heads: a base, and a stride that holds them, in whole vectors of 16 bytes.
inline int kv_check_rows(const void* p, uint64_t stride, uint32_t heads, uint32_t head_dim, uint32_t n_rows)
{
    if (!p || !kv_aligned(p) || (stride & 7u)) return TENT_ERR_INVALID;
    if (stride < (uint64_t)heads * head_dim || stride > ((uint64_t)1 << 60) / (n_rows ? n_rows : 1)) return TENT_ERR_RANGE;
    return TENT_OK;
}

// ---- both: what the kernels work on ----
struct KvCache {
    uint8_t *k, *v;
    uint64_t page_stride;
    uint32_t n_pages, page_shift, heads;
};

inline KvCache kv_cache_dev(const tent_kv_cache& c)
{
    KvCache d{static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.page_stride, (uint32_t)c.n_pages, 0, c.kv_heads};
    while ((1u << d.page_shift) < c.page_tokens) ++d.page_shift;
    return d;
}

// A sequence of a batch, as far as it is what the call says.
struct KvSeq {
    int32_t row0, rows;        // rows 0: none, or a sequence that is left out
    int32_t len;               // tokens with the rows
    bool bad;
};

TENT_KV_BOTH KvSeq kv_sequence(const tent_kv_batch& b, int32_t lo, int32_t hi, int32_t len)
{
    const bool fits = lo >= 0 && hi >= lo && (uint32_t)hi <= b.n_rows && (uint32_t)(hi - lo) <= b.max_rows && len >= 0 &&
                      (uint32_t)len <= b.max_kv;
    return fits ? KvSeq{lo, hi - lo, len, false} : KvSeq{0, 0, 0, true};
}
TENT_KV_BOTH KvSeq kv_sequence(const tent_kv_batch& b, uint32_t s) { return kv_sequence(b, b.row_start[s], b.row_start[s + 1], b.kv_len[s]); }

// Byte offset of the page that holds token t (0 <= t < max_kv) of sequence s; negative where the table names none of the pool.
TENT_KV_BOTH int64_t kv_page_of(const KvCache& c, const tent_kv_batch& b, uint32_t s, uint32_t t)
{
    const uint32_t page = (uint32_t)b.page_table[(uint64_t)s * b.table_stride + (t >> c.page_shift)];
    return page < c.n_pages ? (int64_t)(page * c.page_stride) : -1;
}

// The tokens [lo, hi) that a row sees: `row` of the `rows` last tokens of `len`.
struct KvSpan { int32_t lo, hi; };
TENT_KV_BOTH KvSpan kv_span(int32_t row, int32_t rows, int32_t len, uint32_t window, bool all)
{
    const int32_t hi = all ? len : len - rows + row + 1;
    if (hi <= 0) return KvSpan{0, 0};
    const int32_t lo = window && window < (uint32_t)hi ? hi - (int32_t)window : 0;
    return KvSpan{lo, hi};
}

}  // namespace tent
