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

// The sequences of a batch, for calls that take no pages or need no rows.
inline int kv_check_sequences(const tent_kv_batch* b)
{
    if (!b || b->reserved) return TENT_ERR_INVALID;
    if (b->n_seqs == 0) return TENT_OK;
    if (!b->kv_len || !b->row_start || (((uintptr_t)b->kv_len | (uintptr_t)b->row_start | (uintptr_t)b->errors) & 3u)) return TENT_ERR_INVALID;
    if (b->n_seqs > 65535 || b->n_rows > 0x7FFFFFFFu || (b->n_rows && (b->max_rows < 1 || b->max_rows > b->n_rows)) || b->max_kv > (1u << 30)) return TENT_ERR_RANGE;
    return TENT_OK;
}
inline int kv_check_table(const tent_kv_cache* c, const tent_kv_batch* b)
{
    if (!b->page_table || ((uintptr_t)b->page_table & 3u)) return TENT_ERR_INVALID;
    return b->max_kv > (uint64_t)b->table_stride * c->page_tokens ? TENT_ERR_RANGE : TENT_OK;
}

// Whether one range of bytes has any of another.
inline bool kv_meet(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && (x < y ? y - x < a_bytes : x - y < b_bytes);
}
// Whether values of other places share memory where two tensors have `lists` lists of `width` floats, `stride` (at least width) apart.  They do
// not where the two are one and the same, nor where lists of one lie between those of the other.
inline bool kv_lists_meet(const float* a, const float* b, uint64_t lists, uint64_t width, uint64_t stride)
{
    if (!a || !b || a == b || !width || !lists) return false;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    const uint64_t apart = (x < y ? y - x : x - y) / 4, k = apart / stride, r = apart % stride;
    return (r < width && k < lists) || (stride - r < width && k + 1 < lists);
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

// What a sequence's lists of kept tokens are about: tokens from `base` on, `have` of them, of which `count` entries are kept.  Bad: it stays as it is.
struct KvKept {
    int32_t base, have, count;
    bool bad;
    TENT_KV_BOTH int32_t length() const { return base + count; }         // afterwards; of one that is not bad
    TENT_KV_BOTH int32_t length_up_to(int32_t most) const { return length() < most ? length() : most; }
};
TENT_KV_BOTH KvKept kv_kept(const KvSeq& q, bool by_rows, bool elsewhere, int32_t count, uint32_t most)
{
    KvKept k{by_rows ? q.len - q.rows : 0, by_rows ? q.rows : q.len, count, false};
    k.bad = q.bad || k.base < 0 || count < 0 || (uint32_t)count > most || (!elsewhere && count > k.have) || count > 0x7FFFFFFF - k.base;
    return k;
}

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

// What a row of a tree sees: the context from lo to base, and of the rows, tokens base to len, those that its mask names (`words` of it).
// Of a window the context has what the `deep` rows that it sees leave.
struct KvTreeSpan { int32_t lo, base, len, words; };
TENT_KV_BOTH KvTreeSpan kv_tree_span(int32_t rows, int32_t len, uint32_t window, int32_t deep)
{
    const int32_t base = len - rows, lo = window ? base + deep - (int32_t)window : 0;
    return KvTreeSpan{lo > 0 ? lo : 0, base, len, (rows + 63) >> 6};
}
// The 64 tokens from t0 on as bits; word(i): 64 rows of the mask, 0 for those past the last.
template <class Word>
TENT_KV_BOTH uint64_t kv_tree_bits(const KvTreeSpan& s, int32_t t0, Word word)
{
    const int32_t at = t0 - s.base;                                      // of the first among the rows
    uint64_t bits = at <= -64 ? ~0ull : at < 0 ? ~(~0ull << -at) : 0;
    if (s.lo > t0) bits = s.lo < t0 + 64 ? bits & ~0ull << (s.lo - t0) : 0;
    if (at > -64) {
        if (at < 0) bits |= word(0) << -at;
        else bits |= word(at >> 6) >> (at & 63) | (at & 63 ? word((at >> 6) + 1) << (64 - (at & 63)) : 0);
    }
    return bits;
}

}  // namespace tent
