// Operators that fill, shrink and read the pages of a key/value cache: tent_kv_append, tent_kv_pack, tent_kv_read.
//
// All three move each value once and compute little: HBM bounds them, and latency where there are few rows.  A lane
// works on eight values (16 bytes of a 16-bit row, 4 bytes of codes; four lanes in a row share a block's scale).
//
// Measured, 8 heads of 128 dimensions (and 32 of queries): append of 20,500 rows in 16 bits, 515 MB, 137 us (3.8 TB/s), of one
// row 4 us; pack of 177,500 tokens, 920 MB, 178 us (5.2 TB/s, where a large copy reaches 4.7); read of as many from 4 bits 192 us, of 30,000
// 25 us (6.3 TB/s, much of it from the last-level cache).
#include "kv_elem.h"

namespace tent {
namespace {

// Where the rows of a workgroup lie: found by its first lanes, used by all of it.
constexpr uint32_t kMaxRowTile = 16;
struct RowPlace {
    uint32_t seq, position;
    bool live;                 // the row belongs to a sequence that is not left out, at a position >= 0
};

// The last sequence whose row_start is at most `row`: 64 places at a time, one wave.
__device__ __forceinline__ uint32_t find_sequence(const tent_kv_batch& b, int32_t row, uint32_t lane)
{
    uint32_t lo = 0, n = b.n_seqs;
    while (n > 1) {
        const uint32_t step = (n + 63) / 64, at = lane * step;
        const bool below = at < n && b.row_start[lo + at] <= row;
        const uint32_t below_n = (uint32_t)__popcll(__ballot(below));   // row_start ascends: a prefix of the lanes
        if (below_n == 0) return lo;
        lo += (below_n - 1) * step;
        n -= (below_n - 1) * step;
        n = n < step ? n : step;
    }
    return lo;
}

// Up to 64 sequences are loaded at once, a lane each, so that a row's place is one load away; more of them are searched.  Wrong
// sequences are noted whether or not rows belong to them: by the first workgroup, or, of more than 64, by as many as it takes.
__device__ __forceinline__ void find_rows(RowPlace* to, const KvCache& c, const tent_kv_batch& b, uint32_t row0, uint32_t n)
{
    if (threadIdx.x < 64) {
        const uint32_t lane = threadIdx.x;
        const int32_t row = (int32_t)(row0 + lane);
        uint32_t s = 0;
        KvSeq q{0, 0, 0, false};
        if (b.n_seqs <= 64) {
            const uint32_t at = lane < b.n_seqs ? lane : b.n_seqs - 1;
            const int32_t lo = b.row_start[at], hi = b.row_start[at + 1], len = b.kv_len[at];
            for (uint32_t i = 0; i < n; ++i) {
                const uint32_t before = (uint32_t)__popcll(__ballot(lane < b.n_seqs && lo <= (int32_t)(row0 + i)));
                if (lane == i) s = before ? before - 1 : 0;
            }
            q = kv_sequence(b, __shfl(lo, (int)s, 64), __shfl(hi, (int)s, 64), __shfl(len, (int)s, 64));
            if (blockIdx.x == 0 && kv_sequence(b, lo, hi, len).bad) kv_note(b.errors, TENT_KV_BAD_SEQUENCE);
        } else {
            s = find_sequence(b, (int32_t)row0, lane);
            if (lane < n) {
                while (s + 1 < b.n_seqs && b.row_start[s + 1] <= row) ++s;
                q = kv_sequence(b, s);
            }
        }
        if (lane < n) {
            RowPlace p{0, 0, false};
            if (row >= q.row0 && row < q.row0 + q.rows) {                // a bad sequence has no rows
                const int32_t position = q.len - q.rows + (row - q.row0);
                if (position < 0) kv_note(b.errors, TENT_KV_BAD_POSITION);
                else p = RowPlace{s, (uint32_t)position, true};
            }
            to[lane] = p;
        }
    }
    __syncthreads();
    if (b.n_seqs > 64 && threadIdx.x < 64)                               // behind the barrier, which the others wait at
        for (uint32_t s = blockIdx.x * 64 + threadIdx.x; s < b.n_seqs; s += gridDim.x * 64)
            if (kv_sequence(b, s).bad) kv_note(b.errors, TENT_KV_BAD_SEQUENCE);
}

// A row's page as a byte offset, negative if there is none, and its token in it.
struct PagePlace { int64_t page; uint32_t slot; };
__device__ __forceinline__ PagePlace page_place(const KvCache& c, const tent_kv_batch& b, const RowPlace& p)
{
    return PagePlace{p.live ? kv_page_of(c, b, p.seq, p.position) : -1, p.position & ((1u << c.page_shift) - 1u)};
}

// Byte offsets inside a page of the eight values of chunk `chunk` of a head.
template <int D>
__device__ __forceinline__ uint32_t at16(uint32_t slot, uint32_t heads, uint32_t head, uint32_t chunk)
{
    return ((slot * heads + head) * D + chunk * 8) * 2;
}
template <int D>
__device__ __forceinline__ uint32_t at_codes(uint32_t slot, uint32_t heads, uint32_t head, uint32_t chunk)
{
    return (slot * heads + head) * (D / 2) + chunk * 4;
}
template <int D>
__device__ __forceinline__ uint32_t at_scale(uint32_t slot, uint32_t heads, uint32_t head, uint32_t chunk, uint32_t page_shift)
{
    return ((heads * (D / 2)) << page_shift) + (slot * heads + head) * (D / 32) + chunk / 4;
}

// Writes eight values of a row to its page.  Lanes of a block of 32 come here together.
template <class E, int D, int kBits>
__device__ __forceinline__ void put8(uint8_t* page, uint32_t page_shift, uint32_t slot, uint32_t heads, uint32_t head, uint32_t chunk, u32x4 v)
{
    if constexpr (kBits == 16) {
        dev_store(page + at16<D>(slot, heads, head, chunk), v);
    } else {
        uint32_t byte;
        const uint32_t codes = encode8<E>(v, byte);
        dev_store(page + at_codes<D>(slot, heads, head, chunk), codes);
        if ((chunk & 3u) == 0) dev_store(page + at_scale<D>(slot, heads, head, chunk, page_shift), (uint8_t)byte);
    }
}

template <int kWidth, class F>
__device__ __forceinline__ F sum_lanes(F x)
{
#pragma unroll
    for (int m = 1; m < kWidth; m <<= 1) x += __shfl_xor(x, m, 64);
    return x;
}

// A 64-bit value rounded to 32 bits.  The rounding stands by itself: without the barrier the compiler rounds to 16 bits at once,
// which differs where the 32-bit value is a tie.
__device__ __forceinline__ float in_32(float x) { return x; }
__device__ __forceinline__ float in_32(double x)
{
    float y = (float)x;
    __asm__("" : "+v"(y));
    return y;
}

// A 32-bit value of another lane of the same head.
__device__ __forceinline__ uint32_t of_lane(uint32_t x, uint32_t lane) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)(lane * 4), (int)x); }

struct AppendArgs {
    tent_kv_append_args a;
    KvCache c;
    tent_kv_batch b;
    uint32_t per_row;          // lanes that a row needs: one for every eight values of its heads
    uint32_t side;             // rows that a workgroup takes side by side
    uint32_t first;            // of the launch's workgroups
};

// Eight values of a head, normalised and turned; the lanes of the head come here together.  F: float for queries; double for keys,
// so that a value next to the border of two codes falls on its own side.  `w`: the weights of this lane's dimensions, `cs`: their
// cosines and sines.  What a dimension turns with is in another lane of the head.  `in_64` becomes true, and the result means nothing,
// where a float's range is too short for a mean of squares: of bfloat16 values from 2^60 on, or where neither they nor eps reach 2^-100.
template <class E, int D, class F>
__device__ __forceinline__ u32x4 norm_rotate(const tent_kv_append_args& a, u32x4 raw, uint32_t chunk, bool weighted, u32x4 w, const float* cs, bool& in_64)
{
    constexpr uint32_t kChunks = D / 8;
    if (!weighted && !a.rope) return raw;
    const uint32_t half = a.rope_dim / 16;                               // chunks of one half
    const bool turned = a.rope && chunk < 2 * half;
    const bool pairs = a.flags & TENT_KV_ROPE_PAIRS;
    F x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = (F)E::to_float(raw[i] & 0xFFFFu);
        x[2 * i + 1] = (F)E::to_float(raw[i] >> 16);
    }
    F r = 1;
    if (weighted) {
        F sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
        sum = sum_lanes<kChunks>(sum);
        const F mean = sum * ((F)1 / D) + (F)a.eps;
        if (E::kLarge && sizeof(F) == 4 && !(mean >= (F)0x1p-100 && mean < (F)0x1p120)) in_64 = true;
        r = (F)1 / sqrt(mean);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] *= r * (F)E::to_float(w[i] & 0xFFFFu);
            x[2 * i + 1] *= r * (F)E::to_float(w[i] >> 16);
        }
    }
    if (a.rope && !pairs) {
        const uint32_t partner = (threadIdx.x & 63u) - chunk + (!turned ? chunk : chunk < half ? chunk + half : chunk - half);
        const F sign = chunk < half ? (F)-1 : (F)1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t other = of_lane(raw[i], partner), other_w = weighted ? of_lane(w[i], partner) : 0u;
            F lo = (F)E::to_float(other & 0xFFFFu), hi = (F)E::to_float(other >> 16);
            if (weighted) {
                lo *= r * (F)E::to_float(other_w & 0xFFFFu);
                hi *= r * (F)E::to_float(other_w >> 16);
            }
            if (turned) {
                x[2 * i] = x[2 * i] * (F)cs[2 * i] + sign * lo * (F)cs[8 + 2 * i];
                x[2 * i + 1] = x[2 * i + 1] * (F)cs[2 * i + 1] + sign * hi * (F)cs[9 + 2 * i];
            }
        }
    } else if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F c = (F)cs[i], t = (F)cs[4 + i], p = x[2 * i], q = x[2 * i + 1];
            x[2 * i] = p * c - q * t;
            x[2 * i + 1] = q * c + p * t;
        }
    }
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = E::pack2(in_32(x[2 * i]), in_32(x[2 * i + 1]));
    return out;
}

// A workgroup takes one row, or `side` short ones side by side, or a part of one where there are few; all heads of it (queries, keys, values), a chunk of eight a lane and
// kBatch chunks at a time.  The chunks are on their way while the first wave finds where the row belongs, a chain of two or more loads.
// A lane keeps its chunk number over the heads, as the workgroup is a multiple of a head's lanes, and so its cosines and weights.
constexpr uint32_t kBatch = 4;
template <class E, int D, int kBits>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs g)
{
    __shared__ RowPlace place[kMaxRowTile];
    constexpr uint32_t kChunks = D / 8;
    const tent_kv_append_args& a = g.a;
    const uint32_t row0 = (g.first + blockIdx.x) * g.side, n = g.b.n_rows - row0 < g.side ? g.b.n_rows - row0 : g.side;
    const uint32_t r = g.side == 1 ? 0u : threadIdx.x / g.per_row, x0 = threadIdx.x - r * g.per_row + blockIdx.y * blockDim.x, chunk = x0 % kChunks;
    const uint32_t stride = blockDim.x * gridDim.y;
    const uint64_t row = row0 + r;
    const bool mine = r < n;
    auto load = [&](uint32_t x) -> u32x4 {                               // lanes past the last have nothing
        const uint32_t h = x / kChunks;
        const uint8_t* p;
        if (h < a.q_heads) p = (const uint8_t*)a.q + (row * a.q_stride + (uint64_t)h * D) * 2;
        else if (h < a.q_heads + g.c.heads) p = (const uint8_t*)a.k + (row * a.k_stride + (uint64_t)(h - a.q_heads) * D) * 2;
        else p = (const uint8_t*)a.v + (row * a.v_stride + (uint64_t)(h - a.q_heads - g.c.heads) * D) * 2;
        return dev_load<u32x4>(p + chunk * 16);
    };
    u32x4 raw[kBatch];
    auto load_batch = [&](uint32_t x) {
#pragma unroll
        for (uint32_t i = 0; i < kBatch; ++i)
            if (mine && x + i * stride < g.per_row) raw[i] = load(x + i * stride);
    };
    load_batch(x0);
    u32x4 wq = {0, 0, 0, 0}, wk = {0, 0, 0, 0};
    if (a.q_weight) wq = dev_load<u32x4>((const uint8_t*)a.q_weight + chunk * 16);
    if (a.k_weight) wk = dev_load<u32x4>((const uint8_t*)a.k_weight + chunk * 16);
    find_rows(place, g.c, g.b, row0, n);
    if (!mine) return;
    const RowPlace p = place[r];
    if (!p.live) return;
    const PagePlace to = page_place(g.c, g.b, p);                        // beside the cosines
    float cs[16] = {};
    if (a.rope) {
        const uint32_t at = a.positions ? (uint32_t)a.positions[row] : p.position;
        if (at >= a.rope_rows) {
            if (x0 == 0) kv_note(g.b.errors, TENT_KV_BAD_POSITION | (to.page < 0 ? TENT_KV_BAD_PAGE : 0));
            return;
        }
        const uint32_t half = a.rope_dim / 16;
        if (chunk < 2 * half) {
            const bool pairs = a.flags & TENT_KV_ROPE_PAIRS;
            const float* t = a.rope + (uint64_t)at * a.rope_dim + (pairs ? chunk * 4 : (chunk < half ? chunk : chunk - half) * 8);
            const f32x4 c0 = dev_load<f32x4>(t), s0 = dev_load<f32x4>(t + a.rope_dim / 2);
            const f32x4 c1 = pairs ? s0 : dev_load<f32x4>(t + 4), s1 = pairs ? s0 : dev_load<f32x4>(t + a.rope_dim / 2 + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cs[i] = c0[i];
                cs[4 + i] = c1[i];
                cs[8 + i] = s0[i];
                cs[12 + i] = s1[i];
            }
        }
    }
    if (to.page < 0 && x0 == 0) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
    for (uint32_t x = x0, left = kBatch; x < g.per_row; x += stride, --left) {
        if (left == 0) {
            load_batch(x);
            left = kBatch;
        }
        const u32x4 now = raw[0];
#pragma unroll
        for (uint32_t i = 0; i + 1 < kBatch; ++i) raw[i] = raw[i + 1];
        // cosines and weights are kept as they are: the compiler would keep them in 64 bits, and twice the registers
#pragma unroll
        for (int i = 0; i < 16; ++i) __asm__ volatile("" : "+v"(cs[i]));
        __asm__ volatile("" : "+v"(wq), "+v"(wk));
        const uint32_t h = x / kChunks;
        bool in_64 = false;
        if (h < a.q_heads) {
            u32x4 y = norm_rotate<E, D, float>(a, now, chunk, a.q_weight, wq, cs, in_64);
            if (in_64) y = norm_rotate<E, D, double>(a, now, chunk, a.q_weight, wq, cs, in_64);
            dev_store((uint8_t*)a.q_out + (row * a.q_out_stride + (uint64_t)h * D + chunk * 8) * 2, y);
        } else if (to.page >= 0) {
            const bool is_v = h >= a.q_heads + g.c.heads;
            const uint32_t kh = h - a.q_heads - (is_v ? g.c.heads : 0u);
            const u32x4 y = is_v ? now : norm_rotate<E, D, double>(a, now, chunk, a.k_weight, wk, cs, in_64);
            put8<E, D, kBits>((is_v ? g.c.v : g.c.k) + to.page, g.c.page_shift, to.slot, g.c.heads, kh, chunk, y);
        }
    }
}

struct ReadArgs {
    KvCache c;
    tent_kv_batch b;
    uint8_t *k, *v;
    uint64_t stride;           // bytes
    uint32_t row_tile;
    uint32_t first;            // of the launch's workgroups
};

// A workgroup takes `row_tile` rows, their keys first, then their values, kBatch chunks a lane in flight.
template <class E, int D, int kBits>
__global__ void __launch_bounds__(256) read_kernel(const ReadArgs g)
{
    __shared__ RowPlace place[kMaxRowTile];
    constexpr uint32_t kChunks = D / 8;
    const uint32_t row0 = (g.first + blockIdx.x) * g.row_tile;
    const uint32_t n = g.b.n_rows - row0 < g.row_tile ? g.b.n_rows - row0 : g.row_tile;
    find_rows(place, g.c, g.b, row0, n);
    __shared__ PagePlace pages[kMaxRowTile];
    if (threadIdx.x < n) {
        const PagePlace at = page_place(g.c, g.b, place[threadIdx.x]);
        if (at.page < 0 && place[threadIdx.x].live) kv_note(g.b.errors, TENT_KV_BAD_PAGE);
        pages[threadIdx.x] = at;
    }
    __syncthreads();
    const uint32_t one = g.c.heads * kChunks, all = 2 * n * one;         // chunks of K of a row, and of all there is
    for (uint32_t first = threadIdx.x; first < all; first += kBatch * 256) {
        u32x4 value[kBatch];                                             // 4 bits: the codes, the word that holds the scale, and where in it
        uint32_t where[kBatch];
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint32_t i = first + j * 256 < all ? first + j * 256 : first;
            const bool is_v = i >= n * one;
            const uint32_t x = is_v ? i - n * one : i, r = x / one, y = x - r * one, head = y / kChunks, chunk = y % kChunks;
            const PagePlace p = pages[r];
            where[j] = p.page >= 0 ? 2u : place[r].live ? 1u : 0u;
            const uint8_t* page = (is_v ? g.c.v : g.c.k) + (p.page >= 0 ? p.page : 0);
            const uint32_t slot = p.page >= 0 ? p.slot : 0u;             // of the first page, where there is none
            if constexpr (kBits == 16) {
                value[j] = dev_load<u32x4>(page + at16<D>(slot, g.c.heads, head, chunk));
            } else {
                value[j][0] = dev_load<uint32_t>(page + at_codes<D>(slot, g.c.heads, head, chunk));
                const uint32_t at = at_scale<D>(slot, g.c.heads, head, chunk, g.c.page_shift);
                value[j][1] = dev_load<uint32_t>(page + (at & ~3u));     // a byte's load would be waited for here, to extend it
                value[j][2] = 8 * (at & 3u);
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < kBatch; ++j) {
            const uint32_t i = first + j * 256;
            if (i >= all || where[j] == 0u) continue;
            const bool is_v = i >= n * one;
            const uint32_t x = is_v ? i - n * one : i, r = x / one, y = x - r * one;
            u32x4 out = value[j];
            if constexpr (kBits == 4) out = decode8<E>(value[j][0], scale_of(value[j][1] >> value[j][2] & 0xFFu));
            if (where[j] == 1u) out = u32x4{0, 0, 0, 0};
            dev_stream((is_v ? g.v : g.k) + (row0 + r) * g.stride + (uint64_t)y * 16, out);
        }
    }
}

struct PackArgs {
    KvCache src, dst;
    const int32_t *src_pages, *dst_pages;
    int32_t* errors;
    uint32_t n_pages, parts;   // workgroups for one page of one pool
    uint32_t first;            // of the launch's workgroups
};

// A workgroup takes four chunks a lane of one page of K or V, all four in flight at once.
constexpr uint32_t kPackChunks = 4;
template <class E, int D>
__global__ void __launch_bounds__(256) pack_kernel(const PackArgs g)
{
    constexpr uint32_t kChunks = D / 8;
    const uint32_t block = g.first + blockIdx.x, part = block % g.parts, at = block / g.parts;
    const bool is_v = at >= g.n_pages;
    const uint32_t i = is_v ? at - g.n_pages : at;
    const uint32_t from = (uint32_t)g.src_pages[i], to = (uint32_t)g.dst_pages[i];
    if (from >= g.src.n_pages || to >= g.dst.n_pages) {
        if (threadIdx.x == 0) kv_note(g.errors, TENT_KV_BAD_PAGE);
        return;
    }
    const uint8_t* src = (is_v ? g.src.v : g.src.k) + from * g.src.page_stride;
    uint8_t* dst = (is_v ? g.dst.v : g.dst.k) + to * g.dst.page_stride;
    const uint32_t n = (g.src.heads * kChunks) << g.src.page_shift;      // a multiple of the 8 lanes that share two blocks
    const uint32_t scales = ((g.src.heads * (D / 2)) << g.src.page_shift);
    const uint32_t first = part * blockDim.x * kPackChunks + threadIdx.x;
    u32x4 v[kPackChunks];
#pragma unroll
    for (uint32_t k = 0; k < kPackChunks; ++k) {
        const uint32_t x = first + k * blockDim.x;
        v[k] = x < n ? dev_load<u32x4>(src + (uint64_t)x * 16) : u32x4{0, 0, 0, 0};
    }
    // Four lanes share a block and have it for each k.  They exchange their codes so that lane j of them stores the 16 bytes of k = j.
    const uint32_t lane = threadIdx.x & 63u, j = lane & 3u;
    u32x4 codes;
    uint32_t scale = 0;
#pragma unroll
    for (uint32_t k = 0; k < kPackChunks; ++k) {
        uint32_t byte;
        codes[k] = encode8<E>(v[k], byte);
        scale = j == k ? byte : scale;
    }
    u32x4 mine;                                                          // mine[i]: codes of lane i of the four for k = j
#pragma unroll
    for (uint32_t d = 0; d < 4; ++d) {                                   // from lane j ^ d, which gives what it has for k = j
        const uint32_t k = j ^ d, give = k == 0 ? codes[0] : k == 1 ? codes[1] : k == 2 ? codes[2] : codes[3];
        const uint32_t got = d == 0   ? give
                             : d == 1 ? (uint32_t)__builtin_amdgcn_mov_dpp((int)give, 0xB1, 0xF, 0xF, true)
                             : d == 2 ? (uint32_t)__builtin_amdgcn_mov_dpp((int)give, 0x4E, 0xF, 0xF, true)
                                      : (uint32_t)__builtin_amdgcn_mov_dpp((int)give, 0x1B, 0xF, 0xF, true);
        mine[0] = k == 0 ? got : mine[0];
        mine[1] = k == 1 ? got : mine[1];
        mine[2] = k == 2 ? got : mine[2];
        mine[3] = k == 3 ? got : mine[3];
    }
    // and of 16 lanes, which have four blocks in a row for each k, lanes 0..3 store the scales of k = 0..3
    scale <<= 8 * (lane >> 2 & 3u);
    scale |= (uint32_t)__builtin_amdgcn_mov_dpp((int)scale, 0x124, 0xF, 0xF, true);      // lanes rotated by 4 within 16
    scale |= (uint32_t)__builtin_amdgcn_mov_dpp((int)scale, 0x128, 0xF, 0xF, true);      // by 8
    const uint32_t x = first - j + j * blockDim.x;                       // of the four lanes' first chunk for k = j
    if (x < n) dev_store(dst + (uint64_t)x * 4, mine);
    if ((lane & 12u) == 0) {
        if (x + 16 <= n) dev_store(dst + scales + x / 4, scale);         // a head of 64 values ends inside, a page may
        else
            for (uint32_t i = 0; x + 4 * i < n; ++i) dev_store(dst + scales + x / 4 + i, (uint8_t)(scale >> (8 * i)));
    }
}

template <class E, int D, int kBits>
int launch_append(AppendArgs g, hipStream_t s)
{
    g.per_row = (g.a.q_heads + 2 * g.c.heads) * (D / 8);
    g.side = g.per_row >= 256 ? 1 : 256 / g.per_row;                     // at most 16: a row has a key and a value of 64 at least
    const uint32_t turns = (g.per_row + 255) / 256, threads = g.side > 1 ? 256 : (g.per_row + turns * 64 - 1) / (turns * 64) * 64;
    return launch_blocks(((uint64_t)g.b.n_rows + g.side - 1) / g.side, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((append_kernel<E, D, kBits>), dim3(blocks, (uint64_t)g.b.n_rows * turns <= 512 ? turns : 1), dim3(threads), 0, s, g);
    });
}
// Rows of a workgroup: as many as its lanes take in one batch, fewer where that leaves compute units without one.
template <class E, int D, int kBits>
int launch_read(ReadArgs g, hipStream_t s)
{
    const uint32_t batch = kBatch * 256 / (2 * g.c.heads * (D / 8)), spread = g.b.n_rows / 1024;
    const uint32_t n = batch < spread ? batch : spread;
    g.row_tile = n < 1 ? 1 : n > kMaxRowTile ? kMaxRowTile : n;
    return launch_blocks(((uint64_t)g.b.n_rows + g.row_tile - 1) / g.row_tile, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((read_kernel<E, D, kBits>), dim3(blocks), dim3(256), 0, s, g);
    });
}
template <class E, int D>
int launch_pack(PackArgs g, hipStream_t s)
{
    const uint32_t n = (g.src.heads * (D / 8)) << g.src.page_shift;
    g.parts = (n + 256 * kPackChunks - 1) / (256 * kPackChunks);
    return launch_blocks((uint64_t)2 * g.n_pages * g.parts, [&](uint32_t first, uint32_t blocks) {
        g.first = first;
        hipLaunchKernelGGL((pack_kernel<E, D>), dim3(blocks), dim3(256), 0, s, g);
    });
}

}  // namespace
}  // namespace tent

using namespace tent;

#define TENT_KV_DIM(dim, call) ((dim) == 64 ? call(64) : (dim) == 128 ? call(128) : call(256))

extern "C" uint64_t tent_kv_packed_page(uint32_t page_tokens, uint32_t kv_heads, uint32_t head_dim)
{
    if (!kv_sizes_ok(page_tokens, kv_heads, head_dim)) return 0;
    return (kv_page_bytes(page_tokens, kv_heads, head_dim, 4) + 15) / 16 * 16;
}

extern "C" int tent_kv_append(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_append_args* args, void* stream)
{
    int rc = kv_check_cache(cache);
    if (rc == TENT_OK) rc = kv_check_batch(cache, batch);
    if (rc != TENT_OK) return rc;
    if (!args || args->reserved || (args->flags & ~(uint32_t)TENT_KV_ROPE_PAIRS)) return TENT_ERR_INVALID;
    if (batch->n_seqs == 0 || batch->n_rows == 0) return TENT_OK;
    const uint32_t D = cache->head_dim, n = batch->n_rows;
    if ((rc = kv_check_rows(args->k, args->k_stride, cache->kv_heads, D, n)) != TENT_OK) return rc;
    if ((rc = kv_check_rows(args->v, args->v_stride, cache->kv_heads, D, n)) != TENT_OK) return rc;
    if (args->q_heads > TENT_KV_MAX_HEADS) return TENT_ERR_RANGE;
    if (args->q_heads) {
        if ((rc = kv_check_rows(args->q, args->q_stride, args->q_heads, D, n)) != TENT_OK) return rc;
        if ((rc = kv_check_rows(args->q_out, args->q_out_stride, args->q_heads, D, n)) != TENT_OK) return rc;
        if (args->q == args->q_out && args->q_stride != args->q_out_stride) return TENT_ERR_INVALID;
    }
    if (!kv_aligned(args->q_weight) || !kv_aligned(args->k_weight) || !kv_aligned(args->rope)) return TENT_ERR_INVALID;
    if (!(args->eps >= 0.f) || args->eps > 3.4e38f) return TENT_ERR_RANGE;
    if (args->rope && (args->rope_rows < 1 || args->rope_dim < 16 || args->rope_dim > D || args->rope_dim % 16)) return TENT_ERR_RANGE;
    if ((uintptr_t)args->positions & 3u) return TENT_ERR_INVALID;
    const AppendArgs g{*args, kv_cache_dev(*cache), *batch, 0, 0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_APPEND(dim)                                                                                   \
    (cache->type == TENT_BF16 ? (cache->bits == 16 ? launch_append<Bf16, dim, 16>(g, s) : launch_append<Bf16, dim, 4>(g, s)) \
                              : (cache->bits == 16 ? launch_append<Fp16, dim, 16>(g, s) : launch_append<Fp16, dim, 4>(g, s)))
    return TENT_KV_DIM(D, TENT_APPEND);
}

extern "C" int tent_kv_read(const tent_kv_cache* cache, const tent_kv_batch* batch, void* k_out, void* v_out, uint64_t out_stride,
                            void* stream)
{
    int rc = kv_check_cache(cache);
    if (rc == TENT_OK) rc = kv_check_batch(cache, batch);
    if (rc != TENT_OK) return rc;
    if (batch->n_seqs == 0 || batch->n_rows == 0) return TENT_OK;
    if ((rc = kv_check_rows(k_out, out_stride, cache->kv_heads, cache->head_dim, batch->n_rows)) != TENT_OK) return rc;
    if ((rc = kv_check_rows(v_out, out_stride, cache->kv_heads, cache->head_dim, batch->n_rows)) != TENT_OK) return rc;
    const ReadArgs g{kv_cache_dev(*cache), *batch, static_cast<uint8_t*>(k_out), static_cast<uint8_t*>(v_out), out_stride * 2, 0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_READ(dim)                                                                                     \
    (cache->type == TENT_BF16 ? (cache->bits == 16 ? launch_read<Bf16, dim, 16>(g, s) : launch_read<Bf16, dim, 4>(g, s)) \
                              : (cache->bits == 16 ? launch_read<Fp16, dim, 16>(g, s) : launch_read<Fp16, dim, 4>(g, s)))
    return TENT_KV_DIM(cache->head_dim, TENT_READ);
}

extern "C" int tent_kv_pack(const tent_kv_cache* src, const tent_kv_cache* dst, const int32_t* src_pages, const int32_t* dst_pages,
                            uint32_t n_pages, int32_t* errors, void* stream)
{
    int rc = kv_check_cache(src);
    if (rc == TENT_OK) rc = kv_check_cache(dst);
    if (rc != TENT_OK) return rc;
    if (src->bits != 16 || dst->bits != 4) return TENT_ERR_INVALID;
    if (src->page_tokens != dst->page_tokens || src->kv_heads != dst->kv_heads || src->head_dim != dst->head_dim || src->type != dst->type) return TENT_ERR_RANGE;
    if (n_pages == 0) return TENT_OK;
    if (!src_pages || !dst_pages || (((uintptr_t)src_pages | (uintptr_t)dst_pages | (uintptr_t)errors) & 3u)) return TENT_ERR_INVALID;
    if (n_pages > 0x7FFFFFFFu) return TENT_ERR_RANGE;
    const PackArgs g{kv_cache_dev(*src), kv_cache_dev(*dst), src_pages, dst_pages, errors, n_pages, 0, 0};
    hipStream_t s = static_cast<hipStream_t>(stream);
#define TENT_PACK(dim) (src->type == TENT_BF16 ? launch_pack<Bf16, dim>(g, s) : launch_pack<Fp16, dim>(g, s))
    return TENT_KV_DIM(src->head_dim, TENT_PACK);
}
