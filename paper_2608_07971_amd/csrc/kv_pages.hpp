// Shared by the operations on pages (kv_pages.hip, kv_evict.hip): free pages and
// table entries in bit masks, ranks among them, and the workspace.
#pragma once

#include "kv_internal.hpp"

#include <type_traits>

namespace esp_kv {

constexpr int kThreads = 256;
constexpr int kCopyThreads = 256;
constexpr int kMaxBlocks = 1024;            // blocks of pages, and of entries: added up by every workgroup

// Pages or table entries [0, n) in at most kMaxBlocks blocks of `words` mask words.
struct Blocks {
    int64_t n;
    int32_t words, blocks;
    static Blocks of(int64_t n, int least) {
        const int64_t all = (n + 63) / 64, per = (all + kMaxBlocks - 1) / kMaxBlocks;
        Blocks b{n, int32_t(per > least ? per : least), 0};
        b.blocks = int32_t((all + b.words - 1) / b.words);
        return b;
    }
};

struct Work {
    Blocks pages, entries;
    uint64_t *page_mask;                    // free (or, compact: live) pages
    uint64_t *need_mask, *split_mask;       // entries that take a page; of these, entries that copy one
    int32_t *page_sum, *need_sum, *split_sum, *bad;
    int32_t *count;                         // copies to make
    int2 *copies;                           // from, to
    int32_t *goes;                          // [pages] new places
    int32_t *rows, *row_lengths;            // a table and lengths aside: [sequences][width], [sequences]
    int32_t *cut;                           // [sequences] those that an eviction cuts
    bool at_once;                           // pages are copied by the workgroup that finds them
};

__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

// Bit `at` of a mask, by shifts of 32 bits.
__device__ __forceinline__ bool bit_of(uint64_t mask, int at) { return uint32_t(at & 32 ? mask >> 32 : mask) >> (at & 31) & 1; }

// Sum of x over the workgroup.
__device__ __forceinline__ int block_sum(int x, int *lds) {
#pragma unroll
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// Exclusive prefix of n <= kMaxBlocks values into at[0 .. n], all threads.
__device__ __forceinline__ void prefix(const int32_t *values, int n, int *at, int *lds) {
    int x[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int i = threadIdx.x * 4 + k;
        x[k] = i < n ? values[i] : 0;
    }
#pragma unroll
    for (int k = 0; k < 4; k++) sum += x[k];
    int before = sum;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int v = __shfl_up(before, m);
        before += int(threadIdx.x & 63) >= m ? v : 0;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = before;
    __syncthreads();
    before -= sum;
    for (int w = 0; w < int(threadIdx.x >> 6); w++) before += lds[w];
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int i = threadIdx.x * 4 + k;
        if (i <= n) at[i] = before;
        before += x[k];
    }
    if (threadIdx.x == kThreads - 1 && n == kMaxBlocks) at[n] = before;
    __syncthreads();
}

// Place of the set bit that r others precede.
__device__ __forceinline__ int nth_bit(uint64_t mask, int r) {
    uint32_t m = uint32_t(mask);
    const int low = __popc(m);
    int at = 0;
    if (r >= low) {
        r -= low;
        at = 32;
        m = uint32_t(mask >> 32);
    }
#pragma unroll
    for (int w = 16; w; w >>= 1) {
        const int below = __popc(m & ((1u << w) - 1));
        const bool past = r >= below;
        r -= past ? below : 0;
        at += past ? w : 0;
        m >>= past ? w : 0;
    }
    return at;
}

// The page of rank r among those whose bit is set (flip 0) or clear (flip ~0);
// at(b): how many there are before block b.
template <typename At> __device__ int select(const Work &w, At at, uint64_t flip, int r) {
    int lo = 0, hi = w.pages.blocks - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (at(mid) <= r) lo = mid;
        else hi = mid - 1;
    }
    r -= at(lo);
    const int64_t words = (w.pages.n + 63) / 64, from = int64_t(lo) * w.pages.words;
    for (int x = 0; x < w.pages.words; x += 4) {
        uint64_t m[4];
#pragma unroll
        for (int k = 0; k < 4; k++) m[k] = x + k < w.pages.words && from + x + k < words ? w.page_mask[from + x + k] ^ flip : 0;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int held = __popcll(m[k]);
            if (r < held) return int((from + x + k) * 64 + nth_bit(m[k], r));
            r -= held;
        }
    }
    return -1;
}

// A workgroup copies a page: keys, values and scales of all layers.
__device__ __forceinline__ void copy_page(const Cache &c, int32_t from, int32_t to) {
    const int64_t vectors = int64_t(c.layers) * c.heads * c.tokens * c.dim / 16;
    const int scales = c.layers * 2 * c.heads;
#pragma unroll
    for (int side = 0; side < 2; side++) {
        uint4v *pool = reinterpret_cast<uint4v *>(side ? c.v : c.k);
        for (int64_t at = threadIdx.x; at < vectors; at += kThreads * 4) {
            uint4v x[4];
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (at + j * kThreads < vectors) x[j] = pool[from * vectors + at + j * kThreads];
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (at + j * kThreads < vectors) pool[to * vectors + at + j * kThreads] = x[j];
        }
    }
    for (int i = threadIdx.x; i < scales; i += kThreads) c.scale[int64_t(to) * scales + i] = c.scale[int64_t(from) * scales + i];
}

// Marks the items of block `block` that `has` holds for: four wavefronts, a word each at a time.
template <typename Has> __device__ __forceinline__ void mark(const Blocks &b, int block, uint64_t *mask, int32_t *sum, int *lds, Has has) {
    const int64_t words = (b.n + 63) / 64, from = int64_t(block) * b.words, to = min(words, from + b.words);
    int mine = 0;
    for (int64_t x = from + (threadIdx.x >> 6); x < to; x += 4) {
        const int64_t i = x * 64 + (threadIdx.x & 63);
        const uint64_t m = __ballot(i < b.n && has(i));
        if ((threadIdx.x & 63) == 0) {
            mask[x] = m;
            mine += __popcll(m);
        }
    }
    mine = block_sum(mine, lds);
    if (threadIdx.x == 0) sum[block] = mine;
}

// Calls use(i, held, rank, held2, rank2) for every item of a block: whether its
// bit is set in each of two masks, and how many set bits come before it, from
// `before` and `before2` at the block's start.
template <typename Use>
__device__ __forceinline__ void ranked(const Blocks &b, int block, const uint64_t *mask, int before, const uint64_t *mask2, int before2, Use use) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t words = (b.n + 63) / 64, from = int64_t(block) * b.words, to = min(words, from + b.words);
    for (int64_t x0 = from; x0 < to; x0 += 64) {                 // a word a lane
        const uint64_t m = x0 + lane < to ? mask[x0 + lane] : 0, m2 = x0 + lane < to ? mask2[x0 + lane] : 0;
        int at = __popcll(m), at2 = __popcll(m2);
        const int own = at, own2 = at2;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int v = __shfl_up(at, s), v2 = __shfl_up(at2, s);
            at += lane >= s ? v : 0;
            at2 += lane >= s ? v2 : 0;
        }
        for (int x = wave; x < 64 && x0 + x < to; x += 4) {      // an item a lane
            const uint64_t n = __shfl(m, x), n2 = __shfl(m2, x);
            const int r = before + __shfl(at - own, x), r2 = before2 + __shfl(at2 - own2, x);
            const int64_t i = (x0 + x) * 64 + lane;
            if (i < b.n) use(i, bit_of(n, lane), r + lanes_below(n), bit_of(n2, lane), r2 + lanes_below(n2));
        }
        before += __shfl(at, 63);
        before2 += __shfl(at2, 63);
    }
}

// Lays the work out behind `p`; returns its bytes.
inline size_t lay_out(const esp_kv_cache *c, char *p, Work &w) {
    w.pages = Blocks::of(c->pages, 4);
    w.entries = Blocks::of(int64_t(c->sequences) * c->table_width, 16);
    char *at = p;
    auto take = [&](auto *&to, size_t n) {
        to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(at);
        at += (n * sizeof(*to) + 255) / 256 * 256;
    };
    take(w.count, 1);
    take(w.page_mask, (size_t(w.pages.n) + 63) / 64);
    take(w.need_mask, (size_t(w.entries.n) + 63) / 64);
    take(w.split_mask, (size_t(w.entries.n) + 63) / 64);
    take(w.page_sum, kMaxBlocks);
    take(w.need_sum, kMaxBlocks);
    take(w.split_sum, kMaxBlocks);
    take(w.bad, size_t(c->sequences) > size_t(kMaxBlocks) ? size_t(c->sequences) : size_t(kMaxBlocks));
    take(w.copies, size_t(c->pages));
    take(w.goes, size_t(c->pages));
    take(w.rows, size_t(w.entries.n));
    take(w.row_lengths, size_t(c->sequences));
    take(w.cut, size_t(c->sequences));
    w.at_once = false;
    return size_t(at - p);
}
inline esp_status work_of(const esp_kv_cache *c, void *workspace, size_t bytes, Work &w) {
    const size_t need = lay_out(c, static_cast<char *>(workspace), w);
    return workspace && (reinterpret_cast<uintptr_t>(workspace) & 255) == 0 && bytes >= need ? ESP_OK : ESP_ERR_WORKSPACE;
}

}  // namespace esp_kv
