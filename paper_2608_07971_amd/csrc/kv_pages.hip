// Page operations of the paged 8-bit cache: resize, fork, reorder, compact.
//
// All choices are by index (the lowest free page, in order of sequence and
// slot), so results do not depend on the order of atomics.  An operation is
// three short launches over many workgroups that settle the integers and one
// that copies the pages on the list they left:
//   1  references of dropped pages go down; what is wrong is noted
//   2  free pages and entries that need one are marked in bit masks and counted
//      by blocks
//   3  every workgroup adds up the blocks before its own, so that it knows the
//      rank of its entries and finds the page of a rank by a binary search over
//      the blocks and the bits of one; or, where something is wrong or pages do
//      not suffice, takes step 1 back
// (One workgroup doing all of it took 170 us for 256 sequences of up to 256
// pages in a pool of 65,536; the launches of a step 3-5 us each.)
#include "kv_pages.hpp"

namespace esp_kv {

// ---------------------------------------------------------------------------
// Resize: table entries by blocks
// ---------------------------------------------------------------------------

struct Entry {
    int seq, slot;
    bool wanted;
};
__device__ __forceinline__ Entry entry_of(const Cache &c, const int32_t *lengths, int64_t i) {
    const int seq = int(uint32_t(i) / uint32_t(c.width)), slot = int(uint32_t(i) - uint32_t(seq) * uint32_t(c.width));
    return {seq, slot, slot < (lengths[seq] + c.tokens - 1) >> c.shift};
}
// Calls f(i) for the entries of a block.
template <typename F> __device__ __forceinline__ void each(const Blocks &b, int block, F f) {
    const int64_t from = int64_t(block) * b.words * 64, to = min(b.n, from + int64_t(b.words) * 64);
    for (int64_t i = from + threadIdx.x; i < to; i += kThreads) f(i);
}

__global__ __launch_bounds__(kThreads) void k_resize_drop(Cache c, const int32_t *lengths, Work w) {
    __shared__ int lds[4];
    int bad = 0;
    each(w.entries, blockIdx.x, [&](int64_t i) {
        const Entry e = entry_of(c, lengths, i);
        const int32_t p = c.table[i];
        bad |= lengths[e.seq] < 0 || lengths[e.seq] > int64_t(c.width) << c.shift || p < -1 || p >= c.pages;
        if (p >= 0 && p < c.pages && !e.wanted) atomicAdd(c.refs + p, -1);
    });
    bad = block_sum(bad, lds);
    if (threadIdx.x == 0) w.bad[blockIdx.x] = bad;
}

// Workgroups [0, entries.blocks): entries; the rest: pages.
__global__ __launch_bounds__(kThreads) void k_resize_mark(Cache c, const int32_t *lengths, Work w) {
    __shared__ int lds[4];
    const int b = blockIdx.x;
    if (b >= w.entries.blocks) {
        mark(w.pages, b - w.entries.blocks, w.page_mask, w.page_sum, lds, [&](int64_t p) { return c.refs[p] == 0; });
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t words = (w.entries.n + 63) / 64, from = int64_t(b) * w.entries.words, to = min(words, from + w.entries.words);
    int needs = 0, splits = 0;
    for (int64_t x0 = from + wave; x0 < to; x0 += 16) {          // four words in flight
        int32_t page[4];
#pragma unroll
        for (int k = 0; k < 4; k++) page[k] = x0 + 4 * k < to ? c.table[min((x0 + 4 * k) * 64 + lane, w.entries.n - 1)] : -1;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int64_t x = x0 + 4 * k, i = x * 64 + lane;
            bool need = false, split = false;
            if (x < to && i < w.entries.n) {
                const Entry e = entry_of(c, lengths, i);
                const int last = min(c.lengths[e.seq], lengths[e.seq]);
                // a kept page that ends inside its sequence and still has other owners
                split = e.wanted && page[k] >= 0 && page[k] < c.pages && e.slot == last >> c.shift && (last & (c.tokens - 1)) && c.refs[page[k]] > 1;
                need = split || (e.wanted && page[k] == -1);
            }
            const uint64_t n = __ballot(need), s = __ballot(split);
            if (x < to && lane == 0) {
                w.need_mask[x] = n;
                w.split_mask[x] = s;
            }
            needs += lane == 0 ? __popcll(n) : 0;
            splits += lane == 0 ? __popcll(s) : 0;
        }
    }
    needs = block_sum(needs, lds);
    splits = block_sum(splits, lds);
    if (threadIdx.x == 0) {
        w.need_sum[b] = needs;
        w.split_sum[b] = splits;
    }
}

__global__ __launch_bounds__(kThreads) void k_resize_take(Cache c, const int32_t *lengths, Work w) {
    __shared__ int lds[4], free_at[kMaxBlocks + 1], need_at[kMaxBlocks + 1], split_at[kMaxBlocks + 1];
    int bad = 0;
    for (int b = threadIdx.x; b < w.entries.blocks; b += kThreads) bad |= w.bad[b];
    bad = block_sum(bad, lds);
    prefix(w.page_sum, w.pages.blocks, free_at, lds);
    prefix(w.need_sum, w.entries.blocks, need_at, lds);
    prefix(w.split_sum, w.entries.blocks, split_at, lds);
    const bool short_of = free_at[w.pages.blocks] < need_at[w.entries.blocks];
    if (bad || short_of) {
        each(w.entries, blockIdx.x, [&](int64_t i) {
            const int32_t p = c.table[i];
            if (p >= 0 && p < c.pages && !entry_of(c, lengths, i).wanted) atomicAdd(c.refs + p, 1);
        });
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            *w.count = 0;
            record(c, bad ? ESP_ERR_SHAPE : ESP_ERR_RANGE);
        }
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.count = split_at[w.entries.blocks];
    ranked(w.entries, blockIdx.x, w.need_mask, need_at[blockIdx.x], w.split_mask, split_at[blockIdx.x], [&](int64_t i, bool need, int rank, bool split, int copy) {
        const Entry e = entry_of(c, lengths, i);
        const int32_t p = c.table[i];
        const int to = need ? select(w, [&](int b) { return free_at[b]; }, 0, rank) : -1;
        if (to >= 0) {
            if (split) {
                w.copies[copy] = make_int2(p, to);
                atomicAdd(c.refs + p, -1);
            }
            c.refs[to] = 1;
            c.table[i] = to;
        } else if (!e.wanted && p >= 0) {
            c.table[i] = -1;
        }
        if (e.slot == 0) c.lengths[e.seq] = lengths[e.seq];
    });
    if (w.at_once && split_at[blockIdx.x] < split_at[blockIdx.x + 1]) {
        __syncthreads();
        for (int i = split_at[blockIdx.x]; i < split_at[blockIdx.x + 1]; i++) copy_page(c, w.copies[i].x, w.copies[i].y);
    }
}

// ---------------------------------------------------------------------------
// Fork: a workgroup a child
// ---------------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void k_fork_drop(Cache c, int n, const int32_t *parents, const int32_t *children, Work w) {
    __shared__ int lds[4];
    const int i = blockIdx.x, parent = parents[i], child = children[i];
    const bool there = parent >= 0 && parent < c.sequences && child >= 0 && child < c.sequences;
    int bad = 0;
    for (int j = threadIdx.x; j < n; j += kThreads) bad |= parents[j] == child || (j != i && children[j] == child);
    bad = block_sum(bad, lds) || !there;
    int wrong = 0;
    if (there) {
        const int length = c.lengths[parent];
        wrong = length < 0 || length > int64_t(c.width) << c.shift;
        if (!wrong && (length & (c.tokens - 1))) wrong |= c.table[int64_t(parent) * c.width + (length >> c.shift)] < 0;
        for (int x = threadIdx.x; x < c.width; x += kThreads) {
            const int32_t p = c.table[int64_t(parent) * c.width + x], k = c.table[int64_t(child) * c.width + x];
            wrong |= p < -1 || p >= c.pages || k < -1 || k >= c.pages;
            if (k >= 0 && k < c.pages) atomicAdd(c.refs + k, -1);
        }
    }
    wrong = block_sum(wrong, lds);
    if (threadIdx.x == 0) w.bad[i] = (bad ? 1 : 0) | (wrong ? 2 : 0);
}

__global__ __launch_bounds__(kThreads) void k_mark_free(Cache c, Work w) {
    __shared__ int lds[4];
    mark(w.pages, blockIdx.x, w.page_mask, w.page_sum, lds, [&](int64_t p) { return c.refs[p] == 0; });
}

__global__ __launch_bounds__(kThreads) void k_fork_take(Cache c, int n, const int32_t *parents, const int32_t *children, Work w) {
    __shared__ int lds[4], free_at[kMaxBlocks + 1];
    const int i = blockIdx.x, parent = parents[i], child = children[i];
    auto parted = [&](int j) { return parents[j] >= 0 && parents[j] < c.sequences && (c.lengths[parents[j]] & (c.tokens - 1)) != 0; };
    int invalid = 0, wrong = 0, need = 0, rank = 0;
    for (int j = threadIdx.x; j < n; j += kThreads) {
        const int one = parted(j);
        invalid |= w.bad[j] & 1;
        wrong |= w.bad[j] >> 1;
        need += one;
        rank += j < i ? one : 0;
    }
    invalid = block_sum(invalid, lds);
    wrong = block_sum(wrong, lds);
    need = block_sum(need, lds);
    rank = block_sum(rank, lds);
    prefix(w.page_sum, w.pages.blocks, free_at, lds);
    if (invalid || wrong || free_at[w.pages.blocks] < need) {
        if (parent >= 0 && parent < c.sequences && child >= 0 && child < c.sequences)
            for (int x = threadIdx.x; x < c.width; x += kThreads) {
                const int32_t k = c.table[int64_t(child) * c.width + x];
                if (k >= 0 && k < c.pages) atomicAdd(c.refs + k, 1);
            }
        if (i == 0 && threadIdx.x == 0) {
            *w.count = 0;
            record(c, invalid ? ESP_ERR_INVALID_ARG : wrong ? ESP_ERR_SHAPE : ESP_ERR_RANGE);
        }
        return;
    }
    const int length = c.lengths[parent], part = parted(i) ? length >> c.shift : -1;
    if (threadIdx.x == 0) lds[0] = lds[1] = -1;
    __syncthreads();
    for (int x = threadIdx.x; x < c.width; x += kThreads) {
        int32_t p = c.table[int64_t(parent) * c.width + x];
        if (x == part) {                    // filled only in part: copied
            const int to = select(w, [&](int b) { return free_at[b]; }, 0, rank);
            if (to >= 0) {
                w.copies[rank] = make_int2(p, to);
                c.refs[to] = 1;
                lds[0] = p;
                lds[1] = to;
            }
            p = to;
        } else if (p >= 0) {
            atomicAdd(c.refs + p, 1);
        }
        c.table[int64_t(child) * c.width + x] = p;
    }
    if (threadIdx.x == 0) c.lengths[child] = length;
    if (i == 0 && threadIdx.x == 0) *w.count = need;
    if (!w.at_once) return;
    __syncthreads();
    if (lds[1] >= 0) copy_page(c, lds[0], lds[1]);
}

// ---------------------------------------------------------------------------
// Reorder: a workgroup a sequence; every row is put together aside before any is written.
// Three launches: 256 beams of up to 157 pages of 64 KB, some 110 of them copied, 5.7 + 2.4 + 9
// us; 4 beams 3.5 + 1.7 + 4.5 us.
// ---------------------------------------------------------------------------

constexpr int kInvalid = 1, kWrong = 2, kCopies = 4;

__global__ __launch_bounds__(kThreads) void k_reorder_drop(Cache c, const int32_t *parents, Work w) {
    __shared__ int lds[4];
    const int i = blockIdx.x, parent = parents[i];
    const bool there = parent >= 0 && parent < c.sequences;
    // the partly filled page stays with the parent itself, or else with the first that goes on with it
    int earlier = 0;
    for (int j = threadIdx.x; j < i; j += kThreads) earlier |= parents[j] == parent;
    earlier = block_sum(earlier, lds);
    int wrong = 0, length = 0, part = -1;
    bool copies = false;
    if (there) {
        length = c.lengths[parent];
        wrong = length < 0 || length > int64_t(c.width) << c.shift;
        if (!wrong && (length & (c.tokens - 1))) {
            part = length >> c.shift;
            wrong |= c.table[int64_t(parent) * c.width + part] < 0;
            copies = parents[parent] == parent ? parent != i : earlier != 0;
        }
    }
    for (int x = threadIdx.x; x < c.width; x += kThreads) {
        const int32_t p = there ? c.table[int64_t(parent) * c.width + x] : -1, k = c.table[int64_t(i) * c.width + x];
        const bool ok = p >= -1 && p < c.pages;
        wrong |= !ok || k < -1 || k >= c.pages;
        if (k >= 0 && k < c.pages) atomicAdd(c.refs + k, -1);
        if (p >= 0 && ok && !(copies && x == part)) atomicAdd(c.refs + p, 1);
        w.rows[int64_t(i) * c.width + x] = ok ? p : -1;
    }
    wrong = block_sum(wrong, lds);
    if (threadIdx.x == 0) {
        w.row_lengths[i] = length;
        w.bad[i] = (parent < -1 || parent >= c.sequences ? kInvalid : 0) | (wrong ? kWrong : 0) | (copies ? kCopies : 0);
    }
}

__global__ __launch_bounds__(kThreads) void k_reorder_take(Cache c, Work w) {
    __shared__ int lds[4], free_at[kMaxBlocks + 1];
    const int i = blockIdx.x;
    int invalid = 0, wrong = 0, need = 0, rank = 0;
    for (int j = threadIdx.x; j < c.sequences; j += kThreads) {
        const int b = w.bad[j], one = b / kCopies;
        invalid |= b & kInvalid;
        wrong |= b & kWrong;
        need += one;
        rank += j < i ? one : 0;
    }
    invalid = block_sum(invalid, lds);
    wrong = block_sum(wrong, lds);
    need = block_sum(need, lds);
    rank = block_sum(rank, lds);
    prefix(w.page_sum, w.pages.blocks, free_at, lds);
    const int length = w.row_lengths[i], part = w.bad[i] & kCopies ? length >> c.shift : -1;
    if (invalid || wrong || free_at[w.pages.blocks] < need) {
        for (int x = threadIdx.x; x < c.width; x += kThreads) {
            const int32_t p = w.rows[int64_t(i) * c.width + x], k = c.table[int64_t(i) * c.width + x];
            if (p >= 0 && x != part) atomicAdd(c.refs + p, -1);
            if (k >= 0 && k < c.pages) atomicAdd(c.refs + k, 1);
        }
        if (i == 0 && threadIdx.x == 0) {
            *w.count = 0;
            record(c, invalid ? ESP_ERR_INVALID_ARG : wrong ? ESP_ERR_SHAPE : ESP_ERR_RANGE);
        }
        return;
    }
    if (threadIdx.x == 0) lds[0] = lds[1] = -1;
    __syncthreads();
    for (int x = threadIdx.x; x < c.width; x += kThreads) {
        int32_t p = w.rows[int64_t(i) * c.width + x];
        if (x == part) {
            const int to = select(w, [&](int b) { return free_at[b]; }, 0, rank);
            if (to >= 0) {
                w.copies[rank] = make_int2(p, to);
                c.refs[to] = 1;
                lds[0] = p;
                lds[1] = to;
            }
            p = to;
        }
        c.table[int64_t(i) * c.width + x] = p;
    }
    if (threadIdx.x == 0) c.lengths[i] = length;
    if (i == 0 && threadIdx.x == 0) *w.count = need;
    if (!w.at_once) return;
    __syncthreads();
    if (lds[1] >= 0) copy_page(c, lds[0], lds[1]);
}

// ---------------------------------------------------------------------------
// Compact
// ---------------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void k_compact_mark(Cache c, int32_t *refs_out, Work w) {
    __shared__ int lds[4];
    mark(w.pages, blockIdx.x, w.page_mask, w.page_sum, lds, [&](int64_t p) {
        const int32_t r = c.refs[p];
        w.goes[p] = int32_t(p);
        refs_out[p] = r;
        return r > 0;
    });
}

__global__ __launch_bounds__(kThreads) void k_compact_place(Cache c, int limit, int32_t *refs_out, int32_t *live_out, Work w) {
    __shared__ int lds[4], live_at[kMaxBlocks + 1];
    prefix(w.page_sum, w.pages.blocks, live_at, lds);
    const int live = live_at[w.pages.blocks], per = w.pages.words * 64;
    limit = min(limit < 0 ? live : limit, c.pages);
    // live pages below the limit
    int below = 0;
    if (limit < c.pages) {
        const int b = limit / per;
        for (int64_t x = int64_t(b) * w.pages.words + threadIdx.x; x * 64 < limit; x += kThreads) {
            const uint64_t m = w.page_mask[x];
            below += __popcll(limit - x * 64 >= 64 ? m : m & ((uint64_t(1) << (limit - x * 64)) - 1));
        }
        below = block_sum(below, lds) + live_at[b];
    } else {
        below = live;
    }
    const bool fits = live <= limit;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (live_out) *live_out = live;
        *w.count = fits ? live - below : 0;
        if (!fits) record(c, ESP_ERR_RANGE);
    }
    if (!fits) return;
    ranked(w.pages, blockIdx.x, w.page_mask, live_at[blockIdx.x], w.page_mask, 0, [&](int64_t p, bool is_live, int rank, bool, int) {
        if (!is_live || p < limit) return;
        const int hole = select(w, [&](int b) { return b * per - live_at[b]; }, ~uint64_t(0), rank - below);
        if (hole < 0) return;
        w.copies[rank - below] = make_int2(int(p), hole);
        w.goes[p] = hole;
        refs_out[hole] = c.refs[p];
        refs_out[p] = 0;
    });
}

// Copies the listed pages (keys, values and scales of all layers): 16 KB of a
// page a turn.  Sources and targets are disjoint.  With `goes`: the table
// rewritten to the new places.
__global__ __launch_bounds__(kCopyThreads) void k_copy(Cache c, const int32_t *count, const int2 *copies, const int32_t *goes,
                                                       int32_t *table_out) {
    constexpr int kTurn = kCopyThreads * 4;
    const int64_t vectors = int64_t(c.layers) * c.heads * c.tokens * c.dim / 16;
    const int64_t turns = (vectors + kTurn - 1) / kTurn;
    const int scales = c.layers * 2 * c.heads;
    const int64_t total = *count * 2 * turns;
    for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
        const int64_t pair = u / (2 * turns), rest = u - pair * 2 * turns;
        const int2 m = copies[pair];
        const bool values = rest >= turns;
        uint4v *pool = reinterpret_cast<uint4v *>(values ? c.v : c.k);
        const uint4v *from = pool + m.x * vectors;
        uint4v *to = pool + m.y * vectors;
        const int64_t at = (values ? rest - turns : rest) * kTurn + threadIdx.x;
        uint4v x[4];
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (at + j * kCopyThreads < vectors) x[j] = __builtin_nontemporal_load(from + at + j * kCopyThreads);
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (at + j * kCopyThreads < vectors) __builtin_nontemporal_store(x[j], to + at + j * kCopyThreads);
        if (rest == 0)
            for (int i = threadIdx.x; i < scales; i += kCopyThreads) c.scale[int64_t(m.y) * scales + i] = c.scale[int64_t(m.x) * scales + i];
    }
    if (goes) {
        const int64_t entries = int64_t(c.sequences) * c.width;
        for (int64_t i = int64_t(blockIdx.x) * kCopyThreads + threadIdx.x; i < entries; i += int64_t(gridDim.x) * kCopyThreads) {
            const int32_t p = c.table[i];
            table_out[i] = p >= 0 && p < c.pages ? goes[p] : p;
        }
    }
}

Cache cache_of(const esp_kv_cache *c) {
    Cache o{c->pages, c->layers, c->kv_heads, c->page_tokens, c->head_dim, c->sequences, c->table_width, 0, static_cast<uint8_t *>(c->k),
            static_cast<uint8_t *>(c->v), c->scale, c->table, c->lengths, c->refs, c->status};
    while (1 << o.shift < o.tokens) o.shift++;
    return o;
}

esp_status check_cache(const esp_kv_cache *c) {
    if (!c || !c->k || !c->v || !c->scale || !c->table || !c->lengths || !c->refs || !c->status) return ESP_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15) return ESP_ERR_INVALID_ARG;
    const bool page = c->page_tokens == 16 || c->page_tokens == 32 || c->page_tokens == 64;
    const bool dim = c->head_dim == 64 || c->head_dim == 128;
    if (!page || !dim || c->pages < 1 || c->layers < 1 || c->kv_heads < 1 || c->sequences < 1 || c->table_width < 1) return ESP_ERR_SHAPE;
    if (c->kv_heads > 65536 || c->layers > 65536 || int64_t(c->table_width) * c->page_tokens > INT32_MAX ||
        int64_t(c->sequences) * c->table_width > INT32_MAX || int64_t(c->layers) * c->kv_heads * c->page_tokens * c->head_dim > INT32_MAX)
        return ESP_ERR_SHAPE;
    return ESP_OK;
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

// Bytes of a page up to which fork copies it within its last step, a workgroup a page:
// a fork of one child of 32 / 128 / 256 KB pages takes 10.4 / 12.3 / 15.0 us so, 12.5 /
// 13.7 / 13.9 us with a launch of its own for the copies.
constexpr int64_t kAtOnce = 128 << 10;
// A workgroup of resize's last step has the entries of many sequences, each of which may
// need a copy.  It makes them, one after another, only if there can be no more than these
// and no more bytes.  So / with a launch of its own, 2 KB pages: no or one copy 15.8 /
// 17.1 us, 4 copies 21.5 / 21.1, 16 copies 28.5 / 21.0, 64 copies 57.5 / 23.1; 32 KB pages:
// 4 copies 24.0 / 22.0, 16 copies 36.0 / 21.4; 1,024 copies of 128 KB by four workgroups
// 845 / 70.
constexpr int64_t kResizeCopies = 16, kResizeBytes = 64 << 10;

constexpr int32_t kMostSequences = (1 << 24) - 1;                              // a launch's threads are numbered in 32 bits
int64_t page_bytes(const esp_kv_cache *c) { return 2 * int64_t(c->layers) * c->kv_heads * c->page_tokens * c->head_dim; }
// Copies that one workgroup of resize may have to make: one a sequence of its entries.
int64_t copies_of(const esp_kv_cache *c, const Work &w) {
    const int64_t sequences = (int64_t(w.entries.words) * 64 + c->table_width - 2) / c->table_width + 1;
    return sequences < c->sequences ? sequences : c->sequences;
}
// Workgroups of the copy for at most `most` pages: 2,048 fill the GPU.
unsigned copy_blocks(const esp_kv_cache *c, int64_t most) {
    const int64_t blocks = most * 2 * ((page_bytes(c) / 2 + kCopyThreads * 64 - 1) / (kCopyThreads * 64));
    return unsigned(blocks < 1 ? 1 : blocks < 2048 ? blocks : 2048);
}

}  // namespace

extern "C" esp_status esp_kv_pages_workspace(const esp_kv_cache *cache, int32_t n, size_t *bytes) {
    if (esp_status e = check_cache(cache)) return e;
    if (!bytes) return ESP_ERR_INVALID_ARG;
    if (n < 0 || n > cache->sequences) return ESP_ERR_SHAPE;
    Work w;
    *bytes = lay_out(cache, nullptr, w);
    return ESP_OK;
}

extern "C" esp_status esp_kv_resize(const esp_kv_cache *cache, const int32_t *lengths, void *workspace, size_t workspace_bytes, void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (!lengths) return ESP_ERR_INVALID_ARG;
    Work w;
    if (esp_status e = work_of(cache, workspace, workspace_bytes, w)) return e;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Cache c = cache_of(cache);
    const int64_t copies = copies_of(cache, w);
    w.at_once = copies <= kResizeCopies && copies * page_bytes(cache) <= kResizeBytes;
    k_resize_drop<<<w.entries.blocks, kThreads, 0, s>>>(c, lengths, w);
    k_resize_mark<<<w.entries.blocks + w.pages.blocks, kThreads, 0, s>>>(c, lengths, w);
    k_resize_take<<<w.entries.blocks, kThreads, 0, s>>>(c, lengths, w);
    if (!w.at_once) k_copy<<<copy_blocks(cache, cache->sequences), kCopyThreads, 0, s>>>(c, w.count, w.copies, nullptr, nullptr);
    return launched();
}

extern "C" esp_status esp_kv_fork(const esp_kv_cache *cache, int32_t n, const int32_t *parents, const int32_t *children, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (n < 0 || n > cache->sequences) return ESP_ERR_SHAPE;
    if (n == 0) return ESP_OK;
    if (!parents || !children) return ESP_ERR_INVALID_ARG;
    Work w;
    if (esp_status e = work_of(cache, workspace, workspace_bytes, w)) return e;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Cache c = cache_of(cache);
    w.at_once = page_bytes(cache) <= kAtOnce;
    k_fork_drop<<<n, kThreads, 0, s>>>(c, n, parents, children, w);
    k_mark_free<<<w.pages.blocks, kThreads, 0, s>>>(c, w);
    k_fork_take<<<n, kThreads, 0, s>>>(c, n, parents, children, w);
    if (!w.at_once) k_copy<<<copy_blocks(cache, n), kCopyThreads, 0, s>>>(c, w.count, w.copies, nullptr, nullptr);
    return launched();
}

extern "C" esp_status esp_kv_reorder(const esp_kv_cache *cache, const int32_t *parents, void *workspace, size_t workspace_bytes, void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (!parents) return ESP_ERR_INVALID_ARG;
    if (cache->sequences > kMostSequences) return ESP_ERR_SHAPE;
    Work w;
    if (esp_status e = work_of(cache, workspace, workspace_bytes, w)) return e;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Cache c = cache_of(cache);
    w.at_once = page_bytes(cache) <= kAtOnce;
    k_reorder_drop<<<cache->sequences, kThreads, 0, s>>>(c, parents, w);
    k_mark_free<<<w.pages.blocks, kThreads, 0, s>>>(c, w);
    k_reorder_take<<<cache->sequences, kThreads, 0, s>>>(c, w);
    if (!w.at_once) k_copy<<<copy_blocks(cache, cache->sequences), kCopyThreads, 0, s>>>(c, w.count, w.copies, nullptr, nullptr);
    return launched();
}

extern "C" esp_status esp_kv_compact(const esp_kv_cache *cache, int32_t limit, int32_t *table_out, int32_t *refs_out, int32_t *live,
                                     void *workspace, size_t workspace_bytes, void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (!table_out || !refs_out) return ESP_ERR_INVALID_ARG;
    Work w;
    if (esp_status e = work_of(cache, workspace, workspace_bytes, w)) return e;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Cache c = cache_of(cache);
    k_compact_mark<<<w.pages.blocks, kThreads, 0, s>>>(c, refs_out, w);
    k_compact_place<<<w.pages.blocks, kThreads, 0, s>>>(c, limit, refs_out, live, w);
    k_copy<<<copy_blocks(cache, cache->pages), kCopyThreads, 0, s>>>(c, w.count, w.copies, w.goes, table_out);
    return launched();
}

extern "C" esp_status esp_kv_device_status(const esp_kv_cache *cache, void *stream) {
    if (!cache || !cache->status) return ESP_ERR_INVALID_ARG;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int32_t code = 0, zero = 0;
    if (hipMemcpyAsync(&code, cache->status, 4, hipMemcpyDeviceToHost, s) != hipSuccess || hipStreamSynchronize(s) != hipSuccess) return ESP_ERR_DEVICE;
    if (code && (hipMemcpyAsync(cache->status, &zero, 4, hipMemcpyHostToDevice, s) != hipSuccess || hipStreamSynchronize(s) != hipSuccess)) return ESP_ERR_DEVICE;
    return code >= ESP_OK && code <= ESP_ERR_STATE ? esp_status(code) : ESP_ERR_DEVICE;
}
