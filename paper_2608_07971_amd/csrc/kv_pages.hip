// Page operations of the paged 8-bit cache: resize, fork, compact.
//
// Each is one workgroup that settles the integers (references, free pages,
// table) and a second launch that copies the pages on the list it left.  All
// choices are by index (the lowest free page, in order of sequence and slot),
// so results do not depend on the order of atomics.
#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kIndexThreads = 1024, kIndexWaves = kIndexThreads / 64;
constexpr int kCopyThreads = 256;

struct Work {
    int32_t *count;                  // copies to make
    int2 *copies;                    // [pages] from, to
    int32_t *list;                   // [pages] free pages, lowest first
    int32_t *other;                  // [pages or sequences] replaced pages, marks or new places
};

// References change by atomics and are read past the compute unit's cache.
__device__ __forceinline__ int32_t refs_now(const Cache &c, int32_t p) {
    return __hip_atomic_load(c.refs + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

// Numbers the items i of [0, n) that `has` holds for, in order: each wavefront
// counts a run of its own, the runs are added up, and use(i, rank) is called
// for every item held.  Returns how many there are.  `go(total)` decides after
// the count whether they are used.
template <typename Has, typename Go, typename Use>
__device__ int number(int64_t n, int *lds, Has has, Go go, Use use) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t run = ((n + kIndexWaves - 1) / kIndexWaves + 63) / 64 * 64;
    const int64_t from = min(n, run * wave), to = min(n, from + run);
    int mine = 0;
    for (int64_t i = from; i < to; i += 64) mine += __popcll(__ballot(i + lane < to && has(i + lane)));
    __syncthreads();
    if (lane == 0) lds[wave] = mine;
    __syncthreads();
    int before = 0, total = 0;
    for (int w = 0; w < kIndexWaves; w++) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    if (go(total)) {
        for (int64_t i = from; i < to; i += 64) {
            const bool held = i + lane < to && has(i + lane);
            const uint64_t mask = __ballot(held);
            if (held) use(i + lane, before + lanes_below(mask));
            before += __popcll(mask);
        }
    }
    __syncthreads();
    return total;
}

__global__ __launch_bounds__(kIndexThreads) void k_resize(Cache c, const int32_t *lengths, Work w) {
    __shared__ int lds[kIndexWaves];
    __shared__ int copies;
    const int tid = threadIdx.x;
    const int64_t entries = int64_t(c.sequences) * c.width;
    if (tid == 0) {
        copies = 0;
        *w.count = 0;
    }
    int bad = 0;
    for (int s = tid; s < c.sequences; s += kIndexThreads) bad |= lengths[s] < 0 || lengths[s] > int64_t(c.width) << c.shift;
    for (int64_t i = tid; i < entries; i += kIndexThreads) bad |= c.table[i] < -1 || c.table[i] >= c.pages;
    if (__syncthreads_or(bad)) {
        if (tid == 0) record(c, ESP_ERR_SHAPE);
        return;
    }
    auto wanted = [&](int64_t i, int &seq) {
        seq = int(i / c.width);
        return int(i - int64_t(seq) * c.width) < (lengths[seq] + c.tokens - 1) >> c.shift;
    };
    auto drop = [&](int by) {
        for (int64_t i = tid; i < entries; i += kIndexThreads) {
            int seq;
            const int32_t p = c.table[i];
            if (p >= 0 && !wanted(i, seq)) atomicAdd(c.refs + p, by);
        }
        __threadfence();
        __syncthreads();
    };
    drop(-1);
    // a kept page that ends inside its sequence and still has other owners
    auto split = [&](int64_t i, int seq, int32_t p) {
        const int last = min(c.lengths[seq], lengths[seq]);
        return int(i - int64_t(seq) * c.width) == last >> c.shift && (last & (c.tokens - 1)) && refs_now(c, p) > 1;
    };
    auto needs = [&](int64_t i) {
        int seq;
        const int32_t p = c.table[i];
        return wanted(i, seq) && (p < 0 || split(i, seq, p));
    };
    const int need = number(entries, lds, needs, [](int) { return false; }, [](int64_t, int) {});
    const int have = number(c.pages, lds, [&](int64_t p) { return refs_now(c, int32_t(p)) == 0; }, [&](int total) { return total >= need; },
                            [&](int64_t p, int rank) { if (rank < need) w.list[rank] = int32_t(p); });
    if (have < need) {
        drop(1);
        if (tid == 0) record(c, ESP_ERR_RANGE);
        return;
    }
    __threadfence();
    __syncthreads();
    // the entry alone changes here; splits are judged by references, which change after
    number(entries, lds, needs, [](int) { return true; }, [&](int64_t i, int rank) {
        const int32_t p = c.table[i], to = w.list[rank];
        if (p >= 0) w.copies[atomicAdd(&copies, 1)] = make_int2(p, to);
        w.other[rank] = p;
        c.table[i] = to;
    });
    for (int r = tid; r < need; r += kIndexThreads) {
        c.refs[w.list[r]] = 1;
        if (w.other[r] >= 0) atomicAdd(c.refs + w.other[r], -1);
    }
    for (int64_t i = tid; i < entries; i += kIndexThreads) {
        int seq;
        if (!wanted(i, seq)) c.table[i] = -1;
    }
    __syncthreads();
    for (int s = tid; s < c.sequences; s += kIndexThreads) c.lengths[s] = lengths[s];
    if (tid == 0) *w.count = copies;
}

__global__ __launch_bounds__(kIndexThreads) void k_fork(Cache c, int n, const int32_t *parents, const int32_t *children, Work w) {
    __shared__ int lds[kIndexWaves];
    const int tid = threadIdx.x;
    const int64_t entries = int64_t(n) * c.width;
    if (tid == 0) *w.count = 0;
    int32_t *marks = w.other;
    for (int s = tid; s < c.sequences; s += kIndexThreads) marks[s] = 0;
    __threadfence();
    __syncthreads();
    int bad = 0;
    for (int i = tid; i < n; i += kIndexThreads) {
        const int p = parents[i], k = children[i];
        if (p < 0 || p >= c.sequences || k < 0 || k >= c.sequences) bad = 1;
        else bad |= atomicExch(marks + k, 1);
    }
    __threadfence();
    if (!(bad = __syncthreads_or(bad)))
        for (int i = tid; i < n; i += kIndexThreads) bad |= __hip_atomic_load(marks + parents[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__syncthreads_or(bad)) {
        if (tid == 0) record(c, ESP_ERR_INVALID_ARG);
        return;
    }
    auto parted = [&](int i) { return (c.lengths[parents[i]] & (c.tokens - 1)) != 0; };
    auto entry = [&](const int32_t *of, int64_t i) { return c.table + int64_t(of[i / c.width]) * c.width + i % c.width; };
    for (int i = tid; i < n; i += kIndexThreads) {
        const int length = c.lengths[parents[i]];
        bad |= length < 0 || length > int64_t(c.width) << c.shift;
        if (!bad && parted(i)) bad |= c.table[int64_t(parents[i]) * c.width + (length >> c.shift)] < 0;
    }
    for (int64_t i = tid; i < entries; i += kIndexThreads) {
        const int32_t p = *entry(parents, i), k = *entry(children, i);
        bad |= p < -1 || p >= c.pages || k < -1 || k >= c.pages;
    }
    if (__syncthreads_or(bad)) {
        if (tid == 0) record(c, ESP_ERR_SHAPE);
        return;
    }
    auto drop = [&](int by) {
        for (int64_t i = tid; i < entries; i += kIndexThreads) {
            const int32_t p = *entry(children, i);
            if (p >= 0) atomicAdd(c.refs + p, by);
        }
        __threadfence();
        __syncthreads();
    };
    drop(-1);
    const int need = number(n, lds, [&](int64_t i) { return parted(int(i)); }, [](int) { return false; }, [](int64_t, int) {});
    const int have = number(c.pages, lds, [&](int64_t p) { return refs_now(c, int32_t(p)) == 0; }, [&](int total) { return total >= need; },
                            [&](int64_t p, int rank) { if (rank < need) w.list[rank] = int32_t(p); });
    if (have < need) {
        drop(1);
        if (tid == 0) record(c, ESP_ERR_RANGE);
        return;
    }
    for (int64_t i = tid; i < entries; i += kIndexThreads) {
        const int k = int(i / c.width), slot = int(i - int64_t(k) * c.width);
        const int32_t p = *entry(parents, i);
        if (parted(k) && slot == c.lengths[parents[k]] >> c.shift) continue;
        if (p >= 0) atomicAdd(c.refs + p, 1);
        *entry(children, i) = p;
    }
    number(n, lds, [&](int64_t i) { return parted(int(i)); }, [](int) { return true; }, [&](int64_t i, int rank) {
        const int slot = c.lengths[parents[i]] >> c.shift;
        const int32_t to = w.list[rank];
        w.copies[rank] = make_int2(c.table[int64_t(parents[i]) * c.width + slot], to);
        c.table[int64_t(children[i]) * c.width + slot] = to;
        c.refs[to] = 1;
    });
    for (int i = tid; i < n; i += kIndexThreads) c.lengths[children[i]] = c.lengths[parents[i]];
    if (tid == 0) *w.count = need;
}

__global__ __launch_bounds__(kIndexThreads) void k_compact(Cache c, int limit, int32_t *refs_out, int32_t *live_out, Work w) {
    __shared__ int lds[kIndexWaves];
    const int tid = threadIdx.x;
    const int live = number(c.pages, lds, [&](int64_t p) { return c.refs[p] > 0; }, [](int) { return false; }, [](int64_t, int) {});
    if (limit < 0) limit = live;
    limit = min(limit, c.pages);
    if (tid == 0 && live_out) *live_out = live;
    int32_t *goes = w.other;
    for (int p = tid; p < c.pages; p += kIndexThreads) {
        goes[p] = p;
        refs_out[p] = c.refs[p];
    }
    int moved = 0;
    if (live <= limit) {
        number(limit, lds, [&](int64_t p) { return c.refs[p] <= 0; }, [](int) { return true; }, [&](int64_t p, int rank) { w.list[rank] = int32_t(p); });
        moved = number(c.pages - limit, lds, [&](int64_t p) { return c.refs[limit + p] > 0; }, [](int) { return true; }, [&](int64_t p, int rank) {
            const int32_t from = limit + int32_t(p), to = w.list[rank];
            w.copies[rank] = make_int2(from, to);
            goes[from] = to;
        });
        for (int r = tid; r < moved; r += kIndexThreads) {
            const int2 m = w.copies[r];
            refs_out[m.y] = c.refs[m.x];
            refs_out[m.x] = 0;
        }
    } else if (tid == 0) {
        record(c, ESP_ERR_RANGE);
    }
    if (tid == 0) *w.count = moved;
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
            if (at + j * kCopyThreads < vectors) x[j] = from[at + j * kCopyThreads];
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (at + j * kCopyThreads < vectors) to[at + j * kCopyThreads] = x[j];
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

size_t pages_bytes(const esp_kv_cache *c) {
    const size_t pages = size_t(c->pages), most = pages > size_t(c->sequences) ? pages : size_t(c->sequences);
    return (256 + pages * 12 + most * 4 + 255) / 256 * 256;
}
esp_status work_of(const esp_kv_cache *c, void *workspace, size_t bytes, Work &w) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || bytes < pages_bytes(c)) return ESP_ERR_WORKSPACE;
    char *p = static_cast<char *>(workspace);
    w.count = reinterpret_cast<int32_t *>(p);
    w.copies = reinterpret_cast<int2 *>(p + 256);
    w.list = reinterpret_cast<int32_t *>(p + 256 + size_t(c->pages) * 8);
    w.other = w.list + c->pages;
    return ESP_OK;
}
// Workgroups of the copy for at most `most` pages: 2,048 fill the GPU.
unsigned copy_blocks(const esp_kv_cache *c, int64_t most) {
    const int64_t bytes = int64_t(c->layers) * c->kv_heads * c->page_tokens * c->head_dim;
    const int64_t blocks = most * 2 * ((bytes + kCopyThreads * 64 - 1) / (kCopyThreads * 64));
    return unsigned(blocks < 1 ? 1 : blocks < 2048 ? blocks : 2048);
}

}  // namespace

extern "C" esp_status esp_kv_pages_workspace(const esp_kv_cache *cache, int32_t n, size_t *bytes) {
    if (esp_status e = check_cache(cache)) return e;
    if (!bytes) return ESP_ERR_INVALID_ARG;
    if (n < 0 || n > cache->sequences) return ESP_ERR_SHAPE;
    *bytes = pages_bytes(cache);
    return ESP_OK;
}

extern "C" esp_status esp_kv_resize(const esp_kv_cache *cache, const int32_t *lengths, void *workspace, size_t workspace_bytes, void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (!lengths) return ESP_ERR_INVALID_ARG;
    Work w;
    if (esp_status e = work_of(cache, workspace, workspace_bytes, w)) return e;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Cache c = cache_of(cache);
    k_resize<<<1, kIndexThreads, 0, s>>>(c, lengths, w);
    k_copy<<<copy_blocks(cache, cache->sequences), kCopyThreads, 0, s>>>(c, w.count, w.copies, nullptr, nullptr);
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
    k_fork<<<1, kIndexThreads, 0, s>>>(c, n, parents, children, w);
    k_copy<<<copy_blocks(cache, n), kCopyThreads, 0, s>>>(c, w.count, w.copies, nullptr, nullptr);
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
    k_compact<<<1, kIndexThreads, 0, s>>>(c, limit, refs_out, live, w);
    k_copy<<<copy_blocks(cache, cache->pages), kCopyThreads, 0, s>>>(c, w.count, w.copies, w.other, table_out);
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
