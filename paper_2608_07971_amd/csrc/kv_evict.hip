// Eviction by accumulated attention weight: of a sequence that is cut, every
// layer and key head keeps its own tokens, the last `recent` and those of the
// largest weight, which move together in their order.
//   1  entries whose page is shared, and free pages, are marked; what is wrong is noted
//   2  these entries get pages of their own, pages past the new end go
//   3  a workgroup a layer, sequence and head finds the least weight that stays, marks
//      the tokens in a bit mask and moves their weights together
//   4  a workgroup a layer, sequence, head and side moves the codes
// A token never moves to a higher place, so both moves go through a row once, in place:
// what a stretch of new places takes comes from there or from further on.
#include "kv_pages.hpp"

namespace esp_kv {

struct EvictArgs {
    Cache c;
    const int32_t *keep;
    float *mass;
    uint64_t *kept;                         // [layer][sequence][head][words]: tokens that stay
    int32_t recent, words;
};

__device__ __forceinline__ int pages_of(const Cache &c, int tokens) { return int((uint32_t(tokens) + c.tokens - 1) >> c.shift); }

// Workgroups [0, entries.blocks): entries; the rest: pages.
__global__ __launch_bounds__(kThreads) void k_evict_mark(Cache c, const int32_t *keep, Work w) {
    __shared__ int lds[4];
    const int b = blockIdx.x;
    if (b >= w.entries.blocks) {
        mark(w.pages, b - w.entries.blocks, w.page_mask, w.page_sum, lds, [&](int64_t p) { return c.refs[p] == 0; });
        return;
    }
    int bad = 0;
    mark(w.entries, b, w.need_mask, w.need_sum, lds, [&](int64_t i) {
        const int seq = int(uint32_t(i) / uint32_t(c.width)), slot = int(uint32_t(i) - uint32_t(seq) * uint32_t(c.width));
        const int32_t m = c.lengths[seq], k = keep[seq], p = c.table[i];
        const bool ok = k >= 0 && m >= 0 && m <= int64_t(c.width) << c.shift, cut = ok && m > k;
        const bool page = p >= 0 && p < c.pages;
        bad |= !ok || p < -1 || p >= c.pages || (cut && slot < pages_of(c, m) && !page);
        w.rows[i] = p;
        if (slot == 0) w.row_lengths[seq] = cut ? m : -1;
        return cut && slot < pages_of(c, k) && page && c.refs[p] > 1;
    });
    bad = block_sum(bad, lds);
    if (threadIdx.x == 0) w.bad[b] = bad;
}

__global__ __launch_bounds__(kThreads) void k_evict_take(Cache c, const int32_t *keep, Work w) {
    __shared__ int lds[4], free_at[kMaxBlocks + 1], need_at[kMaxBlocks + 1];
    int bad = 0;
    for (int b = threadIdx.x; b < w.entries.blocks; b += kThreads) bad |= w.bad[b];
    bad = block_sum(bad, lds);
    prefix(w.page_sum, w.pages.blocks, free_at, lds);
    prefix(w.need_sum, w.entries.blocks, need_at, lds);
    const bool go = !bad && free_at[w.pages.blocks] >= need_at[w.entries.blocks];
    if (!go) {
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            *w.count = 0;
            record(c, bad ? ESP_ERR_SHAPE : ESP_ERR_RANGE);
        }
        return;
    }
    if (blockIdx.x == 0) {                  // the sequences that are cut, in order
        int n = 0;
        for (int s0 = 0; s0 < c.sequences; s0 += kThreads) {
            const int seq = s0 + threadIdx.x;
            const bool is = seq < c.sequences && w.row_lengths[seq] >= 0;
            const uint64_t who = __ballot(is);
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __popcll(who);
            __syncthreads();
            int at = n + lanes_below(who);
            for (int k = 0; k < 4; k++) {
                at += k < int(threadIdx.x >> 6) ? lds[k] : 0;
                n += lds[k];
            }
            if (is) w.cut[at] = seq;
        }
        if (threadIdx.x == 0) *w.count = n;
    }
    ranked(w.entries, blockIdx.x, w.need_mask, need_at[blockIdx.x], w.need_mask, 0, [&](int64_t i, bool need, int rank, bool, int) {
        const int seq = int(uint32_t(i) / uint32_t(c.width)), slot = int(uint32_t(i) - uint32_t(seq) * uint32_t(c.width));
        if (w.row_lengths[seq] < 0) return;
        const int32_t p = w.rows[i];
        if (need) {
            const int to = select(w, [&](int b) { return free_at[b]; }, 0, rank);
            if (to >= 0) {
                c.refs[to] = 1;
                c.table[i] = to;
                atomicAdd(c.refs + p, -1);
            }
        } else if (slot >= pages_of(c, keep[seq]) && p >= 0) {
            c.table[i] = -1;
            atomicAdd(c.refs + p, -1);
        }
        if (slot == 0) c.lengths[seq] = keep[seq];
    });
}

// A weight's place in the order of all: NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x != x ? 0 : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Item i of those that are cut: its place, and its number among all.
struct Place {
    int layer, seq, head, number;
};
__device__ __forceinline__ Place place_of(const Cache &c, const Work &w, int i) {
    const int head = i % c.heads, rest = i / c.heads, layer = rest % c.layers, seq = w.cut[rest / c.layers];
    return {layer, seq, head, (layer * c.sequences + seq) * c.heads + head};
}

constexpr int kHeld = 16;                   // weights a thread: rows of up to 4,096 tokens are read once

// 1,024 rows of up to 4,096 weights 20 us, 8 rows of 1,500 11 us: four rounds of counting
// and a walk, each a few barriers.
// The want-th largest weight by its bits, eight at a time from the top; then one pass over
// the tokens in order, equal ones by the lower place.
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictArgs a, Work w) {
    __shared__ int counts[256], at[4], ties[4], picked[2];
    const Cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int item = blockIdx.x, items = *w.count * c.layers * c.heads; item < items; item += gridDim.x) {
        const Place p = place_of(c, w, item);
        const int length = w.row_lengths[p.seq];
        const int keep = a.keep[p.seq], recent = min(a.recent, keep), older = length - recent;
        float *mass = a.mass + int64_t(p.number) * (int64_t(c.width) << c.shift);
        uint64_t *kept = a.kept + int64_t(p.number) * a.words;

        // a thread's first weights stay in registers, longer rows are read again
        float first[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; i++) first[i] = i * kThreads + tid < length ? mass[i * kThreads + tid] : 0.0f;
        uint32_t least = ~0u;                   // of those that stay
        int want = keep - recent;               // and how many equal to it do
        if (want > 0) {
            uint32_t known = 0;
            least = 0;
            for (int shift = 24; shift >= 0; shift -= 8) {
                counts[tid] = 0;
                __syncthreads();
                auto count = [&](float x) {
                    const uint32_t u = order_of(x);
                    if ((u & known) == least) atomicAdd(counts + ((u >> shift) & 255), 1);
                };
#pragma unroll
                for (int i = 0; i < kHeld; i++)
                    if (i * kThreads + tid < older) count(first[i]);
                for (int t = kHeld * kThreads + tid; t < older; t += kThreads) count(mass[t]);
                __syncthreads();
                if (wave == 0) {                // four digits a lane, from the largest
                    int own[4], sum = 0;
#pragma unroll
                    for (int k = 0; k < 4; k++) sum += own[k] = counts[255 - 4 * lane - k];
                    int before = sum;
#pragma unroll
                    for (int m = 1; m < 64; m <<= 1) {
                        const int v = __shfl_up(before, m);
                        before += lane >= m ? v : 0;
                    }
                    before -= sum;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        if (want > before && want <= before + own[k]) {
                            picked[0] = 255 - 4 * lane - k;
                            picked[1] = want - before;
                        }
                        before += own[k];
                    }
                }
                __syncthreads();
                least |= uint32_t(picked[0]) << shift;
                known |= 255u << shift;
                want = picked[1];
                __syncthreads();
            }
        }
        int to = 0, equal = 0;                  // tokens that stay, and those equal to `least`, so far
        auto settle = [&](int t0, float x) {
            const int t = t0 + tid;
            const uint32_t u = order_of(x);
            const bool tie = t < older && u == least;
            const uint64_t same = __ballot(tie);
            if (lane == 0) ties[wave] = __popcll(same);
            __syncthreads();
            int rank = equal + lanes_below(same);
            for (int k = 0; k < 4; k++) {
                rank += k < wave ? ties[k] : 0;
                equal += ties[k];
            }
            const bool stays = t < length && (t >= older || u > least || (tie && rank < want));
            const uint64_t who = __ballot(stays);
            if (lane == 0) {
                at[wave] = __popcll(who);
                if (t < length) kept[t / 64] = who;
            }
            __syncthreads();
            int place = to + lanes_below(who);
            for (int k = 0; k < 4; k++) {
                place += k < wave ? at[k] : 0;
                to += at[k];
            }
            if (stays) mass[place] = x;
            __syncthreads();
        };
#pragma unroll
        for (int i = 0; i < kHeld; i++)
            if (i * kThreads < length) settle(i * kThreads, first[i]);
        for (int t0 = kHeld * kThreads; t0 < length; t0 += kThreads) settle(t0, t0 + tid < length ? mass[t0 + tid] : 0.0f);
    }
}

// kTurn tokens move at a time, whole pages; the mask of kStretch is read at a time.  Shorter
// turns wait more often for their look-ups, longer ones leave the GPU fewer workgroups: 64,
// 128, 256 tokens take 280, 284, 330 us for 1,024 rows of 2,048 kept of up to 4,096 tokens of
// 128, and 40, 23, 16 us for 8 rows of 1,000 of 1,500 tokens of 64.  One size for all launches,
// though the longer one would be better for so few rows.
constexpr int kTurn = 128, kMoveThreads = 4 * kTurn, kMoveWaves = kMoveThreads / 64, kStretch = 2048;

// Where the tokens of a turn come from.
struct Sources {
    int64_t from[kTurn], to[kTurn / 16];    // block of the old page; of the new, of each sixteen
    int32_t page[kTurn / 16];               // the new page of each sixteen, and its scale
    float scale[kTurn / 16];
    int32_t in_page[kTurn];
    float by[kTurn];                        // the old scale over the new
    int32_t rescale[kTurn / 64];            // whether any of these is not 1
};

__device__ __forceinline__ uint32_t code2(float x, float y) { return __builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false); }
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float b0, float b1, float b2, float b3) {
    const half2 a = codes<false>(w, static_cast<half2 *>(nullptr)), b = codes<true>(w, static_cast<half2 *>(nullptr));
    return code2(float(a[0]) * b0, float(a[1]) * b1) | code2(float(b[0]) * b2, float(b[1]) * b3) << 16;
}

// Keys: sixteen bytes a thread.  Values, whose tokens lie innermost: a lane has a dimension,
// and takes the sixteen tokens of a group that stand together there at once; which of their
// bytes go where is the same for all lanes, so that a byte is a permutation whose selector
// lies in a scalar register.
// Bound by memory, with values read in whole sixteens of tokens (1.3 GB in 276 us, 4.8 TB/s,
// where half of the tokens stay): gathered byte by byte 525 us.
template <int Dim, int Page> __global__ __launch_bounds__(kMoveThreads) void k_evict_move(EvictArgs a, Work w) {
    __shared__ int list[kStretch + kTurn];
    __shared__ Sources sources[2];
    const Cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int item = blockIdx.x, items = *w.count * c.layers * c.heads * 2; item < items; item += gridDim.x) {
        const Place p = place_of(c, w, item >> 1);
        const int length = w.row_lengths[p.seq], values = item & 1;
        const uint64_t *kept = a.kept + int64_t(p.number) * a.words;
        const int32_t *old = w.rows + int64_t(p.seq) * c.width, *table = c.table + int64_t(p.seq) * c.width;
        uint8_t *pool = values ? c.v : c.k;

        // Wavefronts, 64 each, find the sources of tokens list[from, from + n), which go to places
        // [done, done + n).
        auto look = [&](int from, int n, int done, Sources &to) {
            const int t = wave * 64 + lane, src = list[from + min(t, n - 1)];
            const int32_t page = old[src / Page];
            const float was = t < n ? *c.block_scale(page, p.layer, values, p.head) : 0.0f;
            float now = was;
#pragma unroll
            for (int m = Page / 2; m; m >>= 1) now = fmaxf(now, __shfl_xor(now, m));
            const float by = now > 0.0f ? was / now : 1.0f;
            to.from[t] = c.block(page, p.layer, p.head);
            to.in_page[t] = src % Page;
            to.by[t] = by;
            const bool any = __any(t < n && by != 1.0f);
            if (lane == 0) to.rescale[wave] = any;
            if (t % 16 == 0 && t < n) {
                const int32_t place = table[(done + t) / Page];
                to.to[t / 16] = c.block(place, p.layer, p.head);
                to.page[t / 16] = place;
                to.scale[t / 16] = now;
            }
        };
        // The new pages' scales, once all of a turn's old ones have been read: no later token
        // comes from these pages.
        auto leave_scales = [&](int n, const Sources &m) {
            const int t = tid * 16;
            if (t < n && t % Page == 0) *c.block_scale(m.page[tid], p.layer, values, p.head) = m.scale[tid];
        };
        auto move_keys = [&](int n, int done, const Sources &m) {
            constexpr int kChunks = Dim / 16, kUnits = kTurn * kChunks / kMoveThreads;
            uint4v x[kUnits];
#pragma unroll
            for (int i = 0; i < kUnits; i++) {
                const int u = tid + i * kMoveThreads, t = min(u / kChunks, n - 1);
                x[i] = *reinterpret_cast<const uint4v *>(pool + m.from[t] + m.in_page[t] * Dim + u % kChunks * 16);
            }
            if (m.rescale[0] | m.rescale[1])
#pragma unroll
                for (int i = 0; i < kUnits; i++) {
                    const float by = m.by[min((tid + i * kMoveThreads) / kChunks, n - 1)];
#pragma unroll
                    for (int k = 0; k < 4; k++) x[i][k] = by != 1.0f ? rescaled(x[i][k], by, by, by, by) : x[i][k];
                }
            __syncthreads();                    // all of them are read before any place is written
            leave_scales(n, m);
#pragma unroll
            for (int i = 0; i < kUnits; i++) {
                const int u = tid + i * kMoveThreads, t = u / kChunks, at = done + t;
                if (t < n) *reinterpret_cast<uint4v *>(pool + m.to[t / 16] + at % Page * Dim + u % kChunks * 16) = x[i];
            }
        };
        auto move_values = [&](int n, int done, int from, const Sources &m) {
            constexpr int kHalves = Dim / 64, kOwn = kTurn * kHalves / kMoveWaves;     // tokens of a wavefront
            const int d = wave % kHalves * 64 + lane, t0 = wave / kHalves * kOwn, own = min(kOwn, n - t0);
            uint4v x[kOwn / 16];
            if (own > 0) {
                const int src = list[from + t0 + min(lane, own - 1)];
                // group of sixteen tokens of the old pages that a lane's token is in; the first of each
                const int before = __shfl_up(src, 1);
                uint64_t firsts = __ballot(lane < own && lane > 0 && src >> 4 != before >> 4);
                auto load = [&](int t) {        // the group of token t
                    const int s = __builtin_amdgcn_readlane(src, t);
                    const int64_t block = m.from[t0 + t];
                    return *reinterpret_cast<const uint4v *>(pool + block + d * Page + (s % Page & ~15));
                };
                uint4v now = load(0), next = now;
                int turns = firsts ? __builtin_ctzll(firsts) : 64;   // the token that the next group begins with
                if (turns < 64) next = load(turns);
#pragma unroll
                for (int i = 0; i < kOwn; i += 4) {
                    uint32_t word = 0;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const int t = i + j;
                        if (t < own) {
                            if (t == turns) {
                                now = next;
                                firsts &= firsts - 1;
                                turns = firsts ? __builtin_ctzll(firsts) : 64;
                                if (turns < 64) next = load(turns);
                            }
                            const uint32_t s = uint32_t(__builtin_amdgcn_readlane(src, t)) & 15, none = 0x0c0c0c0cu;
                            const uint32_t pick = (none & ~(255u << (8 * j))) | (s & 7) << (8 * j);
                            word |= __builtin_amdgcn_perm(now[1], now[0], s < 8 ? pick : none) | __builtin_amdgcn_perm(now[3], now[2], s < 8 ? none : pick);
                        }
                    }
                    x[i / 16][i / 4 % 4] = word;
                }
                if (m.rescale[0] | m.rescale[1])
#pragma unroll
                    for (int i = 0; i < kOwn; i += 4) {
                        const float *by = &m.by[t0 + i];
                        x[i / 16][i / 4 % 4] = rescaled(x[i / 16][i / 4 % 4], by[0], by[1], by[2], by[3]);
                    }
            }
            __syncthreads();                    // all of them are read before any place is written
            leave_scales(n, m);
#pragma unroll
            for (int i = 0; i < kOwn; i += 16) {
                const int left = own - i, at = done + t0 + i;
                if (left <= 0) break;
                uint4v *to = reinterpret_cast<uint4v *>(pool + m.to[(t0 + i) / 16] + d * Page + at % Page);
                if (left < 16) {                // past the end: as it was
                    const uint4v was = *to;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const int more = left - 4 * k;
                        const uint32_t mine = more >= 4 ? ~0u : more <= 0 ? 0u : (1u << (8 * more)) - 1;
                        x[i / 16][k] = (x[i / 16][k] & mine) | (was[k] & ~mine);
                    }
                }
                *to = x[i / 16];
            }
        };

        int held = 0, done = 0;
        const int words = (length + 63) / 64, keep = a.keep[p.seq];
        for (int x0 = 0; x0 < words; x0 += kStretch / 64) {
            const uint64_t m = lane < kStretch / 64 && x0 + lane < words ? kept[x0 + lane] : 0;
            int before = __popcll(m);
            const int own = before;
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) {
                const int v = __shfl_up(before, k);
                before += lane >= k ? v : 0;
            }
            const int all = __shfl(before, 63);
            before -= own;
            for (int x = wave; x < kStretch / 64; x += kMoveWaves) {
                const uint64_t n = __shfl(m, x);
                const int at = held + __shfl(before, x) + lanes_below(n);
                if (bit_of(n, lane)) list[at] = (x0 + x) * 64 + lane;
            }
            held = __builtin_amdgcn_readfirstlane(held + all);
            __syncthreads();
            // tokens of a turn: whole ones, and what is left at the end of all; keep tokens in all, whatever the masses did meanwhile
            auto size = [&](int from, int done) {
                const int n = min(held - from, keep - done);
                return n >= kTurn ? kTurn : x0 + kStretch / 64 >= words || n == keep - done ? n : 0;
            };
            int from = 0, slot = 0, n = size(0, done);
            if (n > 0 && wave < kTurn / 64) look(0, n, done, sources[0]);
            __syncthreads();
            while (n > 0) {
                const int more = size(from + n, done + n);
                if (more > 0 && wave < kTurn / 64) look(from + n, more, done + n, sources[slot ^ 1]);
                if (values) move_values(n, done, from, sources[slot]);
                else move_keys(n, done, sources[slot]);
                __syncthreads();
                from += n;
                done += n;
                n = more;
                slot ^= 1;
            }
            if (done >= keep) break;
            const int rest = held - from, next = tid < rest ? list[from + tid] : 0;
            __syncthreads();
            if (tid < rest) list[tid] = next;
            __syncthreads();
            held = rest;
        }
        __syncthreads();                        // the next item's list goes into the same place
    }
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

// Workgroups that go through the items, of which few may be cut: 264 us with one for each of
// 131,072 layers, sequences and heads of which none is, 14 so.
constexpr int64_t kMostBlocks = 4096;
unsigned blocks_of(int64_t items) { return unsigned(items < kMostBlocks ? items : kMostBlocks); }

int64_t words_of(const esp_kv_cache *c) { return (int64_t(c->table_width) * c->page_tokens + 63) / 64; }
int64_t items_of(const esp_kv_cache *c) { return int64_t(c->layers) * c->kv_heads * c->sequences; }

template <int Dim> void move(const EvictArgs &a, const Work &w, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: k_evict_move<Dim, 16><<<blocks, kMoveThreads, 0, s>>>(a, w); break;
    case 32: k_evict_move<Dim, 32><<<blocks, kMoveThreads, 0, s>>>(a, w); break;
    default: k_evict_move<Dim, 64><<<blocks, kMoveThreads, 0, s>>>(a, w); break;
    }
}

}  // namespace

extern "C" esp_status esp_kv_evict_workspace(const esp_kv_cache *cache, size_t *bytes) {
    if (esp_status e = check_cache(cache)) return e;
    if (!bytes) return ESP_ERR_INVALID_ARG;
    // kernels count items, some launches' worth past the last, and a row's tokens, some turns past the last, in 32 bits
    if (2 * items_of(cache) > INT32_MAX - (kMostBlocks - 1) || int64_t(cache->table_width) * cache->page_tokens > INT32_MAX - kStretch) return ESP_ERR_SHAPE;
    Work w;
    *bytes = lay_out(cache, nullptr, w) + size_t(items_of(cache)) * words_of(cache) * sizeof(uint64_t);
    return ESP_OK;
}

extern "C" esp_status esp_kv_evict(const esp_kv_cache *cache, const int32_t *keep, int32_t recent, float *mass, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    size_t need = 0;
    if (esp_status e = esp_kv_evict_workspace(cache, &need)) return e;
    if (!keep || !mass) return ESP_ERR_INVALID_ARG;
    if (recent < 0) return ESP_ERR_SHAPE;
    Work w;
    if (esp_status e = work_of(cache, workspace, workspace_bytes, w)) return e;
    if (workspace_bytes < need) return ESP_ERR_WORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Cache c = cache_of(cache);
    const size_t before = need - size_t(items_of(cache)) * words_of(cache) * sizeof(uint64_t);
    const EvictArgs a{c, keep, mass, reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + before), recent, int32_t(words_of(cache))};
    k_evict_mark<<<w.entries.blocks + w.pages.blocks, kThreads, 0, s>>>(c, keep, w);
    k_evict_take<<<w.entries.blocks, kThreads, 0, s>>>(c, keep, w);
    const int64_t items = items_of(cache);
    k_evict_select<<<blocks_of(items), kThreads, 0, s>>>(a, w);
    if (c.dim == 64) move<64>(a, w, blocks_of(2 * items), s);
    else move<128>(a, w, blocks_of(2 * items), s);
    return launched();
}
