// The attention weight that cached tokens get from a call's queries:
//   mass[t] = decay mass[t] + sum over queries that see t of exp(scale q . k_t - lse[q])
// for each sequence and key head; tokens that are new begin at 0.
#include "kv_internal.hpp"

namespace esp_kv {

typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 32;                   // (token, query head) rows of a matrix tile
// k_weigh: groups of four wavefronts that share the queries between them, and tiles of rows that
// each takes between two barriers.
constexpr int kGroups = 2, kSubs = 2, kStep = kGroups * kSubs * kRows;
constexpr float kLog2e = 1.4426950408889634f;

struct View {
    void *data;
    int64_t token, head;
};

struct WeighArgs {
    Cache c;
    Rows rows;
    View q;
    const float *lse;
    float *mass;
    float scale, decay;
    int32_t layer, q_heads, group, window, max_new, max_length, shares, wide;
    int32_t over, most;                     // sequences with more (token, query head) rows than `over`, and `most` of them, are this launch's
};

__device__ __forceinline__ float16v product32(half8 x, half8 y, float16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float16v product32(bhalf8 x, bhalf8 y, float16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float4v product16(half8 x, half8 y, float4v z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float4v product16(bhalf8 x, bhalf8 y, float4v z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }
template <typename T> struct Pack;
template <> struct Pack<_Float16> { typedef half8 v8; typedef half2 v2; };
template <> struct Pack<__bf16> { typedef bhalf8 v8; typedef bhalf2 v2; };

// A row of the call; n = 0 where there is nothing to do, or where it cannot be done (`note`: recorded).
__device__ __forceinline__ Row usable(const WeighArgs &a, int b, bool note) {
    Row r{a.rows.offsets[b], a.rows.offsets[b + 1], a.rows.seqs ? a.rows.seqs[b] : b, 0};
    r.n -= r.first;
    bool ok = r.first >= 0 && r.n >= 0 && int64_t(r.first) + r.n <= a.rows.tokens && r.seq >= 0 && r.seq < a.c.sequences;
    if (ok) {
        r.length = a.c.lengths[r.seq];
        ok = r.length >= 0 && r.length <= int64_t(a.c.width) << a.c.shift && r.n <= a.max_new && r.length <= a.max_length;
    }
    if (!ok) {
        if (note) record(a.c, ESP_ERR_SHAPE);
        return Row{};
    }
    if (r.n * a.group <= a.over || r.n * a.group > a.most) r.n = r.length = 0;
    return r;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// The key head's tiles of kTile tokens in order of rows, cut into even shares.  Finds the
// first of share `share` of `shares`, and how many it has.
struct Found {
    int row, tile, count;
};
template <int kTile> __device__ __forceinline__ Found find_share(const WeighArgs &a, int share, int shares, bool note) {
    const int lane = threadIdx.x & 63, rows = a.rows.rows;
    auto tiles_of = [&](int b, bool n) { return b < rows ? (usable(a, b, n).length + kTile - 1) / kTile : 0; };
    int all = 0, held[4];
#pragma unroll
    for (int k = 0; k < 4; k++) all += held[k] = tiles_of(64 * k + lane, note);   // the first 256 are kept
    for (int b = 256; b < rows; b += 256)
#pragma unroll
        for (int k = 0; k < 4; k++) all += tiles_of(b + 64 * k + lane, note);
    all = wave_sum(all);
    const int each = int((int64_t(all) + shares - 1) / shares);
    const int64_t begin = int64_t(share) * each;
    Found f{-1, 0, int(min(int64_t(each), max(int64_t(0), all - begin)))};
    if (f.count == 0) return f;
    for (int b0 = 0, before = 0; b0 < rows; b0 += 256) {
        if (b0)
#pragma unroll
            for (int k = 0; k < 4; k++) held[k] = tiles_of(b0 + 64 * k + lane, false);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            int at = held[k];
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) {
                const int v = __shfl_up(at, m);
                at += lane >= m ? v : 0;
            }
            at += before;                   // tiles up to this row's last
            const uint64_t past = __ballot(begin < at);
            if (past) {
                const int l = __builtin_ctzll(past);
                f.row = b0 + 64 * k + l;
                f.tile = int(begin) - __shfl(at - held[k], l);
                return f;
            }
            before = __shfl(at, 63);
        }
    }
    return f;                               // lengths that changed under the call
}

// Row r of a sequence's (token, query head) rows, going on by the same number each time.
struct Walker {
    int token, head;
    __device__ __forceinline__ Walker() {}
    __device__ __forceinline__ Walker(int r, int group) : token(r / group), head(r - token * group) {}
    // whether the head came round
    __device__ __forceinline__ bool on(int tokens, int heads, int group) {
        token += tokens;
        head += heads;
        const bool round = head >= group;
        if (round) {
            head -= group;
            token++;
        }
        return round;
    }
};

// Eight elements at any alignment.
template <typename T> __device__ __forceinline__ typename Pack<T>::v8 load8(const T *p, bool wide) {
    typename Pack<T>::v8 x;
    if (wide) x = *reinterpret_cast<const typename Pack<T>::v8 *>(p);
    else
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = p[e];
    return x;
}

// A token's keys as one lane of each half holds them for k_weigh: half h's steps 2 i and 2 i + 1
// are elements 32 i + 16 h and on, so that codes are loaded sixteen at a time.
template <typename T, int Dim> struct Keys {
    typedef typename Pack<T>::v8 V8;
    typedef typename Pack<T>::v2 V2;
    uint4v w[Dim / 32];
    __device__ __forceinline__ void load(const uint8_t *token, int half) {
#pragma unroll
        for (int s = 0; s < Dim / 32; s++) w[s] = *reinterpret_cast<const uint4v *>(token + 32 * s + 16 * half);
    }
    __device__ __forceinline__ V8 step(int s) const { return codes8<V8, V2>(w[s / 2][s % 2 * 2], w[s / 2][s % 2 * 2 + 1]); }
};

__device__ __forceinline__ float weight(float product, float scale, float lse) {
    return __builtin_amdgcn_exp2f(__builtin_fmaf(product, scale, -lse) * kLog2e);
}

// Many queries.  A wavefront has 32 cached tokens, which stay in registers as the columns
// of the products; the queries that see them go by, through LDS, kStep rows at a time, of
// which each group of four wavefronts takes kSubs times 32.  So a token's sum is its lanes'
// own, and no two workgroups add to the same place.  Products wait for no read and no
// exponential for another: all of a tile's reads, products, differences and exponentials go
// one kind after another.
// Bound by the wavefronts' vector instructions (a sixteenth of a tile: difference, product,
// exponential, sum): 3 sequences of up to 12,000 tokens, up to 2,048 of them new, 32 query
// heads of 128, 279 GFLOP, 366 us (762 TFLOP/s; up to 535 in the first passes after the GPU was idle).  Queries through registers instead of direct
// into LDS: 457; one group of wavefronts, or four: 509, 489; heads one after another in the
// launch instead of next to each other, so that long shares come last: 449.
template <typename T, int Dim, int Page> __global__ __launch_bounds__(kThreads * kGroups, 4) void k_weigh(WeighArgs a) {
    typedef typename Pack<T>::v8 V8;
    constexpr int kSteps = Dim / 16, kTile = kWaves * 32, kRowBytes = Dim * 2, kAll = kThreads * kGroups;
    constexpr int kPass = kAll / (Dim / 8), kPasses = kStep / kPass;      // rows that the threads load at once, 16 bytes each
    __shared__ __align__(16) uint8_t queries[2][kStep * kRowBytes];
    __shared__ __align__(16) float lses[2][kStep];
    __shared__ __align__(16) int places[2][kStep];
    __shared__ float sums[kGroups][kTile];
    __shared__ bool counts[2][kGroups];     // whether all of a group's rows of a step do
    static_assert(kSubs * kRows == 64, "a group's rows of a step are one wavefront's");

    const Cache &c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int number = __builtin_amdgcn_readfirstlane(tid >> 6), wave = number % kWaves, team = number / kWaves;
    const int share = blockIdx.x / c.heads, head = blockIdx.x - share * c.heads;
    const Found f = find_share<kTile>(a, share, a.shares, blockIdx.x == 0 && tid < 64);
    int b = __builtin_amdgcn_readfirstlane(f.row), tile = __builtin_amdgcn_readfirstlane(f.tile);
    if (b < 0) return;

    // a 16-byte chunk's place in its row of LDS is turned by the row, so that the rows that a
    // matrix step reads at once lie in different banks
    auto turn = [](int row) { return Dim == 128 ? row & 15 : (row >> 1) & 7; };
    const int chunk = (tid % (Dim / 8)) ^ turn(tid / (Dim / 8));
    const uint32_t query_at = (team * (kSubs * kRows) + col) * kRowBytes + (((2 * half) ^ turn(col)) << 4);
    const int tokens_on = kPass / a.group, heads_on = kPass - tokens_on * a.group;
    const int64_t ahead = tokens_on * a.q.token + heads_on * a.q.head, round = a.q.token - a.group * a.q.head;

    for (int left = __builtin_amdgcn_readfirstlane(f.count); left > 0; left--, tile++) {
        Row row = usable(a, b, false);
        while (tile * kTile >= row.length) {
            if (++b >= a.rows.rows) return;
            tile = 0;
            row = usable(a, b, false);
        }
        const int p0 = row.length - row.n, n_rows = row.n * a.group, t0 = tile * kTile;
        // rows that may see a token of the tile
        const int t1 = min(row.length, t0 + kTile) - 1, w0 = t0 + wave * 32, t = w0 + col;
        const int r_from = max(0, t0 - p0) * a.group / kRows * kRows;
        int r_to = n_rows;
        if (a.window > 0) r_to = int(min(int64_t(n_rows), max(int64_t(0), int64_t(t1) + a.window - p0) * a.group));

        int page = t < row.length ? c.table[int64_t(row.seq) * c.width + t / Page] : -1;
        if (t < row.length && (page < 0 || page >= c.pages)) {
            record(c, ESP_ERR_SHAPE);
            page = -1;
        }
        float sum = 0.0f;
        if (r_from < r_to) {
            const float ks = *c.block_scale(max(page, 0), a.layer, 0, head) * a.scale;
            V8 k[kSteps];
            {
                Keys<T, Dim> codes;
                codes.load(c.k + c.block(max(page, 0), a.layer, head) + t % Page * Dim, half);
#pragma unroll
                for (int s = 0; s < kSteps; s++) k[s] = codes.step(s);
            }
            // rows that are not there are read as the last one
            Walker at(r_from + tid / (Dim / 8), a.group);
            const T *base = static_cast<const T *>(a.q.data) + int64_t(row.first) * a.q.token + int64_t(head) * a.group * a.q.head + chunk * 8;
            const T *from = base + at.token * a.q.token + at.head * a.q.head, *last_row = base + (row.n - 1) * a.q.token;
            int own_row = r_from + (tid & (kStep - 1));
            float next_lse = 0.0f;
            int next_place = -1;
            auto load = [&](int buffer) {
#pragma unroll
                for (int i = 0; i < kPasses; i++) {
                    const T *src = at.token < row.n ? from : last_row;
                    uint8_t *to = &queries[buffer][(i * kAll + number * 64) * 16];
                    if (a.wide) {
                        __builtin_amdgcn_global_load_lds(reinterpret_cast<const __attribute__((address_space(1))) void *>(reinterpret_cast<uintptr_t>(src)),
                                                         (__attribute__((address_space(3))) void *)to, 16, 0, 0);
                    } else {
                        *reinterpret_cast<V8 *>(to + lane * 16) = load8<T>(src, false);
                    }
                    from += ahead;
                    if (at.on(tokens_on, heads_on, a.group)) from += round;
                }
                if (tid < kStep) {
                    next_lse = INFINITY;
                    next_place = -1;
                    if (own_row < n_rows) {
                        const Walker w(own_row, a.group);
                        next_lse = a.lse[int64_t(row.first + w.token) * a.q_heads + head * a.group + w.head];
                        next_place = next_lse == -INFINITY ? -1 : p0 + w.token;     // -1: sees nothing, whatever the query holds
                    }
                    own_row += kStep;
                }
            };
            auto put = [&](int buffer) {
                if (tid < kStep) {
                    lses[buffer][tid] = next_lse;
                    places[buffer][tid] = next_place;
                    const bool all = __all(next_place >= 0);
                    if (lane == 0) counts[buffer][number] = all;
                }
                __builtin_amdgcn_s_waitcnt(0x0f70);              // the queries have come in
            };
            auto products = [&](int buffer, int sub, float16v &s) {
                V8 q[kSteps];
#pragma unroll
                for (int i = 0; i < kSteps; i++)
                    q[i] = *reinterpret_cast<const V8 *>(&queries[buffer][0] + ((query_at + sub * kRows * kRowBytes) ^ ((i / 2 * 4 + i % 2) << 4)));
                __builtin_amdgcn_sched_barrier(0);               // all reads on their way before the first product waits
#pragma unroll
                for (int i = 0; i < 16; i++) s[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < kSteps; i++) s = product32(q[i], k[i], s);
            };
            // s[4 y + x]: row 8 y + 4 half + x
            auto add = [&](int buffer, int sub, const float16v &s) {
                const float *lse = &lses[buffer][(team * kSubs + sub) * kRows + 4 * half];
                float e[16];
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const float4v l = *reinterpret_cast<const float4v *>(lse + 8 * y);
#pragma unroll
                    for (int x = 0; x < 4; x++) e[4 * y + x] = __builtin_fmaf(s[4 * y + x], ks, -l[x]);
                }
                __builtin_amdgcn_sched_barrier(0);               // each step for all of them, so that none waits for itself
#pragma unroll
                for (int i = 0; i < 16; i++) e[i] *= kLog2e;
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 16; i++) e[i] = __builtin_amdgcn_exp2f(e[i]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int m = 8; m; m >>= 1)
#pragma unroll
                    for (int i = 0; i < m; i++) e[i] += e[i + m];
                sum += e[0];
            };
            auto add_seen = [&](int buffer, int sub, const float16v &s) {
                const int r = (team * kSubs + sub) * kRows + 4 * half;
#pragma unroll
                for (int y = 0; y < 4; y++)
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const int p = places[buffer][r + 8 * y + x];
                        const float e = weight(s[4 * y + x], ks, lses[buffer][r + 8 * y + x]);
                        sum += t <= p && (a.window <= 0 || t > p - a.window) ? e : 0.0f;
                    }
            };
            Walker seen(r_from + team * kSubs * kRows, a.group);
            const int seen_tokens = kStep / a.group, seen_heads = kStep - seen_tokens * a.group, spread = kSubs * kRows / a.group + 1;
            load(0);
            put(0);
            __syncthreads();
            int buffer = 0;
            for (int r0 = r_from; r0 < r_to; r0 += kStep, buffer ^= 1) {
                const bool more = r0 + kStep < r_to;
                if (more) load(buffer ^ 1);
                const int own0 = r0 + team * kSubs * kRows, first = p0 + seen.token, last = first + spread;
                seen.on(seen_tokens, seen_heads, a.group);
                if (counts[buffer][team] && w0 + 31 <= first && (a.window <= 0 || w0 > last - a.window)) {
#pragma unroll
                    for (int i = 0; i < kSubs; i++) {
                        float16v s;
                        products(buffer, i, s);
                        add(buffer, i, s);
                    }
                } else {
                    for (int i = 0; i < kSubs && own0 + i * kRows < r_to; i++) {
                        float16v s;
                        products(buffer, i, s);
                        add_seen(buffer, i, s);
                    }
                }
                if (more) put(buffer ^ 1);
                __syncthreads();
            }
        }
        sum += __shfl_xor(sum, 32);
        if (half == 0) sums[team][wave * 32 + col] = sum;
        __syncthreads();
        if (team == 0 && half == 0 && page >= 0) {
#pragma unroll
            for (int g = 1; g < kGroups; g++) sum += sums[g][wave * 32 + col];
            float *mass = a.mass + ((int64_t(a.layer) * c.sequences + row.seq) * c.heads + head) * (int64_t(c.width) * Page) + t;
            *mass = t < p0 ? __builtin_fmaf(*mass, a.decay, sum) : sum;
        }
        __syncthreads();                    // the next tile's sums go into the same places
    }
}

// Few queries: kBlocks times 16 rows of a sequence and key head stay in registers while a
// wavefront goes through its share of the tokens, 64 at a time, sixteen a column block of the
// products; the next ones' codes and the pages after these are on their way.  A block's tokens
// lie in one page, so its place and scale are the wavefront's.  More rows take as many rounds,
// each adding to the one before.
// Bound by memory: 64 single tokens of 32 heads on up to 8,192 cached ones of 8 key heads (200
// MB) 43 us where the memory-side cache holds them (4.6 TB/s), 54 us where it does not (60 with
// products of 32 by 32, whose registers leave three wavefronts a SIMD and 32 tokens a turn).
template <typename T, int Dim, int Page, int kBlocks>
__global__ __launch_bounds__(kThreads, kBlocks == 1 ? 4 : 3) void k_weigh_few(WeighArgs a) {
    typedef typename Pack<T>::v8 V8;
    typedef typename Pack<T>::v2 V2;
    constexpr int kSteps = Dim / 32, kTile = 64, kRound = 16 * kBlocks;
    const Cache &c = a.c;
    const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
    const int share = unit / c.heads, head = unit - share * c.heads;
    if (share >= a.shares) return;
    const Found f = find_share<kTile>(a, share, a.shares, unit == 0);
    int b = __builtin_amdgcn_readfirstlane(f.row), tile = __builtin_amdgcn_readfirstlane(f.tile), left = __builtin_amdgcn_readfirstlane(f.count);
    if (b < 0) return;
    for (; left > 0; b++, tile = 0) {
        if (b >= a.rows.rows) return;
        Row row = usable(a, b, false);
        row.n = __builtin_amdgcn_readfirstlane(row.n);
        row.length = __builtin_amdgcn_readfirstlane(row.length);
        const int p0 = row.length - row.n, n_rows = row.n * a.group, end = min(tile + left, (row.length + kTile - 1) / kTile);
        if (tile >= end) continue;
        left -= end - tile;
        const int32_t *table = c.table + int64_t(row.seq) * c.width;
        float *mass = a.mass + ((int64_t(a.layer) * c.sequences + row.seq) * c.heads + head) * (int64_t(c.width) * Page);
        for (int r0 = 0; r0 < n_rows; r0 += kRound) {
            // quarter g's elements of steps 2 i and 2 i + 1: 64 i + 16 g and on, as the codes are loaded
            V8 q[kBlocks][kSteps];
            float lse[kBlocks][4];          // of rows r0 + 16 y + 4 quarter + x
#pragma unroll
            for (int y = 0; y < kBlocks; y++) {
                const Walker w(min(r0 + 16 * y + col, n_rows - 1), a.group);
                const T *from = static_cast<const T *>(a.q.data) + int64_t(row.first + w.token) * a.q.token + int64_t(head * a.group + w.head) * a.q.head;
#pragma unroll
                for (int s = 0; s < kSteps; s++) q[y][s] = load8<T>(from + s / 2 * 64 + 16 * quarter + s % 2 * 8, a.wide);
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    const int r = r0 + 16 * y + 4 * quarter + x;
                    lse[y][x] = INFINITY;
                    if (r < n_rows) {
                        const Walker v(r, a.group);
                        const float l = a.lse[int64_t(row.first + v.token) * a.q_heads + head * a.group + v.head];
                        lse[y][x] = l == -INFINITY ? INFINITY : l;           // infinity: sees nothing, whatever the query holds
                    }
                }
            }
            auto page_of = [&](int i) {
                const int t = i * kTile + lane;
                return i < end && t < row.length ? table[t / Page] : -1;
            };
            struct Tile {
                uint4v codes[4][Dim / 64];
                float scale, mass;          // of the lane's own token
                bool there;
            };
            auto load = [&](Tile &x, int i, int page) {
                const int t = i * kTile + lane;
                x.there = uint32_t(page) < uint32_t(c.pages);
                if (!x.there && i < end && t < row.length && r0 == 0) record(c, ESP_ERR_SHAPE);
                page = x.there ? page : 0;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const uint8_t *block = c.k + c.block(__builtin_amdgcn_readlane(page, 16 * j), a.layer, head);
                    const uint32_t at = uint32_t((16 * j + col) % Page * Dim + 16 * quarter);
#pragma unroll
                    for (int s = 0; s < Dim / 64; s++) x.codes[j][s] = *reinterpret_cast<const uint4v *>(block + (at + 64 * s));
                }
                x.scale = *c.block_scale(page, a.layer, 0, head) * a.scale;
                x.mass = x.there && (t < p0 || r0) ? mass[t] : 0.0f;
            };
            Tile now, next;
            int page = page_of(tile + 1);
            load(now, tile, page_of(tile));
            for (int i = tile; i < end; i++) {
                load(next, i + 1, page);
                page = page_of(i + 2);
                // whether all rows that there are see all of the tile
                const bool whole = i * kTile + kTile - 1 <= p0 && (a.window <= 0 || i * kTile > p0 + row.n - 1 - a.window);
                float own = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    float4v s[kBlocks];
#pragma unroll
                    for (int y = 0; y < kBlocks; y++) s[y] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < kSteps; k++) {
                        const uint4v w = now.codes[j][k / 2];
                        const V8 key = codes8<V8, V2>(w[k % 2 * 2], w[k % 2 * 2 + 1]);
#pragma unroll
                        for (int y = 0; y < kBlocks; y++) s[y] = product16(q[y][k], key, s[y]);
                    }
                    const float ks = __uint_as_float(uint32_t(__builtin_amdgcn_readlane(__float_as_uint(now.scale), 16 * j)));
                    const int t = i * kTile + 16 * j + col;
                    float sum = 0.0f;
#pragma unroll
                    for (int y = 0; y < kBlocks; y++)
#pragma unroll
                        for (int x = 0; x < 4; x++) {
                            const float e = weight(s[y][x], ks, lse[y][x]);
                            const int r = r0 + 16 * y + 4 * quarter + x, p = whole ? 0 : p0 + r / a.group;
                            sum += lse[y][x] != INFINITY && (whole || (t <= p && (a.window <= 0 || t > p - a.window))) ? e : 0.0f;
                        }
                    sum += __shfl_xor(sum, 16);
                    sum += __shfl_xor(sum, 32);
                    own = quarter == j ? sum : own;
                }
                if (now.there) mass[i * kTile + lane] = __builtin_fmaf(now.mass, r0 ? 1.0f : a.decay, own);
                now = next;
            }
        }
    }
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

// Rows (token, query head) a sequence and key head up to which k_weigh_few takes it, in
// rounds of 16 or 32.  So / by k_weigh, 64 sequences of about 3,800 tokens of 128: 48 rows of 4
// key heads 68 / 128 us, 96 rows 89 / 122, 128 rows 106 / 121, 192 rows 160 / 134.
constexpr int kFewRows = 128;
// Its wavefronts, as many as its registers allow at once: three a SIMD for rounds of 32 rows, four
// for 16.  2,048 / 4,096 / 8,192 of the latter: 59 / 54 / 55 us (weights of 64 single tokens of
// 32 heads on up to 8,192 cached ones, 8 key heads).
constexpr int kUnits = 1024, kFewWaves = 3 * kUnits, kFewestWaves = 4 * kUnits;           // kUnits: the GPU's SIMDs
// Workgroups of k_weigh, and of it where few sequences, if any, are its own: 64 single tokens whose
// bound allows more take 94 us beside it, 91 alone (8 key heads, up to 8,040 tokens of 128).
constexpr int kManyBlocks = 16384, kSomeBlocks = 1024;

// How a sequence is weighed: by the most rows that it may have.
enum Kind { kSixteens, kPairs, kMany };
Kind kind_of(int64_t rows) { return rows <= 16 ? kSixteens : rows <= kFewRows ? kPairs : kMany; }
constexpr int32_t kMostOf[] = {16, kFewRows, INT32_MAX};

template <typename T, int Dim, int Page> void launch(const WeighArgs &a, Kind kind, unsigned blocks, hipStream_t s) {
    if (kind == kMany) k_weigh<T, Dim, Page><<<blocks, kThreads * kGroups, 0, s>>>(a);
    else if (kind == kPairs) k_weigh_few<T, Dim, Page, 2><<<blocks, kThreads, 0, s>>>(a);
    else k_weigh_few<T, Dim, Page, 1><<<blocks, kThreads, 0, s>>>(a);
}
template <typename T, int Dim> void launch(const WeighArgs &a, Kind kind, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: launch<T, Dim, 16>(a, kind, blocks, s); break;
    case 32: launch<T, Dim, 32>(a, kind, blocks, s); break;
    default: launch<T, Dim, 64>(a, kind, blocks, s); break;
    }
}
template <typename T> void launch(const WeighArgs &a, Kind kind, unsigned blocks, hipStream_t s) {
    a.c.dim == 64 ? launch<T, 64>(a, kind, blocks, s) : launch<T, 128>(a, kind, blocks, s);
}

// The sequences of one kind; `alone`: no other launch has any.
int64_t shares_of(const WeighArgs &a, Kind kind, bool alone) {
    // shares of a head's tiles: one each where queries are many; else as many as the GPU holds wavefronts
    const int64_t tile = kind == kMany ? kWaves * 32 : 64, most = a.rows.rows * ((int64_t(a.max_length) + tile - 1) / tile);
    const int64_t fill = (kind == kMany ? alone ? kManyBlocks : kSomeBlocks : kind == kPairs ? kFewWaves : kFewestWaves) / a.c.heads + 1;
    return most > INT32_MAX ? -1 : most < fill ? most : fill;
}
esp_status weigh(WeighArgs a, Kind kind, bool alone, int32_t type, hipStream_t s) {
    a.shares = int32_t(shares_of(a, kind, alone));
    const int64_t workers = int64_t(a.shares) * a.c.heads, count = kind == kMany ? workers : (workers + kWaves - 1) / kWaves;
    if (type == ESP_KV_BF16) launch<__bf16>(a, kind, unsigned(count), s);
    else launch<_Float16>(a, kind, unsigned(count), s);
    return launched();
}

}  // namespace

extern "C" esp_status esp_kv_weigh(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                                   const int32_t *offsets, const int32_t *seqs, int32_t q_heads, esp_kv_view q, const float *lse,
                                   float scale, int32_t window, float decay, int32_t max_new, int32_t max_length, float *mass,
                                   void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (type != ESP_KV_BF16 && type != ESP_KV_FP16) return ESP_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || !std::isfinite(decay) || window < 0) return ESP_ERR_INVALID_ARG;
    if (layer < 0 || layer >= cache->layers || rows < 0 || tokens < 0 || tokens > INT32_MAX || max_new < 0 || max_length < 0) return ESP_ERR_SHAPE;
    if (q_heads < 1 || q_heads > 65536 || q_heads % cache->kv_heads) return ESP_ERR_SHAPE;
    if (rows == 0 || tokens == 0 || max_new == 0 || max_length == 0) return ESP_OK;
    if (!offsets || !q.data || !lse || !mass) return ESP_ERR_INVALID_ARG;
    const int32_t group = q_heads / cache->kv_heads;
    if (tokens * group > INT32_MAX - 8 * kStep) return ESP_ERR_SHAPE;
    // tokens of a sequence are counted in 32 bits, some tiles past the last
    const int64_t held = int64_t(cache->table_width) * cache->page_tokens, bound = max_length < held ? max_length : held;
    if (bound > INT32_MAX - 8 * kStep) return ESP_ERR_SHAPE;
    const bool wide = (reinterpret_cast<uintptr_t>(q.data) & 15) == 0 && q.token_stride % 8 == 0 && q.head_stride % 8 == 0;
    WeighArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, View{q.data, q.token_stride, q.head_stride}, lse, mass, scale, decay,
                layer, q_heads, group, window, max_new, max_length, 0, wide, 0, INT32_MAX};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    // what the caller allows a row, and the most that it has if no row is without any: where these are of
    // different kinds, each row goes to the lesser kind if it is of that, else to the greater.  One row of
    // 512 tokens among 511 empty ones, group 4, on 4,096: 52 us, 494 in the rounds of the lesser alone.
    const int64_t allowed = tokens < max_new ? tokens : max_new, even = tokens < rows ? 1 : tokens - rows + 1;
    const Kind least = kind_of((even < allowed ? even : allowed) * group);
    // four rounds of sixteens are no second launch's worth: 16 single tokens with a loose bound 22 / 25 us (64
    // sequences of 32 rows among empty ones 168 / 114)
    const Kind most = least == kSixteens && allowed * group <= 4 * 16 ? least : kind_of(allowed * group);
    if (shares_of(a, least, true) < 0) return ESP_ERR_SHAPE;
    if (least != most) {
        a.most = kMostOf[least];
        if (esp_status e = weigh(a, least, false, type, s)) return e;
        a.over = a.most;
        a.most = INT32_MAX;
    }
    return weigh(a, most, least == most, type, s);
}
