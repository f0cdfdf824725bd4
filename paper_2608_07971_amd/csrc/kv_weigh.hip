// The attention weight that cached tokens get from a call's queries:
//   mass[t] = decay mass[t] + sum over queries that see t of exp(scale q . k_t - lse[q])
// for each sequence and key head; tokens that are new begin at 0.
#include "kv_internal.hpp"

namespace esp_kv {

typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 32;                   // (token, query head) rows of a matrix tile
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
};

__device__ __forceinline__ float16v product32(half8 x, half8 y, float16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float16v product32(bhalf8 x, bhalf8 y, float16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }
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
    if (r.n == 0) r.length = 0;
    return r;
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// A wavefront has kCols times 32 cached tokens, which stay in registers as the
// columns of the products; the queries that see them go by, 32 rows at a time,
// through LDS for all four wavefronts.  So a token's sum is its lane's own, and
// no two workgroups add to the same place.
template <typename T, int Dim, int Page, int kCols> __global__ __launch_bounds__(kThreads) void k_weigh(WeighArgs a) {
    typedef typename Pack<T>::v8 V8;
    typedef typename Pack<T>::v2 V2;
    constexpr int kSteps = Dim / 16, kTile = kWaves * 32 * kCols, kRowBytes = Dim * 2;
    constexpr int kChunks = kRows * Dim / 8 / kThreads;          // 16-byte chunks of a tile of queries a thread stages
    __shared__ __align__(16) uint8_t queries[2][kRows * kRowBytes];
    __shared__ __align__(16) float lses[2][kRows];
    __shared__ __align__(16) int places[2][kRows];
    __shared__ int sums[kWaves], found[2];

    const Cache &c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int head = blockIdx.x / a.shares, share = blockIdx.x - head * a.shares;

    // the head's tiles in order of rows: this workgroup's share of them
    auto tiles_of = [&](int b, bool note) { return b < a.rows.rows ? (usable(a, b, note).length + kTile - 1) / kTile : 0; };
    int all = 0;
    for (int b = tid; b < a.rows.rows; b += kThreads) all += tiles_of(b, blockIdx.x == 0);
    all = wave_sum(all);
    if (lane == 0) sums[wave] = all;
    __syncthreads();
    all = sums[0] + sums[1] + sums[2] + sums[3];
    const int each = (all + a.shares - 1) / a.shares, begin = share * each, end = min(all, begin + each);
    if (begin >= end) return;
    if (tid == 0) found[0] = -1;
    for (int b0 = 0, before = 0; before <= begin && b0 < a.rows.rows; b0 += kThreads) {
        const int own = tiles_of(b0 + tid, false);
        int at = own;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int v = __shfl_up(at, m);
            at += lane >= m ? v : 0;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = at;
        __syncthreads();
        for (int w = 0; w < wave; w++) at += sums[w];
        at += before;                       // tiles up to this row's last
        if (begin < at && begin >= at - own) {
            found[0] = b0 + tid;
            found[1] = begin - (at - own);
        }
        before += sums[0] + sums[1] + sums[2] + sums[3];
    }
    __syncthreads();
    int b = __builtin_amdgcn_readfirstlane(found[0]), tile = __builtin_amdgcn_readfirstlane(found[1]);
    if (b < 0) return;                      // lengths that changed under the call

    auto turn = [](int row) { return Dim == 128 ? row & 15 : (row >> 1) & 7; };
    for (int left = end - begin; left > 0; left--, tile++) {
        Row row = usable(a, b, false);
        while (tile * kTile >= row.length) {
            if (++b >= a.rows.rows) return;
            tile = 0;
            row = usable(a, b, false);
        }
        const int p0 = row.length - row.n, n_rows = row.n * a.group, t0 = tile * kTile;
        // rows that may see a token of the tile
        const int t1 = min(row.length, t0 + kTile) - 1;
        int r_from = max(0, t0 - p0) * a.group / kRows * kRows, r_to = n_rows;
        if (a.window > 0) r_to = int(min(int64_t(n_rows), max(int64_t(0), int64_t(t1) + a.window - p0) * a.group));

        int page[kCols];
        float ks[kCols], sum[kCols];
        V8 k[kCols][kSteps];
#pragma unroll
        for (int j = 0; j < kCols; j++) {
            const int t = t0 + (wave * kCols + j) * 32 + col;
            page[j] = t < row.length ? c.table[int64_t(row.seq) * c.width + t / Page] : -1;
            if (t < row.length && (page[j] < 0 || page[j] >= c.pages)) {
                record(c, ESP_ERR_SHAPE);
                page[j] = -1;
            }
            sum[j] = 0.0f;
        }
        if (r_from < r_to) {
#pragma unroll
            for (int j = 0; j < kCols; j++) {
                const int t = t0 + (wave * kCols + j) * 32 + col, p = max(page[j], 0);
                const uint8_t *from = c.k + c.block(p, a.layer, head) + t % Page * Dim + 16 * half;
                ks[j] = *c.block_scale(p, a.layer, 0, head) * a.scale;
                uint4v w[kSteps / 2];
#pragma unroll
                for (int s = 0; s < kSteps / 2; s++) w[s] = *reinterpret_cast<const uint4v *>(from + 32 * s);
#pragma unroll
                for (int s = 0; s < kSteps / 2; s++) {
                    k[j][2 * s] = codes8<V8, V2>(w[s][0], w[s][1]);
                    k[j][2 * s + 1] = codes8<V8, V2>(w[s][2], w[s][3]);
                }
            }
            // a tile of queries on its way: through registers into LDS
            V8 next[kChunks];
            float next_lse = 0.0f;
            int next_place = -1;
            auto load = [&](int r0) {
#pragma unroll
                for (int i = 0; i < kChunks; i++) {
                    const int u = tid + i * kThreads, r = r0 + u / (Dim / 8), d = u % (Dim / 8) * 8;
                    V8 x{};
                    if (r < n_rows) {
                        const int token = r / a.group, h = head * a.group + r - token * a.group;
                        const T *src = static_cast<const T *>(a.q.data) + int64_t(row.first + token) * a.q.token + int64_t(h) * a.q.head + d;
                        if (a.wide) x = *reinterpret_cast<const V8 *>(src);
                        else
#pragma unroll
                            for (int e = 0; e < 8; e++) x[e] = src[e];
                    }
                    next[i] = x;
                }
                if (tid < kRows) {
                    const int r = r0 + tid, token = r / a.group;
                    next_lse = INFINITY;
                    next_place = -1;
                    if (r < n_rows) {
                        const float l = a.lse[int64_t(row.first + token) * a.q_heads + head * a.group + r - token * a.group];
                        next_lse = l == -INFINITY ? INFINITY : l;            // it sees nothing
                        next_place = p0 + token;
                    }
                }
            };
            load(r_from);
            for (int r0 = r_from; r0 < r_to; r0 += kRows) {
                const int buffer = (r0 / kRows) & 1;
#pragma unroll
                for (int i = 0; i < kChunks; i++) {
                    const int u = tid + i * kThreads, r = u / (Dim / 8), chunk = u % (Dim / 8);
                    *reinterpret_cast<V8 *>(&queries[buffer][r * kRowBytes + ((chunk ^ turn(r)) << 4)]) = next[i];
                }
                if (tid < kRows) {
                    lses[buffer][tid] = next_lse;
                    places[buffer][tid] = next_place;
                }
                __syncthreads();
                if (r0 + kRows < r_to) load(r0 + kRows);
                float16v s[kCols];
#pragma unroll
                for (int j = 0; j < kCols; j++)
#pragma unroll
                    for (int i = 0; i < 16; i++) s[j][i] = 0.0f;
                // half h's steps 2 i and 2 i + 1: elements 32 i + 16 h and on, as the keys were loaded
#pragma unroll
                for (int i = 0; i < kSteps; i++) {
                    const int chunk = i / 2 * 4 + 2 * half + i % 2;
                    const V8 q = *reinterpret_cast<const V8 *>(&queries[buffer][col * kRowBytes + ((chunk ^ turn(col)) << 4)]);
#pragma unroll
                    for (int j = 0; j < kCols; j++) s[j] = product32(q, k[j][i], s[j]);
                }
                const int first = p0 + r0 / a.group, last = p0 + min(r0 + kRows, n_rows) / a.group;
                const int w0 = t0 + wave * kCols * 32, w1 = w0 + kCols * 32 - 1;
                const bool whole = r0 + kRows <= n_rows && w1 <= first && (a.window <= 0 || w0 > last - a.window);
#pragma unroll
                for (int y = 0; y < 4; y++) {            // s[4 y + x]: row 8 y + 4 half + x
                    const float4v l = *reinterpret_cast<const float4v *>(&lses[buffer][8 * y + 4 * half]);
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < kCols; j++)
#pragma unroll
                            for (int x = 0; x < 4; x++) sum[j] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][4 * y + x], ks[j], -l[x]) * kLog2e);
                    } else {
                        const int *at = &places[buffer][8 * y + 4 * half];
#pragma unroll
                        for (int j = 0; j < kCols; j++) {
                            const int t = w0 + j * 32 + col;
#pragma unroll
                            for (int x = 0; x < 4; x++) {
                                const bool seen = t <= at[x] && (a.window <= 0 || t > at[x] - a.window);
                                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][4 * y + x], ks[j], -l[x]) * kLog2e);
                                sum[j] += seen ? e : 0.0f;
                            }
                        }
                    }
                }
            }
            __syncthreads();                // the next tile's queries go into the same places
        }
        float *mass = a.mass + ((int64_t(a.layer) * c.sequences + row.seq) * c.heads + head) * (int64_t(c.width) * Page);
#pragma unroll
        for (int j = 0; j < kCols; j++) {
            const int t = t0 + (wave * kCols + j) * 32 + col;
            const float got = sum[j] + __shfl_xor(sum[j], 32);
            if (half == 0 && t < row.length && page[j] >= 0) mass[t] = t < p0 ? __builtin_fmaf(mass[t], a.decay, got) : got;
        }
    }
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

constexpr int64_t kMostBlocks = ((int64_t(1) << 32) - kThreads) / kThreads;    // a launch's threads are numbered in 32 bits

template <typename T, int Dim, int kCols> void launch(const WeighArgs &a, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: k_weigh<T, Dim, 16, kCols><<<blocks, kThreads, 0, s>>>(a); break;
    case 32: k_weigh<T, Dim, 32, kCols><<<blocks, kThreads, 0, s>>>(a); break;
    default: k_weigh<T, Dim, 64, kCols><<<blocks, kThreads, 0, s>>>(a); break;
    }
}
template <typename T> void launch(const WeighArgs &a, bool many, unsigned blocks, hipStream_t s) {
    if (a.c.dim == 64) many ? launch<T, 64, 2>(a, blocks, s) : launch<T, 64, 1>(a, blocks, s);
    else many ? launch<T, 128, 2>(a, blocks, s) : launch<T, 128, 1>(a, blocks, s);
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
    if (tokens * group > INT32_MAX - kRows) return ESP_ERR_SHAPE;
    const bool many = int64_t(max_new) * group > kRows;
    const int64_t tile = kWaves * 32 * (many ? 2 : 1), most = rows * ((int64_t(max_length) + tile - 1) / tile);
    if (most > INT32_MAX) return ESP_ERR_SHAPE;
    const int64_t fill = (many ? 16384 : 4096) / cache->kv_heads + 1, shares = most < fill ? most : fill;
    if (shares * cache->kv_heads > kMostBlocks) return ESP_ERR_SHAPE;
    const bool wide = (reinterpret_cast<uintptr_t>(q.data) & 15) == 0 && q.token_stride % 8 == 0 && q.head_stride % 8 == 0;
    const WeighArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, View{q.data, q.token_stride, q.head_stride}, lse, mass, scale, decay,
                      layer, q_heads, group, window, max_new, max_length, int32_t(shares), wide};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned blocks = unsigned(shares * cache->kv_heads);
    if (type == ESP_KV_BF16) launch<__bf16>(a, many, blocks, s);
    else launch<_Float16>(a, many, blocks, s);
    return launched();
}
