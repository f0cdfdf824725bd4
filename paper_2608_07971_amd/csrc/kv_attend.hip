// Attention over the paged 8-bit cache.
#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 64;                   // tokens a wavefront takes at a time
constexpr int kCols = 16;                   // (token, query head) rows of a unit: the columns of the matrix products
constexpr float kLift = 14.0f;              // softmax weights are taken times 2^14, so that fp16 holds them down to 2^-38 of the largest
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kNoScale = -200;              // exponent of a value scale below any

struct View {
    void *data;
    int64_t token, head;
};

struct AttendArgs {
    Cache c;
    Rows rows;
    View q, out;
    float *lse;
    float scale;                            // softmax scale times log2 e
    int32_t layer, q_heads, group, window, max_new, max_length, target, wide;
    uint32_t *counters;
    float *partial;
};

// Tiles of tokens that queries at positions [p0, p1] see.
struct Span {
    int from, to;                           // tiles [from, to)
    __device__ __forceinline__ int size() const { return to > from ? to - from : 0; }
};
__device__ __forceinline__ Span span_of(int p0, int p1, int window) {
    if (p1 < 0) return {0, 0};
    const int first = window > 0 ? max(0, max(p0, 0) - window + 1) : 0;
    return {first / kTile, p1 / kTile + 1};
}

// One workgroup's work: tiles of a unit (16 rows of queries of one sequence
// and key head), and how the units of its row are numbered.
struct Plan {
    Row row;
    int unit, chunk, chunks, first, per;    // first: the chunk index of the unit's chunk 0; per: tiles a chunk
    bool any;
};

__device__ __forceinline__ Row usable_row(const AttendArgs &a, int b) {
    Row r{};
    if (b < a.rows.rows) {
        r = row_of(a.c, a.rows, b);
        if (r.n > a.max_new || r.length > a.max_length) {
            record(a.c, ESP_ERR_SHAPE);
            r.n = 0;
        }
    }
    return r;
}

// Work is cut into chunks of `per` tiles, `per` from the sum over all rows, so
// that ragged batches fill the GPU like even ones.  Every wavefront works the
// cut out for itself, a row a lane.
__device__ Plan plan_of(const AttendArgs &a, int index) {
    const int lane = threadIdx.x & 63;
    const int rows = a.rows.rows;
    int64_t total = 0, tokens = 0;
    for (int b = lane; b < rows; b += 64) {
        const Row r = usable_row(a, b);
        tokens += r.n;
        const int units = (r.n * a.group + kCols - 1) / kCols;
        total += int64_t(units) * span_of(r.length - r.n, r.length - 1, a.window).size();
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        total += __shfl_xor(total, m);
        tokens += __shfl_xor(tokens, m);
    }
    Plan p;
    p.any = false;
    if (tokens > a.rows.tokens) {           // rows that overlap: the launch has no room for them
        record(a.c, ESP_ERR_SHAPE);
        return p;
    }
    const int64_t share = (total + a.target - 1) / a.target;
    p.per = int((max(share, int64_t(kWaves)) + kWaves - 1) / kWaves * kWaves);
    int before = 0;
    for (int b0 = 0; b0 < rows; b0 += 64) {
        const Row r = usable_row(a, b0 + lane);
        const int units = (r.n * a.group + kCols - 1) / kCols;
        const int chunks = max(1, (span_of(r.length - r.n, r.length - 1, a.window).size() + p.per - 1) / p.per);
        int sum = units * chunks;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int v = __shfl_up(sum, m);
            sum += lane >= m ? v : 0;
        }
        const uint64_t past = __ballot(before + sum > index);
        if (past) {
            const int at = __builtin_ctzll(past);
            const int in_row = index - before - __shfl(sum - units * chunks, at);
            p.row = Row{__shfl(r.first, at), __shfl(r.n, at), __shfl(r.seq, at), __shfl(r.length, at)};
            p.chunks = __shfl(chunks, at);
            p.unit = in_row / p.chunks;
            p.chunk = in_row - p.unit * p.chunks;
            p.first = index - p.chunk;
            p.any = true;
            break;
        }
        before += __shfl(sum, 63);
    }
    return p;
}

// Maximum and sum over the four lanes that hold one column's tokens.
__device__ __forceinline__ float across_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float across_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ float4v product(half8 x, half8 y, float4v z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float4v product(bhalf8 x, bhalf8 y, float4v z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }

template <typename T> struct Pack;
template <> struct Pack<_Float16> { typedef half8 v8; typedef half2 v2; };
template <> struct Pack<__bf16> { typedef bhalf8 v8; typedef bhalf2 v2; };

// Bytes whose low seven bits are all set: e4m3's NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    const uint32_t hit = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return (hit >> 7) * 0xffu;
}

// A unit's running softmax: column n = lane % 16 of the transposed products,
// so that the statistics of a column lie in the lanes that hold it.
template <int Dim> struct Running {
    float4v o[Dim / 16];                    // row 16 dt + 4 (lane / 16) + i of out^T
    float m, l;                             // largest score (log 2), sum of weights: of this lane's tokens
    int e;                                  // out is held divided by 2^e
};

template <typename T, int Dim> __global__ __launch_bounds__(kThreads) void k_attend(AttendArgs a) {
    typedef typename Pack<T>::v8 V8;
    typedef typename Pack<T>::v2 V2;
    constexpr int kSteps = Dim / 32;        // matrix steps of a score
    constexpr int kTiles = Dim / 16;        // matrix tiles of an output
    constexpr int kPad = Dim + 4;
    __shared__ __align__(16) float so[kWaves][kCols][kPad];
    __shared__ float sm[kWaves][kCols], sl[kWaves][kCols];
    __shared__ int se[kWaves];
    __shared__ uint32_t ticket;

    const Cache &c = a.c;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
    const int head = blockIdx.x % c.heads;
    const Plan p = plan_of(a, blockIdx.x / c.heads);
    if (!p.any) return;
    const Row &row = p.row;

    // this lane's query: row r of the unit is (token r / group, query head r % group)
    const int n_rows = row.n * a.group, r0 = p.unit * kCols, r = r0 + col, p0 = row.length - row.n;
    const int token = r / a.group, q_head = head * a.group + r - token * a.group;
    const int pos = r < n_rows ? p0 + token : -1, low = a.window > 0 ? pos - a.window : -1;
    const int pos_first = p0 + r0 / a.group, pos_last = p0 + (min(r0 + kCols, n_rows) - 1) / a.group;
    Span span = span_of(pos_first, pos_last, a.window);
    span.from += p.chunk * p.per;
    span.to = min(span.to, span.from + p.per);

    V8 q[kSteps];
    {
        const T *src = static_cast<const T *>(a.q.data) + int64_t(row.first + token) * a.q.token + int64_t(q_head) * a.q.head + quad * (Dim / 4);
#pragma unroll
        for (int s = 0; s < kSteps; s++) {
            V8 x{};
            if (r < n_rows) {
                if (a.wide) x = *reinterpret_cast<const V8 *>(src + 8 * s);
                else
#pragma unroll
                    for (int j = 0; j < 8; j++) x[j] = src[8 * s + j];
            }
            q[s] = x;
        }
    }

    Running<Dim> u;
#pragma unroll
    for (int d = 0; d < kTiles; d++) u.o[d] = float4v{0, 0, 0, 0};
    u.m = -INFINITY;
    u.l = 0.0f;
    u.e = kNoScale;

    const int32_t *table = c.table + int64_t(row.seq) * c.width;
    const int in_page = c.tokens - 1;
    const int k_group = col >> 2;           // keys: matrix row 4 k_group + i of tile j is token 16 k_group + 4 j + i
    for (int t = span.from + wave; t < span.to; t += kWaves) {
        const int at_k = t * kTile + 16 * k_group, at_v = t * kTile + 16 * quad;
        int page_k = at_k < row.length ? table[at_k >> c.shift] : -1, page_v = at_v < row.length ? table[at_v >> c.shift] : -1;
        const bool ok = page_v >= 0 && page_v < c.pages;
        if (!ok && at_v < row.length && col == 0) record(c, ESP_ERR_SHAPE);
        if (page_k < 0 || page_k >= c.pages) page_k = 0;       // read something; it is masked below
        if (!ok) page_v = 0;
        const uint8_t *kp = c.k + c.block(page_k, a.layer, head) + ((at_k & in_page) + (col & 3)) * Dim + quad * (Dim / 4);
        const uint8_t *vp = c.v + c.block(page_v, a.layer, head) + (col << c.shift) + (at_v & in_page);
        uint4v kw[4][Dim / 64], vw[kTiles];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int s = 0; s < Dim / 64; s++) kw[j][s] = *reinterpret_cast<const uint4v *>(kp + 4 * j * Dim + 16 * s);
#pragma unroll
        for (int d = 0; d < kTiles; d++) vw[d] = *reinterpret_cast<const uint4v *>(vp + (d << (4 + c.shift)));
        const float k_scale = *c.block_scale(page_v, a.layer, 0, head) * a.scale, v_scale = *c.block_scale(page_v, a.layer, 1, head);

        float4v s[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            s[j] = float4v{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < kSteps; k++) {
                const uint4v w = kw[j][k >> 1];
                s[j] = product(codes8<V8, V2>(w[2 * (k & 1)], w[2 * (k & 1) + 1]), q[k], s[j]);
            }
        }
        const bool whole = t * kTile + kTile - 1 <= pos_first && (a.window <= 0 || t * kTile > pos_last - a.window) && __all(ok);
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int tt = at_v + 4 * j + i;
                s[j][i] = whole || (tt <= pos && tt > low && ok) ? s[j][i] * k_scale : -INFINITY;
                top = fmaxf(top, s[j][i]);
            }
        top = across_max(top);
        if (__any(top > u.m)) {
            const float m = fmaxf(u.m, top), by = u.m == m ? 1.0f : __builtin_amdgcn_exp2f(u.m - m);
            u.m = m;
            u.l *= by;
#pragma unroll
            for (int d = 0; d < kTiles; d++) u.o[d] *= by;
        }
        const float base = u.m == -INFINITY ? 0.0f : u.m - kLift;
        // value scales relative to the largest so far, so that fp16 holds weight * scale
        int e = max(-126, min(126, int((__float_as_uint(v_scale) >> 23) & 255) - 127));
        e = ok ? e : kNoScale;
        e = max(e, __shfl_xor(e, 16));
        e = max(e, __shfl_xor(e, 32));
        if (e > u.e) {
            const float by = ldexpf(1.0f, max(u.e - e, -200));
#pragma unroll
            for (int d = 0; d < kTiles; d++) u.o[d] *= by;
            u.e = e;
        }
        const float v_rel = ldexpf(v_scale, -u.e);
        half8 w[2], seen[2];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int tt = at_v + 4 * j + i;
                const bool vis = whole || (tt <= pos && tt > low && ok);
                const float x = __builtin_amdgcn_exp2f(s[j][i] - base);
                u.l += x;
                w[j >> 1][4 * (j & 1) + i] = vis ? _Float16(x * v_rel) : _Float16(0.0f);
                seen[j >> 1][4 * (j & 1) + i] = vis ? _Float16(1.0f) : _Float16(0.0f);
            }
        if (!whole) {
            // tokens past the end hold anything: their codes become 0.  A NaN that
            // only some rows see must not reach the others through 0 * NaN.
            const int held = ok ? max(0, min(16, row.length - at_v)) : 0;
            uint32_t nans = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int left = held - 4 * i;
                const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
                for (int d = 0; d < kTiles; d++) {
                    vw[d][i] &= keep;
                    nans |= nan_bytes(vw[d][i]);
                }
            }
            if (__any(nans != 0)) {
#pragma unroll
                for (int d = 0; d < kTiles; d++) {
                    float4v hit{0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 2; k++) {
                        const uint32_t x = nan_bytes(vw[d][2 * k]), y = nan_bytes(vw[d][2 * k + 1]);
                        hit = product(codes8<half8, half2>(x & 0x38383838u, y & 0x38383838u), seen[k], hit);
                        vw[d][2 * k] &= ~x;
                        vw[d][2 * k + 1] &= ~y;
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (hit[i] > 0.0f) u.o[d][i] = NAN;
                }
            }
        }
#pragma unroll
        for (int d = 0; d < kTiles; d++)
#pragma unroll
            for (int k = 0; k < 2; k++) u.o[d] = product(codes8<half8, half2>(vw[d][2 * k], vw[d][2 * k + 1]), w[k], u.o[d]);
    }

    // join the wavefronts
    u.l = across_sum(u.l);
#pragma unroll
    for (int d = 0; d < kTiles; d++) *reinterpret_cast<float4v *>(&so[wave][col][16 * d + 4 * quad]) = u.o[d];
    if (quad == 0) {
        sm[wave][col] = u.m;
        sl[wave][col] = u.l;
    }
    if (lane == 0) se[wave] = u.e;
    __syncthreads();
    constexpr int kMine = Dim / 16;         // values of a row a thread finishes
    const int n = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kMine, rn = r0 + n;
    float m = -INFINITY, l = 0.0f, o[kMine];
    int e = kNoScale;
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
        m = fmaxf(m, sm[w][n]);
        e = max(e, se[w]);
    }
#pragma unroll
    for (int i = 0; i < kMine; i++) o[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
        const float f = sm[w][n] == m ? 1.0f : __builtin_amdgcn_exp2f(sm[w][n] - m), g = f * ldexpf(1.0f, max(se[w] - e, -200));
        l = __builtin_fmaf(sl[w][n], f, l);
#pragma unroll
        for (int i = 0; i < kMine; i++) o[i] = __builtin_fmaf(so[w][n][d0 + i], g, o[i]);
    }
    const bool none = m == -INFINITY && !(l != l);
    float lse = none ? -INFINITY : m - kLift + __builtin_log2f(l);
#pragma unroll
    for (int i = 0; i < kMine; i++) o[i] = none ? 0.0f : ldexpf(o[i] / l, e);

    if (p.chunks > 1) {
        // every chunk leaves its part; the last to arrive joins them in order
        float *mine = a.partial + (int64_t(p.first + p.chunk) * c.heads + head) * (kCols * (Dim + 1));
        if (rn < n_rows) {
#pragma unroll
            for (int i = 0; i < kMine; i++) mine[n * Dim + d0 + i] = o[i];
            if (d0 == 0) mine[kCols * Dim + n] = lse;
        }
        __threadfence();
        __syncthreads();
        uint32_t *counter = a.counters + int64_t(p.first) * c.heads + head;
        if (threadIdx.x == 0) ticket = atomicAdd(counter, 1u);
        __syncthreads();
        if (ticket != uint32_t(p.chunks) - 1) return;
        __threadfence();
        if (threadIdx.x == 0) *counter = 0;
        const float *parts = a.partial + (int64_t(p.first) * c.heads + head) * (kCols * (Dim + 1));
        const int64_t step = int64_t(c.heads) * (kCols * (Dim + 1));
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int i = 0; i < kMine; i++) o[i] = 0.0f;
        if (rn < n_rows) {
            bool nan = false;
            for (int k = 0; k < p.chunks; k++) {
                const float x = parts[k * step + kCols * Dim + n];
                nan |= x != x;
                m = fmaxf(m, x);
            }
            for (int k = 0; k < p.chunks; k++) {
                const float x = parts[k * step + kCols * Dim + n], f = x == -INFINITY ? 0.0f : x == m ? 1.0f : __builtin_amdgcn_exp2f(x - m);
                l += f;
#pragma unroll
                for (int i = 0; i < kMine; i++) o[i] = __builtin_fmaf(parts[k * step + n * Dim + d0 + i], f, o[i]);
            }
            if (nan) l = NAN;
        }
        const bool empty = m == -INFINITY && !(l != l);
        lse = empty ? -INFINITY : m + __builtin_log2f(l);
#pragma unroll
        for (int i = 0; i < kMine; i++) o[i] = empty ? 0.0f : o[i] / l;
    }
    if (rn >= n_rows) return;
    const int tok = row.first + rn / a.group, qh = head * a.group + rn % a.group;
    T *dst = static_cast<T *>(a.out.data) + int64_t(tok) * a.out.token + int64_t(qh) * a.out.head + d0;
#pragma unroll
    for (int i = 0; i < kMine; i++) dst[i] = T(o[i]);
    if (d0 == 0 && a.lse) a.lse[int64_t(tok) * a.q_heads + qh] = lse * kLn2;
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

// Chunks that all heads together are cut into: three workgroups of four
// wavefronts fit a compute unit, 256 units.
constexpr int kChunksWanted = 768;

struct Shape {
    int32_t target;
    int64_t chunks;                          // bound on the chunks of one head
    size_t counters, bytes;
};
esp_status shape_of(const esp_kv_cache *c, int32_t rows, int64_t tokens, int32_t q_heads, int32_t max_new, int32_t max_length, Shape &s) {
    if (rows < 0 || tokens < 0 || tokens > INT32_MAX || max_new < 0 || max_length < 0) return ESP_ERR_SHAPE;
    if (q_heads < 1 || q_heads > 65536 || q_heads % c->kv_heads) return ESP_ERR_SHAPE;
    const int64_t group = q_heads / c->kv_heads;
    if (int64_t(max_new) * group > INT32_MAX / 2) return ESP_ERR_SHAPE;
    s.target = kChunksWanted / c->kv_heads > 1 ? kChunksWanted / c->kv_heads : 1;
    const int64_t by_tokens = tokens * group / kCols + rows, by_rows = int64_t(rows) * ((int64_t(max_new) * group + kCols - 1) / kCols);
    s.chunks = (by_tokens < by_rows ? by_tokens : by_rows) + s.target;
    if (s.chunks * c->kv_heads > INT32_MAX) return ESP_ERR_SHAPE;
    s.counters = (size_t(s.chunks) * c->kv_heads * 4 + 255) / 256 * 256;
    s.bytes = s.counters + size_t(s.chunks) * c->kv_heads * kCols * (c->head_dim + 1) * 4;
    return ESP_OK;
}

}  // namespace

extern "C" esp_status esp_kv_attend_workspace(const esp_kv_cache *cache, int32_t rows, int64_t tokens, int32_t q_heads, int32_t max_new,
                                              int32_t max_length, size_t *bytes) {
    if (esp_status e = check_cache(cache)) return e;
    if (!bytes) return ESP_ERR_INVALID_ARG;
    Shape s;
    if (esp_status e = shape_of(cache, rows, tokens, q_heads, max_new, max_length, s)) return e;
    *bytes = s.bytes;
    return ESP_OK;
}

extern "C" esp_status esp_kv_attend(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                                    const int32_t *offsets, const int32_t *seqs, int32_t q_heads, esp_kv_view q, float scale, int32_t window,
                                    int32_t max_new, int32_t max_length, esp_kv_view out, float *lse, void *workspace, size_t workspace_bytes,
                                    void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (type != ESP_KV_BF16 && type != ESP_KV_FP16) return ESP_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || window < 0) return ESP_ERR_INVALID_ARG;
    if (layer < 0 || layer >= cache->layers) return ESP_ERR_SHAPE;
    Shape s;
    if (esp_status e = shape_of(cache, rows, tokens, q_heads, max_new, max_length, s)) return e;
    if (rows == 0 || tokens == 0) return ESP_OK;
    if (!offsets || !q.data || !out.data) return ESP_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < s.bytes) return ESP_ERR_WORKSPACE;
    const bool wide = (reinterpret_cast<uintptr_t>(q.data) & 15) == 0 && q.token_stride % 8 == 0 && q.head_stride % 8 == 0;
    const AttendArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, View{q.data, q.token_stride, q.head_stride},
                       View{out.data, out.token_stride, out.head_stride}, lse, scale * kLog2e, layer, q_heads, q_heads / cache->kv_heads,
                       window, max_new, max_length, s.target, wide, static_cast<uint32_t *>(workspace),
                       reinterpret_cast<float *>(static_cast<char *>(workspace) + s.counters)};
    const hipStream_t h = static_cast<hipStream_t>(stream);
    const unsigned blocks = unsigned(s.chunks * cache->kv_heads);
    if (type == ESP_KV_BF16) cache->head_dim == 64 ? k_attend<__bf16, 64><<<blocks, kThreads, 0, h>>>(a) : k_attend<__bf16, 128><<<blocks, kThreads, 0, h>>>(a);
    else cache->head_dim == 64 ? k_attend<_Float16, 64><<<blocks, kThreads, 0, h>>>(a) : k_attend<_Float16, 128><<<blocks, kThreads, 0, h>>>(a);
    return launched();
}
