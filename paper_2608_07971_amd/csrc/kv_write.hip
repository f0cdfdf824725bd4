// Rotary positions, writing tokens into the paged 8-bit cache, reading them back.
#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kThreads = 256;

struct View {
    void *data;
    int64_t token, head;
};

// The row whose tokens hold token t: the last b with offsets[b] <= t.
__device__ __forceinline__ int row_at(const int32_t *offsets, int rows, int64_t t) {
    int lo = 0, hi = rows - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (offsets[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// ---------------------------------------------------------------------------
// Rotation.  y = m (a cos - b sin, a sin + b cos) for each pair.
// ---------------------------------------------------------------------------

// Elements of pair i of a head; pairs past the rotary part are neighbours that pass through.
__device__ __forceinline__ void pair_of(const Rope &r, int i, int &a, int &b) {
    const int half = r.rotary >> 1;
    const bool split = !r.interleaved && i < half;
    a = split ? i : 2 * i;
    b = split ? i + half : 2 * i + 1;
}

// One pair a thread: any strides and alignment.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_rotate_any(Rope r, View x, View out, const int32_t *positions,
                                                         int64_t tokens, int heads, int dim, float sign) {
    const int64_t pairs = tokens * heads * (dim / 2);
    for (int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x; u < pairs; u += int64_t(gridDim.x) * kThreads) {
        const int i = int(u % (dim / 2));
        const int64_t th = u / (dim / 2);
        const int h = int(th % heads);
        const int64_t t = th / heads;
        int a, b;
        pair_of(r, i, a, b);
        const T *p = static_cast<const T *>(x.data) + t * x.token + h * x.head;
        T *o = static_cast<T *>(out.data) + t * out.token + h * out.head;
        T va = p[a], vb = p[b];
        if (i < r.rotary / 2) {
            float c, s;
            cos_sin(double(positions[t]) * r.turns[i], c, s);
            c *= r.magnitude;
            s *= sign * r.magnitude;
            const float fa = float(va), fb = float(vb);
            va = T(__builtin_fmaf(fa, c, -(fb * s)));
            vb = T(__builtin_fmaf(fa, s, fb * c));
        }
        o[a] = va;
        o[b] = vb;
    }
}

template <typename T> struct Vec8 { T x[8]; };
template <typename T> __device__ __forceinline__ Vec8<T> load8(const T *p) {
    Vec8<T> v;
    const uint4v *q = reinterpret_cast<const uint4v *>(p);
    uint4v *w = reinterpret_cast<uint4v *>(v.x);
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; i++) w[i] = q[i];
    return v;
}
template <typename T> __device__ __forceinline__ void store8(T *p, const Vec8<T> &v) {
    uint4v *q = reinterpret_cast<uint4v *>(p);
    const uint4v *w = reinterpret_cast<const uint4v *>(v.x);
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; i++) q[i] = w[i];
}

// Eight pairs a thread (16 elements), for `per` heads in turn, so that the
// angles are worked out once for them.  Chunk c of a head: the pairs
// [8c, 8c + 8); chunks past the rotary part pass through.
template <typename T>
__device__ __forceinline__ void rotate_chunk(const Rope &r, const View &x, const View &out, int64_t t, int position,
                                             int head, int heads, int c, float sign) {
    const int half = r.rotary >> 1, i0 = 8 * c;
    const bool turn = i0 < half;
    float cs[8], sn[8];
    if (turn) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            cos_sin(double(position) * r.turns[i0 + j], cs[j], sn[j]);
            cs[j] *= r.magnitude;
            sn[j] *= sign * r.magnitude;
        }
    }
    const int a = turn && !r.interleaved ? i0 : 16 * c, b = turn && !r.interleaved ? i0 + half : 16 * c + 8;
    const T *p = static_cast<const T *>(x.data) + t * x.token + int64_t(head) * x.head;
    T *o = static_cast<T *>(out.data) + t * out.token + int64_t(head) * out.head;
    for (int h = 0; h < heads; h++, p += x.head, o += out.head) {
        Vec8<T> u = load8(p + a), v = load8(p + b);
        if (turn && r.interleaved) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                T &va = j < 4 ? u.x[2 * j] : v.x[2 * j - 8], &vb = j < 4 ? u.x[2 * j + 1] : v.x[2 * j - 7];
                const float fa = float(va), fb = float(vb);
                va = T(__builtin_fmaf(fa, cs[j], -(fb * sn[j])));
                vb = T(__builtin_fmaf(fa, sn[j], fb * cs[j]));
            }
        } else if (turn) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const float fa = float(u.x[j]), fb = float(v.x[j]);
                u.x[j] = T(__builtin_fmaf(fa, cs[j], -(fb * sn[j])));
                v.x[j] = T(__builtin_fmaf(fa, sn[j], fb * cs[j]));
            }
        }
        store8(o + a, u);
        store8(o + b, v);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_rotate(Rope r, View x, View out, const int32_t *positions, int64_t tokens,
                                                     int heads, int per, int chunks, float sign) {
    const int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t t = u / chunks;
    const int head = blockIdx.y * per;
    if (t >= tokens) return;
    rotate_chunk<T>(r, x, out, t, positions[t], head, min(per, heads - head), int(u - t * chunks), sign);
}

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

struct AppendArgs {
    Cache c;
    Rows rows;
    Rope rope;           // rotary = 0: none
    View k, v, q, q_out;
    int32_t layer, q_heads, units;
};

__device__ __forceinline__ float block_max(float x, float *lds) {
#pragma unroll
    for (int m = 32; m; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}

// The least exponent e with most <= 448 * 2^e (448 = 1.75 * 2^8), within +-100.
__device__ __forceinline__ float least_scale(float most) {
    const uint32_t b = __float_as_uint(most);
    int e = int(b >> 23) - 127 - ((b & 0x7fffff) <= 0x600000 ? 8 : 7);
    e = max(-100, min(100, e));
    return __uint_as_float(uint32_t(e + 127) << 23);
}

__device__ __forceinline__ uint32_t code2(float a, float b) {
    a = a == a ? fminf(fmaxf(a, -448.0f), 448.0f) : a;
    b = b == b ? fminf(fmaxf(b, -448.0f), 448.0f) : b;
    return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
}

// A workgroup writes one page's new tokens for one head, keys or values: the
// values stay in registers between the largest and the codes.
template <typename T, int Dim, int Page> __device__ void append_block(const AppendArgs &a, int unit, int head, int which) {
    constexpr int kPairs = Dim / 2, kStep = kThreads / kPairs, kRounds = (Page + kStep - 1) / kStep;
    __shared__ float lds[4];
    const Cache &c = a.c;
    // units: a row of n tokens touches at most n / Page + 2 pages
    int lo = 0, hi = a.rows.rows - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.rows.offsets[mid] / Page + 2 * mid <= unit) lo = mid;
        else hi = mid - 1;
    }
    const Row row = row_of(c, a.rows, lo);
    const int p0 = row.length - row.n, from = max(p0, 0);
    const int slot = from / Page + unit - (a.rows.offsets[lo] / Page + 2 * lo);
    if (row.n == 0 || unit < a.rows.offsets[lo] / Page + 2 * lo || int64_t(slot) * Page >= row.length) return;
    const int32_t page = c.table[int64_t(row.seq) * c.width + slot];
    if (page < 0 || page >= c.pages) {
        if (threadIdx.x == 0) record(c, ESP_ERR_SHAPE);
        return;
    }
    const int i = threadIdx.x % kPairs, t0 = threadIdx.x / kPairs;
    int ea = 2 * i, eb = 2 * i + 1;
    const bool turn = which == 0 && i < a.rope.rotary / 2;
    if (which == 0 && a.rope.rotary) pair_of(a.rope, i, ea, eb);
    const double turns = turn ? a.rope.turns[i] : 0.0;
    const View &x = which ? a.v : a.k;
    float va[kRounds], vb[kRounds], most = 0.0f;
#pragma unroll
    for (int k = 0; k < kRounds; k++) {
        const int p = slot * Page + t0 + k * kStep;
        va[k] = vb[k] = 0.0f;
        if (p >= from && p < row.length && t0 + k * kStep < Page) {
            const T *src = static_cast<const T *>(x.data) + int64_t(row.first + (p - p0)) * x.token + head * x.head;
            va[k] = float(src[ea]);
            vb[k] = float(src[eb]);
            if (turn) {
                float cs, sn;
                cos_sin(double(p) * turns, cs, sn);
                cs *= a.rope.magnitude;
                sn *= a.rope.magnitude;
                const float fa = va[k], fb = vb[k];
                va[k] = __builtin_fmaf(fa, cs, -(fb * sn));
                vb[k] = __builtin_fmaf(fa, sn, fb * cs);
            }
            const float ma = fabsf(va[k]), mb = fabsf(vb[k]);
            most = fmaxf(most, fmaxf(ma < INFINITY ? ma : 0.0f, mb < INFINITY ? mb : 0.0f));
        }
    }
    most = block_max(most, lds);
    float *place = c.block_scale(page, a.layer, which, head);
    const bool older = slot * Page < from;
    const float least = least_scale(most), was = *place, scale = older ? fmaxf(was, least) : least;
    uint8_t *block = (which ? c.v : c.k) + c.block(page, a.layer, head);
    const int ta = which ? ea * Page : ea, tb = which ? eb * Page : eb, step = which ? 1 : Dim;
    if (older && scale > was) {
        const float by = was / scale;
        for (int t = t0; slot * Page + t < from; t += kStep) {
            uint8_t *pa = block + ta + t * step, *pb = block + tb + t * step;
            const uint32_t w = uint32_t(*pa) | uint32_t(*pb) << 8;
            const half2 n = codes<false>(w, static_cast<half2 *>(nullptr));
            const uint32_t z = code2(float(n[0]) * by, float(n[1]) * by);
            *pa = uint8_t(z);
            *pb = uint8_t(z >> 8);
        }
    }
    __syncthreads();                                  // every thread has read the old scale
#pragma unroll
    for (int k = 0; k < kRounds; k++) {
        const int t = t0 + k * kStep, p = slot * Page + t;
        if (p >= from && p < row.length && t < Page) {
            const uint32_t z = code2(va[k] / scale, vb[k] / scale);
            block[ta + t * step] = uint8_t(z);
            block[tb + t * step] = uint8_t(z >> 8);
        }
    }
    if (threadIdx.x == 0) *place = scale;
}

// Workgroups [0, units * heads * 2) write; the others turn the queries.
template <typename T, int Dim, int Page> __global__ __launch_bounds__(kThreads) void k_append(AppendArgs a) {
    const int writers = a.units * a.c.heads * 2;
    int w = blockIdx.x;
    if (w < writers) {
        const int which = w & 1;
        w >>= 1;
        append_block<T, Dim, Page>(a, w / a.c.heads, w % a.c.heads, which);
        return;
    }
    constexpr int kChunks = Dim / 16;
    const int64_t u = int64_t(w - writers) * kThreads + threadIdx.x, th = u / kChunks;
    const int64_t t = th / a.q_heads;
    if (t >= a.rows.tokens) return;
    const int b = row_at(a.rows.offsets, a.rows.rows, t);
    const Row row = row_of(a.c, a.rows, b);
    rotate_chunk<T>(a.rope, a.q, a.q_out, t, row.length - row.n + int(t - row.first), int(th - t * a.q_heads), 1,
                    int(u % kChunks), 1.0f);
}

// ---------------------------------------------------------------------------
// Gather: eight values of one token and head a thread.
// ---------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kThreads) void k_gather(Cache c, Rows rows, const int32_t *starts, int layer, T *k, T *v) {
    const int chunks = c.dim / 8;
    const int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int d = int(u % chunks) * 8;
    const int64_t th = u / chunks;
    const int h = int(th % c.heads);
    const int64_t t = th / c.heads;
    if (t >= rows.tokens) return;
    const int b = row_at(rows.offsets, rows.rows, t);
    const Row row = row_of(c, rows, b);
    const int64_t p = int64_t(starts[b]) + (t - row.first);
    Vec8<T> ko{}, vo{};
    if (row.n > 0 && t >= row.first && t < row.first + row.n && p >= 0 && p < row.length) {
        const int32_t page = c.table[int64_t(row.seq) * c.width + (p >> c.shift)];
        if (page < 0 || page >= c.pages) {
            record(c, ESP_ERR_SHAPE);
        } else {
            const int at = int(p & (c.tokens - 1));
            const int64_t block = c.block(page, layer, h);
            const float sk = *c.block_scale(page, layer, 0, h), sv = *c.block_scale(page, layer, 1, h);
            const uint2v kw = *reinterpret_cast<const uint2v *>(c.k + block + int64_t(at) * c.dim + d);
            const half8 kn = codes8<half8, half2>(kw[0], kw[1]);
            const uint8_t *vp = c.v + block + int64_t(d) * c.tokens + at;
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; j++) w[j >> 2] |= uint32_t(vp[int64_t(j) * c.tokens]) << (8 * (j & 3));
            const half8 vn = codes8<half8, half2>(w[0], w[1]);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                ko.x[j] = T(float(kn[j]) * sk);
                vo.x[j] = T(float(vn[j]) * sv);
            }
        }
    }
    store8(k + th * c.dim + d, ko);
    store8(v + th * c.dim + d, vo);
}

}  // namespace esp_kv

// ---------------------------------------------------------------------------
// Entry points
// ---------------------------------------------------------------------------

using namespace esp_kv;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// Whether 16-byte accesses at multiples of 8 elements are aligned.
bool wide(const esp_kv_view &v, int size) {
    return aligned16(v.data) && (v.token_stride * size) % 16 == 0 && (v.head_stride * size) % 16 == 0;
}
View view_of(const esp_kv_view &v) { return {v.data, v.token_stride, v.head_stride}; }
Rope rope_of(const esp_kv_rope *r) { return r ? Rope{r->turns, r->magnitude, r->rotary_dim, r->interleaved} : Rope{nullptr, 1.0f, 0, 0}; }

esp_status check_rope(const esp_kv_rope *r, int32_t dim) {
    if (!r->turns || (r->interleaved != 0 && r->interleaved != 1) || !(r->magnitude == r->magnitude)) return ESP_ERR_INVALID_ARG;
    return r->rotary_dim >= 2 && r->rotary_dim % 2 == 0 && r->rotary_dim <= dim ? ESP_OK : ESP_ERR_SHAPE;
}

esp_status check_rows(int32_t rows, int64_t tokens, const int32_t *offsets) {
    if (rows < 0 || tokens < 0 || tokens > INT32_MAX) return ESP_ERR_SHAPE;
    return rows && tokens && !offsets ? ESP_ERR_INVALID_ARG : ESP_OK;
}

template <typename T>
void rotate(const Rope &r, View x, View out, const int32_t *positions, int64_t tokens, int heads, int dim, float sign,
            bool vector, hipStream_t s) {
    if (vector) {
        const int chunks = dim / 16, per = 4;
        const int64_t blocks = (tokens * chunks + kThreads - 1) / kThreads;
        k_rotate<T><<<dim3(unsigned(blocks), (heads + per - 1) / per), kThreads, 0, s>>>(r, x, out, positions, tokens, heads, per, chunks, sign);
    } else {
        const int64_t blocks = (tokens * heads * (dim / 2) + kThreads - 1) / kThreads;
        k_rotate_any<T><<<unsigned(blocks < 65536 ? blocks : 65536), kThreads, 0, s>>>(r, x, out, positions, tokens, heads, dim, sign);
    }
}

template <typename T, int Dim> void append(const AppendArgs &a, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: k_append<T, Dim, 16><<<blocks, kThreads, 0, s>>>(a); break;
    case 32: k_append<T, Dim, 32><<<blocks, kThreads, 0, s>>>(a); break;
    default: k_append<T, Dim, 64><<<blocks, kThreads, 0, s>>>(a); break;
    }
}

}  // namespace

extern "C" esp_status esp_kv_rope_turns(int32_t rotary_dim, double base, int32_t scaling, double factor, int32_t context,
                                        double *turns, float *magnitude) {
    if (!turns || !magnitude) return ESP_ERR_INVALID_ARG;
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 65536) return ESP_ERR_SHAPE;
    if (!(base > 1.0) || !std::isfinite(base) || scaling < ESP_KV_ROPE_NONE || scaling > ESP_KV_ROPE_PARTS) return ESP_ERR_INVALID_ARG;
    if (scaling != ESP_KV_ROPE_NONE && (!(factor >= 1.0) || !std::isfinite(factor))) return ESP_ERR_INVALID_ARG;
    if (scaling == ESP_KV_ROPE_NTK && rotary_dim < 4) return ESP_ERR_SHAPE;
    if (scaling == ESP_KV_ROPE_PARTS && context < 1) return ESP_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    if (scaling == ESP_KV_ROPE_NTK) base *= pow(factor, rotary_dim / (rotary_dim - 2.0));
    for (int32_t i = 0; i < rotary_dim / 2; i++) {
        double f = pow(base, -2.0 * i / rotary_dim);
        if (scaling == ESP_KV_ROPE_LINEAR) f /= factor;
        if (scaling == ESP_KV_ROPE_PARTS) {
            const double share = fmin(1.0, fmax(0.0, (f * context / two_pi - 1.0) / 31.0));
            f *= share + (1.0 - share) / factor;
        }
        turns[i] = f / two_pi;
    }
    *magnitude = scaling == ESP_KV_ROPE_PARTS ? float(0.1 * log(factor) + 1.0) : 1.0f;
    return ESP_OK;
}

extern "C" esp_status esp_kv_rotate(const esp_kv_rope *rope, int32_t type, int64_t tokens, int32_t heads, int32_t head_dim,
                                    esp_kv_view x, const int32_t *positions, int32_t inverse, esp_kv_view out, void *stream) {
    if (!rope || type < ESP_KV_BF16 || type > ESP_KV_FP32) return ESP_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > INT32_MAX || heads < 0 || heads > 65536 || head_dim < 2 || head_dim % 2 || head_dim > 65536) return ESP_ERR_SHAPE;
    if (esp_status e = check_rope(rope, head_dim)) return e;
    if (tokens == 0 || heads == 0) return ESP_OK;
    if (!x.data || !out.data || !positions) return ESP_ERR_INVALID_ARG;
    const int size = type == ESP_KV_FP32 ? 4 : 2;
    const bool vector = wide(x, size) && wide(out, size) && rope->rotary_dim % 16 == 0 && head_dim % 16 == 0;
    const float sign = inverse ? -1.0f : 1.0f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Rope r = rope_of(rope);
    const View vx = view_of(x), vo = view_of(out);
    if (type == ESP_KV_BF16) rotate<__bf16>(r, vx, vo, positions, tokens, heads, head_dim, sign, vector, s);
    else if (type == ESP_KV_FP16) rotate<_Float16>(r, vx, vo, positions, tokens, heads, head_dim, sign, vector, s);
    else rotate<float>(r, vx, vo, positions, tokens, heads, head_dim, sign, vector, s);
    return launched();
}

extern "C" esp_status esp_kv_append(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                                    const int32_t *offsets, const int32_t *seqs, esp_kv_view k, esp_kv_view v,
                                    const esp_kv_rope *rope, int32_t q_heads, esp_kv_view q, esp_kv_view q_out, void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (type != ESP_KV_BF16 && type != ESP_KV_FP16) return ESP_ERR_INVALID_ARG;
    if (layer < 0 || layer >= cache->layers || q_heads < 0 || q_heads > 65536) return ESP_ERR_SHAPE;
    if (esp_status e = check_rows(rows, tokens, offsets)) return e;
    if (rope) {
        if (esp_status e = check_rope(rope, cache->head_dim)) return e;
        if (rope->rotary_dim % 16) return ESP_ERR_SHAPE;
    }
    if (rows == 0 || tokens == 0) return ESP_OK;
    if (!k.data || !v.data || (q_heads && (!rope || !q.data || !q_out.data))) return ESP_ERR_INVALID_ARG;
    if (q_heads && !(wide(q, 2) && wide(q_out, 2))) return ESP_ERR_INVALID_ARG;
    const int64_t units = tokens / cache->page_tokens + 2 * int64_t(rows);
    const int64_t blocks = units * cache->kv_heads * 2 + (tokens * q_heads * (cache->head_dim / 16) + kThreads - 1) / kThreads;
    if (blocks > INT32_MAX) return ESP_ERR_SHAPE;
    const AppendArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, rope_of(rope), view_of(k), view_of(v), view_of(q), view_of(q_out),
                       layer, q_heads, int32_t(units)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == ESP_KV_BF16) cache->head_dim == 64 ? append<__bf16, 64>(a, unsigned(blocks), s) : append<__bf16, 128>(a, unsigned(blocks), s);
    else cache->head_dim == 64 ? append<_Float16, 64>(a, unsigned(blocks), s) : append<_Float16, 128>(a, unsigned(blocks), s);
    return launched();
}

extern "C" esp_status esp_kv_gather(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                                    const int32_t *offsets, const int32_t *seqs, const int32_t *starts, void *k_out, void *v_out,
                                    void *stream) {
    if (esp_status e = check_cache(cache)) return e;
    if (type != ESP_KV_BF16 && type != ESP_KV_FP16) return ESP_ERR_INVALID_ARG;
    if (layer < 0 || layer >= cache->layers) return ESP_ERR_SHAPE;
    if (esp_status e = check_rows(rows, tokens, offsets)) return e;
    if (rows == 0 || tokens == 0) return ESP_OK;
    if (!starts || !k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return ESP_ERR_INVALID_ARG;
    const int64_t blocks = (tokens * cache->kv_heads * (cache->head_dim / 8) + kThreads - 1) / kThreads;
    if (blocks > INT32_MAX) return ESP_ERR_SHAPE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Rows r{offsets, seqs, rows, tokens};
    if (type == ESP_KV_BF16) k_gather<__bf16><<<unsigned(blocks), kThreads, 0, s>>>(cache_of(cache), r, starts, layer, static_cast<__bf16 *>(k_out), static_cast<__bf16 *>(v_out));
    else k_gather<_Float16><<<unsigned(blocks), kThreads, 0, s>>>(cache_of(cache), r, starts, layer, static_cast<_Float16 *>(k_out), static_cast<_Float16 *>(v_out));
    return launched();
}
