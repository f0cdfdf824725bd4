// Rotary positions, writing tokens into the paged 8-bit cache, reading them back.
#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kThreads = 256;

struct View {
    void *data;
    int64_t token, head;
};

// How many b in [0, rows) have f(b) <= x, f ascending: 64 at a time by the lanes of a wavefront.
template <typename F> __device__ __forceinline__ int count_up_to(int rows, int64_t x, F f) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int b0 = 0; b0 < rows; b0 += 256) {          // four loads in flight
        int held = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) {
            const int b = b0 + 64 * k + lane;
            held += __popcll(__ballot(b < rows && f(b) <= x));
        }
        n += held;
        if (held < 256) break;
    }
    return n;
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
template <typename T> __device__ __forceinline__ void store8(T *p, const Vec8<T> &v) {
    uint4v *q = reinterpret_cast<uint4v *>(p);
    const uint4v *w = reinterpret_cast<const uint4v *>(v.x);
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; i++) q[i] = w[i];
}

// Two 16-byte vectors of a head a thread, for up to kPer heads, so that the
// angles are worked out once for them and their loads are in flight together.
// Neighbouring threads take neighbouring vectors: with halves thread c has
// vectors c and c + n of the turned part's 2 n (a pair's two sides), with
// neighbours as pairs the same vectors, each with pairs of its own; then the
// same of the part that passes through.
// Stream: what is read is not read again soon, and is read past the caches.
// Bound by memory: 403 MB (16,383 tokens, 24 heads of 128 in float32) take 75 us
// at the kernel (5.4 TB/s).
constexpr int kRotateHeads = 4, kAppendHeads = 2;
template <typename T, int kPer, bool Stream>
__device__ __forceinline__ void rotate_chunk(const Rope &r, const View &x, const View &out, int64_t t, int position,
                                             int head, int heads, int dim, int c, float sign) {
    constexpr int kVec = 16 / sizeof(T);
    union Vec {
        uint4v w;
        T x[kVec];
    };
    const int turned = r.rotary / (2 * kVec), rest = dim / (2 * kVec) - turned;
    const bool turn = c < turned;
    const int a = (turn ? c : c + turned) * kVec, b = a + (turn ? turned : rest) * kVec;
    const T *p = static_cast<const T *>(x.data) + t * x.token + int64_t(head) * x.head;
    T *o = static_cast<T *>(out.data) + t * out.token + int64_t(head) * out.head;
    Vec u[kPer], v[kPer];
#pragma unroll
    for (int h = 0; h < kPer; h++) {
        const T *from = p + min(h, heads - 1) * x.head;
        const uint4v *pa = reinterpret_cast<const uint4v *>(from + a), *pb = reinterpret_cast<const uint4v *>(from + b);
        u[h].w = Stream ? __builtin_nontemporal_load(pa) : *pa;
        v[h].w = Stream ? __builtin_nontemporal_load(pb) : *pb;
    }
    if (turn) {
        float cs[kVec], sn[kVec];
#pragma unroll
        for (int j = 0; j < kVec; j++) {
            const int i = !r.interleaved ? a + j : j < kVec / 2 ? a / 2 + j : b / 2 + j - kVec / 2;
            cos_sin(double(position) * r.turns[i], cs[j], sn[j]);
            cs[j] *= r.magnitude;
            sn[j] *= sign * r.magnitude;
        }
        auto pair = [](T &ya, T &yb, float cs, float sn) {
            const float fa = float(ya), fb = float(yb);
            ya = T(__builtin_fmaf(fa, cs, -(fb * sn)));
            yb = T(__builtin_fmaf(fa, sn, fb * cs));
        };
        if (r.interleaved) {
#pragma unroll
            for (int h = 0; h < kPer; h++)
#pragma unroll
                for (int j = 0; j < kVec / 2; j++) {
                    pair(u[h].x[2 * j], u[h].x[2 * j + 1], cs[j], sn[j]);
                    pair(v[h].x[2 * j], v[h].x[2 * j + 1], cs[j + kVec / 2], sn[j + kVec / 2]);
                }
        } else {
#pragma unroll
            for (int h = 0; h < kPer; h++)
#pragma unroll
                for (int j = 0; j < kVec; j++) pair(u[h].x[j], v[h].x[j], cs[j], sn[j]);
        }
    }
#pragma unroll
    for (int h = 0; h < kPer; h++)
        if (h < heads) {
            *reinterpret_cast<uint4v *>(o + h * out.head + a) = u[h].w;
            *reinterpret_cast<uint4v *>(o + h * out.head + b) = v[h].w;
        }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_rotate(Rope r, View x, View out, const int32_t *positions, int64_t tokens,
                                                     int heads, int dim, int chunks, float sign) {
    const int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t t = uint32_t(u) / uint32_t(chunks);           // tokens * chunks < 2^32
    const int head = blockIdx.y * kRotateHeads;
    if (t >= tokens) return;
    rotate_chunk<T, kRotateHeads, true>(r, x, out, t, positions[t], head, min(kRotateHeads, heads - head), dim, int(u - t * chunks), sign);
}

// ---------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------

struct AppendArgs {
    Cache c;
    Rows rows;
    Rope rope;           // rotary = 0: none
    View k, v, q, q_out;
    int32_t layer, q_heads, writers, shares, wide;
};

// The least exponent e with most <= 448 * 2^e (448 = 1.75 * 2^8), within +-100.
__device__ __forceinline__ float least_scale(float most) {
    const uint32_t b = __float_as_uint(most);
    int e = int(b >> 23) - 127 - ((b & 0x7fffff) <= 0x600000 ? 8 : 7);
    e = max(-100, min(100, e));
    return __uint_as_float(uint32_t(e + 127) << 23);
}

// Two codes; infinities take the largest, NaN stays.
__device__ __forceinline__ uint32_t code2(float a, float b) {
    a = a == a ? __builtin_amdgcn_fmed3f(a, -448.0f, 448.0f) : a;
    b = b == b ? __builtin_amdgcn_fmed3f(b, -448.0f, 448.0f) : b;
    return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
}

// Work of a launch's first workgroup, beside the others': records what is wrong with any
// row, also with those that no unit is found for where offsets do not ascend.
__device__ __forceinline__ void check_rows(const Cache &c, const Rows &r) {
    for (int b = threadIdx.x; b < r.rows; b += kThreads) row_of(c, r, b);
}

// A unit is one page that a row's tokens touch: row b's units are numbered from
// offsets[b] / Page + 2 b (n tokens touch at most n / Page + 2 pages).
struct Unit {
    Row row;
    int b, slot, page;                      // page -1: there is none
    int from, to;                           // positions of the row's tokens in this page; from = to: nothing to do
};
template <int Page> __device__ __forceinline__ Unit unit_of(const Cache &c, const Rows &r, int unit, const int32_t *starts) {
    auto base = [&](int b) { return r.offsets[b] / Page + 2 * b; };
    Unit u{};
    const int b = count_up_to(r.rows, unit, base) - 1;
    if (b < 0) return u;
    u.b = b;
    u.row = row_of(c, r, b);
    // new tokens: the last n of the sequence, none before its start; read back: any from `starts` on
    const int64_t first = starts ? int64_t(starts[b]) : int64_t(u.row.length) - u.row.n, last = first + u.row.n;
    if (starts && (first < 0 || last > INT32_MAX)) {
        record(c, ESP_ERR_SHAPE);
        return u;
    }
    const int64_t from = max(first, int64_t(0)), slot = from / Page + unit - base(b);
    if (u.row.n == 0 || unit < base(b) || slot * Page >= last) return u;
    u.slot = int(slot);
    u.from = int(max(from, slot * Page));
    u.to = int(min(last, slot * Page + Page));
    u.page = -1;
    if (slot * Page < u.row.length) {
        u.page = c.table[int64_t(u.row.seq) * c.width + u.slot];
        if (u.page < 0 || u.page >= c.pages) {
            record(c, ESP_ERR_SHAPE);
            u.page = -1;
        }
    }
    return u;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int m = 32; m; m >>= 1) x = fmaxf(x, __shfl_xor(x, m));
    return x;
}
__device__ __forceinline__ float finite_abs(float x) {
    x = fabsf(x);
    return x < INFINITY ? x : 0.0f;
}

template <typename T> struct Vec4 { T x[4]; };
template <typename T> __device__ __forceinline__ Vec4<T> load4(const T *p, bool wide) {
    Vec4<T> v;
    if (wide) *reinterpret_cast<uint2v *>(v.x) = *reinterpret_cast<const uint2v *>(p);
    else
#pragma unroll
        for (int i = 0; i < 4; i++) v.x[i] = p[i];
    return v;
}

// Codes of a page that a growing scale makes smaller: 4 at a time.
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float by) {
    const half2 a = codes<false>(w, static_cast<half2 *>(nullptr)), b = codes<true>(w, static_cast<half2 *>(nullptr));
    return code2(float(a[0]) * by, float(a[1]) * by) | code2(float(b[0]) * by, float(b[1]) * by) << 16;
}

// A block's scale.  `older`: the page has tokens from before.
struct Scale {
    float was, now, by;                     // by: 1 / now, exact for the powers of two that append makes
    bool older;
};
__device__ __forceinline__ Scale scale_of(float was, bool older, float most) {
    const float least = least_scale(most), now = older ? fmaxf(was, least) : least;
    return {was, now, 1.0f / now, older};
}
// The largest over the kTeam wavefronts that share a block; lds[4], a buffer of its own each second time.
template <int kTeam> __device__ __forceinline__ float team_max(float x, float *lds) {
    x = wave_max(x);
    if (kTeam > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) lds[wave] = x;
        __syncthreads();
        for (int i = 0; i < kTeam; i++) x = fmaxf(x, lds[wave / kTeam * kTeam + i]);
    }
    return x;
}

// Sixteen tokens [c0, c0 + 16) of a page (One: the token c0 alone): what of them
// is new is written.  A lane takes four pairs of one token's key, four (heads of
// 128) or eight (of 64) tokens at a time; the values stay in registers between
// the largest and the codes.  Tokens that are not new are read as their nearest
// new one and left out, so that no load waits for another.
template <typename T, int Dim, int Page, bool One, int kTeam>
__device__ __forceinline__ void append_keys(const AppendArgs &a, const Unit &u, int head, int c0, bool active, float *lds) {
    constexpr int kLanes = Dim / 8, kTokens = 64 / kLanes, kRounds = One ? 1 : 16 / kTokens;
    const int lane = threadIdx.x & 63, part = lane % kLanes, first = u.slot * Page;
    const int p0 = One ? lane < kLanes ? c0 : u.to : c0 + lane / kLanes;
    const int half = a.rope.rotary >> 1, i0 = 4 * part;
    const bool turn = i0 < half, apart = turn && !a.rope.interleaved;
    const int ea = apart ? i0 : 8 * part, eb = apart ? i0 + half : 8 * part + 4;      // elements ea.. and eb..
    const T *src = static_cast<const T *>(a.k.data) + head * a.k.head + (int64_t(u.row.first) - (u.row.length - u.row.n)) * a.k.token;
    Vec4<T> va[kRounds], vb[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; k++) {
        const T *from = src + int64_t(max(u.from, min(u.to - 1, p0 + k * kTokens))) * a.k.token;
        va[k] = load4(from + ea, a.wide);
        vb[k] = load4(from + eb, a.wide);
    }
    float *place = a.c.block_scale(u.page, a.layer, 0, head);
    const float was = *place;
    double turns[4];
#pragma unroll
    for (int j = 0; j < 4; j++) turns[j] = turn ? a.rope.turns[i0 + j] : 0.0;
    float x[kRounds][8], most = 0.0f;
#pragma unroll
    for (int k = 0; k < kRounds; k++) {
        const int p = p0 + k * kTokens;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            x[k][j] = float(va[k].x[j]);
            x[k][4 + j] = float(vb[k].x[j]);
        }
        if (a.rope.rotary) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                float cs, sn;
                cos_sin(double(p) * turns[j], cs, sn);
                cs *= a.rope.magnitude;
                sn *= a.rope.magnitude;
                const float fa = apart ? x[k][j] : x[k][2 * j], fb = apart ? x[k][4 + j] : x[k][2 * j + 1];
                const float ya = __builtin_fmaf(fa, cs, -(fb * sn)), yb = __builtin_fmaf(fa, sn, fb * cs);
                if (apart) {
                    x[k][j] = ya;
                    x[k][4 + j] = yb;
                } else if (turn) {
                    x[k][2 * j] = ya;
                    x[k][2 * j + 1] = yb;
                }
            }
        }
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j++) top = fmaxf(top, finite_abs(x[k][j]));
        most = fmaxf(most, p >= u.from && p < u.to ? top : 0.0f);
    }
    const Scale s = scale_of(was, first < u.from, team_max<kTeam>(most, lds));
    if (!active) return;
    uint8_t *block = a.c.k + a.c.block(u.page, a.layer, head);
    if (s.older && s.now > s.was) {         // One: the page's first 16 tokens and on
        const float by = s.was / s.now;
        uint32_t *w = reinterpret_cast<uint32_t *>(block);
        const int from = One ? 0 : c0 - first, to = One ? u.from - first : min(u.from, c0 + 16) - first;
        for (int i = from * (Dim / 4) + lane; i < to * (Dim / 4); i += 64) w[i] = rescaled(w[i], by);
    }
#pragma unroll
    for (int k = 0; k < kRounds; k++) {
        const int p = p0 + k * kTokens;
        if (p >= u.from && p < u.to) {
            uint32_t *to = reinterpret_cast<uint32_t *>(block + (p - first) * Dim);
            to[ea / 4] = code2(x[k][0] * s.by, x[k][1] * s.by) | code2(x[k][2] * s.by, x[k][3] * s.by) << 16;
            to[eb / 4] = code2(x[k][4] * s.by, x[k][5] * s.by) | code2(x[k][6] * s.by, x[k][7] * s.by) << 16;
        }
    }
    if (lane == 0 && (One || c0 == first)) *place = s.now;
}

// ... and their values.  A lane takes all the tokens of one (heads of 64) or two
// dimensions, so that sixteen tokens go out at once, as pages hold them.
template <typename T, int Dim, int Page, bool One, int kTeam>
__device__ __forceinline__ void append_values(const AppendArgs &a, const Unit &u, int head, int c0, bool active, float *lds) {
    constexpr int kDims = Dim / 64, kTokens = One ? 1 : 16;
    const int lane = threadIdx.x & 63, d0 = lane * kDims, first = u.slot * Page;
    const T *src = static_cast<const T *>(a.v.data) + head * a.v.head + (int64_t(u.row.first) - (u.row.length - u.row.n)) * a.v.token + d0;
    union Dims {
        uint32_t w;
        T x[2];
    } v[kTokens];
    if (kDims == 2 && a.wide) {
#pragma unroll
        for (int t = 0; t < kTokens; t++) v[t].w = *reinterpret_cast<const uint32_t *>(src + int64_t(max(u.from, min(u.to - 1, c0 + t))) * a.v.token);
    } else {
#pragma unroll
        for (int t = 0; t < kTokens; t++)
#pragma unroll
            for (int d = 0; d < kDims; d++) v[t].x[d] = src[int64_t(max(u.from, min(u.to - 1, c0 + t))) * a.v.token + d];
    }
    float *place = a.c.block_scale(u.page, a.layer, 1, head);
    const float was = *place;
    float most = 0.0f;
#pragma unroll
    for (int t = 0; t < kTokens; t++)
#pragma unroll
        for (int d = 0; d < kDims; d++) most = fmaxf(most, finite_abs(float(v[t].x[d])));     // a token read twice changes nothing
    const Scale s = scale_of(was, first < u.from, team_max<kTeam>(most, lds));
    if (!active) return;
    uint8_t *block = a.c.v + a.c.block(u.page, a.layer, head) + d0 * Page;
    if (s.older && s.now > s.was) {
        const float by = s.was / s.now;
        const int from = One ? 0 : c0 - first, to = One ? u.from - first : min(u.from, c0 + 16) - first;
        for (int d = 0; d < kDims; d++)
            for (int t = from; t < to; t += 4) {       // a word may reach into the new tokens: these are written after
                uint32_t *w = reinterpret_cast<uint32_t *>(block + d * Page + t);
                *w = rescaled(*w, by);
            }
    }
    if constexpr (One) {
#pragma unroll
        for (int d = 0; d < kDims; d++) block[d * Page + c0 - first] = uint8_t(code2(float(v[0].x[d]) * s.by, 0.0f));
    } else if (c0 + 16 > u.from && c0 < u.to) {
#pragma unroll
        for (int d = 0; d < kDims; d++) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++)
                w[i] = code2(float(v[4 * i].x[d]) * s.by, float(v[4 * i + 1].x[d]) * s.by) | code2(float(v[4 * i + 2].x[d]) * s.by, float(v[4 * i + 3].x[d]) * s.by) << 16;
            uint8_t *to = block + d * Page + (c0 - first);
            if (c0 >= u.from && c0 + 16 <= u.to) {
                *reinterpret_cast<uint4v *>(to) = uint4v{w[0], w[1], w[2], w[3]};
            } else {
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (c0 + i >= u.from && c0 + i < u.to) to[i] = uint8_t(w[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
    if (lane == 0 && (One || c0 == first)) *place = s.now;
}

// Workgroups [0, writers): some of the 2 * heads blocks of one unit, a block by
// as many wavefronts as the page has sixteens of tokens (a single token by one);
// the others turn the queries.  One more, in front, checks the rows.
// Bound by the chain load - largest - scale - store of each block: 256 single tokens
// of 8 key and 32 query heads of 128, 19 MB with the reading back of their pages, 23 us
// in two launches; 9 prompts of up to 4,096 tokens, 175 MB likewise, 55 us (3.2 TB/s).
template <typename T, int Dim, int Page> __global__ __launch_bounds__(kThreads) void k_append(AppendArgs a) {
    constexpr int kTeam = Page / 16, kTeams = 4 / kTeam;
    __shared__ float lds[2][4];
    const int place = int(blockIdx.x) - 1;
    if (place < 0) return check_rows(a.c, a.rows);
    if (place < a.writers) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int unit = place / a.shares, share = place - unit * a.shares;
        const Unit u = unit_of<Page>(a.c, a.rows, unit, nullptr);
        if (u.from >= u.to || u.page < 0) return;
        const int blocks = 2 * a.c.heads;
        if (u.to - u.from == 1) {
            for (int i = share * 4 + wave; i < blocks; i += a.shares * 4) {
                if (i < a.c.heads) append_keys<T, Dim, Page, true, 1>(a, u, i, u.from, true, nullptr);
                else append_values<T, Dim, Page, true, 1>(a, u, i - a.c.heads, u.from, true, nullptr);
            }
            return;
        }
        // even parts keys, odd parts values; every wavefront goes round as often, for the barriers
        const int c0 = u.slot * Page + wave % kTeam * 16, step = a.shares / 2 * kTeams;
        for (int i = 0, head = share / 2 * kTeams + wave / kTeam; i < (a.c.heads + step - 1) / step; i++, head += step) {
            if (share & 1) append_values<T, Dim, Page, false, kTeam>(a, u, min(head, a.c.heads - 1), c0, head < a.c.heads, lds[i & 1]);
            else append_keys<T, Dim, Page, false, kTeam>(a, u, min(head, a.c.heads - 1), c0, head < a.c.heads, lds[i & 1]);
        }
        return;
    }
    constexpr int kChunks = Dim / 16;
    const int groups = (a.q_heads + kAppendHeads - 1) / kAppendHeads;
    const int64_t u = int64_t(place - a.writers) * kThreads + threadIdx.x, tg = u / kChunks;
    const int64_t t = min(tg / groups, a.rows.tokens - 1);
    // the row of the wavefront's first token, then step by step
    const int64_t t_first = __shfl(int(t), 0);
    int b = max(0, count_up_to(a.rows.rows, t_first, [&](int x) { return a.rows.offsets[x]; }) - 1);
    if (tg / groups >= a.rows.tokens) return;
    while (b + 1 < a.rows.rows && a.rows.offsets[b + 1] <= t) b++;
    const Row row = row_of(a.c, a.rows, b);
    const int head = int(tg - t * groups) * kAppendHeads;
    rotate_chunk<T, kAppendHeads, false>(a.rope, a.q, a.q_out, t, row.length - row.n + int(t - row.first), head, min(kAppendHeads, a.q_heads - head), Dim, int(u % kChunks), 1.0f);
}

// ---------------------------------------------------------------------------
// Gather: the same units, read back.
// ---------------------------------------------------------------------------

struct GatherArgs {
    Cache c;
    Rows rows;
    const int32_t *starts;
    int32_t layer, shares, units;
    void *k, *v;
};

template <typename T, int Dim, int Page> __device__ __forceinline__ void gather_block(const GatherArgs &a, const Unit &u, int head, bool values) {
    const int lane = threadIdx.x & 63, first = u.slot * Page;
    const int64_t row_size = int64_t(a.c.heads) * Dim;
    // the output row of the page's first token
    T *out = static_cast<T *>(values ? a.v : a.k) + (int64_t(u.row.first) + first - a.starts[u.b]) * row_size + int64_t(head) * Dim;
    // past the end of the sequence, or without a page: 0
    const int held = u.page < 0 ? u.from : min(u.to, u.row.length);
    for (int t = max(u.from, held) + lane / (Dim / 8); t < u.to; t += 512 / Dim) store8(out + (t - first) * row_size + lane % (Dim / 8) * 8, Vec8<T>{});
    if (held <= u.from) return;
    const float s = *a.c.block_scale(u.page, a.layer, values, head);
    if (!values) {
        constexpr int kLanes = Dim / 8, kTokens = 64 / kLanes;
        const uint8_t *block = a.c.k + a.c.block(u.page, a.layer, head);
        constexpr int kRounds = Page / kTokens;
        const int d = lane % kLanes * 8;
        uint2v w[kRounds];
#pragma unroll
        for (int k = 0; k < kRounds; k++) {            // other tokens of the page are read as the nearest that is asked for
            const int t = max(u.from, min(held - 1, first + k * kTokens + lane / kLanes)) - first;
            w[k] = *reinterpret_cast<const uint2v *>(block + t * Dim + d);
        }
#pragma unroll
        for (int k = 0; k < kRounds; k++) {
            const int t = k * kTokens + lane / kLanes;
            if (first + t < u.from || first + t >= held) continue;
            const half8 n = codes8<half8, half2>(w[k][0], w[k][1]);
            Vec8<T> o;
#pragma unroll
            for (int j = 0; j < 8; j++) o.x[j] = T(float(n[j]) * s);
            store8(out + t * row_size + d, o);
        }
        return;
    }
    constexpr int kDims = Dim / 64;
    const int d0 = lane * kDims;
    const uint8_t *block = a.c.v + a.c.block(u.page, a.layer, head) + d0 * Page;
    uint4v all[Page / 16][kDims];
#pragma unroll
    for (int g = 0; g < Page; g += 16)
#pragma unroll
        for (int d = 0; d < kDims; d++) all[g / 16][d] = *reinterpret_cast<const uint4v *>(block + d * Page + g);
#pragma unroll
    for (int g = 0; g < Page; g += 16) {
        if (first + g + 16 <= u.from || first + g >= held) continue;
        const uint4v(&w)[kDims] = all[g / 16];
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            half8 n[kDims];
#pragma unroll
            for (int d = 0; d < kDims; d++) n[d] = codes8<half8, half2>(w[d][i / 4], w[d][i / 4 + 1]);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int t = g + i + j;
                if (first + t < u.from || first + t >= held) continue;
                typedef T Out __attribute__((ext_vector_type(kDims)));
                Out o;
#pragma unroll
                for (int d = 0; d < kDims; d++) o[d] = T(float(n[d][j]) * s);
                *reinterpret_cast<Out *>(out + t * row_size + d0) = o;
            }
        }
    }
}

template <typename T, int Dim, int Page> __global__ __launch_bounds__(kThreads) void k_gather(GatherArgs a) {
    const int place = int(blockIdx.x) - 1;
    if (place < 0) return check_rows(a.c, a.rows);
    const int w = __builtin_amdgcn_readfirstlane(place * (kThreads / 64) + (threadIdx.x >> 6));
    const int unit = w / a.shares, share = w - unit * a.shares;
    if (unit >= a.units) return;
    const Unit u = unit_of<Page>(a.c, a.rows, unit, a.starts);
    if (u.from < u.to)
        for (int i = share; i < 2 * a.c.heads; i += a.shares) gather_block<T, Dim, Page>(a, u, i % a.c.heads, i >= a.c.heads);
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
    return aligned16(v.data) && v.token_stride * size % 16 == 0 && v.head_stride * size % 16 == 0;
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
        const int chunks = dim / (32 / int(sizeof(T)));
        const int64_t blocks = (tokens * chunks + kThreads - 1) / kThreads;
        k_rotate<T><<<dim3(unsigned(blocks), (heads + kRotateHeads - 1) / kRotateHeads), kThreads, 0, s>>>(r, x, out, positions, tokens, heads, dim, chunks, sign);
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
template <typename T, int Dim> void gather(const GatherArgs &a, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: k_gather<T, Dim, 16><<<blocks, kThreads, 0, s>>>(a); break;
    case 32: k_gather<T, Dim, 32><<<blocks, kThreads, 0, s>>>(a); break;
    default: k_gather<T, Dim, 64><<<blocks, kThreads, 0, s>>>(a); break;
    }
}

// A launch's threads are numbered in 32 bits.
constexpr int64_t kMostThreads = (int64_t(1) << 32) - kThreads;

// Parts of a unit's work, `most` at most, each of `waves` wavefronts: about 16,384
// wavefronts in all, twice what the GPU holds; as few as finish in as many rounds.
int32_t shares_of(int64_t units, int64_t most, int64_t waves) {
    const int64_t fill = 16384 / (units * waves), shares = fill < 1 ? 1 : fill < most ? fill : most, rounds = (most + shares - 1) / shares;
    return int32_t((most + rounds - 1) / rounds);
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
    const int step = 32 / size;             // elements of two vectors
    const bool vector = wide(x, size) && wide(out, size) && rope->rotary_dim % step == 0 && head_dim % step == 0 &&
                        tokens * (head_dim / step) <= kMostThreads;
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
    const int32_t teams = 64 / cache->page_tokens,
                  shares = 2 * shares_of(units, (cache->kv_heads + teams - 1) / teams, 8);
    const int64_t writers = units * shares;
    const int64_t turners = (tokens * ((q_heads + kAppendHeads - 1) / kAppendHeads) * (cache->head_dim / 16) + kThreads - 1) / kThreads;
    if (writers + turners + 1 > kMostThreads / kThreads) return ESP_ERR_SHAPE;
    const unsigned blocks = unsigned(writers + turners + 1);
    // loads of four keys or two values at a time
    auto fours = [](const esp_kv_view &x) { return (reinterpret_cast<uintptr_t>(x.data) & 7) == 0 && x.token_stride % 4 == 0 && x.head_stride % 4 == 0; };
    const AppendArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, rope_of(rope), view_of(k), view_of(v), view_of(q), view_of(q_out),
                       layer, q_heads, int32_t(writers), shares, fours(k) && fours(v)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == ESP_KV_BF16) cache->head_dim == 64 ? append<__bf16, 64>(a, blocks, s) : append<__bf16, 128>(a, blocks, s);
    else cache->head_dim == 64 ? append<_Float16, 64>(a, blocks, s) : append<_Float16, 128>(a, blocks, s);
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
    const int64_t units = tokens / cache->page_tokens + 2 * int64_t(rows);
    const int32_t shares = shares_of(units, 2 * cache->kv_heads, 1);
    const int64_t workers = (units * shares + kThreads / 64 - 1) / (kThreads / 64);
    if (workers + 1 > kMostThreads / kThreads) return ESP_ERR_SHAPE;
    const unsigned blocks = unsigned(workers + 1);
    const GatherArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, starts, layer, shares, int32_t(units), k_out, v_out};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == ESP_KV_BF16) cache->head_dim == 64 ? gather<__bf16, 64>(a, blocks, s) : gather<__bf16, 128>(a, blocks, s);
    else cache->head_dim == 64 ? gather<_Float16, 64>(a, blocks, s) : gather<_Float16, 128>(a, blocks, s);
    return launched();
}
