// Norms of queries and keys for each head, with the position rotation in the
// same pass, and their gradient.
//   n = x r,  r = (sum x^2 / D + eps)^-1/2,  y = m R(p) (n w)
// With g = m R(p)^T dy (the rotation turned back):
//   dw = sum over tokens and heads of g n
//   dx = r (g w - n c),  c = sum (g w n) / D
#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kThreads = 256;
constexpr int kMostDim = 512;

struct View {
    void *data;
    int64_t token, head;
};

// One of queries and keys.
struct Side {
    View x, y;                              // y: outputs, or the gradients that come in
    View dx;
    const void *weight;                     // NULL: ones
    float *partial;                         // [blocks][dim] sums of the weight's gradient
    void *dweight;
    int32_t heads, blocks;
};

struct NormArgs {
    Side side[2];
    Rope rope;
    const int32_t *positions;
    int64_t tokens;
    int32_t dim, wide_weight;               // wide_weight: weights in float32, else of the tensors' type
    float eps, part;                        // part: 1 / dim
};

template <typename T> __device__ __forceinline__ float weight_at(const NormArgs &a, const void *w, int i) {
    return !w ? 1.0f : a.wide_weight ? static_cast<const float *>(w)[i] : float(static_cast<const T *>(w)[i]);
}

// Sum over the kLanes lanes that share a head.
template <int kLanes> __device__ __forceinline__ float team_sum(float x) {
#pragma unroll
    for (int m = kLanes / 2; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// Two vectors of a head a lane, 16 bytes each or, where the turned part's halves are no
// multiple of these, 8, so that both sides of its pairs are its own: with halves lane c has vectors c and c + n of the turned part's 2 n, with
// neighbours as pairs the same vectors with pairs of their own; then the same of
// the part that passes through.
template <typename T, int kBytes> struct Place {
    static constexpr int kVec = kBytes / int(sizeof(T));
    int a, b;                               // elements of the two vectors
    bool turn;
    __device__ __forceinline__ Place(const Rope &r, int dim, int c) {
        const int turned = r.rotary / (2 * kVec), rest = dim / (2 * kVec) - turned;
        turn = c < turned;
        a = (turn ? c : c + turned) * kVec;
        b = a + (turn ? turned : rest) * kVec;
    }
    __device__ __forceinline__ void angles(const Rope &r, int position, float sign, float (&cs)[kVec], float (&sn)[kVec]) const {
#pragma unroll
        for (int j = 0; j < kVec; j++) {
            const int i = !r.interleaved ? a + j : j < kVec / 2 ? a / 2 + j : b / 2 + j - kVec / 2;
            cs[j] = 1.0f;
            sn[j] = 0.0f;
            if (turn) {
                cos_sin(double(position) * r.turns[i], cs[j], sn[j]);
                cs[j] *= r.magnitude;
                sn[j] *= sign * r.magnitude;
            }
        }
    }
    // x: the first vector's elements, then the second's.  What passes through is left alone: a sine
    // of 0 would make NaN of an infinity's partner.
    __device__ __forceinline__ void turn_by(bool interleaved, float (&x)[2 * kVec], const float (&cs)[kVec], const float (&sn)[kVec]) const {
        if (!turn) return;
        auto pair = [](float &u, float &v, float c, float s) {
            const float fu = u, fv = v;
            u = __builtin_fmaf(fu, c, -(fv * s));
            v = __builtin_fmaf(fu, s, fv * c);
        };
        if (interleaved) {
#pragma unroll
            for (int j = 0; j < kVec; j++) pair(x[2 * j], x[2 * j + 1], cs[j], sn[j]);
        } else {
#pragma unroll
            for (int j = 0; j < kVec; j++) pair(x[j], x[kVec + j], cs[j], sn[j]);
        }
    }
};

template <typename T, int kBytes> union Vec {
    typedef uint32_t Words __attribute__((ext_vector_type(kBytes / 4)));
    Words w;
    T x[kBytes / sizeof(T)];
};

template <typename T, int kBytes>
__device__ __forceinline__ void load(const View &v, int64_t t, int head, int a, int b, float (&x)[2 * kBytes / sizeof(T)]) {
    constexpr int kVec = kBytes / int(sizeof(T));
    const T *p = static_cast<const T *>(v.data) + t * v.token + head * v.head;
    Vec<T, kBytes> u, w;
    u.w = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T, kBytes>::Words *>(p + a));
    w.w = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T, kBytes>::Words *>(p + b));
#pragma unroll
    for (int j = 0; j < kVec; j++) {
        x[j] = float(u.x[j]);
        x[kVec + j] = float(w.x[j]);
    }
}
template <typename T, int kBytes>
__device__ __forceinline__ void store(const View &v, int64_t t, int head, int a, int b, const float (&x)[2 * kBytes / sizeof(T)]) {
    constexpr int kVec = kBytes / int(sizeof(T));
    T *p = static_cast<T *>(v.data) + t * v.token + head * v.head;
    Vec<T, kBytes> u, w;
#pragma unroll
    for (int j = 0; j < kVec; j++) {
        u.x[j] = T(x[j]);
        w.x[j] = T(x[kVec + j]);
    }
    *reinterpret_cast<typename Vec<T, kBytes>::Words *>(p + a) = u.w;
    *reinterpret_cast<typename Vec<T, kBytes>::Words *>(p + b) = w.w;
}

// Whose work a workgroup does: queries first, then keys.
__device__ __forceinline__ int side_of(const NormArgs &a, int &block) {
    const int which = block >= a.side[0].blocks;
    block -= which ? a.side[0].blocks : 0;
    return which;
}

// Units (token, group of heads) from `first` on, `step` apart.
struct Walk {
    int64_t token;
    int group, groups, tokens_on, groups_on;
    __device__ __forceinline__ Walk(int first, int step, int n)
        : token(uint32_t(first) / uint32_t(n)), group(int(uint32_t(first) % uint32_t(n))), groups(n), tokens_on(int(uint32_t(step) / uint32_t(n))),
          groups_on(int(uint32_t(step) % uint32_t(n))) {}
    __device__ __forceinline__ void next() {
        token += tokens_on;
        group += groups_on;
        if (group >= groups) {
            group -= groups;
            token++;
        }
    }
};

// kLanes lanes a token and head (dim / (2 vectors) of them at work), kPer heads of a
// token, whose angles are worked out once.  Read past the caches: neither input nor output is
// wanted again here.
// Bound by memory: 16,383 tokens of 32 + 8 heads of 128 in bf16 (336 MB) 69 us (4.9 TB/s); 256
// of them 8.1 us, a chain of loads, sums and angles.
template <typename T, int kBytes, int kLanes, int kPer> __global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
    constexpr int kVec = kBytes / int(sizeof(T)), kTeams = kThreads / kLanes;
    int block = blockIdx.x;
    const Side &s = a.side[side_of(a, block)];
    const int c = threadIdx.x % kLanes, groups = (s.heads + kPer - 1) / kPer;
    const int64_t unit = int64_t(block) * kTeams + threadIdx.x / kLanes, t = unit / groups;
    if (t >= a.tokens) return;              // whole teams leave
    const int head = int(unit - t * groups) * kPer;
    const bool there = c < a.dim / (2 * kVec);
    const Place<T, kBytes> at(a.rope, a.dim, there ? c : 0);
    float x[kPer][2 * kVec], w[2 * kVec], cs[kVec], sn[kVec];
#pragma unroll
    for (int h = 0; h < kPer; h++) load<T, kBytes>(s.x, t, min(head + h, s.heads - 1), at.a, at.b, x[h]);
#pragma unroll
    for (int j = 0; j < kVec; j++) {
        w[j] = weight_at<T>(a, s.weight, at.a + j);
        w[kVec + j] = weight_at<T>(a, s.weight, at.b + j);
    }
    at.angles(a.rope, a.positions[t], 1.0f, cs, sn);
#pragma unroll
    for (int h = 0; h < kPer; h++) {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 2 * kVec; j++) sum = __builtin_fmaf(x[h][j], x[h][j], sum);
        sum = team_sum<kLanes>(there ? sum : 0.0f);
        const float r = rsqrtf(__builtin_fmaf(sum, a.part, a.eps));
#pragma unroll
        for (int j = 0; j < 2 * kVec; j++) x[h][j] = x[h][j] * r * w[j];
        at.turn_by(a.rope.interleaved, x[h], cs, sn);
        if (there && head + h < s.heads) store<T, kBytes>(s.y, t, head + h, at.a, at.b, x[h]);
    }
}

// The gradient of the former 120 us (503 MB, 4.2 TB/s): 152 registers leave three wavefronts a
// SIMD; with four the sums are spilled (178 us), and one head at a time takes 135.
// The same teams, each going through many tokens with the sums of its elements' weight
// gradient in registers; a workgroup's sums go to its row of `partial`, added up by
// k_norm_weights: an order that sizes, types, strides and alignment decide (by the vectors and teams).
template <typename T, int kBytes, int kLanes, int kPer> __global__ __launch_bounds__(kThreads) void k_norm_back(NormArgs a) {
    constexpr int kVec = kBytes / int(sizeof(T)), kTeams = kThreads / kLanes, kOwn = 2 * kVec;
    __shared__ float lds[4][kMostDim];
    int block = blockIdx.x;
    const Side &s = a.side[side_of(a, block)];
    const int c = threadIdx.x % kLanes, groups = (s.heads + kPer - 1) / kPer;
    const bool there = c < a.dim / (2 * kVec);
    const Place<T, kBytes> at(a.rope, a.dim, there ? c : 0);
    float w[kOwn], dw[kOwn];
#pragma unroll
    for (int j = 0; j < kVec; j++) {
        w[j] = weight_at<T>(a, s.weight, at.a + j);
        w[kVec + j] = weight_at<T>(a, s.weight, at.b + j);
    }
#pragma unroll
    for (int j = 0; j < kOwn; j++) dw[j] = 0.0f;
    for (Walk u(block * kTeams + threadIdx.x / kLanes, s.blocks * kTeams, groups); u.token < a.tokens; u.next()) {
        const int64_t t = u.token;
        const int head = u.group * kPer;
        float x[kPer][kOwn], g[kPer][kOwn], cs[kVec], sn[kVec];
#pragma unroll
        for (int h = 0; h < kPer; h++) {
            load<T, kBytes>(s.x, t, min(head + h, s.heads - 1), at.a, at.b, x[h]);
            load<T, kBytes>(s.y, t, min(head + h, s.heads - 1), at.a, at.b, g[h]);
        }
        at.angles(a.rope, a.positions[t], -1.0f, cs, sn);
#pragma unroll
        for (int h = 0; h < kPer; h++) {
            const bool held = there && head + h < s.heads;
            at.turn_by(a.rope.interleaved, g[h], cs, sn);
            float sum = 0.0f, dot = 0.0f;
#pragma unroll
            for (int j = 0; j < kOwn; j++) {
                sum = __builtin_fmaf(x[h][j], x[h][j], sum);
                dot = __builtin_fmaf(g[h][j] * w[j], x[h][j], dot);
            }
            sum = team_sum<kLanes>(there ? sum : 0.0f);
            dot = team_sum<kLanes>(there ? dot : 0.0f);
            const float r = rsqrtf(__builtin_fmaf(sum, a.part, a.eps)), mean = dot * r * a.part;
#pragma unroll
            for (int j = 0; j < kOwn; j++) {
                const float n = x[h][j] * r;
                dw[j] += held ? g[h][j] * n : 0.0f;
                x[h][j] = r * __builtin_fmaf(g[h][j], w[j], -(n * mean));
            }
            if (held) store<T, kBytes>(s.dx, t, head + h, at.a, at.b, x[h]);
        }
    }
    if (!s.dweight) return;
    // over the teams of a wavefront, then over the wavefronts
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < kOwn; j++) {
#pragma unroll
        for (int m = kLanes; m < 64; m <<= 1) dw[j] += __shfl_xor(dw[j], m);
        if ((threadIdx.x & 63) < kLanes && there) lds[wave][j < kVec ? at.a + j : at.b + j - kVec] = dw[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.dim; i += kThreads)
        s.partial[int64_t(block) * a.dim + i] = (lds[0][i] + lds[1][i]) + (lds[2][i] + lds[3][i]);
}

// Any strides, alignment and rotary part: a wavefront a token and head, a pair a lane at a time.
constexpr int kMostPairs = kMostDim / 2 / 64, kAnyHeads = 8;      // heads that angles are worked out for once
template <typename T, bool Back> __global__ __launch_bounds__(kThreads) void k_norm_any(NormArgs a) {
    __shared__ float lds[4][kMostDim];
    int block = blockIdx.x;
    const Side &s = a.side[side_of(a, block)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.dim / 2, half = a.rope.rotary / 2;
    int ea[kMostPairs], eb[kMostPairs];
    float wa[kMostPairs], wb[kMostPairs], da[kMostPairs], db[kMostPairs];
#pragma unroll
    for (int k = 0; k < kMostPairs; k++) {
        const int i = lane + 64 * k;
        const bool apart = !a.rope.interleaved && i < half;
        ea[k] = i >= pairs ? 0 : apart ? i : 2 * i;
        eb[k] = i >= pairs ? 0 : apart ? i + half : 2 * i + 1;
        wa[k] = weight_at<T>(a, s.weight, ea[k]);
        wb[k] = weight_at<T>(a, s.weight, eb[k]);
        da[k] = db[k] = 0.0f;
    }
    const int groups = (s.heads + kAnyHeads - 1) / kAnyHeads;
    for (Walk u(block * 4 + wave, s.blocks * 4, groups); u.token < a.tokens; u.next()) {
        const int64_t t = u.token;
        float cs[kMostPairs], sn[kMostPairs];
#pragma unroll
        for (int k = 0; k < kMostPairs; k++) {
            const int i = lane + 64 * k;
            cs[k] = 1.0f;
            sn[k] = 0.0f;
            if (i < half) {
                cos_sin(double(a.positions[t]) * a.rope.turns[i], cs[k], sn[k]);
                cs[k] *= a.rope.magnitude;
                sn[k] *= a.rope.magnitude;
            }
        }
        for (int head = u.group * kAnyHeads; head < min(s.heads, (u.group + 1) * kAnyHeads); head++) {
            const T *px = static_cast<const T *>(s.x.data) + t * s.x.token + head * s.x.head;
            T *py = static_cast<T *>(s.y.data) + t * s.y.token + head * s.y.head;
            float xa[kMostPairs], xb[kMostPairs], ga[kMostPairs], gb[kMostPairs], sum = 0.0f, dot = 0.0f;
#pragma unroll
            for (int k = 0; k < kMostPairs; k++) {
                xa[k] = xb[k] = ga[k] = gb[k] = 0.0f;
                if (lane + 64 * k < pairs) {
                    xa[k] = float(px[ea[k]]);
                    xb[k] = float(px[eb[k]]);
                    sum = __builtin_fmaf(xa[k], xa[k], __builtin_fmaf(xb[k], xb[k], sum));
                    if (Back) {
                        const float y = float(py[ea[k]]), z = float(py[eb[k]]);
                        const bool turn = lane + 64 * k < half;
                        ga[k] = turn ? __builtin_fmaf(y, cs[k], z * sn[k]) : y;
                        gb[k] = turn ? __builtin_fmaf(z, cs[k], -(y * sn[k])) : z;
                        dot = __builtin_fmaf(ga[k] * wa[k], xa[k], __builtin_fmaf(gb[k] * wb[k], xb[k], dot));
                    }
                }
            }
            sum = team_sum<64>(sum);
            if (Back) dot = team_sum<64>(dot);
            const float r = rsqrtf(__builtin_fmaf(sum, a.part, a.eps)), mean = dot * r * a.part;
            T *out = Back ? static_cast<T *>(s.dx.data) + t * s.dx.token + head * s.dx.head : py;
#pragma unroll
            for (int k = 0; k < kMostPairs; k++) {
                if (lane + 64 * k >= pairs) continue;
                const float na = xa[k] * r, nb = xb[k] * r;
                if (Back) {
                    da[k] += ga[k] * na;
                    db[k] += gb[k] * nb;
                    out[ea[k]] = T(r * __builtin_fmaf(ga[k], wa[k], -(na * mean)));
                    out[eb[k]] = T(r * __builtin_fmaf(gb[k], wb[k], -(nb * mean)));
                } else {
                    const float y = na * wa[k], z = nb * wb[k];
                    const bool turn = lane + 64 * k < half;
                    out[ea[k]] = T(turn ? __builtin_fmaf(y, cs[k], -(z * sn[k])) : y);
                    out[eb[k]] = T(turn ? __builtin_fmaf(y, sn[k], z * cs[k]) : z);
                }
            }
        }
    }
    if (!Back || !s.dweight) return;
#pragma unroll
    for (int k = 0; k < kMostPairs; k++)
        if (lane + 64 * k < pairs) {
            lds[wave][ea[k]] = da[k];
            lds[wave][eb[k]] = db[k];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < a.dim; i += kThreads)
        s.partial[int64_t(block) * a.dim + i] = (lds[0][i] + lds[1][i]) + (lds[2][i] + lds[3][i]);
}

// Sums of the workgroups' rows: 16 elements a workgroup, 64 stretches of rows each.
constexpr int kSumThreads = 1024;
template <typename T> __global__ __launch_bounds__(kSumThreads) void k_norm_weights(NormArgs a) {
    __shared__ float lds[64][17];
    const Side &s = a.side[blockIdx.y];
    if (!s.dweight) return;
    const int i = blockIdx.x * 16 + threadIdx.x % 16, part = threadIdx.x / 16;
    float sum = 0.0f;
    if (i < a.dim)
        for (int b = part; b < s.blocks; b += 512) {    // eight loads in flight
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; k++) x[k] = b + 64 * k < s.blocks ? s.partial[int64_t(b + 64 * k) * a.dim + i] : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; k++) sum += x[k];
        }
    lds[part][threadIdx.x % 16] = sum;
    __syncthreads();
    if (part || i >= a.dim) return;
    for (int k = 1; k < 64; k++) sum += lds[k][threadIdx.x];
    if (a.wide_weight) static_cast<float *>(s.dweight)[i] = sum;
    else static_cast<T *>(s.dweight)[i] = T(sum);
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

constexpr int64_t kMostBlocks = ((int64_t(1) << 32) - kThreads) / kThreads;    // a launch's threads are numbered in 32 bits
constexpr int kPerHeads = 4, kBackHeads = 2;
// Workgroups of a gradient, of queries and keys together: those that the GPU holds at once, or
// twice as many, whose ends lie less far apart, where each still has four turns.  So many / the
// others: 655,320 heads of 128 in bf16 120 / 143 us; 131,168 of 64 in fp16 20 / 24.
constexpr int kBackBlocks = 768;

View view_of(const esp_kv_view &v) { return {v.data, v.token_stride, v.head_stride}; }
// Bytes that accesses at multiples of them may have: 16, 8 or 0 (neither).
int wide(const esp_kv_view &v, int size) {
    const uint64_t all = uint64_t(reinterpret_cast<uintptr_t>(v.data)) | uint64_t(v.token_stride * size) | uint64_t(v.head_stride * size);
    return all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : 0;
}
int lanes_of(int32_t dim, int size, int bytes) {                 // lanes of a head: a power of two
    int n = 1;
    while (n < dim * size / (2 * bytes)) n *= 2;
    return n;
}
int least_of(int a, int b) { return a < b ? a : b; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

esp_status check(const esp_kv_rope *rope, int32_t type, int64_t tokens, int32_t head_dim, int32_t q_heads, int32_t k_heads, int32_t weight_type, float eps) {
    if (!rope || type < ESP_KV_BF16 || type > ESP_KV_FP32 || (weight_type != type && weight_type != ESP_KV_FP32)) return ESP_ERR_INVALID_ARG;
    if (!(eps > 0.0f) || !(eps < INFINITY)) return ESP_ERR_INVALID_ARG;
    if (!rope->turns || (rope->interleaved != 0 && rope->interleaved != 1) || !(rope->magnitude == rope->magnitude)) return ESP_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > INT32_MAX || q_heads < 0 || q_heads > 65536 || k_heads < 0 || k_heads > 65536) return ESP_ERR_SHAPE;
    if (head_dim < 2 || head_dim % 2 || head_dim > kMostDim) return ESP_ERR_SHAPE;
    return rope->rotary_dim >= 2 && rope->rotary_dim % 2 == 0 && rope->rotary_dim <= head_dim ? ESP_OK : ESP_ERR_SHAPE;
}

// Bytes of the vectors that heads are taken as, 0: none.
int vectors(const NormArgs &a, int size, int most) {
    for (int bytes = most; bytes >= 8; bytes /= 2)
        if (a.rope.rotary * size % (2 * bytes) == 0 && a.dim * size % (2 * bytes) == 0 && lanes_of(a.dim, size, bytes) <= 64) return bytes;
    return 0;
}

// Workgroups of a gradient: all at once, shared between queries and keys by their heads.
void share_blocks(NormArgs &a, int64_t tokens, int32_t q_heads, int32_t k_heads, int lanes) {
    const int64_t heads = int64_t(q_heads) + k_heads;
    if (!heads) return;
    const int64_t teams = kThreads / lanes, turns = (tokens * heads + teams * kBackHeads - 1) / (teams * kBackHeads);
    const int64_t want = turns >= 8 * kBackBlocks ? 2 * kBackBlocks : least(turns, kBackBlocks);
    for (int i = 0; i < 2; i++) {
        const int64_t own = i ? k_heads : q_heads;
        a.side[i].blocks = own ? int32_t((want * own + heads - 1) / heads) : 0;
    }
}

template <typename T, int kBytes, int kLanes> void launch(const NormArgs &a, bool back, unsigned blocks, hipStream_t s) {
    if (back) k_norm_back<T, kBytes, kLanes, kBackHeads><<<blocks, kThreads, 0, s>>>(a);
    else k_norm<T, kBytes, kLanes, kPerHeads><<<blocks, kThreads, 0, s>>>(a);
}
template <typename T, int kBytes> void launch(const NormArgs &a, int lanes, bool back, unsigned blocks, hipStream_t s) {
    switch (lanes) {
    case 1: launch<T, kBytes, 1>(a, back, blocks, s); break;
    case 2: launch<T, kBytes, 2>(a, back, blocks, s); break;
    case 4: launch<T, kBytes, 4>(a, back, blocks, s); break;
    case 8: launch<T, kBytes, 8>(a, back, blocks, s); break;
    case 16: launch<T, kBytes, 16>(a, back, blocks, s); break;
    case 32: launch<T, kBytes, 32>(a, back, blocks, s); break;
    default: launch<T, kBytes, 64>(a, back, blocks, s); break;
    }
}
template <typename T> esp_status run(NormArgs &a, bool back, int aligned, hipStream_t s) {
    const int bytes = vectors(a, sizeof(T), aligned), lanes = bytes ? lanes_of(a.dim, sizeof(T), bytes) : 64;
    int64_t blocks = 0;
    for (Side &side : a.side) {
        if (!back && side.heads) {
            const int64_t per = bytes ? kPerHeads : kAnyHeads, groups = (side.heads + per - 1) / per, teams = kThreads / lanes;
            const int64_t need = (a.tokens * groups + teams - 1) / teams;
            if (bytes && need > kMostBlocks / 2) return ESP_ERR_SHAPE;
            side.blocks = int32_t(bytes ? need : least(need, 65536));
        }
        blocks += side.blocks;
    }
    if (blocks == 0) {
    } else if (bytes == 16) {
        launch<T, 16>(a, lanes, back, unsigned(blocks), s);
    } else if (bytes == 8) {
        launch<T, 8>(a, lanes, back, unsigned(blocks), s);
    } else {
        if (back) k_norm_any<T, true><<<unsigned(blocks), kThreads, 0, s>>>(a);
        else k_norm_any<T, false><<<unsigned(blocks), kThreads, 0, s>>>(a);
    }
    if (back && (a.side[0].dweight || a.side[1].dweight)) k_norm_weights<T><<<dim3((a.dim + 15) / 16, 2), kSumThreads, 0, s>>>(a);
    return launched();
}
esp_status run(NormArgs &a, int32_t type, bool back, int aligned, void *stream) {
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (type == ESP_KV_BF16) return run<__bf16>(a, back, aligned, s);
    if (type == ESP_KV_FP16) return run<_Float16>(a, back, aligned, s);
    return run<float>(a, back, aligned, s);
}

}  // namespace

extern "C" esp_status esp_kv_norm_rotate(const esp_kv_rope *rope, int32_t type, int64_t tokens, int32_t head_dim, int32_t q_heads,
                                         int32_t k_heads, esp_kv_view q, esp_kv_view k, const void *q_weight, const void *k_weight,
                                         int32_t weight_type, const int32_t *positions, float eps, esp_kv_view q_out,
                                         esp_kv_view k_out, void *stream) {
    if (esp_status e = check(rope, type, tokens, head_dim, q_heads, k_heads, weight_type, eps)) return e;
    if (tokens == 0 || q_heads + k_heads == 0) return ESP_OK;
    if (!positions || (q_heads && (!q.data || !q_out.data)) || (k_heads && (!k.data || !k_out.data))) return ESP_ERR_INVALID_ARG;
    const int size = type == ESP_KV_FP32 ? 4 : 2;
    NormArgs a{{{view_of(q), view_of(q_out), {}, q_weight, nullptr, nullptr, q_heads, 0}, {view_of(k), view_of(k_out), {}, k_weight, nullptr, nullptr, k_heads, 0}},
               {rope->turns, rope->magnitude, rope->rotary_dim, rope->interleaved}, positions, tokens, head_dim, weight_type == ESP_KV_FP32, eps, 1.0f / float(head_dim)};
    const int aligned = least_of(q_heads ? least_of(wide(q, size), wide(q_out, size)) : 16, k_heads ? least_of(wide(k, size), wide(k_out, size)) : 16);
    return run(a, type, false, aligned, stream);
}

extern "C" esp_status esp_kv_norm_rotate_workspace(int64_t tokens, int32_t head_dim, int32_t q_heads, int32_t k_heads, size_t *bytes) {
    if (!bytes) return ESP_ERR_INVALID_ARG;
    if (tokens < 0 || tokens > INT32_MAX || q_heads < 0 || q_heads > 65536 || k_heads < 0 || k_heads > 65536 || head_dim < 2 || head_dim > kMostDim)
        return ESP_ERR_SHAPE;
    NormArgs a{};
    share_blocks(a, tokens, q_heads, k_heads, lanes_of(head_dim, 2, 16));
    *bytes = (size_t(a.side[0].blocks) + a.side[1].blocks) * head_dim * sizeof(float);
    return ESP_OK;
}

extern "C" esp_status esp_kv_norm_rotate_backward(const esp_kv_rope *rope, int32_t type, int64_t tokens, int32_t head_dim, int32_t q_heads,
                                                  int32_t k_heads, esp_kv_view q, esp_kv_view k, const void *q_weight, const void *k_weight,
                                                  int32_t weight_type, const int32_t *positions, float eps, esp_kv_view q_grad,
                                                  esp_kv_view k_grad, esp_kv_view dq, esp_kv_view dk, void *dq_weight, void *dk_weight,
                                                  void *workspace, size_t workspace_bytes, void *stream) {
    if (esp_status e = check(rope, type, tokens, head_dim, q_heads, k_heads, weight_type, eps)) return e;
    if (tokens == 0) q_heads = k_heads = 0;                        // the weights' gradients are 0
    if (q_heads + k_heads == 0 && !dq_weight && !dk_weight) return ESP_OK;
    if (q_heads + k_heads && !positions) return ESP_ERR_INVALID_ARG;
    if ((q_heads && (!q.data || !q_grad.data || !dq.data)) || (k_heads && (!k.data || !k_grad.data || !dk.data))) return ESP_ERR_INVALID_ARG;
    const int size = type == ESP_KV_FP32 ? 4 : 2;
    NormArgs a{{{view_of(q), view_of(q_grad), view_of(dq), q_weight, nullptr, dq_weight, q_heads, 0},
                {view_of(k), view_of(k_grad), view_of(dk), k_weight, nullptr, dk_weight, k_heads, 0}},
               {rope->turns, rope->magnitude, rope->rotary_dim, rope->interleaved}, positions, tokens, head_dim, weight_type == ESP_KV_FP32, eps, 1.0f / float(head_dim)};
    share_blocks(a, tokens, q_heads, k_heads, lanes_of(head_dim, 2, 16));
    if (dq_weight || dk_weight) {
        const size_t need = (size_t(a.side[0].blocks) + a.side[1].blocks) * head_dim * sizeof(float);
        if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need)) return ESP_ERR_WORKSPACE;
        float *p = static_cast<float *>(workspace);
        a.side[0].partial = p;
        a.side[1].partial = p + size_t(a.side[0].blocks) * head_dim;
    }
    auto both = [&](const esp_kv_view &x, const esp_kv_view &g, const esp_kv_view &d) { return least_of(wide(x, size), least_of(wide(g, size), wide(d, size))); };
    const int aligned = least_of(q_heads ? both(q, q_grad, dq) : 16, k_heads ? both(k, k_grad, dk) : 16);
    return run(a, type, true, aligned, stream);
}
