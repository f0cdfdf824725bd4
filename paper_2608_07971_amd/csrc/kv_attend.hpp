// Shared by the two attention kernels of the paged 8-bit cache.
#pragma once

#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 64;                   // tokens a wavefront takes at a time
constexpr int kDies = 8;                    // workgroups go round the dies
constexpr int kCols = 16;                   // (token, query head) rows of a unit: the columns of the matrix products
// Softmax weights are taken relative to a maximum that is raised only when a
// score passes it by kSlack, times 2^kLift, so that fp16 holds them from 2^14
// down to 2^-34 of the largest.
constexpr float kLift = 10.0f, kSlack = 4.0f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kPromptRows = 128;            // rows of a unit of many new tokens
// Values enter their product in fp16 as code * scale / 2^r, with r the output's exponent.
// That is exact for scales from 2^(r - kNear) to 2^r: e4m3's least step is 2^-9, fp16's
// 2^-24.  Blocks outside of these move r, and the output with it, so that what one block
// gives does not depend on how large others are; r stays within 2^kDown of the largest so
// far, which keeps the output in float32's range.
constexpr int kNear = 15, kDown = 80;
constexpr int kNoScale = -200;              // exponent of a value scale below any
constexpr int kApart = 1000;                // k_prompt: blocks of a tile that have no exponent in common

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
    int32_t layer, q_heads, group, window, max_new, max_length, groups, wide, wide_out, units, splits;
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
template <typename T> struct Pack;
template <> struct Pack<_Float16> { typedef half8 v8; typedef half2 v2; };
template <> struct Pack<__bf16> { typedef bhalf8 v8; typedef bhalf2 v2; };

// Bytes whose low seven bits are all set: e4m3's NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    const uint32_t hit = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return (hit >> 7) * 0xffu;
}

__device__ __forceinline__ void store_pair(float *p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), uint64_t(__float_as_uint(x)) | uint64_t(__float_as_uint(y)) << 32, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_pair(const float *p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float(uint32_t(v)), __uint_as_float(uint32_t(v >> 32)));
}

// Exponent of a scale, and what is left of it: 1 for those that append makes.
__device__ __forceinline__ int exponent(float x) { return max(-126, min(126, int((__float_as_uint(x) >> 23) & 255) - 127)); }
// 2^e, from 2^-126 on.
__device__ __forceinline__ float power(int e) { return __uint_as_float(uint32_t(max(1, min(254, e + 127))) << 23); }
// Four codes times 2^k (the exponent of `by`).
__device__ __forceinline__ half8 scaled8(uint32_t a, uint32_t b, float by) {
    const half2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, by, false), y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, by, true);
    const half2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, by, false), w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, by, true);
    return half8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// Many new tokens: kv_prompt.hip.
void launch_prompt(const AttendArgs &a, int32_t type, hipStream_t stream);

}  // namespace esp_kv
