// Shared by the kernels of the paged 8-bit cache (include/esp_kv.h).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/esp_kv.h"

namespace esp_kv {

typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// The cache as kernels take it, with the strides of its pools.
struct Cache {
    int32_t pages, layers, heads, tokens, dim, sequences, width, shift;   // tokens = 1 << shift
    uint8_t *k, *v;
    float *scale;
    int32_t *table, *lengths, *refs, *status;

    __device__ __forceinline__ int64_t block(int32_t page, int32_t layer, int32_t head) const {
        return ((int64_t(page) * layers + layer) * heads + head) * (int64_t(tokens) * dim);
    }
    __device__ __forceinline__ float *block_scale(int32_t page, int32_t layer, int32_t which, int32_t head) const {
        return scale + ((int64_t(page) * layers + layer) * 2 + which) * heads + head;
    }
};

struct Rope {
    const double *turns;
    float magnitude;
    int32_t rotary, interleaved;
};

// Rows of new tokens: offsets into the packed tokens, the sequence of each.
struct Rows {
    const int32_t *offsets, *seqs;
    int32_t rows;
    int64_t tokens;
};

__device__ __forceinline__ void record(const Cache &c, int32_t code) { atomicCAS(c.status, 0, code); }

// Row b's tokens [first, first + n) with sequence and length; n = 0 where the
// offsets, the sequence or the length are not usable.
struct Row {
    int32_t first, n, seq, length;
};
__device__ __forceinline__ Row row_of(const Cache &c, const Rows &r, int32_t b) {
    Row o{r.offsets[b], r.offsets[b + 1], r.seqs ? r.seqs[b] : b, 0};
    o.n -= o.first;
    bool ok = o.first >= 0 && o.n >= 0 && int64_t(o.first) + o.n <= r.tokens && o.seq >= 0 && o.seq < c.sequences;
    if (ok) {
        o.length = c.lengths[o.seq];
        ok = o.length >= 0 && o.length <= int64_t(c.width) << c.shift;
    }
    if (!ok) {
        record(c, ESP_ERR_SHAPE);
        o.first = o.n = o.length = o.seq = 0;
    }
    return o;
}

// cos and sin of t revolutions.  The position times the frequency is taken in
// binary64, so the fraction of a turn is good to 2^-30 at positions of a
// million; the rest are the Taylor polynomials on an eighth of a turn either
// way (errors under 2.5e-8).
__device__ __forceinline__ void cos_sin(double t, float &c, float &s) {
    const double quarter = __builtin_rint(t * 4.0);
    const float x = float((t - quarter * 0.25) * 6.283185307179586);
    const int q = int(quarter - 4.0 * __builtin_floor(quarter * 0.25));
    const float z = x * x;
    float sn = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040);
    sn = __builtin_fmaf(z, sn, 1.0f / 120);
    sn = __builtin_fmaf(z, sn, -1.0f / 6);
    sn = __builtin_fmaf(z * x, sn, x);
    float cs = __builtin_fmaf(z, 1.0f / 40320, -1.0f / 720);
    cs = __builtin_fmaf(z, cs, 1.0f / 24);
    cs = __builtin_fmaf(z, cs, -0.5f);
    cs = __builtin_fmaf(z, cs, 1.0f);
    const float a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn;
    c = (q == 1 || q == 2) ? -a : a;
    s = (q & 2) ? -b : b;
}

template <int Type> struct TypeOf;
template <> struct TypeOf<ESP_KV_BF16> { typedef __bf16 type; };
template <> struct TypeOf<ESP_KV_FP16> { typedef _Float16 type; };
template <> struct TypeOf<ESP_KV_FP32> { typedef float type; };

// Two e4m3 codes of the lower or upper half of a word as numbers (exact in both types).
template <bool High> __device__ __forceinline__ half2 codes(uint32_t w, half2 *) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, High);
}
template <bool High> __device__ __forceinline__ bhalf2 codes(uint32_t w, bhalf2 *) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, High);
}
template <typename V8, typename V2> __device__ __forceinline__ V8 codes8(uint32_t a, uint32_t b) {
    V2 *t = nullptr;
    const V2 x = codes<false>(a, t), y = codes<true>(a, t), z = codes<false>(b, t), w = codes<true>(b, t);
    return V8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

Cache cache_of(const esp_kv_cache *c);
// Status of a cache descriptor's sizes and pointers (host).
esp_status check_cache(const esp_kv_cache *c);
inline esp_status launched() { return hipGetLastError() == hipSuccess ? ESP_OK : ESP_ERR_DEVICE; }

}  // namespace esp_kv
