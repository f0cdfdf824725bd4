// Beam search's selection: of every request the `width` largest of
//   score[beam] + x[beam][token] - ln sum exp x[beam]
// over its beams and the vocabulary, ties to the lower beam, then by its logits, then the lower
// token.
// Within a beam the order is that of the logits, so one pass finds its best while the sum
// of exponentials runs along; a second launch, a workgroup a request, sums up the splits and
// compares across beams in binary64.
#include "kv_internal.hpp"

namespace esp_kv {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMostWidth = 64;              // a wavefront holds the best so far, one a lane
constexpr int kMostSplits = 16;             // of a beam's vocabulary
constexpr int kEach = 8;                    // logits a lane takes at a time
constexpr int kBatch = 64 * kEach;
constexpr float kLog2e = 1.4426950408889634f;

struct BeamArgs {
    const void *logits;
    int64_t group_stride, beam_stride;
    const float *scores;
    const uint8_t *ended;
    int32_t groups, beams, vocab, width, pad, splits, span;      // span: tokens of a split
    uint64_t *keys;                         // [row][split][width]: the best of each
    double *sums;                           // [row][split]
    float *tops;
    float *out;
    int32_t *parents, *tokens;
};

// A number's bits in an order that integers have; -0 as 0.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float number(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
// Larger is better: the logit, then the lower token.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) { return uint64_t(ordered(x)) << 32 | ~token; }

struct One {                                // a key of 64 bits
    uint64_t k;
    __device__ __forceinline__ bool operator>(const One &o) const { return k > o.k; }
};
struct Two {                                // the sum in binary64, then the lower beam, then its own order (place_of)
    uint64_t k, l;
    __device__ __forceinline__ bool operator>(const Two &o) const { return k > o.k || (k == o.k && l > o.l); }
};
// A beam's order: the logit, then the earlier split and rank there, which is the lower token.
constexpr int kMostBeams = 1024, kPlaces = kMostSplits * kMostWidth;
__device__ __forceinline__ uint64_t place_of(uint32_t beam, uint32_t logit, uint32_t split, uint32_t rank) {
    return (uint64_t(kMostBeams - 1 - beam) << 32 | logit) * kPlaces + (kPlaces - 1 - (split * kMostWidth + rank));
}
// x of the lane whose number differs in the bit With: by rows' permutations and swaps of rows
// and halves, without LDS.
template <int With> __device__ __forceinline__ uint32_t across(uint32_t x, int lane) {
    if constexpr (With == 1) return __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true);                   // quads: 1 0 3 2
    if constexpr (With == 2) return __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true);                   // 2 3 0 1
    if constexpr (With == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x1b, 0xf, 0xf, true), 0x141, 0xf, 0xf, true);   // 3 2 1 0, then eights back to front
    if constexpr (With == 8) return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true);                  // sixteens by eight
    if constexpr (With == 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return lane & 16 ? s[0] : s[1];
    }
    if constexpr (With == 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return lane & 32 ? s[0] : s[1];
    }
}
template <int With> __device__ __forceinline__ uint64_t across(uint64_t x, int lane) {
    return uint64_t(across<With>(uint32_t(x >> 32), lane)) << 32 | across<With>(uint32_t(x), lane);
}
template <int With> __device__ __forceinline__ One across(One a, int lane) { return {across<With>(a.k, lane)}; }
template <int With> __device__ __forceinline__ Two across(Two a, int lane) { return {across<With>(a.k, lane), across<With>(a.l, lane)}; }
__device__ __forceinline__ One from_lane(One a, int lane) { return {uint64_t(__shfl(int64_t(a.k), lane))}; }
__device__ __forceinline__ Two from_lane(Two a, int lane) { return {uint64_t(__shfl(int64_t(a.k), lane)), uint64_t(__shfl(int64_t(a.l), lane))}; }

// Keys of the lanes from the largest on, by a bitonic network.
template <int With, typename K> __device__ __forceinline__ K exchange(K mine, int lane, bool larger) {
    const K other = across<With>(mine, lane);
    return (other > mine) == larger ? other : mine;
}
template <int With, typename K> __device__ __forceinline__ K halved(K mine, int lane, bool down) {      // of a bitonic stretch
    mine = exchange<With>(mine, lane, ((lane & With) == 0) == down);
    if constexpr (With > 1) mine = halved<With / 2>(mine, lane, down);
    return mine;
}
template <typename K> __device__ __forceinline__ K sorted(K mine, int lane) {
    mine = halved<1>(mine, lane, (lane & 2) == 0);
    mine = halved<2>(mine, lane, (lane & 4) == 0);
    mine = halved<4>(mine, lane, (lane & 8) == 0);
    mine = halved<8>(mine, lane, (lane & 16) == 0);
    mine = halved<16>(mine, lane, (lane & 32) == 0);
    return halved<32>(mine, lane, true);
}
// The 64 largest of two sorted sets.
template <typename K> __device__ __forceinline__ K merged(K best, K more, int lane) {
    more = from_lane(more, 63 - lane);
    best = more > best ? more : best;
    return halved<32>(best, lane, true);
}

__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The best keys that a wavefront has seen.  What passes the `width`-th of them
// waits in LDS until there are 64 to be sorted in.
template <typename K> struct Best {
    K best, least;                          // least: the width-th
    K *queue;                               // [128]
    int lane, width, waiting;
    __device__ __forceinline__ void start(K first, K *q, int w) {
        lane = threadIdx.x & 63;
        queue = q;
        width = w;
        waiting = 0;
        best = sorted(first, lane);
        least = from_lane(best, width - 1);
    }
    __device__ __forceinline__ void join(K more) {
        best = merged(best, sorted(more, lane), lane);
        least = from_lane(best, width - 1);
    }
    // there: whether k passes `least`
    __device__ __forceinline__ void offer(K k, bool there) {
        const uint64_t who = __ballot(there);
        if (!who) return;
        if (there) queue[waiting + __builtin_amdgcn_mbcnt_hi(uint32_t(who >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(who), 0))] = k;
        waiting += __popcll(who);
        if (waiting < 64) return;
        wave_fence();
        const K now = queue[lane], rest = queue[64 + lane];
        wave_fence();
        queue[lane] = rest;
        waiting -= 64;
        join(now);
    }
    __device__ __forceinline__ void finish() {
        wave_fence();
        if (waiting) join(lane < waiting ? queue[lane] : K{});
    }
};

// Running sum of exp(x - top).
struct Sum {
    float top, sum;
    __device__ __forceinline__ static float off(float top) { return top == -INFINITY ? 0.0f : top; }
    template <int M, int N> __device__ __forceinline__ void add(const float (&x)[M][N], float most) {
        const float to = fmaxf(top, most), by = off(to);
        float s = sum * __builtin_amdgcn_exp2f((top - by) * kLog2e);
#pragma unroll
        for (int i = 0; i < M; i++)
#pragma unroll
            for (int j = 0; j < N; j++) s += __builtin_amdgcn_exp2f((x[i][j] - by) * kLog2e);
        top = to;
        sum = s;
    }
};

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Eight {
    T x[kEach];
};

// A workgroup a split of a beam's vocabulary.  Each wavefront starts with its lanes' largest
// of the first turn; after that a logit has to pass the width-th best, which few do: these
// are marked in a mask a lane and read once more in one short loop (with the code for them at
// every logit, 119 KB of it, a turn took twice as long).  A row's sums are taken by places
// in the row alone, so copies of a row have equal sums wherever they lie.
// A turn's loads are waited for before its arithmetic (conversion, maximum, difference, product,
// exponential, sum, comparison), and four wavefronts a SIMD do not hide them: 512 rows of 131,072 in
// bf16 (134 MB) 39 us (3.4 TB/s), where reading alone takes 20 to 27; 4 rows of 32,000 8.3 us, a
// chain of loading, sorting and joining.
template <typename T> __global__ __launch_bounds__(kThreads) void k_beam_rows(BeamArgs a) {
    __shared__ One lds[kWaves][128];
    __shared__ float tops[kWaves];
    __shared__ double sums[kWaves];
    constexpr int kFlight = 8 / int(sizeof(T));                  // vectors at a time
    const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const float score = a.scores[row];
    if (!(fabsf(score) < INFINITY) || (a.ended && a.ended[row])) return;        // k_beam_join does not ask for it
    const int group = row / a.beams;
    const T *x = static_cast<const T *>(a.logits) + group * a.group_stride + (row - group * a.beams) * a.beam_stride;
    const int64_t from = int64_t(split) * a.span, to = min(int64_t(a.vocab), from + a.span);

    Eight<T> e[kFlight];
    auto load = [&](int64_t at) {
#pragma unroll
        for (int f = 0; f < kFlight; f++) {
            const int64_t i = at + f * (kWaves * kBatch) + lane * kEach;
            if (i + kEach <= to) {
                e[f] = *reinterpret_cast<const Eight<T> *>(x + i);
            } else {
#pragma unroll
                for (int j = 0; j < kEach; j++) e[f].x[j] = i + j < to ? x[i + j] : T(-INFINITY);
            }
        }
    };
    Best<One> best;
    Sum sum{-INFINITY, 0.0f};
    bool first = true;
    for (int64_t at = from + wave * kBatch; at < to; at += kWaves * kBatch * kFlight) {
        load(at);
        float v[kFlight][kEach];
#pragma unroll
        for (int f = 0; f < kFlight; f++)
#pragma unroll
            for (int j = 0; j < kEach; j++) v[f][j] = float(e[f].x[j]);
        float most[kFlight], top = -INFINITY;
#pragma unroll
        for (int f = 0; f < kFlight; f++) {
            most[f] = v[f][0];
#pragma unroll
            for (int j = 1; j < kEach; j++) most[f] = fmaxf(most[f], v[f][j]);
            top = fmaxf(top, most[f]);
        }
        sum.add(v, top);
        auto token = [&](int i) { return at + i / kEach * (kWaves * kBatch) + lane * kEach + i % kEach; };
        uint64_t own = 0;
        if (first) {                        // starts with each lane's largest
#pragma unroll
            for (int i = 0; i < kFlight * kEach; i++) own = max(own, key_of(v[i / kEach][i % kEach], uint32_t(token(i))));
            best.start(One{own}, lds[wave], a.width);
        }
        const float least = number(uint32_t(best.least.k >> 32));
        uint32_t passes = 0;
        if (first) {
#pragma unroll
            for (int i = 0; i < kFlight * kEach; i++) passes |= v[i / kEach][i % kEach] >= least ? 1u << i : 0;
        } else {                            // of equal ones the earlier is better: a later one has to be larger
            if (!__any(top > least)) continue;
#pragma unroll
            for (int i = 0; i < kFlight * kEach; i++) passes |= v[i / kEach][i % kEach] > least ? 1u << i : 0;
        }
        first = false;
        for (; __any(passes != 0); passes &= passes - 1) {       // few: read once more
            const int64_t t = passes ? token(__builtin_ctz(passes)) : at, held = min(t, to - 1);
            const One k{key_of(t < to ? float(x[held]) : -INFINITY, uint32_t(t))};
            best.offer(k, passes && k > best.least && k.k != own);
        }
    }
    if (first) best.start(One{0}, lds[wave], a.width);           // nothing for this wavefront
    best.finish();
    // over the wavefront, then over the workgroup, in binary64
    float top = sum.top;
#pragma unroll
    for (int m = 32; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    double total = double(sum.sum) * double(__builtin_amdgcn_exp2f((sum.top - Sum::off(top)) * kLog2e));
#pragma unroll
    for (int m = 32; m; m >>= 1) total += __shfl_xor(total, m);
    wave_fence();
    lds[wave][lane] = best.best;
    if (lane == 0) {
        tops[wave] = top;
        sums[wave] = total;
    }
    __syncthreads();
    if (wave) return;
    One all = best.best;
#pragma unroll 1
    for (int w = 1; w < kWaves; w++) all = merged(all, lds[w][lane], lane);
    if (lane < a.width) a.keys[int64_t(blockIdx.x) * a.width + lane] = all.k;
    if (lane == 0) {
#pragma unroll
        for (int w = 1; w < kWaves; w++) top = fmaxf(top, tops[w]);
        total = 0.0;
#pragma unroll
        for (int w = 0; w < kWaves; w++) total += sums[w] * double(__builtin_amdgcn_exp2f((tops[w] - Sum::off(top)) * kLog2e));
        a.tops[blockIdx.x] = top;
        a.sums[blockIdx.x] = total;
    }
}

__device__ __forceinline__ uint64_t ordered(double x) {
    const uint64_t u = uint64_t(__double_as_longlong(x + 0.0));
    return u >> 63 ? ~u : u | uint64_t(1) << 63;
}
__device__ __forceinline__ double number(uint64_t u) { return __longlong_as_double(int64_t(u >> 63 ? u & ~(uint64_t(1) << 63) : ~u)); }

// A workgroup a request (64 of 8 beams 6.4 us, one of 4 beams in 16 splits 4.1 us): beams' sums over
// their splits, then, by one wavefront, the best of what they left.
__global__ __launch_bounds__(kThreads) void k_beam_join(BeamArgs a) {
    __shared__ Two queue[128];
    extern __shared__ double lse[];         // [beams]; NaN: no candidates
    const int group = blockIdx.x, lane = threadIdx.x & 63;
    // the lists' first ones before their second; the first 64 on their way while the sums are made
    const uint32_t lists = a.beams * a.splits, all = lists * a.width;          // at most 2^20
    auto key = [&](uint32_t i) {
        const uint32_t rank = i / lists, list = i - rank * lists;
        return i < all ? a.keys[(int64_t(group) * lists + list) * a.width + rank] : 0;
    };
    const uint64_t early = key(lane);
    for (int b0 = 0; b0 < a.beams; b0 += kThreads / kMostSplits) {             // a beam by as many lanes as it may have splits
        const int b = b0 + threadIdx.x / kMostSplits, i = threadIdx.x % kMostSplits, row = group * a.beams + min(b, a.beams - 1);
        const bool ended = a.ended && a.ended[row], live = !ended && fabsf(a.scores[row]) < INFINITY, there = live && i < a.splits;
        const int64_t at = int64_t(row) * a.splits + min(i, a.splits - 1);
        const float own = there ? a.tops[at] : -INFINITY;
        const double part = there ? a.sums[at] : 0.0;
        float top = own;
#pragma unroll
        for (int m = kMostSplits / 2; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
        double sum = there ? part * exp2((double(own) - Sum::off(top)) * 1.4426950408889634074) : 0.0;
#pragma unroll
        for (int m = kMostSplits / 2; m; m >>= 1) sum += __shfl_xor(sum, m);
        if (i == 0 && b < a.beams) lse[b] = live ? double(top) + log(sum) : ended ? 0.0 : double(NAN);
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;          // the rest is one wavefront's
    Best<Two> best;
    // lists are sorted in this order, too, where sums of a beam are equal but its logits are not: once
    // as many in a row as there are lists have not passed, no other does
    uint32_t quiet = 0;
    for (uint32_t i0 = 0; i0 < all && quiet < lists; i0 += 64) {
        Two k{0, 0};
        if (i0 + lane < all) {
            const uint32_t rank = (i0 + lane) / lists, list = i0 + lane - rank * lists, beam = list / uint32_t(a.splits);
            const int row = group * a.beams + beam;
            const double s = double(a.scores[row]);
            double total = NAN;
            uint32_t logit = 0;
            if (a.ended && a.ended[row]) {
                if (rank == 0 && list == beam * a.splits) total = s;
            } else if (fabs(s) < INFINITY) {
                const uint64_t held = i0 == 0 ? early : key(i0 + lane);
                logit = uint32_t(held >> 32);
                if (held) total = s + (double(number(logit)) - lse[beam]);
            }
            if (fabs(total) < INFINITY) k = {ordered(total), place_of(beam, logit, list - beam * a.splits, rank)};
        }
        if (i0 == 0) {
            best.start(k, queue, a.width);
            continue;
        }
        const bool passes = k > best.least;
        quiet = __any(passes) ? 0 : quiet + 64;
        best.offer(k, passes);
    }
    best.finish();
    if (lane < a.width) {
        const bool there = best.best.k != 0;
        const int64_t at = int64_t(group) * a.width + lane;
        const uint32_t beam = kMostBeams - 1 - uint32_t(best.best.l / kPlaces >> 32), place = kPlaces - 1 - uint32_t(best.best.l % kPlaces);
        const int row = there ? group * a.beams + int(beam) : -1;
        int token = there ? a.pad : -1;
        if (there && !(a.ended && a.ended[row]))
            token = int(~uint32_t(a.keys[(int64_t(row) * a.splits + place / kMostWidth) * a.width + place % kMostWidth]));
        a.out[at] = there ? float(number(best.best.k)) : -INFINITY;
        a.parents[at] = row;
        a.tokens[at] = token;
    }
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

constexpr int kMostVocab = 1 << 30;
constexpr int64_t kMostRows = 1 << 23;      // a launch's threads are numbered in 32 bits

esp_status check(int32_t groups, int32_t beams, int32_t vocab, int32_t width) {
    if (groups < 0 || beams < 1 || beams > kMostBeams || vocab < 1 || vocab > kMostVocab || width < 1 || width > kMostWidth) return ESP_ERR_SHAPE;
    return int64_t(groups) * beams > kMostRows ? ESP_ERR_SHAPE : ESP_OK;
}

// Splits of a beam's vocabulary: as many workgroups as the GPU holds, none of less than a
// turn.  512 rows of 131,072: 1,024 workgroups 40 us, 2,048 57.
void lay_out(BeamArgs &a) {
    const int64_t rows = int64_t(a.groups) * a.beams, turn = kWaves * kBatch;
    const int64_t most = (a.vocab + turn - 1) / turn;
    int64_t splits = rows ? 1024 / rows : 1;
    splits = splits < 1 ? 1 : splits > kMostSplits ? kMostSplits : splits;
    splits = splits > most ? most : splits;
    a.span = int32_t(((a.vocab + splits - 1) / splits + turn - 1) / turn * turn);
    a.splits = int32_t((int64_t(a.vocab) + a.span - 1) / a.span);
}
size_t bytes_of(const BeamArgs &a) {
    const size_t n = size_t(a.groups) * a.beams * a.splits;
    return n * (a.width * sizeof(uint64_t) + sizeof(double) + sizeof(float));
}

}  // namespace

extern "C" esp_status esp_kv_select_beams_workspace(int32_t groups, int32_t beams, int32_t vocab, int32_t width, size_t *bytes) {
    if (!bytes) return ESP_ERR_INVALID_ARG;
    if (esp_status e = check(groups, beams, vocab, width)) return e;
    BeamArgs a{};
    a.groups = groups;
    a.beams = beams;
    a.vocab = vocab;
    a.width = width;
    lay_out(a);
    *bytes = bytes_of(a);
    return ESP_OK;
}

extern "C" esp_status esp_kv_select_beams(int32_t type, int32_t groups, int32_t beams, int32_t vocab, int32_t width, const void *logits,
                                          int64_t group_stride, int64_t beam_stride, const float *scores, const uint8_t *ended,
                                          int32_t pad, float *scores_out, int32_t *parents, int32_t *tokens, void *workspace,
                                          size_t workspace_bytes, void *stream) {
    if (type < ESP_KV_BF16 || type > ESP_KV_FP32) return ESP_ERR_INVALID_ARG;
    if (esp_status e = check(groups, beams, vocab, width)) return e;
    if (ended && (pad < 0 || pad >= vocab)) return ESP_ERR_INVALID_ARG;
    if (groups == 0) return ESP_OK;
    if (!logits || !scores || !scores_out || !parents || !tokens) return ESP_ERR_INVALID_ARG;
    BeamArgs a{logits, group_stride, beam_stride, scores, ended, groups, beams, vocab, width, pad, 0, 0, nullptr, nullptr, nullptr, scores_out, parents, tokens};
    lay_out(a);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < bytes_of(a)) return ESP_ERR_WORKSPACE;
    const size_t n = size_t(groups) * beams * a.splits;
    a.keys = static_cast<uint64_t *>(workspace);
    a.sums = reinterpret_cast<double *>(a.keys + n * width);
    a.tops = reinterpret_cast<float *>(a.sums + n);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const unsigned blocks = unsigned(n);
    if (type == ESP_KV_BF16) k_beam_rows<__bf16><<<blocks, kThreads, 0, s>>>(a);
    else if (type == ESP_KV_FP16) k_beam_rows<_Float16><<<blocks, kThreads, 0, s>>>(a);
    else k_beam_rows<float><<<blocks, kThreads, 0, s>>>(a);
    k_beam_join<<<unsigned(groups), kThreads, size_t(beams) * sizeof(double), s>>>(a);
    return launched();
}
