// Attention of many new tokens over the paged 8-bit cache.
#include "kv_attend.hpp"

#include <type_traits>

namespace esp_kv {

typedef float float16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float16v product32(half8 x, half8 y, float16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float16v product32(bhalf8 x, bhalf8 y, float16v z) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0); }

// A workgroup takes 128 rows (token, query head) of one sequence and key head
// against tiles of 64 tokens, each of its four wavefronts 32 rows.  Codes
// become 16-bit numbers once, on their way into LDS, for all four; while a tile
// is worked on, the codes of the next are on their way into registers.  Scores
// and output are held transposed, as in k_attend: the rows of the key matrix
// are taken in the order that leaves the softmax weights in place for the
// value product.  V's block scales enter as the codes are widened, exactly (kNear),
// K's with the softmax scale.
// Bound by the wavefronts' issue, products and the softmax between them: 3
// sequences of up to 16,000 tokens, up to 2,048 of them new, 32 query heads of 128,
// 847 GFLOP in 930 us (911 TFLOP/s); 16 heads of 64 in a window of 1,000 tokens, 21
// GFLOP in 63.5 us (335 TFLOP/s, a third of it in tiles that only some rows see).
template <typename T, int Dim, int Page> __global__ __launch_bounds__(kThreads, Dim == 64 ? 3 : 2) void k_prompt(AttendArgs a) {
    typedef typename Pack<T>::v8 V8;
    typedef typename Pack<T>::v2 V2;
    constexpr int kSteps = Dim / 16;        // matrix steps of a score
    constexpr int kOut = Dim / 32;          // matrix tiles of an output
    constexpr int kKeyUnits = kTile * Dim / 16 / kThreads, kSegs = Dim / 16;
    constexpr int kKeyRow = Dim * 2;        // bytes of a token in LDS
    constexpr int kHalf = kTile * Dim * 2;  // bytes of a tile's keys in LDS, and of its values
    __shared__ __align__(16) uint8_t lds[2][2 * kHalf];          // two tiles: keys, then values
    __shared__ uint32_t nans[2];
    __shared__ uint32_t ticket;

    const Cache &c = a.c;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 31, half = lane >> 5;
    if (blockIdx.x == 0) {                  // beside the list: what is wrong with any row, also one that no unit is found for
        for (int b = tid; b < a.rows.rows; b += kThreads) usable_row(a, b);
        return;
    }
    // the dies take stretches of the list [head][part][unit], so that a die's cache holds the keys of few heads
    const int place = blockIdx.x - 1, per_die = (gridDim.x - 1) / kDies, item = place % kDies * per_die + place / kDies;
    const int per_head = a.units * a.splits, head = item / per_head;
    if (head >= c.heads) return;
    const int part = (item - head * per_head) / a.units, index = a.units - 1 - (item - head * per_head - part * a.units);

    // units: row b's begin at offsets[b] * group / 128 + b at the earliest
    int lo = 0, hi = a.rows.rows - 1;
    auto base_of = [&](int b) { return int64_t(a.rows.offsets[b]) * a.group / kPromptRows + b; };
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (base_of(mid) <= index) lo = mid;
        else hi = mid - 1;
    }
    Row row = usable_row(a, lo);
    row.first = __builtin_amdgcn_readfirstlane(row.first);
    row.n = __builtin_amdgcn_readfirstlane(row.n);
    row.seq = __builtin_amdgcn_readfirstlane(row.seq);
    row.length = __builtin_amdgcn_readfirstlane(row.length);
    const int64_t unit64 = index - base_of(lo);
    const int n_rows = row.n * a.group;
    if (unit64 < 0 || unit64 * kPromptRows >= n_rows) return;
    const int r0 = __builtin_amdgcn_readfirstlane(int(unit64)) * kPromptRows, p0 = row.length - row.n;

    // this lane's query; the wavefront's and the workgroup's positions
    const int r = r0 + wave * 32 + col, token = r / a.group, q_head = head * a.group + r - token * a.group;
    const int pos = r < n_rows ? p0 + token : -1, low = a.window > 0 ? pos - a.window : -1;
    const int w0 = min(r0 + wave * 32, n_rows - 1), w1 = min(r0 + wave * 32 + 31, n_rows - 1);
    const int pos_first = p0 + w0 / a.group, pos_last = p0 + w1 / a.group;
    Span span = span_of(p0 + r0 / a.group, p0 + min(r0 + kPromptRows - 1, n_rows - 1) / a.group, a.window);
    {
        const int share = (span.size() + a.splits - 1) / a.splits;
        span.from += part * share;
        span.to = min(span.to, span.from + share);
    }

    // the softmax scale's sign goes into the queries, so that a larger product is a larger score
    const float scale = fabsf(a.scale);
    V8 q[kSteps];
    {
        const T *src = static_cast<const T *>(a.q.data) + int64_t(row.first + token) * a.q.token + int64_t(q_head) * a.q.head + 8 * half;
#pragma unroll
        for (int s = 0; s < kSteps; s++) {
            V8 x{};
            if (r < n_rows) {
                if (a.wide) x = *reinterpret_cast<const V8 *>(src + 16 * s);
                else
#pragma unroll
                    for (int j = 0; j < 8; j++) x[j] = src[16 * s + j];
            }
            if (a.scale < 0.0f)
#pragma unroll
                for (int j = 0; j < 8; j++) x[j] = -x[j];
            q[s] = x;
        }
    }
    float16v o[kOut];                       // row 8 b + 4 half + i of tile d: element 32 d + 16 half + 4 b + i
#pragma unroll
    for (int d = 0; d < kOut; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = 0.0f;
    float m_run = -INFINITY, l_run = 0.0f;
    int o_exp = kNoScale, o_top = kNoScale; // exponent of the output, and the largest so far

    const uint32_t page_step = uint32_t(c.layers * c.heads) * (Page * Dim);
    const int64_t block_at = int64_t(a.layer * c.heads + head) * (Page * Dim);
    const uint8_t *keys = c.k + block_at, *vals = c.v + block_at;
    const float *scales = c.scale + 2 * a.layer * c.heads + head;
    const int32_t *table = c.table + int64_t(row.seq) * c.width;

    // What is known of a tile's four groups of 16 tokens: lane g (and 4 + g, ...) has
    // group g's page (-1 none) and scales.
    struct Group {
        int page;
        float k, v;
    };
    auto page_of = [&](int t) {
        const int at = t * kTile + 16 * (lane & 3);
        const int page = at < row.length ? table[at / Page] : -1;
        return uint32_t(page) < uint32_t(c.pages) ? page : -1;
    };
    auto scales_of = [&](int page) {
        const float *p = scales + uint64_t(max(page, 0)) * uint32_t(2 * c.layers * c.heads);
        return Group{page, p[0], p[c.heads]};
    };
    auto lane_float = [&](float x, int g) { return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(__float_as_uint(x), g))); };

    // Unit u of the keys: 16 bytes of token u / kSegs.  Unit u of the values: 16
    // tokens of one dimension, in the order in which pages hold them.  A wavefront's
    // units of one kind lie in one page.
    constexpr int kPageGroups = Page / 16;
    uint32_t key_from[kKeyUnits], value_from[kKeyUnits];         // place in the page
    uint32_t key_to[kKeyUnits], value_to[kKeyUnits];             // and in LDS
    int key_group[kKeyUnits], value_group[kKeyUnits], value_first[kKeyUnits];
    // A 16-byte chunk's place in its row of LDS is turned by the row, so that the 16
    // rows that a matrix step reads at once lie in different banks.
    auto key_turn = [](int token) { return Dim == 128 ? token & 15 : (token >> 1) & 7; };
    auto value_turn = [](int d) { return ((d >> 1) & 3) | ((d >> 2) & 4); };
#pragma unroll
    for (int i = 0; i < kKeyUnits; i++) {
        const int u = tid + i * kThreads, token = u / kSegs, seg = u % kSegs;
        key_from[i] = token % Page * Dim + seg * 16;
        key_to[i] = token * kKeyRow + ((2 * seg ^ key_turn(token)) << 4);
        key_group[i] = __builtin_amdgcn_readfirstlane(token >> 4);
        const int d = u / kPageGroups % Dim, first = u / (kPageGroups * Dim) * kPageGroups, g = first + u % kPageGroups;
        value_from[i] = d * Page + g % kPageGroups * 16;
        value_to[i] = kHalf + d * (kTile * 2) + ((2 * g ^ value_turn(d)) << 4);
        value_group[i] = g;
        value_first[i] = __builtin_amdgcn_readfirstlane(first);
    }
    uint4v kw[kKeyUnits], vw[kKeyUnits];
    // Pages that are not there are read as page 0: what came in is masked.
    auto load = [&](int page) {
#pragma unroll
        for (int i = 0; i < kKeyUnits; i++) {
            const uint32_t pk = max(__builtin_amdgcn_readlane(page, key_group[i]), 0), pv = max(__builtin_amdgcn_readlane(page, value_first[i]), 0);
            kw[i] = *reinterpret_cast<const uint4v *>(keys + uint64_t(pk) * page_step + key_from[i]);
            vw[i] = *reinterpret_cast<const uint4v *>(vals + uint64_t(pv) * page_step + value_from[i]);
        }
    };
    // The exponent that a tile's values are taken relative to: that of the output, or the
    // tile's largest where a block is too far from it; kApart where the blocks are too far
    // from each other, and each has its own, in order.
    auto scale_exponent = [&](const Group &grp) { return grp.page < 0 ? kNoScale : grp.v != 0.0f ? exponent(grp.v) : max(o_exp, -126); };
    auto ref_of = [&](const Group &grp) {
        const int e = scale_exponent(grp);
        auto near = [&](int r) { return __all(e == kNoScale || (e <= r && e >= r - kNear)); };
        if (near(o_exp)) return o_exp;
        int most = kNoScale;
#pragma unroll
        for (int g = 0; g < 4; g++) most = max(most, __builtin_amdgcn_readlane(e, g));
        const int to = max(most, max(o_top, most) - kDown);
        return near(to) ? to : kApart;
    };
    // Where a tile's blocks are apart: after a group of exponent x.
    auto ref_after = [&](int r, int &top, int x) {
        top = max(top, x);
        return x > r || (x > kNoScale && x < r - kNear) ? max(x, top - kDown) : r;
    };
    // Widens the loaded tile into LDS, values divided by 2^r.
    auto store = [&](auto fast, int t, int buffer, const Group &grp, int ref, bool whole) {
        const int e = exponent(grp.v);
        int r = ref;
        if (ref == kApart) {
            const int own = scale_exponent(grp);
            int at = o_exp, top = o_top;
#pragma unroll
            for (int g = 0; g < 4; g++) {
                at = ref_after(at, top, __builtin_amdgcn_readlane(own, g));
                r = (lane & 3) == g ? at : r;
            }
        }
        const float by = power(e - r), rest = ldexpf(grp.v, -e);
        const bool powers = __all(rest == 1.0f || grp.page < 0);
#pragma unroll
        for (int i = 0; i < kKeyUnits; i++) {
            V8 *to = reinterpret_cast<V8 *>(&lds[buffer][key_to[i]]), *to2 = reinterpret_cast<V8 *>(&lds[buffer][key_to[i] ^ 16]);
            *to = codes8<V8, V2>(kw[i][0], kw[i][1]);
            *to2 = codes8<V8, V2>(kw[i][2], kw[i][3]);
        }
#pragma unroll
        for (int i = 0; i < kKeyUnits; i++) {
            if (!decltype(fast)::value && !whole) {     // past the end, or without a page: codes of 0
                const int held = __builtin_amdgcn_readlane(grp.page, value_first[i]) < 0 ? 0 : row.length - t * kTile - 16 * value_group[i];
                uint32_t bad = 0;
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    const int left = held - 4 * x;
                    const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
                    vw[i][x] = vw[i][x] & keep;
                    bad |= nan_bytes(vw[i][x]);
                }
                if (bad) nans[buffer] = t + 1;
            }
            const float f = lane_float(by, value_first[i]);
            half8 x = scaled8(vw[i][0], vw[i][1], f), y = scaled8(vw[i][2], vw[i][3], f);
            if (!powers) {                  // a scale that is no power of two: one more rounding, to fp16
                const float z = __builtin_amdgcn_readlane(grp.page, value_first[i]) < 0 ? 0.0f : lane_float(rest, value_first[i]);
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    x[j] = _Float16(float(x[j]) * z);
                    y[j] = _Float16(float(y[j]) * z);
                }
            }
            *reinterpret_cast<half8 *>(&lds[buffer][value_to[i]]) = x;
            *reinterpret_cast<half8 *>(&lds[buffer][value_to[i] ^ 16]) = y;
        }
    };
    // whether every row of the workgroup sees all of a tile
    const int first_of_all = p0 + r0 / a.group, last_of_all = p0 + min(r0 + kPromptRows - 1, n_rows - 1) / a.group;
    auto inside = [&](int t, const Group &grp) {
        return t * kTile + kTile - 1 <= first_of_all && (a.window <= 0 || t * kTile > last_of_all - a.window) && __all(grp.page >= 0);
    };

    if (tid < 2) nans[tid] = 0;
    Group now{-1, 0.0f, 0.0f}, next{-1, 0.0f, 0.0f};
    int after = -1;                         // pages of the tile after next
    int ref = kNoScale;                     // of the present tile
    if (span.from < span.to) {
        now = scales_of(page_of(span.from));
        load(now.page);
        if (span.from + 1 < span.to) after = page_of(span.from + 1);
        ref = ref_of(now);
        __syncthreads();
        store(std::false_type{}, span.from, 0, now, ref, inside(span.from, now));
    }
    __syncthreads();
    // key row m of a matrix tile is the token whose bits 2 and 3 are those of m exchanged
    const int key_row = (col & 19) | (col & 4) << 1 | (col & 8) >> 1;
    const int value_row = (col & 4) << 2 | (col & 24) >> 1 | (col & 3);
    const uint32_t key_at = key_row * kKeyRow + ((half ^ key_turn(key_row)) << 4);
    const uint32_t value_at = kHalf + value_row * (kTile * 2) + ((half ^ value_turn(value_row)) << 4);
    // A tile, and the next into LDS.  fast: every row of the workgroup sees all of both, and
    // this one's blocks are not apart.
    auto step = [&](auto fast, int t) {
        constexpr bool Fast = decltype(fast)::value;
        const int buffer = (t - span.from) & 1;
        const bool more = Fast || t + 1 < span.to;
        if (more) {
            next = scales_of(after);
            load(next.page);
            if (t + 2 < span.to) after = page_of(t + 2);
        }
        float16v s[2];
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int i = 0; i < 16; i++) s[j][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < kSteps; k++) {
#pragma unroll
            for (int j = 0; j < 2; j++)
                s[j] = product32(*reinterpret_cast<const V8 *>(&lds[buffer][(key_at ^ (k << 5)) + j * 32 * kKeyRow]), q[k], s[j]);
        }
        // the reads stay 2 steps ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int k = 0; k < kSteps - 2; k++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        // s[j][4 b + i]: token 32 j + 16 (b / 2) + 8 half + 4 (b % 2) + i, so that
        // s[g / 2][8 (g % 2) + i] is token 8 half + i of group g
        float ks[4];
        const float scaled = now.k * scale;
#pragma unroll
        for (int g = 0; g < 4; g++) ks[g] = lane_float(scaled, g);
        const bool whole = Fast || (__all(now.page >= 0) && t * kTile + kTile - 1 <= pos_first && (a.window <= 0 || t * kTile > pos_last - a.window));
        if (!whole) {
            bool lost = false;
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const bool ok = __builtin_amdgcn_readlane(now.page, g) >= 0;
                lost |= !ok && t * kTile + 16 * g < row.length;
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int tt = t * kTile + 16 * g + 8 * half + i;
                    s[g >> 1][8 * (g & 1) + i] = tt <= pos && tt > low && ok ? s[g >> 1][8 * (g & 1) + i] * ks[g] : -INFINITY;
                }
                ks[g] = 1.0f;
            }
            if (lost && lane == 0) record(c, ESP_ERR_SHAPE);
        }
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < 4; g++) {
            float x = s[g >> 1][8 * (g & 1)];
#pragma unroll
            for (int i = 1; i < 8; i++) x = fmaxf(x, s[g >> 1][8 * (g & 1) + i]);
            top = fmaxf(top, x * ks[g]);    // ks >= 0
        }
        {
            const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(z[0]), __uint_as_float(z[1]));
        }
        const int to = !Fast && ref == kApart ? o_exp : ref;
        if (__any(top > m_run + kSlack) || to != o_exp) {
            const float m = fmaxf(m_run, top), by = m_run == m ? 1.0f : __builtin_amdgcn_exp2f(m_run - m);
            const float down = by * (to != o_exp ? ldexpf(1.0f, max(o_exp - to, -200)) : 1.0f);
            m_run = m;
            o_exp = to;
            o_top = max(o_top, to);
            l_run *= by;
#pragma unroll
            for (int d = 0; d < kOut; d++) o[d] *= down;
        }
        const float base = m_run == -INFINITY ? 0.0f : m_run - kLift;
        half8 w[4];
#pragma unroll
        for (int g = 0; g < 4; g++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g >> 1][8 * (g & 1) + i], ks[g], -base));
                l_run += x;
                w[g][i] = _Float16(x);
            }
        if (!Fast && nans[buffer] == uint32_t(t + 1)) {
            // A NaN value that only some rows see must not reach the others through
            // 0 * NaN: it is looked for token by token, then it becomes 0 in LDS.
            for (int x = 0; x < kTile; x++) {
                const int tt = t * kTile + x;
                if (tt > pos || tt <= low) continue;
#pragma unroll
                for (int d = 0; d < kOut; d++)
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const _Float16 v = *reinterpret_cast<const _Float16 *>(&lds[buffer][kHalf + (32 * d + 16 * half + i) * (kTile * 2) + ((x >> 3 ^ value_turn(16 * half + i)) << 4) + 2 * (x & 7)]);
                        if (v != v) o[d][i] = NAN;
                    }
            }
            __syncthreads();                // the same for the whole workgroup
            for (int x = tid; x < kTile * Dim; x += kThreads) {
                _Float16 *v = reinterpret_cast<_Float16 *>(lds[buffer] + kHalf) + x;
                if (*v != *v) *v = _Float16(0.0f);
            }
            __syncthreads();
        }
        const int e_own = scale_exponent(now);
#pragma unroll
        for (int g = 0; g < 4; g++) {
            if (!Fast && ref == kApart) {
                const int r = ref_after(o_exp, o_top, __builtin_amdgcn_readlane(e_own, g));
                const float by = ldexpf(1.0f, max(o_exp - r, -200));
                o_exp = r;
#pragma unroll
                for (int d = 0; d < kOut; d++) o[d] *= by;
            }
#pragma unroll
            for (int d = 0; d < kOut; d++)
                o[d] = product32(*reinterpret_cast<const half8 *>(&lds[buffer][(value_at ^ (g << 5)) + d * 32 * (kTile * 2)]), w[g], o[d]);
        }
        if (more) {
            ref = ref_of(next);
            store(fast, t + 1, buffer ^ 1, next, ref, Fast || inside(t + 1, next));
            now = next;
        }
        __syncthreads();
    };
    // tiles that every row sees by its position
    const int seen_from = a.window > 0 ? max(0, last_of_all - a.window + kTile) / kTile : 0, seen_to = (first_of_all + 1) / kTile;
    for (int t = span.from; t < span.to; t++) {
        for (; t >= seen_from && t + 1 < min(seen_to, span.to) && ref != kApart && __all(now.page >= 0 && after >= 0); t++) step(std::true_type{}, t);
        step(std::false_type{}, t);
    }

    // finish: element 32 d + 16 half + x of this lane's row is o[d][x]
    {
        const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(z[0]) + __uint_as_float(z[1]);
    }
    const bool none = m_run == -INFINITY && !(l_run != l_run);
    float lse = none ? -INFINITY : m_run - kLift + __builtin_log2f(l_run);
    const float by = none ? 0.0f : ldexpf(1.0f, max(o_exp, -149)) / l_run;
#pragma unroll
    for (int d = 0; d < kOut; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = none ? 0.0f : o[d][i] * by;

    if (a.splits > 1) {
        // as in k_attend: parts by agent-scope atomics, the last to arrive joins them in order
        constexpr int kPart = kPromptRows * (Dim + 2);
        const int64_t unit_id = int64_t(head) * a.units + index;
        // pair x of lane y of a wavefront lies at 64 x + y; the last pairs hold lse
        float *parts = a.partial + unit_id * a.splits * kPart + wave * (32 * (Dim + 2)) + 2 * lane;
        {
            float *mine = parts + int64_t(part) * kPart;
#pragma unroll
            for (int d = 0; d < kOut; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 2) store_pair(mine + (8 * d + i / 2) * 128, o[d][i], o[d][i + 1]);
            if (half == 0) store_pair(mine + Dim * 32, lse, 0.0f);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) ticket = __hip_atomic_fetch_add(a.counters + unit_id, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (ticket != uint32_t(a.splits) - 1) return;
        if (tid == 0) __hip_atomic_store(a.counters + unit_id, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (r >= n_rows) return;
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int d = 0; d < kOut; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[d][i] = 0.0f;
        bool nan = false;
        for (int k = 0; k < a.splits; k++) {
            const float *from = parts + int64_t(k) * kPart;
            const float x = load_pair(from + Dim * 32 - 64 * half).x, m_new = fmaxf(m, x), was = m == m_new ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            const float f = x == -INFINITY ? 0.0f : x == m_new ? 1.0f : __builtin_amdgcn_exp2f(x - m_new);
            nan |= x != x;
            m = m_new;
            l = l * was + f;
#pragma unroll
            for (int d = 0; d < kOut; d++)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float2 z = load_pair(from + (8 * d + i / 2) * 128);
                    o[d][i] = __builtin_fmaf(z.x, f, o[d][i] * was);
                    o[d][i + 1] = __builtin_fmaf(z.y, f, o[d][i + 1] * was);
                }
        }
        if (nan) l = NAN;
        const bool empty = m == -INFINITY && !nan;
        lse = empty ? -INFINITY : m + __builtin_log2f(l);
#pragma unroll
        for (int d = 0; d < kOut; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[d][i] = empty ? 0.0f : o[d][i] / l;
    }
    if (r >= n_rows) return;
    T *dst = static_cast<T *>(a.out.data) + int64_t(row.first + token) * a.out.token + int64_t(q_head) * a.out.head + 16 * half;
#pragma unroll
    for (int d = 0; d < kOut; d++) {
        V8 x, y;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            x[i] = T(o[d][i]);
            y[i] = T(o[d][8 + i]);
        }
        if (a.wide_out) {
            *reinterpret_cast<V8 *>(dst + 32 * d) = x;
            *reinterpret_cast<V8 *>(dst + 32 * d + 8) = y;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                dst[32 * d + i] = x[i];
                dst[32 * d + 8 + i] = y[i];
            }
        }
    }
    if (half == 0 && a.lse) a.lse[int64_t(row.first + token) * a.q_heads + q_head] = lse * kLn2;
}

template <typename T, int Dim> static void launch_dim(const AttendArgs &a, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: k_prompt<T, Dim, 16><<<blocks, kThreads, 0, s>>>(a); break;
    case 32: k_prompt<T, Dim, 32><<<blocks, kThreads, 0, s>>>(a); break;
    default: k_prompt<T, Dim, 64><<<blocks, kThreads, 0, s>>>(a); break;
    }
}

void launch_prompt(const AttendArgs &a, int32_t type, hipStream_t s) {
    const int64_t items = int64_t(a.units) * a.splits * a.c.heads;
    const unsigned blocks = unsigned((items + kDies - 1) / kDies * kDies) + 1;
    if (type == ESP_KV_BF16) a.c.dim == 64 ? launch_dim<__bf16, 64>(a, blocks, s) : launch_dim<__bf16, 128>(a, blocks, s);
    else a.c.dim == 64 ? launch_dim<_Float16, 64>(a, blocks, s) : launch_dim<_Float16, 128>(a, blocks, s);
}

}  // namespace esp_kv
