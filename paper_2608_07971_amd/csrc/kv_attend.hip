// Attention over the paged 8-bit cache.
#include "kv_attend.hpp"

namespace esp_kv {

// The work of one head is a list of tiles: units (16 rows of queries of one
// sequence and key head) one after another, every unit of a row with as many
// tiles as the row's longest (one where there is none, so that empty rows are
// written too).  The list is cut evenly over the workgroups, which all run at
// once: ragged batches and single long sequences fill the GPU alike, and a
// workgroup has at most two units that it shares with others.
//
// 64 rows of the list at a time, worked out by the first wavefront.
struct Window {
    Row row[64];
    int units[64], tiles[64], end[64];      // end: tiles of the list up to and with this row
};

__device__ __forceinline__ int units_of(const AttendArgs &a, const Row &r) { return (r.n * a.group + kCols - 1) / kCols; }
__device__ __forceinline__ int tiles_of(const AttendArgs &a, const Row &r) { return max(1, span_of(r.length - r.n, r.length - 1, a.window).size()); }

// All threads: the rows from b0 on, `before` tiles before them.
__device__ __forceinline__ void load_window(const AttendArgs &a, int b0, int before, Window &w) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        const Row r = usable_row(a, b0 + lane);
        const int units = units_of(a, r), tiles = tiles_of(a, r);
        int end = units * tiles;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int v = __shfl_up(end, m);
            end += lane >= m ? v : 0;
        }
        w.row[lane] = r;
        w.units[lane] = units;
        w.tiles[lane] = tiles;
        w.end[lane] = before + end;
    }
    __syncthreads();
}

// Maximum and sum over the four lanes that hold one column's tokens.
__device__ __forceinline__ float across_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ int across_max(int x) {
    auto r = __builtin_amdgcn_permlane16_swap(uint32_t(x), uint32_t(x), false, false);
    x = max(int(r[0]), int(r[1]));
    r = __builtin_amdgcn_permlane32_swap(uint32_t(x), uint32_t(x), false, false);
    return max(int(r[0]), int(r[1]));
}
__device__ __forceinline__ float across_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ float4v product(half8 x, half8 y, float4v z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ float4v product(bhalf8 x, bhalf8 y, float4v z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }

// Workgroups of one compute unit, by what the registers hold.
template <int Dim> constexpr int kPerUnit = Dim == 64 ? 3 : 2;

template <bool Stream> __device__ __forceinline__ uint4v fetch(const uint8_t *p) {
    const uint4v *q = reinterpret_cast<const uint4v *>(p);
    return Stream ? __builtin_nontemporal_load(q) : *q;
}

// A wavefront takes 64 tokens of a unit at a time.  Scores and output are held
// transposed (rows tokens or output values, columns queries), so a query's
// statistics lie in the lanes that hold its column, and the weights are in
// place for the value product as the score product leaves them: matrix row
// 4 g + i of score tile j is token 16 g + 4 j + i.  No data passes through LDS
// until the wavefronts join.
// Bound by reading the pages: 256 sequences of up to 8,192 tokens, 8 key heads of
// 128, 1.35 GB in 255 us (5.3 TB/s); 4 of up to 131,001, 1.04 GB in 176 us (5.9 TB/s);
// one of 777 tokens 11 us, a chain of reads: rows twice, table, page, parts.
template <typename T, int Dim, int Page, bool Stream> __global__ __launch_bounds__(kThreads, kPerUnit<Dim>) void k_attend(AttendArgs a) {
    typedef typename Pack<T>::v8 V8;
    typedef typename Pack<T>::v2 V2;
    constexpr int kSteps = Dim / 32;        // matrix steps of a score
    constexpr int kTiles = Dim / 16;        // matrix tiles of an output
    constexpr int kPad = Dim + 4;
    __shared__ __align__(16) float so[kWaves][kCols][kPad];
    __shared__ float sm[kWaves][kCols], sl[kWaves][kCols];
    __shared__ int se[kWaves];
    __shared__ uint32_t ticket;
    __shared__ Window win;

    const Cache &c = a.c;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
    const int turn = blockIdx.x / kDies, head = turn % c.heads, me = turn / c.heads * kDies + blockIdx.x % kDies;
    const int k_group = col >> 2;

    const uint32_t page_step = uint32_t(c.layers * c.heads) * (Page * Dim);
    const int64_t block_at = int64_t(a.layer * c.heads + head) * (Page * Dim);
    const uint8_t *keys = c.k + block_at, *vals = c.v + block_at;
    const float *scales = c.scale + 2 * a.layer * c.heads + head;

    // this workgroup's share [at, stop) of the list
    int64_t total = 0, tokens = 0;
    int units = 0;
    for (int b = lane; b < a.rows.rows; b += 64) {
        const Row r = usable_row(a, b);
        total += int64_t(units_of(a, r)) * tiles_of(a, r);
        tokens += r.n;
        units += units_of(a, r);
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        total += __shfl_xor(total, m);
        tokens += __shfl_xor(tokens, m);
        units += __shfl_xor(units, m);
    }
    if (tokens > a.rows.tokens || total > INT32_MAX) {          // rows that overlap, or a list that cannot be numbered
        if (threadIdx.x == 0) record(c, ESP_ERR_SHAPE);
        return;
    }
    // a tile for every wavefront, unless the units are shorter: a unit each is quicker than several in turn
    const int all = __builtin_amdgcn_readfirstlane(int(total)), each = max(1, __builtin_amdgcn_readfirstlane(units));
    const int per = max(min(kWaves, (all + each - 1) / each), (all + a.groups - 1) / a.groups);
    if (int64_t(me) * per >= all) return;
    int at = me * per;
    const int stop = min(all, at + per);
    int b0 = 0;
    load_window(a, 0, 0, win);
    while (at < stop) {
        // the row that holds list place `at`
        uint64_t past = __ballot(win.end[lane] > at);
        while (!past) {
            b0 += 64;
            if (b0 >= a.rows.rows) break;
            load_window(a, b0, win.end[63], win);
            past = __ballot(win.end[lane] > at);
        }
        if (!past) break;                   // lengths that change during the call
        const int in = __builtin_ctzll(past);
        auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
        const Row row{same(win.row[in].first), same(win.row[in].n), same(win.row[in].seq), same(win.row[in].length)};
        const int tiles = same(win.tiles[in]), row_at = same(win.end[in]) - same(win.units[in]) * tiles;
        const int unit = (at - row_at) / tiles, unit_at = row_at + unit * tiles, skip = at - unit_at;
        const int count = min(tiles - skip, stop - at);
        const int first_part = unit_at / per, parts = (unit_at + tiles - 1) / per - first_part + 1;
        at += count;

        // this lane's query: row r of the sequence is (token r / group, query head r % group)
        const int n_rows = row.n * a.group, r0 = unit * kCols, r = r0 + col, p0 = row.length - row.n;
        const int token = r / a.group, q_head = head * a.group + r - token * a.group;
        const int pos = r < n_rows ? p0 + token : -1, low = a.window > 0 ? pos - a.window : -1;
        const int pos_first = p0 + r0 / a.group, pos_last = p0 + (min(r0 + kCols, n_rows) - 1) / a.group;
        Span span = span_of(pos_first, pos_last, a.window);
        span.from += skip;
        span.to = min(span.to, span.from + count);

        // matrix step 2 s + k of a score takes elements 64 s + 16 quad + 8 k + (0..7)
        V8 q[kSteps];
        {
            const T *src = static_cast<const T *>(a.q.data) + int64_t(row.first + token) * a.q.token + int64_t(q_head) * a.q.head + 16 * quad;
#pragma unroll
            for (int s = 0; s < kSteps; s++) {
                V8 x{};
                if (r < n_rows) {
                    const T *from = src + 64 * (s >> 1) + 8 * (s & 1);
                    if (a.wide) x = *reinterpret_cast<const V8 *>(from);
                    else
#pragma unroll
                        for (int j = 0; j < 8; j++) x[j] = from[j];
                }
                q[s] = x;
            }
        }

        float4v o[kTiles];                  // row 16 d + 4 quad + i of out^T, divided by 2^o_exp
#pragma unroll
        for (int d = 0; d < kTiles; d++) o[d] = float4v{0, 0, 0, 0};
        float m_run = -INFINITY, l_run = 0.0f;   // largest score (log 2); sum of the weights of this lane's tokens
        int o_exp = kNoScale, o_top = kNoScale;      // o_top: the largest so far

        // What a wavefront holds of a tile.  Keys: this lane reads 16 bytes of rows of
        // page_k's tokens; values: 16 tokens of page_v at 16 dimensions.
        const int32_t *table = c.table + int64_t(row.seq) * c.width;
        int page_k = -1, page_v = -1;
        uint4v kw[4][Dim / 64], vw[kTiles];
        float k_scale = 0.0f, v_scale = 0.0f;
        bool ok = false;
        auto pages_of = [&](int t) {
            const int at_k = t * kTile + 16 * k_group, at_v = t * kTile + 16 * quad;
            page_k = at_k < row.length ? table[at_k / Page] : -1;
            page_v = at_v < row.length ? table[at_v / Page] : -1;
        };
        auto load_keys = [&](int t) {
            const int at_k = t * kTile + 16 * k_group;
            const bool k_ok = uint32_t(page_k) < uint32_t(c.pages);
            ok = uint32_t(page_v) < uint32_t(c.pages);
            const uint8_t *kp = keys + uint64_t(k_ok ? page_k : 0) * page_step + ((at_k % Page + (col & 3)) * Dim + quad * 16);
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int s = 0; s < Dim / 64; s++) kw[j][s] = fetch<Stream>(kp + (4 * j * Dim + 64 * s));
            const float *sp = scales + uint64_t(ok ? page_v : 0) * uint32_t(2 * c.layers * c.heads);
            k_scale = sp[0];
            v_scale = sp[c.heads];
            if (!__all(k_ok))               // past the end, or a page that is not there: zeros
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int s = 0; s < Dim / 64; s++) kw[j][s] = k_ok ? kw[j][s] : uint4v{0, 0, 0, 0};
        };
        auto load_values = [&](int t) {
            const int at_v = t * kTile + 16 * quad;
            const bool v_ok = uint32_t(page_v) < uint32_t(c.pages);
            const uint8_t *vp = vals + uint64_t(v_ok ? page_v : 0) * page_step + (col * Page + at_v % Page);
#pragma unroll
            for (int d = 0; d < kTiles; d++) vw[d] = fetch<Stream>(vp + d * 16 * Page);
            if (!__all(v_ok)) {
                if (!v_ok && at_v < row.length && col == 0) record(c, ESP_ERR_SHAPE);
#pragma unroll
                for (int d = 0; d < kTiles; d++) vw[d] = v_ok ? vw[d] : uint4v{0, 0, 0, 0};
            }
        };
        auto scores = [&](float4v (&s)[4]) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                s[j] = float4v{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < kSteps; k++) {
                    const uint4v w = kw[j][k >> 1];
                    s[j] = product(codes8<V8, V2>(w[2 * (k & 1)], w[2 * (k & 1) + 1]), q[k], s[j]);
                }
            }
        };
        // The running maximum takes the tile's scores in; the output follows.
        auto raise = [&](const float4v (&s)[4]) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) top = fmaxf(top, s[j][i]);
            top = across_max(top);
            if (__any(top > m_run + kSlack)) {
                const float m = fmaxf(m_run, top), by = m_run == m ? 1.0f : __builtin_amdgcn_exp2f(m_run - m);
                m_run = m;
                l_run *= by;
#pragma unroll
                for (int d = 0; d < kTiles; d++) o[d] *= by;
            }
        };
        // Weights times values, of which this lane's 16 tokens have a scale of exponent e:
        // in one go, unless the tile's blocks are too far apart.  A scale of 0 is near any.
        auto values = [&](const half8 (&w)[2], int e) {
            auto largest = [&] { return __builtin_amdgcn_readfirstlane(across_max(e)); };
            for (int most = largest(); most > kNoScale; most = largest()) {
                o_top = max(o_top, most);
                if (most > o_exp || most < o_exp - kNear) {
                    const int to = max(most, o_top - kDown);
                    const float by = ldexpf(1.0f, max(o_exp - to, -200));
#pragma unroll
                    for (int d = 0; d < kTiles; d++) o[d] *= by;
                    o_exp = to;
                }
                const bool near = e >= min(o_exp - kNear, most);
                const half8 u[2] = {near ? w[0] : half8{}, near ? w[1] : half8{}};
                const float by = power(e - o_exp);
#pragma unroll
                for (int d = 0; d < kTiles; d++)
#pragma unroll
                    for (int k = 0; k < 2; k++) o[d] = product(scaled8(vw[d][2 * k], vw[d][2 * k + 1], by), u[k], o[d]);
                e = near ? kNoScale : e;
            }
        };

        // Tiles that every row sees whole.  Pages are read two steps ahead, keys and
        // values one: the next keys are asked for as soon as the scores have used the
        // present ones, the next values after the value product, so that a wavefront
        // has a tile in flight nearly always.
        const int in_window = a.window > 0 ? max(0, pos_last - a.window + kTile) / kTile : 0;
        const int whole_from = max(span.from, in_window), whole_to = max(whole_from, min(span.to, (pos_first + 1) / kTile));
        int t = whole_from + wave;
        if (t < whole_to) {
            pages_of(t);
            load_keys(t);
            load_values(t);
            if (t + kWaves < whole_to) pages_of(t + kWaves);
        }
        for (; t < whole_to; t += kWaves) {
            float4v s[4];
            scores(s);
            const float ks = ok ? k_scale * a.scale : 0.0f, vs = v_scale, none = ok ? 0.0f : -INFINITY;
            const bool held_page = ok, more = t + kWaves < whole_to;
            if (more) load_keys(t + kWaves);
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) s[j][i] = __builtin_fmaf(s[j][i], ks, none);
            raise(s);
            const int e = exponent(vs);
            const float base = m_run == -INFINITY ? 0.0f : m_run - kLift, v_rest = held_page ? ldexpf(vs, -e) : 0.0f;
            half8 w[2];
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float x = __builtin_amdgcn_exp2f(s[j][i] - base);
                    l_run += x;
                    w[j >> 1][4 * (j & 1) + i] = _Float16(x * v_rest);
                }
            values(w, !held_page ? kNoScale : vs != 0.0f ? e : max(o_exp, -126));
            if (more) {
                load_values(t + kWaves);
                if (t + 2 * kWaves < whole_to) pages_of(t + 2 * kWaves);
            }
        }

        // The others: at the window's start and at the end.
        const int head_tiles = min(whole_from, span.to) - span.from, rest = head_tiles + max(0, span.to - whole_to);
        for (int x = wave; x < rest; x += kWaves) {
            const int t = x < head_tiles ? span.from + x : whole_to + x - head_tiles, at_v = t * kTile + 16 * quad;
            pages_of(t);
            load_keys(t);
            load_values(t);
            float4v s[4];
            scores(s);
            const float ks = k_scale * a.scale;
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int tt = at_v + 4 * j + i;
                    s[j][i] = tt <= pos && tt > low && ok ? s[j][i] * ks : -INFINITY;
                }
            raise(s);
            const int e = exponent(v_scale);
            const float base = m_run == -INFINITY ? 0.0f : m_run - kLift, v_rest = ldexpf(v_scale, -e);
            half8 w[2], seen[2];
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const bool hidden = s[j][i] == -INFINITY;
                    const float x = __builtin_amdgcn_exp2f(s[j][i] - base);
                    l_run += x;
                    w[j >> 1][4 * (j & 1) + i] = hidden ? _Float16(0.0f) : _Float16(x * v_rest);    // 0 * an infinite scale
                    seen[j >> 1][4 * (j & 1) + i] = hidden ? _Float16(0.0f) : _Float16(1.0f);
                }
            // tokens past the end hold anything: their codes become 0.  A NaN that
            // only some rows see must not reach the others through 0 * NaN.
            const int held = max(0, min(16, row.length - at_v));
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
                        const uint32_t y = nan_bytes(vw[d][2 * k]), z = nan_bytes(vw[d][2 * k + 1]);
                        hit = product(codes8<half8, half2>(y & 0x38383838u, z & 0x38383838u), seen[k], hit);
                        vw[d][2 * k] &= ~y;
                        vw[d][2 * k + 1] &= ~z;
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (hit[i] > 0.0f) o[d][i] = NAN;
                }
            }
            values(w, !ok ? kNoScale : v_scale != 0.0f ? e : max(o_exp, -126));
        }

        // join the wavefronts
        l_run = across_sum(l_run);
        __syncthreads();                    // the unit before has been read
#pragma unroll
        for (int d = 0; d < kTiles; d++) *reinterpret_cast<float4v *>(&so[wave][col][16 * d + 4 * quad]) = o[d];
        if (quad == 0) {
            sm[wave][col] = m_run;
            sl[wave][col] = l_run;
        }
        if (lane == 0) se[wave] = o_exp;
        __syncthreads();
        constexpr int kMine = Dim / 16;     // values of a row a thread finishes
        const int n = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kMine, rn = r0 + n;
        float m = -INFINITY, l = 0.0f, y[kMine];
        int e = kNoScale;
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            m = fmaxf(m, sm[w][n]);
            e = max(e, se[w]);
        }
#pragma unroll
        for (int i = 0; i < kMine; i++) y[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            const float f = sm[w][n] == m ? 1.0f : __builtin_amdgcn_exp2f(sm[w][n] - m), g = f * ldexpf(1.0f, max(se[w] - e, -200));
            l = __builtin_fmaf(sl[w][n], f, l);
#pragma unroll
            for (int i = 0; i < kMine; i++) y[i] = __builtin_fmaf(so[w][n][d0 + i], g, y[i]);
        }
        const bool none = m == -INFINITY && !(l != l);
        float lse = none ? -INFINITY : m - kLift + __builtin_log2f(l);
#pragma unroll
        for (int i = 0; i < kMine; i++) y[i] = none ? 0.0f : ldexpf(y[i] / l, e);

        if (parts > 1) {
            // Every part is left in the place of its workgroup (2 w + 1 for a unit that
            // begins there, 2 w for one that goes on); the last to arrive joins them in
            // order.  Parts and tickets go by agent-scope atomics, which pass the dies'
            // own caches: each thread's stores have been performed (vmcnt 0) before the
            // ticket is drawn.  Fences in their place write the whole cache back and
            // took 110 of 300 us at 512 workgroups.
            constexpr int kPart = kCols * (Dim + 2), kBatch = 8;
            const int64_t step = int64_t(c.heads) * 2 * kPart;
            float *base = a.partial + int64_t(head) * 2 * kPart, *mine = base + me * step + (me == first_part ? kPart : 0);
            if (rn < n_rows) {
#pragma unroll
                for (int i = 0; i < kMine; i += 2) store_pair(mine + n * Dim + d0 + i, y[i], y[i + 1]);
                if (d0 == 0) store_pair(mine + kCols * Dim + 2 * n, lse, 0.0f);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            uint32_t *counter = a.counters + int64_t(first_part) * c.heads + head;
            if (threadIdx.x == 0) ticket = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (ticket != uint32_t(parts) - 1) continue;
            if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            m = -INFINITY;
            l = 0.0f;
#pragma unroll
            for (int i = 0; i < kMine; i++) y[i] = 0.0f;
            if (rn < n_rows) {
                bool nan = false;
                for (int k0 = 0; k0 < parts; k0 += kBatch) {    // so many loads in flight at a time
                    float x[kBatch];
                    float2 z[kBatch][kMine / 2];
#pragma unroll
                    for (int k = 0; k < kBatch; k++) {
                        const int part = min(k0 + k, parts - 1);
                        const float *from = base + (first_part + part) * step + (part ? 0 : kPart);
                        x[k] = load_pair(from + kCols * Dim + 2 * n).x;
#pragma unroll
                        for (int i = 0; i < kMine / 2; i++) z[k][i] = load_pair(from + n * Dim + d0 + 2 * i);
                    }
                    float top = m;
#pragma unroll
                    for (int k = 0; k < kBatch; k++) {
                        nan |= x[k] != x[k];
                        top = fmaxf(top, x[k]);
                    }
                    const float by = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);
                    m = top;
                    l *= by;
#pragma unroll
                    for (int i = 0; i < kMine; i++) y[i] *= by;
#pragma unroll
                    for (int k = 0; k < kBatch; k++) {
                        const float f = k0 + k >= parts || x[k] == -INFINITY ? 0.0f : x[k] == m ? 1.0f : __builtin_amdgcn_exp2f(x[k] - m);
                        l += f;
#pragma unroll
                        for (int i = 0; i < kMine / 2; i++) {
                            y[2 * i] = __builtin_fmaf(z[k][i].x, f, y[2 * i]);
                            y[2 * i + 1] = __builtin_fmaf(z[k][i].y, f, y[2 * i + 1]);
                        }
                    }
                }
                if (nan) l = NAN;
            }
            const bool empty = m == -INFINITY && !(l != l);
            lse = empty ? -INFINITY : m + __builtin_log2f(l);
#pragma unroll
            for (int i = 0; i < kMine; i++) y[i] = empty ? 0.0f : y[i] / l;
        }
        if (rn < n_rows) {
            const int tok = row.first + rn / a.group, qh = head * a.group + rn % a.group;
            T *dst = static_cast<T *>(a.out.data) + int64_t(tok) * a.out.token + int64_t(qh) * a.out.head + d0;
            if (a.wide_out) {
                typedef T Out __attribute__((ext_vector_type(kMine)));
                Out z;
#pragma unroll
                for (int i = 0; i < kMine; i++) z[i] = T(y[i]);
                *reinterpret_cast<Out *>(dst) = z;
            } else {
#pragma unroll
                for (int i = 0; i < kMine; i++) dst[i] = T(y[i]);
            }
            if (d0 == 0 && a.lse) a.lse[int64_t(tok) * a.q_heads + qh] = lse * kLn2;
        }
    }
    if (at < stop && threadIdx.x == 0) record(c, ESP_ERR_SHAPE);
}

}  // namespace esp_kv

using namespace esp_kv;

namespace {

constexpr int kComputeUnits = 256;
// k_prompt from kManyRows rows of a sequence and key head on, if there are kManyUnits units.
// Measured on 8 key heads with 4 query heads each (k_prompt / k_attend), us:
//                                        heads of 128      heads of 64
//   8 sequences of 8,192 tokens, 64 rows    83 /  97          60 /  50
//                                96 rows    99 / 138          71 /  52
//                               128 rows   102 / 166          71 /  91
//   64 of 2,048,                 48 rows   164 / 130          82 /  66
//                                96 rows   171 / 251          84 / 123
//   1 of 16,384,     256 rows (24 units)    86 /  61          45 /  40
//                  1,200 rows (80 units)   132 / 352          90 / 174
constexpr int kManyRows = 96, kManyUnits = 64;

struct Shape {
    bool prompt;
    int32_t groups;                          // k_attend: workgroups of one head
    bool stream;                             // k_attend: keys and values read past the caches
    int32_t units, splits;                   // k_prompt: units of one head at most, parts of each
    size_t counters, bytes;
};
esp_status shape_of(const esp_kv_cache *c, int32_t rows, int64_t tokens, int32_t q_heads, int32_t max_new, int32_t max_length, Shape &s) {
    if (rows < 0 || tokens < 0 || tokens > INT32_MAX || max_new < 0 || max_length < 0) return ESP_ERR_SHAPE;
    if (q_heads < 1 || q_heads > 65536 || q_heads % c->kv_heads) return ESP_ERR_SHAPE;
    const int64_t group = q_heads / c->kv_heads;
    if (int64_t(max_new) * group > INT32_MAX / 2) return ESP_ERR_SHAPE;
    s = Shape{};
    // Counters, all that has to be zero at first, lie in front, as many for every call on caches of this many heads, so that
    // calls of other shapes leave them alone: k_attend takes groups * heads, k_prompt
    // units * heads of at most half its 512 places.
    s.counters = ((size_t(kComputeUnits) * 3 + c->kv_heads) * 4 + 255) / 256 * 256;
    s.bytes = s.counters;
    const int64_t units = rows ? tokens * group / kPromptRows + rows : 0;
    s.prompt = tokens * group >= int64_t(rows) * kManyRows && units * c->kv_heads >= kManyUnits;
    if (s.prompt) {
        const int64_t places = 2 * kComputeUnits;
        // a workgroup each (one part: they are many), one more and some to fill up; a launch's threads are numbered in 32 bits
        if (units * c->kv_heads > (int64_t(1) << 32) / kThreads - 2 * kDies) return ESP_ERR_SHAPE;
        // too few units for the GPU: their tiles are shared out, eight at least to a part
        int64_t splits = places / (units * c->kv_heads);
        if (splits > max_length / (8 * kTile)) splits = max_length / (8 * kTile);
        s.units = int32_t(units);
        s.splits = int32_t(splits > 1 ? splits : 1);
        if (s.splits > 1) s.bytes += size_t(units) * c->kv_heads * s.splits * kPromptRows * (c->head_dim + 2) * 4;
        return ESP_OK;
    }
    const int slots = kComputeUnits * (c->head_dim == 64 ? kPerUnit<64> : kPerUnit<128>);
    s.groups = slots / c->kv_heads > 1 ? slots / c->kv_heads : 1;
    // Read once (one unit a row), and more than the memory-side cache holds twice over: loads
    // that leave no trace, 195 -> 177 us for 1.04 GB; 46 -> 51 us for 268 MB read again and again.
    // By the caller's bounds, for want of others: where these are loose it goes wrong by 3 to 8%
    // (256 sequences of 300 tokens under a bound of 32,768: 48 -> 52 us; 256 of 4,096 with no
    // bound on new tokens: 352 -> 368 us).
    s.stream = int64_t(max_new) * group <= kCols && 2 * int64_t(rows) * max_length * c->kv_heads * c->head_dim > (int64_t(512) << 20);
    // no more than one for every four tiles of the longest rows, or for every unit
    const int64_t few = int64_t(rows) * ((int64_t(max_new) * group + kCols - 1) / kCols), tiles = few * (max_length / kTile + 2);
    const int64_t most = tiles / kWaves + 1 > few ? tiles / kWaves + 1 : few;
    if (most < s.groups) s.groups = int32_t(most);
    s.bytes += size_t(s.groups) * c->kv_heads * 2 * kCols * (c->head_dim + 2) * 4;
    return ESP_OK;
}

}  // namespace

namespace {

template <typename T, int Dim, bool Stream> void launch_dim(const AttendArgs &a, unsigned blocks, hipStream_t s) {
    switch (a.c.tokens) {
    case 16: k_attend<T, Dim, 16, Stream><<<blocks, kThreads, 0, s>>>(a); break;
    case 32: k_attend<T, Dim, 32, Stream><<<blocks, kThreads, 0, s>>>(a); break;
    default: k_attend<T, Dim, 64, Stream><<<blocks, kThreads, 0, s>>>(a); break;
    }
}
template <typename T> void launch(const AttendArgs &a, bool stream, unsigned blocks, hipStream_t s) {
    if (stream) a.c.dim == 64 ? launch_dim<T, 64, true>(a, blocks, s) : launch_dim<T, 128, true>(a, blocks, s);
    else a.c.dim == 64 ? launch_dim<T, 64, false>(a, blocks, s) : launch_dim<T, 128, false>(a, blocks, s);
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
    const bool wide_out = (reinterpret_cast<uintptr_t>(out.data) & 15) == 0 && out.token_stride % 8 == 0 && out.head_stride % 8 == 0;
    const AttendArgs a{cache_of(cache), Rows{offsets, seqs, rows, tokens}, View{q.data, q.token_stride, q.head_stride},
                       View{out.data, out.token_stride, out.head_stride}, lse, scale * kLog2e, layer, q_heads, q_heads / cache->kv_heads,
                       window, max_new, max_length, s.groups, wide, wide_out, s.units, s.splits, static_cast<uint32_t *>(workspace),
                       reinterpret_cast<float *>(static_cast<char *>(workspace) + s.counters)};
    const hipStream_t h = static_cast<hipStream_t>(stream);
    if (s.prompt) {
        launch_prompt(a, type, h);
        return launched();
    }
    const unsigned blocks = unsigned((s.groups + kDies - 1) / kDies * kDies) * unsigned(cache->kv_heads);
    if (type == ESP_KV_BF16) launch<__bf16>(a, s.stream, blocks, h);
    else launch<_Float16>(a, s.stream, blocks, h);
    return launched();
}
