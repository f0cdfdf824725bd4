/*
 * esp_kv.h -- C-ABI of the paged 8-bit key/value cache of the MI355X (gfx950)
 * Elastic Shadow Pricing library (same library file as esp.h).
 *
 * The price loop gives an offline-inference job a configuration: a number of
 * sequences and a number of bytes of GPU memory for its cache.  The calls
 * below are that cache: pages that grow, shrink, fork and move to a smaller
 * budget (resize, fork, compact), writing new tokens with rotary positions in
 * 8 bits (append), and attention over what is held (attend).
 *
 * Layout.  A page holds page_tokens tokens of every layer and key/value head.
 * The pool is page-major, so a pool whose last pages are empty can be cut:
 *   k      [pages][layers][kv_heads][page_tokens][head_dim]   e4m3 (OCP), 1 byte
 *   v      [pages][layers][kv_heads][head_dim][page_tokens]   e4m3, token innermost
 *   scale  [pages][layers][2: k, v][kv_heads]                 float32 >= 0, value = code * scale
 *   table  [sequences][table_width]  page of tokens [i*page_tokens, (i+1)*page_tokens), -1 none
 *   lengths[sequences]               tokens held
 *   refs   [pages]                   table entries that name the page; 0 = free
 * A page that is the partly filled last page of a sequence has one owner:
 * fork and resize copy it rather than share it, so append never writes a
 * page that another sequence reads.
 *
 * Conventions are those of esp.h: a status is returned, nothing throws or
 * aborts, `stream` is a hipStream_t, calls only enqueue work and can be
 * captured in a graph (esp_kv_device_status alone waits).  All pointers are
 * device memory unless marked host.  Every index that the GPU reads from
 * device memory (lengths, offsets, table, sequence numbers) is checked there
 * before it is used; what is found wrong is left out and recorded in
 * *cache->status (the first code is kept until esp_kv_device_status takes it).
 */
#ifndef ESP_KV_H
#define ESP_KV_H

#include "esp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of queries, keys, values and outputs. */
enum { ESP_KV_BF16 = 0, ESP_KV_FP16 = 1, ESP_KV_FP32 = 2 };

typedef struct {
    int32_t pages, layers, kv_heads, page_tokens, head_dim;   /* page_tokens 16, 32 or 64; head_dim 64 or 128 */
    int32_t sequences, table_width;
    void *k, *v;                     /* 16-byte aligned */
    float *scale;
    int32_t *table, *lengths, *refs;
    int32_t *status;                 /* one word, 0 = fine */
} esp_kv_cache;

/* Scaling of rotary positions for contexts beyond the trained one. */
enum {
    ESP_KV_ROPE_NONE = 0,
    ESP_KV_ROPE_LINEAR = 1,          /* every frequency / factor */
    ESP_KV_ROPE_NTK = 2,             /* base * factor^(rot / (rot - 2)): the slowest pair slows by factor, the fastest by nothing */
    ESP_KV_ROPE_PARTS = 3            /* pairs of fewer than 1 turn over `context` slow by factor, of more than 32 by
                                        nothing, linearly between; vectors scaled by 0.1 ln(factor) + 1 */
};

/* A rotation: pair i turns by turns[i] * position revolutions. */
typedef struct {
    const double *turns;             /* [rotary_dim / 2] revolutions per position */
    float magnitude;
    int32_t rotary_dim;              /* even, <= head_dim; the rest of the head passes through */
    int32_t interleaved;             /* pairs (2i, 2i+1), else (i, i + rotary_dim/2) */
} esp_kv_rope;

/* A tensor [tokens][heads][head_dim], the last dimension contiguous; strides in elements. */
typedef struct {
    void *data;
    int64_t token_stride, head_stride;
} esp_kv_view;

/* Host only: turns (host, [rotary_dim/2]) and *magnitude (host) from the base frequency and the scaling. */
esp_status esp_kv_rope_turns(int32_t rotary_dim, double base, int32_t scaling, double factor, int32_t context,
                             double *turns, float *magnitude);

/*
 * out = x with every pair (a, b) of a head turned by the token's position:
 * magnitude * (a cos - b sin, a sin + b cos); inverse != 0 turns the other
 * way, which is the gradient.  positions int32 [tokens], any sign.  out may be
 * x itself (same strides); otherwise the two must not overlap.
 */
esp_status esp_kv_rotate(const esp_kv_rope *rope, int32_t type, int64_t tokens, int32_t heads, int32_t head_dim,
                         esp_kv_view x, const int32_t *positions, int32_t inverse, esp_kv_view out, void *stream);

/*
 * Writes new tokens into the cache.  Row b has the tokens
 * [offsets[b], offsets[b+1]) of k and v (type bf16 or fp16), which are the
 * last ones of sequence seqs[b] (NULL: b): its length has already grown
 * (esp_kv_resize).  Rows name distinct sequences.  Keys are turned by rope
 * (NULL: not; rotary_dim a multiple of 16) at their positions in the sequence.
 * Per page, head and of keys and values apart: e is the least exponent from -100
 * to 100 with max|x| <= 448 * 2^e over the finite new values, the block's scale
 * 2^e, or the old scale where that is larger and the page has older tokens (their
 * codes are divided by the growth, a power of two, so they change only where they
 * leave e4m3's normal range).  Values are rounded to the nearest code once, from
 * float32; infinities, and what lies beyond 448 * 2^100, take the largest code,
 * NaN stays NaN.  q (q_heads > 0): turned the same way into
 * q_out in the same launch; both 16-byte aligned, with strides that keep it so.
 */
esp_status esp_kv_append(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                         const int32_t *offsets, const int32_t *seqs, esp_kv_view k, esp_kv_view v,
                         const esp_kv_rope *rope, int32_t q_heads, esp_kv_view q, esp_kv_view q_out, void *stream);

/*
 * Reads tokens back: row b's tokens [starts[b], starts[b] + offsets[b+1] -
 * offsets[b]) of sequence seqs[b] as numbers, into k_out and v_out
 * [tokens][kv_heads][head_dim], contiguous, type bf16 or fp16.  Tokens past a
 * sequence's end read as 0; a row with a negative start is left out.
 */
esp_status esp_kv_gather(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                         const int32_t *offsets, const int32_t *seqs, const int32_t *starts, void *k_out, void *v_out,
                         void *stream);

/*
 * Attention of q [tokens][q_heads][head_dim] (bf16 or fp16; q_heads a multiple
 * of kv_heads, query head h reads key head h / (q_heads / kv_heads)) over the
 * cache.  Token i of row b's n is at position p = length - n + i of sequence
 * seqs[b] and sees the cached tokens t <= p, with window > 0 those with
 * t > p - window only.
 *   out = sum_t softmax_t(scale * q . k_t) v_t,   lse = ln sum_t exp(scale * q . k_t)
 * A token that sees nothing gets out = 0, lse = -inf.  lse: float32
 * [tokens][q_heads] contiguous, or NULL.  Every sum and statistic is float32;
 * the softmax weights enter the value product rounded to fp16: 2^-11 of each,
 * and those below 2^-34 of the largest vanish.  Values enter it exactly if their
 * block's scale is a power of two, as append's are, whatever other blocks'
 * scales (down to 2^-80 of the largest, then less exactly); with another scale
 * they may be rounded to fp16 first.
 * max_new >= every row's n and max_length >= every length are bounds the
 * caller knows.  They choose the launch and how it reads; loose ones have cost
 * up to a tenth of a call.  A row over either bound is not computed and recorded
 * as ESP_ERR_SHAPE; tokens of no row, or of one that is left out, keep what out
 * and lse held.
 * workspace: at least esp_kv_attend_workspace bytes, 256-byte aligned, the first
 * 4 * (768 + kv_heads) of them zeroed once before its first use and left ready
 * for the next call, of any shape, on a cache of as many kv_heads; calls that
 * may run at the same time need one each, so a graph that may be replayed beside
 * other work needs its own.  Lengths, offsets and sequence numbers must not
 * change while a call that was given them runs: the outputs are then undefined,
 * and the workspace is to be zeroed again before it serves another call.
 */
esp_status esp_kv_attend_workspace(const esp_kv_cache *cache, int32_t rows, int64_t tokens, int32_t q_heads,
                                   int32_t max_new, int32_t max_length, size_t *bytes);
esp_status esp_kv_attend(const esp_kv_cache *cache, int32_t layer, int32_t type, int32_t rows, int64_t tokens,
                         const int32_t *offsets, const int32_t *seqs, int32_t q_heads, esp_kv_view q, float scale,
                         int32_t window, int32_t max_new, int32_t max_length, esp_kv_view out, float *lse,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Bytes that resize, fork (of n children; as many for any n up to sequences) and compact need; 256-byte aligned, contents free. */
esp_status esp_kv_pages_workspace(const esp_kv_cache *cache, int32_t n, size_t *bytes);

/*
 * Sets every sequence's length (int32 [sequences]; 0 frees it).  Pages past
 * the new end lose an owner; new pages are the free ones of lowest index, in
 * order of sequence and slot.  A kept page that is partly filled and still
 * shared is replaced by a copy.  With too few free pages (ESP_ERR_RANGE) or a
 * length outside [0, table_width * page_tokens] (ESP_ERR_SHAPE) nothing changes.
 */
esp_status esp_kv_resize(const esp_kv_cache *cache, const int32_t *lengths, void *workspace, size_t workspace_bytes,
                         void *stream);

/*
 * Sequence children[i] drops its pages and takes parents[i]'s: full pages are
 * shared, a partly filled last page is copied to the lowest free page, in
 * order of i.  Children are distinct and no parent is a child
 * (ESP_ERR_INVALID_ARG); with too few free pages (ESP_ERR_RANGE) nothing changes.
 */
esp_status esp_kv_fork(const esp_kv_cache *cache, int32_t n, const int32_t *parents, const int32_t *children,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Empties the pages from `limit` on (limit < 0: from the number of live pages
 * on): the i-th live page there is copied to the i-th free page below.  The
 * cache's table and refs stay as they are and name the old places, whose bytes
 * are intact, so readers may go on; table_out and refs_out name the new ones
 * (they may be cache->table and cache->refs).  *live (or NULL): live pages.
 * With more live pages than limit (ESP_ERR_RANGE) nothing moves, and
 * table_out and refs_out repeat the old.
 */
esp_status esp_kv_compact(const esp_kv_cache *cache, int32_t limit, int32_t *table_out, int32_t *refs_out,
                          int32_t *live, void *workspace, size_t workspace_bytes, void *stream);

/* Waits for the stream, returns the recorded code (an esp_status) and clears it. */
esp_status esp_kv_device_status(const esp_kv_cache *cache, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ESP_KV_H */
