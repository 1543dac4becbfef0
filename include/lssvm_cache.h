/*
 * lssvm_cache.h - C ABI of the operators over a paged key/value cache.
 *
 * A decision function of this library is a sum over stored points,
 * f(x) = sum_i alpha_i k(x_i, x). Attention is the sum of that kind whose kernel
 * is exp(scale <q, k_j>), normalised over the points a row sees, and whose
 * coefficients are vectors v_j; its points arrive token by token. The operators
 * here keep such points and answer from them: lssvm_rotary turns keys and queries
 * by their positions, lssvm_cache_append writes new tokens into the cache,
 * lssvm_attention evaluates rows over it, lssvm_cache_evict keeps the heaviest.
 *
 * Conventions: those of lssvm.h (device pointers unless marked "host", caller-owned
 * memory, argument checks on the host before any GPU work, lssvm_last_error()),
 * except that every call only enqueues its work on `stream` and returns; nothing is
 * read back and nothing allocated, so calls can be captured into a HIP graph.
 * `stream` belongs to the current device, the one that holds every array.
 *
 * What stands in device memory (page numbers, lengths, offsets) the host does not
 * see. The kernels bound it instead: a length counts at most columns * page keys, a
 * negative one none; offsets count as if cut to [0, tokens]; a page number outside
 * [0, pages) is a hole, whose keys no row sees and which is never written.
 *
 * Rows (tokens x heads) of one call are at most 2^30, their values at most 2^33.
 *
 * dtype (of k, v, x, q and out) is LSSVM_F32, LSSVM_BF16 or LSSVM_F16. Sums, softmax
 * statistics, weights and rotation factors are fp32, angles fp64. Scales are finite in
 * fp32. In 16-bit types attention's probabilities are rounded to the type where tiles of
 * many rows multiply them with the values (half a step each, of fp16 down to 2^-50 of the
 * largest), and enter in two parts where rows are few.
 */
#ifndef LSSVM_CACHE_H_
#define LSSVM_CACHE_H_

#include "lssvm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of these operators besides LSSVM_F32. */
enum { LSSVM_BF16 = 2, LSSVM_F16 = 3 };

/* A paged cache (host struct of device pointers). Key j of sequence s, head h, is
 *     k + p * k_stride[0] + h * k_stride[1] + (j % page) * k_stride[2],
 *     p = table[s * table_stride + j / page],
 * dim contiguous values, with strides in elements; v and weight alike (a weight is
 * one float per key, its slots contiguous). Strides are free as long as no two rows
 * overlap and rows of k and v begin on 16 bytes, so heads may stand before or behind
 * the slots of a page; slots are at most 2^24 values apart. */
typedef struct lssvm_cache {
    void* k;
    void* v;
    float* weight;           /* accumulated weight of every key, or NULL          */
    const int32_t* table;    /* sequences x columns page numbers                  */
    int32_t* lengths;        /* keys of each sequence                             */
    int64_t pages;           /* pages of the pool, 1 .. 2^31 - 1                  */
    int64_t heads;           /* key/value heads, 1 .. 65535                       */
    int64_t page;            /* keys per page, >= 1                               */
    int64_t dim;             /* values per key and head, a multiple of 8, 8 .. 256 */
    int64_t sequences;       /* 1 .. 65535; sequences * heads <= 2^22             */
    int64_t columns;         /* columns of table, >= 1; columns * page <= 2^29    */
    int64_t k_stride[3];     /* page, head, slot                                  */
    int64_t v_stride[3];     /* page, head, slot                                  */
    int64_t weight_stride[2]; /* page, head                                       */
    int64_t table_stride;    /* between rows of table, >= columns                 */
    int32_t dtype;           /* of k and v                                        */
} lssvm_cache;

/* How rotary frequencies are stretched for contexts longer than the trained one. */
enum {
    LSSVM_ROPE_PLAIN = 0,  /* f_i = base^(-i / pairs)                                      */
    LSSVM_ROPE_LINEAR = 1, /* f_i / factor: positions interpolated                         */
    LSSVM_ROPE_NTK = 2,    /* base * factor^(pairs / (pairs - 1)): the slowest pair is
                              stretched by factor, the fastest not at all                  */
    LSSVM_ROPE_YARN = 3    /* by parts: pairs of 32 turns or more over `original` positions
                              as they are, of 1 or fewer divided by factor, between them
                              mixed linearly in their turns (not in their index, as some
                              models do: those bring frequencies of their own); values
                              times 0.1 ln(factor) + 1                                     */
};

/* Writes the `pairs` frequencies (host, fp64) of rotary positions and the factor of
 * the rotated values. pairs >= 1, base > 0 and factor >= 1 finite, original > 0
 * (used by LSSVM_ROPE_YARN only). */
int lssvm_rotary_frequencies(int64_t pairs, double base, int32_t scaling, double factor,
                             double original, double* freqs, double* scale);

/*
 * Rotary positions: pair i of every head of token t is turned by the angle
 * positions[t] * freqs[i] (fp64) and multiplied by scale,
 *     (y0, y1) = scale * (x0 cos - x1 sin, x1 cos + x0 sin).
 *
 * x, out       device, tokens x heads x dim values of dtype; strides of token and
 *              head in elements (host, 2 each), the dim values contiguous. out may be
 *              x itself with the same strides, else no rows of theirs may overlap
 *              (nor, of other strides, all that lies between their first and last).
 * positions    device, tokens integers of position_bytes (4 or 8) bytes; any sign and
 *              size (from 2^53 on as the nearest double). An infinite angle gives NaN.
 * freqs        device, pairs doubles, 0 <= 2 * pairs <= dim. The first 2 * pairs values
 *              of a head are turned; the others are copied.
 * interleaved  nonzero: pair i is (2i, 2i + 1), else (i, i + pairs).
 * transpose    nonzero: the angle is negated, which is the transposed map, so that
 *              the call takes the gradient with respect to y to that of x.
 */
int lssvm_rotary(const void* x, const int64_t* x_stride, void* out, const int64_t* out_stride,
                 int64_t tokens, int64_t heads, int64_t dim, const void* positions,
                 int32_t position_bytes, const double* freqs, int64_t pairs, double scale,
                 int32_t interleaved, int32_t transpose, int32_t dtype, void* stream);

/*
 * Writes new tokens into the cache. Sequence s gets the tokens offsets[s] ..
 * offsets[s + 1] - 1 as its last keys: lengths[s] already counts them. Keys are
 * turned as by lssvm_rotary on the way, values copied, weights set to zero. Tokens
 * outside the offsets, or that no key of the sequence stands for, are left out;
 * what the call does not write stays as it was.
 *
 * k, v       device, tokens x heads x dim values of the cache's dtype, strides as in
 *            lssvm_rotary.
 * offsets    device, sequences + 1 int32 values, not falling.
 * positions  as in lssvm_rotary, of the new tokens; NULL with pairs = 0.
 * freqs, pairs, scale, interleaved  as in lssvm_rotary; pairs = 0 copies the keys.
 */
int lssvm_cache_append(const lssvm_cache* cache, const void* k, const int64_t* k_stride,
                       const void* v, const int64_t* v_stride, int64_t tokens,
                       const int32_t* offsets, const void* positions, int32_t position_bytes,
                       const double* freqs, int64_t pairs, double scale, int32_t interleaved,
                       void* stream);

/* Device workspace of lssvm_attention for `tokens` rows of `heads` heads; 0 if an
 * argument is out of range. With accumulate and few rows (tokens x group up to 32 per
 * sequence) it holds 4 bytes per row and key of columns * page: a table no wider than
 * its sequences need takes less. */
size_t lssvm_attention_workspace_bytes(const lssvm_cache* cache, int64_t tokens, int64_t heads,
                                       int32_t accumulate);

/*
 * Attention of new tokens over the cache. Row i of the n = offsets[s + 1] - offsets[s]
 * rows of sequence s, length L = lengths[s], sees the keys j < L, with causal only
 * those j <= L - n + i (the rows are the last n tokens of the sequence). Query head h
 * reads key/value head h / (heads / cache heads):
 *     p_j = exp(scale <q, k_j>) / sum over the seen j of the same,  out = sum_j p_j v_j.
 * A row that sees no key gets zeros, one that sees only keys of score minus infinity
 * NaNs. A value that is not finite reaches the rows that see its key and no others: as
 * itself, or as a NaN under a score of minus infinity. Rows outside the offsets are left
 * as they were.
 * With accumulate, each key's weight grows by the p_j of all rows and heads of its
 * group, always summed in one order.
 *
 * q, out      device, tokens x heads x dim values of the cache's dtype, strides of
 *             token and head (host, 2 each); they must not overlap, as in lssvm_rotary.
 * heads       query heads, a multiple of the cache's heads, at most 65535.
 * offsets     as in lssvm_cache_append.
 * weight_out  where weight + gain goes, for the keys j < L of every sequence and
 *             nothing else: an array of its own with strides of page and head
 *             (host, 2), or NULL: into cache->weight. No two sequences may share a
 *             page when weights are accumulated.
 * workspace   device, 256-byte aligned, lssvm_attention_workspace_bytes().
 */
int lssvm_attention(const lssvm_cache* cache, const void* q, const int64_t* q_stride,
                    int64_t tokens, int64_t heads, const int32_t* offsets, double scale,
                    int32_t causal, int32_t accumulate, float* weight_out,
                    const int64_t* weight_out_stride, void* out, const int64_t* out_stride,
                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eviction by accumulated weight: of every sequence and head, the keys that stay are
 * the last `recent` and the heaviest of the others, n = min(length, budget) in all
 * (the last n if recent >= n). Of equal weights the lowest index stays; a NaN counts
 * as the lightest. They are copied in their order, with values and weights, to the
 * keys 0 .. n - 1 of the target, whose length becomes n.
 *
 * from, to  caches with weights and the same heads, page, dim, dtype and sequences.
 *           They may share a pool, but to's pages must not be pages of from, and
 *           `to` needs columns * page >= budget.
 * budget    >= 1; recent >= 0.
 * kept      device, sequences x heads x budget int32, contiguous: the kept indices in
 *           rising order, then -1.
 */
int lssvm_cache_evict(const lssvm_cache* from, const lssvm_cache* to, int64_t budget,
                      int64_t recent, int32_t* kept, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LSSVM_CACHE_H_ */
