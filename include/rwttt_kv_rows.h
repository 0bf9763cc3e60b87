/*
 * rwttt_kv_rows.h -- C ABI of the operators on rows of the owners' paged cache
 * (rwttt_kv.h), for AMD Instinct MI355X (gfx950): rotary positions of new queries
 * and keys before they are stored, and stored rows read back.
 *
 * The conventions are those of rwttt_kv.h: status codes, validation before any launch,
 * device pointers 16-byte aligned, rows of heads that are dense, strides between
 * rows in elements of the io type and multiples of 16 bytes, nothing allocated or
 * synchronised, every call safe to capture in a graph.  These calls use no
 * workspace, so they may overlap with any others that do not write what they read.
 */
#ifndef RWTTT_KV_ROWS_H
#define RWTTT_KV_ROWS_H

#include "rwttt_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rotary positions.  `turning` channels of each head turn in pairs, pair i at
 * position p by the angle p w_i:
 *     a' = gain (a cos - b sin),   b' = gain (b cos + a sin)
 * with (a, b) channels i and i + turning / 2 (RWTTT_ROTARY_HALF) or 2 i and 2 i + 1
 * (RWTTT_ROTARY_INTERLEAVED); the head's other channels stay as they are.
 * Frequencies are kept in turns: turns[i] is w_i / 2 pi in units of 2^-64, so that
 * the angle of any position is a 64-bit product that wraps at whole turns, off by p times
 * what turns[i] is off by: half a unit in a table of nearest numbers, and in that of
 * rwttt_kv_turns at most 1 + 24 w_i / 2 pi units (below 5 where w_i is at most 1). */
#define RWTTT_ROTARY_HALF        0
#define RWTTT_ROTARY_INTERLEAVED 1

typedef struct rwttt_kv_rotary {
    uint32_t turning;        /* even, 2..head_dim                                 */
    int32_t  layout;         /* RWTTT_ROTARY_HALF / RWTTT_ROTARY_INTERLEAVED      */
    float    gain;           /* finite; 1 where the context is not stretched      */
    int32_t  inverse;        /* 1: the transposed map, by -p w_i (the gradient of the
                                inputs from that of the outputs), else 0          */
    const uint64_t* turns;   /* device array [turning / 2]                        */
} rwttt_kv_rotary;

/* Frequencies w_i = base^(-2 i / turning), for contexts stretched by `factor`:
 *   RWTTT_ROTARY_PLAIN   as they are (factor is not read)
 *   RWTTT_ROTARY_LINEAR  w_i / factor
 *   RWTTT_ROTARY_BASE    of the base times factor^(turning / (turning - 2)), which
 *                        leaves the fastest pair and slows the slowest by the factor
 *   RWTTT_ROTARY_PARTS   slow pairs only: with t = context w_i / 2 pi the turns over the
 *                        context before it was stretched and r = (t - low) / (high - low)
 *                        kept in [0, 1], w_i (r + (1 - r) / factor)
 * Writes turns[turning / 2] (host memory), to be copied to the device.  Host only.
 * Any other table of frequencies may be used as well.
 * RWTTT_E_INVALID: turning 0, odd or above 256, base not above 1, a number that
 * is not finite, a factor not above 0 (unless PLAIN), turning 2 with BASE, context not
 * above 0 or high not above low with PARTS. */
#define RWTTT_ROTARY_PLAIN  0
#define RWTTT_ROTARY_LINEAR 1
#define RWTTT_ROTARY_BASE   2
#define RWTTT_ROTARY_PARTS  3

rwttt_status rwttt_kv_turns(uint32_t turning, double base, int32_t scaling, double factor, double low,
                            double high, double context, uint64_t* turns);

/* Turn n tokens' queries (q: [n, n_heads, head_dim]) and keys (k: [n, n_kv_heads,
 * head_dim]; io type, rows the strides apart) to positions[n] (device array): into
 * q_out and k_out, which may be q and k themselves with the same stride.  A token
 * of negative position (the -1 of a padded one) is skipped: its rows of the
 * outputs are left as they were.  q with q_out, or k with k_out, may be NULL.
 * Angles' sines and cosines and the products are fp32, the results rounded once; an
 * infinite channel makes its pair what the two products and their sum are.
 * Needs no buffer of the handle but its shape; n = 0 launches nothing.  One launch.
 * Errors: RWTTT_E_INVALID for a bad rotary, null or misaligned pointers, a bad
 * stride, an output that overlaps an input (positions and turns among them) or the other
 * output other than as said (rows of different strides count as overlapping where the spans
 * of all n meet). */
rwttt_status rwttt_kv_rotate(rwttt_kv* kv, const rwttt_kv_rotary* rotary, const int32_t* positions, uint32_t n,
                             const void* q, uint64_t q_stride, void* q_out, uint64_t q_out_stride,
                             const void* k, uint64_t k_stride, void* k_out, uint64_t k_out_stride, void* stream);

/* Read n stored rows back: row i of k and of v ([n, n_kv_heads, head_dim], io type,
 * rows k_stride and v_stride elements apart) is position positions[i] of owner
 * owners[i] ([n] each, as rwttt_kv_extend lists them), rounded once to the io type
 * (exact but for RWTTT_FP8 with scales).  A pair whose owner is
 * outside [0, n_owners) or whose position is outside [0, lengths[owner]) is
 * skipped: its rows of k and v are left as they were.  k or v may be NULL.
 * n = 0 launches nothing.  One launch.
 * Errors: RWTTT_E_INVALID as above, for outputs that overlap each other or what the call
 * may read (the arrays, the table, the layer's pages and scales), or without k, v or table
 * in the handle. */
rwttt_status rwttt_kv_gather(rwttt_kv* kv, uint32_t layer, const int32_t* owners, const int32_t* positions,
                             const int32_t* lengths, uint32_t n, void* k, uint64_t k_stride, void* v,
                             uint64_t v_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RWTTT_KV_ROWS_H */
