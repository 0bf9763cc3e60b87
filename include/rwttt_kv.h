/*
 * rwttt_kv.h -- C ABI of the owners' paged key-value cache, for AMD Instinct
 * MI355X (gfx950): block tables and slot maps from the owners' lengths, new
 * rows stored with key bounds per page, page selection by those bounds, and
 * the attention of one new token per owner.
 *
 * A decode step of an In-Place TTT model attends to each owner's keys and
 * values before the fast-weight MLP whose state rwttt.h serves.  Rows live in
 * pages of page_rows rows; an owner's table row lists its pages in order, so
 * row j of owner r is row j % page_rows of page table[r][j / page_rows].  Free
 * pages wait in a ring.  A step of the cache is:
 *
 *     rwttt_kv_extend     once: lengths -> pages, table, slots of the new rows
 *     per layer:
 *       rwttt_kv_append   new keys and values through the slots
 *       rwttt_kv_select   (long contexts) the pages each query attends to
 *       rwttt_kv_attend   softmax(scale q K^T) V over all, recent or selected rows
 *
 * Lengths, tables and slots stay on the device: no call synchronises, copies
 * to the host or depends on a host value that a step changes, so a step can be
 * captured in a graph.  rwttt_kv_extend writes the new lengths beside the old
 * ones: a step that fails rolls back by keeping the old lengths and ring
 * position, as a WRITE's candidate does (rwttt.h).
 *
 * Conventions, beside those of rwttt.h (status codes, validation before any
 * launch, device pointers 16-byte aligned, nothing allocated or synchronised):
 *  - All tables and index arrays are int32 device arrays, dense row-major.
 *  - q, out and lse are owner-indexed.  `rows` lists the n owners that a call
 *    computes (a device array), or is NULL for all of them, with n = n_owners;
 *    an id outside [0, n_owners) is skipped, and the rows of owners that are
 *    not listed are not touched.
 *  - Strides count elements between consecutive owners' (or tokens') rows; a
 *    row itself is dense.  A row's bytes and the stride's must be multiples
 *    of 16.
 *  - Out-of-range lengths, pages and slots on the device never lead to an
 *    access outside the caller's buffers: lengths are clamped to
 *    [0, max_pages * page_rows], page ids to [0, n_pages), and such slots are
 *    skipped.  What such rows compute is not specified.
 *  - A handle is read-only for its calls except for its workspace: attends,
 *    and selects, that may overlap in time need a handle (and workspace) each.
 */
#ifndef RWTTT_KV_H
#define RWTTT_KV_H

#include "rwttt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* cache element type beside RWTTT_F32 and RWTTT_BF16: OCP e4m3 */
#define RWTTT_FP8  2

#define RWTTT_KV_MAX_OWNERS   4096
#define RWTTT_KV_MAX_ROWS     (1u << 23)   /* largest max_pages * page_rows              */
#define RWTTT_KV_MAX_SELECT   32768        /* largest max_pages that rwttt_kv_select takes */

typedef struct rwttt_kv rwttt_kv;

typedef struct rwttt_kv_config {
    uint32_t n_owners;       /* 1..RWTTT_KV_MAX_OWNERS                            */
    uint32_t n_layers;
    uint32_t n_pages;        /* pages of each layer's cache; n_pages * page_rows < 2^31 */
    uint32_t page_rows;      /* 16, 32, 64, 128 or 256                            */
    uint32_t max_pages;      /* pages an owner may hold: width of the table       */
    uint32_t n_heads;        /* query heads, a multiple of n_kv_heads             */
    uint32_t n_kv_heads;     /* 1..512; n_heads / n_kv_heads <= 128               */
    uint32_t head_dim;       /* 64, 128 or 256                                    */
    int32_t  io_dtype;       /* RWTTT_F32 / RWTTT_BF16: q, new keys and values, out */
    int32_t  cache_dtype;    /* RWTTT_BF16 / RWTTT_FP8, or RWTTT_F32 for fp32 io  */
    uint32_t reserved;       /* must be 0                                         */
    /* Device buffers; each may be NULL when no call of the handle needs it. */
    int32_t* table;          /* [n_owners, max_pages] page ids                    */
    int32_t* ring;           /* [n_pages] free pages, a ring                      */
    void* const* k;          /* host array of n_layers pointers to                */
    void* const* v;          /*   [n_pages, n_kv_heads, page_rows, head_dim]      */
    void* const* bounds;     /* host array of n_layers pointers to int8
                                [n_pages, n_kv_heads, 2, head_dim]: per page and
                                channel, the least and the largest key           */
    const float* k_scale;    /* [n_layers, n_kv_heads]: an 8-bit key times its    */
    const float* v_scale;    /*   head's scale is its value; RWTTT_FP8 only, NULL: 1 */
    const float* bound_step; /* [n_layers, n_kv_heads]: unit of the bounds; needed
                                with bounds.  Scales and steps are positive and
                                normal numbers, and so are their reciprocals      */
    void* workspace;         /* rwttt_kv_workspace_bytes() bytes, 256-byte aligned,
                                all zero when the handle is created (each call
                                leaves its counters zero); rwttt_kv_attend needs
                                it, rwttt_kv_select is faster with it             */
    size_t workspace_bytes;
} rwttt_kv_config;

/* Bytes of device workspace of a handle: counters, partial results of the
 * attention's splits (the head layout fixes their number), and the page scores
 * of at most 256 (owner, kv head) pairs.  Only the shape fields are read. */
rwttt_status rwttt_kv_workspace_bytes(const rwttt_kv_config* cfg, size_t* bytes);

/* Create a handle: copies the pointers, makes no HIP call.  RWTTT_E_INVALID
 * for a bad shape, type or pointer, RWTTT_E_CAPACITY for a small workspace.
 * *out is set only on success; release with rwttt_kv_destroy. */
rwttt_status rwttt_kv_create(const rwttt_kv_config* cfg, rwttt_kv** out);
rwttt_status rwttt_kv_destroy(rwttt_kv* kv);

/* Pages and slots for a step: owner r goes from have[r] rows to want[r].
 * Growing owners take pages from the ring's front, in owner order; shrinking
 * ones (a finished request: want 0; rows taken back: want < have) return the
 * pages behind ceil(want / page_rows), in owner and page order, to its back.
 *   have, want   [n_owners]
 *   pos          {front, count} of the ring before the call
 *   new_pos      the same after it
 *   lengths      [n_owners]: want, or have if the step does not fit
 *   start        [n_owners + 1]: exclusive sums of max(0, want - have)
 *   slots, owners, positions   [cap]: of the new rows, in owner and position
 *                order, the row of the cache (page * page_rows + row), the owner
 *                and its position; -1 behind the last one
 *   result       {status, new rows, pages taken, pages returned}
 * Nothing fits in part: with too few pages or a too small cap the status is
 * RWTTT_E_CAPACITY; with a length or ring position out of range, or more pages
 * returned than the ring has places beside those it holds, it is
 * RWTTT_E_INVALID; then table and ring stay as they are, lengths is have,
 * new_pos is pos, start and the counts are 0 and the maps -1.
 * Pages returned in a call can be taken by the next one.  Table entries behind
 * an owner's last page are not cleared.  The inputs stay as they are, so that
 * a call may be repeated; new_pos and lengths must not alias them.
 * Errors of the call itself: RWTTT_E_INVALID for null or misaligned pointers,
 * arrays that overlap (the table and the ring among them; the inputs may be one
 * another), or a handle without table or ring.  One launch. */
rwttt_status rwttt_kv_extend(rwttt_kv* kv, const int32_t* have, const int32_t* want,
                             const int32_t* pos, int32_t* new_pos, int32_t* lengths, int32_t* start,
                             int32_t* slots, int32_t* owners, int32_t* positions, uint32_t cap,
                             int32_t* result, void* stream);

/* Store n tokens' keys and values (k, v: [n, n_kv_heads, head_dim], io type,
 * rows k_stride and v_stride elements apart) in their slots of layer's cache;
 * a slot outside the cache (the -1 of a padded token) is skipped.  Rounded once
 * to the cache type, to nearest even; to RWTTT_FP8 after a product with
 * 1 / scale and a clamp to +-448.
 * With bounds, the pages' key bounds follow: in units of the head's step, the
 * floor of the least and the ceiling of the largest stored key of each
 * channel, the key times 1 / step in fp32, clamped to +-127.  So a stored key is
 * inside its page's bounds times the step, up to 2^-22 of itself (the product's
 * rounding), if it is within 127 steps; beyond, the bound is 127 steps and does
 * not hold it.  A page whose row 0 is stored forgets its old bounds.  Rows taken
 * back leave bounds wider than they need be, never narrower.  A NaN key leaves
 * its channel's bounds as they are.
 * The tokens of one page must be consecutive in the call (as rwttt_kv_extend
 * lists them), with no skipped slot between them; otherwise which of their
 * bounds remain is not specified.
 * n = 0 launches nothing.  One launch. */
rwttt_status rwttt_kv_append(rwttt_kv* kv, uint32_t layer, const void* k, uint64_t k_stride,
                             const void* v, uint64_t v_stride, const int32_t* slots, uint32_t n,
                             void* stream);

/* The pages that each listed owner's query attends to, for each kv head: the
 * owner's `first` first and `last` last pages, and of the others those with
 * the largest scores, `keep` in all (keep >= first + last, keep >= 1); all of
 * them when it has no more than keep.  pages: [n_owners, n_kv_heads, keep],
 * positions in the owner's table row, ascending, -1 behind the last.
 * The score is what the bounds can add to the logits of the head's (rounded)
 * queries together: no less than the page's keys add, as far as the bounds hold
 * them (see rwttt_kv_append).  With a the largest magnitude in the group's queries and
 * q8 = rint(q * ((1 / a) * 127)), each step rounded to fp32 (0 for a = 0, or so
 * small, below 3.8e-37, that (1 / a) * 127 overflows),
 *     score = sum over the group's queries and channels of max(q8 lo, q8 hi):
 * whole numbers, so that the choice is exact; ties go to the lowest page.
 * Queries that are not finite select some pages, not specified which.
 * Errors: RWTTT_E_INVALID as above or without bounds or table;
 * RWTTT_E_CAPACITY for max_pages above RWTTT_KV_MAX_SELECT. */
rwttt_status rwttt_kv_select(rwttt_kv* kv, uint32_t layer, const void* q, uint64_t q_stride,
                             const int32_t* lengths, const int32_t* rows, uint32_t n, uint32_t first,
                             uint32_t last, uint32_t keep, int32_t* pages, void* stream);

/* Attention of one new token: for each listed owner r and query head i of kv
 * head h,
 *     out[r, i] = sum_j p_j v[j, h],  p = softmax over j of scale * (q[r, i] . k[j, h])
 *     lse[r, i] = log sum_j exp(scale * (q[r, i] . k[j, h]))      (unless lse is NULL)
 * over the owner's rows j < lengths[r]: all of them; with window > 0 the last
 * `window`; with pages (keep per kv head, as rwttt_kv_select writes them) those
 * of the listed pages, and then window must be 0.  Of a list only the first
 * min(keep, pages held) entries are read, and -1 or a page that is not held is
 * passed over.  The new token's own row is among the rows once it is appended
 * and counted.  An owner without rows, a head whose list names none and one
 * all of whose scores are -inf get out = 0 and lse = -inf.  A score of +inf or
 * NaN makes the head's out and lse NaN.  What the pages hold behind an owner's
 * rows, NaN included, has no influence.
 * Products, maxima and sums are held in fp32, out is rounded once.  How a
 * row's sum is split depends on all listed lengths, so its last bits may
 * differ between calls with other lengths; equal calls give equal bits.
 * Errors: RWTTT_E_INVALID as above, or without k, v, table or workspace. */
rwttt_status rwttt_kv_attend(rwttt_kv* kv, uint32_t layer, const void* q, uint64_t q_stride,
                             const int32_t* lengths, const int32_t* rows, uint32_t n, float scale,
                             uint32_t window, const int32_t* pages, uint32_t keep, void* out,
                             uint64_t out_stride, float* lse, void* stream);

/* hipError_t of the last RWTTT_E_HIP returned by this handle (0 if none). */
int32_t rwttt_kv_last_hip_error(const rwttt_kv* kv);

#ifdef __cplusplus
}
#endif

#endif /* RWTTT_KV_H */
