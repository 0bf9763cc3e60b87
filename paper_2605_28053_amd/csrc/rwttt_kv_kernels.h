// Internal launch interface between the host side of the paged cache
// (rwttt_kv_api.cpp) and its kernels (rwttt_kv.hip).  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "rwttt_kv_rows.h"

namespace rwttt {

// Shape of a handle's cache.
struct KvShape {
  int n_owners, n_pages, page_shift, max_pages, kv_heads, group, head_dim;
  int io_bf16, cache;      // cache: RWTTT_F32, RWTTT_BF16, RWTTT_FP8 or RWTTT_FP4
};

struct KvExtendLaunch {
  KvShape s;
  const int32_t *have, *want, *pos;
  int32_t *table, *ring, *new_pos, *lengths, *start, *slots, *owners, *positions, *result;
  uint32_t cap;
};

struct KvAppendLaunch {
  KvShape s;
  const void *k_new, *v_new;
  uint64_t k_stride, v_stride;
  void *k, *v;
  int8_t* bounds;                           // or null
  const float *k_scale, *v_scale, *step;    // of the layer; scales may be null
  const int32_t* slots;
  uint32_t n;
};

struct KvGatherLaunch {
  KvShape s;
  const void *k, *v;                        // of the layer
  const float *k_scale, *v_scale;           // of the layer, may be null
  const int32_t *table, *owners, *positions, *lengths;
  uint32_t n;
  void *k_out, *v_out;                      // one of them may be null
  uint64_t k_stride, v_stride;
};

// One side of a rotation: the rows of `heads` heads of n tokens, and where they go.
struct KvTurnRows {
  const void* in;
  void* out;
  uint64_t in_stride, out_stride;
  int heads;                                // 0: no such side
};

struct KvRotateLaunch {
  int io_bf16, head_dim, turning, interleaved, inverse;
  float gain;
  const uint64_t* turns;
  const int32_t* positions;
  uint32_t n;
  KvTurnRows q, k;
};

struct KvSelectLaunch {
  KvShape s;
  const void* q;
  uint64_t q_stride;
  const int8_t* bounds;
  const int32_t *table, *lengths, *rows;
  uint32_t n, first, last, keep;
  int32_t* pages;
  void* workspace;                          // or null
};

struct KvAttendLaunch {
  KvShape s;
  const void *q, *k, *v;
  const float *k_scale, *v_scale;
  uint64_t q_stride, out_stride;
  const int32_t *table, *lengths, *rows, *pages;
  uint32_t n, n_layers, window, keep;
  float scale;
  void* out;
  float* lse;
  void* workspace;
};

size_t kv_workspace_bytes(const KvShape& shape);
hipError_t launch_kv_extend(const KvExtendLaunch& L, hipStream_t stream);
hipError_t launch_kv_append(const KvAppendLaunch& L, hipStream_t stream);
hipError_t launch_kv_gather(const KvGatherLaunch& L, hipStream_t stream);
hipError_t launch_kv_rotate(const KvRotateLaunch& L, hipStream_t stream);
hipError_t launch_kv_select(const KvSelectLaunch& L, hipStream_t stream);
hipError_t launch_kv_attend(const KvAttendLaunch& L, hipStream_t stream);

}  // namespace rwttt
