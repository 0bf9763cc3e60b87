// Kernels of the owners' paged key-value cache (include/rwttt_kv.h) for
// gfx950: block tables and slot maps, stored rows with key bounds per page,
// page selection, and one new token's attention.

#include "rwttt_kv_kernels.h"
#include "rwttt_kv_rules.h"

#include <type_traits>

namespace rwttt {
namespace {

#include "rwttt_device.h"

typedef const __attribute__((address_space(4))) int32_t* scalar_i32;   // read through the scalar cache

__device__ __forceinline__ scalar_i32 scalar(const int32_t* p) {
  return reinterpret_cast<scalar_i32>(reinterpret_cast<uintptr_t>(p));
}

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// x of another lane by a data-parallel move (no LDS); lanes without a source add 0.
template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, ROWS, 0xf, false));
}
constexpr int kDppXor1 = 0xb1, kDppXor2 = 0x4e, kDppHalfMirror = 0x141, kDppMirror = 0x140;

// Inclusive sum over a wave's lanes: within the rows of 16, then row 0 to 1 and 2
// to 3, then the lower half to the upper.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += dpp<0x111>(x);
  x += dpp<0x112>(x);
  x += dpp<0x114>(x);
  x += dpp<0x118>(x);
  x += dpp<0x142, 0xa>(x);
  x += dpp<0x143, 0xc>(x);
  return x;
}

// Results that another XCD's block reads in the same launch.  Device-scope
// stores and loads go past the XCDs' separate L2s word by word; a fence instead
// would write back and invalidate a whole L2 under the blocks that still stream
// (122 against 30 us for eight owners of 4200 rows).
__device__ __forceinline__ void share(float* p, float a, float b) {
  const uint64_t w = uint64_t(__float_as_uint(b)) << 32 | __float_as_uint(a);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 shared_pair(const float* p) {
  const uint64_t w = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float(uint32_t(w)), __uint_as_float(uint32_t(w >> 32)));
}
// Counts this block; true for the one that finds `others` counted, which leaves the
// counter zero for the next call -- past the L2 too, whose line holds other counters.
__device__ __forceinline__ uint32_t count_in(uint32_t* count, uint32_t others) {
  const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (before == others) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return before == others;
}
// The thread's shared stores have reached the memory that all XCDs see.
__device__ __forceinline__ void shared_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ---------------------------------------------------------------------------
// extend: lengths -> pages, table, slots
// ---------------------------------------------------------------------------
//
// The three prefix sums over the owners (pages taken, pages returned, new rows)
// fix every output, so each block computes them itself -- 8 bytes an owner, from
// the L2 -- and then fills its part of the flattened lists by a binary search:
// one launch, no block waits for another.  Bound by latency: 3.8 us for eight
// owners, 7.4 for 500 with 34000 new rows, 10.0 for 4000.

constexpr int kExtThreads = 256;
constexpr int kExtItems = 512;           // list entries a block fills

// Last owner whose exclusive sum is <= i (owners without entries are passed over).
__device__ __forceinline__ int owner_of(const int* sums, int n, int i) {
  int lo = 0, hi = n;                    // sums[lo] <= i < sums[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int TURNS>
__global__ void __launch_bounds__(kExtThreads) kv_extend_kernel(const KvExtendLaunch p) {
  extern __shared__ int ext_lds[];
  const int n = p.s.n_owners, shift = p.s.page_shift, P = 1 << shift;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int* take = ext_lds;
  int* give = take + n + 1;
  int* add = give + n + 1;
  __shared__ uint32_t wave_sum[kExtThreads / 64][4];
  __shared__ int any_bad;
  if (tid == 0) any_bad = 0;
  __syncthreads();

  // four owners a thread and turn, their lengths kept for the second pass
  const int limit = p.s.max_pages << shift;
  const int turns = (n + 4 * kExtThreads - 1) / (4 * kExtThreads), i0 = tid * 4 * turns;
  int have[TURNS * 4], want[TURNS * 4];
#pragma unroll
  for (int k = 0; k < TURNS; ++k) {
    const int at = i0 + 4 * k;
    const bool on = k < turns;
    if (on && at + 4 <= n) {
      const int4 h = *reinterpret_cast<const int4*>(p.have + at), w = *reinterpret_cast<const int4*>(p.want + at);
      have[4 * k] = h.x, have[4 * k + 1] = h.y, have[4 * k + 2] = h.z, have[4 * k + 3] = h.w;
      want[4 * k] = w.x, want[4 * k + 1] = w.y, want[4 * k + 2] = w.z, want[4 * k + 3] = w.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool there = on && at + j < n;
        have[4 * k + j] = there ? p.have[at + j] : 0;
        want[4 * k + j] = there ? p.want[at + j] : 0;
      }
    }
  }
  const int front = p.pos[0], count = p.pos[1], pages = p.s.n_pages;
  uint32_t t = 0, g = 0, a = 0;          // of a thread: 16 owners of 2^23 rows at most
  int bad = 0;
#pragma unroll
  for (int k = 0; k < TURNS * 4; ++k) {
    bad |= have[k] < 0 || want[k] < 0 || have[k] > limit || want[k] > limit;
    const int h = clampi(have[k], 0, limit), w = clampi(want[k], 0, limit);
    const int ph = (h + P - 1) >> shift, pw = (w + P - 1) >> shift;
    t += max(0, pw - ph);
    g += max(0, ph - pw);
    a += max(0, w - h);
  }
  // Exclusive sums over the threads.  4096 owners have 2^31 pages at most; their new
  // rows pass 32 bits, so the low 16 bits and the rest are summed apart.
  const uint32_t st = wave_scan(t), sg = wave_scan(g), lo = wave_scan(a & 0xffffu), hi = wave_scan(a >> 16);
  if (lane == 63) {
    wave_sum[wave][0] = st;
    wave_sum[wave][1] = sg;
    wave_sum[wave][2] = lo;
    wave_sum[wave][3] = hi;
  }
  if (bad) any_bad = 1;
  __syncthreads();
  long long bt = st - t, bg = sg - g, ba = (long long)lo + ((long long)hi << 16) - a, taken = 0, given = 0, added = 0;
#pragma unroll
  for (int w = 0; w < kExtThreads / 64; ++w) {
    const long long x = wave_sum[w][0], y = wave_sum[w][1], z = wave_sum[w][2] + ((long long)wave_sum[w][3] << 16);
    if (w < wave) {
      bt += x;
      bg += y;
      ba += z;
    }
    taken += x;
    given += y;
    added += z;
  }
  const ExtendVerdict verdict = extend_verdict(!any_bad, front, count, pages, taken, given, added, p.cap);
  const bool ok = verdict == ExtendVerdict::ok;
  const int code = ok ? RWTTT_OK : verdict == ExtendVerdict::invalid ? RWTTT_E_INVALID : RWTTT_E_CAPACITY;
  if (ok) {
#pragma unroll
    for (int k = 0; k < TURNS * 4; ++k) {
      const int ph = (have[k] + P - 1) >> shift, pw = (want[k] + P - 1) >> shift;
      if (k < turns * 4 && i0 + k < n) {
        take[i0 + k] = int(bt);
        give[i0 + k] = int(bg);
        add[i0 + k] = int(ba);
      }
      bt += max(0, pw - ph);
      bg += max(0, ph - pw);
      ba += max(0, want[k] - have[k]);
    }
    if (tid == 0) {
      take[n] = int(taken);
      give[n] = int(given);
      add[n] = int(added);
    }
  }
  __syncthreads();

  const int b = blockIdx.x, step = gridDim.x * kExtThreads, at = b * kExtThreads + tid;
  for (int i = at; i < n + 1; i += step) {
    if (i < n) p.lengths[i] = ok ? p.want[i] : p.have[i];
    p.start[i] = ok ? add[i] : 0;
  }
  if (at == 0) {
    p.new_pos[0] = ok ? int(front + taken >= pages ? front + taken - pages : front + taken) : front;
    p.new_pos[1] = ok ? int(count - taken + given) : count;
    p.result[0] = code;
    p.result[1] = ok ? int(added) : 0;
    p.result[2] = ok ? int(taken) : 0;
    p.result[3] = ok ? int(given) : 0;
  }
  // front < pages, count <= pages and i < pages: at most twice round
  auto ring_at = [&](int i) {
    unsigned x = unsigned(front) + unsigned(i);
    x = x >= unsigned(pages) ? x - unsigned(pages) : x;
    return int(x >= unsigned(pages) ? x - unsigned(pages) : x);
  };
  if (ok) {
    for (int i = at; i < taken; i += step) {
      const int r = owner_of(take, n, i);
      const int ph = (p.have[r] + P - 1) >> shift;
      p.table[size_t(r) * p.s.max_pages + ph + (i - take[r])] = p.ring[ring_at(i)];
    }
    for (int i = at; i < given; i += step) {
      const int r = owner_of(give, n, i);
      const int pw = (p.want[r] + P - 1) >> shift;
      p.ring[ring_at(count + i)] = p.table[size_t(r) * p.s.max_pages + pw + (i - give[r])];
    }
  }
  for (long long i = at; i < p.cap; i += step) {
    int slot = -1, owner = -1, position = -1;
    if (ok && i < added) {
      const int r = owner_of(add, n, int(i));
      const int h = p.have[r], ph = (h + P - 1) >> shift;
      owner = r;
      position = h + (int(i) - add[r]);
      const int lp = position >> shift;
      // a page taken in this call comes from the ring: its table entry may not be written yet
      const int page = lp >= ph ? p.ring[ring_at(take[r] + (lp - ph))] : p.table[size_t(r) * p.s.max_pages + lp];
      if (unsigned(page) < unsigned(pages)) slot = (page << shift) + (position & (P - 1));
    }
    p.slots[i] = slot;
    p.owners[i] = owner;
    p.positions[i] = position;
  }
}

// ---------------------------------------------------------------------------
// append: new rows through the slots, with the pages' key bounds
// ---------------------------------------------------------------------------
//
// Bound by the bytes for a prefill (28000 tokens of eight heads of 128 in bf16,
// 114 MB in and out: 26.4 us, 4.3 TB/s against 4.9 of a plain copy) and by
// latency below a few thousand tokens.
//
// A wave takes one kv head of a run of tokens: 16 bytes a lane, LPR lanes hold a
// row, and all NI loads of keys and of values are in flight at once.  The run's
// rows are stored from the registers.  The bounds of a page belong to the wave
// whose run holds the page's first token of this call: it adds the page's rows
// in its registers to those behind its run, which it reads again (from the L2,
// mostly), so one wave sees all of a page's new keys and no atomics are needed.

// A scaled value, clamped to the largest e4m3 number; NaN stays.
__device__ __forceinline__ float fp8_clamp(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }

template <int IO, int CT> struct AppendRow {   // 16 bytes of io
  static constexpr int E = IO ? 8 : 4;
  static constexpr int W = CT == RWTTT_FP8 ? E / 4 : CT == RWTTT_BF16 ? E / 2 : E;   // words in the cache
  uint32_t raw[4];
  __device__ __forceinline__ void load(const char* src) {
    const u32x4_t t = *reinterpret_cast<const u32x4_t*>(src);
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = t[i];
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (IO) return i & 1 ? bf16_hi(raw[i / 2]) : bf16_lo(raw[i / 2]);
    else return __uint_as_float(raw[i]);
  }
  __device__ __forceinline__ void store(char* dst, float inv_scale) const {
    uint32_t w[W];
    if constexpr (IO && CT == RWTTT_BF16) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = raw[i];
    } else if constexpr (CT == RWTTT_F32) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = raw[i];
    } else if constexpr (CT == RWTTT_BF16) {
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = bf16x2_rne(get(2 * i), get(2 * i + 1));
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = fp8_clamp(get(4 * i + j) * inv_scale);
        const int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
        w[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], v, true));
      }
    }
    if constexpr (W == 4) *reinterpret_cast<u32x4_t*>(dst) = (u32x4_t){w[0], w[1], w[2], w[3]};
    else if constexpr (W == 2) *reinterpret_cast<u32x2_t*>(dst) = (u32x2_t){w[0], w[1]};
    else *reinterpret_cast<uint32_t*>(dst) = w[0];
  }
};

// The value of x as the cache holds it.
template <int CT> __device__ __forceinline__ float stored_value(float x, float scale, float inv_scale) {
  if constexpr (CT == RWTTT_F32) return x;
  if constexpr (CT == RWTTT_BF16) return bf16_lo(bf16_rne(x));
  return __builtin_amdgcn_cvt_f32_fp8(__builtin_amdgcn_cvt_pk_fp8_f32(fp8_clamp(x * inv_scale), 0.f, 0, false), 0) * scale;
}

struct AppendParams {
  KvAppendLaunch L;
  int run;               // tokens a wave looks at
};

template <int IO, int CT, int D, int NI>
__global__ void __launch_bounds__(256) kv_append_kernel(const AppendParams ap) {
  const KvAppendLaunch& p = ap.L;
  constexpr int IOB = IO ? 2 : 4, CB = CT == RWTTT_F32 ? 4 : CT == RWTTT_BF16 ? 2 : 1;
  using Row = AppendRow<IO, CT>;
  constexpr int E = Row::E, LPR = D / E, RPI = 64 / LPR;
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int H = p.s.kv_heads, shift = p.s.page_shift, P = 1 << shift;
  const int h = unit % H, n = int(p.n), t0 = unit / H * ap.run, t1 = min(n, t0 + ap.run);
  if (t0 >= n) return;
  const unsigned rows = unsigned(p.s.n_pages) << shift;
  const int sub = lane / LPR, piece = lane % LPR;
  const char* src_k = static_cast<const char*>(p.k_new) + size_t(h) * D * IOB + piece * 16;
  const char* src_v = static_cast<const char*>(p.v_new) + size_t(h) * D * IOB + piece * 16;
  const size_t pitch_k = p.k_stride * IOB, pitch_v = p.v_stride * IOB;

  Row k[NI], v[NI];
  unsigned slot[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int t = t0 + j * RPI + sub, at = min(t, t1 - 1);
    slot[j] = t < t1 ? unsigned(p.slots[at]) : ~0u;
    k[j].load(src_k + at * pitch_k);
    v[j].load(src_v + at * pitch_v);
  }
  // lane l: the slot of token t0 + l; where the token before is not in its page, the page begins
  const unsigned mine = t0 + lane < n ? unsigned(p.slots[t0 + lane]) : ~0u;
  unsigned before = unsigned(__shfl_up(int(mine), 1));
  if (lane == 0) before = t0 > 0 ? unsigned(p.slots[t0 - 1]) : ~0u;
  const float k_scale = CT == RWTTT_FP8 && p.k_scale ? p.k_scale[h] : 1.f;
  const float v_inv = 1.f / (CT == RWTTT_FP8 && p.v_scale ? p.v_scale[h] : 1.f), k_inv = 1.f / k_scale;
  auto store_rows = [&] {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const size_t at = ((size_t(slot[j] >> shift) * H + h) * P + (slot[j] & (P - 1))) * size_t(D * CB) + piece * (E * CB);
      if (slot[j] < rows) {
        k[j].store(static_cast<char*>(p.k) + at, k_inv);
        v[j].store(static_cast<char*>(p.v) + at, v_inv);
      }
    }
  };
  if (!p.bounds) {
    store_rows();
    return;
  }

  // Rounding, scales and step keep the order, so least and largest are found on
  // the keys as they come in and only these two are rounded.
  float lo[E], hi[E];
  auto widen = [&](const Row& r) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      lo[i] = fminf(lo[i], r.get(i));      // a NaN leaves the bound as it is
      hi[i] = fmaxf(hi[i], r.get(i));
    }
  };
  const bool begins = mine < rows && !(before < rows && before >> shift == mine >> shift);
  for (unsigned long long pages = __ballot(begins && lane < t1 - t0); pages; pages &= pages - 1) {
    const int l0 = __builtin_ctzll(pages), t = t0 + l0;
    const unsigned page = unsigned(__builtin_amdgcn_readlane(int(mine), l0)) >> shift;
    // [t, end): the page's tokens in this call
    bool same = mine < rows && mine >> shift == page;
    unsigned long long miss = __ballot(!same) >> l0;
    int run = miss ? __builtin_ctzll(miss) : 64 - l0, end = t + run;
    bool fresh = __ballot(lane >= l0 && lane < l0 + run && (mine & (P - 1)) == 0) != 0;
    while (end == t0 + 64 || (end > t0 + 64 && run == 64)) {
      const unsigned s = end + lane < n ? unsigned(p.slots[end + lane]) : ~0u;
      same = s < rows && s >> shift == page;
      miss = __ballot(!same);
      run = miss ? __builtin_ctzll(miss) : 64;
      fresh |= __ballot(lane < run && (s & (P - 1)) == 0) != 0;
      if (run == 0) break;
      end += run;
    }
    int8_t* at = p.bounds + (size_t(page) * H + h) * (2 * D) + piece * E;
    uint32_t wl[E / 4], wh[E / 4];
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      wl[i] = reinterpret_cast<const uint32_t*>(at)[i];
      wh[i] = reinterpret_cast<const uint32_t*>(at + D)[i];
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      lo[i] = INFINITY;
      hi[i] = -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int u = t0 + j * RPI + sub;
      if (u >= t && u < min(end, t1)) widen(k[j]);
    }
    constexpr int U = 8;                 // loads in flight behind the run
    for (int u = t1 + sub; u < end; u += U * RPI) {
      Row r[U];
#pragma unroll
      for (int j = 0; j < U; ++j) r[j].load(src_k + min(u + j * RPI, end - 1) * pitch_k);
#pragma unroll
      for (int j = 0; j < U; ++j) widen(r[j]);   // a row twice changes no bound
    }
#pragma unroll
    for (int d = LPR; d < 64; d <<= 1) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        lo[i] = fminf(lo[i], __shfl_xor(lo[i], d));
        hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], d));
      }
    }
    if (sub == 0) {
      const float inv_step = 1.f / p.step[h];
#pragma unroll
      for (int i = 0; i < E / 4; ++i) {
        if (fresh) {
          wl[i] = 0x7f7f7f7fu;
          wh[i] = 0x81818181u;
        }
        uint32_t nl = 0, nh = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = stored_value<CT>(lo[4 * i + j], k_scale, k_inv), y = stored_value<CT>(hi[4 * i + j], k_scale, k_inv);
          const bool none = lo[4 * i + j] > hi[4 * i + j];       // NaN alone
          const float xl = none ? 127.f : floorf(x * inv_step), yh = none ? -127.f : ceilf(y * inv_step);
          const int l = min(int(int8_t(wl[i] >> (8 * j))), int(fminf(fmaxf(xl, -127.f), 127.f)));
          const int u = max(int(int8_t(wh[i] >> (8 * j))), int(fminf(fmaxf(yh, -127.f), 127.f)));
          nl |= uint32_t(l & 0xff) << (8 * j);
          nh |= uint32_t(u & 0xff) << (8 * j);
        }
        reinterpret_cast<uint32_t*>(at)[i] = nl;
        reinterpret_cast<uint32_t*>(at + D)[i] = nh;
      }
    }
  }
  store_rows();                          // last: a wait for a load also waits for the stores before it
}

// ---------------------------------------------------------------------------
// select: the pages with the largest scores
// ---------------------------------------------------------------------------
//
// max(q lo, q hi) is max(q, 0) hi - max(-q, 0) lo, so the group's queries fold
// into two vectors of whole numbers, U = sum max(q8, 0) and V = sum max(-q8, 0),
// before any page is read: a page costs two 8-bit dot products.  U and V reach
// 127 * group, so each is split into two base-128 digits.
//
// Where the rows (one: an owner and kv head) are too few to fill the chip,
// several blocks share one: each scores a part of its pages into the workspace
// and counts itself, and the last one ranks them all.
//
// The ranking counts the scores in bins of their own range, 12 bits of it, in
// LDS, and looks closer only at the bin that the last page kept lies in.
//
// Bound by latency: 64 rows of 2048 pages (30 MB of bounds, four blocks a row) take
// 14.8 us, of which the bounds' loads 9.7 (a plain read of as much: 4.6), the
// exchange between the blocks 2, the ranking 2.5; one block a row takes 19.3 us.

constexpr int kSelRows = 256;            // most rows that several blocks share
// Pages of a part: below, the exchange costs more than it saves.  64 rows of 2048
// pages take 19.3, 16.1, 14.8 and 16.0 us in 1, 2, 4 and 8 parts, 66 rows of up to 564
// pages 8.1 and 8.6 us in 1 and 2.
constexpr int kSelPart = 512;

struct SelectParams {
  KvSelectLaunch L;
  uint32_t* count;       // [rows]: parts that are done, zero between calls
  uint32_t* score;       // [rows][pitch]
  int splits, pitch;
};

// Sum of the values of LPP neighbouring lanes, in each of them.
template <int LPP> __device__ __forceinline__ int lanes_sum(int x) {
  x += int(dpp<kDppXor1>(uint32_t(x)));
  x += int(dpp<kDppXor2>(uint32_t(x)));
  x += int(dpp<kDppHalfMirror>(uint32_t(x)));
  if constexpr (LPP >= 16) x += int(dpp<kDppMirror>(uint32_t(x)));
  if constexpr (LPP >= 32) x += __shfl_xor(x, 16);
  return x;
}

// Exclusive sum over a block's threads.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* waves) {
  const int wave = threadIdx.x >> 6;
  const uint32_t inc = wave_scan(x);
  if ((threadIdx.x & 63) == 63) waves[wave] = inc;
  __syncthreads();
  uint32_t at = inc - x;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) at += w < wave ? waves[w] : 0u;
  return at;
}

template <int IO, int D>
__global__ void __launch_bounds__(kSelThreads) kv_select_kernel(const SelectParams sp) {
  const KvSelectLaunch& p = sp.L;
  extern __shared__ uint32_t key[];      // [pitch] scores, ordered as unsigned numbers
  __shared__ SelectLds<D> lds;
  const int H = p.s.kv_heads, G = p.s.group, shift = p.s.page_shift, P = 1 << shift;
  const int row = blockIdx.x / sp.splits, split = blockIdx.x % sp.splits, i = row / H, h = row % H;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = p.rows ? p.rows[i] : i;
  if (unsigned(r) >= unsigned(p.s.n_owners)) return;
  const int len = clampi(p.lengths[r], 0, p.s.max_pages << shift);
  const int np = (len + P - 1) >> shift, keep = int(p.keep);
  int32_t* out = p.pages + (size_t(r) * H + h) * keep;
  if (np <= keep) {
    for (int j = split * kSelThreads + tid; j < keep; j += sp.splits * kSelThreads) out[j] = j < np ? j : -1;
    return;
  }
  // as many of the row's blocks as its pages are worth
  const int splits = min(sp.splits, max(1, (np + kSelPart / 2) / kSelPart));
  if (split >= splits) return;
  const int chunk = ((np + splits - 1) / splits + 1) & ~1;
  const int j0 = min(np, split * chunk), j1 = min(np, j0 + chunk);

  // the first pages' bounds are on their way while the queries are folded:
  // LPP lanes a page, 16 bytes of its bounds each, the low bounds first
  constexpr int LPP = 2 * D / 16, PPI = 64 / LPP, U = 8;
  const int piece = lane % LPP, sub = lane / LPP;
  const int32_t* table = p.table + size_t(r) * p.s.max_pages;
  const int8_t* bounds = p.bounds + size_t(h) * (2 * D) + piece * 16;
  u32x4_t b[U];
  auto load_bounds = [&](int base) {
    unsigned page[U];
#pragma unroll
    for (int k = 0; k < U; ++k) page[k] = unsigned(table[min(base + k * PPI + sub, np - 1)]);
#pragma unroll
    for (int k = 0; k < U; ++k)
      b[k] = *reinterpret_cast<const u32x4_t*>(bounds + size_t(min(page[k], unsigned(p.s.n_pages - 1))) * H * (2 * D));
  };
  int base = j0 + wave * (PPI * U);
  if (base < j1) load_bounds(base);

  // the group's largest magnitude, then its digits
  float a = 0.f;
  const size_t q0 = size_t(r) * p.q_stride + size_t(h) * G * D;
  for (int j = tid; j < G * D; j += kSelThreads) {
    const float q = IO ? Elem<uint16_t>::get(p.q, q0 + j) : Elem<float>::get(p.q, q0 + j);
    a = fmaxf(a, fabsf(q));
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) a = fmaxf(a, __shfl_xor(a, d));
  if (lane == 0) lds.wave_max[wave] = a;
  __syncthreads();
  a = 0.f;
  for (int w = 0; w < kSelWaves; ++w) a = fmaxf(a, lds.wave_max[w]);
  const float to = query_unit(a);
  if (tid < D) {
    int up = 0, down = 0;
    for (int g = 0; g < G; ++g) {
      const float q = IO ? Elem<uint16_t>::get(p.q, q0 + g * D + tid) : Elem<float>::get(p.q, q0 + g * D + tid);
      const int q8 = int(fminf(fmaxf(rintf(q * to), -127.f), 127.f));   // the clamp only acts on NaN
      up += max(q8, 0);
      down += max(-q8, 0);
    }
    uint8_t* dg = reinterpret_cast<uint8_t*>(lds.digits);
    dg[tid] = uint8_t(up & 127);
    dg[D + tid] = uint8_t(up >> 7);
    dg[2 * D + tid] = uint8_t(down & 127);
    dg[3 * D + tid] = uint8_t(down >> 7);
  }
  __syncthreads();

  const bool low = piece < LPP / 2;
  int d0[4], d1[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int at = (piece % (LPP / 2)) * 4 + w;
    d0[w] = int(lds.digits[low ? 2 : 0][at]);
    d1[w] = int(lds.digits[low ? 3 : 1][at]);
  }
  for (; base < j1; base += kSelWaves * PPI * U) {
    int s[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      int s0 = 0, s1 = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        s0 = __builtin_amdgcn_sdot4(int(b[k][w]), d0[w], s0, false);
        s1 = __builtin_amdgcn_sdot4(int(b[k][w]), d1[w], s1, false);
      }
      s[k] = s0 + (s1 << 7);
      s[k] = low ? -s[k] : s[k];
    }
    if (base + kSelWaves * PPI * U < j1) load_bounds(base + kSelWaves * PPI * U);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      s[k] = lanes_sum<LPP>(s[k]);
      const int j = base + k * PPI + sub;
      if (piece == 0 && j < j1) key[j] = uint32_t(s[k]) ^ 0x80000000u;
    }
  }
  __syncthreads();

  if (splits > 1) {
    uint64_t* shared_key = reinterpret_cast<uint64_t*>(sp.score + size_t(row) * sp.pitch);
    for (int k = j0 / 2 + tid; j0 < j1 && k < (j1 + 1) / 2; k += kSelThreads)
      __hip_atomic_store(shared_key + k, uint64_t(key[2 * k + 1]) << 32 | key[2 * k], __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    shared_done();
    __syncthreads();
    if (tid == 0) lds.pick[0] = count_in(&sp.count[row], uint32_t(splits - 1));
    __syncthreads();
    if (!lds.pick[0]) return;
    for (int k = tid; k < (np + 1) / 2; k += kSelThreads) {
      const uint64_t w = __hip_atomic_load(shared_key + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      key[2 * k] = uint32_t(w);
      key[2 * k + 1] = uint32_t(w >> 32);
    }
    __syncthreads();
  }

  // Pages [f0, f1) are ranked, by v = score - least (rwttt_kv_rules.h).  None is to be
  // taken: no v reaches above ~0.
  const int f0 = int(p.first), f1 = np - int(p.last);
  Rank rank{~0u, 0, 0};
  uint32_t least = ~0u;
  if (const int want = keep - (np - (f1 - f0)); want > 0) {
    uint32_t most = 0;
    for (int j = f0 + tid; j < f1; j += kSelThreads) {
      least = min(least, key[j]);
      most = max(most, key[j]);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      least = min(least, uint32_t(__shfl_xor(int(least), d)));
      most = max(most, uint32_t(__shfl_xor(int(most), d)));
    }
    if (lane == 0) {
      lds.wave_least[wave] = least;
      lds.wave_most[wave] = most;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
      least = min(least, lds.wave_least[w]);
      most = max(most, lds.wave_most[w]);
    }
    rank = rank_begin(most - least, want);
    while (rank.top > 0) {
      constexpr int PER = kSelBins / kSelThreads;
      for (int k = tid; k < kSelBins / 4; k += kSelThreads)
        *reinterpret_cast<u32x4_t*>(lds.hist + 4 * k) = (u32x4_t){0, 0, 0, 0};
      if (tid == 0) lds.pick[3] = 0;
      __syncthreads();
      for (int j = f0 + tid; j < f1; j += kSelThreads) {
        const uint32_t v = key[j] - least;
        if (rank_in(rank, v)) atomicAdd(&lds.hist[rank_bin(rank, v)], 1u);
      }
      __syncthreads();
      uint32_t c[PER], sum = 0;          // the thread's bins, from the top
#pragma unroll
      for (int k = 0; k < PER; ++k) sum += c[k] = lds.hist[kSelBins - 1 - (tid * PER + k)];
      uint32_t above = block_scan(sum, lds.wave_sum[0]);
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (above < uint32_t(rank.want) && above + c[k] >= uint32_t(rank.want)) {
          lds.pick[0] = uint32_t(kSelBins - 1 - (tid * PER + k));
          lds.pick[1] = above;
          lds.pick[2] = c[k];
        }
        above += c[k];
      }
      __syncthreads();
      const uint32_t in_bin = lds.pick[2];
      rank = rank_narrow(rank, lds.pick[0], int(lds.pick[1]), int(in_bin));
      if (rank.top > 0 && in_bin <= uint32_t(kSelThreads)) {
        for (int j = f0 + tid; j < f1; j += kSelThreads) {
          const uint32_t v = key[j] - least;
          if (rank_in(rank, v)) lds.close[atomicAdd(&lds.pick[3], 1u)] = ScoredPage{v, uint32_t(j)};
        }
        __syncthreads();
        if (uint32_t(tid) < in_bin) {
          const ScoredPage mine = lds.close[tid];
          uint32_t larger = 0, before = 0;
          for (uint32_t k = 0; k < in_bin; ++k) {
            const ScoredPage x = lds.close[k];
            larger += x.score > mine.score;
            before += x.score == mine.score && x.page < mine.page;
          }
          if (larger + before == uint32_t(rank.want) - 1) {   // the last page kept
            lds.pick[0] = mine.score;
            lds.pick[1] = before + 1;
          }
        }
        __syncthreads();
        rank = Rank{lds.pick[0], int(lds.pick[1]), 0};
      }
      __syncthreads();
    }
  }
  const uint32_t v0 = rank.v0;
  const int want = rank.want;

  // in order
  const int per = (np + kSelThreads - 1) / kSelThreads, p0 = min(np, tid * per), p1 = min(np, p0 + per);
  uint32_t count = 0;                    // taken for sure, and equal to v0 in the upper half
  for (int j = p0; j < p1; ++j) {
    const bool forced = j < f0 || j >= f1;
    const uint32_t v = key[j] - least;
    count += forced || v > v0 ? 1u : v == v0 ? 0x10000u : 0u;
  }
  const uint32_t at = block_scan(count, lds.wave_sum[1]);
  int so = int(at & 0xffffu), se = int(at >> 16);
  for (int j = p0; j < p1; ++j) {
    const bool forced = j < f0 || j >= f1;
    const uint32_t v = key[j] - least;
    const bool over = forced || v > v0, equal = !over && v == v0;
    if (over || (equal && se < want)) out[so + min(se, want)] = j;
    so += over;
    se += equal;
  }
}

// ---------------------------------------------------------------------------
// attend: one new token over the cache
// ---------------------------------------------------------------------------
//
// Bound by the cache's bytes: a key and a value are used by at most sixteen
// queries.  All work of a call -- tiles of KT rows of every (listed owner, kv
// head, sixteen queries) -- forms one line that is cut into equal parts, one a
// block, so a long owner is spread over the chip and many short ones fill it as
// well.  The block's waves share each row of its part (a row: one owner, head
// and sixteen queries); every wave keeps the running maximum and sum of its
// queries and the unscaled output in registers, and the four are added through
// LDS.  A row that one block holds whole is written there.  Of a row that more
// blocks hold each leaves its partial result in the workspace and counts
// itself; the one that finds the count full joins them in the order of the
// blocks, so the bits do not depend on which it is.
//
// Matrix instructions with the keys as rows and the queries as columns:
// S^T = K Q^T (16 x 16 over the head's channels) leaves each lane 4 rows of one
// query, which is the operand layout of P^T in O^T = V^T P^T when the rows are
// dealt to the tiles so that a lane's 4 + 4 scores are 8 consecutive rows.  So
// neither scores nor probabilities move between lanes.  V arrives with the
// channels of a row in one lane; its transposed operand takes one byte
// permutation for each pair of values.  A probability enters the second product as
// three bf16 terms, and so does a query of fp32 over a narrower cache: they hold all
// 24 bits of it, and the matrix units have the room (with two terms, 16 bits of a
// probability, no call is faster by more than 1%: 31.1 against
// 31.3 us for eight owners of 4200 rows, 331.2 against 331.4 for 32 of 16000).
//
// Measured: 32 owners of 12000-20000 rows, eight kv heads of four queries and 128
// channels in bf16, 2.19 GB: 331 us, 6.6 TB/s, what a plain streaming read of this
// shape reaches.  Smaller calls add 8 to 9 us to their bytes' time: launch 1.7, the
// row table and cuts 1.5, the first tile's loads 2.5, adding the waves' sums 1 and
// the join 3.

constexpr int kAttThreads = 256;

struct AttendParams {
  KvAttendLaunch L;
  uint32_t* count;       // [blocks], then [windows * 2]: results that have been left, zero between calls
  float* part;           // [blocks * 2 + windows * 2][heads][D]
  float* part_ml;        // the same of [2]: maximum (of log2), sum
  int blocks, head_tiles, part_heads, acc_words;
  float scale_log2;      // scale * log2(e)
  bool stream;           // the cache passes through: non-temporal loads
};

constexpr int kAttWaves = kAttThreads / 64;
// Blocks of a row that are joined at once; more go in windows first, since one block
// reads all it joins: a row over all 512 blocks (131072 rows of one head) took 67 us
// that way and takes 27.  The second level costs about 3 us, 48 results no more.
constexpr int kJoinWindow = 32, kJoinDirect = 48;
constexpr int kAttPad = 4;               // floats behind a query's sums in LDS: neighbours in other banks

// Rows of keys a wave takes at a time.
constexpr int tile_rows(int ct) { return ct == RWTTT_F32 ? 16 : 32; }

struct RowRange {
  int base, tiles, held;                 // base: first tile's first row; held: listed pages
};

template <int KT> __device__ __forceinline__ RowRange row_range(const KvAttendLaunch& p, int len) {
  RowRange x{0, 0, 0};
  if (len == 0) return x;
  if (p.pages) {
    const int np = (len + (1 << p.s.page_shift) - 1) >> p.s.page_shift;
    x.held = min(np, int(p.keep));
    x.tiles = ((x.held << p.s.page_shift) + KT - 1) / KT;
  } else {
    const int lo = p.window ? max(0, len - int(p.window)) : 0;
    x.base = lo / KT * KT;
    x.tiles = (len - x.base + KT - 1) / KT;
  }
  return x;
}

// The listed owners in LDS: id (-1: none), rows, and pre[i] = cost of one head's
// rows of the owners before i, pre[n] of all.
struct RowTable {
  int* owner;
  int* len;
  uint32_t* pre;
  __device__ RowTable(uint32_t* lds, int n) : owner(reinterpret_cast<int*>(lds)), len(owner + n), pre(lds + 2 * n) {}
};
__host__ __device__ constexpr size_t row_table_words(int n) { return 3 * size_t(n) + 1; }

template <int KT>
__device__ __forceinline__ void fill_rows(const KvAttendLaunch& p, const RowTable& rt, uint32_t* wave_sum) {
  const int n = int(p.n), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (n + kAttThreads - 1) / kAttThreads, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  auto cost = [&](int len) {
    const int tiles = row_range<KT>(p, len).tiles;
    return row_cost(tiles);
  };
  uint32_t sum = 0;
  for (int i = i0; i < i1; ++i) {
    const int r = p.rows ? p.rows[i] : i;
    const bool there = unsigned(r) < unsigned(p.s.n_owners);
    const int len = there ? clampi(p.lengths[r], 0, p.s.max_pages << p.s.page_shift) : 0;
    rt.owner[i] = there ? r : -1;
    rt.len[i] = len;
    sum += cost(len);
  }
  const uint32_t inc = wave_scan(sum);
  if (lane == 63) wave_sum[wave] = inc;
  __syncthreads();
  uint32_t at = inc - sum;
  for (int w = 0; w < wave; ++w) at += wave_sum[w];
  for (int i = i0; i < i1; ++i) {
    rt.pre[i] = at;
    at += cost(rt.len[i]);
  }
  if (i1 == n && i0 < n) rt.pre[n] = at;
  __syncthreads();
}

template <int W, bool HINT = false> __device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  if constexpr (W == 1) {
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
    w[0] = HINT ? __builtin_nontemporal_load(q) : *q;
  } else if constexpr (W == 2) {
    const u32x2_t* q = reinterpret_cast<const u32x2_t*>(p);
    const u32x2_t t = HINT ? __builtin_nontemporal_load(q) : *q;
    w[0] = t[0];
    w[1] = t[1];
  } else {
    const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p);
    const u32x4_t t = HINT ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = t[i];
  }
}

__device__ __forceinline__ uint32_t fp8_pair(uint32_t w, bool high) {   // exact: e4m3 fits bf16
  const bf16x2_t h = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)
                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ bf16x8_t as_bf16x8(const uint32_t* w) {
  const u32x4_t t = {w[0], w[1], w[2], w[3]};
  return *reinterpret_cast<const bf16x8_t*>(&t);
}

// x = terms[0] + terms[1] + ... in bf16, eight values a lane: three terms keep all
// 24 bits of each.
template <int N> __device__ __forceinline__ void split_bf16(const float* x, bf16x8_t* terms) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int t = 0; t < N; ++t) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = bf16x2_rne(rest[2 * i], rest[2 * i + 1]);
      if (t + 1 < N) {
        rest[2 * i] -= bf16_lo(w[i]);
        rest[2 * i + 1] -= bf16_hi(w[i]);
      }
    }
    terms[t] = as_bf16x8(w);
  }
}

// Layout of one tile.  CT: cache type, D: head dim.
//   keys:   KW 16-byte pieces a lane and 16-row tile; piece s of lane group g
//           holds the channels from key_channel(s, g) on
//   values: NE chunks of VE channels a lane, from value_channel(e, c) on, for
//           each of the KT / 4 rows of the lane's group
template <int CT, int D> struct TileShape {
  static constexpr int B = CT == RWTTT_F32 ? 4 : CT == RWTTT_BF16 ? 2 : 1;
  static constexpr int KT = tile_rows(CT), NT = KT / 16;
  static constexpr int KE = 16 / B, KW = D / (4 * KE);
  static constexpr int VE = D / 16 < KE ? D / 16 : KE, NE = D / 16 / VE, VW = VE * B / 4;
  static constexpr int VR = KT / 4;      // rows of values a lane holds
  static constexpr int NA = D / 16;      // output tiles (four channels a lane)
  __device__ static int key_channel(int s, int g) { return (s * 4 + g) * KE; }
  __device__ static int value_channel(int e, int c) { return (e * 16 + c) * VE; }
};

// Which pages a tile's halves (16 rows each) lie in, and which of their rows count.
template <int NT> struct TileAt {
  uint32_t page[NT];
  int off[NT], from[NT], to[NT];         // rows [from, to) of the half count
};

template <int IO, int CT, int D, bool NT_HINT>
__global__ void __launch_bounds__(kAttThreads, D == 256 ? 1 : 2) kv_attend_kernel(const AttendParams ap) {
  using S = TileShape<CT, D>;
  constexpr int KT = S::KT, NT = S::NT;
  constexpr bool F = CT == RWTTT_F32;
  constexpr int NQ = IO ? 1 : 3, NP = 3;               // bf16 terms of a query, of a probability
  const KvAttendLaunch& p = ap.L;
  __shared__ uint32_t wave_sum[kAttWaves];
  __shared__ float wave_ml[kAttWaves][16][2];
  __shared__ uint32_t last;
  extern __shared__ float wave_acc[];    // [waves][heads][D + kAttPad], then the row table
  const RowTable rt(reinterpret_cast<uint32_t*>(wave_acc + ap.acc_words), int(p.n));
  const uint32_t* pre = rt.pre;
  fill_rows<KT>(p, rt, wave_sum);

  const int n = int(p.n), H = p.s.kv_heads, HT = ap.head_tiles, VH = H * HT, G = p.s.group;
  const int shift = p.s.page_shift, P = 1 << shift;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // owners without rows: 0 and -inf
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int owner = rt.owner[i];
    if (rt.len[i] != 0 || owner < 0) continue;
    for (int d = tid; d < H * G * D; d += kAttThreads) {
      if constexpr (IO) Elem<uint16_t>::put(p.out, size_t(owner) * p.out_stride + d, 0.f);
      else Elem<float>::put(p.out, size_t(owner) * p.out_stride + d, 0.f);
    }
    if (p.lse)
      for (int d = tid; d < H * G; d += kAttThreads) p.lse[size_t(owner) * H * G + d] = -INFINITY;
  }

  const uint64_t total = uint64_t(pre[n]) * VH;
  const int parts = parts_of(total, ap.blocks), b = blockIdx.x;
  if (b >= parts) return;
  const Cut cut(total, parts);
  int i = 0;                             // the listed owner that u lies in
  uint64_t u = total, end = total;       // the block's part, its cuts where they are made
#pragma unroll 1
  for (int k = 1; k >= 0; --k) {
    end = u;
    u = cut.begin(b + k);
    if (u >= total) continue;            // behind the last part
    // 64 owners at a look
    const int stride = (n + 63) / 64;
    i = (__builtin_popcountll(__ballot(lane * stride < n && uint64_t(pre[min(lane * stride, n)]) * VH <= u)) - 1) * stride;
    if (stride > 1)
      i += __builtin_popcountll(__ballot(lane < stride && i + lane < n && uint64_t(pre[min(i + lane, n)]) * VH <= u)) - 1;
    const uint32_t cost = pre[i + 1] - pre[i];
    const uint32_t x = uint32_t(u - uint64_t(pre[i]) * VH) % cost;   // an owner's tiles and heads fit 32 bits
    u += uint64_t(snapped(x, cost)) - x;
  }
  i = __builtin_amdgcn_readfirstlane(i);

  while (u < end) {
    const uint32_t cost = __builtin_amdgcn_readfirstlane(pre[i + 1] - pre[i]);
    const uint32_t x = uint32_t(u - uint64_t(pre[i]) * VH);
    const int vh = __builtin_amdgcn_readfirstlane(int(x / max(cost, 1u)));
    if (cost == 0 || vh == VH) {         // no rows, or the cut moved to the owner's end
      ++i;
      continue;
    }
    const int tiles = int(cost) - kRowCost;
    const uint32_t x0 = __builtin_amdgcn_readfirstlane(x % cost);
    const uint32_t x1 = uint32_t(min(uint64_t(cost), x0 + (end - u)));
    const int seg0 = max(0, int(x0) - kRowCost), seg1 = max(0, int(x1) - kRowCost);
    const uint64_t u0 = u - x0;          // the row's place in the line
    u += x1 - x0;
    const int at_row = i;
    if (x1 == cost && vh == VH - 1) ++i;
    const int t0 = seg0 + int(uint32_t(seg1 - seg0) * wave / kAttWaves);
    const int t1 = seg0 + int(uint32_t(seg1 - seg0) * (wave + 1) / kAttWaves);
    const int owner = __builtin_amdgcn_readfirstlane(rt.owner[at_row]);
    const int len = __builtin_amdgcn_readfirstlane(rt.len[at_row]);
    const RowRange row = row_range<KT>(p, len);
    const int base = row.base, held = row.held;
    const int h = vh / HT, head0 = (vh % HT) * 16, heads = min(16, G - head0);
    const int least = p.window ? max(0, len - int(p.window)) : 0, last_page = (len - 1) >> shift;
    const scalar_i32 table = scalar(p.table + size_t(owner) * p.s.max_pages);
    const scalar_i32 list = scalar(p.pages ? p.pages + (size_t(owner) * H + h) * p.keep : nullptr);

    auto locate = [&](int t) {
      TileAt<NT> at;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int row0 = base + t * KT + j * 16;
        int lp = row0 >> shift;
        at.off[j] = row0 & (P - 1);
        bool none = false;
        if (p.pages) {
          none = lp >= held;
          lp = list[min(lp, held - 1)];
          none = none || unsigned(lp) > unsigned(last_page);
        }
        const int pos = (lp << shift) + at.off[j];
        at.from[j] = clampi(least - pos, 0, 16);
        at.to[j] = none ? 0 : clampi(len - pos, 0, 16);
        at.page[j] = min(uint32_t(table[clampi(lp, 0, last_page)]), uint32_t(p.s.n_pages - 1));
      }
      return at;
    };

    // queries: the lane's column is one of them; piece s of its channels feeds PER operands
    constexpr int PER = F ? 1 : S::KE / 8, QN = F ? D / 16 : D / 32, QW = F || IO ? 4 : 8;
    const char* q_at = static_cast<const char*>(p.q) +
                       (size_t(owner) * p.q_stride + (size_t(h) * G + head0 + (c < heads ? c : 0)) * D) * (IO ? 2 : 4);
    uint32_t qw[QN][QW];
#pragma unroll
    for (int s = 0; s < QN; ++s) {
      const int ch = S::key_channel(s / PER, g) + (s % PER) * 8;
#pragma unroll
      for (int j = 0; j < QW; j += 4) load_words<4>(q_at + ch * (IO ? 2 : 4) + j * 4, &qw[s][j]);
    }
    const float to_log2 = ap.scale_log2 * (CT == RWTTT_FP8 && p.k_scale ? p.k_scale[h] : 1.f);

    float m = -INFINITY, l = 0.f;
    f32x4_t acc[S::NA];
#pragma unroll
    for (int a = 0; a < S::NA; ++a) acc[a] = (f32x4_t){0.f, 0.f, 0.f, 0.f};

    uint32_t kw[NT][S::KW][4];
    uint32_t vw[S::NE][S::VR][S::VW];
    // row of a half that the lane loads: keys, one a lane; values, VR in turn
    const int k_half = NT == 2 ? c >> 3 : 0, v_half = NT == 2 ? g >> 1 : 0;
    auto half_of = [&](const TileAt<NT>& at, const void* cache, int half) {
      const uint32_t page = NT == 2 && half ? at.page[NT - 1] : at.page[0];
      const int off = NT == 2 && half ? at.off[NT - 1] : at.off[0];
      return static_cast<const char*>(cache) + ((size_t(page) * H + h) * P + off) * size_t(D * S::B);
    };
    auto load_keys = [&](const TileAt<NT>& at) {
      const char* src = half_of(at, p.k, k_half);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int rr = NT == 2 ? ((c >> 2) & 1) * 8 + t * 4 + (c & 3) : c;
#pragma unroll
        for (int s = 0; s < S::KW; ++s) load_words<4, NT_HINT>(src + (rr * D + S::key_channel(s, g)) * S::B, kw[t][s]);
      }
    };
    auto load_values = [&](const TileAt<NT>& at) {
      const char* src = half_of(at, p.v, v_half);
#pragma unroll
      for (int e = 0; e < S::NE; ++e)
#pragma unroll
        for (int k = 0; k < S::VR; ++k) {
          const int rr = NT == 2 ? (g & 1) * 8 + k : g * 4 + k;
          load_words<S::VW, NT_HINT>(src + (rr * D + S::value_channel(e, c)) * S::B, vw[e][k]);
        }
    };

    TileAt<NT> at = locate(min(t0, seg1 - 1)), next = at;
    // With the condition the compiler keeps a second set of registers and loads the
    // next tile while this one is in use: 347 against 373 us for 16 owners of 8500
    // rows, head dim 256, fp32.  Three terms of a query leave no room for it.
    constexpr bool kSecondSet = IO || CT != RWTTT_BF16;
    if (!kSecondSet || t0 < t1) {
      load_keys(at);
      load_values(at);
    }
    bf16x8_t q[F ? 1 : NQ][F ? 1 : QN];
    f32x4_t qf[F ? QN : 1];
#pragma unroll
    for (int s = 0; s < QN; ++s) {
#pragma unroll
      for (int j = 0; j < QW; ++j) qw[s][j] = c < heads ? qw[s][j] : 0u;
      if constexpr (F) {
#pragma unroll
        for (int j = 0; j < 4; ++j) qf[s][j] = __uint_as_float(qw[s][j]);
      } else if constexpr (IO) {
        q[0][s] = as_bf16x8(qw[s]);
      } else {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(qw[s][j]);
        bf16x8_t terms[NQ];
        split_bf16<NQ>(f, terms);
#pragma unroll
        for (int k = 0; k < NQ; ++k) q[k][s] = terms[k];
      }
    }
    for (int t = t0; t < t1; ++t) {
      const bool more = t + 1 < t1;
      if (more) next = locate(t + 1);

      // scores: s[j] belongs to the tile's row g * VR + j
      float s[S::VR];
#pragma unroll
      for (int k = 0; k < NT; ++k) {
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
        if constexpr (F) {
#pragma unroll
          for (int a = 0; a < D / 16; ++a)
#pragma unroll
            for (int b = 0; b < 4; ++b)
              sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[k][a][b]), qf[a][b], sc, 0, 0, 0);
        } else {
#pragma unroll
          for (int a = 0; a < D / 32; ++a) {
            bf16x8_t key;
            if constexpr (CT == RWTTT_BF16) {
              key = as_bf16x8(kw[k][a]);
            } else {
              uint32_t wd[4];
#pragma unroll
              for (int b = 0; b < 4; ++b) wd[b] = fp8_pair(kw[k][a / 2][(a & 1) * 2 + b / 2], b & 1);
              key = as_bf16x8(wd);
            }
#pragma unroll
            for (int b = NQ - 1; b >= 0; --b)
              sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[b][a], sc, 0, 0, 0);
          }
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) s[k * 4 + b] = sc[b] * to_log2;
      }
      if (more) load_keys(next);

      bool whole = true;
#pragma unroll
      for (int j = 0; j < NT; ++j) whole = whole && at.from[j] == 0 && at.to[j] == 16;
      // the lane's rows of its half that count
      const int from = (v_half ? at.from[NT - 1] : at.from[0]) - (NT == 2 ? (g & 1) * 8 : g * 4);
      const int to = (v_half ? at.to[NT - 1] : at.to[0]) - (NT == 2 ? (g & 1) * 8 : g * 4);
      if (!whole) {
#pragma unroll
        for (int j = 0; j < S::VR; ++j) s[j] = j >= from && j < to ? s[j] : -INFINITY;
      }
      float top = s[0];
#pragma unroll
      for (int j = 1; j < S::VR; ++j) top = fmaxf(top, s[j]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (__any(top > m)) {
        const float up = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - up);
        m = up;
        l *= f;
#pragma unroll
        for (int a = 0; a < S::NA; ++a) acc[a] *= f;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float pr[S::VR];
#pragma unroll
      for (int j = 0; j < S::VR; ++j) {
        pr[j] = __builtin_amdgcn_exp2f(s[j] - ref);
        l += pr[j];
      }
      if (!whole) {                      // what lies behind an owner's rows may be anything
#pragma unroll
        for (int e = 0; e < S::NE; ++e)
#pragma unroll
          for (int j = 0; j < S::VR; ++j)
#pragma unroll
            for (int b = 0; b < S::VW; ++b) vw[e][j][b] = j >= from && j < to ? vw[e][j][b] : 0u;
      }
      if constexpr (F) {
#pragma unroll
        for (int e = 0; e < S::NE; ++e)
#pragma unroll
          for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              acc[e * 4 + a] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[e][j][a]), pr[j],
                                                                    acc[e * 4 + a], 0, 0, 0);
      } else {
        bf16x8_t pt[NP];
        split_bf16<NP>(pr, pt);
#pragma unroll
        for (int e = 0; e < S::NE; ++e)
#pragma unroll
          for (int a = 0; a < S::VE; ++a) {
            uint32_t wd[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (CT == RWTTT_BF16) {
                wd[j] = __builtin_amdgcn_perm(vw[e][2 * j + 1][a / 2], vw[e][2 * j][a / 2],
                                              a & 1 ? 0x07060302u : 0x05040100u);
              } else {
                wd[j] = fp8_pair(__builtin_amdgcn_perm(vw[e][2 * j + 1][a / 4], vw[e][2 * j][a / 4],
                                                       a & 2 ? 0x07030602u : 0x05010400u),
                                 a & 1);
              }
            }
            const bf16x8_t val = as_bf16x8(wd);
#pragma unroll
            for (int b = NP - 1; b >= 0; --b)
              acc[e * S::VE + a] =
                  __builtin_amdgcn_mfma_f32_16x16x32_bf16(val, pt[b], acc[e * S::VE + a], 0, 0, 0);
          }
      }
      if (more) {
        load_values(next);
        at = next;
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // the waves' sums into LDS: acc[e * VE + a][j] is channel
    // value_channel(e, 4 g + j) + a of query c
    constexpr int DP = D + kAttPad;
    if (g == 0) {
      wave_ml[wave][c][0] = m;
      wave_ml[wave][c][1] = l;
    }
    if (c < heads) {
#pragma unroll
      for (int e = 0; e < S::NE; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int a = 0; a < S::VE; a += 4)
            *reinterpret_cast<f32x4_t*>(wave_acc + (wave * heads + c) * DP + S::value_channel(e, g * 4 + j) + a) =
                (f32x4_t){acc[e * S::VE + a][j], acc[e * S::VE + a + 1][j], acc[e * S::VE + a + 2][j],
                          acc[e * S::VE + a + 3][j]};
    }
    __syncthreads();

    constexpr int LPR = D / 4;           // lanes a query
    const int cols = heads * LPR;
    const float vs = CT == RWTTT_FP8 && p.v_scale ? p.v_scale[h] : 1.f;
    auto write_out = [&](int head, int col, f32x4_t sum, float top, float total_l) {
      const float norm = total_l == 0.f ? 0.f : vs / total_l;
      const size_t d = size_t(owner) * p.out_stride + (size_t(h) * G + head0 + head) * D + col * 4;
      if constexpr (IO)
        *reinterpret_cast<u32x2_t*>(static_cast<uint16_t*>(p.out) + d) =
            (u32x2_t){bf16x2_rne(sum[0] * norm, sum[1] * norm), bf16x2_rne(sum[2] * norm, sum[3] * norm)};
      else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + d) = sum * norm;
      if (p.lse && col == 0)
        p.lse[(size_t(owner) * H + h) * G + head0 + head] =
            total_l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total_l)) * 0.6931471805599453f;
    };
    auto leave = [&](size_t slot, int col, f32x4_t sum, float top, float total_l) {
      share(ap.part + slot * D + col * 4, sum[0], sum[1]);
      share(ap.part + slot * D + col * 4 + 2, sum[2], sum[3]);
      if (col == 0) share(ap.part_ml + slot * 2, top, total_l);
    };
    const bool complete = seg0 == 0 && seg1 == tiles;
    for (int k = tid; k < cols; k += kAttThreads) {
      const int head = k / LPR, col = k % LPR;
      f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
      float top = -INFINITY, sl = 0.f;
#pragma unroll
      for (int v = 0; v < kAttWaves; ++v) top = fmaxf(top, wave_ml[v][head][0]);
#pragma unroll
      for (int v = 0; v < kAttWaves; ++v) {
        const float mv = wave_ml[v][head][0], f = mv == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mv - top);
        sum += f * *reinterpret_cast<const f32x4_t*>(wave_acc + (v * heads + head) * DP + col * 4);
        sl += f * wave_ml[v][head][1];
      }
      if (complete) {
        write_out(head, col, sum, top, sl);
      } else {
        leave((size_t(b) * 2 + (seg0 == 0 ? 1 : 0)) * ap.part_heads + head, col, sum, top, sl);
      }
    }
    if (!complete) {
      // The row's blocks are neighbours.  A few are joined at once; more in windows
      // of 32 neighbours first, then the windows.  Counters: of the row, the one of
      // its first block, since only the last row of a block's part can go on behind
      // it; of a window, one for the row that began before it and one for the row
      // that begins in it and goes on.
      const int b0 = first_part(cut, u0), b1 = last_part(cut, u0, cost);
      const int w = b / kJoinWindow, w0 = b0 / kJoinWindow, w1 = b1 / kJoinWindow;
      bool final = b1 - b0 < kJoinDirect;
      int k0 = final ? b0 : max(b0, w * kJoinWindow), k1 = final ? b1 : min(b1, (w + 1) * kJoinWindow - 1);
      uint32_t* count = final ? &ap.count[b0] : &ap.count[ap.blocks + w * 2 + (w == w0 ? 1 : 0)];
      int slots = 0, first = b0;         // result k is in slot slots + 2 k + (k == first)
#pragma unroll 1
      for (;;) {
        // the block that finds all others counted goes on
        shared_done();
        __syncthreads();
        if (tid == 0) last = count_in(count, uint32_t(k1 - k0));
        __syncthreads();
        if (!last) break;
        const int groups = max(1, kAttThreads / cols);
        float* merge = wave_acc;         // [groups][cols][6] where there is more than one group
        for (int c0 = 0; c0 < cols; c0 += kAttThreads) {
          const int k = groups > 1 ? tid % cols : c0 + tid, part = groups > 1 ? tid / cols : 0;
          const bool on = k < cols && part < groups;
          const int head = k / LPR, col = k % LPR;
          f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
          float top = -INFINITY, sl = 0.f;
          auto add = [&](float xm, float xl, f32x4_t x) {
            const float up = fmaxf(top, xm), ref = up == -INFINITY ? 0.f : up;
            const float f = __builtin_amdgcn_exp2f(top - ref), fx = __builtin_amdgcn_exp2f(xm - ref);
            sum = f * sum + fx * x;
            sl = f * sl + fx * xl;
            top = up;
          };
          if (on) {
            constexpr int U = 4;         // results in flight
#pragma unroll 1
            for (int s = k0 + part; s <= k1; s += U * groups) {
              f32x4_t x[U];
              float2 ml[U];
#pragma unroll
              for (int v = 0; v < U; ++v) {
                const int r = min(s + v * groups, k1);
                const size_t at_r = size_t(slots + 2 * r + (r == first ? 1 : 0)) * ap.part_heads + head;
                const float2 lo = shared_pair(ap.part + at_r * D + col * 4);
                const float2 hi = shared_pair(ap.part + at_r * D + col * 4 + 2);
                ml[v] = shared_pair(ap.part_ml + at_r * 2);
                x[v] = (f32x4_t){lo.x, lo.y, hi.x, hi.y};
              }
#pragma unroll
              for (int v = 0; v < U; ++v)
                if (s + v * groups <= k1) add(ml[v].x, ml[v].y, x[v]);
            }
          }
          if (groups > 1) {
            if (on) {
              float* at_m = merge + size_t(part * cols + k) * 6;
              at_m[0] = top;
              at_m[1] = sl;
#pragma unroll
              for (int d = 0; d < 4; ++d) at_m[2 + d] = sum[d];
            }
            __syncthreads();
            if (on && part == 0)
              for (int v = 1; v < groups; ++v) {
                const float* at_m = merge + size_t(v * cols + k) * 6;
                add(at_m[0], at_m[1], (f32x4_t){at_m[2], at_m[3], at_m[4], at_m[5]});
              }
          }
          if (on && part == 0) {
            if (final) write_out(head, col, sum, top, sl);
            else leave(size_t(ap.blocks * 2 + w * 2 + (w == w0 ? 1 : 0)) * ap.part_heads + head, col, sum, top, sl);
          }
        }
        if (final) break;
        final = true;
        k0 = w0;
        k1 = w1;
        count = &ap.count[b0];
        slots = ap.blocks * 2;
        first = w0;
      }
    }
    __syncthreads();                     // the next row's sums go to the same LDS
  }
}

constexpr int kAttBlocks = 512;          // two a CU

int part_heads_of(int group) { return group < 16 ? group : 16; }

// Rows (an owner and kv head) that several blocks may share in a select.
int select_rows(const KvShape& s) {
  if (s.max_pages > RWTTT_KV_MAX_SELECT) return 0;
  return s.n_owners < kSelRows / s.kv_heads ? s.n_owners * s.kv_heads : kSelRows;
}

// A handle's workspace: the counters first.
struct KvWorkspace {
  uint32_t *attend_count, *select_count, *score;
  float *part, *part_ml;
  size_t bytes;
  KvWorkspace(void* base, const KvShape& s) {
    char* at = static_cast<char*>(base);
    size_t used = 0;
    auto take = [&](size_t n) {
      char* q = at + used;
      used += (n + 255) / 256 * 256;
      return q;
    };
    const size_t windows = kAttBlocks / kJoinWindow * 2;
    const size_t slots = (size_t(kAttBlocks) * 2 + windows) * part_heads_of(s.group);
    const size_t rows = select_rows(s);
    attend_count = reinterpret_cast<uint32_t*>(take((kAttBlocks + windows) * sizeof(uint32_t)));
    select_count = reinterpret_cast<uint32_t*>(take(kSelRows * sizeof(uint32_t)));
    part = reinterpret_cast<float*>(take(slots * s.head_dim * sizeof(float)));
    part_ml = reinterpret_cast<float*>(take(slots * 2 * sizeof(float)));
    score = reinterpret_cast<uint32_t*>(take(rows * select_pitch(s.max_pages) * sizeof(uint32_t)));
    bytes = used;
  }
};

}  // namespace

size_t kv_workspace_bytes(const KvShape& shape) { return KvWorkspace(nullptr, shape).bytes; }

hipError_t launch_kv_extend(const KvExtendLaunch& L, hipStream_t stream) {
  // two map entries a thread; and where the cache is large, blocks for the pages that
  // ending owners may return with no new row beside them, 16 a thread if all do (128000
  // pages of 64 owners: 12.5 us, 299 from one block; a decode step in that cache 8.5 us
  // a call either way)
  const unsigned maps = (L.cap + kExtItems - 1) / kExtItems, pages = (unsigned(L.s.n_pages) + 4095) / 4096;
  const unsigned blocks = maps > pages ? maps : pages;
  const size_t lds = size_t(L.s.n_owners + 1) * 3 * sizeof(int);
  const dim3 grid(blocks < 1 ? 1 : blocks > 512 ? 512 : blocks), block(kExtThreads);
  // sixteen owners' lengths in a thread's registers cost the small calls 2 us
  if (L.s.n_owners <= 4 * kExtThreads) hipLaunchKernelGGL(kv_extend_kernel<1>, grid, block, lds, stream, L);
  else hipLaunchKernelGGL(kv_extend_kernel<RWTTT_KV_MAX_OWNERS / (4 * kExtThreads)>, grid, block, lds, stream, L);
  return hipGetLastError();
}

namespace {

template <int IO, int CT, int D> hipError_t append_go(AppendParams p, hipStream_t stream) {
  // Decode: one token a wave, so that all pages are followed at once.  A prefill:
  // one load of rows a wave, and four where that still makes four waves a SIMD --
  // 32 chunks of 270 tokens (e4m3) take 9.2 us with one and 12.4 with four, 64 of
  // 430 (bf16) 30.0 and 26.4.
  constexpr int RPI = 64 * (IO ? 8 : 4) / D;
  const uint64_t rows = uint64_t(p.L.n) * p.L.s.kv_heads;
  const bool many = rows >= 4096u * 4 * RPI;
  p.run = rows <= 4096 ? 1 : many ? 4 * RPI : RPI;
  const uint64_t units = uint64_t((p.L.n + p.run - 1) / p.run) * p.L.s.kv_heads;
  const dim3 grid(unsigned((units + 3) / 4)), block(256);
  if (many) hipLaunchKernelGGL((kv_append_kernel<IO, CT, D, 4>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((kv_append_kernel<IO, CT, D, 1>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template <int IO, int CT> hipError_t append_dims(const AppendParams& p, hipStream_t stream) {
  return p.L.s.head_dim == 64    ? append_go<IO, CT, 64>(p, stream)
         : p.L.s.head_dim == 128 ? append_go<IO, CT, 128>(p, stream)
                                 : append_go<IO, CT, 256>(p, stream);
}

template <int IO, int CT, int D> hipError_t attend_go(AttendParams p, hipStream_t stream) {
  const uint64_t rows = uint64_t(p.L.n) * p.L.s.kv_heads * p.head_tiles;
  const dim3 grid(unsigned(attend_grid(rows, p.L.s.max_pages << p.L.s.page_shift, tile_rows(CT), p.blocks)));
  const int acc = kAttWaves * p.part_heads * (D + kAttPad), join = kAttThreads * 6;
  p.acc_words = acc < join ? join : acc;
  const size_t lds = (p.acc_words + row_table_words(int(p.L.n))) * sizeof(float);
  auto kernel = p.stream ? kv_attend_kernel<IO, CT, D, true> : kv_attend_kernel<IO, CT, D, false>;
  if (lds > 60 * 1024) {                 // more than 64 KB of the CU's 160 KB has to be asked for
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(kAttThreads), lds, stream, p);
  return hipGetLastError();
}

template <int IO, int CT> hipError_t attend_dims(const AttendParams& p, hipStream_t stream) {
  return p.L.s.head_dim == 64    ? attend_go<IO, CT, 64>(p, stream)
         : p.L.s.head_dim == 128 ? attend_go<IO, CT, 128>(p, stream)
                                 : attend_go<IO, CT, 256>(p, stream);
}

}  // namespace

hipError_t launch_kv_append(const KvAppendLaunch& L, hipStream_t stream) {
  const AppendParams p{L, 1};
  if (L.s.io_bf16) return L.s.cache == RWTTT_BF16 ? append_dims<1, RWTTT_BF16>(p, stream)
                                                  : append_dims<1, RWTTT_FP8>(p, stream);
  return L.s.cache == RWTTT_F32    ? append_dims<0, RWTTT_F32>(p, stream)
         : L.s.cache == RWTTT_BF16 ? append_dims<0, RWTTT_BF16>(p, stream)
                                   : append_dims<0, RWTTT_FP8>(p, stream);
}

hipError_t launch_kv_select(const KvSelectLaunch& L, hipStream_t stream) {
  SelectParams p;
  p.L = L;
  p.pitch = select_pitch(L.s.max_pages);
  const KvWorkspace ws(L.workspace, L.s);
  p.count = ws.select_count;
  p.score = ws.score;
  // about two blocks a CU
  const int rows = int(L.n) * L.s.kv_heads;
  p.splits = 1;
  if (L.workspace && rows <= select_rows(L.s))
    while (p.splits < 8 && p.splits * 2 * rows <= 512 && L.s.max_pages / (p.splits * 2) >= kSelPart) p.splits *= 2;
  const dim3 grid(unsigned(rows * p.splits)), block(kSelThreads);
  const size_t lds = select_lds(L.s.max_pages);
  auto go = [&](auto kernel, bool asks) {
    if (asks) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, block, lds, stream, p);
    return hipGetLastError();
  };
  const int pages = L.s.max_pages;
  if (L.s.io_bf16)
    return L.s.head_dim == 64    ? go(kv_select_kernel<1, 64>, select_asks_for_lds<64>(pages))
           : L.s.head_dim == 128 ? go(kv_select_kernel<1, 128>, select_asks_for_lds<128>(pages))
                                 : go(kv_select_kernel<1, 256>, select_asks_for_lds<256>(pages));
  return L.s.head_dim == 64    ? go(kv_select_kernel<0, 64>, select_asks_for_lds<64>(pages))
         : L.s.head_dim == 128 ? go(kv_select_kernel<0, 128>, select_asks_for_lds<128>(pages))
                               : go(kv_select_kernel<0, 256>, select_asks_for_lds<256>(pages));
}

hipError_t launch_kv_attend(const KvAttendLaunch& L, hipStream_t stream) {
  AttendParams p;
  p.L = L;
  // What is resident at once: two blocks a CU, one for 256 channels, whose registers
  // leave room for no more (16 owners of 8500 rows: 180 us in bf16 and 94 in e4m3 so,
  // 184 and 102 with twice the blocks).
  p.blocks = L.s.head_dim == 256 ? kAttBlocks / 2 : kAttBlocks;
  p.head_tiles = (L.s.group + 15) / 16;
  p.part_heads = part_heads_of(L.s.group);
  const KvWorkspace ws(L.workspace, L.s);
  p.count = ws.attend_count;
  p.part = ws.part;
  p.part_ml = ws.part_ml;
  p.scale_log2 = L.scale * 1.4426950408889634f;
  const size_t row_bytes = size_t(L.s.head_dim) * (L.s.cache == RWTTT_F32 ? 4 : L.s.cache == RWTTT_BF16 ? 2 : 1) * 2;
  p.stream = attend_streams(L.s.n_pages, L.n, L.s.max_pages, L.keep, L.window, uint64_t(1) << L.s.page_shift,
                            (row_bytes << L.s.page_shift) * L.s.kv_heads, L.n_layers);
  if (L.s.io_bf16) return L.s.cache == RWTTT_BF16 ? attend_dims<1, RWTTT_BF16>(p, stream)
                                                  : attend_dims<1, RWTTT_FP8>(p, stream);
  return L.s.cache == RWTTT_F32    ? attend_dims<0, RWTTT_F32>(p, stream)
         : L.s.cache == RWTTT_BF16 ? attend_dims<0, RWTTT_BF16>(p, stream)
                                   : attend_dims<0, RWTTT_FP8>(p, stream);
}

}  // namespace rwttt
