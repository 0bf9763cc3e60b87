// Kernels of the operators on rows (include/rwttt_kv_rows.h) for gfx950: rotary
// positions, and stored rows read back.

#include "rwttt_kv_kernels.h"

#include <type_traits>

namespace rwttt {
namespace {

#include "rwttt_device.h"
#include "rwttt_kv_device.h"

// ---------------------------------------------------------------------------
// rotate: rotary positions
// ---------------------------------------------------------------------------
//
// An angle in turns is position * frequency, both whole numbers (the frequency
// times 2^64), so the product modulo 2^64 is the exact place within a turn, at
// position 1 as at 2^31; taken as a signed number, its conversion keeps the bits
// of small angles as well.  What fp32 drops of an angle is added to its sine and cosine,
// to first order (below 2^-24 of a turn, so the second is below 2^-44).
//
// A block takes some tokens, computes their sines and cosines once into LDS --
// heads share them -- and passes over its part of the rows.  A lane owns whole
// pairs, so a row may be turned in place: with HALF 16 bytes of each partner, with
// INTERLEAVED 16 bytes.  Where a half of the turning channels is no whole number of
// 16 bytes, the partners and the channels behind them are loaded and stored as they lie,
// aligned to their type, and the pairs that are left over one by one.
//
// Bound by the bytes for a prefill: 8192 tokens of 32 + 8 heads of 128 channels in bf16
// (168 MB in and out) take 33 us, 5.1 TB/s, the rate of a copy, and 27 us where the last-level
// cache still holds some of them; 4096 tokens of 100 turning channels (84 MB) 30 us, 44 with
// a lane a pair; a decode step of eight tokens 3.1 us.

constexpr int kRotThreads = 256;

typedef u32x4_t Loose __attribute__((aligned(2)));

template <int IO> struct IoRow {           // 16 bytes of io
  static constexpr int E = IO ? 8 : 4;
  uint32_t w[4];
  __device__ __forceinline__ void load(const char* p) {
    const u32x4_t t = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = t[i];
  }
  // anywhere that an element may be
  __device__ __forceinline__ void load_loose(const char* p) {
    const u32x4_t t = *reinterpret_cast<const Loose*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = t[i];
  }
  template <bool HINT> __device__ __forceinline__ void store_loose(char* p) const {
    const u32x4_t t = {w[0], w[1], w[2], w[3]};
    if (HINT) __builtin_nontemporal_store(t, reinterpret_cast<Loose*>(p));
    else *reinterpret_cast<Loose*>(p) = t;
  }
  template <bool HINT> __device__ __forceinline__ void store(char* p) const {
    const u32x4_t t = {w[0], w[1], w[2], w[3]};
    if (HINT) __builtin_nontemporal_store(t, reinterpret_cast<u32x4_t*>(p));
    else *reinterpret_cast<u32x4_t*>(p) = t;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (IO) return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    else return __uint_as_float(w[i]);
  }
  __device__ __forceinline__ void put_pair(int i, float a, float b) {   // elements 2 i, 2 i + 1
    if constexpr (IO) w[i] = bf16x2_rne(a, b);
    else {
      w[2 * i] = __float_as_uint(a);
      w[2 * i + 1] = __float_as_uint(b);
    }
  }
};

// Division by a number known to the host: floor(2^32 / by) gives the quotient or one less.
struct Divider {
  uint32_t by, magic;
  __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t& rest) const {
    uint32_t q = __umulhi(x, magic);
    rest = x - q * by;
    if (rest >= by) {
      ++q;
      rest -= by;
    }
    return q;
  }
};
Divider divider(uint32_t by) { return {by, uint32_t((uint64_t(1) << 32) / by - (by == 1))}; }

struct RotateParams {
  KvRotateLaunch L;
  int tokens;              // of a block
  Divider units;           // of a head: what one lane takes at a time
  int per_token, part;     // units of a token, of a block's part of them
  Divider whole;           // per_token
};

// How the units of a head are laid out.
enum class Turn { half, interleaved, ragged };   // ragged: HALF of any width

// a b + c d, of fp32 io with one product's rounding taken back, so that the sum's remains.
template <int IO> __device__ __forceinline__ float two_products(float a, float b, float c, float d) {
  const float p = c * d, sum = fmaf(a, b, p);
  if constexpr (IO) return sum;
  return __builtin_isfinite(p) ? sum + fmaf(c, d, -p) : sum;
}
template <int IO> __device__ __forceinline__ float2 turned(float2 x, float2 cs) {
  return make_float2(two_products<IO>(x.x, cs.x, -x.y, cs.y), two_products<IO>(x.y, cs.x, x.x, cs.y));
}

template <int IO, Turn T, int U>
__global__ void __launch_bounds__(kRotThreads) kv_rotate_kernel(const RotateParams rp) {
  const KvRotateLaunch& p = rp.L;
  constexpr int B = IO ? 2 : 4, E = IoRow<IO>::E;
  constexpr bool HINT = U > 1;
  using M = Elem<std::conditional_t<IO, uint16_t, float>>;
  extern __shared__ float2 cs[];         // [tokens][turning / 2]: gain cos, gain sin
  const int half = p.turning / 2, n = int(p.n);
  // ragged: units of pieces of pairs, of single pairs, of pieces behind them, of single channels
  const int pieces = half / E, singles = pieces + half % E, behind = singles + (p.head_dim - p.turning) / E;
  const int t0 = blockIdx.x * rp.tokens, nt = min(rp.tokens, n - t0);
  const int u0 = blockIdx.y * rp.part, span = min(rp.per_token, u0 + rp.part) - u0, total = nt * span;

  for (int i = threadIdx.x; i < nt * half; i += kRotThreads) {
    const int pos = p.positions[t0 + i / half];
    const int64_t place = int64_t(uint64_t(uint32_t(pos)) * p.turns[i % half]);
    const double turn = double(place) * 0x1p-63;                // in half turns, [-1, 1]
    const float near = float(turn), rest = float(turn - double(near)) * 3.14159265f;
    float s, c;
    sincospif(near, &s, &c);
    const float sin = fmaf(c, rest, s), cos = fmaf(-s, rest, c);
    cs[i] = make_float2(cos * p.gain, (p.inverse ? -sin : sin) * p.gain);
  }
  bool waited = false;
  for (int i0 = threadIdx.x; i0 < total || !waited; i0 += U * kRotThreads) {
    // U units, their loads in flight together
    struct Unit {
      char* dst;
      const float2* at;
      int x;                             // -1: none
      int kind;                          // of a ragged one
      IoRow<IO> a, b;
      float2 pair;
    } un[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      Unit& w = un[j];
      const int i = i0 + j * kRotThreads;
      w.x = -1;
      w.kind = 0;
      if (i >= total) continue;
      uint32_t u = i, x;                 // of one token a part of its units, of several all
      const int t = rp.tokens > 1 ? int(rp.whole(i, u)) : 0;
      if (p.positions[t0 + t] < 0) continue;
      int h = int(rp.units(u0 + u, x));
      w.x = int(x);
      const bool is_k = h >= p.q.heads;
      const KvTurnRows& rows = is_k ? p.k : p.q;
      h -= is_k ? p.q.heads : 0;
      const char* src = static_cast<const char*>(rows.in) + ((t0 + t) * rows.in_stride + size_t(h) * p.head_dim) * B;
      w.dst = static_cast<char*>(rows.out) + ((t0 + t) * rows.out_stride + size_t(h) * p.head_dim) * B;
      w.at = cs + t * half;
      if constexpr (T == Turn::half) {
        w.a.load(src + (w.x < pieces ? w.x : w.x + pieces) * 16);
        if (w.x < pieces) w.b.load(src + half * B + w.x * 16);
      } else if constexpr (T == Turn::interleaved) {
        w.a.load(src + w.x * 16);
      } else if (w.x < pieces) {
        w.a.load(src + w.x * 16);
        w.b.load_loose(src + half * B + w.x * 16);
      } else if (w.x < singles) {
        w.x = pieces * E + (w.x - pieces);             // the pair's first channel
        w.kind = 1;
        w.pair = make_float2(M::get(src, w.x), M::get(src, w.x + half));
      } else if (w.x < behind) {
        w.x = p.turning + (w.x - singles) * E;         // the first channel
        w.kind = 2;
        w.a.load_loose(src + w.x * B);
      } else {
        w.x = p.turning + (behind - singles) * E + (w.x - behind);
        w.kind = 3;
        w.pair.x = M::get(src, w.x);
      }
    }
    if (!waited) __syncthreads();
    waited = true;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      Unit& w = un[j];
      if (w.x < 0) continue;
      auto turn_pieces = [&](IoRow<IO>& ra, IoRow<IO>& rb) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 y0 = turned<IO>(make_float2(w.a.get(e), w.b.get(e)), w.at[w.x * E + e]);
          const float2 y1 = turned<IO>(make_float2(w.a.get(e + 1), w.b.get(e + 1)), w.at[w.x * E + e + 1]);
          ra.put_pair(e / 2, y0.x, y1.x);
          rb.put_pair(e / 2, y0.y, y1.y);
        }
      };
      if constexpr (T == Turn::half) {
        if (w.x < pieces) {
          IoRow<IO> ra, rb;
          turn_pieces(ra, rb);
          ra.template store<HINT>(w.dst + w.x * 16);
          rb.template store<HINT>(w.dst + half * B + w.x * 16);
        } else {
          w.a.template store<HINT>(w.dst + (w.x + pieces) * 16);
        }
      } else if constexpr (T == Turn::interleaved) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const int k = w.x * (E / 2) + e;
          if (k < half) {
            const float2 y = turned<IO>(make_float2(w.a.get(2 * e), w.a.get(2 * e + 1)), w.at[k]);
            w.a.put_pair(e, y.x, y.y);
          }
        }
        w.a.template store<HINT>(w.dst + w.x * 16);
      } else if (w.kind == 0) {
        IoRow<IO> ra, rb;
        turn_pieces(ra, rb);
        ra.template store<HINT>(w.dst + w.x * 16);
        rb.template store_loose<HINT>(w.dst + half * B + w.x * 16);
      } else if (w.kind == 1) {
        const float2 y = turned<IO>(w.pair, w.at[w.x]);
        M::put(w.dst, w.x, y.x);
        M::put(w.dst, w.x + half, y.y);
      } else if (w.kind == 2) {
        w.a.template store_loose<HINT>(w.dst + w.x * B);
      } else {
        M::put(w.dst, w.x, w.pair.x);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// gather: stored rows read back
// ---------------------------------------------------------------------------
//
// A wave takes one kv head of a run of rows: LPR lanes hold a row, 16 bytes of
// output each, and the loads of its keys and values are in flight at once behind
// the chain owner -> length and page.  A block's waves take runs behind one another, since
// the powers of a page's rows share lines (with the waves on four heads of the same rows
// 73 MB are fetched instead of 54).  Bound by the bytes, of which the output is the most:
// 48700 rows of eight heads of 128 channels from 4 bits to bf16 (253 MB) take 40 us, 6.2
// TB/s, with non-temporal stores, 75 without; 500 rows 3.3 us.

struct GatherParams {
  KvGatherLaunch L;
  int run;               // rows a wave takes
};

template <int IO, int CT, int D, int NI>
__global__ void __launch_bounds__(256) kv_gather_kernel(const GatherParams gp) {
  const KvGatherLaunch& p = gp.L;
  using Row = CachedRow<IO, CT, D>;
  constexpr int IOB = IO ? 2 : 4, E = Row::E, LPR = D / E, RPI = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int H = p.s.kv_heads, shift = p.s.page_shift, P = 1 << shift;
  const int h = blockIdx.x % H, n = int(p.n), t0 = (blockIdx.x / H * 4 + wave) * gp.run, t1 = min(n, t0 + gp.run);
  if (t0 >= n) return;
  const int sub = lane / LPR, piece = lane % LPR, most = p.s.max_pages << shift;

  int page[NI], row[NI];                 // page -1: skipped
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int t = t0 + j * RPI + sub, at = min(t, t1 - 1);
    const int owner = p.owners[at], pos = p.positions[at];
    const bool there = t < t1 && unsigned(owner) < unsigned(p.s.n_owners);
    const int r = there ? owner : 0;
    const bool held = there && pos >= 0 && pos < min(p.lengths[r], most);
    const int entry = p.table[size_t(r) * p.s.max_pages + (held ? pos >> shift : 0)];
    page[j] = held ? int(min(uint32_t(entry), uint32_t(p.s.n_pages - 1))) : -1;
    row[j] = held ? pos & (P - 1) : 0;
  }
  Row k[NI], v[NI];
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const size_t chunk = size_t(max(page[j], 0)) * H + h;
    if (p.k_out) k[j].load(static_cast<const char*>(p.k), chunk, P, row[j], piece);
    if (p.v_out) v[j].load(static_cast<const char*>(p.v), chunk, P, row[j], piece);
  }
  const float ks = CT == RWTTT_FP8 && p.k_scale ? p.k_scale[h] : 1.f;
  const float vs = CT == RWTTT_FP8 && p.v_scale ? p.v_scale[h] : 1.f;
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const size_t t = size_t(t0 + j * RPI + sub);
    if (page[j] >= 0) {
      const size_t col = size_t(h) * D * IOB + piece * 16;
      if (p.k_out) k[j].template store<true>(static_cast<char*>(p.k_out) + t * p.k_stride * IOB + col, ks);
      if (p.v_out) v[j].template store<true>(static_cast<char*>(p.v_out) + t * p.v_stride * IOB + col, vs);
    }
  }
}

template <int IO, int CT, int D> hipError_t gather_go(GatherParams p, hipStream_t stream) {
  constexpr int RPI = 64 * (IO ? 8 : 4) / D;
  const uint64_t rows = uint64_t(p.L.n) * p.L.s.kv_heads;
  // two loads of rows a wave where that still makes eight waves a SIMD (253 MB of 128
  // channels in bf16 42.4 us, with one 43.3, with four 43.4)
  const bool many = rows >= 8192u * 2 * RPI;
  p.run = many ? 2 * RPI : RPI;
  const dim3 grid(unsigned((p.L.n + 4 * p.run - 1) / (4 * p.run) * p.L.s.kv_heads)), block(256);
  if (many) hipLaunchKernelGGL((kv_gather_kernel<IO, CT, D, 2>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((kv_gather_kernel<IO, CT, D, 1>), grid, block, 0, stream, p);
  return hipGetLastError();
}

template <int IO, int CT> hipError_t gather_dims(const GatherParams& p, hipStream_t stream) {
  return p.L.s.head_dim == 64    ? gather_go<IO, CT, 64>(p, stream)
         : p.L.s.head_dim == 128 ? gather_go<IO, CT, 128>(p, stream)
                                 : gather_go<IO, CT, 256>(p, stream);
}

template <int IO, int U> hipError_t rotate_go(const RotateParams& p, Turn how, dim3 grid, size_t lds, hipStream_t stream) {
  auto kernel = how == Turn::half          ? kv_rotate_kernel<IO, Turn::half, U>
                : how == Turn::interleaved ? kv_rotate_kernel<IO, Turn::interleaved, U>
                                           : kv_rotate_kernel<IO, Turn::ragged, U>;
  hipLaunchKernelGGL(kernel, grid, dim3(kRotThreads), lds, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_gather(const KvGatherLaunch& L, hipStream_t stream) {
  const GatherParams p{L, 1};
  if (L.s.io_bf16) return L.s.cache == RWTTT_BF16  ? gather_dims<1, RWTTT_BF16>(p, stream)
                          : L.s.cache == RWTTT_FP8 ? gather_dims<1, RWTTT_FP8>(p, stream)
                                                   : gather_dims<1, RWTTT_FP4>(p, stream);
  return L.s.cache == RWTTT_F32    ? gather_dims<0, RWTTT_F32>(p, stream)
         : L.s.cache == RWTTT_BF16 ? gather_dims<0, RWTTT_BF16>(p, stream)
         : L.s.cache == RWTTT_FP8  ? gather_dims<0, RWTTT_FP8>(p, stream)
                                   : gather_dims<0, RWTTT_FP4>(p, stream);
}

hipError_t launch_kv_rotate(const KvRotateLaunch& L, hipStream_t stream) {
  RotateParams p;
  p.L = L;
  const int E = L.io_bf16 ? 8 : 4, half = L.turning / 2;
  const Turn how = L.interleaved ? Turn::interleaved : half % E == 0 ? Turn::half : Turn::ragged;
  const bool in_place = (!L.q.heads || L.q.in == L.q.out) && (!L.k.heads || L.k.in == L.k.out);
  // in place the channels that do not turn are where they belong
  const int rest = in_place ? 0 : L.head_dim - L.turning;
  const int of_head = how == Turn::half          ? half / E + rest / E
                      : how == Turn::interleaved ? ((in_place ? L.turning : L.head_dim) + E - 1) / E
                                                 : half / E + half % E + rest / E + rest % E;
  p.units = divider(uint32_t(of_head));
  p.per_token = of_head * (L.q.heads + L.k.heads);
  p.whole = divider(uint32_t(p.per_token));
  // Few units: one a thread, so that all are under way.  Many: four a thread, and the
  // stores with the non-temporal hint, since the chip's caches do not hold what comes out
  // (8192 tokens, 168 MB in and out: 45 us without the hint, 27 to 33 with it).
  const uint64_t units = uint64_t(L.n) * p.per_token;
  const bool many = units > 256u * 8 * kRotThreads;
  const int share = (many ? 4 : 1) * kRotThreads / p.per_token;
  p.tokens = share < 1 ? 1 : share > 16 ? 16 : share;
  if (L.n > (1u << 23) && p.tokens < 2) p.tokens = 2;          // a launch's threads stay below 2^32
  p.part = p.per_token > 1024 * kRotThreads ? (p.per_token + 1023) / 1024 : many ? p.per_token : kRotThreads;
  if (p.tokens > 1) p.part = p.per_token;
  const unsigned blocks = (L.n + p.tokens - 1) / p.tokens, parts = unsigned((p.per_token + p.part - 1) / p.part);
  const dim3 grid(blocks, parts);
  const size_t lds = size_t(p.tokens) * half * sizeof(float2);
  if (many) return L.io_bf16 ? rotate_go<1, 4>(p, how, grid, lds, stream) : rotate_go<0, 4>(p, how, grid, lds, stream);
  return L.io_bf16 ? rotate_go<1, 1>(p, how, grid, lds, stream) : rotate_go<0, 1>(p, how, grid, lds, stream);
}

}  // namespace rwttt
