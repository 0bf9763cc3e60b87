// Attention over a cache of 4 bits: one wave's tiles of one row (an owner, kv head
// and up to sixteen queries).  Included by rwttt_kv.hip.
//
// A tile's rows come in sixteens, each within one page, so that an address is a
// page's buffer, a scalar offset and a lane's own constant one.  The ids of 64 pages at
// a time lie in the lanes of a register and are read from there, with no load between
// one tile and the next.
//
// S^T = K Q^T: codes times their block's power are exact in bf16 (one conversion
// for two), and a lane's 4 scores of each sixteen are 4 consecutive rows.  Two
// sixteens make the 32 rows of an O^T = V^T P^T; its V operand takes two conversions
// and two byte permutations for four values, since a conversion has one power and two
// rows have two.  (The scaled matrix instructions take codes and powers as they lie, but
// add a block's products to 13 bits only: 1e-4 of the products' magnitudes.)
//
// A probability enters as three bf16 terms, its 24 bits cut in eights.  The product
// has sixteen columns and a group seldom so many queries: where they are five or fewer,
// the terms are columns of one product (column c: term c / heads of query c % heads)
// and are added at the row's end; up to eight take two products.  The sum of the
// probabilities is a product with ones.
//
// Bound by HBM for long rows, with the vector units half busy: 32 owners of 12000 to
// 20000 rows, eight kv heads of four queries and 128 channels (540 MB) take 95 to 105 us,
// 5.1 to 5.7 TB/s, by how much of them the last-level cache still holds; the loads alone 88.
// (Two terms of a probability, 16 bits, would take 2% less, 2 to 4% at 256 channels, 2 to 5%
// at 64.)
// Of the steps: scores and values on one tile of
// registers, page ids by scalar loads, probabilities split by rounding 111 us; ids from
// lanes, cut probabilities, the scale within the exponent's product 103; the next tile's
// loads in registers of their own 97.
#pragma once

// How many terms of a group's probabilities one product takes.
constexpr int terms4(int group) { return group <= 5 ? 3 : group <= 8 ? 2 : 1; }

// Pieces of 32 channels of a key (16 where a row has no more than 64) and the D / 16
// channels of a value that a lane holds lie in one block each.
template <int D> struct TileShape4 {
  static constexpr int KT = tile_rows(RWTTT_FP4, D), NT = KT / 16;
  static constexpr int KE = D == 64 ? 16 : 32, KW = D / (4 * KE), PER = KE / 8;
  static constexpr int VE = D / 16, NE = 1, VW = VE <= 8 ? 1 : VE / 8;
  static constexpr int NA = D / 16;
  __device__ static int value_channel(int, int c) { return c * VE; }
};

struct Rows4 {
  const int32_t *table, *list;           // list: null without a selection
  const void *k, *v;
  int h, base, held, len, least, last_page;
  int t0, t1;                            // the wave's tiles
};

template <int IO, int D, bool HINT, int TG>
__device__ __forceinline__ void attend_rows4(const KvAttendLaunch& p, const Rows4& r, float scale_log2, int owner,
                                             int head0, int heads, float& m, float& l, f32x4_t* acc) {
  using S = TileShape4<D>;
  constexpr int NT = S::NT, NQ = IO ? 1 : 3, QN = D / 32, NP = 4 - TG;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int shift = p.s.page_shift, P = 1 << shift;
  if (r.t0 >= r.t1) return;

  // pages [first, first + 64) of the row, one a lane: id and, of a selection, position
  int first = 0;
  uint32_t ids = 0;
  int places = 0;
  auto look = [&](int from) {
    first = from;
    int lp = from + lane;
    if (r.list) {
      lp = lp < r.held ? r.list[lp] : -1;
      places = unsigned(lp) <= unsigned(r.last_page) ? lp : -1;
    }
    ids = min(uint32_t(r.table[clampi(lp, 0, r.last_page)]), uint32_t(p.s.n_pages - 1));
  };
  look((r.base + r.t0 * S::KT) >> shift);

  const uint32_t chunk = uint32_t(fp4_chunk(P, D)), page_bytes = chunk * p.s.kv_heads;   // below 2^25
  struct At {
    size_t at[NT];                       // the sixteen's page and head in the cache
    int off[NT], pos[NT];                // row in the page; position, of a page that is not held beyond all
  };
  struct Tile {
    uint32_t kw[NT][S::KW][4], kp[NT][S::KW];
    uint32_t vw[NT][4][S::VW], vp[NT];   // rows 4 g + i of each sixteen; their powers
    int pos[NT];
  };
  constexpr int kNone = 0x40000000;
  auto locate = [&](int t) {
    At x;
    const int row0 = r.base + t * S::KT;
    if ((row0 >> shift) - first > 63 - (S::KT / 16 - 1)) look(row0 >> shift);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int row = row0 + j * 16, i = (row >> shift) - first;
      x.off[j] = row & (P - 1);
      x.at[j] = size_t(uint32_t(__builtin_amdgcn_readlane(int(ids), i))) * page_bytes + r.h * chunk;
      x.pos[j] = row;
      if (r.list) {
        const int lp = __builtin_amdgcn_readlane(places, i);
        x.pos[j] = lp < 0 ? kNone : (lp << shift) + x.off[j];
      }
    }
    return x;
  };

  // queries, negated if the scale is negative: column c is query c % heads of the tile's, as long
  // as terms are left.  A scale of zero makes them 0, or NaN where they are not finite, so that
  // all scores of the rows that count are alike, and -inf stays that of the others.
  const bool used = c < heads * TG;
  const int column = used ? c % heads : 0, term = c / heads;
  const float sign = scale_log2 == 0.f ? 0.f : scale_log2 < 0.f ? -1.f : 1.f;
  const uint32_t flip = scale_log2 < 0.f ? 0x80008000u : 0u;
  const float to_log2 = scale_log2 == 0.f ? 1.f : fabsf(scale_log2);
  bf16x8_t q[NQ][QN];
#pragma unroll
  for (int s = 0; s < QN; ++s) {
    const int ch = (s / S::PER * 4 + g) * S::KE + s % S::PER * 8;
    const char* src = static_cast<const char*>(p.q) +
                      (size_t(owner) * p.q_stride + (size_t(r.h) * p.s.group + head0 + column) * D + ch) * (IO ? 2 : 4);
    uint32_t w[IO ? 4 : 8];
#pragma unroll
    for (int j = 0; j < (IO ? 4 : 8); j += 4) load_words<4>(src + j * 4, w + j);
    if constexpr (IO) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = used ? w[j] ^ flip : 0u;
      q[0][s] = as_bf16x8(w);
    } else {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = used ? __uint_as_float(w[j]) * sign : 0.f;
      bf16x8_t terms[NQ];
      cut_bf16<NQ, false>(f, terms);
#pragma unroll
      for (int k = 0; k < NQ; ++k) q[k][s] = terms[k];
    }
  }
  if (IO && scale_log2 == 0.f) {         // apart, so that other scales pay for a branch alone
#pragma unroll
    for (int s = 0; s < QN; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[0][s][i] = q[0][s][i] * static_cast<__bf16>(0.f);
  }

  const int k_lane = c * (D / 2) + g * (S::KE / 2), kp_lane = P * (D / 2) + g * S::KE / RWTTT_KV_BLOCK * P + c;
  const int v_lane = 4 * g * (D / 2) + c * (S::VE / 2), vp_lane = P * (D / 2) + c * S::VE / RWTTT_KV_BLOCK * P + 4 * g;
  auto buffer = [&](const void* cache, size_t at) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(cache) + at), 0, int(chunk), 0x27000);
  };
  // The hint is for the keys alone: a line holds two rows, and each load of values takes a
  // half of it (32 owners of 12000-20000 rows: 88 us of loads alone, 96 with the hint on both).
  constexpr int kHint = HINT ? 2 : 0;
  auto load = [&](Tile& y, int t) {
    const At x = locate(t);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const __amdgpu_buffer_rsrc_t b = buffer(r.k, x.at[j]);
      y.pos[j] = x.pos[j];
#pragma unroll
      for (int s = 0; s < S::KW; ++s) {
        if constexpr (S::KE == 32) {
          const u32x4_t w = __builtin_amdgcn_raw_buffer_load_b128(b, k_lane + s * (2 * S::KE), x.off[j] * (D / 2), kHint);
#pragma unroll
          for (int i = 0; i < 4; ++i) y.kw[j][s][i] = w[i];
        } else {
          const u32x2_t w = __builtin_amdgcn_raw_buffer_load_b64(b, k_lane, x.off[j] * (D / 2), kHint);
          y.kw[j][s][0] = w[0], y.kw[j][s][1] = w[1];
        }
        y.kp[j][s] = __builtin_amdgcn_raw_buffer_load_b8(b, kp_lane + s * 4 * P, x.off[j], 0);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const __amdgpu_buffer_rsrc_t b = buffer(r.v, x.at[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int to = v_lane + i * (D / 2), off = x.off[j] * (D / 2);
        if constexpr (D == 64) {
          y.vw[j][i][0] = __builtin_amdgcn_raw_buffer_load_b16(b, to, off, 0);
        } else if constexpr (D == 128) {
          y.vw[j][i][0] = __builtin_amdgcn_raw_buffer_load_b32(b, to, off, 0);
        } else {
          const u32x2_t w = __builtin_amdgcn_raw_buffer_load_b64(b, to, off, 0);
          y.vw[j][i][0] = w[0], y.vw[j][i][1] = w[1];
        }
      }
      y.vp[j] = __builtin_amdgcn_raw_buffer_load_b32(b, vp_lane, x.off[j], 0);
    }
  };

  // what a lane's column takes of a probability: all, less its first 8 bits, or its first 16
  const uint32_t cut1 = term >= 1 ? 0xffff0000u : 0u, cut2 = term >= 2 ? 0xffff0000u : 0u;
  const uint32_t one[4] = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};    // of the column's probabilities, in each element
  auto take = [&](Tile& x) {
    f32x4_t sc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) sc[j] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int a = 0; a < QN; ++a)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        uint32_t wd[4];
        fp4_octet(x.kw[j][a / S::PER][a % S::PER], fp4_unit(x.kp[j][a / S::PER]), wd);
        const bf16x8_t key = as_bf16x8(wd);
#pragma unroll
        for (int b = NQ - 1; b >= 0; --b) sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[b][a], sc[j], 0, 0, 0);
      }

    bool whole = true;
#pragma unroll
    for (int j = 0; j < NT; ++j) whole = whole && x.pos[j] >= r.least && x.pos[j] + 16 <= r.len;
    if (!whole) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = x.pos[j] + 4 * g + i;
          const bool on = pos >= r.least && pos < r.len;
          sc[j][i] = on ? sc[j][i] : -INFINITY;
          // what lies behind an owner's rows may be anything, and its power the NaN's
#pragma unroll
          for (int b = 0; b < S::VW; ++b) x.vw[j][i][b] = on ? x.vw[j][i][b] : 0u;
          if (!on) x.vp[j] = (x.vp[j] & ~(0xffu << (8 * i))) | 127u << (8 * i);
        }
    }
    float top = sc[0][0];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[j][i]);
    top *= to_log2;
    if (__any(top > m)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float up = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - up);
      m = up;
      sum *= f;
#pragma unroll
      for (int a = 0; a < S::NA; ++a) acc[a] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : -m;

#pragma unroll
    for (int u = 0; u < NT; u += 2) {    // 32 rows: operands of one product
      uint32_t pt[NP][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) y[k] = __builtin_amdgcn_exp2f(fmaf(sc[u + i / 2][i % 2 * 2 + k], to_log2, ref));
        // cut: what is left, less its first 8 bits where the mask says so
        auto less = [](float z, uint32_t mask) { return z - __uint_as_float(__float_as_uint(z) & mask); };
        auto pack = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
        if constexpr (TG == 3) {
          pt[0][i] = pack(less(less(y[0], cut1), cut2), less(less(y[1], cut1), cut2));
        } else if constexpr (TG == 2) {
          const float a = less(y[0], 0xffff0000u), b = less(y[1], 0xffff0000u);
          pt[0][i] = term == 0 ? pack(y[0], y[1]) : pack(a, b);
          pt[1][i] = term == 0 ? pack(less(a, 0xffff0000u), less(b, 0xffff0000u)) : 0u;
        } else {
          float a = y[0], b = y[1];
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            pt[k][i] = pack(a, b);
            a = less(a, 0xffff0000u), b = less(b, 0xffff0000u);
          }
        }
      }
#pragma unroll
      for (int b = NP - 1; b >= 0; --b)
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(one), as_bf16x8(pt[b]), sum, 0, 0, 0);
      // two rows' pairs of channels, then two channels' pairs of rows
#pragma unroll
      for (int a = 0; a < S::VE; a += 2) {
        uint32_t even[4], odd[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = u + i / 2, k = i % 2 * 2;
          const uint32_t lo = fp4_pair_at(x.vw[j][k][a / 8], fp4_unit_of(x.vp[j], k), a / 2 % 4);
          const uint32_t hi = fp4_pair_at(x.vw[j][k + 1][a / 8], fp4_unit_of(x.vp[j], k + 1), a / 2 % 4);
          even[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
          odd[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        }
        const bf16x8_t v0 = as_bf16x8(even), v1 = as_bf16x8(odd);
#pragma unroll
        for (int b = NP - 1; b >= 0; --b) {
          acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(pt[b]), acc[a], 0, 0, 0);
          acc[a + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(pt[b]), acc[a + 1], 0, 0, 0);
        }
      }
    }
  };
  // the next tile's loads are under way while one is taken, in registers of their own
  Tile one_tile, other;
  int t = r.t0;
  load(one_tile, t);
  for (; t + 2 < r.t1; t += 2) {
    load(other, t + 1);
    take(one_tile);
    load(one_tile, t + 2);
    take(other);
  }
  if (t + 1 < r.t1) {
    load(other, t + 1);
    take(one_tile);
    one_tile = other;                    // a fourth copy of take() spills
  }
  take(one_tile);
  l = sum[0];
}
