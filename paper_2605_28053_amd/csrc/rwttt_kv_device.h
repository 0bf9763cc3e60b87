// Device-side forms of the paged cache's stored rows, shared by its kernel files.
// Included inside namespace rwttt { namespace { ... } } of each file, behind
// rwttt_device.h.
#pragma once

__device__ __forceinline__ uint32_t fp8_pair(uint32_t w, bool high) {   // exact: e4m3 fits bf16
  const bf16x2_t h = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true)
                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---------------------------------------------------------------------------
// Blocks of 4-bit codes
// ---------------------------------------------------------------------------

// Bytes of a page and head: the rows' codes, then [blocks][rows] powers.
__device__ __forceinline__ constexpr size_t fp4_chunk(int page_rows, int dim) {
  return size_t(page_rows) * (dim / 2 + dim / RWTTT_KV_BLOCK);
}
// Where the power of block b of a row is in its chunk.
__device__ __forceinline__ constexpr size_t fp4_power(int page_rows, int dim, int b, int row) {
  return size_t(page_rows) * (dim / 2) + size_t(b) * page_rows + row;
}

// 2^(e - 127) for a byte e: exponent 255 makes the conversions below NaN.
__device__ __forceinline__ float fp4_unit(uint32_t e) { return __uint_as_float(e << 23); }

// The unit of byte i of four.  Their neighbours' bits stay in the sign and the
// mantissa, which the conversions do not read.
__device__ __forceinline__ float fp4_unit_of(uint32_t four, int i) {
  return __uint_as_float(i < 3 ? four << (23 - 8 * i) : four >> 1);
}

// Codes 2 b and 2 b + 1 of a word as bf16, times the unit: exact.
template <int B> __device__ __forceinline__ uint32_t fp4_pair(uint32_t w, float unit) {
  const bf16x2_t h = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, B);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The same where b is a constant only once its loop is unrolled.
__device__ __forceinline__ uint32_t fp4_pair_at(uint32_t w, float unit, int b) {
  return b == 0 ? fp4_pair<0>(w, unit) : b == 1 ? fp4_pair<1>(w, unit) : b == 2 ? fp4_pair<2>(w, unit) : fp4_pair<3>(w, unit);
}
template <int B> __device__ __forceinline__ f32x2_t fp4_floats(uint32_t w, float unit) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, B);
}
// Eight codes as bf16.
__device__ __forceinline__ void fp4_octet(uint32_t w, float unit, uint32_t* out) {
  out[0] = fp4_pair<0>(w, unit);
  out[1] = fp4_pair<1>(w, unit);
  out[2] = fp4_pair<2>(w, unit);
  out[3] = fp4_pair<3>(w, unit);
}

// The byte E of a block whose largest magnitude has these fp32 bits (a NaN's are
// above infinity's): half a step of the mantissa's first two bits reaches the
// exponent from 1.75 on, where 6 times the smaller power would be as far off as 4
// times the larger.  The limits keep every value of the grid a normal number.
__device__ __forceinline__ uint32_t fp4_exponent(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  const int e = int((top + 0x200000u) >> 23) - 2;
  return uint32_t(min(max(e, 2), 252));
}

// ---------------------------------------------------------------------------
// 16 bytes of io from a stored row
// ---------------------------------------------------------------------------

template <int IO, int CT, int D> struct CachedRow {
  static constexpr int E = IO ? 8 : 4;                       // channels
  static constexpr int B = CT == RWTTT_F32 ? 32 : CT == RWTTT_BF16 ? 16 : CT == RWTTT_FP8 ? 8 : 4;   // bits of one
  static constexpr int W = E * B >= 32 ? E * B / 32 : 1;
  uint32_t w[W], power;
  // Piece `piece` of `row` of chunk (page * heads + head).
  __device__ __forceinline__ void load(const char* cache, size_t chunk, int page_rows, int row, int piece) {
    if constexpr (CT == RWTTT_FP4) {
      const char* at = cache + chunk * fp4_chunk(page_rows, D);
      const char* src = at + row * (D / 2) + piece * (E / 2);
      if constexpr (E == 8) w[0] = *reinterpret_cast<const uint32_t*>(src);
      else w[0] = *reinterpret_cast<const uint16_t*>(src);
      power = *reinterpret_cast<const uint8_t*>(at + fp4_power(page_rows, D, piece * E / RWTTT_KV_BLOCK, row));
    } else {
      const char* src = cache + (chunk * page_rows + row) * size_t(D * B / 8) + piece * (E * B / 8);
      if constexpr (W == 1) {
        w[0] = *reinterpret_cast<const uint32_t*>(src);
      } else if constexpr (W == 2) {
        const u32x2_t t = *reinterpret_cast<const u32x2_t*>(src);
        w[0] = t[0], w[1] = t[1];
      } else {
        const u32x4_t t = *reinterpret_cast<const u32x4_t*>(src);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = t[i];
      }
    }
  }
  // Rounded once to the io type; scale is an 8-bit cache's.
  template <bool HINT> __device__ __forceinline__ void store(char* dst, float scale) const {
    uint32_t o[4];
    if constexpr (CT == RWTTT_FP4) {
      const float unit = fp4_unit(power);
      if constexpr (IO) {
        fp4_octet(w[0], unit, o);
      } else {
        const f32x2_t a = fp4_floats<0>(w[0], unit), b = fp4_floats<1>(w[0], unit);
        o[0] = __float_as_uint(a[0]), o[1] = __float_as_uint(a[1]);
        o[2] = __float_as_uint(b[0]), o[3] = __float_as_uint(b[1]);
      }
    } else if constexpr (CT == RWTTT_FP8) {
      float f[E];
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const uint32_t pair = i & 2 ? fp8_pair(w[i / 4], true) : fp8_pair(w[i / 4], false);
        f[i] = bf16_lo(pair) * scale;
        f[i + 1] = bf16_hi(pair) * scale;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = IO ? bf16x2_rne(f[2 * i % E], f[(2 * i + 1) % E]) : __float_as_uint(f[i]);
    } else if constexpr (CT == RWTTT_BF16 && !IO) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = w[i];
    }
    const u32x4_t t = {o[0], o[1], o[2], o[3]};
    if (HINT) __builtin_nontemporal_store(t, reinterpret_cast<u32x4_t*>(dst));
    else *reinterpret_cast<u32x4_t*>(dst) = t;
  }
};
