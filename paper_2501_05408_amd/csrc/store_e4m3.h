// The 8-bit block store (TEMPO_E4M3): a row's scale and codes (the layout of a tile: tempo_internal.h).
//
// A row x of D values (a step's key or value of one head, in bf16) is kept as D codes of 8 bits (e4m3: 4 bits of
// exponent, 3 of mantissa, largest value 448, no infinities) and one scale byte E:
//     a = max |x_d| over the finite x_d,   e = least whole number >= -111 with a <= 448 * 2^e,   E = e + 127,
//     code_d = x_d * 2^-e rounded to the nearest e4m3 value, ties to even;   NaN where x_d is not finite.
// (With the largest e, 120, codes end at 240: 256 * 2^120 is more than bf16 holds.)
// It stands for code_d * 2^e.  The scale is a power of two, so x_d * 2^-e is exact and the code is one rounding of x_d,
// at most 2^-4 |x_d| off while |x_d| >= 2^(e-6) (below, at most 2^(e-10)); and code_d * 2^e is exact in bf16, which has
// more mantissa bits, with no subnormals: codes that are not zero are at least 2^-9, 2^-9 * 2^-111 is above 2^-126.
// A scale that makes full use of 448 would gain at most one bit at the lower end of the codes' range and none in
// their relative step, and would add a rounding to every value read.
#pragma once

#include "attn_bf16_common.h"

namespace tempo {

// Scale byte of a row whose largest finite |x| has these bf16 bits: a = 1.m * 2^(X - 127) is at most 448 = 1.75 * 2^8
// times 2^(X - 135) if m <= 0.75.
__host__ __device__ inline int scale_byte(uint32_t top) {
  const int E = (int)(top >> 7) - 8 + ((top & 0x7Fu) > 0x60u ? 1 : 0);
  return E < 16 ? 16 : E;
}

__device__ inline float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }             // 2^(E - 127)
__device__ inline float inverse_scale_of(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

__device__ inline float largest_code(uint32_t byte) { return byte == 247u ? 240.f : 448.f; }

// Two bf16 values (low and high half of a word) as codes, in bits 0..15; `most`: largest_code().  For rows that have an element
// that is not finite, or whose codes end at 240.
__device__ inline uint32_t codes_of(uint32_t pair, float inverse, float most) {
  const uint32_t lo = pair << 16, hi = pair & 0xFFFF0000u;
  const float x = __builtin_amdgcn_fmed3f(__builtin_bit_cast(float, lo) * inverse, -most, most);
  const float y = __builtin_amdgcn_fmed3f(__builtin_bit_cast(float, hi) * inverse, -most, most);
  const float a = (lo & 0x7F800000u) == 0x7F800000u ? NAN : x, b = (hi & 0x7F800000u) == 0x7F800000u ? NAN : y;
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// Four values of any other row: one instruction for two (17 instructions a value with the maximum by the way above, 4 by this
// one; 8 x 2047 rows in 8 heads of 128 written and read back 46.8 -> 45.6 us).
__device__ inline uint32_t finite_codes_of(uint32_t a, uint32_t z, float scale) {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  i16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, a), scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, z), scale, true);
  return __builtin_bit_cast(uint32_t, r);
}

// Largest |x| of 8 values, finite or not (bf16 bits).
__device__ inline uint32_t top_of_any(u32x4 x) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t pair = x[i] & 0x7FFF7FFFu;
    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, pair));
  }
  const uint32_t a = top[0], z = top[1];
  return a > z ? a : z;
}

// Larger of the finite |x| of a word's two bf16 values and `top` (bf16 bits).
__device__ inline uint32_t top_of(uint32_t pair, uint32_t top) {
  const uint32_t lo = pair & 0x7FFFu, hi = (pair >> 16) & 0x7FFFu;
  const uint32_t a = lo < 0x7F80u ? lo : 0u, b = hi < 0x7F80u ? hi : 0u;
  const uint32_t m = a > b ? a : b;
  return m > top ? m : top;
}

// 8 consecutive values of a row that D/8 lanes hold side by side: their codes (two words) and the row's scale byte.
struct RowPiece {
  uint32_t lo, hi, scale;
};
// row_max: a maximum over the lanes of the row.
template <typename Max>
__device__ inline RowPiece quantise_with(u32x4 x, Max row_max) {
  uint32_t top = row_max(top_of_any(x));
  RowPiece r;
  if (top <= 0x7F60u) {  // the whole row is finite and its scale byte below 247
    r.scale = (uint32_t)scale_byte(top);
    const float scale = scale_of(r.scale);
    r.lo = finite_codes_of(x.x, x.y, scale);
    r.hi = finite_codes_of(x.z, x.w, scale);
    return r;
  }
  top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = top_of(x[i], top);
  r.scale = (uint32_t)scale_byte(row_max(top));
  const float inverse = inverse_scale_of(r.scale), most = largest_code(r.scale);
  r.lo = codes_of(x.x, inverse, most) | (codes_of(x.y, inverse, most) << 16);
  r.hi = codes_of(x.z, inverse, most) | (codes_of(x.w, inverse, most) << 16);
  return r;
}
// Maximum over the D/8 lanes, all of which or none take part, by lane moves inside a row of 16.
template <int D>
__device__ inline uint32_t row_max(uint32_t v) {
  auto step = [&](int o) { v = (uint32_t)o > v ? (uint32_t)o : v; };
  step(__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));   // lanes 1, 0, 3, 2 of four
  step(__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));   // 2, 3, 0, 1
  step(__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));  // eight lanes reversed
  if (D == 128) step(__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));  // sixteen
  return v;
}
template <int D>
__device__ inline RowPiece quantise_piece(u32x4 x) {
  return quantise_with(x, [](uint32_t v) { return row_max<D>(v); });
}

// Piece `part` of a row into a pool: `slot` of the tile (or of any run of whole groups of it) whose first slot has number
// `first` among the store's `slots`.  Codes of a key row are 8-byte pieces, of a value row single bytes.
template <int D>
__device__ inline void store_piece(uint8_t* pool, int64_t slots, int64_t first, int slot, bool value, int part, const RowPiece& r) {
  if (!value) {
    *reinterpret_cast<uint2*>(pool + first * D + tile_off_k_e4m3(D, slot, 8 * part)) = uint2{r.lo, r.hi};
  } else {
    uint8_t* const to = pool + first * D + tile_off_v_e4m3(D, slot, 8 * part);  // dims 8 part .. +7 lie 16 bytes apart
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to[16 * i] = (uint8_t)(r.lo >> (8 * i));
      to[16 * (4 + i)] = (uint8_t)(r.hi >> (8 * i));
    }
  }
  if (part == 0) pool[slots * D + first + (value ? scale_off_v(slot) : scale_off_k(slot))] = (uint8_t)r.scale;
}

}  // namespace tempo
