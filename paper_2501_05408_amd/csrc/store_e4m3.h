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

// Two bf16 values (low and high half of a word) as codes, in bits 0..15; `most`: largest_code().
__device__ inline uint32_t codes_of(uint32_t pair, float inverse, float most) {
  const uint32_t lo = pair << 16, hi = pair & 0xFFFF0000u;
  const float x = __builtin_amdgcn_fmed3f(__builtin_bit_cast(float, lo) * inverse, -most, most);
  const float y = __builtin_amdgcn_fmed3f(__builtin_bit_cast(float, hi) * inverse, -most, most);
  const float a = (lo & 0x7F800000u) == 0x7F800000u ? NAN : x, b = (hi & 0x7F800000u) == 0x7F800000u ? NAN : y;
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
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
template <int D>
__device__ inline RowPiece quantise_piece(u32x4 x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = top_of(x[i], top);
#pragma unroll
  for (int m = D / 16; m > 0; m >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, m);
    top = o > top ? o : top;
  }
  RowPiece r;
  r.scale = (uint32_t)scale_byte(top);
  const float inverse = inverse_scale_of(r.scale), most = largest_code(r.scale);
  r.lo = codes_of(x.x, inverse, most) | (codes_of(x.y, inverse, most) << 16);
  r.hi = codes_of(x.z, inverse, most) | (codes_of(x.w, inverse, most) << 16);
  return r;
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
