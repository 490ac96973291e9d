// The 8-bit block store: rows are quantised as they are written, and read back as the bf16 values that
// their codes stand for (layout and scale: store_e4m3.h).  Where a row goes is as in kv_store.hip.
#include "attn_bf16_common.h"
#include "store_e4m3.h"

namespace tempo {
namespace {

__device__ inline int rows_of(const StoreParams& p, int b) {
  if (!p.count_per_seq) return INT32_MAX;
  const int n = p.count_per_seq[b];
  return n < 0 ? 0 : n;
}

__device__ inline int step_of(const StoreParams& p, int b) {
  int t = p.t_per_seq ? p.t_per_seq[b] : p.t;
  t = t > p.t ? p.t : t;  // the host validated p.t; never index past it
  return t < 0 ? 0 : t;
}

// First slot of step t's tile in the numbering of all slots of the store, (block, kv head) by (block, kv head).
__device__ inline int64_t tile_slot(const StoreParams& p, int b, int head, int t) {
  const int tile = t >> p.z_log2;
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + (tile & p.tile_mask)], p.num_blocks);
  return ((int64_t)phys * p.Hkv + head) << p.z_log2;
}

__device__ inline int64_t all_slots(const StoreParams& p) { return ((int64_t)p.num_blocks * p.Hkv) << p.z_log2; }

// Row by row: D/8 lanes take a row of 8 values each, keys and values of a (sequence, step, head) side by side, so a
// wavefront writes 64 / (D/4) pairs of rows.  Codes of a key row are 8-byte pieces, of a value row single bytes.
template <int D>
__global__ __launch_bounds__(256) void kv_append_e4m3(StoreParams p, const uint16_t* __restrict__ k_new,
                                                      const uint16_t* __restrict__ v_new) {
  constexpr int LANES = D / 8;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t pair = idx / (2 * LANES);                       // (b, c, head), head fastest
  const bool live = pair < (int64_t)p.batch * p.count * p.Hkv;  // (whole groups of LANES lanes: the exchanges below stay inside)
  const int64_t at = live ? pair : 0;
  const bool value = (idx / LANES) & 1;
  const int part = (int)(idx % LANES), d = 8 * part;
  const int head = (int)(at % p.Hkv);
  const int c = (int)(at / p.Hkv % p.count), b = (int)(at / p.Hkv / p.count);
  const int t = step_of(p, b) + c;
  const int64_t src = (((int64_t)b * p.src_steps + c) * p.Hkv + head) * D + d;
  u32x4 x = *reinterpret_cast<const u32x4*>((value ? v_new : k_new) + src);
  if (p.rope_cos && !value) {  // dims i and i + D/2 of a key are turned together; either lane does it for its own half
    const int other_d = d < D / 2 ? d + D / 2 : d - D / 2;
    u32x4 other = *reinterpret_cast<const u32x4*>(k_new + src - d + other_d);
    if (d < D / 2) rotate_pieces(p.rope_cos, p.rope_sin, t, D / 2, d, x, other);
    else rotate_pieces(p.rope_cos, p.rope_sin, t, D / 2, other_d, other, x);
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = top_of(x[i], top);
#pragma unroll
  for (int m = LANES / 2; m > 0; m >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)top, m);
    top = o > top ? o : top;
  }
  if (!live || c >= rows_of(p, b)) return;
  const uint32_t E = (uint32_t)scale_byte(top);
  const float inverse = inverse_scale_of(E), most = largest_code(E);
  const uint32_t lo = codes_of(x.x, inverse, most) | (codes_of(x.y, inverse, most) << 16);
  const uint32_t hi = codes_of(x.z, inverse, most) | (codes_of(x.w, inverse, most) << 16);
  const int slot = t & ((1 << p.z_log2) - 1);
  const int64_t first = tile_slot(p, b, head, t), scales = all_slots(p) * D + first;
  if (!value) {
    uint8_t* const pool = static_cast<uint8_t*>(p.k_pool);
    *reinterpret_cast<uint2*>(pool + first * D + tile_off_k_e4m3(D, slot, d)) = uint2{lo, hi};
    if (part == 0) pool[scales + scale_off_k(slot)] = (uint8_t)E;
  } else {
    uint8_t* const pool = static_cast<uint8_t*>(p.v_pool);
    uint8_t* const to = pool + first * D + tile_off_v_e4m3(D, slot, d);  // dims d .. d+7 lie 16 bytes apart
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to[16 * i] = (uint8_t)(lo >> (8 * i));
      to[16 * (4 + i)] = (uint8_t)(hi >> (8 * i));
    }
    if (part == 0) pool[scales + scale_off_v(slot)] = (uint8_t)E;
  }
}

// Two codes of a word (its low or high half) as bf16 values.
__device__ inline uint32_t values_of(uint32_t codes, bool high, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, v);
}

// Read-back, element by element: out[b][j - j0][head][d].
template <int D>
__global__ __launch_bounds__(256) void kv_gather_e4m3(StoreParams p, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out,
                                                      int j0, int count) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= (int64_t)p.batch * count * p.Hkv * D) return;
  const int d = (int)(idx % D), head = (int)(idx / D % p.Hkv);
  const int j = j0 + (int)(idx / ((int64_t)D * p.Hkv) % count), b = (int)(idx / ((int64_t)D * p.Hkv * count));
  const int slot = j & ((1 << p.z_log2) - 1);
  const int64_t first = tile_slot(p, b, head, j), scales = all_slots(p) * D + first;
  const uint8_t* const kp = static_cast<const uint8_t*>(p.k_pool);
  const uint8_t* const vp = static_cast<const uint8_t*>(p.v_pool);
  if (k_out) k_out[idx] = (uint16_t)values_of(kp[first * D + tile_off_k_e4m3(D, slot, d)], false, scale_of(kp[scales + scale_off_k(slot)]));
  if (v_out) v_out[idx] = (uint16_t)values_of(vp[first * D + tile_off_v_e4m3(D, slot, d)], false, scale_of(vp[scales + scale_off_v(slot)]));
}

}  // namespace

hipError_t launch_append_e4m3(const StoreParams& p, const void* k_new, const void* v_new, int D, hipStream_t stream) {
  const uint16_t* k = static_cast<const uint16_t*>(k_new);
  const uint16_t* v = static_cast<const uint16_t*>(v_new);
  const int64_t threads = (int64_t)p.batch * p.count * p.Hkv * (D / 4);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (D == 128) return launch(kv_append_e4m3<128>, grid, dim3(256), 0, stream, p, k, v);
  return launch(kv_append_e4m3<64>, grid, dim3(256), 0, stream, p, k, v);
}

hipError_t launch_gather_e4m3(const StoreParams& p, void* k_out, void* v_out, int D, int j0, int count, hipStream_t stream) {
  const int64_t total = (int64_t)p.batch * count * p.Hkv * D;
  if (total == 0) return hipSuccess;
  const dim3 grid((unsigned)((total + 255) / 256));
  uint16_t* k = static_cast<uint16_t*>(k_out);
  uint16_t* v = static_cast<uint16_t*>(v_out);
  if (D == 128) return launch(kv_gather_e4m3<128>, grid, dim3(256), 0, stream, p, k, v, j0, count);
  return launch(kv_gather_e4m3<64>, grid, dim3(256), 0, stream, p, k, v, j0, count);
}

}  // namespace tempo
