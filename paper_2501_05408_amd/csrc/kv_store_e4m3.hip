// The 8-bit block store: rows are quantised as they are written, and read back as the bf16 values that
// their codes stand for (layout and scale: store_e4m3.h).  Where a row goes is as in kv_store.hip.
#include "attn_bf16_common.h"
#include "attn_units.h"
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
// wavefront writes 64 / (D/4) pairs of rows.
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
  const RowPiece r = quantise_piece<D>(x);
  if (!live || c >= rows_of(p, b)) return;
  uint8_t* const pool = static_cast<uint8_t*>(value ? p.v_pool : p.k_pool);
  store_piece<D>(pool, all_slots(p), tile_slot(p, b, head, t), t & ((1 << p.z_log2) - 1), value, part, r);
}

// Two codes of a word (its low or high half) as bf16 values.
__device__ inline uint32_t values_of(uint32_t codes, bool high, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, v);
}

// ---- by 32-slot groups ------------------------------------------------------------------
// One workgroup per (sequence, head, group), half of its wavefronts for the keys, half for the values.  A lane works on a block
// of 4 consecutive slots x 8 consecutive dims, D/8 lanes side by side on the same slots: 16-byte pieces of 4 rows in the
// caller's arrays, and in the store 8 codes of each key row or, of the values, 4 codes (the 4 slots) of each dim, between which
// a block is turned in registers.  The group's images pass through LDS, so that the store is read and written in whole units of
// 1 KiB, the rows in runs of D elements.
// Bound by memory: 8 x 2047 rows in 8 heads of 128 are written in 21.4 us (101 MB, 4.7 TB/s; a large copy moves 4.9) and read
// back in 15.8; by one wavefront a group 4.3 more to write, row by row and element by element 52.6 and 73.2.  What is read once
// or written for good passes the caches by: the caller's rows on the way in (27.4 us without) and on the way out (16 x 4000 rows of
// 8 heads of 64 read back 30.4 us, 198 MB, without 41.2; a sum over them right behind it loses 1.8 of 33).
// 4 words of 4 bytes, a[i] = byte i of every column: columns to rows.
__device__ inline void turn4(uint32_t* a) {
  const uint32_t t0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400), t1 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602);
  const uint32_t t2 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400), t3 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602);
  a[0] = __builtin_amdgcn_perm(t2, t0, 0x05040100);
  a[1] = __builtin_amdgcn_perm(t2, t0, 0x07060302);
  a[2] = __builtin_amdgcn_perm(t3, t1, 0x05040100);
  a[3] = __builtin_amdgcn_perm(t3, t1, 0x07060302);
}

// Offsets of a block inside a group's image: of 8 codes of key slot 4 sg + i, dims 8 part ..; of the 4 codes of dim
// 8 part + k, slots 4 sg .. +3.
template <int D>
__device__ inline int key_piece(int sg, int part, int i) {
  const int tile = sg >> 2, row = 4 * (sg & 3) + i, w = part >> 3, h = (part >> 2) & 1, c = part & 3;
  return ((tile * (D >> 6) + w) * 64 + c * 16 + row) * 16 + h * 8;
}
template <int D>
__device__ inline int value_piece(int sg, int part, int k) {
  const int d = 8 * part + k, c = sg & 3, half = sg >> 2;
  return ((d >> 5) * 64 + c * 16 + (d & 15)) * 16 + ((d >> 4) & 1) * 8 + half * 4;
}
// The image in LDS: 16 bytes more for every 256, so that the pieces that lanes touch together lie in different banks.
__host__ __device__ constexpr int in_lds(int at) { return at + (at >> 8) * 16; }

// The same pieces in the image of a bf16 group: 8 dims of key slot 4 sg + i; dim 8 part + k of slots 4 sg .. +3.
template <int D>
__device__ inline int wide_key_piece(int sg, int part, int i) {
  return (((sg >> 2) * (D >> 5) + (part >> 2)) * 64 + (part & 3) * 16 + 4 * (sg & 3) + i) * 16;
}
template <int D>
__device__ inline int wide_value_piece(int sg, int part, int k) {
  const int d = 8 * part + k;
  return ((d >> 4) * 64 + (sg & 3) * 16 + (d & 15)) * 16 + (sg >> 2) * 8;
}

// kCopy: of a prompt from step 0 on, whose rows are also put into the bf16 store u, as they are held, by the same launch (a prompt
// of 499 steps, 24/8 heads of 128, 20.5 us; by a launch of kv_unpack_e4m3 behind it 23.2).
template <int D, bool kCopy>
__global__ __launch_bounds__(2 * D) void kv_append_groups_e4m3(StoreParams p, UnpackParams u, const uint16_t* __restrict__ k_new,
                                                               const uint16_t* __restrict__ v_new) {
  constexpr int PARTS = D / 8, HALF = D;  // blocks of a group, and threads, for keys and for values
  __shared__ __align__(16) uint8_t images[2][in_lds(32 * D)];
  __shared__ __align__(16) uint8_t wides[2][kCopy ? in_lds(64 * D) : 16];
  const int tid = threadIdx.x % HALF;
  const bool value = __builtin_amdgcn_readfirstlane(threadIdx.x >= HALF);
  uint8_t* const image = images[value];
  const int g = blockIdx.x, head = blockIdx.y, b = blockIdx.z;
  if constexpr (kCopy) {
    if (g == 0 && head == 0) {
      for (int n = threadIdx.x; n < u.tiles; n += 2 * D) u.table[(int64_t)b * u.tiles + n] = b * u.tiles + n;
    }
  }
  const int rows_b = rows_of(p, b) < p.count ? rows_of(p, b) : p.count;
  const int t0 = ((p.t >> 5) + g) << 5;  // first step of this group
  const int first_row = t0 - p.t;        // source row of slot 0 (negative: before the call)
  const int lo = first_row < 0 ? -first_row : 0;
  const int hi = rows_b - first_row < 32 ? rows_b - first_row : 32;  // slots lo .. hi-1 are written
  if (hi <= lo) return;                  // uniform over the workgroup
  const bool whole = lo == 0 && hi == 32;
  const int64_t slot0 = tile_slot(p, b, head, t0) + (t0 & ((1 << p.z_log2) - 1)), scales = all_slots(p) * D + slot0;
  const int64_t row0 = ((int64_t)b * p.src_steps + first_row) * p.Hkv + head;  // (rows are Hkv apart)
  const int part = tid % PARTS, sg = tid / PARTS;
  const uint16_t* const rows = value ? v_new : k_new;
  uint8_t* const pool = static_cast<uint8_t*>(value ? p.v_pool : p.k_pool);

  // The caller's pieces; rows outside the call are read as its nearest row and not written.
  auto row_at = [&](int slot) { return row0 + (int64_t)(slot < lo ? lo : (slot < hi ? slot : hi - 1)) * p.Hkv; };
  u32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(rows + row_at(4 * sg + i) * D + 8 * part));
  if (p.rope_cos && !value) {  // a piece and its partner D/2 dims away are turned together, each lane for its own
    const int other = part < PARTS / 2 ? part + PARTS / 2 : part - PARTS / 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = 4 * sg + i, t = t0 + (slot < lo ? lo : (slot < hi ? slot : hi - 1));
      u32x4 o = *reinterpret_cast<const u32x4*>(rows + row_at(slot) * D + 8 * other);
      if (part < PARTS / 2) rotate_pieces(p.rope_cos, p.rope_sin, t, D / 2, 8 * part, x[i], o);
      else rotate_pieces(p.rope_cos, p.rope_sin, t, D / 2, 8 * other, o, x[i]);
    }
  }
  uint8_t* const wide = wides[value];
  u32x4 held[4];         // (kCopy) what the codes stand for
  uint32_t codes[2][4];  // of slot i, dims 0..3 and 4..7 of the block; values, turned: of dim k, slots 0..3
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const RowPiece r = quantise_piece<D>(x[i]);
    codes[0][i] = r.lo;
    codes[1][i] = r.hi;
    if constexpr (kCopy) {
      const float scale = scale_of(r.scale);
      held[i] = u32x4{values_of(r.lo, false, scale), values_of(r.lo, true, scale), values_of(r.hi, false, scale), values_of(r.hi, true, scale)};
      if (!value) *reinterpret_cast<u32x4*>(wide + in_lds(wide_key_piece<D>(sg, part, i))) = held[i];
    }
    const int slot = 4 * sg + i;
    if (part == 0 && slot >= lo && slot < hi) pool[scales + (value ? scale_off_v(slot) : scale_off_k(slot))] = (uint8_t)r.scale;
    if (!value) *reinterpret_cast<uint2*>(image + in_lds(key_piece<D>(sg, part, i))) = uint2{codes[0][i], codes[1][i]};
  }
  if (value && !whole) {  // this call's slots only, byte by byte: another launch may write the others at the same time
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (4 * sg + i < lo || 4 * sg + i >= hi) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) pool[slot0 * D + value_piece<D>(sg, part, e) + i] = (uint8_t)(codes[e >> 2][i] >> (8 * (e & 3)));
    }
  }
  if (value && whole) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      turn4(codes[q]);
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(image + in_lds(value_piece<D>(sg, part, 4 * q + e))) = codes[q][e];
    }
  }
  if constexpr (kCopy) {
    if (value) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
        *reinterpret_cast<uint2*>(wide + in_lds(wide_value_piece<D>(sg, part, e))) =
            uint2{__builtin_amdgcn_perm(held[1][e >> 1], held[0][e >> 1], sel), __builtin_amdgcn_perm(held[3][e >> 1], held[2][e >> 1], sel)};
      }
    }
  }
  __syncthreads();
  if constexpr (kCopy) {
    const int64_t to = ((((int64_t)b * u.tiles + (t0 >> p.z_log2)) * p.Hkv + head) << p.z_log2) + (t0 & ((1 << p.z_log2) - 1));
    uint8_t* const copy = static_cast<uint8_t*>(value ? u.v : u.k) + to * 2 * D;
#pragma unroll
    for (int i = 0; i < 64 * D / (16 * HALF); ++i) {
      const int at = (i * HALF + tid) * 16;
      *reinterpret_cast<u32x4*>(copy + at) = *reinterpret_cast<const u32x4*>(wide + in_lds(at));
    }
  }
  if (value && !whole) return;
#pragma unroll
  for (int i = 0; i < 32 * D / (16 * HALF); ++i) {
    const int at = (i * HALF + tid) * 16, slot = 16 * (at / (16 * D)) + (tid & 15);  // (a key unit's 16 bytes belong to one slot)
    if (value || (slot >= lo && slot < hi)) *reinterpret_cast<u32x4*>(pool + slot0 * D + at) = *reinterpret_cast<const u32x4*>(image + in_lds(at));
  }
}

// Read-back of steps j0 .. j0+count-1: out[b][j - j0][head][d].
template <int D>
__global__ __launch_bounds__(2 * D) void kv_gather_e4m3(StoreParams p, uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out, int j0, int count) {
  constexpr int PARTS = D / 8, HALF = D;
  __shared__ __align__(16) uint8_t images[2][in_lds(32 * D)];
  const int tid = threadIdx.x % HALF;
  const bool value = __builtin_amdgcn_readfirstlane(threadIdx.x >= HALF);
  uint8_t* const image = images[value];
  const int g = blockIdx.x, head = blockIdx.y, b = blockIdx.z;
  const int t0 = ((j0 >> 5) + g) << 5, first_row = t0 - j0;
  const int lo = first_row < 0 ? -first_row : 0, hi = count - first_row < 32 ? count - first_row : 32;
  const int64_t slot0 = tile_slot(p, b, head, t0) + (t0 & ((1 << p.z_log2) - 1)), scales = all_slots(p) * D + slot0;
  const int64_t row0 = ((int64_t)b * count + first_row) * p.Hkv + head;
  const uint8_t* const pool = static_cast<const uint8_t*>(value ? p.v_pool : p.k_pool);
  uint16_t* const out = value ? v_out : k_out;
  const int part = tid % PARTS, sg = tid / PARTS;
  uint32_t scale[4] = {};  // of the block's slots
  if (out) {
#pragma unroll
    for (int u = 0; u < 32 * D / (16 * HALF); ++u) {
      const int at = (u * HALF + tid) * 16;
      *reinterpret_cast<u32x4*>(image + in_lds(at)) = *reinterpret_cast<const u32x4*>(pool + slot0 * D + at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) scale[i] = pool[scales + (value ? scale_off_v(4 * sg + i) : scale_off_k(4 * sg + i))];
  }
  __syncthreads();
  if (!out) return;
  uint32_t codes[2][4];
  if (value) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
      for (int e = 0; e < 4; ++e) codes[q][e] = *reinterpret_cast<const uint32_t*>(image + in_lds(value_piece<D>(sg, part, 4 * q + e)));
      turn4(codes[q]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 piece = *reinterpret_cast<const uint2*>(image + in_lds(key_piece<D>(sg, part, i)));
      codes[0][i] = piece.x;
      codes[1][i] = piece.y;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * sg + i;
    if (slot < lo || slot >= hi) continue;
    const float s = scale_of(scale[i]);
    const uint32_t a = codes[0][i], z = codes[1][i];
    const u32x4 o = {values_of(a, false, s), values_of(a, true, s), values_of(z, false, s), values_of(z, true, s)};
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(out + (row0 + (int64_t)slot * p.Hkv) * D + 8 * part));
  }
}

// ---- a prompt's keys and values as a bf16 store -----------------------------------------------
// The prompt kernels are bound by the matrix cores and read each key many times, so an 8-bit store's groups are turned into
// bf16 once, into a store laid out in the caller's workspace (u.table, u.k, u.v), which they then read.  A wavefront per
// (sequence, head, group); a unit of codes is two units of bf16, lane by lane.
template <int D>
__global__ __launch_bounds__(64) void kv_unpack_e4m3(StoreParams p, UnpackParams u) {
  const int lane = threadIdx.x;
  const int grp = u.first_group + (int)blockIdx.x, head = blockIdx.y, b = blockIdx.z;
  if (blockIdx.x == 0 && head == 0) {
    for (int n = lane; n < u.tiles; n += 64) u.table[(int64_t)b * u.tiles + n] = b * u.tiles + n;
  }
  const int t0 = grp << 5, in = t0 & ((1 << p.z_log2) - 1);
  const int64_t from = tile_slot(p, b, head, t0) + in, scales = all_slots(p) * D + from;
  const int64_t to = ((((int64_t)b * u.tiles + ((t0 >> p.z_log2) & u.tile_mask)) * p.Hkv + head) << p.z_log2) + in;
  const uint8_t* const k_pool = static_cast<const uint8_t*>(p.k_pool);
  const uint8_t* const v_pool = static_cast<const uint8_t*>(p.v_pool);
  const u32x4* const kp = reinterpret_cast<const u32x4*>(k_pool + from * D) + lane;
  const u32x4* const vp = reinterpret_cast<const u32x4*>(v_pool + from * D) + lane;
  u32x4* const ko = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(u.k) + to * D) + lane;
  u32x4* const vo = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(u.v) + to * D) + lane;
  constexpr int UNITS = D / 32;
  u32x4 k[UNITS], v[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    k[i] = __builtin_nontemporal_load(kp + i * 64);
    v[i] = __builtin_nontemporal_load(vp + i * 64);
  }
  const uint32_t ks = *reinterpret_cast<const uint16_t*>(k_pool + scales + 2 * (lane & 15));
  const uint2 vs = *reinterpret_cast<const uint2*>(v_pool + scales + 8 * (lane >> 4));
  float sv[8];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    sv[r] = scale_of((vs.x >> (8 * r)) & 0xFFu);
    sv[4 + r] = scale_of((vs.y >> (8 * r)) & 0xFFu);
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const float s = scale_of(i < UNITS / 2 ? ks & 0xFFu : ks >> 8);
    ko[(2 * i) * 64] = u32x4{values_of(k[i].x, false, s), values_of(k[i].x, true, s), values_of(k[i].y, false, s), values_of(k[i].y, true, s)};
    ko[(2 * i + 1) * 64] = u32x4{values_of(k[i].z, false, s), values_of(k[i].z, true, s), values_of(k[i].w, false, s), values_of(k[i].w, true, s)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // 8 slots of one dim: exact products, exact in bf16
      float x[8];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t word = v[i][2 * h + r];
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(word, false), z = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
        x[4 * r] = a[0] * sv[4 * r]; x[4 * r + 1] = a[1] * sv[4 * r + 1];
        x[4 * r + 2] = z[0] * sv[4 * r + 2]; x[4 * r + 3] = z[1] * sv[4 * r + 3];
      }
      vo[(2 * i + h) * 64] = pack8(x);
    }
  }
}

}  // namespace

hipError_t launch_unpack_e4m3(const StoreParams& p, const UnpackParams& u, int groups, int D, hipStream_t stream) {
  const dim3 grid((unsigned)groups, (unsigned)p.Hkv, (unsigned)p.batch);
  if (D == 128) return launch(kv_unpack_e4m3<128>, grid, dim3(64), 0, stream, p, u);
  return launch(kv_unpack_e4m3<64>, grid, dim3(64), 0, stream, p, u);
}

hipError_t launch_append_copy_e4m3(const StoreParams& p, const UnpackParams& u, const void* k_new, const void* v_new, int D, hipStream_t stream) {
  const uint16_t* k = static_cast<const uint16_t*>(k_new);
  const uint16_t* v = static_cast<const uint16_t*>(v_new);
  const dim3 grid((unsigned)((p.count + 31) >> 5), (unsigned)p.Hkv, (unsigned)p.batch);
  if (D == 128) return launch((kv_append_groups_e4m3<128, true>), grid, dim3(256), 0, stream, p, u, k, v);
  return launch((kv_append_groups_e4m3<64, true>), grid, dim3(128), 0, stream, p, u, k, v);
}

hipError_t launch_append_e4m3(const StoreParams& p, const void* k_new, const void* v_new, int D, hipStream_t stream) {
  const uint16_t* k = static_cast<const uint16_t*>(k_new);
  const uint16_t* v = static_cast<const uint16_t*>(v_new);
  // Uniform first step and at least one whole 32-slot group: by groups, unless the last one lies in the first one's slots
  // (a ring whose every slot is written, from the middle of a group on), where two launches would be needed.
  const int first_whole = (p.t + 31) >> 5, past_whole = (p.t + p.count) >> 5;
  const int groups = ((p.t + p.count - 1) >> 5) - (p.t >> 5) + 1;
  const int64_t ring_slots = p.tile_mask == INT32_MAX ? INT64_MAX : ((int64_t)p.tile_mask + 1) << p.z_log2;
  if (!p.t_per_seq && past_whole > first_whole && (int64_t)groups * 32 <= ring_slots) {
    const dim3 grid(groups, p.Hkv, p.batch);
    const UnpackParams none = {};
    if (D == 128) return launch((kv_append_groups_e4m3<128, false>), grid, dim3(256), 0, stream, p, none, k, v);
    return launch((kv_append_groups_e4m3<64, false>), grid, dim3(128), 0, stream, p, none, k, v);
  }
  const int64_t threads = (int64_t)p.batch * p.count * p.Hkv * (D / 4);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (D == 128) return launch(kv_append_e4m3<128>, grid, dim3(256), 0, stream, p, k, v);
  return launch(kv_append_e4m3<64>, grid, dim3(256), 0, stream, p, k, v);
}

hipError_t launch_gather_e4m3(const StoreParams& p, void* k_out, void* v_out, int D, int j0, int count, hipStream_t stream) {
  if (count == 0) return hipSuccess;
  const dim3 grid((unsigned)((int)(((int64_t)j0 + count - 1) >> 5) - (j0 >> 5) + 1), (unsigned)p.Hkv, (unsigned)p.batch);
  uint16_t* k = static_cast<uint16_t*>(k_out);
  uint16_t* v = static_cast<uint16_t*>(v_out);
  if (D == 128) return launch(kv_gather_e4m3<128>, grid, dim3(256), 0, stream, p, k, v, j0, count);
  return launch(kv_gather_e4m3<64>, grid, dim3(128), 0, stream, p, k, v, j0, count);
}

}  // namespace tempo
