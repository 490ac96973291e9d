// Rows at positions of their own: rotation by up to four axes on the way into the block store, positions of a tree's nodes, and
// the keeping of the accepted rows of a tree.
//
// A row (a step's key or query of one head) is D/2 pairs (i, i + D/2).  Pair i belongs to an axis a(i) (time, height, width, ...)
// and is turned by the tables' entry (position of the row on that axis, i):
//     y_i = x_i cos - x_(i + D/2) sin,   y_(i + D/2) = x_(i + D/2) cos + x_i sin
// in fp32, rounded once (rope_lo(), rope_hi(): with one axis and positions t + c the bits of the other rotary calls).  The row's
// slot is that of its step, whatever its positions are.
#include <type_traits>

#include "attn_spans.h"
#include "attn_tree.h"
#include "store_e4m3.h"

namespace tempo {
namespace {

__device__ inline int first_step(const int32_t* t_per_seq, int t, int b) {
  int tb = t_per_seq ? t_per_seq[b] : t;
  tb = tb > t ? t : tb;
  return tb < 0 ? 0 : tb;
}

// Eight dims of a row, as they lie in memory and as numbers.
template <typename T>
struct Octet;
template <>
struct Octet<uint16_t> {
  u32x4 w;
  __device__ void load(const uint16_t* from) { w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from)); }
  __device__ void numbers(float* f) const { unpack8(w, f); }
};
template <>
struct Octet<float> {
  f32x4 a, z;
  __device__ void load(const float* from) {
    a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(from));
    z = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(from) + 1);
  }
  __device__ void numbers(float* f) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = a[e], f[4 + e] = z[e];
  }
};
__device__ inline void store_octet(uint16_t* to, const float* f) { *reinterpret_cast<u32x4*>(to) = pack8(f); }
__device__ inline void store_octet(float* to, const float* f) {
  *reinterpret_cast<f32x4*>(to) = f32x4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<f32x4*>(to + 4) = f32x4{f[4], f[5], f[6], f[7]};
}

// Cosines and sines of pairs i0 .. i0+7 of row `row` of the call.
__device__ inline void angles_at(const PlaceParams& p, int64_t row, int half, int i0, float* cs, float* sn) {
  const int32_t* const at = p.positions + row * p.axes;
  auto place = [&](int axis) {
    int v = at[axis < p.axes ? axis : 0];
    v = v < 0 ? 0 : v;
    return (int64_t)(v < p.table_rows ? v : p.table_rows - 1);
  };
  const uint32_t octet = (uint32_t)(p.axis_bits[i0 >> 5] >> (2 * (i0 & 31))) & 0xFFFFu, first = octet & 3u;
  if (octet == first * 0x5555u) {  // one axis
    load_angles(p.rope_cos, place((int)first), half, i0, cs);
    load_angles(p.rope_sin, place((int)first), half, i0, sn);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t entry = place((int)(octet >> (2 * e)) & 3) * half + i0 + e;
    cs[e] = p.rope_cos[entry];
    sn[e] = p.rope_sin[entry];
  }
}

// Where row c of sequence b of the call goes: the slot number of its tile's first slot for kv head 0, and the slot in the tile.
struct RowPlace {
  int64_t first;
  int slot;
};
__device__ inline RowPlace place_of(const PlaceParams& p, int b, int t) {
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + ((t >> p.z_log2) & p.tile_mask)], p.num_blocks);
  return {((int64_t)phys * p.Hkv) << p.z_log2, t & ((1 << p.z_log2) - 1)};
}

// Codes and scale byte of two octets of a row that LANES lanes hold.
template <int LANES>
__device__ inline void quantise_two(u32x4 lo, u32x4 hi, uint2& lo_codes, uint2& hi_codes, uint32_t& scale) {
  auto largest = [](uint32_t v) {
#pragma unroll
    for (int o = 1; o < LANES; o *= 2) {
      const uint32_t other = (uint32_t)__shfl_xor((int)v, o);
      v = other > v ? other : v;
    }
    return v;
  };
  uint32_t a = top_of_any(lo), z = top_of_any(hi), top = largest(a > z ? a : z);
  if (top <= 0x7F60u) {  // (as quantise_with())
    scale = (uint32_t)scale_byte(top);
    const float s = scale_of(scale);
    lo_codes = uint2{finite_codes_of(lo.x, lo.y, s), finite_codes_of(lo.z, lo.w, s)};
    hi_codes = uint2{finite_codes_of(hi.x, hi.y, s), finite_codes_of(hi.z, hi.w, s)};
    return;
  }
  top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = top_of(hi[i], top_of(lo[i], top));
  scale = (uint32_t)scale_byte(largest(top));
  const float inverse = inverse_scale_of(scale), most = largest_code(scale);
  lo_codes = uint2{codes_of(lo.x, inverse, most) | (codes_of(lo.y, inverse, most) << 16), codes_of(lo.z, inverse, most) | (codes_of(lo.w, inverse, most) << 16)};
  hi_codes = uint2{codes_of(hi.x, inverse, most) | (codes_of(hi.y, inverse, most) << 16), codes_of(hi.z, inverse, most) | (codes_of(hi.w, inverse, most) << 16)};
}

// The launch's first workgroups turn queries and keys: D/16 lanes to a row and kHeads of its heads (query heads, then key heads), a
// lane an octet of pairs, whose angles it asks for once.  Then come the values of a bf16 store, by 32-slot groups: a lane eight slots
// by eight dims, read row by row, turned in registers and written as eight 16-byte units (8 bytes or 2 where the call does not write
// all eight slots: 512 rows of 16 trees, 24/8 heads of 128, 8.7 us with 2-byte stores alone, 6.4); of other stores D/8 lanes to a row of a head.
// Bound by memory: 10000 rows of 32/4 heads of 128 with three axes, 205 MB in and out, 50 us of cold rows, 41 back to back (5.0 TB/s).

constexpr int kHeads = 4;

template <int D, typename T, bool k8>
__device__ __forceinline__ void turn_rows(const PlaceParams& p, const T* k_raw, int64_t lane_of_part) {
  constexpr int LANES = D / 16;
  const int chunks = (p.Hq + p.Hrows + kHeads - 1) / kHeads;
  const int64_t unit = lane_of_part / LANES;
  const int part = (int)(lane_of_part % LANES);
  // 8 rows side by side, then the chunks of their heads: the 16-byte units of 8 keys lie together in a bf16 store
  const int64_t all = (int64_t)p.batch * p.count, eight = unit / (8 * chunks);
  const int in = (int)(unit - eight * (8 * chunks)), chunk = in >> 3;
  const int64_t row = eight * 8 + (in & 7);
  if (row >= all) return;
  const int b = (int)(row / p.count), c = (int)(row - (int64_t)b * p.count);
  if (p.count_per_seq && c >= p.count_per_seq[b]) return;  // (all lanes of a row alike)
  const int first = chunk * kHeads, heads = p.Hq + p.Hrows - first < kHeads ? p.Hq + p.Hrows - first : kHeads;
  Octet<T> x[kHeads], y[kHeads];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const int head = h < heads ? first + h : first;  // (not there: read again, so that all requests go out together)
    const T* from = head < p.Hq ? static_cast<const T*>(p.q) + (row * p.Hq + head) * D : k_raw + (row * p.Hrows + head - p.Hq) * D;
    x[h].load(from + 8 * part);
    y[h].load(from + D / 2 + 8 * part);
  }
  RowPlace at = {0, 0};
  if (first + heads > p.Hq) at = place_of(p, b, first_step(p.t_per_seq, p.t, b) + c);
  float cs[8], sn[8];
  angles_at(p, row, D / 2, 8 * part, cs, sn);
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (h >= heads) break;
    const int head = first + h;
    float xs[8], ys[8];
    x[h].numbers(xs);
    y[h].numbers(ys);
    float lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo[e] = rope_lo(xs[e], ys[e], cs[e], sn[e]);
      hi[e] = rope_hi(xs[e], ys[e], cs[e], sn[e]);
    }
    if (head < p.Hq) {
      T* const to = static_cast<T*>(p.q_out) + (row * p.Hq + head) * D + 8 * part;
      store_octet(to, lo);
      store_octet(to + D / 2, hi);
      continue;
    }
    const int64_t slot0 = at.first + ((int64_t)(head - p.Hq) << p.z_log2);
    if constexpr (k8) {
      uint2 lo_codes, hi_codes;
      uint32_t scale;
      quantise_two<LANES>(pack8(lo), pack8(hi), lo_codes, hi_codes, scale);
      uint8_t* const pool = static_cast<uint8_t*>(p.k_pool);
      *reinterpret_cast<uint2*>(pool + slot0 * D + tile_off_k_e4m3(D, at.slot, 8 * part)) = lo_codes;
      *reinterpret_cast<uint2*>(pool + slot0 * D + tile_off_k_e4m3(D, at.slot, 8 * part + D / 2)) = hi_codes;
      const int64_t slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;
      if (part == 0) pool[slots * D + slot0 + scale_off_k(at.slot)] = (uint8_t)scale;
    } else {
      T* const to = static_cast<T*>(p.k_pool) + slot0 * D;
      store_octet(to + (sizeof(T) == 4 ? tile_off_f32(D, at.slot, 8 * part) : tile_off_k_bf16(D, at.slot, 8 * part)), lo);
      store_octet(to + (sizeof(T) == 4 ? tile_off_f32(D, at.slot, 8 * part + D / 2) : tile_off_k_bf16(D, at.slot, 8 * part + D / 2)), hi);
    }
  }
}

// Values of a bf16 store.  Groups of a sequence: those of its steps, of which there are at most `groups`.
template <int D>
__device__ __forceinline__ void value_groups(const PlaceParams& p, const uint16_t* v_new, int64_t at, int groups) {
  constexpr int PARTS = D / 8;
  const int part = (int)(at % PARTS), c = (int)(at / PARTS) & 3;
  const int64_t unit = at / (4 * PARTS);          // (sequence, group, head)
  const int head = (int)(unit % p.Hrows), g = (int)(unit / p.Hrows % groups);
  const int64_t b64 = unit / p.Hrows / groups;
  if (b64 >= p.batch) return;
  const int b = (int)b64, t = first_step(p.t_per_seq, p.t, b), key = ((t >> 5) + g) << 5;
  int rows = p.count;
  if (p.count_per_seq) {
    const int n = p.count_per_seq[b];
    rows = n < 0 ? 0 : (n < rows ? n : rows);
  }
  // the lane's slots are steps key + 4c + 0 .. 3 and the same + 16
  u32x4 w[8];
  bool ours[2] = {true, true}, some = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int row = key + 4 * c + (e & 3) + 16 * (e >> 2) - t;
    const bool there = row >= 0 && row < rows;
    ours[e >> 2] = ours[e >> 2] && there;
    some = some || there;
    w[e] = u32x4{0u, 0u, 0u, 0u};
    if (there) w[e] = *reinterpret_cast<const u32x4*>(v_new + (((int64_t)b * p.count + row) * p.Hrows + head) * D + 8 * part);
  }
  if (!some) return;
  const RowPlace place = place_of(p, b, key);
  u32x4* const to = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.v_pool) + (place.first + ((int64_t)head << p.z_log2)) * D +
                                             tile_off_v_bf16(D, place.slot + 4 * c, 8 * part));
#pragma unroll
  for (int i = 0; i < 8; ++i) {                   // dim 8 part + i of the eight slots
    const uint32_t half = i & 1 ? 0x07060302u : 0x05040100u;
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __builtin_amdgcn_perm(w[2 * e + 1][i >> 1], w[2 * e][i >> 1], half);
    if (ours[0] && ours[1]) {
      to[i] = o;
      continue;
    }
    uint16_t* const each = reinterpret_cast<uint16_t*>(to + i);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (ours[h]) {
        *reinterpret_cast<uint2*>(each + 4 * h) = uint2{o[2 * h], o[2 * h + 1]};
        continue;
      }
#pragma unroll
      for (int e = 4 * h; e < 4 * h + 4; ++e) {
        const int row = key + 4 * c + (e & 3) + 16 * h - t;
        if (row >= 0 && row < rows) each[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
      }
    }
  }
}

// Values of other stores: D/8 lanes to a row of a head.
template <int D, typename T, bool k8>
__device__ __forceinline__ void value_rows(const PlaceParams& p, const T* v_new, int64_t at) {
  constexpr int PARTS = D / 8;
  const int64_t unit = at / PARTS, row = unit / p.Hrows;
  const int part = (int)(at % PARTS), head = (int)(unit - row * p.Hrows);
  if (row >= (int64_t)p.batch * p.count) return;
  const int b = (int)(row / p.count), c = (int)(row - (int64_t)b * p.count);
  if (p.count_per_seq && c >= p.count_per_seq[b]) return;  // (all lanes of a row alike)
  const RowPlace place = place_of(p, b, first_step(p.t_per_seq, p.t, b) + c);
  const int64_t slot0 = place.first + ((int64_t)head << p.z_log2);
  const T* const from = v_new + unit * D + 8 * part;
  if constexpr (k8) {
    const RowPiece r = quantise_piece<D>(*reinterpret_cast<const u32x4*>(from));
    store_piece<D>(static_cast<uint8_t*>(p.v_pool), ((int64_t)p.num_blocks * p.Hkv) << p.z_log2, slot0, place.slot, true, part, r);
  } else {
    Octet<T> w;
    float x[8];
    w.load(from);
    w.numbers(x);
    store_octet(static_cast<T*>(p.v_pool) + slot0 * D + tile_off_f32(D, place.slot, 8 * part), x);
  }
}

template <int D, typename T, bool k8>
__global__ __launch_bounds__(256) void kv_place(PlaceParams p, const T* __restrict__ k_raw, const T* __restrict__ v_new, unsigned turning, int groups) {
  if (blockIdx.x < turning) {
    turn_rows<D, T, k8>(p, k_raw, (int64_t)blockIdx.x * 256 + threadIdx.x);
    return;
  }
  const int64_t at = (int64_t)(blockIdx.x - turning) * 256 + threadIdx.x;
  if constexpr (!k8 && sizeof(T) == 2) value_groups<D>(p, v_new, at, groups);
  else value_rows<D, T, k8>(p, v_new, at);
}

template <typename T, bool k8>
hipError_t launch_place_of(const PlaceParams& p, const void* k_raw, const void* v_new, int D, hipStream_t stream) {
  const int64_t rows = (int64_t)p.batch * p.count, chunks = (p.Hq + p.Hrows + kHeads - 1) / kHeads;
  const int64_t turning = ((rows + 7) / 8 * 8 * chunks * (D / 16) + 255) / 256;
  // steps t .. t + count - 1 touch one group more where they may begin anywhere
  const int groups = p.t_per_seq ? (p.count + 30) / 32 + 1 : ((p.t + p.count - 1) >> 5) - (p.t >> 5) + 1;
  const int64_t lanes = !k8 && sizeof(T) == 2 ? (int64_t)p.batch * groups * p.Hrows * (D / 2) : rows * p.Hrows * (D / 8);
  const dim3 grid((unsigned)(turning + (lanes + 255) / 256)), block(256);
  const T *k = static_cast<const T*>(k_raw), *v = static_cast<const T*>(v_new);
  if (D == 128) return launch((kv_place<128, T, k8>), grid, block, 0, stream, p, k, v, (unsigned)turning, groups);
  return launch((kv_place<64, T, k8>), grid, block, 0, stream, p, k, v, (unsigned)turning, groups);
}

__global__ __launch_bounds__(256) void tree_positions(const int32_t* parents, int32_t* positions, int nodes, int t, const int32_t* t_per_seq) {
  extern __shared__ uint32_t lds[];
  const int b = blockIdx.x;
  const Tree tree = tree_of(parents + (int64_t)b * nodes, nodes, 0, 0, 0, lds);
  const int tb = first_step(t_per_seq, t, b);
  for (int i = threadIdx.x; i < nodes; i += blockDim.x) positions[(int64_t)b * nodes + i] = tb + tree.depth(i);
}

// One workgroup to a (sequence, layer) and `each` kv heads, keys and values: row t + i gets what row t + kept[i] held before the call.
// All rows are read before one is written, so their order does not matter.  Keys move by pieces of eight dims, values by elements,
// which lie 16 bytes apart (64 lanes touch 8 cache lines, by pieces 64).  Bound by the launch and three memory round trips (list, block table, rows).
template <int D, int kDtype>
__global__ __launch_bounds__(256) void kv_keep(KeepParams p, int each) {
  constexpr int PARTS = D / 8;
  using T = typename std::conditional<kDtype == TEMPO_F32, uint32_t, typename std::conditional<kDtype == TEMPO_E4M3, uint8_t, uint16_t>::type>::type;
  struct Piece {
    T e[8];
  };
  extern __shared__ uint32_t lds[];  // pieces of keys, elements of values, (8 bits) scale bytes
  __shared__ int64_t first[2][kKeepRows];  // slot number of the tile's first slot, kv head 0: of the row read, of the row written
  __shared__ int32_t slot[2][kKeepRows];   // in the tile
  __shared__ int32_t listed;
  const int b = blockIdx.y, head0 = blockIdx.x * each, heads = p.Hkv - head0 < each ? p.Hkv - head0 : each, tid = threadIdx.x;
  if (tid == 0) listed = p.count;
  __syncthreads();
  if (tid < p.count) {
    const int n = p.kept[(int64_t)b * p.count + tid];
    const bool there = n >= 0 && n < p.nodes;
    if (!there) atomicMin(&listed, tid);  // (the least of them, whatever their order)
    const int t = first_step(p.t_per_seq, p.t, b);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int step = t + (i || !there ? tid : n);
      const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + ((step >> p.z_log2) & p.tile_mask)], p.num_blocks);
      first[i][tid] = ((int64_t)phys * p.Hkv) << p.z_log2;
      slot[i][tid] = step & ((1 << p.z_log2) - 1);
    }
  }
  __syncthreads();
  const int rows = listed;
  T* const k_pool = static_cast<T*>(p.k_pool[blockIdx.z]);
  T* const v_pool = static_cast<T*>(p.v_pool[blockIdx.z]);
  const int64_t slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;
  const int of_row = heads * PARTS, pieces = rows * of_row, values = rows * heads * D;
  Piece* const keys_held = reinterpret_cast<Piece*>(lds);
  T* const values_held = reinterpret_cast<T*>(keys_held + pieces);
  uint8_t* const scales_held = reinterpret_cast<uint8_t*>(values_held + values);
  auto key_at = [&](int which, int i) {
    const int row = i / of_row, in = i - row * of_row, head = in / PARTS, d = 8 * (in % PARTS), at = slot[which][row];
    const int64_t off = kDtype == TEMPO_F32 ? tile_off_f32(D, at, d) : kDtype == TEMPO_BF16 ? tile_off_k_bf16(D, at, d) : tile_off_k_e4m3(D, at, d);
    return reinterpret_cast<Piece*>(k_pool + (first[which][row] + ((int64_t)(head0 + head) << p.z_log2)) * D + off);
  };
  auto value_at = [&](int which, int i) {
    const int d = i % D, in = i / D, row = in / heads, head = in - row * heads, at = slot[which][row];
    const int64_t off = kDtype == TEMPO_F32 ? tile_off_f32(D, at, d) : kDtype == TEMPO_BF16 ? tile_off_v_bf16(D, at, d) : tile_off_v_e4m3(D, at, d);
    return v_pool + (first[which][row] + ((int64_t)(head0 + head) << p.z_log2)) * D + off;
  };
  auto scale_at = [&](int which, int i) {
    const int row = i / (2 * heads), in = i - row * 2 * heads, value = in >= heads, at = slot[which][row];
    uint8_t* const pool = reinterpret_cast<uint8_t*>(value ? v_pool : k_pool);
    return pool + slots * D + first[which][row] + ((int64_t)(head0 + (value ? in - heads : in)) << p.z_log2) + (value ? scale_off_v(at) : scale_off_k(at));
  };
#pragma unroll 2
  for (int i = tid; i < pieces; i += 256) keys_held[i] = *key_at(0, i);
#pragma unroll 4
  for (int i = tid; i < values; i += 256) values_held[i] = *value_at(0, i);
  if constexpr (kDtype == TEMPO_E4M3) {
    for (int i = tid; i < rows * 2 * heads; i += 256) scales_held[i] = *scale_at(0, i);
  }
  __syncthreads();
#pragma unroll 2
  for (int i = tid; i < pieces; i += 256) *key_at(1, i) = keys_held[i];
#pragma unroll 4
  for (int i = tid; i < values; i += 256) *value_at(1, i) = values_held[i];
  if constexpr (kDtype == TEMPO_E4M3) {
    for (int i = tid; i < rows * 2 * heads; i += 256) *scale_at(1, i) = scales_held[i];
  }
}

// Heads of a workgroup: so many that the workgroups all fit the part (eight to a compute unit), in up to 48 KiB.
template <int kDtype>
hipError_t launch_keep_of(const KeepParams& p, int batch, int layers, int D, hipStream_t stream) {
  const size_t of_head = 2 * (size_t)p.count * (D * (kDtype == TEMPO_F32 ? 4 : kDtype == TEMPO_BF16 ? 2 : 1) + 1);
  int64_t each = ((int64_t)p.Hkv * batch * layers + 2047) / 2048;
  each = each < p.Hkv ? each : p.Hkv;
  each = each < (int64_t)((48 << 10) / of_head) ? each : (int64_t)((48 << 10) / of_head);
  each = each < 1 ? 1 : each;
  const int64_t parts = (p.Hkv + each - 1) / each;
  each = (p.Hkv + parts - 1) / parts;
  const dim3 grid((unsigned)parts, (unsigned)batch, (unsigned)layers), block(256);
  if (D == 128) return launch((kv_keep<128, kDtype>), grid, block, (size_t)each * of_head, stream, p, (int)each);
  return launch((kv_keep<64, kDtype>), grid, block, (size_t)each * of_head, stream, p, (int)each);
}

}  // namespace

hipError_t launch_place(const PlaceParams& p, const void* k_raw, const void* v_new, int D, int dtype, hipStream_t stream) {
  if (dtype == TEMPO_F32) return launch_place_of<float, false>(p, k_raw, v_new, D, stream);
  if (dtype == TEMPO_E4M3) return launch_place_of<uint16_t, true>(p, k_raw, v_new, D, stream);
  return launch_place_of<uint16_t, false>(p, k_raw, v_new, D, stream);
}

hipError_t launch_tree_positions(const int32_t* parents, int32_t* positions, int batch, int nodes, int t, const int32_t* t_per_seq, hipStream_t stream) {
  return launch(tree_positions, dim3((unsigned)batch), dim3(256), tree_lds_bytes(nodes), stream, parents, positions, nodes, t, t_per_seq);
}

hipError_t launch_keep(const KeepParams& p, int batch, int layers, int D, int dtype, hipStream_t stream) {
  if (dtype == TEMPO_F32) return launch_keep_of<TEMPO_F32>(p, batch, layers, D, stream);
  if (dtype == TEMPO_E4M3) return launch_keep_of<TEMPO_E4M3>(p, batch, layers, D, stream);
  return launch_keep_of<TEMPO_BF16>(p, batch, layers, D, stream);
}

}  // namespace tempo
