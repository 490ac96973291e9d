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

__device__ inline void load_octet(const uint16_t* from, float* f) { unpack8(*reinterpret_cast<const u32x4*>(from), f); }
__device__ inline void load_octet(const float* from, float* f) { load_angles(from, 0, 0, 0, f); }
__device__ inline void store_octet(uint16_t* to, const float* f) { *reinterpret_cast<u32x4*>(to) = pack8(f); }
__device__ inline void store_octet(float* to, const float* f) {
  *reinterpret_cast<float4*>(to) = float4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<float4*>(to + 4) = float4{f[4], f[5], f[6], f[7]};
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

// A lane's octet of a row that D/8 lanes hold, turned; its pairs' other halves lie D/16 lanes on.
template <int D>
__device__ inline void turn_octet(const float* cs, const float* sn, bool upper, float* x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float other = __shfl_xor(x[e], D / 16);
    x[e] = upper ? rope_hi(other, x[e], cs[e], sn[e]) : rope_lo(x[e], other, cs[e], sn[e]);
  }
}

// D/8 lanes to a row of one head: the call's query heads, then its key heads, then its value heads.
template <int D, typename T, bool k8>
__global__ __launch_bounds__(256) void kv_place(PlaceParams p, const T* __restrict__ k_raw, const T* __restrict__ v_new) {
  constexpr int LANES = D / 8;
  const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
  const int part = threadIdx.x % LANES, heads = p.Hq + 2 * p.Hrows;
  const int64_t row = unit / heads;  // b * count + c
  int head = (int)(unit - row * heads);
  const int b = (int)(row / p.count), c = (int)(row - (int64_t)b * p.count);
  if (b >= p.batch || (p.count_per_seq && c >= p.count_per_seq[b])) return;  // (all lanes of a row alike)
  const bool query = head < p.Hq, value = !query && head >= p.Hq + p.Hrows;
  const T* from = query ? static_cast<const T*>(p.q) + (row * p.Hq + head) * D
                        : (value ? v_new + (row * p.Hrows + head - p.Hq - p.Hrows) * D : k_raw + (row * p.Hrows + head - p.Hq) * D);
  float x[8];
  load_octet(from + 8 * part, x);
  if (!value) {
    float cs[8], sn[8];
    const bool upper = part >= LANES / 2;
    angles_at(p, row, D / 2, 8 * (upper ? part - LANES / 2 : part), cs, sn);
    turn_octet<D>(cs, sn, upper, x);
  }
  if (query) {
    store_octet(static_cast<T*>(p.q_out) + (row * p.Hq + head) * D + 8 * part, x);
    return;
  }
  head -= value ? p.Hq + p.Hrows : p.Hq;
  const int t = first_step(p.t_per_seq, p.t, b) + c, slot = t & ((1 << p.z_log2) - 1);
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + ((t >> p.z_log2) & p.tile_mask)], p.num_blocks);
  const int64_t first = ((int64_t)phys * p.Hkv + head) << p.z_log2;  // slot number of the tile's first
  if constexpr (k8) {
    const RowPiece r = quantise_piece<D>(pack8(x));
    const int64_t slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;
    store_piece<D>(static_cast<uint8_t*>(value ? p.v_pool : p.k_pool), slots, first, slot, value, part, r);
  } else if constexpr (sizeof(T) == 4) {
    store_octet(static_cast<T*>(value ? p.v_pool : p.k_pool) + first * D + tile_off_f32(D, slot, 8 * part), x);
  } else if (!value) {
    store_octet(static_cast<T*>(p.k_pool) + first * D + tile_off_k_bf16(D, slot, 8 * part), x);
  } else {
    const u32x4 w = pack8(x);
    uint16_t* const to = static_cast<uint16_t*>(p.v_pool) + first * D + tile_off_v_bf16(D, slot, 8 * part);  // dims 8 elements apart
#pragma unroll
    for (int e = 0; e < 8; ++e) to[8 * e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
  }
}

template <typename T, bool k8>
hipError_t launch_place_of(const PlaceParams& p, const void* k_raw, const void* v_new, int D, hipStream_t stream) {
  const int64_t lanes = (int64_t)p.batch * p.count * (p.Hq + 2 * p.Hrows) * (D / 8);
  const dim3 grid((unsigned)((lanes + 255) / 256)), block(256);
  const T *k = static_cast<const T*>(k_raw), *v = static_cast<const T*>(v_new);
  if (D == 128) return launch((kv_place<128, T, k8>), grid, block, 0, stream, p, k, v);
  return launch((kv_place<64, T, k8>), grid, block, 0, stream, p, k, v);
}

__global__ __launch_bounds__(256) void tree_positions(const int32_t* parents, int32_t* positions, int nodes, int t, const int32_t* t_per_seq) {
  extern __shared__ uint32_t lds[];
  const int b = blockIdx.x;
  const Tree tree = tree_of(parents + (int64_t)b * nodes, nodes, 0, 0, 0, lds);
  const int tb = first_step(t_per_seq, t, b);
  for (int i = threadIdx.x; i < nodes; i += blockDim.x) positions[(int64_t)b * nodes + i] = tb + tree.depth(i);
}

// One workgroup to a (sequence, kv head, layer, pool): row t + i gets what row t + kept[i] held before the call.
template <int D, int kDtype>
__global__ __launch_bounds__(256) void kv_keep(KeepParams p) {
  using T = typename std::conditional<kDtype == TEMPO_F32, uint32_t, typename std::conditional<kDtype == TEMPO_E4M3, uint8_t, uint16_t>::type>::type;
  extern __shared__ uint32_t lds[];  // [rows][D] elements, then (8 bits) [rows] scale bytes
  __shared__ int32_t list[kKeepRows];
  __shared__ int32_t listed;
  T* const held = reinterpret_cast<T*>(lds);
  const int b = blockIdx.y, head = blockIdx.x >> 1, tid = threadIdx.x;
  const bool value = (blockIdx.x & 1) != 0;
  if (tid == 0) listed = p.count;
  __syncthreads();
  if (tid < p.count) {
    const int n = p.kept[(int64_t)b * p.count + tid];
    list[tid] = n;
    if (n < 0 || n >= p.nodes) atomicMin(&listed, tid);  // (the least of them, whatever their order)
  }
  __syncthreads();
  const int rows = listed;
  T* const pool = static_cast<T*>(value ? p.v_pool[blockIdx.z] : p.k_pool[blockIdx.z]);
  const int64_t slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;
  const int t = first_step(p.t_per_seq, p.t, b);
  auto tile_of = [&](int step) {
    const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + ((step >> p.z_log2) & p.tile_mask)], p.num_blocks);
    return ((int64_t)phys * p.Hkv + head) << p.z_log2;
  };
  auto place = [&](int step, int d) {
    const int slot = step & ((1 << p.z_log2) - 1);
    const int64_t in = kDtype == TEMPO_F32    ? tile_off_f32(D, slot, d)
                       : kDtype == TEMPO_BF16 ? (value ? tile_off_v_bf16(D, slot, d) : tile_off_k_bf16(D, slot, d))
                                              : (value ? tile_off_v_e4m3(D, slot, d) : tile_off_k_e4m3(D, slot, d));
    return tile_of(step) * D + in;
  };
  auto scale_place = [&](int step) {
    const int slot = step & ((1 << p.z_log2) - 1);
    return slots * D + tile_of(step) + (value ? scale_off_v(slot) : scale_off_k(slot));
  };
  uint8_t* const scales = reinterpret_cast<uint8_t*>(held + rows * D);
  for (int i = tid; i < rows * D; i += 256) {
    if (list[i / D] != i / D) held[i] = pool[place(t + list[i / D], i % D)];
  }
  if (kDtype == TEMPO_E4M3 && tid < rows) scales[tid] = reinterpret_cast<const uint8_t*>(pool)[scale_place(t + list[tid])];
  __syncthreads();
  for (int i = tid; i < rows * D; i += 256) {
    if (list[i / D] != i / D) pool[place(t + i / D, i % D)] = held[i];
  }
  if (kDtype == TEMPO_E4M3 && tid < rows) reinterpret_cast<uint8_t*>(pool)[scale_place(t + tid)] = scales[tid];
}

template <int kDtype>
hipError_t launch_keep_of(const KeepParams& p, int batch, int layers, int D, hipStream_t stream) {
  const dim3 grid((unsigned)(2 * p.Hkv), (unsigned)batch, (unsigned)layers), block(256);
  const size_t lds = (size_t)p.count * (D * (kDtype == TEMPO_F32 ? 4 : kDtype == TEMPO_BF16 ? 2 : 1) + 1) + 4;
  if (D == 128) return launch((kv_keep<128, kDtype>), grid, block, lds, stream, p);
  return launch((kv_keep<64, kDtype>), grid, block, lds, stream, p);
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
