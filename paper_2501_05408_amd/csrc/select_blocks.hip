// Sparse attention's choice of blocks: bounds of the keys of every block, a score of every block for a query, and the
// blocks with the best scores.
//
//   bounds   lo_d = min_j k_jd, hi_d = max_j k_jd over the keys j of a block (of one kv head), once it is complete
//   score    S_n = max over the group's heads g of sum_d max(q_gd lo_d, q_gd hi_d): no key of block n has a larger
//            product with any of the group's queries
//   choice   the first `first` blocks, the `last` newest ones (the newest may be incomplete: it has no bounds yet), and
//            of the others those with the largest S_n, `pick` blocks in all; of equal scores the earlier block
//
// The choice is that of scores summed in 64 bits, in which products of two bf16 values are exact and their sums exact or 1e-16
// off, so that it is the formula's whatever the order of the sums; by fp32 sums alone, blocks whose scores lie within 1e-6 of
// the border would be chosen by rounding.
#include <type_traits>

#include "attn_bf16_common.h"
#include "attn_units.h"
#include "store_e4m3.h"

namespace tempo {
namespace {

__device__ inline int step_of(const int32_t* t_per_seq, int t, int b) {
  int t_b = t_per_seq ? t_per_seq[b] : t;
  t_b = t_b > t ? t : t_b;
  return t_b < 0 ? 0 : t_b;
}

// A value of another lane of the row of 16, by lane moves instead of trips through the LDS permute unit; 0 where there is none.
constexpr int kPairs = 0xB1, kFours = 0x4E, kEights = 0x141, kSixteens = 0x140;  // 1 0 3 2; 2 3 0 1; eight, sixteen lanes reversed
constexpr int kRight = 0x100, kLeft = 0x110;                                    // + n: of the lane n further right / left
template <int How>
__device__ inline int lane_move(int v) { return __builtin_amdgcn_mov_dpp(v, How, 0xF, 0xF, true); }
template <int How>
__device__ inline float lane_move(float v) { return __builtin_bit_cast(float, lane_move<How>(__builtin_bit_cast(int, v))); }
template <int How>
__device__ inline double lane_move(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)lane_move<How>((int)(uint32_t)u), hi = (uint32_t)lane_move<How>((int)(uint32_t)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ inline float row_maximum(float v) {
  v = fmaxf(v, lane_move<kPairs>(v));
  v = fmaxf(v, lane_move<kFours>(v));
  v = fmaxf(v, lane_move<kEights>(v));
  return fmaxf(v, lane_move<kSixteens>(v));
}
__device__ inline float wave_max(float v) { return column_max(row_maximum(v)); }
// Sums over the wavefront's lanes from this one on (kRight) or up to it (kLeft), and its total.
template <int Side>
__device__ inline int wave_sums(int v, int& total) {
  v += lane_move<Side + 1>(v);
  v += lane_move<Side + 2>(v);
  v += lane_move<Side + 4>(v);
  v += lane_move<Side + 8>(v);
  constexpr int end = Side == kRight ? 0 : 15;  // of a row: its total
  const int r0 = __builtin_amdgcn_readlane(v, end), r1 = __builtin_amdgcn_readlane(v, 16 + end);
  const int r2 = __builtin_amdgcn_readlane(v, 32 + end), r3 = __builtin_amdgcn_readlane(v, 48 + end);
  const int row = (threadIdx.x & 63) >> 4;
  total = r0 + r1 + r2 + r3;
  if (Side == kRight) return v + (row == 0 ? r1 + r2 + r3 : row == 1 ? r2 + r3 : row == 2 ? r3 : 0);
  return v + (row == 0 ? 0 : row == 1 ? r0 : row == 2 ? r0 + r1 : r0 + r1 + r2);
}

// ---- bounds -----------------------------------------------------------------------------------
// Values are compared as whole numbers, two to a word: a bf16 value's bits, with all but the sign turned over where it is
// negative, are in the order of the values, NaN above infinity or below minus infinity by its sign.
typedef short i16x2 __attribute__((ext_vector_type(2)));

__device__ inline i16x2 ordered(uint32_t pair) {
  const i16x2 v = __builtin_bit_cast(i16x2, pair);
  return v ^ ((v >> 15) & i16x2{0x7FFF, 0x7FFF});
}
__device__ inline uint32_t values_in_order(i16x2 v) { return __builtin_bit_cast(uint32_t, v ^ ((v >> 15) & i16x2{0x7FFF, 0x7FFF})); }

// Over the 16 lanes of a row of lanes.
template <typename F>
__device__ inline i16x2 reduce_row(i16x2 v, F f) {
  const auto moved = [&](auto how) { return __builtin_bit_cast(i16x2, lane_move<how.value>(__builtin_bit_cast(int, v))); };
  v = f(v, moved(std::integral_constant<int, kPairs>()));
  v = f(v, moved(std::integral_constant<int, kFours>()));
  v = f(v, moved(std::integral_constant<int, kEights>()));
  return f(v, moved(std::integral_constant<int, kSixteens>()));
}

// Bounds of the block of one kv head whose first slot has number `first` among the store's; wavefronts w < D/64 (8-bit store)
// or D/32 (bf16) read the 1 KiB units of their part of the dims, 16 or 8 of them a lane.  Lane (row + 16c) goes through the
// rows row, 16 + row, ... of the block, then the 16 lanes of equal c are reduced.  kFresh: the block's last row is not in the
// store yet; the lane's part of it is in `last` (8 bits: codes, with scale byte last_scale).
// Bound by memory, as long as the comparisons are whole words' (8 x 4096 keys of 4 heads of 128 in blocks of 64, 34 MB:
// 6.7 us, 5.1 TB/s; one value at a time in fp32 10.2; loads that leave the keys in the caches 7.4).
template <int D, bool k8, bool kFresh>
__device__ __forceinline__ void bounds_of_block(const StoreParams& p, int64_t first, int w, int lane, uint16_t* __restrict__ to, u32x4 last,
                                                uint32_t last_scale) {
  constexpr int PER_TILE = k8 ? D / 64 : D / 32;  // units of a row-tile
  constexpr int N = k8 ? 8 : 4;                   // words of two values
  const char* const at = static_cast<const char*>(p.k_pool) + first * (k8 ? D : 2 * D) + w * 1024 + lane * 16;
  const uint8_t* const scales = static_cast<const uint8_t*>(p.k_pool) + ((((int64_t)p.num_blocks * p.Hkv) << p.z_log2) * D + first) + 2 * (lane & 15);
  const auto less = [](i16x2 a, i16x2 z) { return __builtin_elementwise_min(a, z); };
  const auto more = [](i16x2 a, i16x2 z) { return __builtin_elementwise_max(a, z); };
  i16x2 lo[N], hi[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    lo[i] = i16x2{0x7FFF, 0x7FFF};
    hi[i] = i16x2{-0x8000, -0x8000};
  }
  const int groups = 1 << (p.z_log2 - 5);
#pragma unroll 2
  for (int t = 0; t < groups; ++t) {
    u32x4 u[2];
    uint32_t both = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const u32x4* const unit = reinterpret_cast<const u32x4*>(at + (int64_t)(2 * t + r) * PER_TILE * 1024);
      if constexpr (kFresh) u[r] = *unit;  // (a step's own block is read again by its attention)
      else u[r] = __builtin_nontemporal_load(unit);
    }
    if constexpr (k8) both = *reinterpret_cast<const uint16_t*>(scales + 32 * t);
    if (kFresh && t == groups - 1 && (lane & 15) == 15) {
      u[1] = last;
      both = (both & 0xFFu) | (last_scale << 8);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      i16x2 x[N];
      if constexpr (k8) {
        const float scale = scale_of(r == 0 ? both & 0xFFu : both >> 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[2 * i] = ordered(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[r][i], scale, false)));
          x[2 * i + 1] = ordered(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[r][i], scale, true)));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = ordered(u[r][i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        lo[i] = less(lo[i], x[i]);
        hi[i] = more(hi[i], x[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    lo[i] = reduce_row(lo[i], less);
    hi[i] = reduce_row(hi[i], more);
    const i16x2 nan = (hi[i] > (short)0x7F80) | (lo[i] < (short)~0x7F80);  // -1 where there is one, of either sign
    lo[i] = (lo[i] & ~nan) | (nan & (short)0x7FC0);
    hi[i] = (hi[i] & ~nan) | (nan & (short)0x7FC0);
  }
  if ((lane & 15) != 0) return;
  const int c = lane >> 4;
#pragma unroll
  for (int h = 0; h < N / 4; ++h) {
    const int d = k8 ? 64 * w + 32 * h + 8 * c : 32 * w + 8 * c;
    const u32x4 l = {values_in_order(lo[4 * h]), values_in_order(lo[4 * h + 1]), values_in_order(lo[4 * h + 2]), values_in_order(lo[4 * h + 3])};
    const u32x4 m = {values_in_order(hi[4 * h]), values_in_order(hi[4 * h + 1]), values_in_order(hi[4 * h + 2]), values_in_order(hi[4 * h + 3])};
    *reinterpret_cast<u32x4*>(to + d) = l;
    *reinterpret_cast<u32x4*>(to + D + d) = m;
  }
}

// One workgroup per (block of a sequence, kv head).
template <int D, bool k8>
__global__ __launch_bounds__(k8 ? D : 2 * D) void block_bounds(StoreParams p, uint16_t* __restrict__ bounds) {
  const int head = blockIdx.y, b = blockIdx.z;
  const int t_b = step_of(p.t_per_seq, p.t, b);
  int rows = p.count;
  if (p.count_per_seq) rows = p.count_per_seq[b] < rows ? p.count_per_seq[b] : rows;
  const int n = (t_b >> p.z_log2) + (int)blockIdx.x;         // block of the sequence
  const int64_t last = (((int64_t)n + 1) << p.z_log2) - 1;   // its last step
  if (last < t_b || last > (int64_t)t_b + rows - 1) return;  // not completed by the call's steps; uniform
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + n], p.num_blocks);
  const int64_t pair = (int64_t)phys * p.Hkv + head;
  bounds_of_block<D, k8, false>(p, pair << p.z_log2, threadIdx.x >> 6, threadIdx.x & 63, bounds + pair * 2 * D, u32x4{0u, 0u, 0u, 0u}, 0u);
}

// A step's row of one (sequence, kv head) into the store, and the bounds of its block if the step is the block's last.  All
// wavefronts of the workgroup call this; each has the whole key row, so that none waits for the write.
template <int D, bool k8>
__device__ __forceinline__ void write_and_bound(const StoreParams& p, const void* k_new, const void* v_new, uint16_t* bounds, int b, int head) {
  constexpr int LANES = D / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4;
  const int t = step_of(p.t_per_seq, p.t, b), n = t >> p.z_log2, slot = t & ((1 << p.z_log2) - 1);
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + n], p.num_blocks);
  const int64_t pair = (int64_t)phys * p.Hkv + head, first = pair << p.z_log2, slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;
  const int at = lane % (2 * LANES), part = at % LANES;  // lanes: key row, value row, copies of both
  const bool value = at >= LANES;
  const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(value ? v_new : k_new) + ((int64_t)b * p.Hkv + head) * D + 8 * part);
  u32x4 last;  // what lane (15 + 16c) of unit `wave` of the row's tile will hold of it
  uint32_t last_scale = 0;
  if constexpr (k8) {
    const RowPiece r = quantise_piece<D>(x);
    if (wave == 0 && lane < 2 * LANES) store_piece<D>(static_cast<uint8_t*>(value ? p.v_pool : p.k_pool), slots, first, slot, value, part, r);
    const int from = (8 * wave + c) % LANES, other = (8 * wave + 4 + c) % LANES;
    last = u32x4{(uint32_t)__shfl((int)r.lo, from), (uint32_t)__shfl((int)r.hi, from), (uint32_t)__shfl((int)r.lo, other), (uint32_t)__shfl((int)r.hi, other)};
    last_scale = (uint32_t)__shfl((int)r.scale, 0);
  } else {
    if (wave == 0 && lane < LANES) {
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.k_pool) + first * D + tile_off_k_bf16(D, slot, 8 * part)) = x;
    } else if (wave == 0 && lane < 2 * LANES) {
      uint16_t* const to = static_cast<uint16_t*>(p.v_pool) + first * D + tile_off_v_bf16(D, slot, 8 * part);  // (dims lie 8 elements apart)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        to[16 * i] = (uint16_t)x[i];
        to[16 * i + 8] = (uint16_t)(x[i] >> 16);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) last[i] = (uint32_t)__shfl((int)x[i], (4 * wave + c) % LANES);
  }
  if (slot != (1 << p.z_log2) - 1) return;  // uniform
  if (wave < (k8 ? D / 64 : D / 32)) bounds_of_block<D, k8, true>(p, first, wave, lane, bounds + pair * 2 * D, last, last_scale);
}

// ---- scores -----------------------------------------------------------------------------------
// Interval of a score: L <= S_n <= U.  sum_d max(q_d lo_d, q_d hi_d) is the product of [max(q, 0), min(q, 0)] and [hi, lo],
// which the matrix cores take for 16 blocks and 16 heads at a time; how far its fp32 sums are off is bounded by kOff times
// A = sum_d |q_d| max(|lo_d|, |hi_d|), another such product: 2 D = 256 exact products are added in some order, each addition
// off by at most 2^-22 of the sums' magnitude, which A bounds (2^-24 is an fp32 rounding), so by 2^-14 A in all; a sixteenth
// of it covers A's own error and the roundings of L and U.
// Blocks whose interval leaves it open whether they are chosen are scored again, in 64 bits (exact_key), by the kernel that
// chooses: one or two of hundreds.  16 sequences of 512 blocks, 24/8 heads of 128, 34 MB of bounds: 8.2 us behind the chain argument,
// table, bounds; all of them in 64 bits 11.7.
constexpr float kOff = 1.0625f / 16384.f;
constexpr float kLeast = 1e-30f;  // (products below the normal fp32 range)

struct Interval {
  float lo, hi;
};

// A wavefront scores 16 blocks, n0 .. n0+15, of those up to newest - last: lane (row + 16c) holds dims 32s + 8c .. +7 of block
// `row` (phys: its number in the pool), and of the query head that is column `row` of a product.  Lanes row < 4 return the
// interval of block n0 + 4c + row, as a word.
template <int D>
__device__ __forceinline__ uint64_t score_sixteen(const ChooseParams& p, int b, int hkv, int n0, int newest, int& phys) {
  constexpr int KS = D / 32;
  const int lane = threadIdx.x & 63, row = lane & 15, c = lane >> 4;
  const int n = n0 + row <= newest - p.last ? n0 + row : n0;
  phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + n], p.num_blocks);
  const uint16_t* const at = static_cast<const uint16_t*>(p.bounds) + ((int64_t)phys * p.Hkv + hkv) * 2 * D + 8 * c;
  const uint16_t* const q = static_cast<const uint16_t*>(p.q) + ((int64_t)b * p.Hq + (int64_t)hkv * p.G) * D + 8 * c;
  u32x4 x[KS];  // of the first 16 heads; asked for before the bounds, which wait for the table (16 sequences of 512 blocks: 14.9 -> 14.5 us)
#pragma unroll
  for (int s = 0; s < KS; ++s) x[s] = *reinterpret_cast<const u32x4*>(q + (int64_t)(row < p.G ? row : p.G - 1) * D + 32 * s);
  __builtin_amdgcn_sched_barrier(0);  // (or the scheduler puts them behind)
  u32x4 lo[KS], hi[KS], far[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    lo[s] = *reinterpret_cast<const u32x4*>(at + 32 * s);
    hi[s] = *reinterpret_cast<const u32x4*>(at + D + 32 * s);
  }
  float low[4], high[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) low[r] = high[r] = -INFINITY;
  for (int g0 = 0; g0 < p.G; g0 += 16) {
    const int g = g0 + row < p.G ? g0 + row : p.G - 1;
    if (g0 > 0) {
#pragma unroll
      for (int s = 0; s < KS; ++s) x[s] = *reinterpret_cast<const u32x4*>(q + (int64_t)g * D + 32 * s);
    } else {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          far[s][i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, lo[s][i] & 0x7FFF7FFFu),
                                                                             __builtin_bit_cast(i16x2, hi[s][i] & 0x7FFF7FFFu)));
      }
    }
    f32x4 sum = {0.f, 0.f, 0.f, 0.f}, size = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 plus, minus, both;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t pair = x[s][i];  // (a copy: a bit cast of a vector's element takes the vector's first one)
        const uint32_t negative = __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, pair) >> 15);
        plus[i] = pair & ~negative;
        minus[i] = pair & negative;
        both[i] = pair & 0x7FFF7FFFu;
      }
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(hi[s]), as_bf16x8(plus), sum, 0, 0, 0);
      size = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(far[s]), as_bf16x8(both), size, 0, 0, 0);
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(lo[s]), as_bf16x8(minus), sum, 0, 0, 0);
    }
    // lane (column + 16c): blocks n0 + 4c .. +3 for head g0 + column
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float off = fmaf(size[r], kOff, kLeast), l = sum[r] - off, u = sum[r] + off;
      const bool fine = u - l < INFINITY;  // false too where NaN or infinite: left to exact_key
      low[r] = g0 + row < p.G && fine ? fmaxf(low[r], l) : low[r];
      high[r] = g0 + row < p.G ? (fine ? fmaxf(high[r], u) : INFINITY) : high[r];
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {  // over the heads
    low[r] = row_maximum(low[r]);
    high[r] = row_maximum(high[r]);
  }
  const float l = row == 0 ? low[0] : row == 1 ? low[1] : row == 2 ? low[2] : low[3];
  const float u = row == 0 ? high[0] : row == 1 ? high[1] : row == 2 ? high[2] : high[3];
  return (uint64_t)__builtin_bit_cast(uint32_t, u) << 32 | __builtin_bit_cast(uint32_t, l);
}

// kStore: of a whole step, whose row is written, and its block's bounds if it completes it, by the first workgroup of
// every (sequence, kv head): no score reads either, as the newest block is chosen anyway (0: neither; 1: bf16 store; 2: 8-bit).
template <int D, int kStore>
__global__ __launch_bounds__(256) void score_blocks(ChooseParams p, StoreParams store, const void* __restrict__ k_new, const void* __restrict__ v_new) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15;
  const int hkv = blockIdx.y, b = blockIdx.z;
  int part = blockIdx.x;
  if constexpr (kStore != 0) {
    if (part == 0) {
      write_and_bound<D, kStore == 2>(store, k_new, v_new, static_cast<uint16_t*>(p.bounds), b, hkv);
      return;
    }
    --part;
  }
  const int newest = step_of(p.t_per_seq, p.t, b) >> p.z_log2;
  const int n0 = (part * 4 + wave) * 16;
  if (newest < p.pick || n0 > newest - p.last) return;  // all blocks are taken; or only blocks that are taken anyway
  int phys;
  const uint64_t word = score_sixteen<D>(p, b, hkv, n0, newest, phys);
  const int mine = n0 + 4 * (lane >> 4) + row;
  if (row < 4 && mine <= newest - p.last) p.scores[((int64_t)b * p.Hkv + hkv) * p.tiles + mine] = word;
}

// Bits of a score in an order that whole numbers share; NaN above all, 0 below all.
__device__ inline uint64_t key_of(double s) {
  if (s != s) return ~(uint64_t)0;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);  // (-0 and 0 are equal)
  return u >> 63 ? ~u : u | ((uint64_t)1 << 63);
}
__device__ inline uint32_t key_of(float s) {
  const uint32_t u = __builtin_bit_cast(uint32_t, s + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// ---- choice ---------------------------------------------------------------------------------
// One workgroup per (sequence, kv head).  Of the candidates' intervals [L, U], `wanted` have an L of at least the wanted-th
// largest one, so a score below that is not chosen, and at most `wanted` scores exceed the wanted-th largest U, so a score
// above that is.  Both borders are taken a little outwards, at the edges of 512 equal parts of the intervals' range.  What
// lies between them is scored in 64 bits: at most 64 blocks in LDS, where they are ranked one by one; more (equal scores, or
// values far apart) in memory, where the border is searched for among the 64-bit keys, again by parts of their range.
// Bound by latency, 69% of it waiting: 64 of 512 blocks for 128 pairs 6.4 us, of which the kernel's beginning, the words' arrival and
// the bounds' of what is left take a half.
constexpr int kChoose = 512, kWaves = kChoose / 64, kParts = 512, kRanked = 64;
constexpr int kHeads = 16;     // query heads held in LDS
constexpr int kCached = 4096;  // intervals or keys held in LDS; more are read again from memory

__device__ inline uint64_t shfl_xor_u64(uint64_t v, int m) {
  const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)v, m), hi = (uint32_t)__shfl_xor((int)(uint32_t)(v >> 32), m);
  return (uint64_t)hi << 32 | lo;
}

// Sum of `v` over the threads before this one; `total`: over all.  (at: kWaves integers; two barriers apart from other uses.)
__device__ inline int sum_before(int v, int* at, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int all;
  int before = wave_sums<kLeft>(v, all) - v;
  if (lane == 0) at[wave] = all;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? at[w] : 0;
    total += at[w];
  }
  return before;
}

// The part that the wanted-th largest of the values counted in bins[kParts] lies in, how many lie above it, and in it.  One
// wavefront calls this; lane i has parts 8i .. 8i+7.
__device__ inline void find_part(const int* bins, int wanted, int* found) {
  const int lane = threadIdx.x & 63;
  int own[8], sum = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    own[k] = bins[8 * lane + k];
    sum += own[k];
  }
  int all;
  int above = wave_sums<kRight>(sum, all) - sum;
#pragma unroll
  for (int k = 7; k >= 0; --k) {
    if (above < wanted && above + own[k] >= wanted) {
      found[0] = 8 * lane + k;
      found[1] = above;
      found[2] = own[k];
    }
    above += own[k];
  }
}

// Score of block `phys` of the pool in 64 bits for the heads first, first + step, ..., by 16 lanes, in all of them.  ahead: the
// group's first kHeads query heads.  wild: some block's interval has no finite end, as where a product or a sum is not finite; only
// then can the smaller of a dimension's products be NaN, 0 times an infinite bound, which makes the score NaN (asked for every block
// 16 sequences of 512 blocks take 14.8 us, 14.3).
template <int D>
__device__ inline uint64_t exact_key(const ChooseParams& p, const uint16_t* ahead, int b, int hkv, int phys, bool wild, int first = 0, int step = 1) {
  const int d = 8 * (threadIdx.x & 15);
  const bool live = d < D;
  const uint16_t* const at = static_cast<const uint16_t*>(p.bounds) + ((int64_t)clamp_block(phys, p.num_blocks) * p.Hkv + hkv) * 2 * D + (live ? d : 0);
  const uint16_t* const q = static_cast<const uint16_t*>(p.q) + ((int64_t)b * p.Hq + (int64_t)hkv * p.G) * D + (live ? d : 0);
  float l[8], h[8];
  unpack8(*reinterpret_cast<const u32x4*>(at), l);
  unpack8(*reinterpret_cast<const u32x4*>(at + D), h);
  uint64_t best = 0;
  for (int g = first; g < p.G; g += step) {
    float x[8];
    unpack8(g < kHeads ? *reinterpret_cast<const u32x4*>(ahead + g * D + (live ? d : 0)) : *reinterpret_cast<const u32x4*>(q + (int64_t)g * D), x);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = x[e] < 0.f ? l[e] : h[e];  // the larger product's
      sum = fma((double)x[e], (double)m, sum);
    }
    if (wild) {
#pragma unroll 1
      for (int e = 0; e < 8; ++e) sum = __builtin_isunordered(x[e] * l[e], x[e] * h[e]) ? (double)NAN : sum;
    }
    sum = live ? sum : 0.0;
    sum += lane_move<kPairs>(sum);
    sum += lane_move<kFours>(sum);
    sum += lane_move<kEights>(sum);
    sum += lane_move<kSixteens>(sum);
    const uint64_t key = key_of(sum);
    best = key > best ? key : best;
  }
  return best;
}

struct ChooseShared {
  uint64_t cache[kCached];
  int phys[kCached];      // the candidates' blocks in the pool
  __align__(16) uint16_t q[kHeads * 128];
  int bins[2][kParts];
  float range[2][kWaves];
  uint64_t ends[2][kWaves];
  uint64_t ranked_key[kRanked];
  int ranked_at[kRanked];
  int sums[2][kWaves], found[2][3], left, sure, wild, border_at;
  uint64_t border;
};

// The border among 64-bit keys (key_at(n), n = lo .. hi): chosen are keys above cut, and of those equal to it the blocks up to
// cut_at.
template <typename Key>
__device__ void search_border(ChooseShared& sh, Key key_at, int lo, int hi, int wanted, uint64_t& cut, int& cut_at) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t least = ~(uint64_t)0, most = 0;
  for (int n = lo + tid; n <= hi; n += kChoose) {
    const uint64_t key = key_at(n);
    least = key < least ? key : least;
    most = key > most ? key : most;
  }
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    const uint64_t a = shfl_xor_u64(least, m), z = shfl_xor_u64(most, m);
    least = a < least ? a : least;
    most = z > most ? z : most;
  }
  if (lane == 0) {
    sh.ends[0][wave] = least;
    sh.ends[1][wave] = most;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    least = sh.ends[0][w] < least ? sh.ends[0][w] : least;
    most = sh.ends[1][w] > most ? sh.ends[1][w] : most;
  }
  int count = hi - lo + 1;  // candidates in least .. most
  while (least != most && count != wanted) {
    const int bits = 64 - __clzll((long long)(most - least));
    const int shift = bits > 9 ? bits - 9 : 0;
    sh.bins[0][tid] = 0;
    __syncthreads();
    for (int n = lo + tid; n <= hi; n += kChoose) {
      const uint64_t key = key_at(n);
      if (key >= least && key <= most) atomicAdd(&sh.bins[0][(key - least) >> shift], 1);
    }
    __syncthreads();
    if (wave == 0) find_part(sh.bins[0], wanted, sh.found[0]);
    __syncthreads();
    least += (uint64_t)sh.found[0][0] << shift;
    const uint64_t width = ((uint64_t)1 << shift) - 1;
    most = most - least > width ? least + width : most;
    wanted -= sh.found[0][1];
    count = sh.found[0][2];
    __syncthreads();  // found and bins are written again
  }
  cut = least;
  cut_at = INT32_MAX;  // all that are left
  if (count != wanted) {  // one value: the first `wanted` blocks that have it
    const int each = (hi - lo + kChoose) / kChoose, n0 = lo + tid * each;
    int mine = 0, all;
    for (int n = n0; n < n0 + each && n <= hi; ++n) mine += key_at(n) == least;
    int before = sum_before(mine, sh.sums[0], all);
    for (int n = n0; n < n0 + each && n <= hi; ++n) {
      if (key_at(n) == least && ++before == wanted) sh.border_at = n;
    }
    __syncthreads();
    cut_at = sh.border_at;
  }
}

// kScore: few blocks, which the workgroup scores itself; with kStore (score_blocks) as many workgroups more write the rows.
template <int D, bool kScore, int kStore>
__global__ __launch_bounds__(kChoose) void choose_blocks(ChooseParams p, StoreParams store, const void* __restrict__ k_new, const void* __restrict__ v_new) {
  __shared__ ChooseShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.y;
  int hkv = blockIdx.x;
  if constexpr (kStore != 0) {
    if (hkv >= p.Hkv) {
      write_and_bound<D, kStore == 2>(store, k_new, v_new, static_cast<uint16_t*>(p.bounds), b, hkv - p.Hkv);
      return;
    }
  }
  const int newest = step_of(p.t_per_seq, p.t, b) >> p.z_log2;
  const int64_t pair = (int64_t)b * p.Hkv + hkv;
  uint64_t* const scores = p.scores + pair * p.tiles;
  int32_t* const out = p.selected + pair * p.pick;
  const int32_t* const table = p.block_table + (int64_t)b * p.max_blocks_per_seq;
  if (newest < p.pick) {  // all of them
    for (int i = tid; i < p.pick; i += kChoose) out[i] = i <= newest ? i : -1;
    return;
  }
  for (int i = tid; i < (p.G < kHeads ? p.G : kHeads) * (D / 8); i += kChoose)
    reinterpret_cast<u32x4*>(sh.q)[i] = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.q) + ((int64_t)b * p.Hq + (int64_t)hkv * p.G) * D)[i];
  const int lo = p.first, hi = newest - p.last;     // candidates
  const int wanted = p.pick - p.first - p.last;     // of them; fewer than there are
  const bool cached = kScore || hi - lo < kCached;
  auto word_at = [&](int n) { return cached ? sh.cache[n - lo] : scores[n]; };
  auto phys_at = [&](int n) { return cached ? sh.phys[n - lo] : table[n]; };
  auto interval = [&](uint64_t w) {
    return Interval{__builtin_bit_cast(float, (uint32_t)w), __builtin_bit_cast(float, (uint32_t)(w >> 32))};
  };
  constexpr uint32_t kNone = ~0u - 1, kSure = ~0u;  // keys beyond all values': no border; of a block that has been found chosen
  uint32_t sure_above = kNone, open_from = kSure;   // keys of U's outer border and L's
  bool by_key = false;                         // words are 64-bit keys
  uint64_t cut = ~(uint64_t)0;
  int cut_at = -1, open = 0, open_taken = 0;
  auto sure = [&](uint64_t w) { return key_of(interval(w).lo) > sure_above; };
  auto undecided = [&](uint64_t w) { return key_of(interval(w).hi) >= open_from && key_of(interval(w).lo) <= sure_above; };
  if (wanted > 0) {
    if constexpr (kScore) {
      for (int n0 = 16 * wave; n0 <= hi; n0 += 16 * kWaves) {
        int phys;
        const uint64_t word = score_sixteen<D>(p, b, hkv, n0, newest, phys);
        const int row = lane & 15, mine = n0 + 4 * (lane >> 4) + row;
        if (row < 4 && mine >= lo && mine <= hi) sh.cache[mine - lo] = word;
        if (lane < 16 && n0 + lane >= lo && n0 + lane <= hi) sh.phys[n0 + lane - lo] = phys;
      }
      __syncthreads();
    }
    float bottom = -INFINITY, top = -INFINITY;  // the largest finite -L and U
    for (int n = lo + tid; n <= hi; n += kChoose) {
      const uint64_t w = kScore ? sh.cache[n - lo] : scores[n];
      if (!kScore && cached) {
        sh.cache[n - lo] = w;
        sh.phys[n - lo] = table[n];
      }
      const Interval v = interval(w);
      bottom = v.lo > -INFINITY ? fmaxf(bottom, -v.lo) : bottom;
      top = v.hi < INFINITY ? fmaxf(top, v.hi) : top;
    }
    bottom = wave_max(bottom);
    top = wave_max(top);
    if (lane == 0) {
      sh.range[0][wave] = bottom;
      sh.range[1][wave] = top;
    }
    sh.bins[0][tid] = sh.bins[1][tid] = 0;
    if (tid == 0) sh.left = sh.sure = sh.wild = 0;
    if (tid < kRanked) sh.ranked_key[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      bottom = fmaxf(bottom, sh.range[0][w]);
      top = fmaxf(top, sh.range[1][w]);
    }
    const uint32_t least = key_of(-bottom), highest = key_of(top), most = highest < least ? least : highest;
    const int bits = most == least ? 0 : 32 - __clz((int)(most - least));
    const int shift = bits > 9 ? bits - 9 : 0;
    auto part = [&](uint32_t key) { return key <= least ? 0 : ((key < most ? key : most) - least) >> shift; };
    for (int n = lo + tid; n <= hi; n += kChoose) {
      const Interval v = interval(word_at(n));
      atomicAdd(&sh.bins[0][part(key_of(v.lo))], 1);
      atomicAdd(&sh.bins[1][part(key_of(v.hi))], 1);
    }
    __syncthreads();
    if (wave < 2) find_part(sh.bins[wave], wanted, sh.found[wave]);
    __syncthreads();
    // (the first part holds whatever lies below it, the last one whatever lies above)
    open_from = sh.found[0][0] == 0 ? 0u : least + ((uint32_t)sh.found[0][0] << shift);
    const uint32_t past = least + ((uint32_t)(sh.found[1][0] + 1) << shift);  // first key of the next part
    sure_above = sh.found[1][0] == (int)part(most) ? kNone : past - 1;
    int sures = 0;  // of the wavefront
    for (int n = lo + tid; n <= hi; n += kChoose) {
      const uint64_t w = word_at(n);
      sures += __popcll(__ballot(sure(w)));
      if (undecided(w)) {
        const int i = atomicAdd(&sh.left, 1);  // (in any order: ranks do not depend on it)
        if (i < kRanked) sh.ranked_at[i] = n;
        if (interval(w).hi == INFINITY) sh.wild = 1;
      }
    }
    if (lane == 0 && sures) atomicAdd(&sh.sure, sures);  // (lane 0 is in every round that the wavefront is in)
    __syncthreads();
    open = sh.left;
    const bool wild = sh.wild;
    open_taken = wanted - sh.sure;
    if (open > kRanked) {
      // keys instead of intervals: decided blocks above or below all others
      for (int i = tid >> 4; i <= hi - lo; i += kChoose / 16) {
        const uint64_t w = word_at(lo + i);
        uint64_t key = sure(w) ? ~(uint64_t)0 : 0;
        if (undecided(w)) key = exact_key<D>(p, sh.q, b, hkv, phys_at(lo + i), wild);
        if ((lane & 15) == 0) {
          scores[lo + i] = key;
          if (cached) sh.cache[i] = key;
        }
      }
      __syncthreads();
      by_key = true;
      search_border(sh, word_at, lo, hi, wanted, cut, cut_at);
    } else if (open != open_taken) {
      // a block's heads are shared out among as many groups of 16 lanes as there are (64 heads, 4 sequences of 192 blocks: 24.6 -> 12 us)
      const int share = open <= 2 ? 16 : open <= 4 ? 8 : open <= 8 ? 4 : open <= 16 ? 2 : 1;
      for (int i = tid >> 4; i < open * share; i += kChoose / 16) {
        const int at = i / share, first = i % share;
        if (first >= p.G) continue;
        const uint64_t key = exact_key<D>(p, sh.q, b, hkv, phys_at(sh.ranked_at[at]), wild, first, share);
        if ((lane & 15) == 0) atomicMax(reinterpret_cast<unsigned long long*>(&sh.ranked_key[at]), (unsigned long long)key);
      }
      __syncthreads();
      if (tid < open) {
        const uint64_t key = sh.ranked_key[tid];
        const int n = sh.ranked_at[tid];
        int rank = 0;
        for (int i = 0; i < open; ++i) rank += sh.ranked_key[i] > key || (sh.ranked_key[i] == key && sh.ranked_at[i] < n);
        if (rank < open_taken) {
          if (cached) sh.cache[n - lo] = 0x7FFFFFFFu;  // (key_of() of that is kSure)
          else scores[n] = 0x7FFFFFFFu;
        }
      }
      __syncthreads();
    }
  }
  // In ascending order.
  auto chosen = [&](int n) {
    if (n > newest) return false;
    if (n < lo || n > hi) return true;
    if (wanted == 0) return false;
    const uint64_t w = word_at(n);
    if (by_key) return w > cut || (w == cut && n <= cut_at);
    return sure(w) || (open == open_taken && undecided(w));
  };
  int place = 0;
  for (int n0 = 0, round = 0; n0 <= newest; n0 += kChoose, round ^= 1) {
    const bool take = chosen(n0 + tid);
    const uint64_t takes = __ballot(take);
    if (lane == 0) sh.sums[round][wave] = __popcll(takes);
    __syncthreads();  // (the other round's sums are written before, read after it)
    int before = place + __popcll(takes & (((uint64_t)1 << lane) - 1));
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      before += w < wave ? sh.sums[round][w] : 0;
      place += sh.sums[round][w];
    }
    if (take && before < p.pick) out[before] = n0 + tid;
  }
}

}  // namespace

hipError_t launch_block_bounds(const StoreParams& p, void* bounds, int D, int dtype, hipStream_t stream) {
  // blocks that `count` steps touch: known for a uniform first step, else at most one more than they fill
  const int64_t Z = (int64_t)1 << p.z_log2;
  const int64_t blocks = p.t_per_seq ? (p.count - 1) / Z + 2 : (p.t + (int64_t)p.count - 1) / Z - p.t / Z + 1;
  const dim3 grid((unsigned)blocks, (unsigned)p.Hkv, (unsigned)p.batch);
  uint16_t* const to = static_cast<uint16_t*>(bounds);
  if (dtype == TEMPO_E4M3) {
    if (D == 128) return launch((block_bounds<128, true>), grid, dim3(128), 0, stream, p, to);
    return launch((block_bounds<64, true>), grid, dim3(64), 0, stream, p, to);
  }
  if (D == 128) return launch((block_bounds<128, false>), grid, dim3(256), 0, stream, p, to);
  return launch((block_bounds<64, false>), grid, dim3(128), 0, stream, p, to);
}

// Does the workgroup that chooses also score, a launch less?  It streams the bounds of its blocks alone, so they must be few (us, two
// launches / one, 24/8 heads of 128: 1 sequence of 16 blocks 8.5 / 6.2, 128 blocks 8.6 / 7.4, 192 blocks 8.4 / 8.6, 512 blocks 9.4 / 15;
// 16 sequences of 192 blocks 11.0 / 9.4; 64/1 heads, 4 sequences of 80 blocks 10.2 / 8.9, 192 blocks 12 / 14); and with rows to write,
// whose workgroups are as many more and as large, the pairs too (steps of 64 sequences of 192 blocks 55 / 59).
inline bool scores_itself(const ChooseParams& p, int batch, bool writes) {
  return p.tiles <= (p.G <= kHeads ? 192 : 96) && !(writes && (int64_t)batch * p.Hkv > 256);
}

// k_new, v_new: null, or the rows of the step, which are written (and bounded) by the first launch.
template <int D, int kStore>
static hipError_t launch_select(const ChooseParams& p, const StoreParams& store, const void* k_new, const void* v_new, int batch, hipStream_t stream) {
  // (no sequence has more blocks than are taken: nothing to score)
  const int parts = p.tiles > p.pick && p.pick > p.first + p.last ? (p.tiles + 63) / 64 : 0;
  if (scores_itself(p, batch, kStore != 0)) {
    const dim3 grid((unsigned)(p.Hkv * (kStore != 0 ? 2 : 1)), (unsigned)batch);
    return launch((choose_blocks<D, true, kStore>), grid, dim3(kChoose), 0, stream, p, store, k_new, v_new);
  }
  const int workgroups = parts + (kStore != 0 ? 1 : 0);
  if (workgroups > 0) {
    const dim3 grid((unsigned)workgroups, (unsigned)p.Hkv, (unsigned)batch);
    const hipError_t e = launch((score_blocks<D, kStore>), grid, dim3(256), 0, stream, p, store, k_new, v_new);
    if (e != hipSuccess) return e;
  }
  return launch((choose_blocks<D, false, 0>), dim3((unsigned)p.Hkv, (unsigned)batch), dim3(kChoose), 0, stream, p, store, nullptr, nullptr);
}

hipError_t launch_select_blocks(const ChooseParams& p, const StoreParams* store, const void* k_new, const void* v_new, int batch, int D, int dtype,
                                hipStream_t stream) {
  const StoreParams none = {};
  if (!store) return D == 128 ? launch_select<128, 0>(p, none, nullptr, nullptr, batch, stream) : launch_select<64, 0>(p, none, nullptr, nullptr, batch, stream);
  if (dtype == TEMPO_E4M3) return D == 128 ? launch_select<128, 2>(p, *store, k_new, v_new, batch, stream) : launch_select<64, 2>(p, *store, k_new, v_new, batch, stream);
  return D == 128 ? launch_select<128, 1>(p, *store, k_new, v_new, batch, stream) : launch_select<64, 1>(p, *store, k_new, v_new, batch, stream);
}

}  // namespace tempo
