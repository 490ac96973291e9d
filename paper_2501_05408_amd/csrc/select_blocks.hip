// Sparse attention's choice of blocks: bounds of the keys of every block, a score of every block for a query, and the
// blocks with the best scores.
//
//   bounds   lo_d = min_j k_jd, hi_d = max_j k_jd over the keys j of a block (of one kv head), once it is complete
//   score    S_n = max over the group's heads g of sum_d max(q_gd lo_d, q_gd hi_d): no key of block n has a larger
//            product with any of the group's queries
//   choice   the first `first` blocks, the `last` newest ones (the newest may be incomplete: it has no bounds yet), and
//            of the others those with the largest S_n, `pick` blocks in all; of equal scores the earlier block
//
// Scores are summed in 64 bits.  A product of two bf16 values is exact in fp32 and the sum of such products is exact, or
// 1e-16 off, in fp64, so that the choice is that of the formula whatever the order of the sums; in fp32 blocks whose
// scores lie within 1e-6 of the border would be chosen by rounding.
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
  v = f(v, __builtin_bit_cast(i16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true)));
  v = f(v, __builtin_bit_cast(i16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true)));
  v = f(v, __builtin_bit_cast(i16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x141, 0xF, 0xF, true)));
  return f(v, __builtin_bit_cast(i16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x140, 0xF, 0xF, true)));
}

// Bounds of the block of one kv head whose first slot has number `first` among the store's; wavefronts w < D/64 (8-bit store)
// or D/32 (bf16) read the 1 KiB units of their part of the dims, 16 or 8 of them a lane.  Lane (row + 16c) goes through the
// rows row, 16 + row, ... of the block, then the 16 lanes of equal c are reduced.  fresh: the block's last row is not in the
// store yet; the lane's part of it is in `last` (8 bits: codes, with scale byte last_scale).
// Bound by memory, as long as the comparisons are whole words' (8 x 4096 keys of 4 heads of 128 in blocks of 64, 34 MB:
// 7.4 us; one value at a time in fp32 10.2).
template <int D, bool k8>
__device__ __forceinline__ void bounds_of_block(const StoreParams& p, int64_t first, int w, int lane, uint16_t* __restrict__ to, bool fresh, u32x4 last,
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
    for (int r = 0; r < 2; ++r) u[r] = *reinterpret_cast<const u32x4*>(at + (int64_t)(2 * t + r) * PER_TILE * 1024);
    if constexpr (k8) both = *reinterpret_cast<const uint16_t*>(scales + 32 * t);
    if (fresh && t == groups - 1 && (lane & 15) == 15) {
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
  bounds_of_block<D, k8>(p, pair << p.z_log2, threadIdx.x >> 6, threadIdx.x & 63, bounds + pair * 2 * D, false, u32x4{0u, 0u, 0u, 0u}, 0u);
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
  if (wave < (k8 ? D / 64 : D / 32)) bounds_of_block<D, k8>(p, first, wave, lane, bounds + pair * 2 * D, true, last, last_scale);
}

// Bits of a score in an order that whole numbers share; NaN above all.
__device__ inline uint64_t key_of(double s) {
  if (s != s) return ~(uint64_t)0;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);  // (-0 and 0 are equal)
  return u >> 63 ? ~u : u | ((uint64_t)1 << 63);
}

// A wavefront scores 16 blocks: lane (row + 16c) holds dims 32s + 8c .. +7 of block `row`.
// kStore: of a whole step, whose row is written, and its block's bounds if it completes it, by the first workgroup of
// every (sequence, kv head): no score reads either, as the newest block is chosen anyway (0: neither; 1: bf16 store; 2: 8-bit).
template <int D, int kStore>
__global__ __launch_bounds__(256) void score_blocks(ChooseParams p, StoreParams store, const void* __restrict__ k_new, const void* __restrict__ v_new) {
  constexpr int KS = D / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, c = lane >> 4;
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
  const int n = n0 + row <= newest - p.last ? n0 + row : n0;
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + n], p.num_blocks);
  const uint16_t* const at = static_cast<const uint16_t*>(p.bounds) + ((int64_t)phys * p.Hkv + hkv) * 2 * D + 8 * c;
  u32x4 lo[KS], hi[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    lo[s] = *reinterpret_cast<const u32x4*>(at + 32 * s);
    hi[s] = *reinterpret_cast<const u32x4*>(at + D + 32 * s);
  }
  const uint16_t* const q = static_cast<const uint16_t*>(p.q) + ((int64_t)b * p.Hq + (int64_t)hkv * p.G) * D + 8 * c;
  u32x4 u[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) u[s] = *reinterpret_cast<const u32x4*>(q + 32 * s);
  float l[8 * KS], h[8 * KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    unpack8(lo[s], l + 8 * s);
    unpack8(hi[s], h + 8 * s);
  }
  uint64_t best = 0;
  for (int g = 0; g < p.G; ++g) {
    u32x4 now[KS];
    const int ahead = g + 1 < p.G ? g + 1 : g;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      now[s] = u[s];
      u[s] = *reinterpret_cast<const u32x4*>(q + (int64_t)ahead * D + 32 * s);
    }
    double sums[2] = {0.0, 0.0};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float x[8];
      unpack8(now[s], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float m = x[e] < 0.f ? l[8 * s + e] : h[8 * s + e];  // the larger product's
        sums[e & 1] = fma((double)x[e], (double)m, sums[e & 1]);   // (NaN where a bound is)
      }
    }
    double sum = sums[0] + sums[1];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const uint64_t key = key_of(sum);
    best = key > best ? key : best;
  }
  if (c == 0 && n0 + row <= newest - p.last) p.scores[((int64_t)b * p.Hkv + hkv) * p.tiles + n0 + row] = best;
}

// ---- choice ---------------------------------------------------------------------------------
// One workgroup per (sequence, kv head).  The border, the m-th largest key of the candidates: keys are counted in 512 equal
// parts of their range, then of the part that the border lies in, until at most 64 keys are left, which are ranked one by
// one, or the part holds a single value.  Then the chosen blocks in ascending order.  (Counting by the keys' bytes from the
// top down, 256 parts at a time, takes three or four rounds, as scores of one sign share their first byte.)
constexpr int kChoose = 512, kWaves = kChoose / 64, kParts = 512, kRanked = 64;
constexpr int kCached = 4096;  // keys held in LDS; more are read again from memory

__device__ inline uint64_t shfl_xor_u64(uint64_t v, int m) {
  const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)v, m), hi = (uint32_t)__shfl_xor((int)(uint32_t)(v >> 32), m);
  return (uint64_t)hi << 32 | lo;
}

// Sum of `v` over the threads before this one; `total`: over all.  (at: kWaves integers; two barriers apart from other uses.)
__device__ inline int sum_before(int v, int* at, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = v;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(sum, m);
    sum += lane >= m ? o : 0;
  }
  if (lane == 63) at[wave] = sum;
  __syncthreads();
  int before = sum - v;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? at[w] : 0;
    total += at[w];
  }
  return before;
}

__global__ __launch_bounds__(kChoose) void choose_blocks(ChooseParams p) {
  __shared__ uint64_t cache[kCached];
  __shared__ int bins[kParts];
  __shared__ uint64_t ends[2][kWaves];
  __shared__ uint64_t ranked_key[kRanked];
  __shared__ int ranked_at[kRanked];
  __shared__ int sums[2][kWaves], found[3], left, border_at;
  __shared__ uint64_t border;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.y;
  const int newest = step_of(p.t_per_seq, p.t, b) >> p.z_log2;
  const int64_t pair = (int64_t)b * p.Hkv + blockIdx.x;
  const uint64_t* const scores = p.scores + pair * p.tiles;
  int32_t* const out = p.selected + pair * p.pick;
  if (newest < p.pick) {  // all of them
    for (int i = tid; i < p.pick; i += kChoose) out[i] = i <= newest ? i : -1;
    return;
  }
  const int lo = p.first, hi = newest - p.last;  // candidates
  int wanted = p.pick - p.first - p.last;        // of them; fewer than there are
  const bool cached = hi - lo < kCached;
  auto key_at = [&](int n) { return cached ? cache[n - lo] : scores[n]; };
  // Chosen are the candidates with keys above cut, and of those with keys equal to it the ones up to cut_at.
  uint64_t cut = ~(uint64_t)0;
  int cut_at = -1;
  if (wanted > 0) {
    uint64_t least = ~(uint64_t)0, most = 0;
    for (int n = lo + tid; n <= hi; n += kChoose) {
      const uint64_t key = scores[n];
      if (cached) cache[n - lo] = key;
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
      ends[0][wave] = least;
      ends[1][wave] = most;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      least = ends[0][w] < least ? ends[0][w] : least;
      most = ends[1][w] > most ? ends[1][w] : most;
    }
    int count = hi - lo + 1;  // candidates in least .. most
    while (count > kRanked && least != most && count != wanted) {
      const int bits = 64 - __clzll((long long)(most - least));
      const int shift = bits > 9 ? bits - 9 : 0;
      bins[tid] = 0;
      __syncthreads();
      for (int n = lo + tid; n <= hi; n += kChoose) {
        const uint64_t key = key_at(n);
        if (key >= least && key <= most) atomicAdd(&bins[(key - least) >> shift], 1);
      }
      __syncthreads();
      if (wave == 0) {  // lane i: parts 8i .. 8i+7, and how many keys lie above those
        int own[8], sum = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          own[k] = bins[8 * lane + k];
          sum += own[k];
        }
        int above = sum;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
          const int o = __shfl_down(above, m);
          above += lane + m < 64 ? o : 0;
        }
        above -= sum;
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
      __syncthreads();
      least += (uint64_t)found[0] << shift;
      const uint64_t width = ((uint64_t)1 << shift) - 1;
      most = most - least > width ? least + width : most;
      wanted -= found[1];
      count = found[2];
      __syncthreads();  // found and bins are written again
    }
    if (count == wanted) {  // all that are left
      cut = least;
      cut_at = INT32_MAX;
    } else if (least == most) {  // one value: the first `wanted` blocks that have it
      cut = least;
      const int each = (hi - lo + kChoose) / kChoose, n0 = lo + tid * each;
      int mine = 0, all;
      for (int n = n0; n < n0 + each && n <= hi; ++n) mine += key_at(n) == least;
      int before = sum_before(mine, sums[0], all);
      for (int n = n0; n < n0 + each && n <= hi; ++n) {
        if (key_at(n) == least && ++before == wanted) border_at = n;
      }
      __syncthreads();
      cut_at = border_at;
    } else {  // few: the one that wanted - 1 of them come before
      if (tid == 0) left = 0;
      __syncthreads();
      for (int n = lo + tid; n <= hi; n += kChoose) {
        const uint64_t key = key_at(n);
        if (key >= least && key <= most) {
          const int i = atomicAdd(&left, 1);  // (in any order: ranks do not depend on it)
          ranked_key[i] = key;
          ranked_at[i] = n;
        }
      }
      __syncthreads();
      if (tid < count) {
        const uint64_t key = ranked_key[tid];
        const int n = ranked_at[tid];
        int rank = 0;
        for (int i = 0; i < count; ++i) rank += ranked_key[i] > key || (ranked_key[i] == key && ranked_at[i] < n);
        if (rank == wanted - 1) {
          border = key;
          border_at = n;
        }
      }
      __syncthreads();
      cut = border;
      cut_at = border_at;
    }
  }
  // In ascending order: every thread the blocks of one run.
  const int each = (newest + kChoose) / kChoose, n0 = tid * each;
  auto chosen = [&](int n) {
    if (n > newest) return false;
    if (n < lo || n > hi) return true;
    const uint64_t key = key_at(n);
    return key > cut || (key == cut && n <= cut_at);
  };
  int mine = 0, all;
  for (int n = n0; n < n0 + each; ++n) mine += chosen(n);
  int place = sum_before(mine, sums[1], all);
  for (int n = n0; n < n0 + each; ++n) {
    if (chosen(n) && place < p.pick) out[place++] = n;
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

// k_new, v_new: null, or the rows of the step, which are written (and bounded) by the same launch.
template <int D, int kStore>
static hipError_t launch_score(const ChooseParams& p, const StoreParams& store, const void* k_new, const void* v_new, int batch, hipStream_t stream) {
  // (no sequence has more blocks than are taken: nothing to score)
  const int parts = p.tiles > p.pick && p.pick > p.first + p.last ? (p.tiles + 63) / 64 : 0;
  const int workgroups = parts + (kStore != 0 ? 1 : 0);
  if (workgroups == 0) return hipSuccess;
  return launch((score_blocks<D, kStore>), dim3((unsigned)workgroups, (unsigned)p.Hkv, (unsigned)batch), dim3(256), 0, stream, p, store, k_new, v_new);
}

hipError_t launch_select_blocks(const ChooseParams& p, const StoreParams* store, const void* k_new, const void* v_new, int batch, int D, int dtype,
                                hipStream_t stream) {
  const StoreParams none = {};
  hipError_t e;
  if (!store) e = D == 128 ? launch_score<128, 0>(p, none, nullptr, nullptr, batch, stream) : launch_score<64, 0>(p, none, nullptr, nullptr, batch, stream);
  else if (dtype == TEMPO_E4M3) e = D == 128 ? launch_score<128, 2>(p, *store, k_new, v_new, batch, stream) : launch_score<64, 2>(p, *store, k_new, v_new, batch, stream);
  else e = D == 128 ? launch_score<128, 1>(p, *store, k_new, v_new, batch, stream) : launch_score<64, 1>(p, *store, k_new, v_new, batch, stream);
  if (e != hipSuccess) return e;
  return launch(choose_blocks, dim3((unsigned)p.Hkv, (unsigned)batch), dim3(kChoose), 0, stream, p);
}

}  // namespace tempo
