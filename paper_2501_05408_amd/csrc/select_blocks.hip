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

// Smaller / larger of two values; NaN if one is.
__device__ inline float min_nan(float m, float x) { return x < m || x != x ? x : m; }
__device__ inline float max_nan(float m, float x) { return x > m || x != x ? x : m; }

// One workgroup per (block of a sequence, kv head); wavefront w reads the 1 KiB units of its part of the dims: in a bf16
// store 8 dims a lane (unit s = w of each row-tile), in an 8-bit store 16.  Lane (row + 16c) goes through the rows
// row, 16 + row, ... of the block, then the 16 lanes of equal c are reduced.
template <int D, bool k8>
__global__ __launch_bounds__(k8 ? D : 2 * D) void block_bounds(StoreParams p, uint16_t* __restrict__ bounds) {
  constexpr int PER_TILE = k8 ? D / 64 : D / 32;  // units of a row-tile
  constexpr int N = k8 ? 16 : 8;                  // dims a lane holds
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int head = blockIdx.y, b = blockIdx.z;
  const int t_b = step_of(p.t_per_seq, p.t, b);
  int rows = p.count;
  if (p.count_per_seq) rows = p.count_per_seq[b] < rows ? p.count_per_seq[b] : rows;
  const int n = (t_b >> p.z_log2) + (int)blockIdx.x;           // block of the sequence
  const int64_t last = (((int64_t)n + 1) << p.z_log2) - 1;     // its last step
  if (last < t_b || last > (int64_t)t_b + rows - 1) return;    // not completed by the call's steps; uniform
  const int phys = clamp_block(p.block_table[(int64_t)b * p.max_blocks_per_seq + (n & p.tile_mask)], p.num_blocks);
  const int64_t pair = (int64_t)phys * p.Hkv + head, first = pair << p.z_log2;
  const char* const at = static_cast<const char*>(p.k_pool) + first * (k8 ? D : 2 * D) + w * 1024 + lane * 16;
  const uint8_t* const scales = static_cast<const uint8_t*>(p.k_pool) + ((((int64_t)p.num_blocks * p.Hkv) << p.z_log2) * D + first);
  float lo[N], hi[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    lo[i] = INFINITY;
    hi[i] = -INFINITY;
  }
  const int tiles = 1 << (p.z_log2 - 4);
#pragma unroll 4
  for (int t = 0; t < tiles; ++t) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(at + (int64_t)t * PER_TILE * 1024);
    float x[N];
    if constexpr (k8) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const float scale = scale_of(scales[scale_off_k(16 * t + (lane & 15))]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], scale, false);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[i], scale, true);
        x[4 * i] = (float)a[0]; x[4 * i + 1] = (float)a[1]; x[4 * i + 2] = (float)c[0]; x[4 * i + 3] = (float)c[1];
      }
    } else {
      unpack8(u, x);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      lo[i] = min_nan(lo[i], x[i]);
      hi[i] = max_nan(hi[i], x[i]);
    }
  }
#pragma unroll
  for (int m = 8; m > 0; m >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      lo[i] = min_nan(lo[i], __shfl_xor(lo[i], m));
      hi[i] = max_nan(hi[i], __shfl_xor(hi[i], m));
    }
  }
  if ((lane & 15) != 0) return;
  const int c = lane >> 4;
  uint16_t* const to = bounds + pair * 2 * D;
#pragma unroll
  for (int h = 0; h < N / 8; ++h) {
    const int d = k8 ? 64 * w + 32 * h + 8 * c : 32 * w + 8 * c;
    *reinterpret_cast<u32x4*>(to + d) = pack8(lo + 8 * h);
    *reinterpret_cast<u32x4*>(to + D + d) = pack8(hi + 8 * h);
  }
}

// Bits of a score in an order that whole numbers share; NaN above all.
__device__ inline uint64_t key_of(double s) {
  if (s != s) return ~(uint64_t)0;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);  // (-0 and 0 are equal)
  return u >> 63 ? ~u : u | ((uint64_t)1 << 63);
}

// A wavefront scores 16 blocks: lane (row + 16c) holds dims 32s + 8c .. +7 of block `row`.
template <int D>
__global__ __launch_bounds__(256) void score_blocks(ChooseParams p) {
  constexpr int KS = D / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, c = lane >> 4;
  const int hkv = blockIdx.y, b = blockIdx.z;
  const int newest = step_of(p.t_per_seq, p.t, b) >> p.z_log2;
  const int n0 = ((int)blockIdx.x * 4 + wave) * 16;
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
  uint64_t best = 0;
  for (int g = 0; g < p.G; ++g) {
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const u32x4 u = *reinterpret_cast<const u32x4*>(q + g * D + 32 * s);
      float x[8], l[8], h[8];
      unpack8(u, x);
      unpack8(lo[s], l);
      unpack8(hi[s], h);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = x[e] * l[e], z = x[e] * h[e];  // exact
        sum += (double)max_nan(a, z);
      }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const uint64_t key = key_of(sum);
    best = key > best ? key : best;
  }
  if (c == 0 && n0 + row <= newest - p.last) p.scores[((int64_t)b * p.Hkv + hkv) * p.tiles + n0 + row] = best;
}

// One workgroup per (sequence, kv head).  The m-th largest key of the candidates by its bytes from the top down: a
// histogram of the next byte over the keys that share the bytes found so far.  Then the blocks in ascending order.
constexpr int kChoose = 256;

__global__ __launch_bounds__(kChoose) void choose_blocks(ChooseParams p) {
  __shared__ int bins[256];
  __shared__ int at_wave[2][kChoose / 64];
  __shared__ int found[3];  // next byte; keys above it; keys that have it
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
  uint64_t prefix = 0, mask = 0;
  if (wanted > 0) {
    for (int shift = 56; shift >= 0; shift -= 8) {
      bins[tid] = 0;
      __syncthreads();
      for (int n = lo + tid; n <= hi; n += kChoose) {
        const uint64_t key = scores[n];
        if ((key & mask) == prefix) atomicAdd(&bins[(key >> shift) & 255u], 1);
      }
      __syncthreads();
      if (wave == 0) {  // lane i: bins 4i .. 4i+3; how many keys lie in higher bins than those
        int own[4], sum = 0;
        for (int k = 0; k < 4; ++k) {
          own[k] = bins[4 * lane + k];
          sum += own[k];
        }
        int above = sum;
        for (int m = 1; m < 64; m <<= 1) {
          const int o = __shfl_down(above, m);
          above += lane + m < 64 ? o : 0;
        }
        above -= sum;
        for (int k = 3; k >= 0; --k) {
          if (above < wanted && above + own[k] >= wanted) {
            found[0] = 4 * lane + k;
            found[1] = above;
            found[2] = own[k];
          }
          above += own[k];
        }
      }
      __syncthreads();
      prefix |= (uint64_t)found[0] << shift;
      mask |= (uint64_t)255 << shift;
      wanted -= found[1];
      const bool all = found[2] == wanted;  // every key that begins so is taken
      __syncthreads();                      // bins and found are written again
      if (all) break;
    }
  }
  // Keys whose top bytes exceed `prefix` are taken, of those that share them the first `wanted`.
  int taken = 0, equal = 0;
  for (int n0 = 0; n0 <= newest; n0 += kChoose) {
    const int n = n0 + tid;
    const bool candidate = n >= lo && n <= hi && p.pick > p.first + p.last;
    const uint64_t key = candidate ? scores[n] & mask : 0;
    const bool tie = candidate && key == prefix;
    const uint64_t ties = __ballot(tie);
    if (lane == 0) at_wave[0][wave] = __popcll(ties);
    __syncthreads();
    int before = equal;
    for (int w = 0; w < wave; ++w) before += at_wave[0][w];
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    before += __popcll(ties & below);
    const bool take = n <= newest && (n < lo || n > hi || (candidate && key > prefix) || (tie && before < wanted));
    const uint64_t takes = __ballot(take);
    if (lane == 0) at_wave[1][wave] = __popcll(takes);
    __syncthreads();
    int place = taken;
    for (int w = 0; w < wave; ++w) place += at_wave[1][w];
    place += __popcll(takes & below);
    if (take && place < p.pick) out[place] = n;
    for (int w = 0; w < kChoose / 64; ++w) {
      equal += at_wave[0][w];
      taken += at_wave[1][w];
    }
    __syncthreads();
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

hipError_t launch_select_blocks(const ChooseParams& p, int batch, int D, hipStream_t stream) {
  // (no sequence has more blocks than are taken: nothing to score)
  if (p.tiles > p.pick && p.pick > p.first + p.last) {
    const dim3 grid((unsigned)((p.tiles + 63) / 64), (unsigned)p.Hkv, (unsigned)batch);
    const hipError_t e = D == 128 ? launch(score_blocks<128>, grid, dim3(256), 0, stream, p) : launch(score_blocks<64>, grid, dim3(256), 0, stream, p);
    if (e != hipSuccess) return e;
  }
  return launch(choose_blocks, dim3((unsigned)p.Hkv, (unsigned)batch), dim3(kChoose), 0, stream, p);
}

}  // namespace tempo
