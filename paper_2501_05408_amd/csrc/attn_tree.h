// The ancestors of a tree's rows, as bits, from their parents.
//
// parents[i] of row i is a row before it, or anything else: none (a child of the last step before the tree).  With
// A_i = {i} u A_parent(i), doubling: after r rounds a_i holds row i and its 2^r - 1 nearest ancestors, and up_i is the one
// behind them; a round sets a_i |= a_(up_i), up_i = up_(up_i).  log2(depth) rounds of a few LDS reads instead of one read an ancestor.
#pragma once

#include "attn_bf16_common.h"
#include "attn_spans.h"

namespace tempo {

// Words of a row's bits, and of its place in LDS (odd, so that the rows of a wavefront's columns lie in different banks).
__host__ __device__ inline int tree_words(int rows) { return (rows + 31) >> 5; }
__host__ __device__ inline int tree_stride(int rows) { return tree_words(rows) | 1; }
// Bits, ranks above, depths.
inline size_t tree_lds_bytes(int rows) { return (size_t)rows * (tree_stride(rows) + 2) * sizeof(uint32_t); }

namespace {

// Logits that this lane's column does not see become -inf.  bits: of the group's slots, those of the row's ancestors.
template <bool kTree>
__device__ __forceinline__ void mask_span(int key, int lo, int hi, int sinks, uint32_t bits, int lane, float* x) {
  const int c = lane >> 4;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int at = 4 * c + (r & 3) + 16 * (r >> 2), j = key + at;
    bool seen = j <= hi && (j >= lo || j < sinks);
    if (kTree) seen = seen || ((bits >> at) & 1u) != 0;
    x[r] = seen ? x[r] : -INFINITY;
  }
}

struct Tree {
  const uint32_t* seen;   // [rows][stride]: the rows that a row sees
  const int32_t* depths;  // [rows]
  int words, stride;
  __device__ __forceinline__ int depth(int row) const { return depths[row]; }
  // Bit k: row first + k is seen by `row` (first > -32; bits before row 0 and behind the last row are 0).
  __device__ __forceinline__ uint32_t bits(int row, int first) const {
    const int word = first >> 5;
    const uint32_t* const at = seen + row * stride;
    const uint32_t low = word >= 0 && word < words ? at[word] : 0u, high = word + 1 < words ? at[word + 1] : 0u;
    return (uint32_t)((((uint64_t)high << 32) | low) >> (first & 31));
  }
};

// Up to 64 rows: every wavefront does it in its registers, a lane a row, and writes the same words as the others, so that nobody
// waits for anybody (8 nodes of one sequence behind 300 keys: 13.9 us a call with barriers between eight wavefronts, 10.6 without).
__device__ inline Tree small_tree_of(const int32_t* parents, int rows, int window, int sinks, int t, uint32_t* lds) {
  const int words = tree_words(rows), stride = tree_stride(rows), lane = threadIdx.x & 63;
  int32_t* const depths = reinterpret_cast<int32_t*>(lds + rows * stride) + rows;
  const int parent = parents[lane < rows ? lane : 0];
  int up = lane < rows && parent >= 0 && parent < lane ? parent : -1;
  uint32_t low = lane < 32 ? 1u << lane : 0u, high = lane < 32 ? 0u : 1u << (lane - 32);
  while (__any(up >= 0)) {
    const int above = up >= 0 ? up : lane;
    const uint32_t a = (uint32_t)__shfl((int)low, above), z = (uint32_t)__shfl((int)high, above);
    const int next = __shfl(up, above);
    low |= a;
    high |= z;
    up = up >= 0 ? next : -1;
  }
  const int depth = __builtin_popcount(low) + __builtin_popcount(high) - 1;
  if (window > 0 && __any(depth >= window)) {
    uint64_t left = ((uint64_t)high << 32) | low;
    while (__any(left != 0)) {  // (uniform: the lanes' depths are asked for)
      const int bit = left ? __builtin_ctzll(left) : lane;
      const int other = __shfl(depth, bit);
      if (left && depth - other >= window && t + other >= sinks) {
        if (bit < 32) low &= ~(1u << bit);
        else high &= ~(1u << (bit - 32));
      }
      left &= left - 1;
    }
  }
  if (lane < rows) {
    lds[lane * stride] = low;
    if (words > 1) lds[lane * stride + 1] = high;
    depths[lane] = depth;
  }
  return Tree{lds, depths, words, stride};
}

// All threads of the workgroup call this, rows <= 256; lds: tree_lds_bytes().
// A window of `window` positions hides the ancestors that lie further back, but for those among the first `sinks` positions.
__device__ inline Tree tree_of(const int32_t* parents, int rows, int window, int sinks, int t, uint32_t* lds) {
  if (rows <= 64) return small_tree_of(parents, rows, window, sinks, t, lds);
  const int words = tree_words(rows), stride = tree_stride(rows);
  int32_t* const up = reinterpret_cast<int32_t*>(lds + rows * stride);
  int32_t* const depths = up + rows;
  const int tid = threadIdx.x, threads = blockDim.x;
  for (int i = tid; i < rows; i += threads) {
    const int parent = parents[i];
    up[i] = parent >= 0 && parent < i ? parent : -1;
    for (int w = 0; w < words; ++w) lds[i * stride + w] = (i >> 5) == w ? 1u << (i & 31) : 0u;
  }
  __syncthreads();
  // A thread's rows, at most four (256 rows, a single wavefront), are read by all and written behind a barrier.
  for (int reach = 1; reach < rows; reach *= 2) {
    uint32_t more[4][kMaxNodes / 32];
    int next[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = tid + k * threads, above = i < rows ? up[i] : -1;
      next[k] = above >= 0 ? up[above] : -1;
#pragma unroll
      for (int w = 0; w < kMaxNodes / 32; ++w) more[k][w] = above >= 0 && w < words ? lds[above * stride + w] : 0u;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = tid + k * threads;
      if (i < rows) {
        up[i] = next[k];
#pragma unroll
        for (int w = 0; w < kMaxNodes / 32; ++w) {
          if (w < words) lds[i * stride + w] |= more[k][w];
        }
      }
    }
    __syncthreads();
  }
  for (int i = tid; i < rows; i += threads) {
    int n = -1;
    for (int w = 0; w < words; ++w) n += __builtin_popcount(lds[i * stride + w]);
    depths[i] = n;
  }
  __syncthreads();
  if (window > 0 && window < rows) {
    for (int i = tid; i < rows; i += threads) {
      if (depths[i] < window) continue;
      for (int w = 0; w < words; ++w) {
        uint32_t left = lds[i * stride + w], kept = left;
        while (left) {
          const int bit = __builtin_ctz(left);
          left &= left - 1;
          const int depth = depths[32 * w + bit];
          if (depths[i] - depth >= window && t + depth >= sinks) kept &= ~(1u << bit);
        }
        lds[i * stride + w] = kept;
      }
    }
    __syncthreads();
  }
  return Tree{lds, depths, words, stride};
}

}  // namespace
}  // namespace tempo
