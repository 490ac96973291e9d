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

// All threads of the workgroup call this, rows <= 256; lds: tree_lds_bytes().
// A window of `window` positions hides the ancestors that lie further back, but for those among the first `sinks` positions.
__device__ inline Tree tree_of(const int32_t* parents, int rows, int window, int sinks, int t, uint32_t* lds) {
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
