// Attention over a window with sinks, and of a tree of drafted rows, over a bf16 or 8-bit block store; MFMA on gfx950.
//
// Row i of a sequence is step t + i (consecutive steps), or node i of a tree whose keys and values lie in steps t + i: its parent is
// a row before it, or step t - 1.  Its position p_i is its step, or t + its depth.  It sees
//     the keys j < sinks and the keys p_i - window < j <= p_i (without a window: all j <= p_i),
// where of a tree only j < t are counted by their number; of the nodes it sees itself and its ancestors, by their positions.
// out = sum_j w_j v_j / sum_j w_j with w_j = 2^(s log2(e) q.k_j - m), m a running reference.
//
// What a wavefront does with a group of 32 slots is as in attn_units.hip.  The groups that a workgroup's rows see are numbered
// through, those of the sinks before those of the window (span_range()), and cut into splits of whole groups by that number.
#include "attn_combine.h"
#include "attn_image.h"
#include "attn_spans.h"
#include "attn_tree.h"

namespace tempo {
namespace {

// Slots of the group that some row may see, as masks of the lane's value bytes or halves.
template <bool k8>
__device__ __forceinline__ void keep_span(int key, int lo, int last, int sinks, int lane, uint32_t* keep) {
  const int c = lane >> 4;
  constexpr uint32_t kOnes = k8 ? 0xFFu : 0xFFFFu;
#pragma unroll
  for (int i = 0; i < 4; ++i) keep[i] = 0u;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int j = key + 4 * c + (r & 3) + 16 * (r >> 2);
    const uint32_t ones = j <= last && (j >= lo || j < sinks) ? kOnes : 0u;
    if (k8) keep[r >> 2] |= ones << (8 * (r & 3));
    else keep[r >> 1] |= ones << (16 * (r & 1));
  }
}

template <int D, bool k8, bool kTree, bool kRope, int CT>
__global__ __launch_bounds__(512, D == 64 && CT == 2 ? 3 : 1) void attn_spans(SpanParams p) {
  constexpr int KS = D / 32, DT = D / 16;
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nwaves = blockDim.x >> 6;
  const UnitsWork item = units_work(blockIdx.x, blockIdx.y, blockIdx.z, gridDim.x, gridDim.y, gridDim.z, p.Hkv);
  const int hkv = item.hkv, first_col = 16 * CT * item.tile, b = item.b, split = item.split;
  int t_b = p.t_per_seq ? ((const_i32_ptr)p.t_per_seq)[b] : p.t;
  t_b = t_b > p.t ? p.t : (t_b < 0 ? 0 : t_b);
  int rows = p.queries;
  if (p.count_per_seq) {
    const int n = ((const_i32_ptr)p.count_per_seq)[b];
    rows = n < 0 ? 0 : (n < rows ? n : rows);
  }
  const int all_cols = rows * p.G - first_col;  // from this workgroup's first on
  if (all_cols <= 0) return;                    // uniform over the workgroup, as is all that follows
  const SpanRange rg = tile_range(t_b, item.tile, 16 * CT, p.G, rows, p.window, p.sinks, kTree);
  const int from = split * p.split_groups;
  if (from >= rg.groups) return;
  const int past = from + p.split_groups < rg.groups ? from + p.split_groups : rg.groups;
  const int64_t slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;  // of the store
  const_i32_ptr const table = (const_i32_ptr)p.block_table + (int64_t)b * p.max_blocks_per_seq;
  auto slot_of = [&](int key) __attribute__((always_inline)) {
    const int phys = clamp_block(table[(key >> p.z_log2) & p.tile_mask], p.num_blocks);
    return (((int64_t)phys * p.Hkv + hkv) << p.z_log2) + (key & ((1 << p.z_log2) - 1));
  };

  Image<D, k8> g;
  int at = from + wave;
  int key = span_group(rg, at) << 5;
  if (at < past) {
    const int64_t slot = slot_of(key);
    load_image_keys<D, k8>(p, slot, slots, lane, g);
    load_image_values<D, k8>(p, slot, slots, lane, g);
  }

  // The rows' ancestors, where something hangs on them: nodes in the split, or depths.
  const int last_key = (span_group(rg, past - 1) << 5) + 31;
  Tree tree;
  if constexpr (kTree) {
    if (p.window > 0 || last_key >= t_b)
      tree = tree_of(p.parents + (int64_t)b * p.queries, rows, p.window, p.sinks, t_b, reinterpret_cast<uint32_t*>(smem));
  }

  const int first_row = first_col / p.G, row_end = (first_col + 16 * CT - 1) / p.G, last_row = row_end < rows - 1 ? row_end : rows - 1;
  const int last = t_b + last_row;                                            // newest slot that a row may see
  // A group that ends at or before all_hi, and begins at or behind all_lo or lies among the sinks, is seen by all columns.
  const int all_hi = kTree ? t_b - 1 : t_b + first_row;
  const int lo_last = p.window > 0 && last - p.window + 1 > 0 ? last - p.window + 1 : 0;
  int lo_col[CT], hi_col[CT], row_of[CT];
  u32x4 qreg[CT][KS];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = 16 * ct + (lane & 15);
    const bool there = col < all_cols;
    const int row = there ? (first_col + col) / p.G : rows - 1, gq = there ? first_col + col - row * p.G : 0;
    int position = t_b + row;
    if constexpr (kTree) {
      if (p.window > 0) position = t_b + tree.depth(row);
    }
    row_of[ct] = row;
    hi_col[ct] = kTree ? t_b - 1 : position;
    lo_col[ct] = p.window > 0 && position - p.window + 1 > 0 ? position - p.window + 1 : 0;
    const uint16_t* qp = static_cast<const uint16_t*>(p.q) +
                         (((int64_t)b * p.io_steps + row) * p.Hq + (int64_t)hkv * p.G + gq) * D + 8 * (lane >> 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const u32x4 zero = {0u, 0u, 0u, 0u};
      const u32x4 v = *reinterpret_cast<const u32x4*>(qp + 32 * s);
      qreg[ct][s] = there ? v : zero;
    }
    if (kRope) rotate_query<D>(p, position, lane, qreg[ct]);
  }

  // A step's own row lies in the last group; the wavefront that comes to it writes the row (attn_image.h), unless another tile
  // of columns does, and puts it among what it read.
  int key_new = -1;
  void* const stage = smem + nwaves * (32 + (all_cols < 16 ? all_cols : 16) * D);
  if constexpr (!kTree) {
    const int newest = rg.groups - 1;
    if (p.k_new && newest < past && newest >= at && (newest - at) % nwaves == 0) {
      key_new = span_group(rg, newest) << 5;
      const u32x4 x = fetch_new_rows<D>(p, b, hkv, lane);
      if constexpr (k8) write_new_rows<D, kRope>(p, x, t_b, slot_of(key_new), slots, first_col == 0, lane, static_cast<uint8_t*>(stage));
      else write_new_rows_bf16<D, kRope>(p, x, t_b, slot_of(key_new), first_col == 0, lane, static_cast<uint16_t*>(stage));
    }
  }

  WaveState<D> st[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    st[ct].m = kUnseen;
    st[ct].l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) st[ct].acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // The group in the registers; `more`: and request the one whose first key is key_nxt.
  auto group = [&](int key_nxt, bool more) __attribute__((always_inline)) {
    const int64_t slot_nxt = more ? slot_of(key_nxt) : 0;
    if constexpr (!kTree) {
      if (key == key_new) {
        if constexpr (k8) patch_keys<D>(t_b, lane, static_cast<const uint8_t*>(stage), g);
        else patch_keys_bf16<D>(t_b, lane, static_cast<const uint16_t*>(stage), g);
      }
    }
    float x[CT][8];
    image_logits<D, k8, CT>(qreg, g, x);
    if (more) load_image_keys<D, k8>(p, slot_nxt, slots, lane, g);
    const bool cut = key + 31 > all_hi || (key < lo_last && key + 31 >= p.sinks);  // wave-uniform
    if (cut) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        uint32_t bits = 0;
        if constexpr (kTree) {
          if (key + 31 >= t_b) bits = tree.bits(row_of[ct], key - t_b);
        }
        mask_span<kTree>(key, lo_col[ct], hi_col[ct], p.sinks, bits, lane, x[ct]);
      }
    }
    u32x4 w[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) w[ct] = softmax_weights<D, (CT > 1)>(x[ct], p.scale_log2e, lane, st[ct]);
    if constexpr (!kTree) {
      if (key == key_new) {
        if constexpr (k8) patch_values<D>(t_b, lane, static_cast<const uint8_t*>(stage), g);
        else patch_values_bf16<D>(t_b, lane, static_cast<const uint16_t*>(stage), g);
      }
    }
    if (cut) {  // slots that no row sees may be unwritten: values of 0 under the weight of 0
      uint32_t keep[4];
      keep_span<k8>(key, rg.lo, last, p.sinks, lane, keep);
#pragma unroll
      for (int i = 0; i < Image<D, k8>::UNITS; ++i) {
        if constexpr (k8) {
          g.v[i].x &= keep[0]; g.v[i].y &= keep[1]; g.v[i].z &= keep[0]; g.v[i].w &= keep[1];
        } else {
          g.v[i].x &= keep[0]; g.v[i].y &= keep[1]; g.v[i].z &= keep[2]; g.v[i].w &= keep[3];
        }
      }
      if constexpr (k8) {
        g.v_scales.x &= keep[0];
        g.v_scales.y &= keep[1];
      }
    }
    bf16x8 pa[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      if constexpr (k8) pa[ct] = scaled_weights(w[ct], g.v_scales);
      else pa[ct] = as_bf16x8(w[ct]);
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      bf16x8 v;
      if constexpr (k8) {
        const u32x4 u = g.v[dt / 2];
        v = dt & 1 ? operand_of(u.z, u.w, 1.f) : operand_of(u.x, u.y, 1.f);
      } else {
        v = as_bf16x8(g.v[dt]);
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) st[ct].acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[ct], v, st[ct].acc[dt], 0, 0, 0);
    }
    if (more) load_image_values<D, k8>(p, slot_nxt, slots, lane, g);
  };
  if (at < past) {
    for (;;) {
      const int nxt = at + nwaves;
      if (nxt >= past) break;
      const int key_nxt = span_group(rg, nxt) << 5;
      group(key_nxt, true);
      at = nxt;
      key = key_nxt;
    }
    group(0, false);
  }
  if constexpr (kTree) __syncthreads();  // the ancestors lie where the merge writes

  // The wavefronts' results are merged a tile of columns at a time.
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int tile_cols = all_cols - 16 * ct, ncols = tile_cols < 16 ? tile_cols : 16;
    if (ncols <= 0) break;       // uniform over the workgroup
    if (ct > 0) __syncthreads();
    const float l_tot = column_sum(st[ct].l);
    float* sm_m = smem;                  // [nwaves][16]
    float* sm_l = smem + nwaves * 16;    // [nwaves][16]
    float* sm_acc = smem + nwaves * 32;  // [nwaves][ncols][D]
    if (lane < 16) {
      sm_m[wave * 16 + lane] = st[ct].m == kUnseen ? -INFINITY : st[ct].m;
      sm_l[wave * 16 + lane] = l_tot;
    }
    {
      const int n = lane & 15, c = lane >> 4;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 4 * c + r;
        if (j < ncols) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) sm_acc[(wave * ncols + j) * D + 16 * dt + n] = st[ct].acc[dt][r];
        }
      }
    }
    __syncthreads();
    const int first = first_col + 16 * ct;
    if (nwaves == 8) merge_units<D, 8, true>(p, smem, first, ncols, b, hkv, split);
    else if (nwaves == 4) merge_units<D, 4, true>(p, smem, first, ncols, b, hkv, split);
    else if (nwaves == 2) merge_units<D, 2, true>(p, smem, first, ncols, b, hkv, split);
    else merge_units<D, 1, true>(p, smem, first, ncols, b, hkv, split);
  }
}

// Splits of row `at` (row * Hq + head) of sequence b; 0: a row that the call does not answer.
__device__ inline int splits_of(const SpanParams& p, int b, int at) {
  int t_b = p.t_per_seq ? p.t_per_seq[b] : p.t;
  t_b = t_b > p.t ? p.t : (t_b < 0 ? 0 : t_b);
  int rows = p.queries;
  if (p.count_per_seq) {
    const int n = p.count_per_seq[b];
    rows = n < 0 ? 0 : (n < rows ? n : rows);
  }
  const int row = at / p.Hq, column = row * p.G + (at - row * p.Hq) % p.G;
  if (row >= rows) return 0;
  const SpanRange rg = tile_range(t_b, column / p.tile_columns, p.tile_columns, p.G, rows, p.window, p.sinks, p.parents != nullptr);
  return (rg.groups + p.split_groups - 1) / p.split_groups;
}

// One workgroup to a (row, head): any number of splits.
template <int D, bool kBf16>
__global__ __launch_bounds__(256) void combine_spans(SpanParams p) {
  extern __shared__ float smem[];
  const int b = blockIdx.y, at = blockIdx.x;
  const int n = splits_of(p, b, at);
  if (n == 0) return;  // uniform over the workgroup
  const int64_t row = (int64_t)b * gridDim.x + at, orow = (int64_t)b * p.io_steps * p.Hq + at;
  combine_heads<D, kBf16, true>(p.ws_ml + row * p.num_splits * 2, p.ws_acc + row * p.num_splits * D, p.num_splits, n, 1,
                                static_cast<char*>(p.out) + orow * D * (kBf16 ? 2 : 4), smem);
}

// At most 8 splits: a thread to four dims of a (row, head), all of whose partials it asks for at once.
template <int D, bool kBf16>
__global__ __launch_bounds__(256) void combine_spans_few(SpanParams p, int64_t total) {
  constexpr int C4 = D / 4, U = 8;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x, row = idx / C4;
  const int c4 = (int)(idx - row * C4), each = p.Hq * p.queries;
  if (row >= total) return;
  const int b = (int)(row / each), at = (int)(row - (int64_t)b * each);
  const int n = splits_of(p, b, at);
  if (n == 0) return;
  const float* ml = p.ws_ml + row * p.num_splits * 2;
  const float* acc = p.ws_acc + row * p.num_splits * D + 4 * c4;
  float m[U], l[U];
  float4 a[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s = u < n ? u : 0;  // (a split that is there)
    m[u] = ml[2 * s];
    l[u] = ml[2 * s + 1];
    a[u] = *reinterpret_cast<const float4*>(acc + (int64_t)s * D);
    if (u >= n) m[u] = -INFINITY;
  }
  float M = m[0];
#pragma unroll
  for (int u = 1; u < U; ++u) M = fmaxf(M, m[u]);
  if (M == -INFINITY) M = 0.f;
  float L = 0.f;
  float4 A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float w = exp2f(m[u] - M);
    L = fmaf(w, l[u], L);
    A.x = fmaf(w, a[u].x, A.x); A.y = fmaf(w, a[u].y, A.y);
    A.z = fmaf(w, a[u].z, A.z); A.w = fmaf(w, a[u].w, A.w);
  }
  const float inv = 1.0f / L;  // every row sees itself
  const int64_t orow = (int64_t)b * p.io_steps * p.Hq + at;
  if constexpr (!kBf16) {
    *reinterpret_cast<float4*>(static_cast<float*>(p.out) + orow * D + 4 * c4) = float4{A.x * inv, A.y * inv, A.z * inv, A.w * inv};
    return;
  }
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  const bf16x4 o = {(__bf16)(A.x * inv), (__bf16)(A.y * inv), (__bf16)(A.z * inv), (__bf16)(A.w * inv)};
  *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + orow * D + 4 * c4) = o;
}

template <int D, bool k8, bool kTree, bool kRope, int CT>
hipError_t launch_tiles(const SpanParams& p, int batch, int waves, hipStream_t stream) {
  const int columns = p.queries * p.G, tiles = (columns + 16 * CT - 1) / (16 * CT);
  const dim3 grid((unsigned)(p.Hkv * tiles), (unsigned)batch, (unsigned)p.num_splits), block(64 * waves);
  const size_t merge = units_lds_bytes(waves, columns, D) + 2 * D, tree = kTree ? tree_lds_bytes(p.queries) : 0;
  return launch((attn_spans<D, k8, kTree, kRope, CT>), grid, block, merge > tree ? merge : tree, stream, p);
}

template <int D, bool k8, bool kTree>
hipError_t launch_rows(const SpanParams& p, int batch, int waves, hipStream_t stream) {
  if constexpr (!kTree) {
    if (p.rope_cos) {
      if (p.tile_columns == 16) return launch_tiles<D, k8, kTree, true, 1>(p, batch, waves, stream);
      return launch_tiles<D, k8, kTree, true, 2>(p, batch, waves, stream);
    }
  }
  if (p.tile_columns == 16) return launch_tiles<D, k8, kTree, false, 1>(p, batch, waves, stream);
  return launch_tiles<D, k8, kTree, false, 2>(p, batch, waves, stream);
}

template <int D>
hipError_t launch_spans_of(const SpanParams& p, int batch, int dtype, int waves, hipStream_t stream) {
  if (dtype == TEMPO_E4M3) return p.parents ? launch_rows<D, true, true>(p, batch, waves, stream) : launch_rows<D, true, false>(p, batch, waves, stream);
  return p.parents ? launch_rows<D, false, true>(p, batch, waves, stream) : launch_rows<D, false, false>(p, batch, waves, stream);
}

}  // namespace

hipError_t launch_spans(const SpanParams& p, int batch, int D, int dtype, int waves, hipStream_t stream) {
  if (D == 128) return launch_spans_of<128>(p, batch, dtype, waves, stream);
  return launch_spans_of<64>(p, batch, dtype, waves, stream);
}

namespace {
template <int D, bool kBf16>
hipError_t launch_combine_of(const SpanParams& p, int batch, hipStream_t stream) {
  const dim3 block(256);
  if (p.num_splits <= 8) {
    const int64_t total = (int64_t)batch * p.queries * p.Hq;
    return launch((combine_spans_few<D, kBf16>), dim3((unsigned)((total * (D / 4) + 255) / 256)), block, 0, stream, p, total);
  }
  const dim3 grid((unsigned)(p.Hq * p.queries), (unsigned)batch);
  return launch((combine_spans<D, kBf16>), grid, block, (size_t)combine_lds_floats(256, D) * sizeof(float), stream, p);
}
}  // namespace

hipError_t launch_combine_spans(const SpanParams& p, int batch, int D, int dtype, hipStream_t stream) {
  if (dtype == TEMPO_F32) return D == 128 ? launch_combine_of<128, false>(p, batch, stream) : launch_combine_of<64, false>(p, batch, stream);
  return D == 128 ? launch_combine_of<128, true>(p, batch, stream) : launch_combine_of<64, true>(p, batch, stream);
}

}  // namespace tempo
