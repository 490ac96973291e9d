// Attention over a window with sinks, and of a tree, over an fp32 block store; MFMA 16x16x4 on gfx950.
//
// The rows, what they see and how their groups are numbered: attn_spans.hip.  A wavefront takes 16 (row, head) columns and a group
// of 32 slots at a time, as two tiles of 16 rows: logits tile = K (16 slots x 4 dims) Q^T, D/4 steps; answers = P (16 columns x 4
// slots) V, 8 steps a tile of 16 dims.  Lane (row + 16c) of a tile holds dims 16i + 4c .. +3 of its row, so a step contracts the four
// dims 16i + 4c + e of c = 0 .. 3; and the logits that it gets, of slots 4c .. 4c+3 for column (lane & 15), are the operand of the
// second product as they stand.  A tile of answers takes the dims 64h + 4n + e of lanes n, so that values too are read 16 bytes a lane
// (read 4 bytes a lane, where they are used: 145 us for 111, 648 for 536).  All in fp32: for parity and for stores that were made in
// it.  Blocks may be shorter than a group, so every row looks its block up.  A tile of columns streams its keys again, from L2.
// A value that is not finite shows in the columns that see it, and in no other: in groups that some columns see less of than others such
// values are taken for 0 and added to their columns behind the loop, where there are any (us, without / with the check: 2048 steps of
// window 2048 536 / 538, of window 64 58.2 / 59.9; 8 trees of 16 nodes behind 4000 keys 114 / 115; 8 of 100 behind 500, D = 64, 63.3 / 65.5).
// Bound by memory with few columns (16 sequences, 32/8 heads of 128, a step behind a window of 4096 keys: 107 us, 5.0 TB/s), by the
// matrix products and their loads with many (2048 steps of 24/8 heads behind a window of 2048 keys: 538 us, 96 TFLOP/s; 8 trees of 16
// nodes behind 4000 keys: 115 us).
#include "attn_image.h"
#include "attn_spans.h"
#include "attn_tree.h"

namespace tempo {
namespace {

template <int D, bool kTree, bool kRope>
__global__ __launch_bounds__(512) void attn_spans_f32(SpanParams p) {
  constexpr int DT = D / 16;
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 63, c = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nwaves = blockDim.x >> 6;
  const UnitsWork item = units_work(blockIdx.x, blockIdx.y, blockIdx.z, gridDim.x, gridDim.y, gridDim.z, p.Hkv);
  const int hkv = item.hkv, first_col = 16 * item.tile, b = item.b, split = item.split;
  int t_b = p.t_per_seq ? ((const_i32_ptr)p.t_per_seq)[b] : p.t;
  t_b = t_b > p.t ? p.t : (t_b < 0 ? 0 : t_b);
  int rows = p.queries;
  if (p.count_per_seq) {
    const int given = ((const_i32_ptr)p.count_per_seq)[b];
    rows = given < 0 ? 0 : (given < rows ? given : rows);
  }
  const int all_cols = rows * p.G - first_col;  // from this workgroup's first on
  if (all_cols <= 0) return;                    // uniform over the workgroup, as is all that follows
  const SpanRange rg = tile_range(t_b, item.tile, 16, p.G, rows, p.window, p.sinks, kTree);
  const int from = split * p.split_groups;
  if (from >= rg.groups) return;
  const int past = from + p.split_groups < rg.groups ? from + p.split_groups : rg.groups;
  Tree tree;
  if constexpr (kTree)
    tree = tree_of(p.parents + (int64_t)b * p.queries, rows, p.window, p.sinks, t_b, reinterpret_cast<uint32_t*>(smem));

  const int row_end = (first_col + 15) / p.G, last_row = row_end < rows - 1 ? row_end : rows - 1, last = t_b + last_row;
  const bool there = n < all_cols;
  const int row = there ? (first_col + n) / p.G : rows - 1, gq = there ? first_col + n - row * p.G : 0;
  int position = t_b + row;
  if constexpr (kTree) position = t_b + tree.depth(row);
  const int hi_col = kTree ? t_b - 1 : position, lo_col = p.window > 0 && position - p.window + 1 > 0 ? position - p.window + 1 : 0;
  // A group that ends behind all_hi, or begins before lo_last and is not all sinks, is seen less of by some of several rows than by others;
  // in a tree by a single row too, whose ancestors are not all the nodes before it.
  const int all_hi = kTree ? t_b - 1 : t_b + first_col / p.G, lo_last = p.window > 0 && last - p.window + 1 > 0 ? last - p.window + 1 : 0;
  const bool differ = !kRope && (kTree || last_row > first_col / p.G);  // (turned: a single step)
  f32x4 q[DT];
  {
    const float* qp = static_cast<const float*>(p.q) + (((int64_t)b * p.io_steps + row) * p.Hq + (int64_t)hkv * p.G + gq) * D + 4 * c;
#pragma unroll
    for (int i = 0; i < DT; ++i) q[i] = *reinterpret_cast<const f32x4*>(qp + 16 * i);
    if (kRope) {  // a dim's partner D/2 further sits in the same lane
#pragma unroll
      for (int i = 0; i < DT / 2; ++i) {
        const int64_t at = (int64_t)position * (D / 2) + 16 * i + 4 * c;
        const f32x4 cs = *reinterpret_cast<const f32x4*>(p.rope_cos + at), sn = *reinterpret_cast<const f32x4*>(p.rope_sin + at);
        const f32x4 lo = q[i], hi = q[i + DT / 2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          q[i][e] = rope_lo(lo[e], hi[e], cs[e], sn[e]);
          q[i + DT / 2][e] = rope_hi(lo[e], hi[e], cs[e], sn[e]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < DT; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[i][e] = there ? q[i][e] : 0.f;
    }
  }
  float m_run = kUnseen, l_run = 0.f;
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Element offset of a key's row in either pool.  (Keys behind the rows' last are not seen: that one's row in their place.)
  const int32_t* const table = p.block_table + (int64_t)b * p.max_blocks_per_seq;
  auto row_at = [&](int key) {
    const int j = key < last ? key : last;
    const int phys = clamp_block(table[(j >> p.z_log2) & p.tile_mask], p.num_blocks);
    return ((((int64_t)phys * p.Hkv + hkv) << p.z_log2) + (j & ((1 << p.z_log2) - 1))) * D;
  };
  auto cut = [&](int key) __attribute__((always_inline)) { return differ && (key + 31 > all_hi || (key < lo_last && key + 31 >= p.sinks)); };
  bool wrong = false;
  for (int at = from + wave; at < past; at += nwaves) {
    const int key = span_group(rg, at) << 5;
    int64_t off[2];
    float x[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      off[t] = row_at(key + 16 * t + n);
      const float* const kp = static_cast<const float*>(p.k_pool) + off[t] + 4 * c;
      f32x4 k[DT], s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DT; ++i) k[i] = *reinterpret_cast<const f32x4*>(kp + 16 * i);
#pragma unroll
      for (int i = 0; i < DT; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][e], q[i][e], s, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) x[4 * t + r] = s[r];
    }
    f32x4 v[8][D / 64];  // asked for before the weights are known
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int slot = 4 * c + (r & 3);
      const int64_t far = off[r >> 2];
      const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)far, slot), hi = (uint32_t)__shfl((int)(uint32_t)(far >> 32), slot);
      const float* const vp = static_cast<const float*>(p.v_pool) + (int64_t)(((uint64_t)hi << 32) | lo) + 4 * n;
#pragma unroll
      for (int h = 0; h < D / 64; ++h) v[r][h] = *reinterpret_cast<const f32x4*>(vp + 64 * h);
    }
    auto put_off = [&]() __attribute__((always_inline)) {  // a weight of 0 makes NaN of a value that is not finite: such values come later
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int j = key + 4 * c + (r & 3) + 16 * (r >> 2);
        float of = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) of = fmaf(0.f, v[r][dt >> 2][dt & 3], of);
        sum += j <= last && (j >= rg.lo || j < p.sinks) ? of : 0.f;
      }
      if (__any(!(sum == 0.f))) {
        wrong = true;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) v[r][dt >> 2][dt & 3] = fabsf(v[r][dt >> 2][dt & 3]) < INFINITY ? v[r][dt >> 2][dt & 3] : 0.f;
        }
      }
    };
    uint32_t bits = 0;
    if constexpr (kTree) {  // (behind the mask trees take 123 us for 115; steps, before it, 547 for 538)
      if (cut(key)) {
        put_off();
        if (key + 31 >= t_b) bits = tree.bits(row, key - t_b);
      }
    }
    mask_span<kTree>(key, lo_col, hi_col, p.sinks, bits, lane, x);
    float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    mx = column_max(mx) * p.scale_log2e;
    const bool above = mx > m_run;
    if (__any(above && m_run != kUnseen)) {
      const float alpha = above ? fast_exp2(m_run - mx) : 1.f;
      float a[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) a[r] = __shfl(alpha, 4 * c + r);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[dt][r] *= a[r];
      }
    }
    m_run = above ? mx : m_run;
    if constexpr (!kTree) {
      if (cut(key)) put_off();
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float w = fast_exp2(fmaf(x[r], p.scale_log2e, -m_run));
      l_run += w;
      const int j = key + 4 * c + (r & 3) + 16 * (r >> 2);
      const bool some = j <= last && (j >= rg.lo || j < p.sinks);  // (a slot that no row sees may be unwritten)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(w, some ? v[r][dt >> 2][dt & 3] : 0.f, acc[dt], 0, 0, 0);
      }
    }
  }
  if (wrong) {  // such values, one by one, into the columns that see them: infinite or NaN whatever the weight
    int same = lane;
    asm volatile("" : "+v"(same));  // (what both loops have in common is computed anew: registers)
    const int c = same >> 4, n = same & 15;
    for (int at = from + wave; at < past; at += nwaves) {
      const int key = span_group(rg, at) << 5;
      if (!cut(key)) continue;
      uint32_t bits = 0, sees = 0;  // of the group's slots 4c + (r mod 4) + 16 (r / 4), bit r: this lane's column sees it
      if constexpr (kTree) {
        if (key + 31 >= t_b) bits = tree.bits(row, key - t_b);
      }
#pragma unroll 1
      for (int r = 0; r < 8; ++r) {
        const int slot = 4 * c + (r & 3) + 16 * (r >> 2), j = key + slot;
        sees |= ((j <= hi_col && (j >= lo_col || j < p.sinks)) || ((bits >> slot) & 1u) != 0 ? 1u : 0u) << r;
      }
#pragma unroll 1
      for (int r = 0; r < 8; ++r) {
        const int j = key + 4 * c + (r & 3) + 16 * (r >> 2);
        const bool some = j <= last && (j >= rg.lo || j < p.sinks);
        const float* const vp = static_cast<const float*>(p.v_pool) + row_at(j) + 4 * n;
        f32x4 one[D / 64];
#pragma unroll
        for (int h = 0; h < D / 64; ++h) one[h] = *reinterpret_cast<const f32x4*>(vp + 64 * h);
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {  // the slot of lanes 16i ..
          uint32_t seen[4];            // by columns 4c + e
#pragma unroll
          for (int e = 0; e < 4; ++e) seen[e] = ((uint32_t)__shfl((int)sees, 4 * c + e + 16 * i) >> r) & 1u;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const float far = __shfl(some ? one[dt >> 2][dt & 3] : 0.f, n + 16 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[dt][e] += seen[e] && !(fabsf(far) < INFINITY) ? far : 0.f;
          }
        }
      }
    }
  }
  if constexpr (kTree) __syncthreads();  // the ancestors lie where the merge writes

  const int ncols = all_cols < 16 ? all_cols : 16;
  const float l_tot = column_sum(l_run);
  float* const sm_m = smem;                  // [nwaves][16]
  float* const sm_l = smem + nwaves * 16;    // [nwaves][16]
  float* const sm_acc = smem + nwaves * 32;  // [nwaves][ncols][D]
  if (lane < 16) {
    sm_m[wave * 16 + lane] = m_run == kUnseen ? -INFINITY : m_run;
    sm_l[wave * 16 + lane] = l_tot;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int j = 4 * c + r;
    if (j < ncols) {
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        const f32x4 o = {acc[4 * h][r], acc[4 * h + 1][r], acc[4 * h + 2][r], acc[4 * h + 3][r]};
        *reinterpret_cast<f32x4*>(sm_acc + (wave * ncols + j) * D + 64 * h + 4 * n) = o;
      }
    }
  }
  __syncthreads();
  if (nwaves == 8) merge_units<D, 8, true, false>(p, smem, first_col, ncols, b, hkv, split);
  else if (nwaves == 4) merge_units<D, 4, true, false>(p, smem, first_col, ncols, b, hkv, split);
  else if (nwaves == 2) merge_units<D, 2, true, false>(p, smem, first_col, ncols, b, hkv, split);
  else merge_units<D, 1, true, false>(p, smem, first_col, ncols, b, hkv, split);
}

template <int D>
hipError_t launch_f32(const SpanParams& p, int batch, int waves, hipStream_t stream) {
  const int columns = p.queries * p.G, tiles = (columns + 15) / 16;
  const dim3 grid((unsigned)(p.Hkv * tiles), (unsigned)batch, (unsigned)p.num_splits), block(64 * waves);
  const size_t merge = units_lds_bytes(waves, columns, D), tree = p.parents ? tree_lds_bytes(p.queries) : 0, lds = merge > tree ? merge : tree;
  if (p.parents) return launch((attn_spans_f32<D, true, false>), grid, block, lds, stream, p);
  if (p.rope_cos) return launch((attn_spans_f32<D, false, true>), grid, block, lds, stream, p);
  return launch((attn_spans_f32<D, false, false>), grid, block, lds, stream, p);
}

}  // namespace

hipError_t launch_spans_f32(const SpanParams& p, int batch, int D, int waves, hipStream_t stream) {
  if (p.tile_columns != 16) return hipErrorInvalidConfiguration;
  return D == 128 ? launch_f32<128>(p, batch, waves, stream) : launch_f32<64>(p, batch, waves, stream);
}

}  // namespace tempo
