// Partial attention of one split over an 8-bit block store, and over a list of selected blocks of either kind of store;
// MFMA on gfx950.
//
// What is computed, and how a wavefront computes it, is as in attn_partial_bf16.hip: Eq. 1 over one split's key
// positions with a running maximum and sum in fp32; S^T tile = K (16 slots x 32 dims) * Q^T, acc tile = P * V, both
// operands as they lie in the store, streamed by 1 KiB loads without LDS.  What differs:
//   8-bit codes (k8).  A 1 KiB unit holds the operands of two MFMAs.  Keys are turned into bf16 with their row's scale
//     (v_cvt_scalef32_pk_bf16_fp8: exact), so logits need no further factor.  Values are turned into bf16 without a
//     scale and the weight of a slot is multiplied by the slot's scale, a power of two, after it has been rounded to
//     bf16: the products are those of the weights and the values that the codes stand for, and the sum of the weights
//     is that of the rounded ones.  Rounding the weights to bf16 costs as much as rounding the result does.
//   Lists (kSelect).  The positions of a split run over the blocks of a list, [batch][Hkv][pick] block numbers, not over
//     the sequence: position v is slot v mod Z of block list[v div Z].  Entries that name no block at or before the
//     step's are passed over.
// Bound by HBM: 16 sequences of 4096 keys in 8 heads of 128, 135 MB, in 22 us (6.1 TB/s; a streaming read reaches 7.1; the vector
// units are busy 7 of the 22), 8 x 64 listed blocks of 64 bf16 keys, 134 MB, in 22; each byte is fetched once.
// More than 16 (step, head) columns: a wavefront takes 32 (8-bit stores), further workgroups the next ones over the same keys, on
// the same die (units_work()), so that all but one of them read from its L2.
#include "attn_image.h"

namespace tempo {
namespace {

constexpr int kNoKey = -1;  // in the place of a group's first key: none that the step sees

// CT: tiles of 16 columns that a wavefront takes, over the same operands.
// (D = 64, two tiles: 134 registers without the bound, 3 wavefronts to a SIMD; 128 columns 47.9 us, with it 40.6)
template <int D, bool k8, bool kSelect, bool kRope, int CT>
__global__ __launch_bounds__(512, D == 64 && CT == 2 ? 4 : 1) void attn_units(SelectParams p) {
  constexpr int KS = D / 32, DT = D / 16;
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nwaves = blockDim.x >> 6;
  UnitsWork item = {(int)blockIdx.x, 0, (int)blockIdx.y, (int)blockIdx.z};
  if constexpr (!k8 || CT > 1) item = units_work(blockIdx.x, blockIdx.y, blockIdx.z, gridDim.x, gridDim.y, gridDim.z, p.Hkv);  // (else one tile)
  const int hkv = item.hkv, first_col = 16 * CT * item.tile, b = item.b;
  int t_b = p.t_per_seq ? ((const_i32_ptr)p.t_per_seq)[b] : p.t;
  t_b = t_b > p.t ? p.t : (t_b < 0 ? 0 : t_b);
  int split, start, end;  // positions: keys, or places in the list's blocks
  if constexpr (kSelect) {
    split = item.split;
    start = split << p.tps_log2;
    const int last = (p.pick << p.z_log2) - 1, ce = split_end(split, p.tps_log2);
    end = last < ce ? last : ce;
  } else {
    const SeqRange rg = seq_range(t_b, p.window, p.tps_log2, p.queries);
    if (item.split >= rg.nchunks) return;  // uniform over the workgroup
    split = rg.nchunks - 1 - item.split;   // newest first, as in attn_partial_bf16.hip
    const int chunk = rg.chunk0 + split, cs = chunk << p.tps_log2, ce = split_end(chunk, p.tps_log2);
    start = rg.lo > cs ? rg.lo : cs;
    end = rg.hi < ce ? rg.hi : ce;
  }
  const int g_last = end >> 5;
  const int from = kSelect ? 0 : start, upto = kSelect ? t_b : end;  // keys
  const int64_t slots = ((int64_t)p.num_blocks * p.Hkv) << p.z_log2;  // of the store
  const_i32_ptr const table = (const_i32_ptr)p.block_table + (int64_t)b * p.max_blocks_per_seq;
  const_i32_ptr const list = kSelect ? (const_i32_ptr)p.selected + ((int64_t)b * p.Hkv + hkv) * p.pick : nullptr;

  // First key of the group at position group `at`; kNoKey: none that step t_b sees.
  auto key_of = [&](int at) __attribute__((always_inline)) {
    if constexpr (!kSelect) return at << 5;
    const int pos = at << 5, n = list[pos >> p.z_log2];
    if (n < 0 || n > (t_b >> p.z_log2)) return kNoKey;
    const int first = (n << p.z_log2) + (pos & ((1 << p.z_log2) - 1));
    return first <= t_b ? first : kNoKey;
  };
  // From position group `at` on, in this wavefront's turn, the first one with keys.
  auto next_of = [&](int at, int& first) __attribute__((always_inline)) {
    for (; at <= g_last; at += nwaves) {
      first = key_of(at);
      if (!kSelect || first != kNoKey) break;
    }
    return at;
  };
  auto slot_of = [&](int first) __attribute__((always_inline)) {
    const int phys = clamp_block(table[(first >> p.z_log2) & p.tile_mask], p.num_blocks);
    return (((int64_t)phys * p.Hkv + hkv) << p.z_log2) + (first & ((1 << p.z_log2) - 1));
  };

  Image<D, k8> g;
  int key = 0;
  int grp = next_of((start >> 5) + wave, key);
  if (grp <= g_last) {
    const int64_t slot = slot_of(key);
    load_image_keys<D, k8>(p, slot, slots, lane, g);
    load_image_values<D, k8>(p, slot, slots, lane, g);
  }

  // Columns and their ranges, as in attn_partial_bf16.hip.
  const int all_cols = p.queries * p.G - first_col;  // from this workgroup's first on
  const int t_end = t_b + p.queries - 1;
  const int lo_last = (p.window > 0 && t_end - p.window + 1 > 0) ? t_end - p.window + 1 : 0;
  const int all_lo = lo_last > from ? lo_last : from;
  const int all_hi = t_b < upto ? t_b : upto;
  const int seen_hi = t_end < upto ? t_end : upto;
  int lo_col[CT], hi_col[CT];
  u32x4 qreg[CT][KS];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int col = 16 * ct + (lane & 15);
    const int cq = col < all_cols ? (first_col + col) / p.G : p.queries - 1;
    const int gq = col < all_cols ? first_col + col - cq * p.G : 0;
    hi_col[ct] = (t_b + cq) < upto ? (t_b + cq) : upto;
    const int lo_q = (p.window > 0 && t_b + cq - p.window + 1 > 0) ? t_b + cq - p.window + 1 : 0;
    lo_col[ct] = lo_q > from ? lo_q : from;
    const uint16_t* qp = static_cast<const uint16_t*>(p.q) +
                         (((int64_t)b * p.io_steps + cq) * p.Hq + (int64_t)hkv * p.G + gq) * D + 8 * (lane >> 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const u32x4 zero = {0u, 0u, 0u, 0u};
      const u32x4 v = *reinterpret_cast<const u32x4*>(qp + 32 * s);
      qreg[ct][s] = col < all_cols ? v : zero;
    }
    if (kRope) rotate_query<D>(p, t_b + cq, lane, qreg[ct]);
  }

  // A fused write lands in group t_b >> 5, which only the newest split holds.
  int key_new = -1;  // first key of that group, in the wavefront that will reach it
  uint8_t* const stage = reinterpret_cast<uint8_t*>(smem + nwaves * (32 + (all_cols < 16 ? all_cols : 16) * D));
  if constexpr (k8 && !kSelect) {
    const int grp_new = t_b >> 5;
    if (p.k_new && item.split == 0 && grp_new >= grp && (grp_new - grp) % nwaves == 0) {
      key_new = grp_new << 5;
      const u32x4 rows = fetch_new_rows<D>(p, b, hkv, lane);
      write_new_rows<D, kRope>(p, rows, t_b, slot_of(key_new), slots, first_col == 0, lane, stage);
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
    if constexpr (k8 && !kSelect) {
      if (key == key_new) patch_keys<D>(t_b, lane, stage, g);
    }
    float x[CT][8];
    image_logits<D, k8, CT>(qreg, g, x);
    if (more) load_image_keys<D, k8>(p, slot_nxt, slots, lane, g);
    const bool cut = key < all_lo || key > all_hi - 31;  // wave-uniform: some column's range cuts the group
    if (cut) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) mask_logits(key >> 5, lo_col[ct], hi_col[ct], lane, x[ct]);
    }
    u32x4 w[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) w[ct] = softmax_weights<D, (CT > 1)>(x[ct], p.scale_log2e, lane, st[ct]);
    if constexpr (k8 && !kSelect) {
      if (key == key_new) patch_values<D>(t_b, lane, stage, g);
    }
    if (cut) {  // slots that no step of the call sees may be unwritten: codes and scales of 0, bf16 values of 0, under the weight of 0
      if constexpr (k8) {
        const uint2 keep = seen_bytes(key, from, seen_hi, lane);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          g.v[i].x &= keep.x; g.v[i].y &= keep.y; g.v[i].z &= keep.x; g.v[i].w &= keep.y;
        }
        g.v_scales.x &= keep.x;
        g.v_scales.y &= keep.y;
      } else {
        uint32_t keep[4];
        value_masks(key >> 5, from, seen_hi, lane, keep);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          g.v[i].x &= keep[0]; g.v[i].y &= keep[1]; g.v[i].z &= keep[2]; g.v[i].w &= keep[3];
        }
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
  // The last group has a body of its own: behind a condition, requests make every wait one for all of them
  // (attn_partial_bf16.hip).
  if (grp <= g_last) {
    for (;;) {
      int key_nxt = 0;
      const int nxt = next_of(grp + nwaves, key_nxt);
      if (nxt > g_last) break;
      group(key_nxt, true);
      grp = nxt;
      key = key_nxt;
    }
    group(0, false);
  }

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
    if (nwaves == 8) merge_units<D, 8, kSelect>(p, smem, first, ncols, b, hkv, split);
    else if (nwaves == 4) merge_units<D, 4, kSelect>(p, smem, first, ncols, b, hkv, split);
    else if (nwaves == 2) merge_units<D, 2, kSelect>(p, smem, first, ncols, b, hkv, split);
    else merge_units<D, 1, kSelect>(p, smem, first, ncols, b, hkv, split);
  }
}

template <bool k8, bool kSelect, bool kRope, int CT>
hipError_t launch_tiles(const SelectParams& p, int batch, int D, int grid_splits, int waves, hipStream_t stream) {
  const int columns = p.queries * p.G;
  const dim3 grid((unsigned)(p.Hkv * ((columns + 16 * CT - 1) / (16 * CT))), (unsigned)batch, (unsigned)grid_splits), block(64 * waves);
  const size_t lds = units_lds_bytes(waves, columns, D);
  if (D == 128) return launch((attn_units<128, k8, kSelect, kRope, CT>), grid, block, lds, stream, p);
  return launch((attn_units<64, k8, kSelect, kRope, CT>), grid, block, lds, stream, p);
}

// More than 16 columns: 8-bit operands are turned into bf16 once for two tiles.
template <bool k8, bool kSelect, bool kRope>
hipError_t launch_units(const SelectParams& p, int batch, int D, int grid_splits, int waves, hipStream_t stream) {
  if (k8 && p.queries * p.G > 16) return launch_tiles<k8, kSelect, kRope, k8 ? 2 : 1>(p, batch, D, grid_splits, waves, stream);
  return launch_tiles<k8, kSelect, kRope, 1>(p, batch, D, grid_splits, waves, stream);
}

}  // namespace

hipError_t launch_partial_e4m3(const AttnParams& p, int batch, int D, int grid_splits, int waves, hipStream_t stream) {
  SelectParams s;
  static_cast<AttnParams&>(s) = p;
  s.selected = nullptr;
  s.pick = 0;
  if (p.rope_cos) return launch_units<true, false, true>(s, batch, D, grid_splits, waves, stream);
  return launch_units<true, false, false>(s, batch, D, grid_splits, waves, stream);
}

hipError_t launch_partial_selected(const SelectParams& p, int batch, int D, int dtype, int grid_splits, int waves, hipStream_t stream) {
  if (dtype == TEMPO_E4M3) return launch_units<true, true, false>(p, batch, D, grid_splits, waves, stream);
  return launch_units<false, true, false>(p, batch, D, grid_splits, waves, stream);
}

}  // namespace tempo
