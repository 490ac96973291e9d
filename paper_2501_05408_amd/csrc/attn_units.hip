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
#include "attn_bf16_common.h"
#include "attn_units.h"
#include "store_e4m3.h"

namespace tempo {
namespace {

constexpr int kNoKey = -1;  // in the place of a group's first key: none that the step sees

// The register image of a 32-slot group: keys, values, and in an 8-bit store the lane's scale bytes.
template <int D, bool k8>
struct Image {
  static constexpr int UNITS = k8 ? D / 32 : D / 16;  // 1 KiB units of keys, and of values
  u32x4 k[UNITS], v[UNITS];
  uint32_t k_scales;   // slots row, 16 + row
  uint2 v_scales;      // slots 4c..4c+3; 16+4c..16+4c+3
};

template <int D, bool k8>
__device__ __forceinline__ void load_image_keys(const AttnParams& p, int64_t slot, int64_t slots, int lane, Image<D, k8>& g) {
  const char* const at = static_cast<const char*>(p.k_pool) + slot * (k8 ? D : 2 * D) + lane * 16;
#pragma unroll
  for (int i = 0; i < Image<D, k8>::UNITS; ++i) g.k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + i * 1024));
  if constexpr (k8) g.k_scales = *reinterpret_cast<const uint16_t*>(static_cast<const char*>(p.k_pool) + slots * D + slot + 2 * (lane & 15));
}

template <int D, bool k8>
__device__ __forceinline__ void load_image_values(const AttnParams& p, int64_t slot, int64_t slots, int lane, Image<D, k8>& g) {
  const char* const at = static_cast<const char*>(p.v_pool) + slot * (k8 ? D : 2 * D) + lane * 16;
#pragma unroll
  for (int i = 0; i < Image<D, k8>::UNITS; ++i) g.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + i * 1024));
  if constexpr (k8) g.v_scales = *reinterpret_cast<const uint2*>(static_cast<const char*>(p.v_pool) + slots * D + slot + 8 * (lane >> 4));
}

// 8 codes (two words) as a bf16 operand.
__device__ __forceinline__ bf16x8 operand_of(uint32_t a, uint32_t b, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return __builtin_bit_cast(bf16x8, r);
}

// Products of the group's two row tiles with CT tiles of 16 columns; not scaled yet.
template <int D, bool k8, int CT>
__device__ __forceinline__ void image_logits(const u32x4 (*qreg)[D / 32], const Image<D, k8>& g, float (*x)[8]) {
  constexpr int KS = D / 32;
  f32x4 sa[CT], sb[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) sa[ct] = sb[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ka = 1.f, kb = 1.f;
  if constexpr (k8) {
    ka = scale_of(g.k_scales & 0xFFu);
    kb = scale_of(g.k_scales >> 8);
  }
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    bf16x8 a, b;
    if constexpr (k8) {
      const u32x4 u = g.k[s / 2], v = g.k[KS / 2 + s / 2];
      a = s & 1 ? operand_of(u.z, u.w, ka) : operand_of(u.x, u.y, ka);
      b = s & 1 ? operand_of(v.z, v.w, kb) : operand_of(v.x, v.y, kb);
    } else {
      a = as_bf16x8(g.k[s]);
      b = as_bf16x8(g.k[KS + s]);
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      sa[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(qreg[ct][s]), sa[ct], 0, 0, 0);
      sb[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, as_bf16x8(qreg[ct][s]), sb[ct], 0, 0, 0);
    }
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[ct][r] = sa[ct][r];
      x[ct][4 + r] = sb[ct][r];
    }
  }
}

// Which slots of a group this lane's values may be seen of, as masks of their bytes: x of slots 4c..4c+3, y of the others.
__device__ __forceinline__ uint2 seen_bytes(int key0, int v_lo, int v_hi, int lane) {
  const int c = lane >> 4;
  uint2 keep = {0u, 0u};
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int ja = key0 + 4 * c + r, jb = ja + 16;
    keep.x |= ja >= v_lo && ja <= v_hi ? 0xFFu << (8 * r) : 0u;
    keep.y |= jb >= v_lo && jb <= v_hi ? 0xFFu << (8 * r) : 0u;
  }
  return keep;
}

__device__ __forceinline__ float low_of(uint32_t pair) { return __builtin_bit_cast(float, pair << 16); }
__device__ __forceinline__ float high_of(uint32_t pair) { return __builtin_bit_cast(float, pair & 0xFFFF0000u); }

constexpr float kUnseen = -3e38f;  // reference of a column that has seen no key: finite, so that masked logits of -inf get the weight 0

// Online-softmax update of a column's reference, sum and accumulators, and the group's weights, 2^(x scale - reference) in bf16,
// as four words of two.  The sum is that of the rounded weights.  The reference is 2^kSlack above the maximum so far, so that sums
// of a few hundred of the largest values stay finite; wavefronts of two tiles keep an older one until a logit exceeds it, and
// hardly ever rescale their accumulators (16 sequences of 4000 keys, 63 and 126 columns 41.9 -> 37.2 and 74.2 -> 66.6 us; one tile
// gains 1% at most).  That costs accuracy, since the largest weight is a power of two only under its own reference (relative error
// of an answer 0.00217 -> 0.00232; the bf16 kernels for wide blocks 0.0021 to 0.0023), and weights reach 1.
template <int D, bool kKeep>
__device__ __forceinline__ u32x4 softmax_weights(const float* x, float scale, int lane, WaveState<D>& st) {
  float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  mx = column_max(mx) * scale;
  const float top = mx + kSlack;
  const bool above = (kKeep ? mx : top) > st.m;
  if (__any(above && st.m != kUnseen)) {
    const float alpha = above ? fast_exp2(st.m - top) : 1.f;
    float a[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) a[r] = __shfl(alpha, 4 * (lane >> 4) + r);
    st.l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
#pragma unroll
      for (int r = 0; r < 4; ++r) st.acc[dt][r] *= a[r];
    }
  }
  st.m = above ? top : st.m;
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 pair = {(__bf16)fast_exp2(fmaf(x[2 * i], scale, -st.m)), (__bf16)fast_exp2(fmaf(x[2 * i + 1], scale, -st.m))};
    w[i] = __builtin_bit_cast(uint32_t, pair);
    st.l += low_of(w[i]) + high_of(w[i]);
  }
  return w;
}

// The weights of a group's slots, times the scales of their values.
__device__ __forceinline__ bf16x8 scaled_weights(u32x4 w, uint2 scales) {
  uint32_t shift = 23;  // (unknown to the compiler, so that a byte is taken and shifted by one instruction)
  asm("" : "+v"(shift));
  bf16x8 pa;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t four = i < 2 ? scales.x : scales.y;
    const float a = __builtin_bit_cast(float, ((four >> (16 * (i & 1))) & 0xFFu) << shift);
    const float z = __builtin_bit_cast(float, ((four >> (16 * (i & 1) + 8)) & 0xFFu) << shift);
    pa[2 * i] = (__bf16)(low_of(w[i]) * a);
    pa[2 * i + 1] = (__bf16)(high_of(w[i]) * z);
  }
  return pa;
}

// ---- fused write of an 8-bit row (Section 6, "in-place writes") ------------------------------------
// The wavefront that holds step t's group quantises the step's key and value itself: lanes 0 .. D/8-1 hold the key row, 8
// dims each, the next D/8 the value row.  It writes them to the store, and puts them into the group's register image from a
// copy in LDS, [key codes D][value codes D][key scale byte][value scale byte], when it comes to that group.  A launch less
// than writing first (us a step, 24/8 heads of 128, fused / written first: 1 sequence, 300 keys 6.6 / 11.2; 32 sequences, 1000
// keys 12.6 / 15.5; even at 1024 pairs of 4000 keys, 175.0 / 173.3).
template <int D>
__device__ __forceinline__ u32x4 fetch_new_rows(const AttnParams& p, int b, int hkv, int lane) {
  const int lanes = D / 8, at = lane % (2 * lanes);  // (the lanes beyond hold copies)
  const uint16_t* const src = static_cast<const uint16_t*>(at < lanes ? p.k_new : p.v_new) + ((int64_t)b * p.Hkv + hkv) * D + (at % lanes) * 8;
  return *reinterpret_cast<const u32x4*>(src);
}

// slot: the number of the group's first slot among the store's `slots`.
template <int D, bool kRope>
__device__ __forceinline__ void write_new_rows(const AttnParams& p, u32x4 x, int t_b, int64_t slot, int64_t slots, bool store, int lane, uint8_t* stage) {
  constexpr int LANES = D / 8;
  if (kRope) {  // the partner dims, D/2 away, lie in lane ^ (LANES / 2)
    u32x4 other;
#pragma unroll
    for (int w = 0; w < 4; ++w) other[w] = (uint32_t)__shfl_xor((int)x[w], LANES / 2);
    const int d = 8 * (lane % LANES);
    u32x4 lo = d < D / 2 ? x : other, hi = d < D / 2 ? other : x;
    rotate_pieces(p.rope_cos, p.rope_sin, t_b, D / 2, d % (D / 2), lo, hi);
    if (lane < LANES) x = d < D / 2 ? lo : hi;
  }
  const RowPiece r = quantise_piece<D>(x);
  if (lane >= 2 * LANES) return;
  const bool value = lane >= LANES;
  const int part = lane % LANES;
  *reinterpret_cast<uint2*>(stage + lane * 8) = uint2{r.lo, r.hi};
  if (part == 0) stage[2 * D + value] = (uint8_t)r.scale;
  if (store) store_piece<D>(static_cast<uint8_t*>(value ? p.v_pool : p.k_pool), slots, slot, t_b & 31, value, part, r);
}

template <int D>
__device__ __forceinline__ void patch_keys(int t_b, int lane, const uint8_t* stage, Image<D, true>& g) {
  const int u = t_b & 31, row = u & 15, tile = u >> 4, c = lane >> 4;
  if ((lane & 15) != row) return;
#pragma unroll
  for (int w = 0; w < D / 64; ++w) {
    const uint2 a = *reinterpret_cast<const uint2*>(stage + 64 * w + 8 * c), b = *reinterpret_cast<const uint2*>(stage + 64 * w + 32 + 8 * c);
    const u32x4 val = {a.x, a.y, b.x, b.y};
    g.k[w] = tile == 0 ? val : g.k[w];
    g.k[D / 64 + w] = tile == 1 ? val : g.k[D / 64 + w];
  }
  const uint32_t E = stage[2 * D];
  g.k_scales = tile == 0 ? (g.k_scales & 0xFF00u) | E : (g.k_scales & 0xFFu) | (E << 8);
}

template <int D>
__device__ __forceinline__ void patch_values(int t_b, int lane, const uint8_t* stage, Image<D, true>& g) {
  const int u = t_b & 31, row = u & 15, tile = u >> 4, n = lane & 15, shift = 8 * (row & 3);
  if ((lane >> 4) != (row >> 2)) return;
  const uint32_t others = ~(0xFFu << shift);
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
    const uint32_t a = (uint32_t)stage[D + 32 * w + n] << shift, b = (uint32_t)stage[D + 32 * w + 16 + n] << shift;
    g.v[w].x = tile == 0 ? (g.v[w].x & others) | a : g.v[w].x;
    g.v[w].y = tile == 1 ? (g.v[w].y & others) | a : g.v[w].y;
    g.v[w].z = tile == 0 ? (g.v[w].z & others) | b : g.v[w].z;
    g.v[w].w = tile == 1 ? (g.v[w].w & others) | b : g.v[w].w;
  }
  const uint32_t E = (uint32_t)stage[2 * D + 1] << shift;
  g.v_scales.x = tile == 0 ? (g.v_scales.x & others) | E : g.v_scales.x;
  g.v_scales.y = tile == 1 ? (g.v_scales.y & others) | E : g.v_scales.y;
}

// Merge of the workgroup's wavefronts, as in attn_partial_bf16.hip; column j is column first_col + j of the call.
template <int D, int NW, bool kSelect>
__device__ __forceinline__ void merge_units(const AttnParams& p, const float* smem, int first_col, int ncols, int b, int hkv, int split) {
  const float* sm_m = smem;
  const float* sm_l = smem + NW * 16;
  const float* sm_acc = smem + NW * 32;
  // A thread takes 4 dims of a column at a time (one by one, a single wavefront's 16 columns of 128 took 9.5 us a launch of
  // one group, 5.6 now).
  for (int idx = threadIdx.x; idx < ncols * (D / 4); idx += 64 * NW) {
    const int j = idx / (D / 4), d = 4 * (idx % (D / 4));
    float mw[NW], lw[NW];
    f32x4 aw[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      mw[w] = sm_m[w * 16 + j];
      lw[w] = sm_l[w * 16 + j];
      aw[w] = *reinterpret_cast<const f32x4*>(sm_acc + (w * ncols + j) * D + d);
    }
    float M = mw[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, mw[w]);
    const float ref = M == -INFINITY ? 0.f : M;  // nothing seen, or nothing but NaN, which has to show
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const bool seen = lw[w] != 0.f;  // (a column's largest weight is at least 2^-kSlack)
      const float wgt = fast_exp2(mw[w] - ref);
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += seen ? wgt * aw[w][e] : 0.f;
      den += seen ? wgt * lw[w] : 0.f;
    }
    const int jc = (first_col + j) / p.G, jg = first_col + j - jc * p.G;
    if (p.direct) {
      const int64_t orow = ((int64_t)b * p.io_steps + jc) * p.Hq + (int64_t)hkv * p.G + jg;
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (__bf16)(kSelect && den == 0.f ? 0.f : num[e] / den);  // (a list may name no key)
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.out) + orow * D + d) = o;
    } else {
      const int64_t row = ((int64_t)b * p.queries + jc) * p.Hq + (int64_t)hkv * p.G + jg;
      const int64_t part = row * p.num_splits + split;
      *reinterpret_cast<f32x4*>(p.ws_acc + part * D + d) = num;
      if (d == 0) {
        p.ws_ml[part * 2] = M;
        p.ws_ml[part * 2 + 1] = den;
      }
    }
  }
}

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
