// A 32-slot group of a bf16 or 8-bit store as the registers of a wavefront: requests, products, weights, the fused write of an 8-bit
// row, and the merge of a workgroup's wavefronts.  Shared by attn_units.hip, whose head describes the method, and attn_spans.hip.
#pragma once

#include "attn_bf16_common.h"
#include "attn_units.h"
#include "store_e4m3.h"

namespace tempo {
namespace {

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

// The rows of fetch_new_rows(), the key turned to its position.
template <int D, bool kRope>
__device__ __forceinline__ u32x4 turn_new_row(const AttnParams& p, u32x4 x, int t_b, int lane) {
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
  return x;
}

// slot: the number of the group's first slot among the store's `slots`.
template <int D, bool kRope>
__device__ __forceinline__ void write_new_rows(const AttnParams& p, u32x4 x, int t_b, int64_t slot, int64_t slots, bool store, int lane, uint8_t* stage) {
  constexpr int LANES = D / 8;
  x = turn_new_row<D, kRope>(p, x, t_b, lane);
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

// The same for a bf16 row: [key D][value D] in LDS.  (Only the row's own pieces are written: 16 bytes of a key, single values.)
template <int D, bool kRope>
__device__ __forceinline__ void write_new_rows_bf16(const AttnParams& p, u32x4 x, int t_b, int64_t slot, bool store, int lane, uint16_t* stage) {
  constexpr int LANES = D / 8;
  x = turn_new_row<D, kRope>(p, x, t_b, lane);
  if (lane >= 2 * LANES) return;
  *reinterpret_cast<u32x4*>(stage + lane * 8) = x;
  if (!store) return;
  const int part = lane % LANES;
  if (lane < LANES) {
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.k_pool) + slot * D + tile_off_k_bf16(D, t_b & 31, 8 * part)) = x;
  } else {
    uint16_t* const to = static_cast<uint16_t*>(p.v_pool) + slot * D + tile_off_v_bf16(D, t_b & 31, 8 * part);  // dims 8 elements apart
#pragma unroll
    for (int e = 0; e < 8; ++e) to[8 * e] = (uint16_t)(x[e >> 1] >> (16 * (e & 1)));
  }
}

template <int D>
__device__ __forceinline__ void patch_keys_bf16(int t_b, int lane, const uint16_t* stage, Image<D, false>& g) {
  const int u = t_b & 31, row = u & 15, tile = u >> 4, c = lane >> 4;
  if ((lane & 15) != row) return;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const u32x4 val = *reinterpret_cast<const u32x4*>(stage + 32 * s + 8 * c);
    g.k[s] = tile == 0 ? val : g.k[s];
    g.k[D / 32 + s] = tile == 1 ? val : g.k[D / 32 + s];
  }
}

template <int D>
__device__ __forceinline__ void patch_values_bf16(int t_b, int lane, const uint16_t* stage, Image<D, false>& g) {
  const int u = t_b & 31, row = u & 15, tile = u >> 4, n = lane & 15;
  if ((lane >> 4) != (row >> 2)) return;
  const int e = (row & 3) + 4 * tile;  // place of the slot among the lane's 8
  const uint32_t shift = (e & 1) ? 16u : 0u, others = (e & 1) ? 0x0000FFFFu : 0xFFFF0000u;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const uint32_t val = (uint32_t)stage[D + 16 * dt + n] << shift;
#pragma unroll
    for (int w = 0; w < 4; ++w) g.v[dt][w] = w == (e >> 1) ? (g.v[dt][w] & others) | val : g.v[dt][w];
  }
}

// Merge of the workgroup's wavefronts, as in attn_partial_bf16.hip; column j is column first_col + j of the call.
template <int D, int NW, bool kSelect, bool kBf16 = true>
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
    if (p.direct && !kBf16) {
      const int64_t orow = ((int64_t)b * p.io_steps + jc) * p.Hq + (int64_t)hkv * p.G + jg;
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + orow * D + d) = f32x4{num[0] / den, num[1] / den, num[2] / den, num[3] / den};
    } else if (p.direct) {
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

}  // namespace
}  // namespace tempo
