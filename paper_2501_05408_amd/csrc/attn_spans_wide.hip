// Attention over a window with sinks, and of a tree, for many (row, head) columns: prompts, and trees of many nodes or wide groups.
//
// The rows, what they see and how their groups are numbered: attn_spans.hip.  The products as in attn_prefill_bf16.hip: 32 columns
// to a wavefront as the columns of 32x32x16 products (logits = K Q^T, answers = V^T P^T, so that a lane's logits, weights, sum and
// accumulators are of one column), every group of 32 slots staged in LDS once for the workgroup's NW wavefronts, four groups deep,
// the logits of a group computed an iteration ahead of its weights.  What differs: rows see sinks, windows and ancestors; a group
// of an 8-bit store is turned into bf16 on its way into LDS, by the wavefront that fetched the piece (a quarter of the group each),
// instead of by every wavefront that reads it.
#include "attn_bf16_columns32.h"
#include "attn_spans.h"
#include "attn_tree.h"
#include "store_e4m3.h"

namespace tempo {
namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kWaveColumns = 32;

template <bool kTree>
__device__ __forceinline__ void mask_span_tile(int key, int lo, int hi, int sinks, uint32_t bits, int lane, f32x16& x) {
  const int first = 4 * (lane >> 5);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int at = first + 8 * (r >> 2) + (r & 3), j = key + at;
    bool seen = j <= hi && (j >= lo || j < sinks);
    if (kTree) seen = seen || ((bits >> at) & 1u) != 0;
    x[r] = seen ? x[r] : -INFINITY;
  }
}

// Of the 8 slots of lane (n + 16c)'s pieces of values those that some row may see: two to a word.
__device__ __forceinline__ void keep_values(int key, int lo, int last, int sinks, int lane, uint32_t* keep) {
  const int c = (lane >> 4) & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) keep[i] = 0u;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int j = key + 4 * c + (r & 3) + 16 * (r >> 2);
    keep[r >> 1] |= (j <= last && (j >= lo || j < sinks) ? 0xFFFFu : 0u) << (16 * (r & 1));
  }
}

// Eight codes as bf16, under one scale, or under one each.
__device__ __forceinline__ u32x4 bf16_of(uint32_t a, uint32_t b, float scale) {
  const bf16x2 r[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return __builtin_bit_cast(u32x4, r);
}
__device__ __forceinline__ u32x4 bf16_of_each(uint32_t a, uint32_t b, const float* scale) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 v[4] = {__builtin_amdgcn_cvt_pk_f32_fp8(a, false), __builtin_amdgcn_cvt_pk_f32_fp8(a, true),
                      __builtin_amdgcn_cvt_pk_f32_fp8(b, false), __builtin_amdgcn_cvt_pk_f32_fp8(b, true)};
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // (exact: a code has 4 bits)
    const bf16x2 pair = {(__bf16)(v[i][0] * scale[2 * i]), (__bf16)(v[i][1] * scale[2 * i + 1])};
    w[i] = __builtin_bit_cast(uint32_t, pair);
  }
  return w;
}

template <int D, int NW, bool k8, bool kTree, bool kRope>
__global__ __launch_bounds__(64 * NW, 2) void attn_spans_wide(SpanParams p) {
  constexpr int KT = D / 16;                  // 16-dim contraction steps of the logits
  constexpr int OT = D / 32;                  // 32-dim tiles of the output
  constexpr int KU = D / 16;                  // 1 KiB units of one group's keys
  constexpr int UNITS = 2 * KU;               // ... and of its keys and values together
  constexpr int PER_WAVE = UNITS / NW;        // units each wavefront copies per group
  constexpr int NBUF = 4, kBuf = UNITS * 64;
  constexpr int CODES = KU / NW;              // 1 KiB units of codes, of keys or values, that each wavefront turns into bf16
  static_assert(KU % NW == 0, "copy split");
  extern __shared__ u32x4 lds[];              // [NBUF][UNITS][64] x 16 bytes: a group's keys, then its values; then the tree
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // Workgroups go to the 8 dies round-robin by linear index; each die gets a contiguous run of the list, in which the blocks of
  // one (sequence, kv head, split), which read the same keys, are neighbours.
  const unsigned nx = gridDim.x, ny = gridDim.y, total = nx * ny * gridDim.z;
  const unsigned linear = blockIdx.x + nx * (blockIdx.y + ny * blockIdx.z);
  const unsigned die = linear & 7u, share = total >> 3, extra = total & 7u;
  const unsigned item = die * share + (die < extra ? die : extra) + (linear >> 3);
  const unsigned ix = item % nx, iyz = item / nx;
  const int hkv = (int)(iyz % ny), b = (int)(iyz / ny);
  const unsigned nblocks = nx / (unsigned)p.num_splits;
  const int split = (int)(ix / nblocks), block = (int)(nblocks - 1 - ix % nblocks);

  int t_b = p.t_per_seq ? ((const_i32_ptr)p.t_per_seq)[b] : p.t;
  t_b = t_b > p.t ? p.t : (t_b < 0 ? 0 : t_b);
  int rows = p.queries;
  if (p.count_per_seq) {
    const int n = ((const_i32_ptr)p.count_per_seq)[b];
    rows = n < 0 ? 0 : (n < rows ? n : rows);
  }
  const int first = block * (kWaveColumns * NW), all = rows * p.G;  // columns
  if (first >= all) return;                   // uniform over the workgroup, before any barrier
  const int ncols = all - first < kWaveColumns * NW ? all - first : kWaveColumns * NW;
  const int c0 = first / p.G, skip = first - c0 * p.G, row_last = c0 + (skip + ncols - 1) / p.G;
  const SpanRange rg = span_range(t_b, kTree ? 0 : c0, row_last, p.window, p.sinks);
  const int from = split * p.split_groups;
  if (from >= rg.groups) return;
  const int past = from + p.split_groups < rg.groups ? from + p.split_groups : rg.groups;
  const int t_last = t_b + row_last;          // newest slot that a row may see
  auto key_of = [&](int g) { return span_group(rg, g) << 5; };

  // The block-table entries of 64 tiles, one per lane, from that of the first group on.
  const int32_t* table = p.block_table + (int64_t)b * p.max_blocks_per_seq;
  const int tile_last = key_of(past - 1) >> p.z_log2;
  int tile_base = key_of(from) >> p.z_log2;
  uint32_t tile_lo, tile_hi;                  // slot number of the tile's first slot
  auto fetch_entry = [&]() {
    const int tile = tile_base + lane < tile_last ? tile_base + lane : tile_last;
    return table[tile & p.tile_mask];
  };
  auto place_tiles = [&](int found) {
    const uint64_t at = (uint64_t)((int64_t)clamp_block(found, p.num_blocks) * p.Hkv + hkv) << p.z_log2;
    tile_lo = (uint32_t)at;
    tile_hi = (uint32_t)(at >> 32);
    asm volatile("" : "+v"(tile_lo), "+v"(tile_hi));  // waited for here, not among the copies in flight
  };
  const int entry = fetch_entry();

  // This wavefront's rows, and its lane's column.
  const int first_col = kWaveColumns * wave, half = lane >> 5, col = first_col + (lane & 31);
  const bool idle = first_col >= ncols;
  const int wave_end = first_col + kWaveColumns - 1 < ncols - 1 ? first_col + kWaveColumns - 1 : ncols - 1;
  const int r_lo = idle ? c0 : c0 + (skip + first_col) / p.G, r_hi = idle ? c0 : c0 + (skip + wave_end) / p.G;
  const int row = col < ncols ? c0 + (skip + col) / p.G : row_last, gq = col < ncols ? skip + col - (row - c0) * p.G : 0;
  u32x4 qreg[KT];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(p.q) + (((int64_t)b * p.io_steps + row) * p.Hq + (int64_t)hkv * p.G + gq) * D + 8 * half;
#pragma unroll
    for (int s = 0; s < KT; ++s) qreg[s] = *reinterpret_cast<const u32x4*>(qp + 16 * s);
  }
  __builtin_amdgcn_sched_barrier(0);          // ... on their way before the first copies are, and used behind them
  float m_run = -INFINITY;                    // softmax reference of this lane's column (log2 units)
  float l_run = 0.f;                          // running sum over this lane's slots
  f32x16 acc[OT];                             // dims 32 ot + 8 (r / 4) + 4 h + (r mod 4) of this lane's column
#pragma unroll
  for (int ot = 0; ot < OT; ++ot) {
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[ot][r] = 0.f;
  }

  place_tiles(entry);
  auto slot_of = [&](int key) {               // of a group's first slot, among the store's slots
    const int tile = key >> p.z_log2;
    if (tile - tile_base >= 64) {
      tile_base = tile;
      place_tiles(fetch_entry());
    }
    const uint32_t lo = __builtin_amdgcn_readlane(tile_lo, tile - tile_base), hi = __builtin_amdgcn_readlane(tile_hi, tile - tile_base);
    return (((uint64_t)hi << 32) | lo) + (uint32_t)(key & ((1 << p.z_log2) - 1));
  };
  // A group that holds slots no row sees, which may be unwritten: its values there become 0.
  auto masked = [&](int key) { return key + 31 > t_last || (key < rg.lo && key + 31 >= p.sinks); };

  // bf16: wavefront w copies units w, w + NW, ... straight into LDS.  Beyond the last group that one is copied again, into a
  // buffer that nobody reads any more: every iteration then issues the same number of copies, and "all but the newest group has
  // landed" is one counted wait.
  const uint32_t lane_bytes = 16u * (uint32_t)lane;
  auto issue = [&](int at, int g) {
    const uint64_t slot = slot_of(key_of(g < past ? g : past - 1));
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      const int u = wave + NW * i;            // wave-uniform
      char* const pool = static_cast<char*>(u < KU ? p.k_pool : p.v_pool) + slot * (2 * D) + (u < KU ? u : u - KU) * 1024;
      const auto unit = __builtin_amdgcn_make_buffer_rsrc(pool, 0, 1024, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(unit, (lds_ptr)(lds + at + u * 64), 16, lane_bytes, 0, 0, 0);
    }
  };
  auto mask_values = [&](int g, int at) {
    uint32_t keep[4];
    keep_values(key_of(g), rg.lo, t_last, p.sinks, lane, keep);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      const int u = wave + NW * i;
      if (u >= KU) mask_piece(lds + at + u * 64 + lane, keep);
    }
  };
  // 8 bits: the wavefront's codes of a group wait in registers for an iteration, and are turned into the same image.
  struct Codes {
    u32x4 unit[CODES];
    uint32_t k_scales;
    uint2 v_scales;
  };
  auto fetch = [&](int g) {
    const uint64_t slot = slot_of(key_of(g < past ? g : past - 1)), slots = ((uint64_t)p.num_blocks * (uint64_t)p.Hkv) << p.z_log2;
    const char *const k = static_cast<const char*>(p.k_pool), *const v = static_cast<const char*>(p.v_pool);
    Codes c;
#pragma unroll
    for (int i = 0; i < CODES; ++i) {
      const int u = wave + NW * i;            // wave-uniform: keys, then values
      c.unit[i] = *reinterpret_cast<const u32x4*>((u < KU / 2 ? k : v) + slot * D + (u < KU / 2 ? u : u - KU / 2) * 1024 + lane_bytes);
    }
    c.k_scales = *reinterpret_cast<const uint16_t*>(k + slots * D + slot + 2 * (lane & 15));
    c.v_scales = *reinterpret_cast<const uint2*>(v + slots * D + slot + 8 * (lane >> 4));
    return c;
  };
  auto settle = [&](const Codes& c, int g, int at) {
    const int key = key_of(g < past ? g : past - 1);
#pragma unroll
    for (int i = 0; i < CODES; ++i) {
      const int u = wave + NW * i;
      if (u < KU / 2) {                       // keys: tile u / (D / 64), dims from 64 (u mod (D / 64))
        const int tile = u / (D / 64), w = u % (D / 64);
        const float scale = scale_of(tile ? c.k_scales >> 8 : c.k_scales & 0xFFu);
        u32x4* const to = lds + at + (tile * (D / 32) + 2 * w) * 64 + lane;
        to[0] = bf16_of(c.unit[i].x, c.unit[i].y, scale);
        to[64] = bf16_of(c.unit[i].z, c.unit[i].w, scale);
        continue;
      }
      float scale[8];                         // values: dims from 32 (u - KU / 2)
#pragma unroll
      for (int r = 0; r < 8; ++r) scale[r] = scale_of((r < 4 ? c.v_scales.x >> (8 * r) : c.v_scales.y >> (8 * (r - 4))) & 0xFFu);
      u32x4 a = bf16_of_each(c.unit[i].x, c.unit[i].y, scale), z = bf16_of_each(c.unit[i].z, c.unit[i].w, scale);
      if (masked(key)) {
        uint32_t keep[4];
        keep_values(key, rg.lo, t_last, p.sinks, lane, keep);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] &= keep[e];
          z[e] &= keep[e];
        }
      }
      u32x4* const to = lds + at + 2 * u * 64 + lane;  // (KU units of keys before them)
      to[0] = a;
      to[64] = z;
    }
  };
  // landed(): all but the newest group's copies of this wavefront are in LDS.  (Waits and barriers written out: attn_prefill_bf16.hip.)
  auto landed = [&]() {
    if constexpr (k8) return;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((PER_WAVE & 15) | 0x0F70 | ((PER_WAVE >> 4) << 14));  // vmcnt only
    asm volatile("" ::: "memory");
  };
  auto meet = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);       // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // Operands, as in attn_prefill_bf16.hip.
  const int k_lane = ((lane >> 4) & 1) * (D / 32) * 64 + (lane & 15) + 16 * half;
  auto key_operand = [&](int at, int s) { return as_bf16x8(lds[at + k_lane + (s >> 1) * 64 + (s & 1) * 32]); };
  const int v_lane = KU * 64 + ((lane >> 4) & 1) * 64 + (lane & 15) + 16 * half;
  auto value_operand = [&](int at, int chunk, int ot) { return as_bf16x8(lds[at + v_lane + ot * 128 + chunk * 32]); };

  int grp = from, at0 = 0;                    // LDS offset of the buffer of group grp
  auto next = [&](int ahead) { return (at0 + ahead * kBuf) & (NBUF * kBuf - 1); };

  // The first three groups.
  Codes held;
  if constexpr (k8) {
    const Codes a = fetch(from), b = fetch(from + 1), c = fetch(from + 2);
    held = fetch(from + 3);
    settle(a, from, 0);
    settle(b, from + 1, kBuf);
    settle(c, from + 2, 2 * kBuf);
  } else {
#pragma unroll
    for (int i = 0; i < NBUF - 1; ++i) issue(i * kBuf, from + i);
  }
  __builtin_amdgcn_sched_barrier(0);
  Tree tree;
  int position = t_b + row;
  if constexpr (kTree) {
    if (p.window > 0 || key_of(past - 1) + 31 >= t_b) {
      tree = tree_of(p.parents + (int64_t)b * p.queries, rows, p.window, p.sinks, t_b, reinterpret_cast<uint32_t*>(lds + NBUF * kBuf));
      if (p.window > 0) position = t_b + tree.depth(row);
    }
  }
  const int hi_col = kTree ? t_b - 1 : position, lo_col = p.window > 0 && position - p.window + 1 > 0 ? position - p.window + 1 : 0;
#pragma unroll
  for (int s = 0; s < KT; ++s) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    qreg[s] = col < ncols ? qreg[s] : zero;
  }
  if (kRope) {                                // queries arrive unrotated; a dim's partner D/2 further sits in the same lane
#pragma unroll
    for (int s = 0; s < KT / 2; ++s)
      rotate_pieces(p.rope_cos, p.rope_sin, position, D / 2, 16 * s + 8 * half, qreg[s], qreg[s + KT / 2]);
  }

  // The groups in which this wavefront has work, and which of them all of its columns see whole.
  const int whole_hi = kTree ? t_b - 1 : t_b + r_lo;
  const int lo_last = p.window > 0 && t_b + r_hi - p.window + 1 > 0 ? t_b + r_hi - p.window + 1 : 0;
  const int lo_first = kTree ? rg.lo : p.window > 0 && t_b + r_lo - p.window + 1 > 0 ? t_b + r_lo - p.window + 1 : 0;
  const int hi_at = ((t_b + r_hi) >> 5) - rg.g_lo + rg.sink_groups, lo_at = (lo_first >> 5) - rg.g_lo + rg.sink_groups;
  const int own_first = idle ? past : (key_of(from) < p.sinks || lo_at < from ? from : lo_at);
  const int own_last = idle ? past - 1 : (hi_at < past - 1 ? hi_at : past - 1);
  float base = 0.f;                           // m_run, or 0 while the column has seen no key
  float limit = -INFINITY;                    // raw dot product from which on m_run has to move
  auto enter = [&](int g, f32x16& x, float mx) {
    const int key = key_of(g);
    if (key + 31 > whole_hi || (key < lo_last && key + 31 >= p.sinks)) {
      uint32_t bits = 0;
      if constexpr (kTree) {
        if (key + 31 >= t_b) bits = tree.bits(row, key - t_b);
      }
      mask_span_tile<kTree>(key, lo_col, hi_col, p.sinks, bits, lane, x);
      mx = tile_max(x);
    }
    softmax_reference<D>(mx, p.scale_log2e, limit, m_run, base, acc, l_run);
  };
  auto copies = [&]() {                       // into the buffer of group grp - 1, which everybody finished before the last barrier
    if constexpr (k8) {
      settle(held, grp + NBUF - 1, next(NBUF - 1));
      held = fetch(grp + NBUF);
    } else {
      issue(next(NBUF - 1), grp + NBUF - 1);
    }
  };
  auto mask_landed = [&](int g, int at) {
    if constexpr (!k8) {
      if (g < past && masked(key_of(g))) mask_values(g, at);
    }
  };
  auto finish = [&]() {
    landed();
    mask_landed(grp + 2, next(2));
    meet();
    at0 = next(1);
    ++grp;
  };
  landed();
  mask_landed(from, 0);
  mask_landed(from + 1, kBuf);
  meet();
  while (grp < own_first && grp < past) {
    copies();
    finish();
  }
  constexpr int kRead = KT, kSlots = KT + 2 * OT;
  bf16x8 op[kSlots];                          // keys of group grp + 1, then values of group grp
  auto read_operand = [&](int i) {
    op[i] = i < KT ? key_operand(next(1), i) : value_operand(at0, (i - KT) / OT, (i - KT) % OT);
  };
  f32x16 xa, xb;                              // logits of group grp, masked, its reference already moved: in turn
  if (grp <= own_last) {
#pragma unroll
    for (int r = 0; r < 16; ++r) xa[r] = 0.f;
#pragma unroll
    for (int s = 0; s < KT; ++s)
      xa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_operand(at0, s), as_bf16x8(qreg[s]), xa, 0, 0, 0);
    enter(grp, xa, tile_max(xa));
  }
  // Group grp, logits in xc; those of group grp + 1 to xn.
  auto iterate = [&](const f32x16& xc, f32x16& xn) {
#pragma unroll
    for (int i = 0; i < kRead; ++i) read_operand(i);
    u32x4 pa[2];
    float even, mx[5];
#pragma unroll
    for (int r = 0; r < 16; ++r) xn[r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if (s < KT) {
        xn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[s], as_bf16x8(qreg[s]), xn, 0, 0, 0);
      } else {
        const int ot = (s - KT) % OT;
        acc[ot] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[s], as_bf16x8(pa[(s - KT) / OT]), acc[ot], 0, 0, 0);
      }
      if (s + kRead < kSlots) read_operand(s + kRead);
      if (s == KT + OT) copies();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (i * (KT + OT) / 16 == s) softmax_weight(xc, p.scale_log2e, base, i, even, pa, l_run);
      }
      if (s >= KT + OT) {
#pragma unroll
        for (int i = 0; i < 5; ++i) {
          if (i * OT / 5 == s - KT - OT) {
            mx[i] = max3(xn[3 * i], xn[3 * i + 1], xn[3 * i + 2]);
            asm volatile("" : "+v"(mx[i]));   // here, not behind the products
          }
        }
      }
      asm volatile("" : "+v"(l_run));
      __builtin_amdgcn_sched_barrier(0);
    }
    if (grp < own_last) enter(grp + 1, xn, max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], xn[15]), xn[15]));
    finish();
  };
  while (grp <= own_last) {
    iterate(xa, xb);
    if (grp > own_last) break;
    iterate(xb, xa);
  }
  while (grp < past) {
    copies();
    finish();
  }
  // the copies issued last may still be in flight: they must land before the LDS is given up
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  const float l_j = half_sum(l_run);
  if (col >= ncols) return;
  if (p.direct) {                             // every row saw itself
    __bf16* orow = static_cast<__bf16*>(p.out) + (((int64_t)b * p.io_steps + row) * p.Hq + (int64_t)hkv * p.G + gq) * D + 4 * half;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const float inv = 1.0f / l_j;
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x4 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = (__bf16)(acc[ot][4 * i + r] * inv);
        *reinterpret_cast<bf16x4*>(orow + 32 * ot + 8 * i) = o;
      }
    }
  } else {
    const int64_t part = (((int64_t)b * p.queries + row) * p.Hq + (int64_t)hkv * p.G + gq) * p.num_splits + split;
    float* arow = p.ws_acc + part * D + 4 * half;
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(arow + 32 * ot + 8 * i) = f32x4{acc[ot][4 * i], acc[ot][4 * i + 1], acc[ot][4 * i + 2], acc[ot][4 * i + 3]};
    }
    if (half == 0) {
      p.ws_ml[part * 2] = m_run;
      p.ws_ml[part * 2 + 1] = l_j;
    }
  }
}

template <int D, int NW, bool k8>
hipError_t launch_wide(const SpanParams& p, int batch, hipStream_t stream) {
  const int blocks = (p.queries * p.G + p.tile_columns - 1) / p.tile_columns;
  const dim3 grid((unsigned)(blocks * p.num_splits), (unsigned)p.Hkv, (unsigned)batch), block(64 * NW);
  const size_t lds = 4 * (size_t)(D / 8) * 1024 + (p.parents ? tree_lds_bytes(p.queries) : 0);
  if (p.parents) return launch((attn_spans_wide<D, NW, k8, true, false>), grid, block, lds, stream, p);
  if (p.rope_cos) return launch((attn_spans_wide<D, NW, k8, false, true>), grid, block, lds, stream, p);
  return launch((attn_spans_wide<D, NW, k8, false, false>), grid, block, lds, stream, p);
}

}  // namespace

hipError_t launch_spans_wide(const SpanParams& p, int batch, int D, int dtype, hipStream_t stream) {
  const bool k8 = dtype == TEMPO_E4M3;
  if (p.tile_columns != 128) return hipErrorInvalidConfiguration;
  if (D == 128) return k8 ? launch_wide<128, 4, true>(p, batch, stream) : launch_wide<128, 4, false>(p, batch, stream);
  return k8 ? launch_wide<64, 4, true>(p, batch, stream) : launch_wide<64, 4, false>(p, batch, stream);
}

}  // namespace tempo
