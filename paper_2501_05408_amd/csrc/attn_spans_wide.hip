// Attention over a window with sinks, and of a tree, for many (row, head) columns: prompts, and trees of many nodes or wide groups.
//
// The rows, what they see and how their groups are numbered: attn_spans.hip.  The products as in attn_prefill_bf16.hip: 32 columns
// to a wavefront as the columns of 32x32x16 products (logits = K Q^T, answers = V^T P^T, so that a lane's logits, weights, sum and
// accumulators are of one column), every group of 32 slots staged in LDS once for the workgroup's NW wavefronts, the logits of a group
// computed an iteration ahead of its weights.  What differs: rows see sinks, windows and ancestors; tiles of 64 to 128 columns (even ones: a
// wavefront beyond its tile's columns copies, and meets the others); and how groups come into LDS:
//   bf16    copied straight into the image that the products read, four buffers: three groups in flight, one read.
//   8 bits  copied as they lie (codes and scale bytes) into three buffers of their own, and turned from there into bf16 images, three as
//           well, by the wavefront that copied the piece (a quarter of the group each), two groups ahead of the logits.
// LDS of a workgroup, D = 128: bf16 64 KiB, 8 bits 72.75, and the bits of a tree (up to 11 KiB).  Two to a unit, as the splits are planned
// (wide_split_groups()), but for 8-bit trees of more than 206 nodes, one: us, 4 trees of 206 / 208 nodes of 32/4 heads behind 7000 keys
// 158 / 220, bf16 133 / 134.
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

// The same where only one end matters: slots behind `hi`, or before `lo`, which are numbered from the lane's first of the group on (two
// instructions a logit for six).
__device__ __forceinline__ void mask_behind(int hi, f32x16& x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 8 * (r >> 2) + (r & 3) <= hi ? x[r] : -INFINITY;
}
__device__ __forceinline__ void mask_before(int lo, f32x16& x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 8 * (r >> 2) + (r & 3) >= lo ? x[r] : -INFINITY;
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

// Eight codes as bf16, under one scale.
__device__ __forceinline__ u32x4 bf16_of(uint32_t a, uint32_t b, float scale) {
  const bf16x2 r[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return __builtin_bit_cast(u32x4, r);
}
// Codes of 8 slots for each of two dims, under a scale for each slot: a pair of one slot's is turned by one instruction.
__device__ __forceinline__ void bf16_of_slots(u32x4 codes, uint2 scales, u32x4& a, u32x4& z) {
  uint32_t shift = 23;  // (unknown to the compiler, so that a byte is taken and shifted by one instruction)
  asm("" : "+v"(shift));
#pragma unroll
  for (int i = 0; i < 4; ++i) {               // slots 2i, 2i + 1
    const uint32_t both = __builtin_amdgcn_perm(i < 2 ? codes.z : codes.w, i < 2 ? codes.x : codes.y, i & 1 ? 0x07030602u : 0x05010400u);
    const uint32_t four = i < 2 ? scales.x : scales.y;
    const float s = __builtin_bit_cast(float, ((four >> (16 * (i & 1))) & 0xFFu) << shift);
    const float t = __builtin_bit_cast(float, ((four >> (16 * (i & 1) + 8)) & 0xFFu) << shift);
    const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(both, s, false));
    const uint32_t v = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(both, t, true));
    a[i] = __builtin_amdgcn_perm(v, u, 0x05040100u);
    z[i] = __builtin_amdgcn_perm(v, u, 0x07060302u);
  }
}

template <int D, int NW, bool k8, bool kTree, bool kRope>
__global__ __launch_bounds__(64 * NW, 2) void attn_spans_wide(SpanParams p) {
  constexpr int KT = D / 16;                  // 16-dim contraction steps of the logits
  constexpr int OT = D / 32;                  // 32-dim tiles of the output
  constexpr int KU = D / 16;                  // 1 KiB units of one group's keys
  constexpr int UNITS = 2 * KU;               // ... and of its keys and values together
  constexpr int PER_WAVE = UNITS / NW;        // units each wavefront copies per group
  constexpr int NBUF = k8 ? 3 : 4, kBuf = UNITS * 64;
  constexpr int kRaw = KU * 64 + 4 * NW, kRaws = 3;  // 8 bits: a group's codes as they lie in the pools, and the scale bytes for each wavefront
  constexpr int CODES = KU / NW;              // 1 KiB units of codes, of keys or values, that each wavefront turns into bf16
  static_assert(KU % NW == 0, "copy split");
  extern __shared__ u32x4 lds[];              // [NBUF][UNITS][64] x 16 bytes: a group's keys, then its values; 8 bits: [kRaws][kRaw];
                                              // then the tree
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const UnitsWork item = wide_work(blockIdx.x, blockIdx.y, blockIdx.z, gridDim.x, gridDim.y, gridDim.z, p.Hkv,
                                   kTree ? 0 : fewer_keys(p.t, p.window, p.G, p.tile_columns, gridDim.x / (uint32_t)p.Hkv));
  const int hkv = item.hkv, b = item.b, split = item.split, block = item.tile;
  int t_b = p.t_per_seq ? ((const_i32_ptr)p.t_per_seq)[b] : p.t;
  t_b = t_b > p.t ? p.t : (t_b < 0 ? 0 : t_b);
  int rows = p.queries;
  if (p.count_per_seq) {
    const int n = ((const_i32_ptr)p.count_per_seq)[b];
    rows = n < 0 ? 0 : (n < rows ? n : rows);
  }
  const int first = block * p.tile_columns, all = rows * p.G;  // columns
  if (first >= all) return;                   // uniform over the workgroup, before any barrier
  const int ncols = all - first < p.tile_columns ? all - first : p.tile_columns;
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
  constexpr int kSlotBytes = k8 ? D : 2 * D;
  uint32_t tile_lo, tile_hi;                  // byte offset, in either pool, of the tile's first slot
  auto fetch_entry = [&]() {
    const int tile = tile_base + lane < tile_last ? tile_base + lane : tile_last;
    return table[tile & p.tile_mask];
  };
  auto place_tiles = [&](int found) {
    const uint64_t at = ((uint64_t)((int64_t)clamp_block(found, p.num_blocks) * p.Hkv + hkv) << p.z_log2) * kSlotBytes;
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
  // Groups are copied in their order: the next one, at last again and again the split's last, into buffers that nobody reads any
  // more (every iteration then issues the same number of copies, and "all but the newest have landed" is one counted wait).
  // Scalar instructions take the loop's issue slots as others do (94 an iteration and wavefront in its first form, 70 now).
  int next_group = from, next_key = key_of(from);
  auto next_offset = [&]() {                  // byte offset of the group in either pool
    const int tile = next_key >> p.z_log2;
    if (tile - tile_base >= 64) {
      tile_base = tile;
      place_tiles(fetch_entry());
    }
    const uint32_t lo = __builtin_amdgcn_readlane(tile_lo, tile - tile_base), hi = __builtin_amdgcn_readlane(tile_hi, tile - tile_base);
    const uint64_t at = (((uint64_t)hi << 32) | lo) + (uint32_t)(next_key & ((1 << p.z_log2) - 1)) * kSlotBytes;
    if (next_group < past - 1) {
      ++next_group;
      next_key = next_group == rg.sink_groups ? rg.g_lo << 5 : next_key + 32;
    }
    return at;
  };
  // Groups that hold slots no row sees, which may be unwritten: values there become 0.  The last of the sinks, the window's first,
  // the rows' last.
  const int edge_sinks = rg.sink_groups > 0 && 32 * rg.sink_groups > p.sinks ? rg.sink_groups - 1 : -1;
  const int edge_window = 32 * rg.g_lo < rg.lo ? rg.sink_groups : -1;
  const int edge_rows = ((t_last + 1) & 31) != 0 ? rg.groups - 1 : -1;
  auto masked = [&](int g) { return g == edge_sinks || g == edge_window || g == edge_rows; };

  // bf16: wavefront w copies units w, w + NW, ... straight into LDS.
  const uint32_t lane_bytes = 16u * (uint32_t)lane;
  char* const k_units = static_cast<char*>(p.k_pool) + 1024 * wave;
  char* const v_units = static_cast<char*>(p.v_pool) + 1024 * wave;
  auto issue = [&](int at) {
    const uint64_t from_byte = next_offset();
    const auto k = __builtin_amdgcn_make_buffer_rsrc(k_units + from_byte, 0, 1024 * KU, 0x00020000);
    const auto v = __builtin_amdgcn_make_buffer_rsrc(v_units + from_byte, 0, 1024 * KU, 0x00020000);
    u32x4* const to = lds + at + wave * 64;
#pragma unroll
    for (int i = 0; i < PER_WAVE / 2; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(k, (lds_ptr)(to + NW * i * 64), 16, lane_bytes, 1024 * NW * i, 0, 0);
#pragma unroll
    for (int i = 0; i < PER_WAVE / 2; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(v, (lds_ptr)(to + (KU + NW * i) * 64), 16, lane_bytes, 1024 * NW * i, 0, 0);
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
  // 8 bits: codes and scale bytes are copied into LDS as they are, three groups ahead of where a wavefront turns the pieces that it
  // copied itself into the same image: at D = 128 a unit of keys and one of values, at D = 64 one of either.
  constexpr int kCopies = CODES + 2;          // of a wavefront, a group
  const bool key_unit = CODES > 1 || wave < NW / 2;
  const int code_unit = CODES > 1 ? wave : wave % (NW / 2);
  const uint64_t scales_at = (((uint64_t)p.num_blocks * (uint64_t)p.Hkv) << p.z_log2) * D;
  auto fetch = [&](int raw) {
    const uint64_t from_byte = next_offset(), slot = from_byte / D;
    char *const k = static_cast<char*>(p.k_pool), *const v = static_cast<char*>(p.v_pool);
    const auto first = __builtin_amdgcn_make_buffer_rsrc((key_unit ? k : v) + from_byte + 1024 * code_unit, 0, 1024, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(first, (lds_ptr)(lds + raw + wave * 64), 16, lane_bytes, 0, 0, 0);
    if constexpr (CODES > 1) {
      const auto second = __builtin_amdgcn_make_buffer_rsrc(v + from_byte + 1024 * code_unit, 0, 1024, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(second, (lds_ptr)(lds + raw + (wave + NW) * 64), 16, lane_bytes, 0, 0, 0);
    }
    // (each wavefront its own copy of the 32 bytes of keys and of values: another may be a group ahead)
    if (lane < 8) {
      const auto ks = __builtin_amdgcn_make_buffer_rsrc(k + scales_at + slot, 0, 32, 0x00020000);
      const auto vs = __builtin_amdgcn_make_buffer_rsrc(v + scales_at + slot, 0, 32, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ks, (lds_ptr)(lds + raw + KU * 64 + 4 * wave), 4, 4 * lane, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vs, (lds_ptr)(lds + raw + KU * 64 + 4 * wave + 2), 4, 4 * lane, 0, 0, 0);
    }
  };
  struct Codes {
    u32x4 unit[CODES];
    uint32_t k_scales;
    uint2 v_scales;
  };
  // The oldest of three groups in flight.
  auto take = [&](int raw) {
    asm volatile("" ::: "memory");
    constexpr int kLeft = 2 * kCopies;
    __builtin_amdgcn_s_waitcnt((kLeft & 15) | 0x0F70 | ((kLeft >> 4) << 14));  // vmcnt only
    asm volatile("" ::: "memory");
    Codes c;
#pragma unroll
    for (int i = 0; i < CODES; ++i) c.unit[i] = lds[raw + (wave + NW * i) * 64 + lane];
    const char* const scales = reinterpret_cast<const char*>(lds + raw + KU * 64 + 4 * wave);
    c.k_scales = *reinterpret_cast<const uint16_t*>(scales + 2 * (lane & 15));
    c.v_scales = *reinterpret_cast<const uint2*>(scales + 32 + 8 * (lane >> 4));
    return c;
  };
  auto settle = [&](const Codes& c, int g, int at) {
    if (key_unit) {                           // tile code_unit / (D / 64), dims from 64 (code_unit mod (D / 64))
      const int tile = code_unit / (D / 64), w = code_unit % (D / 64);
      const float scale = scale_of((c.k_scales >> (8 * tile)) & 0xFFu);
      u32x4* const to = lds + at + (tile * (D / 32) + 2 * w) * 64 + lane;
      to[0] = bf16_of(c.unit[0].x, c.unit[0].y, scale);
      to[64] = bf16_of(c.unit[0].z, c.unit[0].w, scale);
    }
    if (CODES > 1 || !key_unit) {             // dims from 32 code_unit
      u32x4 a, z;
      bf16_of_slots(c.unit[CODES - 1], c.v_scales, a, z);
      if (masked(g)) {
        uint32_t keep[4];
        keep_values(key_of(g), rg.lo, t_last, p.sinks, lane, keep);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] &= keep[e];
          z[e] &= keep[e];
        }
      }
      u32x4* const to = lds + at + (KU + 2 * code_unit) * 64 + lane;
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
  auto next = [&](int ahead) {
    if constexpr (!k8) return (at0 + ahead * kBuf) & (NBUF * kBuf - 1);
    const int at = at0 + ahead * kBuf;
    return at < NBUF * kBuf ? at : at - NBUF * kBuf;
  };
  int raw0 = NBUF * kBuf;                     // LDS offset of the codes of group grp + 2

  // The first three groups.
  if constexpr (k8) {
    fetch(raw0);
    fetch(raw0 + kRaw);
    fetch(raw0 + 2 * kRaw);
  } else {
#pragma unroll
    for (int i = 0; i < NBUF - 1; ++i) issue(i * kBuf);
  }
  __builtin_amdgcn_sched_barrier(0);
  Tree tree;
  int position = t_b + row;
  if constexpr (kTree) {
    if (p.window > 0 || key_of(past - 1) + 31 >= t_b) {
      tree = tree_of(p.parents + (int64_t)b * p.queries, rows, p.window, p.sinks, t_b, reinterpret_cast<uint32_t*>(lds + NBUF * kBuf + (k8 ? kRaws * kRaw : 0)));
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
  // (numbers of groups: those of the sinks below sink_whole, and whole_first .. whole_last; a few that are whole may not count)
  const int behind = rg.sink_groups - rg.g_lo, sink_whole = (p.sinks >> 5) < rg.sink_groups ? p.sinks >> 5 : rg.sink_groups;
  const int whole_first = ((lo_last + 31) >> 5) + behind, whole_last = ((whole_hi + 1) >> 5) - 1 + behind;
  auto enter = [&](int g, f32x16& x, float mx) {
    if (g >= sink_whole && (g < whole_first || g > whole_last)) {
      const int key = key_of(g);
      if (key < p.sinks || (kTree && key + 31 >= t_b)) {
        uint32_t bits = 0;
        if constexpr (kTree) {
          if (key + 31 >= t_b) bits = tree.bits(row, key - t_b);
        }
        mask_span_tile<kTree>(key, lo_col, hi_col, p.sinks, bits, lane, x);
      } else {
        if (g > whole_last) mask_behind(hi_col - key - 4 * half, x);
        if (g < whole_first) mask_before(lo_col - key - 4 * half, x);
      }
      mx = tile_max(x);
    }
    softmax_reference<D>(mx, p.scale_log2e, limit, m_run, base, acc, l_run);
  };
  Codes codes;
  auto peek = [&]() {
    if constexpr (k8) codes = take(raw0);
  };
  auto copies = [&]() {                       // into the buffer of group grp - 1, which everybody finished before the last barrier
    if constexpr (k8) {
      settle(codes, grp + 2, next(2));
      __builtin_amdgcn_s_waitcnt(0xC07F);     // (they are in registers: the copy may go over them)
      fetch(raw0);
      raw0 = raw0 + kRaw < NBUF * kBuf + kRaws * kRaw ? raw0 + kRaw : NBUF * kBuf;
    } else {
      issue(next(NBUF - 1));
    }
  };
  auto mask_landed = [&](int g, int at) {
    if constexpr (!k8) {
      if (g < past && masked(g)) mask_values(g, at);
    }
  };
  auto finish = [&]() {
    landed();
    mask_landed(grp + 2, next(2));
    meet();
    at0 = next(1);
    ++grp;
  };
  if constexpr (k8) {                         // the first two
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const Codes c = take(raw0 + i * kRaw);
      settle(c, from + i, i * kBuf);
      __builtin_amdgcn_s_waitcnt(0xC07F);
      fetch(raw0 + i * kRaw);
    }
    raw0 += 2 * kRaw;
  }
  landed();
  mask_landed(from, 0);
  mask_landed(from + 1, kBuf);
  meet();
  while (grp < own_first && grp < past) {
    peek();
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
      if (s == KT) peek();
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
    peek();
    copies();
    finish();
  }
  // the copies issued last may still be in flight: they must land before the LDS is used again or given up
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  const float l_j = half_sum(l_run);
  if (p.direct) {                             // every row saw itself
    // Answers leave in whole rows: a wavefront's 32 columns pass through its quarter of the LDS, a column's 16-byte units in an order that
    // spreads them over the banks (4 x 4096 steps, window 1024, 259 us with 8 bytes a lane straight from the registers, 252; window 128
    // 130 and 121.  Partials, 16 bytes a lane, do not gain: 16 ragged trees of 32 nodes 35.9, through LDS 37.4).
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    constexpr int kRow = 2 * D, kUnits = kRow / 16, kRows = 64 / kUnits;
    __syncthreads();                          // all copies have landed, all operands have been read
    if (first_col >= ncols) return;
    char* const own = reinterpret_cast<char*>(lds) + wave * (kWaveColumns * kRow);
    const float inv = 1.0f / l_j;
    const int n = lane & 31, at_row = row * p.Hq + hkv * p.G + gq;
#pragma unroll
    for (int ot = 0; ot < OT; ++ot) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x4 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = (__bf16)(acc[ot][4 * i + r] * inv);
        *reinterpret_cast<bf16x4*>(own + n * kRow + 16 * ((4 * ot + i) ^ (n & (kUnits - 1))) + 8 * half) = o;
      }
    }
    char* const to = static_cast<char*>(p.out) + (int64_t)b * p.io_steps * p.Hq * kRow;
#pragma unroll
    for (int k = 0; k < kWaveColumns / kRows; ++k) {
      const int c = kRows * k + lane / kUnits, unit = lane % kUnits;
      const u32x4 v = *reinterpret_cast<const u32x4*>(own + c * kRow + 16 * (unit ^ (c & (kUnits - 1))));
      const int at = __shfl(at_row, c);
      if (first_col + c < ncols) *reinterpret_cast<u32x4*>(to + (int64_t)at * kRow + 16 * unit) = v;
    }
    return;
  }
  if (col >= ncols) return;
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

template <int D, int NW, bool k8>
hipError_t launch_wide(const SpanParams& p, int batch, hipStream_t stream) {
  const int blocks = (p.queries * p.G + p.tile_columns - 1) / p.tile_columns;
  const dim3 grid((unsigned)(p.Hkv * blocks), (unsigned)batch, (unsigned)p.num_splits), block(64 * NW);
  const size_t lds = (k8 ? 3 * ((size_t)(D / 8 + D / 16) * 1024 + 64 * NW) : 4 * (size_t)(D / 8) * 1024) + (p.parents ? tree_lds_bytes(p.queries) : 0);
  if (p.parents) return launch((attn_spans_wide<D, NW, k8, true, false>), grid, block, lds, stream, p);
  if (p.rope_cos) return launch((attn_spans_wide<D, NW, k8, false, true>), grid, block, lds, stream, p);
  return launch((attn_spans_wide<D, NW, k8, false, false>), grid, block, lds, stream, p);
}

}  // namespace

hipError_t launch_spans_wide(const SpanParams& p, int batch, int D, int dtype, hipStream_t stream) {
  const bool k8 = dtype == TEMPO_E4M3;
  if (p.tile_columns < kWaveColumns || p.tile_columns > 128 || p.tile_columns % kWaveColumns != 0) return hipErrorInvalidConfiguration;
  if (D == 128) return k8 ? launch_wide<128, 4, true>(p, batch, stream) : launch_wide<128, 4, false>(p, batch, stream);
  return k8 ? launch_wide<64, 4, true>(p, batch, stream) : launch_wide<64, 4, false>(p, batch, stream);
}

}  // namespace tempo
