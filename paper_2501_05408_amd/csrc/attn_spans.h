// What the launches of attn_spans*.hip and kv_place.hip take, on top of tempo_internal.h.
#pragma once

#include "attn_units.h"
#include "tempo_internal.h"

namespace tempo {

constexpr int kMaxNodes = 256;  // of a tree: a row's ancestors are 8 words

// Attention of `queries` rows a sequence over the first `sinks` keys, a window, and the nodes of a tree among the rows.
// queries: rows of a sequence (count_per_seq[b] of them, if given); t: step of row 0, for a tree the first node's.
struct SpanParams : AttnParams {
  const int32_t* parents;   // null: rows are consecutive steps; [batch][queries]: row i's parent among the rows, -1: none
  int32_t sinks;
  int32_t tile_columns;     // (row, head) columns of a workgroup, which walks the keys that its own rows see
  int32_t split_groups;     // 32-key groups of a split
};

// The keys that rows first .. last of a sequence whose row 0 is step t see some of, as whole 32-slot groups: `sink_groups` from
// step 0 on, and those from group g_lo to that of the last row's step.  Without a window: from step 0 on.
// A tree's rows are no deeper than their number, so its windows begin where row 0's does.
struct SpanRange {
  int lo;           // first key of the window of the rows' first
  int sink_groups;  // groups of sinks before g_lo
  int g_lo;
  int groups;       // of both
};
__host__ __device__ inline SpanRange span_range(int t, int first, int last, int window, int sinks) {
  SpanRange r;
  r.lo = window > 0 && t + first - window + 1 > 0 ? t + first - window + 1 : 0;
  const int reach = sinks < r.lo ? sinks : r.lo;
  r.g_lo = r.lo >> 5;
  const int g = (int)(((uint32_t)reach + 31u) >> 5);
  r.sink_groups = g < r.g_lo ? g : r.g_lo;
  r.groups = r.sink_groups + ((t + last) >> 5) - r.g_lo + 1;
  return r;
}
__host__ __device__ inline int span_group(const SpanRange& r, int i) { return i < r.sink_groups ? i : i - r.sink_groups + r.g_lo; }

// Rows of the columns of tile `tile`, of a sequence with `rows` rows: the range of its keys.
__host__ __device__ inline SpanRange tile_range(int t, int tile, int tile_columns, int G, int rows, int window, int sinks, bool tree) {
  const int first = (int)((int64_t)tile * tile_columns / G), past = (int)(((int64_t)(tile + 1) * tile_columns - 1) / G);
  return span_range(t, tree ? 0 : first, past < rows - 1 ? past : rows - 1, window, sinks);
}

// What workgroup (x, y, z) takes of a launch for many columns, whose grid is (kv heads * blocks of columns, sequences, splits).  The
// blocks of one (sequence, kv head, split) read the same keys, so they run on one die.  Few blocks: units of work lie on the dies in
// turn (units_work()).  The many of a prompt, whose neighbours read nearly the same windows: each die gets a contiguous run of the
// list of blocks, a unit's last block first, and at its end, so that the die's workgroups end together, one of the list of the units' first
// `fewer` blocks, whose windows begin before step 0: those of an eighth of the units at a time, from the longest on.  (us, unit by unit / so: 4 x 4096
// steps of 24/8 heads of 128, window 1024 249 / 246, 512 176 / 173, 8 bits 275 / 267; 32/8 heads of 64, window 4000 335 / 323; 6000 steps 145 / 145.5.)
constexpr uint32_t kRunBlocks = 8;
__host__ __device__ inline UnitsWork wide_work(uint32_t x, uint32_t y, uint32_t z, uint32_t nx, uint32_t ny, uint32_t nz, int Hkv, uint32_t fewer) {
  const uint32_t blocks = nx / (uint32_t)Hkv;
  if (blocks <= kRunBlocks) return units_work(x, y, z, nx, ny, nz, Hkv);
  const uint32_t total = nx * ny * nz, linear = x + nx * (y + ny * z), die = linear & 7u, at = linear >> 3, units = total / blocks;
  const uint32_t full = blocks - fewer, first = units * full, share = first >> 3, extra = first & 7u;
  const uint32_t begin = die * share + (die < extra ? die : extra), mine = share + (die < extra ? 1 : 0);
  uint32_t unit, block;
  if (at < mine) {
    const uint32_t item = begin + at;
    unit = item / full;
    block = blocks - 1 - (item - unit * full);
  } else {
    const uint32_t item = die * (total >> 3) + (die < (total & 7u) ? die : total & 7u) - begin + at - mine;
    const uint32_t together = (units + 7) >> 3, set = item / (together * fewer), left = units - set * together, width = left < together ? left : together;
    const uint32_t in = item - set * together * fewer, row = in / width;
    unit = set * together + in - row * width;
    block = fewer - 1 - row;
  }
  const uint32_t row = unit / nz;
  return {(int)(row % (uint32_t)Hkv), (int)block, (int)(row / (uint32_t)Hkv), (int)(unit - row * nz)};
}
// Blocks of columns whose first row is nearer to step 0 than its window is long.
__host__ __device__ inline uint32_t fewer_keys(int t, int window, int G, int tile_columns, uint32_t blocks) {
  if (window <= 0 || t >= window) return 0;
  const int64_t n = ((int64_t)(window - t) * G + tile_columns - 1) / tile_columns;
  return n < (int64_t)blocks ? (uint32_t)n : blocks;
}

// Rows at positions of their own.
struct PlaceParams : StoreParams {
  const int32_t* positions;   // [batch][count][axes]
  const void* q;              // [batch][count][Hq][D]; may be null
  void* q_out;
  int32_t Hq;                 // of q; 0: no q
  int32_t Hrows;              // of k_raw and v_new: Hkv, or 0 where only q is turned
  int32_t axes;
  int32_t table_rows;         // positions of the tables
  uint64_t axis_bits[2];      // two bits for each of the 64 (D = 64: 32) pairs: its axis
};

constexpr int kKeepLayers = 64;  // of one launch
constexpr int kKeepRows = 128;   // of a sequence

struct KeepParams {
  void* k_pool[kKeepLayers];
  void* v_pool[kKeepLayers];
  const int32_t* block_table;
  const int32_t* t_per_seq;    // may be null
  const int32_t* kept;         // [batch][count]
  int32_t t;
  int32_t z_log2;
  int32_t max_blocks_per_seq;
  int32_t tile_mask;
  int32_t num_blocks;
  int32_t Hkv;
  int32_t nodes;
  int32_t count;
};

// Weak: the host side can be built without the kernels (its tests record the launches).
#define TEMPO_LAUNCHER __attribute__((weak)) hipError_t
TEMPO_LAUNCHER launch_spans(const SpanParams& p, int batch, int D, int dtype, int waves, hipStream_t stream);
TEMPO_LAUNCHER launch_spans_wide(const SpanParams& p, int batch, int D, int dtype, hipStream_t stream);
TEMPO_LAUNCHER launch_spans_f32(const SpanParams& p, int batch, int D, int waves, hipStream_t stream);
TEMPO_LAUNCHER launch_combine_spans(const SpanParams& p, int batch, int D, int dtype, hipStream_t stream);
TEMPO_LAUNCHER launch_place(const PlaceParams& p, const void* k_raw, const void* v_new, int D, int dtype, hipStream_t stream);
TEMPO_LAUNCHER launch_tree_positions(const int32_t* parents, int32_t* positions, int batch, int nodes, int t, const int32_t* t_per_seq, hipStream_t stream);
TEMPO_LAUNCHER launch_keep(const KeepParams& p, int batch, int layers, int D, int dtype, hipStream_t stream);
#undef TEMPO_LAUNCHER

}  // namespace tempo
