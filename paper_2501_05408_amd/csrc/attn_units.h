// What the launches of attn_units.hip and select_blocks.hip take, on top of tempo_internal.h.
#pragma once

#include "tempo_internal.h"

namespace tempo {

// Attention over a list of blocks: t and t_per_seq are the step's, window and count are not used, one query step.
struct SelectParams : AttnParams {
  const int32_t* selected;  // [B][Hkv][pick] block numbers
  int32_t pick;
};

// What workgroup (x, y, z) takes of a launch of attn_units, whose grid is (kv heads * tiles of columns, sequences, splits).
// Workgroups go to the part's 8 dies, each with its own L2, round-robin by linear index.  The tiles of one (sequence, kv head,
// split) read the same keys, so they are given indexes 8 apart: a run of 8 such units of work is followed by the same units'
// next tiles, all tiles of a unit on one die, whatever the number of heads, and all but the first read from its L2.  The last
// run may be of fewer units, with tiles on neighbouring dies.  (us, tiles a whole row of heads apart / 8 apart: 16 sequences of
// 4000 keys, 32/4 heads of 128, 8 steps 30.4 / 24.2; 64 sequences, 32/1 heads, 4 steps 50.7 / 30.8; lists of 64 blocks of 64 bf16
// keys, 32 sequences, 128/1 heads 119 / 63; 8 heads, where both are the same, 33.1 / 33.3.)
// Indexes are below 2^32: every unit's partials or answers lie in memory.
struct UnitsWork {
  int hkv, tile, b, split;
};
__host__ __device__ inline UnitsWork units_work(uint32_t x, uint32_t y, uint32_t z, uint32_t nx, uint32_t ny, uint32_t nz, int Hkv) {
  if (nx == (uint32_t)Hkv) return {(int)x, 0, (int)y, (int)z};
  const uint32_t tiles = nx / (uint32_t)Hkv, units = (uint32_t)Hkv * ny * nz, linear = x + nx * (y + ny * z);
  const uint32_t run = linear / (8 * tiles), at = linear - run * 8 * tiles, left = units - 8 * run, width = left < 8 ? left : 8;
  const uint32_t tile = at / width, unit = 8 * run + at - tile * width, row = unit / (uint32_t)Hkv;
  return {(int)(unit - row * (uint32_t)Hkv), (int)tile, (int)(row % ny), (int)(row / ny)};
}

// Dynamic LDS of a launch of attn_units: the merge of its wavefronts, and the codes and scale bytes of a new row.
inline size_t units_lds_bytes(int waves, int columns, int D) {
  return (size_t)waves * (32 + (size_t)(columns < 16 ? columns : 16) * D) * sizeof(float) + 2 * (size_t)D + 16;
}

// The bf16 store that an 8-bit store's groups are turned into for a prompt.
struct UnpackParams {
  void* k;                    // [batch * tiles][Hkv][Z * D] bf16
  void* v;
  int32_t* table;             // [batch][tiles]
  int32_t tiles;
  int32_t tile_mask;          // tile n lies in place n & tile_mask
  int32_t first_group;        // of the sequence
};

// Score and choice of blocks.
struct ChooseParams {
  void* bounds;               // [num_blocks][Hkv][2][D] bf16
  const void* q;              // [B][Hq][D] bf16
  const int32_t* block_table;
  const int32_t* t_per_seq;   // may be null
  uint64_t* scores;           // [B][Hkv][tiles]: intervals of the scores, or their order-preserving bits
  int32_t* selected;          // [B][Hkv][pick]
  int32_t t;
  int32_t z_log2;
  int32_t max_blocks_per_seq;
  int32_t num_blocks;
  int32_t Hkv, Hq, G;
  int32_t tiles;              // t / Z + 1
  int32_t pick, first, last;
};

// Weak: the host side can be built without the kernels (its tests record the launches).
#define TEMPO_LAUNCHER __attribute__((weak)) hipError_t
TEMPO_LAUNCHER launch_append_e4m3(const StoreParams& p, const void* k_new, const void* v_new, int D, hipStream_t stream);
TEMPO_LAUNCHER launch_gather_e4m3(const StoreParams& p, void* k_out, void* v_out, int D, int j0, int count, hipStream_t stream);
TEMPO_LAUNCHER launch_append_copy_e4m3(const StoreParams& p, const UnpackParams& u, const void* k_new, const void* v_new, int D, hipStream_t stream);
TEMPO_LAUNCHER launch_unpack_e4m3(const StoreParams& p, const UnpackParams& u, int groups, int D, hipStream_t stream);
TEMPO_LAUNCHER launch_partial_e4m3(const AttnParams& p, int batch, int D, int grid_splits, int waves, hipStream_t stream);
TEMPO_LAUNCHER launch_partial_selected(const SelectParams& p, int batch, int D, int dtype, int grid_splits, int waves, hipStream_t stream);
TEMPO_LAUNCHER launch_combine_selected(const AttnParams& p, int batch, int D, hipStream_t stream);
TEMPO_LAUNCHER launch_block_bounds(const StoreParams& p, void* bounds, int D, int dtype, hipStream_t stream);
TEMPO_LAUNCHER launch_select_blocks(const ChooseParams& p, const StoreParams* store, const void* k_new, const void* v_new, int batch, int D,
                                    int dtype, hipStream_t stream);
#undef TEMPO_LAUNCHER

}  // namespace tempo
