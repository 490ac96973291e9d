// Entry points of drafted trees, windows with sinks, rows at positions of their own and kept rows; the end of tempo_api.hip, whose
// checks they use.
#pragma once

#include "attn_spans.h"

namespace {

// A call of the attention over spans: how its (row, head) columns and its keys are cut.
struct SpanPlan {
  int32_t tile_columns, tiles, split_groups, splits, waves;
};

// Attention over spans is of linear stores.  A launch of so many rows fits whatever the plan: less than 2^31 threads along the grid's first
// axis (tiles of 128 columns and 256 threads, which span_plan() takes where narrower ones would not fit; fp32: 16 columns, 256
// threads at least) and workgroups, which are numbered in 32 bits.
int check_span_store(const tempo_kv* kv, int32_t batch, int32_t Hq, int32_t rows) {
  int rc = check_layout(kv);
  if (rc != TEMPO_OK) return rc;
  if (kv->ring_blocks != 0) return TEMPO_ERR_SHAPE;
  if ((rc = check_heads(kv, batch, Hq)) != TEMPO_OK) return rc;
  if (rows < 1 || rows > (1 << 24) || (int64_t)rows * Hq > (kv->dtype == TEMPO_F32 ? 1 << 26 : 1 << 29)) return TEMPO_ERR_SHAPE;
  const int64_t columns = (int64_t)rows * (Hq / kv->num_kv_heads);
  if ((int64_t)batch * kv->num_kv_heads * ((columns + 15) / 16) > INT32_MAX) return TEMPO_ERR_SHAPE;
  return TEMPO_OK;
}

// Steps t .. t + rows - 1 (of a tree the slots of its nodes), the window (0: none, and no sinks then) and the sinks.
int check_span(const tempo_kv* kv, int32_t t, int32_t rows, int32_t window, int32_t sinks) {
  if (t < 0 || window < 0 || sinks < 0 || t > INT32_MAX - 128 - rows) return TEMPO_ERR_RANGE;
  if (window == 0 && sinks > 0) return TEMPO_ERR_RANGE;
  return check_step(kv, t + rows - 1);
}

// Most 32-key groups that a tile of columns sees, whatever its steps up to t + rows - 1.
int32_t span_groups_bound(int32_t t, int32_t rows, int32_t tile_rows, int32_t window, int32_t sinks) {
  const int64_t all = ((int64_t)t + rows - 1) / 32 + 1;
  if (window == 0) return (int32_t)all;
  const int64_t keys = (int64_t)window + tile_rows - 1;  // a run of so many keys touches ...
  const int64_t some = (keys + 30) / 32 + 1 + ((int64_t)sinks + 31) / 32;
  return (int32_t)(some < all ? some : all);
}

constexpr int64_t kSpanPartials = 131072;  // partials (of a (row, head) and split) of a call at most, if its rows are fewer

// Groups of a split of the kernel for many columns: a time model as make_plan()'s, in nanoseconds.  A workgroup of 128 columns costs
// kWideFixedNs before its first group and behind its last one, hidden behind others only in part; a group, with two or three
// workgroups to a unit (what registers and LDS let in; 8-bit trees of more than 206 nodes at D = 128, one, are not told apart), 560 ns of
// the unit's time at D = 128 and 420 at 64, with one 720 and 540.  The combine reads and writes a partial per (row, head) and split.  Of a
// ragged batch's workgroups about half exist.  (Against lengths of a quarter to four times, over 56675 drawn calls of all tiles: 1.1%.)
constexpr double kWideFixedNs = 8000.0, kWideCombineNs = 4000.0, kWidePartialBytesPerNs = 5000.0;

int32_t wide_split_groups(int64_t units, int32_t groups, int D, int64_t rows, bool ragged, int64_t most) {
  const int64_t resident = D == 128 ? 2 : 3;
  const double alone = D == 128 ? 720.0 : 540.0, shared = D == 128 ? 560.0 : 420.0;
  int32_t best = groups;
  double least = -1.0;
  for (int64_t splits = 1; splits <= most && splits <= 64 && splits <= (groups + 3) / 4; ++splits) {
    const int32_t each = (int32_t)((groups + splits - 1) / splits);
    const int64_t there = (groups + each - 1) / each;  // splits of so many groups
    const int64_t workgroups = ragged ? (units * there * 11 + 19) / 20 : units * there;
    const int64_t whole = (workgroups + kComputeUnits - 1) / kComputeUnits, rounds = (whole + resident - 1) / resident;
    const double at = whole <= 4 ? (double)whole : (double)workgroups / kComputeUnits;  // (many even out)
    const double group = at * shared > (double)rounds * alone ? at * shared : (double)rounds * alone;
    double cost = (double)rounds * kWideFixedNs + each * group;
    if (there > 1) cost += kWideCombineNs + 2.0 * (double)(rows * there) * D * 4 / kWidePartialBytesPerNs * (ragged ? 0.55 : 1.0);
    if (least < 0.0 || cost < least * 0.99) {
      least = cost;
      best = each;
    }
  }
  return best;
}

// Groups up to which a workgroup of up to 32 columns takes all of them, eight wavefronts: a combine costs about 3 us (us, one split of
// eight wavefronts / the best of 2 to 8 splits: bf16, 24/8 heads of 128, one sequence, 10 groups 6.8 / 10.2, 19 groups 7.7 / 10.4, 34 groups
// 11.4 / 9.7; 32/8 heads of 64, 34 groups 8.0 / 9.2, 65 groups 13.0 / 9.7; 8 bits, heads of 128, 32 groups 9.4 / 9.7).
int32_t whole_groups(const tempo_kv* kv) {
  return kv->dtype == TEMPO_E4M3 ? (kv->head_dim == 64 ? 48 : 32) : (kv->head_dim == 64 ? 40 : 24);
}

// Columns of a workgroup: 16 or 32 in the registers of each wavefront, which share the keys out (attn_spans.hip), or 128, 32 to a
// wavefront, over keys in LDS (attn_spans_wide.hip).  Estimates in us: a launch's fixed part; a workgroup's group, of 256 at work
// (for 128 columns by its wavefronts that have some); the combine, where fewer workgroups than units call for splits.  A key is
// fetched from HBM once whatever the tiles.  Fitted to 9 counts of columns of 6 to 190 at 40 shapes of 1 to 48 sequences; us with
// 16 / 32 / 128: 24/8 heads of 128, bf16, 1 sequence of 1000 keys, 63 columns 11.5 / 13.0 / 13.8; 8 of 1000, 96 columns 21 / 17 / 22;
// 16 of 4000, 96 columns 127 / 92 / 67; 32/8 heads of 64, 8 bits, 48 of 1000, 60 columns 27 / 22 / 31; 188 columns 66 / 53 / 46.
// Of a batch whose sequences have steps, or trees, of their own, about half of the longest are taken to be there, though a range
// that is not split takes as long as the longest (16 trees of up to 32 nodes behind up to 4000 keys, 24/8 heads of 128, 8 bits,
// 16 / 32 / 128: 35 / 30 / 44; bf16 61 / 44 / 36).  A group of 8 bits under 32 columns at D = 128 takes a fifth longer where a unit has more
// than one workgroup (its codes are turned by every wavefront, beside the other's): of 8376 drawn calls of that kind this decides 761, which
// are 14% (128 columns taken) and 7% (16) faster for it.  Against the best of the three, over 56675 drawn calls: 1.6% on the mean.
double span_cost_us(const tempo_kv* kv, int64_t pairs, int64_t columns, int64_t rows_heads, int32_t tile, int32_t groups, bool ragged, bool counts) {
  const bool k8 = kv->dtype == TEMPO_E4M3, narrow = kv->head_dim == 64;
  const int at = (k8 ? 2 : 0) + (narrow ? 1 : 0);
  static const double c16[] = {0.36, 0.15, 0.20, 0.105}, c32[] = {0.40, 0.17, 0.25, 0.155}, c128[] = {0.45, 0.20, 0.40, 0.20};
  static const double wave[] = {0.08, 0.04, 0.10, 0.06}, hbm[] = {0.6, 0.3, 0.3, 0.15};
  const double all = (double)((columns + tile - 1) / tile), tiles = counts ? 0.55 * all + 0.25 : all;
  const double there = counts ? 0.55 * (double)columns : (double)columns, mean = ragged ? 0.55 * groups : groups;
  const double workgroups = (double)pairs * tiles, units = kComputeUnits;
  const bool split = workgroups < 192 && groups > (tile == 128 ? 12 : whole_groups(kv));
  double work = workgroups * mean / units;                 // groups one after another on a unit
  if (!split && work < groups) work = groups;
  double each = tile == 16 ? c16[at] : tile == 32 ? c32[at] : c128[at] + wave[at] * there / 32.0 / tiles;
  if (tile == 32 && at == 2 && workgroups > units && !ragged) each *= 1.2;
  const double stream = hbm[at] * (double)pairs * mean / units;
  double cost = (tile == 16 ? 5.0 : tile == 32 ? 7.0 : 9.0) + (each * work > stream ? each * work : stream);
  if (split) {
    const double splits = 512.0 / workgroups < groups / 8.0 ? 512.0 / workgroups : groups / 8.0;
    cost += 5.0 + (double)rows_heads * (counts ? 0.55 : 1.0) * splits * kv->head_dim * 4 / (kWidePartialBytesPerNs * 1000.0);
  }
  return cost;
}

// Wavefronts that share few groups, if four to a workgroup would not fit the part at once: more workgroups side by side hide each other's
// beginnings and ends better (us with 4 / 2 / 1: 3648 of 3 groups, 32 columns, 8 bits, D = 128 65 / 49 / 41; 720 of 4, bf16 28 / 20 / 23; 2048 of 3,
// 16 columns, 8 bits 19.5 / 16.2 / 13.5; D = 64, 1944 of 10, 16 columns, 8 bits 33.5 / 24.6 / 25.7; 1008 of 4, bf16 16.1 / 13.6 / 15.6;
// ragged 768 of 9, 32 columns, D = 128 19.0 / 22.5 / 30.4; steps, D = 128: 1024 of 5, 8 bits 23.8 / 20.8 / 20.0, 2048 of 3, bf16 30.8 / 29.0 / 28.6,
// of 11 65 / 69 / 68, so that such, whose tiles share no keys, are taken up to 8 too).
int32_t few_waves(int64_t workgroups, int32_t tiles, int32_t groups, int D, int32_t tile, bool ragged) {
  const int64_t room = kComputeUnits * (D == 128 ? (tile == 16 ? 12 : 8) : (tile == 16 ? 14 : 12));  // (D = 64, 16 columns: registers let in 16)
  if (groups < 3 || groups > (ragged || tiles == 1 ? 8 : 12) || 4 * workgroups <= room) return 8;
  return !ragged && groups <= 6 && 2 * workgroups > room ? 1 : 2;
}

// Up to 32 columns a split is planned as a step's or block's of as many keys (make_plan()): the kernel streams keys as theirs do.
// (Ragged steps, which make_plan() gives short splits, only where there are fewer workgroups than units: 40 trees of up to 20 nodes
// behind up to 2000 keys, 32/4 heads of 128, 8 bits, one split 35 us, two 50.)
SpanPlan span_plan(const tempo_kv* kv, int32_t batch, int32_t Hq, int32_t rows, int32_t t, bool ragged, bool counts, int32_t window, int32_t sinks,
                   bool tree) {
  SpanPlan s;
  const int32_t G = Hq / kv->num_kv_heads;
  const int64_t columns = (int64_t)rows * G, all = (int64_t)batch * rows * Hq;
  int32_t groups = 0;
  double least = -1.0;
  for (int32_t tile = 16; tile <= 128; tile = tile == 16 ? 32 : 4 * tile) {
    if (tile < 128 && kv->dtype != TEMPO_F32 && (columns + tile - 1) / tile * kv->num_kv_heads * 512 > INT32_MAX) continue;
    int32_t tile_rows = (tile + G - 2) / G + 1;
    tile_rows = tree || tile_rows > rows ? rows : tile_rows;
    const int32_t here = span_groups_bound(t, rows, tile_rows, window, sinks);
    const double cost = span_cost_us(kv, (int64_t)batch * kv->num_kv_heads, columns, all, tile, here, ragged && window == 0, counts);
    if (least < 0.0 || cost < least) {
      least = cost;
      groups = here;
      s.tile_columns = tile;
    }
    if (columns <= tile || kv->dtype == TEMPO_F32) break;  // a wider one holds no more; fp32: 16
  }
  s.tiles = (int32_t)((columns + s.tile_columns - 1) / s.tile_columns);
  // As many wavefronts with columns in every tile (us: 8 trees of 18 nodes behind 6007 keys, 32/4 heads, 144 columns as 2 x 96 34.8, as
  // 128 + 16 37.3; 4 trees of 64 nodes behind 4000 keys, 24/8 heads 25.2 and 26.9).
  if (s.tile_columns > 32) s.tile_columns = (int32_t)((columns + s.tiles - 1) / s.tiles + 31) / 32 * 32;
  const int64_t most = all < kSpanPartials ? kSpanPartials / all : 1;  // splits that the workspace has room for
  if (s.tile_columns <= 32) {
    const int64_t keys = 32 * (int64_t)groups;  // a multiple of the unit of splits, so that windows have no worst alignment
    // tiles of columns are workgroups of their own, as sequences are
    const bool f32 = kv->dtype == TEMPO_F32;  // (whose tiles make_plan() counts itself)
    const int64_t like = f32 ? batch : (int64_t)batch * s.tiles;
    const int32_t queries = f32 ? rows : s.tile_columns / G < 1 ? 1 : s.tile_columns / G < rows ? s.tile_columns / G : rows;
    tempo_plan plan;
    make_plan(kv, like < 65535 ? (int32_t)like : 65535, Hq, (int32_t)(keys - 1 < INT32_MAX - 64 ? keys - 1 : INT32_MAX - 64), 0,
              ragged && window == 0 && like * kv->num_kv_heads < kComputeUnits, queries, most < kMaxSplits ? most : kMaxSplits, &plan);
    s.split_groups = plan.tokens_per_split / 32;
    s.waves = plan.waves;
    if (!f32 && groups <= whole_groups(kv) && like * kv->num_kv_heads <= kComputeUnits) {
      s.split_groups = groups;
      s.waves = groups > 4 ? 8 : groups > 2 ? 4 : groups;
    }
  } else {
    s.split_groups = wide_split_groups((int64_t)batch * kv->num_kv_heads * s.tiles, groups, kv->head_dim, all, ragged && window == 0, most);
    s.waves = 4;
  }
  while ((groups + s.split_groups - 1) / s.split_groups > most) s.split_groups *= 2;
  s.splits = (groups + s.split_groups - 1) / s.split_groups;
  if (s.tile_columns <= 32 && s.splits == 1 && kv->dtype != TEMPO_F32) {
    const int64_t waves = few_waves((int64_t)batch * kv->num_kv_heads * s.tiles, s.tiles, groups, kv->head_dim, s.tile_columns, ragged || counts);
    s.waves = s.waves < waves ? s.waves : (int32_t)waves;
  }
  while (s.waves > 4 && s.tile_columns <= 32 && (int64_t)kv->num_kv_heads * s.tiles * 64 * s.waves > INT32_MAX) s.waves /= 2;
  while (s.tile_columns <= 32 && s.waves > 1 && units_lds_bytes(s.waves, (int)(columns < 16 ? columns : 16), kv->head_dim) > kMaxUnitsLds) s.waves /= 2;
  return s;
}

size_t span_bytes(const tempo_kv* kv, int32_t batch, int32_t Hq, int32_t rows, const SpanPlan& s) {
  return s.splits == 1 ? 256 : plan_bytes(kv, (int64_t)batch * rows * Hq, s.splits);
}

// Of any call with at most `rows` rows a sequence whose tiles of columns see at most `groups` groups.
size_t span_bytes_bound(const tempo_kv* kv, int32_t batch, int32_t Hq, int32_t rows, int32_t groups) {
  const int64_t all = (int64_t)batch * rows * Hq;
  const int64_t partials = all > kSpanPartials / groups ? kSpanPartials : all * groups;
  return plan_bytes(kv, partials, 1);
}

// Everything but the arguments that only one of the entry points has has been checked.
int attend_spans(const tempo_kv* kv, const void* q, void* out, const int32_t* parents, const int32_t* rows_per_seq, int32_t batch, int32_t Hq,
                 int32_t rows, int32_t t, const int32_t* t_per_seq, int32_t window, int32_t sinks, float scale, const SpanPlan& s, void* workspace,
                 hipStream_t stream, const tempo_rope* rope = nullptr, const void* k_new = nullptr, const void* v_new = nullptr) {
  tempo_plan plan = {32, s.splits, s.waves};
  SpanParams p;
  static_cast<AttnParams&>(p) = attn_params(kv, q, out, Hq, t, t_per_seq, window, scale, &plan, workspace, batch, rows);
  p.direct = s.splits == 1;
  p.count_per_seq = rows_per_seq;
  p.parents = parents;
  p.k_new = k_new;
  p.v_new = v_new;
  p.sinks = sinks;
  p.tile_columns = s.tile_columns;
  p.split_groups = s.split_groups;
  if (rope) {
    p.rope_cos = rope->cos;
    p.rope_sin = rope->sin;
  }
  const int rc = launch_status(kv->dtype == TEMPO_F32 ? launch_spans_f32(p, batch, kv->head_dim, s.waves, stream)
                               : s.tile_columns > 32 ? launch_spans_wide(p, batch, kv->head_dim, kv->dtype, stream)
                                                     : launch_spans(p, batch, kv->head_dim, kv->dtype, s.waves, stream),
                               "attn_spans");
  if (rc != TEMPO_OK || p.direct) return rc;
  return launch_status(launch_combine_spans(p, batch, kv->head_dim, kv->dtype, stream), "attn_spans_combine");
}

int check_span_workspace(const tempo_kv* kv, int32_t batch, int32_t Hq, int32_t rows, int32_t t, bool ragged, bool counts, int32_t window,
                         int32_t sinks, bool tree, const void* workspace, size_t workspace_bytes, SpanPlan* plan) {
  const SpanPlan s = *plan = span_plan(kv, batch, Hq, rows, t, ragged, counts, window, sinks, tree);
  const int64_t first = (int64_t)kv->num_kv_heads * s.tiles;  // workgroups along the grid's first axis
  if (first * (s.tile_columns > 32 ? 256 : 64 * s.waves) > INT32_MAX || first * batch * s.splits > INT32_MAX || s.splits > 65535) return TEMPO_ERR_SHAPE;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return TEMPO_ERR_WORKSPACE;
  return workspace_bytes < span_bytes(kv, batch, Hq, rows, s) ? TEMPO_ERR_WORKSPACE : TEMPO_OK;
}

// Positions of a call's rows: tables, axes.
int check_axes(const tempo_rope* rope, const tempo_rope_axes* axes, int32_t head_dim) {
  const int rc = check_rope(rope, head_dim, 0);
  if (rc != TEMPO_OK || !axes) return rc;
  if (axes->axes < 1 || axes->axes > 4) return TEMPO_ERR_SHAPE;
  for (int i = 0; i < head_dim / 2; ++i) {
    if (axes->axis_of_pair[i] >= axes->axes) return TEMPO_ERR_RANGE;
  }
  return TEMPO_OK;
}

PlaceParams place_params(const StoreParams& store, const tempo_rope* rope, const tempo_rope_axes* axes, const int32_t* positions) {
  PlaceParams p;
  static_cast<StoreParams&>(p) = store;
  p.rope_cos = rope->cos;
  p.rope_sin = rope->sin;
  p.positions = positions;
  p.q = nullptr;
  p.q_out = nullptr;
  p.Hq = p.Hrows = 0;
  p.axes = axes ? axes->axes : 1;
  p.table_rows = rope->positions;
  p.axis_bits[0] = p.axis_bits[1] = 0;
  for (int i = 0; axes && i < rope->head_dim / 2; ++i) p.axis_bits[i >> 5] |= (uint64_t)(axes->axis_of_pair[i] & 3u) << (2 * (i & 31));
  return p;
}

}  // namespace

extern "C" {

int tempo_sink_blocks(int32_t window, int32_t sinks, int32_t Z, int32_t queries, int32_t* sink_blocks, int32_t* window_blocks) {
  if (!sink_blocks || !window_blocks) return TEMPO_ERR_NULL;
  if (window < 1 || sinks < 0 || Z < 1 || queries < 1) return TEMPO_ERR_RANGE;
  const int64_t keys = (int64_t)window + queries - 1, turn = (keys + Z - 2) / Z + 1;
  if (turn > INT32_MAX) return TEMPO_ERR_RANGE;
  *sink_blocks = (int32_t)(((int64_t)sinks + Z - 1) / Z);
  *window_blocks = (int32_t)turn;
  return TEMPO_OK;
}

size_t tempo_attn_sinks_workspace_bytes(const tempo_kv* kv, int32_t batch, int32_t num_q_heads, int32_t queries, int32_t max_t,
                                        int32_t window, int32_t sinks) {
  if (check_span_store(kv, batch, num_q_heads, queries) != TEMPO_OK) return 0;
  if (window < 1 || sinks < 0 || max_t < 0 || max_t > INT32_MAX - 128 - queries) return 0;
  return span_bytes_bound(kv, batch, num_q_heads, queries, span_groups_bound(max_t, queries, queries, window, sinks));
}

size_t tempo_attn_tree_workspace_bytes(const tempo_kv* kv, int32_t batch, int32_t num_q_heads, int32_t nodes, int32_t max_t,
                                       int32_t window, int32_t sinks) {
  if (check_span_store(kv, batch, num_q_heads, nodes) != TEMPO_OK || nodes > kMaxNodes) return 0;
  if (window < 0 || sinks < 0 || max_t < 0 || max_t > INT32_MAX - 128 - nodes) return 0;
  return span_bytes_bound(kv, batch, num_q_heads, nodes, span_groups_bound(max_t, nodes, nodes, window, sinks));
}

size_t tempo_prefill_sinks_workspace_bytes(const tempo_kv* kv, int32_t batch, int32_t num_q_heads, int32_t max_t) {
  if (check_span_store(kv, batch, num_q_heads, 1) != TEMPO_OK) return 0;
  if (max_t < 0 || max_t > INT32_MAX - 128) return 0;
  const int32_t rows = max_t < (1 << 24) ? max_t + 1 : 1 << 24;
  return span_bytes_bound(kv, batch, num_q_heads, rows, max_t / 32 + 1);
}

int tempo_attn_tree(const tempo_kv* kv, const void* q, void* out, const int32_t* parents, const int32_t* nodes_per_seq, int32_t batch,
                    int32_t num_q_heads, int32_t nodes, int32_t t, const int32_t* t_per_seq, int32_t window, int32_t sinks, float scale,
                    void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_span_store(kv, batch, num_q_heads, nodes);
  if (rc != TEMPO_OK) return rc;
  if (!q || !out || !parents || (rc = check_store(kv)) != TEMPO_OK) return TEMPO_ERR_NULL;
  if (nodes > kMaxNodes) return TEMPO_ERR_SHAPE;
  if ((rc = check_span(kv, t, nodes, window, sinks)) != TEMPO_OK) return rc;
  if ((rc = check_scale(scale)) != TEMPO_OK) return rc;
  SpanPlan plan;
  if ((rc = check_span_workspace(kv, batch, num_q_heads, nodes, t, t_per_seq != nullptr, nodes_per_seq != nullptr, window, sinks, true, workspace, workspace_bytes, &plan)) != TEMPO_OK) return rc;
  return attend_spans(kv, q, out, parents, nodes_per_seq, batch, num_q_heads, nodes, t, t_per_seq, window, sinks, scale, plan, workspace,
                      static_cast<hipStream_t>(stream));
}

// A call of consecutive steps; k_new set: their rows are written first.  prompt: count_per_seq and many rows.
static int sinks_call(const tempo_kv* kv, const tempo_rope* rope, const void* q, const void* k_new, const void* v_new, void* out, int32_t batch,
                      int32_t Hq, int32_t rows, int32_t t, const int32_t* t_per_seq, const int32_t* count_per_seq, int32_t window, int32_t sinks,
                      float scale, void* workspace, size_t workspace_bytes, void* stream, bool write) {
  int rc = check_span_store(kv, batch, Hq, rows);
  if (rc != TEMPO_OK) return rc;
  if (!q || !out || (write && (!k_new || !v_new)) || (rc = check_store(kv)) != TEMPO_OK) return TEMPO_ERR_NULL;
  if (window < 1) return TEMPO_ERR_RANGE;
  if ((rc = check_span(kv, t, rows, window, sinks)) != TEMPO_OK) return rc;
  if ((rc = check_scale(scale)) != TEMPO_OK) return rc;
  if (rope && (rc = check_rope(rope, kv->head_dim, t + rows - 1)) != TEMPO_OK) return rc;
  if (rope && kv->dtype == TEMPO_F32 && (rows > 1 || count_per_seq)) return TEMPO_ERR_DTYPE;  // rows of several steps are not turned on their way in
  if (write && (int64_t)batch * rows * kv->num_kv_heads * kv->head_dim > INT32_MAX) return TEMPO_ERR_SHAPE;
  SpanPlan plan;
  if ((rc = check_span_workspace(kv, batch, Hq, rows, t, t_per_seq != nullptr, count_per_seq != nullptr, window, sinks, false, workspace, workspace_bytes, &plan)) != TEMPO_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f32 = kv->dtype == TEMPO_F32, fused = write && !f32 && rows == 1 && Hq / kv->num_kv_heads <= 32;  // the attention of a step writes its row itself
  if (write && f32 && rope) {
    const StoreParams p = store_params(kv, batch, t, t_per_seq);
    if ((rc = launch_status(launch_rope_append(p, rope->cos, rope->sin, k_new, v_new, kv->head_dim, kv->dtype, s), "kv_append")) != TEMPO_OK) return rc;
  } else if (write && !fused) {
    StoreParams p = store_params(kv, batch, t, t_per_seq, rows);
    p.count_per_seq = count_per_seq;
    if (rope) {
      p.rope_cos = rope->cos;
      p.rope_sin = rope->sin;
    }
    if ((rc = launch_status(launch_append(p, k_new, v_new, kv->head_dim, kv->dtype, s), "kv_append")) != TEMPO_OK) return rc;
  }
  return attend_spans(kv, q, out, nullptr, count_per_seq, batch, Hq, rows, t, t_per_seq, window, sinks, scale, plan, workspace, s, rope,
                      fused ? k_new : nullptr, fused ? v_new : nullptr);
}

int tempo_attn_sinks(const tempo_kv* kv, const void* q, void* out, int32_t batch, int32_t num_q_heads, int32_t queries, int32_t t,
                     const int32_t* t_per_seq, int32_t window, int32_t sinks, float scale, void* workspace, size_t workspace_bytes,
                     void* stream) {
  return sinks_call(kv, nullptr, q, nullptr, nullptr, out, batch, num_q_heads, queries, t, t_per_seq, nullptr, window, sinks, scale, workspace,
                    workspace_bytes, stream, false);
}

int tempo_decode_step_sinks(const tempo_kv* kv, const void* q, const void* k_new, const void* v_new, void* out, int32_t batch,
                            int32_t num_q_heads, int32_t t, const int32_t* t_per_seq, int32_t window, int32_t sinks, float scale,
                            void* workspace, size_t workspace_bytes, void* stream) {
  return sinks_call(kv, nullptr, q, k_new, v_new, out, batch, num_q_heads, 1, t, t_per_seq, nullptr, window, sinks, scale, workspace,
                    workspace_bytes, stream, true);
}

int tempo_rope_decode_step_sinks(const tempo_kv* kv, const tempo_rope* rope, const void* q_raw, const void* k_raw, const void* v_new, void* out,
                                 int32_t batch, int32_t num_q_heads, int32_t t, const int32_t* t_per_seq, int32_t window, int32_t sinks,
                                 float scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (!rope) return TEMPO_ERR_NULL;
  return sinks_call(kv, rope, q_raw, k_raw, v_new, out, batch, num_q_heads, 1, t, t_per_seq, nullptr, window, sinks, scale, workspace,
                    workspace_bytes, stream, true);
}

int tempo_prefill_sinks(const tempo_kv* kv, const void* q, const void* k_new, const void* v_new, void* out, int32_t batch, int32_t num_q_heads,
                        int32_t t, int32_t count, const int32_t* count_per_seq, int32_t window, int32_t sinks, float scale, void* workspace,
                        size_t workspace_bytes, void* stream) {
  return sinks_call(kv, nullptr, q, k_new, v_new, out, batch, num_q_heads, count, t, nullptr, count_per_seq, window, sinks, scale, workspace,
                    workspace_bytes, stream, true);
}

int tempo_rope_prefill_sinks(const tempo_kv* kv, const tempo_rope* rope, const void* q_raw, const void* k_raw, const void* v_new, void* out,
                             int32_t batch, int32_t num_q_heads, int32_t t, int32_t count, const int32_t* count_per_seq, int32_t window,
                             int32_t sinks, float scale, void* workspace, size_t workspace_bytes, void* stream) {
  if (!rope) return TEMPO_ERR_NULL;
  return sinks_call(kv, rope, q_raw, k_raw, v_new, out, batch, num_q_heads, count, t, nullptr, count_per_seq, window, sinks, scale, workspace,
                    workspace_bytes, stream, true);
}

int tempo_rope_rotate_at(const tempo_rope* rope, const tempo_rope_axes* axes, const int32_t* positions, const void* x, void* y, int32_t dtype,
                         int32_t batch, int32_t count, int32_t heads, void* stream) {
  if (!rope || !positions || !x || !y) return TEMPO_ERR_NULL;
  if (dtype != TEMPO_BF16 && dtype != TEMPO_F32) return TEMPO_ERR_DTYPE;
  if (rope->head_dim != 64 && rope->head_dim != 128) return TEMPO_ERR_SHAPE;
  if (batch < 1 || batch > 65535 || count < 1 || heads < 1 || heads > 65535) return TEMPO_ERR_SHAPE;
  if ((int64_t)count * heads > INT32_MAX || (int64_t)batch * count * heads * rope->head_dim / 8 > INT32_MAX) return TEMPO_ERR_SHAPE;
  const int rc = check_axes(rope, axes, rope->head_dim);
  if (rc != TEMPO_OK) return rc;
  StoreParams none = {};
  none.batch = batch;
  none.count = count;
  PlaceParams p = place_params(none, rope, axes, positions);
  p.q = x;
  p.q_out = y;
  p.Hq = heads;
  return launch_status(launch_place(p, nullptr, nullptr, rope->head_dim, dtype, static_cast<hipStream_t>(stream)), "rope_rotate_at");
}

int tempo_rope_kv_append_at(const tempo_kv* kv, const tempo_rope* rope, const tempo_rope_axes* axes, const int32_t* positions, const void* k_raw,
                            const void* v_new, const void* q_raw, void* q_out, int32_t batch, int32_t num_q_heads, int32_t t,
                            const int32_t* t_per_seq, int32_t count, const int32_t* count_per_seq, void* stream) {
  int rc = check_store(kv);
  if (rc != TEMPO_OK) return rc;
  if (!positions || !k_raw || !v_new || ((q_raw == nullptr) != (q_out == nullptr))) return TEMPO_ERR_NULL;
  if (batch < 1 || batch > 65535 || count < 1 || count > (1 << 24)) return TEMPO_ERR_SHAPE;
  if (q_raw && (rc = check_heads(kv, batch, num_q_heads)) != TEMPO_OK) return rc;
  if (t < 0 || t > INT32_MAX - 64 - count) return TEMPO_ERR_RANGE;
  if ((rc = check_step(kv, t + count - 1)) != TEMPO_OK) return rc;
  if (kv->ring_blocks && (int64_t)count > (int64_t)kv->ring_blocks * kv->block_size) return TEMPO_ERR_RANGE;
  if ((rc = check_axes(rope, axes, kv->head_dim)) != TEMPO_OK) return rc;
  const int64_t heads = (q_raw ? num_q_heads : 0) + 2 * (int64_t)kv->num_kv_heads;
  if (batch * (int64_t)count * heads * kv->head_dim / 8 > INT32_MAX) return TEMPO_ERR_SHAPE;
  StoreParams store = store_params(kv, batch, t, t_per_seq, count);
  store.count_per_seq = count_per_seq;
  PlaceParams p = place_params(store, rope, axes, positions);
  p.Hrows = kv->num_kv_heads;
  p.q = q_raw;
  p.q_out = q_out;
  p.Hq = q_raw ? num_q_heads : 0;
  return launch_status(launch_place(p, k_raw, v_new, kv->head_dim, kv->dtype, static_cast<hipStream_t>(stream)), "rope_kv_append_at");
}

int tempo_tree_positions(const int32_t* parents, int32_t* positions, int32_t batch, int32_t nodes, int32_t t, const int32_t* t_per_seq,
                         void* stream) {
  if (!parents || !positions) return TEMPO_ERR_NULL;
  if (batch < 1 || batch > 65535 || nodes < 1 || nodes > kMaxNodes) return TEMPO_ERR_SHAPE;
  if (t < 0 || t > INT32_MAX - nodes) return TEMPO_ERR_RANGE;
  return launch_status(launch_tree_positions(parents, positions, batch, nodes, t, t_per_seq, static_cast<hipStream_t>(stream)),
                       "tree_positions");
}

int tempo_kv_keep(const tempo_kv* layers, int32_t num_layers, int32_t batch, int32_t t, const int32_t* t_per_seq, int32_t nodes,
                  const int32_t* kept, int32_t count, void* stream) {
  if (!layers || !kept) return TEMPO_ERR_NULL;
  if (num_layers < 1 || batch < 1 || batch > 65535) return TEMPO_ERR_SHAPE;
  if (count < 1 || count > kKeepRows || nodes < 1 || nodes > (1 << 24)) return TEMPO_ERR_SHAPE;
  int rc = TEMPO_OK;
  for (int32_t i = 0; i < num_layers; ++i) {
    const tempo_kv &a = layers[i], &first = layers[0];
    if ((rc = check_store(&a)) != TEMPO_OK) return rc;
    if (a.block_table != first.block_table || a.num_blocks != first.num_blocks || a.max_blocks_per_seq != first.max_blocks_per_seq ||
        a.block_size != first.block_size || a.num_kv_heads != first.num_kv_heads || a.head_dim != first.head_dim || a.dtype != first.dtype ||
        a.ring_blocks != first.ring_blocks)
      return TEMPO_ERR_SHAPE;
    for (int32_t j = 0; j <= i; ++j) {  // (a pool twice would be moved twice, one half of the launch over the other)
      if (layers[j].k_pool == a.v_pool || layers[j].v_pool == a.k_pool || (j < i && (layers[j].k_pool == a.k_pool || layers[j].v_pool == a.v_pool)))
        return TEMPO_ERR_SHAPE;
    }
  }
  if (layers->num_kv_heads > 32767) return TEMPO_ERR_SHAPE;
  const int32_t rows = count > nodes ? count : nodes;
  if (t < 0 || t > INT32_MAX - 64 - rows) return TEMPO_ERR_RANGE;
  if ((rc = check_step(layers, t + rows - 1)) != TEMPO_OK) return rc;
  if (layers->ring_blocks && (int64_t)rows > (int64_t)layers->ring_blocks * layers->block_size) return TEMPO_ERR_RANGE;
  KeepParams p;
  p.block_table = layers->block_table;
  p.t_per_seq = t_per_seq;
  p.kept = kept;
  p.t = t;
  p.z_log2 = ilog2_exact(layers->block_size);
  p.max_blocks_per_seq = layers->max_blocks_per_seq;
  p.tile_mask = tile_mask_of(layers);
  p.num_blocks = layers->num_blocks;
  p.Hkv = layers->num_kv_heads;
  p.nodes = nodes;
  p.count = count;
  for (int32_t at = 0; at < num_layers; at += kKeepLayers) {
    const int32_t n = num_layers - at < kKeepLayers ? num_layers - at : kKeepLayers;
    for (int32_t i = 0; i < kKeepLayers; ++i) {
      p.k_pool[i] = layers[at + (i < n ? i : 0)].k_pool;
      p.v_pool[i] = layers[at + (i < n ? i : 0)].v_pool;
    }
    rc = launch_status(launch_keep(p, batch, n, layers->head_dim, layers->dtype, static_cast<hipStream_t>(stream)), "kv_keep");
    if (rc != TEMPO_OK) return rc;
  }
  return TEMPO_OK;
}

}  // extern "C"
