// host_launches_e4m3.cpp with the launches of windows with sinks, trees, rows at positions and kept rows recorded too, and the
// pure functions by which their workgroups find their work.
#include "host_launches_e4m3.cpp"

namespace tempo {
static hipError_t spans(const char* what, const SpanParams& p, int batch, int D, int waves) {
  return say("%s t=%d rows=%d window=%d sinks=%d tile=%d split_groups=%d splits=%d direct=%d waves=%d tree=%d k=%zu end=%zu", what, p.t, p.queries, p.window,
             p.sinks, p.tile_columns, p.split_groups, p.num_splits, p.direct, waves, p.parents != nullptr, (size_t)p.k_new,
             (size_t)p.ws_acc + (p.direct ? 0 : (size_t)batch * p.queries * p.Hq * p.num_splits * D * 4));
}
hipError_t launch_spans(const SpanParams& p, int batch, int D, int, int waves, hipStream_t) { return spans("spans", p, batch, D, waves); }
hipError_t launch_spans_wide(const SpanParams& p, int batch, int D, int, hipStream_t) { return spans("spans_wide", p, batch, D, 4); }
hipError_t launch_spans_f32(const SpanParams& p, int batch, int D, int waves, hipStream_t) { return spans("spans_f32", p, batch, D, waves); }
hipError_t launch_combine_spans(const SpanParams& p, int batch, int D, int, hipStream_t) { return spans("combine_spans", p, batch, D, 0); }
hipError_t launch_place(const PlaceParams& p, const void* k, const void*, int, int, hipStream_t) {
  return say("place t=%d count=%d Hq=%d Hrows=%d axes=%d rows=%d low=%zu high=%zu k=%zu", p.t, p.count, p.Hq, p.Hrows, p.axes, p.table_rows,
             (size_t)p.axis_bits[0], (size_t)p.axis_bits[1], (size_t)k);
}
hipError_t launch_tree_positions(const int32_t*, int32_t*, int, int nodes, int t, const int32_t*, hipStream_t) { return say("positions t=%d nodes=%d", t, nodes); }
hipError_t launch_keep(const KeepParams& p, int, int layers, int, int, hipStream_t) {
  return say("keep t=%d nodes=%d count=%d layers=%d first=%zu last=%zu", p.t, p.nodes, p.count, layers, (size_t)p.k_pool[0], (size_t)p.v_pool[layers - 1]);
}
}  // namespace tempo

extern "C" {
void span_range_of(int t, int tile, int tile_columns, int G, int rows, int window, int sinks, int tree, int32_t* out) {
  const tempo::SpanRange r = tempo::tile_range(t, tile, tile_columns, G, rows, window, sinks, tree != 0);
  out[0] = r.lo;
  out[1] = r.sink_groups;
  out[2] = r.g_lo;
  out[3] = r.groups;
}
int span_group_of(int t, int first, int last, int window, int sinks, int i) {
  return tempo::span_group(tempo::span_range(t, first, last, window, sinks), i);
}
uint32_t fewer_keys_of(int t, int window, int G, int tile_columns, uint32_t blocks) { return tempo::fewer_keys(t, window, G, tile_columns, blocks); }
void wide_work_of(uint32_t x, uint32_t y, uint32_t z, uint32_t nx, uint32_t ny, uint32_t nz, int Hkv, uint32_t fewer, int32_t* out) {
  const tempo::UnitsWork w = tempo::wide_work(x, y, z, nx, ny, nz, Hkv, fewer);
  out[0] = w.hkv;
  out[1] = w.tile;
  out[2] = w.b;
  out[3] = w.split;
}
}
