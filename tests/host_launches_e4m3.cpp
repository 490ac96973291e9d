// host_launches.cpp with the launches of the 8-bit store and of the attention over selected blocks recorded too.
#include "host_launches.cpp"

namespace tempo {
hipError_t launch_append_e4m3(const StoreParams& p, const void* k, const void* v, int, hipStream_t) {
  return say("append t=%d count=%d steps=%d k=%zu v=%zu", p.t, p.count, p.src_steps, (size_t)k, (size_t)v);
}
hipError_t launch_gather_e4m3(const StoreParams&, void*, void*, int, int j0, int count, hipStream_t) { return say("gather t=%d count=%d", j0, count); }
hipError_t launch_append_copy_e4m3(const StoreParams& p, const UnpackParams& u, const void* k, const void* v, int D, hipStream_t) {
  say("append t=%d count=%d steps=%d k=%zu v=%zu", p.t, p.count, p.src_steps, (size_t)k, (size_t)v);
  const int groups = (p.count + 31) >> 5;
  return say("unpack first=%d groups=%d tiles=%d mask=%d table=%zu k=%zu v=%zu end=%zu", u.first_group, groups, u.tiles, u.tile_mask, (size_t)u.table,
             (size_t)u.k, (size_t)u.v, (size_t)u.v + ((size_t)p.batch * u.tiles * p.Hkv << p.z_log2) * D * 2);
}
hipError_t launch_unpack_e4m3(const StoreParams& p, const UnpackParams& u, int groups, int D, hipStream_t) {
  return say("unpack first=%d groups=%d tiles=%d mask=%d table=%zu k=%zu v=%zu end=%zu", u.first_group, groups, u.tiles, u.tile_mask, (size_t)u.table,
             (size_t)u.k, (size_t)u.v, (size_t)u.v + ((size_t)p.batch * u.tiles * p.Hkv << p.z_log2) * D * 2);
}
hipError_t launch_partial_e4m3(const AttnParams& p, int, int, int grid_splits, int waves, hipStream_t) {
  return attend("partial_e4m3", p, grid_splits, waves);
}
hipError_t launch_partial_selected(const SelectParams& p, int, int, int, int grid_splits, int waves, hipStream_t) {
  return say("selected t=%d pick=%d tps_log2=%d num_splits=%d grid_splits=%d direct=%d waves=%d", p.t, p.pick, p.tps_log2, p.num_splits, grid_splits,
             p.direct, waves);
}
hipError_t launch_combine_selected(const AttnParams& p, int, int, hipStream_t) { return say("combine_selected t=%d num_splits=%d", p.t, p.num_splits); }
hipError_t launch_block_bounds(const StoreParams& p, void*, int, int, hipStream_t) { return say("bounds t=%d count=%d", p.t, p.count); }
hipError_t launch_select_blocks(const ChooseParams& p, const StoreParams* store, const void*, const void*, int, int, int, hipStream_t) {
  return say("select t=%d pick=%d tiles=%d store=%d", p.t, p.pick, p.tiles, store != nullptr);
}
}  // namespace tempo
