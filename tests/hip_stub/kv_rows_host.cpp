// The launches behind kv_rows_api.cpp beside those of kv_host.cpp, and what a plan with trees has on
// the device.
#include "kv_host.cpp"

namespace {
lar::KvWeighArgs weigh{};
lar::KvSelectArgs select_{};
lar::KvKeepArgs keep{};
}  // namespace

namespace lar {
hipError_t launch_kv_weigh(const KvWeighArgs& a, hipStream_t) {
  weigh = a;
  return note();
}
hipError_t launch_kv_select(const KvSelectArgs& a, hipStream_t) {
  select_ = a;
  return note();
}
hipError_t launch_kv_keep(const KvKeepArgs& a, hipStream_t) {
  keep = a;
  return note();
}
}  // namespace lar

extern "C" {
// As stub_plan(), of the last attention: 0: spans, 1: tree stretches, 2: where the runs of each start, 3: the
// trees' joins; 4: waves of a tile and rows of a join's workgroup; 5: `room` words of the records.
int stub_trees(int what, int32_t* to, int room) {
  const void* p = nullptr;
  int n = 0;
  const int32_t two[2] = {attend.tree_waves, attend.tree_join_rows};
  if (what == 0) p = attend.spans, n = room;
  if (what == 1) p = attend.tree, n = attend.n_tree ? attend.tree_at[attend.n_tree] * 10 : 0;
  if (what == 2) p = attend.tree_at, n = attend.n_tree ? attend.n_tree + 1 : 0;
  if (what == 3) p = attend.tree_join, n = attend.n_tree_join * 8;
  if (what == 4) p = two, n = 2;
  if (what == 5) p = attend.trees, n = room;
  if (n) std::memcpy(to, p, sizeof(int32_t) * (n < room ? n : room));
  return n;
}
// Blocks of keys, places of the tables, and whether a call has been handed on since the last time.
int stub_weigh(int32_t* to) {
  to[0] = weigh.n_wide;
  to[1] = weigh.n_seq;
  to[2] = weigh.n_narrow;
  const int was = weigh.after != nullptr;
  weigh.after = nullptr;
  return was;
}
int stub_keep(int32_t* to) {
  to[0] = keep.heads;
  to[1] = keep.n_rows;
  to[2] = keep.fresh;
  to[3] = keep.to == keep.table;
  const int was = keep.rows != nullptr;
  keep.rows = nullptr;
  return was;
}
}
