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
// As stub_plan(), of the last attention: 0: `room` numbers of the spans, 1: `room` words of the records
// (none without trees).
int stub_trees(int what, int32_t* to, int room) {
  const void* p = what == 0 ? (const void*)attend.spans : attend.trees;
  if (!p) return 0;
  std::memcpy(to, p, sizeof(int32_t) * room);
  return room;
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
// Blocks of keys that a sequence's new tokens see; of block i the first key, and the tokens that see it.
int stub_seen_blocks(int32_t ctx, int32_t q_len, int32_t window, int32_t sinks, int32_t i, int32_t* to) {
  const lar::KvSeenBlocks b(ctx - q_len, window, sinks);
  to[0] = b.key(i);
  const lar::KvSeers s(ctx - q_len, q_len, window, sinks, to[0]);
  to[1] = s.t0;
  to[2] = s.t1;
  return b.count(ctx);
}
// The number of the plan that the last call of a kind was made for: weights, selection, move.
uint64_t stub_rows_plan(int what) { return what == 0 ? weigh.plan.id : what == 1 ? select_.plan.id : keep.plan.id; }
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
