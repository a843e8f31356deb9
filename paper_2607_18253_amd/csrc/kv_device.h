// kv_device.h -- what the host (kv_api.cpp) and the kernels (kv_pages.hip, kv_attend.hip)
// of the paged key/value cache share: the geometry, the plan of a token batch and the
// launches.
//
// Cache of one layer: pages of S = 2^sh tokens, [page][kv head][S][D] for K and for V, as
// 16-bit values or as e4m3 codes with one byte per (page, kv head, row): the exponent k of
// the row's scale 2^k, stored as k + 127.
#ifndef LAR_KV_DEVICE_H
#define LAR_KV_DEVICE_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace lar {

enum { kKvF16 = 0, kKvBf16 = 1, kKvE4m3 = 2 };

// Keys of one step of a wave (narrow tiles) and of a workgroup (wide tiles).
constexpr int kNarrowKeys = 32, kWideKeys = 64;
// Query rows -- (token, head of the group) pairs -- of one tile: a wave of the narrow
// kernel has 32, a workgroup of the wide kernel 32 per wave.
constexpr int kNarrowRows = 32, kWideWaves = 8, kWideRows = 32 * kWideWaves;
// Exponents of the e4m3 rows' scales.
constexpr int kKvExpMin = -100, kKvExpMax = 120;

// What a kernel reports to the host.
enum { kKvLostPage = 1, kKvOtherPlan = 2 };

// A new token of the batch: its row of the block table and its position there (< 0: a
// padding row).
struct KvTok {
  int32_t seq, pos;
};

// A stretch of key tiles of one query tile, the work of one wave or workgroup.  Tiles
// are counted over what the tile's rows can see: ns tiles of first tokens (sinks), then
// the tiles from fw on.  slot < 0: the stretch is the whole of its tile and writes the
// result; else its partial sums go to that slot.
struct KvSeg {
  int32_t q0, ntok;   // first new token and number of tokens of the query tile
  int32_t p0;         // position of the first one
  int32_t head, seq;  // kv head; row of the block table
  int32_t ns, fw;
  int32_t t0, t1;     // tiles [t0, t1)
  int32_t slot;
};

// join_rows rows, from row0 on, of a query tile whose key tiles were split: its partial sums
// are in slots [slot, slot + n).
struct KvJoin {
  int32_t q0, ntok, p0, head;
  int32_t slot, n;
  int32_t row0, wide;
};

struct KvGeom {
  int32_t hq, hkv, G, D, sh;
  int32_t dtype, cache;  // kKv*
};

struct KvPool {
  const void *k, *v;
  const uint8_t *ke, *ve;
  uint32_t n_blocks;
};

struct KvRows {
  const void* p;
  int64_t tok, head;  // strides in elements
};

// The plan that a launch was made for.  The device's copy starts with the number of the current
// one: a launch of a captured graph that finds another there touches nothing, since the offsets
// and counts of its arguments belong to the plan that is gone.
struct KvPlanId {
  const uint64_t* now;
  uint64_t id;
};

struct KvAttendArgs {
  KvPlanId plan;
  KvGeom g;
  KvPool pool;
  KvRows q;
  const int32_t* table;
  int32_t cols;
  float scale;        // of the scores, times log2(e)
  int32_t window, sinks;
  void* out;          // [T][hq][D]
  float* lse;         // [T][hq] or null
  const KvSeg *narrow, *wide;
  const int32_t *narrow_at, *wide_at;  // [n + 1] stretches of each wave / workgroup
  int32_t n_narrow, n_wide;            // waves, workgroups
  const KvJoin* join;
  int32_t n_join, join_rows, most_parts;  // most_parts: the most slots of one
  float *narrow_o, *wide_o;            // partial sums of a slot's rows
  float4 *narrow_ml, *wide_ml;         // [slot][rows]: scale of the weights (log2 units) and sums
  int32_t* err;
};

struct KvCopyArgs {
  KvPlanId plan;
  KvGeom g;
  KvPool pool;        // written by an append
  KvRows k, v;        // rows of the batch, [T][hkv][D]
  const int32_t* table;
  int32_t cols, n_tok;
  const KvTok* tok;
  int32_t* err;
};

hipError_t launch_kv_append(const KvCopyArgs& a, hipStream_t stream);
hipError_t launch_kv_read(const KvCopyArgs& a, hipStream_t stream);
hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t stream);

}  // namespace lar

#endif  // LAR_KV_DEVICE_H
