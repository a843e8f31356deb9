// kv_device.h -- what the host (kv_api.cpp, kv_rows_api.cpp, kv_handle.h) and the kernels (kv_pages.hip,
// kv_attend.hip, kv_tree.hip, kv_weigh.hip, kv_select.hip, kv_keep.hip; kv_attend.h, kv_cut.h) of the
// paged key/value cache share: the geometry, the plan of a token batch and the launches.
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

// Tokens of a tree, and of a batch's trees, at most.
constexpr int kMaxTree = 1024, kTreeTokens = 16384;

// What a kernel reports to the host.
enum { kKvLostPage = 1, kKvOtherPlan = 2, kKvBadRows = 3 };

// A new token of the batch: its row of the block table and its position there (< 0: a
// padding row).
struct KvTok {
  int32_t seq, pos;
};

// A sequence of the batch: its first new token, its new tokens and its context with them.  A tree's
// tokens have a record each, from word `tree` of the plan's on (-1: no tree): the token's place
// among those that it follows, then `words` words of bits, which keys it sees of the blocks of 32
// from the one that the first new token is in on.
struct KvSpan {
  int32_t q0, q_len, ctx;
  int32_t tree, words;
  int32_t blocks;  // blocks of kWeighKeys keys that are seen, of the sequences before it that take wide tiles
  int32_t cuts;    // stretches of kSelectStretch rows of those before it
};
constexpr int kWeighKeys = 256;

// The blocks of keys that some new token sees, of a sequence whose first one is at position `base` (< 0: a
// padding row, and token 0 comes first): `sinks` of the first keys, then from `first` on.
struct KvSeenBlocks {
  int32_t sinks, first;
  constexpr KvSeenBlocks(int32_t base, int32_t window, int32_t n_sinks)
      : sinks(n_sinks / kWeighKeys + (n_sinks % kWeighKeys != 0)),
        first(window && base >= window ? (base - window + 1) / kWeighKeys : 0) {
    if (sinks > first) sinks = first;
  }
  constexpr int32_t count(int32_t ctx) const {
    return sinks + (ctx / kWeighKeys + (ctx % kWeighKeys != 0)) - first;
  }
  // the first key of block i
  constexpr int32_t key(int32_t i) const { return (i < sinks ? i : first - sinks + i) * kWeighKeys; }
};

// Of those tokens, by number, the first and the one past the last that see some of the block from key kb on.
struct KvSeers {
  int32_t t0, t1;
  constexpr KvSeers(int32_t base, int32_t q_len, int32_t window, int32_t n_sinks, int32_t kb) : t0(0), t1(q_len) {
    if (kb > base) t0 = kb - base;
    if (base + t0 < 0) t0 = -base;
    if (window && kb >= n_sinks && kb - base < q_len - window - kWeighKeys + 1) t1 = kb - base + window + kWeighKeys - 1;
  }
};

// Contexts that are cut for the selection: stretches of one, one at least, and the working memory, in
// words, of `contexts` sequences and heads with `cuts` of them.  kSelectCuts: the most of one context.
constexpr int kSelectStretch = 4096, kSelectCuts = 256, kSelectDigits = 4, kSelectBins = 512;
constexpr int kv_select_cuts(int32_t ctx) { return ctx > kSelectStretch ? (ctx + (kSelectStretch - 1)) / kSelectStretch : 1; }
constexpr int64_t kv_select_words(int64_t contexts, int64_t cuts) {
  return contexts * 2 * kSelectDigits + (cuts + 3) / 4 * 4 + cuts * kSelectDigits * kSelectBins;
}

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
  const KvSpan* spans;                 // [n_seqs]
  const uint32_t* trees;               // records; null: no sequence has a tree
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

// The sums of the attention's weights.  The narrow tiles of the plan have their keys to themselves;
// the others' keys go by blocks, n_wide of them.
struct KvWeighArgs {
  KvPlanId plan;
  KvGeom g;
  KvPool pool;
  KvRows q;
  const int32_t* table;
  int32_t cols;
  float scale;        // of the scores, times log2(e)
  int32_t window, sinks;
  const float* lse;   // [T][hq]
  const float* before;
  float* after;       // [n_blocks][hkv][S]
  const KvSeg* narrow;
  const int32_t* narrow_at;
  int32_t n_narrow, n_wide;
  const KvSpan* spans;
  int32_t n_seq, cuts;  // cuts: stretches of kSelectStretch rows of all sequences and heads
  int32_t splits;       // workgroups that share the rows of a block of keys; 1: none do
  float* parts;         // their sums
  int32_t* err;
};

struct KvSelectArgs {
  KvPlanId plan;
  KvGeom g;
  const float* weights;  // [n_blocks][hkv][S]
  uint32_t n_blocks;
  const int32_t* table;
  int32_t cols, n_seq, longest;  // longest: context of any
  const KvSpan* spans;
  int32_t budget, first, last;
  int32_t* rows;         // [n_seq][hkv][budget]
  int32_t* work;         // where contexts are cut, else null
  uint32_t* numbers;     // their weights as numbers that order so, by stretches
  int32_t cuts;          // of all sequences and heads
  int32_t* err;
};

struct KvKeepArgs {
  KvPlanId plan;
  KvGeom g;
  KvPool pool;           // written
  float* weights;        // of the rows, or null
  const int32_t *table, *to;
  int32_t cols, to_cols, n_seq;
  const KvSpan* spans;
  const int32_t* rows;   // [n_seq][heads][n_rows], heads hkv or 1
  int32_t heads, n_rows;
  int32_t fresh;         // rows count from the first new token
  int32_t* err;
};

// A launch has less than 2^32 threads.
constexpr bool kv_fits(int64_t groups, int threads) { return groups * threads < (int64_t)1 << 32; }

// Threads for a context: while each has a CU of its own the more the better (256 contexts of 4000 rows: 17, 11
// and 9.6 us with 256, 512 and 1024; of 16000 153, 40 and 27), then as many as leave room for others (1024 of
// 4000: 28, 21 and 37; of 16000 225, 63 and 103), and of many short ones fewest (4096 of 600: 24, 29 and 71).
constexpr int kSelectCus = 256;
constexpr int kv_select_threads(int64_t contexts, int32_t longest) {
  if (contexts <= kSelectCus || longest > 16384) return 1024;
  return contexts <= 4 * kSelectCus || longest > 2048 ? 512 : 256;
}

// The launch of a move: of each list `jobs` workgroups, `shares` for K, as many for V, and one for the rows'
// exponents and weights.
//
// A few passes of a small workgroup, or as many threads as there are, which have fewer barriers for their
// bytes, and then a cache line of a long row for each workgroup (127 contexts to 777 rows of 256 bytes in
// the kernel: 137 us; with 256 threads 141, with whole rows 144, with half lines 166).  Half lines only while
// lists leave CUs over (8 lists of 5000 such rows: 27 us, 39 with lines; 32 of them: 56 and 46).
struct KvKeepShape {
  static constexpr int kFewGroups = 128;  // half the CUs
  int threads, shares = 1, jobs;
  int64_t groups;
  KvKeepShape(const KvGeom& g, int32_t n_seq, int32_t n_rows, bool weights) {
    const int64_t lists = (int64_t)n_seq * g.hkv;
    const int cols = g.D * (g.cache == kKvE4m3 ? 1 : 2) / 16;  // 16 bytes each
    const bool small = n_rows * (int64_t)cols <= 2048;
    threads = small ? 256 : 1024;
    if (!small && cols == 16) shares = 2;
    while (!small && 2 * lists * shares < kFewGroups && cols / shares > 4) shares *= 2;
    jobs = 2 * shares + (g.cache == kKvE4m3 || weights);
    groups = lists * jobs;
  }
};

hipError_t launch_kv_append(const KvCopyArgs& a, hipStream_t stream);
hipError_t launch_kv_read(const KvCopyArgs& a, hipStream_t stream);
hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t stream);
hipError_t launch_kv_tree(const KvAttendArgs& a, hipStream_t stream);
hipError_t launch_kv_weigh(const KvWeighArgs& a, hipStream_t stream);
hipError_t launch_kv_select(const KvSelectArgs& a, hipStream_t stream);
hipError_t launch_kv_keep(const KvKeepArgs& a, hipStream_t stream);

}  // namespace lar

#endif  // LAR_KV_DEVICE_H
