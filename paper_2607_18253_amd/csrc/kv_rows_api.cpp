// kv_rows_api.cpp -- host side of what decides over the rows of a paged key/value cache: the weights
// that they got, which of them stay, and where they go (lar_kv_weigh, _select and _keep in
// include/lar.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>

#include "../../include/lar.h"
#include "kv_handle.h"

using namespace lar;

namespace {

// Bytes of a layer's weights.
uint64_t weight_bytes(const lar_kv* kv, int64_t n_blocks) {
  return ((uint64_t)n_blocks * kv->g.hkv << kv->g.sh) * sizeof(float);
}

lar_status check_grid(lar_kv* kv, int64_t groups, int threads) {
  if (kv_fits(groups, threads)) return LAR_OK;
  return fail(kv, LAR_E_CAPACITY, "a batch of %lld workgroups of %d threads", (long long)groups, threads);
}

lar_status check_table(lar_kv* kv, const int32_t* table, int32_t cols, int64_t need, const char* name) {
  if (!table) return fail(kv, LAR_E_ARG, "null %s", name);
  if (cols < need) return fail(kv, LAR_E_ARG, "%s has %d columns, the planned contexts need %lld", name, cols, (long long)need);
  return LAR_OK;
}

// Workgroups that share the rows of a block of keys, where there are few blocks: two for a CU in all, 2
// blocks of 32 rows of the longest chunk at least for each (of which a window's keys see fewer), sums within
// narrow_o; where that leaves out enough blocks for the time of the sums' launch, 4 us (2048 tokens alone, of 32
// heads of 128: 42 us, 162 with one workgroup for a block of keys; of 4 heads of 64 13 and 158; 100 tokens
// of 32 heads 11 and 15; 33 of them 11 and 9.4).
constexpr int kWeighGroups = 512, kWeighSplits = 32, kWeighLeast = 2, kWeighSaved = 8;
int32_t weigh_splits(const lar_kv* kv) {
  const int64_t groups = std::max<int64_t>(1, kv->blocks * kv->g.hkv), rows = (int64_t)kv->most_new * kv->g.G / 32;
  const int64_t n = std::max<int64_t>(1, std::min({kWeighGroups / groups, rows / kWeighLeast, (int64_t)kWeighSplits}));
  return rows - rows / n >= kWeighSaved ? (int32_t)n : 1;
}

// Working memory for a selection whose contexts are cut, or null where a workgroup takes a whole one.
// Five launches over all rows take 28 us and one for 165k rows; a workgroup 7 us and 0.87 for 1000 rows
// in its registers, 1.5 for 1000 that it reads again for every digit, and all of them one for 200k and 98k rows.
// Cut and whole: 8 contexts of 24k rows 28 and 28 us, of 64k 29 and 105, of 1M 154 and 2124; 256 of 32k 78 and
// 42, of 64k 126 and 167.
constexpr int kSelectWhole = 32768;
int32_t* select_work(const lar_kv* kv) {
  const int64_t narrow = (int64_t)2 * kv->waves * kNarrowRows * kv->g.D;  // words of narrow_o and wide_o
  const int64_t wide = (int64_t)2 * kv->groups * kWideRows * kv->g.D, cuts = kv->cuts * kv->g.hkv;
  if (kv_select_cuts(kv->longest) > kSelectCuts || kv_select_words((int64_t)kv->n_seq * kv->g.hkv, cuts) > narrow ||
      cuts * kSelectStretch > wide)
    return nullptr;
  const double n = kv->longest, all = (double)kv->rows * kv->g.hkv;
  const double whole = n <= kSelectWhole ? std::max(7 + 0.87e-3 * n, all / 200e3) : std::max(1.5e-3 * n, all / 98e3);
  return 28 + all / 165e3 < whole ? (int32_t*)kv->narrow_o : nullptr;
}

}  // namespace

extern "C" {

lar_status lar_kv_weigh(lar_kv* kv, const lar_kv_pages* pages, const lar_kv_rows* q, const int32_t* table,
                        int32_t table_cols, double scale, const float* lse, const float* before, float* weights) {
  if (lar_status st = ready(kv)) return st;
  if (kv->trees) return fail(kv, LAR_E_STATE, "the planned batch has trees, whose tokens are not weighed");
  if (!kv->n_tok) return LAR_OK;
  KvPool pool;
  KvRows qr;
  if (lar_status st = check(kv, pages, table, table_cols, &pool)) return st;
  if (lar_status st = check_rows(kv, q, kv->g.hq, "q", &qr)) return st;
  if (!(scale > 0.0) || !(scale < 1e30)) return fail(kv, LAR_E_ARG, "scale must be positive and finite");
  if (!lse || !before || !weights) return fail(kv, LAR_E_ARG, "null lse, before or weights");
  const uint64_t bytes = weight_bytes(kv, pages->n_blocks);
  const uintptr_t a0 = (uintptr_t)before, b0 = (uintptr_t)weights;
  if (a0 != b0 && a0 < b0 + bytes && b0 < a0 + bytes)
    return fail(kv, LAR_E_ARG, "before and weights must be the same or lie apart");
  if ((int64_t)kv->most_new * kv->g.G > 1 << 30)  // rows of a sequence and head are counted in 32 bits
    return fail(kv, LAR_E_CAPACITY, "%d new tokens of %d heads", kv->most_new, kv->g.G);
  const int32_t splits = weigh_splits(kv);
  if (lar_status st = check_grid(kv, kv->blocks * kv->g.hkv * splits, kWeighKeys)) return st;
  if (kv->window && a0 != b0)  // which carries rows over, by stretches
    if (lar_status st = check_grid(kv, kv->cuts * kv->g.hkv, 256)) return st;
  KvWeighArgs a{};
  a.plan = plan_id(kv);
  a.g = kv->g;
  a.pool = pool;
  a.q = qr;
  a.table = table;
  a.cols = table_cols;
  a.scale = std::max((float)(scale * 1.4426950408889634074), FLT_TRUE_MIN);
  a.window = kv->window;
  a.sinks = kv->sinks;
  a.lse = lse;
  a.before = before;
  a.after = weights;
  a.narrow = (const KvSeg*)(kv->dev + kv->lay.narrow);
  a.narrow_at = (const int32_t*)(kv->dev + kv->lay.narrow_at);
  a.n_narrow = kv->n_narrow;
  a.n_wide = (int32_t)kv->blocks;
  a.spans = (const KvSpan*)(kv->dev + kv->lay.spans);
  a.n_seq = kv->n_seq;
  a.cuts = (int32_t)(kv->cuts * kv->g.hkv);
  a.splits = splits;
  a.parts = kv->narrow_o;
  a.err = kv->err;
  return launch(kv, launch_kv_weigh, a);
}

lar_status lar_kv_select(lar_kv* kv, const float* weights, int64_t n_blocks, const int32_t* table, int32_t table_cols,
                         int32_t budget, int32_t first, int32_t last, int32_t* rows) {
  if (lar_status st = ready(kv)) return st;
  if (budget < 1 || first < 0 || last < 0 || first > budget || last > budget - first)
    return fail(kv, LAR_E_ARG, "a budget of %d rows, the first %d and the last %d among them", budget, first, last);
  if (!kv->n_seq) return LAR_OK;
  if (!weights || !rows) return fail(kv, LAR_E_ARG, "null weights or rows");
  if (n_blocks < 1 || n_blocks > ((((int64_t)1 << 32) - 1) >> kv->g.sh) / kv->g.hkv)
    return fail(kv, LAR_E_ARG, "n_blocks must be in 1 .. (2^32 - 1) / (block_size * n_kv_heads)");
  if (lar_status st = check_table(kv, table, table_cols, kv->all_pages, "block table")) return st;
  const int64_t contexts = (int64_t)kv->n_seq * kv->g.hkv;
  int32_t* const work = select_work(kv);  // in which there is no room for too many
  if (!work)
    if (lar_status st = check_grid(kv, contexts, kv_select_threads(contexts, kv->longest))) return st;
  KvSelectArgs a{};
  a.plan = plan_id(kv);
  a.g = kv->g;
  a.weights = weights;
  a.n_blocks = (uint32_t)n_blocks;
  a.table = table;
  a.cols = table_cols;
  a.n_seq = kv->n_seq;
  a.longest = kv->longest;
  a.spans = (const KvSpan*)(kv->dev + kv->lay.spans);
  a.budget = budget;
  a.first = first;
  a.last = last;
  a.rows = rows;
  a.work = work;
  a.numbers = (uint32_t*)kv->wide_o;
  a.cuts = a.work ? (int32_t)(kv->cuts * kv->g.hkv) : 0;
  a.err = kv->err;
  return launch(kv, launch_kv_select, a);
}

lar_status lar_kv_keep(lar_kv* kv, const lar_kv_pages* pages, const int32_t* table, int32_t table_cols,
                       const int32_t* to_table, int32_t to_cols, const int32_t* rows, int32_t n_rows, int32_t per_head,
                       int32_t fresh, float* weights) {
  if (lar_status st = ready(kv)) return st;
  if (n_rows < 0 || (per_head & ~1) || (fresh & ~1)) return fail(kv, LAR_E_ARG, "n_rows >= 0, per_head and fresh 0 or 1");
  if (!kv->n_seq || !n_rows) return LAR_OK;
  KvPool pool;
  if (!rows) return fail(kv, LAR_E_ARG, "null rows");
  if (lar_status st = check(kv, pages, table, table_cols, &pool)) return st;
  if (lar_status st = check_table(kv, table, table_cols, kv->all_pages, "block table")) return st;
  if (!to_table) {
    to_table = table;
    to_cols = table_cols;
  }
  // a list has no more rows than the context, and of the new tokens none goes up
  const int64_t places = fresh ? kv->longest : std::min(n_rows, kv->longest);
  if (lar_status st = check_table(kv, to_table, to_cols, ceil_div(places, (int64_t)1 << kv->g.sh), "table of the places"))
    return st;
  const KvKeepShape shape(kv->g, kv->n_seq, n_rows, weights != nullptr);
  if (lar_status st = check_grid(kv, shape.groups, shape.threads)) return st;
  KvKeepArgs a{};
  a.plan = plan_id(kv);
  a.g = kv->g;
  a.pool = pool;
  a.weights = weights;
  a.table = table;
  a.to = to_table;
  a.cols = table_cols;
  a.to_cols = to_cols;
  a.n_seq = kv->n_seq;
  a.spans = (const KvSpan*)(kv->dev + kv->lay.spans);
  a.rows = rows;
  a.heads = per_head ? kv->g.hkv : 1;
  a.n_rows = n_rows;
  a.fresh = fresh;
  a.err = kv->err;
  return launch(kv, launch_kv_keep, a);
}

}  // extern "C"
