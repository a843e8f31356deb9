// kv_api.cpp -- host side of the paged key/value cache (lar_kv_* in include/lar.h).
//
// A handle keeps the geometry, the plan of the current token batch and the working memory
// of the attention; the pages belong to the caller.  lar_kv_plan checks the lengths, cuts
// the attention into stretches of equal work and copies the plan to the device from one of
// two pinned buffers; the other calls enqueue kernels, allocate nothing and do not wait.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <functional>
#include <new>
#include <string>
#include <vector>

#include "../../include/lar.h"
#include "kv_device.h"

using namespace lar;

namespace {

constexpr int kStages = 2;  // pinned copies of a plan: one may be on its way while the next is written

size_t up(size_t x) { return (x + 255) & ~size_t(255); }

// Byte offsets of a plan's arrays, the same on the host and on the device, after its number.
struct Layout {
  size_t tok = up(sizeof(uint64_t)), narrow = 0, wide = 0, narrow_at = 0, wide_at = 0, join = 0, end = 0;
  Layout() = default;
  Layout(int64_t n_tok, int64_t n_narrow, int64_t n_wide, int64_t waves, int64_t groups, int64_t n_join) {
    narrow = up(tok + sizeof(KvTok) * n_tok);
    wide = up(narrow + sizeof(KvSeg) * n_narrow);
    narrow_at = up(wide + sizeof(KvSeg) * n_wide);
    wide_at = up(narrow_at + sizeof(int32_t) * (waves + 1));
    join = up(wide_at + sizeof(int32_t) * (groups + 1));
    end = up(join + sizeof(KvJoin) * n_join);
  }
};

}  // namespace

struct lar_kv {
  lar_kv_config cfg{};
  KvGeom g{};
  hipStream_t stream = nullptr;
  int device = 0, cus = 0;
  int waves = 0, groups = 0;  // of the narrow and the wide kernel at most
  size_t cap = 0;             // bytes of a plan at most
  Layout lay;                 // of the current plan
  char* dev = nullptr;
  char* pinned[kStages] = {};
  hipEvent_t done[kStages] = {};
  bool used[kStages] = {};
  int stage = 0;
  float *narrow_o = nullptr, *wide_o = nullptr;
  float4 *narrow_ml = nullptr, *wide_ml = nullptr;
  int32_t* err = nullptr;
  // the plan
  bool planned = false;
  uint64_t plan = 0;  // its number
  int32_t n_seq = 0, n_tok = 0, max_pages = 0, window = 0, sinks = 0;
  int32_t n_narrow = 0, n_wide = 0, n_join = 0, join_rows = 0, most_parts = 0;
  lar_status sticky = LAR_OK;
  std::string msg;
};

namespace {

lar_status fail(lar_kv* kv, lar_status code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    kv->msg = buf;
  } catch (...) {
  }
  return code;
}

#define KV_TRY(kv, expr)                                                           \
  do {                                                                             \
    hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess) return fail(kv, LAR_E_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

// The handle's device is the current one while this lives: the null stream, and calls without
// a stream, go to the current device.
class OnDevice {
 public:
  explicit OnDevice(const lar_kv* kv) {
    int now = 0;
    status_ = hipGetDevice(&now);
    if (status_ != hipSuccess || now == kv->device) return;
    status_ = hipSetDevice(kv->device);
    if (status_ == hipSuccess) before_ = now;
  }
  ~OnDevice() {
    if (before_ >= 0) (void)hipSetDevice(before_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  hipError_t status() const { return status_; }

 private:
  int before_ = -1;
  hipError_t status_ = hipSuccess;
};

// A plan's number, made of all that a plan follows from, so that equal batches have equal plans
// with equal numbers.  Each step maps the numbers one to one: batches that differ in one sequence's
// lengths have different ones, and others the same with a chance of 2^-64.
struct PlanId {
  uint64_t x = 0x243f6a8885a308d3u;  // fraction of pi
  void add(uint32_t a, uint32_t b) {
    x = (x ^ ((uint64_t)a << 32 | b)) * 0x9e3779b97f4a7c15u;  // odd
    x ^= x >> 29;
  }
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The key tiles (of K keys) that the tokens p0 .. p0 + n - 1 of a sequence see: tiles
// [0, ns), then from fw on; their number.
int key_tiles(int64_t p0, int n, int K, int window, int sinks, int* ns, int* fw) {
  const int64_t last = p0 + n - 1;
  *ns = *fw = 0;
  if (last < 0) return 0;
  const int64_t all = last / K + 1;
  const int64_t lo = window ? std::max<int64_t>(0, std::max<int64_t>(p0, 0) - window + 1) : 0;
  const int64_t first = lo / K;
  const int64_t head = std::min<int64_t>(ceil_div(sinks, K), first);  // tiles of sinks before the window
  *ns = (int)head;
  *fw = (int)first;
  return (int)(head + all - first);
}

// Waves of the narrow kernel per CU: the 8 that its registers leave room for, with 8-bit rows
// of 64, which need fewer registers and more rows on their way, 12 (509 requests of 9.2k
// tokens: 1015 us with 8, 933 with 12; 16-bit rows of 64 lose 5 % with 12).
int narrow_per_cu(const KvGeom& g) { return g.D == 64 && g.cache == kKvE4m3 ? 12 : 8; }

// Query tiles of one kernel, in the order in which they are cut into stretches.
struct Tile {
  KvSeg s;
  int tiles;
};

// The split tiles of a plan, and the join list made of them: a workgroup for every `rows` rows.
// Fewer rows leave more threads to share the slots out to, and more CUs to load them; too many
// workgroups take longer to start than that saves.  8 instead of 32 where that makes at most
// kJoins8 workgroups (40 tokens of 4 heads over 400 keys: 14 us, 19 with 32; a limit of 256 takes
// 19), 2 where it makes at most kJoins2 and there are more than kManyParts slots (one token of 4
// heads over 60k keys: 52 us, 55 with 8; over 1000 keys, 32 slots: 10.3 and 9.7).
constexpr int kJoins8 = 512, kJoins2 = 64, kManyParts = 64;
struct Joins {
  int32_t G, most = 0;
  std::vector<KvJoin> tiles;
  void add(const KvSeg& s, int32_t slot, int32_t parts, bool wide) {
    KvJoin j{};
    j.q0 = s.q0;
    j.ntok = s.ntok;
    j.p0 = s.p0;
    j.head = s.head;
    j.slot = slot;
    j.n = parts;
    j.wide = wide;
    tiles.push_back(j);
    most = std::max(most, parts);
  }
  int64_t count(int rows) const {
    int64_t n = 0;
    for (const KvJoin& j : tiles) n += ceil_div((int64_t)j.ntok * G, rows);
    return n;
  }
  int32_t write(KvJoin* list, int32_t* rows) const {
    *rows = most > kManyParts && count(2) <= kJoins2 ? 2 : count(8) <= kJoins8 ? 8 : 32;
    int32_t n = 0;
    for (KvJoin j : tiles)
      for (j.row0 = 0; j.row0 < j.ntok * G; j.row0 += *rows) list[n++] = j;
    return n;
  }
};

// Least key tiles of a wave's run.  A wave takes about 1.1 us for one; joining n parts of r
// rows takes time in proportion to n * r * D, since a workgroup's threads share their quads
// out.  A tile of T key tiles in stretches of L then ends soonest with L = sqrt(T r D * c), here
// from measurements at T = 1179, r = 4 and 8, D = 128 (32 and 52 us with L = 2, 24 and 28 with 8,
// 31 and 33 with 16) and T = 7 to 114, r = 4 (8.6 and 11 us with L = 1 and 2 at T = 7, 15.0 and 13.9
// at T = 114).  From some hundred key tiles on their waves no longer have a SIMD for themselves,
// and runs of one cost more than they save.
int narrow_least(const std::vector<Tile>& tiles, const KvGeom& g) {
  double most = 0;
  int64_t total = 0;
  for (const Tile& t : tiles) total += t.tiles;
  for (const Tile& t : tiles) most = std::max(most, (double)t.tiles * (t.s.ntok * g.G));
  return std::max(total > 512 ? 2 : 1, (int)std::lround(std::sqrt(most * g.D * 5.8e-5)));
}

// Narrow tiles: cuts their key tiles into stretches of equal number, one run of them for each
// of at most `most` waves; a tile that is cut goes to the join.
void cut(const std::vector<Tile>& tiles, int most, int least, KvSeg* segs, int32_t* at, int32_t* n_run,
         Joins* join) {
  int64_t total = 0;  // a tile without keys still has its result to write
  for (const Tile& t : tiles) total += std::max(1, t.tiles);
  int64_t runs = std::max<int64_t>(1, std::min<int64_t>(most, total / least));
  *n_run = 0;
  if (tiles.empty()) return;
  int32_t n_seg = 0, slot = 0;
  int64_t before = 0;  // key tiles before the current tile
  int64_t run = 0;     // run w has key tiles [total * w / runs, total * (w + 1) / runs)
  at[0] = 0;
  for (const Tile& t : tiles) {
    const int64_t n = std::max(1, t.tiles);
    int64_t x = 0;
    const int32_t slot0 = slot;
    int parts = 0;
    while (x < n) {
      int64_t end = total * (run + 1) / runs;
      while (end <= before + x) {
        at[++run] = n_seg;
        end = total * (run + 1) / runs;
      }
      const int64_t y = std::min(n, end - before);
      KvSeg s = t.s;
      s.t0 = (int32_t)x;
      s.t1 = (int32_t)(t.tiles ? y : 0);
      s.slot = x == 0 && y == n ? -1 : slot++;
      segs[n_seg++] = s;
      ++parts;
      x = y;
    }
    if (parts > 1) join->add(t.s, slot0, parts, false);
    before += n;
  }
  while (run < runs) at[++run] = n_seg;
  *n_run = (int32_t)runs;
}

// Wide tiles.  Where they are short for the workgroups: whole tiles where that
// balances, parts of at most `limit` key tiles where it does not, the longest first to the
// workgroup with the least work.  Costs are in key tiles, of about 2 us each.
constexpr int kStart = 2;  // a stretch's queries, first keys and result
// The join: its launch, its slots' latency, and their rows' bytes, written and read at about
// 3 TB/s (2.2 us, 0.07 a slot); a key tile of narrower heads takes less time than that counts for.
double join_cost(int32_t most, int64_t rows, int D) {
  return (1.25 + 0.04 * most + 1.6e-6 * (double)(rows * D)) * (D == 128 ? 1.0 : 1.5);
}
// From this many key tiles per workgroup on parts cost nothing against them, and workgroups
// that read the same keys at the same time from one L2 are worth more.
constexpr int kLong = 128;
constexpr int kXcds = 8;  // workgroup runs are contiguous on an XCD (run_of in kv_attend.hip)

// Long wide tiles: the workgroups of an XCD take neighbouring tiles whole, round by round, so
// that they walk over the same keys together (a chunk of 7681 tokens at 131072: cut in order
// 94 % of the L2's requests went on to memory and a call took 17.9 ms); what is left fills
// them up to equal work, cut where it has to be.
void march(const std::vector<Tile>& tiles, int groups, KvSeg* segs, int32_t* at, int32_t* n_run, Joins* join) {
  struct Part {
    int32_t run, tile, t0, t1;
  };
  std::vector<Part> parts;
  std::vector<int64_t> load(groups, 0);
  std::vector<int32_t> rest;
  int64_t total = 0;
  for (const Tile& t : tiles) total += std::max(1, t.tiles);
  const int64_t target = ceil_div(total, groups);
  int64_t before = 0;
  size_t i = 0;
  for (int x = 0, run0 = 0; x < kXcds; ++x) {
    const int runs = groups / kXcds + (x < groups % kXcds ? 1 : 0);
    // the tiles whose middle lies in this XCD's share
    const size_t first = i;
    while (i < tiles.size() &&
           (x == kXcds - 1 || (2 * before + tiles[i].tiles) * groups < 2 * total * (run0 + runs))) {
      before += std::max(1, tiles[i].tiles);
      ++i;
    }
    size_t rounds = runs ? (i - first) / runs : 0;
    for (; rounds; --rounds) {
      int64_t most = 0;
      for (int w = 0; w < runs; ++w) {
        int64_t n = 0;
        for (size_t k = 0; k < rounds; ++k) n += std::max(1, tiles[first + k * runs + w].tiles);
        most = std::max(most, n);
      }
      if (most <= target) break;
    }
    for (size_t k = 0; k < rounds * runs; ++k) {
      const int w = run0 + (int)(k % runs);
      parts.push_back(Part{w, (int32_t)(first + k), 0, tiles[first + k].tiles});
      load[w] += std::max(1, tiles[first + k].tiles);
    }
    for (size_t k = first + rounds * runs; k < i; ++k) rest.push_back((int32_t)k);
    run0 += runs;
  }
  int w = 0;
  for (int32_t k : rest) {
    const int32_t n = std::max(1, tiles[k].tiles);
    int32_t x = 0;
    while (x < n) {
      while (w < groups - 1 && load[w] >= target) ++w;
      const int32_t y = w < groups - 1 ? (int32_t)std::min<int64_t>(n, x + target - load[w]) : n;
      parts.push_back(Part{w, k, x, std::min(y, tiles[k].tiles)});
      load[w] += y - x;
      x = y;
    }
  }
  std::vector<int32_t> fill(groups + 1, 0), made(tiles.size(), 0), slot(tiles.size(), -1);
  for (const Part& q : parts) {
    ++fill[q.run + 1];
    ++made[q.tile];
  }
  for (int g = 0; g < groups; ++g) fill[g + 1] += fill[g];
  for (int g = 0; g <= groups; ++g) at[g] = fill[g];
  int32_t next = 0;
  for (size_t k = 0; k < tiles.size(); ++k) {
    if (made[k] < 2) continue;
    slot[k] = next;
    join->add(tiles[k].s, next, made[k], true);
    next += made[k];
  }
  for (const Part& q : parts) {  // parts of a tile come in the order of their keys
    KvSeg s = tiles[q.tile].s;
    s.t0 = q.t0;
    s.t1 = q.t1;
    s.slot = made[q.tile] > 1 ? slot[q.tile]++ : -1;
    segs[fill[q.run]++] = s;
  }
  *n_run = groups;
}

void deal(const std::vector<Tile>& tiles, int groups, const KvGeom& g, KvSeg* segs, int32_t* at, int32_t* n_run,
          Joins* join) {
  int64_t total = 0;
  for (const Tile& t : tiles) total += std::max(1, t.tiles);
  *n_run = 0;
  if (tiles.empty()) return;
  if (total / groups >= kLong) {
    march(tiles, groups, segs, at, n_run, join);
    return;
  }
  struct Piece {
    int32_t tile, part, cost;
  };
  const auto parts_of = [](const Tile& t, int64_t limit) { return (int32_t)std::max<int64_t>(1, ceil_div(t.tiles, limit)); };
  const auto cost_of = [](const Tile& t, int32_t parts) { return (int32_t)ceil_div(t.tiles, parts) + kStart; };
  std::vector<Piece> pieces, best;
  std::vector<std::pair<int32_t, int32_t>> load;  // (work, workgroup), the least first
  const auto more = std::greater<std::pair<int32_t, int32_t>>();
  // hands the pieces out; returns the most that a workgroup has
  const auto hand_out = [&](const std::vector<Piece>& p, int32_t* to) {
    load.clear();
    for (int g = 0; g < groups; ++g) load.emplace_back(0, g);
    int32_t most = 0;
    for (size_t i = 0; i < p.size(); ++i) {
      std::pop_heap(load.begin(), load.end(), more);
      load.back().first += p[i].cost;
      most = std::max(most, load.back().first);
      if (to) to[i] = load.back().second;
      std::push_heap(load.begin(), load.end(), more);
    }
    return most;
  };
  const int64_t even = std::max<int64_t>(1, total * 2 / groups);
  int64_t chosen = INT32_MAX, before = 0;
  double least = 1e300;
  for (const int64_t limit : {(int64_t)INT32_MAX, even * 4, even * 2, even * 3 / 2, even, even * 3 / 4, even / 2, even / 4}) {
    if (limit < 1) break;
    pieces.clear();
    int64_t parts = 0, rows = 0;
    int32_t many = 0;
    for (size_t i = 0; i < tiles.size(); ++i) {
      const int32_t n = parts_of(tiles[i], limit);
      if (n > 1) {
        parts += n;
        rows += (int64_t)n * tiles[i].s.ntok * g.G;
        many = std::max(many, n);
      }
      for (int32_t j = 0; j < n; ++j) pieces.push_back(Piece{(int32_t)i, j, cost_of(tiles[i], n)});
    }
    if (parts > 2 * groups) break;             // slots; and the smaller limits have more parts
    if (parts == before && !best.empty()) continue;  // nothing more was cut
    before = parts;
    std::stable_sort(pieces.begin(), pieces.end(), [](const Piece& x, const Piece& y) { return x.cost > y.cost; });
    const double most = hand_out(pieces, nullptr) + (parts ? join_cost(many, rows, g.D) : 0.0);
    if (most < least) {
      least = most;
      chosen = limit;
      best = pieces;
    }
  }
  std::vector<int32_t> to(best.size()), slot(tiles.size(), -1);
  hand_out(best, to.data());
  int32_t next = 0;
  for (size_t i = 0; i < tiles.size(); ++i) {
    const Tile& t = tiles[i];
    const int32_t n = parts_of(t, chosen);
    if (n < 2) continue;
    slot[i] = next;
    join->add(t.s, next, n, true);
    next += n;
  }
  const int32_t runs = (int32_t)std::min<size_t>(groups, best.size());
  std::vector<int32_t> fill(groups + 1, 0);
  for (int32_t g : to) ++fill[g + 1];
  for (int g = 0; g < groups; ++g) fill[g + 1] += fill[g];
  for (int g = 0; g <= runs; ++g) at[g] = fill[g];
  for (size_t i = 0; i < best.size(); ++i) {
    const Tile& t = tiles[best[i].tile];
    const int32_t n = parts_of(t, chosen);
    KvSeg s = t.s;
    s.t0 = (int32_t)((int64_t)t.tiles * best[i].part / n);
    s.t1 = (int32_t)((int64_t)t.tiles * (best[i].part + 1) / n);
    s.slot = n > 1 ? slot[best[i].tile] + best[i].part : -1;
    segs[fill[to[i]]++] = s;
  }
  *n_run = runs;
}

// How many of a device's workgroups the wide tiles of a batch get that has narrow ones too.
// Both need time in proportion to their workgroups until the narrow ones, which are bound by
// memory, reach its rate (with 16-bit rows of 128 from about 150 CUs on), so that most
// batches end sooner with both at work (mixed batch of 3839 tokens: 387 us one after the other,
// 293 together).  Where the two bounds of the narrow ones meet they take more than either: a sum
// of sixth powers (mixed batch: 298 us with the larger of the two).
int split(const std::vector<Tile>& narrow, const std::vector<Tile>& wide, int groups, const KvGeom& g) {
  if (wide.empty()) return 0;
  // microseconds: of a wide key tile and a stretch's start and end, of a narrow one among a
  // CU's eight waves (255 tokens beside 7 chunks of 512 with heads of 64: 161 us, 182 with a time
  // 1.6 times less; 40 tokens beside them: 92 and 103); bytes of a narrow one
  const double wt = g.D == 128 ? 2.1 : 1.35, ws = 8.0, nt = g.D == 128 ? 3.4 : 2.7;
  const double nb = 2.0 * kNarrowKeys * g.D * (g.cache == kKvE4m3 ? 1 : 2), rate = 5.2e6;
  int64_t w = 0, n = 0;
  for (const Tile& t : wide) w += t.tiles;
  for (const Tile& t : narrow) n += t.tiles;
  int best = groups / 2;
  double least = 1e300;
  for (int k = kXcds; k <= groups - kXcds; k += kXcds) {
    const double tw = w * wt / k + std::ceil((double)wide.size() / k) * ws;
    const double tn = std::pow(std::pow(n * nt / ((groups - k) * kWideWaves), 6) + std::pow(n * nb / rate, 6), 1.0 / 6);
    if (std::max(tw, tn) < least) {
      least = std::max(tw, tn);
      best = k;
    }
  }
  return best;
}

bool type16(int32_t t) { return t == LAR_KV_F16 || t == LAR_KV_BF16; }

lar_status ready(lar_kv* kv) {
  if (!kv) return LAR_E_ARG;
  if (kv->sticky != LAR_OK) return kv->sticky;
  if (!kv->planned) return fail(kv, LAR_E_STATE, "no token batch planned (call lar_kv_plan)");
  return LAR_OK;
}

// The arguments that append, read and attend share.
lar_status check(lar_kv* kv, const lar_kv_pages* pages, const int32_t* table, int32_t cols, KvPool* pool) {
  if (lar_status st = ready(kv)) return st;
  if (!pages || !pages->k || !pages->v) return fail(kv, LAR_E_ARG, "null pages");
  if (!table) return fail(kv, LAR_E_ARG, "null block table");
  if (kv->g.cache == kKvE4m3 && (!pages->k_exp || !pages->v_exp))
    return fail(kv, LAR_E_ARG, "an e4m3 cache needs k_exp and v_exp");
  if (((uintptr_t)pages->k | (uintptr_t)pages->v) & 15)
    return fail(kv, LAR_E_ARG, "pages must be aligned to 16 bytes");
  if (pages->n_blocks < 1 ||
      pages->n_blocks > ((((int64_t)1 << 32) - 1) >> kv->g.sh) / kv->g.hkv)
    return fail(kv, LAR_E_ARG, "n_blocks must be in 1 .. (2^32 - 1) / (block_size * n_kv_heads)");
  if (cols < kv->max_pages)
    return fail(kv, LAR_E_ARG, "block table has %d columns, the planned contexts need %d", cols, kv->max_pages);
  *pool = KvPool{pages->k, pages->v, pages->k_exp, pages->v_exp, (uint32_t)pages->n_blocks};
  return LAR_OK;
}

// Rows [T][heads][head_dim] with 16-byte rows.  A stride between things of which there is one
// does not matter.
lar_status check_rows(lar_kv* kv, const lar_kv_rows* r, int heads, const char* name, KvRows* out) {
  if (!r || !r->data) return fail(kv, LAR_E_ARG, "null %s", name);
  if (((uintptr_t)r->data & 15) || (kv->n_tok > 1 && (r->tok_stride & 7)) || (heads > 1 && (r->head_stride & 7)))
    return fail(kv, LAR_E_ARG, "%s: every row must be aligned to 16 bytes", name);
  *out = KvRows{r->data, r->tok_stride, r->head_stride};
  return LAR_OK;
}

// Whether row (t, h) of some rows, at t * a + h * b, and row (t', h') of others with the same
// strides, `delta` further on, have a value in common; rows of D values, T x H of them.  `self`: they
// are the same rows, of which (t, h) = (t', h') does not count.
bool meet(int64_t a, int64_t b, int64_t T, int64_t H, int64_t D, int64_t delta, bool self) {
  for (int64_t h = self ? 0 : 1 - H; h < H; ++h) {
    const __int128 v = (__int128)h * b + delta;  // plus t * a, t = 1 - T .. T - 1: how near to 0?
    const __int128 best = a ? -v / a : 0;
    for (int i = -1; i <= 1; ++i) {
      const int64_t t = (int64_t)std::max<__int128>(1 - T, std::min<__int128>(T - 1, best + i));
      if (self && h == 0 && t == 0) continue;
      const __int128 gap = v + (__int128)t * a;
      if (gap < D && gap > -D) return true;
    }
  }
  return false;
}

// Rows that a call writes: none of them may share memory.
lar_status check_apart(lar_kv* kv, const KvRows& k, const KvRows& v) {
  const int64_t T = kv->n_tok, H = kv->g.hkv, D = kv->g.D;
  const bool rows = (H == 1 || k.head >= D) && (T == 1 || k.tok >= (H > 1 ? (H - 1) * k.head : 0) + D);
  const bool same = (H == 1 || k.head == v.head) && (T == 1 || k.tok == v.tok);
  const auto* kp = (const char*)k.p;
  const auto* vp = (const char*)v.p;
  const auto end = [&](const KvRows& r) { return (T - 1) * r.tok + (H - 1) * r.head + D; };
  const bool far = rows && same && (kp < vp ? (vp - kp) / 2 >= end(k) : (kp - vp) / 2 >= end(v));
  if (far) return LAR_OK;  // as tensors of their own are
  if (meet(k.tok, k.head, T, H, D, 0, true) || meet(v.tok, v.head, T, H, D, 0, true) || kp == vp ||
      (same && meet(k.tok, k.head, T, H, D, (vp - kp) / 2, false)))
    return fail(kv, LAR_E_ARG, "rows of k and v to be written share memory");
  return LAR_OK;
}

KvPlanId plan_id(const lar_kv* kv) { return KvPlanId{(const uint64_t*)kv->dev, kv->plan}; }

KvCopyArgs copy_args(const lar_kv* kv, const KvPool& pool, const int32_t* table, int32_t cols) {
  KvCopyArgs a{};
  a.plan = plan_id(kv);
  a.g = kv->g;
  a.pool = pool;
  a.table = table;
  a.cols = cols;
  a.n_tok = kv->n_tok;
  a.tok = (const KvTok*)(kv->dev + kv->lay.tok);
  a.err = kv->err;
  return a;
}

// A launch on the handle's device and stream.
template <class Args>
lar_status launch(lar_kv* kv, hipError_t (*f)(const Args&, hipStream_t), const Args& a) {
  const OnDevice device(kv);
  KV_TRY(kv, device.status());
  const hipError_t e = f(a, kv->stream);
  return e == hipSuccess ? LAR_OK : fail(kv, LAR_E_HIP, "launch: %s", hipGetErrorString(e));
}

void release(lar_kv* kv) {
  for (void* p : {(void*)kv->dev, (void*)kv->narrow_o, (void*)kv->wide_o, (void*)kv->narrow_ml,
                  (void*)kv->wide_ml, (void*)kv->err})
    if (p) (void)hipFree(p);
  for (int i = 0; i < kStages; ++i) {
    if (kv->pinned[i]) (void)hipHostFree(kv->pinned[i]);
    if (kv->done[i]) (void)hipEventDestroy(kv->done[i]);
  }
}

}  // namespace

extern "C" {

lar_status lar_kv_create(lar_kv** out, const lar_kv_config* cfg) {
  if (!out) return LAR_E_ARG;
  *out = nullptr;
  if (!cfg) return LAR_E_ARG;
  const int S = cfg->block_size;
  if (cfg->n_kv_heads < 1 || cfg->n_kv_heads > 1024 || cfg->n_q_heads < 1 ||
      cfg->n_q_heads % cfg->n_kv_heads || cfg->n_q_heads / cfg->n_kv_heads > 64 ||
      (cfg->head_dim != 64 && cfg->head_dim != 128) || !type16(cfg->dtype) ||
      (cfg->cache_dtype != cfg->dtype && cfg->cache_dtype != LAR_KV_E4M3) || S < 1 || S > 65536 ||
      (S & (S - 1)) || cfg->max_seqs < 1 || cfg->max_seqs > 1 << 20 || cfg->max_tokens < 1 ||
      cfg->max_tokens > 1 << 26 || (int64_t)cfg->max_tokens * cfg->n_kv_heads > 1 << 27 ||
      cfg->reserved != 0)
    return LAR_E_ARG;
  lar_kv* kv = new (std::nothrow) lar_kv;
  if (!kv) return LAR_E_HIP;
  kv->cfg = *cfg;
  kv->stream = static_cast<hipStream_t>(cfg->stream);
  KvGeom& g = kv->g;
  g.hq = cfg->n_q_heads;
  g.hkv = cfg->n_kv_heads;
  g.G = g.hq / g.hkv;
  g.D = cfg->head_dim;
  g.dtype = cfg->dtype;
  g.cache = cfg->cache_dtype;
  while ((1 << g.sh) < S) ++g.sh;
  if (hipGetDevice(&kv->device) != hipSuccess ||
      hipDeviceGetAttribute(&kv->cus, hipDeviceAttributeMultiprocessorCount, kv->device) != hipSuccess) {
    delete kv;
    return LAR_E_HIP;
  }
  kv->waves = kv->cus * narrow_per_cu(g);
  kv->groups = kv->cus;  // a CU holds one workgroup of the wide kernel
  // query tiles: a sequence of n tokens has ceil(n / tokens of a tile) of them per kv head
  const int64_t nt = kNarrowRows / g.G, wt = kWideRows / g.G;
  const int64_t narrow = std::min<int64_t>(cfg->max_seqs, cfg->max_tokens) * g.hkv;
  const int64_t wide = (std::min<int64_t>(cfg->max_seqs, cfg->max_tokens / (nt + 1)) + cfg->max_tokens / wt) * g.hkv;
  kv->cap = Layout(cfg->max_tokens, narrow + kv->waves, wide + narrow + 2 * kv->groups, kv->waves, kv->groups,
                   std::min<int64_t>(narrow, kv->waves) + std::min<int64_t>(wide + narrow, kv->groups) * (kWideRows / 32) + kJoins8).end;
  // every wave or workgroup has two stretches at most that are parts of a tile
  bool ok = hipMalloc((void**)&kv->dev, kv->cap) == hipSuccess &&
            hipMalloc((void**)&kv->narrow_o, sizeof(float) * 2 * kv->waves * kNarrowRows * g.D) == hipSuccess &&
            hipMalloc((void**)&kv->wide_o, sizeof(float) * 2 * kv->groups * kWideRows * g.D) == hipSuccess &&
            hipMalloc((void**)&kv->narrow_ml, sizeof(float4) * 2 * kv->waves * kNarrowRows) == hipSuccess &&
            hipMalloc((void**)&kv->wide_ml, sizeof(float4) * 2 * kv->groups * kWideRows) == hipSuccess &&
            hipMalloc((void**)&kv->err, sizeof(int32_t)) == hipSuccess &&
            hipMemset(kv->err, 0, sizeof(int32_t)) == hipSuccess;
  for (int i = 0; ok && i < kStages; ++i)
    ok = hipHostMalloc((void**)&kv->pinned[i], kv->cap, hipHostMallocDefault) == hipSuccess &&
         hipEventCreateWithFlags(&kv->done[i], hipEventDisableTiming) == hipSuccess;
  if (!ok) {
    release(kv);
    delete kv;
    return LAR_E_HIP;
  }
  *out = kv;
  return LAR_OK;
}

lar_status lar_kv_destroy(lar_kv* kv) {
  if (!kv) return LAR_OK;
  {
    const OnDevice device(kv);
    (void)hipStreamSynchronize(kv->stream);
    release(kv);
  }
  delete kv;
  return LAR_OK;
}

const char* lar_kv_error_string(const lar_kv* kv) { return kv ? kv->msg.c_str() : "null handle"; }

lar_status lar_kv_plan(lar_kv* kv, int32_t n_seqs, const int32_t* q_len, const int32_t* ctx_len,
                       int32_t window, int32_t sinks) {
  if (!kv) return LAR_E_ARG;
  if (n_seqs < 0 || n_seqs > kv->cfg.max_seqs)
    return fail(kv, LAR_E_ARG, "%d sequences, at most %d", n_seqs, kv->cfg.max_seqs);
  if (n_seqs && (!q_len || !ctx_len)) return fail(kv, LAR_E_ARG, "null lengths");
  if (window < 0 || sinks < 0) return fail(kv, LAR_E_ARG, "negative window or sinks");
  const OnDevice device(kv);
  KV_TRY(kv, device.status());
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (kv->stream) KV_TRY(kv, hipStreamIsCapturing(kv->stream, &capture));
  if (capture != hipStreamCaptureStatusNone) return fail(kv, LAR_E_STATE, "no plan under stream capture");
  int64_t T = 0, pages = 0;
  int32_t longest = 0;
  for (int s = 0; s < n_seqs; ++s) {
    if (q_len[s] < 0 || ctx_len[s] < 0 || ctx_len[s] > 1 << 30)
      return fail(kv, LAR_E_ARG, "sequence %d: %d new tokens, context %d", s, q_len[s], ctx_len[s]);
    T += q_len[s];
    if (q_len[s]) longest = std::max(longest, ctx_len[s]);
    if (q_len[s]) pages = std::max<int64_t>(pages, ceil_div(ctx_len[s], (int64_t)1 << kv->g.sh));
  }
  if (T > kv->cfg.max_tokens)
    return fail(kv, LAR_E_ARG, "%lld new tokens, at most %d", (long long)T, kv->cfg.max_tokens);
  // A window of every context hides nothing.  The kernels subtract a shorter one, and then a
  // key of a context, from a position: all within 2^30, so within 32 bits.
  if (window >= longest) window = 0;
  if (!window) sinks = 0;
  PlanId id;
  id.add((uint32_t)window, (uint32_t)sinks);
  for (int s = 0; s < n_seqs; ++s) id.add((uint32_t)q_len[s], (uint32_t)ctx_len[s]);
  // the copy that last left this buffer is done before it is written again
  const int b = kv->stage;
  if (kv->used[b]) KV_TRY(kv, hipEventSynchronize(kv->done[b]));
  char* p = kv->pinned[b];
  const KvGeom& g = kv->g;
  KvTok* tok = (KvTok*)(p + Layout().tok);
  int32_t n_narrow = 0, n_wide = 0, n_join = 0, join_rows = 0, most_parts = 0;
  kv->planned = false;
  try {
    std::vector<Tile> narrow, wide, none;
    const int nt = kNarrowRows / g.G, wt = kWideRows / g.G;
    int64_t q0 = 0;
    for (int s = 0; s < n_seqs; ++s) {
      const int n = q_len[s];
      const int64_t p0 = (int64_t)ctx_len[s] - n;
      for (int r = 0; r < n; ++r) tok[q0 + r] = KvTok{s, (int32_t)(p0 + r)};
      if (!n) continue;
      const bool small = n <= nt;
      const int per = small ? n : wt;
      for (int h = 0; h < g.hkv; ++h)
        for (int r = 0; r < n; r += per) {
          Tile t{};
          t.s.q0 = (int32_t)(q0 + r);
          t.s.ntok = std::min(per, n - r);
          t.s.p0 = (int32_t)(p0 + r);
          t.s.head = h;
          t.s.seq = s;
          t.tiles = key_tiles(p0 + r, t.s.ntok, small ? kNarrowKeys : kWideKeys, window, sinks, &t.s.ns, &t.s.fw);
          (t.tiles ? small ? narrow : wide : none).push_back(t);
        }
      q0 += n;
    }
    // tiles without keys have only their zeros to write: either kernel will do, if they fit
    for (const Tile& t : none) (t.s.ntok <= nt && wide.empty() ? narrow : wide).push_back(t);
    const int64_t nn = (int64_t)narrow.size(), nw = (int64_t)wide.size();
    const Layout L(T, nn ? nn + kv->waves : 0, nw ? nw + 2 * kv->groups : 0, kv->waves, kv->groups,
                   std::min<int64_t>(nn, kv->waves) + std::min<int64_t>(nw, kv->groups) * (kWideRows / 32) + kJoins8);
    if (L.end > kv->cap) return fail(kv, LAR_E_CAPACITY, "plan of %zu bytes, room for %zu", L.end, kv->cap);
    kv->lay = L;
    Joins join{g.G};
    const int groups = nn ? split(narrow, wide, kv->groups, g) : kv->groups;
    cut(narrow, nw ? (kv->groups - groups) * kWideWaves : kv->waves, narrow_least(narrow, g), (KvSeg*)(p + L.narrow),
        (int32_t*)(p + L.narrow_at), &n_narrow, &join);
    deal(wide, groups, g, (KvSeg*)(p + L.wide), (int32_t*)(p + L.wide_at), &n_wide, &join);
    n_join = join.write((KvJoin*)(p + L.join), &join_rows);
    most_parts = join.most;
  } catch (const std::bad_alloc&) {
    return fail(kv, LAR_E_CAPACITY, "out of host memory");
  }
  if (kv->sticky != LAR_OK) {  // an error that was reported ends with the batch it was in
    KV_TRY(kv, hipMemsetAsync(kv->err, 0, sizeof(int32_t), kv->stream));
    kv->sticky = LAR_OK;
  }
  if (T) {
    memcpy(p, &id.x, sizeof id.x);
    KV_TRY(kv, hipMemcpyAsync(kv->dev, p, kv->lay.end, hipMemcpyHostToDevice, kv->stream));
    KV_TRY(kv, hipEventRecord(kv->done[b], kv->stream));
    kv->used[b] = true;
    kv->stage = (b + 1) % kStages;
  }
  kv->n_seq = n_seqs;
  kv->n_tok = (int32_t)T;
  kv->max_pages = (int32_t)pages;
  kv->window = window;
  kv->sinks = sinks;
  kv->plan = id.x;
  kv->n_narrow = n_narrow;
  kv->n_wide = n_wide;
  kv->n_join = n_join;
  kv->join_rows = join_rows;
  kv->most_parts = most_parts;
  kv->planned = true;
  return LAR_OK;
}

lar_status lar_kv_append(lar_kv* kv, const lar_kv_pages* pages, const lar_kv_rows* k, const lar_kv_rows* v,
                         const int32_t* table, int32_t table_cols) {
  if (lar_status st = ready(kv)) return st;
  if (!kv->n_tok) return LAR_OK;
  KvPool pool;
  KvRows kr, vr;
  if (lar_status st = check(kv, pages, table, table_cols, &pool)) return st;
  if (lar_status st = check_rows(kv, k, kv->g.hkv, "k", &kr)) return st;
  if (lar_status st = check_rows(kv, v, kv->g.hkv, "v", &vr)) return st;
  KvCopyArgs a = copy_args(kv, pool, table, table_cols);
  a.k = kr;
  a.v = vr;
  return launch(kv, launch_kv_append, a);
}

lar_status lar_kv_read(lar_kv* kv, const lar_kv_pages* pages, const int32_t* table, int32_t table_cols,
                       const lar_kv_rows* k, const lar_kv_rows* v) {
  if (lar_status st = ready(kv)) return st;
  if (!kv->n_tok) return LAR_OK;
  KvPool pool;
  KvRows kr, vr;
  if (lar_status st = check(kv, pages, table, table_cols, &pool)) return st;
  if (lar_status st = check_rows(kv, k, kv->g.hkv, "k", &kr)) return st;
  if (lar_status st = check_rows(kv, v, kv->g.hkv, "v", &vr)) return st;
  KvCopyArgs a = copy_args(kv, pool, table, table_cols);
  if (lar_status st = check_apart(kv, kr, vr)) return st;
  a.k = kr;
  a.v = vr;
  return launch(kv, launch_kv_read, a);
}

lar_status lar_kv_attend(lar_kv* kv, const lar_kv_pages* pages, const lar_kv_rows* q, const int32_t* table,
                         int32_t table_cols, double scale, void* out, float* lse) {
  if (lar_status st = ready(kv)) return st;
  if (!kv->n_tok) return LAR_OK;
  KvPool pool;
  KvRows qr;
  if (lar_status st = check(kv, pages, table, table_cols, &pool)) return st;
  if (lar_status st = check_rows(kv, q, kv->g.hq, "q", &qr)) return st;
  if (!(scale > 0.0) || !(scale < 1e30)) return fail(kv, LAR_E_ARG, "scale must be positive and finite");
  if (!out || ((uintptr_t)out & 15)) return fail(kv, LAR_E_ARG, "out must be aligned to 16 bytes");
  KvAttendArgs a{};
  a.plan = plan_id(kv);
  a.g = kv->g;
  a.pool = pool;
  a.q = qr;
  a.table = table;
  a.cols = table_cols;
  // Not 0, which would make hidden scores -infinity * 0; scores under the smallest one are as equal.
  a.scale = std::max((float)(scale * 1.4426950408889634074), FLT_TRUE_MIN);
  a.window = kv->window;
  a.sinks = kv->sinks;
  a.out = out;
  a.lse = lse;
  a.narrow = (const KvSeg*)(kv->dev + kv->lay.narrow);
  a.wide = (const KvSeg*)(kv->dev + kv->lay.wide);
  a.narrow_at = (const int32_t*)(kv->dev + kv->lay.narrow_at);
  a.wide_at = (const int32_t*)(kv->dev + kv->lay.wide_at);
  a.n_narrow = kv->n_narrow;
  a.n_wide = kv->n_wide;
  a.join = (const KvJoin*)(kv->dev + kv->lay.join);
  a.n_join = kv->n_join;
  a.join_rows = kv->join_rows;
  a.most_parts = kv->most_parts;
  a.narrow_o = kv->narrow_o;
  a.wide_o = kv->wide_o;
  a.narrow_ml = kv->narrow_ml;
  a.wide_ml = kv->wide_ml;
  a.err = kv->err;
  return launch(kv, launch_kv_attend, a);
}

lar_status lar_kv_sync(lar_kv* kv) {
  if (!kv) return LAR_E_ARG;
  if (kv->sticky != LAR_OK) return kv->sticky;
  const OnDevice device(kv);
  KV_TRY(kv, device.status());
  int32_t e = 0;
  KV_TRY(kv, hipMemcpyAsync(&e, kv->err, sizeof e, hipMemcpyDeviceToHost, kv->stream));
  KV_TRY(kv, hipStreamSynchronize(kv->stream));
  if (e) {
    kv->sticky = LAR_E_STATE;
    return fail(kv, LAR_E_STATE, e == kKvLostPage ? "a block table names a page outside the pool"
                                                  : "a captured call ran under another plan than its own");
  }
  return LAR_OK;
}

}  // extern "C"
