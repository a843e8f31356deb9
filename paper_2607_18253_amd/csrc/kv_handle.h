// kv_handle.h -- the handle of the paged key/value cache and what its entry points (kv_api.cpp,
// kv_rows_api.cpp) have in common: errors, the device, the checks of their arguments, launches.
#ifndef LAR_KV_HANDLE_H
#define LAR_KV_HANDLE_H

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <string>

#include "../../include/lar.h"
#include "kv_device.h"

namespace lar {

constexpr int kKvStages = 2;  // pinned copies of a plan: one may be on its way while the next is written

inline size_t up(size_t x) { return (x + 255) & ~size_t(255); }

// Byte offsets of a plan's arrays, the same on the host and on the device, after its number.
struct KvLayout {
  size_t tok = up(sizeof(uint64_t)), narrow = 0, wide = 0, narrow_at = 0, wide_at = 0, join = 0, spans = 0,
         trees = 0, end = 0;
  KvLayout() = default;
  KvLayout(int64_t n_tok, int64_t n_narrow, int64_t n_wide, int64_t waves, int64_t groups, int64_t n_join,
           int64_t n_seq, int64_t tree_words) {
    narrow = up(tok + sizeof(KvTok) * n_tok);
    wide = up(narrow + sizeof(KvSeg) * n_narrow);
    narrow_at = up(wide + sizeof(KvSeg) * n_wide);
    wide_at = up(narrow_at + sizeof(int32_t) * (waves + 1));
    join = up(wide_at + sizeof(int32_t) * (groups + 1));
    spans = up(join + sizeof(KvJoin) * n_join);
    trees = up(spans + sizeof(KvSpan) * n_seq);
    end = up(trees + sizeof(uint32_t) * tree_words);
  }
};

}  // namespace lar

struct lar_kv {
  lar_kv_config cfg{};
  lar::KvGeom g{};
  hipStream_t stream = nullptr;
  int device = 0, cus = 0;
  int waves = 0, groups = 0;  // of the narrow and the wide kernel at most
  size_t cap = 0;             // bytes of a plan at most
  lar::KvLayout lay;          // of the current plan
  char* dev = nullptr;
  char* pinned[lar::kKvStages] = {};
  hipEvent_t done[lar::kKvStages] = {};
  bool used[lar::kKvStages] = {};
  int stage = 0;
  float *narrow_o = nullptr, *wide_o = nullptr;
  float4 *narrow_ml = nullptr, *wide_ml = nullptr;
  int32_t* err = nullptr;
  // the plan
  bool planned = false;
  uint64_t plan = 0;  // its number
  int32_t n_seq = 0, n_tok = 0, window = 0, sinks = 0;
  int32_t max_pages = 0, all_pages = 0;  // of a context with new tokens, of any
  int32_t longest = 0;                   // context of any
  int64_t blocks = 0;                    // of kWeighKeys keys that are seen, of the sequences that take wide tiles
  int32_t most_new = 0;                  // new tokens of a sequence at most
  int64_t cuts = 0, rows = 0;            // stretches of kSelectStretch rows of all contexts; rows
  int32_t n_narrow = 0, n_wide = 0, n_join = 0, join_rows = 0, most_parts = 0;
  bool trees = false;
  lar_status sticky = LAR_OK;
  std::string msg;
};

namespace lar {

inline lar_status fail(lar_kv* kv, lar_status code, const char* fmt, ...) {
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

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline lar_status ready(lar_kv* kv) {
  if (!kv) return LAR_E_ARG;
  if (kv->sticky != LAR_OK) return kv->sticky;
  if (!kv->planned) return fail(kv, LAR_E_STATE, "no token batch planned (call lar_kv_plan)");
  return LAR_OK;
}

// The arguments that the calls on pages share.
inline lar_status check(lar_kv* kv, const lar_kv_pages* pages, const int32_t* table, int32_t cols, KvPool* pool) {
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
inline lar_status check_rows(lar_kv* kv, const lar_kv_rows* r, int heads, const char* name, KvRows* out) {
  if (!r || !r->data) return fail(kv, LAR_E_ARG, "null %s", name);
  if (((uintptr_t)r->data & 15) || (kv->n_tok > 1 && (r->tok_stride & 7)) || (heads > 1 && (r->head_stride & 7)))
    return fail(kv, LAR_E_ARG, "%s: every row must be aligned to 16 bytes", name);
  *out = KvRows{r->data, r->tok_stride, r->head_stride};
  return LAR_OK;
}

inline KvPlanId plan_id(const lar_kv* kv) { return KvPlanId{(const uint64_t*)kv->dev, kv->plan}; }

// A launch on the handle's device and stream.
template <class Args>
lar_status launch(lar_kv* kv, hipError_t (*f)(const Args&, hipStream_t), const Args& a) {
  const OnDevice device(kv);
  KV_TRY(kv, device.status());
  const hipError_t e = f(a, kv->stream);
  return e == hipSuccess ? LAR_OK : fail(kv, LAR_E_HIP, "launch: %s", hipGetErrorString(e));
}

}  // namespace lar

#endif  // LAR_KV_HANDLE_H
