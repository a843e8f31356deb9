// kv_cut.h -- contexts in stretches of kSelectStretch rows, a workgroup for each of a sequence and kv head.
#ifndef LAR_KV_CUT_H
#define LAR_KV_CUT_H

#include "kv_device.h"

namespace lar {

struct KvCut {
  int seq, head, k, cuts;  // stretch k of the sequence's `cuts`
  int64_t first;           // place of the head's stretches among all
};

// The stretch of workgroup `b`.
__device__ __forceinline__ KvCut kv_cut(const KvSpan* spans, int n_seq, int hkv, int b) {
  int lo = 0, hi = n_seq;  // the last sequence whose stretches start at or before this one
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (spans[mid].cuts * hkv <= b) lo = mid; else hi = mid;
  }
  KvCut c;
  c.seq = lo;
  c.cuts = kv_select_cuts(spans[lo].ctx);
  const int start = spans[lo].cuts * hkv, at = b - start;
  c.head = at / c.cuts;
  c.k = at - c.head * c.cuts;
  c.first = (int64_t)start + (int64_t)c.head * c.cuts;
  return c;
}

}  // namespace lar

#endif  // LAR_KV_CUT_H
