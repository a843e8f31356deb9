// kv_cut.h -- contexts in stretches of kSelectStretch rows, a workgroup for each of a sequence and kv head.
#ifndef LAR_KV_CUT_H
#define LAR_KV_CUT_H

#include "kv_device.h"

namespace lar {

struct KvCut {
  int seq, head, k, cuts;  // stretch k of the sequence's `cuts`
  int64_t first;           // place of the head's stretches among all
};

// The last of n places, in ascending order from 0 on, that is b at most, by whole waves: 64 at a time, one
// load's latency for that many.
template <class Place>
__device__ __forceinline__ int last_to(int n, int b, Place place) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    const int c = __popcll(__ballot(i < n && place(lo + i) <= b));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The stretch of workgroup `b`; those of a sequence start behind those of the ones before it.
__device__ __forceinline__ KvCut kv_cut(const KvSpan* spans, int n_seq, int hkv, int b) {
  KvCut c;
  c.seq = last_to(n_seq, b, [&](int i) { return spans[i].cuts * hkv; });
  c.cuts = kv_select_cuts(spans[c.seq].ctx);
  const int start = spans[c.seq].cuts * hkv, at = b - start;
  c.head = at / c.cuts;
  c.k = at - c.head * c.cuts;
  c.first = (int64_t)start + (int64_t)c.head * c.cuts;
  return c;
}

}  // namespace lar

#endif  // LAR_KV_CUT_H
