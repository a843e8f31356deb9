// kv_select.hip -- which rows of a context stay within a budget.
//
// Of a sequence's n rows and a kv head, the first F and the last L stay, and of those between the
// ones of the largest weights, of equal ones the lowest positions; all in ascending order.  A weight
// is taken as a 32-bit number that orders as it does (-0 as 0, NaN above all), and the smallest one
// to stay is found byte by byte from the top, by counting the values of a byte among the weights
// that agree with it so far.  The positions then come out in one more pass, by prefix sums over
// ballots.  One workgroup for each sequence and kv head.
#include "../../include/lar.h"
#include "kv_device.h"

namespace lar {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// A number that orders as the weight does.
__device__ __forceinline__ uint32_t order(float w) {
  const uint32_t b = __float_as_uint(w + 0.0f);  // -0 + 0 = 0
  return w != w ? 0xffffffffu : b >> 31 ? ~b : b | 0x80000000u;
}

__global__ __launch_bounds__(kThreads) void k_kv_select(KvSelectArgs A) {
  const int seq = blockIdx.x / A.g.hkv, head = blockIdx.x % A.g.hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ int count[256];
  __shared__ int found[2];            // the byte, and how many of it are wanted
  __shared__ int above[kWaves], same[kWaves];
  if (*A.plan.now != A.plan.id) {
    if (tid == 0) *A.err = kKvOtherPlan;
    return;
  }
  const KvSpan s = A.spans[seq];
  const int n = s.ctx, S = 1 << A.g.sh;
  int32_t* rows = A.rows + ((int64_t)seq * A.g.hkv + head) * A.budget;
  if (n <= A.budget) {
    for (int i = tid; i < A.budget; i += kThreads) rows[i] = i < n ? i : -1;
    return;
  }
  const int32_t* table = A.table + (int64_t)seq * A.cols;
  bool lost = false;
  const auto weight = [&](int j) {
    const int32_t page = table[j >> A.g.sh];
    if ((uint32_t)page >= A.n_blocks) {
      lost = true;
      return 0u;
    }
    return order(A.weights[((int64_t)page * A.g.hkv + head) * S + (j & (S - 1))]);
  };
  const int end = n - A.last;                          // first row of the last ones
  int want = A.budget - A.first - A.last;              // rows of those between
  uint32_t least = 0;
  for (int shift = 24; shift >= 0 && want; shift -= 8) {
    if (tid < 256) count[tid] = 0;
    __syncthreads();
    for (int j = A.first + tid; j < end; j += kThreads) {
      const uint32_t x = weight(j);
      if (shift == 24 || (x ^ least) >> (shift + 8) == 0) atomicAdd(&count[x >> shift & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int left = want, b = 255;
      while (count[b] < left) left -= count[b--];
      found[0] = b;
      found[1] = left;
    }
    __syncthreads();
    least |= (uint32_t)found[0] << shift;
    want = found[1];                                   // of those that are equal so far
  }
  // rows above the least, and of the equal ones the first `want`
  int out = 0, equal = 0;
  const bool some = A.budget > A.first + A.last;
  for (int j0 = 0; j0 < n; j0 += kThreads) {
    const int j = j0 + tid;
    bool is_above = false, is_same = false;
    if (j < n) {
      if (j < A.first || j >= end) {
        is_above = true;
      } else if (some) {
        const uint32_t x = weight(j);
        is_above = x > least;
        is_same = x == least;
      }
    }
    const uint64_t ma = __ballot(is_above), ms = __ballot(is_same);
    if (lane == 0) {
      above[wave] = __popcll(ma);
      same[wave] = __popcll(ms);
    }
    __syncthreads();
    int a = out, e = equal, all_a = 0, all_e = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) {
        a += above[w];
        e += same[w];
      }
      all_a += above[w];
      all_e += same[w];
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    a += __popcll(ma & below);                         // rows above the least before this one
    e += __popcll(ms & below);                         // equal ones
    if (is_above || (is_same && e < want)) rows[a + (e < want ? e : want)] = j;
    out += all_a;
    equal += all_e;
    __syncthreads();
  }
  if (lost) *A.err = kKvLostPage;
}

}  // namespace

hipError_t launch_kv_select(const KvSelectArgs& a, hipStream_t stream) {
  k_kv_select<<<a.n_seq * a.g.hkv, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace lar
