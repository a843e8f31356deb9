// kv_weigh.hip -- how much of the attention each row of a key/value cache got.
//
// For key j of a sequence and kv head, over the batch's query rows r of the heads of its group that
// see it,
//     after_j = before_j + sum_r exp(s_rj - lse_r),   s_rj = scale * q_r . k_j,
// with the lse of the attention, so that one pass over K will do; new tokens have before_j = 0.
//
// S = Q K^T by 32x32x16 matrix instructions: a key is a column, held by lanes n and n + 32, and its
// sum over 32 rows is a lane's own.  K goes from the pages into the instructions' registers.
//
//   k_kv_weigh_narrow  the plan's narrow stretches (single tokens, short chunks): a wave has its keys
//                      to itself.  Bound by the bytes of K.
//   k_kv_weigh_wide    chunks: a wave keeps 32 keys and walks over the rows.
//   k_kv_weigh_copy    the sums that no row of the batch adds to, from `before`.
#include "../../include/lar.h"
#include "kv_attend.h"

namespace lar {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ bool other(const KvWeighArgs& A) {
  if (plan_at(A.plan.now, 0) == A.plan.id) return false;
  *A.err = kKvOtherPlan;
  return true;
}

// Row of key j in the pool, of a page that the table names; for a page outside, row 0 of page 0
// with `lost`.
__device__ __forceinline__ uint32_t pool_row(const KvWeighArgs& A, int32_t page, int head, int j, bool& lost) {
  lost = (uint32_t)page >= A.pool.n_blocks;
  return (lost ? 0u : (uint32_t)page) * ((uint32_t)A.g.hkv << A.g.sh) + ((uint32_t)head << A.g.sh) +
         (uint32_t)(j & ((1 << A.g.sh) - 1));
}

// The values of a step t of 16 that half h of a lane has: in memory's order with 8-bit rows, where
// 16 bytes are two steps.
template <bool F8>
__device__ __forceinline__ constexpr int part_of(int t, int h) {
  return F8 ? (2 * (t >> 1) + h) * 16 + (t & 1) * 8 : 16 * t + 8 * h;
}

// K of 32 keys on its way: a lane's share of its key's row.
template <bool BF, bool F8, int D>
struct Keys {
  static constexpr int I = F8 ? D / 32 : D / 16;
  uint4 x[I];
  uint32_t e;
  __device__ __forceinline__ void load(const KvWeighArgs& A, uint32_t row, int h) {
    const char* p = (const char*)A.pool.k + (uint64_t)row * (F8 ? D : 2 * D) + 16 * h;
#pragma unroll
    for (int i = 0; i < I; ++i) x[i] = *(const uint4*)(p + 32 * i);
    e = F8 ? A.pool.ke[row] : 0;
  }
  __device__ __forceinline__ s16x8 part(int t) const {
    using St = Stage<BF, F8, D, 1, 64>;
    return __builtin_bit_cast(s16x8, F8 ? St::widen(x[t >> 1], scale_of(e), t & 1) : x[t]);
  }
};

// 32 query rows: their values, and of the 16 that a lane sums over the log of the sums (log2 units)
// and whether they count.
template <bool F8, int D>
struct Rows {
  s16x8 q[D / 16];
  float l[16];
  uint32_t on;
  // rows `at` .. of the `n` of a kv head (token * G + head of the group), the first token q0
  __device__ __forceinline__ void load(const KvWeighArgs& A, int q0, int head, int at, int n, int lane) {
    const int r = at + (lane & 31), h = lane >> 5, G = A.g.G;
    const int t = r / G, g = r - t * G;
    const int16_t* p = (const int16_t*)A.q.p + (int64_t)(q0 + t) * A.q.tok + (int64_t)(head * G + g) * A.q.head;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      s16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
      if (r < n) z = *(const s16x8*)(p + part_of<F8>(i, h));
      q[i] = z;
    }
    on = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int y = at + key_of(i, h), u = y / G;
      const float z = y < n ? A.lse[(int64_t)(q0 + u) * A.g.hq + head * G + y - u * G] : -__builtin_inff();
      on |= (z != -__builtin_inff() ? 1u : 0u) << i;
      l[i] = z * kLog2e;
    }
  }
};

// Bits of a lane's 16 rows from row `at` on that see key j; rows are tokens from position p0 on.
__device__ __forceinline__ uint32_t seeing(const KvWeighArgs& A, int p0, int at, int h, int j) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int pos = p0 + (at + key_of(i, h)) / A.g.G;
    const bool in = j <= pos && (!A.window || j > pos - A.window || j < A.sinks);
    m |= (in ? 1u : 0u) << i;
  }
  return m;
}

// The weights of a lane's key over the 16 rows in `on`.
template <bool BF, bool F8, int D>
__device__ __forceinline__ float add_up(const Keys<BF, F8, D>& k, const Rows<F8, D>& r, uint32_t on, float c) {
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
  for (int t = 0; t < D / 16; ++t) s = Elem<BF>::mma(r.q[t], k.part(t), s);
  float sum = 0.0f;
  if (__all(on == 0xffffu)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -r.l[i]));
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      sum += on >> i & 1 ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -r.l[i])) : 0.0f;
  }
  return sum;
}

// The key's sum to its place.
__device__ __forceinline__ void put(const KvWeighArgs& A, uint32_t row, bool fresh, float x) {
  A.after[row] = (fresh ? 0.0f : A.before[row]) + x;
}

template <bool BF, bool F8, int D>
__global__ __launch_bounds__(64, 2) void k_kv_weigh_narrow(KvWeighArgs A) {
  const int lane = threadIdx.x, n = lane & 31, h = lane >> 5;
  const int run = run_of(blockIdx.x, A.n_narrow);
  int e = plan_at(A.narrow_at, run + 1), x = plan_at(A.narrow_at, run);
  if (other(A)) e = x;  // nothing to do
  bool any = false;     // a page outside the pool
  for (; x < e; ++x) {
    const KvSeg s = plan_at(A.narrow, x);
    if (s.t0 >= s.t1) continue;
    const int last = s.p0 + s.ntok - 1;  // a narrow tile has all new tokens of its sequence
    const int32_t* table = A.table + (int64_t)s.seq * A.cols;
    const auto look = [&](int t) {
      const int j = tile_key<kNarrowKeys>(s, t) + n;
      return table[(j < last ? j : last) >> A.g.sh];
    };
    Rows<F8, D> rows;
    rows.load(A, s.q0, s.head, 0, s.ntok * A.g.G, lane);
    Keys<BF, F8, D> next;
    bool lost;
    uint32_t row = pool_row(A, look(s.t0), s.head, tile_key<kNarrowKeys>(s, s.t0) + n, lost);
    next.load(A, row, h);
    int32_t page = look(s.t0 + 1 < s.t1 ? s.t0 + 1 : s.t0);
    for (int t = s.t0; t < s.t1; ++t) {
      const Keys<BF, F8, D> k = next;
      const uint32_t at = row;
      const bool gone = lost;
      const int kb = tile_key<kNarrowKeys>(s, t), j = kb + n;
      if (t + 1 < s.t1) {
        row = pool_row(A, page, s.head, tile_key<kNarrowKeys>(s, t + 1) + n, lost);
        next.load(A, row, h);
        if (t + 2 < s.t1) page = look(t + 2);
      }
      const bool masked = kb + kNarrowKeys - 1 > s.p0 || (A.window && kb <= last - A.window && kb + kNarrowKeys > A.sinks);
      const uint32_t on = masked ? rows.on & seeing(A, s.p0, 0, h, j) : rows.on;
      const float sum = add_halves(add_up<BF, F8, D>(k, rows, on, A.scale));
      any |= gone && j <= last;
      if (h == 0 && j <= last && !gone) put(A, at, j >= s.p0, sum);
    }
  }
  if (any) *A.err = kKvLostPage;
}

// One workgroup per kWeighKeys keys of a sequence and kv head, a wave per 32 of them.
template <bool BF, bool F8, int D>
__global__ __launch_bounds__(2 * kWeighKeys, 2) void k_kv_weigh_wide(KvWeighArgs A) {
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % A.g.hkv, block = blockIdx.x / A.g.hkv;
  if (other(A)) return;
  // the last sequence that starts at or before this block: those of its start before it have none
  int lo = 0, hi = A.n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (plan_at(A.spans, mid).blocks <= block) lo = mid; else hi = mid;
  }
  const KvSpan s = plan_at(A.spans, lo);
  const int kb = (block - s.blocks) * kWeighKeys + wave * 32, base = s.ctx - s.q_len, G = A.g.G;
  if (kb >= s.ctx) return;
  const int j = kb + n, last = s.ctx - 1;
  bool lost;
  const uint32_t row = pool_row(A, A.table[(int64_t)lo * A.cols + ((j < last ? j : last) >> A.g.sh)], head, j, lost);
  Keys<BF, F8, D> k;
  k.load(A, row, h);
  // tokens that see some of the keys, from the first one's on
  int t0 = kb > base ? kb - base : 0, t1 = s.q_len;
  if (base + t0 < 0) t0 = -base;
  if (A.window && kb >= A.sinks) t1 = min(t1, A.window + (kb - base + 31));
  float sum = 0.0f;
  for (int at = t0 * G; at < t1 * G; at += 32) {
    Rows<F8, D> rows;
    rows.load(A, s.q0, head, at, t1 * G, lane);
    const int p = base + at / G, q = base + (at + 31) / G;
    const bool masked = kb + 31 > p || (A.window && kb <= q - A.window && kb + 32 > A.sinks);
    const uint32_t on = masked ? rows.on & seeing(A, base, at, h, j) : rows.on;
    sum += add_up<BF, F8, D>(k, rows, on, A.scale);
  }
  sum = add_halves(sum);
  if (j > last || h) return;
  if (lost)
    *A.err = kKvLostPage;
  else
    put(A, row, j >= base, sum);
}

// `before` to `after` for the context of the sequences with new tokens, one workgroup for each
// sequence and kv head.
__global__ __launch_bounds__(256) void k_kv_weigh_copy(KvWeighArgs A) {
  const int seq = blockIdx.x / A.g.hkv, head = blockIdx.x % A.g.hkv;
  if (other(A)) return;
  const KvSpan s = plan_at(A.spans, seq);
  if (s.q_len == 0) return;
  for (int j = threadIdx.x; j < s.ctx - s.q_len; j += 256) {
    bool lost;
    const uint32_t row = pool_row(A, A.table[(int64_t)seq * A.cols + (j >> A.g.sh)], head, j, lost);
    if (lost)
      *A.err = kKvLostPage;
    else
      A.after[row] = A.before[row];
  }
}

template <bool BF, bool F8, int D>
hipError_t run(const KvWeighArgs& a, hipStream_t stream) {
  if (a.window && a.before != a.after) k_kv_weigh_copy<<<a.n_seq * a.g.hkv, 256, 0, stream>>>(a);
  if (a.n_narrow) k_kv_weigh_narrow<BF, F8, D><<<a.n_narrow, 64, 0, stream>>>(a);
  if (a.n_wide) k_kv_weigh_wide<BF, F8, D><<<a.n_wide * a.g.hkv, 2 * kWeighKeys, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool BF, bool F8>
hipError_t run_d(const KvWeighArgs& a, hipStream_t stream) {
  return a.g.D == 128 ? run<BF, F8, 128>(a, stream) : run<BF, F8, 64>(a, stream);
}

}  // namespace

hipError_t launch_kv_weigh(const KvWeighArgs& a, hipStream_t stream) {
  const bool f8 = a.g.cache == kKvE4m3;
  if (a.g.dtype == kKvBf16) return f8 ? run_d<true, true>(a, stream) : run_d<true, false>(a, stream);
  return f8 ? run_d<false, true>(a, stream) : run_d<false, false>(a, stream);
}

}  // namespace lar
