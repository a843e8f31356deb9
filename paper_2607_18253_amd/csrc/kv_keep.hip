// kv_keep.hip -- rows of a key/value cache to the places that they keep.
//
// Row base + rows[i] of a sequence and kv head goes to place base + i: base is 0, or the first new
// token's position for a tree's path.  The rows ascend, so a row never goes up: of the rows that are
// moved one after the other none is written over before it is read, and of those that are moved at
// the same time all are read before one is written.  A workgroup walks over the list of one sequence
// and head in that order, with its share of the columns of K, or of V, or with the rows' exponents
// and weights.  Bound by the rows' bytes, read and written: 674 MB in 146 us, 4.6 TB/s, for 127 contexts.
#include "../../include/lar.h"
#include "kv_device.h"

namespace lar {
namespace {

struct Move {
  uint32_t from, to;  // rows of the pool
  bool on;
};

// What row i of the list is to do.
struct List {
  const KvKeepArgs& A;
  const int32_t *rows, *table, *to;
  int head, base, skip, limit;  // skip: padding rows before the first new token
  int n;                        // entries to look at: as many as can be right, and one that cannot
  bool bad = false, lost = false;
  __device__ __forceinline__ List(const KvKeepArgs& a, int seq, int h) : A(a), head(h) {
    const KvSpan s = A.spans[seq];
    base = A.fresh ? s.ctx - s.q_len : 0;
    skip = base < 0 ? -base : 0;
    limit = A.fresh ? s.q_len : s.ctx;
    n = min(A.n_rows, max(0, limit - skip) + 1);
    rows = A.rows + ((int64_t)seq * A.heads + (A.heads > 1 ? h : 0)) * A.n_rows;
    table = A.table + (int64_t)seq * A.cols;
    to = A.to + (int64_t)seq * A.to_cols;
  }
  __device__ __forceinline__ uint32_t row(int32_t page, int pos) {
    if ((uint32_t)page >= A.pool.n_blocks) {
      lost = true;
      return ~0u;
    }
    return (((uint32_t)page * (uint32_t)A.g.hkv + head) << A.g.sh) + (uint32_t)(pos & ((1 << A.g.sh) - 1));
  }
  // Rows i + k, i + step + k, .. of the list, `i` the same for all threads: all entries are asked for first,
  // then all pages.
  template <int U>
  __device__ __forceinline__ void moves(int i, int k, int step, Move (&m)[U]) {
    int r[U], before[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = -1;
      if (i + u * step >= n) continue;
      const int at = min(i + u * step + k, n - 1);
      r[u] = rows[at];
      before[u] = rows[max(at - 1, 0)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u].on = false;
      if (i + u * step >= n) continue;
      const int at = i + u * step + k;
      if (at >= n || r[u] == -1) continue;  // the list has ended
      if (r[u] >= limit || r[u] < skip + at || (at && (r[u] <= before[u] || before[u] < 0))) {
        bad = true;
        continue;
      }
      m[u].from = (uint32_t)table[(base + r[u]) >> A.g.sh];
      m[u].to = (uint32_t)to[(base + skip + at) >> A.g.sh];
      m[u].on = true;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!m[u].on) continue;
      m[u].from = row((int32_t)m[u].from, base + r[u]);
      m[u].to = row((int32_t)m[u].to, base + skip + i + u * step + k);
      m[u].on = m[u].from != ~0u && m[u].to != ~0u && m[u].from != m[u].to;
    }
  }
};

// Whether a list goes on behind its end.  Of a list that is moved in one pass moves() sees it; in longer ones
// a pass that starts behind the end is not made.  Before the moves: behind them, from the end on, it takes
// the kernel from 56 registers to 70, which leave a CU room for one workgroup of 1024 (127 contexts to 777
// rows each 172 us instead of 146).
template <int THREADS>
__device__ __forceinline__ void look_behind(List& list) {
  for (int i = threadIdx.x + 1; i < list.n; i += THREADS)
    list.bad |= list.rows[i] != -1 && list.rows[i - 1] == -1;
}

// What was loaded has arrived before what follows: a barrier alone waits for no loads.
template <int U>
__device__ __forceinline__ void read(uint4 (&x)[U]) {
#pragma unroll
  for (int u = 0; u < U; ++u) asm volatile("" : "+v"(x[u].x), "+v"(x[u].y), "+v"(x[u].z), "+v"(x[u].w));
}

// Past the caches: what has been moved is read by a later call.
__device__ __forceinline__ void put(char* to, const uint4& x) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  __builtin_nontemporal_store(u32x4{x.x, x.y, x.z, x.w}, (u32x4*)to);
}

// The columns of 16 bytes from `col` on, `cols` of them, of the list's rows.
template <int THREADS, int U>
__device__ __forceinline__ void move_rows(List& list, char* pool, int row_bytes, int col, int cols) {
  const int c = col + threadIdx.x % cols, r = threadIdx.x / cols, step = THREADS / cols;
  Move m[U], next[U];
  list.moves(0, r, step, m);
  for (int i0 = 0; i0 < list.n; i0 += step * U) {
    uint4 x[U] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (m[u].on) x[u] = *(const uint4*)(pool + (uint64_t)m[u].from * row_bytes + c * 16);
    // the rows after these are looked up while these are on their way
    const int i1 = i0 + step * U;
    const bool more = i1 < list.n && list.rows[i1] != -1;  // the same for all
    if (more) list.moves(i1, r, step, next);
    read(x);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (m[u].on) put(pool + (uint64_t)m[u].to * row_bytes + c * 16, x[u]);
    if (!more) break;
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = next[u];
  }
}

template <int THREADS>
__device__ __forceinline__ void move_marks(List& list) {
  const KvKeepArgs& A = list.A;
  const bool f8 = A.g.cache == kKvE4m3;
  uint8_t *ke = (uint8_t*)A.pool.ke, *ve = (uint8_t*)A.pool.ve;
  for (int i0 = 0; i0 < list.n; i0 += THREADS) {
    if (i0 && list.rows[i0] == -1) break;
    Move one[1];
    list.moves(i0, threadIdx.x, THREADS, one);
    const Move m = one[0];
    uint8_t a = 0, b = 0;
    float w = 0.0f;
    if (m.on) {
      if (f8) a = ke[m.from], b = ve[m.from];
      if (A.weights) w = A.weights[m.from];
    }
    uint4 x[1] = {make_uint4(a, b, __float_as_uint(w), 0)};
    read(x);
    __syncthreads();
    if (m.on) {
      if (f8) ke[m.to] = (uint8_t)x[0].x, ve[m.to] = (uint8_t)x[0].y;
      if (A.weights) A.weights[m.to] = __uint_as_float(x[0].z);
    }
  }
}

constexpr int kAtOnce = 4;  // rows that a thread moves at once

// Jobs of a sequence and head: the shares of K, those of V, the marks.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_keep(KvKeepArgs A, int shares, int jobs) {
  const int job = blockIdx.x % jobs, x = blockIdx.x / jobs;
  if (*A.plan.now != A.plan.id) {
    if (threadIdx.x == 0) *A.err = kKvOtherPlan;
    return;
  }
  List list(A, x / A.g.hkv, x % A.g.hkv);
  if (job < 2 * shares) {
    const int bytes = A.g.D * (A.g.cache == kKvE4m3 ? 1 : 2), cols = bytes / 16 / shares;
    if (job == 0 && list.n > THREADS / cols * kAtOnce) look_behind<THREADS>(list);
    move_rows<THREADS, kAtOnce>(list, (char*)(job < shares ? A.pool.k : A.pool.v), bytes, job % shares * cols, cols);
  } else {
    move_marks<THREADS>(list);
  }
  if (list.lost) *A.err = kKvLostPage;
  if (list.bad) *A.err = kKvBadRows;
}

}  // namespace

hipError_t launch_kv_keep(const KvKeepArgs& a, hipStream_t stream) {
  const KvKeepShape s(a.g, a.n_seq, a.n_rows, a.weights != nullptr);
  if (s.threads == 256)
    k_kv_keep<256><<<s.groups, 256, 0, stream>>>(a, s.shares, s.jobs);
  else
    k_kv_keep<1024><<<s.groups, 1024, 0, stream>>>(a, s.shares, s.jobs);
  return hipGetLastError();
}

}  // namespace lar
