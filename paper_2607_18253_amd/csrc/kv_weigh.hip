// kv_weigh.hip -- how much of the attention each row of a key/value cache got.
//
// For key j of a sequence and kv head, over the batch's query rows r of the heads of its group that
// see it,
//     after_j = before_j + sum_r exp(s_rj - lse_r),   s_rj = scale * q_r . k_j,
// with the lse of the attention, so that one pass over K will do; new tokens have before_j = 0.
//
// S = Q K^T by 32x32x16 matrix instructions: a key is a column, held by lanes n and n + 32, and its
// sum over 32 rows is a lane's own, in 32 bits, in an order that the plan fixes: results repeat bit for bit.
//
//   k_kv_weigh_narrow  the plan's narrow stretches (single tokens, short chunks): a wave has its keys
//                      to itself.
//   k_kv_weigh_wide    chunks: a wave keeps 32 or 64 keys that some row sees and walks over the rows.
//   k_kv_weigh_sum     the sums of workgroups that share the rows of a block of keys.
//   k_kv_weigh_copy    under a window, the sums that no row of the batch adds to, from `before`.
#include "../../include/lar.h"
#include "kv_attend.h"
#include "kv_cut.h"

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

// Whether some token sees key j of the context, the first one being at position `base`.  What none sees is
// looked at only where it shares a tile with what one does, and then its page may be gone.
__device__ __forceinline__ bool is_seen(const KvWeighArgs& A, int base, int j) {
  return !A.window || j > base - A.window || j < A.sinks;
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

// Bits of a lane's 16 rows that see key j; row i's token is at position pos(i).
template <class Pos>
__device__ __forceinline__ uint32_t seeing(const KvWeighArgs& A, int j, Pos pos) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int p = pos(i);
    const bool in = j <= p && (!A.window || j > p - A.window || j < A.sinks);
    m |= (in ? 1u : 0u) << i;
  }
  return m;
}

// Whether rows at positions p .. q may not see all the 32 keys from kb on.
__device__ __forceinline__ bool cuts(const KvWeighArgs& A, int p, int q, int kb) {
  return kb + 31 > p || (A.window && kb <= q - A.window && kb + 32 > A.sinks);
}

// The weights of a lane's key over 16 rows: scores s, the logs of the rows' sums (log2 units,
// negated), those of the rows that are `on`.
__device__ __forceinline__ float add_up(const f32x16& s, const float (&l)[16], uint32_t on, float c) {
  float sum = 0.0f;
  if (__all(on == 0xffffu)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, l[i]));
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      sum += on >> i & 1 ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, l[i])) : 0.0f;
  }
  return sum;
}

// The key's sum to its place.
__device__ __forceinline__ void put(const KvWeighArgs& A, uint32_t row, bool fresh, float x) {
  A.after[row] = (fresh ? 0.0f : A.before[row]) + x;
}

// Tiles that a wave has on their way: some 190 KB on a CU of eight.
constexpr int kRing = 3;

// A wave takes its tiles through LDS, where whole rows of a page arrive in wide loads (straight from the
// pages into the instructions' registers each load takes 32 bytes of 32 rows: 154 us), the keys' sums so
// far along with them.  Bound by the bytes of K: 255 tokens over 680 MB of it take 151 us, 4.5 TB/s; larger
// batches come to 5.0, with any number of tiles or waves.

template <bool BF, bool F8, int D>
__global__ __launch_bounds__(64, 2) void k_kv_weigh_narrow(KvWeighArgs A) {
  __shared__ __align__(16) char kt[kNarrowKeys * kRowK<D>];
  using St = Stage<BF, F8, D, kNarrowKeys * (F8 ? D / 16 : D / 8) / 64, 64>;
  constexpr int I = kNarrowKeys / St::kStep;
  const int lane = threadIdx.x, n = lane & 31, h = lane >> 5, G = A.g.G;
  const int r0 = lane / St::kChunks, c = lane % St::kChunks;
  const int run = run_of(blockIdx.x, A.n_narrow);
  int e = plan_at(A.narrow_at, run + 1), x = plan_at(A.narrow_at, run);
  if (other(A)) e = x;  // nothing to do
  bool any = false;     // a page outside the pool
  for (; x < e; ++x) {
    const KvSeg s = plan_at(A.narrow, x);
    if (s.t0 >= s.t1) continue;
    const int last = s.p0 + s.ntok - 1;  // a narrow tile has all new tokens of its sequence
    const int32_t* table = A.table + (int64_t)s.seq * A.cols;
    const auto key = [&](int t) { return tile_key<kNarrowKeys>(s, t < s.t1 ? t : s.t1 - 1) + n; };
    const auto look = [&](int t) {
      const int j = key(t);
      return table[(j < last ? j : last) >> A.g.sh];
    };
    s16x8 q[D / 16];
    float l[16];
    uint32_t rows = 0;
    {
      const int t = n / G, g = n - t * G;
      const int16_t* p = (const int16_t*)A.q.p + (int64_t)(s.q0 + t) * A.q.tok + (int64_t)(s.head * G + g) * A.q.head;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        s16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
        if (t < s.ntok) z = *(const s16x8*)(p + 16 * i + 8 * h);
        q[i] = z;
      }
      float z = -__builtin_inff();
      if (t < s.ntok) z = A.lse[(int64_t)(s.q0 + t) * A.g.hq + s.head * G + g];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = __shfl(z, key_of(i, h));
        rows |= (y != -__builtin_inff() ? 1u : 0u) << i;
        l[i] = -y * kLog2e;
      }
    }
    St st[kRing];
    uint32_t row[kRing], ex[kRing];  // pool row and exponent of this lane's key n
    bool lost[kRing];
    int32_t page[kRing];
    float old[kRing];                // asked for with the tile: a later load would wait for all tiles
    const auto fetch = [&](int u, int t) {  // past the last tile: that one again
      row[u] = pool_row(A, page[u], s.head, key(t), lost[u]);
#pragma unroll
      for (int i = 0; i < I; ++i)
        st[u].k[i] = St::load((const char*)A.pool.k, (uint32_t)__shfl((int)row[u], i * St::kStep + r0), c * 16);
      ex[u] = F8 ? A.pool.ke[row[u]] : 0;
      old[u] = A.before[row[u]];
    };
#pragma unroll
    for (int u = 0; u < kRing; ++u) page[u] = look(s.t0 + u);
#pragma unroll
    for (int u = 0; u < kRing; ++u) {
      fetch(u, s.t0 + u);
      page[u] = look(s.t0 + kRing + u);
    }
    for (int t0 = s.t0; t0 < s.t1; t0 += kRing) {
#pragma unroll
      for (int u = 0; u < kRing; ++u) {
        const int t = t0 + u;
        if (t >= s.t1) break;
        const int kb = tile_key<kNarrowKeys>(s, t), j = kb + n;
        const uint32_t at = row[u];
        const bool gone = lost[u];
        const float before = j < s.p0 ? old[u] : 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i)
          st[u].put_k(kt, i, i * St::kStep + r0, c, F8 ? scale_of((uint32_t)__shfl((int)ex[u], i * St::kStep + r0)) : 0.0f);
        fetch(u, t + kRing);
        page[u] = look(t + 2 * kRing);
        wave_order();
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) sc = Elem<BF>::mma(q[i], k_part<D>(kt, i, lane), sc);
        uint32_t on = rows;
        if (cuts(A, s.p0, last, kb)) {
          const int half = here(h);  // nothing of this is made before: registers
          on &= seeing(A, j, [&](int i) { return s.p0 + key_of(i, half) / G; });
        }
        const float sum = add_halves(add_up(sc, l, on, A.scale));
        any |= gone && j <= last && is_seen(A, s.p0, j);
        if (h == 0 && j <= last && !gone) A.after[at] = before + sum;
        wave_order();
      }
    }
  }
  if (any) *A.err = kKvLostPage;
}

// A row of a kv head as token and head of the group, and the row 32 further on.
struct Place {
  int t, g;
  static __device__ __forceinline__ Place of(int row, int G) { return Place{row / G, row % G}; }
  __device__ __forceinline__ void next(int G, int step, int rest) {
    t += step;
    g += rest;
    if (g >= G) {
      g -= G;
      ++t;
    }
  }
};

// The sequence of block b of keys: the last that starts at or before it, for those of its start before it
// have no blocks.
__device__ __forceinline__ int wide_seq(const KvWeighArgs& A, int b) {
  return last_to(A.n_seq, b, [&](int i) { return A.spans[i].blocks; });
}

// Token of a row that adds nothing: less any key, with any base, it is a negative number of 32 bits (the
// base less a key is -2^26 - kWeighKeys to 2^30).
constexpr int kNoToken = -(3 << 29);

// One workgroup per kWeighKeys keys of a sequence and kv head, KF * 32 of them for a wave, whose
// part of K stays in its registers; 32 rows of Q at a time are in LDS for all waves.  The scores of the
// next rows run beside the exponentials of these, one for a weight at a quarter of the vector unit's rate;
// matrix and vector instructions fill the cycles between them.  2048 tokens of 32 heads over 49k keys of an e4m3
// cache: 793 us, 1020 TFLOP/s (one after the other 1273; 32 keys for a wave 1079).
template <bool BF, bool F8, int D, int KF>
__global__ __launch_bounds__(2 * kWeighKeys / KF, 2) void k_kv_weigh_wide(KvWeighArgs A) {
  constexpr int kThreads = 2 * kWeighKeys / KF, kChunks = D / 8, kStep = kThreads / kChunks;
  constexpr int I = (32 + kStep - 1) / kStep;  // loads of a thread for 32 rows
  struct alignas(16) Block {
    char q[32 * kRowK<D>];
    float l[32];
    int tok[32];  // kNoToken: the row adds nothing
    int all;      // no row is that
  };
  __shared__ Block block[3];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5, G = A.g.G;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x % A.g.hkv, bs = blockIdx.x / A.g.hkv, b = bs % A.n_wide, split = bs / A.n_wide;
  if (other(A)) return;
  const int lo = wide_seq(A, b);
  const KvSpan s = plan_at(A.spans, lo);
  const int base = s.ctx - s.q_len, last = s.ctx - 1;
  const int kb0 = KvSeenBlocks(base, A.window, A.sinks).key(b - s.blocks), kb = kb0 + wave * 32 * KF;
  // tokens that see some of the workgroup's keys; there is one, so t0 < t1 <= q_len, whose rows 32 bits count
  const KvSeers seers(base, s.q_len, A.window, A.sinks, kb0);
  const int t0 = seers.t0, t1 = seers.t1;
  // this workgroup's rows, from row `start` on in `blocks` blocks of 32
  const int step = 32 / G, rest = 32 % G, all_blocks = ((t1 - t0) * G + 31) / 32;
  const int start = t0 * G + 32 * (int)((int64_t)all_blocks * split / A.splits);
  const int blocks = (int)((int64_t)all_blocks * (split + 1) / A.splits) - (int)((int64_t)all_blocks * split / A.splits);
  // rows of Q: this thread's chunks of them, and for the first wave the log of a row's sum
  const int r0 = tid / kChunks, c = tid % kChunks;
  const bool loads = kStep <= 32 || r0 < 32;
  uint4 x[I];
  float z = 0.0f;
  Place at[I], mine = Place::of(start + n, G);
  const int16_t* from[I];
  const int64_t ahead = step * A.q.tok + rest * A.q.head, wrap = A.q.tok - G * A.q.head;
#pragma unroll
  for (int i = 0; i < I; ++i) {
    at[i] = Place::of(start + r0 + i * kStep, G);
    from[i] = (const int16_t*)A.q.p + (int64_t)(s.q0 + at[i].t) * A.q.tok + (int64_t)(head * G + at[i].g) * A.q.head + c * 8;
  }
  int z_tok = 0;
  int left = t1 * G - start;  // rows from the next block's first on
  const auto fetch = [&]() {
    if (rest == 0 && left >= 32) {  // whole blocks, of the same heads
#pragma unroll
      for (int i = 0; i < I; ++i) {
        if (kStep <= 32 || loads) x[i] = *(const uint4*)from[i];
        from[i] += ahead;
        at[i].t += step;
      }
    } else {
#pragma unroll
      for (int i = 0; i < I; ++i) {
        x[i] = make_uint4(0, 0, 0, 0);
        if (loads && at[i].t < t1) x[i] = *(const uint4*)from[i];
        const bool over = at[i].g + rest >= G;
        from[i] += ahead + (over ? wrap : 0);
        at[i].next(G, step, rest);
      }
    }
    left -= 32;
    if (wave == 0) {
      z = mine.t < t1 ? A.lse[(int64_t)(s.q0 + mine.t) * A.g.hq + head * G + mine.g] : -__builtin_inff();
      z_tok = mine.t;
      mine.next(G, step, rest);
    }
  };
  const auto store = [&](Block& to) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (loads) *(uint4*)(to.q + (r0 + i * kStep) * kRowK<D> + c * 16) = x[i];
    if (wave == 0) {
      const bool on = z != -__builtin_inff();
      const int all = __all(on);
      if (h == 0) {
        to.l[n] = -z * kLog2e;
        to.tok[n] = on ? z_tok : kNoToken;
      }
      if (lane == 0) to.all = all;
    }
  };
  s16x8 k[KF][D / 16];
  uint32_t row[KF];
  bool lost[KF];
  float sum[KF];
#pragma unroll
  for (int f = 0; f < KF; ++f) {
    const int j = kb + 32 * f + n;
    row[f] = pool_row(A, A.table[(int64_t)lo * A.cols + ((j < last ? j : last) >> A.g.sh)], head, j, lost[f]);
    Keys<BF, F8, D> y;
    y.load(A, row[f], h);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) k[f][t] = y.part(t);
    sum[f] = 0.0f;
  }
  Place first = Place::of(start, G), final = Place::of(start + 31, G);  // rows of a block
  const auto part = [&](const Block& q, int t) {
    return *(const s16x8*)(q.q + n * kRowK<D> + part_of<F8>(t, h) * 2);
  };
  const auto score = [&](const Block& q, f32x16 (&sc)[KF]) {
#pragma unroll
    for (int f = 0; f < KF; ++f)
#pragma unroll
      for (int y = 0; y < 16; ++y) sc[f][y] = 0.0f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      const s16x8 p = part(q, t);
#pragma unroll
      for (int f = 0; f < KF; ++f) sc[f] = Elem<BF>::mma(p, k[f][t], sc[f]);
    }
  };
  fetch();
  store(block[0]);
  fetch();
  store(block[1]);
  fetch();
  lds_barrier();
  const bool works = kb <= last && blocks > 0;
  f32x16 sa[KF], sb[KF];
  if (works) score(block[0], sa);
  int b0 = 0, b1 = 1, b2 = 2;
  // one block: the scores of the next rows, `next`, beside the exponentials of these, `sc`
  const auto go = [&](f32x16 (&sc)[KF], f32x16 (&next)[KF]) {
    store(block[b2]);
    fetch();
    if (works) {
      const Block &q = block[b0], &qn = block[b1];
      const int p0 = base + first.t, p1 = base + final.t;
      float l[16];
#pragma unroll
      for (int y = 0; y < 16; y += 4) {
        const f32x4 v = *(const f32x4*)(q.l + key_of(y, h));
#pragma unroll
        for (int w = 0; w < 4; ++w) l[y + w] = v[w];
      }
      const bool all = __builtin_amdgcn_readfirstlane(q.all);
      if (all && !cuts(A, p0, p1, kb + 32 * (KF - 1)) && !cuts(A, p0, p1, kb)) {
        float add[KF];
        s16x8 p[kAhead];
#pragma unroll
        for (int t = 0; t < kAhead; ++t) p[t] = part(qn, t);
#pragma unroll
        for (int f = 0; f < KF; ++f) {
          add[f] = 0.0f;
#pragma unroll
          for (int y = 0; y < 16; ++y) next[f][y] = 0.0f;
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
          constexpr int kExps = 16 / (D / 16);
#pragma unroll
          for (int f = 0; f < KF; ++f) next[f] = Elem<BF>::mma(p[t % kAhead], k[f][t], next[f]);
          if (t + kAhead < D / 16) p[t % kAhead] = part(qn, t + kAhead);
#pragma unroll
          for (int f = 0; f < KF; ++f) {
#pragma unroll
            for (int y = t * kExps; y < (t + 1) * kExps; ++y)
              add[f] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[f][y], A.scale, l[y]));
            add[f] = here(add[f]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int f = 0; f < KF; ++f) sum[f] += add[f];
      } else {
        // a row sees key j if its position less j is in 0 .. the window: as unsigned numbers, one
        // comparison
#pragma unroll
        for (int f = 0; f < KF; ++f) {
          const int j = kb + 32 * f + n;
          const uint32_t most = A.window && j >= A.sinks ? (uint32_t)A.window : 0x80000000u;
          float add = 0.0f;
#pragma unroll
          for (int y = 0; y < 16; y += 4) {
            const auto tok = *(const __attribute__((ext_vector_type(4))) int*)(q.tok + key_of(y, h));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[f][y + i], A.scale, l[y + i]));
              add += (uint32_t)(base + tok[i] - j) < most ? v : 0.0f;
            }
          }
          sum[f] += add;
        }
        score(qn, next);
      }
    }
    first.next(G, step, rest);
    final.next(G, step, rest);
    const int z = b0;
    b0 = b1;
    b1 = b2;
    b2 = z;
    lds_barrier();
  };
  for (int i = 0; i < blocks; i += 2) {
    go(sa, sb);
    if (i + 1 < blocks) go(sb, sa);
  }
#pragma unroll
  for (int f = 0; f < KF; ++f) {
    const int j = kb + 32 * f + n;
    const float y = add_halves(sum[f]);
    if (j > last || h) continue;
    if (A.splits > 1)
      A.parts[(int64_t)blockIdx.x * kWeighKeys + j - kb0] = y;
    else if (!lost[f])
      put(A, row[f], j >= base, y);
    else if (is_seen(A, base, j))
      *A.err = kKvLostPage;
  }
}

// The sums of a block's keys over the workgroups that shared its rows, in their order.
__global__ __launch_bounds__(kWeighKeys) void k_kv_weigh_sum(KvWeighArgs A) {
  const int head = blockIdx.x % A.g.hkv, b = blockIdx.x / A.g.hkv;
  if (other(A)) return;
  const int seq = wide_seq(A, b);
  const KvSpan s = plan_at(A.spans, seq);
  const int base = s.ctx - s.q_len;
  const int j = KvSeenBlocks(base, A.window, A.sinks).key(b - s.blocks) + (int)threadIdx.x;
  if (j >= s.ctx) return;
  float y = 0.0f;
#pragma unroll 8
  for (int i = 0; i < A.splits; ++i) y += A.parts[((int64_t)i * gridDim.x + blockIdx.x) * kWeighKeys + threadIdx.x];
  bool lost;
  const uint32_t row = pool_row(A, A.table[(int64_t)seq * A.cols + (j >> A.g.sh)], head, j, lost);
  if (!lost)
    put(A, row, j >= base, y);
  else if (is_seen(A, base, j))
    *A.err = kKvLostPage;
}

// `before` to `after` for the context of the sequences with new tokens, a workgroup for a stretch.  A page
// outside the pool has no weights to carry over; where a token sees it, the other kernels report it.
__global__ __launch_bounds__(256) void k_kv_weigh_copy(KvWeighArgs A) {
  if (other(A)) return;
  const KvCut c = kv_cut(A.spans, A.n_seq, A.g.hkv, blockIdx.x);
  const KvSpan s = A.spans[c.seq];
  if (s.q_len == 0) return;
  const int end = s.ctx - s.q_len, j0 = c.k * kSelectStretch;
  if (j0 >= end) return;
  // all pages are looked up first, of rows past the end the last one's
  constexpr int kRows = kSelectStretch / 256;
  const auto key = [&](int i) { return min(j0 + i * 256 + (int)threadIdx.x, end - 1); };
  const int32_t* table = A.table + (int64_t)c.seq * A.cols;
  uint32_t row[kRows];
  float x[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) row[i] = (uint32_t)table[key(i) >> A.g.sh];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    bool lost;
    row[i] = pool_row(A, (int32_t)row[i], c.head, key(i), lost);
    x[i] = A.before[row[i]];
    if (lost || j0 + i * 256 + (int)threadIdx.x >= end) row[i] = ~0u;  // no row of a pool
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (row[i] != ~0u) A.after[row[i]] = x[i];
}

template <bool BF, bool F8, int D>
hipError_t run(const KvWeighArgs& a, hipStream_t stream) {
  if (a.window && a.before != a.after) k_kv_weigh_copy<<<a.cuts, 256, 0, stream>>>(a);
  if (a.n_narrow) k_kv_weigh_narrow<BF, F8, D><<<a.n_narrow, 64, 0, stream>>>(a);
  if (a.n_wide) {
    const int n = a.n_wide * a.g.hkv;
    // few workgroups: eight waves of 32 keys each
    if (n * a.splits > 256)
      k_kv_weigh_wide<BF, F8, D, 2><<<n * a.splits, kWeighKeys, 0, stream>>>(a);
    else
      k_kv_weigh_wide<BF, F8, D, 1><<<n * a.splits, 2 * kWeighKeys, 0, stream>>>(a);
    if (a.splits > 1) k_kv_weigh_sum<<<n, kWeighKeys, 0, stream>>>(a);
  }
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
