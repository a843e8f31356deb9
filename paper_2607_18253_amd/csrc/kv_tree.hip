// kv_tree.hip -- attention of the sequences of a token batch that have trees of drafted tokens.
//
// A drafted token sees its sequence's context and, of the batch's new tokens, itself and those above
// it in its tree; the sums are those of any token (kv_attend.hip), and so are the numerics of chunks.
// Only key tiles that reach into the tree, or to a window's start, have rows that see different
// keys: there a row's 32 keys are the bits of a word of its record in the plan.
//
//   k_kv_tree  W = 1, 2, 4 or 8 waves, 32 rows each, over the same tiles of keys in LDS; eight waves
//              on a CU.  A tree of n tokens has n rows for each head of a group, 20 to 500: between
//              the single tokens, which the bytes bound, and the chunks, which the matrix
//              instructions do.  One workgroup's tile of all rows reads K and V once, and other
//              workgroups fill in while one waits for its tile.
#include "../../include/lar.h"
#include "kv_attend.h"

namespace lar {
namespace {

// The tree of a query tile's sequence.
struct Tree {
  int base;   // its first token's position
  int block;  // the first key block that bits are about
  int words, first;  // of a record, and the first one's first word
};

__device__ __forceinline__ Tree tree_of(const KvAttendArgs& A, const KvSeg& s) {
  const KvSpan q = plan_at(A.spans, s.seq);
  const int base = q.ctx - q.q_len;
  return Tree{base, (base > 0 ? base : 0) >> 5, q.words, q.tree};
}

// A row of it: what it sees of the keys before the bits' first block, and where its bits are.
struct TreeRow {
  int lo, sinks;
  const uint32_t* bits;  // of key block 0, if there were any
  bool none;             // a padding row: sees nothing
  __device__ __forceinline__ bool sees(const Tree& t, int j) const {
    if (none) return false;
    return j >> 5 < t.block ? j > lo || j < sinks : bits[j >> 5] >> (j & 31) & 1;
  }
};

// Token u of a query tile.
__device__ __forceinline__ TreeRow row_of(const KvAttendArgs& A, const KvSeg& s, const Tree& t, int u) {
  const int pos = s.p0 + u;
  const uint32_t* at = A.trees + (int64_t)t.first + (int64_t)(pos - t.base) * (t.words + 1);
  return TreeRow{A.window ? (int)at[0] - A.window : -1, A.sinks, at + 1 - t.block, pos < 0};
}

// Takes the scores of 32 keys from kb on that the row does not see to -infinity.
__device__ __forceinline__ void hide_of(f32x16& s, const Tree& t, const TreeRow& r, int kb, int h, int window) {
  const int block = kb >> 5;
  if (block < t.block) {
    if (!window) return;  // padding rows are the first of a tree without a context
    const int base = kb + 4 * h, lo = r.lo - base, sinks = r.sinks - base;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = key_of(i, 0);
      s[i] = j > lo || j < sinks ? s[i] : -__builtin_inff();
    }
    return;
  }
  const uint32_t up = block < t.block + t.words && !r.none ? r.bits[block] >> (4 * h) : 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = up >> key_of(i, 0) & 1 ? s[i] : -__builtin_inff();
}

// Adds what clean() took out of V in the stretch's masked tiles to the rows that see it, in the
// result or the partial sums that the wave has just written.
template <bool BF, bool F8, int D, int K>
__device__ __forceinline__ void spread_tree(const KvAttendArgs& A, const KvSeg& s, const Tree& tree, int lane,
                                            int row0, int rows, float* po) {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  const int last = s.p0 + s.ntok - 1, G = A.g.G;
  for (int t = s.t0; t < s.t1; ++t) {
    const int kb = tile_key<K>(s, t);
    if (!is_masked(A, tree.base - 1, last, kb, K)) continue;
    for (int j = kb; j < kb + K && j <= last; ++j) {
      bool lost = false;  // reported before
      const uint32_t row = page_at(A, A.table[(int64_t)s.seq * A.cols + (j >> A.g.sh)], lost) + in_page(A, s.head, j);
      for (int d = lane; d < D; d += 64) {
        float v;
        if (F8) {
          const uint32_t c = ((const uint8_t*)A.pool.v)[(int64_t)row * D + d];
          v = Elem<BF>::value((uint16_t)Elem<BF>::pair(c, scale_of(A.pool.ve[row]), false));
        } else {
          v = Elem<BF>::value(((const uint16_t*)A.pool.v)[(int64_t)row * D + d]);
        }
        if (__builtin_isfinite(v)) continue;
        for (int n = row0; n < row0 + 32 && n < s.ntok * G; ++n) {
          const int u = n / G;
          if (!row_of(A, s, tree, u).sees(tree, j)) continue;
          if (s.slot >= 0) {
            po[part_at<D>(s.slot, rows, s.ntok * G, n, d / 4) + d % 4] += v;
          } else {
            uint16_t* o = (uint16_t*)A.out + ((int64_t)(s.q0 + u) * A.g.hq + s.head * G + n - u * G) * D + d;
            *o = Elem<BF>::one(Elem<BF>::value(*o) + v);
          }
        }
      }
    }
  }
}

template <bool BF, bool F8, int D, int W>
__global__ __launch_bounds__(64 * W, 2) void k_kv_tree(KvAttendArgs A) {
  constexpr int K = W == 1 ? 32 : 64, kRows = 32 * W, kThreads = 64 * W;
  __shared__ __align__(16) char lds[kTileBytes<D, K>];
  static_assert(kRows * kRowK<D> <= kTileBytes<D, K> || W == 8, "a result in LDS");
  __shared__ __align__(16) char more[W == 8 ? kRows * kRowK<D> : 16];
  __shared__ int flag;
  char *const kt = lds, *const vt = lds + K * kRowK<D>;
  using St = Stage<BF, F8, D, (K * (F8 ? D / 16 : D / 8) + kThreads - 1) / kThreads, kThreads>;
  constexpr int I = (K + St::kStep - 1) / St::kStep;
  constexpr bool kAll = St::kStep <= K;  // else there are more threads than chunks
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r0 = tid / St::kChunks, c = tid % St::kChunks;
  const bool loads = kAll || r0 < K;
  const int run = run_of(blockIdx.x, A.n_tree);
  int e = plan_at(A.tree_at, run + 1);
  bool lost = false;  // a page outside the pool
  int x = plan_at(A.tree_at, run);
  if (other_plan(A)) e = x;  // nothing to do
  for (; x < e; ++x) {
    const KvSeg s = plan_at(A.tree, x);
    const Tree tree = tree_of(A, s);
    s16x8 q[D / 16];
    load_q<D>(A, lane_of(A, s, wave * 32 + n), h, q);
    Sums<D> a;
    a.clear();
    const int last = s.p0 + s.ntok - 1;  // position of the last token: keys 0 .. last
    const bool real = wave * 32 < s.ntok * A.g.G;
    const int32_t* table = A.table + (int64_t)s.seq * A.cols;
    const int last_col = last >> A.g.sh;
    // the page of key `lane` of a tile; its pool row; the loads of all rows
    const auto look = [&](int t) {
      const int col = (tile_key<K>(s, t) + (lane & (K - 1))) >> A.g.sh;
      return table[col < last_col ? col : last_col];
    };
    St st;
    uint32_t ex = 0;  // exponents of key `lane`: K, and V << 8
    const auto fetch = [&](int32_t page, int t) {
      const uint32_t src = page_at(A, page, lost) + in_page(A, s.head, tile_key<K>(s, t) + (lane & (K - 1)));
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const uint32_t at = (uint32_t)__shfl((int)src, (i * St::kStep + r0) & (K - 1));
        st.k[i] = St::load((const char*)A.pool.k, at, c * 16);
        st.v[i] = St::load((const char*)A.pool.v, at, c * 16);
      }
      if (F8) ex = A.pool.ke[src] | (uint32_t)A.pool.ve[src] << 8;
    };
    int32_t page = 0;
    if (s.t0 < s.t1) {
      fetch(look(s.t0), s.t0);
      if (s.t0 + 1 < s.t1) page = look(s.t0 + 1);
    }
    if (W > 1) {
      if (tid == 0) flag = 0;
      __syncthreads();
    }
    bool bad = false;
    for (int t = s.t0; t < s.t1; ++t) {
      const int kb = tile_key<K>(s, t);
      const bool masked = is_masked(A, tree.base - 1, last, kb, K);
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int r = i * St::kStep + r0;
        const uint32_t x = F8 ? (uint32_t)__shfl((int)ex, r & (K - 1)) : 0;
        if (!loads) continue;
        st.put_k(kt, i, r, c, scale_of(x));
        if (masked)
          bad |= st.template put_v<true>(vt, i, r, c, last + 1 - kb, scale_of(x >> 8));
        else
          st.template put_v<false>(vt, i, r, c, 0, scale_of(x >> 8));
      }
      if (t + 1 < s.t1) {
        fetch(page, t + 1);
        if (t + 2 < s.t1) page = look(t + 2);
      }
      if (W == 1) wave_order(); else lds_barrier();
      if (real) {
#pragma unroll 1  // registers
        for (int u = 0; u < K / 32; ++u) {
          f32x16 sc[1] = {scores<BF, D>(kt + 32 * u * kRowK<D>, q, n, h)};
          if (masked) {  // the row is looked up again: few tiles are, and registers are short
            const int at = lane_of(A, s, here(wave * 32 + n)).tok - s.q0;
            hide_of(sc[0], tree, row_of(A, s, tree, at), kb + 32 * u, h, A.window);
          }
          raise<BF, D>(a, peak<1>(sc) * A.scale);
          soften<D, 1>(sc, a, A.scale);
          weigh<BF, D, false>(vt + 32 * u * kRowV<D>, sc[0], a, lane);
        }
      }
      if (W == 1) wave_order(); else lds_barrier();
    }
    if (W > 1 && bad) flag = 1;
    finish<BF, D>(A, s, a, lane, wave * 32, kRows, A.narrow_o, A.narrow_ml, (W == 8 ? more : lds) + wave * 32 * kRowK<D>);
    if (W > 1) __syncthreads();  // the flag; and the result's place is free
    if (W > 1 ? flag != 0 : __any(bad)) spread_tree<BF, F8, D, K>(A, s, tree, lane, wave * 32, kRows, A.narrow_o);
    if (W > 1) __syncthreads();  // the flag is read
    if (W == 1) wave_order();
  }
  if (lost) *A.err = kKvLostPage;
}

template <bool BF, bool F8, int D>
void run(const KvAttendArgs& a, hipStream_t stream) {
  const int n = a.n_tree;
  switch (a.tree_waves) {
    case 1: k_kv_tree<BF, F8, D, 1><<<n, 64, 0, stream>>>(a); break;
    case 2: k_kv_tree<BF, F8, D, 2><<<n, 128, 0, stream>>>(a); break;
    case 4: k_kv_tree<BF, F8, D, 4><<<n, 256, 0, stream>>>(a); break;
    default: k_kv_tree<BF, F8, D, 8><<<n, 512, 0, stream>>>(a); break;
  }
}

template <bool BF, bool F8>
void run_d(const KvAttendArgs& a, hipStream_t stream) {
  a.g.D == 128 ? run<BF, F8, 128>(a, stream) : run<BF, F8, 64>(a, stream);
}

}  // namespace

hipError_t launch_kv_tree(const KvAttendArgs& a, hipStream_t stream) {
  const bool f8 = a.g.cache == kKvE4m3;
  if (a.g.dtype == kKvBf16)
    f8 ? run_d<true, true>(a, stream) : run_d<true, false>(a, stream);
  else
    f8 ? run_d<false, true>(a, stream) : run_d<false, false>(a, stream);
  if (const hipError_t e = hipGetLastError()) return e;
  KvAttendArgs j = a;
  j.join = a.tree_join;
  j.n_join = a.n_tree_join;
  j.join_rows = a.tree_join_rows;
  j.most_parts = a.tree_most_parts;
  j.wide_rows = 32 * a.tree_waves;
  j.wide_o = a.narrow_o;
  j.wide_ml = a.narrow_ml;
  return launch_kv_join(j, stream);
}

}  // namespace lar
