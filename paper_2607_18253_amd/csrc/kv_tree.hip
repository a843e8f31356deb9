// kv_tree.hip -- attention of a token batch in which sequences have trees of drafted tokens.
//
// A drafted token sees its sequence's context and, of the batch's new tokens, itself and those above
// it in its tree; the sums are those of any token (kv_attend.hip), and so are the tiles, the numerics
// and the plan's stretches.  Only key tiles that reach into a tree, or to a window's start, have rows
// that see different keys: there a row's 32 keys are the bits of a word of its record in the plan.
// Sequences without a tree are in the same launch.
//
//   k_kv_tree_narrow  one wave per stretch of 32-key tiles, up to 32 rows: single tokens, small trees.
//   k_kv_tree_wide    eight waves, 256 rows, 64-key tiles: larger trees and chunks; and runs of narrow
//                     tiles, one for each wave, in the workgroups after them.
//
// A tree of n tokens has n rows for each head of a group, 20 to 500.  With few of them the bytes of K
// and V bound the wide kernel though most of its waves have no rows: all of them load (125 trees of 5 to 31
// tokens over 642 MB: 143 us with the join, 4.5 TB/s).  With many it is the wide kernel of ordinary batches
// (43 trees of 48 to 64 tokens, 64 heads, e4m3: 632 us, 820 TFLOP/s; as chains there 620).
#include "../../include/lar.h"
#include "kv_attend.h"

namespace lar {
namespace {

constexpr int kNoTree = INT32_MAX;

// The tree of a query tile's sequence.
struct Tree {
  int block;   // the first block of 32 keys that records have bits for, kNoTree without a tree
  int before;  // the last position that all its tokens follow
};

__device__ __forceinline__ Tree tree_of(const KvAttendArgs& A, const KvSeg& s) {
  const KvSpan q = plan_at(A.spans, s.seq);
  const int base = q.ctx - q.q_len;
  return Tree{q.tree < 0 ? kNoTree : (base > 0 ? base : 0) >> 5, base - 1};
}

// The last position up to which every row of a query tile sees all keys, but for a window.
__device__ __forceinline__ int all_to(const Tree& t, const KvSeg& s) { return t.block == kNoTree ? s.p0 : t.before; }

// A row, in one number: its token's position, or with a tree the word of its record's bits that is
// key block 0's, if it had one.
__device__ __forceinline__ int row_of(const KvAttendArgs& A, const KvSeg& s, int u) {
  const KvSpan q = plan_at(A.spans, s.seq);
  if (q.tree < 0) return s.p0 + u;
  const int base = q.ctx - q.q_len;
  return q.tree + (s.q0 + u - q.q0) * (q.words + 1) + 1 - ((base > 0 ? base : 0) >> 5);
}

// The place of its token among those that it follows; 0 for a tree's padding rows.
__device__ __forceinline__ int place_of(const KvAttendArgs& A, const Tree& t, int row) {
  return t.block == kNoTree ? row : (int)A.trees[row - 1 + t.block];
}

__device__ __forceinline__ bool sees(const KvAttendArgs& A, const Tree& t, int row, int j) {
  if (j >> 5 >= t.block) return A.trees[row + (j >> 5)] >> (j & 31) & 1;
  const int p = place_of(A, t, row);
  return j <= p && (!A.window || j > p - A.window || j < A.sinks);
}

// Takes the scores of 32 keys from kb on that the row does not see to -infinity.
__device__ __forceinline__ void hide_keys(const KvAttendArgs& A, f32x16& s, const Tree& t, int row, int kb, int h) {
  if (kb >> 5 >= t.block) {
    const uint32_t up = A.trees[row + (kb >> 5)] >> (4 * h);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = up >> key_of(i, 0) & 1 ? s[i] : -__builtin_inff();
    return;
  }
  const int base = kb + 4 * h, p = place_of(A, t, row) - base;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = key_of(i, 0) <= p ? s[i] : -__builtin_inff();
  if (!A.window) return;
  const int lo = p - A.window, sinks = A.sinks - base;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int j = key_of(i, 0);
    s[i] = j > lo || j < sinks ? s[i] : -__builtin_inff();
  }
}

// As spread() of ordinary batches: adds what clean() took out of V to the rows that see it.
template <bool BF, bool F8, int D, int K, bool ANY>
__device__ __forceinline__ void spread_tree(const KvAttendArgs& A, const KvSeg& s, int lane, int row0, int rows,
                                            float* po) {
  lane = here(lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  const int last = s.p0 + s.ntok - 1, G = A.g.G;
  const Tree tree = tree_of(A, s);
  for (int t = s.t0; t < s.t1; ++t) {
    const int kb = tile_key<K>(s, t);
    if (ANY ? !odd_tile<BF, D, K>(A, s, lane, kb, last) : !is_masked(A, all_to(tree, s), last, kb, K)) continue;
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
          if (!sees(A, tree, row_of(A, s, u), j)) continue;
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

// One wave's run of narrow stretches; `lds`: its tile of 32 keys.
template <bool BF, bool F8, int D>
__device__ __forceinline__ void narrow_run(const KvAttendArgs& A, char* lds, int run, int lane) {
  char *kt = lds, *vt = lds + kNarrowKeys * kRowK<D>;
  using St = Stage<BF, F8, D, kNarrowKeys * (F8 ? D / 16 : D / 8) / 64, 64>;
  constexpr int I = kNarrowKeys / St::kStep;
  const int n = lane & 31, h = lane >> 5;
  const int r0 = lane / St::kChunks, c = lane % St::kChunks;
  int e = plan_at(A.narrow_at, run + 1);
  bool lost = false;  // a page outside the pool
  int x = plan_at(A.narrow_at, run);
  if (other_plan(A)) e = x;  // nothing to do
  for (; x < e; ++x) {
    const KvSeg s = plan_at(A.narrow, x);
    const Tree tree = tree_of(A, s);
    s16x8 q[D / 16];
    load_q<D>(A, lane_of(A, s, n), h, q);
    Sums<D> a;
    a.clear();
    const int last = s.p0 + s.ntok - 1;  // position of the last token: keys 0 .. last
    const int32_t* table = A.table + (int64_t)s.seq * A.cols;
    const int last_col = last >> A.g.sh;
    const auto look = [&](int t) {
      const int col = (tile_key<kNarrowKeys>(s, t) + n) >> A.g.sh;
      return table[col < last_col ? col : last_col];
    };
    St st;
    uint32_t ex = 0;  // exponents of this lane's row n: K, and V << 8
    const auto fetch = [&](int32_t page, int t) {
      const uint32_t src = page_at(A, page, lost) + in_page(A, s.head, tile_key<kNarrowKeys>(s, t) + n);
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const uint32_t at = (uint32_t)__shfl((int)src, i * St::kStep + r0);
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
    bool bad = false;
    for (int t = s.t0; t < s.t1; ++t) {
      const int kb = tile_key<kNarrowKeys>(s, t);
      const bool masked = is_masked(A, all_to(tree, s), last, kb, kNarrowKeys);
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < I; ++i)
        if (!F8) m = max16(m, top_pair(st.v[i]));
      const bool odd = !F8 && __any(top_half(m) >= kInf<BF>);  // as in kv_attend.hip
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int r = i * St::kStep + r0;
        const uint32_t y = F8 ? (uint32_t)__shfl((int)ex, r) : 0;
        st.put_k(kt, i, r, c, scale_of(y));
        if (masked || odd)
          bad |= st.template put_v<true>(vt, i, r, c, last + 1 - kb, scale_of(y >> 8));
        else
          st.template put_v<false>(vt, i, r, c, 0, scale_of(y >> 8));
      }
      if (t + 1 < s.t1) {
        fetch(page, t + 1);
        if (t + 2 < s.t1) page = look(t + 2);
      }
      wave_order();
      f32x16 sc[1] = {scores<BF, D>(kt, q, n, h)};
      if (masked) hide_keys(A, sc[0], tree, row_of(A, s, lane_of(A, s, here(n)).tok - s.q0), kb, h);
      raise<BF, D>(a, peak<1>(sc) * A.scale);
      soften<D, 1>(sc, a, A.scale);
      weigh<BF, D, !F8>(vt, sc[0], a, lane);
      wave_order();
    }
    finish<BF, D>(A, s, a, lane, 0, kNarrowRows, A.narrow_o, A.narrow_ml, lds);
    wave_order();
    if (__any(bad)) spread_tree<BF, F8, D, kNarrowKeys, !F8>(A, s, lane, 0, kNarrowRows, A.narrow_o);
  }
  if (lost) *A.err = kKvLostPage;
}

template <bool BF, bool F8, int D>
__global__ __launch_bounds__(64, 2) void k_kv_tree_narrow(KvAttendArgs A) {
  __shared__ __align__(16) char lds[kTileBytes<D, kNarrowKeys>];
  narrow_run<BF, F8, D>(A, lds, run_of(blockIdx.x, A.n_narrow), threadIdx.x);
}

// Tile t's products run from K t and t + 1 and V t in LDS, while K t + 2 and V t + 1 are on their way
// there from registers and K t + 3 and V t + 2 on theirs from memory.  The numbers of the next
// stretch and the pages of its first tiles are asked for while the last tiles of this one are worked
// on, and its queries and first tiles before this one's result is written.
template <bool BF, bool F8, int D, bool LSE>
__global__ __launch_bounds__(64 * kWideWaves, 2) void k_kv_tree_wide(KvAttendArgs A) {
  constexpr int kTileK = kWideKeys * kRowK<D>, kTileV = kWideKeys * kRowV<D>, kThreads = 64 * kWideWaves;
  constexpr int kNarrow = kTileBytes<D, kNarrowKeys>, kWide = 3 * kTileK + 2 * kTileV;
  __shared__ __align__(16) char lds[kWide > kWideWaves * kNarrow ? kWide : kWideWaves * kNarrow];
  static_assert(kWideWaves * 32 * kRowK<D> <= kWide, "a result in LDS");
  char *const ldk = lds, *const ldv = lds + 3 * kTileK;
  __shared__ int flag;
  using St = Stage<BF, F8, D, (kWideKeys * (F8 ? D / 16 : D / 8) + kThreads - 1) / kThreads, kThreads>;
  constexpr int I = (kWideKeys + St::kStep - 1) / St::kStep;
  constexpr bool kAll = St::kStep <= kWideKeys;  // else 8-bit rows of 64 need half the threads
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r0 = tid / St::kChunks, c = tid % St::kChunks;
  const bool loads = kAll || r0 < kWideKeys;
  if ((int)blockIdx.x >= A.n_wide) {
    const int run = run_of(blockIdx.x - A.n_wide, (A.n_narrow + kWideWaves - 1) / kWideWaves) * kWideWaves + wave;
    if (run < A.n_narrow) narrow_run<BF, F8, D>(A, lds + wave * kNarrow, run, lane);
    return;
  }
  const int run = run_of(blockIdx.x, A.n_wide);
  int e = plan_at(A.wide_at, run + 1);
  bool lost = false;  // a page outside the pool
  int x = plan_at(A.wide_at, run);
  if (other_plan(A)) e = x;  // nothing to do
  const int mask = (1 << A.g.sh) - 1;
  KvSeg s;
  Tree tree;
  s16x8 q[D / 16];
  Sums<D> a;
  int last, wfirst, wlast;
  bool wreal;
  const int32_t* table;
  St st, s1;
  int32_t p0[I], p1[I], p2[I], page[I];  // of a stretch's first tiles; of the next whose K is fetched
  uint32_t row[I], r1s[I];               // pool rows of the last tile whose K was fetched, of the second
  int32_t ahead = 0;                     // the next stretch's numbers, one to a lane
  const auto first = [&](int t) { return tile_key<kWideKeys>(s, t < s.t1 ? t : s.t1 - 1); };
  const auto row_in = [&](int i) { return kAll ? i * St::kStep + r0 : r0 & (kWideKeys - 1); };
  // the pages, and then the pool rows, of a tile whose first key is kb
  const auto look = [&](const int32_t* tab, int last_col, int kb, int32_t (&p)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int col = (kb + row_in(i)) >> A.g.sh;
      p[i] = tab[(uint32_t)(col < last_col ? col : last_col)];
    }
  };
  const auto look_first = [&](const KvSeg& z) {
    const int32_t* tab = A.table + (int64_t)z.seq * A.cols;
    const int last_col = (z.p0 + z.ntok - 1) >> A.g.sh;
    const auto at = [&](int k) { return tile_key<kWideKeys>(z, z.t0 + k < z.t1 ? z.t0 + k : z.t1 - 1); };
    look(tab, last_col, at(0), p0);
    look(tab, last_col, at(1), p1);
    look(tab, last_col, at(2), p2);
  };
  const auto rows = [&](int kb, const int32_t (&p)[I], uint32_t (&r)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      r[i] = page_at(A, p[i], lost) + (in_page(A, s.head, row_in(i)) + (uint32_t)(kb & mask));
  };
  const auto fetch_k = [&](St& y, const uint32_t (&r)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      y.k[i] = St::load((const char*)A.pool.k, r[i], c * 16);
      if (F8) y.ks[i] = A.pool.ke[r[i]];
    }
  };
  const auto fetch_v = [&](St& y, const uint32_t (&r)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      y.v[i] = St::load((const char*)A.pool.v, r[i], c * 16);
      if (F8) y.vs[i] = A.pool.ve[r[i]];
    }
  };
  const auto put_k = [&](const St& y, int at) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (loads) y.put_k(ldk + at, i, i * St::kStep + r0, c, F8 ? scale_of(y.ks[i]) : 0.0f);
  };
  // V of tile t, whose first key is kb; `plain`: every row sees all of it
  const auto put_v = [&](const St& y, int t, int kb, bool plain) {
    char* vt = ldv + (t & 1) * kTileV;
    if (!loads) return;
    if (!plain && is_masked(A, all_to(tree, s), last, kb, kWideKeys)) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < I; ++i)
        bad |= y.template put_v<true>(vt, i, i * St::kStep + r0, c, last + 1 - kb, F8 ? scale_of(y.vs[i]) : 0.0f);
      if (bad) flag = 1;
    } else {
#pragma unroll
      for (int i = 0; i < I; ++i)
        y.template put_v<false>(vt, i, i * St::kStep + r0, c, 0, F8 ? scale_of(y.vs[i]) : 0.0f);
    }
  };
  const auto works = [&](int kb) { return wreal && kb <= wlast; };
  const auto hide_wave = [&](f32x16 (&y)[1], int kb) {
    if (!is_masked(A, wfirst, wlast, kb, 32)) return false;
    const int u = lane_of(A, s, here(wave * 32 + n)).tok - s.q0;  // looked up again: registers
    hide_keys(A, y[0], tree, row_of(A, s, u), kb, h);
    return true;
  };
  s16x8 kf[kAhead];
  // 32 keys from kb on, their scores in `sc`, their maximum taken: exponentials and the product with
  // V, beside the scores of the 32 keys from nb on
  const auto half = [&](int kb, const char* vt, bool more, int nb, const char* kt, const char* kn, f32x16 (&sc)[1],
                        f32x16 (&next)[1], bool plain) {
    if (plain ? !wreal : !works(kb)) return;
    float mx = weigh_and_score<BF, D, LSE>(vt, kt, kn, kf, q, sc, next, a, A.scale, lane);
    if (!plain) {
      if (!more || !works(nb)) return;
      if (hide_wave(next, nb)) mx = peak<1>(next);
    }
    raise<BF, D>(a, mx * A.scale);
  };
  // Takes up stretch x, whose numbers are `s` and whose first pages have been looked up: its queries and
  // first tiles, on their way from here on.
  const auto begin = [&]() {
    tree = tree_of(A, s);
    last = s.p0 + s.ntok - 1;
    // positions of this wave's own rows: keys past the last are not seen by any
    const int wtok = (wave * 32 + 31) / A.g.G, wtok0 = wave * 32 / A.g.G;
    wlast = s.p0 + (wtok < s.ntok ? wtok : s.ntok - 1);
    wfirst = tree.block == kNoTree ? s.p0 + (wtok0 < s.ntok ? wtok0 : s.ntok - 1) : tree.before;
    wreal = wave * 32 < s.ntok * A.g.G;
    table = A.table + (int64_t)s.seq * A.cols;
    uint32_t r0s[I];
    rows(first(s.t0), p0, r0s);
    fetch_k(st, r0s);
    fetch_v(st, r0s);
    rows(first(s.t0 + 1), p1, r1s);
    fetch_k(s1, r1s);
    load_q<D>(A, lane_of(A, s, wave * 32 + n), h, q);
    rows(first(s.t0 + 2), p2, row);
    look(table, last >> A.g.sh, first(s.t0 + 3), page);
  };
  // The next stretch that has keys, from x on; those without have only their zeros to write.
  const auto find = [&]() {
    for (; x < e; ++x) {
      s = plan_at(A.wide, x);
      if (s.t0 < s.t1) break;
      blank<D>(A, s, tid, kThreads);
    }
    if (x >= e) return false;
    look_first(s);
    return true;
  };
  const auto next_one = [&]() {
    KvSeg z;
    z.q0 = __builtin_amdgcn_readlane(ahead, 0);
    z.ntok = __builtin_amdgcn_readlane(ahead, 1);
    z.p0 = __builtin_amdgcn_readlane(ahead, 2);
    z.head = __builtin_amdgcn_readlane(ahead, 3);
    z.seq = __builtin_amdgcn_readlane(ahead, 4);
    z.ns = __builtin_amdgcn_readlane(ahead, 5);
    z.fw = __builtin_amdgcn_readlane(ahead, 6);
    z.t0 = __builtin_amdgcn_readlane(ahead, 7);
    z.t1 = __builtin_amdgcn_readlane(ahead, 8);
    z.slot = __builtin_amdgcn_readlane(ahead, 9);
    return z;
  };
  static_assert(sizeof(KvSeg) == 40);
  bool more = find();
  if (more) begin();
  f32x16 sa[1], sb[1];
  int kc = 0, kn = kTileK, kx = 2 * kTileK;  // K of this tile, the next and the one after
  while (more) {
    a.clear();
    kc = 0;
    kn = kTileK;
    kx = 2 * kTileK;
    __syncthreads();  // the last stretch's tiles and flag are done with
    if (tid == 0) flag = 0;
    __syncthreads();
    put_k(st, kc);
    put_v(st, s.t0, first(s.t0), false);
    put_k(s1, kn);
    fetch_v(st, r1s);
    fetch_k(st, row);
    ahead = ((const int32_t*)(A.wide + (x + 1 < e ? x + 1 : x)))[lane < 10 ? lane : 0];
    lds_barrier();
    if (works(first(s.t0))) {
      sa[0] = scores<BF, D>(ldk, q, n, h);
      hide_wave(sa, first(s.t0));
      raise<BF, D>(a, peak<1>(sa) * A.scale);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = k_part<D>(ldk + 32 * kRowK<D>, i, lane);
    }
    // Tile t; k0 .. k4: the first keys of it and of those after it
    const auto step = [&](int t, int k0, int k1, int k3, int k4, bool plain) {
      put_v(st, t + 1, k1, plain);
      put_k(st, kx);
      uint32_t next_row[I];
      rows(k3, page, next_row);
      fetch_v(st, row);
      fetch_k(st, next_row);
      look(table, last >> A.g.sh, k4, page);
#pragma unroll
      for (int i = 0; i < I; ++i) row[i] = next_row[i];
      const char* vt = ldv + (t & 1) * kTileV;
      half(k0, vt, true, k0 + 32, ldk + kc + 32 * kRowK<D>, ldk + kn, sa, sb, plain);
      half(k0 + 32, vt + 32 * kRowV<D>, plain || t + 1 < s.t1, k1, ldk + kn, ldk + kn + 32 * kRowK<D>, sb, sa, plain);
      const int z = kc;
      kc = kn;
      kn = kx;
      kx = z;
      lds_barrier();
    };
    // Plain tiles, which every row sees whole, follow one another: from the first past the sinks and
    // the windows' starts up to the tree's, or the first row's position.
    const int past = A.window && last >= A.window ? (last - A.window) / kWideKeys + 1 - s.fw + s.ns : 0;
    const int plain0 = past > s.ns ? past : s.ns, all = all_to(tree, s);
    const int plain1 = all < 0 ? 0 : (all + 1) / kWideKeys - s.fw + s.ns;
    int t = s.t0;
    while (t < s.t1) {
      // with the next one plain and four more to come, nothing is left to decide
      const int stop = plain1 - 1 < s.t1 - 4 ? plain1 - 1 : s.t1 - 4;
      if (t >= plain0)
        for (int kb = tile_key<kWideKeys>(s, t); t < stop; ++t, kb += kWideKeys)
          step(t, kb, kb + kWideKeys, kb + 3 * kWideKeys, kb + 4 * kWideKeys, true);
      if (t < s.t1) {
        if (t == s.t1 - 1) {  // where there is no next one: the same one's
          const KvSeg z = next_one();
          if (z.t0 < z.t1) look_first(z);
        }
        step(t, first(t), first(t + 1), first(t + 3), first(t + 4), false);
        ++t;
      }
    }
    const KvSeg done = s;
    more = ++x < e;
    if (more) {
      s = next_one();
      if (s.t0 >= s.t1) more = find();
      if (more) begin();
    }
    finish<BF, D>(A, done, a, lane, wave * 32, kWideRows, A.wide_o, A.wide_ml, lds + wave * 32 * kRowK<D>);
    if (flag) spread_tree<BF, F8, D, kWideKeys, false>(A, done, lane, wave * 32, kWideRows, A.wide_o);
  }
  if (lost) *A.err = kKvLostPage;
}

template <bool BF, bool F8, int D>
void run(const KvAttendArgs& a, hipStream_t stream) {
  const dim3 grid(a.n_wide + (a.n_narrow + kWideWaves - 1) / kWideWaves);
  if (!a.n_wide)
    k_kv_tree_narrow<BF, F8, D><<<a.n_narrow, 64, 0, stream>>>(a);
  else if (a.lse)
    k_kv_tree_wide<BF, F8, D, true><<<grid, 64 * kWideWaves, 0, stream>>>(a);
  else
    k_kv_tree_wide<BF, F8, D, false><<<grid, 64 * kWideWaves, 0, stream>>>(a);
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
  return hipGetLastError();
}

}  // namespace lar
