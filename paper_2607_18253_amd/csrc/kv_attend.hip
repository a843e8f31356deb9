// kv_attend.hip -- attention of a token batch over the pages of a key/value cache.
//
// For new token r of a sequence, at position p, over the keys j it sees (j <= p, and under
// a window W also j > p - W or j < sinks):
//     s_j = scale * q . k_j,   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),
// in one pass over the keys with a running maximum m and sum, all in 32 bits.
//
// A query tile is up to 32 (narrow) or 256 (wide) rows of one sequence and one kv head,
// row = token * G + head of the group, so that K and V are read once for the group.  Both
// kernels compute S^T = K Q^T and O^T = V^T P^T with 32x32x16 matrix instructions: a
// query row is a column, held by lanes n and n + 32, its maximum and sum are a lane's own
// values, and the elements of P^T that a lane holds are those that it has to hand to the
// second product, with its keys in the order  16 t + (j & 3) + 8 (j >> 2) + 4 h  that the
// transposing LDS reads give V^T in.
//
//   k_kv_narrow  one wave per stretch of 32-key tiles: single tokens and short chunks.
//                Bound by the bytes of K and V.  Waves share nothing, so there is no
//                barrier; the next tile is on its way in registers while one is used.
//   k_kv_wide    eight waves, 256 rows, 64-key tiles in LDS for all of them: chunks.
//                Bound by the matrix instructions and the exponentials beside them.
//   k_kv_join    the partial sums of the tiles whose keys were split over waves.
// A batch with both kinds of tiles is one launch of k_kv_wide; one with trees of drafted tokens has
// kernels of its own (kv_tree.hip) before the join.
//
// For the second product P has to be of V's 16-bit type.  Single tokens on a 16-bit cache have
// matrix instructions to spare: each weight is taken as two such values, 16 bits in all.  (On an
// 8-bit cache, whose rows have 4 bits, that would take 509 requests of 9.2k tokens from 1711 to
// 1766 us and the error against 64 bits from 1.34 times that of a 32-bit form to the same.)
// Else it is rounded once (nearest even), an error of the size of the output's own rounding,
// and the result is divided by the sum of the rounded weights, so that nothing is lost of a
// weight that outweighs the others; the log of the sum, where it is asked for, is that of the
// unrounded ones.  f16 has no values below 2^-24, and from 2^-14 down fewer bits: a row's weights
// are scaled so that its largest is 2^11 to 2^15, and what a weight loses at that end is 2^-36
// of the largest at most, 2^-17 of the result for 2^19 keys.  (With largest weights of 1 the
// share of 32767 keys that weigh 2^-23 to 2^-26 of one came out wrong by up to all of it.)
#include "../../include/lar.h"
#include "kv_attend.h"

namespace lar {
namespace {

// ------------------------------------------------------------------ narrow tiles
// One wave's run of stretches; `lds`: its tile of 32 keys.
template <bool BF, bool F8, int D>
__device__ __forceinline__ void narrow(const KvAttendArgs& A, char* lds, int run, int lane) {
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
    s16x8 q[D / 16];
    const Row row = load_q<D>(A, lane_of(A, s, n), h, q);
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
      const bool masked = is_masked(A, s.p0, last, kb, kNarrowKeys);
      uint32_t e[I], m = 0;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        e[i] = F8 ? (uint32_t)__shfl((int)ex, i * St::kStep + r0) : 0;
        st.put_k(kt, i, i * St::kStep + r0, c, scale_of(e[i]));
        if (!F8) m = max16(m, top_pair(st.v[i]));
      }
      // With weights in two parts infinities and NaN are taken out of any tile: the second part may
      // be 0 or have the other sign, and 0 * inf and inf - inf are NaN.  (Finding them takes 9
      // instructions for 16 bytes: 255 decode tokens 255.1 -> 256.5 us.)
      const bool odd = !F8 && __any(top_half(m) >= kInf<BF>);
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int r = i * St::kStep + r0;
        if (masked || odd)
          bad |= st.template put_v<true>(vt, i, r, c, last + 1 - kb, scale_of(e[i] >> 8));
        else
          st.template put_v<false>(vt, i, r, c, 0, scale_of(e[i] >> 8));
      }
      if (t + 1 < s.t1) {
        fetch(page, t + 1);
        if (t + 2 < s.t1) page = look(t + 2);
      }
      wave_order();
      f32x16 sc[1] = {scores<BF, D>(kt, q, n, h)};
      if (masked) hide<1>(sc, row, kb, h, A.window);
      raise<BF, D>(a, peak<1>(sc) * A.scale);
      soften<D, 1>(sc, a, A.scale);
      weigh<BF, D, !F8>(vt, sc[0], a, lane);
      wave_order();
    }
    finish<BF, D>(A, s, a, lane, 0, kNarrowRows, A.narrow_o, A.narrow_ml, lds);
    wave_order();
    if (__any(bad)) spread<BF, F8, D, kNarrowKeys, !F8>(A, s, lane, 0, kNarrowRows, A.narrow_o);
  }
  if (lost) *A.err = kKvLostPage;
}

template <bool BF, bool F8, int D>
__global__ __launch_bounds__(64, 2) void k_kv_narrow(KvAttendArgs A) {
  __shared__ __align__(16) char lds[kTileBytes<D, kNarrowKeys>];
  narrow<BF, F8, D>(A, lds, run_of(blockIdx.x, A.n_narrow), threadIdx.x);
}

// ------------------------------------------------------------------ wide tiles
// The workgroups past n_wide take narrow tiles, a run for each wave: the two kinds share the
// device, one bound by matrix instructions and the other by memory.
//
// LSE: the log of the sums is asked for, which takes the sum of the unrounded weights too
// (7681 tokens at 131072: 15.8 ms with it, 14.8 without; heads of 64: 9.2 and 8.7).
template <bool BF, bool F8, int D, bool LSE>
__global__ __launch_bounds__(64 * kWideWaves, 2) void k_kv_wide(KvAttendArgs A) {
  constexpr int kTileK = kWideKeys * kRowK<D>, kTileV = kWideKeys * kRowV<D>, kThreads = 64 * kWideWaves;
  constexpr int kNarrow = kTileBytes<D, kNarrowKeys>, kWide = 3 * kTileK + 2 * kTileV;
  __shared__ __align__(16) char lds[kWide > kWideWaves * kNarrow ? kWide : kWideWaves * kNarrow];
  static_assert(kWideWaves * 32 * kRowK<D> <= kWide, "a result in LDS");
  char *const ldk = lds, *const ldv = lds + 3 * kTileK;
  __shared__ int flag;
  using St = Stage<BF, F8, D, (kWideKeys * (F8 ? D / 16 : D / 8) + kThreads - 1) / kThreads, kThreads>;
  constexpr int I = (kWideKeys + St::kStep - 1) / St::kStep;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r0 = tid / St::kChunks, c = tid % St::kChunks;
  constexpr bool kAll = St::kStep <= kWideKeys;  // else 8-bit rows of 64 need half the threads
  const bool loads = r0 < kWideKeys;
  if ((int)blockIdx.x >= A.n_wide) {
    const int run = run_of(blockIdx.x - A.n_wide, (A.n_narrow + kWideWaves - 1) / kWideWaves) * kWideWaves + wave;
    if (run < A.n_narrow) narrow<BF, F8, D>(A, lds + wave * kNarrow, run, lane);
    return;
  }
  const int run = run_of(blockIdx.x, A.n_wide);
  int e = plan_at(A.wide_at, run + 1);
  bool lost = false;  // a page outside the pool
  int x = plan_at(A.wide_at, run);
  if (other_plan(A)) e = x;  // nothing to do
  // the current stretch, its queries, and its first keys on their way
  KvSeg s;
  s16x8 q[D / 16];
  Row rw;
  Sums<D> a;
  int last, last_col, wfirst, wlast;
  bool wreal;
  const int32_t* table;
  St st, s0, s1;
  int32_t page[I];            // of the next tile whose K is fetched
  uint32_t row[I], r1s[I];    // pool rows of the last tile whose K was fetched, the next V
  const int mask = (1 << A.g.sh) - 1;
  // Loads are not skipped, so that what waits for one knows how many follow it: past the
  // stretch's end they take its last tile.
  const auto first = [&](int t) { return tile_key<kWideKeys>(s, t < s.t1 ? t : s.t1 - 1); };
  const auto row_of = [&](int i) { return kAll ? i * St::kStep + r0 : r0 & (kWideKeys - 1); };
  // the pages, and then the pool rows, of a tile whose first key is kb
  const auto look = [&](int kb, int32_t (&p)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int col = (kb + row_of(i)) >> A.g.sh;
      p[i] = table[(uint32_t)(col < last_col ? col : last_col)];
    }
  };
  // tiles start at multiples of 64: a key's row in its page is that of its row in the tile,
  // and in pages of more than 64 tokens the tile's place in the page
  const auto rows = [&](int kb, const int32_t (&p)[I], uint32_t (&r)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      r[i] = page_at(A, p[i], lost) + (in_page(A, s.head, row_of(i)) + (uint32_t)(kb & mask));
  };
  const auto fetch_k = [&](St& x, const uint32_t (&r)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      x.k[i] = St::load((const char*)A.pool.k, r[i], c * 16);
      if (F8) x.ks[i] = A.pool.ke[r[i]];
    }
  };
  const auto fetch_v = [&](St& x, const uint32_t (&r)[I]) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      x.v[i] = St::load((const char*)A.pool.v, r[i], c * 16);
      if (F8) x.vs[i] = A.pool.ve[r[i]];
    }
  };
  const auto put_k = [&](const St& x, int at) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (kAll || loads) x.put_k(ldk + at, i, i * St::kStep + r0, c, F8 ? scale_of(x.ks[i]) : 0.0f);
  };
  // V of tile t, whose first key is kb; `plain`: every row sees all of it
  const auto put_v = [&](const St& x, int t, int kb, bool plain) {
    char* vt = ldv + (t & 1) * kTileV;
    if (!kAll && !loads) return;
    if (!plain && is_masked(A, s.p0, last, kb, kWideKeys)) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < I; ++i)
        bad |= x.template put_v<true>(vt, i, i * St::kStep + r0, c, last + 1 - kb, F8 ? scale_of(x.vs[i]) : 0.0f);
      if (bad) flag = 1;
    } else {
#pragma unroll
      for (int i = 0; i < I; ++i)
        x.template put_v<false>(vt, i, i * St::kStep + r0, c, 0, F8 ? scale_of(x.vs[i]) : 0.0f);
    }
  };
  const auto works = [&](int kb) { return wreal && kb <= wlast; };
  s16x8 kf[kAhead];
  // 32 keys from kb on, their scores in `sc`, their maximum taken: exponentials and the
  // product with V, beside the scores of the 32 keys from nb on (past the wave's last key
  // these are of any rows, and not used)
  const auto half = [&](int kb, const char* vt, bool more, int nb, const char* kt, const char* kn,
                        f32x16 (&sc)[1], f32x16 (&next)[1], bool plain) {
    if (plain ? !wreal : !works(kb)) return;
    float mx = weigh_and_score<BF, D, LSE>(vt, kt, kn, kf, q, sc, next, a, A.scale, lane);
    if (!plain && (!more || !works(nb))) return;
    if (!plain && is_masked(A, wfirst, wlast, nb, 32)) {
      hide<1>(next, rw, nb, h, A.window);
      mx = peak<1>(next);
    }
    raise<BF, D>(a, mx * A.scale);
  };
  f32x16 sa[1], sb[1];
  int kc = 0, kn = kTileK, kx = 2 * kTileK;  // K of this tile, the next and the one after
  // Takes up the next stretch that has keys: its queries and first tiles, all on their way
  // at once beside what the last one has left to do.
  const auto next = [&]() {
    for (; x < e; ++x) {
      s = plan_at(A.wide, x);
      if (s.t0 < s.t1) break;
      blank<D>(A, s, tid, kThreads);
    }
    if (x++ >= e) return false;
    rw = load_q<D>(A, lane_of(A, s, wave * 32 + n), h, q);
    last = s.p0 + s.ntok - 1;
    last_col = last >> A.g.sh;
    // positions of this wave's own rows: keys past the last are not seen by any
    const int wtok = (wave * 32 + 31) / A.g.G, wtok0 = wave * 32 / A.g.G;
    wlast = s.p0 + (wtok < s.ntok ? wtok : s.ntok - 1);
    wfirst = s.p0 + (wtok0 < s.ntok ? wtok0 : s.ntok - 1);
    wreal = wave * 32 < s.ntok * A.g.G;
    table = A.table + (int64_t)s.seq * A.cols;
    int32_t p0[I], p1[I], p2[I];
    uint32_t r0s[I];
    look(first(s.t0), p0);
    look(first(s.t0 + 1), p1);
    look(first(s.t0 + 2), p2);
    look(first(s.t0 + 3), page);
    rows(first(s.t0), p0, r0s);
    rows(first(s.t0 + 1), p1, r1s);
    rows(first(s.t0 + 2), p2, row);
    fetch_k(s0, r0s);
    fetch_v(s0, r0s);
    fetch_k(s1, r1s);
    return true;
  };
  bool more = next();
  while (more) {
    a.clear();
    kc = 0;
    kn = kTileK;
    kx = 2 * kTileK;
    __syncthreads();  // the last stretch's tiles and flag are done with
    if (tid == 0) flag = 0;
    __syncthreads();
    put_k(s0, kc);
    put_v(s0, s.t0, first(s.t0), false);
    put_k(s1, kn);
    fetch_v(st, r1s);
    fetch_k(st, row);
    lds_barrier();
    if (works(tile_key<kWideKeys>(s, s.t0))) {
      sa[0] = scores<BF, D>(ldk, q, n, h);
      const int kb = tile_key<kWideKeys>(s, s.t0);
      if (is_masked(A, wfirst, wlast, kb, 32)) hide<1>(sa, rw, kb, h, A.window);
      raise<BF, D>(a, peak<1>(sa) * A.scale);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = k_part<D>(ldk + 32 * kRowK<D>, i, lane);
    }
    // Tile t; k0 .. k4: the first keys of it and of the four after it
    const auto step = [&](int t, int k0, int k1, int k3, int k4, bool plain) {
      // what was fetched beside the last tile goes into LDS beside this one, where all waves
      // are past the tiles that were there
      put_v(st, t + 1, k1, plain);
      put_k(st, kx);
      uint32_t next_row[I];
      rows(k3, page, next_row);
      fetch_v(st, row);
      fetch_k(st, next_row);
      look(k4, page);
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
    // Plain tiles, which every row of the query tile sees whole, follow one another: from the
    // first past the sinks and the last row's window's start up to the first row's position.
    const int past = A.window && last >= A.window ? (last - A.window) / kWideKeys + 1 - s.fw + s.ns : 0;
    const int plain0 = past > s.ns ? past : s.ns;
    const int plain1 = s.p0 < 0 ? 0 : (s.p0 + 1) / kWideKeys - s.fw + s.ns;
    int t = s.t0;
    while (t < s.t1) {
      // with the next one plain and four more to come, nothing is left to decide
      const int stop = plain1 - 1 < s.t1 - 4 ? plain1 - 1 : s.t1 - 4;
      if (t >= plain0)
        for (int kb = tile_key<kWideKeys>(s, t); t < stop; ++t, kb += kWideKeys)
          step(t, kb, kb + kWideKeys, kb + 3 * kWideKeys, kb + 4 * kWideKeys, true);
      if (t < s.t1) {
        step(t, first(t), first(t + 1), first(t + 3), first(t + 4), false);
        ++t;
      }
    }
    const KvSeg done = s;
    more = next();
    finish<BF, D>(A, done, a, lane, wave * 32, kWideRows, A.wide_o, A.wide_ml, lds + wave * 32 * kRowK<D>);
    if (flag) spread<BF, F8, D, kWideKeys, false>(A, done, lane, wave * 32, kWideRows, A.wide_o);
  }
  if (lost) *A.err = kKvLostPage;
}

// ------------------------------------------------------------------ joining split tiles
// One workgroup per join_rows rows of a split tile.  A thread has 4 values of a row; where the
// rows leave threads over, these share out the slots and are joined through LDS, in a fixed order.
// Bound by the latency of the slots' loads, of which each thread has four on their way.
struct Part {
  float m, l, lr;
  f32x4 o;
  // The sums of two parts of a row's keys.
  __device__ __forceinline__ void join(const Part& p) {
    const float top = fmaxf(m, p.m), t = top == -__builtin_inff() ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - t), g = __builtin_amdgcn_exp2f(p.m - t);
    m = top;
    l = __builtin_fmaf(p.l, g, l * f);
    lr = __builtin_fmaf(p.lr, g, lr * f);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(p.o[i], g, o[i] * f);
  }
};

template <bool BF, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_join(KvAttendArgs A) {
  constexpr int kQuads = D / 4;
  __shared__ Part parts[THREADS];
  const KvJoin j = plan_at(A.join, blockIdx.x);
  if (other_plan(A)) return;
  const int rows = j.wide ? kWideRows : kNarrowRows, row0 = j.row0;
  const int have = j.ntok * A.g.G - row0 < A.join_rows ? j.ntok * A.g.G - row0 : A.join_rows;
  const float* po = j.wide ? A.wide_o : A.narrow_o;
  const float4* pml = j.wide ? A.wide_ml : A.narrow_ml;
  const int n = have * kQuads;  // quads of values
  int share = THREADS / n;      // threads on the same one
  share = share < 1 ? 1 : share < j.n ? share : j.n;
  const int mine = n < THREADS ? threadIdx.x / n : 0;
  for (int u = n < THREADS ? threadIdx.x % n : threadIdx.x; u < n; u += THREADS) {
    const int r = u % have, d = (u / have) * 4;
    Part a{-__builtin_inff(), 0.0f, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
    if (mine < share) {
      for (int s = mine; s < j.n; s += 4 * share) {
        Part p[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int x = s + k * share < j.n ? s + k * share : s;
          const float4 ml = pml[(int64_t)(j.slot + x) * rows + row0 + r];
          p[k].m = ml.x;
          p[k].l = ml.y;
          p[k].lr = ml.z;
          p[k].o = *(const f32x4*)(po + part_at<D>(j.slot + x, rows, j.ntok * A.g.G, row0 + r, d / 4));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (s + k * share < j.n) a.join(p[k]);
      }
    }
    // Shares are joined by fours, then what they made (then one round: every thread is here).
    if (share > 1) parts[threadIdx.x] = a;
    for (int k = 1; k < share; k *= 4) {
      __syncthreads();
      if (mine % (4 * k) == 0) {
        const int end = mine + 4 * k < share ? mine + 4 * k : share;
        for (int i = mine + k; i < end; i += k) a.join(parts[i * n + u]);
        parts[threadIdx.x] = a;
      }
    }
    if (mine != 0) continue;
    const int t = (row0 + r) / A.g.G, g = row0 + r - t * A.g.G;
    const bool none = j.p0 + t < 0;
    const float inv = none ? 0.0f : 1.0f / a.lr;
    const int64_t at = (int64_t)(j.q0 + t) * A.g.hq + j.head * A.g.G + g;
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = Elem<BF>::one(none ? 0.0f : a.o[2 * i] * inv) |
             (uint32_t)Elem<BF>::one(none ? 0.0f : a.o[2 * i + 1] * inv) << 16;
    *(uint2*)((uint16_t*)A.out + at * D + d) = make_uint2(w[0], w[1]);
    if (A.lse && d == 0) {
      const float m = a.m == -__builtin_inff() ? 0.0f : a.m;
      A.lse[at] = none ? -__builtin_inff() : (m + __builtin_amdgcn_logf(a.l)) * kLn2;
    }
  }
}

template <bool BF, bool F8, int D>
hipError_t run(const KvAttendArgs& a, hipStream_t stream) {
  if (a.trees) {
    if (const hipError_t e = launch_kv_tree(a, stream)) return e;
  } else if (a.n_wide) {
    const dim3 grid(a.n_wide + (a.n_narrow + kWideWaves - 1) / kWideWaves);
    if (a.lse)
      k_kv_wide<BF, F8, D, true><<<grid, 64 * kWideWaves, 0, stream>>>(a);
    else
      k_kv_wide<BF, F8, D, false><<<grid, 64 * kWideWaves, 0, stream>>>(a);
  } else if (a.n_narrow) {
    k_kv_narrow<BF, F8, D><<<a.n_narrow, 64, 0, stream>>>(a);
  }
  // Many parts: more threads to share them out to (40 tokens of 8 heads over 4000 keys, 16
  // parts of each tile: 15.4 us with 1024 threads, 19.3 with 256); few parts of many tiles:
  // smaller workgroups (255 decode tokens take 1.5 % more with 1024).
  // Few tiles of trees, 1024 quads of values each: 6.7 us, 10.1 with 256 (125 trees of 5 to 31 tokens); with half
  // as many, of heads of 64, they take the same.
  const bool large = a.trees && a.n_join < 512 && a.join_rows * D >= 4096;
  if (a.n_join && (a.most_parts > 8 || large))
    k_kv_join<BF, D, 1024><<<a.n_join, 1024, 0, stream>>>(a);
  else if (a.n_join)
    k_kv_join<BF, D, 256><<<a.n_join, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <bool BF, bool F8>
hipError_t run_d(const KvAttendArgs& a, hipStream_t stream) {
  return a.g.D == 128 ? run<BF, F8, 128>(a, stream) : run<BF, F8, 64>(a, stream);
}

}  // namespace

hipError_t launch_kv_attend(const KvAttendArgs& a, hipStream_t stream) {
  const bool f8 = a.g.cache == kKvE4m3;
  if (a.g.dtype == kKvBf16) return f8 ? run_d<true, true>(a, stream) : run_d<true, false>(a, stream);
  return f8 ? run_d<false, true>(a, stream) : run_d<false, false>(a, stream);
}

}  // namespace lar
