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
// A batch with both kinds of tiles is one launch of k_kv_wide.
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
#include "kv_device.h"
#include "kv_words.h"

namespace lar {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((address_space(3))) char lds_char;

constexpr float kLn2 = 0.693147180559945309f;

// Per 16-bit type, in log2 units: a row's largest weight is 2^kTop when its sums are scaled, and
// may grow by 2^kLag before they are rescaled.
template <bool BF> struct Elem;
template <> struct Elem<true> {
  using x8 = bf16x8;
  static __device__ __forceinline__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ s16x8 pack(f32x8 x) {
    return __builtin_bit_cast(s16x8, __builtin_convertvector(x, bf16x8));
  }
  static __device__ __forceinline__ f32x8 unpack(s16x8 x) {
    return __builtin_convertvector(__builtin_bit_cast(bf16x8, x), f32x8);
  }
  static __device__ __forceinline__ uint32_t pair(uint32_t codes, float s, bool hi) {
    return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, s, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, s, false));
  }
  static __device__ __forceinline__ uint16_t one(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
  }
  static __device__ __forceinline__ float value(uint16_t x) {
    return __uint_as_float((uint32_t)x << 16);
  }
  // c plus the two values of a pair
  static __device__ __forceinline__ float add_pair(uint32_t x, float c) {
    typedef __attribute__((ext_vector_type(2))) __bf16 x2;
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(x2, x), x2{(__bf16)1.0f, (__bf16)1.0f}, c, false);
  }
  static constexpr uint32_t kExp = 0x7f80u;  // exponent bits: all ones where not finite
  static constexpr float kTop = 0.0f, kLag = 8.0f;
};
template <> struct Elem<false> {
  using x8 = f16x8;
  static __device__ __forceinline__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ s16x8 pack(f32x8 x) {
    return __builtin_bit_cast(s16x8, __builtin_convertvector(x, f16x8));
  }
  static __device__ __forceinline__ f32x8 unpack(s16x8 x) {
    return __builtin_convertvector(__builtin_bit_cast(f16x8, x), f32x8);
  }
  static __device__ __forceinline__ uint32_t pair(uint32_t codes, float s, bool hi) {
    return hi ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, s, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, s, false));
  }
  static __device__ __forceinline__ uint16_t one(float x) {
    return __builtin_bit_cast(uint16_t, (_Float16)x);
  }
  static __device__ __forceinline__ float value(uint16_t x) {
    return (float)__builtin_bit_cast(_Float16, x);
  }
  static __device__ __forceinline__ float add_pair(uint32_t x, float c) {
    typedef __attribute__((ext_vector_type(2))) _Float16 x2;
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(x2, x), x2{(_Float16)1.0f, (_Float16)1.0f}, c, false);
  }
  static constexpr uint32_t kExp = 0x7c00u;
  static constexpr float kTop = 11.0f, kLag = 4.0f;  // 2^15 at most: f16 ends at 2^16
};

// Sets infinities and NaN among the 8 16-bit values to 0; whether there were any.
template <bool BF>
__device__ __forceinline__ bool clean(uint4& x) {
  constexpr uint32_t e = Elem<BF>::kExp, eh = e << 16;
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (w[i] & e) == e, hi = (w[i] & eh) == eh;
    w[i] = lo ? w[i] & 0xffff0000u : w[i];
    w[i] = hi ? w[i] & 0x0000ffffu : w[i];
    bad |= lo || hi;
  }
  x = make_uint4(w[0], w[1], w[2], w[3]);
  return bad;
}

// A value that is not known before this point, so that what is made of it is made here and
// not kept in registers across the loops around.
template <class T>
__device__ __forceinline__ T here(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The plan's arrays are not written while a kernel runs: scalar loads.
template <class T>
__device__ __forceinline__ T plan_at(const T* p, int i) {
  constexpr int n = sizeof(T) / 4;
  const auto* w = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(p + i);
  int32_t x[n];
#pragma unroll
  for (int k = 0; k < n; ++k) x[k] = w[k];
  T t;
  __builtin_memcpy(&t, x, sizeof t);
  return t;
}

// Whether the device has another plan now than the launch was made for.
__device__ __forceinline__ bool other_plan(const KvAttendArgs& A) {
  if (plan_at(A.plan.now, 0) == A.plan.id) return false;
  *A.err = kKvOtherPlan;
  return true;
}

// The run of stretches of workgroup `i` of n.  Workgroups go to the 8 XCDs in turn; runs that
// follow one another, which read the same keys or their neighbours, go to one XCD's L2.
__device__ __forceinline__ int run_of(int i, int n) {
  const int x = i & 7, r = n & 7;
  return x * (n >> 3) + (x < r ? x : r) + (i >> 3);
}

// The larger, or the sum, of a lane's value and that of lane ^ 32.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Orders a wave's LDS accesses of different lanes: they run in program order.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A barrier of the workgroup for its LDS alone: loads from memory stay on their way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Key of element i of S^T's 32 keys in a lane of half h.
__device__ __forceinline__ constexpr int key_of(int i, int h) {
  return (i & 3) + 8 * (i >> 2) + 4 * h;
}

// LDS tiles: [key][D] 16-bit values, rows padded.  A K read takes 16 bytes at one place of
// 32 rows: with 16 bytes of padding 16 rows cover the 64 banks.  A V read takes 64 bytes at
// one place of 8 rows: rows 64 bytes apart, modulo the banks, cover them twice.
template <int D> constexpr int kRowK = D * 2 + 16;
template <int D> constexpr int kRowV = D * 2 + 64;
template <int D, int K> constexpr int kTileBytes = K * (kRowK<D> + kRowV<D>);  // K, then V

// A query tile in a wave: this lane's row and what its keys are.
struct Row {
  int pos;    // position of the row's token; < 0: it sees nothing
  int lo;     // keys > lo or < sinks
  int sinks;
  __device__ __forceinline__ bool sees(int j) const {
    return j <= pos && (j > lo || j < sinks);
  }
};

// Takes the scores of keys from kb on that the row does not see to -infinity.
template <int NB>
__device__ __forceinline__ void hide(f32x16 (&s)[NB], const Row& r, int kb, int h, int window) {
  const int base = kb + 4 * h;  // the keys of a lane: base + constants
  const int pos = r.pos - base;
#pragma unroll
  for (int u = 0; u < NB; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[u][i] = 32 * u + key_of(i, 0) <= pos ? s[u][i] : -__builtin_inff();
  if (!window) return;
  const int lo = r.lo - base, sinks = r.sinks - base;
#pragma unroll
  for (int u = 0; u < NB; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = 32 * u + key_of(i, 0);
      s[u][i] = j > lo || j < sinks ? s[u][i] : -__builtin_inff();
    }
}

// The running sums of a wave's 32 rows.
template <int D>
struct Sums {
  f32x16 o[D / 32];  // O^T: row n, value 32 b + key_of(i, h)
  float m, l, lr;    // weights are 2^(score - m); this half's part of their sum, and of what o has
  __device__ __forceinline__ void clear() {
    const float z = here(0.0f);
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = z;
    m = -__builtin_inff();
    l = lr = 0.0f;
  }
};

// S^T of 32 keys, `kt` their rows in LDS.
template <bool BF, int D>
__device__ __forceinline__ f32x16 scores(const char* kt, const s16x8 (&q)[D / 16], int n, int h) {
  f32x16 s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    const s16x8 k = *(const s16x8*)(kt + n * kRowK<D> + h * 16 + t * 32);
    s = Elem<BF>::mma(k, q[t], s);
  }
  return s;
}

// The largest of a row's scores in NB blocks of 32 keys.
template <int NB>
__device__ __forceinline__ float peak(const f32x16 (&s)[NB]) {
  float mx = s[0][0];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i]);
  return max_halves(mx);
}

// Takes a tile's largest scores (times the scale: log2 units) into the running maximum less
// kTop, rescaling the rows' sums where it grew.
template <bool BF, int D>
__device__ __forceinline__ void raise(Sums<D>& a, float mx) {
  if (__any(mx > a.m + (Elem<BF>::kTop + Elem<BF>::kLag))) {
    const float m = fmaxf(mx - Elem<BF>::kTop, a.m);
    const float f = m > a.m ? __builtin_amdgcn_exp2f(a.m - m) : 1.0f;  // 0 from a.m = -inf
    a.m = m;
    a.l *= f;
    a.lr *= f;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) a.o[b][i] *= f;
  }
}

// Scores to their exponentials, into the running sum.
template <int D, int NB>
__device__ __forceinline__ void soften(f32x16 (&s)[NB], Sums<D>& a, float c) {
  const float m = a.m == -__builtin_inff() ? 0.0f : a.m;
  float l = 0.0f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -m));
      l += s[b][i];
    }
  a.l += l;
}

// V^T fragment of 16 keys and 32 values, `vt` the keys' rows in LDS: 16 lanes read 4 keys x
// 16 values and get them by columns.
template <int D>
__device__ __forceinline__ s16x8 v_part(const char* vt, int b, int lane) {
  const int h = lane >> 5, i = lane & 15, g = lane >> 4;
  const char* at = vt + (4 * h + (i >> 2)) * kRowV<D> + (g & 1) * 32 + (i & 3) * 8 + b * 64;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 8 * kRowV<D>));
  s16x8 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = lo[j];
    v[4 + j] = hi[j];
  }
  return v;
}

// The exponentials of 16 keys, rounded, in the order of v_part's keys.
template <bool BF>
__device__ __forceinline__ s16x8 p_part(const f32x16& p, int t) {
  f32x8 x;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = p[8 * t + j];
  return Elem<BF>::pack(x);
}

// x plus the sum of 8 rounded weights.
template <bool BF>
__device__ __forceinline__ float add_rounded(s16x8 pk, float x) {
  const uint4 w = __builtin_bit_cast(uint4, pk);
  return Elem<BF>::add_pair(w.w, Elem<BF>::add_pair(w.z, Elem<BF>::add_pair(w.y, Elem<BF>::add_pair(w.x, x))));
}

// O^T += V^T P^T over 32 keys, `vt` their rows in LDS; TWO: P in two parts, the rounded
// weights and what the rounding left.
template <bool BF, int D, bool TWO>
__device__ __forceinline__ void weigh(const char* vt, const f32x16& p, Sums<D>& a, int lane) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    f32x8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = p[8 * t + j];
    const s16x8 hi = Elem<BF>::pack(x);
    s16x8 lo;
    if (TWO)
      lo = Elem<BF>::pack(x - Elem<BF>::unpack(hi));
    else
      a.lr = add_rounded<BF>(hi, a.lr);
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
      const s16x8 v = v_part<D>(vt + 16 * t * kRowV<D>, b, lane);
      a.o[b] = Elem<BF>::mma(v, hi, a.o[b]);
      if (TWO) a.o[b] = Elem<BF>::mma(v, lo, a.o[b]);
    }
  }
  if (TWO) a.lr = a.l;
}

// K fragments that a wave has on their way from LDS ahead of their use.
constexpr int kAhead = 4;

template <int D>
__device__ __forceinline__ s16x8 k_part(const char* kt, int t, int lane) {
  return *(const s16x8*)(kt + (lane & 31) * kRowK<D> + (lane >> 5) * 16 + t * 32);
}

// Exponentials of 32 keys with scores `s` and their product with V (rows `vt`), beside the
// scores of the next 32 keys (rows `kt`, their first fragments in `k`) into `next`; returns
// the maximum of those, and in `k` the first fragments of rows `kn`.  Exponentials and maxima
// run in the shadow of the matrix instructions, LDS reads four of those ahead, in the order
// written: the exponentials evenly over the scores' instructions and the first of the
// product's, which is as late as they can be.  Of the two waves of a SIMD the one at the
// scores and exponentials goes first, and the other one's product fills in (7681 tokens at
// 131072: 15.0 ms, 15.3 without priorities, 15.5 with all exponentials beside the scores; heads
// of 64: 8.7, 9.2 and 9.3).
template <bool BF, int D, bool LSE>
__device__ __forceinline__ float weigh_and_score(const char* vt, const char* kt, const char* kn, s16x8 (&k)[kAhead],
                                                 const s16x8 (&q)[D / 16], f32x16 (&s)[1], f32x16 (&next)[1],
                                                 Sums<D>& a, float c, int lane) {
  constexpr int kSteps = D / 16, kB = D / 32, kSlots = kSteps + kB;
  const float m = a.m == -__builtin_inff() ? 0.0f : a.m;
  s16x8 pk[2], v[kB];
  f32x16 x;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.0f;
  float l = a.l, lr = a.lr;
  // the exponentials beside matrix instruction `slot`
  const auto exps = [&](int slot) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if (e * kSlots / 16 != slot) continue;
      const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][e], c, -m));
      s[0][e] = y;
      if (LSE) l += y;
      if ((e & 7) == 7) {
        pk[e >> 3] = here(p_part<BF>(s[0], e >> 3));
        lr = add_rounded<BF>(pk[e >> 3], lr);
      }
    }
    if (LSE) l = here(l);
    lr = here(lr);
  };
#pragma unroll
  for (int t = 0; t < kSteps; ++t) {
    x = Elem<BF>::mma(k[t % kAhead], q[t], x);
    if (t + kAhead < kSteps) k[t % kAhead] = k_part<D>(kt, t + kAhead, lane);
    if (t >= kSteps - kB) v[t - (kSteps - kB)] = v_part<D>(vt, t - (kSteps - kB), lane);
    exps(t);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  float mx = x[0];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      a.o[b] = Elem<BF>::mma(v[b], pk[t], a.o[b]);
      if (t == 0) {
        v[b] = v_part<D>(vt + 16 * kRowV<D>, b, lane);
        exps(kSteps + b);
      } else {
#pragma unroll
        for (int i = b * kAhead / kB; i < (b + 1) * kAhead / kB; ++i) k[i] = k_part<D>(kn, i, lane);
#pragma unroll
        for (int i = 16 * b / kB; i < 16 * (b + 1) / kB; ++i) mx = fmaxf(mx, x[i]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  __builtin_amdgcn_s_setprio(1);
  a.l = l;
  a.lr = lr;
  next[0] = x;
  return max_halves(mx);
}

// What a lane of a query tile is: its row's token and head, and what it sees.
struct Lane {
  int tok, qh;   // token of the batch, query head
  bool real;     // the tile has this row
  Row row;
};

__device__ __forceinline__ Lane lane_of(const KvAttendArgs& A, const KvSeg& s, int n) {
  const int t = n / A.g.G;
  Lane x;
  x.real = t < s.ntok;
  const int u = x.real ? t : s.ntok - 1;
  x.tok = s.q0 + u;
  x.qh = s.head * A.g.G + (x.real ? n - t * A.g.G : 0);
  x.row.pos = s.p0 + u;
  x.row.lo = A.window ? x.row.pos - A.window : -1;
  x.row.sinks = A.sinks;
  return x;
}

template <int D>
__device__ __forceinline__ Row load_q(const KvAttendArgs& A, const Lane& x, int h, s16x8 (&q)[D / 16]) {
  const int16_t* p = (const int16_t*)A.q.p + (int64_t)x.tok * A.q.tok + (int64_t)x.qh * A.q.head;
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    s16x8 z = {0, 0, 0, 0, 0, 0, 0, 0};
    if (x.real) z = *(const s16x8*)(p + 16 * t + 8 * h);
    q[t] = z;
  }
  return x.row;
}

// Where a split tile's partial sums are: by blocks of 32 rows, in each 4 values of its rows side
// by side, by quads of values.  `rows`: what a slot has room for; a narrow tile's `real` rows
// have no gaps between them (one token of one head over 60k keys: 24 -> 14 us).
template <int D>
__device__ __forceinline__ int64_t part_at(int slot, int rows, int real, int row, int quad) {
  const int first = row & ~31, n = rows == kNarrowRows ? real : 32;
  return ((int64_t)slot * rows + first) * D + (quad * n + row - first) * 4;
}

// The result of a wave's 32 rows, through LDS (32 rows of `tmp`) so that whole rows are
// written, or their partial sums (`row0`: first row of the wave in the slot, `rows` of one).
template <bool BF, int D>
__device__ __forceinline__ void finish(const KvAttendArgs& A, const KvSeg& s, const Sums<D>& a, int lane,
                                       int row0, int rows, float* po, float4* pml, char* tmp) {
  lane = here(lane);
  const int n = lane & 31, h = lane >> 5, slot = s.slot;
  const Lane x = lane_of(A, s, row0 + n);
  const float l = add_halves(a.l), lr = add_halves(a.lr);
  if (slot >= 0) {
    if (!x.real) return;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        f32x4 y = {a.o[b][i], a.o[b][i + 1], a.o[b][i + 2], a.o[b][i + 3]};
        *(f32x4*)(po + part_at<D>(slot, rows, s.ntok * A.g.G, row0 + n, 8 * b + key_of(i, h) / 4)) = y;
      }
    if (h == 0) pml[(int64_t)slot * rows + row0 + n] = make_float4(a.m, l, lr, 0.0f);
    return;
  }
  const bool none = x.row.pos < 0;
  const float f = none ? 0.0f : 1.0f / lr;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      uint32_t w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float y0 = none ? 0.0f : a.o[b][i + 2 * j] * f;
        const float y1 = none ? 0.0f : a.o[b][i + 2 * j + 1] * f;
        w[j] = Elem<BF>::one(y0) | (uint32_t)Elem<BF>::one(y1) << 16;
      }
      *(uint2*)(tmp + n * kRowK<D> + (32 * b + key_of(i, h)) * 2) = make_uint2(w[0], w[1]);
    }
  if (A.lse && x.real && h == 0) {
    const float m = a.m == -__builtin_inff() ? 0.0f : a.m;
    A.lse[(int64_t)x.tok * A.g.hq + x.qh] = none ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
  wave_order();
  const int have = s.ntok * A.g.G - row0;
  for (int r = lane / (D / 8); r < 32 && r < have; r += 512 / D) {
    const uint4 y = *(const uint4*)(tmp + r * kRowK<D> + lane % (D / 8) * 16);
    const int t = (row0 + r) / A.g.G, g = row0 + r - t * A.g.G;
    *(uint4*)((uint16_t*)A.out + ((int64_t)(s.q0 + t) * A.g.hq + s.head * A.g.G + g) * D + lane % (D / 8) * 8) = y;
  }
}

// The result of a query tile without keys, by `threads` threads: zeros.
template <int D>
__device__ __forceinline__ void blank(const KvAttendArgs& A, const KvSeg& s, int tid, int threads) {
  for (int i = tid; i < s.ntok * A.g.G * (D / 8); i += threads) {
    const int r = i / (D / 8), t = r / A.g.G;
    const int64_t at = (int64_t)(s.q0 + t) * A.g.hq + s.head * A.g.G + r - t * A.g.G;
    *(uint4*)((uint16_t*)A.out + at * D + i % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
    if (A.lse && i % (D / 8) == 0) A.lse[at] = -__builtin_inff();
  }
}

// First key of tile t.
template <int K>
__device__ __forceinline__ int tile_key(const KvSeg& s, int t) {
  return (t < s.ns ? t : s.fw + t - s.ns) * K;
}

// Rows of K and V on their way from the pages into LDS: `I` loads of 16 bytes for each.
template <bool BF, bool F8, int D, int I, int LANES>
struct Stage {
  static constexpr int kChunks = F8 ? D / 16 : D / 8;  // 16-byte chunks of a row in memory
  static constexpr int kStep = LANES / kChunks;        // rows of one load
  uint4 k[I], v[I];
  uint32_t ks[F8 ? I : 1], vs[F8 ? I : 1];             // their exponents (wide tiles)

  // 16 bytes, `at` bytes past the start of a row of the pool
  static __device__ __forceinline__ uint4 load(const char* pool, uint32_t row, uint32_t at) {
    return *(const uint4*)(pool + (uint64_t)row * (kChunks * 16) + at);
  }
  // 16-bit chunk j (of 2 with 8-bit codes) of 16 bytes in memory; s: the row's scale
  static __device__ __forceinline__ uint4 widen(const uint4& x, float s, int j) {
    if (!F8) return x;
    const uint32_t a = j ? x.z : x.x, b = j ? x.w : x.y;
    uint4 o;
    o.x = Elem<BF>::pair(a, s, false);
    o.y = Elem<BF>::pair(a, s, true);
    o.z = Elem<BF>::pair(b, s, false);
    o.w = Elem<BF>::pair(b, s, true);
    return o;
  }
  // Puts load i, row r of the tile, into LDS.
  __device__ __forceinline__ void put_k(char* kt, int i, int r, int c, float scale) const {
#pragma unroll
    for (int j = 0; j < (F8 ? 2 : 1); ++j)
      *(uint4*)(kt + r * kRowK<D> + (F8 ? 2 * c + j : c) * 16) = widen(k[i], scale, j);
  }
  // The same.  MASKED, where rows of the query tile see different keys: a V row from `end` on,
  // which none sees, is cleared, and so are infinities and NaN of the others: in the product they
  // would reach rows that do not see them, as 0 * inf.  Returns whether there were any
  // (spread() adds them).
  template <bool MASKED>
  __device__ __forceinline__ bool put_v(char* vt, int i, int r, int c, int end, float scale) const {
    bool bad = false;
#pragma unroll
    for (int j = 0; j < (F8 ? 2 : 1); ++j) {
      uint4 y = widen(v[i], scale, j);
      if (MASKED) {
        if (r >= end) y = make_uint4(0, 0, 0, 0);
        bad |= clean<BF>(y);
      }
      *(uint4*)(vt + r * kRowV<D> + (F8 ? 2 * c + j : c) * 16) = y;
    }
    return bad;
  }
};

__device__ __forceinline__ float scale_of(uint32_t exp) { return __uint_as_float((exp & 0xff) << 23); }

// First row of a page in the pool; for a page outside it sets `lost` and takes page 0.
__device__ __forceinline__ uint32_t page_at(const KvAttendArgs& A, int32_t page, bool& lost) {
  const bool in = (uint32_t)page < A.pool.n_blocks;
  lost |= !in;
  return (in ? (uint32_t)page : 0u) * ((uint32_t)A.g.hkv << A.g.sh);
}

// Row of key j in its page, of a kv head.  Keys past the last one that the table has are
// read from the last page: rows of the pool, of which no use is made.
__device__ __forceinline__ uint32_t in_page(const KvAttendArgs& A, int head, int j) {
  return ((uint32_t)head << A.g.sh) + (uint32_t)(j & ((1 << A.g.sh) - 1));
}

// Whether some rows at positions p0 .. last may not see all the K keys from kb on: these
// reach past the first row's position or before the last row's window.
__device__ __forceinline__ bool is_masked(const KvAttendArgs& A, int p0, int last, int kb, int K) {
  return kb + K - 1 > p0 || (A.window && kb <= last - A.window && kb + K > A.sinks);
}

// Whether V has infinities or NaN in the K keys from kb on, up to key `last` (16-bit rows).
template <bool BF, int D, int K>
__device__ __forceinline__ bool odd_tile(const KvAttendArgs& A, const KvSeg& s, int lane, int kb, int last) {
  constexpr int kChunks = D / 8;  // 16-byte chunks of a row
  uint32_t m = 0;
  bool lost = false;  // reported before
  for (int j = kb + lane / kChunks; j < kb + K && j <= last; j += 64 / kChunks) {
    const uint32_t row = page_at(A, A.table[(int64_t)s.seq * A.cols + (j >> A.g.sh)], lost) + in_page(A, s.head, j);
    m = max16(m, top_pair(*(const uint4*)((const char*)A.pool.v + (uint64_t)row * (D * 2) + lane % kChunks * 16)));
  }
  return __any(top_half(m) >= kInf<BF>);
}

// Adds what clean() took out of V to the rows that see it, in the result or the partial sums that
// the wave has just written: w * inf is inf whatever the weight w.  That was in the stretch's
// masked tiles, or in ANY.  `row0`: the wave's first row in the query tile.
template <bool BF, bool F8, int D, int K, bool ANY>
__device__ __forceinline__ void spread(const KvAttendArgs& A, const KvSeg& s, int lane, int row0, int rows,
                                       float* po) {
  lane = here(lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  const int last = s.p0 + s.ntok - 1, G = A.g.G;
  for (int t = s.t0; t < s.t1; ++t) {
    const int kb = tile_key<K>(s, t);
    if (ANY ? !odd_tile<BF, D, K>(A, s, lane, kb, last) : !is_masked(A, s.p0, last, kb, K)) continue;
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
          const int u = n / G, pos = s.p0 + u;
          const Row r{pos, A.window ? pos - A.window : -1, A.sinks};
          if (!r.sees(j)) continue;
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
  if (a.n_wide) {
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
  if (a.n_join && a.most_parts > 8)
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
