// kv_attend.h -- what the kernels that attend over the pages of a key/value cache have in common
// (kv_attend.hip, where the mathematics are described, kv_tree.hip, kv_weigh.hip).
#ifndef LAR_KV_ATTEND_H
#define LAR_KV_ATTEND_H

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

}  // namespace
}  // namespace lar

#endif  // LAR_KV_ATTEND_H
