// kv_pages.hip -- rows into and out of the pages of a key/value cache.
//
//   k_kv_append  one thread per 16 bytes of a new token's K row and of its V row.  A
//                16-bit cache takes the row as it is.  An 8-bit cache takes e4m3 codes of
//                x * 2^-k, k the least integer that brings the row's largest finite
//                magnitude to 448 at most, so the scale is exact and the only rounding is
//                that to 3 fraction bits, to nearest even; infinities and NaN become NaN.
//   k_kv_read    the rows of the batch's tokens back as 16-bit values; code * 2^k needs
//                4 significant bits, so this is exact.
// Bound by the bytes of the rows.  The D/8 threads of a row sit in one wave; magnitudes are
// compared as the bits of their 16-bit patterns, K's and V's in one word, over the row by
// lane permutations, and the codes come from the conversion that takes a power of two along.
#include "../../include/lar.h"
#include "kv_device.h"
#include "kv_words.h"

namespace lar {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) short s16x2;

// Pattern of the largest magnitude that is held: its code times its scale is the largest such
// value that the 16-bit type has.
template <bool BF> constexpr uint32_t kHeld = BF ? 0x7f70u : 0x7b80u;  // 1.875 * 2^127, 61440

// Row of (page, head, position) in the pool, or -1 with the sticky error for a page outside.
__device__ __forceinline__ int64_t page_row(const KvGeom& g, const KvPool& pool, int32_t page,
                                            int head, int pos, int32_t* err) {
  if ((uint32_t)page >= pool.n_blocks) {
    *err = kKvLostPage;
    return -1;
  }
  return (((int64_t)page * g.hkv + head) << g.sh) + (pos & ((1 << g.sh) - 1));
}

// The largest pattern of 8 magnitudes.
__device__ __forceinline__ uint32_t top(const uint4& x) { return top_half(top_pair(x)); }

// Whether the device has another plan now than the launch was made for.
__device__ __forceinline__ bool other_plan(const KvCopyArgs& A) {
  if (*A.plan.now == A.plan.id) return false;
  *A.err = kKvOtherPlan;
  return true;
}

// The larger of both halves of a word over the 8 or 16 lanes of a row.
template <int LANES>
__device__ __forceinline__ uint32_t top_of_row(uint32_t m) {
  m = max16(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, false));   // lane ^ 1
  m = max16(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, false));   // lane ^ 2
  m = max16(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, false));  // 7 - lane, of 8
  if (LANES == 16) m = max16(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xf, 0xf, false));
  return m;
}

// Values that are not finite to NaN, and what is too large to what is held; the largest
// finite pattern.
template <bool BF>
__device__ uint32_t hold(uint4& x) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w}, most = 0;
  for (int i = 0; i < 8; ++i) {
    const int sh = 16 * (i & 1);
    uint32_t v = w[i >> 1] >> sh & 0xffffu, a = v & 0x7fffu;
    if (a >= kInf<BF>) {
      v |= 0x7fffu;
    } else {
      a = a < kHeld<BF> ? a : kHeld<BF>;
      v = (v & 0x8000u) | a;
      most = most < a ? a : most;
    }
    w[i >> 1] = (w[i >> 1] & ~(0xffffu << sh)) | v << sh;
  }
  x = make_uint4(w[0], w[1], w[2], w[3]);
  return most;
}

// The least k with magnitude <= 448 * 2^k, within its bounds; a row of zeros has -9.
template <bool BF>
__device__ __forceinline__ int exponent(uint32_t pattern) {
  const float f = BF ? __uint_as_float(pattern << 16) : (float)__builtin_bit_cast(f16x2, pattern)[0];
  const uint32_t b = __float_as_uint(f);
  if (b == 0) return -9;
  const int k = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
  return k < kKvExpMin ? kKvExpMin : k > kKvExpMax ? kKvExpMax : k;
}

// e4m3 codes of x * 2^-k.
template <bool BF>
__device__ __forceinline__ uint2 codes(const uint4& x, int k) {
  const float s = __uint_as_float((uint32_t)(k + 127) << 23);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  s16x2 c[2] = {{0, 0}, {0, 0}};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (BF)
      c[i >> 1] = i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c[i >> 1], __builtin_bit_cast(bf16x2, w[i]), s, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c[i >> 1], __builtin_bit_cast(bf16x2, w[i]), s, false);
    else
      c[i >> 1] = i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c[i >> 1], __builtin_bit_cast(f16x2, w[i]), s, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(c[i >> 1], __builtin_bit_cast(f16x2, w[i]), s, false);
  return make_uint2(__builtin_bit_cast(uint32_t, c[0]), __builtin_bit_cast(uint32_t, c[1]));
}

template <bool BF>
__device__ __forceinline__ uint4 values(uint2 c, uint32_t exp) {
  const float s = __uint_as_float(exp << 23);
  uint4 o;
  if (BF) {
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, s, false));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, s, true));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, s, false));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, s, true));
  } else {
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.x, s, false));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.x, s, true));
    o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.y, s, false));
    o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c.y, s, true));
  }
  return o;
}

// A thread's place: token, head and 16-byte chunk (tokens * heads <= 2^27).
struct Place {
  uint32_t t, head, c;
  const void *k, *v;
  __device__ __forceinline__ Place(const KvCopyArgs& A, int lanes) {
    const uint32_t x = blockIdx.x * 256 + threadIdx.x, r = x / lanes;
    c = x % lanes;
    t = r / (uint32_t)A.g.hkv;
    head = r - t * (uint32_t)A.g.hkv;
    k = (const uint16_t*)A.k.p + (int64_t)t * A.k.tok + (int64_t)head * A.k.head + c * 8;
    v = (const uint16_t*)A.v.p + (int64_t)t * A.v.tok + (int64_t)head * A.v.head + c * 8;
  }
};

template <bool F8, bool BF, int LANES>
__global__ __launch_bounds__(256) void k_kv_append(KvCopyArgs A) {
  const Place at(A, LANES);
  if (at.t >= (uint32_t)A.n_tok) return;
  const KvTok tok = A.tok[at.t];
  if (other_plan(A)) return;
  if (tok.pos < 0) return;
  const int32_t page = A.table[(int64_t)tok.seq * A.cols + (tok.pos >> A.g.sh)];
  uint4 k = *(const uint4*)at.k, v = *(const uint4*)at.v;
  const int64_t row = page_row(A.g, A.pool, page, at.head, tok.pos, A.err);
  if (row < 0) return;
  if (F8) {
    uint32_t m = top_of_row<LANES>(top(k) | top(v) << 16);
    if ((m & 0xffffu) > kHeld<BF> || m >> 16 > kHeld<BF>) {  // the row's threads go together
      const uint32_t mk = hold<BF>(k), mv = hold<BF>(v);
      m = top_of_row<LANES>(mk | mv << 16);
    }
    const int ke = exponent<BF>(m & 0xffffu), ve = exponent<BF>(m >> 16);
    ((uint2*)A.pool.k)[row * LANES + at.c] = codes<BF>(k, ke);
    ((uint2*)A.pool.v)[row * LANES + at.c] = codes<BF>(v, ve);
    if (at.c == 0) {
      ((uint8_t*)A.pool.ke)[row] = (uint8_t)(ke + 127);
      ((uint8_t*)A.pool.ve)[row] = (uint8_t)(ve + 127);
    }
  } else {
    ((uint4*)A.pool.k)[row * LANES + at.c] = k;
    ((uint4*)A.pool.v)[row * LANES + at.c] = v;
  }
}

template <bool F8, bool BF, int LANES>
__global__ __launch_bounds__(256) void k_kv_read(KvCopyArgs A) {
  const Place at(A, LANES);
  if (at.t >= (uint32_t)A.n_tok) return;
  const KvTok tok = A.tok[at.t];
  if (other_plan(A)) return;
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  if (tok.pos >= 0) {
    const int32_t page = A.table[(int64_t)tok.seq * A.cols + (tok.pos >> A.g.sh)];
    const int64_t row = page_row(A.g, A.pool, page, at.head, tok.pos, A.err);
    if (row >= 0) {
      if (F8) {
        k = values<BF>(((const uint2*)A.pool.k)[row * LANES + at.c], A.pool.ke[row]);
        v = values<BF>(((const uint2*)A.pool.v)[row * LANES + at.c], A.pool.ve[row]);
      } else {
        k = ((const uint4*)A.pool.k)[row * LANES + at.c];
        v = ((const uint4*)A.pool.v)[row * LANES + at.c];
      }
    }
  }
  *(uint4*)at.k = k;
  *(uint4*)at.v = v;
}

template <int LANES>
void append(const KvCopyArgs& a, unsigned n, hipStream_t stream) {
  if (a.g.cache != kKvE4m3)
    k_kv_append<false, false, LANES><<<n, 256, 0, stream>>>(a);
  else if (a.g.dtype == kKvBf16)
    k_kv_append<true, true, LANES><<<n, 256, 0, stream>>>(a);
  else
    k_kv_append<true, false, LANES><<<n, 256, 0, stream>>>(a);
}

template <int LANES>
void read(const KvCopyArgs& a, unsigned n, hipStream_t stream) {
  if (a.g.cache != kKvE4m3)
    k_kv_read<false, false, LANES><<<n, 256, 0, stream>>>(a);
  else if (a.g.dtype == kKvBf16)
    k_kv_read<true, true, LANES><<<n, 256, 0, stream>>>(a);
  else
    k_kv_read<true, false, LANES><<<n, 256, 0, stream>>>(a);
}

unsigned blocks(const KvCopyArgs& a) {
  return (unsigned)(((int64_t)a.n_tok * a.g.hkv * (a.g.D / 8) + 255) / 256);
}

}  // namespace

hipError_t launch_kv_append(const KvCopyArgs& a, hipStream_t stream) {
  if (a.g.D == 128)
    append<16>(a, blocks(a), stream);
  else
    append<8>(a, blocks(a), stream);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvCopyArgs& a, hipStream_t stream) {
  if (a.g.D == 128)
    read<16>(a, blocks(a), stream);
  else
    read<8>(a, blocks(a), stream);
  return hipGetLastError();
}

}  // namespace lar
