// kv_pages.hip -- rows into and out of the pages of a key/value cache.
//
//   k_kv_append  one thread per 16 bytes of a new token's K row and of its V row.  A
//                16-bit cache takes the row as it is.  An 8-bit cache takes e4m3 codes of
//                x * 2^-k, k the least integer that brings the row's largest finite
//                magnitude to 448 at most (amax = m * 2^f, 1/2 <= m < 1: k = f - 9, one
//                more where m > 7/8), so the scale is exact and the only rounding is that
//                to 3 fraction bits, to nearest even; infinities and NaN become NaN.
//   k_kv_read    the rows of the batch's tokens back as 16-bit values; code * 2^k needs
//                4 significant bits, so this is exact.
// Bound by the bytes of the rows.  The D/8 threads of a row sit in one wave.
#include "../../include/lar.h"
#include "kv_device.h"

namespace lar {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

// Row index of (page, head, row) in units of rows, or -1 with the sticky error for a page
// outside the pool.
__device__ __forceinline__ int64_t page_row(const KvGeom& g, const KvPool& pool, int32_t page,
                                            int head, int pos, int32_t* err) {
  if ((uint32_t)page >= pool.n_blocks) {
    *err = LAR_E_STATE;
    return -1;
  }
  return (((int64_t)page * g.hkv + head) << g.sh) + (pos & ((1 << g.sh) - 1));
}

template <bool BF>
__device__ __forceinline__ float lo16(uint32_t w) {
  if (BF) return __uint_as_float(w << 16);
  return (float)__builtin_bit_cast(f16x2, w)[0];
}
template <bool BF>
__device__ __forceinline__ float hi16(uint32_t w) {
  if (BF) return __uint_as_float(w & 0xffff0000u);
  return (float)__builtin_bit_cast(f16x2, w)[1];
}

// e4m3 codes of the 8 values of this thread; the row lies in `lanes` (8 or 16) threads.
template <bool BF>
__device__ __forceinline__ uint2 quantise(const uint4& x, int lanes, int* exp_out) {
  const float held = BF ? 0x1.ep+127f : 61440.0f;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  float f[8];
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = lo16<BF>(w[i]);
    f[2 * i + 1] = hi16<BF>(w[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = __builtin_fabsf(f[i]);
    if (a < __builtin_inff()) {  // finite: held to what the 16-bit type takes back
      f[i] = __builtin_copysignf(fminf(a, held), f[i]);
      amax = fmaxf(amax, fminf(a, held));
    } else {
      f[i] = __builtin_nanf("");
    }
  }
  for (int m = 1; m < lanes; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
  int e;
  const float mant = frexpf(amax, &e);
  int k = e - 9 + (mant > 0.875f ? 1 : 0);
  k = k < kKvExpMin ? kKvExpMin : k > kKvExpMax ? kKvExpMax : k;
  *exp_out = k + 127;
  const float s = __uint_as_float((uint32_t)(127 - k) << 23);
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * s, f[1] * s, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * s, f[3] * s, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * s, f[5] * s, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * s, f[7] * s, hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

template <bool BF>
__device__ __forceinline__ uint4 dequantise(uint2 c, uint32_t exp) {
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

template <bool F8, bool BF>
__global__ __launch_bounds__(256) void k_kv_append(KvCopyArgs A) {
  const int lanes = A.g.D >> 3;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = x / lanes;  // (token, head)
  const int c = (int)(x - r * lanes);
  const int64_t t = r / A.g.hkv;
  const int head = (int)(r - t * A.g.hkv);
  if (t >= A.n_tok) return;
  const KvTok tok = A.tok[t];
  if (tok.pos < 0) return;
  const int32_t page = A.table[(int64_t)tok.seq * A.cols + (tok.pos >> A.g.sh)];
  const uint4 k = *(const uint4*)((const uint16_t*)A.k.p + t * A.k.tok + head * A.k.head + c * 8);
  const uint4 v = *(const uint4*)((const uint16_t*)A.v.p + t * A.v.tok + head * A.v.head + c * 8);
  const int64_t row = page_row(A.g, A.pool, page, head, tok.pos, A.err);
  if (row < 0) return;
  if (F8) {
    int ke, ve;
    const uint2 kc = quantise<BF>(k, lanes, &ke), vc = quantise<BF>(v, lanes, &ve);
    ((uint2*)A.pool.k)[row * lanes + c] = kc;
    ((uint2*)A.pool.v)[row * lanes + c] = vc;
    if (c == 0) {
      ((uint8_t*)A.pool.ke)[row] = (uint8_t)ke;
      ((uint8_t*)A.pool.ve)[row] = (uint8_t)ve;
    }
  } else {
    ((uint4*)A.pool.k)[row * lanes + c] = k;
    ((uint4*)A.pool.v)[row * lanes + c] = v;
  }
}

template <bool F8, bool BF>
__global__ __launch_bounds__(256) void k_kv_read(KvCopyArgs A) {
  const int lanes = A.g.D >> 3;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = x / lanes;
  const int c = (int)(x - r * lanes);
  const int64_t t = r / A.g.hkv;
  const int head = (int)(r - t * A.g.hkv);
  if (t >= A.n_tok) return;
  const KvTok tok = A.tok[t];
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  if (tok.pos >= 0) {
    const int32_t page = A.table[(int64_t)tok.seq * A.cols + (tok.pos >> A.g.sh)];
    const int64_t row = page_row(A.g, A.pool, page, head, tok.pos, A.err);
    if (row >= 0) {
      if (F8) {
        k = dequantise<BF>(((const uint2*)A.pool.k)[row * lanes + c], A.pool.ke[row]);
        v = dequantise<BF>(((const uint2*)A.pool.v)[row * lanes + c], A.pool.ve[row]);
      } else {
        k = ((const uint4*)A.pool.k)[row * lanes + c];
        v = ((const uint4*)A.pool.v)[row * lanes + c];
      }
    }
  }
  *(uint4*)((uint16_t*)A.k.p + t * A.k.tok + head * A.k.head + c * 8) = k;
  *(uint4*)((uint16_t*)A.v.p + t * A.v.tok + head * A.v.head + c * 8) = v;
}

template <class Launch>
hipError_t launch(const KvCopyArgs& a, Launch go) {
  const int64_t n = (int64_t)a.n_tok * a.g.hkv * (a.g.D / 8);
  go(dim3((unsigned)((n + 255) / 256)));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const KvCopyArgs& a, hipStream_t stream) {
  return launch(a, [&](dim3 n) {
    if (a.g.cache != kKvE4m3)
      k_kv_append<false, false><<<n, 256, 0, stream>>>(a);
    else if (a.g.dtype == kKvBf16)
      k_kv_append<true, true><<<n, 256, 0, stream>>>(a);
    else
      k_kv_append<true, false><<<n, 256, 0, stream>>>(a);
  });
}

hipError_t launch_kv_read(const KvCopyArgs& a, hipStream_t stream) {
  return launch(a, [&](dim3 n) {
    if (a.g.cache != kKvE4m3)
      k_kv_read<false, false><<<n, 256, 0, stream>>>(a);
    else if (a.g.dtype == kKvBf16)
      k_kv_read<true, true><<<n, 256, 0, stream>>>(a);
    else
      k_kv_read<true, false><<<n, 256, 0, stream>>>(a);
  });
}

}  // namespace lar
