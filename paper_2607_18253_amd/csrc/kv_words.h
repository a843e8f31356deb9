// kv_words.h -- 16-bit floating-point values by their patterns, two in a word.
#ifndef LAR_KV_WORDS_H
#define LAR_KV_WORDS_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace lar {

// Pattern of infinity; those of NaN are larger, finite magnitudes smaller.
template <bool BF> constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;

// The larger ones of two pairs.
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
  typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}

// The largest patterns of 8 magnitudes, of the even and of the odd ones.
__device__ __forceinline__ uint32_t top_pair(const uint4& x) {
  return max16(max16(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), max16(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
}

// The larger half of a word.
__device__ __forceinline__ uint32_t top_half(uint32_t m) { return max16(m, m >> 16) & 0xffffu; }

}  // namespace lar

#endif  // LAR_KV_WORDS_H
