// N adjacent values of a row, as stored: loaded and stored at once (2 to 16 bytes), read and rounded one by one.
#pragma once

#include "dp_internal.h"

namespace dpbk {

template <int DT, int N>
struct Values {
  static constexpr int SIZE = DT == DP_F32 ? 4 : 2, BYTES = N * SIZE;
  static_assert(BYTES == 2 || BYTES == 4 || BYTES == 8 || BYTES == 16, "one access");
  typedef __attribute__((ext_vector_type(BYTES >= 4 ? BYTES / 4 : 1))) uint32_t Words;
  union {
    Words w;
    uint32_t word[BYTES >= 4 ? BYTES / 4 : 1];
  };
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const char* p = static_cast<const char*>(base) + at * SIZE;
    if constexpr (BYTES == 2)
      word[0] = *reinterpret_cast<const uint16_t*>(p);
    else
      w = *reinterpret_cast<const Words*>(p);
  }
  __device__ __forceinline__ void store(void* base, int64_t at) const {
    char* p = static_cast<char*>(base) + at * SIZE;
    if constexpr (BYTES == 2)
      *reinterpret_cast<uint16_t*>(p) = (uint16_t)word[0];
    else
      *reinterpret_cast<Words*>(p) = w;
  }
  __device__ __forceinline__ float get(int k) const {
    if constexpr (DT == DP_F32) return __uint_as_float(word[k]);
    const uint32_t pair = word[k / 2];
    if constexpr (DT == DP_BF16) return __uint_as_float(k & 1 ? pair & 0xFFFF0000u : pair << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(k & 1 ? pair >> 16 : pair & 0xFFFFu));
  }
  // Rounded to nearest even.
  __device__ __forceinline__ void set(const float (&x)[N]) {
    if constexpr (DT == DP_F32) {
#pragma unroll
      for (int k = 0; k < N; ++k) word[k] = __float_as_uint(x[k]);
    } else {
      typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
      typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
#pragma unroll
      for (int k = 0; k < N; k += 2) {
        const float lo = x[k], hi = k + 1 < N ? x[k + 1 < N ? k + 1 : k] : 0.f;
        if constexpr (DT == DP_BF16)
          word[k / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
        else
          word[k / 2] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)lo, (_Float16)hi});
      }
    }
  }
};

}  // namespace dpbk
