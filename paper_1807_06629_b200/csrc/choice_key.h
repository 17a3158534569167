// Order of the logits where the k largest of a row are taken one after the other: the fp32 order in the upper half (NaN above every
// number, -0 = +0), then the index, lower ones above.  Every key is above 0 and below kChoiceAll, so that "below the choice before"
// can start there and as many choices as there are logits can be made: a NaN at index 0 included.  Host code may include it.
#pragma once
#include <cstdint>
#ifdef __CUDACC__
#define PRSGD_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define PRSGD_HOST_DEVICE inline
#endif

namespace prsgd {

constexpr unsigned long long kChoiceAll = ~0ull;
// `bits`: of the logit as fp32
PRSGD_HOST_DEVICE unsigned long long choice_key(uint32_t bits, uint32_t index) {
  const uint32_t size = bits & 0x7FFFFFFFu;
  const uint32_t order = size > 0x7F800000u ? 0xFFFFFFFFu : size == 0u ? 0x80000000u : (bits & 0x80000000u) ? ~bits : bits | 0x80000000u;
  return ((unsigned long long)order << 32) | (0xFFFFFFFEu - index);
}
PRSGD_HOST_DEVICE uint32_t choice_index(unsigned long long key) { return 0xFFFFFFFEu - (uint32_t)key; }

}  // namespace prsgd
