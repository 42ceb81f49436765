// Rows of channels, four to a thread: shared by the sequence operators (internal).
#pragma once
#include "dense.hpp"
#include "graph.hpp"

namespace lms {
namespace {

constexpr int V = 4;                   // channels of a thread

template <typename T>
__device__ __forceinline__ void store4(T* p, int cnt, const float (&v)[V]) {
  if constexpr (sizeof(T) == 2) {
    const v2u q = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    if (cnt >= V) { __builtin_memcpy(p, &q, 8); return; }
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < cnt) p[e] = (T)(q[e >> 1] >> ((e & 1) * 16));
  } else {
    if (cnt >= V) { __builtin_memcpy(p, v, 16); return; }
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < cnt) p[e] = v[e];
  }
}
__device__ __forceinline__ void load4(const float* p, int cnt, float (&v)[V]) {
  if (cnt >= V) { __builtin_memcpy(v, p, 16); return; }
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < cnt ? p[e] : 0.f;
}

#define NEED(cond, ...)        \
  do {                         \
    if (!(cond)) {             \
      set_error(__VA_ARGS__);  \
      return LMS_EINVAL;       \
    }                          \
  } while (0)

inline uint64_t up256(uint64_t b) { return (b + 255) / 256 * 256; }
inline lms_status done(const char* what, hipError_t e) {
  if (e == hipSuccess) return LMS_OK;
  set_error("%s: %s", what, hipGetErrorString(e));
  return LMS_EHIP;
}

}  // namespace
}  // namespace lms
