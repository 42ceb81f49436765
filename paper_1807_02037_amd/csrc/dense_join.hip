// Joins the sums of the splits of a reduction, in order, and does what the epilogue of an unsplit product does.
#include <hip/hip_runtime.h>

#include "dense.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

// Eight columns of a row a thread, the loads of four splits in flight.
template <typename T, int MODE>
__global__ __launch_bounds__(64) void dense_join_kernel(DenseP p) {
  const int vpr = (p.N + 7) / 8;                                  // vectors of a row
  const long long i = (long long)blockIdx.x * 64 + threadIdx.x, v0 = i / vpr;
  const int n = (int)(i - v0 * vpr) * 8, cnt = p.N - n < 8 ? p.N - n : 8;
  const int src = MODE == DENSE_DW ? (int)(v0 / p.M) : 0;         // DW: the rows of one source, then of the other
  const long long row = v0 - src * p.M;
  if (src >= (MODE == DENSE_DW ? p.srcs : 1) || row >= p.M) return;
  const long long plane = p.M * p.N, split = plane * p.srcs;
  const float* at = p.part + src * plane + row * p.N + n;
  auto plus = [](float a, float c) {                              // Q8: sums of 32 bits in the place of floats
    if constexpr (dense_q8(MODE)) return __int_as_float(__float_as_int(a) + __float_as_int(c));
    else return a + c;
  };
  auto add = [&](const float* q, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    int s = 0;
    for (; s + 4 <= p.splits; s += 4) {
      float t[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) load8(q + (s + u) * split, cnt, t[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = plus(v[e], t[u][e]);
    }
    for (; s < p.splits; ++s) {
      float t[8];
      load8(q + s * split, cnt, t);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = plus(v[e], t[e]);
    }
  };
  float v[8], u[8], b[8], r[8], w[8];
  dense_bias8<MODE>(p, n, cnt, b);
  dense_scales8<MODE>(p, n, cnt, w);
  const float scale = dense_scale<MODE>(p, row);
  dense_beside8<T, MODE>(p, row, n, cnt, r);
  add(at, v);
  if constexpr (MODE == DENSE_GATED) add(at + plane, u);
  dense_scaled8<MODE>(scale, w, v);
  dense_finish8<T, MODE>(p, src, row, n, cnt, v, u, b, r);
}

template <typename T, int MODE>
hipError_t launch_join(DenseP& p, hipStream_t s) {
  const long long vectors = (long long)((p.N + 7) / 8) * p.M * (MODE == DENSE_DW ? p.srcs : 1);
  if (vectors > 0xffffff00LL) return hipErrorInvalidValue;        // a grid holds less than 2^32 threads; results this large are not split
  hipLaunchKernelGGL((dense_join_kernel<T, MODE>), dim3((unsigned)((vectors + 63) / 64)), dim3(64), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t dense_join(int mode, bool f32, DenseP& p, hipStream_t s) {
  switch (mode) {
    case DENSE_FWD: return f32 ? launch_join<float, DENSE_FWD>(p, s) : launch_join<uint16_t, DENSE_FWD>(p, s);
    case DENSE_GATED: return f32 ? launch_join<float, DENSE_GATED>(p, s) : launch_join<uint16_t, DENSE_GATED>(p, s);
    case DENSE_DX: return f32 ? launch_join<float, DENSE_DX>(p, s) : launch_join<uint16_t, DENSE_DX>(p, s);
    case DENSE_Q8: return launch_join<uint16_t, DENSE_Q8>(p, s);
    case DENSE_Q8_F32: return launch_join<float, DENSE_Q8_F32>(p, s);
    default: return f32 ? launch_join<float, DENSE_DW>(p, s) : launch_join<uint16_t, DENSE_DW>(p, s);
  }
}

}  // namespace lms
