// Matrix products of language-model layers: parameters, activations and epilogue shared by their kernels (internal).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "conv_tile.hpp"
#include "lms.h"

namespace lms {

// One launch of a product.  Rows i, columns j, reduction index r:
//   DENSE_FWD    out[i][j] = act(sum_r a[i][r] b[r][j] + bias[j]) + res[i][j]; pre[i][j] = the argument of act
//   DENSE_GATED  g = sum_r a[i][r] b0[r][j], u = sum_r a[i][r] b1[r][j]; out = act(g) u; pre, pre1 = g, u.
//                With dh: out, pre1 = dh u act'(g), dh act(g) instead (the gradients of g and u)
//   DENSE_DX     out[i][j] = sum over segments and r of a_s[i][r] b_s[j][r]
//   DENSE_DW     out_s[i][j] = sum_r a[r][i] b_s[r][j] for each source s
enum { DENSE_FWD = 0, DENSE_GATED = 1, DENSE_DX = 2, DENSE_DW = 3 };

struct DenseP {
  const void* a[2];            // operands of the segments (DX), or a[0]
  const void* b[2];            // of the segments (DX) or the sources (GATED, DW)
  void* out[2];                // of the sources (DW), or out[0]
  const float* bias;
  const void* res;
  const void* dh;
  void *pre, *pre1;
  long long M, lda, ldb, ldo, ldr;     // ldr: res and dh; pre and pre1 lie as out
  long long red;               // reduction extent of a segment
  int N;
  int segs, srcs;              // segments of the reduction (1 or 2); sources of columns (1, or 2: GATED, DW)
  int act;
  int out_f32;                 // DW: out is fp32 (else the storage type)
  int splits, stages_per_split, stages;   // the reduction's stages, segments one after the other
  int ntm, ntn, ntiles;
  float* part;                 // splits > 1: sums of a split, [split][source][M][N]
};

// The product by whichever kernel suits (dense_layers.hip): p holds everything up to out_f32, and part, of dense_ws bytes (a function of the sizes alone).
hipError_t dense_product(int mode, bool f32, DenseP& p, hipStream_t s);
uint64_t dense_ws(int mode, bool f32, long long M, int N, long long red, int segs, int srcs);

hipError_t dense_bf16(int mode, DenseP& p, hipStream_t s);        // dense_gemm.hip
uint64_t dense_bf16_ws(int mode, long long M, int N, long long red, int segs, int srcs);
uint64_t dense_f32_ws(int mode, long long M, int N, long long red, int segs, int srcs);
hipError_t dense_f32(int mode, DenseP& p, hipStream_t s);         // dense_f32.hip
hipError_t dense_join(int mode, bool f32, DenseP& p, hipStream_t s);        // dense_join.hip: p.part into the results
bool dense_few_ok(int mode, long long M);                         // few rows (dense_few.hip)
uint64_t dense_few_ws(int mode, bool f32, long long M, int N, long long red);
hipError_t dense_few(int mode, bool f32, DenseP& p, hipStream_t s);

namespace {

// act(v) and act'(v) by the definitions.  exp(x) as 2^(x log2 e) in one instruction and the reciprocal's instruction are each within an ulp, far below
// the rounding of a 16-bit result; for 32 bits the product of x and log2 e adds |x| 2^-24, which counts only where the sigmoid vanishes.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f)); }
constexpr float GELU_A = 0.7978845608028654f, GELU_B = 0.044715f;     // sqrt(2 / pi) and the cubic term of the tanh form

template <int ACT>
__device__ __forceinline__ void act_one(float v, float& value, float& slope) {
  value = v;
  slope = 1.f;
  if constexpr (ACT == LMS_ACT_RELU) { value = v > 0.f ? v : 0.f; slope = v > 0.f ? 1.f : 0.f; }
  if constexpr (ACT == LMS_ACT_SILU) { const float s = sigmoid(v); value = v * s; slope = s + value * (1.f - s); }
  if constexpr (ACT == LMS_ACT_GELU) {
    const float cdf = 0.5f * (1.f + erff(v * 0.70710678f));
    value = v * cdf;
    slope = cdf + v * 0.3989422804f * __builtin_amdgcn_exp2f(v * v * -0.72134752f);        // the density: e^(-v^2/2) / sqrt(2 pi)
  }
  if constexpr (ACT == LMS_ACT_GELU_TANH) {                       // (1 + tanh t) / 2 = sigmoid(2 t)
    const float s = sigmoid(2.f * GELU_A * (v + GELU_B * v * v * v));
    value = v * s;
    slope = s + value * (1.f - s) * 2.f * GELU_A * (1.f + 3.f * GELU_B * v * v);
  }
}
// f(integral_constant<int, act>): one uniform branch around the arithmetic of a vector
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case LMS_ACT_RELU: f(std::integral_constant<int, LMS_ACT_RELU>{}); return;
    case LMS_ACT_SILU: f(std::integral_constant<int, LMS_ACT_SILU>{}); return;
    case LMS_ACT_GELU: f(std::integral_constant<int, LMS_ACT_GELU>{}); return;
    case LMS_ACT_GELU_TANH: f(std::integral_constant<int, LMS_ACT_GELU_TANH>{}); return;
    default: f(std::integral_constant<int, LMS_ACT_NONE>{});
  }
}
// v = act(v)
__device__ __forceinline__ void act8(int act, float (&v)[8]) {
  with_act(act, [&](auto a) {
    float slope;
#pragma unroll
    for (int e = 0; e < 8; ++e) act_one<decltype(a)::value>(v[e], v[e], slope);
  });
}
// the gradients of g and u from that of act(g) u: g = d u act'(g), u = d act(g)
__device__ __forceinline__ void gated_grad8(int act, const float (&d)[8], float (&g)[8], float (&u)[8]) {
  with_act(act, [&](auto a) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float value, slope;
      act_one<decltype(a)::value>(g[e], value, slope);
      g[e] = d[e] * u[e] * slope;
      u[e] = d[e] * value;
    }
  });
}

// Eight consecutive elements of the storage type at any address, the first cnt of them there.  Whole vectors take one 16-byte access (two
// for fp32) whatever the address: the device reads and writes global memory at any alignment.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int cnt, float (&v)[8]) {
  if (cnt >= 8) {
    if constexpr (sizeof(T) == 2) {
      v4u q;
      __builtin_memcpy(&q, p, 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((e & 1) ? (q[e >> 1] & 0xffff0000u) : (q[e >> 1] << 16));
    } else __builtin_memcpy(v, p, 32);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = 0.f;
    if (e < cnt) {
      if constexpr (sizeof(T) == 2) v[e] = bf2f(p[e]);
      else v[e] = p[e];
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int cnt, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const v4u q = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    if (cnt >= 8) { __builtin_memcpy(p, &q, 16); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cnt) p[e] = (T)(q[e >> 1] >> ((e & 1) * 16));
  } else {
    if (cnt >= 8) { __builtin_memcpy(p, v, 32); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cnt) p[e] = v[e];
  }
}

// What is done with eight sums (DENSE_GATED: of g and of u) at row i, columns n .. n+7 (cnt of them exist).  T: storage type.
template <typename T, int MODE>
__device__ __forceinline__ void dense_finish8(const DenseP& p, int src, long long i, int n, int cnt, float (&v)[8], float (&u)[8]) {
  const long long o = i * p.ldo + n;
  if constexpr (MODE == DENSE_DX) store8((T*)p.out[0] + o, cnt, v);
  if constexpr (MODE == DENSE_DW) {
    if (p.out_f32) store8((float*)p.out[src] + o, cnt, v);
    else store8((T*)p.out[src] + o, cnt, v);
  }
  if constexpr (MODE == DENSE_FWD) {
    float r[8];
    if (p.res) load8((const T*)p.res + i * p.ldr + n, cnt, r);
    if (p.bias) {
      float b[8];
      load8(p.bias + n, cnt, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += b[e];
    }
    if (p.pre) store8((T*)p.pre + o, cnt, v);
    act8(p.act, v);
    if (p.res)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    store8((T*)p.out[0] + o, cnt, v);
  }
  if constexpr (MODE == DENSE_GATED) {
    if (p.dh) {
      float d[8];
      load8((const T*)p.dh + i * p.ldr + n, cnt, d);
      gated_grad8(p.act, d, v, u);
      store8((T*)p.out[0] + o, cnt, v);
      store8((T*)p.pre1 + o, cnt, u);
    } else {
      if (p.pre) store8((T*)p.pre + o, cnt, v);
      if (p.pre1) store8((T*)p.pre1 + o, cnt, u);
      act8(p.act, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= u[e];
      store8((T*)p.out[0] + o, cnt, v);
    }
  }
}

// The sums of one split, to be added by dense_join.
__device__ __forceinline__ void dense_part8(const DenseP& p, int split, int src, long long i, int n, int cnt, const float (&v)[8]) {
  store8(p.part + (((long long)split * p.srcs + src) * p.M + i) * p.N + n, cnt, v);
}

// Epilogue of a wave's TM x TN transposed accumulators (lane l of a 32 x 32 one holds row l % 32, columns 8 * (v / 4) + 4 * (l / 32) + v % 4).  32 rows at a time go
// through the wave's own LDS, in order and so without a barrier, and leave as vectors of eight columns.  DENSE_GATED: the first half of the
// columns are of g, the second of u.  m0, n0: the wave's first row and column.
template <typename T, int MODE, int WTN, int TM, int TN>
__device__ __forceinline__ void dense_epilogue(const DenseP& p, const f32x16 (&acc)[TM][TN], unsigned char* lds, long long m0, int n0, int src, int split) {
  constexpr int LDC = WTN + 4, COLS = MODE == DENSE_GATED ? WTN / 2 : WTN, LPR = COLS / 8, RPI = 64 / LPR, QV = 32 / RPI;
  const int lane = threadIdx.x & 63, half = lane >> 5, cg = (lane % LPR) * 8;
  const int n = n0 + cg, cnt = p.N - n < 8 ? p.N - n : 8;
  float* sC = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        *reinterpret_cast<float4*>(sC + (lane & 31) * LDC + j * 32 + 8 * v + 4 * half) =
            make_float4(acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]);
#pragma unroll
    for (int q = 0; q < QV; ++q) {
      const int lr = lane / LPR + q * RPI;
      const long long row = m0 + i * 32 + lr;
      const float* at = sC + lr * LDC + cg;
      float v[8], u[8];
      auto get = [&](const float* s, float (&d)[8]) {
        const float4 lo = *reinterpret_cast<const float4*>(s), hi = *reinterpret_cast<const float4*>(s + 4);
        d[0] = lo.x; d[1] = lo.y; d[2] = lo.z; d[3] = lo.w; d[4] = hi.x; d[5] = hi.y; d[6] = hi.z; d[7] = hi.w;
      };
      get(at, v);
      if constexpr (MODE == DENSE_GATED) get(at + COLS, u);
      if (row >= p.M || cnt <= 0) continue;
      if (p.splits > 1) {
        dense_part8(p, split, src, row, n, cnt, v);
        if constexpr (MODE == DENSE_GATED) dense_part8(p, split, 1, row, n, cnt, u);
      } else dense_finish8<T, MODE>(p, src, row, n, cnt, v, u);
    }
    __builtin_amdgcn_sched_barrier(0);                            // 32 rows after the other: together they are more than the registers hold
  }
}

}  // namespace
}  // namespace lms
