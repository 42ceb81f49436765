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
//   DENSE_Q8     DENSE_FWD of 8-bit integers: the sum times sx[i] sw[j] in its place.  Both operands have the reduction in rows, two elements in each of the
//                "elements" that lda, ldb and red count; DENSE_Q8_F32: out and res are fp32.  The sums are whole numbers of 32 bits, kept as such in part
enum { DENSE_FWD = 0, DENSE_GATED = 1, DENSE_DX = 2, DENSE_DW = 3, DENSE_Q8 = 4, DENSE_Q8_F32 = 5 };
constexpr bool dense_q8(int mode) { return mode == DENSE_Q8 || mode == DENSE_Q8_F32; }

struct DenseP {
  const void* a[2];            // operands of the segments (DX), or a[0]
  const void* b[2];            // of the segments (DX) or the sources (GATED, DW)
  void* out[2];                // of the sources (DW), or out[0]
  const float* bias;
  const float *sx, *sw;        // Q8: what one step of a row of a, and of a row of b, stands for
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
  int job0, jobs;              // of ntiles * splits work-groups, those of this launch (launch_jobs)
  float* part;                 // splits > 1: sums of a split, [split][source][M][N]
};

// The product by whichever kernel suits (dense_layers.hip): p holds everything up to out_f32, and part, of dense_ws bytes (a function of the sizes alone).
hipError_t dense_product(int mode, bool f32, DenseP& p, hipStream_t s);
uint64_t dense_ws(int mode, bool f32, long long M, int N, long long red, int segs, int srcs);

hipError_t dense_bf16(int mode, DenseP& p, hipStream_t s);        // dense_gemm.hip
hipError_t dense_bf16_pair(DenseP& dx, DenseP& dw, bool& taken, hipStream_t s);
uint64_t dense_bf16_ws(int mode, long long M, int N, long long red, int segs, int srcs);
uint64_t dense_f32_ws(int mode, long long M, int N, long long red, int segs, int srcs);
hipError_t dense_f32(int mode, DenseP& p, hipStream_t s);         // dense_f32.hip
hipError_t dense_join(int mode, bool f32, DenseP& p, hipStream_t s);        // dense_join.hip: p.part into the results
bool dense_few_ok(int mode, bool f32, long long M);               // few rows (dense_few.hip)
uint64_t dense_few_ws(int mode, bool f32, long long M, int N, long long red);
hipError_t dense_few(int mode, bool f32, DenseP& p, hipStream_t s);

namespace {

// A grid holds less than 2^32 threads: the work-groups of a product, NT threads each, go in as many launches as that takes.
template <int NT, typename F>
hipError_t launch_jobs(DenseP& p, F&& launch) {
  constexpr long long most = (1LL << 31) / NT;
  const long long total = (long long)p.ntiles * p.splits;
  for (long long at = 0; at < total; at += most) {
    p.job0 = (int)at;
    p.jobs = (int)(total - at < most ? total - at : most);
    launch(dim3((unsigned)xcd_grid(p.jobs)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// A work-group's number among ntiles * splits, or -1.
__device__ __forceinline__ int dense_job(const DenseP& p) {
  const int job = xcd_order(p.jobs);
  return job < 0 ? -1 : p.job0 + job;
}

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
    // The normal distribution's tail is e^(-v^2/2) times erfcx(|v| / sqrt 2) / 2, and the density has the same exponential.  erfcx(z) = t P(t), t = 1 / (1 + 0.35 z):
    // P fitted to the function in fp64 (least squares, reweighted until the relative error was level), off by 4.4e-08 while the exponential is above 0 (|v| < 14.5).  No branches, and small tails
    // keep their relative precision, which 1 + erf loses (the device library's erf took 6 us of a 128 x 128 tile's epilogue).
    const float e = __builtin_amdgcn_exp2f(v * v * -0.72134752f), t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(v), 0.35f * 0.70710678f, 1.f));
    constexpr float C[] = {0.197466275f, 0.197472524f, 0.185208714f, 0.163207615f, 0.113303273f, 0.14348005f, -0.0894003726f, 0.222640154f, -0.174137574f, 0.0407593086f};
    float q = C[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) q = __builtin_fmaf(q, t, C[i]);
    const float tail = 0.5f * q * t * e, cdf = v < 0.f ? tail : 1.f - tail;
    value = v * cdf;
    slope = cdf + v * 0.3989422804f * e;
  }
  if constexpr (ACT == LMS_ACT_GELU_TANH) {                       // (1 + tanh t) / 2 = sigmoid(2 t)
    const float s = sigmoid(2.f * GELU_A * (v + GELU_B * v * v * v));
    value = v * s;
    slope = s + value * (1.f - s) * 2.f * GELU_A * (1.f + 3.f * GELU_B * __builtin_fminf(v * v, 1e30f));     // finite where value (1 - s) is 0
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
// AROUND: around the L2s, which the operands of neighbouring work-groups are to keep (gated forward 8192 x 4096 x 8192 934 -> 905 us).
typedef unsigned v4u_any __attribute__((ext_vector_type(4), aligned(2)));
template <bool AROUND = false, typename T>
__device__ __forceinline__ void store8(T* p, int cnt, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    const v4u q = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    if (cnt >= 8) {
      if constexpr (AROUND) __builtin_nontemporal_store(q, (v4u_any*)p);
      else __builtin_memcpy(p, &q, 16);
      return;
    }
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

// N elements as they lie in memory (as words: in an array of halves the compiler takes the loads apart).
template <typename T, int N>
struct Raw {
  unsigned q[N * sizeof(T) / 4];
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float((e & 1) ? (q[e >> 1] & 0xffff0000u) : (q[e >> 1] << 16));
    else return __uint_as_float(q[e]);
  }
};
template <int N, typename T>
__device__ __forceinline__ Raw<T, N> raw(const T* p, int cnt) {
  Raw<T, N> r;
  if (cnt >= N) { __builtin_memcpy(&r, p, sizeof(r)); return r; }
#pragma unroll
  for (unsigned& w : r.q) w = 0;
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < cnt) {
      if constexpr (sizeof(T) == 2) r.q[e >> 1] |= (unsigned)p[e] << ((e & 1) * 16);
      else r.q[e] = __float_as_uint(p[e]);
    }
  return r;
}

// The operand of the epilogue at row i, columns n ..: residual, or the gradient of act(g) u.  Loaded apart from its use, so that many can be in flight.
template <typename T, int MODE>
__device__ __forceinline__ void dense_beside8(const DenseP& p, long long i, int n, int cnt, float (&r)[8]) {
  const T* q = (const T*)(MODE == DENSE_GATED ? p.dh : p.res);
  if ((MODE == DENSE_FWD || MODE == DENSE_GATED || dense_q8(MODE)) && q) load8(q + i * p.ldr + n, cnt, r);
}
template <int MODE>
__device__ __forceinline__ void dense_bias8(const DenseP& p, int n, int cnt, float (&b)[8]) {
  if ((MODE == DENSE_FWD || dense_q8(MODE)) && p.bias) load8(p.bias + n, cnt, b);
}
// A sum of 8-bit integers into what it stands for: it is rounded to 24 bits, once, then multiplied by both scales' product.  That goes as significands and exponents: the scales' product, or the sum's
// with one of them, may be beyond the type's ends where the result is not.
__device__ __forceinline__ float q8_scaled(int sum, float s, float w) {
  const float m = __builtin_amdgcn_frexp_mantf(s) * __builtin_amdgcn_frexp_mantf(w);
  return __builtin_amdgcn_ldexpf((float)sum * m, __builtin_amdgcn_frexp_expf(s) + __builtin_amdgcn_frexp_expf(w));
}
// s = sx of the row
template <int MODE>
__device__ __forceinline__ void dense_scales8(const DenseP& p, int n, int cnt, float (&w)[8]) {
  if constexpr (dense_q8(MODE)) load8(p.sw + n, cnt, w);
}
template <int MODE>
__device__ __forceinline__ float dense_scale(const DenseP& p, long long i) {
  if constexpr (dense_q8(MODE)) return p.sx[i];
  else return 1.f;
}
template <int MODE>
__device__ __forceinline__ void dense_scaled8(float s, const float (&w)[8], float (&v)[8]) {
  if constexpr (dense_q8(MODE))
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = q8_scaled(__float_as_int(v[e]), s, w[e]);
}

// What is done with eight sums (DENSE_GATED: of g and of u) at row i, columns n .. n+7 (cnt of them exist).  T: storage type.
template <typename T, int MODE>
__device__ __forceinline__ void dense_finish8(const DenseP& p, int src, long long i, int n, int cnt, float (&v)[8], float (&u)[8], const float (&b)[8],
                                              const float (&r)[8]) {
  const long long o = i * p.ldo + n;
  if constexpr (MODE == DENSE_DX) store8<true>((T*)p.out[0] + o, cnt, v);
  if constexpr (MODE == DENSE_DW) {
    if (p.out_f32) store8<true>((float*)p.out[src] + o, cnt, v);
    else store8<true>((T*)p.out[src] + o, cnt, v);
  }
  if constexpr (MODE == DENSE_FWD || dense_q8(MODE)) {
    if (p.bias)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += b[e];
    if (p.pre) store8<true>((T*)p.pre + o, cnt, v);
    act8(p.act, v);
    if (p.res)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    store8<true>((T*)p.out[0] + o, cnt, v);
  }
  if constexpr (MODE == DENSE_GATED) {
    if (p.dh) {
      gated_grad8(p.act, r, v, u);
      store8<true>((T*)p.out[0] + o, cnt, v);
      store8<true>((T*)p.pre1 + o, cnt, u);
    } else {
      if (p.pre) store8<true>((T*)p.pre + o, cnt, v);
      if (p.pre1) store8<true>((T*)p.pre1 + o, cnt, u);
      act8(p.act, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= u[e];
      store8<true>((T*)p.out[0] + o, cnt, v);
    }
  }
}

// The sums of one split, to be added by dense_join.
__device__ __forceinline__ void dense_part8(const DenseP& p, int split, int src, long long i, int n, int cnt, const float (&v)[8]) {
  store8(p.part + (((long long)split * p.srcs + src) * p.M + i) * p.N + n, cnt, v);
}

// Epilogue of a wave's TM x TN transposed accumulators (lane l of a 32 x 32 one holds row l % 32, columns 8 * (v / 4) + 4 * (l / 32) + v % 4).  32 rows at a time go
// through the wave's own LDS, in order and so without a barrier, and leave as vectors of eight columns.  DENSE_GATED: the first half of the
// columns are of g, the second of u.  m0, n0: the wave's first row and column.  Waves whose rows and columns all exist, nearly all of them, take no
// branch per vector, and the 32 rows' residuals are asked for together (behind branches each waited for the one before: 30 us of the 500 of
// 8192 x 8192 x 4096).
template <int MODE, int WTN>
struct EpiShape {
  static constexpr int COLS = MODE == DENSE_GATED ? WTN / 2 : WTN, LPR = COLS / 8, RPI = 64 / LPR, QV = 32 / RPI;   // lanes of a row, rows of an instruction, vectors of a lane in 32 rows
};
// Residuals (or dh) of a wave's first PRE x 32 rows, asked for before the main loop, whose length hides them.
template <int MODE, int WTN, int PRE>
struct Beside {
  static constexpr bool ON = MODE == DENSE_FWD || MODE == DENSE_GATED || MODE == DENSE_Q8;
  typedef EpiShape<MODE, WTN> E;
  v4u q[ON && PRE ? PRE : 1][ON && PRE ? E::QV : 1];
  __device__ __forceinline__ void ask(const DenseP& p, long long m0, int n0, bool whole) {
    const uint16_t* r = (const uint16_t*)(MODE == DENSE_GATED ? p.dh : p.res);
    if constexpr (ON && PRE > 0)
      if (r && whole) {
        const int lane = threadIdx.x & 63;
        r += (m0 + lane / E::LPR) * p.ldr + n0 + lane % E::LPR * 8;
#pragma unroll
        for (int i = 0; i < PRE; ++i)
#pragma unroll
          for (int v = 0; v < E::QV; ++v) __builtin_memcpy(&q[i][v], r + (long long)(i * 32 + v * E::RPI) * p.ldr, 16);
      }
  }
};
// Every row and column of a wave's tile exists, and its sums are whole.
template <int MODE, int WTN, int TM>
__device__ __forceinline__ bool epilogue_whole(const DenseP& p, long long m0, int n0) {
  return p.splits <= 1 && m0 + TM * 32 <= p.M && n0 + EpiShape<MODE, WTN>::COLS <= p.N;
}

template <typename T, int MODE, int WTN, int PRE, int TM, int TN, typename Acc>
__device__ __forceinline__ void dense_epilogue(const DenseP& p, const Acc (&acc)[TM][TN], unsigned char* lds, long long m0, int n0, int src, int split,
                                               const Beside<MODE, WTN, PRE>& pre) {
  typedef EpiShape<MODE, WTN> E;
  constexpr int LDC = WTN + 4, COLS = E::COLS, LPR = E::LPR, RPI = E::RPI, QV = E::QV;
  const int lane = threadIdx.x & 63, half = lane >> 5, cg = (lane % LPR) * 8;
  const int n = n0 + cg, cnt = p.N - n < 8 ? p.N - n : 8;
  float* sC = reinterpret_cast<float*>(lds);
  float b[8], w[8];
  if (p.splits <= 1 && cnt > 0) {
    dense_bias8<MODE>(p, n, cnt, b);
    dense_scales8<MODE>(p, n, cnt, w);
  }
  auto bits = [](auto v) { return __builtin_bit_cast(float, v); };
  auto turn = [&](int i) {                                        // 32 rows into LDS
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        *reinterpret_cast<float4*>(sC + (lane & 31) * LDC + j * 32 + 8 * v + 4 * half) =
            make_float4(bits(acc[i][j][4 * v]), bits(acc[i][j][4 * v + 1]), bits(acc[i][j][4 * v + 2]), bits(acc[i][j][4 * v + 3]));
  };
  auto get = [&](int lr, int at, float (&d)[8]) {
    const float* s = sC + lr * LDC + cg + at;
    const float4 lo = *reinterpret_cast<const float4*>(s), hi = *reinterpret_cast<const float4*>(s + 4);
    d[0] = lo.x; d[1] = lo.y; d[2] = lo.z; d[3] = lo.w; d[4] = hi.x; d[5] = hi.y; d[6] = hi.z; d[7] = hi.w;
  };
  if (epilogue_whole<MODE, WTN, TM>(p, m0, n0)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float r[QV][8], s[QV];
#pragma unroll
      for (int q = 0; q < QV; ++q) {
        s[q] = dense_scale<MODE>(p, m0 + i * 32 + lane / LPR + q * RPI);
        if constexpr (Beside<MODE, WTN, PRE>::ON && PRE > 0) {
          if (i < PRE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) r[q][e] = __uint_as_float((e & 1) ? (pre.q[i < PRE ? i : 0][q][e >> 1] & 0xffff0000u) : (pre.q[i < PRE ? i : 0][q][e >> 1] << 16));
            continue;
          }
        }
        dense_beside8<T, MODE>(p, m0 + i * 32 + lane / LPR + q * RPI, n, 8, r[q]);
      }
      turn(i);
#pragma unroll
      for (int q = 0; q < QV; ++q) {
        const int lr = lane / LPR + q * RPI;
        float v[8], u[8];
        get(lr, 0, v);
        if constexpr (MODE == DENSE_GATED) get(lr, COLS, u);
        dense_scaled8<MODE>(s[q], w, v);
        dense_finish8<T, MODE>(p, src, m0 + i * 32 + lr, n, 8, v, u, b, r[q]);
      }
      __builtin_amdgcn_sched_barrier(0);                          // 32 rows after the other: together they are more than the registers hold
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    turn(i);
    for (int q = 0; q < QV; ++q) {
      const int lr = lane / LPR + q * RPI;
      const long long row = m0 + i * 32 + lr;
      if (row >= p.M || cnt <= 0) continue;
      float v[8], u[8], r[8];
      get(lr, 0, v);
      if constexpr (MODE == DENSE_GATED) get(lr, COLS, u);
      if (p.splits > 1) {
        dense_part8(p, split, src, row, n, cnt, v);
        if constexpr (MODE == DENSE_GATED) dense_part8(p, split, 1, row, n, cnt, u);
      } else {
        dense_beside8<T, MODE>(p, row, n, cnt, r);
        dense_scaled8<MODE>(dense_scale<MODE>(p, row), w, v);
        dense_finish8<T, MODE>(p, src, row, n, cnt, v, u, b, r);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace
}  // namespace lms
