// Linear layer in 8-bit integers: rows of x and columns of w as whole numbers from -127 to 127 with a scale each (include/lms.h has the formulas).
//
// Both operands of the product lie with the reduction in rows of whole 16-byte vectors, zeros behind the last element: the weights are turned once, x as it is quantised.  In bytes the
// product is then that of two bf16 matrices whose reductions lie in rows, and it runs on the same tiles (dense_gemm.hip).
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "kernels.hpp"
#include "rows4.hpp"

namespace lms {

namespace {

constexpr int MAX_K = 1 << 17;         // 127^2 of them stay below 2^31

// The whole number nearest to 127 x / most, ties to even.  bf16: 127 x is exact, and the quotient of 15 by 8 bits is either a tie, which a float holds, or further from one
// than its rounding.  fp32: the same in fp64.  Values of more than 2^119 are scaled first, which is exact where it matters (x above most / 254).
template <typename T>
__device__ __forceinline__ int step_of(float x, float most) {
  if constexpr (sizeof(T) == 2) {
    const float s = most > 0x1p119f ? 0x1p-8f : 1.f;
    return (int)__builtin_rintf((127.f * (x * s)) / (most * s));
  } else return (int)__builtin_rint(127.0 * (double)x / (double)most);
}
// The scale of values whose largest magnitude has these bits: NaN where one of them is not finite, and then all steps are 0.
__device__ __forceinline__ float scale_of(unsigned bits) { return bits >= 0x7f800000u ? __builtin_nanf("") : __uint_as_float(bits) / 127.f; }
__device__ __forceinline__ bool steps(unsigned bits) { return bits != 0u && bits < 0x7f800000u; }

__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// NT threads a row, which hold it in NV vectors of eight each, or, with NV = 0, read it twice.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) void q8_rows_kernel(const T* x, long long ldx, int k, int kp, signed char* xq, float* sx, long long row0) {
  __shared__ unsigned s_most[NT / 64];
  const long long row = row0 + blockIdx.x;
  const T* from = x + row * ldx;
  signed char* to = xq + row * kp;
  const int tid = threadIdx.x;
  Raw<T, 8> held[NV > 0 ? NV : 1];
  unsigned most = 0;
  auto each = [&](auto&& f) {
    if constexpr (NV > 0)
#pragma unroll
      for (int v = 0; v < NV; ++v) f(v, (tid + v * NT) * 8);
    else
      for (int c = tid * 8; c < kp; c += NT * 8) f(0, c);
  };
  each([&](int v, int c) { if (NV > 0) held[v] = raw<8>(from + c, c < k ? k - c : 0); });
  each([&](int v, int c) {
    if constexpr (NV == 0) held[0] = raw<8>(from + c, c < k ? k - c : 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned m = magnitude_bits(held[v].get(e));
      most = most > m ? most : m;
    }
  });
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const unsigned m = __shfl_xor(most, d);
    most = most > m ? most : m;
  }
  if constexpr (NT > 64) {
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) most = most > s_most[w] ? most : s_most[w];
  }
  if (tid == 0) sx[row] = scale_of(most);
  const float top = __uint_as_float(most);
  const bool some = steps(most);
  each([&](int v, int c) {
    if (c >= kp) return;
    if constexpr (NV == 0) held[0] = raw<8>(from + c, c < k ? k - c : 0);
    unsigned q[2] = {0u, 0u};
    if (some)
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e >> 2] |= (unsigned)(step_of<T>(held[v].get(e), top) & 255) << (8 * (e & 3));
    __builtin_memcpy(to + c, q, 8);
  });
}

// 64 columns of the weights: their scales, and the steps turned into rows.
template <typename T>
__global__ __launch_bounds__(256) void q8_weight_kernel(const T* w, long long ldw, int n, int k, int kp, signed char* wq, float* sw) {
  __shared__ unsigned s_most[4][64];
  __shared__ int s_q[64][65];
  const int col = threadIdx.x & 63, way = threadIdx.x >> 6, j = blockIdx.x * 64 + col;
  unsigned most = 0;
  if (j < n)
    for (int r = way; r < k; r += 4) {
      float v;
      if constexpr (sizeof(T) == 2) v = bf2f(w[r * ldw + j]);
      else v = w[r * ldw + j];
      const unsigned m = magnitude_bits(v);
      most = most > m ? most : m;
    }
  s_most[way][col] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) most = most > s_most[i][col] ? most : s_most[i][col];
  if (way == 0 && j < n) sw[j] = scale_of(most);
  const float top = __uint_as_float(most);
  const bool some = steps(most) && j < n;
  for (int r0 = 0; r0 < kp; r0 += 64) {
    __syncthreads();
    for (int r = way; r < 64; r += 4) {
      int q = 0;
      if (some && r0 + r < k) {
        float v;
        if constexpr (sizeof(T) == 2) v = bf2f(w[(r0 + r) * ldw + j]);
        else v = w[(r0 + r) * ldw + j];
        q = step_of<T>(v, top);
      }
      s_q[r][col] = q;
    }
    __syncthreads();
    const int row = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;          // 16 steps of one column
    if (blockIdx.x * 64 + row < n && r0 + part < kp) {
      unsigned q[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 16; ++e) q[e >> 2] |= (unsigned)(s_q[part + e][row] & 255) << (8 * (e & 3));
      __builtin_memcpy(wq + (long long)(blockIdx.x * 64 + row) * kp + r0 + part, q, 16);
    }
  }
}

int pitch(const lms_linear_q8_desc* d) { return (d->k + 15) / 16 * 16; }

template <typename T>
hipError_t quantise(const lms_linear_q8_desc* d, const T* x, signed char* xq, float* sx, hipStream_t s) {
  const int kp = pitch(d);
  const long long ldx = d->ldx ? d->ldx : d->k;
  auto go = [&](auto nt, auto nv) {
    constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
    constexpr long long most = (1LL << 31) / NT;
    for (long long r = 0; r < d->m; r += most) {
      hipLaunchKernelGGL((q8_rows_kernel<T, NT, NV>), dim3((unsigned)(d->m - r < most ? d->m - r : most)), dim3(NT), 0, s, x, ldx, d->k, kp, xq, sx, r);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
#define ROWS(NT, NV) if (kp <= NT * 8 * NV) return go(std::integral_constant<int, NT>{}, std::integral_constant<int, NV>{})
  ROWS(64, 1);
  ROWS(256, 1);
  ROWS(256, 2);
  ROWS(256, 4);
  ROWS(1024, 4);
#undef ROWS
  return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 0>{});
}

uint64_t rows_bytes(const lms_linear_q8_desc* d) { return up256((uint64_t)d->m * pitch(d)); }
uint64_t scale_bytes(const lms_linear_q8_desc* d) { return up256((uint64_t)d->m * 4); }
int mode_of(const lms_linear_q8_desc* d) { return d->dtype == LMS_F32 ? DENSE_Q8_F32 : DENSE_Q8; }
uint64_t product_bytes(const lms_linear_q8_desc* d) { return up256(dense_bf16_ws(mode_of(d), d->m, d->n, pitch(d) / 2, 1, 1)); }

lms_status check(const char* what, const lms_linear_q8_desc* d) {
  NEED(d->m >= 0 && d->n >= 1 && d->k >= 1, "%s: rows must be >= 0, widths >= 1", what);
  NEED(d->m <= 0x7fffffffLL, "%s: more than 2^31 - 1 rows", what);
  NEED(d->n <= 1 << 30, "%s: widths above 2^30", what);
  NEED(d->k <= MAX_K, "%s: more than 2^17 inputs", what);
  NEED(d->act >= LMS_ACT_NONE && d->act <= LMS_ACT_GELU_TANH, "%s: unknown activation %d", what, d->act);
  NEED(d->dtype == LMS_BF16 || d->dtype == LMS_F32, "%s: dtype must be LMS_BF16 or LMS_F32", what);
  const long long most = 1LL << 40, ldx = d->ldx ? d->ldx : d->k, ldw = d->ldw ? d->ldw : d->n, ldy = d->ldy ? d->ldy : d->n, ldr = d->ldr ? d->ldr : d->n;
  NEED(ldx >= d->k && ldw >= d->n && ldy >= d->n && ldr >= d->n, "%s: a row pitch is shorter than the row", what);
  NEED(ldx <= most && ldw <= most && ldy <= most && ldr <= most, "%s: a row pitch is above 2^40", what);
  return LMS_OK;
}
lms_status aligned(const char* what, const lms_linear_q8_desc* d, std::initializer_list<const void*> rows, std::initializer_list<const void*> words, std::initializer_list<const void*> vectors) {
  uintptr_t a = 0, b = 0, c = 0;
  for (const void* q : rows) a |= (uintptr_t)q;
  for (const void* q : words) b |= (uintptr_t)q;
  for (const void* q : vectors) c |= (uintptr_t)q;
  NEED((a & (d->dtype == LMS_F32 ? 3 : 1)) == 0 && (b & 3) == 0, "%s: a pointer is not aligned to its elements", what);
  NEED((c & 15) == 0, "%s: 8-bit rows and the workspace must be aligned to 16 bytes", what);
  return LMS_OK;
}

hipError_t product(const lms_linear_q8_desc* d, const void* xq, const float* sx, const void* wq, const float* sw, const float* bias, const void* res, void* y, void* ws, hipStream_t s) {
  DenseP p{};
  p.a[0] = xq; p.b[0] = wq; p.out[0] = y;
  p.sx = sx; p.sw = sw; p.bias = bias; p.res = res;
  p.M = d->m; p.N = d->n; p.red = pitch(d) / 2;
  p.lda = p.ldb = pitch(d) / 2;
  p.ldo = d->ldy ? d->ldy : d->n;
  p.ldr = d->ldr ? d->ldr : d->n;
  p.segs = 1; p.srcs = 1; p.act = d->act;
  p.part = (float*)ws;
  return dense_bf16(mode_of(d), p, s);
}

}  // namespace

lms_status linear_q8_weight_size(const lms_linear_q8_desc* d, uint64_t* bytes) {
  if (const lms_status st = check("lms_linear_q8_weight_bytes", d)) return st;
  *bytes = (uint64_t)d->n * pitch(d);
  return LMS_OK;
}
lms_status linear_q8_workspace(const lms_linear_q8_desc* d, uint64_t* bytes) {
  if (const lms_status st = check("lms_linear_q8_workspace_bytes", d)) return st;
  *bytes = d->m == 0 ? 0 : rows_bytes(d) + scale_bytes(d) + product_bytes(d);
  return LMS_OK;
}

lms_status linear_q8_weight(const lms_linear_q8_desc* d, const void* w, void* wq, float* sw, void* stream) {
  const char* what = "lms_linear_q8_weight";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {w}, {sw}, {wq})) return st;
  const dim3 grid((unsigned)((d->n + 63) / 64));
  const long long ldw = d->ldw ? d->ldw : d->n;
  hipStream_t s = (hipStream_t)stream;
  if (d->dtype == LMS_F32) hipLaunchKernelGGL(q8_weight_kernel<float>, grid, dim3(256), 0, s, (const float*)w, ldw, d->n, d->k, pitch(d), (signed char*)wq, sw);
  else hipLaunchKernelGGL(q8_weight_kernel<uint16_t>, grid, dim3(256), 0, s, (const uint16_t*)w, ldw, d->n, d->k, pitch(d), (signed char*)wq, sw);
  return done(what, hipGetLastError());
}

lms_status linear_q8_rows(const lms_linear_q8_desc* d, const void* x, void* xq, float* sx, void* stream) {
  const char* what = "lms_linear_q8_rows";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {x}, {sx}, {xq})) return st;
  hipStream_t s = (hipStream_t)stream;
  return done(what, d->dtype == LMS_F32 ? quantise<float>(d, (const float*)x, (signed char*)xq, sx, s) : quantise<uint16_t>(d, (const uint16_t*)x, (signed char*)xq, sx, s));
}

lms_status linear_q8_product(const lms_linear_q8_desc* d, const void* xq, const float* sx, const void* wq, const float* sw, const float* bias, const void* res, void* y, void* ws,
                             void* stream) {
  const char* what = "lms_linear_q8_product";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {res, y}, {sx, sw, bias}, {xq, wq, ws})) return st;
  NEED(res != y || (d->ldr ? d->ldr : d->n) == (d->ldy ? d->ldy : d->n), "%s: res may be y only with the same pitch", what);
  if (d->m == 0) return LMS_OK;
  NEED(ws || product_bytes(d) == 0, "%s: workspace of %llu bytes required", what, (unsigned long long)product_bytes(d));
  return done(what, product(d, xq, sx, wq, sw, bias, res, y, ws, (hipStream_t)stream));
}

lms_status linear_q8_fwd(const lms_linear_q8_desc* d, const void* x, const void* wq, const float* sw, const float* bias, const void* res, void* y, void* ws, void* stream) {
  const char* what = "lms_linear_q8_fwd";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {x, res, y}, {sw, bias}, {wq, ws})) return st;
  NEED(res != y || (d->ldr ? d->ldr : d->n) == (d->ldy ? d->ldy : d->n), "%s: res may be y only with the same pitch", what);
  if (d->m == 0) return LMS_OK;
  NEED(ws, "%s: workspace required", what);
  char* at = (char*)ws;
  float* sx = (float*)(at + rows_bytes(d));
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = d->dtype == LMS_F32 ? quantise<float>(d, (const float*)x, (signed char*)at, sx, s) : quantise<uint16_t>(d, (const uint16_t*)x, (signed char*)at, sx, s);
  if (e == hipSuccess) e = product(d, at, sx, wq, sw, bias, res, y, at + rows_bytes(d) + scale_bytes(d), s);
  return done(what, e);
}

}  // namespace lms
