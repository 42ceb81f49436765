// Distillation loss from a teacher's top logits and its gradient (include/lms.h has the formulas).
//
// A work-group takes a row.  One pass over the row's logits keeps the running maximum and the sum of exponentials relative to it, in fp32, as powers
// of two, which are one instruction; the teacher's k entries lie in LDS.  The gradient scale weight T (q - p) is q for all classes but
// the teacher's: the row leaves as whole vectors, and behind a barrier the teacher's classes are written over.
#include <hip/hip_runtime.h>

#include "dense.hpp"
#include "graph.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

constexpr int MAX_K = 1024;
constexpr float LOG2E = 1.44269504f, LN2 = 0.69314718f;

struct DistillP {
  const void* z;
  const float* t;
  const int32_t* ids;
  const float* weight;
  const float* lse_in;
  float *row_loss, *lse;       // or null
  float* part;                 // weight * row loss, or null
  void* dz;                    // or null
  long long rows, ldz;
  int classes, k;
  float temp, scale;
};

// Maximum and sum over a work-group of NT threads, in a fixed order.
template <int NT, typename F>
__device__ __forceinline__ float group_reduce(float v, float* lds, F&& f) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = f(v, __shfl_xor(v, d));
  __syncthreads();                                                // what the last reduction left has been read
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) v = f(v, lds[w]);
  return v;
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void distill_kernel(DistillP p) {
  __shared__ float s_p[MAX_K], s_q[MAX_K], s_red[NT / 64];
  __shared__ int s_id[MAX_K];
  const auto add = [](float a, float b) { return a + b; };
  const auto larger = [](float a, float b) { return fmaxf(a, b); };
  const int tid = threadIdx.x;
  const long long row = blockIdx.x;
  const T* z = (const T*)p.z + row * p.ldz;
  T* dz = (T*)p.dz + (p.dz ? row * p.ldz : 0);
  const float weight = p.weight ? p.weight[row] : 1.f;
  const float zero8[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto clear = [&]() {
    for (int c = tid * 8; c < p.classes; c += NT * 8) store8(dz + c, p.classes - c, zero8);
  };
  if (weight == 0.f && !p.row_loss && !p.lse) {                   // nothing depends on this row
    if (p.part && tid == 0) p.part[row] = 0.f;
    if (p.dz) clear();
    return;
  }

  // ---- the teacher: p, and the logits of its classes (before any of them is written over: dz may be z) ----
  const float inf = __builtin_inff();
  const float c2 = LOG2E / p.temp;                                // e^((a - b) / T) = 2^((a - b) c2); the difference first: the type's lowest value times c2 is -inf
  float top = -inf;
  for (int j = tid; j < p.k; j += NT) {
    const int id = p.ids[row * p.k + j];
    const float t = p.t[row * p.k + j];
    const bool there = id >= 0 && id < p.classes && !(t == -inf);
    s_id[j] = there ? id : -1;
    s_p[j] = t;
    if (there) {
      top = fmaxf(top, t);
      if constexpr (sizeof(T) == 2) s_q[j] = bf2f(z[id]);
      else s_q[j] = z[id];
    }
  }
  top = group_reduce<NT>(top, s_red, larger);
  float total = 0.f;
  for (int j = tid; j < p.k; j += NT)
    if (s_id[j] >= 0) total += __builtin_amdgcn_exp2f((s_p[j] - top) * c2);
  total = group_reduce<NT>(total, s_red, add);
  const bool some = total > 0.f || total != total;                // total is at least 1 where there is an entry
  if (!some && p.dz && !p.part) { clear(); return; }

  // ---- the student: q = 2^((z - m) c2 - l), m: the largest logit, or lse T ----
  float m, l = 0.f;
  if (p.lse_in) {
    m = p.lse_in[row] * p.temp;
    if (m == -inf) m = 0.f;                                       // all classes masked: q = 0
  } else {
    m = -inf;
    float s = 0.f;
    for (int c = tid * 8; c < p.classes; c += NT * 8) {
      float v[8];
      load8(z + c, p.classes - c, v);
      float high = m;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = c + e < p.classes ? v[e] : -inf;
        high = fmaxf(high, v[e]);
      }
      const float base = high == -inf ? 0.f : high;               // nothing but masked classes so far
      s *= __builtin_amdgcn_exp2f((m - base) * c2);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f((v[e] - base) * c2);
      m = high;
    }
    const float mine = m;
    m = group_reduce<NT>(m, s_red, larger);
    if (m == -inf) m = 0.f;
    s = group_reduce<NT>(s * __builtin_amdgcn_exp2f((mine - m) * c2), s_red, add);
    l = __builtin_amdgcn_logf(s);                                 // -inf where all classes are masked
    if (p.lse && tid == 0) p.lse[row] = m / p.temp + l * LN2;
  }

  if (p.part || p.row_loss) {
    const float log_total = __builtin_amdgcn_logf(total);
    float loss = 0.f;
    for (int j = tid; j < p.k; j += NT)
      if (s_id[j] >= 0) {
        const float log_p = (s_p[j] - top) * c2 - log_total, prob = __builtin_amdgcn_exp2f(log_p);
        if (prob != 0.f) loss += s_q[j] == -inf ? inf : prob * (log_p - ((s_q[j] - m) * c2 - l));     // on a masked class: inf
      }
    loss = group_reduce<NT>(loss, s_red, add) * (LN2 * p.temp * p.temp);
    if (tid == 0) {
      if (p.row_loss) p.row_loss[row] = loss;
      if (p.part) p.part[row] = weight == 0.f ? 0.f : weight * loss;
    }
  }
  if (!p.dz) return;
  if (!some) { clear(); return; }

  // ---- the gradient ----
  const float coef = p.scale * weight * p.temp;
  if (l == -inf) l = 0.f;
  for (int c = tid * 8; c < p.classes; c += NT * 8) {
    float v[8];
    load8(z + c, p.classes - c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = coef * __builtin_amdgcn_exp2f((v[e] - m) * c2 - l);
    store8(dz + c, p.classes - c, v);
  }
  __syncthreads();                                                // the row is there: now the teacher's classes
  const float inv = 1.f / total;
  for (int j = tid; j < p.k; j += NT) {
    const int id = s_id[j];
    if (id < 0) continue;
    float sum = 0.f;
    bool first = true;
    for (int i = 0; i < p.k; ++i)                                 // a class that comes more than once counts with the sum, once
      if (s_id[i] == id) {
        if (i < j) { first = false; break; }
        sum += __builtin_amdgcn_exp2f((s_p[i] - top) * c2) * inv;
      }
    if (!first) continue;
    const float v = coef * (__builtin_amdgcn_exp2f((s_q[j] - m) * c2 - l) - sum);
    if constexpr (sizeof(T) == 2) dz[id] = f2bf(v);
    else dz[id] = v;
  }
}

// loss = scale * sum of part, in fp64 and in a fixed order
__global__ __launch_bounds__(1024) void distill_loss_kernel(const float* part, long long rows, float scale, float* loss) {
  __shared__ double sums[1024];
  double t = 0.0;
  for (long long r = threadIdx.x; r < rows; r += 1024) t += (double)part[r];
  sums[threadIdx.x] = t;
  for (int d = 512; d > 0; d >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < d) sums[threadIdx.x] += sums[threadIdx.x + d];
  }
  if (threadIdx.x == 0) loss[0] = (float)(sums[0] * (double)scale);
}

hipError_t launch_distill(bool f32, const DistillP& p, float* loss, hipStream_t s) {
  if (p.rows > 0) {
    if (f32) hipLaunchKernelGGL((distill_kernel<float, 256>), dim3((unsigned)p.rows), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((distill_kernel<uint16_t, 256>), dim3((unsigned)p.rows), dim3(256), 0, s, p);
  }
  if (loss) hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(1024), 0, s, p.part, p.rows, p.scale, loss);
  return hipGetLastError();
}

#define NEED(cond, ...)        \
  do {                         \
    if (!(cond)) {             \
      set_error(__VA_ARGS__);  \
      return LMS_EINVAL;       \
    }                          \
  } while (0)

lms_status check(const char* what, const lms_distill_desc* d) {
  NEED(d->rows >= 0 && d->classes >= 1, "%s: rows must be >= 0, classes >= 1", what);
  NEED(d->rows <= 0x7fffffffLL, "%s: more than 2^31 - 1 rows", what);
  NEED(d->k >= 1 && d->k <= MAX_K, "%s: k must be in 1 .. %d", what, MAX_K);
  NEED(d->dtype == LMS_BF16 || d->dtype == LMS_F32, "%s: dtype must be LMS_BF16 or LMS_F32", what);
  NEED(d->ldz == 0 || (d->ldz >= d->classes && d->ldz <= (1LL << 40)), "%s: row pitch shorter than the row, or above 2^40", what);
  NEED(d->temperature > 0.f && d->temperature < __builtin_inff(), "%s: the temperature must be positive and finite", what);
  NEED(d->scale == d->scale && d->scale - d->scale == 0.f, "%s: the scale must be finite", what);
  return LMS_OK;
}

}  // namespace

lms_status distill_workspace(const lms_distill_desc* d, int which, uint64_t* bytes) {
  if (const lms_status st = check("lms_distill_workspace_bytes", d)) return st;
  NEED(which >= LMS_DISTILL_FWD && which <= LMS_DISTILL_LOSS_GRAD, "lms_distill_workspace_bytes: unknown call %d", which);
  *bytes = which == LMS_DISTILL_BWD ? 0 : ((uint64_t)d->rows * 4 + 255) / 256 * 256;
  return LMS_OK;
}

lms_status distill(const lms_distill_desc* d, int which, const void* z, const float* t, const int32_t* ids, const float* weight, const float* lse_in, float* loss,
                   float* row_loss, float* lse, void* dz, void* ws, void* stream) {
  const char* what = which == LMS_DISTILL_FWD ? "lms_distill_fwd" : which == LMS_DISTILL_BWD ? "lms_distill_bwd" : "lms_distill_loss_grad";
  if (const lms_status st = check(what, d)) return st;
  const bool f32 = d->dtype == LMS_F32;
  NEED((((uintptr_t)z | (uintptr_t)dz) & (f32 ? 3 : 1)) == 0, "%s: a pointer is not aligned to its elements", what);
  NEED((((uintptr_t)t | (uintptr_t)ids | (uintptr_t)weight | (uintptr_t)lse_in | (uintptr_t)loss | (uintptr_t)row_loss | (uintptr_t)lse) & 3) == 0,
       "%s: a pointer is not aligned to its elements", what);
  NEED(!loss || ws || d->rows == 0, "%s: workspace of %llu bytes required", what, (unsigned long long)d->rows * 4);
  DistillP p{};
  p.z = z; p.t = t; p.ids = ids; p.weight = weight; p.lse_in = lse_in;
  p.row_loss = row_loss; p.lse = lse; p.dz = dz;
  p.part = loss ? (float*)ws : nullptr;
  p.rows = d->rows; p.ldz = d->ldz ? d->ldz : d->classes;
  p.classes = d->classes; p.k = d->k; p.temp = d->temperature; p.scale = d->scale;
  const hipError_t e = launch_distill(f32, p, loss, (hipStream_t)stream);
  if (e != hipSuccess) { set_error("%s: %s", what, hipGetErrorString(e)); return LMS_EHIP; }
  return LMS_OK;
}

}  // namespace lms
