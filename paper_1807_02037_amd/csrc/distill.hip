// Distillation loss from a teacher's top logits and its gradient (include/lms.h has the formulas).
//
// A work-group takes a row and holds it in registers from its one read to the one write of its gradient (longer rows than those hold are read again).  Sums are fp32
// of powers of two, which are one instruction; the teacher's k entries lie in LDS.  The gradient scale weight T (q - p) is q for all classes but
// the teacher's: the row leaves as whole vectors, and the wave that has stored a teacher's class then writes over it.  A wave's stores to one
// address stay in order; a barrier instead would wait until the whole row has arrived in memory.
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
  long long row0;              // first row of this launch
  int classes, k, table;       // table: a power of two, at least 2 k
  float temp, scale;
};

// Two values of every thread of a work-group of NT, by f and g, in a fixed order.
template <int NT, typename F, typename G>
__device__ __forceinline__ void group_reduce(float& v, float& w, float (*lds)[2], F&& f, G&& g) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    v = f(v, __shfl_xor(v, d));
    w = g(w, __shfl_xor(w, d));
  }
  __syncthreads();                                                // what the last reduction left has been read; what the caller wrote is there
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) {
      lds[threadIdx.x >> 6][0] = v;
      lds[threadIdx.x >> 6][1] = w;
    }
    __syncthreads();
    v = lds[0][0];
    w = lds[0][1];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) {
      v = f(v, lds[i][0]);
      w = g(w, lds[i][1]);
    }
  }
}

// Eight logits as they lie in memory; -inf for those beyond the row.
template <typename T>
struct Logits {
  unsigned q[2 * sizeof(T)];
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float((e & 1) ? (q[e >> 1] & 0xffff0000u) : (q[e >> 1] << 16));
    else return __uint_as_float(q[e]);
  }
  __device__ __forceinline__ void load(const T* p, int cnt) {
    if (cnt >= 8) { __builtin_memcpy(q, p, sizeof(q)); return; }
#pragma unroll
    for (unsigned& w : q) w = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < cnt) {
        if constexpr (sizeof(T) == 2) q[e >> 1] = (e & 1) ? (q[e >> 1] & 0xffffu) | (unsigned)p[e] << 16 : (q[e >> 1] & 0xffff0000u) | p[e];
        else q[e] = __float_as_uint(p[e]);
      }
  }
};

// NT threads a row, which hold it in NV vectors of eight logits each, or, with NV = 0, read it again for each pass.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) void distill_kernel(DistillP p) {
  __shared__ float s_red[NT / 64][2];
  __shared__ int s_twice;                                         // a class comes more than once
  extern __shared__ int s_dyn[];
  int* const s_id = s_dyn;                                        // of the entries: class or -1, teacher's logit, student's
  float* const s_p = reinterpret_cast<float*>(s_dyn + p.k);
  float* const s_q = s_p + p.k;
  int* const s_set = s_dyn + 3 * p.k;                             // the classes that come, in a hash table of p.table places
  const auto add = [](float a, float b) { return a + b; };
  const auto larger = [](float a, float b) { return fmaxf(a, b); };
  const float inf = __builtin_inff();
  const int tid = threadIdx.x;
  const long long row = p.row0 + blockIdx.x;
  const T* z = (const T*)p.z + row * p.ldz;
  T* dz = (T*)p.dz + (p.dz ? row * p.ldz : 0);
  const float weight = p.weight ? p.weight[row] : 1.f;
  auto each = [&](auto&& f) {                                     // f(vector, first class)
    if constexpr (NV > 0)
#pragma unroll
      for (int v = 0; v < NV; ++v) f(v, (tid + v * NT) * 8);
    else
      for (int c = tid * 8; c < p.classes; c += NT * 8) f(0, c);
  };
  auto clear = [&]() {
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    each([&](int, int c) { if (c < p.classes) store8(dz + c, p.classes - c, zero); });
  };
  if (weight == 0.f && !p.row_loss && !p.lse) {                   // nothing depends on this row
    if (p.part && tid == 0) p.part[row] = 0.f;
    if (p.dz) clear();
    return;
  }
  // the teacher's entries are asked for before the row: loads come back in order
  const int id0 = tid < p.k ? p.ids[row * p.k + tid] : -1;
  const float t0 = tid < p.k ? p.t[row * p.k + tid] : 0.f;
  Logits<T> held[NV > 0 ? NV : 1];
  if constexpr (NV > 0) each([&](int v, int c) { held[v].load(z + c, p.classes - c); });
  auto logits = [&](int v, int c) -> const Logits<T>& {
    if constexpr (NV == 0) held[0].load(z + c, p.classes - c);
    return held[v];
  };

  // ---- the teacher: p, and the logits of its classes (before any of them is written over: dz may be z) ----
  // e^((a - b) / T) = 2^((a - b) c2); the difference first: the type's lowest value times c2 is -inf.  A T below the least normal number would make c2 inf and the largest class 0 inf.
  const float c2 = fminf(LOG2E / p.temp, 3.4028235e38f);
  float top = -inf;
  if (p.dz) {
    for (int i = tid; i < p.table; i += NT) s_set[i] = -1;
    if (tid == 0) s_twice = 0;
  }
  for (int j = tid; j < p.k; j += NT) {
    const int id = j == tid ? id0 : p.ids[row * p.k + j];
    const float t = j == tid ? t0 : p.t[row * p.k + j];
    const bool there = id >= 0 && id < p.classes && !(t == -inf);
    s_id[j] = there ? id : -1;
    s_p[j] = t;
    if (there) {
      top = fmaxf(top, t);
      if constexpr (sizeof(T) == 2) s_q[j] = bf2f(z[id]);
      else s_q[j] = z[id];
    }
  }

  // ---- the student: q = 2^((z - m) c2 - l), m: the largest logit, or lse T ----
  float m = -inf, s = 0.f, total = 0.f, l = 0.f;
  if (!p.lse_in) each([&](int v, int c) {
    const Logits<T>& x = logits(v, c);
    float high = m;
#pragma unroll
    for (int e = 0; e < 8; ++e) high = fmaxf(high, x.get(e));
    if constexpr (NV == 0) {                                      // the running sum, relative to the running maximum
      const float base = high == -inf ? 0.f : high;               // nothing but masked classes so far
      s *= __builtin_amdgcn_exp2f((m - base) * c2);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f((x.get(e) - base) * c2);
    }
    m = high;
  });
  const float mine = m;
  group_reduce<NT>(m, top, s_red, larger, larger);
  if (p.lse_in) m = p.lse_in[row] * p.temp;
  if (m == -inf) m = 0.f;                                         // all classes masked: q = 0
  if (!p.lse_in) {
    if constexpr (NV > 0) each([&](int v, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f((held[v].get(e) - m) * c2);
    });
    else s *= __builtin_amdgcn_exp2f((mine - m) * c2);
  }
  for (int j = tid; j < p.k; j += NT) {
    const int id = s_id[j];
    if (id < 0) continue;
    total += __builtin_amdgcn_exp2f((s_p[j] - top) * c2);
    if (p.dz)
      for (unsigned at = ((unsigned)id * 2654435761u) >> 16;; ++at) {       // at most half of the places are taken
        const int was = atomicCAS(&s_set[at & (p.table - 1)], -1, id);
        if (was == id) s_twice = 1;
        if (was == -1 || was == id) break;
      }
  }
  group_reduce<NT>(s, total, s_red, add, add);
  const bool some = total > 0.f || total != total;                // total is at least 1 where there is an entry
  if (!p.lse_in) l = __builtin_amdgcn_logf(s);                    // -inf where all classes are masked
  if (p.lse && tid == 0) p.lse[row] = m / p.temp + l * LN2;

  // T^2 sum p (log p - log q) as T sum p (T log p + T log sum - (z - m)): neither the type's lowest value in z nor T^2 overflows on the way to a loss that does not
  if (p.part || p.row_loss) {
    const float log_total = __builtin_amdgcn_logf(total);
    float loss = 0.f, unused = 0.f;
    for (int j = tid; j < p.k; j += NT)
      if (s_id[j] >= 0) {
        const float log_p = (s_p[j] - top) * c2 - log_total, prob = __builtin_amdgcn_exp2f(log_p);
        if (prob != 0.f) loss += s_q[j] == -inf ? inf : prob * (p.temp * LN2 * (log_p + l) - (s_q[j] - m));     // on a masked class: inf
      }
    group_reduce<NT>(loss, unused, s_red, add, add);
    loss *= p.temp;
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
  each([&](int v, int c) {
    if (c >= p.classes) return;
    const Logits<T>& x = logits(v, c);
    float d[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = coef * __builtin_amdgcn_exp2f((x.get(e) - m) * c2 - l);
    store8(dz + c, p.classes - c, d);
  });
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const float inv = 1.f / total;
  const bool twice = s_twice != 0;
  for (int j = tid & 63; j < p.k; j += 64) {                      // every wave looks through the entries for its own classes
    const int id = s_id[j];
    if (id < 0 || ((id / 8 % NT) ^ tid) >= 64) continue;
    float sum = __builtin_amdgcn_exp2f((s_p[j] - top) * c2) * inv;
    if (twice) {                                                  // a class that comes more than once counts with the sum, once
      bool first = true;
      sum = 0.f;
      for (int i = 0; i < p.k; ++i)
        if (s_id[i] == id) {
          if (i < j) { first = false; break; }
          sum += __builtin_amdgcn_exp2f((s_p[i] - top) * c2) * inv;
        }
      if (!first) continue;
    }
    const float v = coef * (__builtin_amdgcn_exp2f((s_q[j] - m) * c2 - l) - sum);
    if constexpr (sizeof(T) == 2) dz[id] = f2bf(v);
    else dz[id] = v;
  }
}

// loss = scale * sum of part, in fp64 and in a fixed order
__global__ __launch_bounds__(512) void distill_loss_kernel(const float* part, long long rows, float scale, float* loss) {
  __shared__ double sums[8];
  double t[4] = {0.0, 0.0, 0.0, 0.0};
  for (long long r = threadIdx.x; r < rows; r += 2048) {
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = r + u * 512 < rows ? part[r + u * 512] : 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) t[u] += (double)v[u];
  }
  double sum = t[0] + t[1] + t[2] + t[3];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += sums[w];
    loss[0] = (float)(sum * (double)scale);
  }
}

// The fewest threads and vectors that hold a row; rows beyond 98304 classes (fp32: 65536) are read again for the gradient.  A grid holds less than 2^32
// threads: more rows go in several launches.
template <typename T>
hipError_t launch_rows(DistillP& p, hipStream_t s) {
  constexpr bool wide = sizeof(T) == 4;
  auto go = [&](auto nt, auto nv) {
    constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
    constexpr long long most = (1LL << 31) / NT;
    for (p.row0 = 0; p.row0 < p.rows; p.row0 += most) {
      const long long take = p.rows - p.row0 < most ? p.rows - p.row0 : most;
      hipLaunchKernelGGL((distill_kernel<T, NT, NV>), dim3((unsigned)take), dim3(NT), (3 * p.k + (p.dz ? p.table : 0)) * 4, s, p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
#define ROWS(NT, NV) if (p.classes <= NT * 8 * NV) return go(std::integral_constant<int, NT>{}, std::integral_constant<int, NV>{})
  ROWS(64, 1);
  ROWS(64, 4);
  ROWS(256, 4);
  ROWS(512, 4);
  ROWS(512, 8);
  if constexpr (!wide) ROWS(512, 13);
  ROWS(1024, 8);
  if constexpr (!wide) ROWS(1024, 12);
#undef ROWS
  return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 0>{});
}

hipError_t launch_distill(bool f32, DistillP& p, float* loss, hipStream_t s) {
  const hipError_t e = f32 ? launch_rows<float>(p, s) : launch_rows<uint16_t>(p, s);
  if (e != hipSuccess || !loss) return e;
  hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(512), 0, s, p.part, p.rows, p.scale, loss);
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
  NEED(d->classes <= 1 << 30, "%s: more than 2^30 classes", what);
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
  NEED(((uintptr_t)ws & 15) == 0, "%s: the workspace is not aligned", what);
  DistillP p{};
  p.z = z; p.t = t; p.ids = ids; p.weight = weight; p.lse_in = lse_in;
  p.row_loss = row_loss; p.lse = lse; p.dz = dz;
  p.part = loss ? (float*)ws : nullptr;
  p.rows = d->rows; p.ldz = d->ldz ? d->ldz : d->classes;
  p.classes = d->classes; p.k = d->k;
  for (p.table = 2; p.table < 2 * p.k;) p.table *= 2;
  p.temp = d->temperature; p.scale = d->scale;
  const hipError_t e = launch_distill(f32, p, loss, (hipStream_t)stream);
  if (e != hipSuccess) { set_error("%s: %s", what, hipGetErrorString(e)); return LMS_EHIP; }
  return LMS_OK;
}

}  // namespace lms
