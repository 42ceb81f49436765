// Group normalisation with an activation, channels last, and its backward pass (include/lms.h has the formulas).
//
// Sums over a sample's positions and a group's channels come from partial ones: a work-group takes a chunk of a sample's positions and up to 256 channels and leaves, for each channel, mean
// and sum of squared deviations (backwards: sums of dv and of dv xhat); a second launch joins the chunks and channels of each group; the third computes the results.  Deviations are from the mean of the rows that a thread holds, and
// means are joined with what their distances add, so that nothing cancels however far the mean is from zero.
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "kernels.hpp"
#include "rows4.hpp"

namespace lms {

namespace {

constexpr int NT = 512, WAVES = NT / 64;
constexpr int U = 8;                   // rows of a thread in flight
constexpr long long PART_BYTES = 96LL << 20;                      // inputs that are read again before they have left the last-level cache

struct NormP {
  const void *x, *dy;
  const float *gamma, *beta;
  const float *mean, *rstd;            // [sample][group]
  float *mean_out, *rstd_out;          // forward: where the join writes them
  void* out;                           // y or dx
  float* part;                         // [sample of the part][chunk][2][channels]
  float* coef;                         // backward: [sample][group][2], means over the group of gamma dv and of gamma dv xhat
  long long s, ldx, ldy, ldo, chunk_rows;
  long long sample0;                   // first sample of the part
  int c, groups, cg, act, chunks, cblocks, lpr;      // lpr: lanes of a row, a power of two
  float eps;
};

// What a thread has of the job: its rows begin at row0 + first and come `stride` apart.
struct Place {
  long long sample, row0, rows;        // rows of the chunk
  int chunk, c, cnt, first, stride;
};
__device__ __forceinline__ Place place(const NormP& p, int job) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rpw = 64 / p.lpr;
  const int cb = job % p.cblocks, at = job / p.cblocks;
  Place t;
  t.chunk = at % p.chunks;
  t.sample = p.sample0 + at / p.chunks;
  const long long begin = t.chunk * p.chunk_rows;
  t.rows = p.s - begin < p.chunk_rows ? p.s - begin : p.chunk_rows;
  t.row0 = t.sample * p.s + begin;
  t.c = (cb * p.lpr + lane % p.lpr) * V;
  t.cnt = p.c - t.c;
  t.first = wave * rpw + lane / p.lpr;
  t.stride = WAVES * rpw;
  return t;
}

// mean, 1 / deviation, gamma and beta of a thread's channels.
struct Coef {
  float mean[V], rstd[V], gamma[V], beta[V];
  int group[V];
  __device__ __forceinline__ Coef(const NormP& p, long long sample, int c) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool there = c + e < p.c;
      group[e] = there ? (c + e) / p.cg : 0;
      mean[e] = p.mean[sample * p.groups + group[e]];
      rstd[e] = p.rstd[sample * p.groups + group[e]];
      gamma[e] = p.gamma && there ? p.gamma[c + e] : 1.f;
      beta[e] = p.beta && there ? p.beta[c + e] : 0.f;
    }
  }
};

// Mean and squared deviations of n values and of nb others, together.
__device__ __forceinline__ void merge(float& n, float (&mean)[V], float (&m2)[V], float nb, const float (&mb)[V], const float (&qb)[V]) {
  const float all = n + nb;
  if (nb == 0.f) return;
  const float share = nb / all;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float d = mb[e] - mean[e];
    mean[e] = __builtin_fmaf(d, share, mean[e]);
    m2[e] += __builtin_fmaf(d * d, n * share, qb[e]);
  }
  n = all;
}

template <typename T>
__global__ __launch_bounds__(NT) void norm_stats_kernel(NormP p) {
  __shared__ float s_n[WAVES][64], s_mean[WAVES][64][V], s_m2[WAVES][64][V];
  const Place t = place(p, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float n = 0.f, mean[V] = {}, m2[V] = {};
  const T* x = (const T*)p.x + t.row0 * p.ldx + t.c;
  if (t.cnt > 0)
    for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
      Raw<T, V> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = raw<V>(x + (r + u * t.stride < t.rows ? r + u * t.stride : r) * p.ldx, t.cnt);
      float nb = 0.f, mb[V] = {}, qb[V] = {};
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * t.stride < t.rows) {
          nb += 1.f;
#pragma unroll
          for (int e = 0; e < V; ++e) mb[e] += v[u].get(e);
        }
      const float inv = 1.f / nb;
#pragma unroll
      for (int e = 0; e < V; ++e) mb[e] *= inv;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * t.stride < t.rows)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float d = v[u].get(e) - mb[e];
            qb[e] = __builtin_fmaf(d, d, qb[e]);
          }
      merge(n, mean, m2, nb, mb, qb);
    }
  s_n[wave][lane] = n;
#pragma unroll
  for (int e = 0; e < V; ++e) { s_mean[wave][lane][e] = mean[e]; s_m2[wave][lane][e] = m2[e]; }
  __syncthreads();
  if (threadIdx.x >= p.lpr || t.cnt <= 0) return;
  for (int i = 0; i < WAVES * (64 / p.lpr); ++i) {                // this column's other rows
    const int w = i / (64 / p.lpr), l = i % (64 / p.lpr) * p.lpr + lane;
    if (w == 0 && l == lane) continue;
    float mb[V], qb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { mb[e] = s_mean[w][l][e]; qb[e] = s_m2[w][l][e]; }
    if (n == 0.f && s_n[w][l] == 0.f) continue;
    merge(n, mean, m2, s_n[w][l], mb, qb);
  }
  float* to = p.part + ((t.sample - p.sample0) * p.chunks + t.chunk) * 2 * p.c + t.c;
  store4(to, t.cnt, mean);
  store4(to + p.c, t.cnt, m2);
}

// Sum of v over a work-group of 256, in a fixed order.
__device__ __forceinline__ float group_sum(float v, float* lds) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Mean and 1 / deviation of a group from its channels' chunks.
__global__ __launch_bounds__(256) void norm_join_kernel(NormP p) {
  __shared__ float lds[4];
  const int g = blockIdx.x % p.groups;
  const long long local = blockIdx.x / p.groups, sample = p.sample0 + local, items = (long long)p.chunks * p.cg;
  const float* part = p.part + local * p.chunks * 2 * p.c + g * p.cg;
  const float inv = 1.f / ((float)p.s * (float)p.cg);
  auto each = [&](auto&& f) {                                     // f(rows, mean, squared deviations)
    for (long long i = threadIdx.x; i < items; i += 256) {
      const int chunk = (int)(i / p.cg), c = (int)(i - (long long)chunk * p.cg);
      const long long left = p.s - chunk * p.chunk_rows;
      const float* at = part + (long long)chunk * 2 * p.c + c;
      f((float)(left < p.chunk_rows ? left : p.chunk_rows), at[0], at[p.c]);
    }
  };
  float sum = 0.f, dev = 0.f;
  each([&](float n, float mean, float) { sum = __builtin_fmaf(n, mean, sum); });
  const float mean = group_sum(sum, lds) * inv;
  // what the rounding of the mean leaves is taken out of it: the deviations' own sum
  float rest = 0.f;
  each([&](float n, float m, float m2) {
    const float d = m - mean;
    rest = __builtin_fmaf(n, d, rest);
    dev += __builtin_fmaf(n * d, d, m2);
  });
  const float shift = group_sum(rest, lds) * inv;
  const float var = group_sum(dev, lds) * inv - shift * shift;
  if (threadIdx.x == 0) {
    p.mean_out[sample * p.groups + g] = mean + shift;
    p.rstd_out[sample * p.groups + g] = 1.f / sqrtf((var > 0.f || var != var ? var : 0.f) + p.eps);
  }
}

template <typename T>
__global__ __launch_bounds__(NT) void norm_apply_kernel(NormP p) {
  // backwards through the jobs: what the statistics read last is still in the cache
  const Place t = place(p, gridDim.x - 1 - blockIdx.x);
  if (t.cnt <= 0) return;
  const Coef k(p, t.sample, t.c);
  float scale[V];
#pragma unroll
  for (int e = 0; e < V; ++e) scale[e] = k.rstd[e] * k.gamma[e];
  const T* x = (const T*)p.x + t.row0 * p.ldx + t.c;
  T* y = (T*)p.out + t.row0 * p.ldo + t.c;
  with_act(p.act, [&](auto act) {
    for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
      Raw<T, V> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = raw<V>(x + (r + u * t.stride < t.rows ? r + u * t.stride : r) * p.ldx, t.cnt);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * t.stride < t.rows) {
          float o[V], slope;
#pragma unroll
          for (int e = 0; e < V; ++e) act_one<decltype(act)::value>(__builtin_fmaf(v[u].get(e) - k.mean[e], scale[e], k.beta[e]), o[e], slope);
          store4(y + (r + u * t.stride) * p.ldo, t.cnt, o);
        }
    }
  });
}

// dv = dy act'(gamma xhat + beta), and xhat.
template <int ACT, typename T>
__device__ __forceinline__ void slope4(const Coef& k, const Raw<T, V>& x, const Raw<T, V>& dy, float (&hat)[V], float (&dv)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    float value, slope;
    hat[e] = (x.get(e) - k.mean[e]) * k.rstd[e];
    act_one<ACT>(__builtin_fmaf(k.gamma[e], hat[e], k.beta[e]), value, slope);
    dv[e] = dy.get(e) * slope;
  }
}

template <typename T>
__global__ __launch_bounds__(NT) void norm_sums_kernel(NormP p) {
  __shared__ float s_a[WAVES][64][V], s_b[WAVES][64][V];
  const Place t = place(p, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float a[V] = {}, b[V] = {};
  if (t.cnt > 0) {
    const Coef k(p, t.sample, t.c);
    const T *x = (const T*)p.x + t.row0 * p.ldx + t.c, *dy = (const T*)p.dy + t.row0 * p.ldy + t.c;
    with_act(p.act, [&](auto act) {
      for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
        Raw<T, V> v[U], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const long long row = r + u * t.stride < t.rows ? r + u * t.stride : r;
          v[u] = raw<V>(x + row * p.ldx, t.cnt);
          d[u] = raw<V>(dy + row * p.ldy, t.cnt);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (r + u * t.stride < t.rows) {
            float hat[V], dv[V];
            slope4<decltype(act)::value, T>(k, v[u], d[u], hat, dv);
#pragma unroll
            for (int e = 0; e < V; ++e) {
              a[e] += dv[e];
              b[e] = __builtin_fmaf(dv[e], hat[e], b[e]);
            }
          }
      }
    });
  }
#pragma unroll
  for (int e = 0; e < V; ++e) { s_a[wave][lane][e] = a[e]; s_b[wave][lane][e] = b[e]; }
  __syncthreads();
  if (threadIdx.x >= p.lpr || t.cnt <= 0) return;
  for (int i = 1; i < WAVES * (64 / p.lpr); ++i) {
    const int w = i / (64 / p.lpr), l = i % (64 / p.lpr) * p.lpr + lane;
#pragma unroll
    for (int e = 0; e < V; ++e) { a[e] += s_a[w][l][e]; b[e] += s_b[w][l][e]; }
  }
  float* to = p.part + (t.sample * p.chunks + t.chunk) * 2 * p.c + t.c;
  store4(to, t.cnt, a);
  store4(to + p.c, t.cnt, b);
}

// Means over a group of gamma dv and of gamma dv xhat.
__global__ __launch_bounds__(256) void norm_join_bwd_kernel(NormP p) {
  __shared__ float lds[4];
  const int g = blockIdx.x % p.groups;
  const long long sample = p.sample0 + blockIdx.x / p.groups, items = (long long)p.chunks * p.cg;
  const float* part = p.part + sample * p.chunks * 2 * p.c + g * p.cg;
  float a = 0.f, b = 0.f;
  for (long long i = threadIdx.x; i < items; i += 256) {
    const int chunk = (int)(i / p.cg), c = (int)(i - (long long)chunk * p.cg);
    const float gamma = p.gamma ? p.gamma[g * p.cg + c] : 1.f;
    const float* at = part + (long long)chunk * 2 * p.c + c;
    a = __builtin_fmaf(gamma, at[0], a);
    b = __builtin_fmaf(gamma, at[p.c], b);
  }
  const float inv = 1.f / ((float)p.s * (float)p.cg);
  a = group_sum(a, lds) * inv;
  b = group_sum(b, lds) * inv;
  if (threadIdx.x == 0) {
    p.coef[(sample * p.groups + g) * 2] = a;
    p.coef[(sample * p.groups + g) * 2 + 1] = b;
  }
}

template <typename T>
__global__ __launch_bounds__(NT) void norm_dx_kernel(NormP p) {
  const Place t = place(p, gridDim.x - 1 - blockIdx.x);
  if (t.cnt <= 0) return;
  const Coef k(p, t.sample, t.c);
  float m1[V], m2[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    m1[e] = p.coef[(t.sample * p.groups + k.group[e]) * 2];
    m2[e] = p.coef[(t.sample * p.groups + k.group[e]) * 2 + 1];
  }
  const T *x = (const T*)p.x + t.row0 * p.ldx + t.c, *dy = (const T*)p.dy + t.row0 * p.ldy + t.c;
  T* dx = (T*)p.out + t.row0 * p.ldo + t.c;
  with_act(p.act, [&](auto act) {
    for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
      Raw<T, V> v[U], d[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long row = r + u * t.stride < t.rows ? r + u * t.stride : r;
        v[u] = raw<V>(x + row * p.ldx, t.cnt);
        d[u] = raw<V>(dy + row * p.ldy, t.cnt);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * t.stride < t.rows) {
          float hat[V], dv[V];
          slope4<decltype(act)::value, T>(k, v[u], d[u], hat, dv);
#pragma unroll
          for (int e = 0; e < V; ++e) dv[e] = k.rstd[e] * (__builtin_fmaf(k.gamma[e], dv[e], -m1[e]) - hat[e] * m2[e]);
          store4(dx + (r + u * t.stride) * p.ldo, t.cnt, dv);
        }
    }
  });
}

// dbeta and dgamma from the sums of all samples' chunks, in order.
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* part, long long rows, int c, float* dgamma, float* dbeta) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, way = threadIdx.x >> 5;
  const long long n = (long long)blockIdx.x * 32 + lane;          // column of 2 c
  float t = 0.f;
  if (n < 2LL * c) {
    long long i = way;
    for (; i + 56 < rows; i += 64) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = part[(i + 8 * u) * 2 * c + n];
      t += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    for (; i < rows; i += 8) t += part[i * 2 * c + n];
  }
  sums[way][lane] = t;
  __syncthreads();
  if (way != 0 || n >= 2LL * c) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) t += sums[w][lane];
  if (n < c) { if (dbeta) dbeta[n] = t; }
  else if (dgamma) dgamma[n - c] = t;
}

// ---- sizes ----
struct Split {
  int lpr, cblocks, chunks;
  long long chunk_rows;
};
Split split_of(const lms_group_norm_desc* d) {
  Split t;
  for (t.lpr = 1; t.lpr < 64 && t.lpr * V < d->c;) t.lpr *= 2;
  t.cblocks = (d->c + t.lpr * V - 1) / (t.lpr * V);
  const long long step = (long long)WAVES * (64 / t.lpr) * U, most = (d->s + step - 1) / step;
  const long long jobs = d->n * t.cblocks, want = jobs >= 2048 ? 1 : (2048 + jobs - 1) / (jobs ? jobs : 1);
  const long long chunks = want < most ? want : most;
  t.chunk_rows = ((d->s + chunks - 1) / chunks + step - 1) / step * step;
  t.chunks = (int)((d->s + t.chunk_rows - 1) / t.chunk_rows);
  return t;
}
// Samples that are taken together.
long long part_samples(const lms_group_norm_desc* d, const Split& t, int tensors) {
  const long long bytes = d->s * d->c * (d->dtype == LMS_F32 ? 4 : 2) * tensors, fit = PART_BYTES / bytes > 0 ? PART_BYTES / bytes : 1;
  const long long jobs = (long long)t.chunks * t.cblocks, groups = d->groups, each = jobs > groups ? jobs : groups, most = (1LL << 22) / each > 0 ? (1LL << 22) / each : 1;
  const long long n = fit < most ? fit : most;
  return n < d->n ? n : d->n;
}

lms_status check(const char* what, const lms_group_norm_desc* d) {
  NEED(d->n >= 0 && d->s >= 1 && d->c >= 1, "%s: samples must be >= 0, positions and channels >= 1", what);
  NEED(d->c <= 1 << 20, "%s: more than 2^20 channels", what);
  NEED(d->n <= 0x7fffffffLL && d->s <= 0x7fffffffLL && d->n * d->s <= 0x7fffffffLL, "%s: more than 2^31 - 1 rows", what);
  NEED(d->groups >= 1 && d->c % d->groups == 0, "%s: the channels must be a multiple of the groups", what);
  NEED(d->act >= LMS_ACT_NONE && d->act <= LMS_ACT_GELU_TANH, "%s: unknown activation %d", what, d->act);
  NEED(d->dtype == LMS_BF16 || d->dtype == LMS_F32, "%s: dtype must be LMS_BF16 or LMS_F32", what);
  NEED(d->eps > 0.f && d->eps < __builtin_inff(), "%s: eps must be positive and finite", what);
  const long long most = 1LL << 40;
  NEED((d->ldx == 0 || (d->ldx >= d->c && d->ldx <= most)) && (d->ldy == 0 || (d->ldy >= d->c && d->ldy <= most)),
       "%s: a row pitch is shorter than the row, or above 2^40", what);
  return LMS_OK;
}
lms_status aligned(const char* what, const lms_group_norm_desc* d, const void* a, const void* b, const void* c, std::initializer_list<const void*> words) {
  const uintptr_t rows = (uintptr_t)a | (uintptr_t)b | (uintptr_t)c;
  uintptr_t w = 0;
  for (const void* q : words) w |= (uintptr_t)q;
  NEED((rows & (d->dtype == LMS_F32 ? 3 : 1)) == 0 && (w & 3) == 0, "%s: a pointer is not aligned to its elements", what);
  return LMS_OK;
}
NormP params(const lms_group_norm_desc* d, const Split& t) {
  NormP p{};
  p.s = d->s; p.c = d->c; p.groups = d->groups; p.cg = d->c / d->groups; p.act = d->act; p.eps = d->eps;
  p.ldx = d->ldx ? d->ldx : d->c; p.ldy = d->ldy ? d->ldy : d->c;
  p.chunks = t.chunks; p.chunk_rows = t.chunk_rows; p.cblocks = t.cblocks; p.lpr = t.lpr;
  return p;
}

template <typename T>
hipError_t forward(const lms_group_norm_desc* d, const Split& t, NormP& p, hipStream_t s) {
  const long long part = part_samples(d, t, 1);
  for (p.sample0 = 0; p.sample0 < d->n; p.sample0 += part) {
    const long long take = d->n - p.sample0 < part ? d->n - p.sample0 : part;
    const dim3 jobs((unsigned)(take * t.chunks * t.cblocks));
    hipLaunchKernelGGL(norm_stats_kernel<T>, jobs, dim3(NT), 0, s, p);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(take * d->groups)), dim3(256), 0, s, p);
    hipLaunchKernelGGL(norm_apply_kernel<T>, jobs, dim3(NT), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t backward(const lms_group_norm_desc* d, const Split& t, NormP& p, float* dgamma, float* dbeta, hipStream_t s) {
  const long long part = part_samples(d, t, 2);
  for (p.sample0 = 0; p.sample0 < d->n; p.sample0 += part) {
    const long long take = d->n - p.sample0 < part ? d->n - p.sample0 : part;
    const dim3 jobs((unsigned)(take * t.chunks * t.cblocks));
    hipLaunchKernelGGL(norm_sums_kernel<T>, jobs, dim3(NT), 0, s, p);
    if (p.out) {
      hipLaunchKernelGGL(norm_join_bwd_kernel, dim3((unsigned)(take * d->groups)), dim3(256), 0, s, p);
      hipLaunchKernelGGL(norm_dx_kernel<T>, jobs, dim3(NT), 0, s, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!dgamma && !dbeta) return hipSuccess;
  hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((2LL * d->c + 31) / 32)), dim3(256), 0, s, p.part, d->n * t.chunks, d->c, dgamma, dbeta);
  return hipGetLastError();
}

uint64_t stat_bytes(const lms_group_norm_desc* d) { return up256((uint64_t)d->n * d->groups * 4); }
uint64_t part_bytes(const lms_group_norm_desc* d, const Split& t, long long samples) { return up256((uint64_t)samples * t.chunks * 2 * d->c * 4); }

}  // namespace

lms_status group_norm_workspace(const lms_group_norm_desc* d, int which, uint64_t* bytes) {
  if (const lms_status st = check("lms_group_norm_workspace_bytes", d)) return st;
  NEED(which == LMS_GROUP_NORM_FWD || which == LMS_GROUP_NORM_BWD, "lms_group_norm_workspace_bytes: unknown call %d", which);
  const Split t = split_of(d);
  if (d->n == 0) *bytes = 0;
  else if (which == LMS_GROUP_NORM_FWD) *bytes = part_bytes(d, t, part_samples(d, t, 1)) + 2 * stat_bytes(d);
  else *bytes = part_bytes(d, t, d->n) + 2 * stat_bytes(d);
  return LMS_OK;
}

lms_status group_norm_fwd(const lms_group_norm_desc* d, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, void* ws, void* stream) {
  const char* what = "lms_group_norm_fwd";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, x, y, nullptr, {gamma, beta, mean, rstd})) return st;
  if (d->n == 0) return LMS_OK;
  NEED(ws, "%s: workspace required", what);
  NEED(((uintptr_t)ws & 15) == 0, "%s: the workspace is not aligned", what);
  const Split t = split_of(d);
  NormP p = params(d, t);
  char* at = (char*)ws;
  p.mean_out = mean ? mean : (float*)at;
  p.rstd_out = rstd ? rstd : (float*)(at + stat_bytes(d));
  p.mean = p.mean_out; p.rstd = p.rstd_out;
  p.part = (float*)(at + 2 * stat_bytes(d));
  p.x = x; p.gamma = gamma; p.beta = beta; p.out = y; p.ldo = p.ldy;
  hipStream_t s = (hipStream_t)stream;
  return done(what, d->dtype == LMS_F32 ? forward<float>(d, t, p, s) : forward<uint16_t>(d, t, p, s));
}

lms_status group_norm_bwd(const lms_group_norm_desc* d, const void* dy, const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd, void* dx,
                          float* dgamma, float* dbeta, void* ws, void* stream) {
  const char* what = "lms_group_norm_bwd";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, dy, x, dx, {gamma, beta, mean, rstd, dgamma, dbeta})) return st;
  NEED(d->n == 0 || ws, "%s: workspace required", what);
  NEED(((uintptr_t)ws & 15) == 0, "%s: the workspace is not aligned", what);
  const Split t = split_of(d);
  NormP p = params(d, t);
  p.coef = (float*)ws;
  p.part = (float*)((char*)ws + 2 * stat_bytes(d));
  p.x = x; p.dy = dy; p.gamma = gamma; p.beta = beta; p.mean = mean; p.rstd = rstd; p.out = dx; p.ldo = p.ldx;
  hipStream_t s = (hipStream_t)stream;
  return done(what, d->dtype == LMS_F32 ? backward<float>(d, t, p, dgamma, dbeta, s) : backward<uint16_t>(d, t, p, dgamma, dbeta, s));
}

}  // namespace lms
