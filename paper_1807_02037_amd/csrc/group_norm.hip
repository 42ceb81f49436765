// Group normalisation with an activation, channels last, and its backward pass (include/lms.h has the formulas).
//
// Sums over a sample's positions and a group's channels come from partial ones: a work-group takes a chunk of a sample's positions and up to 256 channels and leaves, for each channel, mean
// and sum of squared deviations (backwards: sums of dv and of dv xhat); a second launch joins the chunks and channels of each group; the third computes the results.  Deviations are from the mean of the rows that a thread holds, and
// means are joined with what their distances add, so that nothing cancels however far the mean is from zero.  The inputs are read twice: 128^3 positions x 64 channels in bf16, forward, 76 + 8 + 97 us,
// 4.6 TB/s over three passes (a copy of 1 GiB reaches 5.05); sums of powers of x, and samples a part at a time, so that the second read comes from the last-level cache, gave nothing.
//
// Samples that the registers of a work-group hold are read once: see below.
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "kernels.hpp"
#include "rows4.hpp"

namespace lms {

namespace {

constexpr int NT = 512, WAVES = NT / 64;
constexpr int U = 8;                   // rows of a thread in flight

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
  bool there;
};
// WHOLE: at least four channels.  The last vector of a row that would end beyond it begins earlier instead, and its first channels are computed twice, alike.
template <bool WHOLE>
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
  t.there = t.c < p.c;
  if (WHOLE && t.c > p.c - V) t.c = p.c - V;
  t.cnt = WHOLE ? V : p.c - t.c;
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
  const float share = nb * __builtin_amdgcn_rcpf(all);            // within an ulp: it weighs a distance
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float d = mb[e] - mean[e];
    mean[e] = __builtin_fmaf(d, share, mean[e]);
    m2[e] += __builtin_fmaf(d * d, n * share, qb[e]);
  }
  n = all;
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(NT) void norm_stats_kernel(NormP p) {
  __shared__ float s_n[WAVES][64], s_mean[WAVES][64][V], s_m2[WAVES][64][V];
  constexpr int U = 4;                                            // and the next four on their way: registers for four work-groups on a compute unit
  const Place t = place<WHOLE>(p, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float n = 0.f, mean[V] = {}, m2[V] = {};
  const T* x = (const T*)p.x + t.row0 * p.ldx + t.c;
  if (t.there) {
    Raw<T, V> v[U], next[U];
    const T *const begin = x + t.first * p.ldx, *from = begin;
    const long long step = t.stride * p.ldx;
    auto ask = [&](long long r) {                                 // rows beyond the last: the thread's first, for nothing
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = raw<V>(r + u * t.stride < t.rows ? from + u * step : begin, t.cnt);
      from += U * step;
    };
    if (t.first < t.rows) ask(t.first);
    for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = next[u];
      if (r + U * t.stride < t.rows) ask(r + U * t.stride);       // while these are worked on
      float nb = 0.f, mb[V] = {}, qb[V] = {};
      auto batch = [&](auto whole) {
        auto have = [&](int u) { return decltype(whole)::value || r + u * t.stride < t.rows; };
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (have(u)) {
            nb += 1.f;
#pragma unroll
            for (int e = 0; e < V; ++e) mb[e] += v[u].get(e);
          }
        const float inv = decltype(whole)::value ? 1.f / U : 1.f / nb;
#pragma unroll
        for (int e = 0; e < V; ++e) mb[e] *= inv;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (have(u))
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float d = v[u].get(e) - mb[e];
              qb[e] = __builtin_fmaf(d, d, qb[e]);
            }
      };
      if (r + (U - 1) * t.stride < t.rows) batch(std::true_type{});
      else batch(std::false_type{});
      merge(n, mean, m2, nb, mb, qb);
    }
  }
  for (int d = p.lpr; d < 64; d *= 2) {                           // the wave's rows of this column; both sides compute the same
    const bool upper = lane & d;
    float mb[V], qb[V];
    const float nb = __shfl_xor(n, d);
#pragma unroll
    for (int e = 0; e < V; ++e) { mb[e] = __shfl_xor(mean[e], d); qb[e] = __shfl_xor(m2[e], d); }
    if (!upper) merge(n, mean, m2, nb, mb, qb);
  }
  s_n[wave][lane] = n;
#pragma unroll
  for (int e = 0; e < V; ++e) { s_mean[wave][lane][e] = mean[e]; s_m2[wave][lane][e] = m2[e]; }
  __syncthreads();
  if (threadIdx.x >= p.lpr || !t.there) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    float mb[V], qb[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { mb[e] = s_mean[w][lane][e]; qb[e] = s_m2[w][lane][e]; }
    merge(n, mean, m2, s_n[w][lane], mb, qb);
  }
  float* to = p.part + ((t.sample - p.sample0) * p.chunks + t.chunk) * 2 * p.c + t.c;
  store4(to, t.cnt, mean);
  store4(to + p.c, t.cnt, m2);
}

// Sums of v and w over a work-group of JT threads, in a fixed order.
constexpr int JT = 1024;
__device__ __forceinline__ void group_sum(float& v, float& w, float (&lds)[2][JT / 64]) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    v += __shfl_xor(v, d);
    w += __shfl_xor(w, d);
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) { lds[0][threadIdx.x >> 6] = v; lds[1][threadIdx.x >> 6] = w; }
  __syncthreads();
  v = w = 0.f;
#pragma unroll
  for (int i = 0; i < JT / 64; ++i) { v += lds[0][i]; w += lds[1][i]; }
}
// f(chunk, channel of the group, the chunk's two values of the channel) for a group's chunks and channels, four in flight.
template <typename F>
__device__ __forceinline__ void each_partial(const NormP& p, const float* part, F&& f) {
  constexpr int IN_FLIGHT = 4;
  const int items = p.chunks * p.cg, dchunk = JT / p.cg, dc = JT - dchunk * p.cg;
  int chunk = (int)threadIdx.x / p.cg, c = (int)threadIdx.x - chunk * p.cg;
  for (int i = threadIdx.x; i < items; i += IN_FLIGHT * JT) {
    float a[IN_FLIGHT], b[IN_FLIGHT];
    int ch[IN_FLIGHT], cc[IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) {
      ch[u] = chunk;
      cc[u] = c;
      const float* at = part + (i + u * JT < items ? (long long)chunk * 2 * p.c + c : 0);
      a[u] = at[0];
      b[u] = at[p.c];
      chunk += dchunk;
      c += dc;
      if (c >= p.cg) { c -= p.cg; ++chunk; }
    }
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u)
      if (i + u * JT < items) f(ch[u], cc[u], a[u], b[u]);
  }
}

// Mean and 1 / deviation of a group from its channels' chunks.
__global__ __launch_bounds__(JT) void norm_join_kernel(NormP p) {
  __shared__ float lds[2][JT / 64];
  const int g = blockIdx.x % p.groups;
  const long long local = blockIdx.x / p.groups, sample = p.sample0 + local;
  const float* part = p.part + local * p.chunks * 2 * p.c + g * p.cg;
  const float inv = 1.f / ((float)p.s * (float)p.cg);
  const float full = (float)p.chunk_rows, last = (float)(p.s - (p.chunks - 1) * p.chunk_rows);      // rows of a chunk
  float sum = 0.f, unused = 0.f;
  each_partial(p, part, [&](int chunk, int, float mean, float) { sum = __builtin_fmaf(chunk + 1 < p.chunks ? full : last, mean, sum); });
  group_sum(sum, unused, lds);
  const float mean = sum * inv;
  // what the rounding of the mean leaves is taken out of it: the deviations' own sum
  float rest = 0.f, dev = 0.f;
  each_partial(p, part, [&](int chunk, int, float m, float m2) {
    const float n = chunk + 1 < p.chunks ? full : last, d = m - mean;
    rest = __builtin_fmaf(n, d, rest);
    dev += __builtin_fmaf(n * d, d, m2);
  });
  group_sum(rest, dev, lds);
  const float shift = rest * inv, var = dev * inv - shift * shift;
  if (threadIdx.x == 0) {
    p.mean_out[sample * p.groups + g] = mean + shift;
    p.rstd_out[sample * p.groups + g] = 1.f / sqrtf((var > 0.f || var != var ? var : 0.f) + p.eps);
  }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(NT) void norm_apply_kernel(NormP p) {
  // backwards through the jobs: what the statistics read last is still in the cache
  const Place t = place<WHOLE>(p, gridDim.x - 1 - blockIdx.x);
  if (!t.there) return;
  const Coef k(p, t.sample, t.c);
  float scale[V];
#pragma unroll
  for (int e = 0; e < V; ++e) scale[e] = k.rstd[e] * k.gamma[e];
  const long long xstep = t.stride * p.ldx, ystep = t.stride * p.ldo;
  const T* x = (const T*)p.x + (t.row0 + t.first) * p.ldx + t.c;
  T* y = (T*)p.out + (t.row0 + t.first) * p.ldo + t.c;
  with_act(p.act, [&](auto act) {
    for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
      Raw<T, V> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = raw<V>(x + (r + u * t.stride < t.rows ? u * xstep : 0), t.cnt);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * t.stride < t.rows) {
          float o[V], slope;
#pragma unroll
          for (int e = 0; e < V; ++e) act_one<decltype(act)::value>(__builtin_fmaf(v[u].get(e) - k.mean[e], scale[e], k.beta[e]), o[e], slope);
          store4(y + u * ystep, t.cnt, o);
        }
      x += U * xstep;
      y += U * ystep;
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

template <typename T, bool WHOLE>
__global__ __launch_bounds__(NT) void norm_sums_kernel(NormP p) {
  __shared__ float s_a[WAVES][64][V], s_b[WAVES][64][V];
  const Place t = place<WHOLE>(p, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float a[V] = {}, b[V] = {};
  if (t.there) {
    const Coef k(p, t.sample, t.c);
    const long long xstep = t.stride * p.ldx, dstep = t.stride * p.ldy;
    const T *x = (const T*)p.x + (t.row0 + t.first) * p.ldx + t.c, *dy = (const T*)p.dy + (t.row0 + t.first) * p.ldy + t.c;
    with_act(p.act, [&](auto act) {
      for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
        Raw<T, V> v[U], d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const bool have = r + u * t.stride < t.rows;
          v[u] = raw<V>(x + (have ? u * xstep : 0), t.cnt);
          d[u] = raw<V>(dy + (have ? u * dstep : 0), t.cnt);
        }
        x += U * xstep;
        dy += U * dstep;
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
  for (int d = p.lpr; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < V; ++e) { a[e] += __shfl_xor(a[e], d); b[e] += __shfl_xor(b[e], d); }
#pragma unroll
  for (int e = 0; e < V; ++e) { s_a[wave][lane][e] = a[e]; s_b[wave][lane][e] = b[e]; }
  __syncthreads();
  if (threadIdx.x >= p.lpr || !t.there) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w)
#pragma unroll
    for (int e = 0; e < V; ++e) { a[e] += s_a[w][lane][e]; b[e] += s_b[w][lane][e]; }
  float* to = p.part + (t.sample * p.chunks + t.chunk) * 2 * p.c + t.c;
  store4(to, t.cnt, a);
  store4(to + p.c, t.cnt, b);
}

// Means over a group of gamma dv and of gamma dv xhat.
__global__ __launch_bounds__(JT) void norm_join_bwd_kernel(NormP p) {
  __shared__ float lds[2][JT / 64];
  const int g = blockIdx.x % p.groups;
  const long long sample = p.sample0 + blockIdx.x / p.groups;
  float a = 0.f, b = 0.f;
  each_partial(p, p.part + sample * p.chunks * 2 * p.c + g * p.cg, [&](int, int c, float va, float vb) {
    const float gamma = p.gamma ? p.gamma[g * p.cg + c] : 1.f;
    a = __builtin_fmaf(gamma, va, a);
    b = __builtin_fmaf(gamma, vb, b);
  });
  group_sum(a, b, lds);
  const float inv = 1.f / ((float)p.s * (float)p.cg);
  if (threadIdx.x == 0) {
    p.coef[(sample * p.groups + g) * 2] = a * inv;
    p.coef[(sample * p.groups + g) * 2 + 1] = b * inv;
  }
}

template <typename T, bool WHOLE>
__global__ __launch_bounds__(NT) void norm_dx_kernel(NormP p) {
  const Place t = place<WHOLE>(p, gridDim.x - 1 - blockIdx.x);
  if (!t.there) return;
  const Coef k(p, t.sample, t.c);
  float m1[V], m2[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    m1[e] = p.coef[(t.sample * p.groups + k.group[e]) * 2];
    m2[e] = p.coef[(t.sample * p.groups + k.group[e]) * 2 + 1];
  }
  const long long xstep = t.stride * p.ldx, dstep = t.stride * p.ldy, ostep = t.stride * p.ldo;
  const T *x = (const T*)p.x + (t.row0 + t.first) * p.ldx + t.c, *dy = (const T*)p.dy + (t.row0 + t.first) * p.ldy + t.c;
  T* dx = (T*)p.out + (t.row0 + t.first) * p.ldo + t.c;
  with_act(p.act, [&](auto act) {
    for (long long r = t.first; r < t.rows; r += (long long)U * t.stride) {
      Raw<T, V> v[U], d[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool have = r + u * t.stride < t.rows;
        v[u] = raw<V>(x + (have ? u * xstep : 0), t.cnt);
        d[u] = raw<V>(dy + (have ? u * dstep : 0), t.cnt);
      }
      x += U * xstep;
      dy += U * dstep;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * t.stride < t.rows) {
          float hat[V], dv[V];
          slope4<decltype(act)::value, T>(k, v[u], d[u], hat, dv);
#pragma unroll
          for (int e = 0; e < V; ++e) dv[e] = k.rstd[e] * (__builtin_fmaf(k.gamma[e], dv[e], -m1[e]) - hat[e] * m2[e]);
          store4(dx + u * ostep, t.cnt, dv);
        }
      dx += U * ostep;
    }
  });
}

// ---- samples that a work-group holds ----
//
// Groups of whole vectors of eight channels (tokens: of any width, at the price of LDS traffic).  A work-group keeps what it has read in registers from the one read to the one write.
// us, bf16, backward: 8192 tokens x 4096 41 + 5 for gamma and beta (4.9 TB/s; by the launches above 1865), 64 samples of 196 positions x 1024 23 + 5 (3.4 TB/s, two rounds of work-groups each of which waits for its
// loads, its three barriers and its stores in turn; by the launches above 46).

constexpr int W = 8;                   // channels of a vector here

struct ResidentP {
  NormP n;
  long long samples;
  int lanes;                           // tokens: lanes of a row, a power of two
  int span, parts;                     // tokens: lanes that meet by shuffles, a power of two, and how many such make a group
  int block, blocks;                   // images: vectors of a work-group's channels, and how many such blocks there are
  int gv;                              // vectors of a group
};

// eight values of a vector
template <int ACT, typename T>
__device__ __forceinline__ void slope8(const float (&ga)[W], const float (&be)[W], float mean, float rstd, const Raw<T, W>& x, const Raw<T, W>& dy, float (&hat)[W], float (&dv)[W]) {
#pragma unroll
  for (int e = 0; e < W; ++e) {
    float value, slope;
    hat[e] = (x.get(e) - mean) * rstd;
    act_one<ACT>(__builtin_fmaf(ga[e], hat[e], be[e]), value, slope);
    dv[e] = dy.get(e) * slope;
  }
}
// A vector, or zeros.
template <typename T>
__device__ __forceinline__ Raw<T, W> vector(const T* p, bool there) {
  Raw<T, W> r = {};
  if (there) __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
// Makes the compiler compute anew what it has computed of these: kept, it takes twice their registers.
template <typename T, int N>
__device__ __forceinline__ void anew(Raw<T, W> (&t)[N]) {
#pragma unroll
  for (auto& v : t)
#pragma unroll
    for (unsigned& w : v.q) asm volatile("" : "+v"(w));
}
__device__ __forceinline__ void weights8(const NormP& p, int c, bool there, float (&ga)[W], float (&be)[W]) {
#pragma unroll
  for (int e = 0; e < W; ++e) { ga[e] = 1.f; be[e] = 0.f; }
  if (there && p.gamma) load8(p.gamma + c, W, ga);
  if (there && p.beta) load8(p.beta + c, W, be);
}

// Tokens (s = 1).  A row takes `lanes` lanes of K vectors each; rows of a work-group run in parallel, and it goes on to others, the next row's loads out before this one is worked on.  A group's
// vectors meet by shuffles, as far as its lanes go in powers of two within a wave, the rest in LDS, in two buffers by turns: one barrier for up to DIRECT parts, which every thread adds up for itself
// (8192 x 4096 in one group, forward 54 us with a barrier for each of three steps, 42 so).  Backwards the sums for gamma and beta stay in registers until the work-group's last row.
template <typename T, int NT, int K, bool BWD>
__global__ __launch_bounds__(NT) void norm_tokens_kernel(ResidentP q) {
  constexpr int DIRECT = 16;
  __shared__ float s_part[2][2][NT * K], s_sum[2][2][NT * K / DIRECT];
  const NormP& p = q.n;
  const int tid = threadIdx.x, l = tid & (q.lanes - 1), sub = tid / q.lanes, rows = NT / q.lanes, nv = p.c / W, each = q.lanes * K / q.span;     // each: parts of a row
  int buffer = 0;
  auto vec = [&](int j) { return l + j * q.lanes; };
  float ga[K][W], be[K][W], da[BWD ? K : 1][W] = {}, db[BWD ? K : 1][W] = {};
#pragma unroll
  for (int j = 0; j < K; ++j) weights8(p, vec(j) * W, vec(j) < nv, ga[j], be[j]);
  Raw<T, W> x[K], dy[BWD ? K : 1], nx[K], ndy[BWD ? K : 1];
  float mean[BWD ? K : 1], rstd[BWD ? K : 1], nmean[BWD ? K : 1], nrstd[BWD ? K : 1];
  auto ask = [&](long long row) {
    const bool there = row < q.samples;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const bool cnt = there && vec(j) < nv;
      nx[j] = vector((const T*)p.x + row * p.ldx + vec(j) * W, cnt);
      if constexpr (BWD) {
        ndy[j] = vector((const T*)p.dy + row * p.ldy + vec(j) * W, cnt);
        nmean[j] = cnt ? p.mean[row * p.groups + vec(j) / q.gv] : 0.f;
        nrstd[j] = cnt ? p.rstd[row * p.groups + vec(j) / q.gv] : 0.f;
      }
    }
  };
  // a[j] and b[j] of each vector into the sums over its group
  const bool fold = K > 1 && p.groups == 1;                       // a thread's vectors are of one group
  auto join = [&](float (&a)[K], float (&b)[K], bool two) {
    if (fold) {
#pragma unroll
      for (int j = 1; j < K; ++j) {
        a[0] += a[j];
        b[0] += b[j];
        a[j] = b[j] = 0.f;
      }
    }
    for (int d = 1; d < q.span; d *= 2)
#pragma unroll
      for (int j = 0; j < K; ++j) {
        a[j] += __shfl_xor(a[j], d);
        if (two) b[j] += __shfl_xor(b[j], d);
      }
    if (q.parts == 1) return;
    float (&part)[2][NT * K] = s_part[buffer], (&sum)[2][NT * K / DIRECT] = s_sum[buffer];
    buffer ^= 1;
    if (l % q.span == 0)
#pragma unroll
      for (int j = 0; j < K; ++j) {
        part[0][sub * each + vec(j) / q.span] = a[j];
        part[1][sub * each + vec(j) / q.span] = b[j];
      }
    __syncthreads();                                              // this buffer's last readers have come through the other's barrier since
    if (q.parts <= DIRECT) {
#pragma unroll
      for (int j = 0; j < K; ++j) {
        if (fold && j > 0) {
          a[j] = a[0];
          b[j] = b[0];
          continue;
        }
        a[j] = b[j] = 0.f;
        if (vec(j) >= nv) continue;
        const int at = sub * each + vec(j) / q.gv * q.parts;
        for (int k = 0; k < (fold ? q.lanes / q.span : q.parts); ++k) {
          a[j] += part[0][at + k];
          b[j] += part[1][at + k];
        }
      }
      return;
    }
    int team = 1;
    while (team < 64 && team < q.parts && 2 * team * rows * p.groups <= NT) team *= 2;
    for (int i = tid / team; i < rows * p.groups; i += NT / team) {
      const int at = i / p.groups * each + i % p.groups * q.parts;
      float ta = 0.f, tb = 0.f;
      for (int k = tid & (team - 1); k < q.parts; k += team) {
        ta += part[0][at + k];
        tb += part[1][at + k];
      }
      for (int d = 1; d < team; d *= 2) {
        ta += __shfl_xor(ta, d);
        tb += __shfl_xor(tb, d);
      }
      if ((tid & (team - 1)) == 0) { sum[0][i] = ta; sum[1][i] = tb; }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (vec(j) < nv) {
        a[j] = sum[0][sub * p.groups + vec(j) / q.gv];
        b[j] = sum[1][sub * p.groups + vec(j) / q.gv];
      }
  };
  constexpr bool AHEAD = !BWD || NT < 1024;                       // registers
  const float inv = 1.f / (float)p.cg;
  const long long stride = (long long)gridDim.x * rows, first = (long long)blockIdx.x * rows;
  if (AHEAD) ask(first + sub);
  for (long long r0 = first; r0 < q.samples; r0 += stride) {      // the same for the whole work-group
    const long long row = r0 + sub;
    const bool there = row < q.samples;
    if (!AHEAD) ask(row);
#pragma unroll
    for (int j = 0; j < K; ++j) {
      x[j] = nx[j];
      if constexpr (BWD) { dy[j] = ndy[j]; mean[j] = nmean[j]; rstd[j] = nrstd[j]; }
    }
    if (AHEAD && r0 + stride < q.samples) ask(row + stride);
    float a[K], b[K];
    if constexpr (!BWD) {
#pragma unroll
      for (int j = 0; j < K; ++j) {
        a[j] = b[j] = 0.f;
#pragma unroll
        for (int e = 0; e < W; ++e) a[j] += x[j].get(e);
      }
      join(a, b, false);
      float m[K], d2[K];
#pragma unroll
      for (int j = 0; j < K; ++j) {
        m[j] = a[j] * inv;
        d2[j] = b[j] = 0.f;
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float d = vec(j) < nv ? x[j].get(e) - m[j] : 0.f;
          b[j] += d;                                              // what the rounding of the mean left
          d2[j] = __builtin_fmaf(d, d, d2[j]);
        }
      }
      join(d2, b, true);
#pragma unroll
      for (int j = 0; j < K; ++j) {
        const float shift = b[j] * inv, var = d2[j] * inv - shift * shift, rs = 1.f / sqrtf((var > 0.f || var != var ? var : 0.f) + p.eps);
        m[j] += shift;
        if (!there || vec(j) >= nv) continue;
        if (vec(j) % q.gv == 0) {
          p.mean_out[row * p.groups + vec(j) / q.gv] = m[j];
          p.rstd_out[row * p.groups + vec(j) / q.gv] = rs;
        }
        float y[W];
#pragma unroll
        for (int e = 0; e < W; ++e) y[e] = __builtin_fmaf((x[j].get(e) - m[j]) * rs, ga[j][e], be[j][e]);
        act8(p.act, y);
        store8((T*)p.out + row * p.ldo + vec(j) * W, W, y);
      }
    } else {
      float hat[K][W], dv[K][W];
      with_act(p.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < K; ++j) slope8<decltype(act)::value, T>(ga[j], be[j], mean[j], rstd[j], x[j], dy[j], hat[j], dv[j]);
      });
#pragma unroll
      for (int j = 0; j < K; ++j) {
        a[j] = b[j] = 0.f;
#pragma unroll
        for (int e = 0; e < W; ++e) {
          db[j][e] += dv[j][e];
          da[j][e] = __builtin_fmaf(dv[j][e], hat[j][e], da[j][e]);
          dv[j][e] *= ga[j][e];
          a[j] += dv[j][e];
          b[j] = __builtin_fmaf(dv[j][e], hat[j][e], b[j]);
        }
      }
      if (!p.out) continue;
      join(a, b, true);
#pragma unroll
      for (int j = 0; j < K; ++j) {
        if (!there || vec(j) >= nv) continue;
        float d[W];
#pragma unroll
        for (int e = 0; e < W; ++e) d[e] = rstd[j] * ((dv[j][e] - a[j] * inv) - hat[j][e] * (b[j] * inv));
        store8((T*)p.out + row * p.ldo + vec(j) * W, W, d);
      }
    }
  }
  if constexpr (BWD)
    if (p.part) {                                                 // the rows of a wave together first
      const int subs = q.lanes < 64 ? 64 / q.lanes : 1;
      for (int d = q.lanes; d < 64; d *= 2)
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
          for (int e = 0; e < W; ++e) {
            db[j][e] += __shfl_xor(db[j][e], d);
            da[j][e] += __shfl_xor(da[j][e], d);
          }
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (vec(j) < nv && sub % subs == 0) {
          float* to = p.part + ((long long)blockIdx.x * (rows / subs) + sub / subs) * 2 * p.c + vec(j) * W;
          store8(to, W, db[j]);
          store8(to + p.c, W, da[j]);
        }
    }
}

// Tokens whose groups, or rows, are not of whole vectors: the channels' values go through LDS, where a team of lanes sums each group's and finishes
// what is needed of them once (forward 8192 x 4100 in four groups 337 us with a root for each channel, 176 so; 100000 x 100 in five 64 and 46).
template <typename T, int NT, int K, bool BWD>
__global__ __launch_bounds__(NT, K == 1 ? 4 : 2) void norm_tokens_any_kernel(ResidentP q) {
  extern __shared__ float s_any[];
  const NormP& p = q.n;
  const int tid = threadIdx.x, l = tid & (q.lanes - 1), sub = tid / q.lanes, rows = NT / q.lanes, width = q.lanes * K * W;
  float *const s_a = s_any, *const s_b = s_a + rows * width, *const s_sum = s_b + rows * width;         // [row][channel], twice; [row][group][2]
  int team = 1;                                                   // as many lanes for a group as there are for all of them at once
  while (team < 64 && team < p.cg && 2 * team * rows * p.groups <= NT) team *= 2;
  auto at = [&](int j) { return (l + j * q.lanes) * W; };
  auto count = [&](int j) { return p.c - at(j) < W ? p.c - at(j) : W; };
  float ga[K][W], be[K][W], da[BWD ? K : 1][W] = {}, db[BWD ? K : 1][W] = {};
  int group[K][W];
#pragma unroll
  for (int j = 0; j < K; ++j)
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const bool there = at(j) + e < p.c;
      group[j][e] = (there ? at(j) + e : p.c - 1) / p.cg;
      ga[j][e] = there && p.gamma ? p.gamma[at(j) + e] : 1.f;
      be[j][e] = there && p.beta ? p.beta[at(j) + e] : 0.f;
    }
  // two values of each channel's group; forward only two groups' for a vector of eight, if they are not smaller (backward 8192 x 4100 in four groups 225 us so, 212 channel by channel)
  auto of_groups = [&](auto&& get, float (&a)[K][W], float (&b)[K][W]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (!BWD && p.cg >= W) {
        const float2 low = get(group[j][0]), high = get(group[j][W - 1]);
#pragma unroll
        for (int e = 0; e < W; ++e) {
          a[j][e] = group[j][e] == group[j][0] ? low.x : high.x;
          b[j][e] = group[j][e] == group[j][0] ? low.y : high.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float2 t = get(group[j][e]);
          a[j][e] = t.x;
          b[j][e] = t.y;
        }
      }
  };
  // the channels' values into what `finish` makes of the sums over their groups; its i: group i % groups of the work-group's row i / groups
  auto join = [&](float (&a)[K][W], float (&b)[K][W], auto two, auto&& finish) __attribute__((always_inline)) {
    constexpr bool TWO = decltype(two)::value;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < K; ++j) {
      store8(s_a + sub * width + at(j), W, a[j]);
      if constexpr (TWO) store8(s_b + sub * width + at(j), W, b[j]);
    }
    __syncthreads();
    for (int i = tid / team; i < rows * p.groups; i += NT / team) {
      const int from = i / p.groups * width + i % p.groups * p.cg;
      float ta = 0.f, tb = 0.f;
      for (int k = tid & (team - 1); k < p.cg; k += team) {
        ta += s_a[from + k];
        if constexpr (TWO) tb += s_b[from + k];
      }
      for (int d = 1; d < team; d *= 2) {
        ta += __shfl_xor(ta, d);
        if constexpr (TWO) tb += __shfl_xor(tb, d);
      }
      if ((tid & (team - 1)) == 0) {
        float2& to = reinterpret_cast<float2*>(s_sum)[i];
        to = finish(i, ta, tb, to);                               // the same thread's as the time before
      }
    }
    __syncthreads();
    of_groups([&](int g) { return reinterpret_cast<const float2*>(s_sum)[sub * p.groups + g]; }, a, b);
  };
  const float inv = 1.f / (float)p.cg;
  const long long stride = (long long)gridDim.x * rows;
  for (long long r0 = (long long)blockIdx.x * rows; r0 < q.samples; r0 += stride) {       // the same for the whole work-group
    const long long row = r0 + sub;
    const bool there = row < q.samples;
    Raw<T, W> x[K], dy[BWD ? K : 1];
    float a[K][W], b[K][W], mean[BWD ? K : 1][W], rstd[BWD ? K : 1][W];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      x[j] = raw<W>((const T*)p.x + row * p.ldx + at(j), there ? count(j) : 0);
      if constexpr (BWD) {
        dy[j] = raw<W>((const T*)p.dy + row * p.ldy + at(j), there ? count(j) : 0);
      }
    }
    if constexpr (BWD)
      of_groups([&](int g) { return there ? make_float2(p.mean[row * p.groups + g], p.rstd[row * p.groups + g]) : make_float2(0.f, 0.f); }, mean, rstd);
    if constexpr (!BWD) {
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int e = 0; e < W; ++e) { a[j][e] = x[j].get(e); b[j][e] = 0.f; }
      join(a, b, std::false_type{}, [&](int, float sum, float, float2) { return make_float2(sum * inv, 0.f); });
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int e = 0; e < W; ++e) {
          b[j][e] = x[j].get(e) - a[j][e];                        // their sum: what the rounding of the mean left
          a[j][e] = b[j][e] * b[j][e];
        }
      join(a, b, std::true_type{}, [&](int i, float squares, float rest, float2 before) {
        const float shift = rest * inv, var = squares * inv - shift * shift, rs = 1.f / sqrtf((var > 0.f || var != var ? var : 0.f) + p.eps), m = before.x + shift;
        const long long at = r0 + i / p.groups;
        if (at < q.samples) {
          p.mean_out[at * p.groups + i % p.groups] = m;
          p.rstd_out[at * p.groups + i % p.groups] = rs;
        }
        return make_float2(m, rs);
      });
#pragma unroll
      for (int j = 0; j < K; ++j) {
        if (!there || count(j) <= 0) continue;
        float y[W];
#pragma unroll
        for (int e = 0; e < W; ++e) y[e] = __builtin_fmaf((x[j].get(e) - a[j][e]) * b[j][e], ga[j][e], be[j][e]);
        act8(p.act, y);
        store8((T*)p.out + row * p.ldo + at(j), count(j), y);
      }
    } else {
      float hat[K][W], dv[K][W];
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int e = 0; e < W; ++e) hat[j][e] = (x[j].get(e) - mean[j][e]) * rstd[j][e];
      with_act(p.act, [&](auto act) {
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
          for (int e = 0; e < W; ++e) {
            float value, slope;
            act_one<decltype(act)::value>(__builtin_fmaf(ga[j][e], hat[j][e], be[j][e]), value, slope);
            dv[j][e] = dy[j].get(e) * slope;
          }
      });
#pragma unroll
      for (int j = 0; j < K; ++j)
#pragma unroll
        for (int e = 0; e < W; ++e) {
          db[j][e] += dv[j][e];
          da[j][e] = __builtin_fmaf(dv[j][e], hat[j][e], da[j][e]);
          a[j][e] = dv[j][e] *= ga[j][e];
          b[j][e] = dv[j][e] * hat[j][e];
        }
      if (!p.out) continue;
      join(a, b, std::true_type{}, [&](int, float ta, float tb, float2) { return make_float2(ta * inv, tb * inv); });
#pragma unroll
      for (int j = 0; j < K; ++j) {
        if (!there || count(j) <= 0) continue;
        float d[W];
#pragma unroll
        for (int e = 0; e < W; ++e) d[e] = rstd[j][e] * ((dv[j][e] - a[j][e]) - hat[j][e] * b[j][e]);
        store8((T*)p.out + row * p.ldo + at(j), count(j), d);
      }
    }
  }
  if constexpr (BWD)
    if (p.part) {                                                 // the rows of a wave together first
      const int subs = q.lanes < 64 ? 64 / q.lanes : 1;
      for (int d = q.lanes; d < 64; d *= 2)
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
          for (int e = 0; e < W; ++e) {
            db[j][e] += __shfl_xor(db[j][e], d);
            da[j][e] += __shfl_xor(da[j][e], d);
          }
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (count(j) > 0 && sub % subs == 0) {
          float* to = p.part + ((long long)blockIdx.x * (rows / subs) + sub / subs) * 2 * p.c + at(j);
          store8(to, count(j), db[j]);
          store8(to + p.c, count(j), da[j]);
        }
    }
}

// Images: a sample's positions of one block of whole groups, K positions of a vector of channels a thread.
template <typename T, int NT, int K, bool BWD>
__global__ __launch_bounds__(NT, sizeof(T) * K <= 8 ? 4 : 2) void norm_image_kernel(ResidentP q) {
  __shared__ float s_part[2][NT], s_sum[2][256];
  __shared__ float s_chan[BWD ? 2 : 1][BWD ? W : 1][BWD ? NT : 1];
  const NormP& p = q.n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nv = p.c / W;
  const long long sample = blockIdx.x / q.blocks;
  const int v0 = (int)(blockIdx.x % q.blocks) * q.block, mine = nv - v0 < q.block ? nv - v0 : q.block;       // vectors of this block
  const int lanes = NT / q.block, pos = tid / q.block, col = tid - pos * q.block, group = col / q.gv, groups = mine / q.gv;
  const bool there = pos < lanes && col < mine;
  const int c = (v0 + col) * W;
  const long long row0 = sample * p.s;
  float ga[W], be[W];
  weights8(p, c, there, ga, be);
  Raw<T, W> x[K], dy[BWD ? K : 1];
  float mean = 0.f, rstd = 0.f;
  const int left = there ? (int)(p.s - pos) : 0;                  // positions from this thread's first on
  auto have = [&](int j) { return j * lanes < left; };
  {
    const T *px = (const T*)p.x + (row0 + pos) * p.ldx + c, *pd = (const T*)p.dy + (row0 + pos) * p.ldy + c;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      x[j] = vector(px + j * (lanes * p.ldx), have(j));
      if constexpr (BWD) dy[j] = vector(pd + j * (lanes * p.ldy), have(j));
    }
  }
  T* const out = (T*)p.out + (row0 + pos) * p.ldo + c;
  if (BWD && there) {
    mean = p.mean[sample * p.groups + (v0 + col) / q.gv];
    rstd = p.rstd[sample * p.groups + (v0 + col) / q.gv];
  }
  auto join = [&](float& a, float& b) {                           // over the positions and a group's vectors
    __syncthreads();
    s_part[0][tid] = a;
    s_part[1][tid] = b;
    __syncthreads();
    for (int g = wave; g < groups; g += NT / 64) {
      float ta = 0.f, tb = 0.f;
      for (int i = lane; i < lanes * q.gv; i += 64) {
        const int at = i / q.gv * q.block + g * q.gv + i % q.gv;
        ta += s_part[0][at];
        tb += s_part[1][at];
      }
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        ta += __shfl_xor(ta, d);
        tb += __shfl_xor(tb, d);
      }
      if (lane == 0) { s_sum[0][g] = ta; s_sum[1][g] = tb; }
    }
    __syncthreads();
    if (there) { a = s_sum[0][group]; b = s_sum[1][group]; }
  };
  const float inv = 1.f / ((float)p.s * (float)p.cg);
  float a = 0.f, b = 0.f;
  if constexpr (!BWD) {
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int e = 0; e < W; ++e) a += x[j].get(e);               // zeros where there is no position
    join(a, b);
    mean = a * inv;
    a = b = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (have(j))
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float d = x[j].get(e) - mean;
          b += d;
          a = __builtin_fmaf(d, d, a);
        }
    join(a, b);
    const float shift = b * inv, var = a * inv - shift * shift;
    mean += shift;
    rstd = 1.f / sqrtf((var > 0.f || var != var ? var : 0.f) + p.eps);
    if (there && pos == 0 && col % q.gv == 0) {
      p.mean_out[sample * p.groups + (v0 + col) / q.gv] = mean;
      p.rstd_out[sample * p.groups + (v0 + col) / q.gv] = rstd;
    }
    with_act(p.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (have(j)) {
          float y[W], slope;
#pragma unroll
          for (int e = 0; e < W; ++e) act_one<decltype(act)::value>(__builtin_fmaf((x[j].get(e) - mean) * rstd, ga[e], be[e]), y[e], slope);
          store8(out + j * (lanes * p.ldo), W, y);
        }
    });
  } else {
    float da[W] = {}, db[W] = {}, dv[K][W];                       // dv stays, in the place of dy; xhat is computed anew from x
    with_act(p.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < K; ++j) {
        float hat[W];
        slope8<decltype(act)::value, T>(ga, be, mean, rstd, x[j], dy[j], hat, dv[j]);
        if (have(j))
#pragma unroll
          for (int e = 0; e < W; ++e) {
            db[e] += dv[j][e];
            da[e] = __builtin_fmaf(dv[j][e], hat[e], da[e]);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
    });
#pragma unroll
    for (int e = 0; e < W; ++e) {
      a = __builtin_fmaf(ga[e], db[e], a);
      b = __builtin_fmaf(ga[e], da[e], b);
      s_chan[0][e][tid] = db[e];
      s_chan[BWD ? 1 : 0][e][tid] = da[e];
    }
    join(a, b);
    if (p.part)                                                   // 2 W mine sums over the positions' lanes
      for (int i = tid; i < 2 * W * mine; i += NT) {
        const int which = i / (W * mine), rest = i - which * W * mine, v = rest / W, e = rest - v * W;
        float t = 0.f;
        for (int k = 0; k < lanes; ++k) t += s_chan[BWD ? which : 0][e][k * q.block + v];
        p.part[(sample * 2 + which) * p.c + (v0 + v) * W + e] = t;
      }
    if (!p.out) return;
    anew(x);
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (have(j)) {
        float d[W];
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float hat = (x[j].get(e) - mean) * rstd;
          d[e] = rstd * (__builtin_fmaf(ga[e], dv[j][e], -a * inv) - hat * (b * inv));
        }
        store8(out + j * (lanes * p.ldo), W, d);
        __builtin_amdgcn_sched_barrier(0);                        // one vector after the other: registers
      }
  }
}

// dbeta and dgamma from the sums of all samples' chunks, in order, 32 runs of rows at a time (with 8, and a row of sums for each of a wave's rows, 32768 x 256 in one group took 39 us backward, now 19).
constexpr int WAYS = 32;
__global__ __launch_bounds__(32 * WAYS) void norm_weights_kernel(const float* part, long long rows, int c, float* dgamma, float* dbeta) {
  __shared__ float sums[WAYS][32];
  const int lane = threadIdx.x & 31, way = threadIdx.x >> 5;
  const long long n = (long long)blockIdx.x * 32 + lane;          // column of 2 c
  float t = 0.f;
  if (n < 2LL * c) {
    long long i = way;
    for (; i + 7 * WAYS < rows; i += 8 * WAYS) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = part[(i + u * WAYS) * 2 * c + n];
      t += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
    for (; i < rows; i += WAYS) t += part[i * 2 * c + n];
  }
  sums[way][lane] = t;
  __syncthreads();
  if (way != 0 || n >= 2LL * c) return;
#pragma unroll
  for (int w = 1; w < WAYS; ++w) t += sums[w][lane];
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
  const long long jobs = d->n * t.cblocks, want = jobs >= 1024 ? 1 : (1024 + jobs - 1) / (jobs ? jobs : 1);     // four work-groups on each compute unit
  const long long chunks = want < most ? want : most;
  t.chunk_rows = ((d->s + chunks - 1) / chunks + step - 1) / step * step;
  t.chunks = (int)((d->s + t.chunk_rows - 1) / t.chunk_rows);
  return t;
}
// Samples of one launch: 2^22 work-groups of 512 threads are a grid.
long long part_samples(const lms_group_norm_desc* d, const Split& t) {
  const long long jobs = (long long)t.chunks * t.cblocks, each = jobs > 2 * d->groups ? jobs : 2 * d->groups, most = (1LL << 22) / each > 0 ? (1LL << 22) / each : 1;
  return most < d->n ? most : d->n;
}

// How a work-group holds samples, if it does: from the sizes and the type alone.
enum { NOT_HELD, TOKENS, TOKENS_ANY, IMAGES };
struct Held {
  int kind, nt, k, lanes, span, parts, block, blocks;
  long long grid, grid_fwd, rows;      // rows of sums for gamma and beta
  unsigned lds;
};
// Work-groups that go through the tokens.  Forward more of them, with at least four rounds of rows each (32768 x 1024 in 8 groups 50 -> 34 us, 2048 x 4096 with one round each 15 against 12 us);
// backward each leaves its sums for gamma and beta.
constexpr int TOKEN_GROUPS = 512, TOKEN_GROUPS_FWD = 2048;
Held held_of(const lms_group_norm_desc* d) {
  Held h{};
  const int cg = d->c / d->groups, nv = (d->c + W - 1) / W, gv = cg / W;
  if (d->s == 1) {
    int lanes = 1;
    while (lanes < nv) lanes *= 2;
    if (lanes <= 256) { h.nt = 256; h.k = 1; h.lanes = lanes; }
    else if (nv <= 512) { h.nt = 512; h.k = 1; h.lanes = 512; }
    else if (nv <= 1024) { h.nt = 512; h.k = 2; h.lanes = 512; }
    else if (nv <= 2048 && cg % W == 0) { h.nt = 1024; h.k = 2; h.lanes = 1024; }
    else return h;
    const long long rows = h.nt / h.lanes, need = (d->n + rows - 1) / rows;
    h.kind = cg % W ? TOKENS_ANY : TOKENS;
    for (h.span = 1; h.kind == TOKENS && h.span < 64 && gv % (2 * h.span) == 0;) h.span *= 2;
    h.parts = h.kind == TOKENS ? gv / h.span : 0;
    if (h.kind == TOKENS && d->groups == 1 && h.lanes <= 64) {     // the lanes behind the last vector have zeros
      h.span = h.lanes;
      h.parts = 1;
    }
    h.lds = h.kind == TOKENS_ANY ? (unsigned)(h.nt * h.k * W * 8 + rows * d->groups * 8) : 0;
    h.grid = need < TOKEN_GROUPS ? need : TOKEN_GROUPS;
    h.grid_fwd = need / 4 < TOKEN_GROUPS ? h.grid : need / 4 < TOKEN_GROUPS_FWD ? need / 4 : TOKEN_GROUPS_FWD;
    h.rows = h.grid * (h.lanes < 64 ? h.nt / 64 : rows);
    return h;
  }
  if (cg % W) return h;
  // at least 64 channels of whole groups, whose rows are a cache line, and of few positions as many as give all threads one
  const long long fill = 256 / (d->s * gv), line = gv >= 8 ? 1 : (8 + gv - 1) / gv, each = fill > line ? fill : line;
  const int groups = (int)(each < d->groups ? each : d->groups);
  h.block = groups * gv;
  h.blocks = (nv + h.block - 1) / h.block;
  if (h.block > 512) return Held{};
  // the fewest threads whose four positions each hold the sample, else those whose eight do (which leaves half the waves: 64 x 196 x 1024 in bf16 backward 26.4 us with eight of 256 threads)
  for (const int i : {0, 1, 2, 3}) {
    const int nt = i % 2 ? 512 : 256;
    if (h.block > nt) continue;
    const long long k = (d->s + nt / h.block - 1) / (nt / h.block);
    if (k > (i < 2 ? 4 : 8)) continue;
    if (d->n * h.blocks > (1LL << 31) / nt) return Held{};
    h.kind = IMAGES;
    h.nt = nt;
    h.k = k <= 2 ? 2 : k <= 4 ? 4 : 8;
    h.grid = h.grid_fwd = d->n * h.blocks;
    h.rows = d->n;
    return h;
  }
  return Held{};
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

template <typename T, bool BWD>
hipError_t resident(const lms_group_norm_desc* d, const Held& h, const NormP& p, hipStream_t s) {
  ResidentP q{p, d->n, h.lanes, h.span, h.parts, h.block, h.blocks, p.cg / W};
  const dim3 grid((unsigned)(BWD ? h.grid : h.grid_fwd));
#define TOKEN(NT, K) if (h.kind == TOKENS && h.nt == NT && h.k == K) hipLaunchKernelGGL((norm_tokens_kernel<T, NT, K, BWD>), grid, dim3(NT), 0, s, q)
#define IMAGE(NT, K) if (h.kind == IMAGES && h.nt == NT && h.k == K) hipLaunchKernelGGL((norm_image_kernel<T, NT, K, BWD>), grid, dim3(NT), 0, s, q)
#define ANY(NT, K)                                                                                                                                                 \
  if (h.kind == TOKENS_ANY && h.nt == NT && h.k == K) {                                                                                                            \
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(norm_tokens_any_kernel<T, NT, K, BWD>), hipFuncAttributeMaxDynamicSharedMemorySize, \
                                                       NT * K * W * 16);                                                                                          \
    if (attr != hipSuccess) return attr;                                                                                                                           \
    hipLaunchKernelGGL((norm_tokens_any_kernel<T, NT, K, BWD>), grid, dim3(NT), h.lds, s, q);                                                                      \
  }
  ANY(256, 1)
  ANY(512, 1)
  ANY(512, 2)
#undef ANY
  TOKEN(256, 1);
  TOKEN(512, 1);
  TOKEN(512, 2);
  TOKEN(1024, 2);
  IMAGE(256, 2);
  IMAGE(256, 4);
  IMAGE(256, 8);
  IMAGE(512, 2);
  IMAGE(512, 4);
  IMAGE(512, 8);
#undef TOKEN
#undef IMAGE
  return hipGetLastError();
}

template <typename T, bool WHOLE>
hipError_t forward(const lms_group_norm_desc* d, const Split& t, NormP& p, hipStream_t s) {
  const long long part = part_samples(d, t);
  for (p.sample0 = 0; p.sample0 < d->n; p.sample0 += part) {
    const long long take = d->n - p.sample0 < part ? d->n - p.sample0 : part;
    const dim3 jobs((unsigned)(take * t.chunks * t.cblocks));
    hipLaunchKernelGGL((norm_stats_kernel<T, WHOLE>), jobs, dim3(NT), 0, s, p);
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(take * d->groups)), dim3(JT), 0, s, p);
    hipLaunchKernelGGL((norm_apply_kernel<T, WHOLE>), jobs, dim3(NT), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t sum_weights(const float* part, long long rows, int c, float* dgamma, float* dbeta, hipStream_t s) {
  hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((2LL * c + 31) / 32)), dim3(32 * WAYS), 0, s, part, rows, c, dgamma, dbeta);
  return hipGetLastError();
}

template <typename T, bool WHOLE>
hipError_t backward(const lms_group_norm_desc* d, const Split& t, NormP& p, float* dgamma, float* dbeta, hipStream_t s) {
  const long long part = part_samples(d, t);
  for (p.sample0 = 0; p.sample0 < d->n; p.sample0 += part) {
    const long long take = d->n - p.sample0 < part ? d->n - p.sample0 : part;
    const dim3 jobs((unsigned)(take * t.chunks * t.cblocks));
    hipLaunchKernelGGL((norm_sums_kernel<T, WHOLE>), jobs, dim3(NT), 0, s, p);
    if (p.out) {
      hipLaunchKernelGGL(norm_join_bwd_kernel, dim3((unsigned)(take * d->groups)), dim3(JT), 0, s, p);
      hipLaunchKernelGGL((norm_dx_kernel<T, WHOLE>), jobs, dim3(NT), 0, s, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return !dgamma && !dbeta ? hipSuccess : sum_weights(p.part, d->n * t.chunks, d->c, dgamma, dbeta, s);
}

uint64_t stat_bytes(const lms_group_norm_desc* d) { return up256((uint64_t)d->n * d->groups * 4); }
uint64_t part_bytes(const lms_group_norm_desc* d, const Split& t, long long samples) { return up256((uint64_t)samples * t.chunks * 2 * d->c * 4); }

}  // namespace

lms_status group_norm_workspace(const lms_group_norm_desc* d, int which, uint64_t* bytes) {
  if (const lms_status st = check("lms_group_norm_workspace_bytes", d)) return st;
  NEED(which == LMS_GROUP_NORM_FWD || which == LMS_GROUP_NORM_BWD, "lms_group_norm_workspace_bytes: unknown call %d", which);
  const Split t = split_of(d);
  const Held h = held_of(d);
  if (d->n == 0) *bytes = 0;
  else if (h.kind != NOT_HELD) *bytes = 2 * stat_bytes(d) + (which == LMS_GROUP_NORM_BWD ? up256((uint64_t)h.rows * 2 * d->c * 4) : 0);
  else if (which == LMS_GROUP_NORM_FWD) *bytes = part_bytes(d, t, part_samples(d, t)) + 2 * stat_bytes(d);
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
  const Held h = held_of(d);
  if (h.kind != NOT_HELD) return done(what, d->dtype == LMS_F32 ? resident<float, false>(d, h, p, s) : resident<uint16_t, false>(d, h, p, s));
  const bool f32 = d->dtype == LMS_F32;
  if (d->c >= V) return done(what, f32 ? forward<float, true>(d, t, p, s) : forward<uint16_t, true>(d, t, p, s));
  return done(what, f32 ? forward<float, false>(d, t, p, s) : forward<uint16_t, false>(d, t, p, s));
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
  const Held h = held_of(d);
  if (h.kind != NOT_HELD && d->n > 0) {
    if (!dgamma && !dbeta) p.part = nullptr;
    const hipError_t e = d->dtype == LMS_F32 ? resident<float, true>(d, h, p, s) : resident<uint16_t, true>(d, h, p, s);
    return done(what, e != hipSuccess || !p.part ? e : sum_weights(p.part, h.rows, d->c, dgamma, dbeta, s));
  }
  const bool f32 = d->dtype == LMS_F32;
  if (d->c >= V) return done(what, f32 ? backward<float, true>(d, t, p, dgamma, dbeta, s) : backward<uint16_t, true>(d, t, p, dgamma, dbeta, s));
  return done(what, f32 ? backward<float, false>(d, t, p, dgamma, dbeta, s) : backward<uint16_t, false>(d, t, p, dgamma, dbeta, s));
}

}  // namespace lms
