// Verification of drafted tokens (include/lms.h has the rule).
//
// Two launches.  The first sums, for each request, the chunks of the one distribution that its next token comes from, a wave a chunk; every wave finds that distribution by itself, from a few reads of the drafts.
// The second picks the chunk in which the running sum passes the drawn share of the whole, and the class in it.  Differences and sums are fp64: the token is that of exact sums but
// where the drawn number lies within some 2^-50 of a border, and whole numbers have no tolerance.
// Bound by latency, then by memory: us in a graph, 1 x 32003 8.0, 8 x 128000 8.3, 128 x 50304 16.5 (51 MB; launches 10 and 5.4), 512 x 50304 42.9.  Both steps in one launch, a work-group a request, read
// at what one compute unit gets (10.7, 30.7, 18.6, 45.8), so only few classes go that way.
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "kernels.hpp"
#include "rows4.hpp"

namespace lms {

namespace {

constexpr int NT = 256, STEP = NT * 4;  // classes of a work-group at a time, and of a chunk at least
constexpr int MAX_CHUNKS = 256;        // of a request: four a lane
// Few chunks of few requests: both steps by a work-group of FEW threads a request (us in a graph, two launches / one: 1 x 1000 7.1 / 5.8, 1 x 8000 7.8 / 6.4, 1 x 16000 8.0 / 8.2, 64 x 8000 8.6 / 7.1,
// 256 x 16000 13.5 / 12.0; 1 x 32003 8.0 / 11.6, 4000 x 1000 23 / 71 with 1024 threads; call by call from Python 1 x 8000 10.1 / 7.5, 1 x 16000 9.5 / 7.3).
constexpr int FEW = 512, ALONE_REQUESTS = 256, ALONE_CHUNKS = 16;

struct VerifyP {
  const float *p, *q;
  const int32_t *drafted, *counts;
  const float *u, *v;
  int32_t *accepted, *tokens;
  double* sums;                // [request][chunk][2]: of max(p - q, 0) and of p
  long long ldp, ldq;
  int requests, drafts, classes, chunks, chunk;      // chunk: classes of one, a multiple of STEP
};

// Drafts of a request that are accepted: those before the first that is not.  The whole wave takes part.
__device__ __forceinline__ int accepted_drafts(const VerifyP& p, int b, int& count) {
  const int lane = threadIdx.x & 63;
  count = p.counts ? p.counts[b] : p.drafts;
  count = count < 0 ? 0 : count > p.drafts ? p.drafts : count;
  for (int i0 = 0; i0 < count; i0 += 64) {
    const int i = i0 + lane;
    bool good = false;
    if (i < count) {
      const int t = p.drafted[(long long)b * p.drafts + i];
      if (t >= 0 && t < p.classes)
        good = (double)p.u[(long long)b * p.drafts + i] * (double)p.q[((long long)b * p.drafts + i) * p.ldq + t] < (double)p.p[((long long)b * (p.drafts + 1) + i) * p.ldp + t];
    }
    const unsigned long long bad = __ballot(i < count && !good);
    if (bad) return i0 + __builtin_ctzll(bad);
  }
  return count;
}

// Of four classes: max(p - q, 0), and p where it is above 0; nothing for NaN.
__device__ __forceinline__ void masses(const float (&a)[4], const float (&b)[4], double (&r)[4], double (&w)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double d = (double)a[e] - (double)b[e];
    r[e] = d > 0.0 ? d : 0.0;
    w[e] = a[e] > 0.f ? (double)a[e] : 0.0;
  }
}

// The wave's sums over a chunk of the distribution pr, qr: in all lanes.
__device__ __forceinline__ void chunk_sums(const VerifyP& p, const float* pr, const float* qr, int chunk, double& sr, double& sp) {
  const int lane = threadIdx.x & 63, begin = chunk * p.chunk, end = begin + p.chunk < p.classes ? begin + p.chunk : p.classes;
  sr = sp = 0.0;
  for (int c0 = begin; c0 < end; c0 += STEP) {
    float a[4][4], q[4][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int c = c0 + u * 256 + lane * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) a[u][e] = q[u][e] = 0.f;
      if (c < end) load4(pr + c, p.classes - c, a[u]);
      if (c < end && qr) load4(qr + c, p.classes - c, q[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      double r[4], w[4];
      masses(a[u], q[u], r, w);
      sr += (r[0] + r[1]) + (r[2] + r[3]);
      sp += (w[0] + w[1]) + (w[2] + w[3]);
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    sr += __shfl_xor(sr, d);
    sp += __shfl_xor(sp, d);
  }
}

__global__ __launch_bounds__(NT) void verify_sums_kernel(VerifyP p) {
  const long long job = (long long)blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (job >= (long long)p.requests * p.chunks) return;
  const int b = (int)(job / p.chunks), chunk = (int)(job - (long long)b * p.chunks);
  int count;
  const int at = accepted_drafts(p, b, count);
  double sr, sp;
  chunk_sums(p, p.p + ((long long)b * (p.drafts + 1) + at) * p.ldp, at < count ? p.q + ((long long)b * p.drafts + at) * p.ldq : nullptr, chunk, sr, sp);
  if ((threadIdx.x & 63) == 0) {
    p.sums[job * 2] = sr;
    p.sums[job * 2 + 1] = sp;
  }
}

// Sum of the lanes up to this one.
__device__ __forceinline__ double running(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// ALONE: the sums as well, a chunk a wave, in LDS.
template <int NT, bool ALONE>
__global__ __launch_bounds__(NT) void verify_pick_kernel(VerifyP p) {
  constexpr int STEP = NT * 4;
  __shared__ double lds[NT / 64], s_sums[ALONE ? ALONE_CHUNKS : 1][2];
  __shared__ int s_first[NT / 64], s_last[NT / 64];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int count;
  const int at = accepted_drafts(p, b, count);
  const float* pr = p.p + ((long long)b * (p.drafts + 1) + at) * p.ldp;
  const float* qr = at < count ? p.q + ((long long)b * p.drafts + at) * p.ldq : nullptr;
  if constexpr (ALONE) {
    for (int chunk = wave; chunk < p.chunks; chunk += NT / 64) {
      double sr, sp;
      chunk_sums(p, pr, qr, chunk, sr, sp);
      if (lane == 0) { s_sums[chunk][0] = sr; s_sums[chunk][1] = sp; }
    }
    __syncthreads();
  }
  // the chunk: lane l has four, from 4 l on
  constexpr int NONE = 0x7fffffff;
  double er[4], ep[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool there = lane * 4 + e < p.chunks;
    const double* from = ALONE ? nullptr : p.sums + ((long long)b * p.chunks + lane * 4 + e) * 2;
    if constexpr (ALONE) from = s_sums[there ? lane * 4 + e : 0];
    er[e] = there ? from[0] : 0.0;
    ep[e] = there ? from[1] : 0.0;
  }
  const bool rest = __ballot(er[0] > 0.0 || er[1] > 0.0 || er[2] > 0.0 || er[3] > 0.0) != 0;      // else p, which has no more than q anywhere, itself
#pragma unroll
  for (int e = 0; e < 4; ++e) er[e] = rest ? er[e] : ep[e];
  const double four = (er[0] + er[1]) + (er[2] + er[3]), upto = running(four), whole = __shfl(upto, 63), target = (double)p.v[b] * whole;
  double before[4], sofar = upto - four;
  int chunk = NONE, high = -1;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    before[e] = sofar;
    sofar += er[e];
    if (er[e] > 0.0) {
      high = lane * 4 + e;
      if (sofar > target && chunk == NONE) chunk = lane * 4 + e;
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const int f = __shfl_xor(chunk, d), h = __shfl_xor(high, d);
    chunk = chunk < f ? chunk : f;
    high = high > h ? high : h;
  }
  int token = -1;
  if (high >= 0) {                                                // else there is no class to take
    chunk = __builtin_amdgcn_readfirstlane(chunk != NONE ? chunk : high);
    const double pick = chunk % 4 == 0 ? before[0] : chunk % 4 == 1 ? before[1] : chunk % 4 == 2 ? before[2] : before[3];
    double base = __shfl(pick, chunk / 4);
    const int begin = chunk * p.chunk, end = begin + p.chunk < p.classes ? begin + p.chunk : p.classes;
    int last = -1;                                                // the last class with a share so far
    for (int c0 = begin; c0 < end && token < 0; c0 += STEP) {
      const int c = c0 + (int)threadIdx.x * 4;
      float a[4] = {0.f, 0.f, 0.f, 0.f}, q[4] = {0.f, 0.f, 0.f, 0.f};
      if (c < end) load4(pr + c, p.classes - c, a);
      if (c < end && qr) load4(qr + c, p.classes - c, q);
      double r[4], w[4];
      masses(a, q, r, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = rest ? r[e] : w[e];
      const double own = (r[0] + r[1]) + (r[2] + r[3]), wave_upto = running(own);
      __syncthreads();
      if (lane == 63) lds[wave] = wave_upto;
      __syncthreads();
      double sum = base + (wave_upto - own);
      for (int i = 0; i < wave; ++i) sum += lds[i];
      int first = NONE, top = -1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum += r[e];
        if (r[e] > 0.0) {
          top = c + e;
          if (sum > target && first == NONE) first = c + e;
        }
      }
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        const int f = __shfl_xor(first, d), h = __shfl_xor(top, d);
        first = first < f ? first : f;
        top = top > h ? top : h;
      }
      if (lane == 0) { s_first[wave] = first; s_last[wave] = top; }
      __syncthreads();
      for (int i = 0; i < NT / 64; ++i) {
        first = first < s_first[i] ? first : s_first[i];
        last = last > s_last[i] ? last : s_last[i];
        base += lds[i];
      }
      if (first != NONE) token = first;
    }
    if (token < 0) token = last;
  }
  int32_t* out = p.tokens + (long long)b * (p.drafts + 1);
  for (int i = threadIdx.x; i <= p.drafts; i += NT) out[i] = i < at ? p.drafted[(long long)b * p.drafts + i] : i == at ? token : -1;
  if (threadIdx.x == 0) p.accepted[b] = at;
}

void chunks_of(const lms_verify_desc* d, int& chunks, int& chunk) {
  const int steps = (d->classes + STEP - 1) / STEP, per = (steps + MAX_CHUNKS - 1) / MAX_CHUNKS;
  chunk = per * STEP;
  chunks = (steps + per - 1) / per;
}

lms_status check(const char* what, const lms_verify_desc* d) {
  NEED(d->requests >= 0 && d->drafts >= 0 && d->classes >= 1, "%s: requests and drafts must be >= 0, classes >= 1", what);
  NEED(d->requests <= 1 << 20 && d->drafts <= 1 << 10, "%s: more than 2^20 requests, or 2^10 drafts", what);
  NEED(d->classes <= 1 << 30, "%s: more than 2^30 classes", what);
  NEED((long long)d->requests * d->classes <= 1LL << 34, "%s: requests times classes above 2^34", what);
  const long long most = 1LL << 40;
  NEED((d->ldp == 0 || (d->ldp >= d->classes && d->ldp <= most)) && (d->ldq == 0 || (d->ldq >= d->classes && d->ldq <= most)),
       "%s: a row pitch is shorter than the row, or above 2^40", what);
  return LMS_OK;
}

}  // namespace

lms_status verify_workspace(const lms_verify_desc* d, uint64_t* bytes) {
  if (const lms_status st = check("lms_verify_workspace_bytes", d)) return st;
  int chunks, chunk;
  chunks_of(d, chunks, chunk);
  *bytes = up256((uint64_t)d->requests * chunks * 16);
  return LMS_OK;
}

lms_status verify(const lms_verify_desc* d, const float* pr, const float* q, const int32_t* drafted, const int32_t* counts, const float* u, const float* v, int32_t* accepted, int32_t* tokens,
                  void* ws, void* stream) {
  const char* what = "lms_verify";
  if (const lms_status st = check(what, d)) return st;
  if (d->requests == 0) return LMS_OK;
  NEED(d->drafts == 0 || (q && drafted && u), "%s: drafts need q, their tokens and u", what);
  uintptr_t low = 0;
  for (const void* a : {(const void*)pr, (const void*)q, (const void*)drafted, (const void*)counts, (const void*)u, (const void*)v, (const void*)accepted, (const void*)tokens}) low |= (uintptr_t)a;
  NEED((low & 3) == 0, "%s: a pointer is not aligned to its elements", what);
  NEED(ws && ((uintptr_t)ws & 15) == 0, "%s: the workspace is missing or not aligned", what);
  VerifyP p{};
  p.p = pr; p.q = q; p.drafted = drafted; p.counts = counts; p.u = u; p.v = v;
  p.accepted = accepted; p.tokens = tokens; p.sums = (double*)ws;
  p.ldp = d->ldp ? d->ldp : d->classes; p.ldq = d->ldq ? d->ldq : d->classes;
  p.requests = d->requests; p.drafts = d->drafts; p.classes = d->classes;
  chunks_of(d, p.chunks, p.chunk);
  hipStream_t s = (hipStream_t)stream;
  if (p.chunks <= ALONE_CHUNKS && d->requests <= ALONE_REQUESTS) {
    hipLaunchKernelGGL((verify_pick_kernel<FEW, true>), dim3((unsigned)d->requests), dim3(FEW), 0, s, p);
    return done(what, hipGetLastError());
  }
  hipLaunchKernelGGL(verify_sums_kernel, dim3((unsigned)(((long long)d->requests * p.chunks + NT / 64 - 1) / (NT / 64))), dim3(NT), 0, s, p);
  hipLaunchKernelGGL((verify_pick_kernel<NT, false>), dim3((unsigned)d->requests), dim3(NT), 0, s, p);
  return done(what, hipGetLastError());
}

}  // namespace lms
