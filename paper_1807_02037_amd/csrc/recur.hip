// Gated recurrence over packed sequences, its backward pass and its single-token form (include/lms.h has the formulas).
//
// A span of rows maps the state h that enters it to A h + H, A the product of its a, or 0 where a sequence begins in it.  Backwards, with r = a dh, what a row passes to the one before it
// (dh = e + r of the row behind), it maps r to A r + R, A = 0 where a sequence ends in it.  Those zeros are negative, which no product is: behind them what enters does not count, were it NaN.
// Spans compose, so rows need not wait for one another:
// a wave takes a few rows of 256 channels and holds what it has read of them in registers; the waves of a work-group, one after the other in time, exchange their spans in LDS: a chunk.
// Where chunks depend on each other, a first launch leaves each chunk's (A, H), a second composes them into the state that enters each chunk, and the third computes the
// results.  (Taking a part of the line at a time through all three, so that the third reads from the last-level cache, loses more to partly filled launches than it gains: 32768 x 4096 bf16 in
// parts of 96 / 192 MB / one: forward 427 / 362 / 325 us, backward 624 / 580 / 528.)
#include <hip/hip_runtime.h>

#include <cstdlib>
#include <initializer_list>

#include "dense.hpp"
#include "graph.hpp"
#include "kernels.hpp"
#include "rows4.hpp"

namespace lms {

namespace {

constexpr int BLOCK = 64 * V;          // of a wave and of a work-group
constexpr int KEEP = 32;               // rows between the states that the forward pass keeps

struct RecurP {
  const void *x, *g, *o, *dy;
  const int32_t* offsets;
  const float *h0, *dlast;
  void *y, *dx, *dg, *dout;
  float *last, *dh0;
  float* sums;                 // [chunk of the part][2][channels]: A and H, or null
  float* in;                   // [chunk][channels]: state that enters a chunk (backward: r from the chunk behind), or null: none does
  float* kept;                 // [KEEP rows][channels]: state that enters them, or null
  long long rows, ldx, ldy, each;      // each: rows of a sequence where there are no offsets
  int seqs, channels, act;
  int chunk0, chunks, all_chunks;      // chunks of this launch
  int direct;                  // few chunks: each composes those that come before it out of sums itself, and there is no `in`
  int empties;                 // work-groups of a block of channels behind the chunks' that look for sequences without rows
  int lpr, subs;               // lanes of a row, a power of two; runs of rows of a wave, 64 / lpr
};

// Rows of a run, of a whole wave the same for all lanes: which begin a sequence, which end one, which belong to one, and which one.
template <int ROWS>
struct Marks {
  unsigned first, last, live;
  int seq[ROWS];
};
// The borders are read as constants: for a whole wave by scalar loads, which do not wait for the rows that are on their way.
typedef const __attribute__((address_space(4))) int32_t* Borders;
// The last sequence that begins at or before the row; of several at the same place all but the last are empty.  -1: none.
__device__ __forceinline__ int sequence_of(const RecurP& p, long long row, int lo, int hi) {  // offsets[lo] <= row < offsets[hi]; -1 and seqs + 1: any row
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (((Borders)(uintptr_t)p.offsets)[mid] <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}
// w0, wn: first row and number of rows of the wave.  Where it has several runs, they are looked for between the sequences of its first and its last row, which most often are one.
template <int ROWS, bool NARROW>
__device__ __forceinline__ Marks<ROWS> marks(const RecurP& p, long long r0, long long w0, int wn) {
  Marks<ROWS> m = {0u, 0u, 0u, {}};
  const Borders off = (Borders)(uintptr_t)p.offsets;
  int s = 0;
  long long begin = 0, next = 0;
  if (p.offsets) {
    if (w0 >= p.rows) return m;
    s = sequence_of(p, w0, -1, p.seqs + 1);
    begin = s >= 0 ? off[s] : 0;
    next = s < p.seqs ? off[s + 1] : 0;
    if (NARROW && s < p.seqs && next < w0 + wn) {
      const int end = sequence_of(p, w0 + wn - 1, s, p.seqs + 1) + 1;
      s = sequence_of(p, r0, s, end);
      begin = s >= 0 ? off[s] : 0;
      next = s < p.seqs ? off[s + 1] : 0;
    }
  } else {
    s = (int)(r0 / p.each);
    begin = s * p.each;
    next = begin + p.each;
  }
  if (r0 >= p.rows) return m;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const long long row = r0 + r;
    if (s < p.seqs && next <= row) {                              // on to the sequence of this row: most often the next one
      ++s;
      begin = next;
      next = p.offsets ? (s < p.seqs ? off[s + 1] : 0) : begin + p.each;
      if (s < p.seqs && next <= row) {                            // behind any number of empty ones
        s = sequence_of(p, row, s, p.seqs + 1);
        begin = off[s];
        next = s < p.seqs ? off[s + 1] : 0;
      }
    }
    const bool live = row < p.rows && s >= 0 && s < p.seqs;
    m.live |= (unsigned)live << r;
    m.first |= (unsigned)(live && begin == row) << r;
    m.last |= (unsigned)(live && next == row + 1) << r;
    m.seq[r] = live ? s : 0;
  }
  return m;
}

// Of a = sigmoid(g) and 1 - a the smaller one, e / (1 + e) with e = exp(-|g|), and the sign of g: where that is negative it is a, else 1 - a.  The other is one minus it, so both are there to their own
// precision (a difference from an a that is rounded already is off by 1 % at g = 12 and by all at 18), and a gate at its end keeps or replaces all, bit for bit.
__device__ __forceinline__ float share(float g) {
  const float e = __builtin_amdgcn_exp2f(__builtin_fabsf(g) * -1.44269504f);
  return __builtin_copysignf(e * __builtin_amdgcn_rcpf(1.f + e), g);
}
__device__ __forceinline__ float kept_of(float share) { return __builtin_signbitf(share) ? -share : 1.f - share; }     // a
__device__ __forceinline__ float rest_of(float share) { return __builtin_signbitf(share) ? 1.f + share : share; }      // 1 - a

// a h + (1 - a) x
__device__ __forceinline__ float mix(float share, float h, float x) { return __builtin_fmaf(kept_of(share), h, rest_of(share) * x); }

// What leaves a span (a, h) that v enters, and the a of two spans, the one of `second` behind.
__device__ __forceinline__ float through(float a, float v, float h) { return __builtin_signbitf(a) ? h : __builtin_fmaf(a, v, h); }
__device__ __forceinline__ float product(float a, float second) { return __builtin_signbitf(second) ? -0.f : a * second; }

enum { SUM_FWD, APPLY_FWD, SUM_BWD, APPLY_BWD };

constexpr int CHUNK_FWD = 64, CHUNK_BWD = 32;                      // rows of a work-group, times the runs of a wave
static_assert(CHUNK_BWD == KEEP, "a chunk of the backward pass begins where a state is kept");

// Rows of a wave: forward eight, whose raw inputs and gates leave registers for sixteen waves on a compute unit; backward, with twice the tensors, four; in fp32 half of that.
template <typename T, int WAY>
struct Shape {
  static constexpr bool BWD = WAY == SUM_BWD || WAY == APPLY_BWD;
  static constexpr int CHUNK = BWD ? CHUNK_BWD : CHUNK_FWD, WAVES = sizeof(T) == 2 ? 8 : 16, ROWS = CHUNK / WAVES, NT = WAVES * 64;
  static_assert(KEEP % ROWS == 0 && ROWS < 32, "");
};

// WHOLE: at least four channels.  The last vector of a row that would end beyond it begins earlier instead, and its first channels are computed twice, alike.
// NARROW: up to 128 channels.  They leave lanes free, and a wave takes several runs of rows one after the other, which meet by shuffles before the waves do.
template <typename T, int WAY, bool WHOLE, bool NARROW>
__global__ __launch_bounds__((Shape<T, WAY>::NT), 4) void recur_kernel(RecurP p) {
  constexpr int ROWS = Shape<T, WAY>::ROWS, WAVES = Shape<T, WAY>::WAVES, CHUNK = Shape<T, WAY>::CHUNK;
  constexpr bool BWD = Shape<T, WAY>::BWD, STATE = WAY != SUM_BWD;   // STATE: h is computed
  __shared__ float s_a[STATE ? WAVES : 1][BLOCK], s_h[STATE ? WAVES : 1][BLOCK], s_b[BWD ? WAVES : 1][BLOCK], s_r[BWD ? WAVES : 1][BLOCK];
  const int blocks = NARROW ? 1 : (p.channels + BLOCK - 1) / BLOCK, job = blockIdx.x, lane = threadIdx.x & 63;
  const int run = NARROW ? lane / p.lpr : 0, runs = NARROW ? p.subs : 1, col = NARROW ? lane & (p.lpr - 1) : lane;
  const int chunk = job / blocks, at = col * V, c0 = (job - chunk * blocks) * BLOCK + at;
  const unsigned c = WHOLE && c0 > p.channels - V ? p.channels - V : c0;       // an offset of 32 bits from what is the same for the wave
  const bool column = c0 < p.channels;
  const int cnt = WHOLE ? V : p.channels - c0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // sequences without a row keep their states: eight at a time to a wave, by work-groups behind those of the chunks
  if constexpr (WAY == APPLY_FWD || WAY == APPLY_BWD)
    if (chunk >= p.chunks) {
      constexpr int EACH = 8;
      float* to = BWD ? p.dh0 : p.last;
      const float* from = BWD ? p.dlast : p.h0;
      for (long long s0 = ((long long)(chunk - p.chunks) * WAVES + wave) * EACH; s0 < p.seqs; s0 += (long long)p.empties * WAVES * EACH) {
        const int s = (int)s0 + lane;
        const bool empty = lane < EACH && s < p.seqs && (!p.offsets || p.offsets[s] == p.offsets[s + 1]);
        const unsigned long long found = __ballot(empty);
        if (!column) continue;
        float v[EACH][V] = {};
#pragma unroll
        for (int i = 0; i < EACH; ++i)
          if (from && (found >> i & 1)) load4(from + (s0 + i) * p.channels + c, cnt, v[i]);
#pragma unroll
        for (int i = 0; i < EACH; ++i)
          if (found >> i & 1) store4(to + (s0 + i) * p.channels + c, cnt, v[i]);
      }
      return;
    }
  const long long row0 = (long long)(p.chunk0 + chunk) * (CHUNK * runs), r0 = row0 + (wave * runs + run) * ROWS;
  const long long x0 = r0 * p.ldx, y0 = r0 * p.ldy;               // of the first row
  const bool there = column && r0 < p.rows, gated = p.o != nullptr;

  // all that is read of the rows, in flight at once; rows beyond the last: the first, for nothing
  Raw<T, V> x[STATE ? ROWS : 1], g[ROWS], o[WAY == SUM_FWD ? 1 : ROWS], dy[BWD ? ROWS : 1];
  if (there) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const bool have = r0 + r < p.rows;
      const long long xr = x0 + (have ? r * p.ldx : 0), yr = y0 + (have ? r * p.ldy : 0);
      g[r] = raw<V>((const T*)p.g + xr + c, cnt);
      if constexpr (STATE) x[r] = raw<V>((const T*)p.x + xr + c, cnt);
      if constexpr (BWD) dy[r] = raw<V>((const T*)p.dy + yr + c, cnt);
    }
    if constexpr (WAY != SUM_FWD)
      if (gated)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) o[r] = raw<V>((const T*)p.o + x0 + (r0 + r < p.rows ? r * p.ldx : 0) + c, cnt);
  }
  float state[V] = {}, behind[V] = {};                            // h that enters the chunk; r that enters it from behind
  if (column) {
    const long long entry = (long long)(p.chunk0 + chunk) * p.channels;
    if (WAY == APPLY_FWD && p.in) load4(p.in + entry + c, cnt, state);
    if (WAY == APPLY_BWD && p.kept) load4(p.kept + row0 / KEEP * p.channels + c, cnt, state);
    if (WAY == APPLY_BWD && p.in) load4(p.in + entry + p.channels + c, cnt, behind);
  }
  if constexpr (WAY == APPLY_FWD || WAY == APPLY_BWD)
    if (p.direct && column) {
      constexpr int IN_FLIGHT = 4;
      float (&v)[V] = BWD ? behind : state;
      const int before = BWD ? p.chunks - 1 - chunk : chunk;
      for (int i0 = 0; i0 < before; i0 += IN_FLIGHT) {
        float ka[IN_FLIGHT][V], kh[IN_FLIGHT][V];
#pragma unroll
        for (int u = 0; u < IN_FLIGHT; ++u) {
          const int i = i0 + u < before ? i0 + u : i0;
          const float* from = p.sums + (long long)(BWD ? p.chunks - 1 - i : i) * 2 * p.channels + c;
          load4(from, cnt, ka[u]);
          load4(from + p.channels, cnt, kh[u]);
        }
#pragma unroll
        for (int u = 0; u < IN_FLIGHT; ++u)
          if (i0 + u < before)
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = through(ka[u][e], v[e], kh[u][e]);
      }
    }
  const Marks<ROWS> m = marks<ROWS, NARROW>(p, r0, row0 + wave * runs * ROWS, runs * ROWS);
  auto of_sequence = [&](const float* t, int r, float (&v)[V]) __attribute__((always_inline)) {  // the values of row r's sequence, zeros where there are none
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    if (t && column) load4(t + (long long)m.seq[r] * p.channels + c, cnt, v);
  };

  // ---- the wave's spans ----
  float a[ROWS][V], err[BWD ? ROWS : 1][V];                       // a: the gates' shares; err: e = dy act(o)
  if constexpr (BWD) {
    if (gated && there) with_act(p.act, [&](auto act) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float value, slope;
          act_one<decltype(act)::value>(o[r].get(e), value, slope);
          err[r][e] = value * dy[r].get(e);
        }
    });
    else
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) err[r][e] = there ? dy[r].get(e) : 0.f;
  }
  float A[V], H[V], B[V], R[V];                                   // B: A of the way backwards.  R = sum over rows of e times the product of a up to the row, which needs no order from behind
#pragma unroll
  for (int e = 0; e < V; ++e) { A[e] = B[e] = 1.f; H[e] = R[e] = 0.f; }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (STATE && (m.first >> r & 1)) {
      of_sequence(p.h0, r, H);
#pragma unroll
      for (int e = 0; e < V; ++e) A[e] = -0.f;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      a[r][e] = share(there ? g[r].get(e) : 0.f);
      if constexpr (STATE) {
        A[e] *= kept_of(a[r][e]);
        H[e] = mix(a[r][e], H[e], there ? x[r].get(e) : 0.f);
      }
    }
    if constexpr (BWD)
      if (!(m.last & ((1u << r) - 1))) {                          // rows behind a sequence's end pass nothing on
        float d[V] = {};
        const bool end = m.last >> r & 1;
        if (end) of_sequence(p.dlast, r, d);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          B[e] *= kept_of(a[r][e]);
          R[e] = __builtin_fmaf(B[e], err[r][e] + d[e], R[e]);
          if (end) B[e] = -0.f;
        }
      }
  }
  // runs of a wave: A, H become those of the runs up to this one, eA, eH of those before it; B, R of the runs from this one on, eB, eR of those behind it
  float eA[V], eH[V], eB[V], eR[V];
  if constexpr (NARROW) {
    auto meet = [&](float (&a)[V], float (&h)[V], float (&ea)[V], float (&eh)[V], bool back) __attribute__((always_inline)) {
      for (int d = 1; d < runs; d *= 2) {
        const int from = back ? lane + d * p.lpr : lane - d * p.lpr;
        const bool take = back ? run + d < runs : run >= d;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float oa = __shfl(a[e], from), oh = __shfl(h[e], from);
          if (take) {
            h[e] = through(a[e], oh, h[e]);
            a[e] = product(oa, a[e]);
          }
        }
      }
      const int from = back ? lane + p.lpr : lane - p.lpr;
      const bool edge = back ? run == runs - 1 : run == 0;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float oa = __shfl(a[e], from), oh = __shfl(h[e], from);
        ea[e] = edge ? 1.f : oa;
        eh[e] = edge ? 0.f : oh;
      }
    };
    if constexpr (STATE) meet(A, H, eA, eH, false);
    if constexpr (BWD) meet(B, R, eB, eR, true);
  }
  auto put = [&](float (&t)[BLOCK], const float (&v)[V]) { *reinterpret_cast<float4*>(&t[at]) = make_float4(v[0], v[1], v[2], v[3]); };
  if constexpr (STATE)
    if (!NARROW || run == runs - 1) { put(s_a[wave], A); put(s_h[wave], H); }
  if constexpr (BWD)
    if (!NARROW || run == 0) { put(s_b[wave], B); put(s_r[wave], R); }
  __syncthreads();
  auto compose = [&](const float (&sa)[BLOCK], const float (&sh)[BLOCK], float (&v)[V]) __attribute__((always_inline)) {
    const float4 k = *reinterpret_cast<const float4*>(&sa[at]), d = *reinterpret_cast<const float4*>(&sh[at]);
    v[0] = through(k.x, v[0], d.x); v[1] = through(k.y, v[1], d.y); v[2] = through(k.z, v[2], d.z); v[3] = through(k.w, v[3], d.w);
  };
  if constexpr (WAY == SUM_FWD || WAY == SUM_BWD) {
    if (wave != 0 || run != 0 || !column) return;
    float k[V] = {1.f, 1.f, 1.f, 1.f}, d[V] = {};
    for (int i = 0; i < WAVES; ++i) {
      const int w = WAY == SUM_FWD ? i : WAVES - 1 - i;
      const float (&sa)[BLOCK] = WAY == SUM_FWD ? s_a[STATE ? w : 0] : s_b[BWD ? w : 0];
      compose(sa, WAY == SUM_FWD ? s_h[STATE ? w : 0] : s_r[BWD ? w : 0], d);
#pragma unroll
      for (int e = 0; e < V; ++e) k[e] = product(k[e], sa[at + e]);
    }
    float* to = p.sums + (long long)chunk * 2 * p.channels + c;
    store4(to, cnt, k);
    store4(to + p.channels, cnt, d);
    return;
  }
  if constexpr (WAY == APPLY_FWD || WAY == APPLY_BWD) {
    if (!there) return;
    // what was computed of the inputs is computed again from here on: kept, it takes twice the registers of the inputs, and with them the second work-group of a compute unit
    auto anew = [](auto& t) __attribute__((always_inline)) {
#pragma unroll
      for (auto& v : t)
#pragma unroll
        for (unsigned& w : v.q) asm volatile("" : "+v"(w));
    };
    anew(x);
    if constexpr (BWD) { anew(g); anew(o); }
    if constexpr (NARROW)                                         // there a and 1 - a as well (146338 x 64 forward 78 -> 63 us, backward 107 -> 100; 64571 x 640 124 and 126)
#pragma unroll
      for (auto& row : a)
#pragma unroll
        for (float& v : row) asm volatile("" : "+v"(v));
    for (int w = 0; w < wave; ++w) compose(s_a[w], s_h[w], state);
    if constexpr (NARROW)
#pragma unroll
      for (int e = 0; e < V; ++e) state[e] = through(eA[e], state[e], eH[e]);
    auto entry_of = [&](int r) { return (long long)m.seq[r] * p.channels + c; };
    if constexpr (WAY == APPLY_FWD) {
      if (p.kept && r0 % KEEP == 0) store4(p.kept + r0 / KEEP * p.channels + c, cnt, state);
      auto finish = [&](auto act, auto with_gate) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
          if (m.first >> r & 1) of_sequence(p.h0, r, state);
          float y[V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            y[e] = state[e] = mix(a[r][e], state[e], x[r].get(e));
            if constexpr (decltype(with_gate)::value) {
              float value, slope;
              act_one<decltype(act)::value>(o[r].get(e), value, slope);
              y[e] *= value;
            }
          }
          if (!(m.live >> r & 1)) continue;
          store4((T*)p.y + y0 + r * p.ldy + c, cnt, y);
          if ((m.last >> r & 1) && p.last) store4(p.last + entry_of(r), cnt, state);
        }
      };
      if (gated) with_act(p.act, [&](auto act) __attribute__((always_inline)) { finish(act, std::true_type{}); });
      else finish(std::integral_constant<int, LMS_ACT_NONE>{}, std::false_type{});
    } else {
      float h[ROWS][V], now[V];
#pragma unroll
      for (int e = 0; e < V; ++e) now[e] = state[e];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        if (m.first >> r & 1) of_sequence(p.h0, r, now);
#pragma unroll
        for (int e = 0; e < V; ++e) h[r][e] = now[e] = mix(a[r][e], now[e], x[r].get(e));
      }
      for (int w = WAVES - 1; w > wave; --w) compose(s_b[w], s_r[w], behind);
      if constexpr (NARROW)
#pragma unroll
        for (int e = 0; e < V; ++e) behind[e] = through(eB[e], behind[e], eR[e]);
      auto finish = [&](auto act, auto with_gate) __attribute__((always_inline)) {
#pragma unroll
        for (int r = ROWS - 1; r >= 0; --r) {
          if (!(m.live >> r & 1)) continue;
          const bool first = m.first >> r & 1;
          if (m.last >> r & 1) of_sequence(p.dlast, r, behind);
          float before[V], dx[V], dg[V], dout[V];
#pragma unroll
          for (int e = 0; e < V; ++e) before[e] = r > 0 ? h[r > 0 ? r - 1 : 0][e] : state[e];
          if (first) of_sequence(p.h0, r, before);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float dh = err[r][e] + behind[e], rest = rest_of(a[r][e]);
            dx[e] = rest * dh;
            behind[e] = kept_of(a[r][e]) * dh;
            dg[e] = behind[e] * rest * (before[e] - x[r].get(e));
            if constexpr (decltype(with_gate)::value) {
              float value, slope;
              act_one<decltype(act)::value>(o[r].get(e), value, slope);
              dout[e] = dy[r].get(e) * slope * h[r][e];
            }
          }
          const long long to = x0 + r * p.ldx;
          if (p.dx) store4((T*)p.dx + to + c, cnt, dx);
          if (p.dg) store4((T*)p.dg + to + c, cnt, dg);
          if constexpr (decltype(with_gate)::value)
            if (p.dout) store4((T*)p.dout + to + c, cnt, dout);
          if (first && p.dh0) store4(p.dh0 + entry_of(r), cnt, behind);
        }
      };
      if (gated) with_act(p.act, [&](auto act) __attribute__((always_inline)) { finish(act, std::true_type{}); });
      else finish(std::integral_constant<int, LMS_ACT_NONE>{}, std::false_type{});
    }
  }
}

// The states that enter the chunks chunk0 .. chunk0 + chunks of the line from that which enters the first (backwards: r from behind, from that which enters the last): 16 channels, 64 spans of
// chunks, which stay in registers between the two ways through them where they are eight or fewer.  Bound by the reads that follow one another, so many short spans of few channels (us, the
// three launches backward of bf16 with a gate, for 64 channels x 16 spans / 32 x 32 / 16 x 64 / 8 x 128: 200000 x 256 339 / 276 / 269 / 278, 64571 x 640 225 / 207 / 203 / 212, 4096 x 512
// 21.5 / 20.6 / 21.3 / 22.9).
constexpr int JOIN_WIDTH = 16, JOIN_SPANS = 64;
constexpr int JOIN_BLOCKS = 1 << 21;   // blocks of channels of a launch: a grid holds less than 2^32 threads
template <bool BWD>
__global__ __launch_bounds__(JOIN_WIDTH * JOIN_SPANS) void recur_join_kernel(RecurP p, int block0) {
  __shared__ float s_a[JOIN_SPANS][JOIN_WIDTH], s_h[JOIN_SPANS][JOIN_WIDTH];
  const int lane = threadIdx.x & (JOIN_WIDTH - 1), span = threadIdx.x / JOIN_WIDTH, c = (block0 + (int)blockIdx.x) * JOIN_WIDTH + lane;
  const int per = (p.chunks + JOIN_SPANS - 1) / JOIN_SPANS, first = span * per, end = first + per < p.chunks ? first + per : p.chunks;
  const bool there = c < p.channels;
  auto index = [&](int i) { return BWD ? p.chunks - 1 - i : i; };   // i: in the order of composition
  constexpr int U = 8;
  float ka[U], kh[U];
  auto ask = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* from = p.sums + (long long)index(i0 + u < end ? i0 + u : i0) * 2 * p.channels + c;
      ka[u] = from[0];
      kh[u] = from[p.channels];
    }
  };
  float a = 1.f, h = 0.f;
  if (there)
    for (int i0 = first; i0 < end; i0 += U) {
      ask(i0);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u < end) {
          a = product(a, ka[u]);
          h = through(ka[u], h, kh[u]);
        }
    }
  s_a[span][lane] = a;
  s_h[span][lane] = h;
  __syncthreads();
  if (!there) return;
  const bool outer = BWD ? p.chunk0 + p.chunks == p.all_chunks : p.chunk0 == 0;     // nothing enters the line
  float* const edge = p.in + (long long)(BWD ? p.chunk0 + p.chunks : p.chunk0) * p.channels + c;
  float in = outer ? 0.f : *edge;
  if (outer && span == 0) *edge = 0.f;
  for (int s = 0; s < span; ++s) in = through(s_a[s][lane], in, s_h[s][lane]);
  for (int i0 = first; i0 < end; i0 += U) {
    if (per > U) ask(i0);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u < end) {
        in = through(ka[u], in, kh[u]);
        p.in[(long long)(p.chunk0 + (BWD ? index(i0 + u) : i0 + u + 1)) * p.channels + c] = in;
      }
  }
}

// ---- sequences of one length, each by work-groups that walk along it ----
//
// Where there are enough of them for the chip, every tensor is read once: a work-group takes two channels a lane of one sequence and goes through it 64 rows at a time, eight waves of eight rows, the next rows' loads out
// before these are worked on.  The waves' spans meet in LDS, every wave composes all of them, and so each knows the state that the next 64 rows begin with: one barrier a step.  Rows
// beyond a sequence's end pass r on as it is (a = 1, e = 0), so that the gradient of the last state enters there.  32768 x 4096 in bf16 of 8 sequences, with a gate: forward 199 us (5.4 TB/s), backward
// 386 us (4.9 TB/s); a copy of 1 GiB reaches 5.05 TB/s.
constexpr int WV = 2, WBLOCK = 64 * WV, WROWS = 8, WSTEP = 8 * WROWS;

template <typename T, bool BWD>
__global__ __launch_bounds__(512, 2) void recur_walk_kernel(RecurP p) {
  __shared__ float2 s_a[2][8][64], s_h[2][8][64], s_r[2][BWD ? 8 : 1][BWD ? 64 : 1];
  const int blocks = (p.channels + WBLOCK - 1) / WBLOCK, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seq = blockIdx.x / blocks, c0 = (int)(blockIdx.x - seq * blocks) * WBLOCK + lane * WV;
  const unsigned c = c0 > p.channels - WV ? p.channels - WV : c0;  // the last pair of an odd row begins earlier, and its first channel is computed twice, alike
  const bool column = c0 < p.channels, gated = p.o != nullptr;
  const long long row0 = seq * p.each;
  const int each = (int)p.each, steps = (each + WSTEP - 1) / WSTEP, keeps = (each + KEEP - 1) / KEEP;
  typedef Raw<T, WV> Pair;
  Pair x[WROWS], g[WROWS], o[WROWS], dy[BWD ? WROWS : 1], nx[WROWS], ng[WROWS], no[WROWS], ndy[BWD ? WROWS : 1];
  float2 entry = {}, next_entry = {};                             // backward: the state that these rows begin with
  auto pair = [](const T* q) { Pair r; __builtin_memcpy(&r, q, sizeof(r)); return r; };
  auto ask = [&](int step) __attribute__((always_inline)) {
    if (!column) return;
#pragma unroll
    for (int r = 0; r < WROWS; ++r) {
      const int at = step * WSTEP + wave * WROWS + r;
      const long long row = row0 + (at < each ? at : each - 1);
      nx[r] = pair((const T*)p.x + row * p.ldx + c);
      ng[r] = pair((const T*)p.g + row * p.ldx + c);
      if constexpr (BWD) ndy[r] = pair((const T*)p.dy + row * p.ldy + c);
    }
    if (gated)
#pragma unroll
      for (int r = 0; r < WROWS; ++r) {
        const int at = step * WSTEP + wave * WROWS + r;
        no[r] = pair((const T*)p.o + (row0 + (at < each ? at : each - 1)) * p.ldx + c);
      }
    if constexpr (BWD) __builtin_memcpy(&next_entry, p.kept + ((long long)seq * keeps + step * (WSTEP / KEEP)) * p.channels + c, 8);
  };
  const float* from = BWD ? p.dlast : p.h0;
  float2 carry = {};
  if (from && column) __builtin_memcpy(&carry, from + (long long)seq * p.channels + c, 8);
  auto get = [](const float2& v, int e) { return e ? v.y : v.x; };
  auto pass = [](const float2& a, const float2& v, const float2& h) { return make_float2(__builtin_fmaf(a.x, v.x, h.x), __builtin_fmaf(a.y, v.y, h.y)); };
  auto put = [&](T* base, long long row, const float (&v)[WV]) {
    if constexpr (sizeof(T) == 2) {
      const unsigned q = pack_bf16x2(v[0], v[1]);
      __builtin_memcpy(base + row + c, &q, 4);
    } else __builtin_memcpy(base + row + c, v, 8);
  };
  ask(BWD ? steps - 1 : 0);
  for (int i = 0; i < steps; ++i) {
    const int step = BWD ? steps - 1 - i : i, half = i & 1, at0 = step * WSTEP + wave * WROWS;
#pragma unroll
    for (int r = 0; r < WROWS; ++r) {
      x[r] = nx[r]; g[r] = ng[r]; o[r] = no[r];
      if constexpr (BWD) dy[r] = ndy[r];
    }
    entry = next_entry;
    if (i + 1 < steps) ask(BWD ? step - 1 : step + 1);
    float a[WROWS][WV], err[BWD ? WROWS : 1][WV];                  // a: the gates' shares
    if constexpr (BWD) {
      if (gated) with_act(p.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < WROWS; ++r)
#pragma unroll
          for (int e = 0; e < WV; ++e) {
            float value, slope;
            act_one<decltype(act)::value>(o[r].get(e), value, slope);
            err[r][e] = value * dy[r].get(e);
          }
      });
      else
#pragma unroll
        for (int r = 0; r < WROWS; ++r)
#pragma unroll
          for (int e = 0; e < WV; ++e) err[r][e] = dy[r].get(e);
    }
    float2 A = {1.f, 1.f}, H = {0.f, 0.f}, R = {0.f, 0.f}, upto_a[BWD ? 1 : WROWS], upto_h[BWD ? 1 : WROWS];      // upto: A and H of the rows up to each
#pragma unroll
    for (int r = 0; r < WROWS; ++r) {
      const bool live = at0 + r < each;
#pragma unroll
      for (int e = 0; e < WV; ++e) {
        a[r][e] = share(g[r].get(e));
        if constexpr (BWD) {
          a[r][e] = live ? a[r][e] : 0.f;
          err[r][e] = live ? err[r][e] : 0.f;
        }
      }
      A = make_float2(A.x * kept_of(a[r][0]), A.y * kept_of(a[r][1]));
      H = make_float2(mix(a[r][0], H.x, x[r].get(0)), mix(a[r][1], H.y, x[r].get(1)));
      if constexpr (BWD) R = make_float2(__builtin_fmaf(A.x, err[r][0], R.x), __builtin_fmaf(A.y, err[r][1], R.y));
      else { upto_a[r] = A; upto_h[r] = H; }
    }
    s_a[half][wave][lane] = A;
    s_h[half][wave][lane] = H;
    if constexpr (BWD) s_r[half][wave][lane] = R;
    __syncthreads();                                              // the other half is read by none: its readers have written this one since
    float2 state = BWD ? entry : carry, behind = {};
    if constexpr (!BWD) {
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        if (w == wave) state = carry;
        carry = pass(s_a[half][w][lane], carry, s_h[half][w][lane]);
      }
    } else {
      for (int w = 0; w < wave; ++w) state = pass(s_a[half][w][lane], state, s_h[half][w][lane]);
#pragma unroll
      for (int w = 7; w >= 0; --w) {
        if (w == wave) behind = carry;
        carry = pass(s_a[half][w][lane], carry, s_r[half][w][lane]);
      }
    }
    // computed anew from here on: see recur_kernel
    auto anew = [](auto& t) __attribute__((always_inline)) {
#pragma unroll
      for (auto& v : t)
#pragma unroll
        for (unsigned& w : v.q) asm volatile("" : "+v"(w));
    };
    if constexpr (BWD) anew(x);
    if (!column) continue;
    if constexpr (!BWD) {
      if (p.kept && at0 % KEEP == 0 && at0 < each) __builtin_memcpy(p.kept + ((long long)seq * keeps + at0 / KEEP) * p.channels + c, &state, 8);
      auto finish = [&](auto act, auto with_gate) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < WROWS; ++r) {
          float y[WV];
          const float2 h = pass(upto_a[r], state, upto_h[r]);
#pragma unroll
          for (int e = 0; e < WV; ++e) {
            y[e] = get(h, e);
            if constexpr (decltype(with_gate)::value) {
              float value, slope;
              act_one<decltype(act)::value>(o[r].get(e), value, slope);
              y[e] *= value;
            }
          }
          if (at0 + r >= each) continue;
          put((T*)p.y, (row0 + at0 + r) * p.ldy, y);
          if (at0 + r == each - 1 && p.last) __builtin_memcpy(p.last + (long long)seq * p.channels + c, &h, 8);
        }
      };
      if (gated) with_act(p.act, [&](auto act) __attribute__((always_inline)) { finish(act, std::true_type{}); });
      else finish(std::integral_constant<int, LMS_ACT_NONE>{}, std::false_type{});
    } else {
      float2 h[WROWS], now = state;
#pragma unroll
      for (int r = 0; r < WROWS; ++r) h[r] = now = make_float2(mix(a[r][0], now.x, x[r].get(0)), mix(a[r][1], now.y, x[r].get(1)));
      anew(g);
      anew(o);
      auto finish = [&](auto act, auto with_gate) __attribute__((always_inline)) {
#pragma unroll
        for (int r = WROWS - 1; r >= 0; --r) {
          if (at0 + r >= each) continue;
          const float2 before = r > 0 ? h[r > 0 ? r - 1 : 0] : state;
          float dx[WV], dg[WV], dout[WV], back[WV];
#pragma unroll
          for (int e = 0; e < WV; ++e) {
            const float dh = err[r][e] + get(behind, e), rest = rest_of(a[r][e]);
            dx[e] = rest * dh;
            back[e] = kept_of(a[r][e]) * dh;
            dg[e] = back[e] * rest * (get(before, e) - x[r].get(e));
            if constexpr (decltype(with_gate)::value) {
              float value, slope;
              act_one<decltype(act)::value>(o[r].get(e), value, slope);
              dout[e] = dy[r].get(e) * slope * get(h[r], e);
            }
          }
          behind = make_float2(back[0], back[1]);
          const long long to = (row0 + at0 + r) * p.ldx;
          if (p.dx) put((T*)p.dx, to, dx);
          if (p.dg) put((T*)p.dg, to, dg);
          if constexpr (decltype(with_gate)::value)
            if (p.dout) put((T*)p.dout, to, dout);
          if (at0 + r == 0 && p.dh0) __builtin_memcpy(p.dh0 + (long long)seq * p.channels + c, &behind, 8);
        }
      };
      if (gated) with_act(p.act, [&](auto act) __attribute__((always_inline)) { finish(act, std::true_type{}); });
      else finish(std::integral_constant<int, LMS_ACT_NONE>{}, std::false_type{});
    }
  }
}

// One position of each request, its state in a slot.  Rows of the same slot are consecutive positions of one request: the first of them takes them all, in order.  MANY rows: a work-group
// looks through the slots once, not each wave (4096 rows of 2048 channels 80 -> 40 us, 65536 of 256 6.1 -> 1.8 ms).
constexpr int STEP_ROWS = 65536, STEP_FEW = 512;
template <typename T, bool MANY>
__global__ __launch_bounds__(256) void recur_step_kernel(RecurP p, const int32_t* slots, const float* from, float* to, int n) {
  const int blocks = (p.channels + 4 * BLOCK - 1) / (4 * BLOCK), lane = threadIdx.x & 63;
  const int row = blockIdx.x / blocks, c = (blockIdx.x - row * blocks) * 4 * BLOCK + threadIdx.x * V, cnt = p.channels - c;
  const int slot = slots[row];
  if (slot < 0 || slot >= p.seqs) return;
  float h[V] = {};
  if (cnt > 0) load4(from + (long long)slot * p.channels + c, cnt, h);
  auto position = [&](int at) {
    if (cnt <= 0) return;
    const long long i = at * p.ldx + c;
    const Raw<T, V> x = raw<V>((const T*)p.x + i, cnt), g = raw<V>((const T*)p.g + i, cnt);
    Raw<T, V> o;
    if (p.o) o = raw<V>((const T*)p.o + i, cnt);
    float y[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      y[e] = h[e] = mix(share(g.get(e)), h[e], x.get(e));
    }
    if (p.o) with_act(p.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float value, slope;
        act_one<decltype(act)::value>(o.get(e), value, slope);
        y[e] *= value;
      }
    });
    store4((T*)p.y + at * p.ldy + c, cnt, y);
  };
  if constexpr (MANY) {
    constexpr int SEEN = 8;                                       // words in flight
    __shared__ unsigned long long s_same[STEP_ROWS / 64];         // which rows are of this slot
    const int words = (n + 63) / 64, own = row / 64, wave = threadIdx.x >> 6;
    for (int w0 = wave * SEEN; w0 < words; w0 += 4 * SEEN) {
      int there[SEEN];
#pragma unroll
      for (int u = 0; u < SEEN; ++u) {
        const int i = (w0 + u) * 64 + lane;
        there[u] = i < n ? slots[i] : -1;
      }
#pragma unroll
      for (int u = 0; u < SEEN; ++u) {
        const unsigned long long same = __ballot(there[u] == slot);
        if (lane == 0 && w0 + u < words) s_same[w0 + u] = same;
      }
    }
    __syncthreads();
    const unsigned long long until = (2ull << (row & 63)) - 1;    // this row and those before it in its word
    bool earlier = false;
    for (int w = lane; w <= own; w += 64) earlier |= (s_same[w] & (w == own ? until >> 1 : ~0ull)) != 0;
    if (__ballot(earlier)) return;
    position(row);
    for (int w0 = own; w0 < words; w0 += 64) {
      unsigned long long mine = w0 + lane < words ? s_same[w0 + lane] : 0;
      if (w0 + lane == own) mine &= ~until;
      for (unsigned long long found = __ballot(mine != 0); found; found &= found - 1) {
        const int w = w0 + __builtin_ctzll(found);
        for (unsigned long long more = s_same[w] & (w == own ? ~until : ~0ull); more; more &= more - 1) position(w * 64 + __builtin_ctzll(more));
      }
    }
    if (cnt > 0) store4(to + (long long)slot * p.channels + c, cnt, h);
    return;
  }
  for (int i0 = 0; i0 < row; i0 += 64)                            // an earlier row of the slot takes this one
    if (__ballot(i0 + lane < row && slots[i0 + lane < row ? i0 + lane : row] == slot)) return;
  position(row);
  for (int i0 = row + 1; i0 < n; i0 += 64) {
    unsigned long long more = __ballot(i0 + lane < n && slots[i0 + lane < n ? i0 + lane : row] == slot);
    for (; more; more &= more - 1) position(i0 + __builtin_ctzll(more));
  }
  if (cnt > 0) store4(to + (long long)slot * p.channels + c, cnt, h);
}

// Lanes of a row, and rows of a chunk: narrow rows leave a wave several runs.
int lanes_of(int channels) {
  int lanes = 1;
  while (lanes < 64 && lanes * V < channels) lanes *= 2;
  return lanes;
}
int chunk_of(const lms_recur_desc* d, bool bwd) { return (bwd ? CHUNK_BWD : CHUNK_FWD) * (64 / lanes_of(d->channels)); }
long long chunks_of(long long rows, int chunk) { return rows <= chunk ? 1 : (rows + chunk - 1) / chunk; }
// Chunks of one launch: 2^21 work-groups of up to 1024 threads are a grid.
long long most_chunks(const lms_recur_desc* d) {
  const long long most = (1LL << 21) / ((d->channels + BLOCK - 1) / BLOCK);
  return most < 1 ? 1 : most;
}
// Tuning aid: LMS_RECUR_CHUNKS, fewer of them in a launch.  The workspace is that of the most.
long long part_chunks(const lms_recur_desc* d) {
  const char* fewer = getenv("LMS_RECUR_CHUNKS");
  const long long most = most_chunks(d), want = fewer ? atoll(fewer) : 0;
  return want > 0 && want < most ? want : most;
}
uint64_t sums_bytes(const lms_recur_desc* d, int chunk) {
  const long long part = most_chunks(d), all = chunks_of(d->rows, chunk);
  return up256((uint64_t)(part < all ? part : all) * 2 * d->channels * 4);
}
uint64_t in_bytes(const lms_recur_desc* d, int chunk) { return up256((uint64_t)(chunks_of(d->rows, chunk) + 1) * d->channels * 4); }

lms_status check(const char* what, const lms_recur_desc* d, bool step) {
  NEED(d->rows >= 0 && d->channels >= 1 && d->seqs >= 1, "%s: rows must be >= 0, channels and sequences >= 1", what);
  NEED(d->rows <= 0x7fffffffLL - 64, "%s: more than 2^31 - 65 rows", what);
  NEED(d->channels <= 1 << 26 && d->seqs <= 1 << 30, "%s: more than 2^26 channels, or 2^30 sequences", what);
  NEED(d->act >= LMS_ACT_NONE && d->act <= LMS_ACT_GELU_TANH, "%s: unknown activation %d", what, d->act);
  NEED(d->dtype == LMS_BF16 || d->dtype == LMS_F32, "%s: dtype must be LMS_BF16 or LMS_F32", what);
  const long long most = 1LL << 40;
  NEED((d->ldx == 0 || (d->ldx >= d->channels && d->ldx <= most)) && (d->ldy == 0 || (d->ldy >= d->channels && d->ldy <= most)),
       "%s: a row pitch is shorter than the row, or above 2^40", what);
  NEED(!step || d->rows <= STEP_ROWS, "%s: more than %d rows of a step", what, STEP_ROWS);
  return LMS_OK;
}
lms_status lined(const char* what, const lms_recur_desc* d, const int32_t* offsets) {
  NEED(offsets || d->rows % d->seqs == 0, "%s: without offsets the rows must be a multiple of the sequences", what);
  return LMS_OK;
}
// Elements of the storage type, then of 32 bits.
lms_status aligned(const char* what, const lms_recur_desc* d, std::initializer_list<const void*> rows, std::initializer_list<const void*> words) {
  uintptr_t a = 0, b = 0;
  for (const void* q : rows) a |= (uintptr_t)q;
  for (const void* q : words) b |= (uintptr_t)q;
  NEED((a & (d->dtype == LMS_F32 ? 3 : 1)) == 0 && (b & 3) == 0, "%s: a pointer is not aligned to its elements", what);
  return LMS_OK;
}
bool overlap(const lms_recur_desc* d, const float* a, const float* b) {
  const uintptr_t n = (uintptr_t)d->seqs * d->channels * 4, x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + n && y < x + n;
}
RecurP params(const lms_recur_desc* d, int chunk, const void* x, const void* g, const void* o, const int32_t* offsets, const float* h0) {
  RecurP p{};
  p.x = x; p.g = g; p.o = o; p.offsets = offsets; p.h0 = h0;
  p.rows = d->rows; p.ldx = d->ldx ? d->ldx : d->channels; p.ldy = d->ldy ? d->ldy : d->channels;
  p.each = d->rows / d->seqs > 0 ? d->rows / d->seqs : 1;
  p.seqs = d->seqs; p.channels = d->channels; p.act = d->act;
  p.all_chunks = (int)chunks_of(d->rows, chunk);
  p.lpr = lanes_of(d->channels);
  p.subs = 64 / p.lpr;
  return p;
}
// No chunk needs what another leaves: one chunk, or whole sequences in each.
bool alone(const lms_recur_desc* d, int chunk, const int32_t* offsets) { return d->rows <= chunk || (!offsets && chunk % (d->rows / d->seqs) == 0); }

// Whether work-groups walk along sequences of one length, for both directions together, since they share what is kept: by what both are estimated to take.  A step of 64 rows takes
// 8.5 us there and back, on each compute unit one at a time, or as long as the eleven tensors take; the line reads five of them twice and has two more launches each way.
// us, bf16 with a gate, forward + backward, walk / line:
//   sequences x rows x channels   8 x 4096 x 4096  209 + 385 / 336 + 529     4 x 4096 x 4096  175 + 338 / 186 + 276     8 x 2048 x 2048  92 + 177 / 95 + 150
//   32 x 512 x 512  24 + 47 / 32 + 48     16 x 128 x 1024  9 + 14 / 21 + 22     4 x 1024 x 2048  43 + 83 / 32 + 46     1 x 8192 x 4096  331 + 613 / 102 + 149
bool walks(const lms_recur_desc* d, const int32_t* offsets) {
  const long long each = d->rows / d->seqs, groups = (long long)d->seqs * ((d->channels + WBLOCK - 1) / WBLOCK);
  if (offsets || each <= CHUNK_FWD || d->channels < WV || groups >= 1 << 22) return false;
  const double bytes = (double)d->rows * d->channels * (d->dtype == LMS_F32 ? 4 : 2), rounds = (double)((groups + 255) / 256);
  const double steps = (double)((each + WSTEP - 1) / WSTEP) * rounds * 8.5, walk = steps > bytes * 11 / 4.7e6 ? steps : bytes * 11 / 4.7e6;
  return walk < 25.0 + bytes * 16 / 4.9e6;
}
template <bool BWD>
hipError_t walk(const lms_recur_desc* d, const RecurP& p, hipStream_t s) {
  const dim3 grid((unsigned)((long long)d->seqs * ((d->channels + WBLOCK - 1) / WBLOCK)));
  if (d->dtype == LMS_F32) hipLaunchKernelGGL((recur_walk_kernel<float, BWD>), grid, dim3(512), 0, s, p);
  else hipLaunchKernelGGL((recur_walk_kernel<uint16_t, BWD>), grid, dim3(512), 0, s, p);
  return hipGetLastError();
}

template <typename T, int WAY>
hipError_t launch(const RecurP& p, hipStream_t s) {
  const int blocks = (p.channels + BLOCK - 1) / BLOCK;
  const dim3 grid((unsigned)(blocks * (p.chunks + p.empties))), threads((Shape<T, WAY>::NT));
  if (p.subs == 1) hipLaunchKernelGGL((recur_kernel<T, WAY, true, false>), grid, threads, 0, s, p);
  else if (p.channels >= V) hipLaunchKernelGGL((recur_kernel<T, WAY, true, true>), grid, threads, 0, s, p);
  else hipLaunchKernelGGL((recur_kernel<T, WAY, false, true>), grid, threads, 0, s, p);
  return hipGetLastError();
}

// Chunks up to which a launch for the states between them is not worth it (us, forward + backward, with it / without: 256 x 1024 in bf16 16.4 + 17.2 / 14.6 + 15.6, 512 x 960 16.9 + 18.4 / 15.1 + 17.2;
// of 32 chunks, 1024 x 1024 backward 19.4 / 21.3).
constexpr int DIRECT = 16;

constexpr int EMPTIES = 1 << 14;       // work-groups that look for sequences without rows, at most

// in: entries of the states between chunks, sums: of a part.
template <typename T, bool BWD>
hipError_t line(RecurP& p, bool alone, long long part, hipStream_t s) {
  const int parts = (int)((p.all_chunks + part - 1) / part);
  float* const in = p.in;
  if (alone) p.in = nullptr;
  for (int i = 0; i < parts; ++i) {
    p.chunk0 = (int)((BWD ? parts - 1 - i : i) * part);
    p.chunks = (int)(p.all_chunks - p.chunk0 < part ? p.all_chunks - p.chunk0 : part);
    hipError_t e = hipSuccess;
    if (!alone) {
      e = launch<T, BWD ? SUM_BWD : SUM_FWD>(p, s);
      if (e != hipSuccess) return e;
      p.direct = parts == 1 && p.all_chunks <= DIRECT;               // of several parts, the sums are only this one's
      if (p.direct) p.in = nullptr;
      else
        for (int b = 0, all = (p.channels + JOIN_WIDTH - 1) / JOIN_WIDTH; b < all; b += JOIN_BLOCKS)
          hipLaunchKernelGGL(recur_join_kernel<BWD>, dim3((unsigned)(all - b < JOIN_BLOCKS ? all - b : JOIN_BLOCKS)), dim3(JOIN_WIDTH * JOIN_SPANS), 0, s, p, b);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    constexpr int WAY = BWD ? APPLY_BWD : APPLY_FWD, looked = Shape<T, WAY>::WAVES * 8;
    const int blocks = (p.channels + BLOCK - 1) / BLOCK, most = blocks < EMPTIES ? EMPTIES / blocks : 1, need = (p.seqs + looked - 1) / looked;
    p.empties = i > 0 || !(BWD ? p.dh0 : p.last) || !(p.offsets || p.rows == 0) ? 0 : need < most ? need : most;
    e = launch<T, WAY>(p, s);
    if (e != hipSuccess) return e;
    p.empties = 0;
  }
  p.in = in;
  return hipSuccess;
}

}  // namespace

lms_status recur_kept(const lms_recur_desc* d, uint64_t* bytes) {
  if (const lms_status st = check("lms_recur_kept_bytes", d, false)) return st;
  // one for each KEEP rows of the line, or of each sequence
  const uint64_t line = chunks_of(d->rows, KEEP), seqs = d->rows % d->seqs ? 0 : (uint64_t)d->seqs * ((d->rows / d->seqs + KEEP - 1) / KEEP);
  *bytes = d->rows <= CHUNK_BWD ? 0 : up256((line > seqs ? line : seqs) * d->channels * 4);
  return LMS_OK;
}

lms_status recur_workspace(const lms_recur_desc* d, int which, uint64_t* bytes) {
  if (const lms_status st = check("lms_recur_workspace_bytes", d, false)) return st;
  NEED(which == LMS_RECUR_FWD || which == LMS_RECUR_BWD, "lms_recur_workspace_bytes: unknown call %d", which);
  const int chunk = chunk_of(d, which == LMS_RECUR_BWD);
  *bytes = d->rows <= chunk ? 0 : sums_bytes(d, chunk) + in_bytes(d, chunk);
  return LMS_OK;
}

lms_status recur_fwd(const lms_recur_desc* d, const void* x, const void* g, const void* o, const int32_t* offsets, const float* h0, void* y, float* last, void* kept, void* ws,
                     void* stream) {
  const char* what = "lms_recur_fwd";
  if (const lms_status st = check(what, d, false)) return st;
  if (const lms_status st = lined(what, d, offsets)) return st;
  if (const lms_status st = aligned(what, d, {x, g, o, y}, {offsets, h0, last})) return st;
  NEED(!overlap(d, h0, last), "%s: the last states must not overlap the initial ones", what);
  uint64_t need = 0;
  recur_workspace(d, LMS_RECUR_FWD, &need);
  NEED(!need || ws, "%s: workspace of %llu bytes required", what, (unsigned long long)need);
  NEED((((uintptr_t)ws | (uintptr_t)kept) & 15) == 0, "%s: the workspace is not aligned", what);
  const int chunk = chunk_of(d, false);
  RecurP p = params(d, chunk, x, g, o, offsets, h0);
  p.y = y; p.last = last;
  p.kept = d->rows <= CHUNK_BWD ? nullptr : (float*)kept;
  p.sums = (float*)ws;
  p.in = (float*)((char*)ws + sums_bytes(d, chunk));
  const bool whole = alone(d, chunk, offsets);
  const long long part = part_chunks(d);
  hipStream_t s = (hipStream_t)stream;
  if (walks(d, offsets)) return done(what, walk<false>(d, p, s));
  return done(what, d->dtype == LMS_F32 ? line<float, false>(p, whole, part, s) : line<uint16_t, false>(p, whole, part, s));
}

lms_status recur_bwd(const lms_recur_desc* d, const void* dy, const void* x, const void* g, const void* o, const int32_t* offsets, const float* h0, const void* kept, const float* dlast,
                     void* dx, void* dg, void* dout, float* dh0, void* ws, void* stream) {
  const char* what = "lms_recur_bwd";
  if (const lms_status st = check(what, d, false)) return st;
  if (const lms_status st = lined(what, d, offsets)) return st;
  if (const lms_status st = aligned(what, d, {dy, x, g, o, dx, dg, dout}, {offsets, h0, dlast, dh0})) return st;
  NEED(o || !dout, "%s: the gradient of o needs o", what);
  NEED(!overlap(d, dlast, dh0) && !overlap(d, h0, dh0), "%s: the gradient of the initial states must not overlap the states or the gradient of the last ones", what);
  const int chunk = chunk_of(d, true);
  const bool walking = walks(d, offsets), whole = !walking && alone(d, chunk, offsets);
  NEED(whole || kept, "%s: what the forward pass kept is needed", what);
  uint64_t need = 0;
  recur_workspace(d, LMS_RECUR_BWD, &need);
  NEED(!need || ws, "%s: workspace of %llu bytes required", what, (unsigned long long)need);
  NEED((((uintptr_t)ws | (uintptr_t)kept) & 15) == 0, "%s: the workspace is not aligned", what);
  RecurP p = params(d, chunk, x, g, o, offsets, h0);
  p.dy = dy; p.dlast = dlast;
  p.dx = dx; p.dg = dg; p.dout = dout; p.dh0 = dh0;
  p.kept = whole ? nullptr : (float*)const_cast<void*>(kept);
  p.sums = (float*)ws;
  p.in = (float*)((char*)ws + sums_bytes(d, chunk));
  const long long part = part_chunks(d);
  hipStream_t s = (hipStream_t)stream;
  if (walking) return done(what, walk<true>(d, p, s));
  return done(what, d->dtype == LMS_F32 ? line<float, true>(p, whole, part, s) : line<uint16_t, true>(p, whole, part, s));
}

lms_status recur_step(const lms_recur_desc* d, const void* x, const void* g, const void* o, const int32_t* slots, const float* state, float* next, void* y, void* stream) {
  const char* what = "lms_recur_step";
  if (const lms_status st = check(what, d, true)) return st;
  if (const lms_status st = aligned(what, d, {x, g, o, y}, {slots, state, next})) return st;
  NEED(state == next || !overlap(d, state, next), "%s: the new states are the old ones or apart from them", what);
  if (d->rows == 0) return LMS_OK;
  RecurP p = params(d, CHUNK_FWD, x, g, o, nullptr, nullptr);
  p.y = y;
  const long long groups = d->rows * ((d->channels + 4 * BLOCK - 1) / (4 * BLOCK));
  NEED(groups < 1 << 24, "%s: rows times channels above 2^34", what);
  const dim3 grid((unsigned)groups);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, p, slots, state, next, (int)d->rows); };
  if (d->rows <= STEP_FEW) d->dtype == LMS_F32 ? go(recur_step_kernel<float, false>) : go(recur_step_kernel<uint16_t, false>);
  else d->dtype == LMS_F32 ? go(recur_step_kernel<float, true>) : go(recur_step_kernel<uint16_t, true>);
  return done(what, hipGetLastError());
}

}  // namespace lms
