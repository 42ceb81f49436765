// Linear layers and gated projections of few rows (tokens answered one by one): bound by reading the weights once.
//
// A work-group takes CB columns, CB / 8 lanes for eight columns each of one reduction index; the other lanes and waves take others, KU consecutive ones at a
// time: that many 16-byte loads of weights in flight a lane, and one load of each row of x.  Products are ordinary fp32 instructions, which for
// so few rows stay behind the loads.  The partial sums meet by shuffles and in LDS, in a fixed order.
//
// Memory gives its rate only to whole 128-byte lines of a row of weights, and only if all 256 compute units ask.  So layers of at least 16384 columns take CB = 64
// and the whole reduction; narrower ones take 128 columns and split the reduction until there are 256 work-groups, and a second launch joins the
// sums.  Small weights are read in less time than that launch takes: then each work-group keeps the whole reduction, of 16 or 32 columns.
// us (one row, several sets of weights in turn; GB/s of weights):
//                            16 columns   32     64     128 columns, splits 4     8        64, splits 4
//   4096 -> 4096 (34 MB)       18.5                    15.0                   13.5      13.4
//   16384 -> 4096 (134 MB)     57.3                    35.4                   30.6 (4390)
//   2048 -> 2048 (8 MB)         8.9                    11.8                   11.6      10.1
//   gated 4096 -> 8192         61.0      39.0   38.8   32.7 (4105)            36.7      38.4
//   gated 4096 -> 16384        89.6                    55.2 (4863)            57.3      61.6
//   8192 -> 16384 (268 MB)                      52.3 (5134)
#include <hip/hip_runtime.h>

#include "dense.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

constexpr int FT = 512;              // threads

template <typename T, int MODE, int R, int CB>
__global__ __launch_bounds__(FT) void dense_few_kernel(DenseP p) {
  constexpr int S = MODE == DENSE_GATED ? 2 : 1, LC = CB / 8, KG = FT / LC;
  constexpr int KU = S * R * sizeof(T) >= 32 ? 4 : 8;             // registers
  __shared__ float sums[FT / 64][S][R][CB];
  const int job = dense_job(p);
  if (job < 0) return;
  const int split = job / p.ntiles;
  const int tid = threadIdx.x, c = (tid % LC) * 8, n = (job - split * p.ntiles) * CB + c, cnt = p.N - n < 8 ? p.N - n : 8;
  const int rows = (int)p.M;
  const T* x = (const T*)p.a[0];
  float fb[8], fr[8];                                             // of the thread that finishes a row's eight columns
  const bool finisher = tid < R * LC && tid / LC < rows && cnt > 0;
  if (finisher && p.splits == 1) {
    dense_bias8<MODE>(p, n, cnt, fb);
    dense_beside8<T, MODE>(p, tid / LC, n, cnt, fr);
  }
  const T* w[2] = {(const T*)p.b[0] + n, (const T*)p.b[1] + n};

  const long long per = (p.red / p.splits + 7) / 8 * 8, k_begin = split * per, k_end = split + 1 < p.splits && k_begin + per < p.red ? k_begin + per : p.red;

  float acc[S][R][8];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[s][r][e] = 0.f;

  if (cnt > 0)
    for (long long k = k_begin + (long long)(tid / LC) * KU; k < k_end; k += KG * KU) {
      const int have = k_end - k < KU ? (int)(k_end - k) : KU;
      Raw<T, KU> xv[R];
      Raw<T, 8> wv[S][KU];
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int u = 0; u < KU; ++u) wv[s][u] = raw<8>(w[s] + (k + (u < have ? u : 0)) * p.ldb, cnt);   // beyond the end: any row that is there
#pragma unroll
      for (int r = 0; r < R; ++r) xv[r] = raw<KU>(x + (r < rows ? r : 0) * p.lda + k, have);
#pragma unroll
      for (int u = 0; u < KU; ++u) {
        if (u >= have) break;                                     // no product of nothing with what may be infinite
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float b = wv[s][u].get(e);
#pragma unroll
            for (int r = 0; r < R; ++r) acc[s][r][e] = __builtin_fmaf(xv[r].get(u), b, acc[s][r][e]);
          }
      }
    }

  // lanes of a wave with the same columns, then the waves
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = acc[s][r][e];
#pragma unroll
        for (int d = 32; d >= LC; d >>= 1) v += __shfl_xor(v, d);
        acc[s][r][e] = v;
      }
  if ((tid & 63) < LC)
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[tid >> 6][s][r][c + e] = acc[s][r][e];
  __syncthreads();
  if (tid < R * LC) {
    const int r = tid / LC;
    float v[8], u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = u[e] = 0.f;
#pragma unroll
      for (int i = 0; i < FT / 64; ++i) {
        v[e] += sums[i][0][r][c + e];
        if constexpr (S == 2) u[e] += sums[i][1][r][c + e];
      }
    }
    if (!finisher) return;
    if (p.splits > 1) {
      dense_part8(p, split, 0, r, n, cnt, v);
      if constexpr (S == 2) dense_part8(p, split, 1, r, n, cnt, u);
    } else dense_finish8<T, MODE>(p, 0, r, n, cnt, v, u, fb, fr);
  }
}

// Splits of the reduction: see above.  Each keeps at least 256 indices.
int few_splits(int mode, bool f32, int N, long long red) {
  const long long bytes = (long long)N * red * (f32 ? 4 : 2) * (mode == DENSE_GATED ? 2 : 1);
  if (N >= 64 * 256 || bytes < 16000000) return 1;
  const int blocks = (N + 127) / 128, want = (256 + blocks - 1) / blocks;
  const long long most = red / 256;
  return (int)(want < most ? want : most < 1 ? 1 : most);
}

template <typename T, int MODE, int R>
hipError_t few_rows(DenseP& p, hipStream_t s) {
  auto launch = [&](auto cb) {
    constexpr int CB = decltype(cb)::value;
    p.ntiles = (p.N + CB - 1) / CB;
    return launch_jobs<FT>(p, [&](dim3 grid) { hipLaunchKernelGGL((dense_few_kernel<T, MODE, R, CB>), grid, dim3(FT), 0, s, p); });
  };
  if (p.splits > 1) {
    const hipError_t e = launch(std::integral_constant<int, 128>{});
    return e == hipSuccess ? dense_join(MODE, sizeof(T) == 4, p, s) : e;
  }
  if (p.N >= 64 * 256) return launch(std::integral_constant<int, 64>{});
  return p.N >= 32 * 256 ? launch(std::integral_constant<int, 32>{}) : launch(std::integral_constant<int, 16>{});
}

template <typename T, int MODE>
hipError_t few_mode(DenseP& p, hipStream_t s) {
  if (p.M == 1) return few_rows<T, MODE, 1>(p, s);
  if constexpr (sizeof(T) == 4) {
    if constexpr (MODE == DENSE_FWD)
      if (p.M > 4) return few_rows<T, MODE, 8>(p, s);
    if (p.M > 2) return few_rows<T, MODE, 4>(p, s);
  }
  return few_rows<T, MODE, 2>(p, s);
}

}  // namespace

// In bf16 from three rows on the matrix cores' tiles are as fast or faster (us, rows here / there: 4096 -> 4096 4 rows 15.3, 8 rows 17.8 / 13.4; 4096 -> 16384 8 rows 37.6 / 30.7; gated
// 4096 -> 8192 4 rows 35.7 / 34.9); in fp32 they are slower up to eight (24.0 / 29.6), of which a gated projection's do not fit the registers.
bool dense_few_ok(int mode, bool f32, long long M) { return (mode == DENSE_FWD || mode == DENSE_GATED) && M <= (!f32 ? 2 : mode == DENSE_FWD ? 8 : 4); }

uint64_t dense_few_ws(int mode, bool f32, long long M, int N, long long red) {
  const int splits = few_splits(mode, f32, N, red);
  return splits > 1 ? (uint64_t)splits * (mode == DENSE_GATED ? 2 : 1) * M * N * 4 : 0;
}

hipError_t dense_few(int mode, bool f32, DenseP& p, hipStream_t s) {
  p.splits = few_splits(mode, f32, p.N, p.red);
  if (f32) return mode == DENSE_FWD ? few_mode<float, DENSE_FWD>(p, s) : few_mode<float, DENSE_GATED>(p, s);
  return mode == DENSE_FWD ? few_mode<uint16_t, DENSE_FWD>(p, s) : few_mode<uint16_t, DENSE_GATED>(p, s);
}

}  // namespace lms
