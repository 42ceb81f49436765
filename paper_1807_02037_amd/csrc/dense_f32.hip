// Matrix products of language-model layers on fp32 tensors (see DenseP for what a launch computes): exact fp32 products on the matrix cores.
//
// v_mfma_f32_32x32x2_f32 needs 64 cycles for 32 x 32 x 2 products, a sixteenth of the bf16 rate, so feeding it is easy: 128 x 128 outputs a work-group, 32
// of the reduction a stage, through registers one element at a time, at any address, pitch and length.  Each operand lies in LDS as in memory: rows of
// 32 of the reduction where that is contiguous, else rows of 128 columns.  A lane takes elements 8 s + 4 h + t (h: its half of the wave) for product t of step s,
// the same for both operands, so that a row's four come with one 16-byte read.
//
// The matrix cores bound it; see dense_f32.
#include <hip/hip_runtime.h>

#include "dense.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

constexpr int FM = 128, FN = 128, FK = 32;
constexpr int F_ROW = FK + 4, F_COL = FM + 8;                     // row pitches in LDS (floats): reads fall into different banks
constexpr int F_TILE = FM * F_ROW > FK * F_COL ? FM * F_ROW : FK * F_COL;
constexpr int F_LDS = 4 * F_TILE * 4;                             // two stages of two operands
static_assert(F_LDS >= 4 * epi_wave_bytes(64) && 2 * F_LDS <= 163840, "epilogue, two work-groups a compute unit");

template <int MODE>
__global__ __launch_bounds__(256, 2) void dense_f32_kernel(DenseP p) {
  constexpr bool A_FAST = MODE != DENSE_DW, B_FAST = MODE == DENSE_DX;
  constexpr int OUT_N = MODE == DENSE_GATED ? FN / 2 : FN;
  __shared__ __attribute__((aligned(16))) float lds[4 * F_TILE];

  const int job = xcd_order(p.ntiles * p.splits);
  if (job < 0) return;
  const int split = job / p.ntiles, tile = job - split * p.ntiles;
  int tm = tile % p.ntm, tn = tile / p.ntm, src = 0;
  if (MODE == DENSE_DW && p.srcs == 2) {
    const int each = p.ntn / 2;
    src = tn >= each;
    tn -= src * each;
  }
  const long long m0 = (long long)tm * FM;
  const int n0 = tn * OUT_N;
  const int first = split * p.stages_per_split, count = p.stages - first < p.stages_per_split ? p.stages - first : p.stages_per_split;
  const int seg_stages = p.stages / p.segs;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  const int half = lane >> 5, li = lane & 31;

  // Element j of this thread: along the extent, along the reduction.
  auto e_of = [&](bool fast, int j) { return fast ? (tid >> 5) + 8 * j : tid & 127; };
  auto r_of = [&](bool fast, int j) { return fast ? tid & 31 : (tid >> 7) + 2 * j; };
  auto at = [](bool fast, int e, int r) { return fast ? e * F_ROW + r : r * F_COL + e; };
  float ra[16], rb[16];
  auto pull = [&](int it) {
    int s = first + it;
    const bool second = MODE == DENSE_DX && p.segs == 2 && s >= seg_stages;
    if (second) s -= seg_stages;
    const long long r0 = (long long)s * FK;
    const float* a = (const float*)(second ? p.a[1] : p.a[0]);
    const float* b = (const float*)(second || (MODE == DENSE_DW && src) ? p.b[1] : p.b[0]);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const long long e = m0 + e_of(A_FAST, j), r = r0 + r_of(A_FAST, j);
      const bool ok = e < p.M && r < p.red;
      const float v = a[ok ? (A_FAST ? e * p.lda + r : r * p.lda + e) : 0];
      ra[j] = ok ? v : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      int c = e_of(B_FAST, j);
      const float* q = b;
      if (MODE == DENSE_GATED) {                                  // half of the tile's columns from each source
        if (c >= FN / 2) q = (const float*)p.b[1];
        c &= FN / 2 - 1;
      }
      const long long e = n0 + c, r = r0 + r_of(B_FAST, j);
      const bool ok = e < p.N && r < p.red;
      const float v = q[ok ? (B_FAST ? e * p.ldb + r : r * p.ldb + e) : 0];
      rb[j] = ok ? v : 0.f;
    }
  };
  auto push = [&](int buf) {
    float* d = lds + buf * 2 * F_TILE;
#pragma unroll
    for (int j = 0; j < 16; ++j) d[at(A_FAST, e_of(A_FAST, j), r_of(A_FAST, j))] = ra[j];
#pragma unroll
    for (int j = 0; j < 16; ++j) d[F_TILE + at(B_FAST, e_of(B_FAST, j), r_of(B_FAST, j))] = rb[j];
  };
  // first column of the wave's block j within the tile
  auto col = [&](int j) { return MODE == DENSE_GATED ? j * (FN / 2) + wn * 32 : wn * 64 + j * 32; };
  auto four = [&](bool fast, const float* t, int e, int s, float (&v)[4]) {
    if (fast) {
      const float4 q = *reinterpret_cast<const float4*>(t + e * F_ROW + 8 * s + 4 * half);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = t[(8 * s + 4 * half + u) * F_COL + e];
  };

  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  pull(0);
  push(0);
  for (int it = 0; it < count; ++it) {
    __syncthreads();                                              // this stage is in LDS, and every wave is done with the other buffer
    if (it + 1 < count) pull(it + 1);
    const float* t = lds + (it & 1) * 2 * F_TILE;
#pragma unroll
    for (int s = 0; s < FK / 8; ++s) {
      float a[2][4], b[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        four(A_FAST, t, wm * 64 + i * 32 + li, s, a[i]);
        four(B_FAST, t + F_TILE, col(i) + li, s, b[i]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j][u], a[i][u], acc[i][j], 0, 0, 0);
    }
    if (it + 1 < count) push((it + 1) & 1);
  }
  __syncthreads();
  dense_epilogue<float, MODE, 64>(p, acc, reinterpret_cast<unsigned char*>(lds) + wave * epi_wave_bytes(64), m0 + wm * 64, n0 + wn * (MODE == DENSE_GATED ? 32 : 64), src, split);
}

template <int MODE>
hipError_t launch_f32(DenseP& p, hipStream_t s) {
  const int out_n = MODE == DENSE_GATED ? FN / 2 : FN;
  const long long tm = (p.M + FM - 1) / FM, tn = (long long)((p.N + out_n - 1) / out_n) * (MODE == DENSE_DW ? p.srcs : 1);
  if (tm * tn * p.splits > 0x7fffff00LL) return hipErrorInvalidValue;
  p.ntm = (int)tm;
  p.ntn = (int)tn;
  p.ntiles = (int)(tm * tn);
  hipLaunchKernelGGL((dense_f32_kernel<MODE>), dim3((unsigned)xcd_grid((long long)p.ntiles * p.splits)), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t dense_f32(int mode, DenseP& p, hipStream_t s) {
  p.stages = (int)((p.red + FK - 1) / FK) * p.segs;
  p.splits = 1;
  p.stages_per_split = p.stages;
  switch (mode) {
    case DENSE_FWD: return launch_f32<DENSE_FWD>(p, s);
    case DENSE_GATED: return launch_f32<DENSE_GATED>(p, s);
    case DENSE_DX: return launch_f32<DENSE_DX>(p, s);
    default: return launch_f32<DENSE_DW>(p, s);
  }
}

}  // namespace lms
