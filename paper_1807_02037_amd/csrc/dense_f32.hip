// Matrix products of language-model layers on fp32 tensors (see DenseP for what a launch computes): exact fp32 products on the matrix cores.
//
// v_mfma_f32_32x32x2_f32 needs 64 cycles for 32 x 32 x 2 products, a sixteenth of the bf16 rate: 128 x 128 outputs a work-group, or 64 x 64 where there are few, 32 of the
// reduction a stage.  Each operand lies in LDS as in memory: rows of 32 of the reduction where that is contiguous, else rows of columns.  A lane takes
// elements 8 s + 4 h + t (h: its half of the wave) for product t of step s, the same for both operands, so that a row's four come with one 16-byte read.
//
// The matrix cores bound it, at the clock that the device holds under them: 139 TFLOP/s at 4096 x 4096 x 4096 (the library's product 151).
#include <hip/hip_runtime.h>

#include "conv_dma.hpp"
#include "dense.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

// ---- operands on 16-byte boundaries, lengths in multiples of four: loads that write LDS ----
//
// A ring of stages, asked for RING - 1 ahead: the 32 loads and 32 LDS stores of four bytes a thread that a stage takes through registers (below) become four or eight loads of
// sixteen.  Rows along the reduction are 128 bytes long, as in dense_gemm.hip, and permuted alike; rows of columns have their halves of 32 banks exchanged where the
// reduction index has bit 2, so that the two halves of a wave, four rows apart, read different banks.
constexpr int DFK = 32;
template <int EXT, bool FAST, int SUB>
struct F32Operand {
  static constexpr int V = EXT * DFK / (4 * 256);                 // loads per thread
  __device__ static __forceinline__ void where(int v, int& e, int& r) {
    if constexpr (FAST) {
      e = v / 8;
      r = ((v % 8) ^ ((e >> 1) & 7)) * 4;
    } else {
      constexpr int C = SUB / 4;
      const int piece = v / (DFK * C), w = v % (DFK * C);
      r = w / C;
      e = piece * SUB + ((w % C) ^ (8 * ((r >> 2) & 1))) * 4;
    }
  }
  // LDS bytes of this lane's four values of step s (FAST), or of the first of them at step 0
  __device__ static __forceinline__ int base(int e, int half, int s) {
    if constexpr (FAST) return e * 128 + (((2 * s + half) ^ ((e >> 1) & 7)) << 4);
    else return (e / SUB) * (DFK * SUB * 4) + half * (4 * SUB * 4) + ((((e % SUB) >> 2) ^ (8 * half)) << 4) + (e & 3) * 4;
  }
};

template <int MODE, int FM, int RING>
__global__ __launch_bounds__(256, 2) void dense_f32_dma_kernel(DenseP p) {
  constexpr bool A_FAST = MODE != DENSE_DW, B_FAST = MODE == DENSE_DX;
  constexpr int OUT_N = MODE == DENSE_GATED ? FM / 2 : FM, W = FM / 2, TB = W / 32, SUB = MODE == DENSE_GATED ? FM / 2 : FM;
  typedef F32Operand<FM, A_FAST, FM> OpA;
  typedef F32Operand<FM, B_FAST, SUB> OpB;
  constexpr int V = OpA::V, OPERAND = FM * DFK * 4, STAGE = 2 * OPERAND, LOADS = 2 * V;
  static_assert(RING * STAGE >= 4 * epi_wave_bytes(W) && 2 * RING * STAGE <= 163840, "epilogue; two work-groups a compute unit");
  __shared__ __attribute__((aligned(256))) unsigned char lds[RING * STAGE];

  const int job = dense_job(p);
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

  const long long m_left = p.M - m0, n_left = (long long)p.N - n0;
  int a_e[V], a_r[V], b_e[V], b_r[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    OpA::where(tid + j * 256, a_e[j], a_r[j]);
    OpB::where(tid + j * 256, b_e[j], b_r[j]);
    if (MODE == DENSE_GATED) b_e[j] %= SUB;
  }
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)lds + wave * 1024);
  unsigned a_off[V], b_off[V];
  v4u rs_a = {}, rs_b = {}, rs_u = {};
  int to_load = count;
  long long load_r = 0;
  auto enter = [&](int seg, long long r) {                        // the next stage is of segment seg, element r
    load_r = r;
    const long long ao = A_FAST ? m0 * p.lda + r : r * p.lda + m0, bo = B_FAST ? n0 * p.ldb + r : r * p.ldb + n0;
    rs_a = buffer_rsrc((const float*)p.a[MODE == DENSE_DX ? seg : 0] + ao, 0x7fffffff);
    rs_b = buffer_rsrc((const float*)p.b[MODE == DENSE_DX ? seg : MODE == DENSE_DW ? src : 0] + bo, 0x7fffffff);
    if (MODE == DENSE_GATED) rs_u = buffer_rsrc((const float*)p.b[1] + bo, 0x7fffffff);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      a_off[j] = a_e[j] < m_left && r + a_r[j] < p.red ? (unsigned)((A_FAST ? a_e[j] * p.lda + a_r[j] : a_r[j] * p.lda + a_e[j]) * 4) : DMA_OOB;
      b_off[j] = b_e[j] < n_left && r + b_r[j] < p.red ? (unsigned)((B_FAST ? b_e[j] * p.ldb + b_r[j] : b_r[j] * p.ldb + b_e[j]) * 4) : DMA_OOB;
    }
  };
  auto fetch = [&](int buf) {
    const unsigned at = lds0 + buf * STAGE;
#pragma unroll
    for (int j = 0; j < V; ++j) load_lds16(rs_a, at + j * 4096, a_off[j], 0);
#pragma unroll
    for (int j = 0; j < V; ++j) load_lds16(MODE == DENSE_GATED && j >= V / 2 ? rs_u : rs_b, at + OPERAND + j * 4096, b_off[j], 0);
    if (--to_load <= 0) {                                         // beyond the last: nothing but zeros
      rs_a[2] = rs_b[2] = rs_u[2] = 0;
      return;
    }
    load_r += DFK;
    if (MODE == DENSE_DX && load_r >= p.red) { enter(1, 0); return; }
    auto move = [](v4u& rs, long long bytes) {
      const unsigned long long to = ((unsigned long long)rs[1] << 32 | rs[0]) + bytes;
      rs[0] = (unsigned)to;
      rs[1] = (unsigned)(to >> 32);
    };
    move(rs_a, (A_FAST ? DFK : DFK * p.lda) * 4);
    move(rs_b, (B_FAST ? DFK : DFK * p.ldb) * 4);
    if (MODE == DENSE_GATED) move(rs_u, DFK * p.ldb * 4);
    if (load_r + DFK > p.red)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        a_off[j] = load_r + a_r[j] < p.red ? a_off[j] : DMA_OOB;
        b_off[j] = load_r + b_r[j] < p.red ? b_off[j] : DMA_OOB;
      }
  };
  // first column of the wave's block j within the tile
  auto col = [&](int j) { return MODE == DENSE_GATED ? j / (TB / 2 ? TB / 2 : 1) * (FM / 2) + wn * (W / 2) + j % (TB / 2 ? TB / 2 : 1) * 32 : wn * W + j * 32; };
  constexpr int STEPS = DFK / 8;
  int a_rd[TB][A_FAST ? STEPS : 1], b_rd[TB][B_FAST ? STEPS : 1];
#pragma unroll
  for (int i = 0; i < TB; ++i) {
#pragma unroll
    for (int s = 0; s < (A_FAST ? STEPS : 1); ++s) a_rd[i][s] = OpA::base(wm * W + i * 32 + li, half, s);
#pragma unroll
    for (int s = 0; s < (B_FAST ? STEPS : 1); ++s) b_rd[i][s] = OPERAND + OpB::base(col(i) + li, half, s);
  }
  auto four = [](const unsigned char* t, const int* rd, bool fast, int sub, int s, float (&v)[4]) {
    if (fast) {
      const float4 q = *reinterpret_cast<const float4*>(t + rd[s]);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float*>(t + rd[0] + (8 * s + u) * sub * 4);
  };

  f32x16 acc[TB][TB];
#pragma unroll
  for (int i = 0; i < TB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  {
    const int seg = MODE == DENSE_DX && first >= seg_stages ? 1 : 0;
    enter(seg, (long long)(first - seg * seg_stages) * DFK);
  }
#pragma unroll
  for (int u = 0; u < RING - 1; ++u) fetch(u);
  int buf = 0, fill = RING - 1, left = count;                     // this stage's buffer; the next to be filled
  do {                                                            // at least one stage
    wait_barrier<(RING - 2) * LOADS>();                           // this stage has landed, and every wave is done with the buffer before it
    fetch(fill);
    const unsigned char* t = lds + buf * STAGE;
    float a[2][TB][4], b[2][TB][4];
    auto read = [&](int s) {
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        four(t, a_rd[i], A_FAST, FM, s, a[s & 1][i]);
        four(t, b_rd[i], B_FAST, SUB, s, b[s & 1][i]);
      }
    };
    read(0);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (s + 1 < STEPS) read(s + 1);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < TB; ++i)
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[s & 1][j][u], a[s & 1][i][u], acc[i][j], 0, 0, 0);
    }
    buf = buf + 1 < RING ? buf + 1 : 0;
    fill = fill + 1 < RING ? fill + 1 : 0;
  } while (--left > 0);
  wait_loads();
  __syncthreads();
  dense_epilogue<float, MODE, W, 0>(p, acc, lds + wave * epi_wave_bytes(W), m0 + wm * W, n0 + wn * (MODE == DENSE_GATED ? W / 2 : W), src, split, Beside<MODE, W, 0>{});
}

// ---- any address, pitch and length ----
constexpr int FK = 32, F_ROW = FK + 4;                            // reduction elements of a stage; row pitches in LDS (floats): reads fall into different banks

// A work-group computes FM x FM outputs, a wave FM / 2 x FM / 2.
// WIDE: pitches beyond 32-bit offsets within a tile; else loads by buffers, beyond whose end they give zeros.
template <int MODE, int FM, bool WIDE>
__global__ __launch_bounds__(256, FM == 128 ? 2 : 4) void dense_f32_kernel(DenseP p) {
  constexpr bool A_FAST = MODE != DENSE_DW, B_FAST = MODE == DENSE_DX;
  constexpr int FN = FM, OUT_N = MODE == DENSE_GATED ? FN / 2 : FN;
  constexpr int W = FM / 2, TB = W / 32, EL = FM * FK / 256;      // extent of a wave, in blocks of 32; elements of a stage and operand per thread
  constexpr int F_COL = FM + 8;                                    // four rows apart: 32 banks further
  constexpr int F_TILE = FM * F_ROW > FK * F_COL ? FM * F_ROW : FK * F_COL;
  static_assert(16 * F_TILE >= 4 * epi_wave_bytes(W) && (FM == 128 ? 2 : 4) * 16 * F_TILE <= 163840, "two stages of two operands; epilogue; work-groups of a compute unit");
  __shared__ __attribute__((aligned(16))) float lds[4 * F_TILE];

  const int job = dense_job(p);
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
  auto e_of = [&](bool fast, int j) { return fast ? (tid >> 5) + 8 * j : tid & (FM - 1); };
  auto r_of = [&](bool fast, int j) { return fast ? tid & 31 : tid / FM + 256 / FM * j; };
  auto at = [](bool fast, int e, int r) { return fast ? e * F_ROW + r : r * F_COL + e; };
  float ra[2][EL], rb[2][EL];                                     // stages are asked for two ahead
  const unsigned none = DMA_OOB;
  // bytes of an element's row step, and of this thread's first element of a tile
  const long long a_step = (A_FAST ? 8 : 256 / FM) * p.lda * 4, b_step = (B_FAST ? 8 : 256 / FM) * p.ldb * 4;
  const int be = MODE == DENSE_GATED ? e_of(B_FAST, 0) & (FN / 2 - 1) : e_of(B_FAST, 0);
  const unsigned a_at = (unsigned)((A_FAST ? e_of(true, 0) * p.lda + r_of(true, 0) : r_of(false, 0) * p.lda + e_of(false, 0)) * 4);
  const unsigned b_at = (unsigned)((B_FAST ? e_of(true, 0) * p.ldb + r_of(true, 0) : r_of(false, 0) * p.ldb + be) * 4);
  const long long a_end = A_FAST ? (p.M - 1) * p.lda + p.red : (p.red - 1) * p.lda + p.M;     // elements of a segment
  const long long b_end = B_FAST ? (long long)(p.N - 1) * p.ldb + p.red : (p.red - 1) * p.ldb + p.N;
  auto pull = [&](int it, auto set) {
    constexpr int S = decltype(set)::value;
    int s = first + it;
    const bool second = MODE == DENSE_DX && p.segs == 2 && s >= seg_stages;
    if (second) s -= seg_stages;
    const long long r0 = (long long)s * FK;
    const float* a = (const float*)(second ? p.a[1] : p.a[0]);
    const float* b = (const float*)(second || (MODE == DENSE_DW && src) ? p.b[1] : p.b[0]);
    if constexpr (!WIDE) {
      const long long ao = A_FAST ? m0 * p.lda + r0 : r0 * p.lda + m0, bo = B_FAST ? n0 * p.ldb + r0 : r0 * p.ldb + n0;
      auto rsrc = [](const float* q, long long left) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(q), 0, (int)(left < 0x1fffffff ? left * 4 : 0x7ffffffc), 0x00020000);
      };
      const auto rs_a = rsrc(a + ao, a_end - ao), rs_b = rsrc(b + bo, b_end - bo), rs_u = rsrc(MODE == DENSE_GATED ? (const float*)p.b[1] + bo : b, b_end - bo);
      // what lies behind the end of a row is not beyond the buffer: along the reduction, or along the extent
      const unsigned av = (A_FAST ? r0 + r_of(true, 0) < p.red : m0 + e_of(false, 0) < p.M) ? a_at : none;
      const unsigned bv = (B_FAST ? r0 + r_of(true, 0) < p.red : n0 + be < p.N) ? b_at : none;
#pragma unroll
      for (int j = 0; j < EL; ++j) ra[S][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs_a, (int)(av + j * (unsigned)a_step), 0, 0));
      if constexpr (MODE == DENSE_GATED) {                        // half of the tile's columns, whole waves, from each source
        static_assert(FN / 2 >= 64 || MODE != DENSE_GATED, "a wave's columns are of one source");
        const bool up = __builtin_amdgcn_readfirstlane(e_of(false, 0)) >= FN / 2;
        if (up)
#pragma unroll
          for (int j = 0; j < EL; ++j) rb[S][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs_u, (int)(bv + j * (unsigned)b_step), 0, 0));
        else
#pragma unroll
          for (int j = 0; j < EL; ++j) rb[S][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs_b, (int)(bv + j * (unsigned)b_step), 0, 0));
      } else
#pragma unroll
        for (int j = 0; j < EL; ++j) rb[S][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs_b, (int)(bv + j * (unsigned)b_step), 0, 0));
      return;
    }
#pragma unroll
    for (int j = 0; j < EL; ++j) {
      const long long e = m0 + e_of(A_FAST, j), r = r0 + r_of(A_FAST, j);
      const bool ok = e < p.M && r < p.red;
      const float v = a[ok ? (A_FAST ? e * p.lda + r : r * p.lda + e) : 0];
      ra[S][j] = ok ? v : 0.f;
    }
#pragma unroll
    for (int j = 0; j < EL; ++j) {
      int c = e_of(B_FAST, j);
      const float* q = b;
      if (MODE == DENSE_GATED) {
        if (c >= FN / 2) q = (const float*)p.b[1];
        c &= FN / 2 - 1;
      }
      const long long e = n0 + c, r = r0 + r_of(B_FAST, j);
      const bool ok = e < p.N && r < p.red;
      const float v = q[ok ? (B_FAST ? e * p.ldb + r : r * p.ldb + e) : 0];
      rb[S][j] = ok ? v : 0.f;
    }
  };
  auto push = [&](auto set) {                                     // into the buffer of the same number
    constexpr int buf = decltype(set)::value;
    float* d = lds + buf * 2 * F_TILE;
#pragma unroll
    for (int j = 0; j < EL; ++j) d[at(A_FAST, e_of(A_FAST, j), r_of(A_FAST, j))] = ra[buf][j];
#pragma unroll
    for (int j = 0; j < EL; ++j) d[F_TILE + at(B_FAST, e_of(B_FAST, j), r_of(B_FAST, j))] = rb[buf][j];
  };
  // first column of the wave's block j within the tile
  auto col = [&](int j) { return MODE == DENSE_GATED ? j / (TB / 2 ? TB / 2 : 1) * (FN / 2) + wn * (W / 2) + j % (TB / 2 ? TB / 2 : 1) * 32 : wn * W + j * 32; };
  auto four = [&](bool fast, const float* t, int e, int s, float (&v)[4]) {
    if (fast) {
      const float4 q = *reinterpret_cast<const float4*>(t + e * F_ROW + 8 * s + 4 * half);
      v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = t[(8 * s + 4 * half + u) * F_COL + e];
  };

  f32x16 acc[TB][TB];
#pragma unroll
  for (int i = 0; i < TB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  const std::integral_constant<int, 0> even{};
  const std::integral_constant<int, 1> odd{};
  pull(0, even);
  if (count > 1) pull(1, odd);
  push(even);
  auto stage = [&](int it, auto set, auto other) {
    __syncthreads();                                              // this stage is in LDS, and every wave is done with the other buffer
    if (it + 2 < count) pull(it + 2, set);
    const float* t = lds + decltype(set)::value * 2 * F_TILE;
#pragma unroll
    for (int s = 0; s < FK / 8; ++s) {
      float a[TB][4], b[TB][4];
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        four(A_FAST, t, wm * W + i * 32 + li, s, a[i]);
        four(B_FAST, t + F_TILE, col(i) + li, s, b[i]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < TB; ++i)
#pragma unroll
          for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j][u], a[i][u], acc[i][j], 0, 0, 0);
    }
    if (it + 1 < count) push(other);
  };
  for (int it = 0; it < count; it += 2) {
    stage(it, even, odd);
    if (it + 1 < count) stage(it + 1, odd, even);
  }
  __syncthreads();
  dense_epilogue<float, MODE, W, 0>(p, acc, reinterpret_cast<unsigned char*>(lds) + wave * epi_wave_bytes(W), m0 + wm * W, n0 + wn * (MODE == DENSE_GATED ? W / 2 : W), src, split,
                                 Beside<MODE, W, 0>{});
}

// Tile and splits by an estimate as in dense_gemm.hip.  us of a stage of 32: of a work-group alone on its compute unit, and what each adds where there are more.
// us by tile and splits (the starred are taken; operands on 16-byte boundaries):   128: 1    2    4    8      64: 1    2    4    8
//   64 x 4096 x 4096                                                                 273  144   78   47      90   51   33*  35
//   1000 x 1024 x 1000                                                                74   47   35   41      29*  32   37   46
//   2048 x 2048 x 2048                                                               150* 146  158  183     155  167  180  204
//   4096 x 4096 x 4096                                                               992*               1151
// Through registers: 33 for 1000 x 1024 x 1000, 1048 for 4096 x 4096 x 4096.
struct F32Plan { int fm, splits; };
struct F32Cost { int fm, per_cu; double alone, each; };
constexpr F32Cost F32_COSTS[] = {{128, 2, 2.1, 1.95}, {64, 2, 0.66, 0.6}};

constexpr int MAX_SPLITS = 48;

F32Plan f32_plan(int mode, long long M, int N, long long red, int segs, int srcs) {
  const long long stages = (red + FK - 1) / FK * segs;
  F32Plan best = {128, 1};
  double least = 1e300;
  for (const F32Cost& t : F32_COSTS) {
    if (mode == DENSE_GATED && t.fm == 64) continue;              // a wave needs columns of both sources
    const int out_n = mode == DENSE_GATED ? t.fm / 2 : t.fm;
    const long long tiles = (M + t.fm - 1) / t.fm * ((N + out_n - 1) / out_n) * (mode == DENSE_DW ? srcs : 1), slots = 256LL * t.per_cu;
    for (int splits = 1; splits <= MAX_SPLITS; ++splits) {
      const long long per = (stages + splits - 1) / splits, jobs = tiles * splits, rounds = jobs / slots, rest = jobs - rounds * slots;
      if (splits > 1 && per < 4) break;
      const double held = (double)((rest + 255) / 256) * t.each;
      double us = rounds * (per * t.per_cu * t.each + 2.0) + (rest == 0 ? 0.0 : per * (held > t.alone ? held : t.alone) + 2.0);
      if (splits > 1) us += 5.0 + splits * (0.15 + (double)M * N * srcs * 2e-6);
      if (us < least) { least = us; best = {t.fm, splits}; }
    }
  }
  return best;
}

static_assert(FK == DFK, "one plan for both kernels");

template <int MODE, int FM, typename Kernel>
hipError_t launch_f32(Kernel kernel, DenseP& p, hipStream_t s) {
  p.stages = (int)((p.red + FK - 1) / FK) * p.segs;
  p.stages_per_split = (p.stages + p.splits - 1) / p.splits;
  p.splits = (p.stages + p.stages_per_split - 1) / p.stages_per_split;
  const int out_n = MODE == DENSE_GATED ? FM / 2 : FM;
  const long long tm = (p.M + FM - 1) / FM, tn = (long long)((p.N + out_n - 1) / out_n) * (MODE == DENSE_DW ? p.srcs : 1);
  if (tm * tn * p.splits > 0x7fffff00LL) return hipErrorInvalidValue;
  p.ntm = (int)tm;
  p.ntn = (int)tn;
  p.ntiles = (int)(tm * tn);
  const hipError_t e = launch_jobs<256>(p, [&](dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p); });
  return e == hipSuccess && p.splits > 1 ? dense_join(MODE, true, p, s) : e;
}

// As dma_ok of dense_gemm.hip.
bool f32_dma_ok(int mode, const DenseP& p) {
  uintptr_t at = (uintptr_t)p.a[0] | (uintptr_t)p.b[0];
  if (p.segs == 2) at |= (uintptr_t)p.a[1];
  if (p.segs == 2 || p.srcs == 2) at |= (uintptr_t)p.b[1];
  const long long a_len = mode == DENSE_DW ? p.M : p.red, b_len = mode == DENSE_DX ? p.red : p.N;
  return (at & 15) == 0 && ((p.lda | p.ldb | a_len | b_len) & 3) == 0 && p.lda < (1 << 21) && p.ldb < (1 << 21);
}

template <int MODE>
hipError_t f32_mode(DenseP& p, hipStream_t s) {
  const F32Plan plan = f32_plan(MODE, p.M, p.N, p.red, p.segs, p.srcs);
  p.splits = plan.splits;
  if (p.lda >= 1 << 21 || p.ldb >= 1 << 21) return launch_f32<MODE, 128>(dense_f32_kernel<MODE, 128, true>, p, s);
  const bool dma = f32_dma_ok(MODE, p);
  if constexpr (MODE != DENSE_GATED)
    if (plan.fm == 64) return dma ? launch_f32<MODE, 64>(dense_f32_dma_kernel<MODE, 64, 5>, p, s) : launch_f32<MODE, 64>(dense_f32_kernel<MODE, 64, false>, p, s);
  return dma ? launch_f32<MODE, 128>(dense_f32_dma_kernel<MODE, 128, 2>, p, s) : launch_f32<MODE, 128>(dense_f32_kernel<MODE, 128, false>, p, s);
}

}  // namespace

hipError_t dense_f32(int mode, DenseP& p, hipStream_t s) {
  switch (mode) {
    case DENSE_FWD: return f32_mode<DENSE_FWD>(p, s);
    case DENSE_GATED: return f32_mode<DENSE_GATED>(p, s);
    case DENSE_DX: return f32_mode<DENSE_DX>(p, s);
    default: return f32_mode<DENSE_DW>(p, s);
  }
}

uint64_t dense_f32_ws(int mode, long long M, int N, long long red, int segs, int srcs) {
  const int splits = f32_plan(mode, M, N, red, segs, srcs).splits;
  return splits > 1 ? (uint64_t)splits * srcs * M * N * 4 : 0;
}

}  // namespace lms
