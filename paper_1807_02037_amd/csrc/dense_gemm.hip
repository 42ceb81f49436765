// Matrix products of language-model layers in bf16 on the matrix cores (see DenseP for what a launch computes).
//
// A work-group of four waves computes BM x BN outputs; the reduction runs 64 at a time through two buffers in LDS.  Every operand lies in
// LDS as it lies in memory: where the reduction index is contiguous (rows of x, of the gradients, and of w for the data gradient) rows of 64 of it, read as
// they are; where it is not (w for the forward pass, both operands of the weight gradient) rows of 128 columns, or of 64, read with the gfx950 LDS transpose
// read.  So no operand is ever transposed in memory.  Products are taken transposed (the operand of the columns first): a lane then holds four consecutive
// columns of a row, and the epilogue turns 32 rows at a time through LDS into vectors of eight columns.
//
// Two ways into LDS: buffer loads that write LDS, for operands on 16-byte boundaries, where offsets beyond the descriptor read zeros and so
// ragged tiles need no branches; and through registers, at any address and for any length, element by element only where a vector crosses the end of a row.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "conv_dma.hpp"
#include "dense.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

constexpr int DK = 64;               // reduction elements of a stage
constexpr int NKS = DK / 16;         // steps of a stage: one 32x32x16 product per pair of operand fragments
constexpr int DSL = DK / 8;          // 16-byte slots of a row of DK

// 16-byte slots within a row of DK are permuted by this, and 64-byte blocks within a row of W columns by that, so that the rows a read touches at a
// time fall into different banks.
__device__ __forceinline__ int row_swz(int row) { return (row >> 1) & 7; }
template <int W>
__device__ __forceinline__ int col_swz(int r) { return W == 128 ? r & 3 : (r >> 1) & 1; }

template <int BM_, int BN_>
struct DenseTile {
  static constexpr int BM = BM_, BN = BN_, WM = 2, WN = 2, NT = 256;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static constexpr int A_BYTES = BM * DK * 2, B_BYTES = BN * DK * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int AV = A_BYTES / (16 * NT), BV = B_BYTES / (16 * NT);      // vectors of a stage per thread
  static constexpr int EPI_WAVE = epi_wave_bytes(WTN);
  static constexpr int LDS_BYTES = 2 * STAGE > 4 * EPI_WAVE ? 2 * STAGE : 4 * EPI_WAVE;
  static constexpr int OCC = 163840 / LDS_BYTES < 4 ? 163840 / LDS_BYTES : 4;   // work-groups of a compute unit, waves of a SIMD
};

// One operand's tile in LDS: EXT rows or columns of the result by DK of the reduction.
//   RED_FAST: element (e, r) at base[e * ld + r]; in LDS rows e of DK.
//   else:     element (e, r) at base[r * ld + e]; in LDS SUB columns wide pieces of rows r, one after the other.
template <int EXT, bool RED_FAST, int SUB>
struct Operand {
  static constexpr int V = EXT * DK / (8 * 256);        // vectors per thread
  // Vector v: its element along the extent, and along the reduction.
  __device__ static __forceinline__ void where(int v, int& e, int& r) {
    if constexpr (RED_FAST) {
      e = v / DSL;
      r = ((v % DSL) ^ row_swz(e)) * 8;
    } else {
      constexpr int VPR = SUB / 8;
      const int piece = v / (DK * VPR), w = v % (DK * VPR);
      r = w / VPR;
      e = piece * SUB + (((w % VPR) >> 2) ^ col_swz<SUB>(r)) * 32 + (w & 3) * 8;
    }
  }
  // LDS address of this lane's piece of the fragment of elements e0 .. e0+31 (e0: a multiple of 32) at step ks.
  __device__ static __forceinline__ int address(int e0, int ks, int lane) {
    if constexpr (RED_FAST) {
      const int row = e0 + (lane & 31);
      return row * (DK * 2) + (((ks * 2 + (lane >> 5)) ^ row_swz(row)) << 4);
    } else {
      const int li = lane & 15, lg = lane >> 4;
      const int r = ks * 16 + 8 * (lg >> 1) + (li >> 2);
      return (e0 / SUB) * (DK * SUB * 2) + r * (SUB * 2) + ((((e0 % SUB) >> 5) ^ col_swz<SUB>(r)) << 6) + 32 * (lg & 1) + 8 * (li & 3);
    }
  }
  __device__ static __forceinline__ bf16x8 fragment(const unsigned char* at) {
    if constexpr (RED_FAST) return *reinterpret_cast<const bf16x8*>(at);
    else return tr_frag(at, at + 4 * SUB * 2);
  }
};

template <int MODE, int BN>
constexpr int dense_sub() { return MODE == DENSE_GATED ? BN / 2 : (BN < 128 ? BN : 128); }

// Order of the tiles: neighbours in the grid's order share operands in the L2 of an XCD, so a run of tiles covers GROUP rows of tiles by some columns.
constexpr int GROUP = 8;
__device__ __forceinline__ void tile_at(const DenseP& p, int tile, int& tm, int& tn) {
  const int per = GROUP * p.ntn, g = tile / per, first = g * GROUP, rows = p.ntm - first < GROUP ? p.ntm - first : GROUP, w = tile - g * per;
  tm = first + w % rows;
  tn = w / rows;
}

template <typename T, int MODE, bool DMA>
__global__ __launch_bounds__(T::NT, T::OCC) void dense_kernel(DenseP p) {
  constexpr bool A_FAST = MODE != DENSE_DW, B_FAST = MODE == DENSE_DX;
  constexpr int BM = T::BM, BN = T::BN, TM = T::TM, TN = T::TN, AV = T::AV, BV = T::BV, SUB = dense_sub<MODE, BN>();
  constexpr int OUT_N = MODE == DENSE_GATED ? BN / 2 : BN;       // output columns of a tile
  typedef Operand<BM, A_FAST, BM < 128 ? BM : 128> OpA;
  typedef Operand<BN, B_FAST, SUB> OpB;
  extern __shared__ __attribute__((aligned(256))) unsigned char dense_smem[];

  const int job = xcd_order(p.ntiles * p.splits);
  if (job < 0) return;
  const int split = job / p.ntiles;
  int tm, tn;
  tile_at(p, job - split * p.ntiles, tm, tn);
  int src = 0;
  if (MODE == DENSE_DW && p.srcs == 2) {                          // columns of tiles of the one source, then of the other
    const int each = p.ntn / 2;
    src = tn >= each;
    tn -= src * each;
  }
  const long long m0 = (long long)tm * BM;
  const int n0 = tn * OUT_N;
  const int first = split * p.stages_per_split, count = (p.stages - first < p.stages_per_split ? p.stages - first : p.stages_per_split);
  const int seg_stages = p.stages / p.segs;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;

  // ---- loads ----
  const uint16_t* const a0 = (const uint16_t*)p.a[0];
  const uint16_t* const b0 = (const uint16_t*)(MODE == DENSE_DW && src ? p.b[1] : p.b[0]);
  const uint16_t* const a1 = (const uint16_t*)p.a[1];
  const uint16_t* const b1 = (const uint16_t*)p.b[1];
  int a_e[AV], a_r[AV], b_e[BV], b_r[BV];                         // place of a vector in the tile; b_e of DENSE_GATED counts within a source
  unsigned a_off[AV], b_off[BV];
#pragma unroll
  for (int j = 0; j < AV; ++j) {
    OpA::where(tid + j * 256, a_e[j], a_r[j]);
    a_off[j] = m0 + a_e[j] < p.M ? (unsigned)((A_FAST ? a_e[j] * p.lda + a_r[j] : a_r[j] * p.lda + a_e[j]) * 2) : DMA_OOB;
  }
#pragma unroll
  for (int j = 0; j < BV; ++j) {
    OpB::where(tid + j * 256, b_e[j], b_r[j]);
    if (MODE == DENSE_GATED) b_e[j] %= SUB;
    b_off[j] = n0 + b_e[j] < p.N ? (unsigned)((B_FAST ? b_e[j] * p.ldb + b_r[j] : b_r[j] * p.ldb + b_e[j]) * 2) : DMA_OOB;
  }
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)dense_smem + wave * 1024);
  const long long a_end = A_FAST ? (p.M - 1) * p.lda + p.red : (p.red - 1) * p.lda + p.M;     // elements of a segment
  const long long b_end = B_FAST ? (long long)(p.N - 1) * p.ldb + p.red : (p.red - 1) * p.ldb + p.N;

  // stage `it` of this work-group: reduction elements r0 .. r0+63 of a segment
  struct At { const uint16_t *a, *b, *bu; long long a_left, b_left; long long r0; bool whole; };
  auto stage_at = [&](int it) {
    int s = first + it;
    bool second = false;
    if (MODE == DENSE_DX && s >= seg_stages && p.segs == 2) { s -= seg_stages; second = true; }
    At t;
    t.r0 = (long long)s * DK;
    const long long ao = A_FAST ? m0 * p.lda + t.r0 : t.r0 * p.lda + m0, bo = B_FAST ? n0 * p.ldb + t.r0 : t.r0 * p.ldb + n0;
    t.a = (second ? a1 : a0) + ao;
    t.b = (second ? b1 : b0) + bo;
    t.bu = MODE == DENSE_GATED ? b1 + bo : nullptr;
    t.whole = t.r0 + DK <= p.red;
    t.a_left = it < count ? (a_end - ao) * 2 : 0;                 // beyond the last stage: nothing but zeros
    t.b_left = it < count ? (b_end - bo) * 2 : 0;
    return t;
  };
  auto clip = [](long long bytes) { return bytes < 0 ? 0 : bytes; };
  // buffer loads that write LDS
  auto dma_a = [&](const At& t, const v4u& rs, int buf, int j) {
    const bool in = !A_FAST || t.whole || t.r0 + a_r[j] < p.red;  // otherwise the rows beyond the last lie beyond the buffer
    load_lds16(rs, lds0 + buf * T::STAGE + j * 4096, in ? a_off[j] : DMA_OOB, 0);
  };
  auto dma_b = [&](const At& t, const v4u& rs, int buf, int j) {
    const bool in = !B_FAST || t.whole || t.r0 + b_r[j] < p.red;
    load_lds16(rs, lds0 + buf * T::STAGE + T::A_BYTES + j * 4096, in ? b_off[j] : DMA_OOB, 0);
  };
  auto fetch = [&](int it, int buf) {
    const At t = stage_at(it);
    const v4u rs_a = buffer_rsrc(t.a, clip(t.a_left)), rs_b = buffer_rsrc(t.b, clip(t.b_left));
    const v4u rs_u = MODE == DENSE_GATED ? buffer_rsrc(t.bu, clip(t.b_left)) : rs_b;
#pragma unroll
    for (int j = 0; j < AV; ++j) dma_a(t, rs_a, buf, j);
#pragma unroll
    for (int j = 0; j < BV; ++j) dma_b(t, MODE == DENSE_GATED && j >= BV / 2 ? rs_u : rs_b, buf, j);
  };
  // through registers, at any address
  v4u ra[DMA ? 1 : AV], rb[DMA ? 1 : BV];
  auto vector = [&](const uint16_t* q, long long have) {
    v4u v = {0u, 0u, 0u, 0u};
    if (have >= 8) __builtin_memcpy(&v, q, 16);
    else
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (e < have) v[e >> 1] |= (unsigned)q[e] << ((e & 1) * 16);
    return v;
  };
  auto pull = [&](int it) {
    const At t = stage_at(it);
#pragma unroll
    for (int j = 0; j < AV; ++j) {
      const long long red = p.red - t.r0 - a_r[j], ext = p.M - m0 - a_e[j];
      ra[j] = vector(t.a + (A_FAST ? a_e[j] * p.lda + a_r[j] : a_r[j] * p.lda + a_e[j]), red > 0 && ext > 0 ? (A_FAST ? red : ext) : 0);
    }
#pragma unroll
    for (int j = 0; j < BV; ++j) {
      const long long red = p.red - t.r0 - b_r[j], ext = (long long)p.N - n0 - b_e[j];
      rb[j] = vector((MODE == DENSE_GATED && j >= BV / 2 ? t.bu : t.b) + (B_FAST ? b_e[j] * p.ldb + b_r[j] : b_r[j] * p.ldb + b_e[j]),
                     red > 0 && ext > 0 ? (B_FAST ? red : ext) : 0);
    }
  };
  auto push = [&](int buf) {
    unsigned char* d = dense_smem + buf * T::STAGE + tid * 16;
#pragma unroll
    for (int j = 0; j < AV; ++j) *reinterpret_cast<v4u*>(d + j * 4096) = ra[j];
#pragma unroll
    for (int j = 0; j < BV; ++j) *reinterpret_cast<v4u*>(d + T::A_BYTES + j * 4096) = rb[j];
  };

  // ---- LDS read addresses ----
  int a_rd[TM][NKS], b_rd[TN][NKS];
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) {
#pragma unroll
    for (int i = 0; i < TM; ++i) a_rd[i][ks] = OpA::address(wm * T::WTM + i * 32, ks, lane);
#pragma unroll
    for (int j = 0; j < TN; ++j)
      b_rd[j][ks] = T::A_BYTES + OpB::address(MODE == DENSE_GATED ? (j / (TN / 2)) * SUB + (wn * (TN / 2) + j % (TN / 2)) * 32 : wn * T::WTN + j * 32, ks, lane);
  }

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  auto multiply = [&](int buf) {
    const unsigned char* t = dense_smem + buf * T::STAGE;
    bf16x8 af[2][TM], bf[2][TN];
    auto load = [&](int ks) {
#pragma unroll
      for (int j = 0; j < TN; ++j) bf[ks & 1][j] = OpB::fragment(t + b_rd[j][ks]);
#pragma unroll
      for (int i = 0; i < TM; ++i) af[ks & 1][i] = OpA::fragment(t + a_rd[i][ks]);
    };
    load(0);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      if (ks + 1 < NKS) load(ks + 1);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[ks & 1][j], af[ks & 1][i], acc[i][j], 0, 0, 0);
    }
  };

  if constexpr (DMA) {
    fetch(0, 0);
    for (int it = 0; it < count; it += 2) {
      unrolled<2>([&](auto k) {
        constexpr int buf = decltype(k)::value;
        if (it + buf >= count) return;
        wait_barrier<0>();                                        // this stage has landed, and every wave is done with the other buffer
        fetch(it + buf + 1, buf ^ 1);
        multiply(buf);
      });
    }
    wait_loads();
  } else {
    pull(0);
    push(0);
    for (int it = 0; it < count; ++it) {
      __syncthreads();                                            // this stage is in LDS, and every wave is done with the other buffer
      if (it + 1 < count) pull(it + 1);
      multiply(it & 1);
      if (it + 1 < count) push((it + 1) & 1);
    }
  }
  __syncthreads();                                                // the buffers are free for the epilogue
  dense_epilogue<uint16_t, MODE, T::WTN>(p, acc, dense_smem + wave * T::EPI_WAVE, m0 + wm * T::WTM, n0 + wn * (MODE == DENSE_GATED ? T::WTN / 2 : T::WTN), src, split);
}

template <typename T, int MODE, bool DMA>
hipError_t launch_dense(DenseP& p, hipStream_t s) {
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(dense_kernel<T, MODE, DMA>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
  if (attr != hipSuccess) return attr;
  const int out_n = MODE == DENSE_GATED ? T::BN / 2 : T::BN;
  const long long tm = (p.M + T::BM - 1) / T::BM, tn = (long long)((p.N + out_n - 1) / out_n) * (MODE == DENSE_DW ? p.srcs : 1);
  if (tm * tn * p.splits > 0x7fffff00LL) return hipErrorInvalidValue;
  p.ntm = (int)tm;
  p.ntn = (int)tn;
  p.ntiles = (int)(tm * tn);
  hipLaunchKernelGGL((dense_kernel<T, MODE, DMA>), dim3((unsigned)xcd_grid((long long)p.ntiles * p.splits)), dim3(T::NT), T::LDS_BYTES, s, p);
  return hipGetLastError();
}

typedef DenseTile<128, 128> Tile128;

// Loads that write LDS need whole 16-byte vectors: addresses and pitches in multiples of 8 elements, and lengths too, since a vector across the end of a row
// would bring in what lies behind it.  32-bit offsets within a tile bound the pitch.
bool dma_ok(int mode, const DenseP& p) {
  uintptr_t at = (uintptr_t)p.a[0] | (uintptr_t)p.b[0];
  if (p.segs == 2) at |= (uintptr_t)p.a[1];
  if (p.segs == 2 || p.srcs == 2) at |= (uintptr_t)p.b[1];
  const long long a_len = mode == DENSE_DW ? p.M : p.red, b_len = mode == DENSE_DX ? p.red : p.N;
  return (at & 15) == 0 && ((p.lda | p.ldb | a_len | b_len) & 7) == 0 && p.lda < (1 << 21) && p.ldb < (1 << 21);
}

template <int MODE>
hipError_t dense_mode(DenseP& p, hipStream_t s) {
  return dma_ok(MODE, p) ? launch_dense<Tile128, MODE, true>(p, s) : launch_dense<Tile128, MODE, false>(p, s);
}

}  // namespace

hipError_t dense_bf16(int mode, DenseP& p, hipStream_t s) {
  p.stages = (int)((p.red + DK - 1) / DK) * p.segs;
  p.splits = 1;
  p.stages_per_split = p.stages;
  switch (mode) {
    case DENSE_FWD: return dense_mode<DENSE_FWD>(p, s);
    case DENSE_GATED: return dense_mode<DENSE_GATED>(p, s);
    case DENSE_DX: return dense_mode<DENSE_DX>(p, s);
    default: return dense_mode<DENSE_DW>(p, s);
  }
}

}  // namespace lms
