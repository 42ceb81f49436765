// Matrix products of language-model layers in bf16 on the matrix cores (see DenseP for what a launch computes).
//
// A work-group of four waves computes BM x BN outputs; the reduction runs 64 at a time through a ring of two to five stages in LDS.  Every operand lies in
// LDS as it lies in memory: where the reduction index is contiguous (rows of x, of the gradients, and of w for the data gradient) rows of 64 of it, read as
// they are; where it is not (w for the forward pass, both operands of the weight gradient) rows of 128 columns, or of 64, read with the gfx950 LDS transpose
// read.  So no operand is ever transposed in memory.  Products are taken transposed (the operand of the columns first): a lane then holds four consecutive
// columns of a row, and the epilogue turns 32 rows at a time through LDS into vectors of eight columns.
//
// Two ways into LDS: buffer loads that write LDS, for operands on 16-byte boundaries, where offsets beyond the descriptor read zeros and so
// ragged tiles need no branches; and through registers and two stages, at any address and for any length: a vector of columns across the end of a row is the row's last eight,
// shifted; only a partial last stage and rows of fewer than eight columns go element by element.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "conv_dma.hpp"
#include "dense.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

// 16-byte slots within a row of DK reduction elements are permuted by this, and 64-byte blocks within a row of W columns by that, so that the rows a read touches at a
// time fall into different banks.
template <int DK>
__device__ __forceinline__ int row_swz(int row) { return DK == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int W>
__device__ __forceinline__ int col_swz(int r) { return W == 128 ? r & 3 : W == 64 ? (r >> 1) & 1 : 0; }

template <int BM_, int BN_, int DK_, int RING_, int WM_ = 2, int WN_ = 2>
struct DenseTile {
  static constexpr int DK = DK_;                                  // reduction elements of a stage
  static constexpr int RING = RING_;                              // stages in LDS
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NT = 256;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static constexpr int A_BYTES = BM * DK * 2, B_BYTES = BN * DK * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int AV = A_BYTES / (16 * NT), BV = B_BYTES / (16 * NT);      // vectors of a stage per thread
  static constexpr int EPI_WAVE = epi_wave_bytes(WTN);
  static constexpr int LDS_BYTES = RING * STAGE > 4 * EPI_WAVE ? RING * STAGE : 4 * EPI_WAVE;
  static constexpr int OCC = 163840 / LDS_BYTES < 4 ? 163840 / LDS_BYTES : 4;   // work-groups of a compute unit, waves of a SIMD
};

// One operand's tile in LDS: EXT rows or columns of the result by DK of the reduction.
//   RED_FAST: element (e, r) at base[e * ld + r]; in LDS rows e of DK.
//   else:     element (e, r) at base[r * ld + e]; in LDS SUB columns wide pieces of rows r, one after the other.
template <int EXT, bool RED_FAST, int SUB, int DK>
struct Operand {
  static constexpr int NKS = DK / 16, DSL = DK / 8;     // steps of a stage: one 32x32x16 product per pair of operand fragments; 16-byte slots of a row of DK
  static constexpr int V = EXT * DK / (8 * 256);        // vectors per thread
  // Vector v: its element along the extent, and along the reduction.
  __device__ static __forceinline__ void where(int v, int& e, int& r) {
    if constexpr (RED_FAST) {
      e = v / DSL;
      r = ((v % DSL) ^ row_swz<DK>(e)) * 8;
    } else {
      constexpr int VPR = SUB / 8;
      const int piece = v / (DK * VPR), w = v % (DK * VPR);
      r = w / VPR;
      e = piece * SUB + (((w % VPR) >> 2) ^ col_swz<SUB>(r)) * 32 + (w & 3) * 8;
    }
  }
  // LDS address of this lane's piece of the fragment of elements e0 .. e0+31 (e0: a multiple of 32) at step ks: rd[] of N registers from prepare(), plus a constant.
  static constexpr int N = RED_FAST ? NKS : EXT / 32;             // registers: of the steps, or of the fragments (at most)
  __device__ static __forceinline__ int base(int e0, int ks, int lane) {
    if constexpr (RED_FAST) {
      const int row = e0 + (lane & 31);
      return row * (DK * 2) + (((ks * 2 + (lane >> 5)) ^ row_swz<DK>(row)) << 4);
    } else {
      const int li = lane & 15, lg = lane >> 4;
      const int r = 8 * (lg >> 1) + (li >> 2);                    // + 16 ks, which the permutation does not see
      return (e0 / SUB) * (DK * SUB * 2) + r * (SUB * 2) + ((((e0 % SUB) >> 5) ^ col_swz<SUB>(r)) << 6) + 32 * (lg & 1) + 8 * (li & 3);
    }
  }
  template <int TILES, typename F>
  __device__ static __forceinline__ void prepare(int (&rd)[N], int lane, F&& first) {
    if constexpr (RED_FAST)
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) rd[ks] = base(first(0), ks, lane);
    else
#pragma unroll
      for (int i = 0; i < TILES; ++i) rd[i] = base(first(i), 0, lane);
  }
  __device__ static __forceinline__ int address(const int (&rd)[N], int i, int ks) {
    if constexpr (RED_FAST) return rd[ks] + i * (32 * DK * 2);    // fragments of a wave follow one another: 32 rows further the permutation is the same
    else return rd[i] + ks * (16 * SUB * 2);
  }
  __device__ static __forceinline__ bf16x8 fragment(const unsigned char* at) {
    if constexpr (RED_FAST) return *reinterpret_cast<const bf16x8*>(at);
    else return tr_frag(at, at + 4 * SUB * 2);
  }
};

// The reduction lies in rows of b.
template <int MODE>
constexpr bool dense_b_fast() { return MODE == DENSE_DX || dense_q8(MODE); }
template <int MODE, int BN>
constexpr int dense_sub() { return MODE == DENSE_GATED ? BN / 2 : (BN < 128 ? BN : 128); }

// Accumulators, what they leave as, and one product of fragments of 16 bytes a lane: 32 x 32 x 16 in bf16, 32 x 32 x 32 in 8-bit integers, in the same time.
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
template <int MODE>
struct DenseKind {
  typedef std::conditional_t<dense_q8(MODE), i32x16, f32x16> Acc;
  typedef std::conditional_t<MODE == DENSE_Q8_F32, float, uint16_t> Out;
  __device__ static __forceinline__ Acc product(const bf16x8& b, const bf16x8& a, const Acc& c) {
    if constexpr (dense_q8(MODE)) return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(v4i, b), __builtin_bit_cast(v4i, a), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
  }
};

// Order of the tiles: neighbours in the grid's order share operands in the L2 of an XCD, so a run of tiles covers GROUP rows of tiles by some columns.
constexpr int GROUP = 8;
__device__ __forceinline__ void tile_at(const DenseP& p, int tile, int& tm, int& tn) {
  const int per = GROUP * p.ntn, g = tile / per, first = g * GROUP, rows = p.ntm - first < GROUP ? p.ntm - first : GROUP, w = tile - g * per;
  tm = first + w % rows;
  tn = w / rows;
}

template <typename T, int MODE, bool DMA>
__device__ __forceinline__ void dense_tile(const DenseP& p, int job) {
  constexpr bool A_FAST = MODE != DENSE_DW, B_FAST = dense_b_fast<MODE>();
  constexpr int BM = T::BM, BN = T::BN, TM = T::TM, TN = T::TN, AV = T::AV, BV = T::BV, SUB = dense_sub<MODE, BN>();
  constexpr int OUT_N = MODE == DENSE_GATED ? BN / 2 : BN;       // output columns of a tile
  constexpr int DK = T::DK, NKS = DK / 16;
  typedef Operand<BM, A_FAST, BM < 128 ? BM : 128, DK> OpA;
  typedef Operand<BN, B_FAST, SUB, DK> OpB;
  extern __shared__ __attribute__((aligned(256))) unsigned char dense_smem[];

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
  const long long m_left = p.M - m0, n_left = (long long)p.N - n0;
  int a_e[AV], a_r[AV], b_e[BV], b_r[BV];                         // place of a vector in the tile; b_e of DENSE_GATED counts within a source
#pragma unroll
  for (int j = 0; j < AV; ++j) OpA::where(tid + j * 256, a_e[j], a_r[j]);
#pragma unroll
  for (int j = 0; j < BV; ++j) {
    OpB::where(tid + j * 256, b_e[j], b_r[j]);
    if (MODE == DENSE_GATED) b_e[j] %= SUB;
  }
  struct Source { const uint16_t *a, *b, *bu; };
  // the operands at reduction element r of a segment
  auto source = [&](int seg, long long r) {
    const long long ao = A_FAST ? m0 * p.lda + r : r * p.lda + m0, bo = B_FAST ? n0 * p.ldb + r : r * p.ldb + n0;
    const int bs = MODE == DENSE_DX ? seg : MODE == DENSE_DW ? src : 0;
    return Source{(const uint16_t*)p.a[MODE == DENSE_DX ? seg : 0] + ao, (const uint16_t*)p.b[bs] + bo, MODE == DENSE_GATED ? (const uint16_t*)p.b[1] + bo : nullptr};
  };

  // Buffer loads that write LDS.  The descriptors move along the reduction with the stages; the vectors' offsets from them stay, those of rows or columns that do not
  // exist beyond every buffer.  The last stage of a segment may be partial: there the vectors beyond the end are moved out as well, or lie beyond the buffer.
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)dense_smem + wave * 1024);
  unsigned a_off[DMA ? AV : 1], b_off[DMA ? BV : 1];
  v4u rs_a = {}, rs_b = {}, rs_u = {};
  int to_load = count, load_seg = 0;                              // stages not asked for yet
  long long load_r = 0;
  auto enter = [&](int seg, long long r) {                        // the next stage is of segment seg, element r
    load_seg = seg;
    load_r = r;
    const Source t = source(seg, r);
    rs_a = buffer_rsrc(t.a, 0x7fffffff);
    rs_b = buffer_rsrc(t.b, 0x7fffffff);
    if (MODE == DENSE_GATED) rs_u = buffer_rsrc(t.bu, 0x7fffffff);
#pragma unroll
    for (int j = 0; j < AV; ++j) a_off[j] = a_e[j] < m_left ? (unsigned)((A_FAST ? a_e[j] * p.lda + a_r[j] : a_r[j] * p.lda + a_e[j]) * 2) : DMA_OOB;
#pragma unroll
    for (int j = 0; j < BV; ++j) b_off[j] = b_e[j] < n_left ? (unsigned)((B_FAST ? b_e[j] * p.ldb + b_r[j] : b_r[j] * p.ldb + b_e[j]) * 2) : DMA_OOB;
  };
  auto last = [&]() {                                             // the next stage is partial
#pragma unroll
    for (int j = 0; j < AV; ++j) a_off[j] = load_r + a_r[j] < p.red ? a_off[j] : DMA_OOB;
#pragma unroll
    for (int j = 0; j < BV; ++j) b_off[j] = load_r + b_r[j] < p.red ? b_off[j] : DMA_OOB;
  };
  auto advance = [&]() {
    if (--to_load <= 0) {                                         // beyond the last: nothing but zeros
      rs_a[2] = rs_b[2] = rs_u[2] = 0;
      return;
    }
    load_r += DK;
    if (MODE == DENSE_DX && load_r >= p.red) enter(1, 0);
    else {
      auto move = [](v4u& rs, long long bytes) {
        const unsigned long long base = ((unsigned long long)rs[1] << 32 | rs[0]) + bytes;
        rs[0] = (unsigned)base;
        rs[1] = (unsigned)(base >> 32);
      };
      move(rs_a, (A_FAST ? DK : DK * p.lda) * 2);
      move(rs_b, (B_FAST ? DK : DK * p.ldb) * 2);
      if (MODE == DENSE_GATED) move(rs_u, DK * p.ldb * 2);
    }
    if (load_r + DK > p.red) last();
  };
  constexpr int LOADS = AV + BV;
  auto load = [&](unsigned at, int v) {                           // load v of a stage into the buffer at `at`
    if (v < AV) load_lds16(rs_a, lds0 + at + v * 4096, a_off[v < AV ? v : 0], 0);
    else load_lds16(MODE == DENSE_GATED && v - AV >= BV / 2 ? rs_u : rs_b, lds0 + at + T::A_BYTES + (v - AV) * 4096, b_off[v < AV ? 0 : v - AV], 0);
  };
  // Through registers, at any address.  Vectors move along the reduction by pointers.  Rows and columns beyond the last: any that is there, their results are not
  // stored.  A vector of columns across the end of a row is the row's last eight elements, shifted.  The last stage of a segment, if it is partial, and
  // rows of fewer than eight columns go element by element.
  v4u ra[DMA ? 1 : AV], rb[DMA ? 1 : BV];
  const uint16_t *pa[DMA ? 1 : AV], *pb[DMA ? 1 : BV];
  int a_shift = 0, b_shift = 0;                                   // elements; the same for all of a thread's vectors
  const bool tiny = (!A_FAST && p.M < 8) || (!B_FAST && p.N < 8);
  const bool a_cut = !A_FAST && m_left < BM, b_cut = !B_FAST && n_left < OUT_N;
  auto at_start = [&](int seg, long long r0) {
    const Source t = source(seg, r0);
#pragma unroll
    for (int j = 0; j < AV; ++j) {
      const long long most = A_FAST ? m_left - 1 : m_left - 8;
      const long long e = a_e[j] <= most ? a_e[j] : most;         // may lie before the tile
      if (!A_FAST) a_shift = a_e[j] < m_left ? (int)(a_e[j] - e) : 0;
      pa[j] = t.a + (A_FAST ? e * p.lda + a_r[j] : a_r[j] * p.lda + e);
    }
#pragma unroll
    for (int j = 0; j < BV; ++j) {
      const long long most = B_FAST ? n_left - 1 : n_left - 8;
      const long long e = b_e[j] <= most ? b_e[j] : most;
      if (!B_FAST) b_shift = b_e[j] < n_left ? (int)(b_e[j] - e) : 0;
      pb[j] = (MODE == DENSE_GATED && j >= BV / 2 ? t.bu : t.b) + (B_FAST ? e * p.ldb + b_r[j] : b_r[j] * p.ldb + e);
    }
  };
  auto shifted = [](v4u v, int by) {                              // elements by .. 7 to the front
    const unsigned __int128 w = __builtin_bit_cast(unsigned __int128, v) >> (16 * by);
    return __builtin_bit_cast(v4u, w);
  };
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
    const int st = first + it, seg = MODE == DENSE_DX && st >= seg_stages ? 1 : 0;
    const long long r0 = (long long)(st - seg * seg_stages) * DK;
    if (it == 0 || (MODE == DENSE_DX && r0 == 0)) at_start(seg, r0);
    if (r0 + DK <= p.red && !tiny) {
#pragma unroll
      for (int j = 0; j < AV; ++j) {
        __builtin_memcpy(&ra[j], pa[j], 16);
        pa[j] += A_FAST ? DK : DK * p.lda;
      }
#pragma unroll
      for (int j = 0; j < BV; ++j) {
        __builtin_memcpy(&rb[j], pb[j], 16);
        pb[j] += B_FAST ? DK : DK * p.ldb;
      }
      return;
    }
    const Source t = source(seg, r0);
#pragma unroll
    for (int j = 0; j < AV; ++j) {
      const long long red = p.red - r0 - a_r[j], ext = m_left - a_e[j];
      ra[j] = vector(t.a + (A_FAST ? a_e[j] * p.lda + a_r[j] : a_r[j] * p.lda + a_e[j]), red > 0 && ext > 0 ? (A_FAST ? red : ext) : 0);
    }
#pragma unroll
    for (int j = 0; j < BV; ++j) {
      const long long red = p.red - r0 - b_r[j], ext = n_left - b_e[j];
      rb[j] = vector((MODE == DENSE_GATED && j >= BV / 2 ? t.bu : t.b) + (B_FAST ? b_e[j] * p.ldb + b_r[j] : b_r[j] * p.ldb + b_e[j]),
                     red > 0 && ext > 0 ? (B_FAST ? red : ext) : 0);
    }
  };
  auto push = [&](int it) {
    unsigned char* d = dense_smem + (it & 1) * T::STAGE + tid * 16;
    const int st = first + it, seg = MODE == DENSE_DX && st >= seg_stages ? 1 : 0;
    const bool whole = (long long)(st - seg * seg_stages + 1) * DK <= p.red && !tiny;     // else its vectors are in place
    if (a_cut && whole)
#pragma unroll
      for (int j = 0; j < AV; ++j) ra[j] = shifted(ra[j], a_shift);
    if (b_cut && whole)
#pragma unroll
      for (int j = 0; j < BV; ++j) rb[j] = shifted(rb[j], b_shift);
#pragma unroll
    for (int j = 0; j < AV; ++j) *reinterpret_cast<v4u*>(d + j * 4096) = ra[j];
#pragma unroll
    for (int j = 0; j < BV; ++j) *reinterpret_cast<v4u*>(d + T::A_BYTES + j * 4096) = rb[j];
  };

  int a_rd[OpA::N], b_rd[OpB::N];
  OpA::template prepare<TM>(a_rd, lane, [&](int i) { return wm * T::WTM + i * 32; });
  OpB::template prepare<TN>(b_rd, lane, [&](int j) {
    return MODE == DENSE_GATED ? (j / (TN / 2)) * SUB + (wn * (TN / 2) + j % (TN / 2)) * 32 : wn * T::WTN + j * 32;
  });

  const long long wm0 = m0 + wm * T::WTM;                         // the wave's first row and column
  const int wn0 = n0 + wn * (MODE == DENSE_GATED ? T::WTN / 2 : T::WTN);
  constexpr int PRE = !DMA ? 0 : TM < 2 ? TM : 2;
  Beside<MODE, T::WTN, PRE> beside;
  typename DenseKind<MODE>::Acc acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
  bf16x8 af[2][TM], bf[2][TN];                                    // operands are read one step ahead of their products
  auto read = [&](const unsigned char* t, int ks, int f) {        // fragment f of step ks
    if (f < TN) bf[ks & 1][f] = OpB::fragment(t + T::A_BYTES + OpB::address(b_rd, f, ks));
    else af[ks & 1][f - TN] = OpA::fragment(t + OpA::address(a_rd, f - TN, ks));
  };
  auto product = [&](int ks, int q) {
    const int i = q / TN, j = q % TN;
    acc[i][j] = DenseKind<MODE>::product(bf[ks & 1][j], af[ks & 1][i], acc[i][j]);
  };
  auto multiply = [&](int buf) {
    const unsigned char* t = dense_smem + buf * T::STAGE;
#pragma unroll
    for (int f = 0; f < TM + TN; ++f) read(t, 0, f);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) {
      if (ks + 1 < NKS)
#pragma unroll
        for (int f = 0; f < TM + TN; ++f) read(t, ks + 1, f);
#pragma unroll
      for (int q = 0; q < TM * TN; ++q) product(ks, q);
    }
  };

  if constexpr (DMA) {
    // The last step of a stage has its operands in registers before it begins, so the barrier stands in front of it: there every wave is done with this buffer, and
    // the next stage has landed.  From there to the next barrier the loads of the stage RING further go out into this buffer, spread between the
    // products (in a row they fill the queue of the address unit and the products behind them wait), and the next stage's first operands are
    // read: the matrix cores wait for nothing but the waves' skew at the barrier.
    // Products of a stage, counted from the barrier, that loads go out behind: with two buffers the first half, since the next barrier waits for them (2048 x 4096 x 4096
    // 82.9 -> 81.8 us, 8192 x 8192 x 4096 on these tiles 546 -> 517).
    constexpr int SLOTS = NKS * TM * TN / (T::RING == 2 ? 2 : 1);
    constexpr int EARLY = (TM * TN * LOADS + SLOTS - 1) / SLOTS;  // loads of the step behind the barrier
    {
      const int seg = MODE == DENSE_DX && first >= seg_stages ? 1 : 0;
      enter(seg, (long long)(first - seg * seg_stages) * DK);
      if (load_r + DK > p.red) last();
    }
#pragma unroll
    for (int it = 0; it < T::RING; ++it) {
      if (it) advance();
#pragma unroll
      for (int v = 0; v < (it == T::RING - 1 ? EARLY : LOADS); ++v) load(it * T::STAGE, v);
    }
    beside.ask(p, wm0, wn0, epilogue_whole<MODE, T::WTN, TM>(p, wm0, wn0));
    wait_barrier<(T::RING - 2) * LOADS + EARLY>();                // more loads behind those it counts only make it wait longer
#pragma unroll
    for (int f = 0; f < TM + TN; ++f) read(dense_smem, 0, f);
    int it = 0;
    unsigned at = 0, pat = (T::RING - 1) * T::STAGE;              // this stage's buffer, and the last one's
    do {                                                          // at least one stage
      const unsigned nat = at + T::STAGE < T::RING * T::STAGE ? at + T::STAGE : 0;
      const unsigned char *t = dense_smem + at, *next = dense_smem + nat;
      unrolled<NKS>([&](auto s) {
        constexpr int ks = decltype(s)::value;
        if constexpr (ks == NKS - 1) {
          advance();
          wait_barrier<(T::RING - 2) * LOADS>();
        }
#pragma unroll
        for (int q = 0; q < TM * TN; ++q) {
          constexpr int from = (ks + 1) % NKS * TM * TN;          // slot of q = 0
          product(ks, q);
          if (q < TM + TN) read(ks == NKS - 1 ? next : t, (ks + 1) % NKS, q);
#pragma unroll
          for (int v = 0; v < LOADS; ++v)
            if (v * SLOTS / LOADS == from + q) load(ks == NKS - 1 ? at : pat, v);
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (TM + TN > TM * TN)
#pragma unroll
          for (int f = TM * TN; f < TM + TN; ++f) read(ks == NKS - 1 ? next : t, (ks + 1) % NKS, f);
      });
      pat = at;
      at = nat;
    } while (++it < count);
    wait_loads();
  } else {
    pull(0);
    push(0);
    for (int it = 0; it < count; ++it) {
      __syncthreads();                                            // this stage is in LDS, and every wave is done with the other buffer
      if (it + 1 < count) pull(it + 1);
      multiply(it & 1);
      if (it + 1 < count) push(it + 1);
    }
  }
  __syncthreads();                                                // the buffers are free for the epilogue
  dense_epilogue<typename DenseKind<MODE>::Out, MODE, T::WTN, PRE>(p, acc, dense_smem + wave * T::EPI_WAVE, wm0, wn0, src, split, beside);
}

template <typename T, int MODE, bool DMA>
__global__ __launch_bounds__(T::NT, T::OCC) void dense_kernel(DenseP p) {
  const int job = dense_job(p);
  if (job >= 0) dense_tile<T, MODE, DMA>(p, job);
}
// Both products of a backward pass in one launch: of few tiles each, one after the other they leave most compute units idle twice.
template <typename T>
__global__ __launch_bounds__(T::NT, T::OCC) void dense_pair_kernel(DenseP dx, DenseP dw) {
  const int job = xcd_order(dx.ntiles + dw.ntiles);
  if (job < 0) return;
  if (job < dx.ntiles) dense_tile<T, DENSE_DX, true>(dx, job);
  else dense_tile<T, DENSE_DW, true>(dw, job - dx.ntiles);
}

// The 256 x 256 tile, one work-group on a compute unit, a wave on a SIMD.  Rows along the reduction arrive in whole 128-byte lines only if 64 of it are asked for at a time
// (half a line costs what the line costs), and two stages of 64 of both operands ahead are more than the LDS holds.  So each operand has a ring of its own:
// A three units of 64, B two.  One barrier a stage, in front of its last step, whose operands are in registers: there every wave is done with the stage's units.  Behind
// it the next unit of B goes out, spread over the last step and the first of the next stage, and has until that stage's barrier to land; in the two steps
// between goes the next unit of A, which has a stage more.
// TFLOP/s, 8192 x 65536 x 4096 forward, N(0,1): 1327; with rings of four units of 32 of both, two barriers for 64: 1259; A in three units of 64 and B in four of 32, two
// barriers: 1289; two units of 64 of both, whose last loads have no time to land: 1215; without loads 1660 (which bounds nothing else: operands that stay in the
// L2s gain 2 %).  At two stages the first products wait for memory and all compute units meet in their epilogues: 8192 x 8192 x 4096 1295.
struct Tile256 {
  static constexpr int DK = 64, BM = 256, BN = 256, NT = 256;
  static constexpr int UNIT = 256 * DK * 2, A_RING = 3, B_RING = 2, LDS_BYTES = (A_RING + B_RING) * UNIT;
  static_assert(LDS_BYTES == 163840 && LDS_BYTES >= 4 * epi_wave_bytes(128), "the LDS of a compute unit");
};

template <int MODE>
__global__ __launch_bounds__(256, 1) void dense_large_kernel(DenseP p) {
  typedef Tile256 T;
  constexpr bool A_FAST = MODE != DENSE_DW, B_FAST = dense_b_fast<MODE>();
  constexpr int DK = T::DK, BM = T::BM, BN = T::BN, TM = 4, TN = 4, NP = TM * TN, SUB = 128, OUT_N = MODE == DENSE_GATED ? 128 : 256;
  constexpr int V = T::UNIT / (16 * T::NT), B_AT = T::A_RING * T::UNIT;     // loads of a unit per thread; where B's ring begins
  typedef Operand<BM, A_FAST, SUB, DK> OpA;
  typedef Operand<BN, B_FAST, SUB, DK> OpB;
  extern __shared__ __attribute__((aligned(256))) unsigned char dense_smem[];

  const int job = dense_job(p);
  if (job < 0) return;
  const int split = job / p.ntiles;
  int tm, tn, src = 0;
  tile_at(p, job - split * p.ntiles, tm, tn);
  if (MODE == DENSE_DW && p.srcs == 2) {                          // columns of tiles of the one source, then of the other
    const int each = p.ntn / 2;
    src = tn >= each;
    tn -= src * each;
  }
  const long long m0 = (long long)tm * BM;
  const int n0 = tn * OUT_N;
  const int first = split * p.stages_per_split, count = p.stages - first < p.stages_per_split ? p.stages - first : p.stages_per_split;
  const int seg_stages = p.stages / p.segs;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;

  // ---- loads: a stream for each operand, as in dense_kernel ----
  const long long m_left = p.M - m0, n_left = (long long)p.N - n0;
  int a_e[V], a_r[V], b_e[V], b_r[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    OpA::where(tid + j * 256, a_e[j], a_r[j]);
    OpB::where(tid + j * 256, b_e[j], b_r[j]);
    if (MODE == DENSE_GATED) b_e[j] %= SUB;
  }
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)dense_smem + wave * 1024);
  unsigned a_off[V], b_off[V];
  v4u rs_a = {}, rs_b = {}, rs_u = {};
  int a_left = count, b_left = count;                             // units not asked for yet
  long long ar = 0, br = 0;                                       // reduction element of the next unit
  auto a_enter = [&](int seg, long long r) {
    ar = r;
    rs_a = buffer_rsrc((const uint16_t*)p.a[MODE == DENSE_DX ? seg : 0] + (A_FAST ? m0 * p.lda + r : r * p.lda + m0), 0x7fffffff);
#pragma unroll
    for (int j = 0; j < V; ++j)
      a_off[j] = a_e[j] < m_left && r + a_r[j] < p.red ? (unsigned)((A_FAST ? a_e[j] * p.lda + a_r[j] : a_r[j] * p.lda + a_e[j]) * 2) : DMA_OOB;
  };
  auto b_enter = [&](int seg, long long r) {
    br = r;
    const long long o = B_FAST ? n0 * p.ldb + r : r * p.ldb + n0;
    rs_b = buffer_rsrc((const uint16_t*)p.b[MODE == DENSE_DX ? seg : MODE == DENSE_DW ? src : 0] + o, 0x7fffffff);
    if (MODE == DENSE_GATED) rs_u = buffer_rsrc((const uint16_t*)p.b[1] + o, 0x7fffffff);
#pragma unroll
    for (int j = 0; j < V; ++j)
      b_off[j] = b_e[j] < n_left && r + b_r[j] < p.red ? (unsigned)((B_FAST ? b_e[j] * p.ldb + b_r[j] : b_r[j] * p.ldb + b_e[j]) * 2) : DMA_OOB;
  };
  auto move = [](v4u& rs, long long bytes) {
    const unsigned long long base = ((unsigned long long)rs[1] << 32 | rs[0]) + bytes;
    rs[0] = (unsigned)base;
    rs[1] = (unsigned)(base >> 32);
  };
  auto a_next = [&]() {
    if (--a_left <= 0) { rs_a[2] = 0; return; }                   // beyond the last: nothing but zeros
    ar += DK;
    if (MODE == DENSE_DX && ar >= p.red) a_enter(1, 0);
    else move(rs_a, (A_FAST ? DK : DK * p.lda) * 2);
    if (ar + DK > p.red)
#pragma unroll
      for (int j = 0; j < V; ++j) a_off[j] = ar + a_r[j] < p.red ? a_off[j] : DMA_OOB;
  };
  auto b_next = [&]() {
    if (--b_left <= 0) { rs_b[2] = rs_u[2] = 0; return; }
    br += DK;
    if (MODE == DENSE_DX && br >= p.red) b_enter(1, 0);
    else {
      move(rs_b, (B_FAST ? DK : DK * p.ldb) * 2);
      if (MODE == DENSE_GATED) move(rs_u, DK * p.ldb * 2);
    }
    if (br + DK > p.red)
#pragma unroll
      for (int j = 0; j < V; ++j) b_off[j] = br + b_r[j] < p.red ? b_off[j] : DMA_OOB;
  };
  auto a_load = [&](unsigned at, int v) { load_lds16(rs_a, lds0 + at + v * 4096, a_off[v], 0); };
  auto b_load = [&](unsigned at, int v) { load_lds16(MODE == DENSE_GATED && v >= V / 2 ? rs_u : rs_b, lds0 + B_AT + at + v * 4096, b_off[v], 0); };

  int a_rd[OpA::N], b_rd[OpB::N];
  OpA::template prepare<TM>(a_rd, lane, [&](int i) { return wm * 128 + i * 32; });
  OpB::template prepare<TN>(b_rd, lane, [&](int j) { return MODE == DENSE_GATED ? (j / 2) * SUB + (wn * 2 + j % 2) * 32 : wn * 128 + j * 32; });
  const long long wm0 = m0 + wm * 128;                            // the wave's first row and column
  const int wn0 = n0 + wn * (OUT_N / 2);
  Beside<MODE, 128, 2> beside;
  typename DenseKind<MODE>::Acc acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
  bf16x8 af[2][TM], bf[2][TN];                                    // operands are read one step ahead of their products
  auto read = [&](unsigned a, unsigned b, int ks, int f) {        // fragment f of step ks; a, b: the units
    if (f < TN) bf[ks & 1][f] = OpB::fragment(dense_smem + B_AT + b + OpB::address(b_rd, f, ks));
    else af[ks & 1][f - TN] = OpA::fragment(dense_smem + a + OpA::address(a_rd, f - TN, ks));
  };
  // step ks: products, the reads of the next step's operands (a, b: their units), and four loads, from load(l) on, one every four products
  auto step = [&](auto ks_c, unsigned a, unsigned b, auto l_c, auto&& load) {
    constexpr int ks = decltype(ks_c)::value, l = decltype(l_c)::value;
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      acc[q / TN][q % TN] = DenseKind<MODE>::product(bf[ks & 1][q % TN], af[ks & 1][q / TN], acc[q / TN][q % TN]);
      if (q < TM + TN) read(a, b, (ks + 1) % 4, q);
      if (q % 4 == 0) load(l + q / 4);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  static_assert(DK == 64 && V == 8, "four steps a stage, of four loads each");
  const std::integral_constant<int, 0> c0{};
  const std::integral_constant<int, 1> c1{};
  const std::integral_constant<int, 2> c2{};
  const std::integral_constant<int, 3> c3{};
  const std::integral_constant<int, 4> c4{};

  {
    const int seg = MODE == DENSE_DX && first >= seg_stages ? 1 : 0;
    a_enter(seg, (long long)(first - seg * seg_stages) * DK);
    b_enter(seg, (long long)(first - seg * seg_stages) * DK);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) a_load(0, v);
  a_next();
#pragma unroll
  for (int v = 0; v < V; ++v) b_load(0, v);
  b_next();
#pragma unroll
  for (int v = 0; v < V; ++v) a_load(T::UNIT, v);
  a_next();
  unsigned a = 0, b = 0;                                          // this stage's units
  unsigned a_fill = 2 * T::UNIT, b_fill = T::UNIT;                // the units that loads go to
  auto a_fills = [&](int l) { a_load(a_fill, l); };
  auto b_fills = [&](int l) { b_load(b_fill, l); };
#pragma unroll
  for (int l = 0; l < 4; ++l) b_fills(l);
  beside.ask(p, wm0, wn0, epilogue_whole<MODE, 128, TM>(p, wm0, wn0));
  wait_barrier<12>();                                             // unit 0 of each has landed: behind them are unit 1 of A, half of unit 1 of B, and the residuals, which only make it wait longer
#pragma unroll
  for (int f = 0; f < TM + TN; ++f) read(0, 0, 0, f);
  int left = count;                                               // at least one stage
  do {
    const unsigned an = a + T::UNIT < T::A_RING * T::UNIT ? a + T::UNIT : 0u, bn = b ? 0u : (unsigned)T::UNIT;
    step(c0, a, b, c4, b_fills);
    step(c1, a, b, c0, a_fills);
    step(c2, a, b, c4, a_fills);
    a_next();
    b_next();
    a_fill = a;
    b_fill = b;
    wait_barrier<8>();                                            // the unit of A just asked for may be in flight
    step(c3, an, bn, c0, b_fills);
    a = an;
    b = bn;
  } while (--left > 0);
  wait_loads();
  __syncthreads();                                                // the rings are free for the epilogue
  dense_epilogue<typename DenseKind<MODE>::Out, MODE, 128, 2>(p, acc, dense_smem + wave * epi_wave_bytes(128), wm0, wn0, src, split, beside);
}

// Tiles and stages of a product; false: more than an int numbers.
template <typename T, int MODE>
bool dense_grid(DenseP& p) {
  p.stages = (int)((p.red + T::DK - 1) / T::DK) * p.segs;
  p.stages_per_split = (p.stages + p.splits - 1) / p.splits;
  p.splits = (p.stages + p.stages_per_split - 1) / p.stages_per_split;      // none without a stage
  const int out_n = MODE == DENSE_GATED ? T::BN / 2 : T::BN;
  const long long tm = (p.M + T::BM - 1) / T::BM, tn = (long long)((p.N + out_n - 1) / out_n) * (MODE == DENSE_DW ? p.srcs : 1);
  if (tm * tn * p.splits > 0x7fffff00LL) return false;
  p.ntm = (int)tm;
  p.ntn = (int)tn;
  p.ntiles = (int)(tm * tn);
  return true;
}

template <int MODE>
hipError_t launch_large(DenseP& p, hipStream_t s) {
  typedef Tile256 T;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(dense_large_kernel<MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
  if (attr != hipSuccess) return attr;
  if (!dense_grid<T, MODE>(p)) return hipErrorInvalidValue;
  return launch_jobs<T::NT>(p, [&](dim3 grid) { hipLaunchKernelGGL((dense_large_kernel<MODE>), grid, dim3(T::NT), T::LDS_BYTES, s, p); });
}

template <typename T, int MODE, bool DMA>
hipError_t launch_dense(DenseP& p, hipStream_t s) {
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(dense_kernel<T, MODE, DMA>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
  if (attr != hipSuccess) return attr;
  if (!dense_grid<T, MODE>(p)) return hipErrorInvalidValue;
  return launch_jobs<T::NT>(p, [&](dim3 grid) { hipLaunchKernelGGL((dense_kernel<T, MODE, DMA>), grid, dim3(T::NT), T::LDS_BYTES, s, p); });
}

// Deep rings hide what a stage takes to arrive where there is one work-group on a compute unit; two work-groups hide each other's.
typedef DenseTile<128, 128, 64, 2> Tile128;
typedef DenseTile<128, 128, 64, 5> Tile128D;
typedef DenseTile<64, 128, 64, 3> Tile64x128;
typedef DenseTile<64, 64, 64, 5> Tile64;
typedef DenseTile<32, 128, 64, 4, 1, 4> Tile32;
enum { TILE_256, TILE_128, TILE_128D, TILE_64X128, TILE_64, TILE_32 };

// Tile and splits of a reduction, from the sizes alone (workspaces are planned before there are addresses), by an estimate of the time: rounds of work-groups
// through the compute units, stages of 64 of the reduction each, and for splits the join's launch (5 us: 3 on the device, and the host's; 0.15 a split) and its passes over the sums (4 TB/s).  us of a stage, measured
// where a work-group is alone on its compute unit and where all units hold as many as they can (forward, bf16, rows x inputs x outputs):
//                  alone            full
//   256 x 256      1.62             1.62     8192 x 65536 x 4096
//   128 x 128      0.86 (one stage ahead)   1.10     64 x 4096 x 4096, 2048 x 4096 x 4096
//   the same, deep 0.50             0.65     1024 x 2048 x 4096
//   64 x 128       0.48             0.80     512 x 4096 x 4096, 1024 x 2048 x 4096
//   64 x 64        0.33             0.52     64 x 4096 x 4096, 512 x 4096 x 4096
//   32 x 128       0.38             0.62
// Beside its stages a tile costs its first loads and its epilogue: 1 or 2 us where another work-group on the unit covers the rest, but with 256 x 256, where all units
// write 128 KB each at a time, more: LARGE_FIXED, with a residual for the forward product (us, 256 x 256 / 128 x 128: 4096 x 512 x 4096 29 / 25, 4096 x 1024 x 4096 44 / 39, 4096 x 2048 x 4096 69 / 81; 7493 x 960 x 13760, SiLU,
// residual 326 / 244).
// us by tile and splits, of which it takes the starred:
//                         128 x 128: 1    2      4      8     deep: 1  2      4     64 x 128: 1  2     4      64 x 64: 1  2      4
//   24 x 2048 x 8192             30.9   21.3   15.7   16.7    18.9   16.1   14.9       18.8   15.8   13.9       14.3   14.6   15.5   (32 x 128, 4: 13.9*)
//   256 x 2048 x 2048            26.0   17.8   14.9   16.9    19.9   15.6   14.1       16.3   13.9   13.4       12.8*  12.7   13.6
//   512 x 4096 x 4096            61.8   42.2   39.2   51.2    42.9   34.2   43.9       36.0*  39.1   47.1       40.6   47.9   56.1
//   1024 x 2048 x 4096           36.2   38.4   52.7   83.4    27.5*  44.3   62.7       31.2   45.9   61.8       40.0   54.1   70.5
//   2048 x 4096 x 4096           79.5*  107    137    192     85.8   118    164        102    129    148        129    153    173
struct DensePlan { int tile, splits; };
struct TileCost { int tile, bm, bn, per_cu; double alone, full, fixed; };
constexpr TileCost COSTS[] = {{TILE_256, 256, 256, 1, 1.62, 1.62, 0.0}, {TILE_128, 128, 128, 2, 0.86, 1.10, 2.0}, {TILE_128D, 128, 128, 1, 0.50, 0.65, 2.0},
                              {TILE_64X128, 64, 128, 2, 0.48, 0.80, 1.0}, {TILE_64, 64, 64, 2, 0.33, 0.52, 1.0}, {TILE_32, 32, 128, 2, 0.38, 0.62, 1.0}};

constexpr double LARGE_FIXED[] = {20.0, 15.0, 8.0, 5.0, 20.0, 20.0};     // DENSE_FWD, GATED, DX, DW, Q8, Q8_F32

constexpr int MAX_SPLITS = 48;

DensePlan dense_plan(int mode, long long M, int N, long long red, int segs, int srcs) {
  const long long stages = (red + 63) / 64 * segs;
  DensePlan best = {TILE_128, 1};
  double least = 1e300;
  for (const TileCost& t : COSTS) {
    if (mode == DENSE_GATED && (t.tile == TILE_64 || t.tile == TILE_32)) continue;     // a wave needs columns of both sources
    const int out_n = mode == DENSE_GATED ? t.bn / 2 : t.bn;
    const long long tiles = (M + t.bm - 1) / t.bm * ((N + out_n - 1) / out_n) * (mode == DENSE_DW ? srcs : 1), slots = 256LL * t.per_cu;
    const double fixed = t.tile == TILE_256 ? LARGE_FIXED[mode] : t.fixed;
    for (int splits = 1; splits <= MAX_SPLITS; ++splits) {
      const long long per = (stages + splits - 1) / splits, jobs = tiles * splits, rounds = jobs / slots, rest = jobs - rounds * slots;
      if (splits > 1 && per < 2) break;
      double us = rounds * (per * t.full + fixed) + (rest == 0 ? 0.0 : per * (rest > 256 ? t.full : t.alone) + fixed);
      if (splits > 1) us += 5.0 + splits * (0.15 + (double)M * N * srcs * 2e-6);
      if (us < least) { least = us; best = {t.tile, splits}; }
    }
  }
  return best;
}

// Loads that write LDS need whole 16-byte vectors: addresses and pitches in multiples of 8 elements, and lengths too, since a vector across the end of a row
// would bring in what lies behind it.  32-bit offsets within a tile bound the pitch.
bool dma_ok(int mode, const DenseP& p) {
  uintptr_t at = (uintptr_t)p.a[0] | (uintptr_t)p.b[0];
  if (p.segs == 2) at |= (uintptr_t)p.a[1];
  if (p.segs == 2 || p.srcs == 2) at |= (uintptr_t)p.b[1];
  const long long a_len = mode == DENSE_DW ? p.M : p.red, b_len = mode == DENSE_DX || dense_q8(mode) ? p.red : p.N;
  return (at & 15) == 0 && ((p.lda | p.ldb | a_len | b_len) & 7) == 0 && p.lda < (1 << 21) && p.ldb < (1 << 21);
}

// What cannot go by those loads takes the plan's splits, for which the workspace was sized, on one of two tiles through registers: the plan's costs are not theirs.
template <int MODE>
hipError_t dense_mode(DenseP& p, hipStream_t s) {
  const DensePlan plan = dense_plan(MODE, p.M, p.N, p.red, p.segs, p.srcs);
  p.splits = plan.splits;
  hipError_t e;
  const auto at_any_address = [&]() {
    if constexpr (dense_q8(MODE)) return hipErrorInvalidValue;    // never: the layout of its operands is the library's
    else return plan.tile <= TILE_128D ? launch_dense<Tile128, MODE, false>(p, s) : launch_dense<Tile64x128, MODE, false>(p, s);
  };
  if (!dma_ok(MODE, p)) e = at_any_address();
  else if (plan.tile == TILE_256) e = launch_large<MODE>(p, s);
  else if (plan.tile == TILE_128) e = launch_dense<Tile128, MODE, true>(p, s);
  else if (plan.tile == TILE_128D) e = launch_dense<Tile128D, MODE, true>(p, s);
  else if constexpr (MODE == DENSE_GATED) e = launch_dense<Tile64x128, MODE, true>(p, s);
  else if (plan.tile == TILE_64X128) e = launch_dense<Tile64x128, MODE, true>(p, s);
  else if (plan.tile == TILE_64) e = launch_dense<Tile64, MODE, true>(p, s);
  else e = launch_dense<Tile32, MODE, true>(p, s);
  return e == hipSuccess && p.splits > 1 ? dense_join(MODE, false, p, s) : e;
}

}  // namespace

// dx and dw together where both take 64 x 64 tiles and do not split; taken: whether they were.
hipError_t dense_bf16_pair(DenseP& dx, DenseP& dw, bool& taken, hipStream_t s) {
  typedef Tile64 T;
  const DensePlan a = dense_plan(DENSE_DX, dx.M, dx.N, dx.red, dx.segs, dx.srcs), b = dense_plan(DENSE_DW, dw.M, dw.N, dw.red, dw.segs, dw.srcs);
  taken = false;
  if (a.tile != TILE_64 || b.tile != TILE_64 || a.splits != 1 || b.splits != 1 || !dma_ok(DENSE_DX, dx) || !dma_ok(DENSE_DW, dw)) return hipSuccess;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(dense_pair_kernel<T>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
  if (attr != hipSuccess) return attr;
  dx.splits = dw.splits = 1;
  if (!dense_grid<T, DENSE_DX>(dx) || !dense_grid<T, DENSE_DW>(dw)) return hipErrorInvalidValue;
  if ((long long)dx.ntiles + dw.ntiles > (1LL << 31) / T::NT) return hipSuccess;     // more than one grid holds
  taken = true;
  hipLaunchKernelGGL((dense_pair_kernel<T>), dim3((unsigned)xcd_grid((long long)dx.ntiles + dw.ntiles)), dim3(T::NT), T::LDS_BYTES, s, dx, dw);
  return hipGetLastError();
}

hipError_t dense_bf16(int mode, DenseP& p, hipStream_t s) {
  switch (mode) {
    case DENSE_FWD: return dense_mode<DENSE_FWD>(p, s);
    case DENSE_GATED: return dense_mode<DENSE_GATED>(p, s);
    case DENSE_DX: return dense_mode<DENSE_DX>(p, s);
    case DENSE_Q8: return dense_mode<DENSE_Q8>(p, s);
    case DENSE_Q8_F32: return dense_mode<DENSE_Q8_F32>(p, s);
    default: return dense_mode<DENSE_DW>(p, s);
  }
}

uint64_t dense_bf16_ws(int mode, long long M, int N, long long red, int segs, int srcs) {
  const int splits = dense_plan(mode, M, N, red, segs, srcs).splits;
  return splits > 1 ? (uint64_t)splits * srcs * M * N * 4 : 0;
}

}  // namespace lms
