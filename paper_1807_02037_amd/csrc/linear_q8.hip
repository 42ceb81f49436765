// Linear layer in 8-bit integers: rows of x and columns of w as whole numbers from -127 to 127 with a scale each (include/lms.h has the formulas).
//
// Both operands of the product lie with the reduction in rows of whole 16-byte vectors, zeros behind the last element: the weights are turned once, x as it is quantised.  In bytes the
// product is then that of two bf16 matrices whose reductions lie in rows, and it runs on the same tiles (dense_gemm.hip); up to 64 rows have kernels of their own, which read the weights in one round.
// us: 8192 rows, 8192 -> 4096, residual: rows 45 (201 MB at 4.4 TB/s), product 265 to 300 as the clock goes (1.8 to 2.1 P/s; operands of zeros 199); 24 rows, 2048 -> 8192: 3 and 6.
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "conv_dma.hpp"
#include "kernels.hpp"
#include "rows4.hpp"

namespace lms {

namespace {

constexpr int MAX_K = 1 << 17;         // 127^2 of them stay below 2^31

// The whole number nearest to 127 x / most, ties to even.  bf16: 127 x is exact, and the quotient of 15 by 8 bits is either a tie, which a float holds, or further from one
// than its rounding.  fp32: the same in fp64.  Values of more than 2^119 are scaled first, which is exact where it matters (x above most / 254).
template <typename T>
__device__ __forceinline__ int step_of(float x, float most) {
  if constexpr (sizeof(T) == 2) {
    const float s = most > 0x1p119f ? 0x1p-8f : 1.f;
    return (int)__builtin_rintf((127.f * (x * s)) / (most * s));
  } else return (int)__builtin_rint(127.0 * (double)x / (double)most);
}
// The scale of values whose largest magnitude has these bits: NaN where one of them is not finite, and then all steps are 0.
__device__ __forceinline__ float scale_of(unsigned bits) { return bits >= 0x7f800000u ? __builtin_nanf("") : __uint_as_float(bits) / 127.f; }
__device__ __forceinline__ bool steps(unsigned bits) { return bits != 0u && bits < 0x7f800000u; }

__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// NT threads a row, which hold it in NV vectors of eight each, or, with NV = 0, read it twice.
template <typename T, int NT, int NV>
__global__ __launch_bounds__(NT) void q8_rows_kernel(const T* x, long long ldx, int k, int kp, signed char* xq, float* sx, long long row0) {
  __shared__ unsigned s_most[NT / 64];
  const long long row = row0 + blockIdx.x;
  const T* from = x + row * ldx;
  signed char* to = xq + row * kp;
  const int tid = threadIdx.x;
  Raw<T, 8> held[NV > 0 ? NV : 1];
  unsigned most = 0;
  auto each = [&](auto&& f) {
    if constexpr (NV > 0)
#pragma unroll
      for (int v = 0; v < NV; ++v) f(v, (tid + v * NT) * 8);
    else
      for (int c = tid * 8; c < kp; c += NT * 8) f(0, c);
  };
  each([&](int v, int c) { if (NV > 0) held[v] = raw<8>(from + c, c < k ? k - c : 0); });
  each([&](int v, int c) {
    if constexpr (NV == 0) held[0] = raw<8>(from + c, c < k ? k - c : 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned m = magnitude_bits(held[v].get(e));
      most = most > m ? most : m;
    }
  });
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const unsigned m = __shfl_xor(most, d);
    most = most > m ? most : m;
  }
  if constexpr (NT > 64) {
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) most = most > s_most[w] ? most : s_most[w];
  }
  if (tid == 0) sx[row] = scale_of(most);
  const float top = __uint_as_float(most);
  const bool some = steps(most);
  each([&](int v, int c) {
    if (c >= kp) return;
    if constexpr (NV == 0) held[0] = raw<8>(from + c, c < k ? k - c : 0);
    unsigned q[2] = {0u, 0u};
    if (some)
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e >> 2] |= (unsigned)(step_of<T>(held[v].get(e), top) & 255) << (8 * (e & 3));
    __builtin_memcpy(to + c, q, 8);
  });
}

// ---- few rows ----
//
// Bound by reading the weights once.  A wave takes CW columns, its lanes consecutive 16 bytes of the reduction, and has eight loads of weights in flight before anything else happens; the rows of x lie
// in LDS, 4-byte dot products go to whole sums of each lane, and the lanes meet by shuffles: whole numbers, in any order the same.  FUSED: every work-group quantises the rows itself,
// while its weights are on their way, instead of waiting for another launch.  One row, 4096 -> 4096, us in a graph: 5.5 with the same weights again, 7.0 with two sets by turns, 8.4 with weights from memory (2.0 TB/s).  (Products of 32 x 32 x 32 with both operands straight from memory, for 9 to
// 32 rows, took 10.1 us at 24 x 2048 -> 8192 and 58 at 32 x 8192 -> 16384: half a line of each column a load is what the address unit is slow at.)
constexpr int FT = 512, FEW_LDS = 65536 - 256;      // with what the kernel has besides, no more than any launch may have

template <int ACT>
__device__ __forceinline__ float act_value(float v) {
  float value, slope;
  act_one<ACT>(v, value, slope);
  return value;
}

// Sums over the wave of N values of each lane: the i-th in the lanes from 64 / N i on.  Each exchange halves the values that a lane holds: N - 1 of them and the rest of six, where sums one by one take 6 N.
template <int N>
__device__ __forceinline__ int lanes_sum(int (&v)[N]) {
  const int lane = threadIdx.x & 63;
  int d = 32;
#pragma unroll
  for (int half = N / 2; half >= 1; half /= 2, d /= 2) {
    const bool upper = lane & d;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const int keep = upper ? v[i + half] : v[i], give = upper ? v[i] : v[i + half];
      v[i] = keep + __shfl_xor(give, d);
    }
  }
  for (; d >= 1; d /= 2) v[0] += __shfl_xor(v[0], d);
  return v[0];
}

template <typename T, int R, int CW, bool FUSED>
__global__ __launch_bounds__(FT) void q8_few_kernel(DenseP p, const T* x, long long ldx, int k, int kp) {
  constexpr int S = 8 / CW;                                       // loads of a column in flight
  extern __shared__ __attribute__((aligned(16))) signed char s_x[];           // R rows of kp steps
  __shared__ unsigned s_most[R][FT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rows = (int)p.M;
  const int waves = (int)gridDim.x * (FT / 64);
  const signed char* wq = (const signed char*)p.b[0];
  v4u w[CW][S];
  auto ask = [&](int col, int k0) {
#pragma unroll
    for (int j = 0; j < CW; ++j)
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int at = k0 + s * 1024 + lane * 16;
        w[j][s] = v4u{0u, 0u, 0u, 0u};
        if (col + j < p.N && at < kp) w[j][s] = *reinterpret_cast<const v4u*>(wq + (long long)(col + j) * kp + at);
      }
  };
  int col = ((int)blockIdx.x * (FT / 64) + wave) * CW;
  ask(col, 0);
  float sx[R];
  if constexpr (FUSED) {
    constexpr int HELD = 2;
    Raw<T, 8> held[R][HELD];
    unsigned most[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int v = 0; v < HELD; ++v) {
        const int c = (tid + v * FT) * 8;
        held[r][v] = raw<8>(x + (r < rows ? r : 0) * ldx + c, c < k ? k - c : 0);
      }
    auto vec = [&](int r, int v) -> Raw<T, 8> {                   // any vector of a row
      const int c = (tid + v * FT) * 8;
      return raw<8>(x + (r < rows ? r : 0) * ldx + c, c < k ? k - c : 0);
    };
    auto largest = [](unsigned m, const Raw<T, 8>& q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned b = magnitude_bits(q.get(e));
        m = m > b ? m : b;
      }
      return m;
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      most[r] = 0;
#pragma unroll
      for (int v = 0; v < HELD; ++v) most[r] = largest(most[r], held[r][v]);
      for (int v = HELD; v * FT * 8 < kp; ++v) most[r] = largest(most[r], vec(r, v));
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        const unsigned m = __shfl_xor(most[r], d);
        most[r] = most[r] > m ? most[r] : m;
      }
      if (lane == 0) s_most[r][wave] = most[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int i = 0; i < FT / 64; ++i) most[r] = most[r] > s_most[r][i] ? most[r] : s_most[r][i];
      sx[r] = scale_of(most[r]);
      const float top = __uint_as_float(most[r]);
      const bool some = steps(most[r]);
      auto put = [&](int v, const Raw<T, 8>& d) {
        const int c = (tid + v * FT) * 8;
        if (c >= kp) return;
        unsigned q[2] = {0u, 0u};
        if (some)
#pragma unroll
          for (int e = 0; e < 8; ++e) q[e >> 2] |= (unsigned)(step_of<T>(d.get(e), top) & 255) << (8 * (e & 3));
        __builtin_memcpy(s_x + r * kp + c, q, 8);
      };
#pragma unroll
      for (int v = 0; v < HELD; ++v) put(v, held[r][v]);
      for (int v = HELD; v * FT * 8 < kp; ++v) put(v, vec(r, v));
    }
  } else {
    const signed char* xq = (const signed char*)p.a[0];
    for (int i = tid * 16; i < R * kp; i += FT * 16) {
      const int r = i / kp;
      *reinterpret_cast<v4u*>(s_x + i) = *reinterpret_cast<const v4u*>(xq + (long long)(r < rows ? i : i - r * kp));      // rows that are not there: the first
    }
#pragma unroll
    for (int r = 0; r < R; ++r) sx[r] = p.sx[r < rows ? r : 0];
  }
  __syncthreads();
  while (col < p.N) {                                             // uniform in a wave
    int acc[CW][R] = {};
    for (int k0 = 0;;) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int at = k0 + s * 1024 + lane * 16;
        if (at < kp)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const v4u d = *reinterpret_cast<const v4u*>(s_x + r * kp + at);
#pragma unroll
            for (int j = 0; j < CW; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[j][r] = __builtin_amdgcn_sdot4((int)d[i], (int)w[j][s][i], acc[j][r], false);
          }
      }
      k0 += S * 1024;
      if (k0 >= kp) break;
      ask(col, k0);
    }
    const int done = col;
    col += waves * CW;
    if (col < p.N) ask(col, 0);
    constexpr int N = CW * R, SHARE = 64 / N;                     // outputs of the wave; lanes of one: output r CW + j is that of the lanes from (r CW + j) SHARE on
    int all[N];
#pragma unroll
    for (int j = 0; j < CW; ++j)
#pragma unroll
      for (int r = 0; r < R; ++r) all[r * CW + j] = acc[j][r];
    const int mine = lanes_sum<N>(all), r = lane / SHARE / CW, n = done + lane / SHARE % CW;
    if (lane % SHARE == 0 && r < rows && n < p.N) {
      float s = sx[0];
#pragma unroll
      for (int i = 1; i < R; ++i) s = r == i ? sx[i] : s;
      float v = q8_scaled(mine, s, p.sw[n]);
      if (p.bias) v += p.bias[n];
      with_act(p.act, [&](auto act) { v = act_value<decltype(act)::value>(v); });
      if constexpr (sizeof(T) == 2) {
        if (p.res) v += bf2f(((const T*)p.res)[r * p.ldr + n]);
        ((T*)p.out[0])[r * p.ldo + n] = f2bf(v);
      } else {
        if (p.res) v += ((const T*)p.res)[r * p.ldr + n];
        ((T*)p.out[0])[r * p.ldo + n] = v;
      }
    }
  }
}

// ---- some rows ----
//
// ROWS rows and C columns a work-group, its four waves in turn 128 bytes of the reduction each, a whole line of every row and column, straight to LDS.  Each wave has a ring of DEPTH such
// stages for itself and waits for nobody: no barrier before the waves' sums meet.
constexpr int MT = 256, LINE = 128;
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef int v4i __attribute__((ext_vector_type(4)));
constexpr int some_ring(int rows, int c, int depth) { return 4 * depth * (rows + c) * LINE; }

template <typename T, int ROWS, int C, int DEPTH>
__global__ __launch_bounds__(MT) void q8_some_kernel(DenseP p, int kp) {
  constexpr int LA = ROWS / 8, LOADS = LA + C / 8, STAGE = (ROWS + C) * LINE, PITCH = C + 4;       // LA: loads of rows
  constexpr int R = ROWS / C, STEPS = C == 32 ? 4 : 2, PARTS = 8 / STEPS;                          // products of C x C by PARTS pieces of 16 bytes
  static_assert(some_ring(ROWS, C, DEPTH) >= 4 * ROWS * PITCH * 4 && (DEPTH - 1) * LOADS < 64, "the waves' sums take the rings' place; vmcnt has six bits");
  typedef std::conditional_t<C == 32, i32x16, v4i> Acc;
  constexpr int VALUES = sizeof(Acc) / 4;
  extern __shared__ __attribute__((aligned(1024))) unsigned char s_ring[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), rows = (int)p.M, n0 = blockIdx.x * C;
  const int lines = (kp + LINE - 1) / LINE, count = (lines + 3) / 4;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)s_ring + wave * DEPTH * STAGE);
  const v4u rs_a = buffer_rsrc(p.a[0], 0x7fffffff), rs_b = buffer_rsrc((const signed char*)p.b[0] + (long long)n0 * kp, 0x7fffffff);
  // eight rows of a line a load; a row's 16-byte pieces lie in an order of its own, so that the reads of many rows' same piece meet all banks
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
  unsigned off[LOADS];
#pragma unroll
  for (int v = 0; v < LOADS; ++v) {
    const int row = (v < LA ? v : v - LA) * 8 + (lane >> 3);
    off[v] = row < (v < LA ? rows : p.N - n0) ? (unsigned)(row * kp + piece) : DMA_OOB;
  }
  auto ask = [&](int it) __attribute__((always_inline)) {
    const unsigned at = lds0 + it % DEPTH * STAGE, k0 = (it * 4 + wave) * LINE;
    const bool whole = (int)k0 + LINE <= kp, have = (int)k0 + piece < kp;     // beyond the end: zeros
    if (whole) {
#pragma unroll
      for (int v = 0; v < LOADS; ++v) load_lds16(v < LA ? rs_a : rs_b, at + v * 1024, off[v], k0);
    } else {
#pragma unroll
      for (int v = 0; v < LOADS; ++v) load_lds16(v < LA ? rs_a : rs_b, at + v * 1024, have ? off[v] : DMA_OOB, k0);
    }
  };
  const int quad = tid % (C / 4) * 4, cnt = p.N - n0 - quad;
  float sw[V], bias[V] = {};
  load4(p.sw + n0 + quad, cnt, sw);
  if (p.bias) load4(p.bias + n0 + quad, cnt, bias);
#pragma unroll
  for (int it = 0; it < DEPTH; ++it) ask(it);
  Acc acc[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int v = 0; v < VALUES; ++v) acc[r][v] = 0;
  int read[STEPS];
#pragma unroll
  for (int ks = 0; ks < STEPS; ++ks) read[ks] = wave * DEPTH * STAGE + lane % C * LINE + ((ks * PARTS + lane / C) ^ (lane & 7)) * 16;
  for (int it = 0; it < count; ++it) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * LOADS) : "memory");
    const unsigned char* t = s_ring + it % DEPTH * STAGE;
    v4i a[R][STEPS], b[STEPS];
#pragma unroll
    for (int ks = 0; ks < STEPS; ++ks) {
      b[ks] = *reinterpret_cast<const v4i*>(t + read[ks] + ROWS * LINE);
#pragma unroll
      for (int r = 0; r < R; ++r) a[r][ks] = *reinterpret_cast<const v4i*>(t + read[ks] + r * C * LINE);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // this stage's place is free
    ask(it + DEPTH);
#pragma unroll
    for (int ks = 0; ks < STEPS; ++ks)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (C == 32) acc[r] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[ks], a[r][ks], acc[r], 0, 0, 0);
        else acc[r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[ks], a[r][ks], acc[r], 0, 0, 0);
      }
  }
  wait_loads();
  __syncthreads();
  int* const sums = reinterpret_cast<int*>(s_ring);               // [wave][row][column], from the transposed accumulators: lane l has row l % C, columns 4 (l / C) + v % 4, 8 further for each four of v
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int v = 0; v < VALUES / 4; ++v)
      *reinterpret_cast<v4i*>(sums + (wave * ROWS + r * C + lane % C) * PITCH + 8 * v + 4 * (lane / C)) = v4i{acc[r][4 * v], acc[r][4 * v + 1], acc[r][4 * v + 2], acc[r][4 * v + 3]};
  __syncthreads();
  constexpr int EACH = MT / (C / 4);                              // rows at a time
  const int n = n0 + quad;
#pragma unroll
  for (int i0 = 0; i0 < ROWS; i0 += EACH) {
    const int i = i0 + tid / (C / 4);
    if (i >= rows || i >= ROWS || cnt <= 0) continue;
    v4i sum = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += *reinterpret_cast<const v4i*>(sums + (w * ROWS + i) * PITCH + quad);
    const float s = p.sx[i];
    float y[V], beside[V] = {};
    if (p.res) {
      const Raw<T, V> q = raw<V>((const T*)p.res + i * p.ldr + n, cnt);
#pragma unroll
      for (int e = 0; e < V; ++e) beside[e] = q.get(e);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] = q8_scaled(sum[e], s, sw[e]) + bias[e];
    with_act(p.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] = act_value<decltype(act)::value>(y[e]);
    });
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] += beside[e];
    store4((T*)p.out[0] + i * p.ldo + n, cnt, y);
  }
}

// ---- weights, laid out once ----
//
// Columns' largest magnitudes meet in sw as bits, by a maximum whose order does not matter; then tiles are turned through LDS; then the bits become scales.
__global__ __launch_bounds__(256) void q8_clear_kernel(unsigned* most, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) most[i] = 0;
}
__global__ __launch_bounds__(256) void q8_scales_kernel(float* sw, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) sw[i] = scale_of(__float_as_uint(sw[i]));
}

constexpr int WROWS = 256;             // of the reduction, a work-group
constexpr int WBLOCKS = 1 << 14;       // blocks of columns of a launch

template <typename T>
__device__ __forceinline__ float element(const T* p) {
  if constexpr (sizeof(T) == 2) return bf2f(*p);
  else return *p;
}
// 256 columns, eight a thread
template <typename T>
__global__ __launch_bounds__(256) void q8_columns_kernel(const T* w, long long ldw, int n, int k, unsigned* sw, int block0) {
  __shared__ unsigned s_most[8][256];
  const int c = (threadIdx.x & 31) * 8, way = threadIdx.x >> 5, j = (block0 + (int)blockIdx.x) * 256 + c, r0 = blockIdx.y * WROWS, cnt = n - j;
  unsigned most[8] = {};
  if (cnt > 0)
#pragma unroll 4
    for (int r = r0 + way; r < r0 + WROWS; r += 8) {
      const Raw<T, 8> v = raw<8>(w + (long long)(r < k ? r : r0) * ldw + j, cnt);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned m = magnitude_bits(v.get(e));
        most[e] = most[e] > m ? most[e] : m;
      }
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) s_most[way][c + e] = most[e];
  __syncthreads();
  const int col = (block0 + (int)blockIdx.x) * 256 + threadIdx.x;
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = m > s_most[i][threadIdx.x] ? m : s_most[i][threadIdx.x];
  if (col < n) atomicMax(sw + col, m);
}
template <typename T>
__global__ __launch_bounds__(256) void q8_turn_kernel(const T* w, long long ldw, int n, int k, int kp, signed char* wq, const unsigned* sw, int block0) {
  __shared__ int s_q[64][65];
  const int c0 = (block0 + (int)blockIdx.x) * 64, col = threadIdx.x & 63, way = threadIdx.x >> 6, j = c0 + col;
  const unsigned most = j < n ? sw[j] : 0u;
  const float top = __uint_as_float(most);
  const bool some = steps(most);
  for (int r0 = blockIdx.y * WROWS; r0 < (int)(blockIdx.y + 1) * WROWS && r0 < kp; r0 += 64) {
    __syncthreads();
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = r0 + way + 4 * i;
      v[i] = some && r < k ? element(w + (long long)r * ldw + j) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s_q[way + 4 * i][col] = some ? step_of<T>(v[i], top) : 0;
    __syncthreads();
    const int row = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;          // 16 steps of one column
    if (c0 + row < n && r0 + part < kp) {
      unsigned q[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < 16; ++e) q[e >> 2] |= (unsigned)(s_q[part + e][row] & 255) << (8 * (e & 3));
      __builtin_memcpy(wq + (long long)(c0 + row) * kp + r0 + part, q, 16);
    }
  }
}

int pitch(const lms_linear_q8_desc* d) { return (d->k + 15) / 16 * 16; }

template <typename T>
hipError_t lay_out(const lms_linear_q8_desc* d, const T* w, signed char* wq, float* sw, hipStream_t s) {
  const int kp = pitch(d), n = d->n, deep = (kp + WROWS - 1) / WROWS;
  const long long ldw = d->ldw ? d->ldw : d->n;
  const dim3 flat((unsigned)((n + 255) / 256));
  auto blocks = [&](int width, auto&& launch) {
    const int all = (n + width - 1) / width;
    for (int b = 0; b < all; b += WBLOCKS) launch(dim3((unsigned)(all - b < WBLOCKS ? all - b : WBLOCKS), (unsigned)deep), b);
  };
  hipLaunchKernelGGL(q8_clear_kernel, flat, dim3(256), 0, s, (unsigned*)sw, n);
  blocks(256, [&](dim3 grid, int b) { hipLaunchKernelGGL(q8_columns_kernel<T>, grid, dim3(256), 0, s, w, ldw, n, d->k, (unsigned*)sw, b); });
  blocks(64, [&](dim3 grid, int b) { hipLaunchKernelGGL(q8_turn_kernel<T>, grid, dim3(256), 0, s, w, ldw, n, d->k, kp, wq, (const unsigned*)sw, b); });
  hipLaunchKernelGGL(q8_scales_kernel, flat, dim3(256), 0, s, sw, n);
  return hipGetLastError();
}

template <typename T>
hipError_t quantise(const lms_linear_q8_desc* d, const T* x, signed char* xq, float* sx, hipStream_t s) {
  const int kp = pitch(d);
  const long long ldx = d->ldx ? d->ldx : d->k;
  auto go = [&](auto nt, auto nv) {
    constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
    constexpr long long most = (1LL << 31) / NT;
    for (long long r = 0; r < d->m; r += most) {
      hipLaunchKernelGGL((q8_rows_kernel<T, NT, NV>), dim3((unsigned)(d->m - r < most ? d->m - r : most)), dim3(NT), 0, s, x, ldx, d->k, kp, xq, sx, r);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
#define ROWS(NT, NV) if (kp <= NT * 8 * NV) return go(std::integral_constant<int, NT>{}, std::integral_constant<int, NV>{})
  ROWS(64, 1);
  ROWS(256, 1);
  ROWS(256, 2);
  ROWS(256, 4);
  ROWS(1024, 4);
#undef ROWS
  return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 0>{});
}

// One or two rows that fit the LDS.  From three on products of many rows, whose two launches then cost less than the dot products (us, the same weights again, dot products / those: 4096 -> 4096 one row 5.8 / 8, two 7.2 / 8.3,
// four 9.4 / 8.6; 2048 -> 8192 four rows 10.7 / 7.6; 8192 -> 16384 four rows 31.6 / 31.8).
bool few_rows(const lms_linear_q8_desc* d) { return d->m >= 1 && d->m <= 2 && d->m * pitch(d) <= FEW_LDS; }

template <typename T, int R, bool FUSED>
hipError_t few(const lms_linear_q8_desc* d, DenseP& p, const T* x, hipStream_t s) {
  const int kp = pitch(d), steps = (kp + 1023) / 1024;
  auto go = [&](auto cw) {
    constexpr int CW = decltype(cw)::value;
    const long long need = ((long long)d->n + CW * (FT / 64) - 1) / (CW * (FT / 64));
    hipLaunchKernelGGL((q8_few_kernel<T, R, CW, FUSED>), dim3((unsigned)(need < 512 ? need : 512)), dim3(FT), R * kp, s, p, x, d->ldx ? d->ldx : (long long)d->k, d->k, kp);
    return hipGetLastError();
  };
  if (steps >= 8) return go(std::integral_constant<int, 1>{});
  if (steps >= 3) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}
template <typename T>
hipError_t few_product(const lms_linear_q8_desc* d, DenseP& p, const void* x, hipStream_t s) {
  const T* t = (const T*)x;
  if (d->m == 1) return x ? few<T, 1, true>(d, p, t, s) : few<T, 1, false>(d, p, t, s);
  return x ? few<T, 2, true>(d, p, t, s) : few<T, 2, false>(d, p, t, s);
}

template <typename T, int ROWS, int C, int DEPTH>
hipError_t some(const lms_linear_q8_desc* d, DenseP& p, hipStream_t s) {
  constexpr int ring = some_ring(ROWS, C, DEPTH);
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(q8_some_kernel<T, ROWS, C, DEPTH>), hipFuncAttributeMaxDynamicSharedMemorySize, ring);
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((q8_some_kernel<T, ROWS, C, DEPTH>), dim3((unsigned)((d->n + C - 1) / C)), dim3(MT), ring, s, p, pitch(d));
  return hipGetLastError();
}
// Where one round of work-groups takes all columns, and a wave has few enough stages one after the other that the tiles' splits with their join cost more.  us, tiles / this, with the rows' launch of 3:
//   rows                       3             24            64                                    3             32            64
//   1024 -> 1024        7.7 / 6.1     8.4 / 6.5     8.0 / 7.0      4096 -> 6000      13.4 / 9.7    14.3 / 10.3   15.3 / 12.2
//   4096 -> 4096       11.3 / 8.4    12.4 / 9.6    13.8 / 11.6     8192 -> 8192      20.7 / 18.8   21.6 / 21.3   22.9 / 22.7
//   2048 -> 8192       10.2 / 7.5    10.9 / 8.1    10.7 / 9.7      12000 -> 4096     19.0 / 15.5   20.7 / 18.3   21.4 / 24.5
//   8192 -> 2048       12.7 / 10.7   13.5 / 11.3   14.8 / 14.2     16384 -> 8192     32.8 / 35.7   33.6 / 38.8   43.5 / 41.8
bool some_rows(const lms_linear_q8_desc* d) { return d->m >= 3 && d->m <= 64 && d->n <= 256 * 32 && pitch(d) <= (d->m <= 32 ? 12288 : 8192); }
template <typename T>
hipError_t some_product(const lms_linear_q8_desc* d, DenseP& p, hipStream_t s) {
  if (d->n > 256 * 16) return d->m > 32 ? some<T, 64, 32, 3>(d, p, s) : some<T, 32, 32, 4>(d, p, s);
  return d->m > 32 ? some<T, 64, 16, 3>(d, p, s) : some<T, 32, 16, 5>(d, p, s);
}

uint64_t rows_bytes(const lms_linear_q8_desc* d) { return up256((uint64_t)d->m * pitch(d)); }
uint64_t scale_bytes(const lms_linear_q8_desc* d) { return up256((uint64_t)d->m * 4); }
int mode_of(const lms_linear_q8_desc* d) { return d->dtype == LMS_F32 ? DENSE_Q8_F32 : DENSE_Q8; }
uint64_t product_bytes(const lms_linear_q8_desc* d) { return few_rows(d) || some_rows(d) ? 0 : up256(dense_bf16_ws(mode_of(d), d->m, d->n, pitch(d) / 2, 1, 1)); }

lms_status check(const char* what, const lms_linear_q8_desc* d) {
  NEED(d->m >= 0 && d->n >= 1 && d->k >= 1, "%s: rows must be >= 0, widths >= 1", what);
  NEED(d->m <= 0x7fffffffLL, "%s: more than 2^31 - 1 rows", what);
  NEED(d->n <= 1 << 30, "%s: widths above 2^30", what);
  NEED(d->k <= MAX_K, "%s: more than 2^17 inputs", what);
  NEED(d->act >= LMS_ACT_NONE && d->act <= LMS_ACT_GELU_TANH, "%s: unknown activation %d", what, d->act);
  NEED(d->dtype == LMS_BF16 || d->dtype == LMS_F32, "%s: dtype must be LMS_BF16 or LMS_F32", what);
  const long long most = 1LL << 40, ldx = d->ldx ? d->ldx : d->k, ldw = d->ldw ? d->ldw : d->n, ldy = d->ldy ? d->ldy : d->n, ldr = d->ldr ? d->ldr : d->n;
  NEED(ldx >= d->k && ldw >= d->n && ldy >= d->n && ldr >= d->n, "%s: a row pitch is shorter than the row", what);
  NEED(ldx <= most && ldw <= most && ldy <= most && ldr <= most, "%s: a row pitch is above 2^40", what);
  return LMS_OK;
}
lms_status aligned(const char* what, const lms_linear_q8_desc* d, std::initializer_list<const void*> rows, std::initializer_list<const void*> words, std::initializer_list<const void*> vectors) {
  uintptr_t a = 0, b = 0, c = 0;
  for (const void* q : rows) a |= (uintptr_t)q;
  for (const void* q : words) b |= (uintptr_t)q;
  for (const void* q : vectors) c |= (uintptr_t)q;
  NEED((a & (d->dtype == LMS_F32 ? 3 : 1)) == 0 && (b & 3) == 0, "%s: a pointer is not aligned to its elements", what);
  NEED((c & 15) == 0, "%s: 8-bit rows and the workspace must be aligned to 16 bytes", what);
  return LMS_OK;
}

// x: the rows themselves where there are few, then no xq
hipError_t product(const lms_linear_q8_desc* d, const void* x, const void* xq, const float* sx, const void* wq, const float* sw, const float* bias, const void* res, void* y, void* ws, hipStream_t s) {
  DenseP p{};
  p.a[0] = xq; p.b[0] = wq; p.out[0] = y;
  p.sx = sx; p.sw = sw; p.bias = bias; p.res = res;
  p.M = d->m; p.N = d->n; p.red = pitch(d) / 2;
  p.lda = p.ldb = pitch(d) / 2;
  p.ldo = d->ldy ? d->ldy : d->n;
  p.ldr = d->ldr ? d->ldr : d->n;
  p.segs = 1; p.srcs = 1; p.act = d->act;
  p.part = (float*)ws;
  if (few_rows(d)) return d->dtype == LMS_F32 ? few_product<float>(d, p, x, s) : few_product<uint16_t>(d, p, x, s);
  if (some_rows(d)) return d->dtype == LMS_F32 ? some_product<float>(d, p, s) : some_product<uint16_t>(d, p, s);
  return dense_bf16(mode_of(d), p, s);
}

}  // namespace

lms_status linear_q8_weight_size(const lms_linear_q8_desc* d, uint64_t* bytes) {
  if (const lms_status st = check("lms_linear_q8_weight_bytes", d)) return st;
  *bytes = (uint64_t)d->n * pitch(d);
  return LMS_OK;
}
lms_status linear_q8_workspace(const lms_linear_q8_desc* d, uint64_t* bytes) {
  if (const lms_status st = check("lms_linear_q8_workspace_bytes", d)) return st;
  *bytes = d->m == 0 ? 0 : rows_bytes(d) + scale_bytes(d) + product_bytes(d);
  return LMS_OK;
}

lms_status linear_q8_weight(const lms_linear_q8_desc* d, const void* w, void* wq, float* sw, void* stream) {
  const char* what = "lms_linear_q8_weight";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {w}, {sw}, {wq})) return st;
  hipStream_t s = (hipStream_t)stream;
  return done(what, d->dtype == LMS_F32 ? lay_out<float>(d, (const float*)w, (signed char*)wq, sw, s) : lay_out<uint16_t>(d, (const uint16_t*)w, (signed char*)wq, sw, s));
}

lms_status linear_q8_rows(const lms_linear_q8_desc* d, const void* x, void* xq, float* sx, void* stream) {
  const char* what = "lms_linear_q8_rows";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {x}, {sx}, {xq})) return st;
  hipStream_t s = (hipStream_t)stream;
  return done(what, d->dtype == LMS_F32 ? quantise<float>(d, (const float*)x, (signed char*)xq, sx, s) : quantise<uint16_t>(d, (const uint16_t*)x, (signed char*)xq, sx, s));
}

lms_status linear_q8_product(const lms_linear_q8_desc* d, const void* xq, const float* sx, const void* wq, const float* sw, const float* bias, const void* res, void* y, void* ws,
                             void* stream) {
  const char* what = "lms_linear_q8_product";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {res, y}, {sx, sw, bias}, {xq, wq, ws})) return st;
  NEED(res != y || (d->ldr ? d->ldr : d->n) == (d->ldy ? d->ldy : d->n), "%s: res may be y only with the same pitch", what);
  if (d->m == 0) return LMS_OK;
  NEED(ws || product_bytes(d) == 0, "%s: workspace of %llu bytes required", what, (unsigned long long)product_bytes(d));
  return done(what, product(d, nullptr, xq, sx, wq, sw, bias, res, y, ws, (hipStream_t)stream));
}

lms_status linear_q8_fwd(const lms_linear_q8_desc* d, const void* x, const void* wq, const float* sw, const float* bias, const void* res, void* y, void* ws, void* stream) {
  const char* what = "lms_linear_q8_fwd";
  if (const lms_status st = check(what, d)) return st;
  if (const lms_status st = aligned(what, d, {x, res, y}, {sw, bias}, {wq, ws})) return st;
  NEED(res != y || (d->ldr ? d->ldr : d->n) == (d->ldy ? d->ldy : d->n), "%s: res may be y only with the same pitch", what);
  if (d->m == 0) return LMS_OK;
  NEED(ws, "%s: workspace required", what);
  char* at = (char*)ws;
  float* sx = (float*)(at + rows_bytes(d));
  hipStream_t s = (hipStream_t)stream;
  if (few_rows(d)) return done(what, product(d, x, nullptr, nullptr, wq, sw, bias, res, y, nullptr, s));
  hipError_t e = d->dtype == LMS_F32 ? quantise<float>(d, (const float*)x, (signed char*)at, sx, s) : quantise<uint16_t>(d, (const uint16_t*)x, (signed char*)at, sx, s);
  if (e == hipSuccess) e = product(d, nullptr, at, sx, wq, sw, bias, res, y, at + rows_bytes(d) + scale_bytes(d), s);
  return done(what, e);
}

}  // namespace lms
