// Linear layer and gated feed-forward projection: what lms_linear_* and lms_gated_* launch, and the passes beside their matrix products.
#include <hip/hip_runtime.h>

#include "dense.hpp"
#include "graph.hpp"
#include "kernels.hpp"

namespace lms {

namespace {

// ---- gradients that enter the products, and column sums ----
//
// A work-group takes a chunk of 32 rows (more where there are many, so that the chunks' sums stay small) of 512 columns, eight columns a thread: each input is read once, the gradient is written once in the storage type, and
// the columns' sums over the work-group's rows, of the values before rounding, go to part[chunk of rows][n].  sum_rows adds the chunks in order.
// The rounding to bf16 is the price of products on the bf16 matrix cores: dx and dw of a layer with an activation are 0.0023 from the exact result (relative norm) where
// their own rounding alone is 0.0017.  Carrying the rest of each value as a second bf16 operand would restore that and double the products (8192 x 4096 x 4096: 435 of 483 us).
constexpr int PT = 256, PC = 512, LANES = PC / 8, WAYS = PT / LANES;
int chunk_rows(long long m) {
  int rows = 32;
  while (rows < 1024 && m > 2048LL * rows) rows *= 2;
  return rows;
}

struct GradP {
  const void *d, *g, *u;       // gradient that comes in; linear: g = pre; gated: g and u
  void *dz, *du;
  float* part;                 // or null
  long long M, ldd, ldo;       // ldd: d, g, u; ldo: dz, du
  int N, act, gated, rows;     // rows: of a chunk
};

template <typename T>
__global__ __launch_bounds__(PT) void act_grad_kernel(GradP p) {
  __shared__ float sums[WAYS][PC];
  const int across = (p.N + PC - 1) / PC, chunk = blockIdx.x / across, c0 = (int)(blockIdx.x % across) * PC;
  const int c = (threadIdx.x % LANES) * 8, way = threadIdx.x / LANES, n = c0 + c, cnt = p.N - n < 8 ? p.N - n : 8;
  const long long r0 = (long long)chunk * p.rows;
  float total[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  constexpr int U = 4;                                            // rows in flight
  auto rows = [&](auto gated_c, auto slope_c) {                   // what is read: d; g; g and u
    constexpr bool GATED = decltype(gated_c)::value, SLOPE = decltype(slope_c)::value;
    for (int r = way; r < p.rows && r0 + r < p.M; r += WAYS * U) {
      Raw<T, 8> d[U], g[SLOPE ? U : 1], u[GATED ? U : 1];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const long long row = r0 + r + k * WAYS, at = (row < p.M ? row : r0 + r) * p.ldd + n;       // rows beyond the last: one that is there, for nothing
        d[k] = raw<8>((const T*)p.d + at, cnt);
        if constexpr (SLOPE) g[k] = raw<8>((const T*)p.g + at, cnt);
        if constexpr (GATED) u[k] = raw<8>((const T*)p.u + at, cnt);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const long long row = r0 + r + k * WAYS;
        if (row >= p.M) break;
        float dv[8], gv[8], uv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dv[e] = d[k].get(e);
          if constexpr (SLOPE) gv[e] = g[k].get(e);
          if constexpr (GATED) uv[e] = u[k].get(e);
          else uv[e] = 1.f;
        }
        if constexpr (SLOPE) {
          gated_grad8(p.act, dv, gv, uv);
          store8((T*)p.dz + row * p.ldo + n, cnt, gv);
          if constexpr (GATED) store8((T*)p.du + row * p.ldo + n, cnt, uv);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) total[e] += SLOPE ? gv[e] : dv[e];
      }
    }
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (cnt > 0) {
    if (p.gated) rows(yes, yes);
    else if (p.g) rows(no, yes);
    else rows(no, no);
  }
  if (!p.part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[way][c + e] = total[e];
  __syncthreads();
  for (int i = threadIdx.x; i < PC; i += PT)
    if (c0 + i < p.N) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < WAYS; ++w) t += sums[w][i];
      p.part[(long long)chunk * p.N + c0 + i] = t;
    }
}

// out[n] = sum over the chunks of part[chunk][n], in order, for the columns from n0 on
__global__ __launch_bounds__(PT) void sum_rows_kernel(const float* part, long long chunks, int N, int n0, float* out) {
  __shared__ float sums[8][32];
  const int c = threadIdx.x & 31, way = threadIdx.x >> 5, n = n0 + (int)blockIdx.x * 32 + c;
  float t = 0.f;
  if (n < N) {
    long long i = way;
    for (; i + 24 < chunks; i += 32) {
      float v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = part[(i + 8 * u) * N + n];
      t += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; i < chunks; i += 8) t += part[i * N + n];
  }
  sums[way][c] = t;
  __syncthreads();
  if (way == 0 && n < N) {
#pragma unroll
    for (int w = 1; w < 8; ++w) t += sums[w][c];
    out[n] = t;
  }
}

__global__ __launch_bounds__(PT) void zero_kernel(uint16_t* p, long long ld, int N, long long rows, int halves) {
  for (long long i = (long long)blockIdx.x * PT + threadIdx.x; i < rows * N; i += (long long)gridDim.x * PT)
    for (int h = 0; h < halves; ++h) p[(i / N * ld + i % N) * halves + h] = 0;
}

hipError_t act_grad(bool f32, GradP& p, float* sums, hipStream_t s) {
  p.rows = chunk_rows(p.M);
  const long long chunks = (p.M + p.rows - 1) / p.rows;
  const long long groups = chunks * ((p.N + PC - 1) / PC);
  if (groups >= (1LL << 32) / PT) return hipErrorInvalidValue;    // a grid holds less than 2^32 threads; this many have more rows and columns than fit the device's memory
  const dim3 grid((unsigned)groups);
  if (f32) hipLaunchKernelGGL(act_grad_kernel<float>, grid, dim3(PT), 0, s, p);
  else hipLaunchKernelGGL(act_grad_kernel<uint16_t>, grid, dim3(PT), 0, s, p);
  if (sums)
    for (int n0 = 0; n0 < p.N; n0 += 1 << 28)                     // 2^23 work-groups
      hipLaunchKernelGGL(sum_rows_kernel, dim3((unsigned)(((p.N - n0 < 1 << 28 ? p.N - n0 : 1 << 28) + 31) / 32)), dim3(PT), 0, s, p.part, chunks, p.N, n0, sums);
  return hipGetLastError();
}

hipError_t fill_zero(void* out, long long rows, int N, long long ld, bool f32, hipStream_t s) {
  const long long groups = (rows * N + PT - 1) / PT;
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(groups < 1 << 20 ? groups : 1 << 20)), dim3(PT), 0, s, (uint16_t*)out, ld, N, rows, f32 ? 2 : 1);
  return hipGetLastError();
}

// ---- what the two descriptors have in common ----
struct Layer {
  long long m, ldx, ldw, ldy, ldr;
  int n, k, act, srcs;
  bool f32, w32;
};

constexpr uint64_t WS_ALIGN = 256;
uint64_t up(uint64_t b) { return (b + WS_ALIGN - 1) / WS_ALIGN * WS_ALIGN; }
long long grad_pitch(int n) { return (n + 7) / 8 * 8; }
uint64_t grad_bytes(const Layer& l) { return up((uint64_t)l.m * grad_pitch(l.n) * (l.f32 ? 4 : 2)); }
uint64_t chunk_bytes(const Layer& l) { return up((uint64_t)((l.m + chunk_rows(l.m) - 1) / chunk_rows(l.m)) * l.n * 4); }

#define NEED(cond, ...)        \
  do {                         \
    if (!(cond)) {             \
      set_error(__VA_ARGS__);  \
      return LMS_EINVAL;       \
    }                          \
  } while (0)

lms_status check(const char* what, const Layer& l, int dtype, int wgrad_dtype) {
  NEED(l.m >= 0 && l.n >= 1 && l.k >= 1, "%s: rows must be >= 0, widths >= 1", what);
  NEED(l.m <= 0x7fffffffLL, "%s: more than 2^31 - 1 rows", what);
  NEED(l.n <= 1 << 30 && l.k <= 1 << 30, "%s: widths above 2^30", what);
  NEED(l.act >= LMS_ACT_NONE && l.act <= LMS_ACT_GELU_TANH, "%s: unknown activation %d", what, l.act);
  NEED(dtype == LMS_BF16 || dtype == LMS_F32, "%s: dtype must be LMS_BF16 or LMS_F32", what);
  NEED(wgrad_dtype == LMS_F32 || wgrad_dtype == dtype, "%s: wgrad_dtype must be LMS_F32 or the dtype", what);
  NEED(l.ldx >= l.k && l.ldw >= l.n && l.ldy >= l.n && l.ldr >= l.n, "%s: a row pitch is shorter than the row", what);
  const long long most = 1LL << 40;
  NEED(l.ldx <= most && l.ldw <= most && l.ldy <= most && l.ldr <= most, "%s: a row pitch is above 2^40", what);
  return LMS_OK;
}

lms_status linear_layer(const lms_linear_desc* d, Layer& l) {
  l = Layer{d->m, d->ldx ? d->ldx : d->k, d->ldw ? d->ldw : d->n, d->ldy ? d->ldy : d->n, d->ldr ? d->ldr : d->n, d->n, d->k, d->act, 1,
            d->dtype == LMS_F32, d->wgrad_dtype == LMS_F32};
  return check("lms_linear", l, d->dtype, d->wgrad_dtype);
}
lms_status gated_layer(const lms_gated_desc* d, Layer& l) {
  const long long ldh = d->ldh ? d->ldh : d->f;
  l = Layer{d->m, d->ldx ? d->ldx : d->k, d->ldw ? d->ldw : d->f, ldh, ldh, d->f, d->k, d->act, 2, d->dtype == LMS_F32, d->wgrad_dtype == LMS_F32};
  return check("lms_gated", l, d->dtype, d->wgrad_dtype);
}

lms_status aligned(const char* what, const Layer& l, const void* const* p, int count) {
  const uintptr_t low = l.f32 ? 3 : 1;
  for (int i = 0; i < count; ++i) NEED(((uintptr_t)p[i] & low) == 0, "%s: a pointer is not aligned to its elements", what);
  return LMS_OK;
}
// what a call's workspace holds besides nothing
lms_status space(const char* what, uint64_t need, const void* ws) {
  NEED(!need || ws, "%s: workspace of %llu bytes required", what, (unsigned long long)need);
  NEED(((uintptr_t)ws & 15) == 0, "%s: the workspace is not aligned", what);
  return LMS_OK;
}
lms_status done(const char* what, hipError_t e) {
  if (e == hipSuccess) return LMS_OK;
  set_error("%s: %s", what, hipGetErrorString(e));
  return LMS_EHIP;
}

// dx = sum over sources of dz_s w_s^T; dw_s = x^T dz_s
hipError_t layer_grads(const Layer& l, const void* const* dz, long long ldz, const void* x, const void* const* w, void* dx, void* const* dw, float* part, hipStream_t s) {
  DenseP px{}, pw{};
  if (dx) {
    for (int i = 0; i < l.srcs; ++i) { px.a[i] = dz[i]; px.b[i] = w[i]; }
    px.out[0] = dx;
    px.M = l.m; px.N = l.k; px.red = l.n;
    px.lda = ldz; px.ldb = l.ldw; px.ldo = l.ldx;
    px.segs = l.srcs; px.srcs = 1;
    px.part = part;
  }
  if (dw[0]) {
    pw.a[0] = x;
    for (int i = 0; i < l.srcs; ++i) { pw.b[i] = dz[i]; pw.out[i] = dw[i]; }
    pw.M = l.k; pw.N = l.n; pw.red = l.m;
    pw.lda = l.ldx; pw.ldb = ldz; pw.ldo = l.ldw;
    pw.segs = 1; pw.srcs = l.srcs;
    pw.out_f32 = l.w32;
    pw.part = part;
  }
  hipError_t e = hipSuccess;
  if (dx && dw[0] && !l.f32) {
    bool taken;
    e = dense_bf16_pair(px, pw, taken, s);
    if (taken || e != hipSuccess) return e;
  }
  if (dx) e = dense_product(DENSE_DX, l.f32, px, s);
  if (e == hipSuccess && dw[0]) e = dense_product(DENSE_DW, l.f32, pw, s);
  return e;
}

uint64_t grads_ws(const Layer& l, bool dx, bool dw) {
  const uint64_t a = dx ? dense_ws(DENSE_DX, l.f32, l.m, l.k, l.n, l.srcs, 1) : 0, b = dw ? dense_ws(DENSE_DW, l.f32, l.k, l.n, l.m, 1, l.srcs) : 0;
  return up(a > b ? a : b);
}

}  // namespace

uint64_t dense_ws(int mode, bool f32, long long M, int N, long long red, int segs, int srcs) {
  if (dense_few_ok(mode, f32, M)) return dense_few_ws(mode, f32, M, N, red);
  return f32 ? dense_f32_ws(mode, M, N, red, segs, srcs) : dense_bf16_ws(mode, M, N, red, segs, srcs);
}
hipError_t dense_product(int mode, bool f32, DenseP& p, hipStream_t s) {
  if (dense_few_ok(mode, f32, p.M)) return dense_few(mode, f32, p, s);
  return f32 ? dense_f32(mode, p, s) : dense_bf16(mode, p, s);
}

lms_status linear_workspace(const lms_linear_desc* d, int which, uint64_t* bytes) {
  Layer l;
  if (const lms_status st = linear_layer(d, l)) return st;
  NEED(which == LMS_LINEAR_FWD || which == LMS_LINEAR_BWD, "lms_linear_workspace_bytes: unknown call %d", which);
  if (which == LMS_LINEAR_FWD) *bytes = up(dense_ws(DENSE_FWD, l.f32, l.m, l.n, l.k, 1, 1));
  else *bytes = (l.act != LMS_ACT_NONE ? grad_bytes(l) : 0) + chunk_bytes(l) + grads_ws(l, true, true);
  return LMS_OK;
}

lms_status linear_fwd(const lms_linear_desc* d, const void* x, const void* w, const float* bias, const void* res, void* y, void* pre, void* ws, void* stream) {
  Layer l;
  if (const lms_status st = linear_layer(d, l)) return st;
  const void* all[] = {x, w, res, y, pre};
  if (const lms_status st = aligned("lms_linear_fwd", l, all, 5)) return st;
  NEED(((uintptr_t)bias & 3) == 0, "lms_linear_fwd: bias is not aligned to its elements");
  NEED(res != y || l.ldr == l.ldy, "lms_linear_fwd: res may be y only with the same pitch");
  if (l.m == 0) return LMS_OK;
  uint64_t need = 0;
  linear_workspace(d, LMS_LINEAR_FWD, &need);
  if (const lms_status st = space("lms_linear_fwd", need, ws)) return st;
  DenseP p{};
  p.a[0] = x; p.b[0] = w; p.out[0] = y;
  p.bias = bias; p.res = res; p.pre = pre;
  p.M = l.m; p.N = l.n; p.red = l.k;
  p.lda = l.ldx; p.ldb = l.ldw; p.ldo = l.ldy; p.ldr = l.ldr;
  p.segs = 1; p.srcs = 1; p.act = l.act;
  p.part = (float*)ws;
  return done("lms_linear_fwd", dense_product(DENSE_FWD, l.f32, p, (hipStream_t)stream));
}

lms_status linear_bwd(const lms_linear_desc* d, const void* dy, const void* x, const void* w, const void* pre, void* dx, void* dw, float* db, void* ws,
                      void* stream) {
  Layer l;
  if (const lms_status st = linear_layer(d, l)) return st;
  NEED(l.m == 0 || ((!dx || w) && (!dw || x)), "lms_linear_bwd: dx needs w, dw needs x");
  NEED(l.m == 0 || l.act == LMS_ACT_NONE || pre, "lms_linear_bwd: a layer with an activation needs pre");
  const void* all[] = {dy, x, w, pre, dx, dw};
  if (const lms_status st = aligned("lms_linear_bwd", l, all, 6)) return st;
  NEED((((uintptr_t)db | (l.w32 ? (uintptr_t)dw : 0)) & 3) == 0, "lms_linear_bwd: dw or dbias is not aligned to its elements");
  hipStream_t s = (hipStream_t)stream;
  if (l.m == 0) {
    hipError_t e = hipSuccess;
    if (dw) e = fill_zero(dw, l.k, l.n, l.ldw, l.w32, s);
    if (e == hipSuccess && db) e = fill_zero(db, 1, l.n, l.n, true, s);
    return done("lms_linear_bwd", e);
  }
  uint64_t need = 0;
  linear_workspace(d, LMS_LINEAR_BWD, &need);
  if (const lms_status st = space("lms_linear_bwd", need, ws)) return st;
  const bool with_act = l.act != LMS_ACT_NONE;
  const void* dz = dy;
  long long ldz = l.ldy;
  char* at = (char*)ws;
  hipError_t e = hipSuccess;
  if (with_act || db) {
    GradP g{};
    g.d = dy; g.g = with_act ? pre : nullptr;
    g.M = l.m; g.N = l.n; g.act = l.act; g.ldd = l.ldy;
    if (with_act) {
      g.dz = at;
      g.ldo = ldz = grad_pitch(l.n);
      dz = at;
      at += grad_bytes(l);
    }
    if (db) { g.part = (float*)at; at += chunk_bytes(l); }
    e = act_grad(l.f32, g, db, s);
  }
  if (e == hipSuccess) {
    const void* const dzs[] = {dz};
    const void* const wsrc[] = {w};
    void* const dws[] = {dw};
    e = layer_grads(l, dzs, ldz, x, wsrc, dx, dws, (float*)at, s);
  }
  return done("lms_linear_bwd", e);
}

lms_status gated_workspace(const lms_gated_desc* d, int which, uint64_t* bytes) {
  Layer l;
  if (const lms_status st = gated_layer(d, l)) return st;
  NEED(which >= LMS_GATED_FWD && which <= LMS_GATED_BWD_RECOMPUTE, "lms_gated_workspace_bytes: unknown call %d", which);
  const uint64_t fwd = up(dense_ws(DENSE_GATED, l.f32, l.m, l.n, l.k, 1, 2)), grads = grads_ws(l, true, true);
  if (which == LMS_GATED_FWD) *bytes = fwd;
  else *bytes = 2 * grad_bytes(l) + (which == LMS_GATED_BWD_RECOMPUTE && fwd > grads ? fwd : grads);
  return LMS_OK;
}

lms_status gated_fwd(const lms_gated_desc* d, const void* x, const void* wg, const void* wu, void* h, void* g, void* u, void* ws, void* stream) {
  Layer l;
  if (const lms_status st = gated_layer(d, l)) return st;
  const void* all[] = {x, wg, wu, h, g, u};
  if (const lms_status st = aligned("lms_gated_fwd", l, all, 6)) return st;
  if (l.m == 0) return LMS_OK;
  uint64_t need = 0;
  gated_workspace(d, LMS_GATED_FWD, &need);
  if (const lms_status st = space("lms_gated_fwd", need, ws)) return st;
  DenseP p{};
  p.a[0] = x; p.b[0] = wg; p.b[1] = wu; p.out[0] = h;
  p.pre = g; p.pre1 = u;
  p.M = l.m; p.N = l.n; p.red = l.k;
  p.lda = l.ldx; p.ldb = l.ldw; p.ldo = l.ldy; p.ldr = l.ldy;
  p.segs = 1; p.srcs = 2; p.act = l.act;
  p.part = (float*)ws;
  return done("lms_gated_fwd", dense_product(DENSE_GATED, l.f32, p, (hipStream_t)stream));
}

lms_status gated_bwd(const lms_gated_desc* d, const void* dh, const void* x, const void* wg, const void* wu, const void* g, const void* u, void* dx, void* dwg,
                     void* dwu, void* ws, void* stream) {
  Layer l;
  if (const lms_status st = gated_layer(d, l)) return st;
  NEED(!g == !u, "lms_gated_bwd: g and u are both given or both NULL");
  NEED(!dwg == !dwu, "lms_gated_bwd: dwg and dwu are both given or both NULL");
  NEED(l.m == 0 || (wg && wu) || (g && !dx), "lms_gated_bwd: wg and wu are needed for dx, and where g and u are not given");
  NEED(l.m == 0 || x || (g && !dwg), "lms_gated_bwd: x is needed for dwg and dwu, and where g and u are not given");
  const void* all[] = {dh, x, wg, wu, g, u, dx, dwg, dwu};
  if (const lms_status st = aligned("lms_gated_bwd", l, all, 9)) return st;
  NEED(!l.w32 || (((uintptr_t)dwg | (uintptr_t)dwu) & 3) == 0, "lms_gated_bwd: dwg or dwu is not aligned to its elements");
  hipStream_t s = (hipStream_t)stream;
  if (l.m == 0) {
    hipError_t e = hipSuccess;
    if (dwg) e = fill_zero(dwg, l.k, l.n, l.ldw, l.w32, s);
    if (dwu && e == hipSuccess) e = fill_zero(dwu, l.k, l.n, l.ldw, l.w32, s);
    return done("lms_gated_bwd", e);
  }
  uint64_t need = 0;
  gated_workspace(d, g ? LMS_GATED_BWD : LMS_GATED_BWD_RECOMPUTE, &need);
  if (const lms_status st = space("lms_gated_bwd", need, ws)) return st;
  char* at = (char*)ws;
  const long long ldz = grad_pitch(l.n);
  const void* const dz[] = {at, at + grad_bytes(l)};
  hipError_t e;
  if (g) {
    GradP q{};
    q.d = dh; q.g = g; q.u = u;
    q.dz = at; q.du = at + grad_bytes(l);
    q.M = l.m; q.N = l.n; q.act = l.act; q.gated = 1; q.ldd = l.ldy; q.ldo = ldz;
    e = act_grad(l.f32, q, nullptr, s);
  } else {
    DenseP p{};
    p.a[0] = x; p.b[0] = wg; p.b[1] = wu;
    p.dh = dh; p.out[0] = at; p.pre1 = at + grad_bytes(l);
    p.M = l.m; p.N = l.n; p.red = l.k;
    p.lda = l.ldx; p.ldb = l.ldw; p.ldo = ldz; p.ldr = l.ldy;
    p.segs = 1; p.srcs = 2; p.act = l.act;
    p.part = (float*)(at + 2 * grad_bytes(l));
    e = dense_product(DENSE_GATED, l.f32, p, s);
  }
  if (e == hipSuccess) {
    const void* const w[] = {wg, wu};
    void* const dw[] = {dwg, dwu};
    e = layer_grads(l, dz, ldz, x, w, dx, dw, (float*)(at + 2 * grad_bytes(l)), s);
  }
  return done("lms_gated_bwd", e);
}

}  // namespace lms
