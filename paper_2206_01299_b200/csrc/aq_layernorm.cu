// Layer norm of rows, with the residual's addition, and the gradient.
//
//   s = x + residual (rounded to T, as it is stored),  mean = mean s,  rstd = 1 / sqrt(mean (s - mean)^2 + eps)
//   y = (s - mean) rstd w + b
// and with n = (s - mean) rstd, g = dy w:
//   dx = rstd (g - mean g - n mean(g n)) + dsum,   dw = sum over rows of dy n,   db = sum over rows of dy
//
// Bound by memory: two or four T per element forward, three or four backward.  A row stays in registers between its first and its
// last use, so the variance is that of the differences from the mean (no cancellation), and every operand is read once.
//
// Forward: rows up to 2048 elements of 16 bits belong to a warp, which needs no barrier; wider ones to a CTA.
// Backward: a CTA of as many threads as a row has 16-byte pieces (rows of one warp: eight of them) walks over the rows, a thread
// always at the same columns, whose sums of dw and db it keeps in registers; a CTA's sums go to a workspace, which a second
// kernel adds up in a fixed order.  Rows that are not whole 16-byte pieces, or wider than a CTA holds, go through kernels that
// read them again instead.

#include "aq_stage.h"
#include "aq_stage_device.cuh"

namespace aq {
namespace {

// A lane's piece of a row: 16 bytes, or one element where rows are not whole 16-byte pieces.
template <typename T, bool WHOLE> struct Piece;
template <typename T> struct Piece<T, true> {
  static constexpr int N = 8;
  using Raw = uint4;
  static __device__ Raw load(const T* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
  static __device__ void store(T* p, Raw v) { *reinterpret_cast<uint4*>(p) = v; }
  static __device__ void open(Raw v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 a = Num<T>::open(w[i]); f[2 * i] = a.x; f[2 * i + 1] = a.y; }
  }
  static __device__ Raw close(const float* f) {
    return make_uint4(Num<T>::close(f[0], f[1]), Num<T>::close(f[2], f[3]), Num<T>::close(f[4], f[5]), Num<T>::close(f[6], f[7]));
  }
};
template <> struct Piece<float, true> {
  static constexpr int N = 4;
  using Raw = float4;
  static __device__ Raw load(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
  static __device__ void store(float* p, Raw v) { *reinterpret_cast<float4*>(p) = v; }
  static __device__ void open(Raw v, float* f) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
  static __device__ Raw close(const float* f) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <typename T> struct Scalar {
  static __device__ float open(T x) { return (float)x; }
  static __device__ T close(float x) { return Num<T>::one(x); }
};
template <> struct Scalar<float> {
  static __device__ float open(float x) { return x; }
  static __device__ float close(float x) { return x; }
};
template <typename T> struct Piece<T, false> {
  static constexpr int N = 1;
  using Raw = T;
  static __device__ Raw load(const T* p) { return *p; }
  static __device__ void store(T* p, Raw v) { *p = v; }
  static __device__ void open(Raw v, float* f) { f[0] = Scalar<T>::open(v); }
  static __device__ Raw close(const float* f) { return Scalar<T>::close(f[0]); }
};

__device__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// Sum over the W warps of a CTA, the same for every thread; `shared` holds W values and is free again after the next call's barrier
// (callers alternate between two).
template <int W> __device__ float cta_sum(float x, float* shared) {
  x = warp_sum(x);
  if (W == 1) return x;
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < W; ++i) s += shared[i];
  return s;
}

// ---- forward -------------------------------------------------------------------------------------------------

// W warps to a row, P pieces to a lane; four rows to a CTA where a row is a warp's.
template <typename T, bool WHOLE, int W, int P>
__global__ void __launch_bounds__(W == 1 ? 128 : 32 * W) layer_norm_kernel(const LayerNormArgs a) {
  using Pc = Piece<T, WHOLE>;
  constexpr int N = Pc::N, kThreads = 32 * W;
  __shared__ float shared[2][W];
  const long long row = W == 1 ? (long long)blockIdx.x * 4 + threadIdx.x / 32 : blockIdx.x;
  const int lane = W == 1 ? threadIdx.x & 31 : threadIdx.x;
  next_may_launch();
  wait_for_previous();
  if (W == 1 && row >= a.rows) return;
  const int pieces = a.hidden / N;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  typename Pc::Raw v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = lane + i * kThreads;
    if (at < pieces) v[i] = Pc::load(x + at * N);
  }
  float total = 0.0f;
  if (a.residual) {
    const T* const r = static_cast<const T*>(a.residual) + row * a.ldr;
    T* const sum = a.sum ? static_cast<T*>(a.sum) + row * a.lds : nullptr;
    typename Pc::Raw o[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = lane + i * kThreads;
      if (at < pieces) o[i] = Pc::load(r + at * N);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = lane + i * kThreads;
      if (at >= pieces) continue;
      float f[N], e[N];
      Pc::open(v[i], f);
      Pc::open(o[i], e);
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] += e[j];
      v[i] = Pc::close(f);
      if (sum) Pc::store(sum + at * N, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (lane + i * kThreads >= pieces) continue;
    float f[N];
    Pc::open(v[i], f);
#pragma unroll
    for (int j = 0; j < N; ++j) total += f[j];
  }
  const float inverse = 1.0f / (float)a.hidden;
  const float mean = cta_sum<W>(total, shared[0]) * inverse;
  float squares = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (lane + i * kThreads >= pieces) continue;
    float f[N];
    Pc::open(v[i], f);
#pragma unroll
    for (int j = 0; j < N; ++j) squares = fmaf(f[j] - mean, f[j] - mean, squares);
  }
  const float rstd = 1.0f / sqrtf(fmaf(cta_sum<W>(squares, shared[1]), inverse, a.eps));
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  T* const y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = lane + i * kThreads;
    if (at >= pieces) continue;
    float f[N], w[N], b[N];
    Pc::open(v[i], f);
    if (a.w) {
      Pc::open(Pc::load(static_cast<const T*>(a.w) + at * N), w);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = 1.0f;
    }
    if (a.b) {
      Pc::open(Pc::load(static_cast<const T*>(a.b) + at * N), b);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) b[j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = fmaf((f[j] - mean) * rstd, w[j], b[j]);
    Pc::store(y + at * N, Pc::close(f));
  }
}

// Any width: a CTA goes over its row three times, with sums in binary64.
constexpr int kLongThreads = 1024;
__device__ double long_sum(double x, double* shared) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x / 32] = x;
  __syncthreads();
  x = 0.0;
#pragma unroll
  for (int i = 0; i < kLongThreads / 32; ++i) x += shared[i];
  return x;
}
template <typename T>
__global__ void __launch_bounds__(kLongThreads) layer_norm_long_kernel(const LayerNormArgs a) {
  __shared__ double shared[2][kLongThreads / 32];
  next_may_launch();
  wait_for_previous();
  const long long row = blockIdx.x;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* const r = a.residual ? static_cast<const T*>(a.residual) + row * a.ldr : nullptr;
  T* const sum = r && a.sum ? static_cast<T*>(a.sum) + row * a.lds : nullptr;
  // x may be gone once the sum is stored in its place
  auto value = [&](int j) { return r ? Scalar<T>::close(Scalar<T>::open(x[j]) + Scalar<T>::open(r[j])) : x[j]; };
  double total = 0.0, squares = 0.0;
  for (int j = threadIdx.x; j < a.hidden; j += kLongThreads) {
    const T s = value(j);
    if (sum) sum[j] = s;
    total += (double)Scalar<T>::open(s);
  }
  const float mean = (float)(long_sum(total, shared[0]) / a.hidden);
  for (int j = threadIdx.x; j < a.hidden; j += kLongThreads) {
    const float d = Scalar<T>::open(sum ? sum[j] : value(j)) - mean;
    squares += (double)d * d;
  }
  const float rstd = 1.0f / sqrtf((float)(long_sum(squares, shared[1]) / a.hidden) + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const T* const w = static_cast<const T*>(a.w);
  const T* const b = static_cast<const T*>(a.b);
  T* const y = static_cast<T*>(a.y) + row * a.ldy;
  for (int j = threadIdx.x; j < a.hidden; j += kLongThreads) {
    const float n = (Scalar<T>::open(sum ? sum[j] : value(j)) - mean) * rstd;
    y[j] = Scalar<T>::close(fmaf(n, w ? Scalar<T>::open(w[j]) : 1.0f, b ? Scalar<T>::open(b[j]) : 0.0f));
  }
}

template <typename T, bool WHOLE, int W, int P> cudaError_t run(const LayerNormArgs& a, cudaStream_t s) {
  const unsigned ctas = (unsigned)(W == 1 ? (a.rows + 3) / 4 : a.rows);
  return launch(layer_norm_kernel<T, WHOLE, W, P>, dim3(ctas), W == 1 ? 128 : 32 * W, 0, s, a);
}

template <typename T> cudaError_t run_forward(const LayerNormArgs& a, cudaStream_t s) {
  if (a.whole) {
    const int pieces = a.hidden / Piece<T, true>::N;
    if (pieces <= 32) return run<T, true, 1, 1>(a, s);
    if (pieces <= 64) return run<T, true, 1, 2>(a, s);
    if (pieces <= 128) return run<T, true, 1, 4>(a, s);
    if (pieces <= 256) return run<T, true, 1, 8>(a, s);
    if (pieces <= 512) return run<T, true, 4, 4>(a, s);
    if (pieces <= 1024) return run<T, true, 4, 8>(a, s);
    if (pieces <= 4096) return run<T, true, 16, 8>(a, s);
  } else {
    if (a.hidden <= 256) return run<T, false, 1, 8>(a, s);
    if (a.hidden <= 1024) return run<T, false, 1, 32>(a, s);
    if (a.hidden <= 8192) return run<T, false, 8, 32>(a, s);
  }
  return launch(layer_norm_long_kernel<T>, dim3((unsigned)a.rows), kLongThreads, 0, s, a);
}

// ---- gradient ------------------------------------------------------------------------------------------------

constexpr int kGradRows = 2;                  // rows of a CTA (of a warp, where a row is a warp's) at a time
constexpr int kGradCtasPerSm = 2;

// Sums of four values over a warp: halves are exchanged first, so that six shuffles do for twenty.  Lane l gets value l / 8.
__device__ float warp_sum4(const float* v, int lane) {
  const bool up = lane & 16, side = lane & 8;
  const float a = (up ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[2], 16);
  const float b = (up ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, up ? v[1] : v[3], 16);
  float x = (side ? b : a) + __shfl_xor_sync(0xffffffffu, side ? a : b, 8);
#pragma unroll
  for (int o = 4; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// WARP: a row is a warp's, eight rows' walks to a CTA.  Otherwise the CTA has a thread to every piece of a row.
template <typename T, bool WARP, int MAX>
__global__ void __launch_bounds__(MAX, MAX <= 256 ? kGradCtasPerSm : 1) layer_norm_grad_kernel(const LayerNormGradArgs a) {
  using Pc = Piece<T, true>;
  constexpr int N = Pc::N, R = kGradRows;
  __shared__ float4 exchange[2][WARP ? 1 : MAX / 32];
  __shared__ float sums[WARP ? 2 : 1][WARP ? 8 : 1][WARP ? 32 * N : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, warps = blockDim.x / 32;
  const int piece = WARP ? lane : threadIdx.x;
  next_may_launch();
  wait_for_previous();
  const bool holds = piece < a.hidden / N;
  const int column = holds ? piece * N : 0;                   // a thread without a piece reads the row's first and uses nothing of it
  const long long walks = WARP ? (long long)gridDim.x * 8 : gridDim.x;
  const long long walk = WARP ? (long long)blockIdx.x * 8 + warp : blockIdx.x;
  const T* const s_rows = static_cast<const T*>(a.s) + column;
  const T* const g_rows = static_cast<const T*>(a.dy) + column;
  const T* const k_rows = a.dsum ? static_cast<const T*>(a.dsum) + column : nullptr;
  T* const o_rows = a.dx ? static_cast<T*>(a.dx) + column : nullptr;
  float w[N], dw[N], db[N];
#pragma unroll
  for (int j = 0; j < N; ++j) { w[j] = 1.0f; dw[j] = 0.0f; db[j] = 0.0f; }
  if (a.w) Pc::open(Pc::load(static_cast<const T*>(a.w) + column), w);
  const float inverse = 1.0f / (float)a.hidden;
  typename Pc::Raw ns[R], ng[R], nk[R];
  float nmean[R], nrstd[R];
  auto load = [&](long long row) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const long long r = min(row + i, a.rows - 1);
      ns[i] = Pc::load(s_rows + r * a.lds);
      ng[i] = Pc::load(g_rows + r * a.lddy);
      if (k_rows) nk[i] = Pc::load(k_rows + r * a.ldds);
      nmean[i] = __ldg(a.mean + r);
      nrstd[i] = __ldg(a.rstd + r);
    }
  };
  long long row = walk * R;
  if (row < a.rows) load(row);
  int turn = 0;
  for (; row < a.rows; row += walks * R, turn ^= 1) {
    float n[R][N], g[R][N], rstd[R], part[2 * R];
    typename Pc::Raw skip[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      Pc::open(ns[i], n[i]);
      Pc::open(ng[i], g[i]);
      skip[i] = nk[i];
      rstd[i] = nrstd[i];
      const bool counts = holds && row + i < a.rows;
      part[2 * i] = part[2 * i + 1] = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        n[i][j] = (n[i][j] - nmean[i]) * rstd[i];
        if (counts) {                                          // what does not may be NaN or infinite: left out, not times 0
          dw[j] = fmaf(g[i][j], n[i][j], dw[j]);
          db[j] += g[i][j];
        }
        g[i][j] *= w[j];
        part[2 * i] += g[i][j];
        part[2 * i + 1] = fmaf(g[i][j], n[i][j], part[2 * i + 1]);
      }
      if (!holds) part[2 * i] = part[2 * i + 1] = 0.0f;
    }
    if (row + walks * R < a.rows) load(row + walks * R);
    if (!o_rows) continue;
    const float x = warp_sum4(part, lane);                     // value lane / 8
    float joined[4];
    if (WARP) {
#pragma unroll
      for (int i = 0; i < 4; ++i) joined[i] = __shfl_sync(0xffffffffu, x, 8 * i);
    } else {
      if (lane % 8 == 0) reinterpret_cast<float*>(&exchange[turn][warp])[lane / 8] = x;
      __syncthreads();
      joined[0] = joined[1] = joined[2] = joined[3] = 0.0f;
      for (int i = 0; i < warps; ++i) {
        const float4 o = exchange[turn][i];
        joined[0] += o.x; joined[1] += o.y; joined[2] += o.z; joined[3] += o.w;
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (!holds || row + i >= a.rows) continue;
      const float c1 = joined[2 * i] * inverse, c2 = joined[2 * i + 1] * inverse;
      float o[N], k[N];
#pragma unroll
      for (int j = 0; j < N; ++j) o[j] = rstd[i] * (g[i][j] - fmaf(n[i][j], c2, c1));
      if (k_rows) {
        Pc::open(skip[i], k);
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] += k[j];
      }
      Pc::store(o_rows + (row + i) * a.lddx, Pc::close(o));
    }
  }
  if (!a.dw && !a.db) return;
  float* const out = a.partials + (long long)blockIdx.x * 2 * a.hidden;
  if (WARP) {
#pragma unroll
    for (int j = 0; j < N; ++j) { sums[0][warp][lane * N + j] = dw[j]; sums[1][warp][lane * N + j] = db[j]; }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * a.hidden; e += 256) {
      const int t = e >= a.hidden, j = e - t * a.hidden;
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += sums[t][i][j];
      out[e] = s;
    }
  } else if (holds) {
#pragma unroll
    for (int j = 0; j < N; ++j) { out[column + j] = dw[j]; out[a.hidden + column + j] = db[j]; }
  }
}

// Any width and alignment: sums of dw and db by columns, a thread to a column and four walks to a CTA, before dx is written (which may be dy).
constexpr int kColumns = 64, kWalks = 4;
template <typename T>
__global__ void __launch_bounds__(kColumns * kWalks) layer_norm_columns_kernel(const LayerNormGradArgs a) {
  __shared__ float sums[2][kWalks][kColumns];
  const int column = blockIdx.x * kColumns + threadIdx.x, at = min(column, a.hidden - 1);
  next_may_launch();
  wait_for_previous();
  float dw = 0.0f, db = 0.0f;
  const T* const s = static_cast<const T*>(a.s) + at;
  const T* const g = static_cast<const T*>(a.dy) + at;
#pragma unroll 4
  for (long long row = (long long)blockIdx.y * kWalks + threadIdx.y; row < a.rows; row += (long long)gridDim.y * kWalks) {
    const float n = (Scalar<T>::open(s[row * a.lds]) - __ldg(a.mean + row)) * __ldg(a.rstd + row), dy = Scalar<T>::open(g[row * a.lddy]);
    dw = fmaf(dy, n, dw);
    db += dy;
  }
  sums[0][threadIdx.y][threadIdx.x] = dw;
  sums[1][threadIdx.y][threadIdx.x] = db;
  __syncthreads();
  if (threadIdx.y < 2 && column < a.hidden) {
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < kWalks; ++i) x += sums[threadIdx.y][i][threadIdx.x];
    a.partials[((long long)blockIdx.y * 2 + threadIdx.y) * a.hidden + column] = x;
  }
}

constexpr int kRowThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kRowThreads) layer_norm_rows_kernel(const LayerNormGradArgs a) {
  __shared__ float shared[2][kRowThreads / 32];
  next_may_launch();
  wait_for_previous();
  const long long row = blockIdx.x;
  const T* const s = static_cast<const T*>(a.s) + row * a.lds;
  const T* const dy = static_cast<const T*>(a.dy) + row * a.lddy;
  const T* const skip = a.dsum ? static_cast<const T*>(a.dsum) + row * a.ldds : nullptr;
  const T* const w = static_cast<const T*>(a.w);
  T* const dx = static_cast<T*>(a.dx) + row * a.lddx;
  const float mean = a.mean[row], rstd = a.rstd[row];
  float sum_g = 0.0f, sum_gn = 0.0f;
  for (int j = threadIdx.x; j < a.hidden; j += kRowThreads) {
    const float n = (Scalar<T>::open(s[j]) - mean) * rstd, g = Scalar<T>::open(dy[j]) * (w ? Scalar<T>::open(w[j]) : 1.0f);
    sum_g += g;
    sum_gn = fmaf(g, n, sum_gn);
  }
  const float c1 = cta_sum<kRowThreads / 32>(sum_g, shared[0]) / a.hidden, c2 = cta_sum<kRowThreads / 32>(sum_gn, shared[1]) / a.hidden;
  for (int j = threadIdx.x; j < a.hidden; j += kRowThreads) {
    const float n = (Scalar<T>::open(s[j]) - mean) * rstd, g = Scalar<T>::open(dy[j]) * (w ? Scalar<T>::open(w[j]) : 1.0f);
    const float o = rstd * (g - fmaf(n, c2, c1));
    dx[j] = Scalar<T>::close(skip ? o + Scalar<T>::open(skip[j]) : o);
  }
}

// dw and db from the sums of the CTAs: a warp's lanes take neighbouring columns, the warps of a CTA every eighth row of sums.
__global__ void __launch_bounds__(256) layer_norm_join_kernel(const float* partials, int parts, int hidden, float* dw, float* db) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const long long e = (long long)blockIdx.x * 32 + lane;
  next_may_launch();
  wait_for_previous();
  float s = 0.0f;
  if (e < 2ll * hidden) {
#pragma unroll 8
    for (int i = warp; i < parts; i += 8) s += __ldcg(partials + i * 2ll * hidden + e);
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp || e >= 2ll * hidden) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += sums[i][lane];
  float* const out = e < hidden ? dw : db;
  if (out) out[e < hidden ? e : e - hidden] = s;
}

// How a gradient is computed: rows of a warp, rows of a CTA with a thread to a piece, or by columns and rows apart.
struct GradPlan { int threads; bool warp, apart; long long parts; };
template <typename T> GradPlan grad_plan(const LayerNormGradArgs& a) {
  const int pieces = a.hidden / Piece<T, true>::N;
  GradPlan p{};
  p.apart = !a.whole || pieces > 1024;
  if (p.apart) {
    const long long strips = (a.hidden + kColumns - 1) / kColumns, walks = (a.rows + kWalks - 1) / kWalks;
    const long long most = (8ll * a.sms + strips - 1) / strips;
    p.parts = walks < most ? walks : most;
    return p;
  }
  p.warp = pieces <= 32;
  p.threads = p.warp ? 256 : (pieces + 31) / 32 * 32;
  // as many CTAs as are resident at a time
  const int per_sm = p.threads > 256 ? 1 : kGradCtasPerSm * (256 / p.threads);
  const long long batches = (a.rows + kGradRows * (p.warp ? 8 : 1) - 1) / (kGradRows * (p.warp ? 8 : 1));
  p.parts = batches < (long long)per_sm * a.sms ? batches : (long long)per_sm * a.sms;
  return p;
}

template <typename T> cudaError_t run_grad(const LayerNormGradArgs& a, cudaStream_t s) {
  const GradPlan p = grad_plan<T>(a);
  const bool sums = a.dw || a.db;
  cudaError_t e = cudaSuccess;
  if (p.apart) {
    if (sums) e = launch(layer_norm_columns_kernel<T>, dim3((unsigned)((a.hidden + kColumns - 1) / kColumns), (unsigned)p.parts), dim3(kColumns, kWalks), 0, s, a);
    if (e == cudaSuccess && a.dx) e = launch(layer_norm_rows_kernel<T>, dim3((unsigned)a.rows), dim3(kRowThreads), 0, s, a);
  } else if (p.warp) {
    e = launch(layer_norm_grad_kernel<T, true, 256>, dim3((unsigned)p.parts), dim3(p.threads), 0, s, a);
  } else if (p.threads <= 256) {
    e = launch(layer_norm_grad_kernel<T, false, 256>, dim3((unsigned)p.parts), dim3(p.threads), 0, s, a);
  } else {
    e = launch(layer_norm_grad_kernel<T, false, 1024>, dim3((unsigned)p.parts), dim3(p.threads), 0, s, a);
  }
  if (e != cudaSuccess || !sums) return e;
  return launch(layer_norm_join_kernel, dim3((unsigned)((2ll * a.hidden + 31) / 32)), dim3(256), 0, s, (const float*)a.partials, (int)p.parts, a.hidden, a.dw, a.db);
}

}  // namespace

cudaError_t launch_layer_norm(int dtype, const LayerNormArgs& a, cudaStream_t s) {
  if (dtype == AQ_FP16) return run_forward<__half>(a, s);
  if (dtype == AQ_BF16) return run_forward<__nv_bfloat16>(a, s);
  return run_forward<float>(a, s);
}
long long layer_norm_grad_parts(int dtype, const LayerNormGradArgs& a) {
  if (dtype == AQ_FP16) return grad_plan<__half>(a).parts;
  if (dtype == AQ_BF16) return grad_plan<__nv_bfloat16>(a).parts;
  return grad_plan<float>(a).parts;
}
cudaError_t launch_layer_norm_grad(int dtype, const LayerNormGradArgs& a, cudaStream_t s) {
  if (dtype == AQ_FP16) return run_grad<__half>(a, s);
  if (dtype == AQ_BF16) return run_grad<__nv_bfloat16>(a, s);
  return run_grad<float>(a, s);
}

}  // namespace aq
