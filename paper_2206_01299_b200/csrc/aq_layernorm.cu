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
// Forward: rows up to 256 pieces of 16 bytes belong to a warp, which needs no barrier; wider ones to a CTA.  32768 x 1600 fp16 with a
// residual 68 to 70 us, 0.92 to 0.95 of a plain copy's bandwidth.
// Backward: a CTA of as many threads as a row has eight elements (up to 256 elements: eight warps with a row each; over 2048: sixteen to
// a thread) walks over the rows, a thread always at the same columns, whose sums of dw and db it keeps in registers, in binary32 over all of its rows
// (110 of 32768 x 1600's, rows / 148 at most); a CTA's sums go to a workspace, which a second kernel adds up in a fixed order.  Rows come ahead through shared memory by asynchronous copies.  32768 x 1600 fp16 with a gradient
// along the stream 77 to 83 us (0.77 to 0.84): two CTAs of 120 registers a thread, and 25 instructions an element with a barrier for every two rows;
// issue 0.44.  16384 x 1600 binary32 68 us (0.95).  What did not help: three CTAs at 80 registers (spills, 83 to 125 us), forming n and g again after
// the barrier instead of keeping them (89 us), one row or four at a time (106 us, 87 us), a thread's copies side by side in shared memory (115 us).
// Rows that begin inside a piece: forward a row's pieces are those of the grid it lies on, the first and last by elements; backward a CTA takes
// every `period`-th row, which begin alike, so that its columns stay.  16384 x 1601 fp16: 78 us and 49 us (one element at a time: 217 and 152).
// Backward, rows over 8192 elements are read once for the columns' sums and once for dx (4096 x 12000 fp16: 126 us, element by element 269). Rows of
// operands that begin differently, and forward rows over 4096 pieces, go element by element through kernels that read them again.

#include "aq_stage.h"
#include "aq_stage_device.cuh"

namespace aq {
namespace {

template <typename T> struct Scalar {
  static __device__ float open(T x) { return (float)x; }
  static __device__ T close(float x) { return Num<T>::one(x); }
};
template <> struct Scalar<float> {
  static __device__ float open(float x) { return x; }
  static __device__ float close(float x) { return x; }
};

// A lane's piece of a row: 16 bytes, or one element where rows do not begin on 16-byte boundaries.  Loads are ordinary ones, not those for data that
// nothing writes while a kernel runs: outputs may take the inputs' places, and a kernel may start while the one before still writes its operands.
template <typename T, bool WHOLE> struct Piece;
template <typename T> struct Piece<T, true> {
  static constexpr int N = 8;
  using Raw = uint4;
  static __device__ Raw load(const T* p) { return *reinterpret_cast<const uint4*>(p); }
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
  static __device__ Raw load(const float* p) { return *reinterpret_cast<const float4*>(p); }
  static __device__ void store(float* p, Raw v) { *reinterpret_cast<float4*>(p) = v; }
  static __device__ void open(Raw v, float* f) { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
  static __device__ Raw close(const float* f) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <typename T> struct Piece<T, false> {
  static constexpr int N = 1;
  using Raw = T;
  static __device__ Raw load(const T* p) { return *p; }
  static __device__ void store(T* p, Raw v) { *p = v; }
  static __device__ void open(Raw v, float* f) { f[0] = Scalar<T>::open(v); }
  static __device__ Raw close(const float* f) { return Scalar<T>::close(f[0]); }
};

// A piece of which a row has the elements [lo, hi) only: zeros around them, and only they are stored.
template <typename Pc, typename T> __device__ typename Pc::Raw load_piece(const T* p, int lo, int hi) {
  if (lo <= 0 && hi >= Pc::N) return Pc::load(p);
  float f[Pc::N];
#pragma unroll
  for (int j = 0; j < Pc::N; ++j) f[j] = j >= lo && j < hi ? Scalar<T>::open(p[j]) : 0.0f;
  return Pc::close(f);
}
template <typename Pc, typename T> __device__ void store_piece(T* p, typename Pc::Raw v, int lo, int hi) {
  if (lo <= 0 && hi >= Pc::N) {
    Pc::store(p, v);
    return;
  }
  float f[Pc::N];
  Pc::open(v, f);
#pragma unroll
  for (int j = 0; j < Pc::N; ++j)
    if (j >= lo && j < hi) p[j] = Scalar<T>::close(f[j]);
}
// N values at p, which are a piece of [0, hidden) that begins at `at`: where that is off the 16-byte boundaries, out of the two pieces that hold them.
template <typename Pc, typename T> __device__ void load_weights(const T* w, int at, int hidden, float* f) {
  constexpr int N = Pc::N;
  if (N == 1 || at < N || at + 2 * N > hidden) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = at + j >= 0 && at + j < hidden ? Scalar<T>::open(w[at + j]) : 0.0f;
    return;
  }
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(w + at) & 15);   // the same for a whole warp
  const uint4* const from = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(w + at) - off);
  const uint4 a = *from, b = off ? from[1] : a;
  uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (off & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) v[i] = v[i + 2];
  }
  if (off & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) v[i] = v[i + 1];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], (off & 3) * 8);
  typename Pc::Raw raw;
  memcpy(&raw, v, sizeof raw);
  Pc::open(raw, f);
}

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

// W warps to a row, P pieces to a lane; four rows to a CTA where a row is a warp's.  EDGE: rows may begin and end inside a piece, all operands'
// at the same place (a row's first piece then begins before it), and w and b are off the boundaries.
template <typename T, bool WHOLE, bool EDGE, int W, int P>
__global__ void __launch_bounds__(W == 1 ? 128 : 32 * W) layer_norm_kernel(const LayerNormArgs a) {
  using Pc = Piece<T, WHOLE>;
  constexpr int N = Pc::N, kStep = 32 * W * N;
  __shared__ float shared[2][W];
  const long long row = W == 1 ? (long long)blockIdx.x * 4 + threadIdx.x / 32 : blockIdx.x;
  const int lane = W == 1 ? threadIdx.x & 31 : threadIdx.x;
  next_may_launch();
  wait_for_previous();
  if (W == 1 && row >= a.rows) return;
  const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
  const int first = lane * N - (EDGE ? (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % N) : 0);   // of the lane's first piece; the others are kStep apart
  auto at = [&](int i) { return first + i * kStep; };
  auto lo = [&](int i) { return EDGE ? -at(i) : 0; };         // of a piece's elements those in the row
  auto hi = [&](int i) { return EDGE ? a.hidden - at(i) : N; };
  auto has = [&](int i) { return at(i) < a.hidden; };
  typename Pc::Raw v[P];
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (has(i)) v[i] = load_piece<Pc>(x + at(i), lo(i), hi(i));
  if (a.residual) {
    const T* const r = static_cast<const T*>(a.residual) + row * a.ldr;
    T* const sum = a.sum ? static_cast<T*>(a.sum) + row * a.lds : nullptr;
    typename Pc::Raw o[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (has(i)) o[i] = load_piece<Pc>(r + at(i), lo(i), hi(i));
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (!has(i)) continue;
      float f[N], e[N];
      Pc::open(v[i], f);
      Pc::open(o[i], e);
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] += e[j];
      v[i] = Pc::close(f);
      if (sum) store_piece<Pc>(sum + at(i), v[i], lo(i), hi(i));
    }
  }
  float total = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (!has(i)) continue;
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
    if (!has(i)) continue;
    float f[N];
    Pc::open(v[i], f);
    if (!EDGE || (lo(i) <= 0 && hi(i) >= N)) {
#pragma unroll
      for (int j = 0; j < N; ++j) squares = fmaf(f[j] - mean, f[j] - mean, squares);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j >= lo(i) && j < hi(i)) squares = fmaf(f[j] - mean, f[j] - mean, squares);
    }
  }
  const float rstd = 1.0f / sqrtf(fmaf(cta_sum<W>(squares, shared[1]), inverse, a.eps));
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  T* const y = static_cast<T*>(a.y) + row * a.ldy;
  const T* const wt = static_cast<const T*>(a.w);
  const T* const bs = static_cast<const T*>(a.b);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (!has(i)) continue;
    float f[N], w[N], b[N];
    Pc::open(v[i], f);
    if (!wt) {
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = 1.0f;
    } else if (EDGE) {
      load_weights<Pc>(wt, at(i), a.hidden, w);
    } else {
      Pc::open(Pc::load(wt + at(i)), w);
    }
    if (!bs) {
#pragma unroll
      for (int j = 0; j < N; ++j) b[j] = 0.0f;
    } else if (EDGE) {
      load_weights<Pc>(bs, at(i), a.hidden, b);
    } else {
      Pc::open(Pc::load(bs + at(i)), b);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = fmaf((f[j] - mean) * rstd, w[j], b[j]);
    store_piece<Pc>(y + at(i), Pc::close(f), lo(i), hi(i));
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

template <typename T, bool WHOLE, bool EDGE, int W, int P> cudaError_t run(const LayerNormArgs& a, cudaStream_t s) {
  const unsigned ctas = (unsigned)(W == 1 ? (a.rows + 3) / 4 : a.rows);
  return launch(layer_norm_kernel<T, WHOLE, EDGE, W, P>, dim3(ctas), dim3(W == 1 ? 128 : 32 * W), 0, s, a);
}
template <typename T> cudaError_t run_long(const LayerNormArgs& a, cudaStream_t s) {
  return launch(layer_norm_long_kernel<T>, dim3((unsigned)a.rows), dim3(kLongThreads), 0, s, a);
}
// Pieces of 16 bytes; a shifted row may need one more.
template <typename T, bool EDGE> cudaError_t run_pieces(const LayerNormArgs& a, cudaStream_t s) {
  constexpr int N = Piece<T, true>::N;
  const int pieces = (a.hidden + (EDGE ? N - 1 : 0) + N - 1) / N;
  if (pieces <= 32) return run<T, true, EDGE, 1, 1>(a, s);
  if (pieces <= 64) return run<T, true, EDGE, 1, 2>(a, s);
  if (pieces <= 128) return run<T, true, EDGE, 1, 4>(a, s);
  if (pieces <= 256) return run<T, true, EDGE, 1, 8>(a, s);
  if (pieces <= 512) return run<T, true, EDGE, 4, 4>(a, s);
  if (pieces <= 1024) return run<T, true, EDGE, 8, 4>(a, s);
  if (pieces <= 2048) return run<T, true, EDGE, 16, 4>(a, s);
  if (pieces <= 4096) return run<T, true, EDGE, 16, 8>(a, s);
  return run_long<T>(a, s);
}
template <typename T> cudaError_t run_forward(const LayerNormArgs& a, cudaStream_t s) {
  if (a.rows_at == kRowsWhole) return run_pieces<T, false>(a, s);
  if (a.rows_at == kRowsAlike) return run_pieces<T, true>(a, s);
  if (a.hidden <= 256) return run<T, false, true, 1, 8>(a, s);
  if (a.hidden <= 1024) return run<T, false, true, 1, 32>(a, s);
  if (a.hidden <= 2048) return run<T, false, true, 8, 8>(a, s);
  if (a.hidden <= 8192) return run<T, false, true, 8, 32>(a, s);
  return run_long<T>(a, s);
}

// ---- gradient ------------------------------------------------------------------------------------------------

// Sixteen bytes of a row in pairs.
template <typename T> struct Pairs {
  static constexpr int N = 4;
  static __device__ void open(uint4 raw, float2* f) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = Num<T>::open(w[i]);
  }
  static __device__ uint4 close(const float2* f) {
    return make_uint4(Num<T>::close(f[0].x, f[0].y), Num<T>::close(f[1].x, f[1].y), Num<T>::close(f[2].x, f[2].y), Num<T>::close(f[3].x, f[3].y));
  }
};
template <> struct Pairs<float> {
  static constexpr int N = 2;
  static __device__ void open(uint4 raw, float2* f) {
    f[0] = make_float2(__uint_as_float(raw.x), __uint_as_float(raw.y));
    f[1] = make_float2(__uint_as_float(raw.z), __uint_as_float(raw.w));
  }
  static __device__ uint4 close(const float2* f) { return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y)); }
};

// Sums of V values over a warp: halves are exchanged first, so that a handful of shuffles do for 5 V.  Lane l gets value l / (32 / V).
template <int V> __device__ float warp_sums(const float* v, int lane) {
  float x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = v[i];
#pragma unroll
  for (int n = V / 2, o = 16; n; n /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] = (up ? x[i + n] : x[i]) + __shfl_xor_sync(0xffffffffu, up ? x[i] : x[i + n], o);
  }
#pragma unroll
  for (int o = 16 / V; o; o >>= 1) x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
  return x[0];
}

// Sums of dw and db are kept in rows of whole sectors: pieces of a sector cost as much to write as all of it.
__host__ __device__ constexpr int padded_hidden(int hidden) { return (hidden + 7) / 8 * 8; }
__device__ void store_sums(float* to, const float2* f, int pairs) {
  if (pairs == 4) {
    asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"f"(f[0].x), "f"(f[0].y), "f"(f[1].x), "f"(f[1].y), "f"(f[2].x), "f"(f[2].y), "f"(f[3].x), "f"(f[3].y), "l"(to) : "memory");
  } else {
    *reinterpret_cast<float4*>(to) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
  }
}

constexpr int kGradWalks = 8;                 // rows' walks of a CTA where a row is a warp's
constexpr int kGradSlots = 2;                 // batches of rows that a thread has in shared memory: the one it works on and the next
// A CTA's threads have Q pieces of 16 bytes of a row each (WARP: a warp's lanes, and eight walks to a CTA) and take R rows at a time.  The next rows
// are copied to shared memory meanwhile, each thread's elements by itself and for itself.  Elements behind a row's end are zeros there and add
// nothing to any sum.  EDGE: rows begin inside a piece, every `period`-th one at the same place; a CTA (a warp) takes rows that do.
template <typename T, bool EDGE, bool WARP, int R, int Q, int MAX, int CTAS>
__global__ void __launch_bounds__(MAX, CTAS) layer_norm_grad_kernel(const LayerNormGradArgs a) {
  using Ps = Pairs<T>;
  constexpr int H = Ps::N, N = 2 * H, V = 2 * R;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float exchange[2][WARP ? 1 : MAX / 32][V];
  __shared__ float2 stats[kGradSlots][MAX / 32][R];
  __shared__ float sums[WARP ? 2 : 1][WARP ? kGradWalks : 1][WARP ? 32 * N * Q : 1];
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), warps = blockDim.x / 32;
  const bool skip = a.dsum != nullptr;
  // shared memory: the threads' 16 bytes of a piece side by side; a piece, a row of three arrays and a slot further on
  constexpr uint32_t kPart = MAX * 16, kRow = 3 * Q * kPart, kSlot = R * kRow;
  const uint32_t mine = shared_address(ring) + threadIdx.x * 16;
  next_may_launch();
  wait_for_previous();
  const int walks = WARP ? gridDim.x * kGradWalks : gridDim.x, walk = WARP ? blockIdx.x * kGradWalks + warp : blockIdx.x;
  // rows: `kind`, kind + period ... begin at the same place in their first piece; of those, every walk of the kind takes R at a time in turn
  const int period = EDGE ? a.period : 1, kind = EDGE ? walk % period : 0, turn = EDGE ? walk / period : walk;
  const int shift = EDGE ? (int)(kind * (a.lds % N) % N) : 0;
  int column[Q], lo[Q], hi[Q];                                 // of the thread's elements those in the row
  float2 w[Q][H], dw[Q][H], db[Q][H];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const NormPiece piece = norm_piece(WARP ? lane + 32 * q : (int)(threadIdx.x + q * blockDim.x), N, shift, a.hidden);
    column[q] = piece.column;
    lo[q] = EDGE ? piece.lo : 0;
    hi[q] = piece.hi;
#pragma unroll
    for (int j = 0; j < H; ++j) w[q][j] = dw[q][j] = db[q][j] = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (j < lo[q] || j >= hi[q]) continue;
      (j & 1 ? w[q][j / 2].y : w[q][j / 2].x) = a.w ? Scalar<T>::open(static_cast<const T*>(a.w)[column[q] + j]) : 1.0f;
    }
  }
  const float inverse = 1.0f / (float)a.hidden;
  // the next batch's rows: addresses move on by constants
  const long long first = kind + (long long)turn * R * period, kinds = (a.rows - kind + period - 1) / period;   // rows of the kind
  const T *s = static_cast<const T*>(a.s) + first * a.lds, *g = static_cast<const T*>(a.dy) + first * a.lddy;
  const T* k = skip ? static_cast<const T*>(a.dsum) + first * a.ldds : nullptr;
  T* o = a.dx ? static_cast<T*>(a.dx) + first * a.lddx : nullptr;
  const float* stat = (lane & 1 ? a.rstd : a.mean) + first + (lane % V) / 2 * period;
  const int step = walks * R, each = walks / period * R;       // rows, and rows of the kind, from one batch to the next
  int left = (int)max(kinds - (long long)turn * R, 0ll), here = left;   // rows of the kind from the next batch to ask for on; from the one that is worked on
  auto ask = [&](int slot) {
    const uint32_t there = mine + slot * kSlot;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (i >= left) break;
      const long long r = i * period;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int bytes = hi[q] * (int)sizeof(T), at = norm_copy_from(column[q], hi[q], shift);
        const uint32_t to = there + i * kRow + q * kPart;
        copy16(to, s + r * a.lds + at, bytes);
        copy16(to + Q * kPart, g + r * a.lddy + at, bytes);
        if (skip) copy16(to + 2 * Q * kPart, k + r * a.ldds + at, bytes);
      }
    }
    if (lane < V && lane / 2 < left) copy4(shared_address(&stats[slot][warp][0]) + lane * 4, stat);   // mean and rstd of the rows, for the warp
    s += step * a.lds;
    g += step * a.lddy;
    if (skip) k += step * a.ldds;
    stat += step;
    left -= each;
  };
  if (left > 0) ask(0);
  copies_end();
  int slot = 0;
#pragma unroll 1
  for (; here > 0; here -= each, slot ^= 1) {
    __syncwarp();                                              // the warp has read the other slot's statistics
    if (left > 0) ask(slot ^ 1);
    copies_end();
    copies_wait<1>();
    __syncwarp();
    const uint32_t now = mine + slot * kSlot;
    auto take = [&](int i, int array, int q, float2* f) { Ps::open(shared16(now + i * kRow + (array * Q + q) * kPart), f); };
    float sum[V], rstds[R];
    float2 n[R][Q][H], y[R][Q][H];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      sum[2 * i] = sum[2 * i + 1] = 0.0f;
      if (i >= here) break;
      const float2 st = stats[slot][warp][i];
      const float mean = st.x, rstd = rstds[i] = st.y;
      const bool far = fabsf(mean) > 1e15f;                    // a zero's n may be infinite (rstd is 3e22 at most), whatever the row's elements have
      float2 sg = make_float2(0.0f, 0.0f), sgn = sg;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        take(i, 0, q, n[i][q]);
        take(i, 1, q, y[i][q]);
#pragma unroll
        for (int j = 0; j < H; ++j) n[i][q][j] = mul2(add2(n[i][q][j], both(-mean)), both(rstd));
        if (EDGE && lo[q]) {                                   // what the row before left there
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (j < lo[q]) (j & 1 ? n[i][q][j / 2].y : n[i][q][j / 2].x) = (j & 1 ? y[i][q][j / 2].y : y[i][q][j / 2].x) = 0.0f;
        }
        if (far) {                                             // places behind the row's end, which hold zeros
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (j >= hi[q]) (j & 1 ? n[i][q][j / 2].y : n[i][q][j / 2].x) = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < H; ++j) {
          dw[q][j] = fma2(y[i][q][j], n[i][q][j], dw[q][j]);
          db[q][j] = add2(db[q][j], y[i][q][j]);
          y[i][q][j] = mul2(y[i][q][j], w[q][j]);
          sg = add2(sg, y[i][q][j]);
          sgn = fma2(y[i][q][j], n[i][q][j], sgn);
        }
      }
      sum[2 * i] = sg.x + sg.y;
      sum[2 * i + 1] = sgn.x + sgn.y;
    }
    if (!o) continue;
    float x = warp_sums<V>(sum, lane);                         // value lane / (32 / V)
    if (WARP) {
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = __shfl_sync(0xffffffffu, x, i * (32 / V)) * inverse;
    } else {
      if (lane % (32 / V) == 0) exchange[slot][warp][lane / (32 / V)] = x;
      __syncthreads();
      x = 0.0f;
      for (int i = lane / V; i < warps; i += 32 / V) x += exchange[slot][i][lane % V];
#pragma unroll
      for (int m = V; m < 32; m *= 2) x += __shfl_xor_sync(0xffffffffu, x, m);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = __shfl_sync(0xffffffffu, x, i) * inverse;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (i >= here) break;
      const float rstd = rstds[i];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (hi[q] <= lo[q]) continue;
        float2 f[H];
        if (skip) take(i, 2, q, f);
#pragma unroll
        for (int j = 0; j < H; ++j) {
          const float2 d = add2(fma2(n[i][q][j], both(-sum[2 * i + 1]), y[i][q][j]), both(-sum[2 * i]));
          f[j] = skip ? fma2(d, both(rstd), f[j]) : mul2(d, both(rstd));
        }
        T* const to = o + (long long)(i * period) * a.lddx + column[q];
        if (hi[q] - lo[q] == N) {
          *reinterpret_cast<uint4*>(to) = Ps::close(f);
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (j >= lo[q] && j < hi[q]) to[j] = Scalar<T>::close(j & 1 ? f[j / 2].y : f[j / 2].x);
        }
      }
    }
    o += step * a.lddx;
  }
  if (!a.dw && !a.db) return;
  const int padded = padded_hidden(a.hidden);
  float* const out = a.partials + (long long)blockIdx.x * 2 * padded;
  if (WARP) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j < lo[q] || j >= hi[q]) continue;
        sums[0][warp][column[q] + j] = j & 1 ? dw[q][j / 2].y : dw[q][j / 2].x;
        sums[WARP ? 1 : 0][warp][column[q] + j] = j & 1 ? db[q][j / 2].y : db[q][j / 2].x;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * padded; e += blockDim.x) {
      const int t = e >= padded, j = e - t * padded;
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < (WARP ? kGradWalks : 1); ++i) s += sums[WARP ? t : 0][i][j];
      out[e] = s;
    }
  } else if (EDGE) {                                           // by way of the ring, which holds two sums per column and more
    __syncthreads();
    float* const f = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j < lo[q] || j >= hi[q]) continue;
        f[column[q] + j] = j & 1 ? dw[q][j / 2].y : dw[q][j / 2].x;
        f[padded + column[q] + j] = j & 1 ? db[q][j / 2].y : db[q][j / 2].x;
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < padded / 2; e += blockDim.x) reinterpret_cast<float4*>(out)[e] = reinterpret_cast<const float4*>(f)[e];
  } else {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (!hi[q]) continue;
      store_sums(out + column[q], dw[q], H);
      store_sums(out + padded + column[q], db[q], H);
    }
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
  double total_w = 0.0, total_b = 0.0;                         // of up to 64 rows' sums in binary32 each
  const T* const s = static_cast<const T*>(a.s) + at;
  const T* const g = static_cast<const T*>(a.dy) + at;
  const long long step = (long long)gridDim.y * kWalks;
  for (long long row = (long long)blockIdx.y * kWalks + threadIdx.y; row < a.rows;) {
    float dw = 0.0f, db = 0.0f;
    const int n_rows = (int)min((a.rows - row + step - 1) / step, 64ll);
#pragma unroll 8
    for (int i = 0; i < n_rows; ++i, row += step) {
      const float n = (Scalar<T>::open(s[row * a.lds]) - a.mean[row]) * a.rstd[row], dy = Scalar<T>::open(g[row * a.lddy]);
      dw = fmaf(dy, n, dw);
      db += dy;
    }
    total_w += (double)dw;
    total_b += (double)db;
  }
  sums[0][threadIdx.y][threadIdx.x] = (float)total_w;
  sums[1][threadIdx.y][threadIdx.x] = (float)total_b;
  __syncthreads();
  if (threadIdx.y < 2 && column < a.hidden) {
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < kWalks; ++i) x += sums[threadIdx.y][i][threadIdx.x];
    a.partials[((long long)blockIdx.y * 2 + threadIdx.y) * padded_hidden(a.hidden) + column] = x;
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
  double total_g = 0.0, total_gn = 0.0;                        // of up to 64 elements' sums in binary32 each: rows are as wide as 2^20
  for (int j = threadIdx.x; j < a.hidden;) {
    float sum_g = 0.0f, sum_gn = 0.0f;
    const int n_columns = min((a.hidden - j + kRowThreads - 1) / kRowThreads, 64);
#pragma unroll 8
    for (int i = 0; i < n_columns; ++i, j += kRowThreads) {
      const float n = (Scalar<T>::open(s[j]) - mean) * rstd, g = Scalar<T>::open(dy[j]) * (w ? Scalar<T>::open(w[j]) : 1.0f);
      sum_g += g;
      sum_gn = fmaf(g, n, sum_gn);
    }
    total_g += (double)sum_g;
    total_gn += (double)sum_gn;
  }
  const float c1 = cta_sum<kRowThreads / 32>((float)total_g, shared[0]) / a.hidden, c2 = cta_sum<kRowThreads / 32>((float)total_gn, shared[1]) / a.hidden;
#pragma unroll 4
  for (int j = threadIdx.x; j < a.hidden; j += kRowThreads) {
    const float n = (Scalar<T>::open(s[j]) - mean) * rstd, g = Scalar<T>::open(dy[j]) * (w ? Scalar<T>::open(w[j]) : 1.0f);
    const float o = rstd * (g - fmaf(n, c2, c1));
    dx[j] = Scalar<T>::close(skip ? o + Scalar<T>::open(skip[j]) : o);
  }
}

// The same for wide rows on 16-byte boundaries: a lane has a piece of 16 bytes, the warps of a CTA take rows in turn.
constexpr int kStripWarps = 8;
template <typename T>
__global__ void __launch_bounds__(32 * kStripWarps) layer_norm_strips_kernel(const LayerNormGradArgs a) {
  using Ps = Pairs<T>;
  constexpr int H = Ps::N, N = 2 * H;
  __shared__ float2 sums[2][kStripWarps][32 * H];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, column = (blockIdx.x * 32 + lane) * N;
  const int hi = min(max(a.hidden - column, 0), N);
  next_may_launch();
  wait_for_previous();
  float2 total_w[H], total_b[H];                              // of up to 64 rows' sums each
#pragma unroll
  for (int j = 0; j < H; ++j) total_w[j] = total_b[j] = make_float2(0.0f, 0.0f);
  const long long step = (long long)gridDim.y * kStripWarps;
  auto walk = [&](auto load) {                                // load: a piece of a row
    for (long long row = (long long)blockIdx.y * kStripWarps + warp; row < a.rows;) {
      float2 dw[H], db[H];
#pragma unroll
      for (int j = 0; j < H; ++j) dw[j] = db[j] = make_float2(0.0f, 0.0f);
      const int rows = (int)min((a.rows - row + step - 1) / step, 64ll);
#pragma unroll 4
      for (int i = 0; i < rows; ++i, row += step) {
        float2 n[H], y[H];
        load(static_cast<const T*>(a.s) + row * a.lds + column, n);
        load(static_cast<const T*>(a.dy) + row * a.lddy + column, y);
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int j = 0; j < H; ++j) {
          n[j] = mul2(add2(n[j], both(-mean)), both(rstd));
          dw[j] = fma2(y[j], n[j], dw[j]);
          db[j] = add2(db[j], y[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < H; ++j) {
        total_w[j] = add2(total_w[j], dw[j]);
        total_b[j] = add2(total_b[j], db[j]);
      }
    }
  };
  if (hi == N) {
    walk([](const T* p, float2* f) { Ps::open(*reinterpret_cast<const uint4*>(p), f); });
  } else if (hi) {
    walk([hi](const T* p, float2* f) {
#pragma unroll
      for (int j = 0; j < N; ++j) (j & 1 ? f[j / 2].y : f[j / 2].x) = j < hi ? Scalar<T>::open(p[j]) : 0.0f;
    });
  }
#pragma unroll
  for (int j = 0; j < H; ++j) { sums[0][warp][lane * H + j] = total_w[j]; sums[1][warp][lane * H + j] = total_b[j]; }
  __syncthreads();
  const int padded = padded_hidden(a.hidden);
  for (int e = threadIdx.x; e < 2 * 32 * N; e += 32 * kStripWarps) {
    const int t = e >= 32 * N, j = e - t * 32 * N, c = blockIdx.x * 32 * N + j;
    if (c >= a.hidden) continue;
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < kStripWarps; ++i) x += reinterpret_cast<const float*>(sums[t][i])[j];
    a.partials[((long long)blockIdx.y * 2 + t) * padded + c] = x;
  }
}

// dx of wide rows that begin alike in all operands: a CTA has a row in registers, P pieces of 16 bytes to a thread.  Without EDGE they are whole
// pieces on 16-byte boundaries, and so is w.  Four pieces go into 64 registers and two CTAs on a multiprocessor (one, at 66: 172 instead of 127 us for
// 4096 x 12000 fp16).
constexpr int kWideThreads = 512;
template <typename T, bool EDGE, int P>
__global__ void __launch_bounds__(kWideThreads, P == 4 ? 2 : 1) layer_norm_wide_kernel(const LayerNormGradArgs a) {
  using Pc = Piece<T, true>;
  constexpr int N = Pc::N, kStep = kWideThreads * N;
  __shared__ float shared[2][kWideThreads / 32];
  next_may_launch();
  wait_for_previous();
  const long long row = blockIdx.x;
  const T* const s = static_cast<const T*>(a.s) + row * a.lds;
  const T* const dy = static_cast<const T*>(a.dy) + row * a.lddy;
  const T* const skip = a.dsum ? static_cast<const T*>(a.dsum) + row * a.ldds : nullptr;
  const T* const wt = static_cast<const T*>(a.w);
  T* const dx = static_cast<T*>(a.dx) + row * a.lddx;
  const int first = (int)threadIdx.x * N - (EDGE ? (int)(reinterpret_cast<uintptr_t>(s) / sizeof(T) % N) : 0);
  auto at = [&](int i) { return first + i * kStep; };
  auto lo = [&](int i) { return EDGE ? -at(i) : 0; };
  auto hi = [&](int i) { return EDGE ? a.hidden - at(i) : N; };
  auto weights = [&](int i, float* w) {
    if (!wt) {
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = 1.0f;
    } else if (EDGE) {
      load_weights<Pc>(wt, at(i), a.hidden, w);
    } else {
      Pc::open(Pc::load(wt + at(i)), w);
    }
  };
  typename Pc::Raw vs[P], vy[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (at(i) >= a.hidden) continue;
    vs[i] = load_piece<Pc>(s + at(i), lo(i), hi(i));
    vy[i] = load_piece<Pc>(dy + at(i), lo(i), hi(i));
  }
  const float mean = a.mean[row], rstd = a.rstd[row];
  float sum_g = 0.0f, sum_gn = 0.0f;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (at(i) >= a.hidden) continue;
    float f[N], g[N], w[N];
    Pc::open(vs[i], f);
    Pc::open(vy[i], g);
    weights(i, w);
#pragma unroll
    for (int j = 0; j < N; ++j) {                              // elements around the row have dy of zero
      g[j] *= w[j];
      sum_g += g[j];
      if (EDGE && (j < lo(i) || j >= hi(i))) continue;         // but mean rstd may be infinite where no element of the row is
      sum_gn = fmaf(g[j], (f[j] - mean) * rstd, sum_gn);
    }
  }
  const float inverse = 1.0f / (float)a.hidden;
  const float c1 = cta_sum<kWideThreads / 32>(sum_g, shared[0]) * inverse, c2 = cta_sum<kWideThreads / 32>(sum_gn, shared[1]) * inverse;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (at(i) >= a.hidden) continue;
    float f[N], g[N], w[N];
    Pc::open(vs[i], f);
    Pc::open(vy[i], g);
    weights(i, w);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = rstd * (g[j] * w[j] - fmaf((f[j] - mean) * rstd, c2, c1));
    if (skip) {
      Pc::open(load_piece<Pc>(skip + at(i), lo(i), hi(i)), g);
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] += g[j];
    }
    store_piece<Pc>(dx + at(i), Pc::close(f), lo(i), hi(i));
  }
}

// dw and db from the sums of the CTAs: a warp's lanes take neighbouring columns, the warps of a CTA every kJoinWarps-th row of sums.
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) layer_norm_join_kernel(const float* partials, int parts, int hidden, float* dw, float* db) {
  __shared__ float sums[kJoinWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, padded = padded_hidden(hidden);
  const long long e = (long long)blockIdx.x * 32 + lane;
  next_may_launch();
  wait_for_previous();
  float s = 0.0f;
  if (e < 2ll * padded) {
#pragma unroll 8
    for (int i = warp; i < parts; i += kJoinWarps) s += __ldcg(partials + i * 2ll * padded + e);
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp) return;
#pragma unroll
  for (int i = 1; i < kJoinWarps; ++i) s += sums[i][lane];
  const long long column = e < padded ? e : e - padded;
  float* const out = e < padded ? dw : db;
  if (out && column < hidden && e < 2ll * padded) out[column] = s;
}

// How a gradient is computed: rows of a warp, rows of a CTA, or by columns and rows apart.  Threads have eight elements of a row, or
// sixteen of rows wider than 2048, and as many CTAs run as are resident at a time.
constexpr int kGradSmall = 64, kGradNarrow = 256, kGradWide = 512;   // threads of the CTAs that registers and shared memory are cut for
constexpr int kGradRows = 2;                                  // rows at a time, where threads have eight elements
constexpr int kSharedOfSm = 227 * 1024;
struct GradPlan { int threads, most, each, period; bool warp, apart, edge; long long parts; };
GradPlan grad_plan(const LayerNormGradArgs& a) {
  GradPlan p{};
  const int piece = 16 / a.size;
  p.edge = a.rows_at == kRowsAlike;
  const int span = a.hidden + (p.edge ? piece - 1 : 0);       // a shifted row's first piece begins before it
  p.period = 1;
  for (long long ld = a.lds; p.edge && ld * p.period % piece;) ++p.period;   // at most eight
  p.each = span <= 8 * kGradNarrow ? 8 : 16;
  p.apart = a.rows_at == kRowsAny || span > 16 * kGradWide;
  if (p.apart) {
    const int columns = a.rows_at == kRowsWhole ? 32 * piece : kColumns, of_cta = a.rows_at == kRowsWhole ? kStripWarps : kWalks;
    const long long strips = (a.hidden + columns - 1) / columns, walks = (a.rows + of_cta - 1) / of_cta;
    const long long most = (8ll * a.sms + strips - 1) / strips;
    p.parts = walks < most ? walks : most;
    return p;
  }
  p.warp = span <= 8 * 32;
  const int pieces = (span + piece - 1) / piece, of_thread = p.each / piece;
  p.threads = p.warp ? 32 * kGradWalks : ((pieces + of_thread - 1) / of_thread + 31) / 32 * 32;
  const int rows = p.each == 8 ? kGradRows : 1;
  p.most = p.threads <= kGradSmall ? kGradSmall : p.threads <= kGradNarrow ? kGradNarrow : kGradWide;
  const int bytes = p.most * kGradSlots * rows * 3 * of_thread * 16;
  int per_sm = kGradWide / p.most * (p.most / p.threads);
  if (per_sm > kSharedOfSm / (bytes + 2048)) per_sm = kSharedOfSm / (bytes + 2048);
  const int batch = rows * (p.warp ? kGradWalks : 1);
  const long long batches = (a.rows + batch - 1) / batch, most = (long long)per_sm * a.sms;
  // four batches to a CTA at least, if every multiprocessor has one all the same
  const long long few = batches / 4 > a.sms ? batches / 4 : batches < a.sms ? batches : a.sms;
  p.parts = few < most ? few : most;
  if (!p.warp) p.parts = (p.parts + p.period - 1) / p.period * p.period;   // as many walks of every kind of rows
  return p;
}

template <typename T, bool EDGE, bool WARP, int R, int Q, int MAX, int CTAS> cudaError_t start_grad(LayerNormGradArgs a, const GradPlan& p, cudaStream_t s) {
  a.period = p.period;
  const auto kernel = layer_norm_grad_kernel<T, EDGE, WARP, R, Q, MAX, CTAS>;
  constexpr int kBytes = MAX * kGradSlots * R * 3 * Q * 16;   // as grad_plan has it
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared(reinterpret_cast<const void*>(kernel), kBytes, allowed);
  if (e != cudaSuccess) return e;
  return launch(kernel, dim3((unsigned)p.parts), dim3(p.threads), kBytes, s, a);
}

template <typename T, bool EDGE> cudaError_t run_walks(const LayerNormGradArgs& a, const GradPlan& p, cudaStream_t s) {
  constexpr int kPiece = 16 / sizeof(T);
  if (p.warp) return start_grad<T, EDGE, true, kGradRows, 8 / kPiece, kGradNarrow, 2>(a, p, s);
  if (p.each == 8 && p.most == kGradSmall) return start_grad<T, EDGE, false, kGradRows, 8 / kPiece, kGradSmall, 8>(a, p, s);
  if (p.each == 8) return start_grad<T, EDGE, false, kGradRows, 8 / kPiece, kGradNarrow, 2>(a, p, s);
  if (p.most <= kGradNarrow) return start_grad<T, EDGE, false, 1, 16 / kPiece, kGradNarrow, 2>(a, p, s);
  return start_grad<T, EDGE, false, 1, 16 / kPiece, kGradWide, 1>(a, p, s);
}

template <typename T> cudaError_t run_grad(const LayerNormGradArgs& a, cudaStream_t s) {
  constexpr int kPiece = 16 / sizeof(T);
  const GradPlan p = grad_plan(a);
  const bool sums = a.dw || a.db;
  cudaError_t e = cudaSuccess;
  if (p.apart) {                                              // dw and db before dx, which may be dy or s
    if (sums && a.rows_at == kRowsWhole) {
      e = launch(layer_norm_strips_kernel<T>, dim3((unsigned)((a.hidden + 32 * kPiece - 1) / (32 * kPiece)), (unsigned)p.parts), dim3(32 * kStripWarps), 0, s, a);
    } else if (sums) {
      e = launch(layer_norm_columns_kernel<T>, dim3((unsigned)((a.hidden + kColumns - 1) / kColumns), (unsigned)p.parts), dim3(kColumns, kWalks), 0, s, a);
    }
    if (e == cudaSuccess && a.dx) {
      const bool whole = a.rows_at == kRowsWhole && a.hidden % kPiece == 0 && reinterpret_cast<uintptr_t>(a.w) % 16 == 0;
      const int span = a.hidden + kPiece - 1;
      const dim3 rows((unsigned)a.rows), threads(kWideThreads);
      // four pieces where they hold a row; binary32 rows that come here are wider
      constexpr int kFew = sizeof(T) == 2 ? 4 : 8, kFewSpan = kFew * kWideThreads * kPiece, kSpan = 8 * kWideThreads * kPiece;
      static_assert(sizeof(T) == 2 || 4 * kWideThreads * kPiece <= 16 * kGradWide, "rows of four binary32 pieces go by the other kernel");
      if (whole && a.hidden <= kFewSpan) e = launch(layer_norm_wide_kernel<T, false, kFew>, rows, threads, 0, s, a);
      else if (whole && a.hidden <= kSpan) e = launch(layer_norm_wide_kernel<T, false, 8>, rows, threads, 0, s, a);
      else if (a.rows_at != kRowsAny && span <= kFewSpan) e = launch(layer_norm_wide_kernel<T, true, kFew>, rows, threads, 0, s, a);
      else if (a.rows_at != kRowsAny && span <= kSpan) e = launch(layer_norm_wide_kernel<T, true, 8>, rows, threads, 0, s, a);
      else e = launch(layer_norm_rows_kernel<T>, dim3((unsigned)a.rows), dim3(kRowThreads), 0, s, a);
    }
  } else {
    e = p.edge ? run_walks<T, true>(a, p, s) : run_walks<T, false>(a, p, s);
  }
  if (e != cudaSuccess || !sums) return e;
  return launch(layer_norm_join_kernel, dim3((unsigned)((2ll * padded_hidden(a.hidden) + 31) / 32)), dim3(32 * kJoinWarps), 0, s, (const float*)a.partials, (int)p.parts, a.hidden, a.dw, a.db);
}

}  // namespace

cudaError_t launch_layer_norm(int dtype, const LayerNormArgs& a, cudaStream_t s) {
  if (dtype == AQ_FP16) return run_forward<__half>(a, s);
  if (dtype == AQ_BF16) return run_forward<__nv_bfloat16>(a, s);
  return run_forward<float>(a, s);
}
long long layer_norm_grad_bytes(const LayerNormGradArgs& a) { return grad_plan(a).parts * 2 * padded_hidden(a.hidden) * (long long)sizeof(float); }
cudaError_t launch_layer_norm_grad(int dtype, const LayerNormGradArgs& a, cudaStream_t s) {
  if (dtype == AQ_FP16) return run_grad<__half>(a, s);
  if (dtype == AQ_BF16) return run_grad<__nv_bfloat16>(a, s);
  return run_grad<float>(a, s);
}

}  // namespace aq
