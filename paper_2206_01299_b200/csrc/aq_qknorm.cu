// RMS norm of query and key heads with the position rotation, and the gradient.
//
//   y = w x r,  r = 1 / sqrt(mean x^2 + eps);   o_e = y_e cos_e + y_partner(e) sn_e
// where an element's factors are cos_i and -sin_i (first member of its pair), cos_i and +sin_i (second), or 1 and 0
// (not rotated).  The gradient turns back with -sn and then, with n = x r and g = w dy,
//   dx = r (g - n mean(g n)),   dw = sum over rows and heads of dy n.
//
// Bound by memory: 2 T per element forward, 3 T backward, and a position's factors once per token.  A warp takes one
// token; the lanes of a head are the next power of two of its 16-byte pieces, so a warp holds 32 / lanes heads at a time
// and every lane keeps the same elements of all of them: their weights and rotation factors are loaded once per token.

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/aq_b200.h"
#include "aq_stage.h"

namespace aq {
namespace {

constexpr int kQkThreads = 256, kQkWarps = kQkThreads / 32;
constexpr int kInFlight = 4;                  // passes whose loads are issued together

template <typename T> struct Half2;
template <> struct Half2<__half> {
  static __device__ float2 open(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
  static __device__ uint32_t close(float a, float b) { const __half2 p = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&p); }
};
template <> struct Half2<__nv_bfloat16> {
  static __device__ float2 open(uint32_t u) { return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
  static __device__ uint32_t close(float a, float b) { const __nv_bfloat162 p = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&p); }
};
template <typename T> __device__ void open8(uint4 v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 p = Half2<T>::open(w[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
}
template <typename T> __device__ uint4 close8(const float* f) {
  return make_uint4(Half2<T>::close(f[0], f[1]), Half2<T>::close(f[2], f[3]), Half2<T>::close(f[4], f[5]), Half2<T>::close(f[6], f[7]));
}

// how a lane reaches the other members of its pairs
enum { kPairsInLane = 0, kPairsByShuffle = 1, kPairsByShared = 2 };

// One lane's view of its token: which elements of a head it holds, and their factors.
template <typename T, int W, int MODE>
struct Lane {
  int lane, piece, slot;                      // 16-byte piece of the head; head within the pass
  bool holds;
  int partner;                                // kPairsByShuffle: lane of the pairs' other members
  float cs[8], sn[8];
  float* shared;                              // kPairsByShared: 256 floats of this warp

  __device__ Lane(const QkArgs& a, float* sh) {
    lane = threadIdx.x & 31;
    piece = lane & (W - 1);
    slot = lane / W;
    holds = piece < a.head_dim / 8;
    shared = sh;
    const int step = a.rot_dim / 16;          // pieces between the members of a pair
    partner = lane;
    if (MODE == kPairsByShuffle && piece < 2 * step) partner = lane + (piece < step ? step : -step);
  }
  __device__ void factors(const QkArgs& a, int position) {
    const float* const table = a.cos_sin + (long long)position * a.rot_dim;
    const int half = a.rot_dim / 2;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = piece * 8 + j;
      cs[j] = 1.0f;
      sn[j] = 0.0f;
      if (holds && e < a.rot_dim) {
        const bool second = a.interleaved ? e & 1 : e >= half;
        const int i = a.interleaved ? e >> 1 : second ? e - half : e;
        cs[j] = __ldg(table + i);
        const float s = __ldg(table + half + i);
        sn[j] = second ? s : -s;
      }
    }
  }
  // y_e cos_e + y_partner(e) sn_e * sign
  __device__ void rotate(const QkArgs& a, float* y, float sign) {
    float other[8];
    if (MODE == kPairsInLane) {
#pragma unroll
      for (int j = 0; j < 8; ++j) other[j] = y[j ^ 1];
    } else if (MODE == kPairsByShuffle) {
#pragma unroll
      for (int j = 0; j < 8; ++j) other[j] = __shfl_sync(0xffffffffu, y[j], partner);
    } else {
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 8; ++j) shared[lane * 8 + j] = y[j];
      __syncwarp();
      const int half = a.rot_dim / 2;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = piece * 8 + j;
        const int to = e >= a.rot_dim ? e : e < half ? e + half : e - half;
        other[j] = shared[slot * W * 8 + to];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = fmaf(y[j], cs[j], other[j] * (sn[j] * sign));
  }
};

template <int W> __device__ float sum_over_head(float x) {
#pragma unroll
  for (int o = W / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

template <typename T> __device__ void load_weights(const void* w, int piece, bool holds, float* f) {
  if (w && holds) {
    open8<T>(__ldg(static_cast<const uint4*>(w) + piece), f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 1.0f;
  }
}

// Position of a token; -1 and the status bit when it is outside the table.
__device__ int position_of(const QkArgs& a, long long token) {
  if (!a.rot_dim) return 0;
  const int p = a.positions[token];
  if (p >= 0 && p < a.n_positions) return p;
  if ((threadIdx.x & 31) == 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
  return -1;
}

// Passes [p0, p1) over the heads of one tensor of one token.
template <typename T, int W, int MODE>
__device__ void forward_heads(const QkArgs& a, Lane<T, W, MODE>& l, const void* in, void* out, int heads, const float* w, bool valid, int p0, int p1) {
  const uint4* const src = static_cast<const uint4*>(in);
  uint4* const dst = static_cast<uint4*>(out);
  const int pieces = a.head_dim / 8;
  const float inv = 1.0f / (float)a.head_dim;
  for (int p = p0; p < p1; p += kInFlight) {
    uint4 v[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int head = (p + i) * (32 / W) + l.slot;
      v[i] = make_uint4(0, 0, 0, 0);
      if (p + i < p1 && head < heads && l.holds) v[i] = __ldcs(src + head * pieces + l.piece);
    }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (p + i >= p1) break;
      const int head = (p + i) * (32 / W) + l.slot;
      float y[8], ss = 0.0f;
      open8<T>(v[i], y);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(y[j], y[j], ss);
      const float r = rsqrtf(fmaf(sum_over_head<W>(ss), inv, a.eps));
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] *= r * w[j];
      l.rotate(a, y, 1.0f);
      if (head < heads && l.holds) dst[head * pieces + l.piece] = valid ? close8<T>(y) : make_uint4(0, 0, 0, 0);
    }
  }
}

template <typename T, int W, int MODE>
__global__ void __launch_bounds__(kQkThreads) qk_kernel(const QkArgs a, int splits, int passes_per_task) {
  __shared__ float exchange[MODE == kPairsByShared ? kQkWarps * 256 : 1];
  const long long task = (long long)blockIdx.x * kQkWarps + threadIdx.x / 32;
  const long long token = task / splits;
  if (token >= a.rows) return;
  const int passes_q = (a.heads_q + 32 / W - 1) / (32 / W), passes = passes_q + (a.heads_k + 32 / W - 1) / (32 / W);
  const int p0 = (int)(task % splits) * passes_per_task, p1 = min(p0 + passes_per_task, passes);
  Lane<T, W, MODE> l(a, exchange + (MODE == kPairsByShared ? (threadIdx.x / 32) * 256 : 0));
  const int position = position_of(a, token);
  l.factors(a, max(position, 0));
  float w[8];
  if (p0 < passes_q) {
    load_weights<T>(a.wq, l.piece, l.holds, w);
    forward_heads<T, W, MODE>(a, l, static_cast<const T*>(a.q) + token * a.q_stride, static_cast<T*>(a.q_out) + token * a.q_out_stride,
                              a.heads_q, w, position >= 0, p0, min(p1, passes_q));
  }
  if (p1 > passes_q) {
    load_weights<T>(a.wk, l.piece, l.holds, w);
    forward_heads<T, W, MODE>(a, l, static_cast<const T*>(a.k) + token * a.k_stride, static_cast<T*>(a.k_out) + token * a.k_out_stride,
                              a.heads_k, w, position >= 0, max(p0 - passes_q, 0), p1 - passes_q);
  }
}

// ---- gradient ------------------------------------------------------------------------------------------------

template <typename T, int W, int MODE>
__device__ void backward_heads(const QkArgs& a, Lane<T, W, MODE>& l, const void* in, const void* grad, void* out, int heads, const float* w,
                               float* dw, bool valid) {
  const uint4* const src = static_cast<const uint4*>(in);
  const uint4* const gsrc = static_cast<const uint4*>(grad);
  uint4* const dst = static_cast<uint4*>(out);
  const int pieces = a.head_dim / 8;
  const float inv = 1.0f / (float)a.head_dim;
  const int passes = (heads + 32 / W - 1) / (32 / W);
  constexpr int U = kInFlight / 2;
  for (int p = 0; p < passes; p += U) {
    uint4 v[U], g[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int head = (p + i) * (32 / W) + l.slot;
      v[i] = g[i] = make_uint4(0, 0, 0, 0);
      if (head < heads && l.holds) { v[i] = __ldcs(src + head * pieces + l.piece); g[i] = __ldcs(gsrc + head * pieces + l.piece); }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (p + i >= passes) break;
      const int head = (p + i) * (32 / W) + l.slot;
      const bool mine = head < heads && l.holds;
      float n[8], dy[8], ss = 0.0f, dot = 0.0f;
      open8<T>(v[i], n);
      open8<T>(g[i], dy);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(n[j], n[j], ss);
      const float r = rsqrtf(fmaf(sum_over_head<W>(ss), inv, a.eps));
      l.rotate(a, dy, -1.0f);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[j] *= r;
        if (mine && valid) dw[j] = fmaf(dy[j], n[j], dw[j]);
        dy[j] *= w[j];
        dot = fmaf(dy[j], n[j], dot);
      }
      const float mean = sum_over_head<W>(dot) * inv;
#pragma unroll
      for (int j = 0; j < 8; ++j) dy[j] = r * (dy[j] - n[j] * mean);
      if (mine) dst[head * pieces + l.piece] = valid ? close8<T>(dy) : make_uint4(0, 0, 0, 0);
    }
  }
}

template <typename T, int W, int MODE>
__global__ void __launch_bounds__(kQkThreads) qk_grad_kernel(const QkArgs a) {
  __shared__ float exchange[MODE == kPairsByShared ? kQkWarps * 256 : 1];
  __shared__ float sums[kQkWarps][2][256];
  __shared__ bool last;
  const int warp = threadIdx.x / 32, tid = threadIdx.x;
  Lane<T, W, MODE> l(a, exchange + (MODE == kPairsByShared ? warp * 256 : 0));
  float wq[8], wk[8], dwq[8] = {}, dwk[8] = {};
  load_weights<T>(a.wq, l.piece, l.holds, wq);
  load_weights<T>(a.wk, l.piece, l.holds, wk);
  for (long long token = (long long)blockIdx.x * kQkWarps + warp; token < a.rows; token += (long long)gridDim.x * kQkWarps) {
    const int position = position_of(a, token);
    l.factors(a, max(position, 0));
    backward_heads<T, W, MODE>(a, l, static_cast<const T*>(a.q) + token * a.q_stride, static_cast<const T*>(a.gq) + token * a.gq_stride,
                               static_cast<T*>(a.q_out) + token * a.q_out_stride, a.heads_q, wq, dwq, position >= 0);
    backward_heads<T, W, MODE>(a, l, static_cast<const T*>(a.k) + token * a.k_stride, static_cast<const T*>(a.gk) + token * a.gk_stride,
                               static_cast<T*>(a.k_out) + token * a.k_out_stride, a.heads_k, wk, dwk, position >= 0);
  }
  // the sums of dw: heads of a warp, warps of a CTA, then CTAs, each in a fixed order
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int o = 16; o >= W; o >>= 1) {
      dwq[j] += __shfl_xor_sync(0xffffffffu, dwq[j], o);
      dwk[j] += __shfl_xor_sync(0xffffffffu, dwk[j], o);
    }
    if (l.slot == 0) { sums[warp][0][l.piece * 8 + j] = dwq[j]; sums[warp][1][l.piece * 8 + j] = dwk[j]; }
  }
  __syncthreads();
  float* const mine = a.partials + (long long)blockIdx.x * 512;
  for (int i = tid; i < 2 * a.head_dim; i += kQkThreads) {
    const int t = i / a.head_dim, e = i % a.head_dim;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kQkWarps; ++w) s += sums[w][t][e];
    mine[t * 256 + e] = s;
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  for (int i = tid; i < 2 * a.head_dim; i += kQkThreads) {
    const int t = i / a.head_dim, e = i % a.head_dim;
    float s = 0.0f;
    for (unsigned b = 0; b < gridDim.x; ++b) s += __ldcg(a.partials + (long long)b * 512 + t * 256 + e);
    float* const out = t ? a.dwk : a.dwq;
    if (out) out[e] = s;
  }
  if (tid == 0) *a.ticket = 0;
}

template <typename T, int W, int MODE>
cudaError_t run(const QkArgs& a, bool backward, cudaStream_t s) {
  const int per_pass = 32 / W;
  if (backward) {
    const long long ctas = (a.rows + kQkWarps - 1) / kQkWarps, most = 4ll * a.sms < kQkGradCtas ? 4ll * a.sms : kQkGradCtas;
    qk_grad_kernel<T, W, MODE><<<(unsigned)(ctas < most ? ctas : most), kQkThreads, 0, s>>>(a);
    return cudaGetLastError();
  }
  const int passes = (a.heads_q + per_pass - 1) / per_pass + (a.heads_k + per_pass - 1) / per_pass;
  // few tokens: several warps share one, down to a pass each, until every multiprocessor has sixteen warps
  int per_task = passes;
  while (per_task > 1 && a.rows * ((passes + per_task - 1) / per_task) < 16ll * a.sms) per_task = (per_task + 1) / 2;
  const int splits = (passes + per_task - 1) / per_task;
  const long long ctas = (a.rows * splits + kQkWarps - 1) / kQkWarps;
  qk_kernel<T, W, MODE><<<(unsigned)ctas, kQkThreads, 0, s>>>(a, splits, per_task);
  return cudaGetLastError();
}

template <typename T, int W>
cudaError_t run_mode(const QkArgs& a, bool backward, cudaStream_t s) {
  if (a.interleaved || a.rot_dim == 0) return run<T, W, kPairsInLane>(a, backward, s);
  if (a.rot_dim % 16 == 0) return run<T, W, kPairsByShuffle>(a, backward, s);
  return run<T, W, kPairsByShared>(a, backward, s);          // half a rotation is no whole number of 16-byte pieces
}

template <typename T>
cudaError_t run_lanes(const QkArgs& a, bool backward, cudaStream_t s) {
  const int pieces = a.head_dim / 8;
  if (pieces <= 4) return run_mode<T, 4>(a, backward, s);
  if (pieces <= 8) return run_mode<T, 8>(a, backward, s);
  if (pieces <= 16) return run_mode<T, 16>(a, backward, s);
  return run_mode<T, 32>(a, backward, s);
}

}  // namespace

cudaError_t launch_qk(int dtype, const QkArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_lanes<__half>(a, false, s) : run_lanes<__nv_bfloat16>(a, false, s);
}
cudaError_t launch_qk_grad(int dtype, const QkArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_lanes<__half>(a, true, s) : run_lanes<__nv_bfloat16>(a, true, s);
}

}  // namespace aq
