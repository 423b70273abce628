// RMS norm of query and key heads with the position rotation, and the gradient.
//
//   y = w x r,  r = 1 / sqrt(mean x^2 + eps);   o_e = y_e cos_e + y_partner(e) sn_e
// where an element's factors are cos_i and -sin_i (first member of its pair), cos_i and +sin_i (second), or 1 and 0
// (not rotated).  The gradient turns back with -sn and then, with n = x r and g = w dy,
//   dx = r (g - n mean(g n)),   dw = sum over rows and heads of dy n.
//
// The lanes of a head are the next power of two of its 16-byte pieces, so a warp holds 32 / lanes heads at a time (a pass) and
// every lane keeps the same elements of all of them: their weights and factors are formed once, as a_e = w_e cos_e and
// b_e = w_partner sn_e, and a head costs o_e = r (a_e x_e + b_e x_partner).  Partners are exchanged as they were loaded, two
// values a word.  A warp's loads are all issued before it waits for its token's position.
//
// Bound by memory in the first place, 2 T per element forward and 3 T backward and a position's factors once per token, with the
// issue of instructions (about 15 per element) close behind.  Forward, 32768 tokens of 25 + 25 heads of 64: 77 to 82 us, 5.1 to
// 5.4 TB/s (issue slots 0.73 under a profiler); backward, 16384 tokens of 24 + 8 heads of 64: 50.5 us, 4.0 TB/s (issue slots 0.62, 16 warps).  What did not help: two pieces a lane, which spares the exchange
// but doubles the registers (92 us, 68 us); rings in shared memory filled by bulk copies (81 us, 72 us) or, backward, by
// asynchronous copies (56 us); instructions on pairs of binary32 values.

#include "aq_stage.h"
#include "aq_stage_device.cuh"

namespace aq {
namespace {

constexpr int kQkThreads = 256, kQkWarps = kQkThreads / 32;
constexpr int kCtas = 4, kGradCtas = 2;       // CTAs on a multiprocessor that the registers are cut for
// Passes of a forward warp at most, whose loads are all in flight: seven are what 64 registers hold.  At 32768 tokens of 50
// heads of 64, 77 us; with eight 84 us (three CTAs) or 86 us (four, spilling), with four 94 us (a token's factors are formed
// again for every batch).
constexpr int kPasses = 7;
constexpr int kGradPasses = 2;                // ... of a backward warp at a time, two loads each, and the next ones': 55 us at 16384 tokens of
                                              // 32 heads of 64; with one 70 us, with three 59 us

template <typename T> __device__ void open8(uint4 v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 p = Num<T>::open(w[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
}
template <typename T> __device__ uint4 close8(const float* f) {
  return make_uint4(Num<T>::close(f[0], f[1]), Num<T>::close(f[2], f[3]), Num<T>::close(f[4], f[5]), Num<T>::close(f[6], f[7]));
}

// how a lane reaches the other members of its pairs
enum { kPairsInLane = 0, kPairsByShuffle = 1, kPairsByShared = 2 };

// Which elements of a head a lane holds, and where their partners are.
template <typename T, int W, int MODE>
struct Lane {
  int lane, piece, slot;                      // 16-byte piece of the head; head within the pass
  bool holds;
  int partner;                                // kPairsByShuffle: lane of the pairs' other members
  int half;
  T* shared;                                  // kPairsByShared: 256 values of this warp, and where in them the partners of
  int at[4];                                  // two neighbouring elements begin (half a rotation of an even number of elements)

  __device__ Lane(const QkArgs& a, T* sh) {
    lane = threadIdx.x & 31;
    piece = lane & (W - 1);
    slot = lane / W;
    holds = piece < a.head_dim / 8;
    shared = sh;
    half = a.rot_dim / 2;
    const int step = a.rot_dim / 16;          // pieces between the members of a pair
    partner = lane;
    if (MODE == kPairsByShuffle && piece < 2 * step) partner = lane + (piece < step ? step : -step);
    if (MODE == kPairsByShared) {
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j] = slot * W * 8 + partner_of(a, piece * 8 + 2 * j);
    }
  }
  __device__ int partner_of(const QkArgs& a, int e) const {
    if (e >= a.rot_dim) return e;
    return a.interleaved ? e ^ 1 : e < half ? e + half : e - half;
  }
  // cs, sn: factors of the lane's elements
  __device__ void factors(const QkArgs& a, int position, float* cs, float* sn) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) { cs[j] = 1.0f; sn[j] = 0.0f; }
    const int e0 = piece * 8;
    if (e0 >= a.rot_dim) return;
    const float* const table = a.cos_sin + (long long)position * a.rot_dim;
    if (MODE == kPairsByShuffle) {            // whole pieces: eight consecutive pairs, all first or all second members
      const bool second = e0 >= half;
      const float4* const c = reinterpret_cast<const float4*>(table + (second ? e0 - half : e0));
      const float4* const s = reinterpret_cast<const float4*>(table + (second ? e0 : e0 + half));
      const float4 c0 = __ldg(c), c1 = __ldg(c + 1), s0 = __ldg(s), s1 = __ldg(s + 1);
      const float sign = second ? 1.0f : -1.0f;
      cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
      sn[0] = sign * s0.x; sn[1] = sign * s0.y; sn[2] = sign * s0.z; sn[3] = sign * s0.w;
      sn[4] = sign * s1.x; sn[5] = sign * s1.y; sn[6] = sign * s1.z; sn[7] = sign * s1.w;
      return;
    }
    if (MODE == kPairsInLane && a.rot_dim % 8 == 0) {   // four consecutive pairs
      const float4 c = __ldg(reinterpret_cast<const float4*>(table + e0 / 2)), s = __ldg(reinterpret_cast<const float4*>(table + half + e0 / 2));
      cs[0] = cs[1] = c.x; cs[2] = cs[3] = c.y; cs[4] = cs[5] = c.z; cs[6] = cs[7] = c.w;
      sn[0] = -s.x; sn[1] = s.x; sn[2] = -s.y; sn[3] = s.y; sn[4] = -s.z; sn[5] = s.z; sn[6] = -s.w; sn[7] = s.w;
      return;
    }
    if (MODE == kPairsByShared && half % 2 == 0) {      // two consecutive pairs
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const int e = e0 + j;
        if (e >= a.rot_dim) break;
        const bool second = e >= half;
        const float2 c = __ldg(reinterpret_cast<const float2*>(table + (second ? e - half : e))), s = __ldg(reinterpret_cast<const float2*>(table + (second ? e : e + half)));
        cs[j] = c.x;
        cs[j + 1] = c.y;
        sn[j] = second ? s.x : -s.x;
        sn[j + 1] = second ? s.y : -s.y;
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = e0 + j;
      if (e >= a.rot_dim) break;
      const bool second = a.interleaved ? e & 1 : e >= half;
      const int i = a.interleaved ? e >> 1 : second ? e - half : e;
      cs[j] = __ldg(table + i);
      const float s = __ldg(table + half + i);
      sn[j] = second ? s : -s;
    }
  }
  // values of the partners of a lane's elements; x: the lane's own
  __device__ void partners(const QkArgs& a, uint4 v, const float* x, float* xp) const {
    if (MODE == kPairsInLane) {
#pragma unroll
      for (int j = 0; j < 8; ++j) xp[j] = x[j ^ 1];
    } else if (MODE == kPairsByShuffle) {
      uint4 o;
      o.x = __shfl_sync(0xffffffffu, v.x, partner);
      o.y = __shfl_sync(0xffffffffu, v.y, partner);
      o.z = __shfl_sync(0xffffffffu, v.z, partner);
      o.w = __shfl_sync(0xffffffffu, v.w, partner);
      open8<T>(o, xp);
    } else {
      __syncwarp();
      reinterpret_cast<uint4*>(shared)[lane] = v;
      __syncwarp();
      if (half % 2 == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = Num<T>::open(*reinterpret_cast<const uint32_t*>(shared + at[j]));
          xp[2 * j] = f.x;
          xp[2 * j + 1] = f.y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) xp[j] = (float)shared[slot * W * 8 + partner_of(a, piece * 8 + j)];
      }
    }
  }
};

template <int W> __device__ float sum_over_head(float x) {
#pragma unroll
  for (int o = W / 2; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// weights of the lane's elements
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
  const int p = __ldg(a.positions + token);
  if (p >= 0 && p < a.n_positions) return p;
  if ((threadIdx.x & 31) == 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
  return -1;
}

__device__ float inverse_root(float x) { float y; asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// blockIdx.y: a batch of `per` passes of the queries' heads (the first batches_q) or the keys'
template <typename T, int W, int MODE>
__global__ void __launch_bounds__(kQkThreads, MODE == kPairsByShared ? kCtas - 1 : kCtas) qk_kernel(const QkArgs a, int batches_q, int per) {
  __shared__ __align__(16) T exchange[MODE == kPairsByShared ? kQkWarps * 256 : 8];
  constexpr int H = 32 / W;
  const long long token = (long long)blockIdx.x * kQkWarps + threadIdx.x / 32;
  next_may_launch();
  wait_for_previous();
  if (token >= a.rows) return;
  const bool keys = (int)blockIdx.y >= batches_q;
  const int heads = keys ? a.heads_k : a.heads_q, pieces = a.head_dim / 8;
  const int p0 = ((int)blockIdx.y - (keys ? batches_q : 0)) * per, passes = min(per, (heads - p0 * H + H - 1) / H);
  const Lane<T, W, MODE> l(a, exchange + (MODE == kPairsByShared ? (threadIdx.x / 32) * 256 : 0));
  // 16-byte pieces of the row; a lane without one in a pass reads the row's last and stores nothing
  const int step = H * pieces, last = heads * pieces - 1, at = (p0 * H + l.slot) * pieces + l.piece;
  const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const T*>(keys ? a.k : a.q) + token * (keys ? a.k_stride : a.q_stride));
  uint4* const dst = reinterpret_cast<uint4*>(static_cast<T*>(keys ? a.k_out : a.q_out) + token * (keys ? a.k_out_stride : a.q_out_stride));
  uint4 v[kPasses];
#pragma unroll
  for (int i = 0; i < kPasses; ++i)
    if (i < passes) v[i] = __ldcs(src + min(at + i * step, last));
  const int position = position_of(a, token);
  if (position < 0) {
    for (int i = 0; i < passes; ++i)
      if (l.holds && at + i * step <= last) dst[at + i * step] = make_uint4(0, 0, 0, 0);
    return;
  }
  float fa[8], fb[8];
  l.factors(a, position, fa, fb);
  const void* const weights = keys ? a.wk : a.wq;
  if (weights) {
    float w[8], wp[8];
    load_weights<T>(weights, l.piece, l.holds, w);
    if (MODE == kPairsInLane) {
#pragma unroll
      for (int j = 0; j < 8; ++j) wp[j] = w[j ^ 1];
    } else if (MODE == kPairsByShuffle) {
      load_weights<T>(weights, l.partner & (W - 1), l.holds, wp);
    } else {
      const T* const w0 = static_cast<const T*>(weights);
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const int e = l.piece * 8 + j, to = l.holds ? l.partner_of(a, e) : 0, to1 = l.holds ? l.partner_of(a, e + 1) : 0;
        if (l.half % 2 == 0) {
          const float2 f = Num<T>::open(__ldg(reinterpret_cast<const uint32_t*>(w0 + to)));
          wp[j] = f.x;
          wp[j + 1] = f.y;
        } else {
          wp[j] = (float)w0[to];
          wp[j + 1] = (float)w0[to1];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) { fa[j] *= w[j]; fb[j] *= wp[j]; }
  }
  const float inv = 1.0f / (float)a.head_dim;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    if (i >= passes) break;
    float x[8], xp[8], ss = 0.0f;
    open8<T>(v[i], x);
    l.partners(a, v[i], x, xp);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(x[j], x[j], ss);
    const float r = inverse_root(fmaf(sum_over_head<W>(l.holds ? ss : 0.0f), inv, a.eps));
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = r * fmaf(fa[j], x[j], fb[j] * xp[j]);
    if (l.holds && at + i * step <= last) dst[at + i * step] = close8<T>(o);
  }
}

// ---- gradient ------------------------------------------------------------------------------------------------

// CTAs [0, ctas_q) take the queries' heads, the others the keys'.  A warp walks over tokens, kGradPasses passes at a time, the
// next ones on their way while these are worked on.
template <typename T, int W, int MODE>
__global__ void __launch_bounds__(kQkThreads, kGradCtas) qk_grad_kernel(const QkArgs a, int ctas_q) {
  __shared__ __align__(16) T exchange[MODE == kPairsByShared ? kQkWarps * 256 : 8];
  __shared__ float sums[kQkWarps][256];
  __shared__ float4 joined[kQkThreads];
  __shared__ bool last_cta;
  constexpr int H = 32 / W, U = kGradPasses;
  const int warp = threadIdx.x / 32, tid = threadIdx.x;
  next_may_launch();
  wait_for_previous();
  const bool keys = (int)blockIdx.x >= ctas_q;
  const int heads = keys ? a.heads_k : a.heads_q, pieces = a.head_dim / 8;
  const int cta = (int)blockIdx.x - (keys ? ctas_q : 0), ctas = keys ? (int)gridDim.x - ctas_q : ctas_q;
  const Lane<T, W, MODE> l(a, exchange + (MODE == kPairsByShared ? warp * 256 : 0));
  float w[8], dw[8] = {};
  load_weights<T>(keys ? a.wk : a.wq, l.piece, l.holds, w);
  const int passes = (heads + H - 1) / H, step = H * pieces, last = heads * pieces - 1, at = l.slot * pieces + l.piece;
  const float inv = 1.0f / (float)a.head_dim;
  const T* const x_rows = static_cast<const T*>(keys ? a.k : a.q);
  const T* const g_rows = static_cast<const T*>(keys ? a.gk : a.gq);
  T* const o_rows = static_cast<T*>(keys ? a.k_out : a.q_out);
  const long long x_stride = keys ? a.k_stride : a.q_stride, g_stride = keys ? a.gk_stride : a.gq_stride, o_stride = keys ? a.k_out_stride : a.q_out_stride;
  const long long stride = (long long)ctas * kQkWarps;
  long long token = (long long)cta * kQkWarps + warp;
  uint4 nv[U], ng[U];
  int next_position = 0;
  auto load = [&](long long t, int p) {
    const uint4* const src = reinterpret_cast<const uint4*>(x_rows + t * x_stride);
    const uint4* const gsrc = reinterpret_cast<const uint4*>(g_rows + t * g_stride);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int from = min(at + (p + i) * step, last);         // a lane without a piece reads the row's last and uses nothing of it
      nv[i] = __ldcs(src + from);
      ng[i] = __ldcs(gsrc + from);
    }
    if (p == 0 && a.rot_dim) next_position = __ldg(a.positions + t);
  };
  if (token < a.rows) load(token, 0);
  float cs[8], sn[8];
  for (; token < a.rows; token += stride) {
    int position = 0;
    if (a.rot_dim) {
      position = next_position;
      if (position < 0 || position >= a.n_positions) {
        if ((tid & 31) == 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
        position = -1;
      }
    }
    l.factors(a, max(position, 0), cs, sn);
    uint4* const dst = reinterpret_cast<uint4*>(o_rows + token * o_stride);
    for (int p = 0; p < passes; p += U) {
      uint4 v[U], g[U];
#pragma unroll
      for (int i = 0; i < U; ++i) { v[i] = nv[i]; g[i] = ng[i]; }
      if (p + U < passes) load(token, p + U);
      else if (token + stride < a.rows) load(token + stride, 0);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (p + i >= passes) break;
        float x[8], dy[8], dyp[8], ss = 0.0f, dot = 0.0f;
        open8<T>(v[i], x);
        open8<T>(g[i], dy);
        l.partners(a, g[i], dy, dyp);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dy[j] = fmaf(dy[j], cs[j], -dyp[j] * sn[j]);           // turned back
          ss = fmaf(x[j], x[j], ss);
          dyp[j] = dy[j] * w[j];
          dot = fmaf(dyp[j], x[j], dot);
        }
        const bool mine = l.holds && at + (p + i) * step <= last;
        const float r = inverse_root(fmaf(sum_over_head<W>(l.holds ? ss : 0.0f), inv, a.eps));
        const float mean = sum_over_head<W>(l.holds ? dot : 0.0f) * inv * r * r * r;
        const bool counts = mine && position >= 0;               // what does not may be NaN or infinite: left out, not times 0
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          dw[j] = counts ? fmaf(dy[j] * r, x[j], dw[j]) : dw[j];
          dyp[j] = fmaf(dyp[j], r, -x[j] * mean);
        }
        if (mine) dst[at + (p + i) * step] = position >= 0 ? close8<T>(dyp) : make_uint4(0, 0, 0, 0);
      }
    }
  }
  // the sums of dw: heads of a warp, warps of a CTA, then CTAs, each in a fixed order
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int o = 16; o >= W; o >>= 1) dw[j] += __shfl_xor_sync(0xffffffffu, dw[j], o);
    if (l.slot == 0) sums[warp][l.piece * 8 + j] = dw[j];
  }
  __syncthreads();
  if (tid < a.head_dim) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kQkWarps; ++i) s += sums[i][tid];
    a.partials[(long long)blockIdx.x * 256 + tid] = s;
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) last_cta = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last_cta) return;
  __threadfence();
  // the last CTA: a thread has four columns of every n-th CTA's sums; the threads of a column then join
  const int columns = a.head_dim / 4, n = kQkThreads / columns, column = tid % columns, row = tid / columns;
  for (int t = 0; t < 2; ++t) {
    const int from = t ? ctas_q : 0, to = t ? (int)gridDim.x : ctas_q;
    float4 s = make_float4(0, 0, 0, 0);
    if (row < n) {
#pragma unroll 8
      for (int b = from + row; b < to; b += n) {
        const float4 o = __ldcg(reinterpret_cast<const float4*>(a.partials + (long long)b * 256) + column);
        s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
      }
    }
    joined[tid] = s;
    __syncthreads();
    float* const out = t ? a.dwk : a.dwq;
    if (row == 0 && out) {
      for (int i = 1; i < n; ++i) {
        const float4 o = joined[i * columns + column];
        s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
      }
      out[column * 4] = s.x; out[column * 4 + 1] = s.y; out[column * 4 + 2] = s.z; out[column * 4 + 3] = s.w;
    }
    __syncthreads();
  }
  if (tid == 0) *a.ticket = 0;
}

template <typename T, int W, int MODE>
cudaError_t run(const QkArgs& a, bool backward, cudaStream_t s) {
  constexpr int H = 32 / W;
  const int passes_q = (a.heads_q + H - 1) / H, passes_k = (a.heads_k + H - 1) / H;
  const long long token_ctas = (a.rows + kQkWarps - 1) / kQkWarps;
  if (backward) {
    // one wave of CTAs, shared between queries and keys by their passes
    const int most = kGradCtas * a.sms < kQkGradCtas ? kGradCtas * a.sms : kQkGradCtas;
    int nq = passes_q ? (int)((long long)most * passes_q / (passes_q + passes_k)) : 0;
    if (passes_q && nq < 1) nq = 1;
    if (passes_k && nq > most - 1) nq = most - 1;
    int nk = passes_k ? most - nq : 0;
    if (nq > token_ctas) nq = (int)token_ctas;
    if (nk > token_ctas) nk = (int)token_ctas;
    return launch(qk_grad_kernel<T, W, MODE>, dim3((unsigned)(nq + nk)), kQkThreads, 0, s, a, nq);
  }
  // batches of as equal a number of passes as possible; few tokens: smaller ones, down to a pass each, until every
  // multiprocessor has sixteen warps
  auto batches = [&](int passes, int per) { return (passes + per - 1) / per; };
  const int longest = passes_q > passes_k ? passes_q : passes_k;
  int per = (longest + batches(longest, kPasses) - 1) / batches(longest, kPasses);
  while (per > 1 && a.rows * (batches(passes_q, per) + batches(passes_k, per)) < 16ll * a.sms) per = (per + 1) / 2;
  const int nq = batches(passes_q, per), nk = batches(passes_k, per);
  return launch(qk_kernel<T, W, MODE>, dim3((unsigned)token_ctas, (unsigned)(nq + nk)), kQkThreads, 0, s, a, nq, per);
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
