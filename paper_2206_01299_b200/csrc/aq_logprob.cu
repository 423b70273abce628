// Log probabilities of given tokens with the row's entropy and top alternatives, and their gradient.
//
// One pass over a row of V logits keeps, per thread, a reference m and the sums
//   s = sum 2^(y - m),   t = sum 2^(y - m) (y - m),      y = c x,  c = scale * log2(e),
// which join by rescaling to a common reference.  Then, in natural logarithms,
//   ln S = ln2 (log2 s + m - y_max),  lse = scale x_max + ln S,  logprob = scale (x_target - x_max) - ln S,
//   entropy = ln2 (log2 s - t / s).
// Every value is taken relative to the row's maximum before it is rounded, so that the size of the logits
// costs no digits.

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "../../include/aq_b200.h"
#include "aq_stage.h"

namespace cg = cooperative_groups;

namespace aq {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kGroups = kRowThreads / 4;      // four neighbouring threads share one maximum for the alternatives
constexpr int kCandidates = 1024;             // logits that may tie with or beat the threshold before the slow way is taken
static_assert(kGroups >= kMaxTop, "the threshold needs as many group maxima as alternatives");
constexpr int kCluster = 8;                   // CTAs that share a row when there are few rows; portable cluster size
static_assert(kCluster * kMaxTop <= kCandidates, "the lists of a cluster are merged in one buffer");

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLog2eRest = 1.925963e-8f;    // log2(e) - kLog2e
constexpr float kUnset = -1e38f;              // reference before the first finite value
constexpr float kGone = -1e4f;                // exponents below give exactly 0; also keeps 0 * -infinity out of t
constexpr float kFar = 1e7f;                  // largest |y| whose rounding (half a unit there) the sums take in their stride
constexpr float kSlack = 8.0f;                // how far a value may exceed the reference before it is moved: 2^8 is
                                              // nothing to a binary32 sum, and the move leaves the loop's common path

// 16 bytes of logits.
template <typename T> struct Pack;
template <> struct Pack<float> {
  static constexpr int N = 4;
  static __device__ float top(uint4 v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ void open(uint4 v, float* f) { f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w); }
  static __device__ uint4 close(const float* f) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); }
  static __device__ float one(float x) { return x; }
  static __device__ float round(float x) { return x; }
};
template <> struct Pack<__half> {
  static constexpr int N = 8;
  static __device__ __half2 h(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
  static __device__ float top(uint4 v) {
    const float2 f = __half22float2(__hmax2(__hmax2(h(v.x), h(v.y)), __hmax2(h(v.z), h(v.w))));
    return fmaxf(f.x, f.y);
  }
  static __device__ void open(uint4 v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 p = __half22float2(h(w[i])); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
  }
  static __device__ uint4 close(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&p); }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ float one(__half x) { return __half2float(x); }
  static __device__ __half round(float x) { return __float2half_rn(x); }
};
template <> struct Pack<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __nv_bfloat162 h(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }
  static __device__ float top(uint4 v) {
    const float2 f = __bfloat1622float2(__hmax2(__hmax2(h(v.x), h(v.y)), __hmax2(h(v.z), h(v.w))));
    return fmaxf(f.x, f.y);
  }
  static __device__ void open(uint4 v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ uint4 close(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&p); }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
};

__device__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// max(x, bound) that keeps a NaN
__device__ float at_least(float x, float bound) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(bound)); return y; }

struct Sums {
  float m = kUnset, s = 0.0f, t = 0.0f;
  __device__ void move_to(float to) {
    const float d = fmaxf(m - to, kGone), e = exp2_fast(d);
    t = (t + s * d) * e;
    s *= e;
    m = to;
  }
  __device__ void add(float x, float c) {
    const float d = at_least(fmaf(x, c, -m), kGone), e = exp2_fast(d);
    s += e;
    t = fmaf(e, d, t);
  }
  __device__ void join(float m2, float s2, float t2) {
    Sums o;
    o.m = m2; o.s = s2; o.t = t2;
    const float to = fmaxf(m, m2);
    move_to(to);
    o.move_to(to);
    s += o.s;
    t += o.t;
  }
};

// A logit and its id as one number that orders like (value falling, id rising); 0 is no logit's.
__device__ unsigned long long key_of(float x, unsigned id) {
  const unsigned b = __float_as_uint(x + 0.0f);                         // -0 counts as 0
  return ((unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | (0xffffffffu - id);
}
__device__ unsigned id_of(unsigned long long key) { return 0xffffffffu - (unsigned)key; }
__device__ float value_of(unsigned long long key) {
  const unsigned b = (unsigned)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}

struct RowShared {
  float m[kRowWarps], s[kRowWarps], t[kRowWarps], top[kRowWarps];
  float group_top[kGroups];
  int groups[kGroups];
  int n_groups, n_found;
  float threshold;
  unsigned long long best[kRowWarps];
  unsigned long long found[kCandidates];
  unsigned long long list[kMaxTop];          // this CTA's alternatives, falling
  float cta_m, cta_s, cta_t, cta_top;        // this CTA's sums and largest logit
};

// The part of a row that one CTA reads: `head` elements up to the first 16-byte boundary, whole vectors, `tail`
// elements.  Element ids of the part are contiguous from `first`.
template <typename T> struct Part {
  const T* row;
  const uint4* vec;
  int n_vec;
  int head, tail;
  unsigned first, vec_first, tail_first, count;
  __device__ Part(const T* r, unsigned vocab, unsigned rank, unsigned ranks) {
    constexpr int N = Pack<T>::N;
    row = r;
    const unsigned off = (unsigned)((16u - (unsigned)(reinterpret_cast<uintptr_t>(r) & 15u)) & 15u) / (unsigned)sizeof(T);
    const unsigned all_head = off < vocab ? off : vocab;
    const unsigned all_vec = (vocab - all_head) / N;
    const unsigned per = (all_vec + ranks - 1) / ranks;
    const unsigned v0 = min(rank * per, all_vec), v1 = min(v0 + per, all_vec);
    n_vec = (int)(v1 - v0);
    head = rank == 0 ? (int)all_head : 0;
    vec_first = all_head + v0 * N;
    first = rank == 0 ? 0u : vec_first;
    vec = reinterpret_cast<const uint4*>(r + vec_first);
    tail_first = all_head + all_vec * N;
    tail = rank == ranks - 1 ? (int)(vocab - tail_first) : 0;
    count = (unsigned)head + (unsigned)n_vec * N + (unsigned)tail;
  }
  // the edge element of thread tid (head first, then tail), if it has one
  __device__ bool edge(int tid, unsigned* id) const {
    if (tid < head) { *id = (unsigned)tid; return true; }
    if (tid >= 32 && tid - 32 < tail) { *id = tail_first + (unsigned)(tid - 32); return true; }
    return false;
  }
};

// The k largest of sh.found[0..n) (unique keys) to sh.list, falling; missing places 0.
__device__ void select_found(RowShared& sh, int n, int k) {
  const int tid = threadIdx.x;
  if (tid < k) sh.list[tid] = 0ull;
  __syncthreads();
  for (int i = tid; i < n; i += kRowThreads) {
    const unsigned long long mine = sh.found[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += sh.found[j] > mine;
    if (rank < k && mine) sh.list[rank] = mine;
  }
  __syncthreads();
}

// This CTA's k alternatives to sh.list.  The k-th largest of the 64 group maxima is a lower bound of the k-th
// largest logit, and only groups whose maximum reaches it can hold one: about k of them, whose elements are read
// again (from L2) and compared.  Measured beside the pass that needs the maxima anyway, this is what keeps the
// alternatives nearly free; a sorted list in every thread would cost the loop a compare and a branch per element.
template <typename T>
__device__ void alternatives(RowShared& sh, const Part<T>& part, float my_top, int k) {
  constexpr int N = Pack<T>::N;
  const int tid = threadIdx.x;
  float g = fmaxf(my_top, __shfl_xor_sync(0xffffffffu, my_top, 1));
  g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
  if ((tid & 3) == 0) sh.group_top[tid >> 2] = g;
  if (tid == 0) { sh.n_groups = 0; sh.n_found = 0; }
  __syncthreads();
  if (tid < kGroups) {
    const float mine = sh.group_top[tid];
    int rank = 0;
    for (int j = 0; j < kGroups; ++j) { const float o = sh.group_top[j]; rank += o > mine || (o == mine && j < tid); }
    if (rank == k - 1) sh.threshold = mine;
  }
  __syncthreads();
  const float threshold = sh.threshold;
  if (tid < kGroups && sh.group_top[tid] >= threshold) sh.groups[atomicAdd(&sh.n_groups, 1)] = tid;
  __syncthreads();
  const int n_groups = sh.n_groups, rounds = (part.n_vec + kRowThreads - 1) / kRowThreads;
  auto offer = [&](float x, unsigned id) {
    if (x >= threshold) {
      const int at = atomicAdd(&sh.n_found, 1);
      if (at < kCandidates) sh.found[at] = key_of(x, id);
    }
  };
  for (long long w = tid; w < 4ll * n_groups * rounds; w += kRowThreads) {
    const int rest = (int)(w >> 2), v = (rest / n_groups) * kRowThreads + sh.groups[rest % n_groups] * 4 + (int)(w & 3);
    if (v < part.n_vec) {
      float f[N];
      Pack<T>::open(__ldg(part.vec + v), f);
#pragma unroll
      for (int i = 0; i < N; ++i) offer(f[i], part.vec_first + (unsigned)v * N + i);
    }
  }
  unsigned id;
  if (part.edge(tid, &id)) offer(Pack<T>::one(part.row[id]), id);
  __syncthreads();
  if (sh.n_found <= kCandidates) {
    select_found(sh, sh.n_found, k);
    return;
  }
  // too many logits at or above the threshold (whole stretches of equal ones): the next largest key, k times
  unsigned long long below = ~0ull;
  for (int r = 0; r < k; ++r) {
    unsigned long long best = 0ull;
    for (int v = tid; v < part.n_vec; v += kRowThreads) {
      float f[N];
      Pack<T>::open(__ldg(part.vec + v), f);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned long long key = f[i] == f[i] ? key_of(f[i], part.vec_first + (unsigned)v * N + i) : 0ull;
        if (key < below && key > best) best = key;
      }
    }
    if (part.edge(tid, &id)) {
      const float x = Pack<T>::one(part.row[id]);
      const unsigned long long key = x == x ? key_of(x, id) : 0ull;
      if (key < below && key > best) best = key;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) { const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o); if (other > best) best = other; }
    if ((tid & 31) == 0) sh.best[tid >> 5] = best;
    __syncthreads();
    best = 0ull;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) if (sh.best[w] > best) best = sh.best[w];
    if (tid == 0) sh.list[r] = best;
    below = best;                                 // 0 once there is nothing left: every later place is 0 too
    __syncthreads();
  }
}

__device__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

// One row, or one of gridDim's clusters' shares of it: kRanks CTAs to a row.
template <typename T, int kRanks>
__global__ void __launch_bounds__(kRowThreads) logprob_kernel(const LogprobArgs a) {
  constexpr int N = Pack<T>::N, U = 4;
  __shared__ RowShared sh;
  const int tid = threadIdx.x;
  const unsigned rank = kRanks > 1 ? blockIdx.x % kRanks : 0;
  const long long row = blockIdx.x / kRanks;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  const Part<T> part(x, (unsigned)a.vocab, rank, kRanks);
  const float c = a.scale * kLog2e;

  Sums acc;
  float top = -CUDART_INF_F;
  for (int v0 = tid; v0 < part.n_vec; v0 += U * kRowThreads) {
    uint4 v[U];
    float f[N];
    if (v0 + (U - 1) * kRowThreads < part.n_vec) {
#pragma unroll
      for (int i = 0; i < U; ++i) v[i] = __ldcs(part.vec + v0 + i * kRowThreads);
      float here = Pack<T>::top(v[0]);
#pragma unroll
      for (int i = 1; i < U; ++i) here = fmaxf(here, Pack<T>::top(v[i]));
      top = fmaxf(top, here);
      if (here * c > acc.m + kSlack) acc.move_to(here * c);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        Pack<T>::open(v[i], f);
#pragma unroll
        for (int j = 0; j < N; ++j) acc.add(f[j], c);
      }
    } else {
#pragma unroll
      for (int i = 0; i < U - 1; ++i) {
        if (v0 + i * kRowThreads >= part.n_vec) break;
        v[0] = __ldcs(part.vec + v0 + i * kRowThreads);
        const float here = Pack<T>::top(v[0]);
        top = fmaxf(top, here);
        if (here * c > acc.m + kSlack) acc.move_to(here * c);
        Pack<T>::open(v[0], f);
#pragma unroll
        for (int j = 0; j < N; ++j) acc.add(f[j], c);
      }
    }
  }
  unsigned id;
  if (part.edge(tid, &id)) {
    const float e = Pack<T>::one(x[id]);
    top = fmaxf(top, e);
    if (e * c > acc.m + kSlack) acc.move_to(e * c);
    acc.add(e, c);
  }

  const float my_top = top;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    acc.join(__shfl_xor_sync(0xffffffffu, acc.m, o), __shfl_xor_sync(0xffffffffu, acc.s, o), __shfl_xor_sync(0xffffffffu, acc.t, o));
  }
  top = warp_max(top);
  if ((tid & 31) == 0) { sh.m[tid >> 5] = acc.m; sh.s[tid >> 5] = acc.s; sh.t[tid >> 5] = acc.t; sh.top[tid >> 5] = top; }
  __syncthreads();
  Sums cta;
  float cta_top = -CUDART_INF_F;
#pragma unroll
  for (int w = 0; w < kRowWarps; ++w) { cta.join(sh.m[w], sh.s[w], sh.t[w]); cta_top = fmaxf(cta_top, sh.top[w]); }
  const int k = a.top_k;
  if (k) {
    if (cta_top == -CUDART_INF_F && cta.s == cta.s) {          // nothing but -infinity: the first ids
      if (tid < k) sh.list[tid] = (unsigned)tid < part.count ? key_of(-CUDART_INF_F, part.first + tid) : 0ull;
      __syncthreads();
    } else {
      alternatives(sh, part, my_top, k);
    }
  }

  if constexpr (kRanks > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    if (tid == 0) { sh.cta_m = cta.m; sh.cta_s = cta.s; sh.cta_t = cta.t; sh.cta_top = cta_top; }
    cluster.sync();
    if (rank == 0) {
      for (int r = 1; r < kRanks; ++r) {
        const RowShared* o = cluster.map_shared_rank(&sh, r);
        cta.join(o->cta_m, o->cta_s, o->cta_t);
        cta_top = fmaxf(cta_top, o->cta_top);
      }
      for (int i = tid; i < kRanks * k; i += kRowThreads) sh.found[i] = cluster.map_shared_rank(&sh, i / k)->list[i % k];
    }
    cluster.sync();                                            // the other CTAs' shared memory is no longer needed
    if (rank != 0) return;
    if (k) select_found(sh, kRanks * k, k);
  }

  // statistics of the row
  float ln_s, lse, entropy;
  bool none = false;
  if (fabsf(cta_top) * c > kFar && cta_top > -CUDART_INF_F) {
    // logits so large that rounding the reference already moves it by whole units: once more, relative to the largest
    float s = 0.0f, t = 0.0f;
    if (a.scale * cta_top > -CUDART_INF_F) {
      for (long long i = tid; i < a.vocab; i += kRowThreads) {
        const float d = at_least((Pack<T>::one(x[i]) - cta_top) * c, kGone), e = exp2_fast(d);
        s += e;
        t = fmaf(e, d, t);
      }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) { s += __shfl_xor_sync(0xffffffffu, s, o); t += __shfl_xor_sync(0xffffffffu, t, o); }
    __syncthreads();
    if ((tid & 31) == 0) { sh.s[tid >> 5] = s; sh.t[tid >> 5] = t; }
    __syncthreads();
    s = t = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) { s += sh.s[w]; t += sh.t[w]; }
    none = s == 0.0f;
    ln_s = logf(s);
    entropy = ln_s - kLn2 * (t / s);
  } else {
    none = cta.s == 0.0f;
    ln_s = kLn2 * (log2f(cta.s) - fmaf(cta_top, c, -cta.m));
    entropy = kLn2 * (log2f(cta.s) - cta.t / cta.s);
  }
  lse = fmaf(a.scale, cta_top, ln_s);
  if (none) { lse = -CUDART_INF_F; entropy = 0.0f; }
  if (tid == 0) {
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = entropy;
    if (a.targets) {
      const int32_t target = a.targets[row];
      float lp = 0.0f;
      if (target >= 0 && target < a.vocab) lp = none ? -CUDART_INF_F : a.scale * (Pack<T>::one(x[target]) - cta_top) - ln_s;
      else if (target >= 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
      if (a.logprob) a.logprob[row] = lp;
    }
  }
  if (tid < k) {
    const unsigned long long key = sh.list[tid];
    if (a.top_ids) a.top_ids[row * k + tid] = key ? (int32_t)id_of(key) : -1;
    if (a.top_logprobs) a.top_logprobs[row * k + tid] = !key ? CUDART_NAN_F : none ? -CUDART_INF_F : a.scale * (value_of(key) - cta_top) - ln_s;
  }
}

// ---- gradient ------------------------------------------------------------------------------------------------

constexpr float kFarLse = 4096.0f;            // half a unit of lse in its last place there is 1/4096
constexpr int kGradVecs = 4;                  // 16-byte vectors per thread

// One piece of one row: d = scale p (A + B log2 p) and the target's term, where ln p = z - lse.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) logprob_grad_kernel(const LogprobGradArgs a, int pieces) {
  constexpr int N = Pack<T>::N;
  const int tid = threadIdx.x;
  const long long row = blockIdx.x / (unsigned)pieces;
  const unsigned piece = blockIdx.x % (unsigned)pieces;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const out = static_cast<T*>(a.d_logits) + row * a.ld_d;
  const unsigned vocab = (unsigned)a.vocab;
  const float c = a.scale * kLog2e;
  // c's own rounding matters to binary32 outputs only
  const float c_lo = fmaf(a.scale, kLog2eRest, fmaf(a.scale, kLog2e, -c));
  const float lse = a.lse[row], entropy = a.d_entropy ? a.entropy[row] : 0.0f;
  const float gh = a.d_entropy ? a.d_entropy[row] : 0.0f;
  int32_t target = a.targets ? a.targets[row] : -1;
  if (target >= 0 && (unsigned)target >= vocab) {
    if (tid == 0 && piece == 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
    target = -1;
  }
  const float gl = target >= 0 && a.d_logprob ? a.d_logprob[row] : 0.0f;
  const float at_target = gl * a.scale;

  if (!(fabsf(lse) <= kFarLse)) {
    // the first piece's CTA does the whole row: zeros where the row has no distribution; else the logits are so large
    // that lse has no digits left for ln p, and the row's own sum is formed again, relative to its largest logit
    if (piece) return;
    __shared__ float part[kRowWarps];
    float top = -CUDART_INF_F;
    for (unsigned i = tid; i < vocab; i += kRowThreads) top = fmaxf(top, Pack<T>::one(x[i]));
    top = warp_max(top);
    if ((tid & 31) == 0) part[tid >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) top = fmaxf(top, part[w]);
    __syncthreads();
    float s = 0.0f;
    for (unsigned i = tid; i < vocab; i += kRowThreads) s += exp2_fast(at_least((Pack<T>::one(x[i]) - top) * c, kGone));
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((tid & 31) == 0) part[tid >> 5] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w) s += part[w];
    const bool none = lse == -CUDART_INF_F;
    const float log2s = log2f(s);
    for (unsigned i = tid; i < vocab; i += kRowThreads) {
      const float d = at_least((Pack<T>::one(x[i]) - top) * c - log2s, kGone), p = exp2_fast(d);
      const float v = -a.scale * p * (gl + gh * (d * kLn2 + entropy)) + (i == (unsigned)target ? at_target : 0.0f);
      out[i] = Pack<T>::round(none ? 0.0f : v);
    }
    return;
  }

  // p = 2^(x c - lse log2(e)) with the rounding of the second product put back as a factor of the coefficients
  const float ref = lse * kLog2e;
  const float back = exp2_fast(-fmaf(lse, kLog2eRest, fmaf(lse, kLog2e, -ref)));
  const float coef_a = -a.scale * back * fmaf(gh, entropy, gl), coef_b = -a.scale * back * gh * kLn2;
  auto grad = [&](float v) {
    float d;
    if (sizeof(T) == 4) {
      v = at_least(v, -1e36f);                                   // -infinity times c_lo could be +infinity
      d = fmaf(v, c_lo, fmaf(v, c, -ref));
    } else {
      d = fmaf(v, c, -ref);
    }
    d = at_least(d, kGone);
    return exp2_fast(d) * fmaf(coef_b, d, coef_a);
  };
  const unsigned per = kRowThreads * kGradVecs * N;
  const unsigned misalign = (unsigned)(reinterpret_cast<uintptr_t>(out) & 15u);
  if (misalign == (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u)) {
    const unsigned off = ((16u - misalign) & 15u) / (unsigned)sizeof(T);
    const unsigned head = off < vocab ? off : vocab;
    const unsigned n_vec = (vocab - head) / N, tail = vocab - head - n_vec * N;
    const uint4* const vx = reinterpret_cast<const uint4*>(x + head);
    uint4* const vo = reinterpret_cast<uint4*>(out + head);
    const unsigned v0 = piece * (kRowThreads * kGradVecs) + tid;
    uint4 v[kGradVecs];
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) if (v0 + i * kRowThreads < n_vec) v[i] = __ldcs(vx + v0 + i * kRowThreads);
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) {
      const unsigned at = v0 + i * kRowThreads;
      if (at < n_vec) {
        float f[N];
        Pack<T>::open(v[i], f);
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = grad(f[j]);
        const unsigned t = (unsigned)target - head - at * N;     // target's place in this vector, if it is in it
        if (t < (unsigned)N) {
#pragma unroll
          for (int j = 0; j < N; ++j) if (t == (unsigned)j) f[j] += at_target;
        }
        __stcs(vo + at, Pack<T>::close(f));
      }
    }
    if (piece == 0) {                                            // the elements before the first and after the last vector
      unsigned i = 0xffffffffu;
      if ((unsigned)tid < head) i = tid;
      else if (tid >= 32 && (unsigned)(tid - 32) < tail) i = head + n_vec * N + (tid - 32);
      if (i != 0xffffffffu) out[i] = Pack<T>::round(grad(Pack<T>::one(x[i])) + (i == (unsigned)target ? at_target : 0.0f));
    }
  } else {
    // rows that no common vector boundary serves: element by element
    const unsigned i0 = piece * per, i1 = min(i0 + per, vocab);
    for (unsigned i = i0 + tid; i < i1; i += kRowThreads)
      out[i] = Pack<T>::round(grad(Pack<T>::one(x[i])) + (i == (unsigned)target ? at_target : 0.0f));
  }
}

template <typename T>
cudaError_t run(const LogprobArgs& a, cudaStream_t s) {
  // A row to a CTA when there are rows for half of the multiprocessors; below, a cluster of eight to a row.
  if (a.rows * 2 >= a.sms || a.vocab < 4096) {
    logprob_kernel<T, 1><<<(unsigned)a.rows, kRowThreads, 0, s>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.rows * kCluster);
  cfg.blockDim = dim3(kRowThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<T, kCluster>, a);
}

template <typename T>
cudaError_t run_grad(const LogprobGradArgs& a, cudaStream_t s) {
  const long long per = (long long)kRowThreads * kGradVecs * Pack<T>::N;
  const long long pieces = (a.vocab + per - 1) / per;
  // a grid has at most 2^31 - 1 CTAs: more rows go in several launches
  const long long most = 0x7fffffffll / pieces;
  LogprobGradArgs b = a;
  for (long long r = 0; r < a.rows; r += most) {
    b.rows = a.rows - r < most ? a.rows - r : most;
    logprob_grad_kernel<T><<<(unsigned)(b.rows * pieces), kRowThreads, 0, s>>>(b, (int)pieces);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    b.logits = static_cast<const T*>(b.logits) + b.rows * b.ld;
    b.d_logits = static_cast<T*>(b.d_logits) + b.rows * b.ld_d;
    b.lse += b.rows;
    if (b.targets) b.targets += b.rows;
    if (b.entropy) b.entropy += b.rows;
    if (b.d_logprob) b.d_logprob += b.rows;
    if (b.d_entropy) b.d_entropy += b.rows;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_logprob(int dtype, const LogprobArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run<__half>(a, s) : dtype == AQ_BF16 ? run<__nv_bfloat16>(a, s) : run<float>(a, s);
}

cudaError_t launch_logprob_grad(int dtype, const LogprobGradArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_grad<__half>(a, s) : dtype == AQ_BF16 ? run_grad<__nv_bfloat16>(a, s) : run_grad<float>(a, s);
}

}  // namespace aq
