// Log probabilities of given tokens with the row's entropy and top alternatives, and their gradient.
//
// One pass over a row of V logits keeps, per thread, a reference m and the sums
//   s = sum 2^(y - m),   t = sum 2^(y - m) (y - m),      y = c x,  c = scale * log2(e),
// which join by rescaling to a common reference.  Then, in natural logarithms,
//   ln S = ln2 (log2 s + m - y_max),  lse = scale x_max + ln S,  logprob = scale (x_target - x_max) - ln S,
//   entropy = ln2 (log2 s - t / s).
// Every value is taken relative to the row's maximum before it is rounded, so that the size of the logits
// costs no digits.
//
// Three limits lie close together: memory (8192 x 50304 bf16: 126 us), one exponential a logit (91 us) and the issue of
// instructions (about 80 us); the pass takes 164 to 179 us, 4.6 to 5.0 TB/s (2048 rows under a profiler: issue slots 0.68,
// exponentials 0.55, DRAM 0.54).  The gradient reads and writes each logit once: 4096 x 50257 bf16 134 to 140 us, 5.9 to 6.1 TB/s.  What did not help the pass: loads one step ahead (180 us), rows streamed through a ring in shared
// memory by CTAs that stay, instructions on pairs of binary32 values, 128 threads to a row.

#include <cooperative_groups.h>
#include <math_constants.h>

#include "aq_stage.h"
#include "aq_stage_device.cuh"

namespace cg = cooperative_groups;

namespace aq {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kRowCtas = 7;                   // CTAs on a multiprocessor that the registers are cut for: 168 us at 8192 x 50304 bf16;
                                              // six 176 us, five 184 us, eight 170 us
constexpr int kGroups = kRowThreads / 4;      // four neighbouring threads share one maximum for the alternatives
constexpr int kCandidates = 1024;             // logits that may tie with or beat the threshold before the slow way is taken
static_assert(kGroups >= kMaxTop, "the threshold needs as many group maxima as alternatives");
constexpr int kCluster = 8;                   // CTAs that share a row when there are few rows; portable cluster size
static_assert(kCluster * kMaxTop <= kCandidates, "the lists of a cluster are merged in one buffer");

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLog2eRest = 1.925963e-8f;    // log2(e) - kLog2e
constexpr float kUnset = -1e6f;               // reference before the first larger value: what lies below it adds 0
constexpr float kGone = -1e4f;                // exponents below give exactly 0; also keeps 0 * -infinity out of t
constexpr float kClear = 200.0f;              // exponentials this far below the largest are 0 in binary32 sums
constexpr float kFar = 1e6f;                  // largest |y| of a row's maximum that the sums take in their stride: its rounding is 1/32 there
constexpr float kHuge = 1e38f;                // exponents beyond are about to overflow
constexpr float kSlack = 8.0f;                // how far a value may exceed the reference before it is moved: 2^8 is
                                              // nothing to a binary32 sum, and the move leaves the loop's common path

__device__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
__device__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
// max(x, bound) that keeps a NaN
__device__ float at_least(float x, float bound) { float y; asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(bound)); return y; }

// 16 bytes of logits.  So that nothing is ever infinity times 0, masked ones (-infinity, or anything below kLow) are raised to
// kLow first where that takes half an instruction each (fp16): their exponentials stay 0 as long as the row's largest logit is
// far above.  Elsewhere kLow is -infinity and the exponents are held at kGone.  NaNs stay either way.
template <typename T> struct Pack;
template <> struct Pack<float> {
  static constexpr int N = 4;
  static constexpr float kLow = -__builtin_huge_valf();
  static __device__ void raise(uint32_t (&)[4]) {}
  static __device__ float held(float d) { return at_least(d, kGone); }
  static __device__ uint32_t larger(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
  static __device__ float largest(uint32_t a) { return __uint_as_float(a); }
  static __device__ float2 open2(const uint32_t (&w)[4], int i) { return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])); }
  static __device__ void open(uint4 v, float* f) { f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w); }
  static __device__ uint4 close(const float* f) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); }
  static __device__ float one(float x) { return x; }
  static __device__ float round(float x) { return x; }
};
template <typename T, typename T2> struct Pack16 {
  static constexpr int N = 8;
  static __device__ T2 h(uint32_t u) { return *reinterpret_cast<T2*>(&u); }
  static __device__ uint32_t u(T2 v) { return *reinterpret_cast<const uint32_t*>(&v); }
  static __device__ uint32_t larger(uint32_t a, uint32_t b) { return u(__hmax2(h(a), h(b))); }
  static __device__ float largest(uint32_t a) { const float2 f = Num<T>::open(a); return fmaxf(f.x, f.y); }
  static __device__ float2 open2(const uint32_t (&w)[4], int i) { return Num<T>::open(w[i]); }
  static __device__ void open(uint4 v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 p = Num<T>::open(w[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
  }
  static __device__ uint4 close(const float* f) {
    return make_uint4(Num<T>::close(f[0], f[1]), Num<T>::close(f[2], f[3]), Num<T>::close(f[4], f[5]), Num<T>::close(f[6], f[7]));
  }
  static __device__ T round(float x) { return Num<T>::one(x); }
};
template <> struct Pack<__half> : Pack16<__half, __half2> {
  static constexpr float kLow = -65504.0f;
  static __device__ float held(float d) { return d; }
  static __device__ void raise(uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = u(__hmax2_nan(h(w[i]), h(0xfbfffbffu)));
  }
  static __device__ float one(__half x) { return __half2float(x); }
};
template <> struct Pack<__nv_bfloat16> : Pack16<__nv_bfloat16, __nv_bfloat162> {
  static constexpr float kLow = -__builtin_huge_valf();
  static __device__ void raise(uint32_t (&)[4]) {}
  static __device__ float held(float d) { return at_least(d, kGone); }
  static __device__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
};

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
};

// The same while a thread reads: even and odd elements apart.
struct Sums2 {
  float m = kUnset, s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
  // one or more raised vectors whose largest element is `here`
  template <typename T, int COUNT>
  __device__ void add(const uint32_t (&w)[COUNT][4], float here, float c) {
    if (here * c > m + kSlack) {
      const float d = fmaxf(m - here * c, kGone), e = exp2_fast(d);
      t0 = fmaf(s0, d, t0) * e;
      t1 = fmaf(s1, d, t1) * e;
      s0 *= e;
      s1 *= e;
      m = here * c;
    }
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
#pragma unroll
      for (int j = 0; j < Pack<T>::N / 2; ++j) {
        const float2 v = Pack<T>::open2(w[i], j);
        const float d0 = Pack<T>::held(fmaf(v.x, c, -m)), d1 = Pack<T>::held(fmaf(v.y, c, -m)), e0 = exp2_fast(d0), e1 = exp2_fast(d1);
        s0 += e0;
        s1 += e1;
        t0 = fmaf(e0, d0, t0);
        t1 = fmaf(e1, d1, t1);
      }
  }
  __device__ Sums whole() const {
    Sums o;
    o.m = m; o.s = s0 + s1; o.t = t0 + t1;
    return o;
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

// What the CTAs of a row send to the first of them: sums, largest logit and alternatives.
struct FromCta {
  float m, s, t, top;
  unsigned long long list[kMaxTop];
};

struct RowShared {
  float m[kRowWarps], s[kRowWarps], t[kRowWarps], top[kRowWarps];
  float group_top[kGroups];
  int groups[kGroups];
  int n_groups, n_found;
  float threshold, row_s, row_top;
  unsigned long long best[kRowWarps];
  unsigned long long found[kCandidates];
  unsigned long long list[kMaxTop];          // this CTA's alternatives, falling
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

// The largest key of a warp's lanes.
__device__ unsigned long long warp_best(unsigned long long key) {
  const unsigned high = __reduce_max_sync(0xffffffffu, (unsigned)(key >> 32));
  const unsigned low = __reduce_max_sync(0xffffffffu, (unsigned)(key >> 32) == high ? (unsigned)key : 0u);
  return ((unsigned long long)high << 32) | low;
}

// The k largest of sh.found[0..n) (unique keys) to sh.list, falling; missing places 0.  One warp.
__device__ void select_found(RowShared& sh, int n, int k) {
  const int lane = threadIdx.x & 31;
  if (n <= 128) {                                  // every key counts those above it
    if (lane < k) sh.list[lane] = 0ull;
    __syncwarp();
    for (int i = lane; i < n; i += 32) {
      const unsigned long long mine = sh.found[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += sh.found[j] > mine;
      if (rank < k && mine) sh.list[rank] = mine;
    }
    __syncwarp();
    return;
  }
  unsigned long long below = ~0ull;                // the largest that is left, k times
  for (int r = 0; r < k; ++r) {
    unsigned long long best = 0ull;
    for (int i = lane; i < n; i += 32) { const unsigned long long key = sh.found[i]; if (key < below && key > best) best = key; }
    below = warp_best(best);
    if (lane == 0) sh.list[r] = below;
  }
  __syncwarp();
}

// The k-th largest of the group maxima, and the groups that reach it.  One warp, two groups a lane.
template <typename T>
__device__ void find_groups(RowShared& sh, int k) {
  static_assert(kGroups == 64, "two groups a lane");
  const int lane = threadIdx.x & 31;
  const float g0 = sh.group_top[lane], g1 = sh.group_top[lane + 32];
  float v0 = g0, v1 = g1, threshold = -CUDART_INF_F;
  for (int i = 0; i < k; ++i) {                    // takes the largest away, k times
    const float largest = fmaxf(v0, v1);
    threshold = warp_max(largest);
    if (threshold <= Pack<T>::kLow) break;         // masked logits were raised to kLow
    const unsigned have = __ballot_sync(0xffffffffu, largest == threshold);
    if (lane == __ffs(have) - 1) { if (v0 == threshold) v0 = -CUDART_INF_F; else v1 = -CUDART_INF_F; }
  }
  if (threshold <= Pack<T>::kLow) threshold = -CUDART_INF_F;
  const unsigned in0 = __ballot_sync(0xffffffffu, g0 >= threshold), in1 = __ballot_sync(0xffffffffu, g1 >= threshold), below = (1u << lane) - 1u;
  if (g0 >= threshold) sh.groups[__popc(in0 & below)] = lane;
  if (g1 >= threshold) sh.groups[__popc(in0) + __popc(in1 & below)] = lane + 32;
  if (lane == 0) { sh.threshold = threshold; sh.n_groups = __popc(in0) + __popc(in1); sh.n_found = 0; }
}

// The logits of this warp's share of those groups, read again, that reach the threshold.
template <typename T>
__device__ void collect(RowShared& sh, const Part<T>& part) {
  constexpr int N = Pack<T>::N, U = 4;
  const int tid = threadIdx.x, lane = tid & 31, rounds = (part.n_vec + kRowThreads - 1) / kRowThreads;
  const float threshold = sh.threshold;
  auto offer = [&](float x, unsigned id) {
    if (x >= threshold && x > -CUDART_INF_F) {
      const int at = atomicAdd(&sh.n_found, 1);
      if (at < kCandidates) sh.found[at] = key_of(x, id);
    }
  };
  const int n_groups = sh.n_groups;
  for (int g = tid >> 5; g < n_groups; g += kRowWarps) {
    const int first = sh.groups[g] * 4 + (lane & 3);
    for (int r = lane >> 2; r < rounds; r += 8 * U) {          // eight rounds of the group's four threads at a time
      uint4 v[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int at = (r + 8 * i) * kRowThreads + first;
        if (at < part.n_vec) v[i] = __ldg(part.vec + at);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int at = (r + 8 * i) * kRowThreads + first;
        if (at < part.n_vec) {
          float f[N];
          Pack<T>::open(v[i], f);
#pragma unroll
          for (int j = 0; j < N; ++j) offer(f[j], part.vec_first + (unsigned)at * N + j);
        }
      }
    }
  }
  unsigned id;
  if (part.edge(tid, &id)) offer(Pack<T>::one(part.row[id]), id);
}

// Too many logits at or above the threshold (whole stretches of equal ones): the next largest key, k times.  The whole CTA.
template <typename T>
__device__ void next_largest(RowShared& sh, const Part<T>& part, int k) {
  constexpr int N = Pack<T>::N;
  const int tid = threadIdx.x;
  unsigned id;
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

// Sums of a warp's lanes, relative to the largest reference among them.
__device__ void join_lanes(Sums& a) {
  const float to = warp_max(a.m);
  a.move_to(to);
  a.s = warp_sum(a.s);
  a.t = warp_sum(a.t);
}

// Whether the sums of a pass do not stand: logits so large that rounding the reference already moves it by whole units, or so
// low (all of them masked, perhaps) that raising the masked ones to kLow would show, or a scale so large that they overflow.
template <typename T> __device__ bool far(float top, float s, float c) {
  if (top == -CUDART_INF_F && s == 0.0f) return false;         // nothing but -infinity
  const float above = (top - Pack<T>::kLow) * c;
  return fabsf(top) * c > kFar || (Pack<T>::kLow > -CUDART_INF_F && (above < kClear || above > kHuge));
}
// c; a scale near the end of binary32 would make it infinite
__device__ float base2(float scale) { return fminf(scale * kLog2e, 3.4e38f); }

// Calls f with every logit of a row; the whole CTA, `part` being all of the row.
template <typename T, typename F> __device__ void each_logit(const Part<T>& part, F f) {
  constexpr int N = Pack<T>::N, U = 4;
  for (int v0 = threadIdx.x; v0 < part.n_vec; v0 += U * kRowThreads) {
    uint4 v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) if (v0 + i * kRowThreads < part.n_vec) v[i] = __ldg(part.vec + v0 + i * kRowThreads);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (v0 + i * kRowThreads < part.n_vec) {
        float x[N];
        Pack<T>::open(v[i], x);
#pragma unroll
        for (int j = 0; j < N; ++j) f(x[j]);
      }
    }
  }
  unsigned id;
  if (part.edge(threadIdx.x, &id)) f(Pack<T>::one(part.row[id]));
}

// The sums of such a row once more, relative to its largest logit as it stands: s, t and top to sh.  The whole CTA.
template <typename T>
__device__ void far_row(RowShared& sh, const Part<T>& part, float scale) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float c = base2(scale);
  float top = -CUDART_INF_F, s = 0.0f, t = 0.0f;
  each_logit(part, [&](float x) { top = fmaxf(top, x); });
  top = warp_max(top);
  __syncthreads();
  if (lane == 0) sh.top[warp] = top;
  __syncthreads();
  top = warp_max(lane < kRowWarps ? sh.top[lane] : -CUDART_INF_F);
  const bool empty = scale * top == -CUDART_INF_F;             // NaNs apart, which the sum is to show
  each_logit(part, [&](float x) {
    if (empty && x == x) return;
    const float d = at_least((x - top) * c, kGone), e = exp2_fast(d);
    s += e;
    t = fmaf(e, d, t);
  });
  s = warp_sum(s);
  t = warp_sum(t);
  __syncthreads();
  if (lane == 0) { sh.top[warp] = top; sh.s[warp] = s; sh.t[warp] = t; sh.m[warp] = 0.0f; }
  __syncthreads();
}

// COUNT vectors of a thread
template <typename T, int COUNT>
__device__ void take(uint32_t (&w)[COUNT][4], Sums2& sums, float& top, float c) {
  uint32_t large = 0;
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    Pack<T>::raise(w[i]);
    const uint32_t l = Pack<T>::larger(Pack<T>::larger(w[i][0], w[i][1]), Pack<T>::larger(w[i][2], w[i][3]));
    large = i ? Pack<T>::larger(large, l) : l;
  }
  const float here = Pack<T>::largest(large);
  top = fmaxf(top, here);
  sums.template add<T, COUNT>(w, here, c);
}

// One row to a CTA, or (few rows) to a cluster of kRanks, each with its share of it; the first one joins what they send it.
// The alternatives: the k-th largest of the 64 maxima of four neighbouring threads is a lower bound of the k-th
// largest logit, and only groups whose maximum reaches it can hold one: about k of them, whose elements are read again (from
// L2) and compared.  The pass itself needs the maxima anyway, so that the alternatives cost it nothing; a sorted list in every
// thread would cost a compare and a branch per element.  What follows the pass is left to one warp where it can be: done by
// all eight it was nearly as many instructions as the pass.
template <typename T, int kRanks>
__global__ void __launch_bounds__(kRowThreads, kRanks > 1 ? 1 : kRowCtas) logprob_kernel(const LogprobArgs a) {
  constexpr int U = 4;
  __shared__ RowShared sh;
  __shared__ FromCta from[kRanks];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  next_may_launch();
  wait_for_previous();
  const unsigned rank = kRanks > 1 ? blockIdx.x % kRanks : 0;
  const long long row = blockIdx.x / kRanks;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  const Part<T> part(x, (unsigned)a.vocab, rank, kRanks);
  const float c = base2(a.scale);
  if constexpr (kRanks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");

  Sums2 sums;
  float top = Pack<T>::kLow;
  for (int v0 = tid; v0 < part.n_vec; v0 += U * kRowThreads) {
    if (v0 + (U - 1) * kRowThreads < part.n_vec) {
      uint32_t w[U][4];
#pragma unroll
      for (int i = 0; i < U; ++i) { const uint4 v = __ldcs(part.vec + v0 + i * kRowThreads); w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w; }
      take<T, U>(w, sums, top, c);
    } else {
#pragma unroll 1
      for (int v1 = v0; v1 < part.n_vec; v1 += kRowThreads) {
        const uint4 v = __ldcs(part.vec + v1);
        uint32_t w[1][4] = {{v.x, v.y, v.z, v.w}};
        take<T, 1>(w, sums, top, c);
      }
    }
  }
  Sums acc = sums.whole();
  unsigned id;
  if (part.edge(tid, &id)) {
    const float e = Pack<T>::one(x[id]);
    top = fmaxf(top, e);
    if (e * c > acc.m + kSlack) acc.move_to(e * c);
    acc.add(e, c);
  }

  const int k = a.top_k;
  if (k) {
    float g = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
    if ((tid & 3) == 0) sh.group_top[tid >> 2] = g;
  }
  join_lanes(acc);
  top = warp_max(top);
  if (lane == 0) { sh.m[warp] = acc.m; sh.s[warp] = acc.s; sh.t[warp] = acc.t; sh.top[warp] = top; }
  __syncthreads();
  if (k) {
    if (warp == 0) find_groups<T>(sh, k);
    __syncthreads();
    collect(sh, part);
    __syncthreads();
    if (sh.n_found > kCandidates) next_largest(sh, part, k);
  }
  if (warp == 0) {
    if (k && sh.n_found <= kCandidates) {
      const int n = sh.n_found;
      select_found(sh, n, k);
      if (lane == 0 && n < k) {                   // fewer than k above -infinity: the first ids that hold -infinity follow
        int at = n;
        for (unsigned i = 0; at < k && i < part.count; ++i)
          if (Pack<T>::one(x[part.first + i]) == -CUDART_INF_F) sh.list[at++] = key_of(-CUDART_INF_F, part.first + i);
      }
      __syncwarp();
    }
    acc = Sums();
    if (lane < kRowWarps) { acc.m = sh.m[lane]; acc.s = sh.s[lane]; acc.t = sh.t[lane]; }
    join_lanes(acc);
    top = warp_max(lane < kRowWarps ? sh.top[lane] : Pack<T>::kLow);
  }
  if constexpr (kRanks > 1) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");           // all of the row's CTAs have begun: the first one's memory is there
    if (warp == 0) {
      FromCta* const to = cg::this_cluster().map_shared_rank(from, 0) + rank;
      if (lane == 0) { to->m = acc.m; to->s = acc.s; to->t = acc.t; to->top = top; }
      if (lane < k) to->list[lane] = sh.list[lane];
      __syncwarp();
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if (rank != 0) return;                                     // nobody reads the memory of the others
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == 0) {
      acc = Sums();
      if (lane < kRanks) { acc.m = from[lane].m; acc.s = from[lane].s; acc.t = from[lane].t; }
      join_lanes(acc);
      top = warp_max(lane < kRanks ? from[lane].top : Pack<T>::kLow);
      if (k) {
        for (int i = lane; i < kRanks * k; i += 32) sh.found[i] = from[i / k].list[i % k];
        __syncwarp();
        select_found(sh, kRanks * k, k);
      }
    }
  }
  if (tid == 0) { sh.row_s = acc.s; sh.row_top = top; }
  __syncthreads();
  const bool again = far<T>(sh.row_top, sh.row_s, c);
  if (again) {
    far_row(sh, Part<T>(x, (unsigned)a.vocab, 0, 1), a.scale);
    acc = Sums();
    acc.m = 0.0f;
    if (lane < kRowWarps) { acc.s = sh.s[lane]; acc.t = sh.t[lane]; }
    acc.s = warp_sum(acc.s);
    acc.t = warp_sum(acc.t);
    top = sh.top[0];
  }
  if (warp != 0) return;

  // acc is relative to the reference acc.m, or (again) to the largest logit itself
  const float log2s = log2f(acc.s), ln_s = kLn2 * (again ? log2s : log2s - fmaf(top, c, -acc.m));
  const bool none = acc.s == 0.0f;
  if (lane == 0) {
    if (a.lse) a.lse[row] = none ? -CUDART_INF_F : fmaf(a.scale, top, ln_s);
    if (a.entropy) a.entropy[row] = none ? 0.0f : kLn2 * (log2s - acc.t / acc.s);
    if (a.targets) {
      const int32_t target = a.targets[row];
      float lp = 0.0f;
      if (target >= 0 && target < a.vocab) lp = none ? -CUDART_INF_F : a.scale * (Pack<T>::one(x[target]) - top) - ln_s;
      else if (target >= 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
      if (a.logprob) a.logprob[row] = lp;
    }
  }
  if (lane < k) {
    const unsigned long long key = sh.list[lane];
    if (a.top_ids) a.top_ids[row * k + lane] = key ? (int32_t)id_of(key) : -1;
    if (a.top_logprobs) a.top_logprobs[row * k + lane] = !key ? CUDART_NAN_F : none ? -CUDART_INF_F : a.scale * (value_of(key) - top) - ln_s;
  }
}

// ---- short rows ----------------------------------------------------------------------------------------------
//
// A row of up to kShort logits is a warp's: it stays in registers, so that the largest logit is known before the sums are
// formed, relative to it, and the alternatives are taken from the registers one by one.  8192 rows of 257 bf16 logits
// with twenty alternatives 39 us, without any 7 us (a CTA to a row: 230 and 17 us).

constexpr int kShort = 1024;

template <typename T>
__global__ void __launch_bounds__(kRowThreads) logprob_short_kernel(const LogprobArgs a) {
  constexpr int N = Pack<T>::N, kVecs = kShort / N / 32;
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
  next_may_launch();
  wait_for_previous();
  if (row >= a.rows) return;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  const Part<T> part(x, (unsigned)a.vocab, 0, 1);
  uint4 v[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) if (lane + 32 * i < part.n_vec) v[i] = __ldcs(part.vec + lane + 32 * i);
  // the elements before the first and after the last vector: lanes 0.. and 16..
  const bool edge = lane < part.head || (lane >= 16 && lane - 16 < part.tail);
  const unsigned edge_id = lane < part.head ? (unsigned)lane : part.tail_first + (unsigned)(lane - 16);
  const float edge_x = edge ? Pack<T>::one(x[edge_id]) : 0.0f;
  // f(value, id) of all of this lane's logits
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (32 * i >= part.n_vec) break;
      if (lane + 32 * i < part.n_vec) {
        float e[N];
        Pack<T>::open(v[i], e);
#pragma unroll
        for (int j = 0; j < N; ++j) f(e[j], part.vec_first + (unsigned)(lane + 32 * i) * N + j);
      }
    }
    if (edge) f(edge_x, edge_id);
  };
  const float c = base2(a.scale);
  float top = -CUDART_INF_F, s = 0.0f, t = 0.0f;
  each([&](float e, unsigned) { top = fmaxf(top, e); });
  top = warp_max(top);
  const bool empty = a.scale * top == -CUDART_INF_F;           // NaNs apart, which the sum is to show
  each([&](float e, unsigned) {
    if (empty && e == e) return;
    const float d = at_least((e - top) * c, kGone), p = exp2_fast(d);
    s += p;
    t = fmaf(p, d, t);
  });
  s = warp_sum(s);
  t = warp_sum(t);
  const bool none = s == 0.0f;
  const float log2s = log2f(s), ln_s = kLn2 * log2s;
  if (lane == 0) {
    if (a.lse) a.lse[row] = none ? -CUDART_INF_F : fmaf(a.scale, top, ln_s);
    if (a.entropy) a.entropy[row] = none ? 0.0f : kLn2 * (log2s - t / s);
    if (a.targets) {
      const int32_t target = a.targets[row];
      float lp = 0.0f;
      if (target >= 0 && target < a.vocab) lp = none ? -CUDART_INF_F : a.scale * (Pack<T>::one(x[target]) - top) - ln_s;
      else if (target >= 0) atomicOr(a.status, (uint32_t)AQ_ST_BAD_ID);
      if (a.logprob) a.logprob[row] = lp;
    }
  }
  const int k = a.top_k;
  unsigned long long mine = 0ull, taken = ~0ull, best = 0ull;  // this lane's place in the list; the last key taken; this lane's best below it
  for (int r = 0; r < k; ++r) {
    if (best >= taken || r == 0) {
      best = 0ull;
      each([&](float e, unsigned id) {
        const unsigned long long key = e == e ? key_of(e, id) : 0ull;
        if (key < taken && key > best) best = key;
      });
    }
    __syncwarp();
    taken = warp_best(best);
    if (lane == r) mine = taken;
    if (!taken) break;                                         // nothing left
  }
  if (lane < k) {
    if (a.top_ids) a.top_ids[row * k + lane] = mine ? (int32_t)id_of(mine) : -1;
    if (a.top_logprobs) a.top_logprobs[row * k + lane] = !mine ? CUDART_NAN_F : none ? -CUDART_INF_F : a.scale * (value_of(mine) - top) - ln_s;
  }
}

// ---- gradient ------------------------------------------------------------------------------------------------

constexpr float kFarLse = 4096.0f;            // half a unit of lse in its last place there is 1/4096
// eight: 147 us at 4096 x 50257 bf16 with cold caches; four 151 us, twelve 154 us
constexpr int kGradVecs = 8;                  // 16-byte vectors per thread

// One piece of one row: d = scale p (A + B log2 p) and the target's term, where ln p = z - lse.  LANES threads to a piece: a CTA,
// or a warp where that holds a whole row (8192 rows of 257 bf16 logits: 8 us against 22).
template <typename T, int LANES>
__global__ void __launch_bounds__(kRowThreads) logprob_grad_kernel(const LogprobGradArgs a, int pieces) {
  constexpr int N = Pack<T>::N;
  const int tid = threadIdx.x % LANES;
  next_may_launch();
  wait_for_previous();
  const long long row = LANES == 32 ? (long long)blockIdx.x * kRowWarps + threadIdx.x / 32 : blockIdx.x / (unsigned)pieces;
  const unsigned piece = LANES == 32 ? 0u : blockIdx.x % (unsigned)pieces;
  if (LANES == 32 && row >= a.rows) return;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const out = static_cast<T*>(a.d_logits) + row * a.ld_d;
  const unsigned vocab = (unsigned)a.vocab;
  const float c = base2(a.scale);
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

  if (lse == -CUDART_INF_F) {                                    // no distribution: zeros
    const unsigned i0 = piece * (LANES * kGradVecs * N), i1 = min(i0 + LANES * kGradVecs * N, vocab);
    for (unsigned i = i0 + tid; i < i1; i += LANES) out[i] = Pack<T>::round(0.0f);
    return;
  }
  const float ref = lse * kLog2e, low = Pack<T>::kLow * c - ref;
  if (!(fabsf(lse) <= kFarLse) || low > -kClear || (Pack<T>::kLow > -CUDART_INF_F && low < -kHuge)) {
    // the first piece's CTA does the whole row: the logits are so large that lse has no digits left for ln p (or so low or little
    // scaled that raising the masked ones would show, or scaled so much that they overflow), and the row's own sum is formed again,
    // relative to its largest logit.  Three passes by one CTA: 4096 x 50264 bf16 rows 156 us with one in a hundred of them so,
    // 190 us with one in ten, 476 us with all (120 us with none; binary32, twice the bytes, 820 us with all).
    if (piece) return;
    __shared__ float part[kRowWarps];
    float top = -CUDART_INF_F;
    for (unsigned i = tid; i < vocab; i += LANES) top = fmaxf(top, Pack<T>::one(x[i]));
    top = warp_max(top);
    if (LANES > 32) {
      if ((tid & 31) == 0) part[tid >> 5] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) top = fmaxf(top, part[w]);
      __syncthreads();
    }
    float s = 0.0f;
    for (unsigned i = tid; i < vocab; i += LANES) s += exp2_fast(at_least((Pack<T>::one(x[i]) - top) * c, kGone));
    s = warp_sum(s);
    if (LANES > 32) {
      if ((tid & 31) == 0) part[tid >> 5] = s;
      __syncthreads();
      s = 0.0f;
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) s += part[w];
    }
    const float log2s = log2f(s);
    for (unsigned i = tid; i < vocab; i += LANES) {
      const float d = at_least((Pack<T>::one(x[i]) - top) * c - log2s, kGone), p = exp2_fast(d);
      const float v = -a.scale * p * (gl + gh * (d * kLn2 + entropy)) + (i == (unsigned)target ? at_target : 0.0f);
      out[i] = Pack<T>::round(v);
    }
    return;
  }

  // p = 2^(x c - lse log2(e)) with the rounding of the second product put back as a factor of the coefficients
  const float back = exp2_fast(-fmaf(lse, kLog2eRest, fmaf(lse, kLog2e, -ref)));
  const float coef_a = -a.scale * back * fmaf(gh, entropy, gl), coef_b = -a.scale * back * gh * kLn2;
  auto grad = [&](float v) {                                      // of a raised logit
    float d = fmaf(v, c, -ref);
    if (sizeof(T) == 4) d = fmaf(at_least(v, -1e30f), c_lo, d);    // -infinity times c_lo could be +infinity
    d = Pack<T>::held(d);
    return exp2_fast(d) * fmaf(coef_b, d, coef_a);
  };
  const unsigned per = LANES * kGradVecs * N;
  const unsigned misalign = (unsigned)(reinterpret_cast<uintptr_t>(out) & 15u);
  if (misalign == (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u)) {
    const unsigned off = ((16u - misalign) & 15u) / (unsigned)sizeof(T);
    const unsigned head = off < vocab ? off : vocab;
    const unsigned n_vec = (vocab - head) / N, tail = vocab - head - n_vec * N;
    const uint4* const vx = reinterpret_cast<const uint4*>(x + head);
    uint4* const vo = reinterpret_cast<uint4*>(out + head);
    const unsigned v0 = piece * (LANES * kGradVecs) + tid;
    uint4 v[kGradVecs];
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) if (v0 + i * LANES < n_vec) v[i] = __ldcs(vx + v0 + i * LANES);
#pragma unroll
    for (int i = 0; i < kGradVecs; ++i) {
      const unsigned at = v0 + i * LANES;
      if (at < n_vec) {
        float f[N];
        uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        Pack<T>::raise(w);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
          const float2 x2 = Pack<T>::open2(w, j);
          f[2 * j] = grad(x2.x);
          f[2 * j + 1] = grad(x2.y);
        }
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
      else if (tid >= 16 && (unsigned)(tid - 16) < tail) i = head + n_vec * N + (tid - 16);
      if (i != 0xffffffffu) out[i] = Pack<T>::round(grad(at_least(Pack<T>::one(x[i]), Pack<T>::kLow)) + (i == (unsigned)target ? at_target : 0.0f));
    }
  } else {
    // rows that no common vector boundary serves: element by element
    const unsigned i0 = piece * per, i1 = min(i0 + per, vocab);
    for (unsigned i = i0 + tid; i < i1; i += LANES)
      out[i] = Pack<T>::round(grad(at_least(Pack<T>::one(x[i]), Pack<T>::kLow)) + (i == (unsigned)target ? at_target : 0.0f));
  }
}

template <typename T>
cudaError_t run(const LogprobArgs& a, cudaStream_t s) {
  // Short rows; up to half of that where many alternatives are asked for, which the short kernel takes one by one (8192 rows of
  // 1000 bf16 logits: with 5 alternatives 34 us on either, with 20 103 us against 68; of 257: 39 against 230).
  if (a.vocab <= (a.top_k <= 8 ? kShort : kShort / 2)) return launch(logprob_short_kernel<T>, dim3((unsigned)((a.rows + kRowWarps - 1) / kRowWarps)), kRowThreads, 0, s, a);
  // A row to a CTA when there are rows for half of the multiprocessors; below, a cluster of eight to a row.
  if (a.rows * 2 >= a.sms || a.vocab < 4096) return launch(logprob_kernel<T, 1>, dim3((unsigned)a.rows), kRowThreads, 0, s, a);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.rows * kCluster);
  cfg.blockDim = dim3(kRowThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<T, kCluster>, a);
}

template <typename T>
cudaError_t run_grad(const LogprobGradArgs& a, cudaStream_t s) {
  const long long per = (long long)kRowThreads * kGradVecs * Pack<T>::N;
  if (a.vocab <= per / kRowWarps) return launch(logprob_grad_kernel<T, 32>, dim3((unsigned)((a.rows + kRowWarps - 1) / kRowWarps)), kRowThreads, 0, s, a, 1);
  const long long pieces = (a.vocab + per - 1) / per;
  // a grid has at most 2^31 - 1 CTAs: more rows go in several launches
  const long long most = 0x7fffffffll / pieces;
  LogprobGradArgs b = a;
  for (long long r = 0; r < a.rows; r += most) {
    b.rows = a.rows - r < most ? a.rows - r : most;
    const cudaError_t e = launch(logprob_grad_kernel<T, kRowThreads>, dim3((unsigned)(b.rows * pieces)), kRowThreads, 0, s, b, (int)pieces);
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
