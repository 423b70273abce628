// One optimizer step over many tensors (AdamW, moments in 32 bits or in 8) and the 2-norm of their gradients.
//
//   g' = factor g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
//   p = p - lr decay p - (lr / c1) m / (sqrt(v / c2) + eps),   c = 1 - beta^step
//
// Every element is read once and written once and shares nothing with another, so the step is bound by memory.  The tensors'
// addresses and sizes travel in the launch's arguments: a captured graph holds them, and no copy has to arrive before the
// kernel may start.  A CTA takes a run of neighbouring chunks of 2048 elements, of one tensor after the other; a warp 256
// elements of a chunk, eight to a lane.
//
// Moments in 8 bits.  A warp's 256 elements are a block with one scale per moment: the smallest power of two that keeps the
// block's largest magnitude in the format (m e4m3, up to 1.75 * 2^8; v e5m2, up to 1.75 * 2^15).  Powers of two, since scaling by them
// rounds nothing.  v changes by a thousandth of itself in a step, less than a hundredth of the distance between two values of
// e5m2: rounded to the nearest it would never move.  So roundings are random: the value goes to its upper neighbour where
// its place between the two and a random fraction add up to one, 16 bits each for m and v from a hash of the element's index and the step
// (two multiplications; a Weyl sequence over the steps is cheaper, but what v becomes depends on the sequence's past, and
// v then falls 13 percent too fast).  In the bits of a binary32 that is one addition below the last bit that is kept.
// This step's p goes by the m and v before they are rounded.  The products and sums of m and v are rounded one by one (no
// fused multiply-add), so that the stored codes are a matter of the formula and not of the compiler.

#include "aq_stage.h"
#include "aq_stage_device.cuh"

namespace aq {
namespace {

constexpr int kAdamThreads = 256, kAdamWarps = kAdamThreads / 32;
constexpr int kAdamCtas = 4, kNormCtasPerSm = 8;
constexpr uint32_t kRoot3 = 0xBB67AE85u, kGolden = 0x9E3779B9u;   // fractions of the square root of 3 and of the golden ratio, times 2^32

template <int N> struct Table {
  AdamPart part[N];
  long long first[N + 1];                     // chunks of the tensors before this one
  int n;
};

// Eight values of a lane.  Wide: neighbours, by 16-byte accesses; otherwise every 32nd element.
template <typename T> struct Eight {
  static __device__ void load(const T* p, float* f) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 a = Num<T>::open(w[i]); f[2 * i] = a.x; f[2 * i + 1] = a.y; }
  }
  static __device__ void store(T* p, const float* f) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(Num<T>::close(f[0], f[1]), Num<T>::close(f[2], f[3]), Num<T>::close(f[4], f[5]), Num<T>::close(f[6], f[7])));
  }
  static __device__ float one(T x) { return (float)x; }
  static __device__ T back(float x) { return Num<T>::one(x); }
};
template <> struct Eight<float> {
  static __device__ void load(const float* p, float* f) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  static __device__ void store(float* p, const float* f) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
  }
  static __device__ float one(float x) { return x; }
  static __device__ float back(float x) { return x; }
};

// Which elements of a tensor a lane has: `wide` ones are all there.
struct Lane8 {
  bool wide;
  long long at;                               // of the first
  long long numel;
  __device__ long long place(int j) const { return wide ? at + j : at + 32 * j; }
  __device__ bool has(int j) const { return wide || at + 32 * j < numel; }
};

template <typename T> __device__ void take(const Lane8& l, const void* from, float* f) {
  const T* const p = static_cast<const T*>(from) + l.at;
  if (l.wide) {
    Eight<T>::load(p, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = l.has(j) ? Eight<T>::one(p[32 * j]) : 0.0f;
  }
}
template <typename T> __device__ void put(const Lane8& l, void* to, const float* f) {
  T* const p = static_cast<T*>(to) + l.at;
  if (l.wide) {
    Eight<T>::store(p, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (l.has(j)) p[32 * j] = Eight<T>::back(f[j]);
  }
}
__device__ uint2 take_codes(const Lane8& l, const void* from) {
  const uint8_t* const p = static_cast<const uint8_t*>(from) + l.at;
  if (l.wide) return __ldcs(reinterpret_cast<const uint2*>(p));
  uint32_t c[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) c[j] = l.has(j) ? p[32 * j] : 0;
  return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
}
__device__ void put_codes(const Lane8& l, void* to, const uint32_t* c) {
  uint8_t* const p = static_cast<uint8_t*>(to) + l.at;
  if (l.wide) {
    __stcs(reinterpret_cast<uint2*>(p), make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (l.has(j)) p[32 * j] = (uint8_t)c[j];
  }
}

__device__ float2 half_pair(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
// values of eight codes, before the scale; every one is a binary16 number
__device__ void open_e4m3(uint2 c, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint16_t two = (uint16_t)((i < 2 ? c.x : c.y) >> (16 * (i & 1)));
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
    const float2 a = half_pair(h);
    f[2 * i] = a.x;
    f[2 * i + 1] = a.y;
  }
}
__device__ void open_e5m2(uint2 c, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {               // e5m2 is the upper byte of a binary16
    const uint32_t two = (i < 2 ? c.x : c.y) >> (16 * (i & 1));
    const float2 a = half_pair((two & 0xffu) << 8 | (two & 0xff00u) << 16);
    f[2 * i] = a.x;
    f[2 * i + 1] = a.y;
  }
}

// A block's scale 2^k from its largest magnitude, given as the bits of the binary32; top: the format's largest exponent.
// The formats end at 1.75 * 2^top, so a magnitude above 1.75 of its octave counts to the next one.  Infinities and NaN: NaN.
__device__ int scale_exponent(uint32_t largest, int top) { return max((int)((largest + 0x1fffffu) >> 23) - 127 - top, -126); }
__device__ float power_of_two(int k) { return __uint_as_float((uint32_t)(127 + k) << 23); }

struct Clock { float step_size, root_c2, lr; uint32_t key; };

// The random bits of an element at a step: for m the lower half, for v the upper.
__device__ uint32_t step_key(uint32_t step) {
  uint32_t k = step * kGolden;
  k = (k ^ (k >> 16)) * kRoot3;
  k = (k ^ (k >> 15)) * kGolden;
  return k ^ (k >> 16);
}
__device__ uint32_t random_bits(uint32_t place, uint32_t key) {
  uint32_t u = (place + key) * kRoot3;
  u = (u ^ (u >> 15)) * kGolden;
  return u ^ (u >> 16);
}

__device__ double power(double base, uint64_t n) {
  double p = 1.0;
  for (; n; n >>= 1) {
    if (n & 1) p *= base;
    base *= base;
  }
  return p;
}

template <typename T, int BITS, int N>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtas) adamw_kernel(const __grid_constant__ Table<N> table, const __grid_constant__ AdamScalars a) {
  __shared__ Clock shared_clock;
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  next_may_launch();
  wait_for_previous();
  const float factor = a.factor ? __ldg(a.factor) : 1.0f;
  if (!(fabsf(factor) < __int_as_float(0x7f800000))) return;   // a step that is to be left out
  if (threadIdx.x == 0) {
    const float lr = a.d_lr ? __ldg(a.d_lr) : a.lr;
    float c1 = a.c1, c2 = a.c2;
    uint32_t step = a.step;
    if (a.d_step) {
      const int64_t t = max(__ldg(reinterpret_cast<const long long*>(a.d_step)), 1ll);
      step = (uint32_t)t;
      c1 = (float)(1.0 - power(a.beta1_exact, (uint64_t)t));
      c2 = (float)(1.0 - power(a.beta2_exact, (uint64_t)t));
    }
    shared_clock = Clock{lr / c1, sqrtf(1.0f / c2), lr, step_key(step)};
  }
  __syncthreads();
  const Clock clock = shared_clock;

  const long long chunks = table.first[table.n];
  long long c = chunks * blockIdx.x / gridDim.x;
  const long long end = chunks * (blockIdx.x + 1) / gridDim.x;
  int t = 0;
  for (int hi = table.n; hi - t > 1;) {       // the tensor that has chunk c
    const int mid = (t + hi) / 2;
    if (table.first[mid] <= c) t = mid; else hi = mid;
  }
  for (; c < end; ++c) {
    while (table.first[t + 1] <= c) ++t;
    const AdamPart& part = table.part[t];
    const long long base = (c - table.first[t]) * kAdamChunk + warp * 256;
    if (base >= part.numel) continue;
    Lane8 l;
    l.numel = part.numel;
    l.wide = (part.flags & kPartWide) && base + 256 <= part.numel;
    l.at = base + (l.wide ? lane * 8 : lane);
    float g[8], p[8], m[8], v[8];
    uint2 cm, cv;
    float sm = 0.0f, sv = 0.0f;
    const long long block = base / 256;
    if (part.flags & kPartGradF32) take<float>(l, part.grad, g); else take<T>(l, part.grad, g);
    if (part.master) take<float>(l, part.master, p); else take<T>(l, part.param, p);
    if (BITS == 32) {
      take<float>(l, part.m, m);
      take<float>(l, part.v, v);
    } else {
      cm = take_codes(l, part.m);
      cv = take_codes(l, part.v);
      sm = part.m_scale[block];
      sv = part.v_scale[block];
      open_e4m3(cm, m);
      open_e5m2(cv, v);
    }
    uint32_t largest_m = 0, largest_v = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (BITS == 8) { m[j] = __fmul_rn(m[j], sm); v[j] = __fmul_rn(v[j], sv); }
      const float gj = __fmul_rn(g[j], factor);
      m[j] = __fadd_rn(__fmul_rn(m[j], a.beta1), __fmul_rn(gj, a.rest1));
      v[j] = __fadd_rn(__fmul_rn(v[j], a.beta2), __fmul_rn(__fmul_rn(gj, gj), a.rest2));
      if (BITS == 8) {
        largest_m = max(largest_m, __float_as_uint(m[j]) & 0x7fffffffu);
        largest_v = max(largest_v, __float_as_uint(v[j]) & 0x7fffffffu);
      }
      float root;
      asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v[j]));
      const float update = __fdividef(m[j], fmaf(root, clock.root_c2, a.eps));
      p[j] -= fmaf(clock.step_size, update, clock.lr * part.decay * p[j]);
    }
    if (part.master) put<float>(l, part.master, p);
    put<T>(l, part.param, p);
    if (BITS == 32) {
      put<float>(l, part.m, m);
      put<float>(l, part.v, v);
    } else {
      largest_m = __reduce_max_sync(0xffffffffu, largest_m);
      largest_v = __reduce_max_sync(0xffffffffu, largest_v);
      const int km = scale_exponent(largest_m, 8), kv = scale_exponent(largest_v, 15);
      const float im = power_of_two(-km), iv = power_of_two(-kv);
      uint32_t em[8], ev[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t u = random_bits((uint32_t)l.place(j), clock.key);
        // scaled so that the formats' exponents are binary32's smallest, subnormal numbers among them
        const float ym = __fmul_rn(__fmul_rn(fabsf(m[j]), im), 0x1p-120f), yv = __fmul_rn(__fmul_rn(v[j], iv), 0x1p-112f);
        em[j] = min((__float_as_uint(ym) + ((u & 0xffffu) << 4)) >> 20, 0x7eu) | (__float_as_uint(m[j]) >> 24 & 0x80u);
        ev[j] = max(min((__float_as_uint(yv) + ((u >> 16) << 5)) >> 21, 0x7bu), v[j] > 0.0f ? 1u : 0u);
      }
      put_codes(l, part.m, em);
      put_codes(l, part.v, ev);
      if (lane == 0) {
        const float nan = __int_as_float(0x7fc00000);
        part.m_scale[block] = largest_m < 0x7f800000u ? power_of_two(km) : nan;
        part.v_scale[block] = largest_v < 0x7f800000u ? power_of_two(kv) : nan;
      }
    }
  }
}

// ---- 2-norm of the gradients ------------------------------------------------------------------------------------

// Squares of eight elements are added in binary32, then everything in binary64: a stage has up to billions of them.
template <typename T, int N>
__global__ void __launch_bounds__(kAdamThreads) grad_norm_kernel(const __grid_constant__ Table<N> table, const __grid_constant__ NormScalars a) {
  __shared__ double sums[kAdamWarps];
  __shared__ bool last_cta;
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  next_may_launch();
  wait_for_previous();
  const long long chunks = table.first[table.n];
  long long c = chunks * blockIdx.x / gridDim.x;
  const long long end = chunks * (blockIdx.x + 1) / gridDim.x;
  int t = 0;
  for (int hi = table.n; hi - t > 1;) {
    const int mid = (t + hi) / 2;
    if (table.first[mid] <= c) t = mid; else hi = mid;
  }
  double sum = 0.0;
#pragma unroll 1
  for (; c < end; ++c) {
    while (table.first[t + 1] <= c) ++t;
    const AdamPart& part = table.part[t];
    const long long base = (c - table.first[t]) * kAdamChunk + warp * 256;
    if (base >= part.numel) continue;
    Lane8 l;
    l.numel = part.numel;
    l.wide = (part.flags & kPartWide) && base + 256 <= part.numel;
    l.at = base + (l.wide ? lane * 8 : lane);
    float g[8], s = 0.0f;
    if (part.flags & kPartGradF32) take<float>(l, part.grad, g); else take<T>(l, part.grad, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(g[j], g[j], s);
    sum += (double)s;
  }
  auto join = [&](double x) {                 // the CTA's sum, for thread 0
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) sums[warp] = x;
    __syncthreads();
    x = 0.0;
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < kAdamWarps; ++i) x += sums[i];
    }
    return x;
  };
  sum = join(sum);
  if (threadIdx.x == 0) {
    __stcg(a.partials + blockIdx.x, sum);
    __threadfence();
    last_cta = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last_cta) return;
  __threadfence();
  sum = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kAdamThreads) sum += __ldcg(a.partials + i);
  sum = join(sum);
  if (threadIdx.x) return;
  *a.ticket = 0;
  double* const before = a.partials + kNormCtas;
  if (!a.first) sum += *before;
  if (!a.last) { *before = sum; return; }
  const double norm = sqrt(sum) * a.inv_scale;
  const bool fine = norm <= 1.7976931348623157e308;
  if (a.norm) *a.norm = (float)norm;
  if (a.factor) *a.factor = fine ? (float)(a.inv_scale * fmin(1.0, a.max_norm / (norm + 1e-6))) : __int_as_float(0x7fc00000);
  if (a.step && fine) ++*a.step;
}

template <int N> void fill(Table<N>& table, const AdamPart* parts, int n) {
  long long chunks = 0;
  for (int i = 0; i < n; ++i) {
    table.part[i] = parts[i];
    table.first[i] = chunks;
    chunks += (parts[i].numel + kAdamChunk - 1) / kAdamChunk;
  }
  for (int i = n; i <= N; ++i) table.first[i] = chunks;
  table.n = n;
}

template <int N, typename Kernel, typename Scalars>
cudaError_t start(Kernel kernel, const AdamPart* parts, int n, const Scalars& a, long long ctas, cudaStream_t s) {
  Table<N> table;
  fill(table, parts, n);
  const long long chunks = table.first[n];
  const unsigned grid = (unsigned)(chunks < 1 ? 1 : chunks < ctas ? chunks : ctas);
  return launch(kernel, dim3(grid), kAdamThreads, 0, s, table, a);
}

// Most calls of few tensors are short: a small table spares them 30 KB of arguments.
constexpr int kSmallTable = 24;

template <typename T, int BITS> cudaError_t run_adamw(const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s) {
  if (n <= kSmallTable) return start<kSmallTable>(adamw_kernel<T, BITS, kSmallTable>, parts, n, a, (long long)kAdamCtas * sms, s);
  return start<kAdamTable>(adamw_kernel<T, BITS, kAdamTable>, parts, n, a, (long long)kAdamCtas * sms, s);
}

template <typename T> cudaError_t run_norm(const AdamPart* parts, int n, const NormScalars& a, int sms, cudaStream_t s) {
  const long long most = (long long)kNormCtasPerSm * sms < kNormCtas ? (long long)kNormCtasPerSm * sms : kNormCtas;
  if (n <= kSmallTable) return start<kSmallTable>(grad_norm_kernel<T, kSmallTable>, parts, n, a, most, s);
  return start<kAdamTable>(grad_norm_kernel<T, kAdamTable>, parts, n, a, most, s);
}

}  // namespace

cudaError_t launch_adamw(int dtype, int state_bits, const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  if (state_bits == 8) {
    if (dtype == AQ_FP16) return run_adamw<__half, 8>(parts, n, a, sms, s);
    if (dtype == AQ_BF16) return run_adamw<__nv_bfloat16, 8>(parts, n, a, sms, s);
    return run_adamw<float, 8>(parts, n, a, sms, s);
  }
  if (dtype == AQ_FP16) return run_adamw<__half, 32>(parts, n, a, sms, s);
  if (dtype == AQ_BF16) return run_adamw<__nv_bfloat16, 32>(parts, n, a, sms, s);
  return run_adamw<float, 32>(parts, n, a, sms, s);
}

cudaError_t launch_grad_norm(int dtype, const AdamPart* parts, int n, const NormScalars& a, int sms, cudaStream_t s) {
  if (dtype == AQ_FP16) return run_norm<__half>(parts, n, a, sms, s);
  if (dtype == AQ_BF16) return run_norm<__nv_bfloat16>(parts, n, a, sms, s);
  return run_norm<float>(parts, n, a, sms, s);
}

}  // namespace aq
