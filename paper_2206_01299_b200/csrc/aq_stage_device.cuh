// Device pieces that the stage operators' kernels share: 16-bit types, mbarriers with bounded waits, programmatic launch.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/aq_b200.h"

namespace aq {
namespace {

template <typename T> struct Num;
template <> struct Num<__half> {
  static __device__ __half one(float x) { return __float2half_rn(x); }
  static __device__ float2 open(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
  static __device__ uint32_t close(float a, float b) { const __half2 p = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&p); }
};
template <> struct Num<__nv_bfloat16> {
  static __device__ __nv_bfloat16 one(float x) { return __float2bfloat16_rn(x); }
  static __device__ float2 open(uint32_t u) { return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
  static __device__ uint32_t close(float a, float b) { const __nv_bfloat162 p = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&p); }
};

// programmatic launch: the next kernel of the stream may be placed; the results of the previous one are needed from here
__device__ void next_may_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ void barrier_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
constexpr uint32_t kSleepNs = 100000;         // how long a try may sleep: a thread that polls takes issue slots and power from the products
__device__ bool barrier_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity), "r"(kSleepNs) : "memory");
  return done != 0;
}
__device__ unsigned long long now_ns() { unsigned long long t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
// Waits for a phase; false (and the status bit) when it has not come within four seconds: the caller leaves its loop.
__device__ __noinline__ bool barrier_wait_long(uint32_t bar, uint32_t parity, uint32_t* status) {
  const unsigned long long until = now_ns() + 4000000000ull;
  do {
    for (int i = 0; i < 64; ++i)
      if (barrier_try(bar, parity)) return true;
  } while (now_ns() < until);
  atomicOr(status, (uint32_t)AQ_ST_STALLED);
  return false;
}
__device__ bool barrier_wait(uint32_t bar, uint32_t parity, uint32_t* status) {
#pragma unroll 1
  for (int i = 0; i < 16; ++i)
    if (barrier_try(bar, parity)) return true;
  return barrier_wait_long(bar, parity, status);
}
// one lane waits for its warp
__device__ bool warp_wait(int lane, uint32_t bar, uint32_t parity, uint32_t* status) {
  int ok = 1;
  if (lane == 0) ok = barrier_wait(bar, parity, status);
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}

// A launch that may be placed while the stream's previous kernel drains (the kernels wait for its results themselves).
template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 ctas, unsigned threads, size_t shared, cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = ctas;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = s;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace
}  // namespace aq
