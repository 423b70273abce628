// Gated feed-forward product and its gradient.
//
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u;   dg = dh u act'(g),  du = dh act(g),
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x.

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/aq_b200.h"
#include "aq_stage.h"

namespace aq {
namespace {

template <typename T> struct Num;
template <> struct Num<__half> {
  static __device__ float to(__half x) { return __half2float(x); }
  static __device__ __half from(float x) { return __float2half_rn(x); }
};
template <> struct Num<__nv_bfloat16> {
  static __device__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
};

// act(g) and act'(g)
template <int ACT> __device__ void activation(float g, float* a, float* da) {
  if (ACT == AQ_ACT_GELU) {
    const float cdf = 0.5f * erfcf(-0.70710678f * g);
    *a = g * cdf;
    *da = fmaf(g * 0.3989422804f, __expf(-0.5f * g * g), cdf);
    return;
  }
  // g sigmoid(y): y = g, or the cubic whose sigmoid is (1 + tanh(y / 2)) / 2
  const float y = ACT == AQ_ACT_SILU ? g : 1.5957691216f * g * fmaf(0.044715f * g, g, 1.0f);
  const float dy = ACT == AQ_ACT_SILU ? 1.0f : 1.5957691216f * fmaf(3.0f * 0.044715f * g, g, 1.0f);
  const float sig = __fdividef(1.0f, 1.0f + __expf(-y));
  *a = g * sig;
  *da = sig + g * sig * (1.0f - sig) * dy;
}

// 64 x 64 sums of products, 16 deep at a time: c[i][j] += sum_k A(row0 + i, k) B(col0 + j, k), element (i, k) of A at
// A[i * ar + k * ak].
template <typename T>
__device__ void products(float (&c)[4][4], const T* A, long long ar, long long ak, long long rows, const T* B, long long br, long long bk,
                         long long cols, long long row0, long long col0, long long depth, float (*sa)[65], float (*sb)[65]) {
  const int tid = threadIdx.x, ti = tid / 16, tj = tid % 16;
  for (long long k0 = 0; k0 < depth; k0 += 16) {
    __syncthreads();
    for (int i = tid; i < 1024; i += 256) {
      const int r = i / 16, k = i % 16;
      sa[k][r] = row0 + r < rows && k0 + k < depth ? Num<T>::to(A[(row0 + r) * ar + (k0 + k) * ak]) : 0.0f;
      sb[k][r] = col0 + r < cols && k0 + k < depth ? Num<T>::to(B[(col0 + r) * br + (k0 + k) * bk]) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = fmaf(sa[k][ti * 4 + i], sb[k][tj * 4 + j], c[i][j]);
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(256) ffn_kernel(const FfnArgs a) {
  __shared__ float sa[16][65], sb[16][65];
  const long long row0 = (long long)blockIdx.x * 64, col0 = (long long)blockIdx.y * 64;
  float cg[4][4] = {}, cu[4][4] = {};
  products<T>(cg, static_cast<const T*>(a.x), a.ldx, 1, a.rows, static_cast<const T*>(a.wg), a.ldw, 1, a.inner, row0, col0, a.hidden, sa, sb);
  products<T>(cu, static_cast<const T*>(a.x), a.ldx, 1, a.rows, static_cast<const T*>(a.wu), a.ldw, 1, a.inner, row0, col0, a.hidden, sa, sb);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long r = row0 + threadIdx.x / 16 * 4 + i, c = col0 + threadIdx.x % 16 * 4 + j;
      if (r >= a.rows || c >= a.inner) continue;
      float act, dact;
      activation<ACT>(cg[i][j], &act, &dact);
      static_cast<T*>(a.h)[r * a.ldh + c] = Num<T>::from(act * cu[i][j]);
      if (a.g) {
        static_cast<T*>(a.g)[r * a.ldgu + c] = Num<T>::from(cg[i][j]);
        static_cast<T*>(a.u)[r * a.ldgu + c] = Num<T>::from(cu[i][j]);
      }
    }
}

// dg and du to the workspace
template <typename T, int ACT>
__global__ void __launch_bounds__(256) ffn_dgu_kernel(const FfnGradArgs a) {
  const long long n = a.rows * a.inner;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long r = i / a.inner, c = i % a.inner;
    float act, dact;
    activation<ACT>(Num<T>::to(static_cast<const T*>(a.g)[r * a.ldgu + c]), &act, &dact);
    const float dh = Num<T>::to(static_cast<const T*>(a.dh)[r * a.lddh + c]), u = Num<T>::to(static_cast<const T*>(a.u)[r * a.ldgu + c]);
    static_cast<T*>(a.dg)[i] = Num<T>::from(dh * u * dact);
    static_cast<T*>(a.du)[i] = Num<T>::from(dh * act);
  }
}

template <typename T>
__device__ void store_tile(const float (&c)[4][4], void* out, long long ld, long long rows, long long cols, long long row0, long long col0) {
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long r = row0 + threadIdx.x / 16 * 4 + i, k = col0 + threadIdx.x % 16 * 4 + j;
      if (r < rows && k < cols) static_cast<T*>(out)[r * ld + k] = Num<T>::from(c[i][j]);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) ffn_dx_kernel(const FfnGradArgs a) {
  __shared__ float sa[16][65], sb[16][65];
  const long long row0 = (long long)blockIdx.x * 64, col0 = (long long)blockIdx.y * 64;
  float c[4][4] = {};
  products<T>(c, static_cast<const T*>(a.dg), a.inner, 1, a.rows, static_cast<const T*>(a.wg), 1, a.ldw, a.hidden, row0, col0, a.inner, sa, sb);
  products<T>(c, static_cast<const T*>(a.du), a.inner, 1, a.rows, static_cast<const T*>(a.wu), 1, a.ldw, a.hidden, row0, col0, a.inner, sa, sb);
  store_tile<T>(c, a.dx, a.lddx, a.rows, a.hidden, row0, col0);
}

template <typename T>
__global__ void __launch_bounds__(256) ffn_dw_kernel(const FfnGradArgs a) {
  __shared__ float sa[16][65], sb[16][65];
  const long long row0 = (long long)blockIdx.x * 64, col0 = (long long)blockIdx.y * 64;
  float c[4][4] = {};
  products<T>(c, static_cast<const T*>(blockIdx.z ? a.du : a.dg), 1, a.inner, a.inner, static_cast<const T*>(a.x), 1, a.ldx, a.hidden, row0, col0, a.rows, sa, sb);
  store_tile<T>(c, blockIdx.z ? a.dwu : a.dwg, a.lddw, a.inner, a.hidden, row0, col0);
}

unsigned tiles(long long n) { return (unsigned)((n + 63) / 64); }

template <typename T>
cudaError_t run(const FfnArgs& a, cudaStream_t s) {
  const dim3 grid(tiles(a.rows), tiles(a.inner));
  if (a.act == AQ_ACT_SILU) ffn_kernel<T, AQ_ACT_SILU><<<grid, 256, 0, s>>>(a);
  else if (a.act == AQ_ACT_GELU) ffn_kernel<T, AQ_ACT_GELU><<<grid, 256, 0, s>>>(a);
  else ffn_kernel<T, AQ_ACT_GELU_TANH><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t run_grad(const FfnGradArgs& a, cudaStream_t s) {
  const unsigned ctas = (unsigned)a.sms * 8;
  if (a.act == AQ_ACT_SILU) ffn_dgu_kernel<T, AQ_ACT_SILU><<<ctas, 256, 0, s>>>(a);
  else if (a.act == AQ_ACT_GELU) ffn_dgu_kernel<T, AQ_ACT_GELU><<<ctas, 256, 0, s>>>(a);
  else ffn_dgu_kernel<T, AQ_ACT_GELU_TANH><<<ctas, 256, 0, s>>>(a);
  if (a.dx) ffn_dx_kernel<T><<<dim3(tiles(a.rows), tiles(a.hidden)), 256, 0, s>>>(a);
  if (a.dwg) ffn_dw_kernel<T><<<dim3(tiles(a.inner), tiles(a.hidden), 2), 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_ffn(int dtype, const FfnArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run<__half>(a, s) : run<__nv_bfloat16>(a, s);
}
cudaError_t launch_ffn_grad(int dtype, const FfnGradArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_grad<__half>(a, s) : run_grad<__nv_bfloat16>(a, s);
}

}  // namespace aq
