// Launch-layer interface between the stage handle's C ABI (aq_stage_api.cu) and its kernels
// (aq_logprob.cu, aq_qknorm.cu, aq_ffn.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace aq {

constexpr int kMaxTop = 32;               // alternatives aq_token_logprobs reports at most

struct LogprobArgs {
  const void* logits;
  long long rows, vocab, ld;
  const int32_t* targets;                 // may be null
  float scale;
  int top_k;
  float *logprob, *entropy, *lse;         // may be null
  int32_t* top_ids;                       // may be null
  float* top_logprobs;                    // may be null
  uint32_t* status;
  int sms;
};

struct LogprobGradArgs {
  const void* logits;
  long long rows, vocab, ld;
  const int32_t* targets;                 // may be null
  float scale;
  const float *lse, *entropy;             // entropy may be null
  const float *d_logprob, *d_entropy;     // may be null
  void* d_logits;
  long long ld_d;
  uint32_t* status;
};

struct QkArgs {
  int heads_q, heads_k, head_dim, rot_dim, interleaved;
  float eps;
  long long n_positions, rows;
  const void *q, *k;                      // inputs
  long long q_stride, k_stride;
  const void *wq, *wk;                    // may be null
  const float* cos_sin;                   // may be null
  const int32_t* positions;               // may be null
  const void *gq, *gk;                    // gradients of the outputs (backward only)
  long long gq_stride, gk_stride;
  void *q_out, *k_out;                    // outputs: q, k forward; dq, dk backward
  long long q_out_stride, k_out_stride;
  float *dwq, *dwk;                       // backward only, may be null
  float* partials;                        // [kQkGradCtas][2][256] sums of dwq, dwk of each CTA
  uint32_t* ticket;                       // CTAs that have written theirs; 0 between calls
  uint32_t* status;
  int sms;
};
constexpr int kQkGradCtas = 1024;         // most CTAs of the backward kernel

struct FfnArgs {
  const void* x; long long ldx;
  const void *wg, *wu; long long ldw;
  long long rows; int hidden, inner, act;
  void* h; long long ldh;
  void *g, *u; long long ldgu;            // may be null
  uint32_t* status;
  uint32_t* next;                         // two counters of the CTA pairs; 0 between calls
  int pairs;                              // CTA pairs resident at a time
};

struct FfnGradArgs {
  const void* dh; long long lddh;
  const void* x; long long ldx;
  const void *wg, *wu; long long ldw;
  const void *g, *u; long long ldgu;
  long long rows; int hidden, inner, act;
  void* dx; long long lddx;               // may be null
  void *dwg, *dwu; long long lddw;        // may be null
  void *dg, *du;                          // T[rows][inner], workspace
  float* partial;                         // workspace, ffn_grad_partial_bytes of it
  uint32_t* status;
  uint32_t* next;
  int sms, pairs;
};

cudaError_t launch_logprob(int dtype, const LogprobArgs& a, cudaStream_t s);
cudaError_t launch_logprob_grad(int dtype, const LogprobGradArgs& a, cudaStream_t s);
cudaError_t launch_qk(int dtype, const QkArgs& a, cudaStream_t s);
cudaError_t launch_qk_grad(int dtype, const QkArgs& a, cudaStream_t s);
cudaError_t ffn_resident_pairs(int* pairs);       // of the current device
// bytes of `partial` that a call needs; goes by the sizes, pairs and which outputs there are
long long ffn_grad_partial_bytes(const FfnGradArgs& a);
cudaError_t launch_ffn(int dtype, const FfnArgs& a, cudaStream_t s);
cudaError_t launch_ffn_grad(int dtype, const FfnGradArgs& a, cudaStream_t s);

}  // namespace aq
