// Launch-layer interface between the stage handle's C ABI (aq_stage_api.cu) and its kernels
// (aq_logprob.cu, aq_qknorm.cu, aq_ffn.cu, aq_layernorm.cu, aq_adamw.cu).
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

// Where the rows of a layer norm's operands begin: all on 16-byte boundaries (forward: w and b too, and rows are whole pieces of 16
// bytes), at the same distance from one in all operands (gradient: the first rows on boundaries), or anywhere.
enum { kRowsWhole = 0, kRowsAlike = 1, kRowsAny = 2 };

struct LayerNormArgs {
  const void* x; long long ldx;
  const void* residual; long long ldr;    // may be null
  const void *w, *b;                      // may be null
  float eps;
  long long rows; int hidden;
  void* sum; long long lds;               // may be null
  void* y; long long ldy;
  float *mean, *rstd;                     // may be null
  int rows_at;                            // where rows begin
};

struct LayerNormGradArgs {
  const void* dy; long long lddy;
  const void* dsum; long long ldds;       // may be null
  const void* s; long long lds;
  const void* w;                          // may be null
  const float *mean, *rstd;
  long long rows; int hidden;
  void* dx; long long lddx;               // may be null
  float *dw, *db;                         // may be null
  float* partials;                        // workspace, layer_norm_grad_bytes of it: sums of dw and db of each CTA
  int rows_at, period;                    // period: rows from one to the next that begins at the same place in a 16-byte piece; set by the launch
  int size, sms;                          // size: of an element
};

// The `index`-th piece of n elements of a row of the layer norm's gradient.  Rows begin `shift` elements behind a 16-byte boundary and pieces lie on
// boundaries, so the first one's column is -shift; of a piece's elements [lo, hi) are the row's, none where hi is 0.
struct NormPiece { int column, lo, hi; };
__host__ __device__ inline NormPiece norm_piece(int index, int n, int shift, int hidden) {
  const int column = index * n - shift, rest = hidden - column;
  return {column, column < 0 ? -column : 0, rest < 0 ? 0 : rest < n ? rest : n};
}
// Column from which the asynchronous copy of a piece's first hi elements begins.  The copy of none has to begin on a boundary as well, which a
// shifted row itself does not.
__host__ __device__ inline int norm_copy_from(int column, int hi, int shift) { return hi ? column : -shift; }

// A tensor of a step, or a part of a long one, as the kernels read it.
struct AdamPart {
  void* param;
  float* master;                          // may be null
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;               // 8-bit moments only
  uint32_t numel;                         // at most kPartMost: longer tensors come in several
  uint32_t place;                         // index of its first element in its tensor, mod 2^32
  float decay;
  uint32_t flags;                         // kPartWide, kPartGradF32
};
constexpr uint32_t kPartMost = 1u << 30;
constexpr uint32_t kPartWide = 1;         // every address is a multiple of eight elements, or as many elements behind one as flags >> kPartShiftBit says
constexpr int kPartShiftBit = 8;          // with 8-bit moments only, whose blocks are counted from the tensor's beginning
constexpr uint32_t kPartGradF32 = 2;      // the gradient is binary32 beside 16-bit parameters
constexpr int kAdamTable = 400;           // tensors of a launch: 72 bytes each and 4 of a running count, of 32764 bytes of arguments

struct AdamScalars {
  float beta1, rest1, beta2, rest2, one;  // rest: 1 - beta; one: 1
  float eps, lr, c1, c2;                  // c: 1 - beta^step
  double beta1_exact, beta2_exact;
  uint32_t step;                          // mod 2^32
  const float* factor;                    // may be null
  const float* d_lr;                      // may be null
  const int64_t* d_step;                  // may be null
};

struct NormScalars {
  double* partials;                       // a CTA's sum each, kNormCtas; behind them the sum of the launches before
  uint32_t* ticket;                       // CTAs that have written theirs; 0 between calls
  bool first, last;                       // of the launches of a call
  double inv_scale, max_norm;             // max_norm: infinite for none
  float *norm, *factor;                   // may be null
  int64_t* step;                          // may be null
};
constexpr int kNormCtas = 2048;

cudaError_t launch_logprob(int dtype, const LogprobArgs& a, cudaStream_t s);
cudaError_t launch_logprob_grad(int dtype, const LogprobGradArgs& a, cudaStream_t s);
cudaError_t launch_qk(int dtype, const QkArgs& a, cudaStream_t s);
cudaError_t launch_qk_grad(int dtype, const QkArgs& a, cudaStream_t s);
cudaError_t ffn_resident_pairs(int* pairs);       // of the current device
// bytes of `partial` that a call needs; goes by the sizes, pairs and which outputs there are
long long ffn_grad_partial_bytes(const FfnGradArgs& a);
cudaError_t launch_ffn(int dtype, const FfnArgs& a, cudaStream_t s);
cudaError_t launch_ffn_grad(int dtype, const FfnGradArgs& a, cudaStream_t s);
cudaError_t launch_layer_norm(int dtype, const LayerNormArgs& a, cudaStream_t s);
// bytes of `partials` that a call with dw or db needs; goes by the sizes, the row stride of s, rows_at and sms
long long layer_norm_grad_bytes(const LayerNormGradArgs& a);
cudaError_t launch_layer_norm_grad(int dtype, const LayerNormGradArgs& a, cudaStream_t s);
// `parts`: 0..kAdamTable tensors, none of them empty; they travel in the launch's arguments
cudaError_t launch_adamw(int dtype, int state_bits, const AdamPart* parts, int n, const AdamScalars& a, int sms, cudaStream_t s);
cudaError_t launch_grad_norm(int dtype, const AdamPart* parts, int n, const NormScalars& a, int sms, cudaStream_t s);

}  // namespace aq
