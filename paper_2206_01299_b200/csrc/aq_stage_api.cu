// C ABI of the stage operators: handle, argument checks, workspace.  Nothing here computes on the CPU.

#include "../../include/aq_b200.h"
#include "aq_stage.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

// A workspace that was outgrown while a captured graph may still hold its address.
struct KeptBlock {
  void* block;
  KeptBlock* next;
};

struct aq_stage {
  int device = 0, sms = 0, pairs = 0;
  int dtype = AQ_FP16;
  cudaStream_t stream = nullptr;
  uint32_t* status = nullptr;
  uint32_t *ticket = nullptr, *next = nullptr;   // in the status word's allocation
  float* partials = nullptr;              // aq_qk_norm_rope_grad, aq_grad_norm
  void* work = nullptr;                   // aq_gated_ffn_grad, aq_layer_norm_grad
  size_t work_bytes = 0;
  bool work_captured = false;             // a stream capture has taken its address
  KeptBlock* kept = nullptr;              // freed with the handle
  char err[256] = {0};
  int err_code = AQ_OK;
};

namespace {

thread_local char g_stage_err[256] = "";
thread_local int g_stage_code = AQ_OK;

int fail(aq_stage* st, int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(st ? st->err : g_stage_err, 256, fmt, ap);
  va_end(ap);
  (st ? st->err_code : g_stage_code) = code;
  return code;
}

int cuda_fail(aq_stage* st, cudaError_t e, const char* what) {
  cudaGetLastError();                        // reported here, not by whatever asks the runtime next
  return fail(st, e == cudaErrorMemoryAllocation ? AQ_ENOMEM : AQ_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

bool misaligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// The handle's device must be current for launches on its stream; restored on exit.
struct DeviceGuard {
  int prev = -1;
  explicit DeviceGuard(int dev) {
    cudaGetDevice(&prev);
    if (prev != dev) cudaSetDevice(dev);
    else prev = -1;
  }
  ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

int launched(aq_stage* st, cudaError_t e, const char* what) { return e == cudaSuccess ? AQ_OK : cuda_fail(st, e, what); }

// Makes the workspace at least that large.  A block whose address went into a captured graph is kept until the handle is destroyed,
// for the graph may be replayed at any time; any other may still be used by work in flight, so the stream is drained before it is freed.
int ensure_work(aq_stage* st, size_t bytes) {
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  cudaError_t e = cudaStreamIsCapturing(st->stream, &capture);
  if (e != cudaSuccess) return cuda_fail(st, e, "cudaStreamIsCapturing");
  if (st->work_bytes >= bytes) {
    if (capture != cudaStreamCaptureStatusNone) st->work_captured = true;
    return AQ_OK;
  }
  if (capture != cudaStreamCaptureStatusNone)
    return fail(st, AQ_EUNSUPPORTED, "the workspace has to grow to %zu bytes, which a stream capture does not allow: run the call once before", bytes);
  if (st->work_captured) {
    KeptBlock* const k = new (std::nothrow) KeptBlock{st->work, st->kept};
    if (!k) return fail(st, AQ_ENOMEM, "host allocation failed");
    st->kept = k;
  } else {
    e = cudaStreamSynchronize(st->stream);
    if (e != cudaSuccess) return cuda_fail(st, e, "cudaStreamSynchronize");
    cudaFree(st->work);
  }
  st->work = nullptr;
  st->work_bytes = 0;
  st->work_captured = false;
  e = cudaMalloc(&st->work, bytes);
  if (e != cudaSuccess) return cuda_fail(st, e, "workspace");
  st->work_bytes = bytes;
  return AQ_OK;
}

int check_rows_vocab(aq_stage* st, const char* who, int64_t rows, int64_t vocab, int64_t ld, float scale) {
  if (rows < 0 || rows > 0x7fffffffll) return fail(st, AQ_EINVAL, "%s: rows must be in 0..2^31-1", who);
  if (vocab < 1 || vocab > 0x7fffffffll) return fail(st, AQ_EINVAL, "%s: vocab must be in 1..2^31-1", who);
  if (ld < vocab) return fail(st, AQ_EINVAL, "%s: ld is smaller than vocab", who);
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(st, AQ_EINVAL, "%s: scale must be positive and finite", who);
  return AQ_OK;
}

int check_ffn(aq_stage* st, const char* who, int64_t rows, int hidden, int inner, int act) {
  if (st->dtype == AQ_FP32) return fail(st, AQ_EUNSUPPORTED, "%s: 16-bit types only", who);
  if (rows < 0 || rows > 0x7fffffffll - 4096) return fail(st, AQ_EINVAL, "%s: rows out of range", who);
  if (hidden < 1 || inner < 1 || hidden > (1 << 24) || inner > (1 << 24)) return fail(st, AQ_EINVAL, "%s: hidden and inner must be in 1..2^24", who);
  if (hidden % 8 || inner % 8) return fail(st, AQ_EUNSUPPORTED, "%s: hidden and inner must be multiples of 8", who);
  if (act != AQ_ACT_SILU && act != AQ_ACT_GELU && act != AQ_ACT_GELU_TANH) return fail(st, AQ_EINVAL, "%s: unknown activation %d", who, act);
  return AQ_OK;
}

// A T[..][cols] operand with a row stride: present, aligned, rows that do not overlap.
int check_matrix(aq_stage* st, const char* who, const char* name, const void* p, int64_t ld, int64_t cols) {
  if (!p || misaligned(p, 16)) return fail(st, AQ_EINVAL, "%s: %s is null or not 16-byte aligned", who, name);
  if (ld < cols || ld % 8 || ld > (1ll << 38)) return fail(st, AQ_EINVAL, "%s: the row stride of %s must be a multiple of 8 and at least %lld", who, name, (long long)cols);
  return AQ_OK;
}

int check_qk(aq_stage* st, const char* who, const aq_qk_shape* sh, int64_t rows, const void* wq, const void* wk, const float* cos_sin,
             const int32_t* positions) {
  if (st->dtype == AQ_FP32) return fail(st, AQ_EUNSUPPORTED, "%s: 16-bit types only", who);
  if (!sh) return fail(st, AQ_EINVAL, "%s: null shape", who);
  if (rows < 0 || rows > 0x7fffffffll) return fail(st, AQ_EINVAL, "%s: rows out of range", who);
  if (sh->heads_q < 0 || sh->heads_k < 0 || sh->heads_q > 65536 || sh->heads_k > 65536 || sh->heads_q + sh->heads_k < 1)
    return fail(st, AQ_EINVAL, "%s: heads_q and heads_k must be in 0..65536, one of them positive", who);
  if (sh->head_dim < 8 || sh->head_dim > 256 || sh->head_dim % 8) return fail(st, AQ_EINVAL, "%s: head_dim must be a multiple of 8 in 8..256 (got %d)", who, sh->head_dim);
  if (sh->rot_dim < 0 || sh->rot_dim > sh->head_dim || sh->rot_dim % 2) return fail(st, AQ_EINVAL, "%s: rot_dim must be even and in 0..head_dim (got %d)", who, sh->rot_dim);
  if (!(sh->eps >= 0.0f) || !std::isfinite(sh->eps)) return fail(st, AQ_EINVAL, "%s: eps must be finite and not negative", who);
  if (misaligned(wq, 16) || misaligned(wk, 16)) return fail(st, AQ_EINVAL, "%s: wq or wk is not 16-byte aligned", who);
  if (sh->rot_dim) {
    if (!cos_sin || misaligned(cos_sin, 16) || !positions || misaligned(positions, 4)) return fail(st, AQ_EINVAL, "%s: cos_sin or positions is null or misaligned", who);
    if (sh->n_positions < 1 || sh->n_positions > 0x7fffffffll) return fail(st, AQ_EINVAL, "%s: n_positions must be in 1..2^31-1", who);
  }
  return AQ_OK;
}

aq::QkArgs qk_args(aq_stage* st, const aq_qk_shape* sh, int64_t rows, const void* wq, const void* wk, const float* cos_sin, const int32_t* positions) {
  aq::QkArgs a{};
  a.heads_q = sh->heads_q; a.heads_k = sh->heads_k; a.head_dim = sh->head_dim; a.rot_dim = sh->rot_dim;
  a.interleaved = sh->interleaved != 0; a.eps = sh->eps; a.n_positions = sh->n_positions; a.rows = rows;
  a.wq = wq; a.wk = wk; a.cos_sin = cos_sin; a.positions = positions;
  a.partials = st->partials; a.ticket = st->ticket; a.status = st->status; a.sms = st->sms;
  return a;
}

unsigned size_of(int dtype) { return dtype == AQ_FP32 ? 4 : 2; }

// How the rows of a layer norm's operands lie to one another and to 16-byte boundaries.
struct NormRows {
  bool some = false, begin = true, whole = true, alike = true;   // begin: the first rows on boundaries; whole: all
  int64_t place = 0, stride = 0;                                 // in elements, mod a piece
};

// A T[..][hidden] operand of the layer norm: element alignment and any stride do.
int check_norm_rows(aq_stage* st, const char* who, const char* name, const void* p, int64_t ld, int64_t hidden, NormRows* r) {
  const unsigned size = size_of(st->dtype);
  if (!p || misaligned(p, size)) return fail(st, AQ_EINVAL, "%s: %s is null or misaligned", who, name);
  if (ld < hidden || ld > (1ll << 38)) return fail(st, AQ_EINVAL, "%s: the row stride of %s must be at least %lld", who, name, (long long)hidden);
  const int64_t piece = 16 / size, place = (int64_t)(reinterpret_cast<uintptr_t>(p) / size % piece), stride = ld % piece;
  if (r->some && (place != r->place || stride != r->stride)) r->alike = false;
  if (place) r->begin = false;
  if (place || stride) r->whole = false;
  r->some = true;
  r->place = place;
  r->stride = stride;
  return AQ_OK;
}

int check_norm(aq_stage* st, const char* who, int64_t rows, int hidden, const void* w, const void* b) {
  if (rows < 0 || rows > 0x7fffffffll) return fail(st, AQ_EINVAL, "%s: rows must be in 0..2^31-1", who);
  if (hidden < 1 || hidden > (1 << 20)) return fail(st, AQ_EINVAL, "%s: hidden must be in 1..2^20 (got %d)", who, hidden);
  const unsigned size = size_of(st->dtype);
  if (misaligned(w, size) || misaligned(b, size)) return fail(st, AQ_EINVAL, "%s: w or b is misaligned", who);
  return AQ_OK;
}

// Two operands in one place have to have the same rows.
int check_in_place(aq_stage* st, const char* who, const void* out, int64_t ld_out, const void* in, int64_t ld_in) {
  if (out && out == in && ld_out != ld_in) return fail(st, AQ_EINVAL, "%s: in place, the row strides must be equal", who);
  return AQ_OK;
}

int check_adam_tensor(aq_stage* st, const char* who, int64_t i, const aq_adam_tensor& t) {
  if (t.numel < 0 || t.numel > (1ll << 40)) return fail(st, AQ_EINVAL, "%s: tensor %lld: numel must be in 0..2^40", who, (long long)i);
  if (t.grad_dtype != st->dtype && t.grad_dtype != AQ_FP32) return fail(st, AQ_EINVAL, "%s: tensor %lld: grad_dtype must be the handle's element type or AQ_FP32", who, (long long)i);
  if (t.numel && (!t.grad || misaligned(t.grad, size_of(t.grad_dtype)))) return fail(st, AQ_EINVAL, "%s: tensor %lld: grad is null or misaligned", who, (long long)i);
  return AQ_OK;
}

int check_adam_state(aq_stage* st, const char* who, int64_t i, const aq_adam_tensor& t, int bits) {
  if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay)) return fail(st, AQ_EINVAL, "%s: tensor %lld: weight_decay must be finite and not negative", who, (long long)i);
  if (!t.numel) return AQ_OK;
  if (!t.param || misaligned(t.param, size_of(st->dtype))) return fail(st, AQ_EINVAL, "%s: tensor %lld: param is null or misaligned", who, (long long)i);
  if (t.master && st->dtype == AQ_FP32) return fail(st, AQ_EINVAL, "%s: tensor %lld: binary32 parameters have no master copy", who, (long long)i);
  if (misaligned(t.master, 4)) return fail(st, AQ_EINVAL, "%s: tensor %lld: master is misaligned", who, (long long)i);
  if (!t.m || !t.v || (bits == 32 && (misaligned(t.m, 4) || misaligned(t.v, 4)))) return fail(st, AQ_EINVAL, "%s: tensor %lld: m or v is null or misaligned", who, (long long)i);
  if (bits == 8 && (!t.m_scale || !t.v_scale || misaligned(t.m_scale, 4) || misaligned(t.v_scale, 4)))
    return fail(st, AQ_EINVAL, "%s: tensor %lld: m_scale or v_scale is null or misaligned", who, (long long)i);
  // with scales, m and v are codes, a quarter of what a step of 32 bits reads and writes
  if (bits == 32 && (t.m_scale || t.v_scale)) return fail(st, AQ_EINVAL, "%s: tensor %lld: m_scale and v_scale belong to state_bits 8", who, (long long)i);
  return AQ_OK;
}

// Elements of p until the next multiple of eight of them.
int until_eight(const void* p, int bytes) { return (int)((8 - (reinterpret_cast<uintptr_t>(p) / bytes & 7)) & 7); }

// The next tensors that are not empty, from element *from of tensor *i on, in parts of at most kPartMost elements, at most kAdamTable of
// them; bits 0: gradients only.
int gather_parts(aq_stage* st, const aq_adam_tensor* tensors, int64_t n, int bits, int64_t* i, int64_t* from, aq::AdamPart* parts) {
  int have = 0;
  for (; *i < n; ++*i, *from = 0) {
    const aq_adam_tensor& t = tensors[*i];
    const int size = (int)size_of(st->dtype), grad_size = (int)size_of(t.grad_dtype), state_size = bits == 8 ? 1 : 4;
    // how far all addresses are from a multiple of eight elements, if they agree
    const int head = until_eight(t.grad, grad_size);
    bool agree = true;
    if (bits) agree = until_eight(t.param, size) == head && (!t.master || until_eight(t.master, 4) == head) && until_eight(t.m, state_size) == head && until_eight(t.v, state_size) == head;
    const bool f32 = t.grad_dtype == AQ_FP32 && st->dtype != AQ_FP32;
    for (int64_t count; *from < t.numel; *from += count) {
      if (have == aq::kAdamTable) return have;
      const int64_t e = *from;
      // a few elements by themselves, and the rest begins where wide accesses may; blocks of 8-bit moments are counted from the beginning and stay
      const bool first = agree && head && e == 0 && bits != 8;
      count = first ? head : aq::kPartMost;
      if (count > t.numel - e) count = t.numel - e;
      auto at = [e](const void* p, int bytes) { return p ? const_cast<char*>(static_cast<const char*>(p)) + e * bytes : nullptr; };
      aq::AdamPart& p = parts[have++];
      p = aq::AdamPart{};
      p.grad = at(t.grad, grad_size);
      if (bits) {
        p.param = at(t.param, size);
        p.master = t.master ? t.master + e : nullptr;
        p.m = at(t.m, state_size);
        p.v = at(t.v, state_size);
        if (bits == 8) { p.m_scale = t.m_scale + e / 256; p.v_scale = t.v_scale + e / 256; }
        p.decay = t.weight_decay;
      }
      p.numel = (uint32_t)count;
      p.place = (uint32_t)e;
      p.flags = (agree && !first ? aq::kPartWide : 0u) | (agree && bits == 8 ? (uint32_t)((8 - head) & 7) << aq::kPartShiftBit : 0u) | (f32 ? aq::kPartGradF32 : 0u);
    }
  }
  return have;
}

#define AQ_TRY(expr) do { const int rc_ = (expr); if (rc_ != AQ_OK) return rc_; } while (0)

}  // namespace

extern "C" {

aq_stage* aq_stage_create(void) {
  g_stage_err[0] = 0;
  g_stage_code = AQ_OK;
  aq_stage* st = new (std::nothrow) aq_stage();
  if (!st) { fail(nullptr, AQ_ENOMEM, "host allocation failed"); return nullptr; }
  cudaError_t e = cudaGetDevice(&st->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&st->sms, cudaDevAttrMultiProcessorCount, st->device);
  if (e == cudaSuccess) e = aq::ffn_resident_pairs(&st->pairs);
  if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&st->status), 256);
  if (e == cudaSuccess) e = cudaMemset(st->status, 0, 256);
  if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void**>(&st->partials), sizeof(float) * aq::kQkGradCtas * 2 * 256);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();                    // the memset above is on another stream than the handle's may be
  if (e != cudaSuccess) {
    cuda_fail(nullptr, e, "aq_stage_create");
    cudaFree(st->status);
    cudaFree(st->partials);
    delete st;
    return nullptr;
  }
  st->ticket = st->status + 16;
  st->next = st->status + 32;
  return st;
}

void aq_stage_destroy(aq_stage* st) {
  if (!st) return;
  DeviceGuard guard(st->device);
  cudaStreamSynchronize(st->stream);
  cudaFree(st->status);
  cudaFree(st->partials);
  cudaFree(st->work);
  while (st->kept) {
    KeptBlock* const k = st->kept;
    st->kept = k->next;
    cudaFree(k->block);
    delete k;
  }
  delete st;
}

int aq_stage_configure(aq_stage* st, int key, int64_t value) {
  if (!st) return AQ_EINVAL;
  switch (key) {
    case AQ_DTYPE:
      if (value != AQ_FP16 && value != AQ_BF16 && value != AQ_FP32) return fail(st, AQ_EINVAL, "AQ_DTYPE must be AQ_FP16, AQ_BF16 or AQ_FP32");
      st->dtype = (int)value;
      return AQ_OK;
    case AQ_STREAM:
      st->stream = reinterpret_cast<cudaStream_t>(static_cast<intptr_t>(value));
      return AQ_OK;
    default:
      return fail(st, AQ_EINVAL, "unknown key %d for a stage handle", key);
  }
}

int aq_stage_status(aq_stage* st, uint32_t* bits_host) {
  if (!st) return AQ_EINVAL;
  if (!bits_host) return fail(st, AQ_EINVAL, "aq_stage_status: null pointer");
  DeviceGuard guard(st->device);
  cudaError_t e = cudaMemcpyAsync(bits_host, st->status, sizeof(uint32_t), cudaMemcpyDeviceToHost, st->stream);
  if (e == cudaSuccess) e = cudaMemsetAsync(st->status, 0, 256, st->stream);   // and the counters, which a kernel that gave up leaves as they were
  if (e == cudaSuccess) e = cudaStreamSynchronize(st->stream);
  return launched(st, e, "aq_stage_status");
}

const char* aq_stage_last_error(aq_stage* st) { return st ? st->err : g_stage_err; }
int aq_stage_last_error_code(aq_stage* st) { return st ? st->err_code : g_stage_code; }

int aq_token_logprobs(aq_stage* st, const void* logits, int64_t rows, int64_t vocab, int64_t ld, const int32_t* targets,
                      float scale, int top_k, float* logprob, float* entropy, float* lse, int32_t* top_ids, float* top_logprobs) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_token_logprobs";
  AQ_TRY(check_rows_vocab(st, who, rows, vocab, ld, scale));
  if (top_k < 0 || top_k > aq::kMaxTop || top_k > vocab) return fail(st, AQ_EINVAL, "%s: top_k must be in 0..min(vocab, %d) (got %d)", who, aq::kMaxTop, top_k);
  if (rows == 0) return AQ_OK;
  const unsigned size = st->dtype == AQ_FP32 ? 4 : 2;
  if (!logits || misaligned(logits, size)) return fail(st, AQ_EINVAL, "%s: logits is null or misaligned", who);
  if (misaligned(targets, 4) || misaligned(logprob, 4) || misaligned(entropy, 4) || misaligned(lse, 4) || misaligned(top_ids, 4) || misaligned(top_logprobs, 4))
    return fail(st, AQ_EINVAL, "%s: misaligned pointer", who);
  if (logprob && !targets) return fail(st, AQ_EINVAL, "%s: logprob without targets", who);
  DeviceGuard guard(st->device);
  const aq::LogprobArgs a{logits, rows, vocab, ld, targets, scale, top_ids || top_logprobs ? top_k : 0, logprob, entropy, lse, top_ids, top_logprobs, st->status, st->sms};
  return launched(st, aq::launch_logprob(st->dtype, a, st->stream), who);
}

int aq_token_logprobs_grad(aq_stage* st, const void* logits, int64_t rows, int64_t vocab, int64_t ld, const int32_t* targets,
                           float scale, const float* lse, const float* entropy, const float* d_logprob, const float* d_entropy,
                           void* d_logits, int64_t ld_d) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_token_logprobs_grad";
  AQ_TRY(check_rows_vocab(st, who, rows, vocab, ld, scale));
  if (ld_d < vocab) return fail(st, AQ_EINVAL, "%s: ld_d is smaller than vocab", who);
  if (rows == 0) return AQ_OK;
  const unsigned size = st->dtype == AQ_FP32 ? 4 : 2;
  if (!logits || misaligned(logits, size) || !d_logits || misaligned(d_logits, size)) return fail(st, AQ_EINVAL, "%s: logits or d_logits is null or misaligned", who);
  if (!lse || misaligned(lse, 4) || misaligned(targets, 4) || misaligned(entropy, 4) || misaligned(d_logprob, 4) || misaligned(d_entropy, 4))
    return fail(st, AQ_EINVAL, "%s: lse is null, or a pointer is misaligned", who);
  if (d_logprob && !targets) return fail(st, AQ_EINVAL, "%s: d_logprob without targets", who);
  if (d_entropy && !entropy) return fail(st, AQ_EINVAL, "%s: d_entropy without entropy", who);
  if (logits == d_logits && ld != ld_d) return fail(st, AQ_EINVAL, "%s: in place, ld and ld_d must be equal", who);
  DeviceGuard guard(st->device);
  const aq::LogprobGradArgs a{logits, rows, vocab, ld, targets, scale, lse, entropy, d_logprob, d_entropy, d_logits, ld_d, st->status};
  return launched(st, aq::launch_logprob_grad(st->dtype, a, st->stream), who);
}

int aq_gated_ffn(aq_stage* st, const void* x, int64_t ldx, const void* wg, const void* wu, int64_t ldw, int64_t rows, int hidden,
                 int inner, int act, void* h, int64_t ldh, void* g, void* u, int64_t ldgu) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_gated_ffn";
  AQ_TRY(check_ffn(st, who, rows, hidden, inner, act));
  if (!g != !u) return fail(st, AQ_EINVAL, "%s: g and u are given both or not at all", who);
  if (rows == 0) return AQ_OK;
  AQ_TRY(check_matrix(st, who, "x", x, ldx, hidden));
  AQ_TRY(check_matrix(st, who, "wg", wg, ldw, hidden));
  AQ_TRY(check_matrix(st, who, "wu", wu, ldw, hidden));
  AQ_TRY(check_matrix(st, who, "h", h, ldh, inner));
  if (g) {
    AQ_TRY(check_matrix(st, who, "g", g, ldgu, inner));
    AQ_TRY(check_matrix(st, who, "u", u, ldgu, inner));
  }
  DeviceGuard guard(st->device);
  const aq::FfnArgs a{x, ldx, wg, wu, ldw, rows, hidden, inner, act, h, ldh, g, u, ldgu, st->status, st->next, st->pairs};
  return launched(st, aq::launch_ffn(st->dtype, a, st->stream), who);
}

int aq_gated_ffn_grad(aq_stage* st, const void* dh, int64_t lddh, const void* x, int64_t ldx, const void* wg, const void* wu,
                      int64_t ldw, const void* g, const void* u, int64_t ldgu, int64_t rows, int hidden, int inner, int act,
                      void* dx, int64_t lddx, void* dwg, void* dwu, int64_t lddw) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_gated_ffn_grad";
  AQ_TRY(check_ffn(st, who, rows, hidden, inner, act));
  if (!dwg != !dwu) return fail(st, AQ_EINVAL, "%s: dwg and dwu are given both or not at all", who);
  if (dwg) {
    AQ_TRY(check_matrix(st, who, "dwg", dwg, lddw, hidden));
    AQ_TRY(check_matrix(st, who, "dwu", dwu, lddw, hidden));
  }
  DeviceGuard guard(st->device);
  if (rows == 0) {                                           // no token: the weights' gradients are sums of nothing
    for (void* p : {dwg, dwu}) {
      if (!p) continue;
      const cudaError_t e = cudaMemset2DAsync(p, (size_t)lddw * 2, 0, (size_t)hidden * 2, (size_t)inner, st->stream);
      if (e != cudaSuccess) return cuda_fail(st, e, who);
    }
    return AQ_OK;
  }
  AQ_TRY(check_matrix(st, who, "dh", dh, lddh, inner));
  AQ_TRY(check_matrix(st, who, "x", x, ldx, hidden));
  AQ_TRY(check_matrix(st, who, "wg", wg, ldw, hidden));
  AQ_TRY(check_matrix(st, who, "wu", wu, ldw, hidden));
  AQ_TRY(check_matrix(st, who, "g", g, ldgu, inner));
  AQ_TRY(check_matrix(st, who, "u", u, ldgu, inner));
  if (dx) AQ_TRY(check_matrix(st, who, "dx", dx, lddx, hidden));
  if (!dx && !dwg) return AQ_OK;
  const size_t half = ((size_t)rows * (size_t)inner * 2 + 255) & ~(size_t)255;
  aq::FfnGradArgs a{dh, lddh, x, ldx, wg, wu, ldw, g, u, ldgu, rows, hidden, inner, act, dx, lddx, dwg, dwu, lddw,
                    nullptr, nullptr, nullptr, st->status, st->next, st->sms, st->pairs};
  AQ_TRY(ensure_work(st, 2 * half + (size_t)aq::ffn_grad_partial_bytes(a)));
  a.dg = st->work;
  a.du = static_cast<char*>(st->work) + half;
  a.partial = reinterpret_cast<float*>(static_cast<char*>(st->work) + 2 * half);
  return launched(st, aq::launch_ffn_grad(st->dtype, a, st->stream), who);
}

int aq_qk_norm_rope(aq_stage* st, const aq_qk_shape* shape, int64_t rows, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                    const void* wq, const void* wk, const float* cos_sin, const int32_t* positions,
                    void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_qk_norm_rope";
  AQ_TRY(check_qk(st, who, shape, rows, wq, wk, cos_sin, positions));
  if (rows == 0) return AQ_OK;
  const int64_t nq = (int64_t)shape->heads_q * shape->head_dim, nk = (int64_t)shape->heads_k * shape->head_dim;
  if (nq) {
    AQ_TRY(check_matrix(st, who, "q", q, q_stride, nq));
    AQ_TRY(check_matrix(st, who, "q_out", q_out, q_out_stride, nq));
    if (q == q_out && q_stride != q_out_stride) return fail(st, AQ_EINVAL, "%s: in place, the strides must be equal", who);
  }
  if (nk) {
    AQ_TRY(check_matrix(st, who, "k", k, k_stride, nk));
    AQ_TRY(check_matrix(st, who, "k_out", k_out, k_out_stride, nk));
    if (k == k_out && k_stride != k_out_stride) return fail(st, AQ_EINVAL, "%s: in place, the strides must be equal", who);
  }
  DeviceGuard guard(st->device);
  aq::QkArgs a = qk_args(st, shape, rows, wq, wk, cos_sin, positions);
  a.q = q; a.q_stride = q_stride; a.k = k; a.k_stride = k_stride;
  a.q_out = q_out; a.q_out_stride = q_out_stride; a.k_out = k_out; a.k_out_stride = k_out_stride;
  return launched(st, aq::launch_qk(st->dtype, a, st->stream), who);
}

int aq_qk_norm_rope_grad(aq_stage* st, const aq_qk_shape* shape, int64_t rows, const void* dq_out, int64_t dq_out_stride,
                         const void* dk_out, int64_t dk_out_stride, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                         const void* wq, const void* wk, const float* cos_sin, const int32_t* positions,
                         void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, float* dwq, float* dwk) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_qk_norm_rope_grad";
  AQ_TRY(check_qk(st, who, shape, rows, wq, wk, cos_sin, positions));
  if (misaligned(dwq, 4) || misaligned(dwk, 4)) return fail(st, AQ_EINVAL, "%s: dwq or dwk is misaligned", who);
  DeviceGuard guard(st->device);
  if (rows == 0) {                                           // no token: the weights' gradients are sums of nothing
    for (float* p : {dwq, dwk}) {
      if (!p) continue;
      const cudaError_t e = cudaMemsetAsync(p, 0, sizeof(float) * (size_t)shape->head_dim, st->stream);
      if (e != cudaSuccess) return cuda_fail(st, e, who);
    }
    return AQ_OK;
  }
  const int64_t nq = (int64_t)shape->heads_q * shape->head_dim, nk = (int64_t)shape->heads_k * shape->head_dim;
  if (nq) {
    AQ_TRY(check_matrix(st, who, "dq_out", dq_out, dq_out_stride, nq));
    AQ_TRY(check_matrix(st, who, "q", q, q_stride, nq));
    AQ_TRY(check_matrix(st, who, "dq", dq, dq_stride, nq));
    if (dq == dq_out && dq_stride != dq_out_stride) return fail(st, AQ_EINVAL, "%s: in place, the strides must be equal", who);
  }
  if (nk) {
    AQ_TRY(check_matrix(st, who, "dk_out", dk_out, dk_out_stride, nk));
    AQ_TRY(check_matrix(st, who, "k", k, k_stride, nk));
    AQ_TRY(check_matrix(st, who, "dk", dk, dk_stride, nk));
    if (dk == dk_out && dk_stride != dk_out_stride) return fail(st, AQ_EINVAL, "%s: in place, the strides must be equal", who);
  }
  aq::QkArgs a = qk_args(st, shape, rows, wq, wk, cos_sin, positions);
  a.q = q; a.q_stride = q_stride; a.k = k; a.k_stride = k_stride;
  a.gq = dq_out; a.gq_stride = dq_out_stride; a.gk = dk_out; a.gk_stride = dk_out_stride;
  a.q_out = dq; a.q_out_stride = dq_stride; a.k_out = dk; a.k_out_stride = dk_stride;
  a.dwq = dwq; a.dwk = dwk;
  return launched(st, aq::launch_qk_grad(st->dtype, a, st->stream), who);
}

int aq_layer_norm(aq_stage* st, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* w, const void* b, float eps,
                  int64_t rows, int hidden, void* sum, int64_t lds, void* y, int64_t ldy, float* mean, float* rstd) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_layer_norm";
  NormRows r;
  AQ_TRY(check_norm(st, who, rows, hidden, w, b));
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(st, AQ_EINVAL, "%s: eps must be finite and not negative", who);
  if (misaligned(mean, 4) || misaligned(rstd, 4)) return fail(st, AQ_EINVAL, "%s: mean or rstd is misaligned", who);
  if (sum && !residual) return fail(st, AQ_EINVAL, "%s: sum without residual", who);
  if (rows == 0) return AQ_OK;
  AQ_TRY(check_norm_rows(st, who, "x", x, ldx, hidden, &r));
  AQ_TRY(check_norm_rows(st, who, "y", y, ldy, hidden, &r));
  if (residual) AQ_TRY(check_norm_rows(st, who, "residual", residual, ldr, hidden, &r));
  if (sum) AQ_TRY(check_norm_rows(st, who, "sum", sum, lds, hidden, &r));
  if (sum && sum == y) return fail(st, AQ_EINVAL, "%s: sum and y are two outputs", who);
  AQ_TRY(check_in_place(st, who, y, ldy, x, ldx));
  AQ_TRY(check_in_place(st, who, y, ldy, residual, ldr));
  AQ_TRY(check_in_place(st, who, sum, lds, x, ldx));
  AQ_TRY(check_in_place(st, who, sum, lds, residual, ldr));
  DeviceGuard guard(st->device);
  const bool whole = r.whole && hidden % (16 / size_of(st->dtype)) == 0 && !misaligned(w, 16) && !misaligned(b, 16);
  const aq::LayerNormArgs a{x, ldx, residual, ldr, w, b, eps, rows, hidden, sum, lds, y, ldy, mean, rstd,
                            whole ? aq::kRowsWhole : r.alike ? aq::kRowsAlike : aq::kRowsAny};
  return launched(st, aq::launch_layer_norm(st->dtype, a, st->stream), who);
}

int aq_layer_norm_grad(aq_stage* st, const void* dy, int64_t lddy, const void* dsum, int64_t ldds, const void* s, int64_t lds, const void* w,
                       const float* mean, const float* rstd, int64_t rows, int hidden, void* dx, int64_t lddx, float* dw, float* db) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_layer_norm_grad";
  NormRows r;
  AQ_TRY(check_norm(st, who, rows, hidden, w, nullptr));
  if (misaligned(dw, 4) || misaligned(db, 4)) return fail(st, AQ_EINVAL, "%s: dw or db is misaligned", who);
  DeviceGuard guard(st->device);
  if (rows == 0) {                                           // no token: the weights' gradients are sums of nothing
    for (float* p : {dw, db}) {
      if (!p) continue;
      const cudaError_t e = cudaMemsetAsync(p, 0, sizeof(float) * (size_t)hidden, st->stream);
      if (e != cudaSuccess) return cuda_fail(st, e, who);
    }
    return AQ_OK;
  }
  AQ_TRY(check_norm_rows(st, who, "dy", dy, lddy, hidden, &r));
  AQ_TRY(check_norm_rows(st, who, "s", s, lds, hidden, &r));
  if (dsum) AQ_TRY(check_norm_rows(st, who, "dsum", dsum, ldds, hidden, &r));
  if (dx) AQ_TRY(check_norm_rows(st, who, "dx", dx, lddx, hidden, &r));
  AQ_TRY(check_in_place(st, who, dx, lddx, dy, lddy));
  AQ_TRY(check_in_place(st, who, dx, lddx, dsum, ldds));
  AQ_TRY(check_in_place(st, who, dx, lddx, s, lds));
  if (!mean || !rstd || misaligned(mean, 4) || misaligned(rstd, 4)) return fail(st, AQ_EINVAL, "%s: mean or rstd is null or misaligned", who);
  if (!dx && !dw && !db) return AQ_OK;
  aq::LayerNormGradArgs a{dy, lddy, dsum, ldds, s, lds, w, mean, rstd, rows, hidden, dx, lddx, dw, db, nullptr,
                          r.whole ? aq::kRowsWhole : r.alike && r.begin ? aq::kRowsAlike : aq::kRowsAny, 1, (int)size_of(st->dtype), st->sms};
  if (dw || db) AQ_TRY(ensure_work(st, (size_t)aq::layer_norm_grad_bytes(a)));
  a.partials = static_cast<float*>(st->work);
  return launched(st, aq::launch_layer_norm_grad(st->dtype, a, st->stream), who);
}

int aq_grad_norm(aq_stage* st, const aq_adam_tensor* tensors, int64_t n, double inv_scale, double max_norm, float* norm, float* factor, int64_t* step) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_grad_norm";
  if (n < 0 || (n && !tensors)) return fail(st, AQ_EINVAL, "%s: tensors is null, or n is negative", who);
  if (!((float)inv_scale > 0.0f) || !std::isfinite((float)inv_scale)) return fail(st, AQ_EINVAL, "%s: inv_scale must be positive and finite in binary32", who);
  if (!(max_norm >= 0.0)) return fail(st, AQ_EINVAL, "%s: max_norm must not be negative or NaN", who);
  if (misaligned(norm, 4) || misaligned(factor, 4) || misaligned(step, 8)) return fail(st, AQ_EINVAL, "%s: misaligned pointer", who);
  for (int64_t i = 0; i < n; ++i) AQ_TRY(check_adam_tensor(st, who, i, tensors[i]));
  DeviceGuard guard(st->device);
  aq::NormScalars a{reinterpret_cast<double*>(st->partials), st->ticket, true, false, inv_scale, max_norm > 0.0 ? max_norm : INFINITY, norm, factor, step};
  aq::AdamPart parts[aq::kAdamTable];
  for (int64_t i = 0, from = 0; !a.last; a.first = false) {
    const int have = gather_parts(st, tensors, n, 0, &i, &from, parts);
    a.last = i >= n;
    AQ_TRY(launched(st, aq::launch_grad_norm(st->dtype, parts, have, a, st->sms, st->stream), who));
  }
  return AQ_OK;
}

int aq_adamw(aq_stage* st, const aq_adamw_config* config, const aq_adam_tensor* tensors, int64_t n, const float* factor, const float* d_lr,
             const int64_t* d_step) {
  if (!st) return AQ_EINVAL;
  const char* who = "aq_adamw";
  if (!config) return fail(st, AQ_EINVAL, "%s: null config", who);
  if (n < 0 || (n && !tensors)) return fail(st, AQ_EINVAL, "%s: tensors is null, or n is negative", who);
  if (config->state_bits != 32 && config->state_bits != 8) return fail(st, AQ_EINVAL, "%s: state_bits must be 32 or 8 (got %d)", who, config->state_bits);
  if (!(config->beta1 >= 0.0 && config->beta1 < 1.0 && config->beta2 >= 0.0 && config->beta2 < 1.0)) return fail(st, AQ_EINVAL, "%s: beta1 and beta2 must be in [0, 1)", who);
  if (!(config->eps >= 1e-12) || !(config->eps < 1e30)) return fail(st, AQ_EINVAL, "%s: eps must be in 1e-12..1e30", who);
  if (!d_lr && !std::isfinite((float)config->lr)) return fail(st, AQ_EINVAL, "%s: lr must be finite", who);
  if (!d_step && config->step < 1) return fail(st, AQ_EINVAL, "%s: step counts from 1", who);
  if (misaligned(factor, 4) || misaligned(d_lr, 4) || misaligned(d_step, 8)) return fail(st, AQ_EINVAL, "%s: misaligned pointer", who);
  for (int64_t i = 0; i < n; ++i) {
    AQ_TRY(check_adam_tensor(st, who, i, tensors[i]));
    AQ_TRY(check_adam_state(st, who, i, tensors[i], config->state_bits));
  }
  DeviceGuard guard(st->device);
  aq::AdamScalars a{};
  a.beta1 = (float)config->beta1; a.rest1 = (float)(1.0 - config->beta1);
  a.beta2 = (float)config->beta2; a.rest2 = (float)(1.0 - config->beta2);
  a.one = 1.0f;
  a.beta1_exact = config->beta1; a.beta2_exact = config->beta2;
  a.eps = (float)config->eps;
  a.factor = factor; a.d_lr = d_lr; a.d_step = d_step;
  if (!d_lr) a.lr = (float)config->lr;
  if (!d_step) {
    a.step = (uint32_t)config->step;
    a.c1 = (float)(1.0 - std::pow(config->beta1, (double)config->step));
    a.c2 = (float)(1.0 - std::pow(config->beta2, (double)config->step));
  }
  aq::AdamPart parts[aq::kAdamTable];
  for (int64_t i = 0, from = 0; i < n;) {
    const int have = gather_parts(st, tensors, n, config->state_bits, &i, &from, parts);
    AQ_TRY(launched(st, aq::launch_adamw(st->dtype, config->state_bits, parts, have, a, st->sms, st->stream), who));
  }
  return AQ_OK;
}

}  // extern "C"
