// C ABI of the kernel-level entry points: argument checks, then the launcher.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>
#include <new>
#include <vector>

#include "../../include/mimose.h"
#include "kernels.h"

// sets what mimose_last_error(NULL) returns on this thread (mimose.cpp)
void mimose_set_thread_error(const char* msg);

namespace {
inline bool bad_dtype(int d) { return d != 0 && d != 1; }
inline int done() { return hipGetLastError() == hipSuccess ? MIMOSE_OK : MIMOSE_ERR_HIP; }
inline bool bad_head(int d) { return d != 32 && d != 64; }
// refuses a call: what mimose_last_error(NULL) returns says why
int refuse(const char* op, const char* why) {
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", op, why);
  mimose_set_thread_error(buf);
  return MIMOSE_ERR_INVALID_ARG;
}
// what is wrong with rows of logits and the gradient beside them, or null
const char* bad_logits(int dtype, const void* logits, int64_t ld, const int32_t* labels, const void* dlogits, int T, int V) {
  if (bad_dtype(dtype)) return "dtype must be 0 (fp32) or 1 (bf16)";
  if (T < 0 || V < 1 || ld < V) return "T >= 0, V >= 1 and ld >= V required";
  if (T > 0 && (!logits || !labels)) return "logits and labels must be given";
  const uintptr_t es = mk::elt_size(dtype), a = (uintptr_t)logits, b = (uintptr_t)dlogits;
  if (ld > INT32_MAX) return "ld too large";
  if (a % es || b % es || (uintptr_t)labels % 4) return "a pointer is not aligned to its elements";
  const uintptr_t bytes = T > 0 ? ((uintptr_t)(T - 1) * ld + ld) * es : 0;
  if (b && a != b && a < b + bytes && b < a + bytes) return "dlogits overlaps the logits without being them";
  return nullptr;
}
}  // namespace

extern "C" {

int mimose_op_gemm(int32_t dtype, const void* A, int64_t lda, int32_t a_kmajor, const void* B, int64_t ldb,
                   int32_t b_kmajor, void* C, int64_t ldc, int32_t c_f32, int32_t M, int32_t N, int32_t K,
                   const void* bias, const void* resid, int64_t ldr, void* gelu_out, int32_t gelu,
                   float* a_rowsum, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (bad_dtype(dtype) || !A || !B || !C || M < 0 || N < 0 || K < 0 || gelu < 0 || gelu > 2) return MIMOSE_ERR_INVALID_ARG;
  if (lda < (a_kmajor ? K : M) || ldb < (b_kmajor ? K : N) || ldc < N || (resid && ldr < N)) return MIMOSE_ERR_INVALID_ARG;
  mk::GemmArgs g{A, lda, a_kmajor != 0, B, ldb, b_kmajor != 0, C, ldc, c_f32 != 0, M, N, K};
  g.bias = bias; g.resid = resid; g.ldr = ldr; g.gelu_out = gelu_out; g.gelu = gelu; g.a_rowsum = a_rowsum;
  g.workspace = workspace; g.workspace_bytes = workspace_bytes;
  if (!mk::gemm(dtype, g, (hipStream_t)stream)) return MIMOSE_ERR_INVALID_ARG;
  return done();
}

uint64_t mimose_op_gemm_workspace_bytes(int32_t M, int32_t N) {
  return M > 0 && N > 0 ? mk::gemm_workspace_bytes(M, N) : 0;
}

uint64_t mimose_op_gemm_long_k_workspace_bytes(int32_t N) { return N > 0 ? mk::gemm_long_k_workspace_bytes(N) : 0; }

int mimose_op_layernorm_fwd(int32_t dtype, const void* x, int32_t x_f32, const void* gamma, const void* beta, void* y,
                            int32_t T, int32_t H, float eps, void* stream) {
  if (bad_dtype(dtype) || !x || !gamma || !beta || !y || T < 0 || H < 1 || H > mk::kMaxRowWidth) return MIMOSE_ERR_INVALID_ARG;
  mk::layernorm_fwd(dtype, x, x_f32 != 0, gamma, beta, y, T, H, eps, (hipStream_t)stream);
  return done();
}

int mimose_op_layernorm_bwd(int32_t dtype, const void* dy, int32_t dy_f32, const void* x, int32_t x_f32,
                            const void* gamma, void* dx, const void* add, float* dgamma, float* dbeta, float* partial,
                            int32_t T, int32_t H, float eps, void* stream) {
  if (bad_dtype(dtype) || !dy || !x || !gamma || !dx || !dgamma || !dbeta || !partial || T < 0 || H < 1 ||
      H > mk::kMaxRowWidth || add == dx || (dx == dy && dtype == 1 && dy_f32))
    return MIMOSE_ERR_INVALID_ARG;
  mk::layernorm_bwd(dtype, dy, dy_f32 != 0, x, x_f32 != 0, gamma, dx, add, dgamma, dbeta, partial, T, H, eps,
                    (hipStream_t)stream);
  return done();
}

int32_t mimose_op_partial_rows(int32_t T) { return mk::partial_rows(T); }

int mimose_op_layernorm_bwd_noalloc(int32_t dtype, const void* dy, int32_t dy_f32, const void* x, int32_t x_f32,
                                    const void* gamma, void* dx, const void* add, float* dgamma, float* dbeta,
                                    int32_t T, int32_t H, float eps, void* stream) {
  if (bad_dtype(dtype) || !dy || !x || !gamma || !dx || !dgamma || !dbeta || T < 0 || H < 1 || H > mk::kMaxRowWidth ||
      add == dx || (dx == dy && dtype == 1 && dy_f32)) {
    mimose_set_thread_error("mimose_op_layernorm_bwd_noalloc: bad argument");
    return MIMOSE_ERR_INVALID_ARG;
  }
  const int rc = mk::layernorm_bwd_static(dtype, dy, dy_f32 != 0, x, x_f32 != 0, gamma, dx, add, dgamma, dbeta, T, H, eps,
                                          (hipStream_t)stream);
  if (rc == -1) {
    char buf[200];
    snprintf(buf, sizeof buf,
             "mimose_op_layernorm_bwd_noalloc: %d rows of %d need %lld scratch floats, the fixed array holds %llu",
             T, H, (long long)mk::partial_rows(T) * 2 * H, (unsigned long long)mk::kStaticPartialFloats);
    mimose_set_thread_error(buf);
    return MIMOSE_ERR_INVALID_ARG;
  }
  if (rc != 0) {
    mimose_set_thread_error("mimose_op_layernorm_bwd_noalloc: address of the scratch array not available");
    return MIMOSE_ERR_HIP;
  }
  return done();
}

uint64_t mimose_op_layernorm_bwd_noalloc_max_floats(void) { return mk::kStaticPartialFloats; }

int mimose_op_gelu_bwd(int32_t dtype, void* d, const void* pre, int64_t n, int32_t tanh_form, void* stream) {
  if (bad_dtype(dtype) || !d || !pre || n < 0) return MIMOSE_ERR_INVALID_ARG;
  mk::gelu_bwd(dtype, d, pre, n, tanh_form, (hipStream_t)stream);
  return done();
}

static bool bad_p(float p) { return !(p >= 0.f) || !(p < 1.f); }
static mk::DropDesc make_desc(float p, uint64_t seed, uint32_t site, uint32_t step) {
  mk::DropDesc d;
  if (p <= 0.f) return d;
  d.thr = (uint32_t)std::min(std::floor((double)p * 4294967296.0 + 0.5), 4294967295.0);
  d.scale = (float)(1.0 / (1.0 - (double)p));
  d.k0 = (uint32_t)seed; d.k1 = (uint32_t)(seed >> 32);
  d.site = site; d.step = step;
  return d;
}

int mimose_op_attention_fwd(int32_t dtype, const void* qkv, void* ctx, float* lse, const int32_t* lengths, int32_t B,
                            int32_t L, int32_t nh, int32_t d, int32_t causal, float p_drop, uint64_t seed,
                            uint32_t site, uint32_t step, void* stream) {
  if (bad_dtype(dtype) || !qkv || !ctx || !lse || B < 0 || L < 0 || nh < 1 || bad_head(d) || bad_p(p_drop))
    return MIMOSE_ERR_INVALID_ARG;
  mk::attention_fwd(dtype, qkv, ctx, lse, mk::Rows{lengths, nullptr, 0}, B, L, nh, d, causal, make_desc(p_drop, seed, site, step),
                    (hipStream_t)stream);
  return done();
}

int mimose_op_attention_bwd(int32_t dtype, const void* qkv, const void* ctx, const void* dctx, const float* lse,
                            float* delta, void* dqkv, const int32_t* lengths, int32_t B, int32_t L, int32_t nh,
                            int32_t d, int32_t causal, float p_drop, uint64_t seed, uint32_t site, uint32_t step,
                            void* stream) {
  if (bad_dtype(dtype) || !qkv || !ctx || !dctx || !lse || !delta || !dqkv || B < 0 || L < 0 || nh < 1 || bad_head(d) ||
      bad_p(p_drop))
    return MIMOSE_ERR_INVALID_ARG;
  mk::attention_bwd(dtype, qkv, ctx, dctx, lse, delta, dqkv, mk::Rows{lengths, nullptr, 0}, B, L, nh, d, causal,
                    make_desc(p_drop, seed, site, step), (hipStream_t)stream);
  return done();
}

int mimose_op_dropout(int32_t dtype, void* dst, const void* src, int32_t io_f32, const void* resid, int64_t n, float p,
                      uint64_t seed, uint32_t site, uint32_t step, void* stream) {
  if (bad_dtype(dtype) || !dst || !src || n < 0 || bad_p(p)) return MIMOSE_ERR_INVALID_ARG;
  mk::dropout_apply(dtype, dst, src, io_f32 != 0, resid, n, make_desc(p, seed, site, step), mk::Rows(), 0, 0, 0, (hipStream_t)stream);
  return done();
}

int mimose_op_dropout_layernorm_fwd(int32_t dtype, void* x, int32_t x_f32, const void* resid, const void* gamma,
                                    const void* beta, void* y, int32_t T, int32_t H, float eps, float p, uint64_t seed,
                                    uint32_t site, uint32_t step, void* stream) {
  if (bad_dtype(dtype) || !x || !resid || !gamma || !beta || T < 0 || H < 1 || H > mk::kMaxRowWidth || bad_p(p))
    return MIMOSE_ERR_INVALID_ARG;
  mk::dropout_layernorm_fwd(dtype, x, x_f32 != 0, resid, gamma, beta, y, T, H, eps, make_desc(p, seed, site, step), mk::Rows(), 0, 0,
                            (hipStream_t)stream);
  return done();
}

int mimose_op_layernorm_bwd_dropout(int32_t dtype, const void* dy, int32_t dy_f32, const void* x, int32_t x_f32,
                                    const void* gamma, void* dx, const void* add, void* masked, float* dgamma, float* dbeta,
                                    float* partial, int32_t T, int32_t H, float eps, float p, uint64_t seed, uint32_t site,
                                    uint32_t step, void* stream) {
  if (bad_dtype(dtype) || !dy || !x || !gamma || !dx || !masked || !dgamma || !dbeta || !partial || T < 0 || H < 1 ||
      H > mk::kMaxRowWidth || add == dx || masked == dx || masked == dy || (dx == dy && dtype == 1 && dy_f32) || bad_p(p))
    return MIMOSE_ERR_INVALID_ARG;
  mk::LnBwdMasked ex;
  ex.masked = masked; ex.d = make_desc(p, seed, site, step);
  mk::layernorm_bwd_rows(dtype, dy, dy_f32 != 0, x, x_f32 != 0, gamma, dx, add, partial, T, H, eps, ex, (hipStream_t)stream);
  mk::layernorm_bwd_reduce(partial, dgamma, dbeta, nullptr, T, H, (hipStream_t)stream);
  return done();
}

int mimose_op_softmax_xent(int32_t dtype, void* logits, int64_t ld, const int32_t* labels, float* row_loss,
                           float* loss, int32_t T, int32_t V, int32_t n_valid, void* stream) {
  if (bad_dtype(dtype) || !logits || !labels || !row_loss || !loss || T < 0 || V < 1 || ld < V) return MIMOSE_ERR_INVALID_ARG;
  mk::softmax_xent(dtype, logits, ld, labels, row_loss, loss, T, V, n_valid, (hipStream_t)stream);
  return done();
}

uint64_t mimose_op_token_loss_workspace_bytes(int32_t T) { return mk::token_loss_workspace_bytes(T); }

int mimose_op_token_logprob(int32_t dtype, const void* logits, int64_t ld, const int32_t* labels, float* logp, int32_t T, int32_t V,
                            void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const op = "mimose_op_token_logprob";
  if (const char* why = bad_logits(dtype, logits, ld, labels, nullptr, T, V)) return refuse(op, why);
  if (T == 0) return MIMOSE_OK;
  if (!logp) return refuse(op, "logp must be given");
  if (workspace && ((uintptr_t)workspace & 15)) return refuse(op, "workspace must be 16-byte aligned");
  if (workspace && workspace_bytes < mk::token_loss_workspace_bytes(T)) return refuse(op, "workspace smaller than mimose_op_token_loss_workspace_bytes");
  mk::token_logprob(dtype, logits, ld, labels, logp, T, V, (hipStream_t)stream);
  return done();
}

int mimose_op_preference_loss(int32_t dtype, const void* logits, int64_t ld, const int32_t* labels, const int32_t* ends, int32_t pairs,
                              int32_t L, const float* ref_logp, float beta, float smoothing, void* dlogits, float* logp, float* seq_logp,
                              float* margin, float* loss, int32_t T, int32_t V, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const op = "mimose_op_preference_loss";
  if (const char* why = bad_logits(dtype, logits, ld, labels, dlogits, T, V)) return refuse(op, why);
  if (pairs < 1 || pairs > mk::kMostPairs) return refuse(op, "1 to 2^21 pairs required");
  if (!ends && (L < 0 || (int64_t)2 * pairs * L != T)) return refuse(op, "without ends, T must be 2 * pairs * L");
  if (!ref_logp || !seq_logp || !margin || !loss || (T > 0 && !logp)) return refuse(op, "ref_logp, logp, seq_logp, margin and loss must be given");
  if (const char* why = mk::bad_preference(beta, smoothing)) return refuse(op, why);
  if (T > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < mk::token_loss_workspace_bytes(T)))
    return refuse(op, "workspace must be 16-byte aligned and of mimose_op_token_loss_workspace_bytes");
  mk::PreferenceArgs a;
  a.ends = ends; a.pairs = pairs; a.L = L; a.ref_logp = ref_logp; a.beta = beta; a.smoothing = smoothing;
  a.seq_logp = seq_logp; a.margin = margin; a.loss = loss;
  mk::preference_loss(dtype, logits, ld, labels, a, dlogits, logp, T, V, workspace, (hipStream_t)stream);
  return done();
}

int mimose_op_policy_loss(int32_t dtype, const void* logits, int64_t ld, const int32_t* labels, const float* old_logp,
                          const float* ref_logp, const float* advantage, const float* weight, float scale, float clip_low,
                          float clip_high, float kl_weight, void* dlogits, float* rows, float* stats, int32_t T, int32_t V,
                          void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const op = "mimose_op_policy_loss";
  if (const char* why = bad_logits(dtype, logits, ld, labels, dlogits, T, V)) return refuse(op, why);
  if (!stats || (T > 0 && (!old_logp || !advantage || !rows))) return refuse(op, "old_logp, advantage, rows and stats must be given");
  if ((uintptr_t)rows & 15) return refuse(op, "rows must be 16-byte aligned");
  if (!std::isfinite(scale)) return refuse(op, "scale must be finite");
  if (const char* why = mk::bad_policy(clip_low, clip_high, kl_weight, ref_logp != nullptr)) return refuse(op, why);
  if (workspace && ((uintptr_t)workspace & 15)) return refuse(op, "workspace must be 16-byte aligned");
  if (workspace && workspace_bytes < mk::token_loss_workspace_bytes(T)) return refuse(op, "workspace smaller than mimose_op_token_loss_workspace_bytes");
  mk::PolicyArgs a;
  a.old_logp = old_logp; a.ref_logp = ref_logp; a.advantage = advantage; a.weight = weight;
  a.scale = scale; a.ratio_low = 1.f - clip_low; a.ratio_high = 1.f + clip_high; a.kl_weight = kl_weight;
  a.rows = rows; a.stats = stats;
  mk::policy_loss(dtype, logits, ld, labels, a, dlogits, T, V, (hipStream_t)stream);
  return done();
}

// chunks of a list of tensors, or -1 with what is wrong with it
static int64_t adamw_chunks(const mimose_adamw_tensor* t, int32_t count, int32_t state_bits, const char** why) {
  *why = nullptr;
  if (!t || count < 1) *why = "at least one tensor required";
  else if (state_bits != 8 && state_bits != 32) *why = "state_bits must be 8 or 32";
  if (*why) return -1;
  int64_t chunks = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].n < 0) *why = "a tensor has a negative element count";
    else if (t[i].n == 0) continue;
    else if (!t[i].master || !t[i].grad || !t[i].m || !t[i].v) *why = "master, grad, m and v of a tensor must be given";
    else if (((uintptr_t)t[i].master | (uintptr_t)t[i].grad | (uintptr_t)t[i].m | (uintptr_t)t[i].v | (uintptr_t)t[i].lowp) & 15)
      *why = "master, lowp, grad, m and v of a tensor must be 16-byte aligned";
    else if (state_bits == 8 && (!t[i].m_scale || !t[i].v_scale || (((uintptr_t)t[i].m_scale | (uintptr_t)t[i].v_scale) & 3)))
      *why = "states in 8 bits need m_scale and v_scale, aligned to their elements";
    if (*why) return -1;
    chunks += (t[i].n + mk::kAdamChunk - 1) / mk::kAdamChunk;
    if (chunks >= (1 << 20)) { *why = "too many elements: 2^34 at most"; return -1; }   // a grid's threads are counted in 32 bits
  }
  return chunks;
}
static uint64_t adamw_entries_bytes(int32_t count, int32_t state_bits) {
  const uint64_t e = state_bits == 8 ? sizeof(mk::Adam8Tensor) : sizeof(mk::AdamTensor);
  return (e * (uint64_t)count + 255) / 256 * 256;
}

uint64_t mimose_op_adamw_table_bytes(const mimose_adamw_tensor* tensors, int32_t count, int32_t state_bits) {
  const char* why;
  const int64_t chunks = adamw_chunks(tensors, count, state_bits, &why);
  if (chunks < 0) { refuse("mimose_op_adamw_table_bytes", why); return 0; }
  return adamw_entries_bytes(count, state_bits) + (uint64_t)(chunks > 0 ? chunks : 1) * sizeof(mk::AdamChunk);
}

int mimose_op_adamw_table(const mimose_adamw_tensor* tensors, int32_t count, int32_t state_bits, void* device, uint64_t bytes,
                          mimose_adamw_table* out, void* stream) {
  const char* const op = "mimose_op_adamw_table";
  const char* why;
  const int64_t chunks = adamw_chunks(tensors, count, state_bits, &why);
  if (chunks < 0) return refuse(op, why);
  const uint64_t entries = adamw_entries_bytes(count, state_bits), need = entries + (uint64_t)(chunks > 0 ? chunks : 1) * sizeof(mk::AdamChunk);
  if (!out || !device || ((uintptr_t)device & 15) || bytes < need)
    return refuse(op, "out and 16-byte aligned device memory of mimose_op_adamw_table_bytes must be given");
  try {
    std::vector<char> host(need, 0);
    mk::AdamChunk* c = (mk::AdamChunk*)(host.data() + entries);
    for (int32_t i = 0; i < count; ++i) {
      const mimose_adamw_tensor& t = tensors[i];
      if (state_bits == 8)
        ((mk::Adam8Tensor*)host.data())[i] = {t.master, t.lowp, t.grad, (uint8_t*)t.m, (uint8_t*)t.v, t.m_scale, t.v_scale, t.n, t.decay != 0, 0};
      else
        ((mk::AdamTensor*)host.data())[i] = {t.master, t.lowp, t.grad, (float*)t.m, (float*)t.v, t.n, t.decay != 0, 0};
      for (int64_t s = 0; s < t.n; s += mk::kAdamChunk) *c++ = mk::AdamChunk{i, 0, s};
    }
    if (hipMemcpyAsync(device, host.data(), need, hipMemcpyHostToDevice, (hipStream_t)stream) != hipSuccess ||
        hipStreamSynchronize((hipStream_t)stream) != hipSuccess) {
      (void)hipGetLastError();
      mimose_set_thread_error("mimose_op_adamw_table: copy to the device failed");
      return MIMOSE_ERR_HIP;
    }
  } catch (const std::bad_alloc&) {
    return refuse(op, "no host memory for the table");
  }
  out->device = device; out->tensors = count; out->chunks = (int32_t)chunks; out->state_bits = state_bits; out->reserved_ = 0;
  return MIMOSE_OK;
}

int mimose_op_adamw_step(const mimose_adamw_table* table, const mimose_adamw_cfg* cfg, int64_t step, void* stream) {
  const char* const op = "mimose_op_adamw_step";
  if (!table || !table->device || table->tensors < 1 || table->chunks < 0 || table->chunks >= (1 << 20) ||
      (table->state_bits != 8 && table->state_bits != 32) || !cfg)
    return refuse(op, "a table of mimose_op_adamw_table and cfg must be given");
  if (const char* why = mk::bad_adamw(cfg->lr, cfg->beta1, cfg->beta2, cfg->eps, cfg->weight_decay)) return refuse(op, why);
  if (step < 1) return refuse(op, "updates are numbered from 1");
  const mk::AdamHyper h = mk::adamw_hyper(cfg->lr, cfg->beta1, cfg->beta2, cfg->eps, cfg->weight_decay, step);
  const mk::AdamChunk* chunks = (const mk::AdamChunk*)((const char*)table->device + adamw_entries_bytes(table->tensors, table->state_bits));
  if (table->state_bits == 8) mk::adamw8_update((const mk::Adam8Tensor*)table->device, chunks, table->chunks, h, step, (hipStream_t)stream);
  else mk::adamw_update(mk::BF16, (const mk::AdamTensor*)table->device, chunks, table->chunks, h, (hipStream_t)stream);
  return done();
}

int mimose_op_embed_fwd(int32_t dtype, const int32_t* ids, const void* tok, const void* pos, const void* gamma,
                        const void* beta, void* sum_out, void* y, int32_t B, int32_t L, int32_t H, float eps,
                        int32_t has_ln, void* stream) {
  if (bad_dtype(dtype) || !ids || !tok || !pos || !y || B < 0 || L < 0 || H < 1 || H > mk::kMaxRowWidth) return MIMOSE_ERR_INVALID_ARG;
  if (has_ln && (!gamma || !beta)) return MIMOSE_ERR_INVALID_ARG;
  mk::embed_fwd(dtype, ids, tok, pos, gamma, beta, sum_out, y, mk::Rows(), B * L, B, L, H, eps, has_ln, (hipStream_t)stream);
  return done();
}

int mimose_op_embed_bwd(int32_t dtype, const void* d, const int32_t* ids, const int32_t* order, const int32_t* seg,
                        int32_t n_seg, float* dtok, float* dpos, int32_t B, int32_t L, int32_t H, int32_t max_seq,
                        void* stream) {
  if (bad_dtype(dtype) || !d || !ids || !order || !seg || !dtok || !dpos || B < 0 || L < 0 || H < 1 || n_seg < 0 || max_seq < L)
    return MIMOSE_ERR_INVALID_ARG;
  mk::embed_bwd(dtype, d, ids, order, seg, n_seg, dtok, dpos, mk::Rows(), B, L, H, max_seq, (hipStream_t)stream);
  return done();
}

}  // extern "C"
