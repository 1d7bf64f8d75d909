// C ABI of the kernel-level entry points: argument checks, then the launcher.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <functional>
#include <new>
#include <utility>
#include <vector>

#include "../../include/mimose.h"
#include "kernels.h"
#include "muon.h"

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
// Rows of an operand, or (rows = 1) a plain array: where they begin, elements from one to the next, elements of each, bytes of one.
struct RowSet { const void* at; int64_t ld, width, rows, es; bool plain = false; };
bool overlap(const RowSet& a, const RowSet& b) {
  if (!a.at || !b.at || a.rows < 1 || b.rows < 1) return false;
  const int64_t la = a.ld * a.es, lb = b.ld * b.es, wa = a.width * a.es, wb = b.width * b.es;
  const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
  if (x >= y + (uintptr_t)((b.rows - 1) * lb + wb) || y >= x + (uintptr_t)((a.rows - 1) * la + wa)) return false;
  if (a.rows == 1 || b.rows == 1 || la != lb) return true;
  const int64_t d = (((int64_t)(y - x)) % la + la) % la;   // columns of rows of one pitch: b's begin d bytes behind a's
  return d < wa || d + wb > la;
}
// what is wrong with the sizes of packed attention, or null
const char* bad_packed(int dtype, const int32_t* ends, int32_t n_seq, int32_t T, int32_t nh, int32_t nkv, int32_t d, float scale) {
  if (bad_dtype(dtype)) return "dtype must be 0 (fp32) or 1 (bf16)";
  if (T < 0 || n_seq < 0) return "T >= 0 and n_seq >= 0 required";
  if (nh < 1 || nkv < 1 || nh % nkv) return "n_heads must be a multiple of n_kv_heads";
  if (d != 32 && d != 64 && d != 128) return "head_dim must be 32, 64 or 128";
  if (!std::isfinite(scale) || !(scale > 0.f)) return "scale must be finite and above 0";
  if (n_seq > 0 && (!ends || (uintptr_t)ends % 4)) return "ends must be given, aligned to its elements";
  if (!mk::packed_attention_fits(T, n_seq, nh)) return "too many rows, sequences and heads for one launch";
  return nullptr;
}
// what is wrong with the operands, the first n_in of which are read and the others written, or null
const char* bad_rows(const RowSet* s, int n_in, int n) {
  for (int i = 0; i < n; ++i) {
    if (!s[i].at) return "every operand must be given";
    if (s[i].plain) {
      if ((uintptr_t)s[i].at % 4) return "lse is not aligned to its elements";
    } else {
      if (s[i].ld < s[i].width || s[i].ld >= mk::kPackedLd) return "a leading dimension must cover its heads and be below 2^21";
      if ((uintptr_t)s[i].at % 16 || s[i].ld * s[i].es % 16) return "operands and their rows must be 16-byte aligned";
    }
  }
  for (int i = n_in; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(s[i], s[j])) return "an operand that is written overlaps another";
  return nullptr;
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

int mimose_op_packed_attention_fwd(int32_t dtype, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                   void* out, int64_t ldo, float* lse, const int32_t* ends, int32_t n_seq, int32_t T, int32_t nh,
                                   int32_t nkv, int32_t d, int32_t causal, float scale, void* stream) {
  const char* const op = "mimose_op_packed_attention_fwd";
  if (const char* why = bad_packed(dtype, ends, n_seq, T, nh, nkv, d, scale)) return refuse(op, why);
  if (T == 0 || n_seq == 0) return MIMOSE_OK;
  const int64_t es = mk::elt_size(dtype), w = (int64_t)nh * d, wk = (int64_t)nkv * d, n = T, stats = (int64_t)nh * T;
  const RowSet s[] = {{q, ldq, w, n, es}, {k, ldk, wk, n, es}, {v, ldv, wk, n, es}, {ends, n_seq, n_seq, 1, 4, true}, {out, ldo, w, n, es},
                      {lse, stats, stats, 1, 4, true}};
  if (const char* why = bad_rows(s, 4, 6)) return refuse(op, why);
  mk::PackedAttention p;
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse; p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo;
  p.ends = ends; p.n_seq = n_seq; p.T = T; p.n_heads = nh; p.n_kv_heads = nkv; p.scale = scale;
  mk::packed_attention_fwd(dtype, p, d, causal, (hipStream_t)stream);
  return done();
}

uint64_t mimose_op_packed_attention_bwd_workspace_bytes(int32_t T, int32_t nh, int32_t nkv, int32_t d) {
  return T > 0 && nh > 0 && nkv > 0 && d > 0 ? mk::packed_attention_bwd_workspace_bytes(T, nh, nkv, d) : 0;
}

int mimose_op_packed_attention_bwd(int32_t dtype, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                   const void* out, int64_t ldo, const float* lse, const void* dout, int64_t lddo, void* dq, int64_t lddq,
                                   void* dk, int64_t lddk, void* dv, int64_t lddv, const int32_t* ends, int32_t n_seq, int32_t T,
                                   int32_t nh, int32_t nkv, int32_t d, int32_t causal, float scale, void* workspace,
                                   uint64_t workspace_bytes, void* stream) {
  const char* const op = "mimose_op_packed_attention_bwd";
  if (const char* why = bad_packed(dtype, ends, n_seq, T, nh, nkv, d, scale)) return refuse(op, why);
  if (T == 0 || n_seq == 0) return MIMOSE_OK;
  const int64_t es = mk::elt_size(dtype), w = (int64_t)nh * d, wk = (int64_t)nkv * d, n = T, stats = (int64_t)nh * T;
  const int64_t need = (int64_t)mk::packed_attention_bwd_workspace_bytes(T, nh, nkv, d);
  if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < (uint64_t)need)
    return refuse(op, "workspace must be 16-byte aligned and of mimose_op_packed_attention_bwd_workspace_bytes");
  const RowSet s[] = {{q, ldq, w, n, es}, {k, ldk, wk, n, es}, {v, ldv, wk, n, es}, {out, ldo, w, n, es}, {dout, lddo, w, n, es},
                      {ends, n_seq, n_seq, 1, 4, true}, {lse, stats, stats, 1, 4, true}, {dq, lddq, w, n, es}, {dk, lddk, wk, n, es}, {dv, lddv, wk, n, es},
                      {workspace, need, need, 1, 1, true}};
  if (const char* why = bad_rows(s, 7, 11)) return refuse(op, why);
  mk::PackedAttention p;
  p.q = q; p.k = k; p.v = v; p.out = const_cast<void*>(out); p.lse = const_cast<float*>(lse); p.dout = dout; p.dq = dq; p.dk = dk; p.dv = dv;
  p.ldq = ldq; p.ldk = ldk; p.ldv = ldv; p.ldo = ldo; p.lddo = lddo; p.lddq = lddq; p.lddk = lddk; p.lddv = lddv;
  p.ends = ends; p.n_seq = n_seq; p.T = T; p.n_heads = nh; p.n_kv_heads = nkv; p.scale = scale;
  mk::packed_attention_bwd(dtype, p, d, causal, workspace, (hipStream_t)stream);
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

// A list of matrices laid out: entries, units of work and scratch.  why: null, or what is wrong with the list.
struct MuonPlan {
  std::vector<mk::MuonMatrix> mats;
  std::vector<mk::MuonChunk> chunks;
  std::vector<mk::MuonTile> tiles[6];                  // cells; tri and full on tiles of 128; the three products' on tiles of 256
  std::vector<int32_t> starts;                         // for each part and product: where each block's tiles of 256 begin in the list
  mimose_muon_table table = {};
  const char* why = nullptr;
  uint64_t bytes() const {
    size_t n = mats.size() * sizeof(mk::MuonMatrix) + chunks.size() * sizeof(mk::MuonChunk);
    for (const auto& t : tiles) n += t.size() * sizeof(mk::MuonTile);
    return std::max<size_t>(16, n + starts.size() * sizeof(int32_t));
  }
};
static int64_t muon_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
static int64_t muon_chunk(int64_t n) { return std::max<int64_t>(8192, muon_up((n + 1023) / 1024, 4096)); }   // at most 1024 sums of a matrix
static int64_t muon_scratch(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1 || mk::muon_small(rows, cols)) return 0;
  const int64_t mp = muon_up(std::min(rows, cols), mk::kMuonTile), np = muon_up(std::max(rows, cols), mk::kMuonTile), n = rows * cols;
  return 4 * mp * np + 4 * mp * mp + muon_up((n + muon_chunk(n) - 1) / muon_chunk(n) * 8, 256);
}
static const char* bad_muon_list(const mimose_muon_matrix* t, int32_t count, int32_t parts) {
  if (!t || count < 1) return "at least one matrix required";
  if (parts < 1 || parts > 64) return "1 to 64 parts required";
  struct Range { uintptr_t from, to; bool written; };
  std::vector<Range> all;
  int64_t chunks = 0, tiles = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].rows < 0 || t[i].cols < 0 || t[i].rows > mk::kMuonSide || t[i].cols > mk::kMuonSide) return "a matrix has a side below 0 or above 2^20";
    const int64_t n = (int64_t)t[i].rows * t[i].cols;
    if (n == 0) continue;
    if (!t[i].master || !t[i].grad || !t[i].momentum) return "master, grad and momentum of a matrix must be given";
    if (((uintptr_t)t[i].master | (uintptr_t)t[i].grad | (uintptr_t)t[i].momentum | (uintptr_t)t[i].lowp) & 15)
      return "master, lowp, grad and momentum of a matrix must be 16-byte aligned";
    const uintptr_t f = (uintptr_t)n * 4;
    all.push_back({(uintptr_t)t[i].master, (uintptr_t)t[i].master + f, true});
    all.push_back({(uintptr_t)t[i].momentum, (uintptr_t)t[i].momentum + f, true});
    all.push_back({(uintptr_t)t[i].grad, (uintptr_t)t[i].grad + f, false});
    if (t[i].lowp) all.push_back({(uintptr_t)t[i].lowp, (uintptr_t)t[i].lowp + f / 2, true});
    chunks += (n + muon_chunk(n) - 1) / muon_chunk(n);
    tiles += muon_up(t[i].rows, mk::kMuonTile) / mk::kMuonTile * (muon_up(t[i].cols, mk::kMuonTile) / mk::kMuonTile);
    if (chunks >= (1 << 22) || tiles >= (1 << 22)) return "too many elements: 2^36 at most";   // a grid's threads are counted in 32 bits
  }
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t end = 0, end_written = 0;
  for (const Range& r : all) {
    if (r.from < (r.written ? end : end_written)) return "memory that is written belongs to two matrices, or to two of a matrix' tensors";
    end = std::max(end, r.to);
    if (r.written) end_written = std::max(end_written, r.to);
  }
  return nullptr;
}
// Deals tiles of 256 out to the blocks of one launch.  Runs of up to 16 neighbouring tiles of a matrix stay on one XCD, whose L2 they
// share; runs go to the XCD with least work, the largest first, and there its tiles to the block with least.  A tile's work is its
// k tiles and about four for its store.  Dealt out in equal numbers instead, in the list's order, the blocks of some XCDs get
// the long tiles: 24 layers of 1024 (4096 wide), the first product takes 390 us instead of 263.
static void muon_deal(std::vector<mk::MuonTile>& tiles, size_t from, const std::vector<mk::MuonMatrix>& mats, int stage, std::vector<int32_t>& starts) {
  constexpr int XCDS = 8, BLOCKS = mk::kMuonBlocks / XCDS;
  struct Run { size_t from, to; int64_t each; };   // tiles, and the work of one
  std::vector<Run> runs;
  for (size_t i = from; i < tiles.size();) {
    const mk::MuonMatrix& m = mats[tiles[i].matrix];
    size_t j = i;
    while (j < tiles.size() && j < i + 16 && tiles[j].matrix == tiles[i].matrix) ++j;
    runs.push_back({i, j, ((stage == 1 ? std::max(m.rows, m.cols) : std::min(m.rows, m.cols)) + 63) / 64 + 4});
    i = j;
  }
  std::stable_sort(runs.begin(), runs.end(), [](const Run& a, const Run& b) { return a.each * (int64_t)(a.to - a.from) > b.each * (int64_t)(b.to - b.from); });
  typedef std::pair<int64_t, int> Load;                  // work so far, XCD or block
  std::vector<Load> xcds;
  std::vector<Run> of[XCDS];
  for (int x = 0; x < XCDS; ++x) xcds.push_back({0, x});
  for (const Run& r : runs) {
    std::pop_heap(xcds.begin(), xcds.end(), std::greater<Load>());
    of[xcds.back().second].push_back(r);
    xcds.back().first += r.each * (int64_t)(r.to - r.from);
    std::push_heap(xcds.begin(), xcds.end(), std::greater<Load>());
  }
  std::vector<std::vector<mk::MuonTile>> mine(mk::kMuonBlocks);
  for (int x = 0; x < XCDS; ++x) {
    std::stable_sort(of[x].begin(), of[x].end(), [](const Run& a, const Run& b) { return a.each > b.each; });
    std::vector<Load> blocks;
    for (int b = 0; b < BLOCKS; ++b) blocks.push_back({0, b * XCDS + x});
    for (const Run& r : of[x])
      for (size_t i = r.from; i < r.to; ++i) {
        std::pop_heap(blocks.begin(), blocks.end(), std::greater<Load>());
        mine[blocks.back().second].push_back(tiles[i]);
        blocks.back().first += r.each;
        std::push_heap(blocks.begin(), blocks.end(), std::greater<Load>());
      }
  }
  size_t at = from;
  for (const auto& list : mine) {
    starts.push_back((int32_t)(at - from));
    for (const mk::MuonTile& t : list) tiles[at++] = t;
  }
  starts.push_back((int32_t)(at - from));
}
// An order of the lists of tiles of 128 in which a matrix' tiles stay on one XCD, in all lists: block b runs on XCD b % 8, and what one
// product leaves of a matrix in that XCD's L2 the next one finds there.  A matrix with more than an eighth of the work is cut
// into as many runs as it has eighths.  Runs go to the XCD with least work, the largest first; places that are left over name no matrix.
static void muon_spread(std::vector<mk::MuonTile>* lists, const size_t* from, int n_lists, const std::vector<int64_t>& work, int32_t first) {
  constexpr int XCDS = 8;
  int64_t all = 0;
  for (int64_t w : work) all += w;
  struct Run { int32_t matrix; int part, parts; int64_t work; };
  std::vector<Run> runs;
  for (size_t m = 0; m < work.size(); ++m) {
    if (!work[m]) continue;
    const int parts = (int)std::max<int64_t>(1, (work[m] * XCDS + all - 1) / all);
    for (int k = 0; k < parts; ++k) runs.push_back({(int32_t)m, k, parts, work[m] / parts});
  }
  std::stable_sort(runs.begin(), runs.end(), [](const Run& a, const Run& b) { return a.work > b.work; });
  std::vector<std::vector<int>> xcd_of(work.size());
  for (size_t m = 0; m < work.size(); ++m) xcd_of[m].assign(XCDS, 0);
  int64_t load[XCDS] = {};
  for (const Run& r : runs) {
    const int x = (int)(std::min_element(load, load + XCDS) - load);
    load[x] += r.work;
    xcd_of[r.matrix][r.part] = x;
  }
  std::vector<int> parts_of(work.size(), 1);
  for (const Run& r : runs) parts_of[r.matrix] = r.parts;
  for (int l = 0; l < n_lists; ++l) {
    std::vector<mk::MuonTile>& list = lists[l];
    std::vector<mk::MuonTile> queue[XCDS];
    for (size_t i = from[l]; i < list.size();) {
      size_t j = i;
      while (j < list.size() && list[j].matrix == list[i].matrix) ++j;
      const int32_t m = list[i].matrix - first;
      for (size_t k = i; k < j; ++k) queue[xcd_of[m][(k - i) * parts_of[m] / (j - i)]].push_back(list[k]);
      i = j;
    }
    size_t longest = 0;
    for (const auto& q : queue) longest = std::max(longest, q.size());
    list.resize(from[l]);
    for (size_t i = 0; i < longest; ++i)
      for (const auto& q : queue) list.push_back(i < q.size() ? q[i] : mk::MuonTile{-1, 0, 0});
  }
}
static MuonPlan muon_plan(const mimose_muon_matrix* t, int32_t count, int32_t parts) {
  MuonPlan p;
  if ((p.why = bad_muon_list(t, count, parts))) return p;
  // the smallest scratch that takes the list in so many parts, in its order
  auto parts_of = [&](int64_t room) {
    int k = 1;
    int64_t used = 0;
    for (int32_t i = 0; i < count; ++i) {
      const int64_t s = muon_scratch(t[i].rows, t[i].cols);
      if (used + s > room) { ++k; used = 0; }
      used += s;
    }
    return k;
  };
  int64_t low = 0, high = 0;
  for (int32_t i = 0; i < count; ++i) {
    const int64_t s = muon_scratch(t[i].rows, t[i].cols);
    low = std::max(low, s);
    high += s;
  }
  while (low < high) {
    const int64_t mid = low + (high - low) / 2;
    if (parts_of(mid) <= parts) high = mid; else low = mid + 1;
  }
  mimose_muon_table& out = p.table;
  out.workspace_bytes = std::max<uint64_t>(16, (uint64_t)high);
  int part = 0;
  int64_t used = 0;
  int32_t first = 0;                                       // of the part's matrices
  // tiles of `side` of a matrix, in groups of four rows of tiles: blocks that run at the same time share rows and columns
  auto cover = [](std::vector<mk::MuonTile>& to, int32_t matrix, int64_t mp, int64_t np, int side, bool tri) {
    const int mt = (int)((mp + side - 1) / side), nt = (int)((np + side - 1) / side);
    for (int i0 = 0; i0 < mt; i0 += 4)
      for (int j = tri ? i0 : 0; j < nt; ++j)
        for (int i = i0; i < std::min(i0 + 4, mt) && (!tri || i <= j); ++i) to.push_back({matrix, (uint16_t)i, (uint16_t)j});
  };
  auto close = [&]() {
    // Tiles of 256 for matrices that they pad to no more than 1.6 times the work, where there are enough to fill the device: the last
    // product of 24 layers of 1024 takes 0.45 ms an iteration on them and 0.68 on tiles of 128.
    const int32_t end = (int32_t)p.mats.size();
    auto fits = [](const mk::MuonMatrix& m) {
      return m.mp > mk::kMuonTile && 10 * muon_up(m.mp, 256) * muon_up(m.np, 256) <= 16 * (int64_t)m.mp * m.np;
    };
    int64_t tiles = 0;
    for (int32_t i = std::max(first, out.small); i < end; ++i)
      if (fits(p.mats[i])) tiles += muon_up(p.mats[i].mp, 256) / 256 * (muon_up(p.mats[i].np, 256) / 256);
    // The others' symmetric products on tiles of 64 where those of 128 are few, or have 18 % more of padding; their last product where they
    // are fewer still.  A step on tiles of 128, the symmetric products on those of 64, all three on those of 64: one matrix of 301 131,
    // 89 and 77 us; 4 of 512 (40 and 64 tiles of 128) 160, 112 and 95; 12 of 384 (72, 108) 141, 109 and 111; a layer of 768 (126, 432)
    // 417, 348 and 361; 5 layers of 301, 77 and 999 (180, 360, much padding) 202, 151 and 154; 12 of 640 (180, 300) 231, 238 and 262;
    // 2 of 2048 (272, 512) 581, 620 and 699.
    int64_t coarse[2] = {}, quarters[2] = {};                // of the symmetric products, of the last one
    auto count = [](int64_t* to, int64_t mt, int64_t nt) { to[0] += mt * (mt + 1) / 2; to[1] += mt * nt; };
    for (int32_t i = std::max(first, out.small); i < end; ++i) {
      const mk::MuonMatrix& m = p.mats[i];
      if (tiles >= 256 && fits(m)) continue;
      const int64_t shorter = std::min(m.rows, m.cols), longer = std::max(m.rows, m.cols);
      count(coarse, m.mp / mk::kMuonTile, m.np / mk::kMuonTile);
      count(quarters, muon_up(shorter, mk::kMuonFine) / mk::kMuonFine, muon_up(longer, mk::kMuonFine) / mk::kMuonFine);
    }
    const bool fine[2] = {coarse[0] < 160 || 118 * quarters[0] < 400 * coarse[0], coarse[1] < 100};
    for (int k = 0; k < 2; ++k)
      if (fine[k]) out.fine[k] |= (uint64_t)1 << part;
    std::vector<int64_t> work(end - first, 0);
    size_t from[3];
    for (int k = 0; k < 3; ++k) from[k] = p.tiles[k].size();
    for (int large = 0; large < 2; ++large) {                // the small tiles' cells come first
      for (int32_t i = std::max(first, out.small); i < end; ++i) {
        const mk::MuonMatrix& m = p.mats[i];
        if ((tiles >= 256 && fits(m)) != (large != 0)) continue;
        cover(p.tiles[0], i, m.mp, m.np, mk::kMuonTile, false);
        if (large) {
          cover(p.tiles[3], i, m.mp, m.mp, 256, true);
          cover(p.tiles[4], i, m.mp, m.mp, 256, true);
          cover(p.tiles[5], i, m.mp, m.np, 256, false);
        } else {
          const int32_t shorter = std::min(m.rows, m.cols), longer = std::max(m.rows, m.cols);
          cover(p.tiles[1], i, shorter, shorter, fine[0] ? mk::kMuonFine : mk::kMuonTile, true);
          cover(p.tiles[2], i, shorter, longer, fine[1] ? mk::kMuonFine : mk::kMuonTile, false);
          work[i - first] = (int64_t)m.mp * m.mp * m.np;
        }
      }
      if (!large) muon_spread(p.tiles, from, 3, work, first);
    }
    for (int s = 1; s <= 3; ++s) muon_deal(p.tiles[2 + s], part ? out.units[3 + s][part - 1] : 0, p.mats, s, p.starts);
    out.units[0][part] = (int32_t)p.chunks.size();
    for (int k = 0; k < 6; ++k) out.units[1 + k][part] = (int32_t)p.tiles[k].size();
    first = end;
  };
  for (int small = 1; small >= 0; --small)                 // the small ones come first, by themselves
    for (int32_t i = 0; i < count; ++i) {
      const int64_t rows = t[i].rows, cols = t[i].cols, n = rows * cols, s = muon_scratch(rows, cols);
      if (n == 0 || mk::muon_small(rows, cols) != (small != 0)) continue;
      if (used + s > high) { close(); ++part; used = 0; }
      mk::MuonMatrix m = {t[i].master, (uint16_t*)t[i].lowp, t[i].grad, t[i].momentum};
      m.rows = (int32_t)rows;
      m.cols = (int32_t)cols;
      if (small) {
        ++out.small;
      } else {
        m.chunk = muon_chunk(n);
        m.mp = (int32_t)muon_up(std::min(rows, cols), mk::kMuonTile);
        m.np = (int32_t)muon_up(std::max(rows, cols), mk::kMuonTile);
        const int64_t x = 2 * (int64_t)m.mp * m.np, a = 2 * (int64_t)m.mp * m.mp;
        m.x[0] = (uint64_t)used; m.x[1] = m.x[0] + x; m.a = m.x[1] + x; m.b = m.a + a; m.partial = m.b + a;
        for (int64_t c = 0; c < n; c += m.chunk) p.chunks.push_back({(int32_t)p.mats.size(), 0, c});
      }
      used += s;
      p.mats.push_back(m);
    }
  close();
  out.parts = part + 1;
  out.matrices = (int32_t)p.mats.size();
  return p;
}

uint64_t mimose_op_muon_table_bytes(const mimose_muon_matrix* matrices, int32_t count, int32_t parts) {
  const char* const op = "mimose_op_muon_table_bytes";
  try {
    const MuonPlan p = muon_plan(matrices, count, parts);
    if (p.why) { refuse(op, p.why); return 0; }
    return p.bytes();
  } catch (const std::bad_alloc&) {
    refuse(op, "no host memory for the table");
    return 0;
  }
}

int mimose_op_muon_table(const mimose_muon_matrix* matrices, int32_t count, int32_t parts, void* device, uint64_t bytes,
                         mimose_muon_table* out, void* stream) {
  const char* const op = "mimose_op_muon_table";
  try {
    MuonPlan p = muon_plan(matrices, count, parts);
    if (p.why) return refuse(op, p.why);
    if (!out || !device || ((uintptr_t)device & 15) || bytes < p.bytes())
      return refuse(op, "out and 16-byte aligned device memory of mimose_op_muon_table_bytes must be given");
    std::vector<char> host(p.bytes(), 0);
    char* to = host.data();
    auto put = [&](const void* from, size_t n) { if (n) memcpy(to, from, n); to += n; };
    put(p.mats.data(), p.mats.size() * sizeof(mk::MuonMatrix));
    put(p.chunks.data(), p.chunks.size() * sizeof(mk::MuonChunk));
    for (const auto& list : p.tiles) put(list.data(), list.size() * sizeof(mk::MuonTile));
    put(p.starts.data(), p.starts.size() * sizeof(int32_t));
    if (hipMemcpyAsync(device, host.data(), host.size(), hipMemcpyHostToDevice, (hipStream_t)stream) != hipSuccess ||
        hipStreamSynchronize((hipStream_t)stream) != hipSuccess) {
      (void)hipGetLastError();
      mimose_set_thread_error("mimose_op_muon_table: copy to the device failed");
      return MIMOSE_ERR_HIP;
    }
    *out = p.table;
    out->device = device;
  } catch (const std::bad_alloc&) {
    return refuse(op, "no host memory for the table");
  }
  return MIMOSE_OK;
}

int mimose_op_muon_step(const mimose_muon_table* table, const mimose_muon_cfg* cfg, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* const op = "mimose_op_muon_step";
  const char* const no_table = "a table of mimose_op_muon_table and cfg must be given";
  if (!table || !table->device || table->matrices < 0 || table->parts < 1 || table->parts > 64 || table->small < 0 ||
      table->small > table->matrices || !cfg)
    return refuse(op, no_table);
  for (const auto& ends : table->units)
    for (int i = 0; i < table->parts; ++i)
      if (ends[i] < (i ? ends[i - 1] : 0) || ends[i] >= (1 << 23)) return refuse(op, no_table);
  if (const char* why = mk::bad_muon(cfg->lr, cfg->momentum, cfg->weight_decay, cfg->rms, cfg->eps, cfg->iterations)) return refuse(op, why);
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < table->workspace_bytes)
    return refuse(op, "workspace must be 16-byte aligned and of table->workspace_bytes");
  const mk::MuonHyper h = {cfg->lr, cfg->momentum, cfg->weight_decay, cfg->rms, cfg->eps, cfg->nesterov != 0, cfg->iterations};
  const mk::MuonMatrix* mats = (const mk::MuonMatrix*)table->device;
  mk::muon_update_small(mats, table->small, h, (hipStream_t)stream);
  const int last = table->parts - 1;
  const mk::MuonChunk* chunks = (const mk::MuonChunk*)(mats + table->matrices);
  const mk::MuonTile* lists[6] = {(const mk::MuonTile*)(chunks + table->units[0][last])};
  for (int k = 1; k < 6; ++k) lists[k] = lists[k - 1] + table->units[k][last];
  const int32_t* starts = (const int32_t*)(lists[5] + table->units[6][last]);
  for (int i = 0; i <= last; ++i) {
    int from[7], count[7];
    for (int k = 0; k < 7; ++k) {
      from[k] = i ? table->units[k][i - 1] : 0;
      count[k] = table->units[k][i] - from[k];
    }
    mk::MuonUnits u;
    u.chunks = chunks + from[0]; u.n_chunks = count[0];
    u.cells = lists[0] + from[1]; u.n_cells = count[1];
    u.tri = lists[1] + from[2]; u.n_tri = count[2];
    u.full = lists[2] + from[3]; u.n_full = count[3];
    u.fine_tri = table->fine[0] >> i & 1;
    u.fine_full = table->fine[1] >> i & 1;
    for (int s = 0; s < 3; ++s, starts += mk::kMuonBlocks + 1) {
      u.large_tiles[s] = lists[3 + s] + from[4 + s];
      u.large[s] = count[4 + s] ? starts : nullptr;
    }
    mk::muon_update(mats, u, workspace, h, (hipStream_t)stream);
  }
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
