// C-ABI wrappers of the single operations, and the dispatch between the MFMA attention
// kernels for bf16 and the fp32 ones.
#include <math.h>
#include <mutex>
#include "kernels.h"

mosaic_status launch_attention_fwd_f32(hipStream_t s, int quota, int dtype, int B, int N, int H, int Hkv, int d,
                                          int causal, const void* qkv, void* O, float* lse);
mosaic_status launch_attention_bwd_f32(hipStream_t s, int quota, int dtype, int B, int N, int H, int Hkv, int d,
                                          int causal, const void* qkv, const void* O, const float* lse,
                                          const void* dO, void* dqkv, float* delta);

bool attention_mfma_supported(int dtype, int d);
mosaic_status launch_attention_fwd_mfma(hipStream_t s, int quota, int B, int N, int H, int Hkv, int d, int causal,
                                        const void* qkv, void* O, float* lse);
mosaic_status launch_attention_bwd_mfma(hipStream_t s, int quota, int B, int N, int H, int Hkv, int d, int causal,
                                        const void* qkv, const void* O, const float* lse, const void* dO, void* dqkv,
                                        float* delta);

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The MFMA kernels address one sample's packed q|k|v rows with 32-bit byte offsets (buffer
// descriptors); a tile may start up to 63 rows past the end.  Longer slices take the
// fp32 kernels, which index with 64 bits.
static bool attn_slice_fits32(int N, int H, int Hkv, int d) {
  return ((int64_t)N + 64) * ((int64_t)H + 2 * Hkv) * d * 2 < ((int64_t)1 << 32);
}

static mosaic_status check_attn(int B, int N, int H, int Hkv, int d) {
  if (B <= 0 || N <= 0 || H <= 0 || d <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "attention sizes must be positive");
  if (Hkv <= 0 || H % Hkv) MOSAIC_FAIL(MOSAIC_EINVAL, "key/value heads (%d) must divide the query heads (%d)", Hkv, H);
  if (d > 128) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "head size %d > 128", d);
  return MOSAIC_OK;
}

mosaic_status launch_attention_fwd(hipStream_t s, int quota, int dtype, int B, int N, int H, int Hkv, int d, int causal,
                                   const void* qkv, void* O, float* lse) {
  MOSAIC_TRY(check_attn(B, N, H, Hkv, d));
  if (attention_mfma_supported(dtype, d) && attn_slice_fits32(N, H, Hkv, d) && aligned16(qkv) && aligned16(O))
    return launch_attention_fwd_mfma(s, quota, B, N, H, Hkv, d, causal, qkv, O, lse);
  return launch_attention_fwd_f32(s, quota, dtype, B, N, H, Hkv, d, causal, qkv, O, lse);
}

mosaic_status launch_attention_bwd(hipStream_t s, int quota, int dtype, int B, int N, int H, int Hkv, int d, int causal,
                                   const void* qkv, const void* O, const float* lse, const void* dO, void* dqkv,
                                   float* delta) {
  MOSAIC_TRY(check_attn(B, N, H, Hkv, d));
  if (attention_mfma_supported(dtype, d) && attn_slice_fits32(N, H, Hkv, d) && aligned16(qkv) && aligned16(O) && aligned16(dO) && aligned16(dqkv)) {
    return launch_attention_bwd_mfma(s, quota, B, N, H, Hkv, d, causal, qkv, O, lse, dO, dqkv, delta);
  }
  return launch_attention_bwd_f32(s, quota, dtype, B, N, H, Hkv, d, causal, qkv, O, lse, dO, dqkv, delta);
}

static mosaic_status check_common(int32_t quota, int32_t dtype) {
  if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) MOSAIC_FAIL(MOSAIC_EINVAL, "bad dtype %d", dtype);
  DeviceInfo di;
  MOSAIC_TRY(mosaic_device_info(&di));
  if (quota <= 0 || quota > di.cu_count) MOSAIC_FAIL(MOSAIC_EQUOTA, "quota %d outside [1, %d]", quota, di.cu_count);
  return MOSAIC_OK;
}

#define NONNULL(p) if (!(p)) MOSAIC_FAIL(MOSAIC_EINVAL, "null pointer: " #p)

extern "C" {

mosaic_status mosaic_op_linear_fwd(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t k, int64_t n,
                                   const void* X, const void* W, const void* bias, const void* R, void* Y) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(X); NONNULL(W); NONNULL(Y);
  if (T < 0 || k <= 0 || n <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad linear sizes");
  return launch_gemm((hipStream_t)stream, quota, dtype, true, false, T, n, k, X, k, W, n, Y, n, bias, R);
}

mosaic_status mosaic_op_linear_dgrad(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t k, int64_t n,
                                     const void* dY, const void* W, const void* R, void* dX) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(dY); NONNULL(W); NONNULL(dX);
  if (T < 0 || k <= 0 || n <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad linear sizes");
  return launch_gemm((hipStream_t)stream, quota, dtype, true, true, T, k, n, dY, n, W, n, dX, k, nullptr, R);
}

size_t mosaic_op_colsum_scratch_bytes(int64_t n) { return colsum_scratch_bytes(n); }

size_t mosaic_op_linear_wgrad_scratch_bytes(int64_t T, int64_t k, int64_t n) {
  return align_up(gemm_splitk_scratch_bytes(k, n, T), 256) + colsum_scratch_bytes(n);
}

mosaic_status mosaic_op_linear_wgrad(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t k, int64_t n,
                                     const void* X, const void* dY, void* dW, void* db, void* scratch) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(X); NONNULL(dY); NONNULL(dW);
  if (T < 0 || k <= 0 || n <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad linear sizes");
  NONNULL(scratch);
  if ((uintptr_t)scratch % 16) MOSAIC_FAIL(MOSAIC_EINVAL, "scratch must be 16-byte aligned");
  if (T == 0) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "weight gradient over zero tokens");
  MOSAIC_TRY(launch_gemm((hipStream_t)stream, quota, dtype, false, false, k, n, T, X, k, dY, n, dW, n, nullptr, nullptr, scratch));
  if (db) MOSAIC_TRY(launch_colsum((hipStream_t)stream, quota, dtype, T, n, dY, db,
                                   (char*)scratch + align_up(gemm_splitk_scratch_bytes(k, n, T), 256)));
  return MOSAIC_OK;
}

mosaic_status mosaic_op_attention_fwd(void* stream, int32_t quota, int32_t dtype, int32_t B, int32_t N, int32_t H,
                                      int32_t d, int32_t causal, const void* qkv, void* O, float* lse) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(qkv); NONNULL(O); NONNULL(lse);
  return launch_attention_fwd((hipStream_t)stream, quota, dtype, B, N, H, H, d, causal, qkv, O, lse);
}

mosaic_status mosaic_op_attention_bwd(void* stream, int32_t quota, int32_t dtype, int32_t B, int32_t N, int32_t H,
                                      int32_t d, int32_t causal, const void* qkv, const void* O, const float* lse,
                                      const void* dO, void* dqkv, float* delta) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(qkv); NONNULL(O); NONNULL(lse); NONNULL(dO); NONNULL(dqkv); NONNULL(delta);
  return launch_attention_bwd((hipStream_t)stream, quota, dtype, B, N, H, H, d, causal, qkv, O, lse, dO, dqkv, delta);
}

mosaic_status mosaic_op_attention_gqa_fwd(void* stream, int32_t quota, int32_t dtype, int32_t B, int32_t N, int32_t H,
                                          int32_t Hkv, int32_t d, int32_t causal, const void* qkv, void* O, float* lse) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(qkv); NONNULL(O); NONNULL(lse);
  return launch_attention_fwd((hipStream_t)stream, quota, dtype, B, N, H, Hkv, d, causal, qkv, O, lse);
}

mosaic_status mosaic_op_attention_gqa_bwd(void* stream, int32_t quota, int32_t dtype, int32_t B, int32_t N, int32_t H,
                                          int32_t Hkv, int32_t d, int32_t causal, const void* qkv, const void* O,
                                          const float* lse, const void* dO, void* dqkv, float* delta) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(qkv); NONNULL(O); NONNULL(lse); NONNULL(dO); NONNULL(dqkv); NONNULL(delta);
  return launch_attention_bwd((hipStream_t)stream, quota, dtype, B, N, H, Hkv, d, causal, qkv, O, lse, dO, dqkv, delta);
}

mosaic_status mosaic_op_norm_fwd(void* stream, int32_t quota, int32_t dtype, int32_t norm, int64_t T, int64_t h,
                                 float eps, const void* x, const void* gamma, const void* beta, void* y, float* stats) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(x); NONNULL(gamma); NONNULL(y); NONNULL(stats);
  if (norm == MOSAIC_LAYERNORM) NONNULL(beta);
  if (T < 0 || h <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad norm sizes");
  return launch_norm_fwd((hipStream_t)stream, quota, dtype, norm, T, h, eps, x, gamma, beta, y, stats);
}

size_t mosaic_op_norm_bwd_scratch_bytes(int64_t h) { return norm_bwd_scratch_bytes(h); }

mosaic_status mosaic_op_norm_bwd(void* stream, int32_t quota, int32_t dtype, int32_t norm, int64_t T, int64_t h,
                                 const void* x, const void* gamma, const float* stats, const void* dy, const void* R,
                                 void* dx, void* dgamma, void* dbeta, void* scratch) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(x); NONNULL(gamma); NONNULL(stats); NONNULL(dy); NONNULL(dx); NONNULL(dgamma); NONNULL(scratch);
  if (norm == MOSAIC_LAYERNORM) NONNULL(dbeta);
  if (T < 0 || h <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad norm sizes");
  return launch_norm_bwd((hipStream_t)stream, quota, dtype, norm, T, h, x, gamma, stats, dy, R, dx, dgamma, dbeta, scratch);
}

// Scratch of the entry point for callers that cannot allocate: the partial column sums of the
// norm backward for rows of up to kStaticNormMaxH elements.  Each GPU holds its own copy of the
// array at its own address; host code never uses the array's name as an address, only the
// pointer that hipGetSymbolAddress returned with that GPU current.
constexpr int64_t kStaticNormMaxH = 5120;
constexpr size_t kStaticScratchBytes = (size_t)512 * 2 * kStaticNormMaxH * sizeof(float);   // 20 MiB
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

static mosaic_status static_scratch_ptr(void** out) {
  constexpr int kMaxDevices = 64;
  static std::mutex mu;
  static void* ptr[kMaxDevices] = {};
  int dev = 0;
  MOSAIC_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "device index %d beyond the %d this table holds", dev, kMaxDevices);
  std::lock_guard<std::mutex> lk(mu);
  if (!ptr[dev]) {
    void* p = nullptr;
    MOSAIC_HIP(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
    if (!p) MOSAIC_FAIL(MOSAIC_EHIP, "hipGetSymbolAddress returned a null address");
    ptr[dev] = p;
  }
  *out = ptr[dev];
  return MOSAIC_OK;
}

size_t mosaic_op_norm_bwd_static_max_h(void) { return (size_t)kStaticNormMaxH; }

mosaic_status mosaic_op_norm_bwd_static(void* stream, int32_t quota, int32_t dtype, int32_t norm, int64_t T, int64_t h,
                                        const void* x, const void* gamma, const float* stats, const void* dy,
                                        const void* R, void* dx, void* dgamma, void* dbeta) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(x); NONNULL(gamma); NONNULL(stats); NONNULL(dy); NONNULL(dx); NONNULL(dgamma);
  if (norm == MOSAIC_LAYERNORM) NONNULL(dbeta);
  if (T < 0 || h <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad norm sizes");
  if (h > kStaticNormMaxH || norm_bwd_scratch_bytes(h, false) > kStaticScratchBytes)
    MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "row width %lld exceeds the %lld elements the built-in scratch covers; "
                "use mosaic_op_norm_bwd with a caller-provided scratch", (long long)h, (long long)kStaticNormMaxH);
  void* sc = nullptr;
  MOSAIC_TRY(static_scratch_ptr(&sc));
  return launch_norm_bwd((hipStream_t)stream, quota, dtype, norm, T, h, x, gamma, stats, dy, R, dx, dgamma, dbeta, sc);
}

mosaic_status mosaic_op_gelu_fwd(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* z, void* a) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(z); NONNULL(a);
  return launch_gelu_fwd((hipStream_t)stream, quota, dtype, n, z, a);
}

mosaic_status mosaic_op_gelu_bwd(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* z, const void* da, void* dz) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(z); NONNULL(da); NONNULL(dz);
  return launch_gelu_bwd((hipStream_t)stream, quota, dtype, n, z, da, dz);
}

mosaic_status mosaic_op_swiglu_fwd(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t f, const void* gu, void* a) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(gu); NONNULL(a);
  return launch_swiglu_fwd((hipStream_t)stream, quota, dtype, T, f, gu, a);
}

mosaic_status mosaic_op_linear_act_fwd(void* stream, int32_t quota, int32_t dtype, int32_t act, int64_t T, int64_t k, int64_t n,
                                       const void* X, const void* W, const void* bias, void* Z, void* A) {
  MOSAIC_TRY(check_common(quota, dtype));
  if (T < 0 || k <= 0 || n < 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad linear shape T=%lld k=%lld n=%lld", (long long)T, (long long)k, (long long)n);
  NONNULL(X); NONNULL(W); NONNULL(Z); NONNULL(A);
  return launch_linear_act_fwd((hipStream_t)stream, quota, dtype, act, T, k, n, X, W, bias, Z, A);
}

mosaic_status mosaic_op_swiglu_bwd(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t f, const void* gu,
                                   const void* da, void* dgu) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(gu); NONNULL(da); NONNULL(dgu);
  return launch_swiglu_bwd((hipStream_t)stream, quota, dtype, T, f, gu, da, dgu);
}

mosaic_status mosaic_op_gelu_tanh_fwd(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* z, void* a) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(z); NONNULL(a);
  return launch_gelu_tanh_fwd((hipStream_t)stream, quota, dtype, n, z, a);
}

mosaic_status mosaic_op_gelu_tanh_bwd(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* z, const void* da, void* dz) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(z); NONNULL(da); NONNULL(dz);
  return launch_gelu_tanh_bwd((hipStream_t)stream, quota, dtype, n, z, da, dz);
}

size_t mosaic_op_rope_table_bytes(int32_t N, int32_t d) { return (N > 0 && d > 0) ? rope_table_bytes(N, d) : 0; }

mosaic_status mosaic_op_rope_table(void* stream, int32_t quota, int32_t N, int32_t d, float base, void* table) {
  MOSAIC_TRY(check_common(quota, MOSAIC_F32));
  NONNULL(table);
  return launch_rope_table((hipStream_t)stream, quota, N, d, base, table);
}

mosaic_status mosaic_op_rope(void* stream, int32_t quota, int32_t dtype, int32_t B, int32_t N, int32_t H, int32_t d,
                             int32_t direction, void* qkv, const void* table) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(qkv); NONNULL(table);
  return launch_rope((hipStream_t)stream, quota, dtype, B, N, H, H, d, direction, qkv, table);
}

mosaic_status mosaic_op_adamw(void* stream, int32_t quota, int32_t dtype, int64_t n, void* params, const void* grads,
                              float* m, float* v, float* master, float lr, float beta1, float beta2, float eps,
                              float weight_decay, int64_t step) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(params); NONNULL(grads); NONNULL(m); NONNULL(v);
  if (n < 0) MOSAIC_FAIL(MOSAIC_EINVAL, "negative element count");
  return launch_adamw((hipStream_t)stream, quota, dtype, n, params, grads, m, v, master, lr, beta1, beta2, eps, weight_decay, step);
}

size_t mosaic_op_rope_axes_table_bytes(int32_t d) { return d > 0 ? rope_axes_table_bytes(d) : 0; }

mosaic_status mosaic_op_rope_axes_table(void* stream, int32_t quota, int32_t d, int32_t n_axes, const int32_t* sections, int32_t order, float base,
                                        void* table) {
  NONNULL(sections); NONNULL(table);
  if (d <= 0 || d % 2) MOSAIC_FAIL(MOSAIC_EINVAL, "head size %d is not positive and even", d);
  if (d > 256) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "head size %d > 256", d);
  if (n_axes < 1 || n_axes > MOSAIC_MAX_AXES) MOSAIC_FAIL(MOSAIC_EINVAL, "%d position axes; 1 to %d", n_axes, MOSAIC_MAX_AXES);
  if (order < MOSAIC_AXES_SPLIT || order > MOSAIC_AXES_DEALT) MOSAIC_FAIL(MOSAIC_EINVAL, "bad order of axes %d", order);
  if (!(base > 0.f) || base > 3.4028234e38f) MOSAIC_FAIL(MOSAIC_EINVAL, "rotary base must be positive and finite");
  int64_t sum = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (sections[a] < 0) MOSAIC_FAIL(MOSAIC_EINVAL, "axis %d has %d pairs", a, sections[a]);
    sum += sections[a];
  }
  if (sum > d / 2) MOSAIC_FAIL(MOSAIC_EINVAL, "the axes have %lld pairs, a head %d", (long long)sum, d / 2);
  if ((uintptr_t)table % 16) MOSAIC_FAIL(MOSAIC_EINVAL, "the table must be 16-byte aligned");
  MOSAIC_TRY(check_common(quota, MOSAIC_F32));
  return launch_rope_axes_table((hipStream_t)stream, quota, d, n_axes, sections, order, base, table);
}

// what the calls on packed rows share; `rotates`: there is a table
static mosaic_status check_heads(int32_t dtype, int64_t T, int32_t H, int32_t Hkv, int32_t d, int32_t pairing, int32_t n_axes, const int32_t* pos,
                                 const void* table) {
  if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) MOSAIC_FAIL(MOSAIC_EINVAL, "bad dtype %d", dtype);
  if (T < 0 || H <= 0 || Hkv <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad sizes T=%lld H=%d Hkv=%d", (long long)T, H, Hkv);
  if (H % Hkv) MOSAIC_FAIL(MOSAIC_EINVAL, "key/value heads (%d) must divide the query heads (%d)", Hkv, H);
  if (d <= 0 || d % 2) MOSAIC_FAIL(MOSAIC_EINVAL, "head size %d is not positive and even", d);
  if (d > 256) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "head size %d > 256", d);
  if (((int64_t)H + 2 * (int64_t)Hkv) * d > INT32_MAX) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "rows of more than 2^31 - 1 elements");
  if (T > ((int64_t)1 << 58) / (((int64_t)H + 2 * Hkv) * d)) MOSAIC_FAIL(MOSAIC_EINVAL, "%lld tokens", (long long)T);
  if (pairing != MOSAIC_PAIR_ADJACENT && pairing != MOSAIC_PAIR_HALVES) MOSAIC_FAIL(MOSAIC_EINVAL, "bad pairing %d", pairing);
  if (table) {
    NONNULL(pos);
    if (n_axes < 1 || n_axes > MOSAIC_MAX_AXES) MOSAIC_FAIL(MOSAIC_EINVAL, "%d position axes; 1 to %d", n_axes, MOSAIC_MAX_AXES);
    if ((uintptr_t)table % 16) MOSAIC_FAIL(MOSAIC_EINVAL, "the table must be 16-byte aligned");
  }
  return MOSAIC_OK;
}
static mosaic_status check_qk_norm(int32_t norm, float eps) {
  if (norm != MOSAIC_LAYERNORM && norm != MOSAIC_RMSNORM) MOSAIC_FAIL(MOSAIC_EINVAL, "bad norm kind %d", norm);
  if (!(eps > 0.f)) MOSAIC_FAIL(MOSAIC_EINVAL, "eps must be positive");
  return MOSAIC_OK;
}
#define APART(p, pn, q, qn) if (overlap(p, pn, q, qn)) MOSAIC_FAIL(MOSAIC_EINVAL, #p " overlaps " #q)

mosaic_status mosaic_op_rope_axes(void* stream, int32_t quota, int32_t dtype, int64_t T, int32_t H, int32_t Hkv, int32_t d, int32_t pairing,
                                  int32_t direction, int32_t n_axes, const int32_t* pos, const void* table, const void* x, void* y) {
  NONNULL(table); NONNULL(x); NONNULL(y);
  MOSAIC_TRY(check_heads(dtype, T, H, Hkv, d, pairing, n_axes, pos, table));
  if (direction != 1 && direction != -1) MOSAIC_FAIL(MOSAIC_EINVAL, "direction must be +1 or -1");
  const int64_t bytes = T * (H + 2 * Hkv) * d * (int64_t)dtype_size(dtype);
  if (x != y) APART(x, bytes, y, bytes);
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_qk_norm_rope_fwd((hipStream_t)stream, quota, dtype, MOSAIC_NORM_NONE, T, H, Hkv, d, 0.f, pairing, direction, n_axes, pos, table, x,
                                 nullptr, nullptr, nullptr, nullptr, y);
}

mosaic_status mosaic_op_qk_norm_rope_fwd(void* stream, int32_t quota, int32_t dtype, int32_t norm, int64_t T, int32_t H, int32_t Hkv, int32_t d,
                                         float eps, int32_t pairing, int32_t n_axes, const int32_t* pos, const void* table, const void* x,
                                         const void* gamma_q, const void* beta_q, const void* gamma_k, const void* beta_k, void* y) {
  NONNULL(x); NONNULL(gamma_q); NONNULL(gamma_k); NONNULL(y);
  MOSAIC_TRY(check_qk_norm(norm, eps));
  if (norm == MOSAIC_LAYERNORM) { NONNULL(beta_q); NONNULL(beta_k); }
  MOSAIC_TRY(check_heads(dtype, T, H, Hkv, d, pairing, n_axes, pos, table));
  const int64_t bytes = T * (H + 2 * Hkv) * d * (int64_t)dtype_size(dtype);
  if (x != y) APART(x, bytes, y, bytes);
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_qk_norm_rope_fwd((hipStream_t)stream, quota, dtype, norm, T, H, Hkv, d, eps, pairing, +1, n_axes, pos, table, x, gamma_q, beta_q,
                                 gamma_k, beta_k, y);
}

size_t mosaic_op_qk_norm_rope_bwd_scratch_bytes(int32_t d) { return d > 0 ? qk_norm_rope_bwd_scratch_bytes(d) : 0; }

mosaic_status mosaic_op_qk_norm_rope_bwd(void* stream, int32_t quota, int32_t dtype, int32_t norm, int64_t T, int32_t H, int32_t Hkv, int32_t d,
                                         float eps, int32_t pairing, int32_t n_axes, const int32_t* pos, const void* table, const void* x,
                                         const void* gamma_q, const void* gamma_k, const void* dy, void* dx, void* dgamma_q, void* dbeta_q,
                                         void* dgamma_k, void* dbeta_k, void* scratch) {
  NONNULL(x); NONNULL(gamma_q); NONNULL(gamma_k); NONNULL(dy); NONNULL(dx); NONNULL(dgamma_q); NONNULL(dgamma_k); NONNULL(scratch);
  MOSAIC_TRY(check_qk_norm(norm, eps));
  if (norm == MOSAIC_LAYERNORM) { NONNULL(dbeta_q); NONNULL(dbeta_k); }
  MOSAIC_TRY(check_heads(dtype, T, H, Hkv, d, pairing, n_axes, pos, table));
  const int64_t bytes = T * (H + 2 * Hkv) * d * (int64_t)dtype_size(dtype);
  APART(x, bytes, dx, bytes);
  if (dy != dx) APART(dy, bytes, dx, bytes);
  if ((uintptr_t)scratch % 16) MOSAIC_FAIL(MOSAIC_EINVAL, "scratch must be 16-byte aligned");
  // the gains' and shifts' gradients are sums that a second launch takes from scratch
  const int64_t gain = d * (int64_t)dtype_size(dtype), needed = (int64_t)qk_norm_rope_bwd_scratch_bytes(d);
  const bool layer = norm == MOSAIC_LAYERNORM;
  const void* const sums[] = {dgamma_q, dgamma_k, layer ? dbeta_q : nullptr, layer ? dbeta_k : nullptr};
  const char* const names[] = {"dgamma_q", "dgamma_k", "dbeta_q", "dbeta_k"};
  for (int i = 0; i < 4; ++i) {
    if (overlap(sums[i], gain, dx, bytes) || overlap(sums[i], gain, scratch, needed)) MOSAIC_FAIL(MOSAIC_EINVAL, "%s overlaps dx or scratch", names[i]);
    for (int j = 0; j < i; ++j)
      if (overlap(sums[i], gain, sums[j], gain)) MOSAIC_FAIL(MOSAIC_EINVAL, "%s overlaps %s", names[i], names[j]);
  }
  APART(scratch, needed, x, bytes); APART(scratch, needed, dy, bytes); APART(scratch, needed, dx, bytes);
  APART(scratch, needed, gamma_q, gain); APART(scratch, needed, gamma_k, gain);
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_qk_norm_rope_bwd((hipStream_t)stream, quota, dtype, norm, T, H, Hkv, d, eps, pairing, n_axes, pos, table, x, gamma_q, gamma_k, dy, dx,
                                 dgamma_q, dbeta_q, dgamma_k, dbeta_k, scratch);
}

size_t mosaic_op_pack8_scale_bytes(int64_t n) { return n > 0 ? pack8_scale_bytes(n) : 0; }

// sizes that the packed calls take: their products fit 64 bits with room for the element size
static mosaic_status check_packed(int32_t dtype, int64_t rows, int64_t cols) {
  if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) MOSAIC_FAIL(MOSAIC_EINVAL, "bad dtype %d", dtype);
  if (rows < 0 || cols < 0 || (cols > 0 && rows > ((int64_t)1 << 58) / cols)) MOSAIC_FAIL(MOSAIC_EINVAL, "bad size %lld x %lld", (long long)rows, (long long)cols);
  return MOSAIC_OK;
}

mosaic_status mosaic_op_pack8(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* x, void* q, void* scale) {
  NONNULL(x); NONNULL(q); NONNULL(scale);
  MOSAIC_TRY(check_packed(dtype, n, 1));
  const int64_t bytes = n * (int64_t)dtype_size(dtype), scales = (int64_t)mosaic_op_pack8_scale_bytes(n);
  APART(x, bytes, q, n); APART(x, bytes, scale, scales); APART(q, n, scale, scales);
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_pack8((hipStream_t)stream, quota, dtype, n, x, q, scale);
}

mosaic_status mosaic_op_unpack8(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* q, const void* scale, void* x) {
  NONNULL(q); NONNULL(scale); NONNULL(x);
  MOSAIC_TRY(check_packed(dtype, n, 1));
  const int64_t bytes = n * (int64_t)dtype_size(dtype);
  APART(x, bytes, q, n); APART(x, bytes, scale, (int64_t)mosaic_op_pack8_scale_bytes(n));
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_unpack8((hipStream_t)stream, quota, dtype, n, q, scale, x);
}

static mosaic_status check_act(int32_t dtype, int32_t act, int64_t T, int64_t f) {
  if (act != MOSAIC_GELU && act != MOSAIC_SWIGLU && act != MOSAIC_GELU_TANH) MOSAIC_FAIL(MOSAIC_EINVAL, "bad activation %d", act);
  return check_packed(dtype, T, f);
}

mosaic_status mosaic_op_act_fwd_pack8(void* stream, int32_t quota, int32_t dtype, int32_t act, int64_t T, int64_t f, const void* z, void* a, void* zq,
                                      void* zscale) {
  NONNULL(z); NONNULL(a); NONNULL(zq); NONNULL(zscale);
  MOSAIC_TRY(check_act(dtype, act, T, f));
  const int64_t es = (int64_t)dtype_size(dtype), m = T * f, n = act == MOSAIC_SWIGLU ? 2 * m : m, scales = (int64_t)mosaic_op_pack8_scale_bytes(n);
  APART(z, n * es, a, m * es); APART(z, n * es, zq, n); APART(z, n * es, zscale, scales);
  APART(a, m * es, zq, n); APART(a, m * es, zscale, scales); APART(zq, n, zscale, scales);
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_act_fwd_pack8((hipStream_t)stream, quota, dtype, act, T, f, z, a, zq, zscale);
}

mosaic_status mosaic_op_act_bwd_pack8(void* stream, int32_t quota, int32_t dtype, int32_t act, int64_t T, int64_t f, const void* zq, const void* zscale,
                                      const void* da, void* dz, void* a) {
  NONNULL(zq); NONNULL(zscale); NONNULL(da); NONNULL(dz);
  MOSAIC_TRY(check_act(dtype, act, T, f));
  const int64_t es = (int64_t)dtype_size(dtype), m = T * f, n = act == MOSAIC_SWIGLU ? 2 * m : m, scales = (int64_t)mosaic_op_pack8_scale_bytes(n);
  if (da != dz || act == MOSAIC_SWIGLU) APART(da, m * es, dz, n * es);
  APART(dz, n * es, zq, n); APART(dz, n * es, zscale, scales);
  if (a) { APART(a, m * es, da, m * es); APART(a, m * es, dz, n * es); APART(a, m * es, zq, n); APART(a, m * es, zscale, scales); }
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_act_bwd_pack8((hipStream_t)stream, quota, dtype, act, T, f, zq, zscale, da, dz, a);
}

size_t mosaic_op_linear_wgrad_pack8_scratch_bytes(int32_t dtype, int64_t T, int64_t k, int64_t n) {
  return T > 0 && k > 0 && n > 0 ? linear_wgrad_pack8_scratch_bytes(dtype, T, k, n) : 0;
}

mosaic_status mosaic_op_linear_wgrad_pack8(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t k, int64_t n, const void* Xq, const void* Xscale,
                                           const void* dY, void* dW, void* db, void* scratch) {
  NONNULL(Xq); NONNULL(Xscale); NONNULL(dY); NONNULL(dW); NONNULL(scratch);
  if (T < 0 || k <= 0 || n <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad linear sizes");
  if (T == 0) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "weight gradient over zero tokens");
  MOSAIC_TRY(check_packed(dtype, T, k)); MOSAIC_TRY(check_packed(dtype, T, n)); MOSAIC_TRY(check_packed(dtype, k, n));
  if (T > INT32_MAX || k > INT32_MAX || n > INT32_MAX) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "sizes past 2^31 - 1: %lld x %lld x %lld", (long long)T, (long long)k, (long long)n);
  const int vn = dtype == MOSAIC_BF16 ? 8 : 4;
  if (db && n % vn) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "column sums of rows of %lld elements, not a multiple of %d", (long long)n, vn);
  if ((uintptr_t)scratch % 16) MOSAIC_FAIL(MOSAIC_EINVAL, "scratch must be 16-byte aligned");
  const int64_t es = (int64_t)dtype_size(dtype), scales = (int64_t)mosaic_op_pack8_scale_bytes(T * k), needed = (int64_t)mosaic_op_linear_wgrad_pack8_scratch_bytes(dtype, T, k, n);
  APART(dW, k * n * es, Xq, T * k); APART(dW, k * n * es, Xscale, scales); APART(dW, k * n * es, dY, T * n * es);
  APART(scratch, needed, Xq, T * k); APART(scratch, needed, Xscale, scales); APART(scratch, needed, dY, T * n * es); APART(scratch, needed, dW, k * n * es);
  if (db) {
    APART(db, n * es, Xq, T * k); APART(db, n * es, Xscale, scales); APART(db, n * es, dY, T * n * es); APART(db, n * es, dW, k * n * es);
    APART(db, n * es, scratch, needed);
  }
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_linear_wgrad_pack8((hipStream_t)stream, quota, dtype, T, k, n, Xq, Xscale, dY, dW, db, scratch);
}

// the calls with a loss over a vocabulary: `dX`, `dtable` and `scratch` as given (null: none)
static mosaic_status check_ce(int32_t dtype, int64_t T, int64_t h, int64_t V, float smoothing, float denom, const void* targets, const void* X, const void* table,
                              const void* loss, const void* losses, bool grad, const void* dX, const void* dtable, const void* scratch) {
  NONNULL(table); NONNULL(loss); NONNULL(scratch);
  if (T != 0) { NONNULL(targets); NONNULL(X); }          // an empty tensor has no address
  if (grad && T != 0 && !dX && !dtable) MOSAIC_FAIL(MOSAIC_EINVAL, "null pointers: neither dX nor dtable is asked for");
  if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) MOSAIC_FAIL(MOSAIC_EINVAL, "bad dtype %d", dtype);
  if (T < 0 || h <= 0 || V <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad sizes T=%lld h=%lld V=%lld", (long long)T, (long long)h, (long long)V);
  if (!(smoothing >= 0.f) || !(smoothing < 1.f)) MOSAIC_FAIL(MOSAIC_EINVAL, "label smoothing must lie in [0, 1)");
  if (!(denom >= 0.f) || denom > 3.4028234e38f) MOSAIC_FAIL(MOSAIC_EINVAL, "the denominator must be positive and finite, or 0 for the mean");
  const int64_t es = (int64_t)dtype_size(dtype);
  if (T > INT32_MAX / 2 || h > (1 << 20) || V > (1 << 22) || V > ((int64_t)1 << 32) / es / h - 1)
    MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "T=%lld h=%lld V=%lld: tables of 4 GiB or more, or sizes past 2^30 tokens, 2^20 values a row or 2^22 rows", (long long)T, (long long)h, (long long)V);
  if (dtype == MOSAIC_BF16 && h % 8) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "rows of %lld bf16 elements, not a multiple of 8", (long long)h);
  if (dtype == MOSAIC_BF16 && (((uintptr_t)X | (uintptr_t)table | (uintptr_t)dX | (uintptr_t)dtable) & 15)) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "bf16 tensors off 16-byte boundaries");
  if ((uintptr_t)scratch % 256) MOSAIC_FAIL(MOSAIC_EINVAL, "scratch must be 256-byte aligned");
  struct Span { const char* name; const void* p; int64_t n; };
  const int64_t rows = T * h * es, words = V * h * es;
  const Span in[] = {{"targets", targets, 4 * T}, {"X", X, rows}, {"table", table, words}};
  const Span out[] = {{"loss", loss, 4}, {"losses", losses, 4 * T}, {"dX", dX, rows}, {"dtable", dtable, words}, {"scratch", scratch, (int64_t)linear_ce_scratch_bytes(dtype, T, h, V, grad)}};
  for (int o = 0; o < 5; ++o) {
    for (const Span& i : in) if (overlap(out[o].p, out[o].n, i.p, i.n)) MOSAIC_FAIL(MOSAIC_EINVAL, "%s overlaps %s", out[o].name, i.name);
    for (int q = 0; q < o; ++q) if (overlap(out[o].p, out[o].n, out[q].p, out[q].n)) MOSAIC_FAIL(MOSAIC_EINVAL, "%s overlaps %s", out[o].name, out[q].name);
  }
  return MOSAIC_OK;
}

static size_t ce_scratch(int32_t dtype, int64_t T, int64_t h, int64_t V, bool grad) {
  if ((dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) || T < 0 || h <= 0 || V <= 0 || T > INT32_MAX / 2 || h > (1 << 20) || V > (1 << 22)) return 0;
  return linear_ce_scratch_bytes(dtype, T, h, V, grad);
}
size_t mosaic_op_linear_ce_fwd_scratch_bytes(int32_t dtype, int64_t T, int64_t h, int64_t V) { return ce_scratch(dtype, T, h, V, false); }
size_t mosaic_op_linear_ce_grad_scratch_bytes(int32_t dtype, int64_t T, int64_t h, int64_t V) { return ce_scratch(dtype, T, h, V, true); }

mosaic_status mosaic_op_linear_ce_fwd(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t h, int64_t V, float smoothing, float denom,
                                      const int32_t* targets, const void* X, const void* table, float* loss, float* losses, void* scratch) {
  MOSAIC_TRY(check_ce(dtype, T, h, V, smoothing, denom, targets, X, table, loss, losses, false, nullptr, nullptr, scratch));
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_linear_ce((hipStream_t)stream, quota, dtype, T, h, V, smoothing, denom, targets, X, table, loss, losses, false, nullptr, nullptr, scratch);
}

mosaic_status mosaic_op_linear_ce_grad(void* stream, int32_t quota, int32_t dtype, int64_t T, int64_t h, int64_t V, float smoothing, float denom,
                                       const int32_t* targets, const void* X, const void* table, float* loss, float* losses, void* dX, void* dtable,
                                       void* scratch) {
  MOSAIC_TRY(check_ce(dtype, T, h, V, smoothing, denom, targets, X, table, loss, losses, true, dX, dtable, scratch));
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_linear_ce((hipStream_t)stream, quota, dtype, T, h, V, smoothing, denom, targets, X, table, loss, losses, true, dX, dtable, scratch);
}

static mosaic_status grouped(void* stream, int32_t quota, int32_t dtype, GroupedForm form, int64_t T, int32_t groups, int64_t k, int64_t n,
                             const int32_t* offsets, const void* A, const void* B, void* C) {
  if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) MOSAIC_FAIL(MOSAIC_EINVAL, "bad dtype %d", dtype);
  if (T < 0 || groups < 0 || k <= 0 || n <= 0) MOSAIC_FAIL(MOSAIC_EINVAL, "bad sizes T=%lld groups=%d k=%lld n=%lld", (long long)T, groups, (long long)k, (long long)n);
  if (groups > 1024) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "%d groups; up to 1024", groups);
  if (T > INT32_MAX / 2 || k > (1 << 28) || n > (1 << 28) || k * n > (int64_t)1 << 40) MOSAIC_FAIL(MOSAIC_EUNSUPPORTED, "sizes T=%lld k=%lld n=%lld", (long long)T, (long long)k, (long long)n);
  const int64_t es = (int64_t)dtype_size(dtype), x = T * k * es, y = T * n * es, w = groups * k * n * es;
  const int64_t a = form == GROUPED_DGRAD ? y : x, b = form == GROUPED_WGRAD ? y : w, c = form == GROUPED_FWD ? y : form == GROUPED_DGRAD ? x : w;
  if (overlap(C, c, A, a) || overlap(C, c, B, b) || overlap(C, c, offsets, 4 * ((int64_t)groups + 1))) MOSAIC_FAIL(MOSAIC_EINVAL, "the output overlaps an input");
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_grouped((hipStream_t)stream, quota, dtype, form, T, groups, k, n, offsets, A, B, C);
}

mosaic_status mosaic_op_grouped_linear_fwd(void* stream, int32_t quota, int32_t dtype, int64_t T, int32_t groups, int64_t k, int64_t n, const int32_t* offsets,
                                           const void* X, const void* W, void* Y) {
  NONNULL(offsets);
  if (T != 0) { NONNULL(X); NONNULL(Y); }
  if (groups != 0) NONNULL(W);
  return grouped(stream, quota, dtype, GROUPED_FWD, T, groups, k, n, offsets, X, W, Y);
}

mosaic_status mosaic_op_grouped_linear_dgrad(void* stream, int32_t quota, int32_t dtype, int64_t T, int32_t groups, int64_t k, int64_t n, const int32_t* offsets,
                                             const void* dY, const void* W, void* dX) {
  NONNULL(offsets);
  if (T != 0) { NONNULL(dY); NONNULL(dX); }
  if (groups != 0) NONNULL(W);
  return grouped(stream, quota, dtype, GROUPED_DGRAD, T, groups, k, n, offsets, dY, W, dX);
}

mosaic_status mosaic_op_grouped_linear_wgrad(void* stream, int32_t quota, int32_t dtype, int64_t T, int32_t groups, int64_t k, int64_t n, const int32_t* offsets,
                                             const void* X, const void* dY, void* dW) {
  NONNULL(offsets);
  if (T != 0) { NONNULL(X); NONNULL(dY); }
  if (groups != 0) NONNULL(dW);
  return grouped(stream, quota, dtype, GROUPED_WGRAD, T, groups, k, n, offsets, X, dY, dW);
}

mosaic_status mosaic_op_dropout(void* stream, int32_t quota, int32_t dtype, int64_t n, float p, uint64_t site, const uint64_t* rng, const void* x,
                                const void* R, void* y) {
  NONNULL(rng);
  if (n != 0) { NONNULL(x); NONNULL(y); }
  if (!(p >= 0.f) || !(p <= 1.f)) MOSAIC_FAIL(MOSAIC_EINVAL, "the probability of dropping must lie in [0, 1]");
  if ((uintptr_t)rng % 8) MOSAIC_FAIL(MOSAIC_EINVAL, "rng must be 8-byte aligned");
  MOSAIC_TRY(check_packed(dtype, n, 1));
  const int64_t bytes = n * (int64_t)dtype_size(dtype);
  if (x != y) APART(x, bytes, y, bytes);
  if (R != y) APART(R, bytes, y, bytes);
  APART(rng, 16, y, bytes);
  MOSAIC_TRY(check_common(quota, dtype));
  return launch_dropout((hipStream_t)stream, quota, dtype, n, (uint32_t)lrintf(p * 65536.f), site, rng, x, R, y);
}

size_t mosaic_op_mse_scratch_bytes(void) { return mse_scratch_bytes(); }

mosaic_status mosaic_op_mse(void* stream, int32_t quota, int32_t dtype, int64_t n, const void* y, const void* target,
                            void* dy, float* loss, void* scratch) {
  MOSAIC_TRY(check_common(quota, dtype));
  NONNULL(y); NONNULL(target); NONNULL(dy); NONNULL(loss); NONNULL(scratch);
  return launch_mse((hipStream_t)stream, quota, dtype, n, y, target, dy, loss, scratch);
}

}  // extern "C"
