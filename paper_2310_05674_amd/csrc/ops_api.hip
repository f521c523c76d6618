// Op-level C entry points (include/sama_ops.h): thin argument checks around the kernel launchers.
#include <algorithm>
#include <cmath>
#include <math.h>
#include <mutex>
#include <string>
#include "../../include/sama_ops.h"
#include "kernels.h"
#include "sequence_ops.h"
#include "token_ops.h"

using namespace sama;

// Scratch of sama_op_adapt_norm_static: the per-block partial sums of ||v||^2 that sama_op_adapt_norm takes from its
// caller.  One copy per GPU the library runs on, alive until the process ends; host code never uses the array's name
// as an address, only the per-device pointers resolved below.
static __device__ __align__(256) double scratch[EW_MAX_BLOCKS];

namespace {
constexpr int MAX_DEVICES = 64;
std::mutex g_scratch_mutex;
double* g_scratch_ptr[MAX_DEVICES] = {};   // device address of `scratch` on each GPU, resolved at the first call there
thread_local std::string g_ops_error;

// The current device's copy of `scratch`; null (and g_ops_error set) if it cannot be resolved.
double* static_scratch() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) { g_ops_error = "no current HIP device (or device index above 63)"; return nullptr; }
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (g_scratch_ptr[dev] == nullptr) {
    double* p = nullptr;
    const hipError_t e = hipGetSymbolAddress((void**)&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || p == nullptr) { g_ops_error = std::string("hipGetSymbolAddress(scratch): ") + hipGetErrorString(e); return nullptr; }
    g_scratch_ptr[dev] = p;
  }
  return g_scratch_ptr[dev];
}

sama_status refuse(const char* op, const char* why) { g_ops_error = std::string(op) + ": " + why; return SAMA_EINVAL; }
sama_status launched(const char* op) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return SAMA_OK;
  g_ops_error = std::string(op) + ": " + hipGetErrorString(e);
  return SAMA_EHIP;
}
bool is_dtype(int32_t t) { return t == SAMA_DTYPE_FP32 || t == SAMA_DTYPE_BF16; }
int value_bytes(int32_t dtype) { return dtype == SAMA_DTYPE_BF16 ? 2 : 4; }
// aligned to a value, and rows x ld values within the address space
bool is_rows(const void* p, int32_t dtype, int64_t rows, int64_t ld) {
  return (uintptr_t)p % value_bytes(dtype) == 0 && ld <= ((int64_t)1 << 40) && (rows == 0 || ld <= ((int64_t)1 << 46) / rows);
}
constexpr int64_t MOST_TOKENS = (int64_t)1 << 30;
// what the embedding calls have in common
const char* check_embedding(const int32_t* ids, int64_t n, int32_t V, int32_t d, float scale, int32_t pad_id) {
  if (n < 0 || n > MOST_TOKENS) return "n must be 0 to 2^30";
  if (V < 1 || d < 1) return "V and d must be positive";
  if (n > 0 && ids == nullptr) return "null ids";
  if ((uintptr_t)ids % 4 != 0) return "ids must be aligned to 4 bytes";
  if (!std::isfinite(scale)) return "scale must be finite";
  if (pad_id < -1) return "pad_id must be -1 (none) or an id";
  return nullptr;
}
// what the feed-forward calls have in common
const char* check_glu(int64_t T, int32_t d, int32_t F, int32_t dtype) {
  if (!is_dtype(dtype)) return "dtype must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16";
  if (T < 0 || T > ((int64_t)1 << 22)) return "T must be 0 to 2^22";
  // offsets in a tile's slab are 32 bits: 255 rows of 2 F values, F + 127 rows of d values
  if (d < 1 || F < 1 || d > (1 << 20) || F > (1 << 20)) return "d and F must be 1 to 2^20";
  if ((int64_t)d * F >= ((int64_t)1 << (dtype == SAMA_DTYPE_BF16 ? 29 : 28))) return "d F must be below 2^29 in bf16, 2^28 in fp32";
  if (dtype == SAMA_DTYPE_BF16 && (d % 8 != 0 || F % 8 != 0)) return "d and F must be multiples of 8 in bf16";
  return nullptr;
}
bool is_glu_rows(const void* p, int64_t ld, int32_t d, int32_t dtype) {
  return p != nullptr && ld >= d && ld <= ((int64_t)1 << 21) && (dtype == SAMA_DTYPE_BF16 ? ((uintptr_t)p & 15) == 0 && ld % 8 == 0 : ((uintptr_t)p & 3) == 0);
}
bool is_glu_dense(const void* p, int32_t dtype) { return p != nullptr && ((uintptr_t)p & (dtype == SAMA_DTYPE_BF16 ? 15 : 3)) == 0; }
}  // namespace

extern "C" {

// Diagnostic switches (include/sama_ops.h): block shape of the bf16 GEMM, 0 = heuristic.
void sama_dev_gemm_shape(int32_t shape) { gemm_bf16_force_shape(shape); }
sama_status sama_dev_gemm_rows(uint64_t choice) { return gemm_bf16_force_rows(choice) ? SAMA_OK : SAMA_EINVAL; }
sama_status sama_dev_gemm_counts(int64_t* counts, int32_t n) {
  if (counts == nullptr || n != GEMM_COUNTS) return SAMA_EINVAL;
  gemm_bf16_take_counts(counts);
  return SAMA_OK;
}
// 0 keeps every launch of the encoder's backward pass on the context's stream, 2 uses the second one, 1 decides by size / 0 makes the optimizer slices wait for its end.
void sama_dev_side_stream(int32_t mode) { encoder_side_stream(mode); }
void sama_dev_side_sink(int32_t on) { encoder_side_sink(on != 0); }

sama_status sama_op_gemm_bf16(const void* A, int64_t lda, int32_t a_trans, const void* B, const void* B2, int64_t ldb,
                              int32_t b_trans, int32_t M, int32_t N, int32_t K, const float* bias, float* C32, void* C16,
                              int64_t ldc, void* hip_stream) {
  if (!A || !B || (!C32 && !C16)) return SAMA_EINVAL;
  GemmBf16Args g{};
  g.A = (const bf16_t*)A; g.lda = lda; g.a_trans = a_trans ? 1 : 0;
  g.B = (const bf16_t*)B; g.B2 = (const bf16_t*)B2; g.ldb = ldb; g.b_trans = b_trans ? 1 : 0;
  g.M = M; g.N = N; g.K = K; g.ldc = ldc; g.bias = bias; g.C32 = C32; g.C16 = (bf16_t*)C16;
  if (check_gemm_bf16(g) != nullptr) return SAMA_EINVAL;
  (void)hipGetLastError();
  launch_gemm_bf16((hipStream_t)hip_stream, g);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_gemm_bf16_batch(int32_t count, const void* const* A, const void* const* B, const void* const* B2,
                                    float* const* C32, const int32_t* M, const int32_t* N, const int32_t* K, int32_t a_trans,
                                    int32_t b_trans, void* hip_stream) {
  if (count < 1 || count > GEMM_MAX_BATCH || !A || !B || !C32 || !M || !N || !K) return SAMA_EINVAL;
  GemmBf16Args g[GEMM_MAX_BATCH];
  for (int k = 0; k < count; ++k) {
    if (!A[k] || !B[k] || !C32[k] || (B2 && !B2[k])) return SAMA_EINVAL;
    g[k] = GemmBf16Args{};
    g[k].A = (const bf16_t*)A[k]; g[k].a_trans = a_trans ? 1 : 0; g[k].lda = a_trans ? M[k] : K[k];
    g[k].B = (const bf16_t*)B[k]; g[k].B2 = B2 ? (const bf16_t*)B2[k] : nullptr; g[k].b_trans = b_trans ? 1 : 0;
    g[k].ldb = b_trans ? K[k] : N[k];
    g[k].M = M[k]; g[k].N = N[k]; g[k].K = K[k]; g[k].ldc = N[k]; g[k].C32 = C32[k];
  }
  if (check_gemm_bf16_batch(g, count) != nullptr) return SAMA_EINVAL;
  (void)hipGetLastError();
  launch_gemm_bf16_batch((hipStream_t)hip_stream, g, count);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

size_t sama_op_gelu_table_bytes(void) { return gelu_table_bytes(); }
sama_status sama_op_gemm_bf16_gelu(const void* A, const void* B, const void* B2, int32_t b_trans, int32_t M, int32_t N, int32_t K,
                                   const void* aux16, void* pre16, float* C32, void* table, void* hip_stream) {
  if (!A || !B || !B2 || !C32 || !table || ((uintptr_t)table & 15) != 0) return SAMA_EINVAL;
  GemmBf16Args g{};
  g.A = (const bf16_t*)A; g.lda = K;
  g.B = (const bf16_t*)B; g.B2 = (const bf16_t*)B2; g.b_trans = b_trans ? 1 : 0; g.ldb = b_trans ? K : N;
  g.M = M; g.N = N; g.K = K; g.ldc = N; g.C32 = C32; g.gelu_tab = (const float*)table;
  g.act = aux16 ? GEMM_ACT_GELU_BWD : GEMM_ACT_GELU_FWD;
  g.aux16 = (const bf16_t*)aux16; g.C16_pre = aux16 ? nullptr : (bf16_t*)pre16;
  if (check_gemm_bf16(g) != nullptr) return SAMA_EINVAL;
  (void)hipGetLastError();
  launch_gelu_tables((hipStream_t)hip_stream, (float*)table);
  launch_gemm_bf16((hipStream_t)hip_stream, g);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_gemm_bf16_residual(int32_t count, const void* A, const void* B, const void* B2, int32_t M, int32_t N, int32_t K,
                                       const float* params, const float* v, const float* eps, const float* x, const float* stats,
                                       float* C32, const int32_t* rows, void* hip_stream) {
  if (count < 1 || count > 2 || !A || !B || !B2 || !params || !x || !C32 || (v != nullptr) != (eps != nullptr)) return SAMA_EINVAL;
  GemmBf16Args g[2];
  for (int k = 0; k < count; ++k) {
    const int64_t row0 = (int64_t)k * M;
    g[k] = GemmBf16Args{};
    g[k].A = (const bf16_t*)A + row0 * K; g[k].lda = K;
    g[k].B = (const bf16_t*)B; g[k].B2 = (const bf16_t*)B2 + (int64_t)k * N * K; g[k].b_trans = 1; g[k].ldb = K;
    g[k].M = M; g[k].N = N; g[k].K = K; g[k].ldc = N; g[k].rows = rows;
    g[k].bias = params; g[k].bias_v = v; g[k].beps = eps; g[k].bsign = v ? (k == 0 ? 1.f : -1.f) : 0.f;
    g[k].res32 = x + row0 * N; g[k].C32 = C32 + row0 * N;
    if (stats) { g[k].ln_mean = stats + row0; g[k].ln_rstd = count * M; g[k].ln_g = N; g[k].ln_b = 2 * N; }
  }
  if (check_gemm_bf16_batch(g, count) != nullptr) return SAMA_EINVAL;
  (void)hipGetLastError();
  launch_gemm_bf16_batch((hipStream_t)hip_stream, g, count);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_adam(float* g, float* m, float* v, float* theta, void* theta16, int64_t n, int64_t n16, int64_t t,
                         float lr, float beta1, float beta2, float eps, float weight_decay, void* hip_stream) {
  if (!g || !m || !v || !theta || n < 0 || n16 < 0 || n16 > n || t < 1) return SAMA_EINVAL;
  if (((uintptr_t)g | (uintptr_t)m | (uintptr_t)v | (uintptr_t)theta) & 15 || ((uintptr_t)theta16 & 7)) return SAMA_EINVAL;
  AdamArgs a{};
  a.beta1 = beta1; a.one_m_beta1 = (float)(1.0 - (double)beta1); a.beta2 = beta2; a.one_m_beta2 = (float)(1.0 - (double)beta2);
  a.lr_c1 = (float)((double)lr / (1.0 - pow((double)beta1, (double)t)));
  a.c2 = (float)(1.0 / sqrt(1.0 - pow((double)beta2, (double)t)));
  a.eps = eps; a.weight_decay = weight_decay;
  (void)hipGetLastError();
  launch_adam((hipStream_t)hip_stream, g, m, v, theta, (bf16_t*)theta16, n, theta16 ? n16 : 0, a);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_adapt_norm(const float* g, const float* m, const float* v, const float* gmeta, float* vdir, double* partial,
                               int64_t n, int64_t t, float lr, float beta1, float beta2, float eps, float alpha, float* scalars,
                               int64_t* status, void* hip_stream) {
  if (!g || !m || !v || !gmeta || !vdir || !partial || !scalars || !status || n < 1 || t < 1) return SAMA_EINVAL;
  if (((uintptr_t)g | (uintptr_t)m | (uintptr_t)v | (uintptr_t)gmeta | (uintptr_t)vdir) & 15) return SAMA_EINVAL;
  const double c1 = 1.0 / (1.0 - pow((double)beta1, (double)t)), c2 = 1.0 / sqrt(1.0 - pow((double)beta2, (double)t));
  AdaptArgs ad{};
  ad.mode = 0; ad.one_m_beta1 = (float)(1.0 - (double)beta1); ad.one_m_beta2 = (float)(1.0 - (double)beta2);
  ad.lr_c1_c2 = (float)((double)lr * c1 * c2); ad.c2 = (float)c2; ad.eps = eps;
  (void)hipGetLastError();
  launch_adapt_norm((hipStream_t)hip_stream, g, m, v, gmeta, vdir, partial, n, ad, alpha, scalars, status);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_adapt_norm_static(const float* g, const float* m, const float* v, const float* gmeta, float* vdir, int64_t n,
                                      int64_t t, float lr, float beta1, float beta2, float eps, float alpha, float* scalars,
                                      int64_t* status, void* hip_stream) {
  g_ops_error.clear();
  if (n > SAMA_OP_STATIC_MAX_N) {
    g_ops_error = "sama_op_adapt_norm_static: n exceeds SAMA_OP_STATIC_MAX_N (2^29 elements); use sama_op_adapt_norm with a caller-owned scratch";
    return SAMA_EINVAL;
  }
  double* partial = static_scratch();
  if (partial == nullptr) return SAMA_EHIP;
  const sama_status s = sama_op_adapt_norm(g, m, v, gmeta, vdir, partial, n, t, lr, beta1, beta2, eps, alpha, scalars, status, hip_stream);
  if (s == SAMA_EINVAL) g_ops_error = "sama_op_adapt_norm_static: null or misaligned pointer, n < 1 or t < 1";
  return s;
}

const char* sama_op_last_error(void) { return g_ops_error.c_str(); }

sama_status sama_op_perturb_lo(const float* theta, const float* vdir, const float* eps_ptr, void* lo_p, void* lo_m, int64_t n16,
                               void* hip_stream) {
  if (!theta || !vdir || !eps_ptr || !lo_p || !lo_m || n16 < 0) return SAMA_EINVAL;
  if ((((uintptr_t)theta | (uintptr_t)vdir) & 15) || (((uintptr_t)lo_p | (uintptr_t)lo_m) & 7)) return SAMA_EINVAL;
  (void)hipGetLastError();
  launch_perturb_lo((hipStream_t)hip_stream, theta, vdir, eps_ptr, (bf16_t*)lo_p, (bf16_t*)lo_m, n16);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_nudge(float* theta, const float* vdir, const float* eps_ptr, void* theta16, int64_t n, int64_t n16,
                          void* hip_stream) {
  if (!theta || !vdir || !eps_ptr || n < 0 || n16 < 0 || n16 > n) return SAMA_EINVAL;
  if ((((uintptr_t)theta | (uintptr_t)vdir) & 15) || ((uintptr_t)theta16 & 7)) return SAMA_EINVAL;
  (void)hipGetLastError();
  launch_nudge((hipStream_t)hip_stream, theta, vdir, eps_ptr, nullptr, (bf16_t*)theta16, nullptr, n, theta16 ? n16 : 0);
  return hipGetLastError() == hipSuccess ? SAMA_OK : SAMA_EHIP;
}

sama_status sama_op_embedding(const void* table, int32_t table_dtype, int64_t ld_table, const int32_t* ids, int64_t n, int32_t V, int32_t d,
                              float scale, int32_t pad_id, void* out, int32_t out_dtype, int64_t ld_out, void* hip_stream) {
  static const char* const op = "sama_op_embedding";
  g_ops_error.clear();
  if (!is_dtype(table_dtype) || !is_dtype(out_dtype)) return refuse(op, "types must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16");
  if (const char* e = check_embedding(ids, n, V, d, scale, pad_id)) return refuse(op, e);
  if (n == 0) return SAMA_OK;
  if (!table || !out) return refuse(op, "null table or output");
  if (ld_table < d || ld_out < d) return refuse(op, "a stride is smaller than a row");
  if (!is_rows(table, table_dtype, V, ld_table) || !is_rows(out, out_dtype, n, ld_out)) return refuse(op, "a pointer is not aligned to its values, or a stride is too large");
  EmbeddingArgs a{};
  a.table = table; a.ldt = ld_table; a.table_bf16 = table_dtype == SAMA_DTYPE_BF16; a.ids = ids; a.n = n; a.V = V; a.d = d; a.scale = scale; a.pad = pad_id;
  a.out = out; a.ldo = ld_out; a.out_bf16 = out_dtype == SAMA_DTYPE_BF16;
  (void)hipGetLastError();
  launch_embedding((hipStream_t)hip_stream, a);
  return launched(op);
}

size_t sama_op_embedding_grad_bytes(int64_t n, int32_t V, int32_t d) {
  return n < 0 || n > MOST_TOKENS || V < 1 || d < 1 ? 0 : embedding_grad_bytes(n, V, d);
}

sama_status sama_op_embedding_grad(const void* dy, int32_t dy_dtype, int64_t ld_dy, const int32_t* ids, int64_t n, int32_t V, int32_t d, float scale,
                                   int32_t pad_id, int32_t accumulate, void* grad, int32_t grad_dtype, int64_t ld_grad, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  static const char* const op = "sama_op_embedding_grad";
  g_ops_error.clear();
  if (!is_dtype(dy_dtype) || !is_dtype(grad_dtype)) return refuse(op, "types must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16");
  if (const char* e = check_embedding(ids, n, V, d, scale, pad_id)) return refuse(op, e);
  if (accumulate != 0 && accumulate != 1) return refuse(op, "accumulate must be 0 or 1");
  if (!grad || (n > 0 && !dy)) return refuse(op, "null gradient or dy");
  if ((n > 0 && ld_dy < d) || ld_grad < d) return refuse(op, "a stride is smaller than a row");
  if ((n > 0 && !is_rows(dy, dy_dtype, n, ld_dy)) || !is_rows(grad, grad_dtype, V, ld_grad)) return refuse(op, "a pointer is not aligned to its values, or a stride is too large");
  if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < embedding_grad_bytes(n, V, d)) {
    (void)refuse(op, "workspace missing, not aligned to 256 bytes or smaller than sama_op_embedding_grad_bytes()");
    return SAMA_EWORKSPACE;
  }
  if (accumulate && n == 0) return SAMA_OK;
  EmbeddingGradArgs a{};
  a.dy = dy; a.ldy = ld_dy; a.dy_bf16 = dy_dtype == SAMA_DTYPE_BF16; a.ids = ids; a.n = n; a.V = V; a.d = d; a.scale = scale; a.pad = pad_id;
  a.accumulate = accumulate != 0; a.grad = grad; a.ldg = ld_grad; a.grad_bf16 = grad_dtype == SAMA_DTYPE_BF16;
  if (!embedding_grad_fits(a)) return refuse(op, "V above 2^30, or more tokens of this width than a launch has room for");
  (void)hipGetLastError();
  launch_embedding_grad((hipStream_t)hip_stream, a, workspace);
  return launched(op);
}

size_t sama_op_grad_clip_bytes(void) { return grad_clip_bytes(); }

sama_status sama_op_grad_clip(int64_t count, void* const* grads, const int64_t* counts, const int32_t* dtypes, float max_norm, float* out,
                              float* norm_out, int64_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
  static const char* const op = "sama_op_grad_clip";
  g_ops_error.clear();
  if (count < 0 || (count > 0 && (!grads || !counts || !dtypes))) return refuse(op, "null list, or a negative count");
  if (!(max_norm > 0.f)) return refuse(op, "max_norm must be positive");
  if (!norm_out || (uintptr_t)norm_out % 4 != 0 || (uintptr_t)out % 4 != 0 || (uintptr_t)status % 8 != 0) return refuse(op, "null norm_out, or a misaligned output");
  if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < grad_clip_bytes()) {
    (void)refuse(op, "workspace missing, not aligned to 256 bytes or smaller than sama_op_grad_clip_bytes()");
    return SAMA_EWORKSPACE;
  }
  int64_t total = 0;
  for (int64_t k = 0; k < count; ++k) {
    if (!is_dtype(dtypes[k])) return refuse(op, "types must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16");
    if (counts[k] < 0 || counts[k] > ((int64_t)1 << 40) || (counts[k] > 0 && (!grads[k] || (uintptr_t)grads[k] % value_bytes(dtypes[k]) != 0)))
      return refuse(op, "a gradient is null, misaligned or of a negative size");
    total += counts[k];
    if (total > ((int64_t)1 << 40)) return refuse(op, "more than 2^40 values");
  }
  (void)hipGetLastError();
  launch_grad_clip((hipStream_t)hip_stream, GradList{grads, counts, dtypes}, count, max_norm, norm_out, out, status, workspace);
  return launched(op);
}

size_t sama_op_glu_ffn_bytes(int64_t T, int32_t d, int32_t F, int32_t dtype) {
  if (check_glu(T, d, F, dtype) != nullptr) return 0;
  return std::max<size_t>(256, dtype == SAMA_DTYPE_BF16 ? glu_ffn_bytes(T, d, F) : glu_ffn_f32_bytes(T, d, F));
}
size_t sama_op_glu_ffn_saved_bytes(int64_t T, int32_t F, int32_t dtype) {
  if (check_glu(T, 8, F, dtype) != nullptr) return 0;
  return std::max<size_t>(256, dtype == SAMA_DTYPE_BF16 ? glu_ffn_saved_bytes(T, F) : glu_ffn_f32_saved_bytes(T, F));
}
size_t sama_op_glu_ffn_grad_bytes(int64_t T, int32_t d, int32_t F, int32_t dtype) {
  if (check_glu(T, d, F, dtype) != nullptr) return 0;
  return std::max<size_t>(256, dtype == SAMA_DTYPE_BF16 ? glu_ffn_grad_bytes(T, d, F) : glu_ffn_f32_grad_bytes(T, d, F));
}

sama_status sama_op_glu_ffn(const void* x, int64_t ldx, const void* w_in, const void* w_out, int64_t T, int32_t d, int32_t F, int32_t act, int32_t dtype,
                            void* y, int64_t ldy, void* hidden, void* saved, void* workspace, size_t workspace_bytes, void* hip_stream) {
  static const char* const op = "sama_op_glu_ffn";
  g_ops_error.clear();
  if (const char* e = check_glu(T, d, F, dtype)) return refuse(op, e);
  if (act != SAMA_ACT_SILU && act != SAMA_ACT_GELU) return refuse(op, "act must be SAMA_ACT_SILU or SAMA_ACT_GELU");
  if (T == 0) return SAMA_OK;
  if (!is_glu_rows(x, ldx, d, dtype) || !is_glu_rows(y, ldy, d, dtype)) return refuse(op, "x or y is null or misaligned, or its stride is too small, too large or (bf16) no multiple of 8");
  if (!is_glu_dense(w_in, dtype) || !is_glu_dense(w_out, dtype) || !is_glu_dense(hidden, dtype)) return refuse(op, "a weight or hidden is null or misaligned");
  if (((uintptr_t)saved & 15) != 0) return refuse(op, "saved must be 16-byte aligned");
  if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < sama_op_glu_ffn_bytes(T, d, F, dtype)) {
    (void)refuse(op, "workspace missing, not aligned to 256 bytes or smaller than sama_op_glu_ffn_bytes()");
    return SAMA_EWORKSPACE;
  }
  GluFfnArgs a{};
  a.x = x; a.ldx = ldx; a.w_in = w_in; a.w_out = w_out; a.T = T; a.d = d; a.F = F; a.act = act; a.y = y; a.ldy = ldy; a.hidden = hidden; a.saved = saved;
  (void)hipGetLastError();
  if (dtype == SAMA_DTYPE_BF16) launch_glu_ffn((hipStream_t)hip_stream, a, workspace);
  else launch_glu_ffn_f32((hipStream_t)hip_stream, a, workspace);
  return launched(op);
}

sama_status sama_op_glu_ffn_grad(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w_in, const void* w_out, const void* hidden,
                                 const void* saved, int64_t T, int32_t d, int32_t F, int32_t act, int32_t dtype, void* dx, int64_t lddx, void* dw_in,
                                 void* dw_out, int32_t dw_dtype, void* workspace, size_t workspace_bytes, void* hip_stream) {
  static const char* const op = "sama_op_glu_ffn_grad";
  g_ops_error.clear();
  if (const char* e = check_glu(T, d, F, dtype)) return refuse(op, e);
  if (act != SAMA_ACT_SILU && act != SAMA_ACT_GELU) return refuse(op, "act must be SAMA_ACT_SILU or SAMA_ACT_GELU");
  if (dw_dtype != dtype && dw_dtype != SAMA_DTYPE_FP32) return refuse(op, "dw_dtype must be dtype or SAMA_DTYPE_FP32");
  if (!is_glu_dense(dw_in, dtype) || !is_glu_dense(dw_out, dtype)) return refuse(op, "a weight's gradient is null or misaligned");
  if (T > 0) {
    if (!is_glu_rows(x, ldx, d, dtype) || !is_glu_rows(dy, lddy, d, dtype) || !is_glu_rows(dx, lddx, d, dtype))
      return refuse(op, "x, dy or dx is null or misaligned, or its stride is too small, too large or (bf16) no multiple of 8");
    if (!is_glu_dense(w_in, dtype) || !is_glu_dense(w_out, dtype) || !is_glu_dense(hidden, dtype)) return refuse(op, "a weight or hidden is null or misaligned");
    if (saved == nullptr || ((uintptr_t)saved & 15) != 0) return refuse(op, "saved must be what the forward call wrote, 16-byte aligned");
  }
  if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < sama_op_glu_ffn_grad_bytes(T, d, F, dtype)) {
    (void)refuse(op, "workspace missing, not aligned to 256 bytes or smaller than sama_op_glu_ffn_grad_bytes()");
    return SAMA_EWORKSPACE;
  }
  (void)hipGetLastError();
  if (T == 0) {
    const int64_t words = dw_dtype == SAMA_DTYPE_FP32 ? (int64_t)d * F : (int64_t)d * F / 2;   // bf16: d F is even
    launch_fill_f32((hipStream_t)hip_stream, (float*)dw_in, 0.f, 2 * words);
    launch_fill_f32((hipStream_t)hip_stream, (float*)dw_out, 0.f, words);
    return launched(op);
  }
  GluFfnGradArgs a{};
  a.dy = dy; a.lddy = lddy; a.x = x; a.ldx = ldx; a.w_in = w_in; a.w_out = w_out; a.hidden = hidden; a.saved = saved; a.T = T; a.d = d; a.F = F; a.act = act;
  a.dx = dx; a.lddx = lddx; a.dw_in = dw_in; a.dw_out = dw_out; a.dw_fp32 = dw_dtype == SAMA_DTYPE_FP32;
  if (dtype == SAMA_DTYPE_BF16) launch_glu_ffn_grad((hipStream_t)hip_stream, a, workspace);
  else launch_glu_ffn_grad_f32((hipStream_t)hip_stream, a, workspace);
  return launched(op);
}
// ---- sequences
namespace {
constexpr int64_t MOST_ROTARY_TOKENS = (int64_t)1 << 23, MOST_DISTILL_TOKENS = (int64_t)1 << 22, MOST_HEAD_ROWS = (int64_t)1 << 28;
constexpr int32_t MOST_KEY_HEADS = 1 << 20;
// [tokens][heads][width] of any alignment
bool is_heads(const void* p, int32_t dtype, int64_t tokens, int64_t heads, int64_t width, int64_t ld, int64_t hs) {
  return ld >= width && hs >= width && is_rows(p, dtype, tokens, ld) && is_rows(p, dtype, heads, hs);
}
const char* check_attention_sizes(int64_t Tq, int64_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t dtype) {
  if (!is_dtype(dtype)) return "the type must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16";
  if (Hk < 1 || Hq < Hk || Hq % Hk != 0 || Hq / Hk > 64) return "Hq must be 1 to 64 times Hk";
  // workgroups of up to 512 threads for each key head and each 32 rows or more: 0.63 of the 2^32 work items of a launch at most
  if (Hk > MOST_KEY_HEADS) return "Hk must be up to 2^20";
  if (D < 8 || D > 128 || D % 8 != 0) return "D must be a multiple of 8, up to 128";
  if (Tq < 0 || Tk < 0 || Tq > MOST_HEAD_ROWS / Hq || Tk > MOST_HEAD_ROWS / Hk) return "Tq Hq and Tk Hk must be 0 to 2^28";
  return nullptr;
}
bool is_attention_heads(const sama_heads& t, int64_t tokens, const sama_attention& a, bool packed) {
  const int unit = a.dtype == SAMA_DTYPE_BF16 ? 8 : 4;
  if (tokens == 0) return true;
  if (t.p == nullptr || (uintptr_t)t.p % 16 != 0 || t.ld % unit != 0 || t.hs % unit != 0) return false;
  if (t.ld < a.D || t.hs < a.D || t.ld > ((int64_t)1 << 21) || t.hs > ((int64_t)1 << 40)) return false;
  return !packed || (a.Hq / a.Hk - 1) * t.hs * value_bytes(a.dtype) < ((int64_t)1 << 30);
}
const char* check_attention(const sama_attention& a, bool grad) {
  if (const char* e = check_attention_sizes(a.Tq, a.Tk, a.Hq, a.Hk, a.D, a.dtype)) return e;
  if (!(a.scale > 0.f) || !std::isfinite(a.scale)) return "scale must be positive and finite";
  if (a.cap != 0.f && !(a.cap >= 1e-3f && a.cap <= 4096.f)) return "cap must be 0 (none), or 1e-3 to 4096";
  if (a.Tq > 0 && (a.spans == nullptr || (uintptr_t)a.spans % 8 != 0)) return "spans missing, or not aligned to 8 bytes";
  if ((uintptr_t)a.at % 4 != 0 || (uintptr_t)a.slopes % 4 != 0 || (uintptr_t)a.lse % 4 != 0) return "at, slopes or lse is not aligned to its values";
  if (a.slopes != nullptr && a.at == nullptr && a.Tq != a.Tk) return "slopes need the queries' places (at) where Tq is not Tk";
  if (!is_attention_heads(a.q, a.Tq, a, grad) || !is_attention_heads(a.k, a.Tk, a, false) || !is_attention_heads(a.v, a.Tk, a, false) ||
      !is_attention_heads(a.out, a.Tq, a, false))
    return "q, k, v or out is missing, not aligned to 16 bytes, or has a stride that is too small, too large or not a multiple of 16 bytes";
  if (!grad) return nullptr;
  if (a.Tq > 0 && a.lse == nullptr) return "null lse";
  if (!is_attention_heads(a.dout, a.Tq, a, true) || !is_attention_heads(a.dq, a.Tq, a, false) || !is_attention_heads(a.dk, a.Tk, a, false) ||
      !is_attention_heads(a.dv, a.Tk, a, false))
    return "dout, dq, dk or dv is missing, not aligned to 16 bytes, or has a stride that is too small, too large or not a multiple of 16 bytes";
  return nullptr;
}
AttentionArgs attention_args(const sama_attention& s) {
  auto heads = [](const sama_heads& h) { return Heads{h.p, h.ld, h.hs}; };
  AttentionArgs a{};
  a.q = heads(s.q); a.k = heads(s.k); a.v = heads(s.v); a.out = heads(s.out); a.dout = heads(s.dout); a.dq = heads(s.dq); a.dk = heads(s.dk); a.dv = heads(s.dv);
  a.spans = s.spans; a.at = s.at; a.slopes = s.slopes; a.lse = s.lse; a.Tq = s.Tq; a.Tk = s.Tk; a.Hq = s.Hq; a.Hk = s.Hk; a.D = s.D; a.scale = s.scale; a.cap = s.cap;
  return a;
}
const char* check_distill(const void* z, int64_t ldz, int32_t dtype, int64_t T, int32_t V, const int32_t* ids, const float* teacher, int32_t K, float tau) {
  if (!is_dtype(dtype)) return "the type must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16";
  if (T < 0 || T > MOST_DISTILL_TOKENS) return "T must be 0 to 2^22";
  if (V < 1 || V > (1 << 30)) return "V must be 1 to 2^30";   // places in a row are 32 bits, behind its end too
  if (K < 1 || K > DISTILL_MAX_ENTRIES) return "K must be 1 to 256";
  if (!(tau >= 1e-4f && tau <= 1e4f)) return "temperature must be 1e-4 to 1e4";
  if (T == 0) return nullptr;
  if (!z || !ids || !teacher) return "null logits, ids or teacher";
  if ((uintptr_t)ids % 4 != 0 || (uintptr_t)teacher % 4 != 0) return "ids or teacher is not aligned to its values";
  if (ldz < V || !is_rows(z, dtype, T, ldz)) return "logits are not aligned to their values, or their stride is smaller than a row or too large";
  return nullptr;
}
}  // namespace

sama_status sama_op_rotary(const void* x, int64_t ldx, int64_t hsx, int64_t T, int32_t H, int32_t D, int32_t dtype, const int32_t* positions, int32_t axes,
                           const int32_t* sections, double base, int32_t neighbours, int32_t inverse, void* out, int64_t ldo, int64_t hso, void* hip_stream) {
  static const char* const op = "sama_op_rotary";
  g_ops_error.clear();
  if (!is_dtype(dtype)) return refuse(op, "the type must be SAMA_DTYPE_FP32 or SAMA_DTYPE_BF16");
  if (T < 0 || T > MOST_ROTARY_TOKENS) return refuse(op, "T must be 0 to 2^23");
  if (H < 1 || D < 2 || (int64_t)H * D > (1 << 20)) return refuse(op, "H must be positive, D at least 2 and H D up to 2^20");
  if (axes < 1 || axes > ROTARY_MAX_AXES || sections == nullptr) return refuse(op, "axes must be 1 to 4, with a section each");
  int64_t pairs = 0;
  for (int k = 0; k < axes; ++k) {
    if (sections[k] < 0 || sections[k] > ROTARY_MAX_PAIRS) return refuse(op, "a section must be 0 to 128 pairs");
    pairs += sections[k];
  }
  if (pairs < 1 || pairs > ROTARY_MAX_PAIRS || 2 * pairs > D) return refuse(op, "the sections must be 1 to 128 pairs together, and fit in D");
  if (!(base >= 1e-6) || !std::isfinite(base)) return refuse(op, "base must be finite, and at least 1e-6");   // below it turns of far positions have no fraction left in 64 bits
  if ((neighbours != 0 && neighbours != 1) || (inverse != 0 && inverse != 1)) return refuse(op, "neighbours and inverse must be 0 or 1");
  if (T == 0) return SAMA_OK;
  if (!x || !out || !positions) return refuse(op, "null x, output or positions");
  if ((uintptr_t)positions % 4 != 0) return refuse(op, "positions must be aligned to 4 bytes");
  if (!is_heads(x, dtype, T, H, D, ldx, hsx) || !is_heads(out, dtype, T, H, D, ldo, hso)) return refuse(op, "a pointer is not aligned to its values, or a stride is smaller than a head or too large");
  if (out == x && (ldx != ldo || hsx != hso)) return refuse(op, "in place the strides must be the same");
  RotaryArgs a{};
  a.x = Heads{x, ldx, hsx}; a.out = out; a.ldo = ldo; a.hso = hso; a.T = T; a.H = H; a.D = D; a.R = (int)(2 * pairs); a.axes = axes; a.positions = positions;
  a.sections = sections; a.base = base; a.neighbours = neighbours != 0; a.inverse = inverse != 0; a.bf16 = dtype == SAMA_DTYPE_BF16;
  (void)hipGetLastError();
  launch_rotary((hipStream_t)hip_stream, a);
  return launched(op);
}

size_t sama_op_attention_bytes(int64_t Tq, int64_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t dtype) {
  return check_attention_sizes(Tq, Tk, Hq, Hk, D, dtype) != nullptr ? 0 : attention_bytes(Tq, Tk, Hq, Hk, D, dtype == SAMA_DTYPE_BF16);
}
size_t sama_op_attention_grad_bytes(int64_t Tq, int64_t Tk, int32_t Hq, int32_t Hk, int32_t D, int32_t dtype) {
  return check_attention_sizes(Tq, Tk, Hq, Hk, D, dtype) != nullptr ? 0 : attention_grad_bytes(Tq, Tk, Hq, Hk, D);
}
sama_status sama_op_attention(const sama_attention* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  static const char* const op = "sama_op_attention";
  g_ops_error.clear();
  if (args == nullptr) return refuse(op, "null arguments");
  if (const char* e = check_attention(*args, false)) return refuse(op, e);
  if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < attention_bytes(args->Tq, args->Tk, args->Hq, args->Hk, args->D, args->dtype == SAMA_DTYPE_BF16)) {
    (void)refuse(op, "workspace missing, not aligned to 256 bytes or smaller than sama_op_attention_bytes()");
    return SAMA_EWORKSPACE;
  }
  if (args->Tq == 0) return SAMA_OK;
  (void)hipGetLastError();
  launch_attention((hipStream_t)hip_stream, attention_args(*args), args->dtype == SAMA_DTYPE_BF16, workspace);
  return launched(op);
}
sama_status sama_op_attention_grad(const sama_attention* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  static const char* const op = "sama_op_attention_grad";
  g_ops_error.clear();
  if (args == nullptr) return refuse(op, "null arguments");
  if (const char* e = check_attention(*args, true)) return refuse(op, e);
  if (!workspace || (uintptr_t)workspace % 256 != 0 || workspace_bytes < attention_grad_bytes(args->Tq, args->Tk, args->Hq, args->Hk, args->D)) {
    (void)refuse(op, "workspace missing, not aligned to 256 bytes or smaller than sama_op_attention_grad_bytes()");
    return SAMA_EWORKSPACE;
  }
  if (args->Tq == 0 && args->Tk == 0) return SAMA_OK;
  (void)hipGetLastError();
  launch_attention_grad((hipStream_t)hip_stream, attention_args(*args), args->dtype == SAMA_DTYPE_BF16, workspace);
  return launched(op);
}
sama_status sama_op_attention_spans(const int32_t* offsets, int64_t documents, const int32_t* prefix, int32_t causal, int64_t T, int32_t* spans, void* hip_stream) {
  static const char* const op = "sama_op_attention_spans";
  g_ops_error.clear();
  if (documents < 0 || documents > ((int64_t)1 << 30) || T < 0 || T > MOST_HEAD_ROWS) return refuse(op, "documents must be 0 to 2^30 and T 0 to 2^28");
  if (causal != 0 && causal != 1) return refuse(op, "causal must be 0 or 1");
  if (T == 0) return SAMA_OK;
  if (!offsets || !spans) return refuse(op, "null offsets or spans");
  if ((uintptr_t)offsets % 4 != 0 || (uintptr_t)prefix % 4 != 0 || (uintptr_t)spans % 8 != 0) return refuse(op, "offsets or prefix is not aligned to its values, or spans not to 8 bytes");
  (void)hipGetLastError();
  launch_attention_spans((hipStream_t)hip_stream, offsets, documents, prefix, causal != 0, T, spans);
  return launched(op);
}

sama_status sama_op_distill(const void* logits, int64_t ldz, int32_t dtype, int64_t T, int32_t V, const int32_t* ids, const float* teacher, int32_t K, float temperature,
                            float* loss, float* saved, void* hip_stream) {
  static const char* const op = "sama_op_distill";
  g_ops_error.clear();
  if (const char* e = check_distill(logits, ldz, dtype, T, V, ids, teacher, K, temperature)) return refuse(op, e);
  if (T == 0) return SAMA_OK;
  if (!loss || !saved || (uintptr_t)loss % 4 != 0 || (uintptr_t)saved % 4 != 0) return refuse(op, "loss or saved is null or not aligned to its values");
  DistillArgs a{};
  a.z = logits; a.ldz = ldz; a.bf16 = dtype == SAMA_DTYPE_BF16; a.T = T; a.V = V; a.K = K; a.ids = ids; a.teacher = teacher; a.tau = temperature; a.loss = loss; a.saved = saved;
  (void)hipGetLastError();
  launch_distill((hipStream_t)hip_stream, a);
  return launched(op);
}
sama_status sama_op_distill_grad(const void* logits, int64_t ldz, int32_t dtype, int64_t T, int32_t V, const int32_t* ids, const float* teacher, int32_t K, float temperature,
                                 const float* dloss, const float* saved, void* dlogits, int64_t lddz, void* hip_stream) {
  static const char* const op = "sama_op_distill_grad";
  g_ops_error.clear();
  if (const char* e = check_distill(logits, ldz, dtype, T, V, ids, teacher, K, temperature)) return refuse(op, e);
  if (T == 0) return SAMA_OK;
  if (!dloss || !saved || (uintptr_t)dloss % 4 != 0 || (uintptr_t)saved % 4 != 0) return refuse(op, "dloss or saved is null or not aligned to its values");
  if (!dlogits || lddz < V || !is_rows(dlogits, dtype, T, lddz)) return refuse(op, "dlogits are null or not aligned to their values, or their stride is smaller than a row or too large");
  if (dlogits == logits && lddz != ldz) return refuse(op, "in place the strides must be the same");
  DistillArgs a{};
  a.z = logits; a.ldz = ldz; a.bf16 = dtype == SAMA_DTYPE_BF16; a.T = T; a.V = V; a.K = K; a.ids = ids; a.teacher = teacher; a.tau = temperature;
  a.dloss = dloss; a.saved = const_cast<float*>(saved); a.dz = dlogits; a.lddz = lddz;
  (void)hipGetLastError();
  launch_distill_grad((hipStream_t)hip_stream, a);
  return launched(op);
}

sama_status sama_dev_glu_tile(int32_t tile) { return glu_ffn_force_tile(tile) ? SAMA_OK : SAMA_EINVAL; }

}  // extern "C"
