// Launchers of the operators of a token model's step: embedding and its gradient, gradient clipping, the gated feed-forward block.
// Internal; the C ABI is include/sama_ops.h, which says what each argument means and checks it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "common.h"

namespace sama {

struct EmbeddingArgs {
  const void* table; int64_t ldt; bool table_bf16;
  const int32_t* ids; int64_t n; int V, d;
  float scale; int pad;
  void* out; int64_t ldo; bool out_bf16;
};
void launch_embedding(hipStream_t, const EmbeddingArgs&);

struct EmbeddingGradArgs {
  const void* dy; int64_t ldy; bool dy_bf16;
  const int32_t* ids; int64_t n; int V, d;      // n < 2^31
  float scale; int pad; bool accumulate;
  void* grad; int64_t ldg; bool grad_bf16;
};
size_t embedding_grad_bytes(int64_t n, int V, int d);
bool embedding_grad_fits(const EmbeddingGradArgs&);   // its launches have less than 2^32 threads
void launch_embedding_grad(hipStream_t, const EmbeddingGradArgs&, void* workspace);

struct GradList { void* const* p; const int64_t* n; const int32_t* dtype; };   // SAMA_DTYPE_*
size_t grad_clip_bytes();
// norm[0] = ||g||, norm[1] = the factor; out: flat fp32, or null (in place); status may be null
void launch_grad_clip(hipStream_t, const GradList& g, int64_t count, double max_norm, float* norm, float* out, int64_t* status, void* workspace);

// The gated feed-forward block (glu_ffn.hip; fp32 that its tiles cannot load: glu_ffn_f32.hip), shapes as in include/sama_ops.h.
enum { GLU_SILU = 0, GLU_GELU = 1 };
struct GluFfnArgs {
  const void* x; int64_t ldx; const void *w_in, *w_out;
  int64_t T; int d, F, act;
  void* y; int64_t ldy; void *hidden, *saved;
};
struct GluFfnGradArgs {
  const void* dy; int64_t lddy; const void* x; int64_t ldx; const void *w_in, *w_out, *hidden, *saved;
  int64_t T; int d, F, act;
  void* dx; int64_t lddx; void *dw_in, *dw_out; bool dw_fp32;
};
size_t glu_ffn_saved_bytes(int64_t T, int F);
size_t glu_ffn_bytes(int64_t T, int d, int F);
size_t glu_ffn_grad_bytes(int64_t T, int d, int F);
void launch_glu_ffn(hipStream_t, const GluFfnArgs&, void* workspace);
void launch_glu_ffn_grad(hipStream_t, const GluFfnGradArgs&, void* workspace);
size_t glu_ffn_f32_saved_bytes(int64_t T, int F);
size_t glu_ffn_f32_bytes(int64_t T, int d, int F);
size_t glu_ffn_f32_grad_bytes(int64_t T, int d, int F);
void launch_glu_ffn_f32(hipStream_t, const GluFfnArgs&, void* workspace);
void launch_glu_ffn_grad_f32(hipStream_t, const GluFfnGradArgs&, void* workspace);
// ... of any width, stride and alignment
size_t glu_ffn_plain_bytes(int64_t T, int F);
size_t glu_ffn_plain_grad_bytes(int64_t T, int F);
void launch_glu_ffn_plain(hipStream_t, const GluFfnArgs&, void* workspace);
void launch_glu_ffn_grad_plain(hipStream_t, const GluFfnGradArgs&, void* workspace);
bool glu_ffn_force_tile(int tile);   // tuning hook: 0 = heuristic; false for a tile that there is not

}  // namespace sama
