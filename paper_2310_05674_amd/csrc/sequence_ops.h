// Launchers of the operators of a token model's sequences: rotary positions, attention within spans of keys, distillation from a teacher's top logits.
// Internal; the C ABI is include/sama_ops.h, which says what each argument means and checks it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "common.h"

namespace sama {

constexpr int ROTARY_MAX_AXES = 4, ROTARY_MAX_PAIRS = 128;
struct Heads { const void* p; int64_t ld, hs; };   // [tokens][heads][width], strides in values

struct RotaryArgs {
  Heads x; void* out; int64_t ldo, hso;
  int64_t T; int H, D, R, axes;                    // R: width that is turned
  const int32_t* positions;                        // [axes][T]
  const int32_t* sections;                         // host
  double base; bool neighbours, inverse, bf16;
};
void launch_rotary(hipStream_t, const RotaryArgs&);

constexpr int DISTILL_MAX_ENTRIES = 256;
struct DistillArgs {
  const void* z; int64_t ldz; bool bf16;
  int64_t T; int V, K;
  const int32_t* ids; const float* teacher;
  float tau;
  float *loss, *saved;                             // saved [T][2] = largest logit, sum of exp((z - it) / tau)
  const float* dloss; void* dz; int64_t lddz;      // of the gradient
};
void launch_distill(hipStream_t, const DistillArgs&);
void launch_distill_grad(hipStream_t, const DistillArgs&);

// Attention (attention.hip, attention_grad.hip), shapes as in include/sama_ops.h.
struct AttentionArgs {
  Heads q, k, v, out, dout, dq, dk, dv;            // what is written has its const cast away
  const int32_t *spans, *at; const float* slopes;
  float* lse;                                      // [Tq][Hq], natural, or null in the forward pass
  int64_t Tq, Tk; int Hq, Hk, D;
  float scale, cap;
};
void launch_attention_spans(hipStream_t, const int32_t* offsets, int64_t documents, const int32_t* prefix, bool causal, int64_t T, int32_t* spans);
size_t attention_bytes(int64_t Tq, int64_t Tk, int Hq, int Hk, int D, bool bf16);
size_t attention_grad_bytes(int64_t Tq, int64_t Tk, int Hq, int Hk, int D);
void launch_attention(hipStream_t, const AttentionArgs&, bool bf16, void* workspace);
void launch_attention_grad(hipStream_t, const AttentionArgs&, bool bf16, void* workspace);

}  // namespace sama
