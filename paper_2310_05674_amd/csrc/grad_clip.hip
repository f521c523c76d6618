// The global norm of many gradients, and the gradients scaled so that it does not exceed a bound:
//   norm = sqrt(sum over all tensors of g^2),  factor = min(1, max_norm / (norm + 1e-6)),  out = factor g.
// Bound by memory: every gradient is read for the norm, and read and written for the scaling, unless the factor is 1 and the result
// goes where the gradients are.  Squares are added in 64 bits (no overflow and no loss whatever the sizes are; four values a clock and CU
// arrive from memory, far fewer than its 64-bit units take), in a fixed order.
//
// The tensors' pointers and sizes travel in the kernel's arguments, up to TENSORS a launch: nothing is copied to the device first, so a call
// may be captured.  A tensor is cut into units, a block takes every so many-th unit of all of them.  One launch of each kernel for
// models of up to TENSORS tensors: the blocks of the second add the partial sums up for themselves instead of waiting for a last block.
// The second kernel walks the units backwards: the end of the gradients is what the last-level cache still holds.
#include <algorithm>
#include <cmath>
#include "kernels.h"
#include "token_ops.h"

namespace sama {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int TENSORS = 112, UNIT = 8192, THREADS = 256, PARTIALS = 2048;

struct ClipTable {
  int count, units;
  double max_norm;
  double* partial; int partials, add;   // add: to what earlier launches left
  float* norm; int64_t* status;         // of the second kernel's first launch
  float* out;
  void* p[TENSORS];
  int64_t n[TENSORS];
  int64_t to[TENSORS];                  // place in out
  int32_t first[TENSORS + 1];           // unit
  uint32_t bf16[(TENSORS + 31) / 32];
};
static_assert(sizeof(ClipTable) <= 4000, "kernel arguments");

// the tensor that a unit belongs to, found by a wave at once
__device__ __forceinline__ int tensor_of(const ClipTable& t, int unit) {
  const int lane = threadIdx.x & 63;
  int k = -1;
#pragma unroll
  for (int c = 0; c < TENSORS; c += 64) k += __popcll(__ballot(c + lane < t.count && t.first[min(c + lane, TENSORS)] <= unit));
  return __builtin_amdgcn_readfirstlane(k);
}
// values before the first 16-byte boundary
__device__ __forceinline__ int ahead(const void* p, int size) { return (int)((16 - ((uintptr_t)p & 15)) & 15) / size; }

template <typename T>
__device__ __forceinline__ double square_sum(const T* p, int64_t n, int64_t at) {
  constexpr int V = 16 / sizeof(T), PER = UNIT / THREADS / V;
  auto sq = [](float x) { return (double)x * (double)x; };
  auto val = [](T x) { if constexpr (sizeof(T) == 2) return bf16_to_f32(x); else return x; };
  double s = 0.0;
  const int head = (int)min((int64_t)ahead(p, sizeof(T)), n);
  if (at == 0 && (int)threadIdx.x < head) s += sq(val(p[threadIdx.x]));
  p += head; n -= head;
  if (at + UNIT <= n) {
    uint4 v[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) v[u] = *reinterpret_cast<const uint4*>(p + at + (int64_t)(u * THREADS + threadIdx.x) * V);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) s += sq(__uint_as_float(w[k]));
        else s += sq(__uint_as_float(w[k] << 16)) + sq(__uint_as_float(w[k] & 0xffff0000u));
      }
    }
  } else {
    for (int64_t i = at + threadIdx.x; i < n; i += THREADS) s += sq(val(p[i]));
  }
  return s;
}

__device__ __forceinline__ double block_sum64(double s, double* red) {
  s = wave_sum(s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < THREADS / 64; ++w) s += red[w];
  return s;
}

__global__ __launch_bounds__(THREADS) void k_square_sums(ClipTable t) {
  __shared__ double red[THREADS / 64];
  double s = 0.0;
  for (int unit = blockIdx.x; unit < t.units; unit += gridDim.x) {
    const int k = tensor_of(t, unit);
    const int64_t at = (int64_t)(unit - t.first[k]) * UNIT;
    s += (t.bf16[k >> 5] >> (k & 31)) & 1 ? square_sum(static_cast<const bf16_t*>(t.p[k]), t.n[k], at)
                                           : square_sum(static_cast<const float*>(t.p[k]), t.n[k], at);
  }
  s = block_sum64(s, red);
  if (threadIdx.x == 0) t.partial[blockIdx.x] = t.add ? t.partial[blockIdx.x] + s : s;
}

template <typename T, typename O>
__device__ __forceinline__ void scale_unit(const T* p, O* to, int64_t n, int64_t at, float f) {
  constexpr int V = 16 / sizeof(T), PER = UNIT / THREADS / V;
  auto one = [&](int64_t i) {
    if constexpr (sizeof(T) == 4) to[i] = p[i] * f;
    else if constexpr (sizeof(O) == 2) to[i] = f32_to_bf16(bf16_to_f32(p[i]) * f);
    else to[i] = bf16_to_f32(p[i]) * f;
  };
  const int head = (int)min((int64_t)ahead(p, sizeof(T)), n);
  if (at == 0 && (int)threadIdx.x < head) one(threadIdx.x);
  p += head; to += head; n -= head;
  if (at + UNIT <= n && ((uintptr_t)to & 15) == 0) {
    uint4 v[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) v[u] = *reinterpret_cast<const uint4*>(p + at + (int64_t)(u * THREADS + threadIdx.x) * V);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      O* const o = to + at + (int64_t)(u * THREADS + threadIdx.x) * V;
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4*>(o) = (f32x4){__uint_as_float(w[0]) * f, __uint_as_float(w[1]) * f, __uint_as_float(w[2]) * f, __uint_as_float(w[3]) * f};
      } else {
        float x[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16) * f; x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u) * f; }
        if constexpr (sizeof(O) == 2) {
          *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
        } else {
          *reinterpret_cast<f32x4*>(o) = (f32x4){x[0], x[1], x[2], x[3]};
          *reinterpret_cast<f32x4*>(o + 4) = (f32x4){x[4], x[5], x[6], x[7]};
        }
      }
    }
  } else {
    const int64_t end = min(at + UNIT, n);
    for (int64_t i = at + threadIdx.x; i < end; i += THREADS) one(i);
  }
}

__global__ __launch_bounds__(THREADS) void k_clip(ClipTable t) {
  __shared__ double red[THREADS / 64];
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < PARTIALS; i += THREADS) s += i + (int)threadIdx.x < t.partials ? t.partial[i + threadIdx.x] : 0.0;
  const double norm = sqrt(block_sum64(s, red));
  const bool finite = norm <= 1.7976931348623157e308;
  const float factor = finite ? (float)fmin(1.0, t.max_norm / (norm + 1e-6)) : 1.f;
  if (t.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) {
    t.norm[0] = (float)norm; t.norm[1] = factor;
    if (t.status != nullptr) *t.status = finite ? 0 : 1;
  }
  if (t.out == nullptr && factor == 1.f) return;
  for (int unit = t.units - 1 - (int)blockIdx.x; unit >= 0; unit -= gridDim.x) {
    const int k = tensor_of(t, unit);
    const int64_t at = (int64_t)(unit - t.first[k]) * UNIT;
    const bool half = (t.bf16[k >> 5] >> (k & 31)) & 1;
    if (t.out != nullptr) {
      if (half) scale_unit(static_cast<const bf16_t*>(t.p[k]), t.out + t.to[k], t.n[k], at, factor);
      else scale_unit(static_cast<const float*>(t.p[k]), t.out + t.to[k], t.n[k], at, factor);
    } else {
      if (half) scale_unit(static_cast<const bf16_t*>(t.p[k]), static_cast<bf16_t*>(t.p[k]), t.n[k], at, factor);
      else scale_unit(static_cast<const float*>(t.p[k]), static_cast<float*>(t.p[k]), t.n[k], at, factor);
    }
  }
}
}  // namespace

size_t grad_clip_bytes() { return PARTIALS * sizeof(double); }

void launch_grad_clip(hipStream_t st, const GradTensor* g, int64_t count, double max_norm, float* norm, float* out, int64_t* status, void* workspace) {
  // launches: the next tensors that are not empty, up to TENSORS of them and 2^30 units
  auto next = [&](int64_t& k, int64_t& flat, ClipTable& t) {
    t.count = t.units = 0;
    for (uint32_t& w : t.bf16) w = 0;
    for (; k < count && t.count < TENSORS; ++k) {
      if (g[k].n == 0) continue;
      const int64_t units = (g[k].n + UNIT - 1) / UNIT;
      if (t.count > 0 && t.units + units > (1 << 30)) break;
      t.p[t.count] = g[k].p; t.n[t.count] = g[k].n; t.to[t.count] = flat; t.first[t.count] = t.units;
      if (g[k].bf16) t.bf16[t.count >> 5] |= 1u << (t.count & 31);
      flat += g[k].n; t.units += (int)units; ++t.count;
    }
    t.first[t.count] = t.units;
  };
  ClipTable t{};
  int most = 0;
  for (int64_t k = 0, flat = 0; k < count;) { next(k, flat, t); most = std::max(most, t.units); }
  const int blocks = std::max(1, std::min(most, PARTIALS));
  t.max_norm = max_norm; t.partial = static_cast<double*>(workspace); t.partials = blocks; t.out = out;
  ProfScope ps(st, F_OTHER, 0.0);
  int64_t k = 0, flat = 0;
  t.add = 0;
  do {
    next(k, flat, t);
    launch_kernel(ps, k_square_sums, blocks, THREADS, 0, st, t);
    t.add = 1;
  } while (k < count);
  k = flat = 0;
  t.norm = norm; t.status = status;
  const bool scale = out != nullptr || !std::isinf(max_norm);
  do {
    next(k, flat, t);
    launch_kernel(ps, k_clip, scale ? std::max(1, std::min(t.units, PARTIALS)) : 1, THREADS, 0, st, t);
    t.norm = nullptr; t.status = nullptr;
  } while (scale && k < count);
}

}  // namespace sama
