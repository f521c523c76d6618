// Distillation from a teacher's top logits.  For a token with student logits z [V] and listed entries (id_k, t_k):
//   p = softmax over its entries of t / tau,  q = softmax over the vocabulary of z / tau,
//   loss = tau^2 sum_k p_k (log p_k - log q_{id_k}),  dz_j = g tau (q_j - sum over the k with id_k = j of p_k)  for dloss = g.
// Bound by memory: the loss reads z once (the running maximum and sum of a softmax), the gradient reads z and writes dz once, with the row's maximum and sum
// that the loss kept.  A workgroup takes a token; what concerns its entries is done by as many threads, in 64 bits (256 of them at most), because the loss is a
// small difference where student and teacher agree.
// Entries outside the vocabulary, or of a logit of minus infinity, are none; a token without entries has loss and gradient zero, and its logits are not read.
#include <algorithm>
#include <cmath>
#include <limits>
#include "kernels.h"
#include "sequence_ops.h"

namespace sama {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr float LOG2E = 1.44269504088896340736f;

template <typename E> constexpr int VALUES = 16 / sizeof(E);
template <typename E> __device__ __forceinline__ float value(E x) {
  if constexpr (sizeof(E) == 2) return bf16_to_f32(x);
  else return x;
}
template <typename E> __device__ __forceinline__ E rounded(float x) {
  if constexpr (sizeof(E) == 2) return f32_to_bf16(x);
  else return x;
}
template <typename E> __device__ __forceinline__ void unpack(const uint4& w, float (&x)[VALUES<E>]) {
  const uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(E) == 2) { x[2 * i] = __uint_as_float(d[i] << 16); x[2 * i + 1] = __uint_as_float(d[i] & 0xffff0000u); }
    else x[i] = __uint_as_float(d[i]);
  }
}
template <typename E> __device__ __forceinline__ uint4 pack(const float (&x)[VALUES<E>]) {
  if constexpr (sizeof(E) == 2) return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  else return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}

// over a workgroup; `red` holds a value for each wave
template <int THREADS, typename T, typename F>
__device__ __forceinline__ T block_join(T x, T* red, F op) {
  x = join_wave(x, op);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) x = op(x, red[w]);
  return x;
}

// A thread's entry, if it has one, and its probability.  Up to 64 entries are the first wave's: every wave looks whether there are any, and nobody waits for the first one's
// exponentials before the row's loads.
struct Entry { int id; bool there; double p, logp; float z; };
template <typename E, int THREADS>
__device__ __forceinline__ bool entries(const DistillArgs& a, int64_t row, Entry& e, double* red) {
  const bool one_wave = a.K <= 64;
  const int k = one_wave ? threadIdx.x & 63 : threadIdx.x;
  e = Entry{-1, false, 0.0, 0.0, 0.f};
  float t = 0.f;
  if (k < a.K) {
    e.id = a.ids[row * a.K + k];
    t = a.teacher[row * a.K + k];
    e.there = e.id >= 0 && e.id < a.V && t != -std::numeric_limits<float>::infinity();
  }
  if (!(one_wave ? __any(e.there) : __syncthreads_or(e.there))) return false;
  if (one_wave && threadIdx.x >= 64) { e.id = -1; e.there = false; return true; }
  if (e.there) e.z = value<E>(static_cast<const E*>(a.z)[row * a.ldz + e.id]);
  const double low = -std::numeric_limits<double>::infinity(), tau = a.tau;
  auto larger = [](double x, double y) { return fmax(x, y); };
  auto add = [](double x, double y) { return x + y; };
  const double mine = e.there ? (double)t : low, top = one_wave ? join_wave(mine, larger) : block_join<THREADS>(mine, red, larger);
  const double x = ((double)t - top) / tau, w = e.there ? exp(x) : 0.0;
  const double sum = one_wave ? join_wave(w, add) : block_join<THREADS>(w, red, add);
  e.p = w / sum; e.logp = x - log(sum);
  return true;
}

// The values before the first 16-byte boundary of a row, its pieces, and the first value behind them.
template <typename E> __device__ __forceinline__ void split_row(const E* row, int V, int& head, int& pieces, int& tail) {
  head = min(V, (int)(((16 - ((uintptr_t)row & 15)) & 15) / sizeof(E)));
  pieces = (V - head) / VALUES<E>;
  tail = head + pieces * VALUES<E>;
}

// Tokens are workgroups along x, and where that would be more work items than one dimension of a launch holds (2^32 - 1), half of them along y.
__device__ __forceinline__ int64_t token_of_workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

template <typename E, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill(DistillArgs a) {
  __shared__ double red64[THREADS / 64];
  __shared__ float2 red[THREADS / 64];
  const int64_t row = token_of_workgroup();
  if (row >= a.T) return;
  Entry e;
  if (!entries<E, THREADS>(a, row, e, red64)) {
    if (threadIdx.x == 0) { a.loss[row] = 0.f; a.saved[2 * row] = 0.f; a.saved[2 * row + 1] = 1.f; }
    return;
  }
  const float c = LOG2E / a.tau;
  const E* const z = static_cast<const E*>(a.z) + row * a.ldz;
  int head, pieces, tail;
  split_row(z, a.V, head, pieces, tail);
  // starting at the lowest number, not at minus infinity, keeps minus infinity from being subtracted from itself
  float m = -std::numeric_limits<float>::max(), s = 0.f;
  auto one = [&](float x) {
    if (x > m) { s *= __builtin_amdgcn_exp2f((m - x) * c); m = x; }
    s += __builtin_amdgcn_exp2f((x - m) * c);
  };
  if ((int)threadIdx.x < head) one(value<E>(z[threadIdx.x]));
  const uint4* const body = reinterpret_cast<const uint4*>(z + head);
  constexpr int AHEAD = 4;
  for (int i = threadIdx.x; i < pieces; i += AHEAD * THREADS) {
    uint4 w[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) if (i + u * THREADS < pieces) w[u] = body[i + u * THREADS];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i + u * THREADS >= pieces) break;
      float x[VALUES<E>];
      unpack<E>(w[u], x);
      float top = m;
#pragma unroll
      for (int v = 0; v < VALUES<E>; ++v) top = fmaxf(top, x[v]);
      if (top > m) { s *= __builtin_amdgcn_exp2f((m - top) * c); m = top; }
#pragma unroll
      for (int v = 0; v < VALUES<E>; ++v) s += __builtin_amdgcn_exp2f((x[v] - m) * c);
    }
  }
  if (tail + (int)threadIdx.x < a.V) one(value<E>(z[tail + threadIdx.x]));
  // each wave's maximum and sum, then all of them
  const float top_w = join_wave(m, [](float x, float y) { return fmaxf(x, y); });
  const float sum_w = join_wave(s * __builtin_amdgcn_exp2f((m - top_w) * c), [](float x, float y) { return x + y; });
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(top_w, sum_w);
  __syncthreads();
  const bool one_wave = a.K <= 64;
  if (one_wave && threadIdx.x >= 64) return;
  float top = red[0].x, sum = 0.f;
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) top = fmaxf(top, red[i].x);
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) sum += red[i].y * __builtin_amdgcn_exp2f((red[i].x - top) * c);
  const double logq = ((double)e.z - (double)top) / (double)a.tau - log((double)sum), part = e.p == 0.0 ? 0.0 : e.p * (e.logp - logq);
  auto add = [](double x, double y) { return x + y; };
  const double loss = one_wave ? join_wave(part, add) : block_join<THREADS>(part, red64, add);
  if (threadIdx.x == 0) {
    a.loss[row] = (float)((double)a.tau * (double)a.tau * loss);
    a.saved[2 * row] = top; a.saved[2 * row + 1] = sum;
  }
}

template <typename E, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill_grad(DistillArgs a) {
  __shared__ double red64[THREADS / 64];
  __shared__ int s_id[DISTILL_MAX_ENTRIES];
  __shared__ float s_p[DISTILL_MAX_ENTRIES];
  const int64_t row = a.T - 1 - token_of_workgroup();   // from the end, which the loss read last: the last-level cache may still have it
  if (row < 0) return;
  const E* const z = static_cast<const E*>(a.z) + row * a.ldz;
  E* const dz = static_cast<E*>(a.dz) + row * a.lddz;
  int head, pieces, tail;
  split_row(dz, a.V, head, pieces, tail);
  uint4* const to = reinterpret_cast<uint4*>(dz + head);
  Entry e;
  if (!entries<E, THREADS>(a, row, e, red64)) {
    if ((int)threadIdx.x < head) dz[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < pieces; i += THREADS) to[i] = make_uint4(0, 0, 0, 0);
    if (tail + (int)threadIdx.x < a.V) dz[tail + threadIdx.x] = 0;
    return;
  }
  if ((int)threadIdx.x < a.K) { s_id[threadIdx.x] = e.there ? e.id : -1; s_p[threadIdx.x] = (float)e.p; }
  const float c = LOG2E / a.tau, top = a.saved[2 * row], g = a.dloss[row] * a.tau, inv = 1.f / a.saved[2 * row + 1], w = g * inv;
  const float zk = e.z;
  asm volatile("" ::"v"(zk));   // dz may be z: every entry's logit is here before any is overwritten
  __syncthreads();
  auto grad = [&](float x) { return __builtin_amdgcn_exp2f((x - top) * c) * w; };
  if ((int)threadIdx.x < head) dz[threadIdx.x] = rounded<E>(grad(value<E>(z[threadIdx.x])));
  if ((((uintptr_t)z ^ (uintptr_t)dz) & 15) == 0) {
    const uint4* const body = reinterpret_cast<const uint4*>(z + head);
    constexpr int AHEAD = 4;
    for (int i = threadIdx.x; i < pieces; i += AHEAD * THREADS) {
      uint4 p[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) if (i + u * THREADS < pieces) p[u] = body[i + u * THREADS];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (i + u * THREADS >= pieces) break;
        float x[VALUES<E>];
        unpack<E>(p[u], x);
#pragma unroll
        for (int v = 0; v < VALUES<E>; ++v) x[v] = grad(x[v]);
        to[i + u * THREADS] = pack<E>(x);
      }
    }
  } else {
    for (int i = head + threadIdx.x; i < tail; i += THREADS) dz[i] = rounded<E>(grad(value<E>(z[i])));
  }
  if (tail + (int)threadIdx.x < a.V) dz[tail + threadIdx.x] = rounded<E>(grad(value<E>(z[tail + threadIdx.x])));
  // the listed values once more, by the first entry of each id
  __syncthreads();
  if (!e.there) return;
  float p = 0.f;
  for (int k = 0; k < a.K; ++k) {
    if (s_id[k] != e.id) continue;
    if (k < (int)threadIdx.x) return;
    p += s_p[k];
  }
  dz[e.id] = rounded<E>((__builtin_amdgcn_exp2f((zk - top) * c) * inv - p) * g);
}

// Waves of a row, us at 256 / 512 / 1024 threads (T x V, loss and gradient): 37 x 8192 fp32: 4.3 / 3.9 / 4.1 and 5.0 / 4.7 / 4.7; 4096 x 8192 fp32: 22.7 / 22.0 / 30.2 and
// 44.2 / 43.2 / 43.0; 4096 x 30522 bf16: 41.4 / 39.6 / 44.5 and 105 / 97.2 / 97.2; 37 x 50304 fp32: 9.3 / 6.5 / 6.4 and 10.7 / 8.3 / 8.1; 4096 x 50304 fp32: 139 / 136 / 132 and
// 329 / 321 / 310.  The last are 6.2 and 5.3 TB/s (a copy: 5.0).
constexpr int LOSS_THREADS = 512, GRAD_THREADS = 1024;
template <typename E>
void launch(hipStream_t st, const DistillArgs& a, bool grad) {
  ProfScope ps(st, F_OTHER, (double)a.T * a.V * sizeof(E) * (grad ? 2 : 1));
  const int64_t most = ((int64_t)1 << 32) / (grad ? GRAD_THREADS : LOSS_THREADS) - 1;
  const dim3 grid = a.T <= most ? dim3((unsigned)a.T) : dim3((unsigned)((a.T + 1) / 2), 2);
  if (grad) launch_kernel(ps, k_distill_grad<E, GRAD_THREADS>, grid, GRAD_THREADS, 0, st, a);
  else launch_kernel(ps, k_distill<E, LOSS_THREADS>, grid, LOSS_THREADS, 0, st, a);
}
void launch_either(hipStream_t st, const DistillArgs& a, bool grad) { a.bf16 ? launch<bf16_t>(st, a, grad) : launch<float>(st, a, grad); }
}  // namespace

void launch_distill(hipStream_t st, const DistillArgs& a) { launch_either(st, a, false); }
void launch_distill_grad(hipStream_t st, const DistillArgs& a) { launch_either(st, a, true); }

}  // namespace sama
