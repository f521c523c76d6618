// The global norm of many gradients, and the gradients scaled so that it does not exceed a bound:
//   norm = sqrt(sum over all tensors of g^2),  factor = min(1, max_norm / (norm + 1e-6)),  out = factor g.
// Bound by memory: every gradient is read for the norm, and read and written for the scaling, unless the factor is 1 and the result
// goes where the gradients are.  Squares are added in 64 bits (no overflow and no loss whatever the sizes are; four values a clock and CU
// arrive from memory, far fewer than its 64-bit units take), in a fixed order.
//
// The tensors' pointers and sizes travel in the kernel's arguments, up to TENSORS a launch: nothing is copied to the device first, so a call
// may be captured.  A tensor is cut into units of 32 KB, a block takes a run of them.  One launch of each kernel for
// models of up to TENSORS tensors: the blocks of the second add the partial sums up for themselves instead of waiting for a last block, while
// their first unit is on its way.  Up to PARTIALS blocks: 217 MB of bf16 matrices and fp32 vectors into 434 MB of flat gradient take 148 us (5.9 TB/s of
// what is read twice and written), with 2048 blocks 154, and 154 with 4096 blocks that walk backwards in the second kernel, towards what the last-level
// cache should still hold; 25 MB into a flat gradient, out of the caches, 17.3 us, of which two launches are a third.  Matrices alone, into `out` / in place: 6.3 million fp32
// values 16.0 / 16.0, 108 million 246 / 268, in bf16 146 / 130.  A tensor whose place in `out` is off 16 bytes (any behind one of odd length) goes out value by value and
// is read once more: 319 for 246, bf16 255 for 146.
#include <algorithm>
#include <cmath>
#include "../../include/sama_ops.h"
#include "kernels.h"
#include "token_ops.h"

namespace sama {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int TENSORS = 112, THREADS = 256, PER = 8, UNIT_BYTES = THREADS * PER * 16, PARTIALS = 4096;

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

// A tensor's values before its first 16-byte boundary, fewer than eight, belong to its unit 0 beside that unit's 32 KB.
struct Unit {
  int k;             // tensor
  int64_t n, at;     // values behind those, of them the unit begins with number `at`
  const char* p;     // the tensor
  int head, half;
  __device__ __forceinline__ int size() const { return half ? 2 : 4; }
  __device__ __forceinline__ int values() const { return UNIT_BYTES >> (half ? 1 : 2); }
  __device__ __forceinline__ bool whole() const { return at + values() <= n; }
};
__device__ __forceinline__ Unit unit_at(const ClipTable& t, int k, int unit) {
  Unit u;
  u.k = k;
  u.half = (t.bf16[k >> 5] >> (k & 31)) & 1;
  u.p = static_cast<const char*>(t.p[k]);
  u.head = (int)min((int64_t)((16 - ((uintptr_t)u.p & 15)) & 15) / u.size(), t.n[k]);
  u.n = t.n[k] - u.head;
  u.at = (int64_t)(unit - t.first[k]) * u.values();
  return u;
}
// the tensor that a unit belongs to, found by a wave at once
__device__ __forceinline__ int tensor_of(const ClipTable& t, int unit) {
  const int lane = threadIdx.x & 63;
  int k = -1;
#pragma unroll
  for (int c = 0; c < TENSORS; c += 64) k += __popcll(__ballot(c + lane < t.count && t.first[min(c + lane, TENSORS)] <= unit));
  return __builtin_amdgcn_readfirstlane(k);
}
// `halves`: a thread's eight bf16 values of a piece are two times four, 2 KB apart, so that the fp32 values they become are stored in whole lines
__device__ __forceinline__ void load_whole(const Unit& u, bool halves, uint4 (&v)[PER]) {
  const char* const p = u.p + ((u.head + u.at) << (u.half ? 1 : 2));
  if (halves) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint2 a = *reinterpret_cast<const uint2*>(p + (2 * i * THREADS + threadIdx.x) * 8), b = *reinterpret_cast<const uint2*>(p + ((2 * i + 1) * THREADS + threadIdx.x) * 8);
      v[i] = make_uint4(a.x, a.y, b.x, b.y);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = *reinterpret_cast<const uint4*>(p + (i * THREADS + threadIdx.x) * 16);
}
__device__ __forceinline__ float value_at(const Unit& u, int64_t i) {   // i: of the tensor
  return u.half ? bf16_to_f32(reinterpret_cast<const bf16_t*>(u.p)[i]) : reinterpret_cast<const float*>(u.p)[i];
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ double block_sum64(double s, double* red) {
  s = wave_sum(s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < THREADS / 64; ++w) s += red[w];
  return s;
}
// a block's run of the units
__device__ __forceinline__ void run_of(int units, int& from, int& to) {
  from = (int)((int64_t)units * blockIdx.x / gridDim.x);
  to = (int)((int64_t)units * (blockIdx.x + 1) / gridDim.x);
}

__global__ __launch_bounds__(THREADS) void k_square_sums(ClipTable t) {
  __shared__ double red[THREADS / 64];
  double s[4] = {};
  auto add = [&](int i, float x) { s[i & 3] += (double)x * (double)x; };
  int from, to;
  run_of(t.units, from, to);
  if (from < to) {
    int k = tensor_of(t, from);
    for (int unit = from; unit < to; ++unit) {
      while (unit >= t.first[k + 1]) ++k;
      const Unit u = unit_at(t, k, unit);
      if (u.at == 0 && (int)threadIdx.x < u.head) add(0, value_at(u, threadIdx.x));
      if (u.whole()) {
        uint4 v[PER];
        load_whole(u, false, v);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (u.half) { add(e, low(w[e])); add(e + 2, high(w[e])); }
            else add(e, __uint_as_float(w[e]));
          }
        }
      } else {
        for (int64_t i = u.at + threadIdx.x; i < u.n; i += THREADS) add(0, value_at(u, u.head + i));
      }
    }
  }
  const double sum = block_sum64((s[0] + s[1]) + (s[2] + s[3]), red);
  if (threadIdx.x == 0) t.partial[blockIdx.x] = t.add ? t.partial[blockIdx.x] + sum : sum;
}

// Results go past the caches, which keep the gradients for the second reading instead, and the next norm does not wait for them to be written back: the 217 MB
// above take 196 us with ordinary stores instead of 156, the 25 MB the same with both.
__device__ __forceinline__ void store_once(char* p, f32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(p)); }
// The factor as two, applied one after the other: 1 and itself, or 2^-64 and 2^64 times itself where it is so small that fp32 would hold it in fewer bits (norms beyond
// fp32's range).  The first product is exact, unless the second rounds to zero.
struct Factor {
  float first, second;
  __device__ __forceinline__ float operator()(float x) const { return x * first * second; }
};
// One unit, whose values are in v if it is a whole one, times f to `dest` (the tensor's place): bf16 in place, else fp32.
__device__ __forceinline__ void scale_unit(const Unit& u, const uint4 (&v)[PER], void* dest, bool to_bf16, Factor f) {
  auto one = [&](int64_t i) {
    const float x = f(value_at(u, i));
    if (to_bf16) static_cast<bf16_t*>(dest)[i] = f32_to_bf16(x);
    else static_cast<float*>(dest)[i] = x;
  };
  if (u.at == 0 && (int)threadIdx.x < u.head) one(threadIdx.x);
  char* const at = static_cast<char*>(dest) + ((u.head + u.at) << (to_bf16 ? 1 : 2));
  if (u.whole() && ((uintptr_t)at & 15) == 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      const int piece = i * THREADS + threadIdx.x;
      if (!u.half) {
        store_once(at + piece * 16, (f32x4){f(__uint_as_float(w[0])), f(__uint_as_float(w[1])), f(__uint_as_float(w[2])), f(__uint_as_float(w[3]))});
      } else if (to_bf16) {
        *reinterpret_cast<uint4*>(at + piece * 16) = make_uint4(pack_bf16x2(f(low(w[0])), f(high(w[0]))), pack_bf16x2(f(low(w[1])), f(high(w[1]))),
                                                                pack_bf16x2(f(low(w[2])), f(high(w[2]))), pack_bf16x2(f(low(w[3])), f(high(w[3]))));
      } else {
        const int first = 2 * i * THREADS + threadIdx.x;
        store_once(at + first * 16, (f32x4){f(low(w[0])), f(high(w[0])), f(low(w[1])), f(high(w[1]))});
        store_once(at + (first + THREADS) * 16, (f32x4){f(low(w[2])), f(high(w[2])), f(low(w[3])), f(high(w[3]))});
      }
    }
  } else {
    const int64_t end = min(u.at + u.values(), u.n);
    for (int64_t i = u.at + threadIdx.x; i < end; i += THREADS) one(u.head + i);
  }
}

__global__ __launch_bounds__(THREADS) void k_clip(ClipTable t) {
  __shared__ double red[THREADS / 64];
  double s = 0.0;
  double part[PARTIALS / THREADS];
#pragma unroll
  for (int i = 0; i < PARTIALS / THREADS; ++i) part[i] = i * THREADS + (int)threadIdx.x < t.partials ? t.partial[i * THREADS + threadIdx.x] : 0.0;
  int from, to;
  run_of(t.units, from, to);
  int k = 0;
  Unit u{};
  uint4 v[PER] = {};
  if (from < to) {
    k = tensor_of(t, from);
    u = unit_at(t, k, from);
    if (u.whole()) load_whole(u, t.out != nullptr && u.half, v);
  }
#pragma unroll
  for (int i = 0; i < PARTIALS / THREADS; ++i) s += part[i];
  const double norm = sqrt(block_sum64(s, red));
  const bool finite = norm <= 1.7976931348623157e308;
  const double exact = finite ? fmin(1.0, t.max_norm / (norm + 1e-6)) : 1.0;
  const float factor = (float)exact;
  const Factor scale = exact < 0x1p-100 ? Factor{0x1p-64f, (float)(exact * 0x1p64)} : Factor{1.f, factor};
  if (t.norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) {
    t.norm[0] = (float)norm; t.norm[1] = factor;
    if (t.status != nullptr) *t.status = finite ? 0 : 1;
  }
  if (t.out == nullptr && factor == 1.f) return;
  for (int unit = from; unit < to; ++unit) {
    if (unit > from) {
      while (unit >= t.first[k + 1]) ++k;
      u = unit_at(t, k, unit);
      if (u.whole()) load_whole(u, t.out != nullptr && u.half, v);
    }
    if (t.out != nullptr) scale_unit(u, v, t.out + t.to[k], false, scale);
    else scale_unit(u, v, t.p[k], u.half != 0, scale);
  }
}
}  // namespace

size_t grad_clip_bytes() { return PARTIALS * sizeof(double); }

void launch_grad_clip(hipStream_t st, const GradList& g, int64_t count, double max_norm, float* norm, float* out, int64_t* status, void* workspace) {
  // launches: the next tensors that are not empty, up to TENSORS of them and 2^30 units
  auto next = [&](int64_t& k, int64_t& flat, ClipTable& t) {
    t.count = t.units = 0;
    for (uint32_t& w : t.bf16) w = 0;
    for (; k < count && t.count < TENSORS; ++k) {
      if (g.n[k] == 0) continue;
      const bool bf16 = g.dtype[k] == SAMA_DTYPE_BF16;
      const int64_t each = bf16 ? UNIT_BYTES / 2 : UNIT_BYTES / 4, units = (g.n[k] + each - 1) / each;
      if (t.count > 0 && t.units + units > (1 << 30)) break;
      t.p[t.count] = g.p[k]; t.n[t.count] = g.n[k]; t.to[t.count] = flat; t.first[t.count] = t.units;
      if (bf16) t.bf16[t.count >> 5] |= 1u << (t.count & 31);
      flat += g.n[k]; t.units += (int)units; ++t.count;
    }
    t.first[t.count] = t.units;
  };
  ClipTable t{};
  int most = 0;
  int64_t total = 0;
  for (int64_t k = 0, flat = 0; k < count;) { next(k, flat, t); most = std::max(most, t.units); total = flat; }
  const int blocks = std::max(1, std::min(most, PARTIALS));
  t.max_norm = max_norm; t.partial = static_cast<double*>(workspace); t.partials = blocks; t.out = out;
  ProfScope ps(st, F_OTHER, 12.0 * total);
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
