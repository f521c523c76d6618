// Embedding lookup with scaling, out[i] = scale * table[id_i], and its gradient, grad[v] (+)= scale * sum over the i with id_i = v
// of dy[i].  Both move bytes: a row of the table and of the output for each token; the real rows of dy once and every row of the
// table's gradient once.
//
// The gradient sorts the tokens by id, which gives every id's rows one after the other in ascending i, and sums each run in a fixed
// order in 32 bits: the same bits from call to call, without an atomic on a sum.  Two launches.
//   k_token_sort   A workgroup owns a range of ids (V / 512 of them or so) and looks through all tokens twice, 16 waves a section of
//                  them each: it counts its ids and those below its range, turns the counts into places, and puts its tokens there, a
//                  wave 64 at a time in order (ranks among equal ids by ballots).  No workgroup waits for another.  The rows of the
//                  gradient without a token are zeroed here, while others still sort: for a vocabulary of 30522 and 4096 tokens that
//                  is most of all bytes.
//   k_token_sum    16 waves of `P` sorted rows each and a slice of the columns.  Runs inside a wave go out directly, runs over waves
//                  are joined through LDS, runs over workgroups through partial sums that the last of them to finish adds in order.
//                  A fixed number of rows to a workgroup and not of ids: texts have one token in ten the same, and padding more.
#include <algorithm>
#include "kernels.h"
#include "token_ops.h"

namespace sama {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<bf16_t>(bf16_t x) { return bf16_to_f32(x); }

// VEC neighbouring values of either type; VEC > 1: aligned to their size, at most 16 bytes of them
template <typename T, int VEC>
struct Values;
template <typename T>
struct Values<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32<T>(v); }
};
template <>
struct Values<float, 4> {
  f32x4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x4*>(p); }
  __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v[0]; f[1] = v[1]; f[2] = v[2]; f[3] = v[3]; }
};
template <>
struct Values<bf16_t, 4> {
  uint2 v;
  __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float (&f)[4]) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u); f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
};
template <>
struct Values<bf16_t, 8> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { f[2 * k] = __uint_as_float(w[k] << 16); f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u); }
  }
};
__device__ __forceinline__ void put(float* p, const float (&f)[1]) { *p = f[0]; }
__device__ __forceinline__ void put(bf16_t* p, const float (&f)[1]) { *p = f32_to_bf16(f[0]); }
__device__ __forceinline__ void put(float* p, const float (&f)[4]) { *reinterpret_cast<f32x4*>(p) = (f32x4){f[0], f[1], f[2], f[3]}; }
__device__ __forceinline__ void put(bf16_t* p, const float (&f)[4]) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])); }
__device__ __forceinline__ void put(float* p, const float (&f)[8]) {
  *reinterpret_cast<f32x4*>(p) = (f32x4){f[0], f[1], f[2], f[3]};
  *reinterpret_cast<f32x4*>(p + 4) = (f32x4){f[4], f[5], f[6], f[7]};
}
__device__ __forceinline__ void put(bf16_t* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// ---------------------------------------------------------------------------------------------------- lookup
struct LookupArgs {
  const void* table; int64_t ldt;
  const int32_t* ids; int64_t n; int V, d;
  float scale; int pad;
  void* out; int64_t ldo;
  int rows;             // of a block
  uint32_t pieces, magic;   // of a row; ceil(2^32 / pieces)
};

// A block takes `rows` rows, its threads the pieces of VEC values of all of them one after the other, U of them at a time so that
// the loads of the ids, then those of the rows, are under way together.
template <typename TI, typename TO, int VEC, int U>
__global__ __launch_bounds__(256) void k_embedding(LookupArgs a) {
  const TI* const table = static_cast<const TI*>(a.table);
  TO* const out = static_cast<TO*>(a.out);
  for (int64_t row0 = (int64_t)blockIdx.x * a.rows; row0 < a.n; row0 += (int64_t)gridDim.x * a.rows) {
  const uint32_t here = (uint32_t)min((int64_t)a.rows, a.n - row0), total = here * a.pieces;
  for (uint32_t i0 = threadIdx.x; i0 < total; i0 += 256 * U) {
    Values<TI, VEC> v[U];
    uint32_t row[U], col[U];
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = min(i0 + 256 * u, total - 1);
      row[u] = a.pieces == 1 ? i : a.rows == 1 ? 0 : (uint32_t)(((uint64_t)i * a.magic) >> 32);   // i / pieces: i pieces < 2^32
      col[u] = (i - row[u] * a.pieces) * VEC;
      id[u] = a.ids[row0 + row[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].load(table + (int64_t)min(max(id[u], 0), a.V - 1) * a.ldt + col[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 256 * u >= total) break;
      float f[VEC];
      v[u].get(f);
      const bool pad = a.pad >= 0 && id[u] == a.pad;
#pragma unroll
      for (int k = 0; k < VEC; ++k) f[k] = pad ? 0.f : f[k] * a.scale;
      put(out + (row0 + row[u]) * a.ldo + col[u], f);
    }
  }
  }
}

template <typename TI, typename TO, int VEC>
void launch_lookup(hipStream_t st, ProfScope& ps, LookupArgs a) {
  a.pieces = a.d / VEC;
  a.magic = a.pieces == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + a.pieces - 1) / a.pieces);
  // four pieces a thread where that leaves 1024 blocks and more
  const bool many = a.n * a.pieces >= (int64_t)1024 * 1024;
  a.rows = (int)std::max<int64_t>(1, (many ? 1024 : 256) / a.pieces);
  const uint32_t blocks = (uint32_t)std::min<int64_t>((a.n + a.rows - 1) / a.rows, 1 << 20);
  if (many) launch_kernel(ps, k_embedding<TI, TO, VEC, 4>, blocks, 256, 0, st, a);
  else launch_kernel(ps, k_embedding<TI, TO, VEC, 1>, blocks, 256, 0, st, a);
}
template <typename TI, typename TO>
void launch_lookup(hipStream_t st, ProfScope& ps, const LookupArgs& a) {
  constexpr int VEC = sizeof(TI) == 2 && sizeof(TO) == 2 ? 8 : 4;
  const uintptr_t at = (uintptr_t)a.table | (uintptr_t)(a.ldt * sizeof(TI)), to = (uintptr_t)a.out | (uintptr_t)(a.ldo * sizeof(TO));
  const bool wide = a.d % VEC == 0 && at % (VEC * sizeof(TI)) == 0 && to % (VEC * sizeof(TO)) == 0;
  if (wide) launch_lookup<TI, TO, VEC>(st, ps, a);
  else launch_lookup<TI, TO, 1>(st, ps, a);
}

// ---------------------------------------------------------------------------------------------------- gradient: the sort
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, SORT_RANGE = 512;   // ids of a workgroup at most
constexpr int SUM_WAVES = 16;

struct SortArgs {
  const int32_t* ids; int n, V, pad, range;
  int32_t *order, *sorted, *start;   // [n] token of each place, [n] its id, [V + 1] first place of each id
  uint32_t* tickets; int ntickets;
  void* grad; int64_t ldg; int d, elem;   // rows to zero (null: none), bytes of a value
};

__global__ __launch_bounds__(SORT_THREADS) void k_token_sort(SortArgs a) {
  extern __shared__ int32_t place[];         // [waves][range]: counts, then the next place of each id for each wave's tokens
  __shared__ int32_t s_wave[SORT_WAVES], s_below[SORT_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lo = blockIdx.x * a.range, range = min(a.range, a.V - lo);
  for (int i = blockIdx.x * SORT_THREADS + tid; i < a.ntickets; i += gridDim.x * SORT_THREADS) a.tickets[i] = 0;
  for (int i = tid; i < SORT_WAVES * range; i += SORT_THREADS) place[i] = 0;
  __syncthreads();
  const int section = ((a.n + SORT_WAVES - 1) / SORT_WAVES + 63) / 64 * 64;
  const int first = min(wave * section, a.n), last = min(first + section, a.n);   // (wave * section <= n + 15 * 64)
  int32_t* const mine = place + wave * range;
  // which of its range's ids a token has; `below`: it has a smaller one
  auto of = [&](int id, bool& below) {
    const bool real = a.pad < 0 || id != a.pad;
    id = min(max(id, 0), a.V - 1) - lo;
    below = real && id < 0;
    return real && id >= 0 && id < range ? id : -1;
  };
  int below = 0;
#pragma unroll 8
  for (int i = first + lane; i < last; i += 64) {
    bool b;
    const int id = of(a.ids[i], b);
    below += b ? 1 : 0;
    if (id >= 0) atomicAdd(mine + id, 1);
  }
  __syncthreads();
  // places: ids in order, of an id the waves in order
  int total = 0;
  if (tid < range)
    for (int w = 0; w < SORT_WAVES; ++w) total += place[w * range + tid];
  int upto = total;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const int t = __shfl_up(upto, s, 64);
    if (lane >= s) upto += t;
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) below += __shfl_xor(below, s, 64);
  if (lane == 63) s_wave[wave] = upto;
  if (lane == 0) s_below[wave] = below;
  __syncthreads();
  int at = upto - total;
  for (int w = 0; w < SORT_WAVES; ++w) at += s_below[w] + (w < wave ? s_wave[w] : 0);
  if (tid < range) {
    a.start[lo + tid] = at;
    if (lo + tid == a.V - 1) a.start[a.V] = at + total;
    for (int w = 0; w < SORT_WAVES; ++w) {
      const int c = place[w * range + tid];
      place[w * range + tid] = total > 0 ? at : -1;
      at += c;
    }
  }
  __syncthreads();
  // the rows nobody has: a wave a row, before it sorts, so that the stores drain meanwhile
  if (a.grad != nullptr) {
    const int64_t bytes = (int64_t)a.d * a.elem, ld = a.ldg * a.elem;
    const bool wide = (((uintptr_t)a.grad | (uintptr_t)ld | (uintptr_t)bytes) & 15) == 0;
    for (int r = wave; r < range; r += SORT_WAVES) {
      if (mine[r] >= 0) continue;
      char* const row = static_cast<char*>(a.grad) + (lo + r) * ld;
      if (wide) {
        for (int64_t b = lane * 16; b < bytes; b += 1024) *reinterpret_cast<uint4*>(row + b) = make_uint4(0, 0, 0, 0);
      } else {
        for (int64_t b = lane * 2; b < bytes; b += 128) *reinterpret_cast<uint16_t*>(row + b) = 0;
      }
    }
  }
  // (each wave reads and changes its own places from here on)
  const int bits = range > 1 ? 32 - __builtin_clz(range - 1) : 0;
  constexpr int AHEAD = 4;   // groups of 64 tokens whose ids are loaded before the ones at hand are placed
  int32_t next_ids[AHEAD];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) next_ids[u] = a.ids[min(i0 + 64 * u + lane, a.n - 1)];
  };
  if (first < last) fetch(first);
  for (int i0 = first; i0 < last; i0 += 64 * AHEAD) {
    int32_t ids[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ids[u] = next_ids[u];
    if (i0 + 64 * AHEAD < last) fetch(i0 + 64 * AHEAD);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + 64 * u + lane;
      bool b;
      const int id = i < last ? of(ids[u], b) : -1;
      uint64_t peers = __ballot(id >= 0);
      if (peers == 0) continue;
      for (int k = 0; k < bits; ++k) {
        const bool set = (id >> k) & 1;
        const uint64_t with = __ballot(set);
        peers &= set ? with : ~with;
      }
      if (id >= 0) {
        const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(peers >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)peers, 0)), next = mine[id];
        a.order[next + rank] = i;
        a.sorted[next + rank] = lo + id;
        if (rank == 0) mine[id] = next + __popcll(peers);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------- gradient: the sums
struct SumArgs {
  const void* dy; int64_t ldy;
  const int32_t *order, *sorted, *start; int V, d;
  float scale; int accumulate;
  void* grad; int64_t ldg;
  float* part; uint32_t* tickets;   // [chunks][head, tail][d rounded up to whole slices]; [chunks][slices]
};
__device__ __forceinline__ void publish_pair(float* p, float x, float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), ((uint64_t)__float_as_uint(y) << 32) | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <int VEC>
__device__ __forceinline__ void publish_values(float* p, const float (&f)[VEC]) {
  if constexpr (VEC == 1) __hip_atomic_store(p, f[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else
#pragma unroll
    for (int k = 0; k < VEC; k += 2) publish_pair(p + k, f[k], f[k + 1]);
}
template <int VEC>
__device__ __forceinline__ void collect_values(const float* p, float (&f)[VEC]) {
  if constexpr (VEC == 1) f[0] = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else
#pragma unroll
    for (int k = 0; k < VEC; k += 2) {
      const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p + k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      f[k] = __uint_as_float((uint32_t)v); f[k + 1] = __uint_as_float((uint32_t)(v >> 32));
    }
}

template <typename TI, typename TO, int VEC, int P>
__global__ __launch_bounds__(SUM_WAVES * 64) void k_token_sum(SumArgs a) {
  constexpr int CHUNK = SUM_WAVES * P, SLICE = 64 * VEC;
  __shared__ float s_head[SUM_WAVES][SLICE];   // a wave's part of a run that began before it
  __shared__ int s_last[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = blockIdx.x, slice = blockIdx.y, slices = gridDim.y;
  const int m = a.start[a.V], c0 = chunk * CHUNK;                   // tokens that count
  if (c0 >= m) return;
  const int c1 = min(c0 + CHUNK, m);
  const int q0 = min(c0 + wave * P, c1), nq = min(P, c1 - q0);
  const int col = slice * SLICE + lane * VEC;
  const bool have = col < a.d;                                      // (d is a multiple of VEC)
  const TI* const dy = static_cast<const TI*>(a.dy) + (have ? col : 0);
  TO* const grad = static_cast<TO*>(a.grad);
  auto finish = [&](int id, const float (&s)[VEC]) {
    if (!have) return;
    TO* const p = grad + (int64_t)id * a.ldg + col;
    float f[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] = s[k] * a.scale;
    if (a.accumulate) {
      Values<TO, (sizeof(TO) == 4 && VEC == 8) ? 4 : VEC> old;
      if constexpr (sizeof(TO) == 4 && VEC == 8) {
        float o[4];
        old.load(p); old.get(o);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] += o[k];
        old.load(p + 4); old.get(o);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[4 + k] += o[k];
      } else {
        float o[VEC];
        old.load(p); old.get(o);
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] += o[k];
      }
    }
    put(p, f);
  };
  auto head_out = [&](const float (&s)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) s_head[wave][k * 64 + lane] = s[k];
  };
  auto head_add = [&](int w, float (&s)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) s[k] += s_head[w][k * 64 + lane];
  };

  // ---- this wave's rows
  float acc[VEC] = {};
  bool own_run = false;      // the run at the wave's end began here and goes on behind it
  int tail_id = -1;
  if (nq > 0) {
    const int my = min(q0 + lane, c1 - 1);
    const int my_id = a.sorted[my], my_row = a.order[my];
    const int before = q0 > 0 ? a.sorted[q0 - 1] : -1, behind = q0 + nq < m ? a.sorted[q0 + nq] : -1;
    constexpr int B = P < 8 ? P : 8;
    int run = before;
    bool began = false;
    for (int j0 = 0; j0 < nq; j0 += B) {
      Values<TI, VEC> v[B];
#pragma unroll
      for (int j = 0; j < B; ++j) v[j].load(dy + (int64_t)__builtin_amdgcn_readlane(my_row, min(j0 + j, nq - 1)) * a.ldy);
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (j0 + j >= nq) break;
        const int id = __builtin_amdgcn_readlane(my_id, j0 + j);
        float f[VEC];
        v[j].get(f);
        if (id != run) {
          if (j0 + j > 0) {
            if (began) finish(run, acc);
            else head_out(acc);
          }
          run = id; began = true;
#pragma unroll
          for (int k = 0; k < VEC; ++k) acc[k] = f[k];
        } else {
#pragma unroll
          for (int k = 0; k < VEC; ++k) acc[k] += f[k];
        }
      }
    }
    if (!began) head_out(acc);
    else if (run == behind) { own_run = true; tail_id = run; }
    else finish(run, acc);
  }
  __syncthreads();

  // ---- runs over waves; those over workgroups leave their part
  const int64_t width = (int64_t)slices * SLICE;
  float* const parts = a.part + slice * SLICE + lane * VEC;   // of chunk c: + (2 c + which) width
  const int head_id = a.sorted[c0], last_id = a.sorted[c1 - 1];
  const int head_from = a.start[head_id], head_to = a.start[head_id + 1];
  const bool head_over = head_from < c0;                                   // the first run began in an earlier workgroup
  const int tail_from = a.start[last_id], tail_to = a.start[last_id + 1];
  const bool tail_over = tail_to > c1 && tail_from >= c0;                  // the last one begins here and goes on
  auto upto_wave = [&](int to) { return (min(to, c1) - 1 - c0) / P; };     // the wave of a run's last row here
  if (wave == 0 && head_over) {
    float s[VEC] = {};
    for (int w = 0; w <= upto_wave(head_to); ++w) head_add(w, s);
    publish_values<VEC>(parts + (2 * (int64_t)chunk) * width, s);
  }
  if (own_run) {
    const int to = a.start[tail_id + 1];
    for (int w = wave + 1; w <= upto_wave(to); ++w) head_add(w, acc);
    if (to > c1) publish_values<VEC>(parts + (2 * (int64_t)chunk + 1) * width, acc);
    else finish(tail_id, acc);
  }
  if (!head_over && !tail_over) return;                                    // the same for the workgroup
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                         // what this wave published has arrived (see last_block)
  __syncthreads();
  auto chunks_of = [&](int from, int to) { return (to - 1) / CHUNK - from / CHUNK + 1; };
  if (threadIdx.x == 0) {
    auto arrive = [&](int from, int to) {
      const uint32_t before = __hip_atomic_fetch_add(a.tickets + (int64_t)(from / CHUNK) * slices + slice, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      return before == (uint32_t)chunks_of(from, to) - 1u ? 1 : 0;
    };
    s_last[0] = head_over ? arrive(head_from, head_to) : 0;
    s_last[1] = tail_over ? arrive(tail_from, tail_to) : 0;
  }
  __syncthreads();
  const bool last[2] = {s_last[0] != 0, s_last[1] != 0};
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!last[which]) continue;
    const int id = which == 0 ? head_id : last_id, from = which == 0 ? head_from : tail_from, to = which == 0 ? head_to : tail_to;
    const int first_chunk = from / CHUNK, count = chunks_of(from, to), each = (count + SUM_WAVES - 1) / SUM_WAVES;
    float s[VEC] = {};
    const int k1 = min((wave + 1) * each, count);
    for (int k0 = wave * each; k0 < k1; k0 += 4) {
      float f[4][VEC];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = min(k0 + u, k1 - 1);
        collect_values<VEC>(parts + (2 * (int64_t)(first_chunk + k) + (k == 0 ? 1 : 0)) * width, f[u]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (k0 + u < k1) {
#pragma unroll
          for (int k = 0; k < VEC; ++k) s[k] += f[u][k];
        }
    }
    head_out(s);
    __syncthreads();
    if (wave == 0) {
      float t[VEC] = {};
      for (int w = 0; w < SUM_WAVES; ++w) head_add(w, t);
      finish(id, t);
    }
    __syncthreads();
  }
}

// Sorted rows of a wave: the most of 16 to 1 that leave the chip 256 workgroups.
int sum_rows(int64_t n, int slices) {
  int p = 16;
  while (p > 1 && (n + SUM_WAVES * p - 1) / (SUM_WAVES * p) * slices < 256) p /= 2;
  return p;
}
// What a call needs for the widest slices, and for the narrowest: pointers and strides that a call comes with decide between them.
int slices_of(int d, int vec) { return (d + 64 * vec - 1) / (64 * vec); }

struct GradPlan { int P, slices; int64_t chunks; size_t order, sorted, start, tickets, part, bytes; };
GradPlan plan_grad(int64_t n, int V, int d, int vec) {
  GradPlan g{};
  g.slices = slices_of(d, vec);
  g.P = sum_rows(n, g.slices);
  g.chunks = (n + SUM_WAVES * g.P - 1) / (SUM_WAVES * g.P);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  g.order = take((size_t)n * 4); g.sorted = take((size_t)n * 4); g.start = take(((size_t)V + 1) * 4);
  // room for the most chunks that n or fewer tokens may be cut into (sum_rows)
  const int64_t most = std::max((n + SUM_WAVES * 16 - 1) / (SUM_WAVES * 16), std::min<int64_t>((n + SUM_WAVES - 1) / SUM_WAVES, 512 / g.slices + 2));
  g.tickets = take((size_t)most * g.slices * 4);
  g.part = take((size_t)most * 2 * g.slices * 64 * vec * 4);
  g.bytes = at;
  return g;
}

template <typename TI, typename TO, int VEC>
void launch_sum(hipStream_t st, ProfScope& ps, const SumArgs& s, const GradPlan& g) {
  const dim3 grid((uint32_t)g.chunks, g.slices);
  switch (g.P) {
    case 16: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 16>, grid, SUM_WAVES * 64, 0, st, s);
    case 8: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 8>, grid, SUM_WAVES * 64, 0, st, s);
    case 4: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 4>, grid, SUM_WAVES * 64, 0, st, s);
    case 2: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 2>, grid, SUM_WAVES * 64, 0, st, s);
    default: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 1>, grid, SUM_WAVES * 64, 0, st, s);
  }
}

// Values a lane takes: 16 bytes of dy, where every row of dy and of the gradient allows it.
int grad_vec(const EmbeddingGradArgs& a) {
  const int se = a.dy_bf16 ? 2 : 4, ge = a.grad_bf16 ? 2 : 4, vec = a.dy_bf16 ? 8 : 4;
  const uintptr_t at = (uintptr_t)a.dy | (uintptr_t)(a.ldy * se), to = (uintptr_t)a.grad | (uintptr_t)(a.ldg * ge);
  return a.d % vec == 0 && at % 16 == 0 && to % std::min(16, vec * ge) == 0 ? vec : 1;
}
}  // namespace

void launch_embedding(hipStream_t st, const EmbeddingArgs& e) {
  if (e.n == 0) return;
  LookupArgs a{};
  a.table = e.table; a.ldt = e.ldt; a.ids = e.ids; a.n = e.n; a.V = e.V; a.d = e.d; a.scale = e.scale; a.pad = e.pad; a.out = e.out; a.ldo = e.ldo;
  ProfScope ps(st, F_OTHER, 0.0);
  if (e.table_bf16 && e.out_bf16) launch_lookup<bf16_t, bf16_t>(st, ps, a);
  else if (e.table_bf16) launch_lookup<bf16_t, float>(st, ps, a);
  else if (e.out_bf16) launch_lookup<float, bf16_t>(st, ps, a);
  else launch_lookup<float, float>(st, ps, a);
}

size_t embedding_grad_bytes(int64_t n, int V, int d) {
  return std::max({plan_grad(n, V, d, 8).bytes, plan_grad(n, V, d, 4).bytes, plan_grad(n, V, d, 1).bytes});
}

void launch_embedding_grad(hipStream_t st, const EmbeddingGradArgs& e, void* workspace) {
  const int vec = grad_vec(e);
  const GradPlan g = plan_grad(e.n, e.V, e.d, vec);
  char* const ws = static_cast<char*>(workspace);
  ProfScope ps(st, F_OTHER, 0.0);
  SortArgs s{};
  s.ids = e.ids; s.n = (int)e.n; s.V = e.V; s.pad = e.pad;
  // two workgroups to a CU, which sort and zero by turns
  s.range = std::min(SORT_RANGE, std::max(1, (e.V + 511) / 512));
  s.order = (int32_t*)(ws + g.order); s.sorted = (int32_t*)(ws + g.sorted); s.start = (int32_t*)(ws + g.start);
  s.tickets = (uint32_t*)(ws + g.tickets); s.ntickets = (int)(g.chunks * g.slices);
  s.grad = e.accumulate ? nullptr : e.grad; s.ldg = e.ldg; s.d = e.d; s.elem = e.grad_bf16 ? 2 : 4;
  launch_kernel(ps, k_token_sort, (e.V + s.range - 1) / s.range, SORT_THREADS, SORT_WAVES * s.range * 4, st, s);
  if (e.n == 0) return;
  SumArgs a{};
  a.dy = e.dy; a.ldy = e.ldy; a.order = s.order; a.sorted = s.sorted; a.start = s.start; a.V = e.V; a.d = e.d; a.scale = e.scale;
  a.accumulate = e.accumulate; a.grad = e.grad; a.ldg = e.ldg; a.part = (float*)(ws + g.part); a.tickets = s.tickets;
  auto go = [&](auto ti, auto to, auto wide) {
    typedef decltype(ti) TI;
    typedef decltype(to) TO;
    if (vec > 1) launch_sum<TI, TO, decltype(wide)::value>(st, ps, a, g);
    else launch_sum<TI, TO, 1>(st, ps, a, g);
  };
  const std::integral_constant<int, 8> eight;
  const std::integral_constant<int, 4> four;
  if (e.dy_bf16 && e.grad_bf16) go(bf16_t{}, bf16_t{}, eight);
  else if (e.dy_bf16) go(bf16_t{}, float{}, eight);
  else if (e.grad_bf16) go(float{}, bf16_t{}, four);
  else go(float{}, float{}, four);
}

}  // namespace sama
