// Embedding lookup with scaling, out[i] = scale * table[id_i], and its gradient, grad[v] (+)= scale * sum over the i with id_i = v
// of dy[i].  Both move bytes: a row of the table and of the output for each token; the real rows of dy once and every row of the
// table's gradient once.
//
// Measured on an MI355X: the lookup beside its kernel; the gradient of 4096 tokens of 768 into 30522 rows of fp32 23.7 us for 106 MB (94 MB of them written: 13.5
// us by themselves), of 65521 tokens of 1024 in bf16, a quarter padding, into 50304 rows 78 us for 307 MB; of 703 tokens of 256 into 8192 rows 6.2 us.
//
// The gradient sorts the tokens by id, which gives every id's rows one after the other in ascending i, and sums each run in a fixed
// order in 32 bits: the same bits from call to call, without an atomic on a sum.  Two launches, and for a few tokens one (k_token_few).
//   k_token_sort   A workgroup owns every 256th id and looks through all tokens, 16 waves a section of them each: it counts its ids and
//                  those of the workgroups before it, turns the counts into places, and puts its tokens there, a wave 64 at a time in order
//                  (ranks among equal ids by ballots).  Every 256th and not 256th parts of the table: the low ids are the frequent ones of
//                  most vocabularies, and one workgroup had half of the tokens.  No workgroup waits for another.
//                  Beside each a second one zeroes a share of the gradient: for a vocabulary of 30522 and 4096 tokens that is most of all
//                  bytes, and sorting hides behind it.  Zeroing only the rows that stay so, in the launch behind this one, moves a fifth
//                  less and takes longer; so does leaving just those there that do not hide behind the sort (30 us instead of 24 for the first
//                  of the above, 78 to 91 instead of 78 for the second).
//   k_token_sum    8 waves of `P` sorted rows each and a slice of the columns.  Runs inside a wave go out directly, runs over waves
//                  are joined through LDS, runs over workgroups through partial sums that the last of them to finish adds in order.
//                  A fixed number of rows to a workgroup and not of ids: texts have one token in ten the same, and padding more.
#include <algorithm>
#include <type_traits>
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

// What passes through the caches once: rows of dy, each read by one workgroup, and the rows that are summed, which go out among the zeroed rows still on their
// way.  us for 65521 tokens of 1024 into 50304 rows, 4096 of 768 into 30522: kept 88.0, 27.2, these stores 83.3, 25.5, the loads as well 78.0, 25.7,
// the zeroing as well 77.0, 27.8.
template <typename T, int VEC>
__device__ __forceinline__ Values<T, VEC> load_once(const T* p) {
  Values<T, VEC> v;
  if constexpr (VEC * sizeof(T) == 16) {
    typedef decltype(v.v) V;
    v.v = __builtin_bit_cast(V, __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)));
  } else {
    v.load(p);
  }
  return v;
}
template <int VEC>
__device__ __forceinline__ void put_once(bf16_t* p, const float (&f)[VEC]) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  if constexpr (VEC == 8) __builtin_nontemporal_store((u4){pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])}, reinterpret_cast<u4*>(p));
  else if constexpr (VEC == 4) __builtin_nontemporal_store((u2){pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])}, reinterpret_cast<u2*>(p));
  else put(p, f);
}
template <int VEC>
__device__ __forceinline__ void put_once(float* p, const float (&f)[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int k = 0; k < VEC; k += 4) __builtin_nontemporal_store((f32x4){f[k], f[k + 1], f[k + 2], f[k + 3]}, reinterpret_cast<f32x4*>(p + k));
  } else {
    put(p, f);
  }
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
// the loads of the ids, then those of the rows, are under way together.  Bound by memory: 32768 tokens of 1024, a quarter of them padding, from an fp32 table
// into bf16 in 21.0 us, 90 MB of distinct rows and output (4.3 TB/s; 168 MB with what the caches answer); 128 tokens of 256 in 5.2, which is the call: the
// kernel takes 2.4.
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
  // four pieces a thread where that leaves 1024 blocks and more, else one (the first of the above 25.5 us with one, the second the same with either)
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
  // rows in pieces of 16 bytes (of the fp32 side) where both sides allow it: 32768 x 1024, ids evenly spread, 30.3 us, a value at a time 44.1
  const bool wide = a.d % VEC == 0 && at % (VEC * sizeof(TI)) == 0 && to % (VEC * sizeof(TO)) == 0;
  if (wide) launch_lookup<TI, TO, VEC>(st, ps, a);
  else launch_lookup<TI, TO, 1>(st, ps, a);
}

// ---------------------------------------------------------------------------------------------------- gradient: the sort
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, SORT_RANGE = 512;   // ids of a workgroup at most
constexpr int SUM_WAVES = 8;
// The order of the ids: id mod 2^lg, then id / 2^lg, of which there are up to `range`.
struct IdOrder {
  int lg, range;
  __host__ __device__ __forceinline__ int groups() const { return 1 << lg; }
  __host__ __device__ __forceinline__ int64_t places() const { return (int64_t)groups() * range; }
  __host__ __device__ __forceinline__ int64_t place(int id) const { return (int64_t)(id & (groups() - 1)) * range + (id >> lg); }
};
IdOrder order_of(int V) {
  IdOrder o{8, 0};   // a workgroup to a CU
  while (((V - 1) >> o.lg) + 1 > SORT_RANGE) ++o.lg;
  o.range = ((V - 1) >> o.lg) + 1;
  return o;
}

// lanes of the set below this one, + from
__device__ __forceinline__ int rank_in(uint64_t lanes, int from) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, from));
}
// the lanes of `among` that have this lane's id, of `bits` bits: of the first few ids that there are one by one, then by a ballot for each bit
__device__ __forceinline__ uint64_t lanes_with(int id, uint64_t among, int bits) {
  uint64_t same = 0, left = among;
#pragma unroll 1
  for (int k = 0; k < 4 && left != 0; ++k) {
    const int v = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
    const uint64_t with = __ballot(id == v) & left;
    if (id == v) same = with;
    left &= ~with;
  }
  if (left == 0) return same;
  uint64_t rest = left;
  for (int k = 0; k < bits; ++k) {
    const bool set = (id >> k) & 1;
    const uint64_t with = __ballot(set);
    rest &= set ? with : ~with;
  }
  return left >> (threadIdx.x & 63) & 1 ? rest : same;
}
typedef int i4 __attribute__((ext_vector_type(4), aligned(4)));   // a load of 16 bytes wants no more than a word's alignment

struct SortArgs {
  const int32_t* ids; int n, V, pad;
  IdOrder o;
  int32_t *order, *sorted, *start;   // [n] token of each place, [n] its id, [groups range + 1] first place of each id in the order of the ids
  uint32_t* tickets; int ntickets;
  char* grad; int64_t row, ld, rows; int fills;   // bytes of a row of the gradient and from one to the next; workgroups that zero them
};

// Zeroes a share of the gradient's rows, all of them: which have no token is not known yet.
__device__ __forceinline__ void zero_share(const SortArgs& a, int share) {
  const int tid = threadIdx.x;
  const bool dense = a.row == a.ld, wide = (((uintptr_t)a.grad | (uintptr_t)a.ld | (uintptr_t)a.row) & 15) == 0;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  if (dense && wide) {
    const int64_t pieces = a.rows * (a.row / 16), each = (pieces + a.fills - 1) / a.fills;
    const int64_t from = share * each, to = min(from + each, pieces);
    for (int64_t i = from + tid; i < to; i += SORT_THREADS) *reinterpret_cast<f32x4*>(a.grad + i * 16) = zero;
    return;
  }
  for (int64_t r = (int64_t)share * SORT_WAVES + (tid >> 6); r < a.rows; r += (int64_t)a.fills * SORT_WAVES) {
    char* const row = a.grad + r * a.ld;
    if (wide) {
      for (int64_t b = (tid & 63) * 16; b < a.row; b += 1024) *reinterpret_cast<f32x4*>(row + b) = zero;
    } else {
      for (int64_t b = (tid & 63) * 2; b < a.row; b += 128) *reinterpret_cast<uint16_t*>(row + b) = 0;
    }
  }
}

// A wave's tokens are read once: those of the workgroup's ids go, in order, into a list in LDS of LIST places.  A wave that has more of them (of an id
// that half a batch consists of) reads its tokens again instead.  Looking through the ids is bound by instructions, each of the 256 workgroups
// looks at all of them: six vector instructions for 64, the rest is on masks in scalar registers.
constexpr int LIST = 1024, GROUP = 256, LIST_BITS = 23;   // tokens a wave takes at a time, four neighbours a lane; bits of a token's number in its section
static_assert(SORT_RANGE <= 1 << (32 - LIST_BITS), "the list has the id above them");
__global__ __launch_bounds__(SORT_THREADS) void k_token_sort(SortArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint32_t s_list[];   // [waves][LIST]: token of the section, id
  int32_t* const place = reinterpret_cast<int32_t*>(s_list + SORT_WAVES * LIST);   // [waves][range]: counts, then the next place of each id for each wave's tokens
  __shared__ int32_t s_wave[SORT_WAVES], s_below[SORT_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blockIdx.x >= (uint32_t)a.o.groups()) return zero_share(a, blockIdx.x - a.o.groups());
  const int own = blockIdx.x, range = a.o.range, mask = a.o.groups() - 1, lg = a.o.lg, most = a.V - 1, n = a.n;
  const int pad = a.pad >= 0 ? a.pad : INT32_MIN;                  // (ids below zero are taken as -1: none is that)
  for (int i = blockIdx.x * SORT_THREADS + tid; i < a.ntickets; i += a.o.groups() * SORT_THREADS) a.tickets[i] = 0;
  int32_t* const mine = place + wave * range;
  for (int i = lane; i < range; i += 64) mine[i] = 0;
  // an odd number of KB: sections 16 KB apart would begin in one channel of the L2, and all workgroups read the same at the same time
  const int section = (((n + SORT_WAVES - 1) / SORT_WAVES + GROUP - 1) / GROUP | 1) * GROUP;
  const int first = (int)min((int64_t)wave * section, (int64_t)n), last = (int)min((int64_t)first + section, (int64_t)n);
  const int bits = range > 1 ? 32 - __builtin_clz(range - 1) : 0;
  auto clamped = [&](int id) { return min(max(id, 0), most); };
  const int room = section <= 1 << LIST_BITS ? LIST : 0;
  int below = 0, listed = 0;                 // tokens of workgroups before this one, of this one: the same in every lane
  auto look = [&](int i0, i4 now, auto whole) {
    const int t[4] = {max(now[0], -1), max(now[1], -1), max(now[2], -1), max(now[3], -1)};
    bool here[4];
    uint64_t have[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int g = clamped(t[e]) & mask;
      const bool counts = t[e] != pad && (decltype(whole)::value || i0 + 4 * lane + e < last);
      here[e] = counts && g == own;
      have[e] = __ballot(here[e]);
      below += __popcll(__ballot(counts && g < own));
    }
    if ((have[0] | have[1] | have[2] | have[3]) == 0) return;
    int at = listed;
#pragma unroll
    for (int e = 0; e < 4; ++e) at = rank_in(have[e], at);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (here[e]) {   // (a list that is too short is not used)
        s_list[wave * LIST + min(at, LIST - 1)] = (uint32_t)(i0 - first + 4 * lane + e) | (uint32_t)(clamped(t[e]) >> lg) << LIST_BITS;
        ++at;
      }
      listed += __popcll(have[e]);
    }
  };
  constexpr int AHEAD = 4;
  const int groups = (last - first) / GROUP;   // whole ones
  const int32_t* const ids = a.ids + first + 4 * lane;
  i4 next[AHEAD] = {};
  auto fetch = [&](int g) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) if (g + u < groups) next[u] = *reinterpret_cast<const i4*>(ids + (int64_t)(g + u) * GROUP);
  };
  fetch(0);
  for (int g = 0; g < groups; g += AHEAD) {
    i4 now[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) now[u] = next[u];
    fetch(g + AHEAD);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) if (g + u < groups) look(first + (g + u) * GROUP, now[u], std::true_type{});
  }
  if (first + groups * GROUP < last) {
    const int i = first + groups * GROUP + 4 * lane;
    look(first + groups * GROUP, (i4){a.ids[min(i, n - 1)], a.ids[min(i + 1, n - 1)], a.ids[min(i + 2, n - 1)], a.ids[min(i + 3, n - 1)]}, std::false_type{});
  }
  // f(id or -1, token) for this wave's tokens of the workgroup's ids, 64 in order at a time
  auto each = [&](auto f) {
    if (listed <= room) {
      for (int k0 = 0; k0 < listed; k0 += 64) {
        const uint32_t v = s_list[wave * LIST + min(k0 + lane, LIST - 1)];
        f(k0 + lane < listed ? (int)(v >> LIST_BITS) : -1, first + (int)(v & ((1u << LIST_BITS) - 1)));
      }
      return;
    }
    constexpr int DEEP = 8;
    int32_t ahead[DEEP];
    auto load = [&](int i0) {
#pragma unroll
      for (int u = 0; u < DEEP; ++u) ahead[u] = a.ids[min(i0 + 64 * u + lane, n - 1)];
    };
    load(first);
    for (int i0 = first; i0 < last; i0 += 64 * DEEP) {
      int32_t ids[DEEP];
#pragma unroll
      for (int u = 0; u < DEEP; ++u) ids[u] = ahead[u];
      if (i0 + 64 * DEEP < last) load(i0 + 64 * DEEP);
#pragma unroll
      for (int u = 0; u < DEEP; ++u) {
        const int i = i0 + 64 * u + lane, id = clamped(ids[u]);
        f(i < last && (id & mask) == own && max(ids[u], -1) != pad ? id >> lg : -1, i);
      }
    }
  };
  each([&](int id, int) {
    uint64_t some = __ballot(id >= 0);
    if (some == 0) return;
    some = lanes_with(id, some, bits);
    if (id >= 0 && rank_in(some, 0) == 0) mine[id] += __popcll(some);   // the first of each id: no two lanes at one place
  });
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
  if (lane == 63) s_wave[wave] = upto;
  if (lane == 0) s_below[wave] = below;
  __syncthreads();
  int at = upto - total;
  for (int w = 0; w < SORT_WAVES; ++w) at += s_below[w] + (w < wave ? s_wave[w] : 0);
  if (tid < range) {
    a.start[(int64_t)own * range + tid] = at;
    if (own == mask && tid == range - 1) a.start[a.o.places()] = at + total;
    for (int w = 0; w < SORT_WAVES; ++w) {
      const int c = place[w * range + tid];
      place[w * range + tid] = at;
      at += c;
    }
  }
  __syncthreads();
  each([&](int id, int token) {   // (each wave reads and changes its own places)
    uint64_t peers = __ballot(id >= 0);
    if (peers == 0) return;
    peers = lanes_with(id, peers, bits);
    if (id >= 0) {
      const int rank = rank_in(peers, 0), to = mine[id];
      a.order[to + rank] = token;
      a.sorted[to + rank] = (id << lg) + own;
      if (rank == 0) mine[id] = to + __popcll(peers);
    }
  });
}

// ---------------------------------------------------------------------------------------------------- gradient: the sums
struct SumArgs {
  const void* dy; int64_t ldy;
  const int32_t *order, *sorted, *start; int n, d;
  IdOrder o;
  float scale; int accumulate;
  void* grad; int64_t ldg;
  int slices;                       // of the columns
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

template <typename TO, int VEC>
__device__ __forceinline__ void put_sum(TO* p, const float (&s)[VEC], float scale, int accumulate) {
  float f[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) f[k] = s[k] * scale;
  if (accumulate) {
    constexpr int STEP = sizeof(TO) == 4 && VEC == 8 ? 4 : VEC;
#pragma unroll
    for (int k0 = 0; k0 < VEC; k0 += STEP) {
      Values<TO, STEP> old;
      float o[STEP];
      old.load(p + k0); old.get(o);
#pragma unroll
      for (int k = 0; k < STEP; ++k) f[k0 + k] += o[k];
    }
  }
  put_once(p, f);
}

template <typename TI, typename TO, int VEC, int P>
__global__ __launch_bounds__(SUM_WAVES * 64) void k_token_sum(SumArgs a) {
  constexpr int CHUNK = SUM_WAVES * P, SLICE = 64 * VEC;
  __shared__ float s_head[SUM_WAVES][SLICE];   // a wave's part of a run that began before it
  __shared__ int s_last[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slices = a.slices, chunk = blockIdx.x / slices, slice = blockIdx.x - chunk * slices;
  // what is read first does not wait for the number of tokens that count (what lies behind them is not used)
  const int c0 = chunk * CHUNK, q = c0 + wave * P;
  const int my_id = a.sorted[min(q + lane, a.n - 1)], my_row = a.order[min(q + lane, a.n - 1)];
  const int around = a.sorted[lane == 0 ? max(min(q, a.n) - 1, 0) : min(q + P, a.n - 1)], head_id = a.sorted[c0];
  const int m = a.start[a.o.places()];
  if (c0 >= m) return;
  const int c1 = min(c0 + CHUNK, m);
  const int q0 = min(q, c1), nq = min(P, c1 - q0);
  const int last_id = a.sorted[c1 - 1];
  const int *const head_at = a.start + a.o.place(head_id), *const tail_at = a.start + a.o.place(last_id);
  const int head_from = head_at[0], head_to = head_at[1], tail_from = tail_at[0], tail_to = tail_at[1];
  const int col = slice * SLICE + lane * VEC;
  const bool have = col < a.d;                                      // (d is a multiple of VEC)
  const TI* const dy = static_cast<const TI*>(a.dy) + (have ? col : 0);
  TO* const grad = static_cast<TO*>(a.grad);
  auto finish = [&](int id, const float (&s)[VEC]) {
    if (have) put_sum(grad + (int64_t)id * a.ldg + col, s, a.scale, a.accumulate);
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
    const int before = q0 > 0 ? __builtin_amdgcn_readlane(around, 0) : -1, behind = q0 + nq < m ? __builtin_amdgcn_readlane(around, 1) : -1;
    constexpr int B = P < 8 ? P : 8;
    int run = before;
    bool began = false;
    for (int j0 = 0; j0 < nq; j0 += B) {
      Values<TI, VEC> v[B];
#pragma unroll
      for (int j = 0; j < B; ++j) v[j] = load_once<TI, VEC>(dy + (int64_t)__builtin_amdgcn_readlane(my_row, min(j0 + j, nq - 1)) * a.ldy);
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
  const bool head_over = head_from < c0;                                   // the first run began in an earlier workgroup
  const bool tail_over = tail_to > c1 && tail_from >= c0;                  // the last one begins here and goes on
  auto upto_wave = [&](int to) { return (min(to, c1) - 1 - c0) / P; };     // the wave of a run's last row here
  if (wave == 0 && head_over) {
    float s[VEC] = {};
    for (int w = 0; w <= upto_wave(head_to); ++w) head_add(w, s);
    publish_values<VEC>(parts + (2 * (int64_t)chunk) * width, s);
  }
  if (own_run) {
    const int to = a.start[a.o.place(tail_id) + 1];
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

// ---------------------------------------------------------------------------------------------------- gradient: few tokens in one launch
// A workgroup owns every 256th id and a slice of the columns: it looks through all ids, lists its tokens in order, sorts them by id in LDS, sums
// the runs, a wave an equal share of the sorted rows, and zeroes its other rows meanwhile.  Nobody waits for another workgroup, nothing passes through
// memory.  What bounds it is one launch and the id with the most tokens, whose rows one CU reads at 45 GB/s, while the two launches above spread them over
// the chip but cost one more and the way through memory between them.  us, two launches / this one, ids by Zipf's law of exponent 1.1 (the most frequent 13 %):
//   tokens            64           256          703          1024
//   8192 x 256     9.6 / 5.5                 10.8 / 6.2
//   8192 x 512    10.3 / 6.1   11.2 / 6.5    11.7 / 9.4   11.9 / 11.4
//   2000 x 768     9.0 / 6.5   10.2 / 6.8    10.4 / 7.4   10.9 / 7.8
//   8192 x 1024   12.2 / 10.5  13.1 / 11.1   13.7 / 12.4  14.4 / 14.5
//   30522 x 512   15.4 / 12.7  16.1 / 15.0   16.7 / 16.7  16.7 / 18.7
// 703 tokens of 8192 x 256, half of them of one id: 10.9 / 10.5, all: 12.5 / 19.5.  So: up to 1024 tokens, up to 32 MB of gradient to be written (a workgroup's
// rows are 256 apart: zeroing more than that takes longer than in the sort's own share), up to four slices.
constexpr int FEW_TOKENS = 1024, FEW_WAVES = FEW_TOKENS / 64, FEW_BITS = 16, FEW_SLICES = 4;   // a thread looks at one id; bits of a token in the list
constexpr int64_t FEW_BYTES = 32 << 20;
struct FewArgs {
  const void* dy; int64_t ldy;
  const int32_t* ids; int n, V, d, pad, bits, slices;   // bits of id / 256
  float scale; int accumulate;
  void* grad; int64_t ldg;
};
template <typename TI, typename TO, int VEC>
__global__ __launch_bounds__(FEW_WAVES * 64) void k_token_few(FewArgs a) {
  constexpr int GROUPS = 256, SLICE = 64 * VEC, HEADS = FEW_WAVES * SLICE;
  __shared__ __attribute__((aligned(16))) uint32_t s_work[HEADS > FEW_TOKENS ? HEADS : FEW_TOKENS];   // the list, later the waves' parts of runs that began before them
  __shared__ uint32_t s_sorted[FEW_TOKENS];
  __shared__ __attribute__((aligned(16))) int32_t s_count[SORT_RANGE], s_to[SORT_RANGE];              // of each id: its tokens, where they go (in the end: where they end)
  __shared__ int32_t s_wave[FEW_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int own = blockIdx.x / a.slices, slice = blockIdx.x - own * a.slices;
  const int pad = a.pad >= 0 ? a.pad : INT32_MIN, most = a.V - 1, n = a.n;
  const int t = tid < n ? a.ids[tid] : 0;
  if (tid < SORT_RANGE) s_count[tid] = 0;
  __syncthreads();
  // ---- this workgroup's tokens, in order (the atomics are on counts)
  const int clamped = min(max(t, 0), most), local = clamped >> 8;
  const bool here = tid < n && max(t, -1) != pad && (clamped & (GROUPS - 1)) == own;
  const uint64_t tokens = __ballot(here);
  if (here) atomicAdd(&s_count[local], 1);
  if (lane == 0) s_wave[wave] = __popcll(tokens);
  __syncthreads();
  int m = 0, before_me = 0;
#pragma unroll
  for (int w = 0; w < FEW_WAVES; ++w) {
    if (w < wave) before_me += s_wave[w];
    m += s_wave[w];
  }
  if (here) s_work[rank_in(tokens, before_me)] = (uint32_t)tid | (uint32_t)local << FEW_BITS;
  __syncthreads();
  const int col = slice * SLICE + lane * VEC;
  const bool have = col < a.d;                                      // (d is a multiple of VEC)
  TO* const grad = static_cast<TO*>(a.grad) + (int64_t)own * a.ldg + (have ? col : 0);
  const int64_t next = (int64_t)GROUPS * a.ldg;
  // ---- one wave sorts them, the others zero the rows of the ids that have none
  if (wave == 0) {
    static_assert(SORT_RANGE == 64 * 8, "ids of a lane");
    int c[8], sum = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) { c[k] = s_count[8 * lane + k]; sum += c[k]; }
    int upto = sum;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int v = __shfl_up(upto, s, 64);
      if (lane >= s) upto += v;
    }
    upto -= sum;
#pragma unroll
    for (int k = 0; k < 8; ++k) { s_to[8 * lane + k] = upto; upto += c[k]; }
    for (int k0 = 0; k0 < m; k0 += 64) {
      const bool there = k0 + lane < m;
      const uint32_t v = there ? s_work[k0 + lane] : 0;
      const int id = there ? (int)(v >> FEW_BITS) : -1;
      const uint64_t same = lanes_with(id, __ballot(there), a.bits);
      if (there) {
        const int rank = rank_in(same, 0), to = s_to[id];
        s_sorted[to + rank] = v;
        if (rank == 0) s_to[id] = to + __popcll(same);
      }
    }
  } else if (!a.accumulate && have) {
    const int rows = own > most ? 0 : (most - own) / GROUPS + 1;
    const float zero[VEC] = {};
    for (int r = wave - 1; r < rows; r += FEW_WAVES - 1)
      if (s_count[r] == 0) put(grad + r * next, zero);
  }
  __syncthreads();
  // ---- the sums
  const int P = (m + FEW_WAVES - 1) / FEW_WAVES, q0 = min(wave * P, m), q1 = min(q0 + P, m);
  float* const s_head = reinterpret_cast<float*>(s_work);
  const TI* const dy = static_cast<const TI*>(a.dy) + (have ? col : 0);
  auto head_out = [&](const float (&s)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) s_head[wave * SLICE + k * 64 + lane] = s[k];
  };
  auto finish = [&](int id, const float (&s)[VEC]) {
    if (have) put_sum(grad + id * next, s, a.scale, a.accumulate);
  };
  float acc[VEC] = {};
  int open = -1;             // the run at the wave's end began here and goes on behind it
  if (q0 < q1) {
    const int before = q0 > 0 ? (int)(__builtin_amdgcn_readfirstlane(s_sorted[q0 - 1]) >> FEW_BITS) : -1;
    const int behind = q1 < m ? (int)(__builtin_amdgcn_readfirstlane(s_sorted[q1]) >> FEW_BITS) : -1;
    constexpr int B = 8;
    int run = before;
    bool began = false;
    for (int j0 = q0; j0 < q1; j0 += B) {
      const uint32_t mine = s_sorted[min(j0 + (lane & (B - 1)), q1 - 1)];
      Values<TI, VEC> v[B];
#pragma unroll
      for (int j = 0; j < B; ++j)
        if (j == 0 || j0 + j < q1) v[j] = load_once<TI, VEC>(dy + (int64_t)(__builtin_amdgcn_readlane(mine, j) & ((1u << FEW_BITS) - 1)) * a.ldy);
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (j0 + j >= q1) break;
        const int id = (int)((uint32_t)__builtin_amdgcn_readlane(mine, j) >> FEW_BITS);
        float f[VEC];
        v[j].get(f);
        if (id != run) {
          if (j0 + j > q0) {
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
    else if (run == behind) open = run;
    else finish(run, acc);
  }
  __syncthreads();
  if (open >= 0) {
    const int last = (s_to[open] - 1) / P;
    for (int w = wave + 1; w <= last; ++w)
#pragma unroll
      for (int k = 0; k < VEC; ++k) acc[k] += s_head[w * SLICE + k * 64 + lane];
    finish(open, acc);
  }
}

// Sorted rows of a wave: the most of 16 to 1 that leave the chip 512 workgroups.  4096 tokens of 768 into 30522 rows 23.7 us, with 256 workgroups 23.6, with
// 1024 26.8; 65521 of 1024 the same with all.
int sum_rows(int64_t n, int slices) {
  int p = 16;
  while (p > 1 && (n + SUM_WAVES * p - 1) / (SUM_WAVES * p) * slices < 512) p /= 2;
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
  g.order = take((size_t)n * 4); g.sorted = take((size_t)n * 4); g.start = take(((size_t)order_of(V).places() + 1) * 4);
  // room for the most chunks that n or fewer tokens may be cut into (sum_rows)
  const int64_t most = std::max((n + SUM_WAVES * 16 - 1) / (SUM_WAVES * 16), std::min<int64_t>((n + SUM_WAVES - 1) / SUM_WAVES, 1024 / g.slices + 2));
  g.tickets = take((size_t)most * g.slices * 4);
  g.part = take((size_t)most * 2 * g.slices * 64 * vec * 4);
  g.bytes = at;
  return g;
}

template <typename TI, typename TO, int VEC>
void launch_sum(hipStream_t st, ProfScope& ps, const SumArgs& s, const GradPlan& g) {
  const uint32_t grid = (uint32_t)(g.chunks * g.slices);
  switch (g.P) {
    case 16: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 16>, grid, SUM_WAVES * 64, 0, st, s);
    case 8: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 8>, grid, SUM_WAVES * 64, 0, st, s);
    case 4: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 4>, grid, SUM_WAVES * 64, 0, st, s);
    case 2: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 2>, grid, SUM_WAVES * 64, 0, st, s);
    default: return launch_kernel(ps, k_token_sum<TI, TO, VEC, 1>, grid, SUM_WAVES * 64, 0, st, s);
  }
}

template <typename TI, typename TO>
void launch_few(hipStream_t st, ProfScope& ps, const FewArgs& a, int vec) {
  constexpr int VEC = sizeof(TI) == 2 ? 8 : 4;
  if (vec > 1) launch_kernel(ps, k_token_few<TI, TO, VEC>, 256 * slices_of(a.d, VEC), FEW_WAVES * 64, 0, st, a);
  else launch_kernel(ps, k_token_few<TI, TO, 1>, 256 * slices_of(a.d, 1), FEW_WAVES * 64, 0, st, a);
}

// Values a lane takes: 16 bytes of dy, where every row of dy and of the gradient allows it: 4096 tokens of 768, ids evenly spread, into 30522 rows 23.6 us, a
// value at a time 25.8.
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

bool embedding_grad_fits(const EmbeddingGradArgs& e) {
  const GradPlan g = plan_grad(e.n, e.V, e.d, grad_vec(e));
  return e.V <= (1 << 30) && g.chunks * g.slices < ((int64_t)1 << 32) / (SUM_WAVES * 64);
}

void launch_embedding_grad(hipStream_t st, const EmbeddingGradArgs& e, void* workspace) {
  const int vec = grad_vec(e);
  const GradPlan g = plan_grad(e.n, e.V, e.d, vec);
  char* const ws = static_cast<char*>(workspace);
  ProfScope ps(st, F_OTHER, 0.0);
  if (e.n <= FEW_TOKENS && order_of(e.V).lg == 8 && g.slices <= FEW_SLICES && (e.accumulate || e.V * (int64_t)e.d * (e.grad_bf16 ? 2 : 4) <= FEW_BYTES)) {
    FewArgs a{};
    a.dy = e.dy; a.ldy = e.ldy; a.ids = e.ids; a.n = (int)e.n; a.V = e.V; a.d = e.d; a.pad = e.pad;
    while (order_of(e.V).range > 1 << a.bits) ++a.bits;
    a.slices = g.slices;
    a.scale = e.scale; a.accumulate = e.accumulate; a.grad = e.grad; a.ldg = e.ldg;
    if (e.dy_bf16 && e.grad_bf16) launch_few<bf16_t, bf16_t>(st, ps, a, vec);
    else if (e.dy_bf16) launch_few<bf16_t, float>(st, ps, a, vec);
    else if (e.grad_bf16) launch_few<float, bf16_t>(st, ps, a, vec);
    else launch_few<float, float>(st, ps, a, vec);
    return;
  }
  SortArgs s{};
  s.ids = e.ids; s.n = (int)e.n; s.V = e.V; s.pad = e.pad;
  s.o = order_of(e.V);
  s.grad = (char*)e.grad; s.row = (int64_t)e.d * (e.grad_bf16 ? 2 : 4); s.ld = e.ldg * (e.grad_bf16 ? 2 : 4); s.rows = e.V;
  s.fills = e.accumulate ? 0 : 256;
  s.order = (int32_t*)(ws + g.order); s.sorted = (int32_t*)(ws + g.sorted); s.start = (int32_t*)(ws + g.start);
  s.tickets = (uint32_t*)(ws + g.tickets); s.ntickets = (int)(g.chunks * g.slices);
  static bool configured = false;   // more than 64 KB of LDS with the largest ranges
  if (!configured) {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_token_sort), hipFuncAttributeMaxDynamicSharedMemorySize, SORT_WAVES * (SORT_RANGE + LIST) * 4);
    configured = true;
  }
  launch_kernel(ps, k_token_sort, s.o.groups() + s.fills, SORT_THREADS, SORT_WAVES * (s.o.range + LIST) * 4, st, s);
  if (e.n == 0) return;
  SumArgs a{};
  a.slices = g.slices;
  a.dy = e.dy; a.ldy = e.ldy; a.order = s.order; a.sorted = s.sorted; a.start = s.start; a.n = s.n; a.o = s.o; a.d = e.d; a.scale = e.scale;
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
