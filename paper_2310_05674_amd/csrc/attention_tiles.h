// What the attention kernels (attention.hip, attention_grad.hip) have in common: fragments of 32 rows by 16 of the contraction, tiles of rows in LDS and their
// loads, the scores' transformation, and products that keep what is not finite out of results that do not see it.
//
// All three products of a pass run on 32x32 matrix instructions, 32x32x16 in bf16 and eight of 32x32x2 in fp32, with a lane holding eight of a row's sixteen
// contraction indices: lane l, row l % 32, h = l / 32, indices 8 h + t.  The result has column l % 32 and, in register r, row 8 (r / 4) + 4 h + r % 4.  Scores are
// computed transposed (rows: the tile in LDS, columns: what a wave keeps in registers), so a lane holds scores of one row of its own, its softmax needs one exchange
// between two lanes, and eight neighbouring registers are already a fragment of the second product, if its contraction is taken in the order
// (h, t) -> 8 (t / 4) + 4 h + t % 4, which the other operand's transposed fetch follows.
#pragma once
#include <limits>
#include <type_traits>
#include "kernels.h"
#include "sequence_ops.h"

namespace sama {
namespace attn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef const __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef const __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef const __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) void lds_void;
constexpr int LDS_MAX = 160 * 1024;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr float INF = std::numeric_limits<float>::infinity();

template <typename E> using Frag = std::conditional_t<sizeof(E) == 2, bf16x8, f32x8>;
__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x16 zeros() { return (f32x16){0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}; }
// registers 8 half .. of a result as a fragment; in bf16 this is where probabilities and score gradients are rounded, once, because the products run on bf16 operands
template <typename E> __device__ __forceinline__ Frag<E> fragment(const f32x16& x, int half) {
  if constexpr (sizeof(E) == 2) {
    union { bf16x8 v; uint32_t w[4]; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u.w[i] = pack_bf16x2(x[8 * half + 2 * i], x[8 * half + 2 * i + 1]);
    return u.v;
  } else {
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[8 * half + i];
    return v;
  }
}
template <typename E> __device__ __forceinline__ Frag<E> zero_fragment() {
  if constexpr (sizeof(E) == 2) return __builtin_bit_cast(bf16x8, (u32x4){0, 0, 0, 0});
  else return (f32x8){0, 0, 0, 0, 0, 0, 0, 0};
}
// eight values of a row in global memory, 16-byte aligned
template <typename E> __device__ __forceinline__ Frag<E> load_fragment(const E* p) {
  if constexpr (sizeof(E) == 2) return *reinterpret_cast<const bf16x8*>(p);
  else { const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4); return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
}
// Waits here for fragments from global memory.  Left to the compiler the wait is where they are first used, inside the loop, and there it would be for the loads of the next tile as well.
template <typename F, int N> __device__ __forceinline__ void arrived(F (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}
__device__ __forceinline__ int register_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// Tiles in LDS: rows of DP values, their 16-byte pieces permuted within the row so that both fetches fill all banks: sixteen rows at the same piece, and four
// neighbouring rows at 64 neighbouring bytes.
template <typename E, int DP> struct Tile {
  static constexpr int ROW = DP * sizeof(E), PIECES = ROW / 16, DF = DP / 32, KS = DP / 16;
  static_assert(PIECES == 8 || PIECES % 16 == 0, "row");
  static __device__ __forceinline__ int permuted(int r) {
    if constexpr (PIECES == 8) return (((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1);
    else return ((r & 3) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1);
  }
  // A lane's place in a tile for either fetch, to be added to where the tile is (a multiple of ROW); which piece of a row is meant is then one exclusive or.
  static __device__ __forceinline__ uint32_t row_lane(int lane) {
    return (lane & 31) * ROW + ((permuted(lane & 31) ^ (lane >> 5) * (int)(sizeof(E) / 2)) << 4);
  }
  static __device__ __forceinline__ uint32_t column_lane(int lane) {
    const int h = lane >> 5;
    if constexpr (sizeof(E) == 2) {
      const int r = 4 * h + ((lane & 15) >> 2), piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
      return r * ROW + ((piece ^ permuted(r)) << 4) + (lane & 1) * 8;
    } else {
      return 4 * h * ROW + ((((lane & 31) >> 2) ^ permuted(4 * h)) << 4) + (lane & 3) * 4;
    }
  }
  // rows row0 + lane % 32, contraction 16 ks ..
  static __device__ __forceinline__ Frag<E> rows(uint32_t at, int row0, int ks) {
    if constexpr (sizeof(E) == 2) {
      return *(lds_bf16x8*)(uintptr_t)((at ^ (uint32_t)(ks << 5)) + row0 * ROW);
    } else {
      const f32x4 a = *(lds_f32x4*)(uintptr_t)((at ^ (uint32_t)(ks << 6)) + row0 * ROW), b = *(lds_f32x4*)(uintptr_t)((at ^ (uint32_t)(ks << 6 | 16)) + row0 * ROW);
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  // transposed: column 32 df + lane % 32 of rows row0 .. row0 + 15, in the order above
  static __device__ __forceinline__ Frag<E> columns(uint32_t at, int row0, int df) {
    if constexpr (sizeof(E) == 2) {
      union { bf16x8 v; s16x4 q[2]; } u;
#pragma unroll
      for (int t = 0; t < 2; ++t) u.q[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)((at ^ (uint32_t)(df << 6 | t << 4)) + (row0 + 8 * t) * ROW));
      return u.v;
    } else {
      f32x8 v;
#pragma unroll
      for (int t = 0; t < 8; ++t) v[t] = *(lds_float*)(uintptr_t)((at ^ (uint32_t)((df << 7) ^ ((t & 3) << 6) ^ ((t >> 2) << 4))) + (row0 + 8 * (t >> 2) + (t & 3)) * ROW);
      return v;
    }
  }
};

// Loads go from memory straight to LDS, 1 KB a wave and instruction, through buffer descriptors that begin at the tile's first row: what lies behind the last row
// or the row's last value reads as zero, and offsets stay below 2^31.
constexpr uint32_t NOWHERE = 0x80000000u, MOST = 0x7fffffffu;
struct Source {   // tiles of `step` bytes each, from `at` on
  uint64_t at, left; uint32_t step;
  __device__ __forceinline__ Source(const void* p, int64_t bytes, int64_t step_) : at((uint64_t)(uintptr_t)p), left((uint64_t)bytes), step((uint32_t)step_) {}
  __device__ __forceinline__ u32x4 tile(uint32_t t) const {
    const uint64_t off = (uint64_t)t * step, from = at + off, rest = left - off;
    return (u32x4){(uint32_t)from, (uint32_t)(from >> 32), rest > MOST ? MOST : (uint32_t)rest, 0x00020000u};
  }
  static __device__ __forceinline__ u32x4 nothing() { return (u32x4){0, 0, 0, 0x00020000u}; }   // reads as zero
};
__device__ __forceinline__ void load_to_lds(uint32_t to, uint32_t offset, u32x4 from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(from) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_void*)p); }

// ROWS rows of a tensor by WAVES waves: neighbouring tokens', or with `heads` the packed rows of G heads a token, see GROUP.
constexpr int GROUP = 64;   // packed rows: GROUP / G whole tokens, their heads one after the other, and what is left of 64 rows stays empty
template <typename E, int DP, int ROWS, int WAVES> struct Loads {
  typedef Tile<E, DP> T;
  static constexpr int BYTES = ROWS * T::ROW, N = BYTES / 1024 / WAVES;
  static_assert(BYTES % (1024 * WAVES) == 0, "loads");
  uint32_t offset[N];
  __device__ __forceinline__ void init(int64_t ld, int64_t hs, int G, int D, int wave, int lane) {
    const int tokens = GROUP / G;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const int at = (q * WAVES + wave) * 1024 + lane * 16, r = at / T::ROW, piece = (at % T::ROW / 16) ^ T::permuted(r), in = r % GROUP;
      const uint32_t row = (uint32_t)(G == 1 ? r : r / GROUP * tokens + in / G) * (uint32_t)ld + (uint32_t)(G == 1 ? 0 : in % G) * (uint32_t)hs;
      offset[q] = (G == 1 || in < tokens * G) && piece * 16 < D * (int)sizeof(E) ? row * (uint32_t)sizeof(E) + piece * 16 : NOWHERE;
    }
  }
  __device__ __forceinline__ void issue_one(int q, uint32_t lds, u32x4 from, int wave) const { load_to_lds(lds + (q * WAVES + wave) * 1024, offset[q], from); }
  __device__ __forceinline__ void issue(uint32_t lds, u32x4 from, int wave) const {
#pragma unroll
    for (int q = 0; q < N; ++q) issue_one(q, lds, from, wave);
  }
};
// nothing is on its way to LDS any more: before a wave ends, or uses LDS for something else
__device__ __forceinline__ void drain_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// everything a wave has asked for is in LDS, for all of them
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Scores in units of log 2: scale s, or cap tanh(scale s / cap), less slope |distance|.
enum { PLAIN = 0, CAPPED = 1, BIASED = 2 };
template <typename E, int SHAPE> struct Scores {
  float factor, in, out;     // s -> the exponent of e^2y for y = scale s / cap; cap log2(e)
  __device__ __forceinline__ Scores(float scale, float cap) : factor(scale * LOG2E), in(SHAPE & CAPPED ? (sizeof(E) == 2 ? 2.f * LOG2E : 1.f) * scale / cap : 0.f), out(cap * LOG2E) {}
  // The score, and what its derivative is multiplied by.  tanh y = 1 - 2 r, 1 - tanh^2 y = 4 r (1 - r) for r = 1 / (1 + e^2y): within 2^-22 of cap in all, 2^-17 of
  // a score for a cap of 30 and 2^-10 for the largest, where bf16 probabilities are rounded by 2^-9; in fp32 small scores want the library's tanh, whose error is relative.
  __device__ __forceinline__ float operator()(float s, float slope, float distance, float& bend) const {
    float x;
    if constexpr ((SHAPE & CAPPED) == 0) {
      x = s * factor;
    } else if constexpr (sizeof(E) == 2) {
      const float r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * in)), four = 4.f * r;
      x = fmaf(-2.f * out, r, out);
      bend = fmaf(-four, r, four);
    } else {
      const float t = tanhf(s * in);
      x = t * out;
      bend = fmaf(-t, t, 1.f);
    }
    if constexpr ((SHAPE & BIASED) != 0) x = fmaf(-slope, fabsf(distance), x);
    return x;
  }
};

// A run of TOTAL fetches, each used by use(i, fragment) AHEAD steps later.  Left to itself the compiler waits for each fragment right after asking for it.  What else a step does, such
// as a load of the next tile, which takes 90 clocks when several are issued at once, is spread over the run by use().
template <int TOTAL, int AHEAD_, typename F, typename Fetch, typename Use>
__device__ __forceinline__ void pipeline(Fetch fetch, Use use) {
  constexpr int AHEAD = AHEAD_ < TOTAL ? AHEAD_ : TOTAL;
  F x[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) x[i] = fetch(i);
#pragma unroll
  for (int i = 0; i < TOTAL; ++i) {
    use(i, x[i % AHEAD]);
    if (i + AHEAD < TOTAL) x[i % AHEAD] = fetch(i + AHEAD);
  }
}
template <typename E> constexpr int ROWS_AHEAD = sizeof(E) == 2 ? 4 : 2;

// The keys of a subtile of 32 that a lane sees, as bits, for its registers: bit 8 (r / 4) + r % 4 is register r's.
__device__ __forceinline__ uint32_t seen_keys(int2 span, int k0, int h) {
  const int lo = min(max(span.x - k0, 0), 32), hi = min(max(span.y - k0, 0), 32);
  const uint32_t below_hi = hi >= 32 ? 0xffffffffu : (1u << hi) - 1u, below_lo = lo >= 32 ? 0xffffffffu : (1u << lo) - 1u;
  return (below_hi & ~below_lo) >> (4 * h);
}
__device__ __forceinline__ int seen_bit(int r) { return 8 * (r >> 2) + (r & 3); }
// x where the bit is set, else `other`
__device__ __forceinline__ float where_seen(uint32_t seen, int r, float x, float other) {
  const uint32_t m = (uint32_t)((int32_t)(seen << (31 - seen_bit(r))) >> 31);
  return __uint_as_float((__float_as_uint(x) & m) | (__float_as_uint(other) & ~m));
}

// acc[df] += (columns 32 df .. of 16 N of a tile's rows)^T times the N fragments b.  The columns are fetched ahead of the arithmetic that makes b.
//
// Where some of a lane's weights are zero because it does not see the row (its bit of `seen` clear): zero times infinity or NaN is NaN, so a row that is not finite
// would reach lanes that do not see it.  The rows are looked through first, and if one is not finite, the product runs twice: with zeros for what is not, and with
// what is beyond every number where a lane sees such a value and nothing elsewhere.  One loop for both, because sums that leave a branch in two versions are copied.
template <typename E, int DP, int N> struct Columns {
  Frag<E> a[N][DP / 32];
  __device__ __forceinline__ void fetch(uint32_t tile, int row0) {   // tile: of a lane, see column_lane
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int df = 0; df < DP / 32; ++df) a[s][df] = Tile<E, DP>::columns(tile, row0 + 16 * s, df);
  }
};
template <typename E> __device__ __forceinline__ float add_unless_finite(const Frag<E>& x, float check) {   // check + 0 x
  if constexpr (sizeof(E) == 2) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 zero = {(__bf16)0.f, (__bf16)0.f};
    const union { bf16x8 v; bf16x2 w[4]; } u = {x};
#pragma unroll
    for (int i = 0; i < 4; ++i) check = __builtin_amdgcn_fdot2_f32_bf16(u.w[i], zero, check, false);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) check = fmaf(x[i], 0.f, check);
  }
  return check;
}
template <typename E, int DP>
__device__ __forceinline__ bool all_finite(uint32_t tile, int row0) {   // tile: of a lane, see row_lane
  float check = 0.f;
#pragma unroll
  for (int ks = 0; ks < DP / 16; ++ks) check = add_unless_finite<E>(Tile<E, DP>::rows(tile, row0, ks), check);
  return !__any(check != check);
}
template <typename E> __device__ __forceinline__ void split_finite(const Frag<E> x, Frag<E>& finite, Frag<E>& rest) {
  if constexpr (sizeof(E) == 2) {
    union { bf16x8 v; uint16_t w[8]; } a, f, r;
    a.v = x;
#pragma unroll
    for (int i = 0; i < 8; ++i) { const bool bad = (a.w[i] & 0x7f80) == 0x7f80; f.w[i] = bad ? 0 : a.w[i]; r.w[i] = bad ? 0x7f7f : 0; }
    finite = f.v; rest = r.v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool bad = (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
      finite[i] = bad ? 0.f : x[i]; rest[i] = bad ? std::numeric_limits<float>::max() : 0.f;
    }
  }
}
template <typename E, int DP, int N>
__device__ __forceinline__ void add_product(f32x16 (&acc)[DP / 32], Columns<E, DP, N>& x, Frag<E> (&b)[N], bool finite, uint32_t seen, uint32_t tile, int row0) {
  if (!finite) {
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int df = 0; df < DP / 32; ++df) { Frag<E> rest; split_finite<E>(x.a[s][df], x.a[s][df], rest); }
  }
  for (int turn = 0;; ++turn) {
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int df = 0; df < DP / 32; ++df) acc[df] = mma(x.a[s][df], b[s], acc[df]);
    if (finite || turn == 1) break;
    asm volatile("" : "+v"(seen));   // here and not before, where it would be for nothing
    x.fetch(tile, row0);
#pragma unroll
    for (int s = 0; s < N; ++s) {
#pragma unroll
      for (int df = 0; df < DP / 32; ++df) { Frag<E> rest; split_finite<E>(x.a[s][df], rest, x.a[s][df]); }
#pragma unroll
      for (int t = 0; t < 8; ++t) b[s][t] = (seen >> seen_bit(8 * s + t) & 1) ? 3e38f : 0.f;
    }
  }
}

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) x = min(x, __shfl_xor(x, k));
  return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) x = max(x, __shfl_xor(x, k));
  return x;
}
__device__ __forceinline__ float other_half_max(float x) { return join32(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float other_half_sum(float x) { return join32(x, [](float a, float b) { return a + b; }); }

// keys [first, end) of a query, none as [0, 0)
__device__ __forceinline__ int2 span_of(const int32_t* spans, int64_t query, int keys) {
  const int2 s = reinterpret_cast<const int2*>(spans)[query];
  const int first = max(s.x, 0), end = min(s.y, keys);
  return first < end ? make_int2(first, end) : make_int2(0, 0);
}

// 32 columns of a result, df, from lane's registers to its row
template <typename E>
__device__ __forceinline__ void store_columns(E* row, int df, int D, const f32x16& x, float factor, int h) {
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int d = 32 * df + 8 * b + 4 * h;
    if (d >= D) continue;
    if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(row + d) = make_uint2(pack_bf16x2(x[4 * b] * factor, x[4 * b + 1] * factor), pack_bf16x2(x[4 * b + 2] * factor, x[4 * b + 3] * factor));
    else *reinterpret_cast<f32x4*>(row + d) = (f32x4){x[4 * b] * factor, x[4 * b + 1] * factor, x[4 * b + 2] * factor, x[4 * b + 3] * factor};
  }
}

// Rows of a workgroup that walks the keys: 128 (four waves side by side), 64 (two, and two groups of keys) or 32 (four groups of keys, two where rows have 512 bytes).  What decides is how many
// workgroups there are, how many fit a CU, and how much of a tile the rows of a workgroup see.  us of the forward pass and of dq, causal; workgroups of 64 in brackets:
//   bf16, width 64: never 128.  16 heads of 8192 in one text (2048): 240 and 271 with 128, 216 and 264 with 64; 16 on 4 of 8111 in 23 texts (2028): 50 and 59, 42 and 48.  64 or 32, 12 heads of
//     4096 in 4 texts (768): 51 and 55, 44 and 48; in 41: 15 and 18, 23 and 26; 8 heads of 2000 in two (256): 32 and 33, 20 and 22.
//   fp32, width 64: never 128.  12 heads of 6000 in two texts (1128): 358 and 504 with 128, 311 and 418 with 64.  64 or 32, 12 heads of 4096 in 4 texts (768): 164 and 215, 173 and 220; in 41:
//     47 and 60, 63 and 75; 8 heads of 3500 in ten (440): 69 and 92, 56 and 70.
//   bf16, width 128: 16 heads on 8 of 8192 in one text (2048): 345 and 404 with 128, 414 and 478 with 64; 16 of 6000 in 20 texts (1504): 60 and 72, 59 and 66 (the rule takes 128, for long texts' sake).  64 or 32, 12 heads of 4096 in
//     4 texts (768): 73 and 80, 103 and 111; 8 of 3500 in ten (440): 31 and 34, 39 and 42; of 2000 in two (256): 43 and 45, 30 and 32.
//   fp32, width 128: 64 takes the time of 32.  128 or 32, a training step of 12 heads of 4096 in 4 texts (768): 1487, 1714; of 8 heads of 3500 in one (440): 1697, 1742; of 2000 (250): 995, 717.
inline int rows_of_workgroup(int64_t rows, int Hk, int width, bool bf16) {
  const int64_t of_128 = (rows + 127) / 128 * Hk, of_64 = (rows + 63) / 64 * Hk;
  if (width > 64 && of_128 >= (bf16 ? 512 : 192)) return 128;
  if (width > 64 && !bf16) return 32;
  return of_64 >= (width > 64 ? 384 : bf16 ? 1024 : 640) ? 64 : 32;
}

}  // namespace attn
}  // namespace sama
