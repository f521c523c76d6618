// The gated feed-forward block on the matrix cores, in bf16 with fp32 accumulation or in fp32: for T tokens of width d and F hidden values
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wo^T                                        (W_in = [Wg; Wu] [2F x d], Wo [d x F])
//   dh = dy Wo, dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu, dW_in = [dg; du]^T x, dWo = dy^T h.
// 6 T d F operations forward and 12 backward in four launches:
//   k_glu_up      both projections of a tile of tokens and hidden values in one workgroup, the rows of Wg and Wu sixteen by sixteen in turn, so that
//                 a lane has g and u of the same values and h is all that leaves it (for training also g and u, see below)
//   k_glu_dgate   dh, and out of it [dg, du] in the epilogue; dh is never stored
//   k_glu_product y; and dx, dW_in and dWo side by side: three products that read the same [dg, du] and none of which fills the chip alone.  Where the
//                 tiles of a product are too few, or a few too many for a round, the contraction is cut as well, and k_glu_join adds the parts
#include <algorithm>
#include <cmath>
#include <iterator>
#include <type_traits>
#include <utility>
#include "kernels.h"
#include "token_ops.h"

namespace sama {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;
constexpr int LDS_MAX = 160 * 1024;
// Elements E: bf16_t or float.  A slab is 128 bytes of the contraction, 64 or 32 indices, two k-steps of 64 bytes; a lane's operand of a k-step is 16 bytes,
// for one 16x16x32 product in bf16 or four of 16x16x4 in fp32.
constexpr int SLAB = 128;
template <typename E> constexpr uint32_t DEPTH = SLAB / sizeof(E);

// BM x BN outputs of a workgroup, by WGM x WGN multiplying waves; NSTAGE slabs of the contraction in LDS; PW waves that only load (0: the
// multiplying ones do); YP: fragments of B per piece of a k-step (0: all); RD: reads of a piece lie among the first 1 / RD of the products of the piece
// before it (0: ahead of its own products).
template <int BM_, int BN_, int WGM_, int WGN_, int NSTAGE_, int PW_, int YP_, int RD_, int PER_CU_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, NSTAGE = NSTAGE_, PW = PW_, RD = RD_, PER_CU = PER_CU_;
  static constexpr int WAVES = WGM * WGN, LW = PW > 0 ? PW : WAVES, THREADS = (WAVES + PW) * 64;
  static constexpr int WM = BM / WGM, WN = BN / WGN, XT = WM / 16, YT = WN / 16;
  static constexpr int YP = YP_ > 0 ? YP_ : YT, NP = YT / YP;
  static constexpr int A_BYTES = BM * SLAB, B_BYTES = BN * SLAB, STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int NLA = A_BYTES / 1024 / LW, NLB = B_BYTES / 1024 / LW, NL = NLA + NLB;
  static constexpr int LDS_BYTES = NSTAGE * STAGE_BYTES;
  static_assert(LDS_BYTES * PER_CU <= LDS_MAX && WM % 16 == 0 && WN % 32 == 0 && YT % YP == 0, "tile");
  static_assert(A_BYTES % (1024 * LW) == 0 && B_BYTES % (1024 * LW) == 0 && NL * (NSTAGE - 2) <= 63, "loads");
};

template <typename F, int... I>
__device__ __forceinline__ void static_for_each(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) { static_for_each(std::make_integer_sequence<int, N>{}, f); }

// An operand: KC, storage [rows][k] with the contraction index contiguous, staged in LDS [row][slab], or KS, storage [k][rows], staged [slab][rows] and fetched with
// the transposing read (bf16) or a word at a time (fp32).  Swizzles as in gemm_bf16.hip: of KC the 16-byte pieces of a row by (row / 2) % 8, of KS
// pieces of 16 rows of a k-row by a function of k, so that the lanes of a fetch fill all banks.
// PAIRS (KC): the rows of a tile are sixteen of the first half of the matrix, the same sixteen of the second half, and so on.
enum { KC, KS, PAIRS };
template <typename E, int R>
__device__ __forceinline__ int chunk_swizzle(int kr) {
  constexpr int NC = R / 16;
  static_assert(NC % 8 == 0 || NC == 4 || NC == 2, "tile width");
  if constexpr (sizeof(E) == 4) return (kr >> 2) & (NC == 2 ? 1 : 3);   // the four k-rows that a fetch of a word reads, four apart
  else if constexpr (NC == 2) return (kr >> 3) & 1;
  else return NC % 8 == 0 ? (kr & 3) | ((kr >> 1) & 4) : ((kr >> 1) & 1) | ((kr >> 2) & 2);
}
struct Operand {
  const void* p; uint32_t ld, rows;   // rows: of the matrix (KC) or its columns (KS); PAIRS: of a half
};
// Byte offset, from the slab's first element, of the 16 bytes that belong at byte `at` of its stage, and their contraction index.
template <typename E, int S, int R>
__device__ __forceinline__ uint32_t piece_offset(uint32_t at, const Operand& o, uint32_t& k) {
  constexpr uint32_t Z = sizeof(E);
  if constexpr (S == KS) {
    constexpr uint32_t RB = R * Z, PP = Z;   // pieces of 16 bytes in 16 rows
    const uint32_t kr = at / RB, q = at % RB / 16, ql = ((q / PP) ^ (uint32_t)chunk_swizzle<E, R>((int)kr)) * PP + q % PP;
    k = kr;
    return kr * o.ld * Z + ql * 16;
  } else {
    const uint32_t r = at / SLAB, c = at % SLAB / 16 ^ (r / 2) % 8;
    k = c * (16 / Z);
    const uint32_t row = S == KC ? r : (r / 32) * 16 + r % 16 + ((r / 16) & 1) * o.rows;
    return row * o.ld * Z + c * 16;
  }
}
template <typename E, int S, int R>
__device__ __forceinline__ int fetch_lane_offset(int lane, int ks_or_frag) {
  if constexpr (S == KS && sizeof(E) == 4) {
    const int kr = 4 * (lane >> 4);                             // and the three behind it; the same swizzle for kr + 16
    return kr * R * 4 + ((ks_or_frag ^ chunk_swizzle<E, R>(kr)) * 64) + 4 * (lane & 15);
  } else if constexpr (S == KS) {
    const int j = lane & 15, kr = 8 * (lane >> 4) + (j >> 2);   // the swizzle is the same for kr + 4 and kr + 32
    return kr * R * 2 + ((ks_or_frag ^ chunk_swizzle<E, R>(kr)) * 32) + 8 * (j & 3);
  } else {
    const int r = lane & 15;
    return r * 128 + (((4 * ks_or_frag + (lane >> 4)) ^ (r / 2) % 8) * 16);
  }
}

// Loads go through buffer descriptors: what lies behind the last value of a matrix reads as zero, so that tiles may hang over in rows and, of KS,
// in the contraction; the pieces of a KC slab behind the end of the contraction are sent out of range.  The descriptor begins at the slab's
// first element, so offsets stay below 2^31 whatever the size of the matrix.
constexpr uint32_t NOWHERE = 0x80000000u, MOST = 0x7fffffffu;
struct Window {
  uint64_t at, left;   // address of the next slab, bytes from there to the end of the matrix
  __device__ __forceinline__ u32x4 descriptor() const {
    return (u32x4){(uint32_t)at, (uint32_t)(at >> 32), left > MOST ? MOST : (uint32_t)left, 0x00020000u};
  }
  __device__ __forceinline__ void step(uint32_t bytes) { at += bytes; left -= bytes; }
};
template <typename E, int S>
__device__ __forceinline__ Window window(const Operand& o, uint32_t row0, uint32_t k0, uint32_t K) {
  Window w;
  const uint64_t first = S == KS ? (uint64_t)k0 * o.ld + row0 : (uint64_t)row0 * o.ld + k0;
  const uint64_t end = S == KS ? (uint64_t)(K - 1) * o.ld + o.rows : (uint64_t)((S == PAIRS ? 2 : 1) * o.rows - 1) * o.ld + K;
  w.at = (uint64_t)(uintptr_t)o.p + sizeof(E) * first;
  w.left = sizeof(E) * (end - first);
  return w;
}

template <int NL, int W>
__device__ __forceinline__ void wait_loads(int younger) {
  if constexpr (W == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else {
    if (younger >= W) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NL * W) : "memory");
    else wait_loads<NL, W - 1>(younger);
  }
}

// acc = the products of rows i0.. of A and j0.. of B over slabs [slab0, slab0 + slabs) of the contraction K.  D = B-fragment x A-fragment: a lane has
// four neighbouring columns 4 (lane / 16) .. + 3 of row lane % 16 of each 16 x 16 fragment.  Every wave of the workgroup calls it; those that only load
// come back without results.  No wave may read or write the stages any more when it is called.
template <typename T, typename E, int SA, int SB>
__device__ __forceinline__ void contract(f32x4 (&acc)[T::XT][T::YT], unsigned char* smem, const Operand& A, const Operand& B, uint32_t i0, uint32_t j0,
                                         uint32_t K, uint32_t slab0, int slabs) {
  constexpr int XT = T::XT, YT = T::YT, NSTAGE = T::NSTAGE;
  constexpr int RD = T::RD == 0 && SA != KS && SB != KS ? 9 : T::RD;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lw = T::PW > 0 ? wave - T::WAVES : wave;
  const bool loader = T::PW == 0 || wave >= (uint32_t)T::WAVES;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)smem;
  uint32_t offA[T::NLA], offB[T::NLB], ragged = 0;      // ragged: loads of a KC operand that are behind the contraction's end in its last slab
  Window wa{}, wb{};
  constexpr uint32_t BK = DEPTH<E>;
  const uint32_t stepA = SA == KS ? SLAB * A.ld : SLAB, stepB = SB == KS ? SLAB * B.ld : SLAB;
  const bool to_end = K % BK != 0 && slab0 + slabs == (K + BK - 1) / BK;
  int next = 0;
  uint32_t next_at = lds0 + lw * 1024;
  auto load = [&](uint32_t to, uint32_t off, u32x4 from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off), "s"(from) : "memory", "m0");
  };
  auto issue = [&]() {
    if (next >= slabs) return;
    const u32x4 da = wa.descriptor(), db = wb.descriptor();
    if (to_end && next == slabs - 1) {
#pragma unroll
      for (int q = 0; q < T::NLA; ++q) if (SA != KS && (ragged >> q & 1)) offA[q] = NOWHERE;
#pragma unroll
      for (int q = 0; q < T::NLB; ++q) if (SB != KS && (ragged >> (T::NLA + q) & 1)) offB[q] = NOWHERE;
    }
#pragma unroll
    for (int q = 0; q < T::NLA; ++q) load(next_at + q * T::LW * 1024, offA[q], da);
#pragma unroll
    for (int q = 0; q < T::NLB; ++q) load(next_at + T::A_BYTES + q * T::LW * 1024, offB[q], db);
    wa.step(stepA); wb.step(stepB);
    next_at = (next + 1) % NSTAGE == 0 ? lds0 + lw * 1024 : next_at + T::STAGE_BYTES;
    ++next;
  };
  auto arrive = [&](int sl) {   // slab sl is there for everybody, the stage of slab sl - 1 is free
    if (loader) wait_loads<T::NL, NSTAGE - 2>(slabs - 1 - sl);
    __builtin_amdgcn_s_barrier();
    if (loader) issue();
  };
  if (loader) {
    wa = window<E, SA>(A, i0, slab0 * BK, K); wb = window<E, SB>(B, j0, slab0 * BK, K);
    const uint32_t last_k = (K - 1) % BK;
#pragma unroll
    for (int q = 0; q < T::NLA; ++q) { uint32_t k; offA[q] = piece_offset<E, SA, T::BM>((q * T::LW + lw) * 1024 + lane * 16, A, k); if (k > last_k) ragged |= 1u << q; }
#pragma unroll
    for (int q = 0; q < T::NLB; ++q) { uint32_t k; offB[q] = piece_offset<E, SB, T::BN>((q * T::LW + lw) * 1024 + lane * 16, B, k); if (k > last_k) ragged |= 1u << (T::NLA + q); }
#pragma unroll
    for (int s = 0; s < NSTAGE - 1; ++s) issue();
  }
  if (T::PW > 0 && loader) {
    for (int i = 0; i < slabs; ++i) arrive(i);
    return;
  }

  const int wr = (int)(wave / T::WGN) * T::WM, wc = (int)(wave % T::WGN) * T::WN;
#pragma unroll
  for (int x = 0; x < XT; ++x)
#pragma unroll
    for (int y = 0; y < YT; ++y) acc[x][y] = (f32x4){0.f, 0.f, 0.f, 0.f};
  constexpr int STEPS = 2;
  int fa[SA == KS ? XT : STEPS], fb[SB == KS ? YT : STEPS];
  if (SA != KS) {
#pragma unroll
    for (int ks = 0; ks < STEPS; ++ks) fa[ks] = fetch_lane_offset<E, SA, T::BM>(lane, ks) + wr * SLAB;
  } else {
#pragma unroll
    for (int x = 0; x < XT; ++x) fa[x] = fetch_lane_offset<E, SA, T::BM>(lane, (wr >> 4) + x);
  }
  if (SB != KS) {
#pragma unroll
    for (int ks = 0; ks < STEPS; ++ks) fb[ks] = fetch_lane_offset<E, SB, T::BN>(lane, ks) + wc * SLAB;
  } else {
#pragma unroll
    for (int y = 0; y < YT; ++y) fb[y] = fetch_lane_offset<E, SB, T::BN>(lane, (wc >> 4) + y);
  }
  typedef std::conditional_t<sizeof(E) == 4, f32x4, bf16x8> Frag;
  auto fetch = [&](const unsigned char* s, auto strided, auto r, const int* f, int frag, int ks) -> Frag {
    constexpr int R = decltype(r)::value;
    if constexpr (!decltype(strided)::value) {
      return *reinterpret_cast<const Frag*>(s + f[ks] + frag * 16 * SLAB);
    } else if constexpr (sizeof(E) == 4) {
      const float* const p = reinterpret_cast<const float*>(s + f[frag] + ks * 16 * R * 4);
      return (f32x4){p[0], p[R], p[2 * R], p[3 * R]};
    } else {
      const unsigned char* const p = s + f[frag] + ks * 32 * R * 2;
      union { bf16x8 v; s16x4 h[2]; } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * R * 2));
      return u.v;
    }
  };
  auto fetchA = [&](const unsigned char* s, int x, int ks) { return fetch(s, std::bool_constant<SA == KS>{}, std::integral_constant<int, T::BM>{}, fa, x, ks); };
  auto fetchB = [&](const unsigned char* s, int y, int ks) { return fetch(s + T::A_BYTES, std::bool_constant<SB == KS>{}, std::integral_constant<int, T::BN>{}, fb, y, ks); };

  // pieces of a slab, products of a piece: in fp32 four for each pair of fragments, all pairs before the next four, so that none waits for the one before it
  constexpr int YP = T::YP, NP = T::NP, NT = STEPS * NP, SUB = sizeof(E) == 4 ? 4 : 1, NM = XT * YP * SUB;
  static_assert(NT % 2 == 0, "operand double buffer parity");
  Frag av[2][XT], bv[2][YP];
  auto mfma = [&](auto t, auto m) {
    constexpr int T_ = t, M_ = m % (XT * YP), ks = T_ / NP, y0 = T_ % NP * YP, x = M_ / YP, yy = M_ % YP, y = (x & 1) ? YP - 1 - yy : yy;
    if constexpr (sizeof(E) == 4) acc[x][y0 + y] = __builtin_amdgcn_mfma_f32_16x16x4f32(bv[T_ & 1][y][m / (XT * YP)], av[ks & 1][x][m / (XT * YP)], acc[x][y0 + y], 0, 0, 0);
    else acc[x][y0 + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bv[T_ & 1][y], av[ks & 1][x], acc[x][y0 + y], 0, 0, 0);
  };
  constexpr int READS = YP + XT;
  auto operands = [](int t) { return YP + (t % NP == 0 ? XT : 0); };
  auto read = [&](const unsigned char* at, auto t, auto r) {
    constexpr int T_ = t, R_ = r, ks = T_ / NP, p = T_ % NP, wa1 = p == 0 ? 1 : 0;
    if constexpr (wa1 == 1 && R_ == 0) av[ks & 1][0] = fetchA(at, 0, ks);
    else if constexpr (R_ - wa1 < YP) bv[T_ & 1][R_ - wa1] = fetchB(at, p * YP + R_ - wa1, ks);
    else av[ks & 1][R_ - YP] = fetchA(at, R_ - YP, ks);
  };
  auto read_all = [&](const unsigned char* at, auto t) {
    static_for<READS>([&](auto r) { if constexpr (decltype(r)::value < operands(decltype(t)::value)) read(at, t, r); });
  };
  auto multiply = [&](auto t) {
    if (RD != 0) __builtin_amdgcn_sched_barrier(0);
    static_for<NM>([&](auto m) { mfma(t, m); });
    if (RD != 0) __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply_reading = [&](auto t, const unsigned char* at, auto tn) {
    constexpr int nr = operands(decltype(tn)::value);
    constexpr auto before = [](int m) { const int b = (m * nr * RD + NM - 1) / NM; return b < nr ? b : nr; };
    __builtin_amdgcn_sched_barrier(0);
    static_for<NM>([&](auto m) {
      static_for<READS>([&](auto r) { if constexpr (decltype(r)::value >= before(decltype(m)::value) && decltype(r)::value < before(decltype(m)::value + 1)) read(at, tn, r); });
      __builtin_amdgcn_sched_barrier(0);
      mfma(t, m);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto stage_of = [&](int sl) { return smem + (sl % NSTAGE) * T::STAGE_BYTES; };
  arrive(0);
  if constexpr (RD == 0) {
    for (int i = 0; i < slabs; ++i) {
      if (i > 0) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        arrive(i);
      }
      const unsigned char* const at = stage_of(i);
      static_for<NT>([&](auto t) { read_all(at, t); multiply(t); });
    }
  } else {
    read_all(stage_of(0), std::integral_constant<int, 0>{});
    for (int i = 0; i + 1 < slabs; ++i) {
      const unsigned char* const at = stage_of(i);
      static_for<NT - 1>([&](auto t) { multiply_reading(t, at, std::integral_constant<int, decltype(t)::value + 1>{}); });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      arrive(i + 1);
      multiply_reading(std::integral_constant<int, NT - 1>{}, stage_of(i + 1), std::integral_constant<int, 0>{});
    }
    const unsigned char* const at = stage_of(slabs - 1);
    static_for<NT - 1>([&](auto t) { multiply_reading(t, at, std::integral_constant<int, decltype(t)::value + 1>{}); });
    multiply(std::integral_constant<int, NT - 1>{});
  }
}

// ---------------------------------------------------------------------------------------------------- epilogues
__device__ __forceinline__ uint2 packed(f32x4 v) { return make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); }
// Of two neighbouring fragments lanes 16 apart exchange halves: a lane then has eight neighbouring columns, 16 (g & 1) + 8 (g / 2) on, g = lane / 16.
__device__ __forceinline__ uint4 side_by_side(f32x4 a, f32x4 b) {
  uint2 v0 = packed(a), v1 = packed(b);
  u32x2 r = __builtin_amdgcn_permlane16_swap(v0.x, v1.x, false, false); v0.x = r[0]; v1.x = r[1];
  r = __builtin_amdgcn_permlane16_swap(v0.y, v1.y, false, false); v0.y = r[0]; v1.y = r[1];
  return make_uint4(v0.x, v0.y, v1.x, v1.y);
}
__device__ __forceinline__ int pair_column(int lane) { return 16 * ((lane >> 4) & 1) + 8 * (lane >> 5); }

// The gate and its derivative: silu(g) = g s, silu'(g) = s + g s (1 - s) with s = 1 / (1 + exp(-g)); gelu(g) = g P(g), gelu'(g) = P(g) + g p(g) with the
// normal distribution P and its density p.  In fp32 with the full-precision exp and erf: 1 + erf leaves
// P within 6e-8, which below -5 is as large as P.  In bf16, where the result is rounded to 2^-9 of itself, with the
// hardware's exp2 and reciprocal, and P through its logarithm, which is smooth: P(-x) = 2^q(x) for x >= 0 with a q of degree seven, fitted here to log2 P(-x) on
// [0, 7.5] (Chebyshev points, errors beyond 3.5 counting less).  Its errors: 4e-6 of P down to -3.5, 5e-5 down to -6, 1.6e-4 down to -7.5, where P is 3e-14; behind the fitted end
// they pass the rounding to bf16 (2 % at -9, two thirds at -12), of a P of 1e-19 and less, while q falls on to minus infinity.  Of gelu 6e-7
// anywhere.  An exp2 and eight multiply-adds, where an erf by exp and reciprocal is twice that, and the epilogue of a tile has nothing to hide it
// behind: both projections of 4096 x 768 x 2048 29.3 us instead of 30.9, 26.0 without any gate.
__device__ __forceinline__ float normal_cdf(float g) {
  const float x = fabsf(g);
  float q = -1.72933608e-06f;
  q = fmaf(q, x, 5.9637081e-05f); q = fmaf(q, x, -0.000916504301f); q = fmaf(q, x, 0.00845899247f); q = fmaf(q, x, -0.0538729616f);
  q = fmaf(q, x, -0.458539814f); q = fmaf(q, x, -1.15122414f); q = fmaf(q, x, -0.999997795f);
  const float below = __builtin_amdgcn_exp2f(q);
  return g < 0.f ? below : 1.f - below;
}
template <typename E, int ACT>
__device__ __forceinline__ void gate_and_slope(float g, float& a, float& da) {
  if constexpr (ACT == GLU_GELU) {
    float cdf, ez;
    if constexpr (sizeof(E) == 4) { cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f)); ez = expf(-0.5f * g * g); }
    else { cdf = normal_cdf(g); ez = __builtin_amdgcn_exp2f(-0.72134752044448170f * g * g); }
    a = g * cdf; da = fmaf(g * 0.39894228040143268f, ez, cdf);
  } else {
    float s;
    if constexpr (sizeof(E) == 4) s = 1.f / (1.f + expf(-g));
    else s = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    a = g * s; da = fmaf(a, 1.f - s, s);
  }
}
template <typename E, int ACT>
__device__ __forceinline__ float gate(float g) {
  float a, da;
  gate_and_slope<E, ACT>(g, a, da);
  return a;
}

// g and u as the backward pass finds them: their leading 24 bits (2^-15, where the rounding to bf16 that follows is 2^-8), four values of each in
// three words, so that a lane's part of a 16 x 16 fragment is 16 and 8 bytes.  Blocks of 16 rows by 16 columns in row order, 1 KB and 512 bytes of
// one block side by side: every store and load is whole lines.  Held in bf16 they would be 8 bytes of 12 and would double the error
// of the gradients, in fp32 16.
// They go past the caches, which keep the operands: 8192 x 1024 x 4096 620 -> 600 us for both passes, and no size is slower.
constexpr int SAVED_BLOCK = 1536;
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void pack24(f32x4 v, uint32_t (&w)[3]) {
  const uint32_t b[4] = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  w[0] = __builtin_amdgcn_perm(b[1], b[0], 0x05030201);
  w[1] = __builtin_amdgcn_perm(b[2], b[1], 0x06050302);
  w[2] = __builtin_amdgcn_perm(b[3], b[2], 0x07060503);
}
__device__ __forceinline__ f32x4 unpack24(uint32_t w0, uint32_t w1, uint32_t w2) {
  return (f32x4){__uint_as_float(w0 << 8), __uint_as_float(__builtin_amdgcn_perm(w1, w0, 0x0504030c)),
                 __uint_as_float(__builtin_amdgcn_perm(w2, w1, 0x0403020c)), __uint_as_float(w2 & 0xffffff00u)};
}

struct TileOrder { uint32_t tiles, per_xcd, tm, tn; };   // tm x tn tiles
// Workgroups are dealt to the eight XCDs in turn; each gets a run of the tiles, in groups of eight tile rows, column by column.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t& ti, uint32_t& tj) {
  const uint32_t width = 8 * tn, grp = id / width, rest = id - grp * width, high = min(tm - grp * 8, 8u);
  tj = rest / high; ti = grp * 8 + rest - tj * high;
}

struct UpArgs {
  Operand x, w;          // w: PAIRS
  uint32_t T, F, d;
  TileOrder order;
  void* h;               // [T x F]
  void* saved;           // or null
};
template <typename T, typename E, int ACT>
__global__ __launch_bounds__(T::THREADS) void k_glu_up(UpArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t id = (blockIdx.x & 7) * a.order.per_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= a.order.per_xcd || id >= a.order.tiles) return;
  uint32_t ti, tj;
  tile_of(id, a.order.tm, a.order.tn, ti, tj);
  const uint32_t i0 = ti * T::BM, j0 = tj * (T::BN / 2);
  f32x4 acc[T::XT][T::YT];
  contract<T, E, KC, PAIRS>(acc, smem, a.x, a.w, i0, j0, a.d, 0, (a.d + DEPTH<E> - 1) / DEPTH<E>);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= (uint32_t)T::WAVES) return;
  const int lane = threadIdx.x & 63;
  const uint32_t row0 = i0 + (wave / T::WGN) * T::WM, col0 = j0 + (wave % T::WGN) * (T::WN / 2);
  const uint32_t blocks = (a.F + 15) / 16;
  constexpr int GR = T::YT / 2;                     // granules of 16 hidden values
  static_for<T::XT>([&](auto x_) {
    constexpr int x = x_;
    if (row0 + 16 * x >= a.T) return;
    const uint32_t row = row0 + 16 * x + (lane & 15);
    E* const to = static_cast<E*>(a.h) + (uint64_t)row * a.F;
    f32x4 h[GR];
    static_for<GR>([&](auto q_) {
      constexpr int q = q_;
      const f32x4 g = acc[x][2 * q], u = acc[x][2 * q + 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) h[q][e] = gate<E, ACT>(g[e]) * u[e];
      const uint32_t col = col0 + 16 * q + 4 * (lane >> 4);
      if constexpr (sizeof(E) == 4) {
        if (row < a.T && col < a.F) {
          *reinterpret_cast<f32x4*>(to + col) = h[q];
          if (a.saved != nullptr) {
            float* const b = static_cast<float*>(a.saved) + (uint64_t)row * (2 * a.F) + col;
            *reinterpret_cast<f32x4*>(b) = g;
            *reinterpret_cast<f32x4*>(b + a.F) = u;
          }
        }
      } else if (a.saved != nullptr && col0 + 16 * q < a.F) {
        unsigned char* const b = static_cast<unsigned char*>(a.saved) + ((uint64_t)((row0 >> 4) + x) * blocks + (col0 >> 4) + q) * SAVED_BLOCK;
        uint32_t wg[3], wu[3];
        pack24(g, wg); pack24(u, wu);
        __builtin_nontemporal_store((u32x4){wg[0], wg[1], wg[2], wu[0]}, reinterpret_cast<u32x4*>(b + lane * 16));
        __builtin_nontemporal_store((words2){wu[1], wu[2]}, reinterpret_cast<words2*>(b + 1024 + lane * 8));
      }
    });
    if constexpr (sizeof(E) == 2 && GR == 1) {
      const uint32_t col = col0 + 4 * (lane >> 4);
      if (row < a.T && col < a.F) *reinterpret_cast<uint2*>(to + col) = packed(h[0]);
    } else if constexpr (sizeof(E) == 2) {
      static_for<GR / 2>([&](auto q_) {
        constexpr int q = 2 * q_;
        const uint4 v = side_by_side(h[q], h[q + 1]);
        const uint32_t col = col0 + 16 * q + pair_column(lane);
        if (row < a.T && col < a.F) *reinterpret_cast<uint4*>(to + col) = v;
      });
    }
  });
}

struct DgateArgs {
  Operand dy, w;         // w: KS
  uint32_t T, F, d;
  TileOrder order;
  const void* saved;
  void* dpre;            // [T x 2F]: dg, du
};
template <typename T, typename E, int ACT>
__global__ __launch_bounds__(T::THREADS) void k_glu_dgate(DgateArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t id = (blockIdx.x & 7) * a.order.per_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= a.order.per_xcd || id >= a.order.tiles) return;
  uint32_t ti, tj;
  tile_of(id, a.order.tm, a.order.tn, ti, tj);
  const uint32_t i0 = ti * T::BM, j0 = tj * T::BN;
  f32x4 acc[T::XT][T::YT];
  contract<T, E, KC, KS>(acc, smem, a.dy, a.w, i0, j0, a.d, 0, (a.d + DEPTH<E> - 1) / DEPTH<E>);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= (uint32_t)T::WAVES) return;
  const int lane = threadIdx.x & 63;
  const uint32_t row0 = i0 + (wave / T::WGN) * T::WM, col0 = j0 + (wave % T::WGN) * T::WN;
  const uint32_t blocks = (a.F + 15) / 16;
  auto backward = [&](f32x4 g, f32x4 u, f32x4 dh, f32x4& dg, f32x4& du) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float s, ds;
      gate_and_slope<E, ACT>(g[e], s, ds);
      dg[e] = dh[e] * (u[e] * ds); du[e] = dh[e] * s;
    }
  };
  if constexpr (sizeof(E) == 4) {
    static_for<T::XT>([&](auto x_) {
      constexpr int x = x_;
      const uint32_t row = row0 + 16 * x + (lane & 15);
      float* const to = static_cast<float*>(a.dpre) + (uint64_t)row * (2 * a.F);
      static_for<T::YT>([&](auto y_) {
        const uint32_t col = col0 + 16 * decltype(y_)::value + 4 * (lane >> 4);
        if (row >= a.T || col >= a.F) return;
        const float* const b = static_cast<const float*>(a.saved) + (uint64_t)row * (2 * a.F) + col;
        f32x4 dg, du;
        backward(*reinterpret_cast<const f32x4*>(b), *reinterpret_cast<const f32x4*>(b + a.F), acc[x][decltype(y_)::value], dg, du);
        *reinterpret_cast<f32x4*>(to + col) = dg;
        *reinterpret_cast<f32x4*>(to + a.F + col) = du;
      });
    });
  } else {
    // Two neighbouring fragments at a time, AHEAD pairs of g and u on their way: with one, a wave of the 256 x 256 tile waits for memory sixteen times in a row.
    constexpr int H = T::YT / 2, N = T::XT * H, AHEAD = N < 5 ? N : 5;
    struct { uint4 p; uint2 r; } v[AHEAD][2];
    const uint32_t last_row = (a.T - 1) >> 4;
    auto fetch = [&](auto n_) {
      constexpr int n = n_, x = n / H, h = n % H;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t block = min((col0 >> 4) + 2 * h + k, blocks - 1);
        const unsigned char* const b = static_cast<const unsigned char*>(a.saved) + ((uint64_t)min((row0 >> 4) + x, last_row) * blocks + block) * SAVED_BLOCK;
        v[n % AHEAD][k].p = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(b + lane * 16)));
        v[n % AHEAD][k].r = __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const words2*>(b + 1024 + lane * 8)));
      }
    };
    static_for<AHEAD>([&](auto n) { fetch(n); });
    static_for<N>([&](auto n_) {
      constexpr int n = n_, x = n / H, h = n % H;
      f32x4 dg[2], du[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 p = v[n % AHEAD][k].p;
        const uint2 r = v[n % AHEAD][k].r;
        backward(unpack24(p.x, p.y, p.z), unpack24(p.w, r.x, r.y), acc[x][2 * h + k], dg[k], du[k]);
      }
      if constexpr (n + AHEAD < N) fetch(std::integral_constant<int, n + AHEAD>{});
      const uint4 vg = side_by_side(dg[0], dg[1]), vu = side_by_side(du[0], du[1]);
      const uint32_t row = row0 + 16 * x + (lane & 15), col = col0 + 32 * h + pair_column(lane);
      bf16_t* const to = static_cast<bf16_t*>(a.dpre) + (uint64_t)row * (2 * a.F) + col;
      if (row < a.T && col < a.F) {
        *reinterpret_cast<uint4*>(to) = vg;
        *reinterpret_cast<uint4*>(to + a.F) = vu;
      }
    });
  }
}

// ---------------------------------------------------------------------------------------------------- products in pieces
// One to three products in a launch.  A tile's contraction may be cut into `parts` equal ones: each is a workgroup of its own, which leaves its sums in `part`, a
// fragment of 16 x 16 after the other as the lanes hold them, and k_glu_join adds those of a tile in the order of the contraction.  (Added by the last of
// a tile's workgroups to finish, in the same launch: two thousand clocks of waiting for stores, ticket and loads in one workgroup after the other, 15 us
// where the launch of its own takes 5, and the code for it took registers from the products.)
constexpr int MAX_PRODUCTS = 3;
struct Product {
  Operand A, B;
  uint32_t M, N, K, tm, tn, slabs, parts;
  uint32_t first;        // piece: of all the products before, a multiple of 8
  void* C; uint32_t ldc; int strided_a, c32;
  float* part;           // [parts][tiles][BM x BN]
};
struct ProductArgs {
  Product p[MAX_PRODUCTS];
  int count;
};
// one row of fragments of a wave's part of a tile
template <typename T>
__device__ __forceinline__ void store_row(const f32x4 (&c)[T::YT], const Product& p, uint32_t row0, uint32_t col0) {
  const int lane = threadIdx.x & 63;
  const uint32_t row = row0 + (lane & 15);
  if (p.c32) {
    float* const to = static_cast<float*>(p.C) + (uint64_t)row * p.ldc;
    static_for<T::YT>([&](auto y_) {
      const uint32_t col = col0 + 16 * decltype(y_)::value + 4 * (lane >> 4);
      if (row < p.M && col < p.N) *reinterpret_cast<f32x4*>(to + col) = c[decltype(y_)::value];
    });
  } else {
    bf16_t* const to = static_cast<bf16_t*>(p.C) + (uint64_t)row * p.ldc;
    static_for<T::YT / 2>([&](auto h_) {
      constexpr int h = h_;
      const uint4 v = side_by_side(c[2 * h], c[2 * h + 1]);
      const uint32_t col = col0 + 32 * h + pair_column(lane);
      if (row < p.M && col < p.N) *reinterpret_cast<uint4*>(to + col) = v;
    });
  }
}

// KIND 0: forward (A and B KC); 1: gradients, dx with A KC and B KS, the weights' with both KS
template <typename T, typename E, int KIND>
__global__ __launch_bounds__(T::THREADS) void k_glu_product(ProductArgs a) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  int k = 0;
  while (k + 1 < a.count && blockIdx.x >= a.p[k + 1].first) ++k;
  const Product& p = a.p[k];
  const uint32_t tiles = p.tm * p.tn, pieces = tiles * p.parts, per_xcd = (pieces + 7) / 8, b = blockIdx.x - p.first, id = (b & 7) * per_xcd + (b >> 3);
  if ((b >> 3) >= per_xcd || id >= pieces) return;
  const uint32_t part = p.parts > 1 ? id / tiles : 0, tile = id - part * tiles;
  const uint32_t slab0 = p.parts > 1 ? part * p.slabs / p.parts : 0;
  const int slabs = (int)((p.parts > 1 ? (part + 1) * p.slabs / p.parts : p.slabs) - slab0);
  uint32_t ti, tj;
  tile_of(tile, p.tm, p.tn, ti, tj);
  const uint32_t i0 = ti * T::BM, j0 = tj * T::BN;
  f32x4 acc[T::XT][T::YT];
  if constexpr (KIND == 0) contract<T, E, KC, KC>(acc, smem, p.A, p.B, i0, j0, p.K, slab0, slabs);
  else if (p.strided_a) contract<T, E, KS, KS>(acc, smem, p.A, p.B, i0, j0, p.K, slab0, slabs);
  else contract<T, E, KC, KS>(acc, smem, p.A, p.B, i0, j0, p.K, slab0, slabs);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave >= (uint32_t)T::WAVES) return;
  if (p.parts == 1) {
    const uint32_t row0 = i0 + (wave / T::WGN) * T::WM, col0 = j0 + (wave % T::WGN) * T::WN;
    static_for<T::XT>([&](auto x) { store_row<T>(acc[decltype(x)::value], p, row0 + 16 * decltype(x)::value, col0); });
  } else {
    float* const to = p.part + ((uint64_t)id * T::WAVES + wave) * (T::XT * T::YT * 256) + (threadIdx.x & 63) * 4;
    static_for<T::XT>([&](auto x_) {
      static_for<T::YT>([&](auto y_) { *reinterpret_cast<f32x4*>(to + (decltype(x_)::value * T::YT + decltype(y_)::value) * 256) = acc[decltype(x_)::value][decltype(y_)::value]; });
    });
  }
}

// A wave adds two neighbouring fragments of a tile.
template <typename T>
__global__ __launch_bounds__(256) void k_glu_join(ProductArgs a) {
  constexpr uint32_t PAIRS_OF = T::WAVES * T::XT * T::YT / 2;   // of a tile
  uint64_t id = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  int k = 0;
  while (k < a.count && (a.p[k].parts == 1 || id >= (uint64_t)a.p[k].tm * a.p[k].tn * PAIRS_OF)) {
    if (a.p[k].parts > 1) id -= (uint64_t)a.p[k].tm * a.p[k].tn * PAIRS_OF;
    ++k;
  }
  if (k == a.count) return;
  const Product& p = a.p[k];
  const uint32_t tiles = p.tm * p.tn, tile = (uint32_t)(id / PAIRS_OF), pair = (uint32_t)(id % PAIRS_OF);
  const uint32_t wave = pair / (T::XT * T::YT / 2), x = pair % (T::XT * T::YT / 2) / (T::YT / 2), h = pair % (T::YT / 2);
  const int lane = threadIdx.x & 63;
  const uint64_t step = (uint64_t)tiles * T::BM * T::BN;
  const float* from = p.part + ((uint64_t)tile * T::WAVES + wave) * (T::XT * T::YT * 256) + (x * T::YT + 2 * h) * 256 + lane * 4;
  f32x4 sum[2] = {*reinterpret_cast<const f32x4*>(from), *reinterpret_cast<const f32x4*>(from + 256)};
  uint32_t n = p.parts - 1;
  for (; n >= 3; n -= 3) {
    f32x4 v[3][2];
#pragma unroll
    for (int u = 0; u < 3; ++u) { from += step; v[u][0] = *reinterpret_cast<const f32x4*>(from); v[u][1] = *reinterpret_cast<const f32x4*>(from + 256); }
#pragma unroll
    for (int u = 0; u < 3; ++u) { sum[0] += v[u][0]; sum[1] += v[u][1]; }
  }
  for (; n > 0; --n) {
    from += step;
    sum[0] += *reinterpret_cast<const f32x4*>(from); sum[1] += *reinterpret_cast<const f32x4*>(from + 256);
  }
  uint32_t ti, tj;
  tile_of(tile, p.tm, p.tn, ti, tj);
  const uint32_t row = ti * T::BM + (wave / T::WGN) * T::WM + 16 * x + (lane & 15), col0 = tj * T::BN + (wave % T::WGN) * T::WN + 32 * h;
  if (p.c32) {
    float* const to = static_cast<float*>(p.C) + (uint64_t)row * p.ldc;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t col = col0 + 16 * y + 4 * (lane >> 4);
      if (row < p.M && col < p.N) *reinterpret_cast<f32x4*>(to + col) = sum[y];
    }
  } else {
    const uint4 v = side_by_side(sum[0], sum[1]);
    const uint32_t col = col0 + pair_column(lane);
    if (row < p.M && col < p.N) *reinterpret_cast<uint4*>(static_cast<bf16_t*>(p.C) + (uint64_t)row * p.ldc + col) = v;
  }
}

// ---------------------------------------------------------------------------------------------------- a few tokens
// With up to 16 NT tokens reading the weights is the work, 6 d F bytes, and a product over slabs in LDS is mostly waiting: loads, barrier, loads.  Here a wave
// takes 16 rows of weights and a share of the contraction, in the operand layout straight from memory (lane r + 16 q: eight values of row r), AHEAD
// steps of 32 at once, so that nearly all of a workgroup's weights are asked for before the first arrives; the tokens are the other operand, and
// come from the caches.  The waves' shares meet in LDS, in order.  What it measures stands at launch_glu_ffn().
template <int NA, int NT>
__device__ __forceinline__ void contract_few(f32x4 (&acc)[NA][NT], const bf16_t* w, uint64_t next_w, const bf16_t* x, uint32_t ldx, uint32_t T, uint32_t K, uint32_t step0,
                                             uint32_t step1) {
  const int lane = threadIdx.x & 63, q = lane >> 4;
  constexpr int AHEAD = NA * NT == 1 ? 8 : 4;
#pragma unroll
  for (int n = 0; n < NA; ++n)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
  const bf16_t* xr[NT];   // (tokens that are not there: the last one's results again, which nobody stores)
#pragma unroll
  for (int t = 0; t < NT; ++t) xr[t] = x + (uint64_t)min(16 * t + (lane & 15), T - 1) * ldx;
  for (uint32_t s0 = step0; s0 < step1; s0 += AHEAD) {
    bf16x8 a[AHEAD][NA], b[AHEAD][NT];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const uint32_t k = min(32 * min(s0 + s, step1 - 1) + 8 * q, K - 8);   // K is a multiple of 8
#pragma unroll
      for (int n = 0; n < NA; ++n) a[s][n] = *reinterpret_cast<const bf16x8*>(w + n * next_w + k);
#pragma unroll
      for (int t = 0; t < NT; ++t) b[s][t] = *reinterpret_cast<const bf16x8*>(xr[t] + k);
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      if (s0 + s >= step1) break;
      if (32 * (s0 + s) + 8 * q >= K) {                                     // behind the end: zeros on both sides
#pragma unroll
        for (int n = 0; n < NA; ++n) a[s][n] = bf16x8{};
#pragma unroll
        for (int t = 0; t < NT; ++t) b[s][t] = bf16x8{};
      }
#pragma unroll
      for (int n = 0; n < NA; ++n)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s][n], b[s][t], acc[n][t], 0, 0, 0);
    }
  }
}
__device__ __forceinline__ uint32_t share_of(uint32_t steps, uint32_t share, uint32_t of) { return steps * share / of; }

// h (and what the backward pass wants) of 16 hidden values: a wave an eighth of the contraction
template <int NT, int ACT>
__global__ __launch_bounds__(512) void k_glu_up_few(UpArgs a) {
  __shared__ f32x4 part[8][2][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t f0 = blockIdx.x * 16, steps = (a.d + 31) / 32;
  f32x4 acc[2][NT];
  const bf16_t* const w = static_cast<const bf16_t*>(a.w.p) + (uint64_t)min(f0 + (lane & 15), a.F - 1) * a.d;
  contract_few<2, NT>(acc, w, (uint64_t)a.F * a.d, static_cast<const bf16_t*>(a.x.p), a.x.ld, a.T, a.d, share_of(steps, wave, 8), share_of(steps, wave + 1, 8));
#pragma unroll
  for (int t = 0; t < NT; ++t) { part[wave][0][t][lane] = acc[0][t]; part[wave][1][t][lane] = acc[1][t]; }
  __syncthreads();
  if (wave >= NT || 16 * wave >= (int)a.T) return;
  const int t = wave;
  f32x4 g = part[0][0][t][lane], u = part[0][1][t][lane], h;
#pragma unroll
  for (int k = 1; k < 8; ++k) { g += part[k][0][t][lane]; u += part[k][1][t][lane]; }
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = gate<bf16_t, ACT>(g[e]) * u[e];
  if (a.saved != nullptr) {
    unsigned char* const b = static_cast<unsigned char*>(a.saved) + ((uint64_t)t * ((a.F + 15) / 16) + blockIdx.x) * SAVED_BLOCK;
    uint32_t wg[3], wu[3];
    pack24(g, wg); pack24(u, wu);
    *reinterpret_cast<uint4*>(b + lane * 16) = make_uint4(wg[0], wg[1], wg[2], wu[0]);
    *reinterpret_cast<uint2*>(b + 1024 + lane * 8) = make_uint2(wu[1], wu[2]);
  }
  const uint32_t row = 16 * t + (lane & 15), col = f0 + 4 * (lane >> 4);
  if (row < a.T && col < a.F) *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.h) + (uint64_t)row * a.F + col) = packed(h);
}

struct DownFewArgs { const bf16_t *h, *w; uint32_t T, F, d; bf16_t* y; uint32_t ldy; };
constexpr int DOWN_WAVES = 16;
template <int NT>
__global__ __launch_bounds__(DOWN_WAVES * 64) void k_glu_down_few(DownFewArgs a) {
  __shared__ f32x4 part[DOWN_WAVES][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t r0 = blockIdx.x * 16, steps = (a.F + 31) / 32;
  f32x4 acc[1][NT];
  contract_few<1, NT>(acc, a.w + (uint64_t)min(r0 + (lane & 15), a.d - 1) * a.F, 0, a.h, a.F, a.T, a.F, share_of(steps, wave, DOWN_WAVES), share_of(steps, wave + 1, DOWN_WAVES));
#pragma unroll
  for (int t = 0; t < NT; ++t) part[wave][t][lane] = acc[0][t];
  __syncthreads();
  if (wave >= NT || 16 * wave >= (int)a.T) return;
  f32x4 s = part[0][wave][lane];
  for (int k = 1; k < DOWN_WAVES; ++k) s += part[k][wave][lane];
  const uint32_t row = 16 * wave + (lane & 15), col = r0 + 4 * (lane >> 4);
  if (row < a.T && col < a.d) *reinterpret_cast<uint2*>(a.y + (uint64_t)row * a.ldy + col) = packed(s);
}

// Up to four tokens: four rows of weights to a workgroup, 256 bytes of each a load (in the 4 x 4 x 4 product of sixteen blocks a block is the next
// eight values of the contraction), so that four times as many workgroups ask for weights.  Lane 4 b + i: row, and token, i of block b.  One token, us: 1024 x 4096
// 5.2 + 4.1 (25 MB: 2.7 TB/s with the launches, of which there is nothing to hide them behind), 16 rows at a time 5.6 + 7.3; 2048 x 5504 10.5 + 5.4 (68 MB:
// 4.3 TB/s), 14.1 + 10.8.
__device__ __forceinline__ f32x4 contract_rows(const bf16_t* w, const bf16_t* x, uint32_t K, uint32_t step0, uint32_t step1) {
  const uint32_t b = (threadIdx.x & 63) >> 2;
  constexpr int AHEAD = 4;
  union Piece { bf16x8 v; s16x4 h[2]; };
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (uint32_t s0 = step0; s0 < step1; s0 += AHEAD) {
    Piece p[AHEAD], t[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const uint32_t k = min(128 * min(s0 + s, step1 - 1) + 8 * b, K - 8);
      p[s].v = *reinterpret_cast<const bf16x8*>(w + k);
      t[s].v = *reinterpret_cast<const bf16x8*>(x + k);
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      if (s0 + s >= step1) break;
      if (128 * (s0 + s) + 8 * b >= K) { p[s].v = bf16x8{}; t[s].v = bf16x8{}; }
#pragma unroll
      for (int e = 0; e < 2; ++e) acc = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(p[s].h[e], t[s].h[e], acc, 0, 0, 0);
    }
  }
  const auto add = [](float x, float y) { return x + y; };
#pragma unroll
  for (int e = 0; e < 4; ++e) {   // over the blocks: lanes 32, 16, 8 and 4 apart
    acc[e] = join16(join32(acc[e], add), add);
    acc[e] += rot16<8>(acc[e]);
    acc[e] += rot16<4>(acc[e]);
  }
  return acc;                     // in every block's lane j: the four rows' products with token j
}
template <int ACT>
__global__ __launch_bounds__(256) void k_glu_up_rows(UpArgs a) {
  __shared__ f32x4 part[4][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 3;
  const uint32_t f0 = blockIdx.x * 4, steps = (a.d + 127) / 128;
  const f32x4 acc = contract_rows(static_cast<const bf16_t*>(a.w.p) + (uint64_t)(f0 + i + (wave & 1) * a.F) * a.d, static_cast<const bf16_t*>(a.x.p) + (uint64_t)min((uint32_t)i, a.T - 1) * a.x.ld, a.d,
                                  share_of(steps, wave >> 1, 2), share_of(steps, (wave >> 1) + 1, 2));
  if (lane < 4) part[wave][lane] = acc;
  __syncthreads();
  if (threadIdx.x >= a.T) return;
  const f32x4 g = part[0][i] + part[2][i], u = part[1][i] + part[3][i];
  f32x4 h;
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = gate<bf16_t, ACT>(g[e]) * u[e];
  if (a.saved != nullptr) {
    unsigned char* const b = static_cast<unsigned char*>(a.saved) + (uint64_t)(f0 >> 4) * SAVED_BLOCK;
    const int at = 16 * ((f0 >> 2) & 3) + i;      // the lane of a fragment that has these four columns
    uint32_t wg[3], wu[3];
    pack24(g, wg); pack24(u, wu);
    *reinterpret_cast<uint4*>(b + at * 16) = make_uint4(wg[0], wg[1], wg[2], wu[0]);
    *reinterpret_cast<uint2*>(b + 1024 + at * 8) = make_uint2(wu[1], wu[2]);
  }
  *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.h) + (uint64_t)i * a.F + f0) = packed(h);
}
__global__ __launch_bounds__(512) void k_glu_down_rows(DownFewArgs a) {
  __shared__ f32x4 part[8][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 3;
  const uint32_t r0 = blockIdx.x * 4, steps = (a.F + 127) / 128;
  const f32x4 acc = contract_rows(a.w + (uint64_t)(r0 + i) * a.F, a.h + (uint64_t)min((uint32_t)i, a.T - 1) * a.F, a.F, share_of(steps, wave, 8), share_of(steps, wave + 1, 8));
  if (lane < 4) part[wave][lane] = acc;
  __syncthreads();
  if (threadIdx.x >= a.T) return;
  f32x4 s = part[0][i];
#pragma unroll
  for (int k = 1; k < 8; ++k) s += part[k][i];
  *reinterpret_cast<uint2*>(a.y + (uint64_t)i * a.ldy + r0) = packed(s);
}

// ---------------------------------------------------------------------------------------------------- launches
// us, silu and training for 8192 x 1024 x 4096, gelu and forward only for 4096 x 768 x 2048; + k_glu_join (matrix work alone at the 1515 TFLOP/s of a large product
// 91, 45, 45 and 227, and 17 and 9):
//               k_glu_up   y        k_glu_dgate   gradients      k_glu_up   y
//   256 x 256     155      68 + 16      127       307 + 15         28.8     22.4 + 10.7
//   256 x 128     158      58           130       347 + 10         27.6     18.0 + 7.3
//   128 x 128     212      76           126       346              33.1     17.2
//   64 x 64       268      110         149       604              44.9     21.2
// The large tiles read the least from LDS for a product and are bound by power in the loop (1.5 us of a slab; k_glu_up without its epilogue 126 us); what is left is
// the epilogue, whose 67 MB of h and 201 MB of g and u nothing hides: two workgroups to a CU, workgroups out of step and deeper stages gained nothing.  The
// smaller ones are for sizes whose large tiles do not fill the chip.  128 x 96 for y, whose 256 tiles the second size would fill exactly, takes 16.2 us.
typedef Tile<256, 256, 2, 4, 2, 0, 2, 0, 1> T256;
typedef Tile<256, 128, 4, 2, 3, 4, 2, 2, 1> T192;   // (the number between: 192; the weights' gradients in bf16 keep 3 of its registers in scratch, 16 bytes a lane)
typedef Tile<128, 128, 2, 4, 4, 4, 0, 1, 1> T128;
// Waves that only load also in the small ones: a wave that multiplies between its barriers asks for the next slab too late when there are two or three to a
// SIMD.  us without / with, forward and backward: fp32 512 x 256 x 688 50.2 / 45.5, 6299 x 264 x 528 220 / 205; bf16 300 x 768 x 2048 41.1 / 36.8, 700 x 512 x 1368
// 36.2 / 35.1, 2100 x 80 x 216 29.5 / 26.5.
typedef Tile<64, 64, 2, 2, 4, 4, 0, 1, 2> T64;
typedef Tile<32, 32, 2, 1, 6, 2, 0, 1, 3> T32;

template <auto KERNEL, typename T, typename A>
void launch_big(ProfScope& ps, hipStream_t st, uint32_t grid, const A& a) {
  static bool configured = false;   // per kernel: raise the dynamic LDS limit once
  if (!configured) {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
    configured = true;
  }
  launch_kernel(ps, KERNEL, grid, T::THREADS, T::LDS_BYTES, st, a);
}
TileOrder order_of(uint32_t M, uint32_t N, uint32_t bm, uint32_t bn) {
  TileOrder o{};
  o.tm = (M + bm - 1) / bm; o.tn = (N + bn - 1) / bn; o.tiles = o.tm * o.tn; o.per_xcd = (o.tiles + 7) / 8;
  return o;
}
template <int NT>
void launch_few(ProfScope& ps, hipStream_t st, const UpArgs& u, const DownFewArgs& w, int act) {
  const uint32_t up = (u.F + 15) / 16, down = (w.d + 15) / 16;
  if (act == GLU_GELU) launch_kernel(ps, k_glu_up_few<NT, GLU_GELU>, up, 512, 0, st, u);
  else launch_kernel(ps, k_glu_up_few<NT, GLU_SILU>, up, 512, 0, st, u);
  launch_kernel(ps, k_glu_down_few<NT>, down, DOWN_WAVES * 64, 0, st, w);
}
void launch_rows(ProfScope& ps, hipStream_t st, const UpArgs& u, const DownFewArgs& w, int act) {
  if (act == GLU_GELU) launch_kernel(ps, k_glu_up_rows<GLU_GELU>, u.F / 4, 256, 0, st, u);
  else launch_kernel(ps, k_glu_up_rows<GLU_SILU>, u.F / 4, 256, 0, st, u);
  launch_kernel(ps, k_glu_down_rows, w.d / 4, 512, 0, st, w);
}
template <typename T, typename E>
void launch_up(ProfScope& ps, hipStream_t st, UpArgs a, int act) {
  a.order = order_of(a.T, a.F, T::BM, T::BN / 2);
  if (act == GLU_GELU) launch_big<k_glu_up<T, E, GLU_GELU>, T>(ps, st, 8 * a.order.per_xcd, a);
  else launch_big<k_glu_up<T, E, GLU_SILU>, T>(ps, st, 8 * a.order.per_xcd, a);
}
template <typename T, typename E>
void launch_dgate(ProfScope& ps, hipStream_t st, DgateArgs a, int act) {
  a.order = order_of(a.T, a.F, T::BM, T::BN);
  if (act == GLU_GELU) launch_big<k_glu_dgate<T, E, GLU_GELU>, T>(ps, st, 8 * a.order.per_xcd, a);
  else launch_big<k_glu_dgate<T, E, GLU_SILU>, T>(ps, st, 8 * a.order.per_xcd, a);
}
// ---- which tile, and into how many parts a contraction is cut, by what a launch costs in us: pieces are started in their order, longest first, each on the
// workgroup slot that is free first; a piece takes its slabs' time, by how many workgroups share the CU, and `fixed`; parts are written, read and added.
// The times are those of operands with the contraction contiguous, and of the 64 x 64 and 32 x 32 tiles before these had waves that only load.  Where they are off, us
// planned / taken: y of 4096 x 768 x 2048 in 64 x 64 tiles 29.9 / 21.2; 67 MB of parts 26 / 14 to 16; the gradients of 8192 x 1024 x 4096, whose operands run along the other
// index (1.8 us of a 256 x 256 slab), 252 / 293 to 310.  Training, every launch in one tile / as planned: 1021 x 520 x 1368 52.0 at best (64 x 64) / 47.7,
// 4096 x 768 x 2048 156.2 (128 x 128) / 152.6.
struct TileCost { int tile, bm, bn, per_cu; double one, full, fixed; };   // us of a slab with one workgroup to a CU and with per_cu
constexpr TileCost COST16[] = {{256, 256, 256, 1, 1.50, 1.50, 6.0}, {192, 256, 128, 1, 0.85, 0.85, 4.0}, {128, 128, 128, 1, 0.52, 0.52, 2.5}, {64, 64, 64, 2, 0.27, 0.42, 1.5}, {32, 32, 32, 3, 0.20, 0.37, 1.2}};
constexpr TileCost COST32[] = {{128, 128, 128, 1, 2.00, 2.00, 3.0}, {64, 64, 64, 2, 0.72, 1.10, 2.0}, {32, 32, 32, 3, 0.32, 0.60, 1.5}};
constexpr double JOIN_LAUNCH = 3.5, JOIN_BYTES = 1.0 / 3.0e6;   // us; us a byte of the parts, written and read
constexpr uint32_t LEAST_SLABS = 4, MOST_PARTS = 16;            // of a part; of a tile
// Most bytes of parts that a launch may have, for the sizes in `a`, however they are cut: grows with the number of tokens.
uint64_t most_part_bytes(const TileCost& c, const ProductArgs& a, uint32_t depth) {
  uint64_t pieces = 0;
  for (int k = 0; k < a.count; ++k) {
    const uint64_t tiles = (uint64_t)((a.p[k].M + c.bm - 1) / c.bm) * ((a.p[k].N + c.bn - 1) / c.bn), slabs = (a.p[k].K + depth - 1) / depth;
    pieces += tiles * std::min<uint64_t>(MOST_PARTS, std::max<uint64_t>(1, slabs / LEAST_SLABS));
  }
  return std::min<uint64_t>(pieces, 512 * c.per_cu) * c.bm * c.bn * 4;
}
// The time of a launch of pieces in this order: `n` pieces of length us, ...
double makespan(const uint64_t* n, const double* length, int count, uint64_t slots) {
  // slots by the time they are free, a few distinct ones
  struct Free { double at; uint64_t n; } f[40] = {{0.0, slots}};
  int nf = 1;
  double end = 0.0;
  for (int k = 0; k < count; ++k) {
    uint64_t left = n[k];
    if (left > 8 * slots) {   // whole rounds at once
      const uint64_t rounds = left / slots - 4;
      for (int i = 0; i < nf; ++i) f[i].at += rounds * length[k];
      left -= rounds * slots;
    }
    while (left > 0) {
      int first = 0;
      for (int i = 1; i < nf; ++i) if (f[i].at < f[first].at) first = i;
      const uint64_t take = std::min(left, f[first].n);
      const double done = f[first].at + length[k];
      end = std::max(end, done);
      left -= take;
      f[first].n -= take;
      int same = -1;
      for (int i = 0; i < nf; ++i) if (std::abs(f[i].at - done) < 1e-9) same = i;
      if (same >= 0) f[same].n += take;
      else if (f[first].n == 0) f[first] = {done, take};
      else if (nf < 40) f[nf++] = {done, take};
      else f[first].n += take;   // (too many distinct times: as good as free)
      if (f[first].n == 0) f[first] = f[--nf];
    }
  }
  return end;
}
struct Plan { int tile; uint32_t parts[MAX_PRODUCTS]; int order[MAX_PRODUCTS]; double cost; };
int g_force_tile = 0, g_force_parts = 0;
template <typename E, int N>
Plan plan_products(const TileCost (&costs)[N], const ProductArgs& a, int force_tile) {
  Plan best{0, {}, {}, 0.0};
  for (const TileCost& c : costs) {
    if (force_tile != 0 && c.tile != force_tile) continue;
    const uint64_t room = most_part_bytes(c, a, DEPTH<E>);
    uint64_t tiles[MAX_PRODUCTS] = {};
    uint32_t slabs[MAX_PRODUCTS] = {}, most[MAX_PRODUCTS] = {1, 1, 1};
    for (int k = 0; k < a.count; ++k) {
      tiles[k] = (uint64_t)((a.p[k].M + c.bm - 1) / c.bm) * ((a.p[k].N + c.bn - 1) / c.bn);
      slabs[k] = (a.p[k].K + DEPTH<E> - 1) / DEPTH<E>;
      most[k] = std::min(MOST_PARTS, std::max(1u, slabs[k] / LEAST_SLABS));
    }
    const uint64_t slots = 256 * c.per_cu;
    for (uint32_t s0 = 1; s0 <= most[0]; s0 *= 2)
      for (uint32_t s1 = 1; s1 <= most[1]; s1 *= 2)
        for (uint32_t s2 = 1; s2 <= most[2]; s2 *= 2) {
          uint32_t parts[MAX_PRODUCTS] = {s0, s1, s2};
          if (g_force_parts != 0) for (int k = 0; k < a.count; ++k) parts[k] = std::min(most[k], (uint32_t)g_force_parts);
          uint64_t bytes = 0, pieces = 0;
          for (int k = 0; k < a.count; ++k) {
            pieces += tiles[k] * parts[k];
            if (parts[k] > 1) bytes += tiles[k] * parts[k] * c.bm * c.bn * 4;
          }
          if (bytes > room && g_force_parts == 0) continue;
          if (bytes > room) for (int k = 0; k < a.count; ++k) parts[k] = 1;
          Plan p{c.tile, {parts[0], parts[1], parts[2]}, {0, 1, 2}, 0.0};
          const double slab = pieces <= 256 ? c.one : c.full;   // with one more some CU has two, and the launch waits for it
          double length[MAX_PRODUCTS], sorted[MAX_PRODUCTS];
          uint64_t n[MAX_PRODUCTS];
          for (int k = 0; k < a.count; ++k) length[k] = (double)((slabs[k] + parts[k] - 1) / parts[k]) * slab + c.fixed;
          std::sort(p.order, p.order + a.count, [&](int x, int y) { return length[x] != length[y] ? length[x] > length[y] : x < y; });
          for (int k = 0; k < a.count; ++k) { sorted[k] = length[p.order[k]]; n[k] = tiles[p.order[k]] * parts[p.order[k]]; }
          p.cost = makespan(n, sorted, a.count, slots) + (bytes > 0 ? JOIN_LAUNCH + bytes * JOIN_BYTES : 0.0);
          if (best.tile == 0 || p.cost < best.cost) best = p;
        }
  }
  return best;
}
template <typename T, typename E, int KIND>
void launch_products(ProfScope& ps, hipStream_t st, const ProductArgs& in, const Plan& plan, float* part) {
  ProductArgs a{};
  a.count = in.count;
  uint32_t blocks = 0;
  uint64_t join = 0;
  for (int k = 0; k < a.count; ++k) {
    Product& p = a.p[k];
    p = in.p[plan.order[k]];
    p.parts = plan.parts[plan.order[k]];
    p.tm = (p.M + T::BM - 1) / T::BM; p.tn = (p.N + T::BN - 1) / T::BN; p.slabs = (p.K + DEPTH<E> - 1) / DEPTH<E>; p.first = blocks; p.part = part;
    const uint32_t pieces = p.tm * p.tn * p.parts;
    blocks += (pieces + 7) / 8 * 8;
    if (p.parts > 1) { part += (uint64_t)pieces * T::BM * T::BN; join += (uint64_t)p.tm * p.tn * (T::WAVES * T::XT * T::YT / 2); }
  }
  launch_big<k_glu_product<T, E, KIND>, T>(ps, st, blocks, a);
  if (join > 0) launch_kernel(ps, k_glu_join<T>, (uint32_t)((join + 3) / 4), 256, 0, st, a);
}
template <typename E, typename F>
void with_tile(int tile, F f) {
  if constexpr (sizeof(E) == 2) {
    if (tile == 256) return f(T256{});
    if (tile == 192) return f(T192{});
  }
  if (tile >= 128) f(T128{});
  else if (tile == 64) f(T64{});
  else f(T32{});
}
template <typename E, int KIND>
void products(ProfScope& ps, hipStream_t st, const ProductArgs& a, float* part) {
  Plan plan;
  if constexpr (sizeof(E) == 2) plan = plan_products<E>(COST16, a, g_force_tile);
  else plan = plan_products<E>(COST32, a, std::min(g_force_tile, 128));
  with_tile<E>(plan.tile, [&](auto t) { launch_products<decltype(t), E, KIND>(ps, st, a, plan, part); });
}
// the tile of a product that is not cut
template <typename E>
int whole_tile(int64_t M, int64_t N, int64_t K) {
  ProductArgs a{};
  a.count = 1; a.p[0].M = (uint32_t)M; a.p[0].N = (uint32_t)N; a.p[0].K = (uint32_t)K;
  double best = 0.0;
  int tile = 0;
  auto look = [&](const TileCost& c) {
    const uint64_t n = (uint64_t)((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn), slots = 256 * c.per_cu;
    const double length = (double)((K + DEPTH<E> - 1) / DEPTH<E>) * (n <= 256 ? c.one : c.full) + 2 * c.fixed;
    const double cost = (double)((n + slots - 1) / slots) * length;
    if (tile == 0 || cost < best) { tile = c.tile; best = cost; }
  };
  if constexpr (sizeof(E) == 2) for (const TileCost& c : COST16) look(c);
  else for (const TileCost& c : COST32) look(c);
  return g_force_tile == 0 ? tile : sizeof(E) == 4 ? std::min(g_force_tile, 128) : g_force_tile;
}
template <typename E>
size_t part_bytes(const ProductArgs& a) {
  uint64_t most = 256;
  if constexpr (sizeof(E) == 2) for (const TileCost& c : COST16) most = std::max(most, most_part_bytes(c, a, DEPTH<E>));
  else for (const TileCost& c : COST32) most = std::max(most, most_part_bytes(c, a, DEPTH<E>));
  return most;
}
size_t up256(size_t b) { return (b + 255) / 256 * 256; }

template <typename E>
size_t forward_bytes(int64_t T, int d, int F) {
  ProductArgs s{};
  s.count = 1; s.p[0].M = (uint32_t)T; s.p[0].N = d; s.p[0].K = F;
  return part_bytes<E>(s);
}
template <typename E>
size_t backward_bytes(int64_t T, int d, int F) {
  ProductArgs s{};
  s.count = 3; s.p[0].M = (uint32_t)T; s.p[0].N = d; s.p[0].K = 2 * F; s.p[1].M = 2 * F; s.p[1].N = d; s.p[1].K = (uint32_t)T; s.p[2].M = d; s.p[2].N = F; s.p[2].K = (uint32_t)T;
  return up256((size_t)T * 2 * F * sizeof(E)) + part_bytes<E>(s);
}

template <typename E>
void forward(hipStream_t st, const GluFfnArgs& g, void* workspace) {
  constexpr bool BF16 = sizeof(E) == 2;
  const uint32_t T = (uint32_t)g.T, d = g.d, F = g.F;
  ProfScope ps(st, BF16 ? F_GEMM_NT : F_GEMM_F32, 6.0 * T * (double)d * F);
  UpArgs u{};
  u.x = Operand{g.x, (uint32_t)g.ldx, T}; u.w = Operand{g.w_in, d, F};
  u.T = T; u.F = F; u.d = d; u.h = g.hidden; u.saved = g.saved;
  // Few tokens without tiles.  us a call, this way / by tiles: 512 x 1368 1 token 10.2 / 13.7, 16 11.4 / 14.0, 32 12.2 / 14.3, 48 14.7 / 14.5; 1024 x 4096 1
  // 9.5 / 19.5, 5 13.1 / 19.6, 16 15.4 / 19.7, 32 20.1 / 20.2, 48 25.6 / 20.2; 2048 x 5504 1 15.0 / 27.2, 4 19.6 / 27.3, 5 27.7 / 27.3, 16 33.5 / 27.6.
  if (BF16 && g_force_tile == 0 && (T <= 4 || (T <= 32 && (uint64_t)d * F <= (1u << 22)))) {
    const DownFewArgs w{(const bf16_t*)g.hidden, (const bf16_t*)g.w_out, T, F, d, (bf16_t*)g.y, (uint32_t)g.ldy};
    if (T <= 4) launch_rows(ps, st, u, w, g.act);
    else if (T <= 16) launch_few<1>(ps, st, u, w, g.act);
    else launch_few<2>(ps, st, u, w, g.act);
    return;
  }
  with_tile<E>(whole_tile<E>(T, 2 * (int64_t)F, d), [&](auto t) { launch_up<decltype(t), E>(ps, st, u, g.act); });
  ProductArgs s{};
  s.count = 1;
  Product& p = s.p[0];
  p.A = Operand{g.hidden, F, T}; p.B = Operand{g.w_out, F, d};
  p.M = T; p.N = d; p.K = F; p.C = g.y; p.ldc = (uint32_t)g.ldy; p.c32 = !BF16;
  products<E, 0>(ps, st, s, (float*)workspace);
}

template <typename E>
void backward(hipStream_t st, const GluFfnGradArgs& g, void* workspace) {
  constexpr bool BF16 = sizeof(E) == 2;
  const uint32_t T = (uint32_t)g.T, d = g.d, F = g.F;
  void* const dpre = workspace;
  ProfScope ps(st, BF16 ? F_GEMM_NN : F_GEMM_F32, 12.0 * T * (double)d * F);
  DgateArgs e{};
  e.dy = Operand{g.dy, (uint32_t)g.lddy, T}; e.w = Operand{g.w_out, F, F};
  e.T = T; e.F = F; e.d = d; e.saved = g.saved; e.dpre = dpre;
  with_tile<E>(whole_tile<E>(T, F, d), [&](auto t) { launch_dgate<decltype(t), E>(ps, st, e, g.act); });
  ProductArgs s{};
  s.count = 3;
  s.p[0].A = Operand{dpre, 2 * F, T}; s.p[0].B = Operand{g.w_in, d, d};
  s.p[0].M = T; s.p[0].N = d; s.p[0].K = 2 * F; s.p[0].C = g.dx; s.p[0].ldc = (uint32_t)g.lddx; s.p[0].c32 = !BF16;
  s.p[1].A = Operand{dpre, 2 * F, 2 * F}; s.p[1].B = Operand{g.x, (uint32_t)g.ldx, d};
  s.p[1].M = 2 * F; s.p[1].N = d; s.p[1].K = T; s.p[1].C = g.dw_in; s.p[1].ldc = d;
  s.p[2].A = Operand{g.dy, (uint32_t)g.lddy, d}; s.p[2].B = Operand{g.hidden, F, F};
  s.p[2].M = d; s.p[2].N = F; s.p[2].K = T; s.p[2].C = g.dw_out; s.p[2].ldc = F;
  for (int k = 1; k < 3; ++k) { s.p[k].strided_a = 1; s.p[k].c32 = g.dw_fp32; }
  products<E, 1>(ps, st, s, (float*)((char*)dpre + up256((size_t)T * 2 * F * sizeof(E))));
}
// fp32 operands that the tiles can load: rows in pieces of 16 bytes
bool pieces32(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 4 == 0; }
}  // namespace

bool glu_ffn_force_tile(int t) {
  const int tile = t % 1000;
  if (t < 0 || (tile != 0 && std::none_of(std::begin(COST16), std::end(COST16), [&](const TileCost& c) { return c.tile == tile; }))) return false;   // no plan would have it
  g_force_tile = tile; g_force_parts = t / 1000;
  return true;
}

size_t glu_ffn_saved_bytes(int64_t T, int F) { return (size_t)((T + 15) / 16) * ((F + 15) / 16) * SAVED_BLOCK; }
size_t glu_ffn_bytes(int64_t T, int d, int F) { return forward_bytes<bf16_t>(T, d, F); }
size_t glu_ffn_grad_bytes(int64_t T, int d, int F) { return backward_bytes<bf16_t>(T, d, F); }
void launch_glu_ffn(hipStream_t st, const GluFfnArgs& g, void* workspace) { forward<bf16_t>(st, g, workspace); }
void launch_glu_ffn_grad(hipStream_t st, const GluFfnGradArgs& g, void* workspace) { backward<bf16_t>(st, g, workspace); }

size_t glu_ffn_f32_saved_bytes(int64_t T, int F) { return (size_t)T * 2 * F * 4; }
size_t glu_ffn_f32_bytes(int64_t T, int d, int F) { return std::max(forward_bytes<float>(T, d, F), glu_ffn_plain_bytes(T, F)); }
size_t glu_ffn_f32_grad_bytes(int64_t T, int d, int F) { return std::max(backward_bytes<float>(T, d, F), glu_ffn_plain_grad_bytes(T, F)); }
// fp32 whose rows are pieces of 16 bytes goes through the tiles: 512 x 256 x 688 with gelu 45.5 us forward and backward, of any width, stride and alignment through the
// products of the MLPs: 512 x 255 x 687 69 us; both keep g and u in the same place, so a forward call of the one
// may be followed by a backward call of the other.
void launch_glu_ffn_f32(hipStream_t st, const GluFfnArgs& g, void* workspace) {
  const bool tiles = g.d % 4 == 0 && g.F % 4 == 0 && pieces32(g.x, g.ldx) && pieces32(g.y, g.ldy) && pieces32(g.w_in, 0) && pieces32(g.w_out, 0) && pieces32(g.hidden, 0);
  if (tiles) forward<float>(st, g, workspace);
  else launch_glu_ffn_plain(st, g, workspace);
}
void launch_glu_ffn_grad_f32(hipStream_t st, const GluFfnGradArgs& g, void* workspace) {
  const bool tiles = g.d % 4 == 0 && g.F % 4 == 0 && pieces32(g.x, g.ldx) && pieces32(g.dy, g.lddy) && pieces32(g.dx, g.lddx) && pieces32(g.w_in, 0) && pieces32(g.w_out, 0) &&
                     pieces32(g.hidden, 0) && pieces32(g.dw_in, 0) && pieces32(g.dw_out, 0);
  if (tiles) backward<float>(st, g, workspace);
  else launch_glu_ffn_grad_plain(st, g, workspace);
}

}  // namespace sama
