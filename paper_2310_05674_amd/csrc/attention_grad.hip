// Gradients of attention (attention.hip), from q, k, v, the output o, its gradient do and the logarithm of each row's sum:
//   p_ij = exp(s_ij - lse_i),  dp_ij = do_i . v_j,  delta_i = do_i . o_i,  ds_ij = p_ij (dp_ij - delta_i) (1 - tanh^2 if capped)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,   i over all queries and heads that share k_j and v_j.
// Scores are formed again, in two launches: one walks the keys for a tile of rows (dq), one the rows for a tile of keys (dk, dv).  That is seven products where five
// would do if one launch made both; but then one side would have to be added up in memory by workgroups as they come, in an order of their own.
// k_attention_delta goes ahead: delta, and what else the second launch needs of each row, laid out in the order in which it is read.
//
// Bound by products where texts are long: 8192 causal tokens in bf16, 16 heads of 128 on 8 key heads, take 383 us for dq (6 D operations a pair, 1077 TFLOP/s) and 652 for dk and dv (8 D, 843).
// Short texts are bound by each workgroup's chain of spans, first loads, tiles and the join of its groups: 8111 tokens in 23 texts, 16 heads of 64 on 4, 48 and 100 us.
#include <algorithm>
#include <cmath>
#include "attention_tiles.h"

namespace sama {
namespace {
using namespace attn;

// Of each row of a group (GROUP packed rows): planes of 64 words.
enum { LSE, DELTA, FIRST, END, AT, SLOPE, PLANES };
constexpr int RECORD = PLANES * GROUP * 4;   // bytes of a group
struct Rows {
  uint32_t* record;   // [Hk][groups][PLANES][GROUP]; LSE and SLOPE in units of log 2
  int2* range;        // [groups]: first key and end of what a group's rows see
  int groups;
};

// o was rounded to the gradients' type, and delta with it: off by 2^-9 |do| |o| or so.  A row of many keys, whose o is a mean, hardly shows that, three keys do: dq off by 0.0046 of
// its norm.  So a 16-bit row of at most FEW keys has delta = sum_j p_ij dp_ij from its keys themselves. 60 drawn cases from one token to 3000: at most 0.0046 without, 0.0027 with FEW
// = 8 or 16.  The launch takes 11.9 us with it and 8.5 without (8111 packed tokens, 16 heads of 64).
constexpr int FEW = 8;   // two a lane

template <typename E, int SHAPE>
__global__ __launch_bounds__(256) void k_attention_delta(AttentionArgs a, Rows rows) {
  const int G = a.Hq / a.Hk, tokens = GROUP / G, hk = blockIdx.x % a.Hk, group = blockIdx.x / a.Hk;
  const int r = threadIdx.x >> 2, part = threadIdx.x & 3;
  const int64_t query = (int64_t)group * tokens + r / G;
  const int head = hk * G + r % G;
  int2 span = make_int2(0, 0);
  if (r < tokens * G && query < a.Tq) span = span_of(a.spans, query, (int)a.Tk);
  const bool some = span.x < span.y;
  float sum = 0.f;
  if (some) {
    const E* const o = static_cast<const E*>(a.out.p) + query * a.out.ld + head * a.out.hs;
    const E* const d = static_cast<const E*>(a.dout.p) + query * a.dout.ld + head * a.dout.hs;
    Frag<E> x[4], y[4];   // all on their way together
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = 8 * part + 32 * u;
      x[u] = i < a.D ? load_fragment<E>(o + i) : zero_fragment<E>(); y[u] = i < a.D ? load_fragment<E>(d + i) : zero_fragment<E>();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)x[u][e], (float)y[u][e], sum);
  }
  const float lse = some ? a.lse[query * a.Hq + head] * LOG2E : 0.f, slope = some && a.slopes != nullptr ? a.slopes[head] * LOG2E : 0.f;
  const int at = some ? (a.at != nullptr ? a.at[query] : (int)query) : 0;
  sum += __shfl_xor(sum, 1); sum += __shfl_xor(sum, 2);
  if (some && sizeof(E) == 2 && span.y - span.x <= FEW) {
    sum = 0.f;
    const E* const q = static_cast<const E*>(a.q.p) + query * a.q.ld + head * a.q.hs;
    const E* const d = static_cast<const E*>(a.dout.p) + query * a.dout.ld + head * a.dout.hs;
    const E* const k = static_cast<const E*>(a.k.p) + hk * a.k.hs;
    const E* const v = static_cast<const E*>(a.v.p) + hk * a.v.hs;
    const Scores<E, SHAPE> score(a.scale, a.cap);
    // two keys a lane, with as many loads on their way as there are registers for: one after the other, the keys of one such row are all that the launch waits for
    const int j0 = span.x + part, j1 = j0 + 4;
    const int64_t in0 = min(j0, span.y - 1), in1 = min(j1, span.y - 1);
    const E *const k0 = k + in0 * a.k.ld, *const k1 = k + in1 * a.k.ld, *const v0 = v + in0 * a.v.ld, *const v1 = v + in1 * a.v.ld;
    float s0 = 0.f, s1 = 0.f, dp0 = 0.f, dp1 = 0.f;
    for (int i = 0; i < a.D; i += 32) {
      Frag<E> x[4], y[4], xk0[4], xk1[4], xv0[4], xv1[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int c = min(i + 8 * u, a.D - 8);
        x[u] = load_fragment<E>(q + c); y[u] = load_fragment<E>(d + c);
        xk0[u] = load_fragment<E>(k0 + c); xk1[u] = load_fragment<E>(k1 + c); xv0[u] = load_fragment<E>(v0 + c); xv1[u] = load_fragment<E>(v1 + c);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i + 8 * u >= a.D) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s0 = fmaf((float)x[u][e], (float)xk0[u][e], s0); s1 = fmaf((float)x[u][e], (float)xk1[u][e], s1);
          dp0 = fmaf((float)y[u][e], (float)xv0[u][e], dp0); dp1 = fmaf((float)y[u][e], (float)xv1[u][e], dp1);
        }
      }
    }
    float bend;
    if (j0 < span.y) sum = __builtin_amdgcn_exp2f(score(s0, slope, (float)(at - j0), bend) - lse) * dp0;
    if (j1 < span.y) sum = fmaf(__builtin_amdgcn_exp2f(score(s1, slope, (float)(at - j1), bend) - lse), dp1, sum);
    sum += __shfl_xor(sum, 1); sum += __shfl_xor(sum, 2);
  }
  if (part == 0) {
    uint32_t* const to = rows.record + ((int64_t)hk * rows.groups + group) * (PLANES * GROUP) + r;
    to[LSE * GROUP] = __float_as_uint(lse);
    to[DELTA * GROUP] = __float_as_uint(sum);
    to[FIRST * GROUP] = span.x; to[END * GROUP] = span.y;
    to[AT * GROUP] = at;
    to[SLOPE * GROUP] = __float_as_uint(slope);
  }
  if (hk == 0) {   // the range, by the rows of each wave and then all
    __shared__ int s_lo[4], s_hi[4];
    const int lo = wave_min(some ? span.x : 0x7fffffff), hi = wave_max(span.y);
    if ((threadIdx.x & 63) == 0) { s_lo[threadIdx.x >> 6] = lo; s_hi[threadIdx.x >> 6] = hi; }
    __syncthreads();
    if (threadIdx.x == 0) rows.range[group] = make_int2(min(min(s_lo[0], s_lo[1]), min(s_lo[2], s_lo[3])), max(max(s_hi[0], s_hi[1]), max(s_hi[2], s_hi[3])));
  }
}

// ------------------------------------------------------------------------------------------------------ dq
template <typename E, int DP_, int WM_>
struct QConfig {
  static constexpr int DP = DP_, WM = WM_;
  static constexpr int KG = WM > 2 ? 1 : WM > 1 || sizeof(E) * DP > 256 ? 2 : 4;
  static constexpr int NS = WM > 2 && sizeof(E) * DP <= 256 ? 2 : 1;
  static constexpr int WAVES = WM * KG, THREADS = WAVES * 64, BM = 32 * WM, BK = 32 * NS * KG;
  static constexpr int KV = BK * DP * (int)sizeof(E), JOIN = KG == 1 ? 0 : WAVES * DP * 32 * 4, LDS = 4 * KV > JOIN ? 4 * KV : JOIN;
  static constexpr int PER_EU = sizeof(E) * DP <= 256 ? 2 : 1;
  static_assert(LDS <= LDS_MAX, "LDS");
};
template <typename E, typename C, int SHAPE>
__global__ __launch_bounds__(C::THREADS, C::PER_EU) void k_attention_dq(AttentionArgs a, Rows recs, int tiles) {
  extern __shared__ __align__(1024) unsigned char smem[];
  typedef Tile<E, C::DP> T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int rw = wave / C::KG, kg = wave % C::KG;
  const int G = a.Hq / a.Hk, rows = (int)a.Tq * G, D = a.D, tokens = GROUP / G;
  const int hk = blockIdx.x % a.Hk, tile = tiles - 1 - blockIdx.x / a.Hk;
  const int row = tile * C::BM + rw * 32 + (lane & 31), query = min(row, rows - 1) / G, in = min(row, rows - 1) % G, head = hk * G + in;
  const int2 span = span_of(a.spans, query, (int)a.Tk);
  const int r0 = min(tile * C::BM + lane % C::BM, rows - 1), r1 = min(tile * C::BM + (lane + 64) % C::BM, rows - 1);
  const int2 s0 = span_of(a.spans, r0 / G, (int)a.Tk), s1 = span_of(a.spans, r1 / G, (int)a.Tk);
  const int lo = __builtin_amdgcn_readfirstlane(wave_min(min(s0.x < s0.y ? s0.x : 0x7fffffff, s1.x < s1.y ? s1.x : 0x7fffffff)));
  const int hi = __builtin_amdgcn_readfirstlane(wave_max(max(s0.y, s1.y)));
  const int end = hi > lo ? (hi - lo + C::BK - 1) / C::BK : 0;
  auto seen_from = [&](int i) {
    for (; i < end; ++i) {
      const int k0 = lo + i * C::BK;
      if (__any((s0.x < k0 + C::BK && s0.y > k0) || (s1.x < k0 + C::BK && s1.y > k0))) break;
    }
    return i;
  };
  Loads<E, C::DP, C::BK, C::WAVES> lk, lv;
  lk.init(a.k.ld, 0, 1, D, wave, lane);
  lv.init(a.v.ld, 0, 1, D, wave, lane);
  const E* const kp = static_cast<const E*>(a.k.p) + hk * a.k.hs;
  const E* const vp = static_cast<const E*>(a.v.p) + hk * a.v.hs;
  const uint32_t lds = lds_address(smem), row_lane = T::row_lane(lane), column_lane = T::column_lane(lane);
  const Source ks(kp + (int64_t)lo * a.k.ld, ((a.Tk - 1 - lo) * a.k.ld + D) * (int64_t)sizeof(E), C::BK * a.k.ld * (int64_t)sizeof(E));
  const Source vs(vp + (int64_t)lo * a.v.ld, ((a.Tk - 1 - lo) * a.v.ld + D) * (int64_t)sizeof(E), C::BK * a.v.ld * (int64_t)sizeof(E));
  int t = seen_from(0);
  if (t < end) { lk.issue(lds, ks.tile(t), wave); lv.issue(lds + C::KV, vs.tile(t), wave); }

  Frag<E> q[T::KS], d[T::KS];
  {
    const E* const p = static_cast<const E*>(a.q.p) + query * a.q.ld + head * a.q.hs;
    const E* const g = static_cast<const E*>(a.dout.p) + query * a.dout.ld + head * a.dout.hs;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
      q[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(p + 16 * ks + 8 * h) : zero_fragment<E>();
      d[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(g + 16 * ks + 8 * h) : zero_fragment<E>();
    }
  }
  const uint32_t* const rec = recs.record + ((int64_t)hk * recs.groups + query / tokens) * (PLANES * GROUP) + query % tokens * G + in;
  const float lse = __uint_as_float(rec[LSE * GROUP]), delta = __uint_as_float(rec[DELTA * GROUP]);
  const float slope = SHAPE & BIASED ? __uint_as_float(rec[SLOPE * GROUP]) : 0.f;
  const int at = SHAPE & BIASED ? (int)rec[AT * GROUP] : 0;
  arrived(q); arrived(d);
  const Scores<E, SHAPE> score(a.scale, a.cap);
  f32x16 dq[T::DF];
#pragma unroll
  for (int df = 0; df < T::DF; ++df) dq[df] = zeros();

  for (int stage = 0; t < end; stage ^= 1) {
    const int next = seen_from(t + 1);
    wait_loads();
    const u32x4 next_k = next < end ? ks.tile(next) : Source::nothing(), next_v = next < end ? vs.tile(next) : Source::nothing();
    const uint32_t next_at = lds + (stage ^ 1) * 2 * C::KV;
    constexpr int LOADS = (lk.N + lv.N) / C::NS;   // in each subtile
    auto load = [&](int i) { if (i < lk.N) lk.issue_one(i, next_at, next_k, wave); else lv.issue_one(i - lk.N, next_at + C::KV, next_v, wave); };
    const uint32_t k_rows = lds + stage * 2 * C::KV + row_lane, v_rows = k_rows + C::KV, k_cols = lds + stage * 2 * C::KV + column_lane;
    const int first = lo + t * C::BK + kg * 32 * C::NS;
    t = next;
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      const int k0 = first + 32 * n, row0 = (kg * C::NS + n) * 32;
      f32x16 s, dp;
      pipeline<2 * T::KS, ROWS_AHEAD<E>, Frag<E>>([&](int i) { return T::rows(i < T::KS ? k_rows : v_rows, row0, i % T::KS); }, [&](int i, const Frag<E>& x) {
        if (i < T::KS) s = mma(x, q[i], i == 0 ? zeros() : s);
        else dp = mma(x, d[i - T::KS], i == T::KS ? zeros() : dp);
#pragma unroll
        for (int j = i * LOADS / (2 * T::KS); j < (i + 1) * LOADS / (2 * T::KS); ++j) load(n * LOADS + j);
      });
      if (!__any(span.x < k0 + 32 && span.y > k0)) continue;   // (not sooner: the loads are every wave's)
      Columns<E, C::DP, 2> columns;
      columns.fetch(k_cols, row0);
      const bool whole = __all(span.x <= k0 && span.y >= k0 + 32);
      const float away = (float)(at - k0 - 4 * h);
      uint32_t seen = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float bend = 1.f;
        const float x = score(s[r], slope, away - (float)(8 * (r >> 2) + (r & 3)), bend);
        const float p = __builtin_amdgcn_exp2f(x - lse);
        s[r] = SHAPE & CAPPED ? p * (dp[r] - delta) * bend : p * (dp[r] - delta);
      }
      if (!whole) {
        seen = seen_keys(span, k0, h);
        const uint32_t matters = span.y - span.x > 1 ? seen : 0;   // a single key has probability 1, whatever its score
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = where_seen(matters, r, s[r], 0.f);
      }
      Frag<E> ds[2] = {fragment<E>(s, 0), fragment<E>(s, 1)};
      add_product<E, C::DP, 2>(dq, columns, ds, whole || all_finite<E, C::DP>(k_rows, row0), seen, k_cols, row0);
    }
  }
  drain_loads();
  if constexpr (C::KG > 1) {   // the groups' sums; a wave then has 32 of the columns
    __syncthreads();
    float* const part = reinterpret_cast<float*>(smem) + rw * C::KG * C::DP * 32;   // [KG][DP][32]
#pragma unroll
    for (int df = 0; df < T::DF; ++df)
#pragma unroll
      for (int r = 0; r < 16; ++r) part[(kg * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)] = dq[df][r];
    __syncthreads();
#pragma unroll
    for (int df = 0; df < T::DF; ++df) {
      if (df % C::KG != kg) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < C::KG; ++g) x += part[(g * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)];
        dq[df][r] = x;
      }
    }
  }
  if (row >= rows) return;
  E* const to = const_cast<E*>(static_cast<const E*>(a.dq.p)) + query * a.dq.ld + head * a.dq.hs;
#pragma unroll
  for (int df = 0; df < T::DF; ++df) if (C::KG == 1 || df % C::KG == kg) store_columns<E>(to, df, D, dq[df], a.scale, h);
}

// ------------------------------------------------------------------------------------------------------ dk, dv
// Tiles of GROUPS groups of rows, one after the other, that have rows which see one of the keys [first, end): their numbers, then -1.
template <int GROUPS> struct Steps {
  const int2* range; int groups, first, end, at = 0;
  uint64_t ahead = 0;                                // which of the 64 tiles before `at` are still to come
  __device__ __forceinline__ Steps(const Rows& r, int first_, int end_) : range(r.range), groups(r.groups), first(first_), end(end_) {}
  __device__ __forceinline__ int next(int lane) {
    while (ahead == 0) {
      if (at * GROUPS >= groups) return -1;
      bool any = false;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int group = (at + lane) * GROUPS + g;
        if (group < groups) { const int2 s = range[group]; any |= s.x < end && s.y > first; }
      }
      ahead = __ballot(any);
      at += 64;
    }
    const int bit = __builtin_ctzll(ahead);
    ahead &= ahead - 1;
    return at - 64 + bit;
  }
};
template <typename E> __device__ __forceinline__ Source rows_source(const Heads& x, const AttentionArgs& a, int hk, int groups) {
  const int G = a.Hq / a.Hk;
  return Source(static_cast<const E*>(x.p) + (int64_t)hk * G * x.hs, ((a.Tq - 1) * x.ld + (G - 1) * x.hs + a.D) * (int64_t)sizeof(E), groups * (GROUP / G) * x.ld * (int64_t)sizeof(E));
}
template <typename C> __device__ __forceinline__ void load_records(u32x4 from, uint32_t stage_at, int wave, int lane) {
#pragma unroll
  for (int i = 0; i < C::REC_LOADS; ++i) {
    const uint32_t at = (i * C::WAVES + wave) * 1024;
    if (at < C::REC) load_to_lds(stage_at + 2 * C::QD + at, at + lane * 16 < C::GROUPS * RECORD ? at + lane * 16 : NOWHERE, from);
  }
}
// Of a subtile's rows, as bits for a lane's registers: those that see the key, and of them those that see another one too: a single key has probability 1, whatever its score,
// so its ds is zero.
__device__ __forceinline__ uint2 seen_rows(const uint32_t* rec, int key, int h) {
  uint2 bits = make_uint2(0, 0);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int at = 8 * q + 4 * h;
    const u32x4 from = *reinterpret_cast<const u32x4*>(rec + FIRST * GROUP + at), to = *reinterpret_cast<const u32x4*>(rec + END * GROUP + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bit = key >= (int)from[i] && key < (int)to[i] ? 1u << seen_bit(4 * q + i) : 0;
      bits.x |= bit;
      bits.y |= to[i] - from[i] > 1 ? bit : 0;
    }
  }
  return bits;
}

// Waves work in pairs on the same 32 keys: the first has k in registers, forms the scores and p, and adds up dv; the second has v, forms dp and, with the first one's p
// through LDS, ds, and adds up dk.  One wave for both needs 300 registers at a width of 128, which leaves one to a SIMD and nothing to do while it waits.
template <typename E, int DP_, int WK_, int QG_, int NS_>
struct KConfig {
  static constexpr int DP = DP_, WK = WK_, QG = QG_, NS = NS_;                    // pairs side by side over keys, over rows; 32 rows each of a pair's part of a tile
  static constexpr int PAIRS = WK * QG, WAVES = 2 * PAIRS, THREADS = WAVES * 64, KEYS = 32 * WK, BQ = 32 * NS * QG, GROUPS = BQ / GROUP;
  static constexpr int QD = BQ * DP * (int)sizeof(E), REC = (GROUPS * RECORD + 1023) / 1024 * 1024, STAGE = 2 * QD + REC;
  static constexpr int P = 2 * STAGE, LDS = P + PAIRS * NS * 4096;                // the pairs' p, fp32
  static constexpr int REC_LOADS = (REC / 1024 + WAVES - 1) / WAVES;
  static_assert(BQ % GROUP == 0 && LDS <= LDS_MAX && 2 * QG * DP * 32 * 4 <= LDS, "LDS");
};
template <typename E, typename C, int SHAPE>
__global__ __launch_bounds__(C::THREADS, 2) void k_attention_dkv(AttentionArgs a, Rows recs) {
  extern __shared__ __align__(1024) unsigned char smem[];
  typedef Tile<E, C::DP> T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int pair = wave % C::PAIRS, kw = pair / C::QG, qg = pair % C::QG;
  const bool second = wave >= C::PAIRS;   // (waves four apart share a SIMD: one of either kind, which want its units at different times)
  const int G = a.Hq / a.Hk, D = a.D, tokens = GROUP / G;
  const int hk = blockIdx.x % a.Hk, k_first = blockIdx.x / a.Hk * C::KEYS;   // the first keys, which most rows of a causal text see, first
  const int key0 = k_first + kw * 32, key = key0 + (lane & 31);
  Steps<C::GROUPS> step_list(recs, k_first, k_first + C::KEYS);
  Loads<E, C::DP, C::BQ, C::WAVES> lq, ld;
  lq.init(a.q.ld, a.q.hs, G, D, wave, lane);
  ld.init(a.dout.ld, a.dout.hs, G, D, wave, lane);
  const uint32_t lds = lds_address(smem), row_lane = T::row_lane(lane), column_lane = T::column_lane(lane);
  const Source qs = rows_source<E>(a.q, a, hk, C::GROUPS), ds = rows_source<E>(a.dout, a, hk, C::GROUPS);
  const Source rs(recs.record + (int64_t)hk * recs.groups * (PLANES * GROUP), (int64_t)recs.groups * RECORD, C::GROUPS * RECORD);
  int step = step_list.next(lane);
  if (step >= 0) { load_records<C>(rs.tile(step), lds, wave, lane); lq.issue(lds, qs.tile(step), wave); ld.issue(lds + C::QD, ds.tile(step), wave); }

  Frag<E> f[T::KS];   // the keys' k, or v
  {
    const Heads& from = second ? a.v : a.k;
    const E* const p = static_cast<const E*>(from.p) + min((int64_t)key, a.Tk - 1) * from.ld + hk * from.hs;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) f[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(p + 16 * ks + 8 * h) : zero_fragment<E>();
  }
  arrived(f);
  const Scores<E, SHAPE> score(a.scale, a.cap);
  float* const shared_p = reinterpret_cast<float*>(smem + C::P) + pair * C::NS * 1024 + lane * 4;
  f32x16 sum[T::DF];   // dv, or dk
#pragma unroll
  for (int df = 0; df < T::DF; ++df) sum[df] = zeros();

  for (int stage = 0; step >= 0; stage ^= 1) {
    const int next = step_list.next(lane);
    wait_loads();
    const bool more = next >= 0;
    const u32x4 next_q = more ? qs.tile(next) : Source::nothing(), next_d = more ? ds.tile(next) : Source::nothing();
    const uint32_t next_at = lds + (stage ^ 1) * C::STAGE;
    if (more) load_records<C>(rs.tile(next), next_at, wave, lane);
    step = next;
    const uint32_t q_tile = lds + stage * C::STAGE, d_tile = q_tile + C::QD;
    const uint32_t rows = (second ? d_tile : q_tile) + row_lane, other_rows = (second ? q_tile : d_tile) + row_lane, columns_at = (second ? q_tile : d_tile) + column_lane;
    const uint32_t* const recs_at = reinterpret_cast<const uint32_t*>(smem + stage * C::STAGE + 2 * C::QD);
    auto record = [&](int n) { const int row0 = (qg * C::NS + n) * 32; return recs_at + row0 / GROUP * (PLANES * GROUP) + row0 % GROUP; };
    f32x16 s[C::NS];
    f32x4 stat[C::NS][4];                        // lse, or delta, of the rows that a lane's registers are of
    Frag<E> b[C::NS][2];
    int first[C::NS], end[C::NS];
#pragma unroll
    for (int n = 0; n < C::NS; ++n) { first[n] = (int)record(n)[FIRST * GROUP + (lane & 31)]; end[n] = (int)record(n)[END * GROUP + (lane & 31)]; }
#pragma unroll
    for (int n = 0; n < C::NS; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) stat[n][q] = *reinterpret_cast<const f32x4*>(record(n) + (second ? DELTA : LSE) * GROUP + 8 * q + 4 * h);
    constexpr int STEPS = C::NS * T::KS, LOADS = lq.N + ld.N;
    pipeline<STEPS, ROWS_AHEAD<E>, Frag<E>>([&](int i) { return T::rows(rows, (qg * C::NS + i / T::KS) * 32, i % T::KS); }, [&](int i, const Frag<E>& x) {
      s[i / T::KS] = mma(x, f[i % T::KS], i % T::KS == 0 ? zeros() : s[i / T::KS]);
#pragma unroll
      for (int j = i * LOADS / STEPS; j < (i + 1) * LOADS / STEPS; ++j) { if (j < lq.N) lq.issue_one(j, next_at, next_q, wave); else ld.issue_one(j - lq.N, next_at + C::QD, next_d, wave); }
    });
    bool some[C::NS], whole[C::NS];
    uint32_t seen[C::NS];
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      some[n] = __any(first[n] < key0 + 32 && end[n] > key0);
      whole[n] = __all(first[n] <= key0 && end[n] >= key0 + 32);
      seen[n] = 0;
    }
    auto mask = [&](int n) {
      const uint2 bits = seen_rows(record(n), key, h);
      seen[n] = bits.x;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[n][r] = where_seen(second ? bits.y : bits.x, r, s[n][r], 0.f);
    };
    if (!second) {
#pragma unroll
      for (int n = 0; n < C::NS; ++n) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 slope = {}, bent; u32x4 place = {};
          if (SHAPE & BIASED) { slope = *reinterpret_cast<const f32x4*>(record(n) + SLOPE * GROUP + 8 * q + 4 * h); place = *reinterpret_cast<const u32x4*>(record(n) + AT * GROUP + 8 * q + 4 * h); }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 4 * q + i;
            float bend = 1.f;
            const float x = score(s[n][r], slope[i], (float)((int)place[i] - key), bend);
            s[n][r] = __builtin_amdgcn_exp2f(x - stat[n][q][i]);
            bent[i] = SHAPE & CAPPED ? s[n][r] * bend : s[n][r];
          }
          *reinterpret_cast<f32x4*>(shared_p + n * 1024 + q * 256) = bent;
        }
        if (!whole[n]) mask(n);
        b[n][0] = fragment<E>(s[n], 0); b[n][1] = fragment<E>(s[n], 1);
      }
    }
    __syncthreads();
    if (second) {
      f32x4 p[C::NS][4];
#pragma unroll
      for (int n = 0; n < C::NS; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) p[n][q] = *reinterpret_cast<const f32x4*>(shared_p + n * 1024 + q * 256);
      __builtin_amdgcn_sched_group_barrier(0x100, 4 * C::NS, 0);   // all of them are on their way before the first is waited for
#pragma unroll
      for (int n = 0; n < C::NS; ++n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = p[n][r >> 2][r & 3] * (s[n][r] - stat[n][r >> 2][r & 3]);
        if (!whole[n]) mask(n);
        b[n][0] = fragment<E>(s[n], 0); b[n][1] = fragment<E>(s[n], 1);
      }
    }
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      if (!some[n]) continue;
      const int row0 = (qg * C::NS + n) * 32;
      const bool finite = whole[n] || all_finite<E, C::DP>(other_rows, row0);
      constexpr int N = sizeof(E) * C::DP > 256 ? 1 : 2;   // fragments at a time: 64 registers of columns at most
#pragma unroll
      for (int half = 0; half < 2; half += N) {
        Columns<E, C::DP, N> columns;
        Frag<E> weights[N];
#pragma unroll
        for (int i = 0; i < N; ++i) weights[i] = b[n][half + i];
        columns.fetch(columns_at, row0 + 16 * half);
        add_product<E, C::DP, N>(sum, columns, weights, finite, seen[n] >> (16 * half), columns_at, row0 + 16 * half);
      }
    }
  }
  drain_loads();
  if constexpr (C::QG > 1) {   // the row groups' sums; a wave then has some of the columns
    float* const part = reinterpret_cast<float*>(smem) + (second ? C::QG * C::DP * 32 : 0);                     // [QG][DP][32]
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < C::WK; ++kk) {
      if (kk == kw) {
#pragma unroll
        for (int df = 0; df < T::DF; ++df)
#pragma unroll
          for (int r = 0; r < 16; ++r) part[(qg * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)] = sum[df][r];
      }
      __syncthreads();
      if (kk == kw) {
#pragma unroll
        for (int df = 0; df < T::DF; ++df) {
          if (df % C::QG != qg) continue;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float x = 0.f;
#pragma unroll
            for (int g = 0; g < C::QG; ++g) x += part[(g * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)];
            sum[df][r] = x;
          }
        }
      }
      __syncthreads();
    }
  }
  if (key >= a.Tk) return;
  const Heads& out = second ? a.dk : a.dv;
  E* const to = const_cast<E*>(static_cast<const E*>(out.p)) + (int64_t)key * out.ld + hk * out.hs;
#pragma unroll
  for (int df = 0; df < T::DF; ++df) if (C::QG == 1 || df % C::QG == qg) store_columns<E>(to, df, D, sum[df], second ? a.scale : 1.f, h);
}

// The same with one wave for both, where its registers are enough for two waves to a SIMD (bf16, widths up to 64): one barrier a tile instead of two, and nothing to hand over.
template <typename E, int DP_, int WK_, int QG_, int NS_>
struct OneConfig {
  static constexpr int DP = DP_, WK = WK_, QG = QG_, NS = NS_;
  static constexpr int WAVES = WK * QG, THREADS = WAVES * 64, KEYS = 32 * WK, BQ = 32 * NS * QG, GROUPS = BQ / GROUP;
  static constexpr int QD = BQ * DP * (int)sizeof(E), REC = (GROUPS * RECORD + 1023) / 1024 * 1024, STAGE = 2 * QD + REC, LDS = 2 * STAGE;
  static constexpr int REC_LOADS = (REC / 1024 + WAVES - 1) / WAVES;
  static_assert(BQ % GROUP == 0 && LDS <= LDS_MAX && WK * QG * DP * 32 * 4 <= LDS, "LDS");
};
template <typename E, typename C, int SHAPE>
__global__ __launch_bounds__(C::THREADS, 2) void k_attention_dkv_one(AttentionArgs a, Rows recs) {
  extern __shared__ __align__(1024) unsigned char smem[];
  typedef Tile<E, C::DP> T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int kw = wave / C::QG, qg = wave % C::QG;
  const int G = a.Hq / a.Hk, D = a.D, tokens = GROUP / G;
  const int hk = blockIdx.x % a.Hk, k_first = blockIdx.x / a.Hk * C::KEYS;
  const int key0 = k_first + kw * 32, key = key0 + (lane & 31);
  Steps<C::GROUPS> step_list(recs, k_first, k_first + C::KEYS);
  Loads<E, C::DP, C::BQ, C::WAVES> lq, ld;
  lq.init(a.q.ld, a.q.hs, G, D, wave, lane);
  ld.init(a.dout.ld, a.dout.hs, G, D, wave, lane);
  const uint32_t lds = lds_address(smem), row_lane = T::row_lane(lane), column_lane = T::column_lane(lane);
  const Source qs = rows_source<E>(a.q, a, hk, C::GROUPS), ds = rows_source<E>(a.dout, a, hk, C::GROUPS);
  const Source rs(recs.record + (int64_t)hk * recs.groups * (PLANES * GROUP), (int64_t)recs.groups * RECORD, C::GROUPS * RECORD);
  int step = step_list.next(lane);
  if (step >= 0) { load_records<C>(rs.tile(step), lds, wave, lane); lq.issue(lds, qs.tile(step), wave); ld.issue(lds + C::QD, ds.tile(step), wave); }

  Frag<E> k[T::KS], v[T::KS];
  {
    const int64_t from = min((int64_t)key, a.Tk - 1);
    const E* const kp = static_cast<const E*>(a.k.p) + from * a.k.ld + hk * a.k.hs;
    const E* const vp = static_cast<const E*>(a.v.p) + from * a.v.ld + hk * a.v.hs;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
      k[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(kp + 16 * ks + 8 * h) : zero_fragment<E>();
      v[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(vp + 16 * ks + 8 * h) : zero_fragment<E>();
    }
  }
  arrived(k); arrived(v);
  const Scores<E, SHAPE> score(a.scale, a.cap);
  f32x16 dk[T::DF], dv[T::DF];
#pragma unroll
  for (int df = 0; df < T::DF; ++df) { dk[df] = zeros(); dv[df] = zeros(); }

  for (int stage = 0; step >= 0; stage ^= 1) {
    const int next = step_list.next(lane);
    wait_loads();
    const bool more = next >= 0;
    const u32x4 next_q = more ? qs.tile(next) : Source::nothing(), next_d = more ? ds.tile(next) : Source::nothing();
    const uint32_t next_at = lds + (stage ^ 1) * C::STAGE;
    if (more) load_records<C>(rs.tile(next), next_at, wave, lane);
    step = next;
    const uint32_t q_rows = lds + stage * C::STAGE + row_lane, q_cols = lds + stage * C::STAGE + column_lane, d_rows = q_rows + C::QD, d_cols = q_cols + C::QD;
    constexpr int LOADS = (lq.N + ld.N) / C::NS;   // in each subtile
    auto load = [&](int j) { if (j < lq.N) lq.issue_one(j, next_at, next_q, wave); else ld.issue_one(j - lq.N, next_at + C::QD, next_d, wave); };
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      const int row0 = (qg * C::NS + n) * 32;
      const uint32_t* const rec = reinterpret_cast<const uint32_t*>(smem + stage * C::STAGE + 2 * C::QD) + row0 / GROUP * (PLANES * GROUP) + row0 % GROUP;
      const int first = (int)rec[FIRST * GROUP + (lane & 31)], end = (int)rec[END * GROUP + (lane & 31)];
      f32x16 s, dp;
      pipeline<2 * T::KS, ROWS_AHEAD<E>, Frag<E>>([&](int i) { return T::rows(i < T::KS ? q_rows : d_rows, row0, i % T::KS); }, [&](int i, const Frag<E>& x) {
        if (i < T::KS) s = mma(x, k[i], i == 0 ? zeros() : s);
        else dp = mma(x, v[i - T::KS], i == T::KS ? zeros() : dp);
#pragma unroll
        for (int j = i * LOADS / (2 * T::KS); j < (i + 1) * LOADS / (2 * T::KS); ++j) load(n * LOADS + j);
      });
      if (!__any(first < key0 + 32 && end > key0)) continue;   // (not sooner: the loads are every wave's)
      const bool whole = __all(first <= key0 && end >= key0 + 32);
      Columns<E, C::DP, 2> columns;
      columns.fetch(d_cols, row0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = 8 * q + 4 * h;
        const f32x4 lse = *reinterpret_cast<const f32x4*>(rec + LSE * GROUP + at), delta = *reinterpret_cast<const f32x4*>(rec + DELTA * GROUP + at);
        f32x4 slope = {}; u32x4 place = {};
        if (SHAPE & BIASED) { slope = *reinterpret_cast<const f32x4*>(rec + SLOPE * GROUP + at); place = *reinterpret_cast<const u32x4*>(rec + AT * GROUP + at); }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * q + i;
          float bend = 1.f;
          const float x = score(s[r], slope[i], (float)((int)place[i] - key), bend);
          s[r] = __builtin_amdgcn_exp2f(x - lse[i]);
          dp[r] = SHAPE & CAPPED ? s[r] * (dp[r] - delta[i]) * bend : s[r] * (dp[r] - delta[i]);
        }
      }
      uint32_t seen = 0;
      if (!whole) {
        const uint2 bits = seen_rows(rec, key, h);
        seen = bits.x;
#pragma unroll
        for (int r = 0; r < 16; ++r) { s[r] = where_seen(bits.x, r, s[r], 0.f); dp[r] = where_seen(bits.y, r, dp[r], 0.f); }
      }
      Frag<E> p[2] = {fragment<E>(s, 0), fragment<E>(s, 1)}, w[2] = {fragment<E>(dp, 0), fragment<E>(dp, 1)};
      Columns<E, C::DP, 2> q_columns;
      q_columns.fetch(q_cols, row0);
      add_product<E, C::DP, 2>(dv, columns, p, whole || all_finite<E, C::DP>(d_rows, row0), seen, d_cols, row0);
      add_product<E, C::DP, 2>(dk, q_columns, w, whole || all_finite<E, C::DP>(q_rows, row0), seen, q_cols, row0);
    }
  }
  drain_loads();
  auto finish = [&](f32x16 (&x)[T::DF], const Heads& out, float factor) {
    if constexpr (C::QG > 1) {   // the row groups' sums; a wave then has some of the columns
      float* const part = reinterpret_cast<float*>(smem) + kw * C::QG * C::DP * 32;                     // [QG][DP][32]
      __syncthreads();
#pragma unroll
      for (int df = 0; df < T::DF; ++df)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[(qg * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)] = x[df][r];
      __syncthreads();
#pragma unroll
      for (int df = 0; df < T::DF; ++df) {
        if (df % C::QG != qg) continue;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float sum = 0.f;
#pragma unroll
          for (int g = 0; g < C::QG; ++g) sum += part[(g * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)];
          x[df][r] = sum;
        }
      }
    }
    if (key >= a.Tk) return;
    E* const to = const_cast<E*>(static_cast<const E*>(out.p)) + (int64_t)key * out.ld + hk * out.hs;
#pragma unroll
    for (int df = 0; df < T::DF; ++df) if (C::QG == 1 || df % C::QG == qg) store_columns<E>(to, df, D, x[df], factor, h);
  };
  finish(dk, a.dk, a.scale);
  finish(dv, a.dv, 1.f);
}

template <auto KERNEL, typename C, typename... A>
void launch(ProfScope& ps, int64_t blocks, hipStream_t st, A... a) {
  static const bool once = [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    return true;
  }();
  (void)once;
  launch_kernel(ps, KERNEL, dim3((unsigned)blocks), C::THREADS, C::LDS, st, a...);
}
template <typename E, int DP, int SHAPE>
void launch_all(hipStream_t st, const AttentionArgs& a, const Rows& rows) {
  ProfScope ps(st, F_OTHER, 0.0);
  const int64_t count = a.Tq * (a.Hq / a.Hk);
  if (a.Tq > 0) launch_kernel(ps, k_attention_delta<E, SHAPE>, dim3((unsigned)((int64_t)rows.groups * a.Hk)), 256, 0, st, a, rows);
  auto rows_of = [&](auto config) {
    typedef decltype(config) C;
    const int64_t n = (count + C::BM - 1) / C::BM;
    launch<&k_attention_dq<E, C, SHAPE>, C>(ps, n * a.Hk, st, a, rows, (int)n);
  };
  auto by_rows = [&] {
    const int n = rows_of_workgroup(count, a.Hk, DP, sizeof(E) == 2);
    if constexpr (DP > 64) if (n == 128) return rows_of(QConfig<E, DP, 4>{});
    if constexpr (sizeof(E) * DP <= 256) if (n == 64) return rows_of(QConfig<E, DP, 2>{});
    rows_of(QConfig<E, DP, 1>{});
  };
  if (a.Tq > 0) by_rows();
  if (a.Tk == 0) return;
  auto pairs = [&](auto config) {
    typedef decltype(config) C;
    launch<&k_attention_dkv<E, C, SHAPE>, C>(ps, (a.Tk + C::KEYS - 1) / C::KEYS * a.Hk, st, a, rows);
  };
  auto ones = [&](auto config) {
    typedef decltype(config) C;
    launch<&k_attention_dkv_one<E, C, SHAPE>, C>(ps, (a.Tk + C::KEYS - 1) / C::KEYS * a.Hk, st, a, rows);
  };
  // How many waves a workgroup has side by side over keys, how many groups over rows: the more workgroups of 128 keys there are, the fewer groups.  us of dk and dv, causal, at that many (-: not measured):
  //   bf16, width 64: 16 heads of 8192 in one text (1024) 368 with 128 keys, 445 with 32 and four groups of rows; of 6000 in five (752) 32 keys 186; 16 on 4 of 8111 in 23 texts (256) 303, 174
  //     with 64 keys, 101 with 32
  //   bf16, width 128, pairs of waves over 128, 64, 32 keys: 16 of 8192 on 8 in one text (512) 688, 1008, 1491; 12 of 4096 in 4 texts (384) 172, 155, 194, in 41 60, 65, 100 (64 keys for both); 8 of 3200 in 4 texts
  //     (200) 134, 100, 87, in 30 44, 37, 58; 8 of 4096 on 4 in 4 texts (128) -, 236, 144
  //   fp32, width 64: 12 of 6000 in two texts (564) 574, 552, 579; of 4096 in 4 (384) -, 255, 269; 8 of 3200 in 4 (200) 325, 176, 134, in 30 97, 57, 65
  //   fp32, width 128, 64 keys or 32, two groups of rows: 16 of 6000 in 3 texts (752) 1132, 1244; 12 of 4096 in 41 (384) 156, 159; 8 of 4096 in 4 (256) 393, 361; of 1500 in 4 (96) 159, 103
  const int64_t blocks = (a.Tk + 127) / 128 * a.Hk;
  if constexpr (sizeof(E) == 2 && DP == 64) {
    if (blocks >= 1024) ones(OneConfig<E, DP, 4, 1, 2>{});
    else ones(OneConfig<E, DP, 1, 4, 1>{});
  } else if constexpr (sizeof(E) == 2) {
    if (blocks >= 512) pairs(KConfig<E, DP, 4, 1, 2>{});
    else if (blocks >= 192) pairs(KConfig<E, DP, 2, 2, 1>{});
    else pairs(KConfig<E, DP, 1, 4, 1>{});
  } else if constexpr (DP == 64) {
    if (blocks >= 256) pairs(KConfig<E, DP, 2, 2, 1>{});
    else pairs(KConfig<E, DP, 1, 4, 1>{});
  } else {
    if (blocks >= 384) pairs(KConfig<E, DP, 2, 2, 1>{});
    else pairs(KConfig<E, DP, 1, 2, 1>{});
  }
}
template <typename E, int DP>
void launch_width(hipStream_t st, const AttentionArgs& a, const Rows& rows) {
  switch ((a.cap > 0.f ? CAPPED : 0) | (a.slopes != nullptr ? BIASED : 0)) {
    case PLAIN: return launch_all<E, DP, PLAIN>(st, a, rows);
    case CAPPED: return launch_all<E, DP, CAPPED>(st, a, rows);
    case BIASED: return launch_all<E, DP, BIASED>(st, a, rows);
    default: return launch_all<E, DP, CAPPED | BIASED>(st, a, rows);
  }
}
int64_t groups_of(int64_t Tq, int G) { const int64_t tokens = GROUP / G; return (Tq + tokens - 1) / tokens; }
}  // namespace

size_t attention_grad_bytes(int64_t Tq, int64_t, int Hq, int Hk, int) { return (size_t)groups_of(Tq, Hq / Hk) * (RECORD * (size_t)Hk + sizeof(int2)) + 256; }

void launch_attention_grad(hipStream_t st, const AttentionArgs& a, bool bf16, void* workspace) {
  const int64_t groups = groups_of(a.Tq, a.Hq / a.Hk);
  Rows rows{static_cast<uint32_t*>(workspace), nullptr, (int)groups};
  rows.range = reinterpret_cast<int2*>(static_cast<unsigned char*>(workspace) + (size_t)groups * RECORD * a.Hk);
  if (bf16) a.D <= 64 ? launch_width<bf16_t, 64>(st, a, rows) : launch_width<bf16_t, 128>(st, a, rows);
  else a.D <= 64 ? launch_width<float, 64>(st, a, rows) : launch_width<float, 128>(st, a, rows);
}

}  // namespace sama
