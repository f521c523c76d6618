// Gradients of attention (attention.hip), from q, k, v, the output o, its gradient do and the logarithm of each row's sum:
//   p_ij = exp(s_ij - lse_i),  dp_ij = do_i . v_j,  delta_i = do_i . o_i,  ds_ij = p_ij (dp_ij - delta_i) (1 - tanh^2 if capped)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,   i over all queries and heads that share k_j and v_j.
// Scores are formed again, in two launches: one walks the keys for a tile of rows (dq), one the rows for a tile of keys (dk, dv).  That is seven products where five
// would do if one launch made both; but then one side would have to be added up in memory by workgroups as they come, in an order of their own.
// k_attention_delta goes ahead: delta, and what else the second launch needs of each row, laid out in the order in which it is read.
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

template <typename E>
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
    for (int i = 8 * part; i < a.D; i += 32) {
      const Frag<E> x = load_fragment<E>(o + i), y = load_fragment<E>(d + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)x[e], (float)y[e], sum);
    }
  }
  sum += __shfl_xor(sum, 1); sum += __shfl_xor(sum, 2);
  if (part == 0) {
    uint32_t* const to = rows.record + ((int64_t)hk * rows.groups + group) * (PLANES * GROUP) + r;
    to[LSE * GROUP] = __float_as_uint(some ? a.lse[query * a.Hq + head] * LOG2E : 0.f);
    to[DELTA * GROUP] = __float_as_uint(sum);
    to[FIRST * GROUP] = span.x; to[END * GROUP] = span.y;
    to[AT * GROUP] = some ? (a.at != nullptr ? a.at[query] : (int)query) : 0;
    to[SLOPE * GROUP] = __float_as_uint(some && a.slopes != nullptr ? a.slopes[head] * LOG2E : 0.f);
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
  static constexpr int KG = WM > 1 ? 1 : sizeof(E) * DP > 256 ? 2 : 4;
  static constexpr int NS = WM > 1 && sizeof(E) * DP <= 256 ? 2 : 1;
  static constexpr int WAVES = WM * KG, THREADS = WAVES * 64, BM = 32 * WM, BK = 32 * NS * KG;
  static constexpr int KV = BK * DP * (int)sizeof(E), LDS = 4 * KV;
  static constexpr int PER_EU = sizeof(E) * DP <= 256 ? 2 : 1;
  static_assert(LDS <= LDS_MAX && KG * DP * 32 * 4 <= LDS, "LDS");
};
template <typename E, typename C, bool SHAPED>
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
  auto issue = [&](int i, int stage) {
    const int64_t k0 = lo + (int64_t)i * C::BK;
    const u32x4 dk = descriptor(kp + k0 * a.k.ld, ((a.Tk - 1 - k0) * a.k.ld + D) * (int64_t)sizeof(E));
    const u32x4 dv = descriptor(vp + k0 * a.v.ld, ((a.Tk - 1 - k0) * a.v.ld + D) * (int64_t)sizeof(E));
    lk.issue(lds + stage * 2 * C::KV, dk, wave);
    lv.issue(lds + stage * 2 * C::KV + C::KV, dv, wave);
  };
  int t = seen_from(0);
  if (t < end) issue(t, 0);

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
  const float slope = SHAPED ? __uint_as_float(rec[SLOPE * GROUP]) : 0.f;
  const int at = SHAPED ? (int)rec[AT * GROUP] : 0;
  const Shape shape(a.scale, a.cap);
  const float c = a.scale * LOG2E;
  f32x16 dq[T::DF];
#pragma unroll
  for (int df = 0; df < T::DF; ++df) dq[df] = zeros();

  for (int stage = 0; t < end; stage ^= 1) {
    const int next = seen_from(t + 1);
    wait_loads();
    if (next < end) issue(next, stage ^ 1);
    const uint32_t k_rows = lds + stage * 2 * C::KV + row_lane, v_rows = k_rows + C::KV, k_cols = lds + stage * 2 * C::KV + column_lane;
    const int first = lo + t * C::BK + kg * 32 * C::NS;
    t = next;
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      const int k0 = first + 32 * n, row0 = (kg * C::NS + n) * 32;
      if (!__any(span.x < k0 + 32 && span.y > k0)) continue;
      f32x16 s = row_product<E, C::DP>(k_rows, row0, q), dp = row_product<E, C::DP>(v_rows, row0, d);
      interleave<2 * T::KS, 4, ROW_READS<E>, PRODUCTS<E>>();
      Columns<E, C::DP, 2> columns;
      columns.fetch(k_cols, row0);
      const bool whole = __all(span.x <= k0 && span.y >= k0 + 32);
      const int away = at - k0 - 4 * h;
      uint32_t seen = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float bend = 1.f, x = s[r] * c;
        if (SHAPED) x = shape.score<E>(s[r], slope, fabsf((float)(away - 8 * (r >> 2) - (r & 3))), bend);
        const float p = __builtin_amdgcn_exp2f(x - lse);
        s[r] = SHAPED ? p * (dp[r] - delta) * bend : p * (dp[r] - delta);
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
  if constexpr (C::KG > 1) {   // the groups' sums; a wave then has 32 of the columns
    __syncthreads();
    float* const part = reinterpret_cast<float*>(smem);                     // [KG][DP][32]
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
template <typename E, typename C, bool SHAPED>
__global__ __launch_bounds__(C::THREADS, 2) void k_attention_dkv(AttentionArgs a, Rows recs) {
  extern __shared__ __align__(1024) unsigned char smem[];
  typedef Tile<E, C::DP> T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int pair = wave % C::PAIRS, kw = pair / C::QG, qg = pair % C::QG;
  const bool second = wave >= C::PAIRS;   // (waves four apart share a SIMD: one of either kind, which want its units at different times)
  const int G = a.Hq / a.Hk, D = a.D, tokens = GROUP / G;
  const int hk = blockIdx.x % a.Hk, k_first = blockIdx.x / a.Hk * C::KEYS;   // the first keys, which most rows of a causal text see, first
  const int key0 = k_first + kw * 32, key = key0 + (lane & 31);
  // steps of GROUPS groups; which of the next 64 have rows that see one of the workgroup's keys
  const int steps = (recs.groups + C::GROUPS - 1) / C::GROUPS;
  int at_step = 0;
  uint64_t ahead = 0;
  auto next_step = [&]() {   // the next step, or `steps`
    while (ahead == 0) {
      if (at_step >= steps) return steps;
      bool any = false;
#pragma unroll
      for (int g = 0; g < C::GROUPS; ++g) {
        const int group = (at_step + lane) * C::GROUPS + g;
        if (group < recs.groups) { const int2 s = recs.range[group]; any |= s.x < k_first + C::KEYS && s.y > k_first; }
      }
      ahead = __ballot(any);
      at_step += 64;
    }
    const int bit = __builtin_ctzll(ahead);
    ahead &= ahead - 1;
    return at_step - 64 + bit;
  };
  Loads<E, C::DP, C::BQ, C::WAVES> lq, ld;
  lq.init(a.q.ld, a.q.hs, G, D, wave, lane);
  ld.init(a.dout.ld, a.dout.hs, G, D, wave, lane);
  const uint32_t lds = lds_address(smem), row_lane = T::row_lane(lane), column_lane = T::column_lane(lane);
  auto issue = [&](int step, int stage) {
    const int64_t group = (int64_t)step * C::GROUPS, q0 = group * tokens;
    const E* const q = static_cast<const E*>(a.q.p) + q0 * a.q.ld + (int64_t)hk * G * a.q.hs;
    const E* const d = static_cast<const E*>(a.dout.p) + q0 * a.dout.ld + (int64_t)hk * G * a.dout.hs;
    const u32x4 dq = descriptor(q, ((a.Tq - 1 - q0) * a.q.ld + (G - 1) * a.q.hs + D) * (int64_t)sizeof(E));
    const u32x4 dd = descriptor(d, ((a.Tq - 1 - q0) * a.dout.ld + (G - 1) * a.dout.hs + D) * (int64_t)sizeof(E));
    const u32x4 dr = descriptor(recs.record + ((int64_t)hk * recs.groups + group) * (PLANES * GROUP), (recs.groups - group) * RECORD);
    lq.issue(lds + stage * C::STAGE, dq, wave);
    ld.issue(lds + stage * C::STAGE + C::QD, dd, wave);
#pragma unroll
    for (int i = 0; i < C::REC_LOADS; ++i) {
      const uint32_t at = (i * C::WAVES + wave) * 1024;
      if (at < C::REC) load_to_lds(lds + stage * C::STAGE + 2 * C::QD + at, at + lane * 16 < C::GROUPS * RECORD ? at + lane * 16 : NOWHERE, dr);
    }
  };
  int step = next_step();
  if (step < steps) issue(step, 0);

  Frag<E> f[T::KS];   // the keys' k, or v
  {
    const Heads& from = second ? a.v : a.k;
    const E* const p = static_cast<const E*>(from.p) + min((int64_t)key, a.Tk - 1) * from.ld + hk * from.hs;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) f[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(p + 16 * ks + 8 * h) : zero_fragment<E>();
  }
  const Shape shape(a.scale, a.cap);
  const float c = a.scale * LOG2E;
  float* const shared_p = reinterpret_cast<float*>(smem + C::P) + pair * C::NS * 1024 + lane * 4;
  f32x16 sum[T::DF];   // dv, or dk
#pragma unroll
  for (int df = 0; df < T::DF; ++df) sum[df] = zeros();

  for (int stage = 0; step < steps; stage ^= 1) {
    const int next = next_step();
    wait_loads();
    if (next < steps) issue(next, stage ^ 1);
    step = next;
    const uint32_t q_tile = lds + stage * C::STAGE, d_tile = q_tile + C::QD;
    const uint32_t rows = (second ? d_tile : q_tile) + row_lane, other_rows = (second ? q_tile : d_tile) + row_lane, columns_at = (second ? q_tile : d_tile) + column_lane;
    const uint32_t* const recs_at = reinterpret_cast<const uint32_t*>(smem + stage * C::STAGE + 2 * C::QD);
    f32x16 s[C::NS];
    Frag<E> b[C::NS][2];
    bool some[C::NS], whole[C::NS];
    uint32_t seen[C::NS], matters[C::NS];
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      const int row0 = (qg * C::NS + n) * 32;
      const uint32_t* const rec = recs_at + row0 / GROUP * (PLANES * GROUP) + row0 % GROUP;
      const int first = (int)rec[FIRST * GROUP + (lane & 31)], end = (int)rec[END * GROUP + (lane & 31)];
      some[n] = __any(first < key0 + 32 && end > key0);
      whole[n] = __all(first <= key0 && end >= key0 + 32);
      seen[n] = matters[n] = 0;
      if (some[n] && !whole[n]) {                // a single key has probability 1, whatever its score: its ds is zero
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int at = 8 * q + 4 * h;
          const u32x4 from = *reinterpret_cast<const u32x4*>(rec + FIRST * GROUP + at), to = *reinterpret_cast<const u32x4*>(rec + END * GROUP + at);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bit = key >= (int)from[i] && key < (int)to[i] ? 1u << seen_bit(4 * q + i) : 0;
            seen[n] |= bit;
            matters[n] |= to[i] - from[i] > 1 ? bit : 0;
          }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      if (some[n]) {
        s[n] = row_product<E, C::DP>(rows, (qg * C::NS + n) * 32, f);
        interleave<T::KS, 4, ROW_READS<E>, PRODUCTS<E>>();
      }
    }
    if (!second) {
#pragma unroll
      for (int n = 0; n < C::NS; ++n) {
        if (!some[n]) continue;
        const int row0 = (qg * C::NS + n) * 32;
        const uint32_t* const rec = recs_at + row0 / GROUP * (PLANES * GROUP) + row0 % GROUP;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int at = 8 * q + 4 * h;
          const f32x4 lse = *reinterpret_cast<const f32x4*>(rec + LSE * GROUP + at);
          f32x4 slope = {}, bent; u32x4 place = {};
          if (SHAPED) { slope = *reinterpret_cast<const f32x4*>(rec + SLOPE * GROUP + at); place = *reinterpret_cast<const u32x4*>(rec + AT * GROUP + at); }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 4 * q + i;
            float bend = 1.f, x = s[n][r] * c;
            if (SHAPED) x = shape.score<E>(s[n][r], slope[i], fabsf((float)((int)place[i] - key)), bend);
            s[n][r] = __builtin_amdgcn_exp2f(x - lse[i]);
            bent[i] = SHAPED ? s[n][r] * bend : s[n][r];
          }
          *reinterpret_cast<f32x4*>(shared_p + n * 1024 + q * 256) = bent;
        }
        if (!whole[n]) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] = where_seen(seen[n], r, s[n][r], 0.f);
        }
        b[n][0] = fragment<E>(s[n], 0); b[n][1] = fragment<E>(s[n], 1);
      }
    }
    __syncthreads();
    if (second) {
#pragma unroll
      for (int n = 0; n < C::NS; ++n) {
        if (!some[n]) continue;
        const int row0 = (qg * C::NS + n) * 32;
        const uint32_t* const rec = recs_at + row0 / GROUP * (PLANES * GROUP) + row0 % GROUP;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 delta = *reinterpret_cast<const f32x4*>(rec + DELTA * GROUP + 8 * q + 4 * h), p = *reinterpret_cast<const f32x4*>(shared_p + n * 1024 + q * 256);
#pragma unroll
          for (int i = 0; i < 4; ++i) { const int r = 4 * q + i; s[n][r] = p[i] * (s[n][r] - delta[i]); }
        }
        if (!whole[n]) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[n][r] = where_seen(matters[n], r, s[n][r], 0.f);
        }
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

constexpr int64_t MANY = 256;

template <auto KERNEL, typename C, typename... A>
void launch(ProfScope& ps, int64_t blocks, hipStream_t st, A... a) {
  static const bool once = [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    return true;
  }();
  (void)once;
  launch_kernel(ps, KERNEL, dim3((unsigned)blocks), C::THREADS, C::LDS, st, a...);
}
template <typename E, int DP, bool SHAPED>
void launch_all(hipStream_t st, const AttentionArgs& a, const Rows& rows) {
  ProfScope ps(st, F_OTHER, 0.0);
  const int64_t count = a.Tq * (a.Hq / a.Hk);
  if (a.Tq > 0) launch_kernel(ps, k_attention_delta<E>, dim3((unsigned)((int64_t)rows.groups * a.Hk)), 256, 0, st, a, rows);
  if (a.Tq == 0) {
  } else if ((count + 127) / 128 * a.Hk >= MANY) {
    typedef QConfig<E, DP, 4> C;
    launch<&k_attention_dq<E, C, SHAPED>, C>(ps, (count + 127) / 128 * a.Hk, st, a, rows, (int)((count + 127) / 128));
  } else {
    typedef QConfig<E, DP, 1> C;
    launch<&k_attention_dq<E, C, SHAPED>, C>(ps, (count + 31) / 32 * a.Hk, st, a, rows, (int)((count + 31) / 32));
  }
  if (a.Tk == 0) return;
  auto dkv = [&](auto config) {
    typedef decltype(config) C;
    launch<&k_attention_dkv<E, C, SHAPED>, C>(ps, (a.Tk + C::KEYS - 1) / C::KEYS * a.Hk, st, a, rows);
  };
  if constexpr (sizeof(E) * DP > 256) {
    if ((a.Tk + 63) / 64 * a.Hk >= MANY) dkv(KConfig<E, DP, 2, 2, 1>{});
    else dkv(KConfig<E, DP, 1, 2, 1>{});
  } else {
    if ((a.Tk + 127) / 128 * a.Hk >= 2 * MANY) dkv(KConfig<E, DP, 4, 1, 2>{});
    else if ((a.Tk + 63) / 64 * a.Hk >= MANY) dkv(KConfig<E, DP, 2, 2, 1>{});
    else dkv(KConfig<E, DP, 1, 4, 1>{});
  }
}
template <typename E, int DP>
void launch_width(hipStream_t st, const AttentionArgs& a, const Rows& rows) {
  if (a.cap > 0.f || a.slopes != nullptr) launch_all<E, DP, true>(st, a, rows);
  else launch_all<E, DP, false>(st, a, rows);
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
