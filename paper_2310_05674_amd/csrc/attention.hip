// Attention of queries over the keys of their spans.  For query i, head h and the key head h' that it shares with G - 1 others:
//   s_j = scale q_i . k_j, capped: cap tanh(s_j / cap), biased: - slope_h |at_i - j|,   p = softmax of s over begin_i <= j < end_i,   o_i = sum_j p_j v_j.
// One pass over the keys with the running maximum and sum of the softmax: 4 D operations a pair, nothing of the scores leaves the registers.
//
// The G heads of a key head are rows of the same tiles (row = query G + head), so K and V are read once for all of them.  A workgroup has 32 WM rows and walks the
// tiles of keys between its rows' first and last; tiles that no row sees are left out.  Its four waves have 32 rows each, or share 64 or 32 with different keys of a tile for each half or quarter of
// them (KG groups; see rows_of_workgroup), and where workgroups are few the keys are split between several, joined by k_attention_join.
//
// Long texts are bound by products: 8192 causal tokens in bf16, 16 heads of 128 on 8 key heads, take 330 us, 834 TFLOP/s.  Short ones by each workgroup's chain of spans, first loads, tiles and
// join: 8111 tokens in 23 texts, 16 heads of 64 on 4, 43 us, of which products alone would be 8.5.  New tokens by memory: 3 over 24001 keys each, 16 heads of 128 on 4, 28.0 us, 5.3 TB/s.
#include <algorithm>
#include <cmath>
#include "attention_tiles.h"

namespace sama {
namespace {
using namespace attn;

template <typename E, int DP_, int WM_, int KG_, int NS_>
struct Config {
  static constexpr int DP = DP_, WM = WM_, KG = KG_, NS = NS_;                    // waves side by side over rows, over keys; 32 keys each of a wave's part of a tile
  static constexpr int WAVES = WM * KG, THREADS = WAVES * 64, BM = 32 * WM, BK = 32 * NS * KG;
  static constexpr int KV = BK * DP * (int)sizeof(E), JOIN = KG == 1 ? 0 : WAVES * (DP * 32 * 4 + 256);
  static constexpr int LDS = 4 * KV > JOIN ? 4 * KV : JOIN;                       // K and V, two stages; the groups' parts
  static constexpr int PER_EU = sizeof(E) * DP <= 256 ? 2 : 1;
  static_assert(LDS <= LDS_MAX, "LDS");
};

struct Parts { float* o; float* lse; int count; };   // of split keys: [count][Hk][rows][D] and [count][Hk][rows]

template <typename E, typename C, int SHAPE>
__global__ __launch_bounds__(C::THREADS, C::PER_EU) void k_attention(AttentionArgs a, Parts parts, int tiles) {
  extern __shared__ __align__(1024) unsigned char smem[];
  typedef Tile<E, C::DP> T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int rw = wave / C::KG, kg = wave % C::KG;
  const int G = a.Hq / a.Hk, rows = (int)a.Tq * G, D = a.D;
  const int hk = blockIdx.x % a.Hk, tile = tiles - 1 - blockIdx.x / a.Hk;   // the last queries, which see the most of a causal text, first
  const int row = tile * C::BM + rw * 32 + (lane & 31), query = min(row, rows - 1) / G, head = hk * G + min(row, rows - 1) % G;
  const int2 span = span_of(a.spans, query, (int)a.Tk);
  // spans of all of the workgroup's rows, two a lane
  const int r0 = min(tile * C::BM + lane % C::BM, rows - 1), r1 = min(tile * C::BM + (lane + 64) % C::BM, rows - 1);
  const int2 s0 = span_of(a.spans, r0 / G, (int)a.Tk), s1 = span_of(a.spans, r1 / G, (int)a.Tk);
  const int lo = __builtin_amdgcn_readfirstlane(wave_min(min(s0.x < s0.y ? s0.x : 0x7fffffff, s1.x < s1.y ? s1.x : 0x7fffffff)));
  const int hi = __builtin_amdgcn_readfirstlane(wave_max(max(s0.y, s1.y)));
  int t = 0, end = hi > lo ? (hi - lo + C::BK - 1) / C::BK : 0;
  if (parts.count > 1) {
    const int64_t n = end;
    t = (int)(n * blockIdx.y / parts.count); end = (int)(n * (blockIdx.y + 1) / parts.count);
  }
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
  t = seen_from(t);
  if (t < end) { lk.issue(lds, ks.tile(t), wave); lv.issue(lds + C::KV, vs.tile(t), wave); }

  Frag<E> q[T::KS];
  {
    const E* const p = static_cast<const E*>(a.q.p) + query * a.q.ld + head * a.q.hs;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) q[ks] = 16 * ks + 8 * h < D ? load_fragment<E>(p + 16 * ks + 8 * h) : zero_fragment<E>();
  }
  arrived(q);
  const Scores<E, SHAPE> score(a.scale, a.cap);
  const float slope = SHAPE & BIASED ? a.slopes[head] * LOG2E : 0.f;
  const int at = SHAPE & BIASED ? (a.at != nullptr ? a.at[query] : query) : 0;
  const float c = SHAPE != PLAIN ? 1.f : a.scale * LOG2E;
  f32x16 o[T::DF];
#pragma unroll
  for (int df = 0; df < T::DF; ++df) o[df] = zeros();
  float m = -INF, l = 0.f;   // of the scores before the factor c; l: of the lane's own keys

  for (int stage = 0; t < end; stage ^= 1) {
    const int next = seen_from(t + 1);
    wait_loads();
    const u32x4 next_k = next < end ? ks.tile(next) : Source::nothing(), next_v = next < end ? vs.tile(next) : Source::nothing();
    const uint32_t next_at = lds + (stage ^ 1) * 2 * C::KV;
    constexpr int LOADS = lk.N + lv.N;
    auto load = [&](int i) { if (i < lk.N) lk.issue_one(i, next_at, next_k, wave); else lv.issue_one(i - lk.N, next_at + C::KV, next_v, wave); };
    const uint32_t k_rows = lds + stage * 2 * C::KV + row_lane, v_rows = k_rows + C::KV, v_cols = lds + stage * 2 * C::KV + C::KV + column_lane;
    const int k0 = lo + t * C::BK + kg * 32 * C::NS;   // the wave's first key
    t = next;
    f32x16 s[C::NS];
    constexpr int STEPS = C::NS * T::KS;
    pipeline<STEPS, ROWS_AHEAD<E>, Frag<E>>([&](int i) { return T::rows(k_rows, (kg * C::NS + i / T::KS) * 32, i % T::KS); }, [&](int i, const Frag<E>& x) {
      s[i / T::KS] = mma(x, q[i % T::KS], i % T::KS == 0 ? zeros() : s[i / T::KS]);
#pragma unroll
      for (int j = i * LOADS / STEPS; j < (i + 1) * LOADS / STEPS; ++j) load(j);
    });
    if (!__any(span.x < k0 + 32 * C::NS && span.y > k0)) continue;   // (not sooner: the loads are every wave's)
    constexpr int AHEAD = C::DP * sizeof(E) > 128 ? 1 : 2;   // sets of columns: 16 registers or 32 in bf16
    Columns<E, C::DP, 2> columns[AHEAD];
    columns[0].fetch(v_cols, kg * C::NS * 32);
    if (SHAPE != PLAIN) {
      const float away = (float)(at - k0 - 4 * h);
#pragma unroll
      for (int n = 0; n < C::NS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) { float bend; s[n][r] = score(s[n][r], slope, away - (float)(32 * n + 8 * (r >> 2) + (r & 3)), bend); }
    }
    const bool whole = __all(span.x <= k0 && span.y >= k0 + 32 * C::NS);
    uint32_t seen[C::NS] = {};
    if (!whole) {
#pragma unroll
      for (int n = 0; n < C::NS; ++n) {
        seen[n] = seen_keys(span, k0 + 32 * n, h);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = where_seen(seen[n], r, s[n][r], -INF);
      }
    }
    float top = m;
#pragma unroll
    for (int n = 0; n < C::NS; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
    top = other_half_max(top);
    if (__any(top > m)) {
      const float shrink = m == -INF ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
      l *= shrink;
#pragma unroll
      for (int df = 0; df < T::DF; ++df)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[df][r] *= shrink;
      m = top;
    }
    const float base = m == -INF ? 0.f : m * c;
    float sum = 0.f;
    Frag<E> p[C::NS][2];
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
#pragma unroll
      for (int r = 0; r < 16; ++r) { s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], c, -base)); sum += s[n][r]; }
      p[n][0] = fragment<E>(s[n], 0); p[n][1] = fragment<E>(s[n], 1);
    }
    l += sum;
#pragma unroll
    for (int n = 0; n < C::NS; ++n) {
      const int row0 = (kg * C::NS + n) * 32;
      if (AHEAD > 1 && n + 1 < C::NS) columns[(n + 1) % AHEAD].fetch(v_cols, row0 + 32);
      const bool finite = whole || all_finite<E, C::DP>(v_rows, row0);
      add_product<E, C::DP, 2>(o, columns[n % AHEAD], p[n], finite, seen[n], v_cols, row0);
      if (AHEAD == 1 && n + 1 < C::NS) columns[0].fetch(v_cols, row0 + 32);
    }
  }

  drain_loads();
  l = other_half_sum(l);
  if constexpr (C::KG > 1) {   // the groups' parts, each of its own maximum, through LDS; a wave then has 32 of the columns
    __syncthreads();
    float* const part = reinterpret_cast<float*>(smem) + rw * C::KG * (C::DP * 32 + 64);   // [KG][DP][32]
    float* const stat = part + C::KG * C::DP * 32;                                           // [KG][2][32]
#pragma unroll
    for (int df = 0; df < T::DF; ++df)
#pragma unroll
      for (int r = 0; r < 16; ++r) part[(kg * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)] = o[df][r];
    if (h == 0) { stat[(kg * 2) * 32 + lane] = m; stat[(kg * 2 + 1) * 32 + lane] = l; }
    __syncthreads();
    float top = -INF, factor[C::KG];
#pragma unroll
    for (int g = 0; g < C::KG; ++g) top = fmaxf(top, stat[2 * g * 32 + (lane & 31)]);
    l = 0.f;
#pragma unroll
    for (int g = 0; g < C::KG; ++g) {
      const float mg = stat[2 * g * 32 + (lane & 31)];
      factor[g] = mg == -INF ? 0.f : __builtin_amdgcn_exp2f((mg - top) * c);
      l += stat[(2 * g + 1) * 32 + (lane & 31)] * factor[g];
    }
    m = top;
#pragma unroll
    for (int df = 0; df < T::DF; ++df) {
      if (df % C::KG != kg) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < C::KG; ++g) x = fmaf(part[(g * C::DP + 32 * df + register_row(r, h)) * 32 + (lane & 31)], factor[g], x);
        o[df][r] = x;
      }
    }
  }
  if (row >= rows) return;
  // Without a key: nothing.  Scores of minus infinity alone have no softmax, so the row's sum of zero makes out NaN; a part of the row that has no others leaves that to the join.
  const bool none = parts.count > 1 ? m == -INF && l == 0.f : span.x >= span.y;
  const float inv = none ? 0.f : 1.f / l, lse = none ? -INF : m * c + log2f(l);
  const bool first = kg == 0 && h == 0;
  if (parts.count > 1) {
    const int64_t at_row = ((int64_t)blockIdx.y * a.Hk + hk) * rows + row;
    if (first) parts.lse[at_row] = lse;
#pragma unroll
    for (int df = 0; df < T::DF; ++df) if (C::KG == 1 || df % C::KG == kg) store_columns<float>(parts.o + at_row * D, df, D, o[df], inv, h);
  } else {
    E* const p = const_cast<E*>(static_cast<const E*>(a.out.p)) + query * a.out.ld + head * a.out.hs;
    if (first && a.lse != nullptr) a.lse[(int64_t)query * a.Hq + head] = lse * LN2;
#pragma unroll
    for (int df = 0; df < T::DF; ++df) if (C::KG == 1 || df % C::KG == kg) store_columns<E>(p, df, D, o[df], inv, h);
  }
}

// The parts of split keys, weighted by what each holds of the row's sum.  A workgroup takes a row: four columns a thread, and eight threads to those, each with every eighth part: the
// parts' loads are then on their way together (48 rows of 64 parts take 5 us, and 41 with one thread for all parts of its columns).
constexpr int MOST_PARTS = 64;
template <typename E>
__global__ __launch_bounds__(256) void k_attention_join(AttentionArgs a, Parts parts) {
  __shared__ float s_weight[MOST_PARTS], s_total[2];
  __shared__ f32x4 s_part[8][32];
  const int G = a.Hq / a.Hk, rows = (int)a.Tq * G, quad = threadIdx.x & 31, share = threadIdx.x >> 5;
  const int64_t of_row = blockIdx.x, step = (int64_t)a.Hk * rows;
  if (threadIdx.x < 64) {
    const float lse = (int)threadIdx.x < parts.count ? parts.lse[threadIdx.x * step + of_row] : -INF;
    const float top = join_wave(lse, [](float x, float y) { return fmaxf(x, y); });
    const float w = lse == -INF ? 0.f : __builtin_amdgcn_exp2f(lse - top), sum = wave_sum(w);
    s_weight[threadIdx.x] = w;
    if (threadIdx.x == 0) { s_total[0] = top; s_total[1] = sum; }
  }
  __syncthreads();
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  if (4 * quad < a.D) {
#pragma unroll 8
    for (int p = share; p < parts.count; p += 8) {
      const f32x4 o = *reinterpret_cast<const f32x4*>(parts.o + (p * step + of_row) * a.D + 4 * quad);
      x += o * s_weight[p];   // a weight of zero too: what is not finite in a part far below the others stays so, and a part without keys holds zeros
    }
  }
  s_part[share][quad] = x;
  __syncthreads();
  if (share != 0 || 4 * quad >= a.D) return;
#pragma unroll
  for (int g = 1; g < 8; ++g) x += s_part[g][quad];
  const float sum = s_total[1];
  const int hk = (int)(of_row / rows), row = (int)(of_row - (int64_t)hk * rows), query = row / G, head = hk * G + row % G;
  float inv = 1.f / sum;
  if (sum == 0.f) { const int2 span = span_of(a.spans, query, (int)a.Tk); if (span.x >= span.y) inv = 0.f; }   // else scores of minus infinity alone: out is NaN
  E* const o = const_cast<E*>(static_cast<const E*>(a.out.p)) + query * a.out.ld + head * a.out.hs + 4 * quad;
  if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
  else *reinterpret_cast<f32x4*>(o) = x * inv;
  if (quad == 0 && a.lse != nullptr) a.lse[(int64_t)query * a.Hq + head] = sum == 0.f ? -INF : (s_total[0] + log2f(sum)) * LN2;
}

__global__ __launch_bounds__(256) void k_attention_spans(const int32_t* offsets, int documents, const int32_t* prefix, int causal, int T, int2* spans) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= T) return;
  int lo = -1, hi = documents;   // offsets[lo] <= t < offsets[hi]; offsets beyond the ends are as if they were far away
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (offsets[mid] <= t) lo = mid; else hi = mid;
  }
  int2 s = make_int2(0, 0);
  if (lo >= 0 && t < offsets[lo + 1]) {
    const int first = max(offsets[lo], 0);
    s = make_int2(first, min(offsets[lo + 1], T));
    if (causal) s.y = min(s.y, max(t + 1, prefix == nullptr ? 0 : first + min(max(prefix[lo], 0), T)));
  }
  spans[t] = s;
}

// What a call looks like: rows of a workgroup, and into how many parts the keys are cut.  Where even workgroups of 32 rows leave CUs without one the keys are split, into as many parts as
// there is room for at once: workgroups of 128 KB of LDS have a CU each, those of 64 KB (bf16, widths up to 64) share it in twos.  us of two new tokens over caches of 24000 keys each, by the
// workgroups before the split and the parts:
//   bf16, width 128: 5 in 51 parts 29, in 64 38; 10 in 25 45, in 51 50; 33 in 7 142, in 15 145.  fp32, width 64: 5 in 51 37, in 64 51; 10 in 25 56, in 51 64; 33 in 7 179, in 15 174
//   fp32, width 128: 5 in 51 95, in 64 149; 10 in 25 176, in 51 185
// Two rounds, where that is one part more than twice as many and parts are few but long enough: bf16, width 128, 100 in 5 443, in 2 482; 130 in 3 602, in 1 763 (of 2048 keys each: 57, 61, but 100 in 5
// 45, in 2 42); fp32, width 64, 100 in 5 521, in 2 629; 130 in 3 782, in 1 1139; fp32, width 128, 130 in 3 2698, in 1 4002; bf16, width 64, 200 in 5 472, in 2 526 (of 2048 keys: 43, 40).
constexpr int64_t LEAST_KEYS = 512, CUS = 256;
constexpr int narrow_groups(int row_bytes) { return row_bytes > 256 ? 2 : 4; }                        // KG of workgroups of 32 rows
constexpr int narrow_lds(int row_bytes) { return 4 * 32 * narrow_groups(row_bytes) * row_bytes; }
struct Plan { int rows, tiles, parts; };
Plan plan(int64_t Tq, int64_t Tk, int Hq, int Hk, int width, bool bf16) {
  const int64_t rows = Tq * (Hq / Hk), narrow = (rows + 31) / 32 * Hk, places = CUS * (LDS_MAX / narrow_lds(width * (bf16 ? 2 : 4)));
  Plan p;
  p.rows = rows_of_workgroup(rows, Hk, width, bf16);
  p.tiles = (int)((rows + p.rows - 1) / p.rows);
  p.parts = 1;
  if (rows > 0 && narrow <= CUS) {
    const int64_t one = places / narrow, two = 2 * places / narrow, parts = one <= 2 && two > 2 * one && Tk >= 2 * LEAST_KEYS * two ? two : one;
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>({parts, Tk / LEAST_KEYS, MOST_PARTS}));
  }
  return p;
}

template <typename E, typename C, int SHAPE>
void launch(hipStream_t st, const AttentionArgs& a, const Plan& p, void* workspace) {
  static const bool once = [] {
    (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&k_attention<E, C, SHAPE>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    return true;
  }();
  (void)once;
  const int64_t rows = a.Tq * (a.Hq / a.Hk);
  Parts parts{static_cast<float*>(workspace), nullptr, p.parts};
  parts.lse = parts.o + (size_t)p.parts * a.Hk * rows * a.D;
  ProfScope ps(st, F_OTHER, 0.0);
  launch_kernel(ps, k_attention<E, C, SHAPE>, dim3((unsigned)(p.tiles * (int64_t)a.Hk), p.parts), C::THREADS, C::LDS, st, a, parts, p.tiles);
  if (p.parts > 1) launch_kernel(ps, k_attention_join<E>, dim3((unsigned)(rows * a.Hk)), 256, 0, st, a, parts);
}
template <typename E, int DP>
void launch_width(hipStream_t st, const AttentionArgs& a, void* workspace) {
  const Plan p = plan(a.Tq, a.Tk, a.Hq, a.Hk, DP, sizeof(E) == 2);
  auto run = [&](auto config) {
    typedef decltype(config) C;
    switch ((a.cap > 0.f ? CAPPED : 0) | (a.slopes != nullptr ? BIASED : 0)) {
      case PLAIN: return launch<E, C, PLAIN>(st, a, p, workspace);
      case CAPPED: return launch<E, C, CAPPED>(st, a, p, workspace);
      case BIASED: return launch<E, C, BIASED>(st, a, p, workspace);
      default: return launch<E, C, CAPPED | BIASED>(st, a, p, workspace);
    }
  };
  constexpr bool LONG = sizeof(E) * DP > 256;
  if constexpr (DP > 64) if (p.rows == 128) return run(Config<E, DP, 4, 1, LONG ? 1 : 2>{});
  if constexpr (!LONG) if (p.rows == 64) return run(Config<E, DP, 2, 2, 1>{});
  typedef Config<E, DP, 1, narrow_groups(DP * sizeof(E)), 1> Narrow;
  static_assert(Narrow::LDS == narrow_lds(DP * sizeof(E)), "what plan() counts with");
  run(Narrow{});
}
}  // namespace

void launch_attention_spans(hipStream_t st, const int32_t* offsets, int64_t documents, const int32_t* prefix, bool causal, int64_t T, int32_t* spans) {
  ProfScope ps(st, F_OTHER, 8.0 * T);
  launch_kernel(ps, k_attention_spans, dim3((unsigned)((T + 255) / 256)), 256, 0, st, offsets, (int)documents, prefix, causal ? 1 : 0, (int)T, reinterpret_cast<int2*>(spans));
}

size_t attention_bytes(int64_t Tq, int64_t Tk, int Hq, int Hk, int D, bool bf16) {
  const Plan p = plan(Tq, Tk, Hq, Hk, D <= 64 ? 64 : 128, bf16);
  return p.parts <= 1 ? 256 : (size_t)p.parts * Tq * Hq * (D + 1) * sizeof(float);
}
void launch_attention(hipStream_t st, const AttentionArgs& a, bool bf16, void* workspace) {
  if (bf16) a.D <= 64 ? launch_width<bf16_t, 64>(st, a, workspace) : launch_width<bf16_t, 128>(st, a, workspace);
  else a.D <= 64 ? launch_width<float, 64>(st, a, workspace) : launch_width<float, 128>(st, a, workspace);
}

}  // namespace sama
