// Rotary positions with several axes: of each head's first R values, pair i turns by the angle phi_i = pos[axis(i)] base^(-2 i / R),
//   (x, y) -> (x cos phi - y sin phi, x sin phi + y cos phi),
// and by -phi_i in the inverse, which is also the gradient.  Bound by memory: every value is read and written once,
// 134 MB for 16384 tokens and 32 heads of 64 in bf16: 28.8 us, 4.7 TB/s (21.5 us where the values are still in the last-level cache).
//
// A workgroup takes a few tokens: first their cosines and sines into LDS, one pair a thread, then all heads, 16 bytes of a row (of both halves) a thread.  Angles
// are 64-bit turns: at position 10^6 an fp32 angle has two digits left behind the point.  The turn is reduced to an eighth either way in 64 bits, so that what is
// rounded to fp32 is at most an eighth of a turn and its sine and cosine are within 1.5 units of the last place.
#include <algorithm>
#include <cmath>
#include "kernels.h"
#include "sequence_ops.h"

namespace sama {
namespace {

constexpr int THREADS = 256, MAX_ANGLES = 2048;

struct RotaryTable {
  RotaryArgs a;
  int tokens;                               // of a workgroup
  double rate[ROTARY_MAX_PAIRS];            // turns for each position
  uint8_t axis[ROTARY_MAX_PAIRS];
};
static_assert(sizeof(RotaryTable) <= 4000, "kernel arguments");

template <typename E, int V> struct alignas(V * sizeof(E)) Piece { E v[V]; };
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(bf16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ void put(float& to, float x) { to = x; }
__device__ __forceinline__ void put(bf16_t& to, float x) { to = f32_to_bf16(x); }

// V: values of a piece (1: rows that do not consist of such pieces).  PAIRED: neighbours turn together, else value i with i + R / 2.
template <typename E, int V, bool PAIRED>
__global__ __launch_bounds__(THREADS) void k_rotary(RotaryTable t) {
  const RotaryArgs& a = t.a;
  __shared__ float2 turn[MAX_ANGLES];
  const int pairs = a.R / 2;
  const int64_t first = (int64_t)blockIdx.x * t.tokens;
  const int count = (int)min((int64_t)t.tokens, a.T - first);
  for (int i = threadIdx.x; i < count * pairs; i += THREADS) {
    const int token = i / pairs, pair = i - token * pairs;
    const double turns = (double)a.positions[t.axis[pair] * a.T + first + token] * t.rate[pair];
    const double part = turns - rint(turns), quarter = rint(4.0 * part);
    float s, c;
    sincospif((float)(2.0 * (part - 0.25 * quarter)), &s, &c);
    const int q = (int)quarter & 3;
    const float cq = q & 1 ? -s : c, sq = q & 1 ? c : s;            // a quarter further, then half a turn
    turn[i] = make_float2(q & 2 ? -cq : cq, (q & 2) != (a.inverse ? 2 : 0) ? -sq : sq);
  }
  __syncthreads();
  const bool in_place = a.out == a.x.p;
  const int turned = V == 1 ? pairs : PAIRED ? a.R / V : pairs / V, units = turned + (in_place ? 0 : (a.D - a.R) / V);
  const int per_token = units * a.H;
  typedef Piece<E, V> P;
  for (int i = threadIdx.x; i < count * per_token; i += THREADS) {
    const int token = i / per_token, rest = i - token * per_token, head = rest / units, u = rest - head * units;
    const E* const x = static_cast<const E*>(a.x.p) + (first + token) * a.x.ld + head * a.x.hs;
    E* const y = static_cast<E*>(a.out) + (first + token) * a.ldo + head * a.hso;
    const float2* const w = turn + token * pairs;
    if (u >= turned) {
      const int at = a.R + (u - turned) * V;
      *reinterpret_cast<P*>(y + at) = *reinterpret_cast<const P*>(x + at);
    } else if (PAIRED && V > 1) {
      P p = *reinterpret_cast<const P*>(x + u * V);
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        const float2 cs = w[u * (V / 2) + e];
        const float m = value(p.v[2 * e]), n = value(p.v[2 * e + 1]);
        put(p.v[2 * e], m * cs.x - n * cs.y); put(p.v[2 * e + 1], m * cs.y + n * cs.x);
      }
      *reinterpret_cast<P*>(y + u * V) = p;
    } else {
      const int at = PAIRED ? 2 * u : u * V, other = PAIRED ? at + 1 : at + pairs;
      P p = *reinterpret_cast<const P*>(x + at), r = *reinterpret_cast<const P*>(x + other);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 cs = w[u * V + e];
        const float m = value(p.v[e]), n = value(r.v[e]);
        put(p.v[e], m * cs.x - n * cs.y); put(r.v[e], m * cs.y + n * cs.x);
      }
      *reinterpret_cast<P*>(y + at) = p; *reinterpret_cast<P*>(y + other) = r;
    }
  }
}

template <typename E, int V>
void launch(hipStream_t st, const RotaryTable& t) {
  ProfScope ps(st, F_OTHER, 2.0 * t.a.T * t.a.H * t.a.D * sizeof(E));
  const dim3 grid((unsigned)((t.a.T + t.tokens - 1) / t.tokens));
  if (t.a.neighbours) launch_kernel(ps, k_rotary<E, V, true>, grid, THREADS, 0, st, t);
  else launch_kernel(ps, k_rotary<E, V, false>, grid, THREADS, 0, st, t);
}
}  // namespace

void launch_rotary(hipStream_t st, const RotaryArgs& a) {
  RotaryTable t;
  t.a = a;
  const int pairs = a.R / 2;
  const double step = 2.0 / a.R * std::log2(a.base);
  for (int axis = 0, i = 0; axis < a.axes; ++axis)
    for (int end = i + a.sections[axis]; i < end; ++i) { t.axis[i] = (uint8_t)axis; t.rate[i] = std::exp2(-step * i) * 0.15915494309189533577; }
  // 32 KB of rows a workgroup, fewer where that would leave CUs without one; no more angles than LDS is set aside for
  const int size = a.bf16 ? 2 : 4;
  const int64_t tokens = std::min<int64_t>({32768 / ((int64_t)a.H * a.D * size), a.T / 1024, MAX_ANGLES / pairs});
  t.tokens = (int)std::max<int64_t>(tokens, 1);
  auto fits = [&](int v) {
    const int bytes = v * size;
    return (uintptr_t)a.x.p % bytes == 0 && (uintptr_t)a.out % bytes == 0 && a.x.ld % v == 0 && a.x.hs % v == 0 && a.ldo % v == 0 && a.hso % v == 0 &&
           (a.neighbours ? a.R : pairs) % v == 0 && (a.D - a.R) % v == 0;
  };
  if (a.bf16) {
    if (fits(8)) launch<bf16_t, 8>(st, t);
    else if (fits(4)) launch<bf16_t, 4>(st, t);
    else launch<bf16_t, 1>(st, t);
  } else {
    if (fits(4)) launch<float, 4>(st, t);
    else launch<float, 1>(st, t);
  }
}

}  // namespace sama
