// Rows of a rotary table (cllm_rope_table): amplitude * (cos, sin)(p f_i) for positions p and
// frequencies f_i.
//
// The angle in turns is held as a 64-bit fraction g_i = f_i / 2 pi mod 1, so that p g_i is exact modulo
// a turn in one integer multiplication, whatever the position (the product p f_i itself would need 24
// bits beside those of the turns).
//
// Bound: the bytes written, 8 to a pair; the arithmetic (25 instructions a pair) is close behind.  Measured: 2^20
// positions of 64 pairs 73.9 us, 7.3 TB/s (110 with a product, a division and the library's functions for
// every pair); 8192 of 32 2.4 us, of which a launch is 1.9.
#include "internal.cuh"
#include "paged.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTurns = 16;  // stores of a thread, at most

struct RopeArgs {
  float2* table;
  unsigned first, positions;
  int per;               // pairs of a position
  int unit, lanes, side; // positions of a unit (an even number of pairs), its threads, units side by side in a CTA
  int turns;             // stores of a thread
  float amplitude;
  unsigned long long g[kRopeDims / 2];
};

// (cos, sin) of a fraction of a turn in 2^-64: what is left of it beside the nearest quarter, as y
// eighths of a turn, |y| <= 1, and the Taylor series of both at (pi / 4) y to y^10, whose rests are
// below 2^-28.  (y is the high word's 32 bits rounded to 24: off by 2^-24 of itself.)
__device__ __forceinline__ float2 cos_sin(unsigned long long turn) {
  const unsigned hi = static_cast<unsigned>(turn >> 32), quarter = (hi + (1u << 29)) >> 30;
  const float y = static_cast<float>(static_cast<int>(static_cast<unsigned>(turn >> 30))) * 0x1p-31f, z = y * y;
  constexpr double q = 0.78539816339744830962, q2 = q * q;  // pi / 4
  constexpr float s1 = q, s3 = -q * q2 / 6, s5 = q * q2 * q2 / 120, s7 = -q * q2 * q2 * q2 / 5040,
                  s9 = q * q2 * q2 * q2 * q2 / 362880;
  constexpr float c2 = -q2 / 2, c4 = q2 * q2 / 24, c6 = -q2 * q2 * q2 / 720, c8 = q2 * q2 * q2 * q2 / 40320,
                  c10 = -q2 * q2 * q2 * q2 * q2 / 3628800;
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, s9, s7), s5), s3), s1);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, c10, c8), c6), c4), c2), 1.f);
  const float u = quarter & 1 ? s : c, v = quarter & 1 ? c : s;  // cos (q + a) = -+ sin a where q is odd
  return make_float2(__uint_as_float(__float_as_uint(u) ^ ((quarter + 1) << 30 & 0x80000000u)),
                     __uint_as_float(__float_as_uint(v) ^ (quarter << 30 & 0x80000000u)));
}

// A thread keeps its two pairs of a unit and goes from unit to unit: a step adds to its fractions.
__global__ void __launch_bounds__(kRopeThreads) paged_rope_kernel(const __grid_constant__ RopeArgs a) {
  const int at = threadIdx.x / a.lanes, e = (threadIdx.x - at * a.lanes) * 2;
  pdl_launch_dependents();
  if (at >= a.side) return;
  const int o0 = e >= a.per, o1 = e + 1 >= a.per;  // position in the unit
  const unsigned long long g0 = a.g[e - o0 * a.per], g1 = a.g[e + 1 - o1 * a.per];
  unsigned pos = (blockIdx.x * (a.side * a.turns) + at) * static_cast<unsigned>(a.unit);
  const unsigned step = a.side * a.unit;
  unsigned long long x = (a.first + pos + o0) * g0, y = (a.first + pos + o1) * g1;
  float2* to = a.table + static_cast<size_t>(pos) * a.per + e;
  pdl_wait();
#pragma unroll 2
  for (int k = 0; k < a.turns; ++k) {
    if (pos + o0 >= a.positions) break;
    const float2 u = cos_sin(x), v = cos_sin(y);
    if (pos + o1 < a.positions) {
      *reinterpret_cast<float4*>(to) = make_float4(a.amplitude * u.x, a.amplitude * u.y, a.amplitude * v.x, a.amplitude * v.y);
    } else {
      *to = make_float2(a.amplitude * u.x, a.amplitude * u.y);
    }
    x += step * g0, y += step * g1;
    pos += step, to += static_cast<size_t>(step) * a.per;
  }
}

}  // namespace

cudaError_t launch_rope_table(float* table, int first, int positions, int dims, const unsigned long long* turns,
                              float amplitude, cudaStream_t s) {
  RopeArgs a;
  a.table = reinterpret_cast<float2*>(table);
  a.first = first, a.positions = positions, a.per = dims / 2, a.amplitude = amplitude;
  a.unit = a.per % 2 ? 2 : 1;  // (a store takes two pairs)
  a.lanes = a.per * a.unit / 2;
  a.side = kRopeThreads / a.lanes;
  const int units = (positions - 1) / a.unit + 1;
  a.turns = min(max(units / (a.side * 152 * 8), 1), kRopeTurns);
  for (int i = 0; i < kRopeDims / 2; ++i) a.g[i] = i < a.per ? turns[i] : 0;
  return launch_after(paged_rope_kernel, dim3((units - 1) / (a.side * a.turns) + 1), kRopeThreads, 0, s, a);
}

}  // namespace cllm
