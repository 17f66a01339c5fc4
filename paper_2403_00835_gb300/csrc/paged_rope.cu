// Rows of a rotary table (cllm_rope_table): amplitude * (cos, sin)(p f_i) for positions p and
// frequencies f_i.
//
// The angle in turns is held as a 64-bit fraction g_i = f_i / 2 pi mod 1, so that p g_i is exact modulo
// a turn in one integer multiplication, whatever the position (the product p f_i itself would need 24
// bits beside those of the turns).
//
// Bound: the bytes written, 8 to a pair.
#include "internal.cuh"
#include "paged.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopePairs = 16;  // pairs of a thread, two to a store

struct RopeArgs {
  float4* table;
  long long pairs;  // all of the table's
  unsigned first;
  int per;          // pairs of a position
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

__global__ void __launch_bounds__(kRopeThreads) paged_rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ unsigned long long g[kRopeDims / 2];
  if (threadIdx.x < static_cast<unsigned>(a.per)) g[threadIdx.x] = a.g[threadIdx.x];
  __syncthreads();
  pdl_launch_dependents();
  const long long base = static_cast<long long>(blockIdx.x) * (kRopeThreads * kRopePairs);
  const long long p0 = base / a.per;
  const int left = static_cast<int>(base - p0 * a.per);
  auto value = [&](unsigned pos, int i) {
    const float2 x = cos_sin(pos * g[i]);
    return make_float2(a.amplitude * x.x, a.amplitude * x.y);
  };
  pdl_wait();
#pragma unroll 4
  for (int u = 0; u < kRopePairs / 2; ++u) {
    const int e = (u * kRopeThreads + static_cast<int>(threadIdx.x)) * 2;  // this thread's pair of the block
    if (base + e >= a.pairs) break;
    unsigned pos = (left + e) / a.per;
    int i = left + e - pos * a.per;
    pos += a.first + static_cast<unsigned>(p0);
    const float2 x = value(pos, i);
    if (++i == a.per) i = 0, ++pos;
    float4* to = a.table + ((base + e) >> 1);
    if (base + e + 1 < a.pairs) {
      const float2 y = value(pos, i);
      *to = make_float4(x.x, x.y, y.x, y.y);
    } else {
      *reinterpret_cast<float2*>(to) = x;
    }
  }
}

}  // namespace

cudaError_t launch_rope_table(float* table, int first, int positions, int dims, const unsigned long long* turns,
                              float amplitude, cudaStream_t s) {
  RopeArgs a;
  a.table = reinterpret_cast<float4*>(table);
  a.first = first, a.per = dims / 2, a.amplitude = amplitude;
  a.pairs = static_cast<long long>(positions) * a.per;
  for (int i = 0; i < kRopeDims / 2; ++i) a.g[i] = i < a.per ? turns[i] : 0;
  constexpr long long block = kRopeThreads * kRopePairs;
  return launch_after(paged_rope_kernel, dim3(static_cast<unsigned>((a.pairs + block - 1) / block)), kRopeThreads, 0, s, a);
}

}  // namespace cllm
