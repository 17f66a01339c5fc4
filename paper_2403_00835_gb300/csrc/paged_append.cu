// The write of a step's keys and values into their pages (cllm_paged_append,
// cllm_paged_append_heads), with norms of K and Q per head and their rotary embedding:
//
//   norm(x) = x / sqrt(sum x^2 / hd + eps) * gain
//   rope(x)_i = x_i cos - x_j sin,  rope(x)_j = x_j cos + x_i sin,  j = i + r/2, or i even and j = i + 1
//
// in fp32, rounded once.  Bound: HBM, every value read once and written once.
// A thread holds two pieces of 16 bytes of a head and their cosines and sines, which serve all
// of its heads of that row; the threads of a head are neighbours, which add up its squares.
// The loads of two heads are under way before the row's slot and position are known.
//
// Small CTAs (2 warps) of a row each: a CTA's heads are a loop of several turns after one wait for
// slot, position and table, and 14 to 16 of them on an SM keep its loads apart in time.  Measured, 8192
// rows of 32 + 2 x 32 heads of 128 in bf16: rotated 62.5 us, 6.5 TB/s; normalised too 66.8, 6.1
// (CTAs of 4 warps 61.4 and 67.3 to 71, of 8 warps 70.9 and 94.5; one head's loads at a time 63.2
// and 76, three 62.4 and 65 to 69, four 62.0 and 72); 256 rows of 32 + 2 x 8 heads 3.2 us, 16 rows 2.2 us (an
// empty launch of the kind takes 1.9).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "act.cuh"
#include "paged.cuh"
#include "internal.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kAppendThreads = 64;
constexpr int kAppendAhead = 2;  // heads of a thread on their way

template <class T> struct Vec16;  // 16 bytes of T as floats
template <> struct Vec16<float> {
  static constexpr int n = 4;
  static __device__ void unpack(const uint4& x, float (&v)[4]) {
    v[0] = __uint_as_float(x.x), v[1] = __uint_as_float(x.y), v[2] = __uint_as_float(x.z), v[3] = __uint_as_float(x.w);
  }
  static __device__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};
template <> struct Vec16<__half> {
  static constexpr int n = 8;
  static __device__ void unpack(const uint4& x, float (&v)[8]) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
  }
  static __device__ uint4 pack(const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ void unpack(const uint4& x, float (&v)[8]) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ uint4 pack(const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};

// Head h of a row, queries first, then keys, then values: where it comes from, and goes to.
template <class T, int HD>
__device__ __forceinline__ const T* head_from(const PagedAppendArgs& a, int t, int h) {
  if (h < a.H) return static_cast<const T*>(a.q) + t * a.q_row + static_cast<size_t>(h) * HD;
  const int g = h - a.H;
  return g < a.Hkv ? static_cast<const T*>(a.k) + t * a.k_row + static_cast<size_t>(g) * HD
                   : static_cast<const T*>(a.v) + t * a.v_row + static_cast<size_t>(g - a.Hkv) * HD;
}
template <class T, int HD>
__device__ __forceinline__ T* head_to(const PagedAppendArgs& a, int t, int h, size_t at) {
  if (h < a.H) return static_cast<T*>(a.q_out) + t * a.qo_row + static_cast<size_t>(h) * HD;
  const int g = h - a.H;
  return (g < a.Hkv ? static_cast<T*>(a.kp) + g * a.s_head : static_cast<T*>(a.vp) + (g - a.Hkv) * a.s_head) + at;
}

// What a launch's heads need: a rotation of whole heads in halves (or none), any rotation, norms too.
enum AppendKind { kWhole, kTurned, kNormed };

// grid: (rows, parts); the heads of a row, queries first, are dealt to the parts.  A thread's
// two pieces of 16 bytes: pairs of halves are element by element of two pieces, r/2 apart; what is
// not rotated comes in neighbouring pieces after them.  Neighbours in pairs lie in one piece.
template <class T, int HD, AppendKind KIND>
__global__ void __launch_bounds__(kAppendThreads, KIND == kNormed ? 14 : 16) paged_append_kernel(const PagedAppendArgs a) {
  using V = Vec16<T>;
  constexpr int kLanes = HD / 2 / V::n;             // threads of one head
  constexpr int kHeads = kAppendThreads / kLanes;   // heads at a time
  constexpr int U = kAppendAhead;
  const int t = blockIdx.x, lane = threadIdx.x % kLanes;
  const int all = a.H + 2 * a.Hkv, step = kHeads * gridDim.y, turned_heads = a.rope != nullptr ? a.H + a.Hkv : 0;
  // pieces between the two of a thread that is rotated
  const int half = KIND == kWhole || a.interleaved ? kLanes : a.dims / 2 / V::n;
  const int p0 = lane < half ? lane : 2 * lane, p1 = lane < half ? lane + half : 2 * lane + 1;
  const bool turn0 = KIND == kWhole || p0 * V::n < a.dims, turn1 = KIND == kWhole || p1 * V::n < a.dims;
  const bool inter = KIND != kWhole && a.interleaved;
  pdl_launch_dependents();
  pdl_wait();
  // (all lanes of a warp go round together: with norms they exchange sums)
  int h0 = blockIdx.y * kHeads + threadIdx.x / kLanes;
  const int end = all + (threadIdx.x % 32) / kLanes;
  uint4 x[U], y[U];
  auto load = [&] {  // the next heads, U at a time
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * step;
      if (h < all) {
        const T* from = head_from<T, HD>(a, t, h);
        x[u] = *reinterpret_cast<const uint4*>(from + p0 * V::n);
        y[u] = *reinterpret_cast<const uint4*>(from + p1 * V::n);
      } else {
        x[u] = y[u] = make_uint4(0, 0, 0, 0);
      }
    }
  };
  load();
  const long long slot = a.slots[t];
  const bool stored = slot >= 0 && (slot >> a.page_shift) < a.n_pages;
  bool skip = false;  // a position outside the table: the row is left out
  float2 cs[V::n];
  if (a.rope != nullptr) {
    const int pos = a.positions[t];
    skip = static_cast<unsigned>(pos) >= static_cast<unsigned>(a.max_pos);
    if (!skip) {
      const float2* row = a.rope + static_cast<size_t>(pos) * ((KIND == kWhole ? HD : a.dims) / 2);
#pragma unroll
      for (int i = 0; i < V::n; i += 2) {
        // half: the n pairs of this thread; interleaved: n / 2 of either piece
        const int at = !inter ? p0 * V::n + i : (i < V::n / 2 ? p0 : p1 - 1) * (V::n / 2) + i;
        if (i < V::n / 2 || !inter ? turn0 : turn1) {
          const float4 c = *reinterpret_cast<const float4*>(row + at);
          cs[i] = make_float2(c.x, c.y);
          cs[i + 1] = make_float2(c.z, c.w);
        }
      }
    }
  }
  if (threadIdx.x == 0 && blockIdx.y == 0 && (skip || (slot != -1 && !stored))) atomicOr(a.err, DERR_CAPACITY);
  if (skip) return;
  const long long page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
  const size_t at = static_cast<size_t>(page * a.s_page + off * a.s_pos);
  for (; h0 < end; h0 += U * step, load()) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * step;
      const bool live = h < all && (stored || h < a.H);
      const T* gain = nullptr;
      if constexpr (KIND == kNormed) gain = h < a.H ? static_cast<const T*>(a.q_gain) : h < a.H + a.Hkv ? static_cast<const T*>(a.k_gain) : nullptr;
      if (KIND != kNormed && !live) continue;
      if (KIND == kNormed || h < turned_heads) {
        float v[V::n], w[V::n];
        V::unpack(x[u], v);
        V::unpack(y[u], w);
        if constexpr (KIND == kNormed) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < V::n; ++i) sum = fmaf(v[i], v[i], fmaf(w[i], w[i], sum));
#pragma unroll
          for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
          if (!live) continue;
          if (gain != nullptr) {
            const float r = rsqrtf(sum * (1.f / HD) + a.eps);
            float g[V::n];
            V::unpack(*reinterpret_cast<const uint4*>(gain + p0 * V::n), g);
#pragma unroll
            for (int i = 0; i < V::n; ++i) v[i] *= r * g[i];
            V::unpack(*reinterpret_cast<const uint4*>(gain + p1 * V::n), g);
#pragma unroll
            for (int i = 0; i < V::n; ++i) w[i] *= r * g[i];
          }
        }
        if (h < turned_heads) {
          if (inter) {
#pragma unroll
            for (int i = 0; i < V::n; i += 2) {
              const float e = v[i], f = v[i + 1], c = cs[i / 2].x, s = cs[i / 2].y;
              if (turn0) v[i] = e * c - f * s, v[i + 1] = f * c + e * s;
            }
#pragma unroll
            for (int i = 0; i < V::n; i += 2) {
              const float e = w[i], f = w[i + 1], c = cs[(V::n + i) / 2].x, s = cs[(V::n + i) / 2].y;
              if (turn1) w[i] = e * c - f * s, w[i + 1] = f * c + e * s;
            }
          } else if (turn0) {
#pragma unroll
            for (int i = 0; i < V::n; ++i) {
              const float e = v[i], f = w[i];
              v[i] = e * cs[i].x - f * cs[i].y;
              w[i] = f * cs[i].x + e * cs[i].y;
            }
          }
        }
        if (KIND != kNormed || gain != nullptr || h < turned_heads) x[u] = V::pack(v), y[u] = V::pack(w);
      }
      T* to = head_to<T, HD>(a, t, h, at);
      *reinterpret_cast<uint4*>(to + p0 * V::n) = x[u];
      *reinterpret_cast<uint4*>(to + p1 * V::n) = y[u];
    }
  }
}

template <class T>
cudaError_t launch_append(const PagedAppendArgs& a, cudaStream_t s) {
  const int kHeads = kAppendThreads / (a.hd / 2 / Vec16<T>::n);
  // few rows: a row's heads are spread over as many CTAs as there are groups of heads
  const int groups = (a.H + 2 * a.Hkv + kHeads - 1) / kHeads;
  const dim3 grid(a.T, a.T < 2 * 152 ? groups : 1);
  auto launch = [&](auto kernel) { return launch_after(kernel, grid, kAppendThreads, 0, s, a); };
  auto kind = [&](auto whole, auto turned, auto normed) {
    if (a.q_gain != nullptr || a.k_gain != nullptr) return launch(normed);
    return a.interleaved || (a.rope != nullptr && a.dims != a.hd) ? launch(turned) : launch(whole);
  };
  if (a.hd == 128)
    return kind(paged_append_kernel<T, 128, kWhole>, paged_append_kernel<T, 128, kTurned>, paged_append_kernel<T, 128, kNormed>);
  return kind(paged_append_kernel<T, 64, kWhole>, paged_append_kernel<T, 64, kTurned>, paged_append_kernel<T, 64, kNormed>);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, int dtype, cudaStream_t s) {
  if (dtype == CLLM_F32) return launch_append<float>(a, s);
  if (dtype == CLLM_BF16) return launch_append<__nv_bfloat16>(a, s);
  return launch_append<__half>(a, s);
}

}  // namespace cllm
