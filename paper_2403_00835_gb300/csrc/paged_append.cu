// The write of a step's keys and values into their pages (cllm_paged_append),
// with the rotary embedding of K and Q:
//
//   rope(x)_i = x_i cos - x_{i+h/2} sin,  rope(x)_{i+h/2} = x_{i+h/2} cos + x_i sin
//
// in fp32, rounded once.  Bound: HBM, every value read once and written once.
// A thread holds 16 bytes of each half of a head and their cosines and sines,
// which serve all of its heads of that row; a row's threads cover 32 (16 in
// fp32) heads at a time, so loads and stores are whole 128-byte lines.  Measured: 8192
// rows, 32 + 2 x 32 heads of 128 in bf16: 64.7 us, 6.3 TB/s; 256 rows 3.6 us, 16 rows 1.9 us (an
// empty launch of the kind takes 1.9).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "act.cuh"
#include "paged.cuh"
#include "internal.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kAppendThreads = 256;

template <class T> struct Vec16;  // 16 bytes of T as floats
template <> struct Vec16<float> {
  static constexpr int n = 4;
  static __device__ void load(const float* p, float (&v)[4]) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
  }
  static __device__ void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <> struct Vec16<__half> {
  static constexpr int n = 8;
  static __device__ void load(const __half* p, float (&v)[8]) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
  }
  static __device__ void store(__half* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ void load(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  }
};

// Head h of row t, queries first, then keys, then values: where it comes from and goes to.
template <class T>
struct HeadAt {
  const T* src = nullptr;  // null: nothing to do
  T* dst = nullptr;
};
template <class T, int HD>
__device__ __forceinline__ HeadAt<T> head_at(const PagedAppendArgs& a, int t, int h, size_t at, bool stored) {
  HeadAt<T> r;
  if (h < a.H) {
    r.src = static_cast<const T*>(a.q) + t * a.q_row + static_cast<size_t>(h) * HD;
    r.dst = static_cast<T*>(a.q_out) + t * a.qo_row + static_cast<size_t>(h) * HD;
  } else if (stored && h < a.H + 2 * a.Hkv) {
    const int g = h - a.H;
    if (g < a.Hkv) {
      r.src = static_cast<const T*>(a.k) + t * a.k_row + static_cast<size_t>(g) * HD;
      r.dst = static_cast<T*>(a.kp) + at + g * a.s_head;
    } else {
      r.src = static_cast<const T*>(a.v) + t * a.v_row + static_cast<size_t>(g - a.Hkv) * HD;
      r.dst = static_cast<T*>(a.vp) + at + (g - a.Hkv) * a.s_head;
    }
  }
  return r;
}

// grid: (rows, parts); the heads of a row, queries first, are dealt to the parts.  A thread's
// two pieces of 16 bytes: pairs of halves are element by element of two pieces, r/2 apart; what is
// not rotated comes in neighbouring pieces after them.  Neighbours in pairs lie in one piece.
template <class T, int HD, bool NORM>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(const PagedAppendArgs a) {
  using V = Vec16<T>;
  constexpr int kLanes = HD / 2 / V::n;             // threads of one head
  constexpr int kHeads = kAppendThreads / kLanes;   // heads at a time
  const int t = blockIdx.x, lane = threadIdx.x % kLanes;
  const int all = a.H + 2 * a.Hkv, step = kHeads * gridDim.y;
  const int half = a.interleaved ? kLanes : a.dims / 2 / V::n;  // pieces between the two of a thread that is rotated
  const int p0 = lane < half ? lane : 2 * lane, p1 = lane < half ? lane + half : 2 * lane + 1;
  const bool turn0 = p0 * V::n < a.dims, turn1 = p1 * V::n < a.dims;
  pdl_launch_dependents();
  pdl_wait();
  const long long slot = a.slots[t];
  const bool stored = slot >= 0 && (slot >> a.page_shift) < a.n_pages;
  bool skip = false;  // a position outside the table: the row is left out
  float2 cs[V::n];
  if (a.rope != nullptr) {
    const int pos = a.positions[t];
    skip = static_cast<unsigned>(pos) >= static_cast<unsigned>(a.max_pos);
    if (!skip) {
      const float2* row = a.rope + static_cast<size_t>(pos) * (a.dims / 2);
#pragma unroll
      for (int i = 0; i < V::n; i += 2) {
        // half: the n pairs of this thread; interleaved: n / 2 of either piece
        const int at = !a.interleaved ? p0 * V::n + i : (i < V::n / 2 ? p0 : p1 - 1) * (V::n / 2) + i;
        if (i < V::n / 2 || !a.interleaved ? turn0 : turn1) {
          const float4 x = *reinterpret_cast<const float4*>(row + at);
          cs[i] = make_float2(x.x, x.y);
          cs[i + 1] = make_float2(x.z, x.w);
        }
      }
    }
  }
  if (threadIdx.x == 0 && blockIdx.y == 0 && (skip || (slot != -1 && !stored))) atomicOr(a.err, DERR_CAPACITY);
  if (skip) return;
  const long long page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
  const size_t at = static_cast<size_t>(page * a.s_page + off * a.s_pos);
  // (all lanes of a warp go round together: they exchange sums)
  for (int h0 = blockIdx.y * kHeads + threadIdx.x / 32 * (32 / kLanes); h0 < all; h0 += step) {
    const int h = h0 + threadIdx.x % 32 / kLanes;
    const HeadAt<T> w = head_at<T, HD>(a, t, h, at, stored);
    const bool key = h >= a.H;
    const T* gain = NORM && h < a.H + a.Hkv ? static_cast<const T*>(key ? a.k_gain : a.q_gain) : nullptr;
    const bool turned = h < a.H + a.Hkv && a.rope != nullptr;
    if constexpr (!NORM) {
      if (w.src == nullptr) continue;
      if (!turned) {
        const uint4 x = *reinterpret_cast<const uint4*>(w.src + p0 * V::n), y = *reinterpret_cast<const uint4*>(w.src + p1 * V::n);
        *reinterpret_cast<uint4*>(w.dst + p0 * V::n) = x;
        *reinterpret_cast<uint4*>(w.dst + p1 * V::n) = y;
        continue;
      }
    }
    float x[V::n], y[V::n];
    if (w.src != nullptr) {
      V::load(w.src + p0 * V::n, x);
      V::load(w.src + p1 * V::n, y);
    } else {
#pragma unroll
      for (int i = 0; i < V::n; ++i) x[i] = y[i] = 0.f;
    }
    if constexpr (NORM) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < V::n; ++i) sum = fmaf(x[i], x[i], fmaf(y[i], y[i], sum));
#pragma unroll
      for (int d = 1; d < kLanes; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (w.src == nullptr) continue;
      if (gain != nullptr) {
        const float r = rsqrtf(sum * (1.f / HD) + a.eps);
        float g[V::n];
        V::load(gain + p0 * V::n, g);
#pragma unroll
        for (int i = 0; i < V::n; ++i) x[i] *= r * g[i];
        V::load(gain + p1 * V::n, g);
#pragma unroll
        for (int i = 0; i < V::n; ++i) y[i] *= r * g[i];
      }
    }
    if (turned) {
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < V::n; i += 2) {
          const float u = x[i], v = x[i + 1], c = cs[i / 2].x, s = cs[i / 2].y;
          if (turn0) x[i] = u * c - v * s, x[i + 1] = v * c + u * s;
        }
#pragma unroll
        for (int i = 0; i < V::n; i += 2) {
          const float u = y[i], v = y[i + 1], c = cs[(V::n + i) / 2].x, s = cs[(V::n + i) / 2].y;
          if (turn1) y[i] = u * c - v * s, y[i + 1] = v * c + u * s;
        }
      } else if (turn0) {
#pragma unroll
        for (int i = 0; i < V::n; ++i) {
          const float u = x[i], v = y[i];
          x[i] = u * cs[i].x - v * cs[i].y;
          y[i] = v * cs[i].x + u * cs[i].y;
        }
      }
    }
    V::store(w.dst + p0 * V::n, x);
    V::store(w.dst + p1 * V::n, y);
  }
}

template <class T>
cudaError_t launch_append(const PagedAppendArgs& a, cudaStream_t s) {
  const int kHeads = kAppendThreads / (a.hd / 2 / Vec16<T>::n);
  // few rows: a row's heads are spread over as many CTAs as there are groups of heads
  const int groups = (a.H + 2 * a.Hkv + kHeads - 1) / kHeads;
  const dim3 grid(a.T, a.T < 2 * 152 ? groups : 1);
  auto launch = [&](auto kernel) { return launch_after(kernel, grid, kAppendThreads, 0, s, a); };
  if (a.q_gain != nullptr || a.k_gain != nullptr)
    return a.hd == 128 ? launch(paged_append_kernel<T, 128, true>) : launch(paged_append_kernel<T, 64, true>);
  return a.hd == 128 ? launch(paged_append_kernel<T, 128, false>) : launch(paged_append_kernel<T, 64, false>);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, int dtype, cudaStream_t s) {
  if (dtype == CLLM_F32) return launch_append<float>(a, s);
  if (dtype == CLLM_BF16) return launch_append<__nv_bfloat16>(a, s);
  return launch_append<__half>(a, s);
}

}  // namespace cllm
