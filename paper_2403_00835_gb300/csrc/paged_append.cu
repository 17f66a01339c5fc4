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

// grid: (rows, parts); the heads of a row, queries first, are dealt to the parts.
template <class T, int HD>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(const PagedAppendArgs a) {
  using V = Vec16<T>;
  constexpr int kLanes = HD / 2 / V::n;             // threads of one head
  constexpr int kHeads = kAppendThreads / kLanes;   // heads at a time
  const int t = blockIdx.x, d = (threadIdx.x % kLanes) * V::n;
  const int all = a.H + 2 * a.Hkv, step = kHeads * gridDim.y;
  pdl_launch_dependents();
  pdl_wait();
  const long long slot = a.slots[t];
  const bool stored = slot >= 0 && (slot >> a.page_shift) < a.n_pages;
  bool rotated = a.rope != nullptr;
  float2 cs[V::n];
  if (rotated) {
    const int pos = a.positions[t];
    rotated = static_cast<unsigned>(pos) < static_cast<unsigned>(a.max_pos);
    if (rotated) {
#pragma unroll
      for (int i = 0; i < V::n; i += 2) {
        const float4 x = *reinterpret_cast<const float4*>(a.rope + static_cast<size_t>(pos) * (HD / 2) + d + i);
        cs[i] = make_float2(x.x, x.y);
        cs[i + 1] = make_float2(x.z, x.w);
      }
    }
  }
  const bool skip = a.rope != nullptr && !rotated;  // a position outside the table: the row is left out
  if (threadIdx.x == 0 && blockIdx.y == 0 && (skip || (slot != -1 && !stored))) atomicOr(a.err, DERR_CAPACITY);
  if (skip) return;
  const long long page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
  const size_t at = static_cast<size_t>(page * a.s_page + off * a.s_pos);
  for (int h = blockIdx.y * kHeads + threadIdx.x / kLanes; h < all; h += step) {
    const T* src;
    T* dst;
    if (h < a.H) {
      src = static_cast<const T*>(a.q) + t * a.q_row + static_cast<size_t>(h) * HD;
      dst = static_cast<T*>(a.q_out) + t * a.qo_row + static_cast<size_t>(h) * HD;
    } else {
      if (!stored) break;
      const int g = h - a.H;
      if (g < a.Hkv) {
        src = static_cast<const T*>(a.k) + t * a.k_row + static_cast<size_t>(g) * HD;
        dst = static_cast<T*>(a.kp) + at + g * a.s_head;
      } else {
        src = static_cast<const T*>(a.v) + t * a.v_row + static_cast<size_t>(g - a.Hkv) * HD;
        dst = static_cast<T*>(a.vp) + at + (g - a.Hkv) * a.s_head;
      }
    }
    if (rotated && h < a.H + a.Hkv) {
      float x[V::n], y[V::n];
      V::load(src + d, x);
      V::load(src + d + HD / 2, y);
#pragma unroll
      for (int i = 0; i < V::n; ++i) {
        const float u = x[i], w = y[i];
        x[i] = u * cs[i].x - w * cs[i].y;
        y[i] = w * cs[i].x + u * cs[i].y;
      }
      V::store(dst + d, x);
      V::store(dst + d + HD / 2, y);
    } else {
      const uint4 x = *reinterpret_cast<const uint4*>(src + d), y = *reinterpret_cast<const uint4*>(src + d + HD / 2);
      *reinterpret_cast<uint4*>(dst + d) = x;
      *reinterpret_cast<uint4*>(dst + d + HD / 2) = y;
    }
  }
}

template <class T>
cudaError_t launch_append(const PagedAppendArgs& a, cudaStream_t s) {
  const int kHeads = kAppendThreads / (a.hd / 2 / Vec16<T>::n);
  // few rows: a row's heads are spread over as many CTAs as there are groups of heads
  const int groups = (a.H + 2 * a.Hkv + kHeads - 1) / kHeads;
  const dim3 grid(a.T, a.T < 2 * 152 ? groups : 1);
  return launch_after(a.hd == 128 ? paged_append_kernel<T, 128> : paged_append_kernel<T, 64>, grid, kAppendThreads, 0, s,
                      a);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, int dtype, cudaStream_t s) {
  if (dtype == CLLM_F32) return launch_append<float>(a, s);
  if (dtype == CLLM_BF16) return launch_append<__nv_bfloat16>(a, s);
  return launch_append<__half>(a, s);
}

}  // namespace cllm
