// Verification of drafted tokens (cllm_verify): two launches.
//
//   p(x) = 2^(c (z_x - m)) / S,  S = sum_v 2^(c (z_v - m)),  c = log2(e) / temperature,  m = max z
//   a draft stands:  u q(x) < p(x);   next = argmax_v max(p - q, 0)_v / e_v
//
// The first kernel reads all logits once, a row in as many shares as fill the GPU: a thread
// keeps its running maximum and sum; the CTA that brings a row's last share adds them up in order and
// judges its draft.  The second finds each request's first row whose draft falls, and runs
// the race over that row, its vocabulary in parts; results meet in one atomicMax on (ratio, lowest
// index), whose order does not matter.
//
// c is held in two floats, the first rounded down, so that both products of an infinite
// difference have its sign.  Sums and probabilities are in fp32; a draft's own probability is
// taken in fp64 (its border decides), one a row.
//
// Bound: HBM, the logits.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.cuh"
#include "paged.cuh"
#include "ptx.cuh"
#include "verify.cuh"

namespace cllm {

namespace {

constexpr int kVThreads = 256, kVWarps = kVThreads / 32;
constexpr float kLog2eHi = 1.44269502162933349609f, kLog2eLo = 1.9259629911e-8f;

template <class T> struct Logits;  // 16 bytes of logits
template <> struct Logits<float> {
  static constexpr int n = 4;
  static __device__ void unpack(const uint4& x, float (&v)[4]) {
    v[0] = __uint_as_float(x.x), v[1] = __uint_as_float(x.y), v[2] = __uint_as_float(x.z), v[3] = __uint_as_float(x.w);
  }
  static __device__ float one(const float* p) { return *p; }
};
template <> struct Logits<__half> {
  static constexpr int n = 8;
  static __device__ void unpack(const uint4& x, float (&v)[8]) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
  }
  static __device__ float one(const __half* p) { return __half2float(*p); }
};
template <> struct Logits<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ void unpack(const uint4& x, float (&v)[8]) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(u[i] << 16), v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
  static __device__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};

// c = log2(e) / t in two floats, hi < c.
struct Heat {
  float hi, lo;
  int kind;  // 0, kNothing or kGreedy
};
__device__ __forceinline__ Heat heat_of(const VerifyArgs& a, int b) {
  if (a.race == nullptr) return {0.f, 0.f, kGreedy};
  const float t = a.temperature != nullptr ? a.temperature[b] : 1.f;
  if (!(t >= 0.f) || t > 0x1p40f) return {0.f, 0.f, kNothing};
  if (t < 0x1p-60f) return {0.f, 0.f, kGreedy};
  float hi = __fdiv_rn(kLog2eHi, t), rest = fmaf(-hi, t, kLog2eHi) + kLog2eLo;
  if (!(rest > 0.f)) {
    hi = __uint_as_float(__float_as_uint(hi) - 1);
    rest = fmaf(-hi, t, kLog2eHi) + kLog2eLo;
  }
  return {hi, rest / t, 0};
}
// c (z - m); m: at least z, or 0 where all are -inf
__device__ __forceinline__ float exponent(const Heat& c, float z, float m) {
  const float d = z - m;
  return fmaf(d, c.hi, d * c.lo);
}
// The sum of 2^(c (z - max)) over some values; max -inf: none of them is above that.
struct Share {
  float max, sum;
};
__device__ __forceinline__ Share plus(const Heat& c, const Share& x, const Share& y) {
  const float m = fmaxf(x.max, y.max), base = m == -INFINITY ? 0.f : m;
  return {m, x.sum * ex2_ftz(exponent(c, x.max, base)) + y.sum * ex2_ftz(exponent(c, y.max, base))};
}
__device__ __forceinline__ Share warp_plus(const Heat& c, Share s) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const Share o{__shfl_xor_sync(~0u, s.max, d), __shfl_xor_sync(~0u, s.sum, d)};
    s = plus(c, s, o);
  }
  return s;
}
// A value with its index, larger for larger values and then lower indices; 0: none.
__device__ __forceinline__ unsigned long long key_of(float v, int at) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return static_cast<unsigned long long>(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | ~static_cast<uint32_t>(at);
}
__device__ __forceinline__ int index_of(unsigned long long key) { return static_cast<int>(~static_cast<uint32_t>(key)); }
constexpr unsigned long long kBadKey = ~0ull;  // a value that is no number
__device__ __forceinline__ unsigned long long warp_largest(unsigned long long k) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const unsigned long long o = __shfl_xor_sync(~0u, k, d);
    if (o > k) k = o;
  }
  return k;
}
__device__ __forceinline__ unsigned long long pack(const Share& s) {
  return static_cast<unsigned long long>(__float_as_uint(s.max)) << 32 | __float_as_uint(s.sum);
}
__device__ __forceinline__ Share unpack(unsigned long long x) {
  return {__uint_as_float(static_cast<uint32_t>(x >> 32)), __uint_as_float(static_cast<uint32_t>(x))};
}

// The request that row `row` belongs to, by a warp: the last one that begins at or before it (-1: none).
__device__ __forceinline__ int request_of(const VerifyArgs& a, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = a.batch;  // among requests [lo, lo + n)
  for (;;) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const unsigned before = __ballot_sync(~0u, lane * step < n && a.row_start[at] <= row);
    if (before == 0) return -1;
    const int k = 31 - __clz(before);
    lo += k * step;
    if (step == 1) return lo;
    n = min(step, n - k * step);
  }
}
struct Rows {
  int first, end;
  bool live;
};
__device__ __forceinline__ Rows rows_of(const VerifyArgs& a, int b) {
  Rows r{a.row_start[b], a.row_start[b + 1], false};
  r.live = r.first >= 0 && r.end > r.first && r.end <= a.rows && r.end - r.first <= a.seq_len[b];
  return r;
}

// Vectors of 16 bytes from the first boundary on, single values before and after.
template <class T, class Vec, class One>
__device__ __forceinline__ void for_logits(const T* z, int from, int to, Vec vec, One one) {
  constexpr int n = Logits<T>::n, U = 4;
  const int tid = threadIdx.x, off = static_cast<int>(reinterpret_cast<uintptr_t>(z + from) & 15) / static_cast<int>(sizeof(T));
  const int head = min((n - off) % n, to - from), vecs = (to - from - head) / n, tail = from + head + vecs * n;
  const uint4* p = reinterpret_cast<const uint4*>(z + from + head);
  for (int i = tid; i < vecs; i += U * kVThreads) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * kVThreads < vecs) x[u] = p[i + u * kVThreads];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * kVThreads < vecs) vec(x[u], from + head + (i + u * kVThreads) * n);
  }
  if (tid < head) one(Logits<T>::one(z + from + tid), from + tid);
  if (tid < to - tail) one(Logits<T>::one(z + tail + tid), tail + tid);
}

template <class T>
__global__ void __launch_bounds__(kVThreads) verify_rows_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ unsigned long long sm[kVWarps];
  __shared__ int sm_request;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  pdl_launch_dependents();
  pdl_wait();
  if (warp == 0) {
    const int b = request_of(a, row);
    if (lane == 0) sm_request = b;
  }
  __syncthreads();
  const int b = sm_request;
  const Rows r = b >= 0 ? rows_of(a, b) : Rows{0, 0, false};
  if (!r.live) {
    if (b >= 0 && row < r.end && split == 0 && tid == 0 && a.target_probs != nullptr) a.target_probs[row] = 0.f;
    return;
  }
  if (row >= r.end) return;  // behind the last request
  const Heat c = heat_of(a, b);
  const T* z = static_cast<const T*>(a.logits) + row * a.logits_row;
  const int v0 = split * a.split_len, v1 = min(v0 + a.split_len, a.vocab);
  constexpr int n = Logits<T>::n;
  const bool greedy = c.kind == kGreedy;
  unsigned long long mine;
  if (greedy) {
    float top = -INFINITY;
    int at = a.vocab;
    bool bad = false;
    auto take = [&](float x, int i) {
      bad |= x != x;
      if (x > top || (x == top && i < at)) top = x, at = i;
    };
    for_logits<T>(z, v0, v1, [&](const uint4& raw, int i) {
      float x[n];
      Logits<T>::unpack(raw, x);
#pragma unroll
      for (int j = 0; j < n; ++j) take(x[j], i + j);
    }, take);
    mine = warp_largest(bad ? kBadKey : key_of(top, at));
  } else {
    Share s{-INFINITY, 0.f};
    auto raise = [&](float top) {
      if (!(top > s.max)) return;
      s.sum *= ex2_ftz(exponent(c, s.max, top));
      s.max = top;
    };
    auto base = [&] { return s.max == -INFINITY ? 0.f : s.max; };
    if (c.kind == 0)
      for_logits<T>(z, v0, v1, [&](const uint4& raw, int) {
        float x[n];
        Logits<T>::unpack(raw, x);
        float top = x[0];
#pragma unroll
        for (int j = 1; j < n; ++j) top = fmaxf(top, x[j]);
        raise(top);
        const float m = base();
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < n; ++j) t[j & 1] += ex2_ftz(exponent(c, x[j], m));
        s.sum += t[0] + t[1];
      }, [&](float x, int) {
        raise(x);
        s.sum += ex2_ftz(exponent(c, x, base()));
      });
    mine = pack(warp_plus(c, s));
  }
  if (lane == 0) sm[warp] = mine;
  __syncthreads();
  if (warp != 0) return;
  auto join = [&](unsigned long long x) { return greedy ? warp_largest(x) : pack(warp_plus(c, unpack(x))); };
  const unsigned long long none = greedy ? 0ull : pack(Share{-INFINITY, 0.f});
  mine = join(lane < kVWarps ? sm[lane] : none);
  if (a.splits > 1) {
    int last = 0;
    if (lane == 0) {
      a.shares[static_cast<size_t>(row) * a.splits + split] = mine;
      __threadfence();
      last = atomicAdd(&a.row_tickets[row], 1) == a.splits - 1;
      if (last) a.row_tickets[row] = 0;
      __threadfence();
    }
    last = __shfl_sync(~0u, last, 0);
    if (!last) return;
    unsigned long long all = none;
    for (int k = lane; k < a.splits; k += 32) {
      const unsigned long long x = __ldcg(a.shares + static_cast<size_t>(row) * a.splits + k);
      all = greedy ? (x > all ? x : all) : pack(plus(c, unpack(all), unpack(x)));
    }
    mine = join(all);
  }
  if (lane != 0) return;
  // the row's verdict
  VerifyRow f{0.f, 0.f, c.kind, -1};
  const int draft = row + 1 < r.end ? a.tokens[row + 1] : -1;
  const bool drafted = static_cast<unsigned>(draft) < static_cast<unsigned>(a.vocab);
  float p = 0.f;
  if (greedy) {
    f.top = index_of(mine);
    if (mine == kBadKey || mine >> 32 == key_of(-INFINITY, 0) >> 32) f.verdict = kNothing;
    else if (drafted && draft == f.top) f.verdict |= kStands, p = 1.f;
  } else if (c.kind == 0) {
    const Share s = unpack(mine);
    f.max = s.max, f.sum = s.sum;
    if (!(s.sum > 0.f && s.sum < INFINITY)) {
      f.verdict = kNothing;
    } else if (drafted) {
      const double d = static_cast<double>(Logits<T>::one(z + draft)) - s.max;
      const double px = exp2(d * c.hi + d * c.lo) / s.sum;
      const float q = a.draft_probs != nullptr ? a.draft_probs[row * a.probs_row + draft] : 1.f;
      if (static_cast<double>(a.uniforms[row]) * q < px) f.verdict |= kStands;
      p = static_cast<float>(px);
    }
  }
  a.found[row] = f;
  if (a.target_probs != nullptr) a.target_probs[row] = p;
}

// The race over values [from, to) of a row: the largest w / e and its index.
template <class T>
__device__ __forceinline__ unsigned long long race(const Heat& c, const VerifyRow& f, const T* z, const float* e, const float* q,
                                                   int skip, int from, int to) {
  const float inv = 1.f / f.sum;
  float best = 0.f;
  int at = 0;
  auto take = [&](float x, float ev, float qv, int v) {
    const float w = fmaf(ex2_ftz(exponent(c, x, f.max)), inv, -qv), ratio = __fdividef(w, ev);
    if (ratio > best && v != skip) best = ratio, at = v;
  };
  constexpr int U = 8;
  for (int v = from + static_cast<int>(threadIdx.x); v < to; v += U * kVThreads) {
    float x[U], ev[U], qv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = v + u * kVThreads;
      x[u] = -INFINITY, ev[u] = 1.f, qv[u] = 0.f;
      if (i < to) {
        x[u] = Logits<T>::one(z + i), ev[u] = e[i];
        if (q != nullptr) qv[u] = q[i];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) take(x[u], ev[u], qv[u], v + u * kVThreads);
  }
  return warp_largest(best > 0.f ? key_of(best, at) : 0ull);
}

template <class T>
__global__ void __launch_bounds__(kVThreads) verify_draw_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ unsigned long long sm[kVWarps];
  __shared__ int sm_last, sm_none;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.y, part = blockIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  const Rows r = rows_of(a, b);
  if (!r.live) {
    if (part == 0 && tid == 0) a.accepted[b] = 0, a.next[b] = -1;
    return;
  }
  // the first row whose draft does not stand (the last row has none)
  int row = r.first;
  VerifyRow f;
  for (;; row += 32) {
    const bool in = row + lane < r.end;
    VerifyRow mine{0.f, 0.f, kNothing, -1};
    if (in) mine = a.found[row + lane];
    const unsigned falls = __ballot_sync(~0u, !(mine.verdict & kStands));
    if (falls == 0) continue;
    const int k = __ffs(falls) - 1;
    row += k;
    f = {__shfl_sync(~0u, mine.max, k), __shfl_sync(~0u, mine.sum, k), __shfl_sync(~0u, mine.verdict, k),
         __shfl_sync(~0u, mine.top, k)};
    break;
  }
  if (f.verdict & (kNothing | kGreedy)) {
    if (part == 0 && tid == 0) a.accepted[b] = row - r.first + 1, a.next[b] = f.verdict & kNothing ? -1 : f.top;
    return;
  }
  const Heat c = heat_of(a, b);
  const int draft = row + 1 < r.end ? a.tokens[row + 1] : -1;
  const bool drafted = static_cast<unsigned>(draft) < static_cast<unsigned>(a.vocab);
  const T* z = static_cast<const T*>(a.logits) + row * a.logits_row;
  const float* e = a.race + b * a.race_row;
  const float* q = drafted && a.draft_probs != nullptr ? a.draft_probs + row * a.probs_row : nullptr;
  const int skip = drafted && a.draft_probs == nullptr ? draft : -1;
  const int v0 = part * a.part_len, v1 = min(v0 + a.part_len, a.vocab);
  auto whole = [&](unsigned long long k) {  // of all warps, in warp 0
    __syncthreads();
    if (lane == 0) sm[warp] = k;
    __syncthreads();
    return warp == 0 ? warp_largest(lane < kVWarps ? sm[lane] : 0ull) : 0ull;
  };
  unsigned long long best = whole(race<T>(c, f, z, e, q, skip, v0, v1));
  if (a.parts > 1) {
    if (tid == 0) {
      if (best != 0) atomicMax(a.best + b, best);
      __threadfence();
      sm_last = atomicAdd(a.request_tickets + b, 1) == a.parts - 1;
      __threadfence();
      if (sm_last) {
        best = atomicExch(a.best + b, 0ull);
        a.request_tickets[b] = 0;
      }
    }
    __syncthreads();
    if (!sm_last) return;
  }
  if (tid == 0) sm_none = best == 0;
  __syncthreads();
  if (sm_none) best = whole(race<T>(c, f, z, e, nullptr, -1, 0, a.vocab));  // nothing is left beside q: from p itself
  if (tid == 0) a.accepted[b] = row - r.first + 1, a.next[b] = best != 0 ? index_of(best) : -1;
}

template <class T>
cudaError_t launch(const VerifyArgs& a, cudaStream_t s) {
  if (a.rows > 0) {
    const cudaError_t e = launch_after(verify_rows_kernel<T>, dim3(a.rows * a.splits), kVThreads, 0, s, a);
    if (e != cudaSuccess) return e;
  }
  return launch_after(verify_draw_kernel<T>, dim3(a.parts, a.batch), kVThreads, 0, s, a);
}

}  // namespace

cudaError_t launch_verify(VerifyArgs a, int dtype, int sms, cudaStream_t s) {
  // shares of a row (parts of a vocabulary): as many as give each SM 8 CTAs (4), of 2048 values at least
  auto cut = [&](int rows, int per_sm, int& pieces, int& len) {
    const int want = (per_sm * sms + rows - 1) / rows, most = (a.vocab + 2047) / 2048;
    pieces = want < most ? want : most;
    len = ((a.vocab + pieces - 1) / pieces + 7) & ~7;
    pieces = (a.vocab + len - 1) / len;
  };
  cut(max(a.rows, 1), 8, a.splits, a.split_len);
  cut(a.batch, 4, a.parts, a.part_len);
  if (dtype == CLLM_F32) return launch<float>(a, s);
  if (dtype == CLLM_BF16) return launch<__nv_bfloat16>(a, s);
  return launch<__half>(a, s);
}

}  // namespace cllm
