// Verification of drafted tokens (cllm_verify): two launches.
//
//   p(x) = 2^(c (z_x - m)) / S,  S = sum_v 2^(c (z_v - m)),  c = log2(e) / temperature,  m = max z
//   a draft stands:  u q(x) < p(x);   next = argmax_v max(p - q, 0)_v / e_v
//
// The first kernel reads all logits once, a row in as many shares as there are warps on the GPU, or in one CTA's: a
// lane keeps its running maximum and sum; the warp that brings a row's last share (a CTA's first warp) adds them up in
// order and judges its draft.  The second finds each request's first row whose draft falls, and
// runs the race over that row, its vocabulary in parts; results meet in one atomicMax on (ratio, lowest
// index), whose order does not matter.
//
// c is held in two floats, the first rounded down, so that both products of an infinite
// difference have its sign.  Sums and probabilities are in fp32.
//
// Bound: HBM, the logits, then the race and the deciding rows (which are in L2 where all logits
// are).  Measured: 768 rows of 131072 in bf16 (201 MB) 37 us, 5.4 TB/s, as long as a bare reduction of these bytes
// takes (39); 1536 rows 65 us, 6.2 TB/s.  The race of 102 requests over them (81 MB) 16 us.
// 16 rows of 32000 in fp32: 8.6 us for both, two launches and their trips to L2.
// Next vectors are loaded while these are summed: 36.9 us against 42 without.  More warps with fewer registers
// 42, CTAs of 8 warps that reduce a share together 40 to 44, shares a half or a quarter as long 41
// and 45; requests to L2 ahead of the race's loads change nothing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.cuh"
#include "paged.cuh"
#include "ptx.cuh"
#include "verify.cuh"

namespace cllm {

namespace {

// CTAs of two warps: the warps have nothing to do with one another, and a CTA's place is free when both have ended.
constexpr int kVThreads = 64, kVWarps = kVThreads / 32;
constexpr int kDrawWarps = 24;  // of the second kernel on an SM
constexpr float kLog2eHi = 1.44269502162933349609f, kLog2eLo = 1.9259629911e-8f;

// 16 bytes of logits.  kNone: four bytes of -inf.
template <class T> struct Logits;
template <> struct Logits<float> {
  static constexpr int n = 4;
  static constexpr uint32_t kNone = 0xff800000u;
  static __device__ float2 pair(const uint4& x, int i) {
    return i == 0 ? make_float2(__uint_as_float(x.x), __uint_as_float(x.y)) : make_float2(__uint_as_float(x.z), __uint_as_float(x.w));
  }
  static __device__ float one(const float* p) { return *p; }
  static __device__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
  }
  // the largest of some vectors; NaN if one is (else without notice)
  template <bool NAN_TOO, int U>
  static __device__ float top(const uint4 (&x)[U]) {
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 v = pair(x[u], i);
        m = NAN_TOO ? max_nan(m, max_nan(v.x, v.y)) : fmaxf(m, fmaxf(v.x, v.y));
      }
    return m;
  }
};
template <class T, class T2>
struct Logits16 {
  static constexpr int n = 8;
  template <bool NAN_TOO, int U>
  static __device__ float top(const uint4 (&x)[U]) {
    auto two = [](uint32_t w) { return *reinterpret_cast<const T2*>(&w); };
    auto larger = [](T2 a, T2 b) { return NAN_TOO ? __hmax2_nan(a, b) : __hmax2(a, b); };
    T2 m = two(x[0].x);
#pragma unroll
    for (int u = 0; u < U; ++u) m = larger(m, larger(larger(two(x[u].x), two(x[u].y)), larger(two(x[u].z), two(x[u].w))));
    const float lo = Logits<T>::wide(m.x), hi = Logits<T>::wide(m.y);
    return NAN_TOO ? Logits<float>::max_nan(lo, hi) : fmaxf(lo, hi);
  }
  static __device__ uint32_t word(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }
};
template <> struct Logits<__half> : Logits16<__half, __half2> {
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static __device__ float wide(__half x) { return __half2float(x); }
  static __device__ float2 pair(const uint4& x, int i) {
    const uint32_t w = word(x, i);
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
  static __device__ float one(const __half* p) { return __half2float(*p); }
};
template <> struct Logits<__nv_bfloat16> : Logits16<__nv_bfloat16, __nv_bfloat162> {
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ float2 pair(const uint4& x, int i) {
    const uint32_t w = word(x, i);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};

__device__ __forceinline__ float rcp_ftz(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// c = log2(e) / t in two floats, hi < c.
struct Heat {
  float hi, lo;
  int kind;  // 0, kNothing or kGreedy
};
__device__ __forceinline__ Heat heat_of(const VerifyArgs& a, float t) {
  if (a.race == nullptr) return {0.f, 0.f, kGreedy};
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
__device__ __forceinline__ float2 exponents(const Heat& c, float2 z, float m) {
  const float2 d = add2(z, make_float2(-m, -m));
  return fma2(d, make_float2(c.hi, c.hi), mul2(d, make_float2(c.lo, c.lo)));
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

// A request's rows and temperature: loads of one trip.
struct Request {
  int first, end, len;
  float heat;
  __device__ bool live(const VerifyArgs& a) const {
    return first >= 0 && end > first && end <= a.rows && end - first <= len;
  }
};
__device__ __forceinline__ Request request(const VerifyArgs& a, int b) {
  return {a.row_start[b], a.row_start[b + 1], a.seq_len[b], a.temperature != nullptr ? a.temperature[b] : 1.f};
}
// The one that row `row` belongs to, by a warp: the last that begins at or before it (end -1: none).
__device__ __forceinline__ Request request_of(const VerifyArgs& a, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = a.batch;  // among requests [lo, lo + n)
  while (n > 32) {
    const int step = (n + 31) / 32;
    const unsigned before = __ballot_sync(~0u, lane * step < n && a.row_start[lo + lane * step] <= row);
    const int k = before != 0 ? 31 - __clz(before) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  const Request r = lane < n ? request(a, lo + lane) : Request{0, -1, 0, 0.f};
  const unsigned before = __ballot_sync(~0u, lane < n && r.first <= row);
  if (before == 0) return {0, -1, 0, 0.f};
  const int k = 31 - __clz(before);
  return {__shfl_sync(~0u, r.first, k), __shfl_sync(~0u, r.end, k), __shfl_sync(~0u, r.len, k), __shfl_sync(~0u, r.heat, k)};
}

// Values [from, to) of a row for a warp: vectors of 16 bytes from the first boundary on, U of a lane
// at a time, and up to n - 1 single ones before and after.
template <class T, int U>
struct Span {
  static constexpr int n = Logits<T>::n;
  const uint4* p;
  const T* z;
  int from, to, head, vecs;
  __device__ Span(const T* row, int from, int to) : z(row), from(from), to(to) {
    const int past = static_cast<int>(reinterpret_cast<uintptr_t>(row + from) & 15) / static_cast<int>(sizeof(T));
    head = min((n - past) % n, to - from);
    vecs = (to - from - head) / n;
    p = reinterpret_cast<const uint4*>(row + from + head);
  }
  __device__ void load(uint4 (&x)[U], int i) const {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      constexpr uint32_t none = Logits<T>::kNone;
      x[u] = make_uint4(none, none, none, none);
      if (i + u * 32 < vecs) x[u] = p[i + u * 32];
    }
  }
  __device__ int index(int i, int u) const { return from + head + (i + u * 32) * n; }  // of a vector's first value
  template <class One>
  __device__ void single(One one) const {
    const int tail = from + head + vecs * n, i = threadIdx.x & 31;
    if (i < head) one(Logits<T>::one(z + from + i), from + i);
    if (i < to - tail) one(Logits<T>::one(z + tail + i), tail + i);
  }
};

// A warp takes a share of a row.  W warps of a CTA: all of a row's shares, which meet in shared memory; W = 1:
// any shares, which meet in memory, counted by the row's ticket.
template <class T, int W>
__global__ void __launch_bounds__(W == 1 ? kVThreads : 32 * W, W == 1 ? kVerifyWarps / kVWarps : kVerifyWarps / W)
    verify_rows_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ unsigned long long sm[W];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, unit = blockIdx.x * kVWarps + warp;
  const int row = W > 1 ? blockIdx.x : unit / a.splits, split = W > 1 ? warp : unit - row * a.splits;
  pdl_launch_dependents();
  pdl_wait();
  if (row >= a.rows) return;
  const T* z = static_cast<const T*>(a.logits) + row * a.logits_row;
  const int v0 = min(split * a.split_len, a.vocab), v1 = min(v0 + a.split_len, a.vocab);
  constexpr int U = 4;
  const Span<T, U> span(z, v0, v1);
  // (vectors, the draft, its logit and its numbers are on their way while the row's request is looked for)
  uint4 x[U];
  int i = lane;
  const int draft = row + 1 < a.rows ? a.tokens[row + 1] : -1;
  const float u = a.race != nullptr ? a.uniforms[row] : 0.f;
  span.load(x, i);
  const bool known = static_cast<unsigned>(draft) < static_cast<unsigned>(a.vocab);
  const float zx = known ? Logits<T>::one(z + draft) : 0.f;
  const float qx = known && a.draft_probs != nullptr ? a.draft_probs[row * a.probs_row + draft] : 1.f;
  const Request r = request_of(a, row);
  if (row >= r.end) return;  // behind the last request
  if (!r.live(a)) {
    if (split == 0 && lane == 0 && a.target_probs != nullptr) a.target_probs[row] = 0.f;
    return;
  }
  const Heat c = heat_of(a, r.heat);
  const bool greedy = c.kind == kGreedy, drafted = known && row + 1 < r.end;
  unsigned long long mine;
  if (greedy) {
    float top = -INFINITY;
    int at = a.vocab;
    bool bad = false;
    for (; i - lane < span.vecs; i += U * 32, span.load(x, i)) {
      const float m = Logits<T>::template top<true>(x);
      bad |= m != m;
      if (m > top) {
        top = m;
        at = a.vocab;
#pragma unroll
        for (int u = U - 1; u >= 0; --u)
#pragma unroll
          for (int j = Logits<T>::n / 2 - 1; j >= 0; --j) {
            const float2 v = Logits<T>::pair(x[u], j);
            if (v.y == m) at = span.index(i, u) + 2 * j + 1;
            if (v.x == m) at = span.index(i, u) + 2 * j;
          }
      }
    }
    span.single([&](float v, int k) {
      bad |= v != v;
      if (v > top || (v == top && k < at)) top = v, at = k;
    });
    mine = warp_largest(bad ? kBadKey : key_of(top, at));
  } else {
    Share s{-INFINITY, 0.f};
    auto raise = [&](float top) {
      if (!(top > s.max)) return;
      s.sum *= ex2_ftz(exponent(c, s.max, top));
      s.max = top;
    };
    auto base = [&] { return s.max == -INFINITY ? 0.f : s.max; };
    if (c.kind == 0) {
      auto add = [&](const uint4 (&x)[U]) {
        raise(Logits<T>::template top<false>(x));
        const float m = base();
        float2 t[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < Logits<T>::n / 2; ++j) {
            const float2 e = exponents(c, Logits<T>::pair(x[u], j), m);
            t[j & 1] = add2(t[j & 1], make_float2(ex2_ftz(e.x), ex2_ftz(e.y)));
          }
        s.sum += (t[0].x + t[0].y) + (t[1].x + t[1].y);
      };
      // (the next vectors are on their way meanwhile)
      uint4 y[U];
      for (; i - lane < span.vecs; i += 2 * U * 32) {
        span.load(y, i + U * 32);
        add(x);
        span.load(x, i + 2 * U * 32);
        add(y);
      }
      span.single([&](float v, int) {
        raise(v);
        s.sum += ex2_ftz(exponent(c, v, base()));
      });
    }
    mine = pack(warp_plus(c, s));
  }
  auto join = [&](unsigned long long x) { return greedy ? warp_largest(x) : pack(warp_plus(c, unpack(x))); };
  const unsigned long long none = greedy ? 0ull : pack(Share{-INFINITY, 0.f});
  if constexpr (W > 1) {
    if (lane == 0) sm[warp] = mine;
    __syncthreads();
    if (warp != 0) return;
    mine = join(lane < W ? sm[lane] : none);
  } else if (a.splits > 1) {
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
    __syncwarp();  // (orders the lanes' reads behind the first lane's fence, which a shuffle does not)
    unsigned long long all = none;
    for (int k = lane; k < a.splits; k += 32) {
      const unsigned long long x = __ldcg(a.shares + static_cast<size_t>(row) * a.splits + k);
      all = greedy ? (x > all ? x : all) : pack(plus(c, unpack(all), unpack(x)));
    }
    mine = join(all);
  }
  if (lane != 0) return;
  // the row's verdict
  VerifyRow f{0.f, 0.f, c.kind, drafted ? draft : -1};
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
      // (difference and exponent in two floats, so that their rounding does not count)
      const float d = zx - s.max, back = d - zx, rest = (zx - (d - back)) - (s.max + back), hi = d * c.hi;
      const float lo = hi > -INFINITY ? fmaf(d, c.hi, -hi) + fmaf(rest, c.hi, d * c.lo) : 0.f;
      p = exp2f(hi) * fmaf(lo, 0.693147180559945f, 1.f) / s.sum;
      if (u * qx < p) f.verdict |= kStands;
    }
  }
  a.found[row] = f;
  if (a.target_probs != nullptr) a.target_probs[row] = p;
}

// A lane's race values from v on, as far as they are there (aligned).
template <class T>
__device__ __forceinline__ void race_values(float4 (&e0)[Logits<T>::n / 4], const float* e, int v, int to) {
#pragma unroll
  for (int k = 0; k < Logits<T>::n / 4; ++k)
    if (v + 4 * k + 4 <= to) e0[k] = *reinterpret_cast<const float4*>(e + v + 4 * k);
}

// The race over values [from, to) of a row, by a warp: the largest w / e and its index.  Where rows
// begin on boundaries of 16 bytes, in vectors, of which a lane keeps the largest ratio and the
// vector's place; which of the vector's values it was is found at the end.  (A branch for every
// value that is larger than those before took half the time: a warp has a hundred of them.)
// Other rows go one value at a time: 128 requests of 4 to 8 rows in bf16 28.6 us at 50257 tokens, 25.7 at 50256 (in
// fp32 37.7 both).
template <class T, bool PROBS>
struct Race {
  static constexpr int n = Logits<T>::n;
  const Heat& c;
  const VerifyRow& f;
  const T* z;
  const float *e, *q;
  int skip;
  float inv;
  __device__ Race(const Heat& c, const VerifyRow& f, const T* z, const float* e, const float* q, int skip)
      : c(c), f(f), z(z), e(e), q(q), skip(skip), inv(PROBS ? 1.f / f.sum : 1.f) {}  // (a common factor does not matter)
  struct Piece {
    uint4 x;
    float4 e[n / 4], q[PROBS ? n / 4 : 1];
  };
  __device__ float ratio(float power, float ev, float qv) const {
    return (PROBS ? fmaf(power, inv, -qv) : power) * rcp_ftz(ev);
  }
  __device__ void load(Piece& p, int v, int end, const float4* e0 = nullptr) const {
    if (v >= end) return;
    p.x = *reinterpret_cast<const uint4*>(z + v);
#pragma unroll
    for (int k = 0; k < n / 4; ++k) {
      p.e[k] = e0 != nullptr ? e0[k] : *reinterpret_cast<const float4*>(e + v + 4 * k);
      if (PROBS) p.q[k] = *reinterpret_cast<const float4*>(q + v + 4 * k);
    }
  }
  __device__ void ratios(const Piece& p, int v, float (&r)[n]) const {
#pragma unroll
    for (int k = 0; k < n / 4; ++k) {
      const float2 a = exponents(c, Logits<T>::pair(p.x, 2 * k), f.max), b = exponents(c, Logits<T>::pair(p.x, 2 * k + 1), f.max);
      const float4 qv = PROBS ? p.q[k] : make_float4(0.f, 0.f, 0.f, 0.f);
      r[4 * k] = ratio(ex2_ftz(a.x), p.e[k].x, qv.x);
      r[4 * k + 1] = ratio(ex2_ftz(a.y), p.e[k].y, qv.y);
      r[4 * k + 2] = ratio(ex2_ftz(b.x), p.e[k].z, qv.z);
      r[4 * k + 3] = ratio(ex2_ftz(b.y), p.e[k].w, qv.w);
    }
    if (static_cast<unsigned>(skip - v) < static_cast<unsigned>(n)) {
#pragma unroll
      for (int j = 0; j < n; ++j)
        if (j == skip - v) r[j] = 0.f;
    }
  }
  __device__ unsigned long long run(int from, int to, const float4* e0) const {  // e0: the lane's first race values, if aligned
    const int lane = threadIdx.x & 31;
    float best = 0.f;
    int at = 0, v = from;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(z + from) | reinterpret_cast<uintptr_t>(e + from) |
                           (PROBS ? reinterpret_cast<uintptr_t>(q + from) : 0);
    if ((bits & 15) == 0) {
      const int whole = from + (to - from) / n * n;
      auto take = [&](const Piece& p, int v) {
        if (v >= whole) return;
        float r[n];
        ratios(p, v, r);
        float m = fmaxf(r[0], r[1]);
#pragma unroll
        for (int j = 2; j < n; j += 2) m = fmaxf(m, fmaxf(r[j], r[j + 1]));
        if (m > best) best = m, at = v;
      };
      // (the next piece is on its way meanwhile)
      Piece p0, p1;
      v = from + lane * n;
      load(p0, v, whole, e0);
      for (; v < whole; v += 64 * n) {
        load(p1, v + 32 * n, whole);
        take(p0, v);
        load(p0, v + 64 * n, whole);
        take(p1, v + 32 * n);
      }
      if (best > 0.f) {
        float r[n];
        load(p0, at, whole);
        ratios(p0, at, r);
        int j = 0;
#pragma unroll
        for (int k = n - 1; k >= 0; --k)
          if (r[k] == best) j = k;
        at += j;
      }
      v = whole;
    }
    constexpr int S = 8;
    for (v += lane; v < to; v += S * 32) {
      float x[S], ev[S], qv[S];
#pragma unroll
      for (int u = 0; u < S; ++u) {
        const int i = v + u * 32;
        x[u] = -INFINITY, ev[u] = 1.f, qv[u] = 0.f;
        if (i < to) {
          x[u] = Logits<T>::one(z + i), ev[u] = e[i];
          if (PROBS) qv[u] = q[i];
        }
      }
#pragma unroll
      for (int u = 0; u < S; ++u) {
        const float r = ratio(ex2_ftz(exponent(c, x[u], f.max)), ev[u], qv[u]);
        if (r > best && v + u * 32 != skip) best = r, at = v + u * 32;
      }
    }
    return warp_largest(best > 0.f ? key_of(best, at) : 0ull);
  }
};

// A warp takes a part of a request's deciding row; W as in the first kernel.
template <class T, int W>
__global__ void __launch_bounds__(W == 1 ? kVThreads : 32 * W, W == 1 ? kDrawWarps / kVWarps : W == 4 ? 6 : 1)
    verify_draw_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ unsigned long long sm[W];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, unit = blockIdx.x * kVWarps + warp;
  const int b = W > 1 ? blockIdx.x : unit / a.parts, part = W > 1 ? warp : unit - b * a.parts;
  const bool first = part == 0 && lane == 0;
  pdl_launch_dependents();
  pdl_wait();
  if (b >= a.batch) return;
  const Request r = request(a, b);
  const int v0 = min(part * a.part_len, a.vocab), v1 = min(v0 + a.part_len, a.vocab);
  const float* e = a.race + b * a.race_row;
  // (the race's first values are on their way while the deciding row is looked for)
  float4 e0[Logits<T>::n / 4];
  const bool ahead = a.race != nullptr && (reinterpret_cast<uintptr_t>(e + v0) & 15) == 0;
  if (ahead) race_values<T>(e0, e, v0 + lane * Logits<T>::n, v1);
  const Heat c = heat_of(a, r.heat);
  if (!r.live(a)) {
    if (first) a.accepted[b] = 0, a.next[b] = -1;
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
    if (first) a.accepted[b] = row - r.first + 1, a.next[b] = f.verdict & kNothing ? -1 : f.top;
    return;
  }
  const T* z = static_cast<const T*>(a.logits) + row * a.logits_row;
  // (f.top: the draft that fell, -1: none)
  unsigned long long best =
      f.top >= 0 && a.draft_probs != nullptr
          ? Race<T, true>(c, f, z, e, a.draft_probs + row * a.probs_row, -1).run(v0, v1, e0)
          : Race<T, false>(c, f, z, e, nullptr, f.top).run(v0, v1, e0);
  if constexpr (W > 1) {
    if (lane == 0) sm[warp] = best;
    __syncthreads();
    if (warp != 0) return;
    best = warp_largest(lane < W ? sm[lane] : 0ull);
  } else if (a.parts > 1) {
    int last = 0;
    if (lane == 0) {
      if (best != 0) atomicMax(a.best + b, best);
      __threadfence();
      last = atomicAdd(a.request_tickets + b, 1) == a.parts - 1;
      if (last) {
        __threadfence();
        best = atomicExch(a.best + b, 0ull);
        a.request_tickets[b] = 0;
      }
    }
    if (!__shfl_sync(~0u, last, 0)) return;
    best = __shfl_sync(~0u, best, 0);
  }
  if (best == 0) best = Race<T, false>(c, f, z, e, nullptr, -1).run(0, a.vocab, nullptr);  // nothing is left beside q: from p itself
  if (lane == 0) a.accepted[b] = row - r.first + 1, a.next[b] = best != 0 ? index_of(best) : -1;
}

template <class T, int W>
cudaError_t launch_rows(const VerifyArgs& a, cudaStream_t s) {
  if (W > 1) return launch_after(verify_rows_kernel<T, W>, dim3(a.rows), 32 * W, 0, s, a);
  const long long units = static_cast<long long>(a.rows) * a.splits;
  return launch_after(verify_rows_kernel<T, W>, dim3((units + kVWarps - 1) / kVWarps), kVThreads, 0, s, a);
}
template <class T, int W>
cudaError_t launch_draw(const VerifyArgs& a, cudaStream_t s) {
  if (W > 1) return launch_after(verify_draw_kernel<T, W>, dim3(a.batch), 32 * W, 0, s, a);
  const long long units = static_cast<long long>(a.batch) * a.parts;
  return launch_after(verify_draw_kernel<T, W>, dim3((units + kVWarps - 1) / kVWarps), kVThreads, 0, s, a);
}

template <class T>
cudaError_t launch(VerifyArgs a, int sms, cudaStream_t s) {
  auto cut = [&](int pieces, int& n, int& len, bool all) {  // the vocabulary in pieces (`all`: of which some may be empty)
    len = ((a.vocab + pieces - 1) / pieces + 7) & ~7;
    n = all ? pieces : (a.vocab + len - 1) / len;
  };
  // as many pieces as warps that the GPU holds, of `least` values at least
  auto spread = [&](int rows, int warps, int least) { return min(max(warps / rows, 1), (a.vocab + least - 1) / least); };
  // CTAs of W warps where the vocabulary is short and all of them are on the GPU at once: their shares meet in
  // shared memory, where others' meet through a fence and two atomics.  (With CTAs of 4, of 16 warps, and without, bf16: 4 x 4
  // rows of 1000 4.6, -, 6.1 us; 30 x 5 of 5000 6.5, 7.6, 9.1; 8 x 8 of 12000 -, 6.8, 9.1; 60 x 5 of 32000 -, 10.2, 13.6;
  // 10 x 8 of 64000 -, 12.7, 12.9; 4 x 6 of 131072 in fp32 -, 21.5, 11.0.  Rows of fp32 are twice the bytes to the same SM,
  // and still as fast or faster up to here: 16 rows of 32768 8.8 and 8.9 us, 8 x 8 of 32000 9.3 and 10.2, 60 x 5 12.6 and 13.6.)
  auto group = [&](int rows, int warps) {
    return a.vocab <= 8192 && 4ll * rows <= warps ? 4 : a.vocab <= 32768 && 16ll * rows <= warps ? 16 : 1;
  };
  if (a.rows > 0) {
    const int w = group(a.rows, kVerifyWarps * sms);
    cut(w > 1 ? w : spread(a.rows, kVerifyWarps * sms, 1024), a.splits, a.split_len, w > 1);
    const cudaError_t e = w == 4 ? launch_rows<T, 4>(a, s) : w == 16 ? launch_rows<T, 16>(a, s) : launch_rows<T, 1>(a, s);
    if (e != cudaSuccess) return e;
  }
  const int w = group(a.batch, 16 * sms);
  cut(w > 1 ? w : spread(a.batch, kDrawWarps * sms, 512), a.parts, a.part_len, w > 1);
  return w == 4 ? launch_draw<T, 4>(a, s) : w == 16 ? launch_draw<T, 16>(a, s) : launch_draw<T, 1>(a, s);
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, int dtype, int sms, cudaStream_t s) {
  if (dtype == CLLM_F32) return launch<float>(a, sms, s);
  if (dtype == CLLM_BF16) return launch<__nv_bfloat16>(a, sms, s);
  return launch<__half>(a, sms, s);
}

}  // namespace cllm
