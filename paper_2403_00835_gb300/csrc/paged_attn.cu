// Attention of new tokens over a paged cache (cllm_paged_attention) on the FMA units.
//
//   o = sum_k p_k v_k / sum_k p_k,  p_k = 2^(scale log2(e) q.k - m),  m the running maximum
//
// in one pass over the keys: fp32 throughout.  A CTA holds a tile of BM rows (tokens
// times the query heads of one key/value head) and takes its keys 64 at a time, the
// next 64 on their way (cp.async) meanwhile.  A thread computes BM/16 rows x 4 scores,
// and of the output BM/16 rows x HD/16 columns; with BM = 64 a shared-memory load of 16
// bytes serves 8 to 11 multiply-adds, which bounds it near half the FMA rate, with BM =
// 16 (few rows) a quarter of that.
//
// Measured: a chunk of 1024 tokens, 32 heads of 128: 312 us, 27.5 TFLOP/s; 16 requests of one
// token, 32 heads on 8, at 2000 keys: 90 us, 2.9 TB/s; a block of 8 tokens, 4 heads of 64, at
// 32 to 96 keys: 6.8 us, a launch's start and round trips to tables and pages.
#include "paged.cuh"
#include "paged_walk.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kPThreads = 256;
constexpr int kPChunk = 64;  // 2^6

template <int HD, int BM>
struct PagedSmem {
  float q[BM][HD + 4];
  float k[2][kPChunk][HD + 4];
  float v[2][kPChunk][HD + 4];
  float p[BM][kPChunk + 4];
  unsigned scan[32];
  RunStart run;
  unsigned bad[2];  // rows whose result is not finite
  int last;
};

__device__ __forceinline__ float4 ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void st4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ bool finite4(float4 v) {
  return isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w);
}

template <int HD, int BM>
__global__ void __launch_bounds__(kPThreads, 1)
    paged_attn_kernel(const __grid_constant__ PagedAttnArgs a, const PagedGeom g) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  using T = float;
  PagedSmem<HD, BM>& s = *reinterpret_cast<PagedSmem<HD, BM>*>(smem_raw);
  constexpr int R = BM / 16, C = HD / 64;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  pdl_launch_dependents();
  pdl_wait();
  if (a.batch > kWarpRequests) run_start_block(a, g, &s.run, s.scan);
  else if (tid < 32) run_start_warp(a, g, &s.run);
  __syncthreads();
  PagedWalk w;
  w.begin(s.run);
  Piece p;
  while (w.next(a, g, p)) {
    const int rows = p.nt * a.group;
    __syncthreads();
    if (tid < 2) s.bad[tid] = 0;
    for (int i = tid; i < BM * (HD / 4); i += kPThreads) {
      const int r = i / (HD / 4), d = i % (HD / 4) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < rows) {
        const int tok = (r * a.group_inv >> 16), hh = p.h * a.group + r % a.group;
        x = ld4(static_cast<const T*>(a.q) + static_cast<long long>(p.row0 + p.t0 + tok) * a.q_row + hh * a.q_head + d);
      }
      *reinterpret_cast<float4*>(&s.q[r][d]) = x;
    }
    RowKeys rk[R];
    float m[R], l[R];
    float4 o[R][C];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = ty * R + i;
      rk[i] = row_keys(a, p.n, p.len, p.row0, p.t0 + (min(r, rows - 1) * a.group_inv >> 16));
      m[i] = -INFINITY, l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // 8 lanes to a key; keys that no row of the tile sees become zeros
    auto load = [&](int c) {
      const int st = (c - p.ca) & 1;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int key = (tid >> 3) + 32 * u, pos = c * kPChunk + key;
        const T *kp = nullptr, *vp = nullptr;
        if (pos >= p.lo && pos < p.hi) kp = pool_row<T>(a, a.k, p.b, p.h, pos), vp = pool_row<T>(a, a.v, p.b, p.h, pos);
#pragma unroll
        for (int d = (tid & 7) * 4; d < HD; d += 32) {
          if (kp != nullptr) {
            cp_async16(&s.k[st][key][d], kp + d);
            cp_async16(&s.v[st][key][d], vp + d);
          } else {
            *reinterpret_cast<float4*>(&s.k[st][key][d]) = make_float4(0.f, 0.f, 0.f, 0.f);
            *reinterpret_cast<float4*>(&s.v[st][key][d]) = make_float4(0.f, 0.f, 0.f, 0.f);
          }
        }
      }
      cp_async_commit();
    };
    const bool live = (tid >> 5) * 2 * R < rows;  // some row of the warp is
    if (p.ca < p.cb) load(p.ca);
    for (int c = p.ca; c < p.cb; ++c) {
      const int kb = c * kPChunk, st = (c - p.ca) & 1;
      if (c + 1 < p.cb) {
        load(c + 1);
        cp_async_wait_but1();
      } else {
        cp_async_wait_all();
      }
      __syncthreads();
      if (live) {
        float x[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 4
        for (int d = 0; d < HD; d += 4) {
          float4 kv[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) kv[j] = ld4(&s.k[st][tx + 16 * j][d]);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float4 q = ld4(&s.q[ty * R + i][d]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              x[i][j] = fmaf(q.w, kv[j].w, fmaf(q.z, kv[j].z, fmaf(q.y, kv[j].y, fmaf(q.x, kv[j].x, x[i][j]))));
          }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const uint32_t b0 = key_bits(rk[i], kb), b1 = key_bits(rk[i], kb + 32);
          const bool see[4] = {(b0 >> tx & 1) != 0, (b0 >> (tx + 16) & 1) != 0, (b1 >> tx & 1) != 0,
                               (b1 >> (tx + 16) & 1) != 0};
          float cm = -INFINITY;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[i][j] = see[j] ? x[i][j] * a.scale_log2 : -INFINITY;
            cm = fmaxf(cm, x[i][j]);
          }
#pragma unroll
          for (int d = 1; d < 16; d <<= 1) cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, d));
          const float nm = fmaxf(m[i], cm), base = nm == -INFINITY ? 0.f : nm;
          const float f = exp2f(m[i] - base);
          m[i] = nm;
          l[i] *= f;
#pragma unroll
          for (int e = 0; e < C; ++e) o[i][e].x *= f, o[i][e].y *= f, o[i][e].z *= f, o[i][e].w *= f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float pr = exp2f(x[i][j] - base);
            l[i] += pr;
            s.p[ty * R + i][tx + 16 * j] = pr;
          }
        }
        __syncwarp();  // (a warp's probabilities are its own rows')
#pragma unroll 2
        for (int key = 0; key < kPChunk; key += 4) {
          float pr[R][4];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float4 t = ld4(&s.p[ty * R + i][key]);
            pr[i][0] = t.x, pr[i][1] = t.y, pr[i][2] = t.z, pr[i][3] = t.w;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < C; ++e) {
              const float4 v = ld4(&s.v[st][key + u][tx * 4 + 64 * e]);
#pragma unroll
              for (int i = 0; i < R; ++i) {
                o[i][e].x = fmaf(pr[i][u], v.x, o[i][e].x);
                o[i][e].y = fmaf(pr[i][u], v.y, o[i][e].y);
                o[i][e].z = fmaf(pr[i][u], v.z, o[i][e].z);
                o[i][e].w = fmaf(pr[i][u], v.w, o[i][e].w);
              }
            }
        }
      }
      __syncthreads();  // (the buffer is loaded anew by the next turn)
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
#pragma unroll
    for (int i = 0; i < R; ++i) m[i] = share_max(m[i], l[i]);

    auto store = [&](int r, int d, float4 x, float mm, float ll) {  // a row's 4 columns from d
      const int tok = (r * a.group_inv >> 16), hh = p.h * a.group + r % a.group;
      const size_t row = static_cast<size_t>(p.row0 + p.t0 + tok);
      const bool any = ll != 0.f;
      if (any) x = make_float4(x.x / ll, x.y / ll, x.z / ll, x.w / ll);
      else x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (!finite4(x) && ll == ll) atomicOr(&s.bad[r >> 5], 1u << (r & 31));
      st4(static_cast<T*>(a.out) + row * a.out_row + hh * a.out_head + d, x);
      if (d == 0 && a.lse != nullptr)
        a.lse[row * a.H + hh] = any ? (mm + log2f(ll)) * 0.69314718055994530942f : -INFINITY;
    };
    bool done = true;
    if (p.whole()) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (ty * R + i < rows) {
#pragma unroll
          for (int e = 0; e < C; ++e) store(ty * R + i, tx * 4 + 64 * e, o[i][e], m[i], l[i]);
        }
    } else {
      const int slot = w.slot(p, blockIdx.x), c0 = w.first_cta(p), c1 = w.last_cta(p);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int r = ty * R + i;
        if (r < rows) {
#pragma unroll
          for (int e = 0; e < C; ++e)
            st4(a.part_o + (static_cast<size_t>(slot) * kPagedPartRows + r) * HD + tx * 4 + 64 * e, o[i][e]);
          if (tx == 0) a.part_ml[slot * kPagedPartRows + r] = make_float2(m[i], l[i]);
        }
      }
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        s.last = atomicAdd(&a.tickets[c0].arrived, 1) == c1 - c0;
        if (s.last) a.tickets[c0].arrived = 0;
        __threadfence();
      }
      __syncthreads();
      done = s.last;
      if (done) {
        for (int i = tid; i < rows * (HD / 4); i += kPThreads) {
          const int r = i / (HD / 4), d = i % (HD / 4) * 4;
          float mm = -INFINITY, ll = 0.f;
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int c = c0; c <= c1; ++c) {
            const int sl = w.slot(p, c) * kPagedPartRows + r;
            const float2 ml = __ldcg(a.part_ml + sl);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(a.part_o + static_cast<size_t>(sl) * HD + d));
            if (ml.x == -INFINITY) continue;  // this part of the keys holds none that the row sees
            const float nm = fmaxf(mm, ml.x), f = exp2f(mm - nm), u = exp2f(ml.x - nm);
            mm = nm;
            ll = ll * f + ml.y * u;
            x = make_float4(x.x * f + y.x * u, x.y * f + y.y * u, x.z * f + y.z * u, x.w * f + y.w * u);
          }
          store(r, d, x, mm, ll);
        }
      }
    }
    __syncthreads();
    if (done)
      for (int r = tid >> 5; r < rows; r += kPThreads / 32)
        if (s.bad[r >> 5] >> (r & 31) & 1)
          exact_row<T, HD>(a, p.b, p.h, p.n, p.len, p.row0, p.t0 + (r * a.group_inv >> 16), p.h * a.group + r % a.group);
  }
}

template <int HD, int BM>
cudaError_t launch(const PagedAttnArgs& a, int grid, cudaStream_t s) {
  const PagedGeom g{BM / a.group, BM / a.group, 6, 1, 2, 2};
  return launch_after(paged_attn_kernel<HD, BM>, dim3(grid), kPThreads, sizeof(PagedSmem<HD, BM>), s, a, g);
}

template <int HD, int BM>
cudaError_t attr() {
  return cudaFuncSetAttribute(paged_attn_kernel<HD, BM>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              sizeof(PagedSmem<HD, BM>));
}

}  // namespace

cudaError_t paged_attention_f32_set_attributes() {
  cudaError_t e = attr<64, 16>();
  if (e == cudaSuccess) e = attr<128, 16>();
  if (e == cudaSuccess) e = attr<64, 64>();
  return e == cudaSuccess ? attr<128, 64>() : e;
}

cudaError_t launch_paged_attention_f32(const PagedAttnArgs& a, int hd, int grid, cudaStream_t s) {
  // rows of one key/value head in an average request
  const long long rows = (static_cast<long long>(a.rows) + a.batch - 1) / a.batch * a.group;
  // (tiles of 16 and of 64 rows: 16 requests of one token at 2000 keys 90 and 152 us, one
  // block of 8 tokens at 32 to 96 keys 6.8 and 10.5 us)
  if (rows <= 16 && a.group <= 16) return hd == 64 ? launch<64, 16>(a, grid, s) : launch<128, 16>(a, grid, s);
  return hd == 64 ? launch<64, 64>(a, grid, s) : launch<128, 64>(a, grid, s);
}

}  // namespace cllm
