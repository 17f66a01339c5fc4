// Attention of few rows over a paged cache (cllm_paged_attention), fp16 and bf16
// pools: greedy decoding and blocks of a few tokens, up to 16 rows to a key/value head.
//
//   S = Q K^T,  p = 2^(scale log2(e) S - m),  O = sum p V,  l = sum p,  out = O / l
//
// in one pass over the keys.  The keys' bytes bound the work (16 rows x 128 keys are
// 1 MFLOP to 64 KB), and what there is to lose is latency: the tensor-memory kernel
// hands a chunk from loads to MMAs to rows to MMAs and back, with one warp of a
// slot at work on 16 rows.  Here 4 warps take every chunk of 64 keys, each all rows x 16
// keys, with warp-level MMAs, scores and probabilities in registers, and its own running
// maximum, sum and output; they meet at the tile's end only, in shared memory.  Warp 4
// streams K and V through a ring of 64-key tiles.  Two CTAs share an SM, so that one's
// tile has its beginning or end while the other's streams.  A row's keys are dealt to the
// warps in fixed order, so results do not depend on timing.
//
// Measured: 8 blocks of 16 tokens at 600 keys, 32 heads: 13.6 us, 6.1 TB/s (the tensor-memory
// kernel: 20.0); 64 requests of one token at 300 keys, 32 heads on 8: 15.9 us, 5.0 TB/s (28.1);
// 128 of one token at 100 keys, 32 heads: 58 us (102); 16 of one token at 4096 keys, 32 heads
// on 8: 51 us, 5.3 TB/s (46: where lengths are long the other's deeper ring is worth more
// than this one's short ends; the host, which chooses, knows the tables' width, a bound on the lengths,
// and does not use it); one
// block of 16 at 144 keys: 7.8 us (8.9), of which a launch's start, the first loads' latency
// and cold instructions are about 5.
//
// Rounding: as in the tensor-memory kernel, P goes to the pools' type, in fp16 at 2^7 times its value.
#include "paged_pipe.cuh"

namespace cllm {

namespace {

constexpr int kFewWarps = 4, kFewThreads = 32 * (kFewWarps + 1);

template <int HD>
struct FewSmem {
  static constexpr int kShift = 6, kRing = HD == 128 ? 4 : 8;
  static constexpr int kTile = kFewKeys * HD * 2;
  static constexpr int kRows = kFewRows, kRowWarps = kFewWarps, kPartRows = 32, kBands = 1;
  static constexpr bool kAhead = false, kIssuer = false;
  alignas(1024) uint8_t q[1][kRows * HD * 2];
  alignas(1024) uint8_t ring[kRing][kTile];
  float o[kFewWarps][kFewRows][HD + 4];  // the warps' outputs at a tile's end
  float2 wml[kFewWarps][kFewRows];
  unsigned scan[32];                     // of run_start_block
  uint64_t full[kRing], empty[kRing], qfull, qempty;
  uint64_t pfull[kPagePieces], pempty[kPagePieces];
  PagePiece piece[kPagePieces], cut[2];  // (cut: to be merged after the run)
  RunStart run;
  unsigned bad[8];
  int abort, busy, last, claim;
};
static_assert(2 * (sizeof(FewSmem<128>) + 1024) <= 228 * 1024, "two CTAs to an SM");
static_assert(1 << FewSmem<64>::kShift == kFewKeys, "keys of a tile");

template <class T> struct Mma16;
template <> struct Mma16<__half> {
  static __device__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    mma_f16_16816(d, a, b0, b1);
  }
};
template <> struct Mma16<__nv_bfloat16> {
  static __device__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    mma_bf16_16816(d, a, b0, b1);
  }
};

// 16-byte piece `c` of row `row` of a tile with the 128-byte swizzle, 64 columns of all rows after another.
__device__ __forceinline__ uint32_t tile_addr(uint32_t base, int rows, int row, int c) {
  return base + (c >> 3) * rows * 128 + row * 128 + (((c & 7) ^ (row & 7)) << 4);
}

template <class T, int HD>
__device__ __forceinline__ void run_few(FewSmem<HD>& s, const PagedAttnArgs& a, const PagedGeom& g) {
  using S = FewSmem<HD>;
  constexpr int KW = kFewWarps, KEYS = kFewKeys / KW;  // warps that share a row's keys, keys of a warp in a chunk
  static_assert(KEYS == 16, "a k step of the second product");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int quad = lane >> 2, col = (lane & 3) * 2, tt = g.slot_tok;
  auto warp_wait = [&](uint64_t* bar, uint32_t parity) { page_wait(bar, parity, &s.abort, &s.busy); };
  RingAt<S::kRing> at;
  RingAt<kPagePieces> pat;
  uint32_t nq = 0;       // pieces with keys so far
  int cuts = 0, before0 = 0, before1 = 0;  // parts to be merged; thread 0: the parts of them that were there before
  for (;; ++pat) {
    if (!piece_wait(&s.pfull[pat.i], pat.phase)) break;
    const PagePiece& p = s.piece[pat.i];
    if (p.end) break;
    const int n = p.chunks, rows = p.nt * a.group, lo = p.lo, hi = p.hi, ca = p.ca;
    float o[HD / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < HD / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    if (n > 0) {
      uint32_t q[HD / 16][4];
      warp_wait(&s.qfull, nq++ & 1);
      const uint32_t qb = smem_u32(s.q[0]);
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk) ldmatrix_x4_a(q[kk], tile_addr(qb, S::kRows, lane & 15, kk * 2 + (lane >> 4)));
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.qempty);
      auto keys_of = [&](int r) {  // of row r of the tile
        return row_keys(a, p.n, p.len, p.row0, p.t0 + (min(r, rows - 1) * a.group_inv >> 16));
      };
      // keys [from, to) are seen by both of this lane's rows
      const int from = keys_of(quad + 8).lo, to = a.mask != nullptr ? p.len - p.n : keys_of(quad).hi;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const int kb = (ca + i) * kFewKeys + warp * KEYS;  // this warp's keys: [kb, kb + KEYS)
        const bool some = kb < hi && kb + KEYS > lo;
        const uint32_t kt = at.i, k_phase = at.phase;
        ++at;
        const uint32_t vt = at.i, v_phase = at.phase;
        ++at;
        float x[KEYS / 8][4];
        warp_wait(&s.full[kt], k_phase);
        if (some) {
          const uint32_t base = smem_u32(s.ring[kt]);
#pragma unroll
          for (int j = 0; j < KEYS / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = 0.f;
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk)
#pragma unroll
            for (int j = 0; j < KEYS / 16; ++j) {
              uint32_t b[4];
              const int key = warp * KEYS + j * 16 + (lane >> 4) * 8 + (lane & 7);
              ldmatrix_x4_a(b, tile_addr(base, kFewKeys, key, kk * 2 + (lane >> 3 & 1)));
              Mma16<T>::mma(x[2 * j], q[kk], b[0], b[1]);
              Mma16<T>::mma(x[2 * j + 1], q[kk], b[2], b[3]);
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.empty[kt]);
        if (some) {
          if (__any_sync(0xffffffffu, from > kb || kb + KEYS > to)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int c = 0; c < (KEYS + 31) / 32; ++c) {
                const uint32_t see = key_bits(keys_of(quad + 8 * u), kb + 32 * c) >> col;
#pragma unroll
                for (int j = 4 * c; j < min(4 * c + 4, KEYS / 8); ++j) {
                  if (!(see >> (j - 4 * c) * 8 & 1)) x[j][2 * u] = -INFINITY;
                  if (!(see >> ((j - 4 * c) * 8 + 1) & 1)) x[j][2 * u + 1] = -INFINITY;
                }
              }
          }
          float cm[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            cm[u] = -INFINITY;
#pragma unroll
            for (int j = 0; j < KEYS / 8; ++j) cm[u] = fmaxf(cm[u], fmaxf(x[j][2 * u], x[j][2 * u + 1]));
            cm[u] = fmaxf(cm[u], __shfl_xor_sync(0xffffffffu, cm[u], 1));
            cm[u] = fmaxf(cm[u], __shfl_xor_sync(0xffffffffu, cm[u], 2)) * a.scale_log2;
          }
          const bool grow0 = cm[0] > m[0] + kPageSlack || (m[0] == -INFINITY && cm[0] > m[0]);
          const bool grow1 = cm[1] > m[1] + kPageSlack || (m[1] == -INFINITY && cm[1] > m[1]);
          if (__any_sync(0xffffffffu, grow0 || grow1)) {
            const float f0 = grow0 ? ex2_ftz(m[0] - cm[0]) : 1.f, f1 = grow1 ? ex2_ftz(m[1] - cm[1]) : 1.f;
            if (grow0) m[0] = cm[0];
            if (grow1) m[1] = cm[1];
            l[0] *= f0, l[1] *= f1;
#pragma unroll
            for (int j = 0; j < HD / 8; ++j) o[j][0] *= f0, o[j][1] *= f0, o[j][2] *= f1, o[j][3] *= f1;
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float nm = m[u] == -INFINITY ? 0.f : Pack16<T>::kTop - m[u];
#pragma unroll
            for (int j = 0; j < KEYS / 8; ++j) {
              x[j][2 * u] = ex2_ftz(fmaf(x[j][2 * u], a.scale_log2, nm));
              x[j][2 * u + 1] = ex2_ftz(fmaf(x[j][2 * u + 1], a.scale_log2, nm));
              l[u] += x[j][2 * u] + x[j][2 * u + 1];
            }
          }
        }
        warp_wait(&s.full[vt], v_phase);
        if (some) {
          if (lo > kb || hi < kb + KEYS) {
            // keys that no row of the tile sees (not loaded, or what the page held before): p
            // is 0 there, and so is V
            for (int c = lane; c < KEYS * HD / 8; c += 32) {
              const int k = c / (HD / 8), key = kb + k;
              if (key < lo || key >= hi)
                *reinterpret_cast<uint4*>(s.ring[vt] + (c % (HD / 8) >> 3) * kFewKeys * 128 + (warp * KEYS + k) * 128 +
                                          (c & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            // (before the tile is loaded anew)
            fence_proxy_async_smem();
            __syncwarp();
          }
          const uint32_t base = smem_u32(s.ring[vt]);
#pragma unroll
          for (int j = 0; j < KEYS / 16; ++j) {
            const uint32_t pa[4] = {Pack16<T>::pack(x[2 * j][0], x[2 * j][1]), Pack16<T>::pack(x[2 * j][2], x[2 * j][3]),
                                    Pack16<T>::pack(x[2 * j + 1][0], x[2 * j + 1][1]),
                                    Pack16<T>::pack(x[2 * j + 1][2], x[2 * j + 1][3])};
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) {
              uint32_t b[4];
              ldmatrix_x4_trans_a(b, tile_addr(base, kFewKeys, warp * KEYS + j * 16 + (lane & 15), d * 2 + (lane >> 4)));
              Mma16<T>::mma(o[2 * d], pa, b[0], b[1]);
              Mma16<T>::mma(o[2 * d + 1], pa, b[2], b[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.empty[vt]);
      }
    }
    // the warps' shares meet in shared memory
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
      l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
      m[u] = share_max(m[u], l[u]);
      if ((lane & 3) == 0) s.wml[warp][quad + 8 * u] = make_float2(m[u], l[u]);
#pragma unroll
      for (int j = 0; j < HD / 8; ++j)
        *reinterpret_cast<float2*>(&s.o[warp][quad + 8 * u][j * 8 + col]) = make_float2(o[j][2 * u], o[j][2 * u + 1]);
    }
    all_rows<S>();
    const bool whole = p.whole;
    const int part_rows = rows_of_part<S>(a, p);
    float4* part = part_of<S, HD>(a, p.slot);
    float2* part_ml = part_ml_of<S>(a, p.slot);
    for (int i = tid; i < rows * (HD / 8); i += 32 * kFewWarps) {
      // (a result's columns side by side, a part's rows)
      const int r = whole ? i / (HD / 8) : i % rows, d8 = whole ? i % (HD / 8) : i / rows;
      float mm = -INFINITY, ll = 0.f;
      float2 ml[KW];
#pragma unroll
      for (int c = 0; c < KW; ++c) {
        ml[c] = s.wml[c][r];
        mm = fmaxf(mm, ml[c].x);
      }
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
#pragma unroll
      for (int c = 0; c < KW; ++c) {
        if (ml[c].x == -INFINITY) continue;  // none of its keys is seen
        const float4* from = reinterpret_cast<const float4*>(&s.o[c][r][d8 * 8]);
        const float4 u = from[0], w = from[1];
        const float f = ex2_ftz(ml[c].x - mm);
        ll = fmaf(ml[c].y, f, ll);
        x = make_float4(fmaf(u.x, f, x.x), fmaf(u.y, f, x.y), fmaf(u.z, f, x.z), fmaf(u.w, f, x.w));
        y = make_float4(fmaf(w.x, f, y.x), fmaf(w.y, f, y.y), fmaf(w.z, f, y.z), fmaf(w.w, f, y.w));
      }
      if (!whole) {
        part[2 * d8 * part_rows + r] = x;
        part[(2 * d8 + 1) * part_rows + r] = y;
        if (d8 == 0) part_ml[r] = make_float2(share_max(mm, ll), ll);
        continue;
      }
      const float f = ll != 0.f ? 1.f / ll : 0.f;
      const float z[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
      uint32_t u[4];
      float any = 0.f;  // (0 * x is NaN for an infinity or NaN)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v0 = ll != 0.f ? z[2 * e] * f : 0.f, v1 = ll != 0.f ? z[2 * e + 1] * f : 0.f;
        any = fmaf(v0, 0.f, fmaf(v1, 0.f, any));
        u[e] = Pack16<T>::pack(v0, v1);
      }
      if (any != 0.f && ll == ll) atomicOr(&s.bad[r >> 5], 1u << (r & 31));
      const int rt = r * a.group_inv >> 16, tok = p.t0 + rt, head = p.h * a.group + r - rt * a.group;
      T* out = static_cast<T*>(a.out) + static_cast<long long>(p.row0 + tok) * a.out_row + head * a.out_head + d8 * 8;
      *reinterpret_cast<uint4*>(out) = make_uint4(u[0], u[1], u[2], u[3]);
      if (d8 == 0) store_lse<T>(a, p, tok, head, mm, ll);
    }
    all_rows<S>();  // (s.o and s.wml are free again)
    if (whole) {
      redo_bad<T, HD>(s, a, p, tt);
    } else {
      const int before = arrive_part<S>(a, p);
      // nothing waits for the counter's answer here: whether this CTA has to merge the
      // tile is seen to after the run (whose first and last pieces may be parts)
      (cuts == 0 ? before0 : before1) = before;
      if (tid < sizeof(PagePiece) / 4) reinterpret_cast<int*>(&s.cut[cuts])[tid] = reinterpret_cast<const int*>(&p)[tid];
      ++cuts;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.pempty[pat.i]);
  }
#pragma unroll 1
  for (int k = cuts - 1; k >= 0; --k) finish_cut<T, HD>(s, a, s.cut[k], tt, k == 0 ? before0 : before1);
}

template <class T, int HD>
__global__ void __launch_bounds__(kFewThreads, 2)
    paged_attn_few_kernel(const __grid_constant__ PagedMaps m, const __grid_constant__ PagedAttnArgs a, const PagedGeom g,
                          const int hold) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  FewSmem<HD>& s = *reinterpret_cast<FewSmem<HD>*>(smem_raw);
  if (smem_u32(smem_raw) & 1023u) {  // (the swizzle's atoms; shared memory starts on one)
    pdl_wait();
    if (threadIdx.x == 0) atomicOr(a.err, DERR_SHAPE);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < FewSmem<HD>::kRing; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], kFewWarps);
    }
    mbar_init(&s.qfull, 1);
    mbar_init(&s.qempty, kFewWarps);
    for (int i = 0; i < kPagePieces; ++i) {
      mbar_init(&s.pfull[i], 1);
      mbar_init(&s.pempty[i], kFewWarps);
    }
    s.abort = s.busy = 0;
    fence_mbar_init();
  }
  if (threadIdx.x < 8) s.bad[threadIdx.x] = 0;
  if (threadIdx.x == kFewThreads - 1) {
    tma_prefetch_desc(&m.q);
    tma_prefetch_desc(&m.k);
    tma_prefetch_desc(&m.v);
  }
  pdl_launch_dependents();
  pdl_wait();  // (nothing of the calls before is read above)
  if (a.batch > kWarpRequests) run_start_block(a, g, &s.run, s.scan);
  __syncthreads();
  if (threadIdx.x >= 32 * kFewWarps) issue_loads<HD>(s, a, g, m, hold);
  else run_few<T, HD>(s, a, g);
  __syncthreads();
  if (threadIdx.x == 0 && s.abort) atomicOr(a.err, DERR_TIMEOUT);
}

template <class T, int HD>
cudaError_t launch_few(const PagedMaps& m, const PagedAttnArgs& a, int hold, int sms, cudaStream_t s) {
  const int tt = kFewRows / a.group;
  return launch_after(paged_attn_few_kernel<T, HD>, dim3(2 * sms), kFewThreads, sizeof(FewSmem<HD>), s, m, a,
                      PagedGeom{tt, tt, FewSmem<HD>::kShift, 1, 4, 3}, hold);
}

template <class T, int HD>
cudaError_t attr() {
  return cudaFuncSetAttribute(paged_attn_few_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              sizeof(FewSmem<HD>));
}

}  // namespace

cudaError_t paged_attention_few_set_attributes() {
  cudaError_t e = attr<__half, 64>();
  if (e == cudaSuccess) e = attr<__half, 128>();
  if (e == cudaSuccess) e = attr<__nv_bfloat16, 64>();
  return e == cudaSuccess ? attr<__nv_bfloat16, 128>() : e;
}

cudaError_t launch_paged_attention_few(const PagedAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int dtype,
                                       int hd, int hold, int sms, cudaStream_t s) {
  PagedMaps m;
  m.k = k;
  m.v = v;
  if (!paged_query_map(&m.q, a, dtype, hd, kFewRows)) return cudaErrorInvalidValue;
  if (dtype == CLLM_BF16)
    return hd == 64 ? launch_few<__nv_bfloat16, 64>(m, a, hold, sms, s)
                    : launch_few<__nv_bfloat16, 128>(m, a, hold, sms, s);
  return hd == 64 ? launch_few<__half, 64>(m, a, hold, sms, s) : launch_few<__half, 128>(m, a, hold, sms, s);
}

}  // namespace cllm
