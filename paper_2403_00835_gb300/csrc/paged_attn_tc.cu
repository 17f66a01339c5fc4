// Attention of new tokens over a paged cache (cllm_paged_attention), fp16 and bf16
// pools, on tcgen05.
//
//   S = Q K^T,  p = 2^(scale log2(e) S - m),  O = sum p V,  l = sum p,  out = O / l
//
// in one pass over the keys, 128 at a time.  One persistent CTA per SM walks its
// share of the launch's units (paged_walk.cuh): warp 9 streams K and V through a
// ring of 128-key tiles, a TMA box per page and 64 columns; warp 8 issues the MMAs
// (S into tensor memory, then P from tensor memory times V); 4 warps per slot
// hold a row of S per thread, so maximum and sum need no exchange, and write P over S.
//
// The two slots (S/P and O in 256 tensor-memory columns each) hide each other's
// latency.  A tile of more than 128 rows has 128 rows in each, which share K and V; a tile
// of up to 128 rows (a block of a few tokens, greedy decoding) has all its rows in
// both, slot t taking every other chunk of keys, and the halves are merged at the end.
// Rows are tokens times the query heads of a key/value head, so grouped heads
// read K and V once.
//
// Rounding: P goes to the pools' type as the A operand of the second MMA (S, m, l and O
// stay fp32).  Each p keeps the relative precision of the values it multiplies,
// and its error averages over the keys; l sums the unrounded p.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"
#include "paged_walk.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kTcThreads = 384;  // warps 0-3, 4-7: the slots' rows; 8 MMAs; 9 loads; 10, 11 idle
constexpr int kTcRegsLow = 72, kTcRegsRow = 216;
static_assert(128 * kTcRegsLow + 256 * kTcRegsRow <= kTcThreads * 168, "register split");
constexpr int kTcRows = 128, kTcChunk = 128;
// A row's running maximum follows only growth of more than this (in log2): P may
// then reach 2^8, and O in tensor memory is rarely rescaled.
constexpr float kTcSlack = 8.f;

template <int HD>
struct TcSmem {
  static constexpr int kRing = HD == 128 ? 5 : 10;
  static constexpr int kTile = kTcChunk * HD * 2;
  alignas(1024) uint8_t q[2][kTcRows * HD * 2];
  alignas(1024) uint8_t ring[kRing][kTile];
  float2 ml[2][kTcRows];  // also the scratch of run_start
  uint64_t full[kRing], empty[kRing], qfull, qempty, sfull[2], pready[2], ofull[2], ofree, drain;
  RunStart run;
  unsigned bad[8];  // rows whose result is not finite
  uint32_t tmem;
  int abort, busy, last;
};
static_assert(sizeof(TcSmem<128>) <= 227 * 1024 && sizeof(TcSmem<64>) <= 227 * 1024, "shared memory");

struct TcMaps {
  CUtensorMap q, k, v;
};

// mbar_wait, but time in which a warp redoes rows (busy) does not count, and once
// a wait has run out the others end at once.
__device__ __forceinline__ bool tc_wait(uint64_t* bar, uint32_t parity, volatile int* abort, volatile int* busy) {
  if (mbar_try_wait(bar, parity)) return true;
  if (*abort) return false;
  uint64_t t0 = globaltimer_ns();
  uint32_t it = 0;
  while (!mbar_try_wait(bar, parity)) {
    if ((++it & 15u) == 0) {
      if (*abort) return false;
      if (*busy) t0 = globaltimer_ns();
      if (globaltimer_ns() - t0 > kWaitBudgetNs) {
        *abort = 1;
        return false;
      }
    }
  }
  return true;
}

// The chunks of a piece that a slot works on: indices first, first + step, .. < end
// (relative to the piece).
struct SlotChunks {
  int first, end, step;
  __device__ bool any() const { return first < end; }
  __device__ bool has(int i) const { return i >= first && i < end && (i - first) % step == 0; }
  __device__ int last() const { return first + (end - 1 - first) / step * step; }
};
__device__ __forceinline__ SlotChunks slot_chunks(const PagedAttnArgs& a, const Piece& p, int tt, int t) {
  const int n = p.cb - p.ca;
  if (p.nt <= tt) return {t, n, 2};
  const int t0 = p.t0 + t * tt, t1 = min(p.t0 + p.nt, t0 + tt);
  const TileKeys k = tile_keys(a, p.n, p.len, t0, t1);
  return {max(0, k.lo / kTcChunk - p.ca), min(n, (k.hi + kTcChunk - 1) / kTcChunk - p.ca), 1};
}

// Ring position of a piece's loads (K0 K1 V0 K2 V1 .. V(n-1)), relative to its first.
__device__ __forceinline__ int ring_k(int i) { return i == 0 ? 0 : 2 * i - 1; }
__device__ __forceinline__ int ring_v(int i, int n) { return i == n - 1 ? 2 * n - 1 : 2 * i + 2; }

template <class T> struct TcType;
template <> struct TcType<__half> {
  static __device__ uint32_t pack(float a, float b) { return pack_f16x2(a, b); }
  static constexpr uint32_t idesc(int n, bool mn) { return idesc_f16_f32(kTcRows, n, mn); }
};
template <> struct TcType<__nv_bfloat16> {
  static __device__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
  static constexpr uint32_t idesc(int n, bool mn) { return idesc_bf16_f32(kTcRows, n, mn); }
};

template <class T, int HD>
__device__ __forceinline__ void issue_loads(TcSmem<HD>& s, const PagedAttnArgs& a, const PagedGeom& g, const TcMaps& m) {
  constexpr int NH = HD / 64, NR = TcSmem<HD>::kRing;
  const int lane = threadIdx.x & 31, tt = g.tile_tok / 2, P = 1 << a.page_shift;
  const int box = min(P, kTcChunk), boxes = kTcChunk / box;
  uint32_t r = 0, pieces = 0;  // loads so far, pieces with keys so far
  bool ok = true;
  PagedWalk w;
  w.begin(a, g, s.run);
  Piece p;
  while (ok && w.next(a, g, p)) {
    if (p.empty()) continue;
    const int n = p.cb - p.ca;
    auto tile = [&](const CUtensorMap* map, int c) {  // 128 keys from chunk c: those pages that hold keys of the tile
      const int kb = c * kTcChunk, slot = r % NR;
      if (r >= NR) ok = tc_wait(&s.empty[slot], (r / NR - 1) & 1, &s.abort, &s.busy);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      const int b0 = max(p.lo - kb, 0) / box, b1 = (min(p.hi - kb, kTcChunk) + box - 1) / box;
      if (lane == 0) mbar_arrive_expect_tx(&s.full[slot], (b1 - b0) * box * HD * 2);
      __syncwarp();
      const int j = lane / NH, half = lane % NH;  // (boxes * NH <= 32)
      if (j >= b0 && j < b1 && j < boxes) {
        const int pos = kb + j * box;
        int page = __ldg(a.table + static_cast<size_t>(p.b) * a.table_width + (pos >> a.page_shift));
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.n_pages)) {
          atomicOr(a.err, DERR_CAPACITY);
          page = a.n_pages;  // outside the map: reads as zeros
        }
        tma_load_5d(s.ring[slot] + half * kTcChunk * 128 + j * box * 128, map, &s.full[slot], half * 64, pos & (P - 1), p.h,
                    page, a.layer);
      }
      ++r;
    };
    if (pieces > 0) ok = tc_wait(&s.qempty, (pieces - 1) & 1, &s.abort, &s.busy);
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) break;
    const int slots = p.nt > tt ? 2 : 1;
    if (lane == 0) mbar_arrive_expect_tx(&s.qfull, slots * NH * tt * a.group * 128);
    __syncwarp();
    if (lane < slots * NH)
      tma_load_3d(s.q[lane / NH] + lane % NH * kTcRows * 128, &m.q, &s.qfull, lane % NH * 64, p.h * a.group,
                  p.row0 + p.t0 + lane / NH * tt);
    ++pieces;
    tile(&m.k, p.ca);
    for (int i = 0; ok && i < n; ++i) {
      if (i + 1 < n) tile(&m.k, p.ca + i + 1);
      if (ok) tile(&m.v, p.ca + i);
    }
  }
  if (!ok && lane == 0) {  // loads in flight land before the CTA leaves
    for (uint32_t i = r > NR ? r - NR : 0; i < r; ++i) mbar_wait(&s.full[i % NR], (i / NR) & 1, nullptr);
    if (pieces > 0) mbar_wait(&s.qfull, (pieces - 1) & 1, nullptr);
  }
}

template <class T, int HD>
__device__ __forceinline__ void issue_mmas(TcSmem<HD>& s, const PagedAttnArgs& a, const PagedGeom& g, uint32_t tmem, int hold) {
  constexpr int NR = TcSmem<HD>::kRing;
  constexpr uint32_t id_s = TcType<T>::idesc(kTcChunk, false), id_o = TcType<T>::idesc(HD, true);
  const int lane = threadIdx.x & 31, tt = g.tile_tok / 2;
  uint32_t r = 0, pieces = 0, np[2] = {0, 0};  // loads of the pieces before, pieces, P tiles taken
  bool ok = true;
  PagedWalk w;
  w.begin(a, g, s.run);
  Piece p;
  while (ok && w.next(a, g, p)) {
    if (p.empty()) continue;
    const int n = p.cb - p.ca;
    const bool two = p.nt > tt;  // 128 rows in each slot
    const SlotChunks sc[2] = {slot_chunks(a, p, tt, 0), slot_chunks(a, p, tt, 1)};
    if (lane == 0) {
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && tc_wait(bar, parity, &s.abort, &s.busy);
        tc_fence_after();
      };
      auto landed = [&](int at) { wait(&s.full[(r + at) % NR], ((r + at) / NR) & 1); };
      auto release = [&](int at) {
        if (ok) tc_commit(&s.empty[(r + at) % NR]);
      };
      auto mma_s = [&](int t, int i) {  // S of slot t over chunk i
        if (!ok) return;
        const uint32_t qa = smem_u32(s.q[two ? t : 0]), ka = smem_u32(s.ring[(r + ring_k(i)) % NR]);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const uint32_t off = (kk >> 2) * kTcRows * 128 + (kk & 3) * 32;
          tc_mma_f16(tmem + t * 256, sdesc_kmajor_sw128(qa + off), sdesc_kmajor_sw128(ka + off), id_s, kk > 0);
        }
        tc_commit(&s.sfull[t]);
      };
      auto mma_o = [&](int t, int i) {  // O of slot t += P V of chunk i
        if (hold > 0 && i + 1 >= hold) ok = false;  // test hook: as if this thread's wait had run out
        wait(&s.pready[t], np[t] & 1);
        ++np[t];
        if (!ok) return;
        const uint32_t va = smem_u32(s.ring[(r + ring_v(i, n)) % NR]);
#pragma unroll
        for (int kk = 0; kk < kTcChunk / 16; ++kk)
          tc_mma_f16_ts(tmem + t * 256 + 128, tmem + t * 256 + kk * 8, sdesc_mnmajor_sw128(va + kk * 16 * 128, kTcChunk * 128),
                        id_o, i > sc[t].first || kk > 0);
        if (i == sc[t].last()) tc_commit(&s.ofull[t]);
      };
      wait(&s.qfull, pieces & 1);
      landed(0);
      if (two) {
        for (int t = 0; t < 2; ++t)
          if (sc[t].has(0)) mma_s(t, 0);
        release(0);
        if (n == 1 && ok) tc_commit(&s.qempty);
        for (int i = 0; ok && i < n; ++i) {
          landed(ring_v(i, n));
          if (i + 1 < n) landed(ring_k(i + 1));
          if (i == 0 && pieces > 0) wait(&s.ofree, (pieces - 1) & 1);
          for (int t = 0; t < 2; ++t) {
            if (sc[t].has(i)) mma_o(t, i);
            if (i + 1 < n && sc[t].has(i + 1)) mma_s(t, i + 1);
          }
          release(ring_v(i, n));
          if (i + 1 < n) release(ring_k(i + 1));
          if (i + 2 == n && ok) tc_commit(&s.qempty);
        }
      } else {
        mma_s(0, 0);
        release(0);
        if (n > 1) {
          landed(ring_k(1));
          mma_s(1, 1);
          release(ring_k(1));
        }
        if (n <= 2 && ok) tc_commit(&s.qempty);
        for (int i = 0; ok && i < n; ++i) {
          landed(ring_v(i, n));
          if (i == 0 && pieces > 0) wait(&s.ofree, (pieces - 1) & 1);
          mma_o(i & 1, i);
          release(ring_v(i, n));
          if (i + 2 < n) {
            landed(ring_k(i + 2));
            mma_s(i & 1, i + 2);
            release(ring_k(i + 2));
            if (i + 3 == n && ok) tc_commit(&s.qempty);
          }
        }
      }
      if (!ok) {
        s.abort = 1;
        tc_commit(&s.drain);  // MMAs in flight end before the CTA leaves
        mbar_wait(&s.drain, 0, nullptr);
      }
    }
    ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
    r += 2 * n;
    ++pieces;
    np[0] = __shfl_sync(0xffffffffu, np[0], 0);
    np[1] = __shfl_sync(0xffffffffu, np[1], 0);
  }
}

// The rows: softmax of every chunk, then the outputs.  After a wait has run out the
// warps go on without waiting (their results are void), so that none is missing
// at a barrier of the 8.
template <class T, int HD>
__device__ __forceinline__ void run_rows(TcSmem<HD>& s, const PagedAttnArgs& a, const PagedGeom& g, uint32_t tmem) {
  constexpr int NR = TcSmem<HD>::kRing;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t = warp >> 2, tt = g.tile_tok / 2;
  const int row = (warp & 3) * 32 + lane;
  const uint32_t ts = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);  // this warp's lanes, slot 0
  const uint32_t mine = ts + t * 256;
  auto warp_wait = [&](uint64_t* bar, uint32_t parity) {
    if (lane == 0) tc_wait(bar, parity, &s.abort, &s.busy);
    __syncwarp();
    tc_fence_after();
  };
  auto all_rows = [&] { named_bar_sync(1, 256); };
  uint32_t r = 0, ns = 0, no[2] = {0, 0};  // loads of the pieces before, S tiles of this slot, outputs of both
  PagedWalk w;
  w.begin(a, g, s.run);
  Piece p;
  while (w.next(a, g, p)) {
    const int n = p.cb - p.ca;
    const bool two = p.nt > tt;
    const int tok0 = two ? t * tt : 0, ntok = two ? min(tt, p.nt - tok0) : p.nt;
    const int rows = ntok * a.group, tok = p.t0 + tok0 + min(row, rows - 1) / a.group;
    const int head = p.h * a.group + row % a.group;
    const RowKeys rk = row_keys(a, p.n, p.len, p.row0, tok);
    const SlotChunks sc[2] = {slot_chunks(a, p, tt, 0), slot_chunks(a, p, tt, 1)};
    const bool band = (warp & 3) * 32 < rows;  // some row of the warp is live
    float m = -INFINITY, l = 0.f;
    if (!p.empty()) {
      for (int i = t == 0 ? sc[0].first : sc[1].first; i < sc[t].end; i += sc[t].step) {
        const int kb = (p.ca + i) * kTcChunk;
        warp_wait(&s.sfull[t], ns++ & 1);
        if (p.lo > kb || p.hi < kb + kTcChunk) {
          // keys of the chunk that no row of the tile sees (not loaded, or what the
          // page held before): p is 0 there, and so is V
          const int v = r + ring_v(i, n);
          warp_wait(&s.full[v % NR], (v / NR) & 1);
          if (kb + row < p.lo || kb + row >= p.hi) {
#pragma unroll
            for (int c = 0; c < HD / 8; ++c)
              *reinterpret_cast<uint4*>(s.ring[v % NR] + (c >> 3) * kTcChunk * 128 + row * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
        }
        if (band) {
          float x0[64], x1[64];
          tmem_ld64(mine, x0);
          tmem_ld64(mine + 64, x1);
          const bool sees_all = rk.lo <= kb && kb + kTcChunk <= (rk.bits != nullptr ? rk.ctx : rk.hi);
          if (__any_sync(0xffffffffu, !sees_all)) {
            const uint32_t b0 = key_bits(rk, kb), b1 = key_bits(rk, kb + 32), b2 = key_bits(rk, kb + 64), b3 = key_bits(rk, kb + 96);
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (!(b0 >> j & 1)) x0[j] = -INFINITY;
              if (!(b1 >> j & 1)) x0[32 + j] = -INFINITY;
              if (!(b2 >> j & 1)) x1[j] = -INFINITY;
              if (!(b3 >> j & 1)) x1[32 + j] = -INFINITY;
            }
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < 64; j += 4)
#pragma unroll
            for (int u = 0; u < 4; ++u) m4[u] = fmaxf(m4[u], fmaxf(x0[j + u], x1[j + u]));
          const float cm = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * a.scale_log2;
          if (i == sc[t].first) {
            m = cm;
          } else {
            const bool grow = cm > m + kTcSlack || (m == -INFINITY && cm > m);
            if (__any_sync(0xffffffffu, grow)) {
              const float nm = grow ? cm : m;
              const float f = grow ? ex2_ftz(m - nm) : 1.f;
              l *= f;
              m = nm;
#pragma unroll 1
              for (int d = 0; d < HD; d += 64) {
                float o[64];
                tmem_ld64(mine + 128 + d, o);
                uint32_t u[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(o[j] * f);
                tmem_st32(mine + 128 + d, u);
#pragma unroll
                for (int j = 0; j < 32; ++j) u[j] = __float_as_uint(o[32 + j] * f);
                tmem_st32(mine + 128 + d + 32, u);
              }
            }
          }
          const float nm = m == -INFINITY ? 0.f : -m;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
          uint32_t pk[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float p0 = ex2_ftz(fmaf(x0[2 * j], a.scale_log2, nm)), p1 = ex2_ftz(fmaf(x0[2 * j + 1], a.scale_log2, nm));
            sum[j & 3] += p0 + p1;
            pk[j] = TcType<T>::pack(p0, p1);
          }
          tmem_st32(mine, pk);
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float p0 = ex2_ftz(fmaf(x1[2 * j], a.scale_log2, nm)), p1 = ex2_ftz(fmaf(x1[2 * j + 1], a.scale_log2, nm));
            sum[j & 3] += p0 + p1;
            pk[j] = TcType<T>::pack(p0, p1);
          }
          tmem_st32(mine + 32, pk);
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.pready[t]);
      }
    }
    const bool whole = p.whole();
    const int cta0 = whole ? 0 : w.first_cta(p), cta1 = whole ? 0 : w.last_cta(p);
    const size_t slot_row = whole ? 0 : static_cast<size_t>(w.slot(p, blockIdx.x)) * kPagedPartRows;
    // `count` columns of a row from column d: a result, or a partial one
    auto store16 = [&](const float (&o)[16], int rr, int d, float scale, bool live) {
      if (!live) return false;
      if (!whole) {
        float4* po = reinterpret_cast<float4*>(a.part_o + (slot_row + rr) * HD + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) po[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        return false;
      }
      T* out = static_cast<T*>(a.out) + static_cast<long long>(p.row0 + tok) * a.out_row + head * a.out_head + d;
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 16; j += 8) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = scale != 0.f ? o[j + 2 * e] * scale : 0.f, y = scale != 0.f ? o[j + 2 * e + 1] * scale : 0.f;
          bad |= !isfinite(x) || !isfinite(y);
          u[e] = TcType<T>::pack(x, y);
        }
        *reinterpret_cast<uint4*>(out + j) = make_uint4(u[0], u[1], u[2], u[3]);
      }
      return bad;
    };
    auto store_lse = [&](int row_tok, int hh, float mm, float ll) {
      if (a.lse != nullptr)
        a.lse[static_cast<size_t>(p.row0 + row_tok) * a.H + hh] = ll != 0.f ? (mm + log2f(ll)) * 0.69314718055994530942f : -INFINITY;
    };
    auto redo = [&](int rr) {  // (the whole warp)
      __syncwarp();
      if (lane == 0) atomicAdd(&s.busy, 1);
      exact_row<T, HD>(a, p, p.t0 + (two ? rr / kTcRows * tt : 0) + (rr % kTcRows) / a.group, p.h * a.group + (rr % kTcRows) % a.group);
      if (lane == 0) atomicAdd(&s.busy, -1);
    };
    bool shared_rows = false;  // rows whose columns several warps have written
    if (two) {
      const bool has = sc[t].any() && !p.empty();
      if (has) warp_wait(&s.ofull[t], no[t] & 1);
      const bool live = row < rows;
      const float scale = l != 0.f ? 1.f / l : 0.f;
      bool bad = false;
      if (band) {
#pragma unroll 1
        for (int d = 0; d < HD; d += 16) {
          float o[16];
          if (has) tmem_ld16(mine + 128 + d, o);
          else
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = 0.f;
          bad |= store16(o, t * kTcRows + row, d, scale, live);
        }
      }
      if (live) {
        if (whole) store_lse(tok, head, m, l);
        else a.part_ml[slot_row + t * kTcRows + row] = make_float2(m, l);
      }
      if (whole)
        for (unsigned redo_rows = __ballot_sync(0xffffffffu, bad); redo_rows; redo_rows &= redo_rows - 1)
          redo(t * kTcRows + (warp & 3) * 32 + __ffs(redo_rows) - 1);
    } else {
      // both slots hold these rows, each over half of the keys; slot t's warps finish
      // the t-th half of the columns
      s.ml[t][row] = make_float2(m, l);
      all_rows();
      const float2 ml0 = s.ml[0][row], ml1 = s.ml[1][row];
      bool has[2];
      for (int u = 0; u < 2; ++u) {
        has[u] = sc[u].any() && !p.empty();
        if (has[u]) warp_wait(&s.ofull[u], no[u] & 1);
      }
      const bool use0 = has[0] && ml0.x != -INFINITY, use1 = has[1] && ml1.x != -INFINITY;
      const float mm = fmaxf(ml0.x, ml1.x);
      const float f0 = use0 ? ex2_ftz(ml0.x - mm) : 0.f, f1 = use1 ? ex2_ftz(ml1.x - mm) : 0.f;
      const float ll = (use0 ? ml0.y * f0 : 0.f) + (use1 ? ml1.y * f1 : 0.f);
      const float scale = ll != 0.f ? 1.f / ll : 0.f;
      const bool live = row < rows;
      bool bad = false;
      if (band) {
#pragma unroll 1
        for (int d = t * (HD / 2); d < (t + 1) * (HD / 2); d += 16) {
          float o[16], o1[16];
          if (has[0]) tmem_ld16(ts + 128 + d, o);
          if (has[1]) tmem_ld16(ts + 256 + 128 + d, o1);
#pragma unroll
          for (int j = 0; j < 16; ++j) o[j] = (use0 ? o[j] * f0 : 0.f) + (use1 ? o1[j] * f1 : 0.f);
          bad |= store16(o, row, d, scale, live);
        }
      }
      if (live && t == 0) {
        if (whole) store_lse(tok, head, mm, ll);
        else a.part_ml[slot_row + row] = make_float2(mm, ll);
      }
      if (bad) atomicOr(&s.bad[row >> 5], 1u << (row & 31));
      shared_rows = whole;
    }
    if (!p.empty()) {  // the accumulators may be overwritten
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.ofree);
      r += 2 * n;
      for (int u = 0; u < 2; ++u) no[u] += sc[u].any();
    }
    if (!whole) {
      __threadfence();
      all_rows();
      if (tid == 0) {
        s.last = atomicAdd(a.tickets + cta0, 1) == cta1 - cta0;
        if (s.last) a.tickets[cta0] = 0;
        __threadfence();
      }
      all_rows();
      if (s.last) {
        // merge the parts of the tile in order, 4 columns of a row per thread
        const int items = p.nt * a.group * (HD / 4);
        for (int i = tid; i < items; i += 256) {
          const int k = i / (HD / 4), d = i % (HD / 4) * 4, kt = k / a.group, hh = p.h * a.group + k % a.group;
          const int rr = two && kt >= tt ? kTcRows + (kt - tt) * a.group + k % a.group : k;
          float mm = -INFINITY, ll = 0.f;
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int c = cta0; c <= cta1; ++c) {
            const size_t at = static_cast<size_t>(w.slot(p, c)) * kPagedPartRows + rr;
            const float2 ml = __ldcg(a.part_ml + at);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(a.part_o + at * HD + d));
            const bool use = ml.x != -INFINITY;
            const float nm = fmaxf(mm, ml.x), f = mm == -INFINITY ? 0.f : ex2_ftz(mm - nm), u = use ? ex2_ftz(ml.x - nm) : 0.f;
            mm = nm;
            ll = ll * f + (use ? ml.y * u : 0.f);
            x.x = x.x * f + (use ? y.x * u : 0.f);
            x.y = x.y * f + (use ? y.y * u : 0.f);
            x.z = x.z * f + (use ? y.z * u : 0.f);
            x.w = x.w * f + (use ? y.w * u : 0.f);
          }
          const float scale = ll != 0.f ? 1.f / ll : 0.f;
          x = ll != 0.f ? make_float4(x.x * scale, x.y * scale, x.z * scale, x.w * scale) : make_float4(0.f, 0.f, 0.f, 0.f);
          if (!isfinite(x.x) || !isfinite(x.y) || !isfinite(x.z) || !isfinite(x.w)) atomicOr(&s.bad[rr >> 5], 1u << (rr & 31));
          *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + static_cast<long long>(p.row0 + p.t0 + kt) * a.out_row + hh * a.out_head + d) =
              make_uint2(TcType<T>::pack(x.x, x.y), TcType<T>::pack(x.z, x.w));
          if (d == 0) store_lse(p.t0 + kt, hh, mm, ll);
        }
        shared_rows = true;
      }
    }
    if (!two || !whole) all_rows();  // (rows written by several warps; s.ml is free again)
    if (shared_rows) {
      unsigned any = 0;
      for (int i = 0; i < 8; ++i) any |= s.bad[i];
      if (any) {
        for (int rr = warp; rr < 256; rr += 8)
          if (s.bad[rr >> 5] >> (rr & 31) & 1) redo(rr);
        all_rows();
        if (tid < 8) s.bad[tid] = 0;
        all_rows();
      }
    }
  }
}

template <class T, int HD>
__global__ void __launch_bounds__(kTcThreads, 1)
    paged_attn_tc_kernel(const __grid_constant__ TcMaps m, const __grid_constant__ PagedAttnArgs a, const PagedGeom g,
                         const int hold) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  TcSmem<HD>& s = *reinterpret_cast<TcSmem<HD>*>(smem_raw);
  if (smem_u32(smem_raw) & 1023u) {  // (the swizzle's atoms; shared memory starts on one)
    if (threadIdx.x == 0) atomicOr(a.err, DERR_SHAPE);
    return;
  }
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < TcSmem<HD>::kRing; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    mbar_init(&s.qfull, 1);
    mbar_init(&s.qempty, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&s.sfull[t], 1);
      mbar_init(&s.pready[t], 4);
      mbar_init(&s.ofull[t], 1);
    }
    mbar_init(&s.ofree, 8);
    mbar_init(&s.drain, 1);
    s.abort = s.busy = 0;
    fence_mbar_init();
  }
  if (threadIdx.x < 8) s.bad[threadIdx.x] = 0;
  if (warp == 8) {
    tmem_alloc(&s.tmem, 512);
    tmem_relinquish();
  }
  run_start(a, g, &s.run, reinterpret_cast<long long*>(s.ml));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  if (warp >= 8) {
    setmaxnreg_dec<kTcRegsLow>();
    if (warp == 8) issue_mmas<T, HD>(s, a, g, tmem, hold);
    else if (warp == 9) issue_loads<T, HD>(s, a, g, m);
  } else {
    setmaxnreg_inc<kTcRegsRow>();
    run_rows<T, HD>(s, a, g, tmem);
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && s.abort) atomicOr(a.err, DERR_TIMEOUT);
  if (warp == 8) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <class T, int HD>
cudaError_t launch_tc(const TcMaps& m, const PagedAttnArgs& a, int hold, int grid, cudaStream_t s) {
  const PagedGeom g{2 * (kTcRows / a.group), kTcChunk, 2};
  paged_attn_tc_kernel<T, HD><<<grid, kTcThreads, sizeof(TcSmem<HD>), s>>>(m, a, g, hold);
  return cudaGetLastError();
}

}  // namespace

cudaError_t paged_attention_tc_set_attributes() {
  cudaError_t e = cudaFuncSetAttribute(paged_attn_tc_kernel<__half, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(TcSmem<64>));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attn_tc_kernel<__half, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(TcSmem<128>));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attn_tc_kernel<__nv_bfloat16, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(TcSmem<64>));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attn_tc_kernel<__nv_bfloat16, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(TcSmem<128>));
  return e;
}

bool paged_pool_map(CUtensorMap* m, const void* pool, const cllm_paged_desc& d) {
  const cuuint64_t dims[5] = {static_cast<cuuint64_t>(d.head_dim), static_cast<cuuint64_t>(d.page_size),
                              static_cast<cuuint64_t>(d.n_kv_heads), static_cast<cuuint64_t>(d.n_pages),
                              static_cast<cuuint64_t>(d.layers)};
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(d.stride_pos) * 2, static_cast<cuuint64_t>(d.stride_head) * 2,
                                 static_cast<cuuint64_t>(d.stride_page) * 2, static_cast<cuuint64_t>(d.stride_layer) * 2};
  const cuuint32_t box[5] = {64, static_cast<cuuint32_t>(d.page_size < kTcChunk ? d.page_size : kTcChunk), 1, 1, 1};
  return make_map_nd(m, d.dtype == CLLM_BF16, pool, 5, dims, strides, box);
}

cudaError_t launch_paged_attention_tc(const PagedAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int dtype, int hd,
                                      int hold, int grid, cudaStream_t s) {
  TcMaps m;
  m.k = k;
  m.v = v;
  // queries of a tile: group heads of 128 / group tokens, row = token * group + head
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(hd), static_cast<cuuint64_t>(a.H), static_cast<cuuint64_t>(a.rows)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(a.q_head) * 2, static_cast<cuuint64_t>(a.q_row) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(a.group), static_cast<cuuint32_t>(kTcRows / a.group)};
  if (!make_map_nd(&m.q, dtype == CLLM_BF16, a.q, 3, dims, strides, box)) return cudaErrorInvalidValue;
  if (dtype == CLLM_BF16)
    return hd == 64 ? launch_tc<__nv_bfloat16, 64>(m, a, hold, grid, s) : launch_tc<__nv_bfloat16, 128>(m, a, hold, grid, s);
  return hd == 64 ? launch_tc<__half, 64>(m, a, hold, grid, s) : launch_tc<__half, 128>(m, a, hold, grid, s);
}

}  // namespace cllm
