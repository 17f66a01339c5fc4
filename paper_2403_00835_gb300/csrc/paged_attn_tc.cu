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
// The two slots (S/P and O in 256 tensor-memory columns each) hide each other's latency;
// P V starts on the first 64 keys of a chunk while the rows work on the others.  A tile
// of more than 128 rows has 128 rows in each slot, which share K and V.  A tile of up to 128
// rows has all its rows in both, slot t taking every other chunk of keys, and the halves
// are merged at the end.  A tile of up to 64 (32) rows is laid out in 2 (4) bands of the 128
// lanes, the same queries in each: the MMAs cost what they did, but a band's warps take
// the maximum and the exponentials of their half (quarter) of a chunk's keys only, P being
// 0 for the others, and the bands' O are summed with the slots'.  Rows are tokens times
// the query heads of a key/value head, so grouped heads read K and V once.
//
// Bound: for long tiles no unit by itself (2048 tokens after 4096, 32 heads: 164 us, 1.05
// PFLOP/s; a chunk of 2 x 128 rows x 128 keys takes 3850 cycles, 2048 of them the MMAs' at their
// full rate; counters: tensor pipe 41 % of the cycles, the exponentials' pipe 21 %, issue slots 35 %)
// but the row warps' dependent steps from S to P, which the other slot's MMAs hide in part; HBM for
// long contexts (16 tokens, 32 heads on 8, over 131072: 91 us, 5.9 TB/s); what a piece costs beside its keys (2 to 3 us:
// its first loads, S and O one after another) for short ones (8 requests of 32 tokens, 256
// to 1024 keys, 32 heads: 26.5 us, 3.5 TB/s).
//
// Rounding: P goes to the pools' type as the A operand of the second MMA, which takes no
// wider one beside 16-bit values (S, m, l and O stay fp32).  A p is off by at most 2^-8 of itself
// in bf16, 2^-11 in fp16 down to 2^-21 of the row's largest, errors that average over the
// keys, and below that in fp16 by 2^-32 of the largest; l sums the unrounded p.  Against 64
// bits results are off by 0.0020-0.0023 (bf16) and 0.00026-0.00028 (fp16) relative, rounding alone
// by 0.0017 and 0.00021.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged_pipe.cuh"

namespace cllm {

namespace {

constexpr int kTcThreads = 320;  // warps 0-3, 4-7: the slots' rows; 8 MMAs; 9 loads
constexpr int kTcRows = 128, kTcShift = 7, kTcChunk = 1 << kTcShift, kTcHalf = 64;
template <int HD, int NB>
struct TcSmem {
  static constexpr int kRows = kTcRows, kRowWarps = 8, kShift = kTcShift, kPartRows = 2 * kTcRows, kBands = NB;
  static constexpr bool kAhead = true, kIssuer = true;
  static constexpr int kRing = HD == 128 ? 5 : 10;
  static constexpr int kTile = kTcChunk * HD * 2;
  alignas(1024) uint8_t q[2][kTcRows * HD * 2];
  alignas(1024) uint8_t ring[kRing][kTile];
  float2 ml[2][kTcRows];  // also the scratch of run_start
  uint64_t full[kRing], empty[kRing], qfull, qempty, ofree, drain;
  // of a slot: S is there; P of a half of the keys is; the piece's O is
  uint64_t sfull[2], pready[2][2], ofull[2];
  // a piece is there; the rows, the issuer are done with it
  uint64_t pfull[kPagePieces], pempty[kPagePieces], pfree[kPagePieces];
  PagePiece piece[kPagePieces], cut[2];  // (cut: to be merged after the run)
  RunStart run;
  unsigned bad[8];  // rows whose result is not finite
  uint32_t tmem;
  int abort, busy, last, claim;
};
static_assert(sizeof(TcSmem<128, 1>) <= 227 * 1024 && sizeof(TcSmem<64, 1>) <= 227 * 1024, "shared memory");

template <class T> struct TcType;
template <> struct TcType<__half> {
  static constexpr uint32_t idesc(int n, bool mn) { return idesc_f16_f32(kTcRows, n, mn); }
};
template <> struct TcType<__nv_bfloat16> {
  static constexpr uint32_t idesc(int n, bool mn) { return idesc_bf16_f32(kTcRows, n, mn); }
};

// Ring position of a piece's V tiles (loaded as K0 K1 V0 K2 V1 .. V(n-1)), relative to K0.
__device__ __forceinline__ int ring_v(int i, int n) { return i == n - 1 ? 2 * n - 1 : 2 * i + 2; }

// The MMAs of the CTA, by one warp, whose instructions are what its chunks cost beside
// the tensor cores' own time (it shares its scheduler with two row warps): descriptors
// are made once and moved by an add, and what decides about them is known to be the
// same in all lanes.  (Made anew for every MMA they held the warp up for 8800 cycles per
// chunk of 256 rows, against 2048 of tensor-core time.)
template <class T, int HD, int NB>
__device__ __forceinline__ void issue_mmas(TcSmem<HD, NB>& s, uint32_t tmem, int hold) {
  const int lane = threadIdx.x & 31;
  tmem = __reduce_max_sync(0xffffffffu, tmem);
  constexpr int NR = TcSmem<HD, NB>::kRing;
  constexpr uint32_t id_s = TcType<T>::idesc(kTcChunk, false), id_o = TcType<T>::idesc(HD, true);
  // low words of the descriptors of the first tile (the address field, in 16 bytes, never carries out of them)
  const uint64_t dq = sdesc_kmajor_sw128(smem_u32(s.q[0])), dk = sdesc_kmajor_sw128(smem_u32(s.ring[0])),
                 dv = sdesc_mnmajor_sw128(smem_u32(s.ring[0]), kTcChunk * 128);
  const uint32_t q_lo = static_cast<uint32_t>(dq), k_lo = static_cast<uint32_t>(dk), v_lo = static_cast<uint32_t>(dv);
  const uint32_t q_hi = static_cast<uint32_t>(dq >> 32), k_hi = static_cast<uint32_t>(dk >> 32),
                 v_hi = static_cast<uint32_t>(dv >> 32);
  auto desc = [](uint32_t lo, uint32_t hi) { return static_cast<uint64_t>(hi) << 32 | lo; };
  RingAt<NR> at;
  RingAt<kPagePieces> pat;
  uint32_t pieces = 0, nc0 = 0, nc1 = 0;  // pieces so far, chunks of each slot
  bool ok = true;
  {
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && (__all_sync(0xffffffffu, mbar_try_wait(bar, parity)) ||
                  __all_sync(0xffffffffu, page_wait_on(bar, parity, &s.abort, &s.busy)));
      tc_fence_after();
    };
    auto same = [](int x) { return static_cast<int>(__reduce_max_sync(0xffffffffu, static_cast<unsigned>(x))); };
    for (;; ++pat) {
      wait(&s.pfull[pat.i], pat.phase);
      if (!ok) break;
      const PagePiece& p = s.piece[pat.i];
      if (same(p.end)) break;
      const int n = same(p.chunks);
      const bool two = same(p.two);
      const SlotChunks c0{same(p.c[0].first), same(p.c[0].end), two ? 1 : 2},
          c1{same(p.c[1].first), same(p.c[1].end), two ? 1 : 2};
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.pfree[pat.i]);
      if (n == 0) continue;
      auto next_tile = [&] {  // the next tile of the ring, landed
        const uint32_t slot = at.i;
        wait(&s.full[slot], at.phase);
        ++at;
        return slot;
      };
      auto release = [&](uint32_t slot) {
        if (ok) tc_commit_warp(&s.empty[slot]);
      };
      auto mma_s = [&](int t, uint32_t slot) {  // S of slot t over the keys of a tile
        if (!ok) return;
        const uint32_t qa = q_lo + (two && t ? sizeof(s.q[0]) >> 4 : 0), ka = k_lo + slot * (TcSmem<HD, NB>::kTile >> 4);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * kTcRows * 128 + (kk & 3) * 32) >> 4;
          tc_mma_f16_warp(tmem + t * 256, desc(qa + off, q_hi), desc(ka + off, k_hi), id_s, kk > 0);
        }
        tc_commit_warp(&s.sfull[t]);
      };
      auto mma_o = [&](int t, uint32_t slot, int i, const SlotChunks& c) {  // O of slot t += P V of chunk i
        if (hold > 0 && i + 1 >= hold) ok = false;  // test hook: as if this thread's wait had run out
        const uint32_t phase = (t ? nc1++ : nc0++) & 1;
        const uint32_t va = v_lo + slot * (TcSmem<HD, NB>::kTile >> 4), first = i > c.first;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          wait(&s.pready[t][b], phase);
          if (!ok) return;
#pragma unroll
          for (int kk = b * kTcHalf / 16; kk < (b + 1) * kTcHalf / 16; ++kk)
            tc_mma_f16_ts_warp(tmem + t * 256 + 128, tmem + t * 256 + kk * 8, desc(va + (kk * 16 * 128 >> 4), v_hi), id_o,
                               kk > 0 ? 1u : first);
        }
        if (i + c.step >= c.end) tc_commit_warp(&s.ofull[t]);
      };
      wait(&s.qfull, pieces & 1);
      const uint32_t k0 = next_tile();
      if (two) {
        if (c0.has(0)) mma_s(0, k0);
        if (c1.has(0)) mma_s(1, k0);
        release(k0);
        if (n == 1 && ok) tc_commit_warp(&s.qempty);
        for (int i = 0; ok && i < n; ++i) {
          const bool more = i + 1 < n;
          const uint32_t k = more ? next_tile() : 0, v = next_tile();
          if (i == 0 && pieces > 0) wait(&s.ofree, (pieces - 1) & 1);
          if (c0.has(i)) mma_o(0, v, i, c0);
          if (more && c0.has(i + 1)) mma_s(0, k);
          if (c1.has(i)) mma_o(1, v, i, c1);
          if (more && c1.has(i + 1)) mma_s(1, k);
          release(v);
          if (more) release(k);
          if (i + 2 == n && ok) tc_commit_warp(&s.qempty);
        }
      } else {
        mma_s(0, k0);
        release(k0);
        if (n > 1) {
          const uint32_t k = next_tile();
          mma_s(1, k);
          release(k);
        }
        if (n <= 2 && ok) tc_commit_warp(&s.qempty);
        auto step = [&](int t, int i, const SlotChunks& c) {
          const uint32_t v = next_tile();
          if (i == 0 && pieces > 0) wait(&s.ofree, (pieces - 1) & 1);
          mma_o(t, v, i, c);
          release(v);
          if (i + 2 < n) {
            const uint32_t k = next_tile();
            mma_s(t, k);
            release(k);
            if (i + 3 == n && ok) tc_commit_warp(&s.qempty);
          }
        };
        for (int i = 0; ok && i < n; i += 2) {
          step(0, i, c0);
          if (ok && i + 1 < n) step(1, i + 1, c1);
        }
      }
      if (!ok) break;
      ++pieces;
    }
    if (!ok) *const_cast<volatile int*>(&s.abort) = 1;
    if (!ok || pieces > 0) {
      // MMAs in flight end before the CTA leaves, also when it is another role that gave up
      tc_commit_warp(&s.drain);
      mbar_wait(&s.drain, 0, nullptr);
    }
  }
}

// The rows: softmax of every chunk, then the outputs.  After a wait has run out the
// warps go on without waiting (their results are void), so that none is missing
// at a barrier of the 8.
template <class T, int HD, int NB>
__device__ __forceinline__ void run_rows(TcSmem<HD, NB>& s, const PagedAttnArgs& a, const PagedGeom& g, uint32_t tmem) {
  constexpr int NR = TcSmem<HD, NB>::kRing;
  constexpr int BR = kTcRows / NB, W = kTcChunk / NB;  // rows of a band, its keys of a chunk
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t = warp >> 2, tt = g.slot_tok;
  const int at = (warp & 3) * 32 + lane;           // this thread's lane of tensor memory,
  const int row = at % BR, col0 = at / BR * W;     // its row of the tile, and the band's first key
  const uint32_t ts = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);  // this warp's lanes, slot 0
  const uint32_t mine = ts + t * 256;
  auto warp_wait = [&](uint64_t* bar, uint32_t parity) {
    if (lane == 0) page_wait(bar, parity, &s.abort, &s.busy);
    __syncwarp();
    tc_fence_after();
  };
  uint32_t r = 0, ns = 0, no[2] = {0, 0};  // loads of the pieces before, chunks of this slot, pieces of both
  int cuts = 0, before0 = 0, before1 = 0;  // parts to be merged; thread 0: the parts of them that were there before
  RingAt<kPagePieces> pat;
  for (;; ++pat) {
    if (!piece_wait(&s.pfull[pat.i], pat.phase)) break;
    const PagePiece& p = s.piece[pat.i];
    if (p.end) break;
    const int n = p.chunks;
    const bool two = NB == 1 && p.two;
    const int tok0 = two ? t * tt : 0;
    const int rows = (two ? min(tt, p.nt - tok0) : p.nt) * a.group;  // live rows of this slot
    const int tok = p.t0 + tok0 + min(row, rows - 1) / a.group;
    const bool band = row - lane < rows;  // some row of the warp is live
    float m = -INFINITY, l = 0.f;
    if (n > 0) {
      const int first = p.c[t].first, end = p.c[t].end, step = p.c[t].step, lo = p.lo, hi = p.hi;
      RowKeys rk = row_keys(a, p.n, p.len, p.row0, tok);
      const int all_to = rk.bits != nullptr ? rk.ctx : rk.hi;  // every key from rk.lo to here is seen
      for (int i = first; i < end; i += step) {
        const int kb = (p.ca + i) * kTcChunk;
        warp_wait(&s.sfull[t], ns++ & 1);
        if (lo > kb || hi < kb + kTcChunk) {
          // keys of the chunk that no row of the tile sees (not loaded, or what the
          // page held before): p is 0 there, and so is V
          const int v = r + ring_v(i, n);
          warp_wait(&s.full[v % NR], (v / NR) & 1);
          const int z0 = max(lo - kb, 0), z1 = min(hi - kb, kTcChunk);  // keys seen: [z0, z1)
          // (16 bytes each, 64 columns of the keys after another)
          for (int c = at; c < kTcChunk * HD / 8; c += kTcRows) {
            const int key = c >> 3 & (kTcChunk - 1);
            if (key < z0 || key >= z1) *reinterpret_cast<uint4*>(s.ring[v % NR] + c * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
        }
        // (32 columns at a time, the next ones under way; the loops are kept small: a
        // call of a few microseconds runs its code cold)
        uint32_t x[2][32], z[32];
        float2 base, sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        float cm = -INFINITY;
        if (NB > 1 && band) {
          // this band's keys; the others' probabilities are zeros in its rows
#pragma unroll
          for (int u = 0; u < W / 32; ++u) tmem_ld32_start(mine + col0 + 32 * u, x[u]);
#pragma unroll
          for (int u = 0; u < W / 32; ++u) tmem_wait32(x[u]);
          uint32_t zero[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) zero[j] = 0;
#pragma unroll
          for (int c = 0; c < kTcChunk; c += 32)
            if (c < col0 || c >= col0 + W) tmem_st16(mine + c / 2, zero);
          if (__any_sync(0xffffffffu, rk.lo > kb + col0 || kb + col0 + W > all_to)) {
            rk = row_keys(a, p.n, p.len, p.row0, tok);
#pragma unroll
            for (int u = 0; u < W / 32; ++u) {
              const uint32_t see = key_bits(rk, kb + col0 + 32 * u);
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(see >> j & 1)) x[u][j] = 0xff800000u;
            }
          }
          float m2[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int u = 0; u < W / 32; ++u)
#pragma unroll
            for (int j = 0; j < 32; j += 2)
              m2[j >> 1 & 1] = fmaxf(m2[j >> 1 & 1], fmaxf(__uint_as_float(x[u][j]), __uint_as_float(x[u][j + 1])));
          cm = fmaxf(m2[0], m2[1]) * a.scale_log2;
        }
        if (NB == 1 && band) {
          if (__any_sync(0xffffffffu, rk.lo > kb || kb + kTcChunk > all_to)) {
            // some row does not see every key: what it does not see becomes -inf
            rk = row_keys(a, p.n, p.len, p.row0, tok);
#pragma unroll 1
            for (int c = 0; c < kTcChunk; c += 32) {
              tmem_ld32_start(mine + c, x[0]);
              const uint32_t see = key_bits(rk, kb + c);
              tmem_wait32(x[0]);
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(see >> j & 1)) x[0][j] = 0xff800000u;
              tmem_st32(mine + c, x[0]);
            }
            tmem_st_wait();
          }
          float m2[2] = {-INFINITY, -INFINITY};
          tmem_ld32_start(mine, x[0]);
#pragma unroll 1
          for (int c = 0; c < kTcChunk; c += 64) {
            tmem_wait32(x[0]);
            tmem_ld32_start(mine + c + 32, x[1]);
#pragma unroll
            for (int j = 0; j < 32; j += 4)
#pragma unroll
              for (int u = 0; u < 2; ++u)
                m2[u] = fmaxf(m2[u], fmaxf(__uint_as_float(x[0][j + 2 * u]), __uint_as_float(x[0][j + 2 * u + 1])));
            tmem_wait32(x[1]);
            tmem_ld32_start(mine + (c + 64 & 127), x[0]);  // (at the end: the first columns again, for the next loop)
#pragma unroll
            for (int j = 0; j < 32; j += 4)
#pragma unroll
              for (int u = 0; u < 2; ++u)
                m2[u] = fmaxf(m2[u], fmaxf(__uint_as_float(x[1][j + 2 * u]), __uint_as_float(x[1][j + 2 * u + 1])));
          }
          cm = fmaxf(m2[0], m2[1]) * a.scale_log2;
        }
        if (band) {
          if (i == first) {
            m = cm;
          } else {
            const bool grow = cm > m + kPageSlack || (m == -INFINITY && cm > m);
            if (__any_sync(0xffffffffu, grow)) {
              // (the P V before is done: this S was issued after it)
              const float nm = grow ? cm : m;
              const float f = grow ? ex2_ftz(m - nm) : 1.f;
              l *= f;
              m = nm;
#pragma unroll 1
              for (int d = 0; d < HD; d += 32) {
                uint32_t(&y)[32] = NB == 1 ? x[1] : z;
                tmem_ld32_start(mine + 128 + d, y);
                tmem_wait32(y);
#pragma unroll
                for (int j = 0; j < 32; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * f);
                tmem_st32(mine + 128 + d, y);
              }
            }
          }
          const float nm = m == -INFINITY ? 0.f : Pack16<T>::kTop - m;
          base = make_float2(nm, nm);
        }
        const float2 scale = make_float2(a.scale_log2, a.scale_log2);
        auto probabilities = [&](uint32_t (&v)[32], int c) {  // columns c .. c + 31 into columns c / 2 ..
          uint32_t pk[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float2 e = fma2(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), scale, base);
            e.x = ex2_ftz(e.x);
            e.y = ex2_ftz(e.y);
            sum[j & 1] = add2(sum[j & 1], e);
            pk[j] = Pack16<T>::pack(e.x, e.y);
          }
          tmem_st16(mine + c / 2, pk);
        };
        if constexpr (NB > 1) {
          if (band) {
#pragma unroll
            for (int u = 0; u < W / 32; ++u) probabilities(x[u], col0 + 32 * u);
            tmem_st_wait();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.pready[t][0]), mbar_arrive(&s.pready[t][1]);
        }
#pragma unroll 1
        for (int b = NB == 1 ? 0 : 2; b < 2; ++b) {
          if (band) {
            tmem_wait32(x[0]);
            tmem_ld32_start(mine + b * kTcHalf + 32, x[1]);
            probabilities(x[0], b * kTcHalf);
            tmem_wait32(x[1]);
            if (b == 0) tmem_ld32_start(mine + kTcHalf, x[0]);
            probabilities(x[1], b * kTcHalf + 32);
            tmem_st_wait();
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.pready[t][b]);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      }
      m = share_max(m, l);
    }
    const bool whole = p.whole;
    // a part: [HD / 4][rows][4], so that the rows' threads write and read side by side
    const int part_rows = rows_of_part<TcSmem<HD, NB>>(a, p);
    float4* part = part_of<TcSmem<HD, NB>, HD>(a, p.slot);
    float2* part_ml = part_ml_of<TcSmem<HD, NB>>(a, p.slot);
    const int head = p.h * a.group + row % a.group;
    // 16 columns of a row from column d: a result, or a part of one
    auto store16 = [&](const float (&o)[16], int rr, int d, float scale, bool live) {
      if (!live) return false;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          part[(d / 4 + j) * part_rows + rr] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        return false;
      }
      T* out = static_cast<T*>(a.out) + static_cast<long long>(p.row0 + tok) * a.out_row + head * a.out_head + d;
      return write16(out, o, scale);
    };
    if (two) {
      const bool has = p.c[t].any();
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
        if (whole) store_lse<T>(a, p, tok, head, m, l);
        else part_ml[t * kTcRows + row] = make_float2(m, l);
      }
      if (whole)
        for (unsigned redo_rows = __ballot_sync(0xffffffffu, bad); redo_rows; redo_rows &= redo_rows - 1)
          redo<T, HD>(s, a, p, tt, t * kTcRows + (warp & 3) * 32 + __ffs(redo_rows) - 1);
    } else if constexpr (NB > 1) {
      // each band of each slot holds these rows over some of the keys: the bands' sums
      // of the slots meet in shared memory (s.q[1], which tiles of one slot's rows leave
      // free), half of the columns at a time
      constexpr int CW = HD / 2;
      static_assert(sizeof(s.q[1]) >= kTcRows * CW * 4, "columns of all bands");
      s.ml[t][at] = make_float2(m, l);
      all_rows<TcSmem<HD, NB>>();
      float mm = -INFINITY, ll = 0.f;
#pragma unroll
      for (int u = 0; u < 2 * NB; ++u) mm = fmaxf(mm, s.ml[u & 1][(u >> 1) * BR + row].x);
#pragma unroll
      for (int u = 0; u < 2 * NB; ++u) {
        const float2 o = s.ml[u & 1][(u >> 1) * BR + row];
        if (o.x != -INFINITY) ll = fmaf(o.y, ex2_ftz(o.x - mm), ll);
      }
      const float m0 = s.ml[0][at].x, m1 = s.ml[1][at].x;
      for (int u = 0; u < 2; ++u)
        if (p.c[u].any()) warp_wait(&s.ofull[u], no[u] & 1);
      const bool use0 = m0 != -INFINITY, use1 = m1 != -INFINITY;
      const float f0 = use0 ? ex2_ftz(m0 - mm) : 0.f, f1 = use1 ? ex2_ftz(m1 - mm) : 0.f;
      const float scale = ll != 0.f ? 1.f / ll : 0.f;
      const bool live = row < rows;
      float4* sum = reinterpret_cast<float4*>(s.q[1]);  // [band][CW / 4][row]
      bool bad = false;
#pragma unroll 1
      for (int d = 0; d < HD; d += CW) {
        if (band) {
#pragma unroll 1
          for (int c = t * (CW / 2); c < (t + 1) * (CW / 2); c += 16) {
            float o[16], o1[16];
            // (what a slot without keys holds is not used)
            tmem_ld16x2(ts + 128 + d + c, ts + 256 + 128 + d + c, o, o1);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = (use0 ? o[j] * f0 : 0.f) + (use1 ? o1[j] * f1 : 0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              sum[(at / BR * (CW / 4) + c / 4 + j) * BR + row] =
                  make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
          }
        }
        all_rows<TcSmem<HD, NB>>();
        if (tid < CW / 16 * BR && live) {
          const int c = tid / BR * 16;
          float o[16];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float4 y = sum[(c / 4 + j) * BR + row];
#pragma unroll
            for (int b = 1; b < NB; ++b) {
              const float4 w = sum[(b * (CW / 4) + c / 4 + j) * BR + row];
              y = make_float4(y.x + w.x, y.y + w.y, y.z + w.z, y.w + w.w);
            }
            o[4 * j] = y.x, o[4 * j + 1] = y.y, o[4 * j + 2] = y.z, o[4 * j + 3] = y.w;
          }
          bad |= store16(o, row, d + c, scale, live);
        }
        all_rows<TcSmem<HD, NB>>();
      }
      if (live && tid < BR) {
        if (whole) store_lse<T>(a, p, tok, head, mm, ll);
        else part_ml[row] = make_float2(share_max(mm, ll), ll);
      }
      if (bad) atomicOr(&s.bad[row >> 5], 1u << (row & 31));
    } else {
      // both slots hold these rows, each over half of the keys; slot t's warps finish
      // the t-th half of the columns
      s.ml[t][row] = make_float2(m, l);
      all_rows<TcSmem<HD, NB>>();
      const float2 ml0 = s.ml[0][row], ml1 = s.ml[1][row];
      bool has[2];
      for (int u = 0; u < 2; ++u) {
        has[u] = p.c[u].any();
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
          tmem_ld16x2(ts + 128 + d, ts + 256 + 128 + d, o, o1);  // (what a slot without keys holds is not used)
#pragma unroll
          for (int j = 0; j < 16; ++j) o[j] = (use0 ? o[j] * f0 : 0.f) + (use1 ? o1[j] * f1 : 0.f);
          bad |= store16(o, row, d, scale, live);
        }
      }
      if (live && t == 0) {
        if (whole) store_lse<T>(a, p, tok, head, mm, ll);
        else part_ml[row] = make_float2(share_max(mm, ll), ll);
      }
      if (bad) atomicOr(&s.bad[row >> 5], 1u << (row & 31));
    }
    if (n > 0) {  // the accumulators may be overwritten
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.ofree);
      r += 2 * n;
      for (int u = 0; u < 2; ++u) no[u] += p.c[u].any();
    }
    if (!whole) {
      const int before = arrive_part<TcSmem<HD, NB>>(a, p);
      // nothing waits for the counter's answer here: whether this CTA has to merge the
      // tile is seen to after the run (whose first and last pieces may be parts)
      (cuts == 0 ? before0 : before1) = before;
      if (tid < sizeof(PagePiece) / 4) reinterpret_cast<int*>(&s.cut[cuts])[tid] = reinterpret_cast<const int*>(&p)[tid];
      ++cuts;
    } else if (!two) {
      all_rows<TcSmem<HD, NB>>();  // (s.ml is free again)
      redo_bad<T, HD>(s, a, p, tt);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.pempty[pat.i]);
  }
#pragma unroll 1
  for (int k = cuts - 1; k >= 0; --k) finish_cut<T, HD>(s, a, s.cut[k], tt, k == 0 ? before0 : before1);
}

template <class T, int HD, int NB>
__global__ void __launch_bounds__(kTcThreads, 1)
    paged_attn_tc_kernel(const __grid_constant__ PagedMaps m, const __grid_constant__ PagedAttnArgs a, const PagedGeom g,
                         const int hold) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  TcSmem<HD, NB>& s = *reinterpret_cast<TcSmem<HD, NB>*>(smem_raw);
  if (smem_u32(smem_raw) & 1023u) {  // (the swizzle's atoms; shared memory starts on one)
    pdl_wait();
    if (threadIdx.x == 0) atomicOr(a.err, DERR_SHAPE);
    return;
  }
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < TcSmem<HD, NB>::kRing; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    mbar_init(&s.qfull, 1);
    mbar_init(&s.qempty, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&s.sfull[t], 1);
      mbar_init(&s.pready[t][0], 4);
      mbar_init(&s.pready[t][1], 4);
      mbar_init(&s.ofull[t], 1);
    }
    for (int i = 0; i < kPagePieces; ++i) {
      mbar_init(&s.pfull[i], 1);
      mbar_init(&s.pempty[i], 8);
      mbar_init(&s.pfree[i], 1);
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
  if (threadIdx.x == kTcThreads - 1) {
    tma_prefetch_desc(&m.q);
    tma_prefetch_desc(&m.k);
    tma_prefetch_desc(&m.v);
  }
  pdl_launch_dependents();
  pdl_wait();  // (nothing of the calls before is read above)
  if (a.batch > kWarpRequests) run_start_block(a, g, &s.run, reinterpret_cast<unsigned*>(s.ml));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  if (warp == 8) issue_mmas<T, HD, NB>(s, tmem, hold);
  else if (warp == 9) issue_loads<HD>(s, a, g, m, 0);
  else run_rows<T, HD, NB>(s, a, g, tmem);
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && s.abort) atomicOr(a.err, DERR_TIMEOUT);
  if (warp == 8) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <class T, int HD, int NB>
cudaError_t launch_tc(const PagedMaps& m, const PagedAttnArgs& a, int hold, int grid, cudaStream_t s) {
  const int tt = kTcRows / NB / a.group;
  // Tiles of 256 rows read K and V once for twice the rows (2048 tokens after 4096, 32
  // heads: 165 us, 170 with tiles of 128); with fewer of them than CTAs their keys
  // would have to be cut and their rows merged, so they are halved instead (4 requests of 61
  // tokens, 32 heads on 8, 700 to 1100 keys: 17.6 us, 34 with tiles of 256).
  const long long per_request = (static_cast<long long>(a.rows) + a.batch - 1) / a.batch;
  const bool two = NB == 1 && per_request > tt && (per_request + 2 * tt - 1) / (2 * tt) * a.batch * a.Hkv >= grid;
  const PagedGeom g{two ? 2 * tt : tt, tt, kTcShift, 2, 8, 8};
  return launch_after(paged_attn_tc_kernel<T, HD, NB>, dim3(grid), kTcThreads, sizeof(TcSmem<HD, NB>), s, m, a, g, hold);
}

template <class T, int HD>
cudaError_t launch_bands(const PagedMaps& m, const PagedAttnArgs& a, int bands, int hold, int grid, cudaStream_t s) {
  return bands == 4   ? launch_tc<T, HD, 4>(m, a, hold, grid, s)
         : bands == 2 ? launch_tc<T, HD, 2>(m, a, hold, grid, s)
                      : launch_tc<T, HD, 1>(m, a, hold, grid, s);
}

template <class T, int HD, int NB>
cudaError_t attr() {
  return cudaFuncSetAttribute(paged_attn_tc_kernel<T, HD, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              sizeof(TcSmem<HD, NB>));
}
template <class T, int HD>
cudaError_t attrs() {
  cudaError_t e = attr<T, HD, 1>();
  if (e == cudaSuccess) e = attr<T, HD, 2>();
  return e == cudaSuccess ? attr<T, HD, 4>() : e;
}

}  // namespace

cudaError_t paged_attention_tc_set_attributes() {
  cudaError_t e = attrs<__half, 64>();
  if (e == cudaSuccess) e = attrs<__half, 128>();
  if (e == cudaSuccess) e = attrs<__nv_bfloat16, 64>();
  return e == cudaSuccess ? attrs<__nv_bfloat16, 128>() : e;
}

bool paged_pool_map(CUtensorMap* m, const void* pool, const cllm_paged_desc& d, int keys) {
  const cuuint64_t dims[5] = {static_cast<cuuint64_t>(d.head_dim), static_cast<cuuint64_t>(d.page_size),
                              static_cast<cuuint64_t>(d.n_kv_heads), static_cast<cuuint64_t>(d.n_pages),
                              static_cast<cuuint64_t>(d.layers)};
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(d.stride_pos) * 2, static_cast<cuuint64_t>(d.stride_head) * 2,
                                 static_cast<cuuint64_t>(d.stride_page) * 2, static_cast<cuuint64_t>(d.stride_layer) * 2};
  const cuuint32_t box[5] = {64, static_cast<cuuint32_t>(d.page_size < keys ? d.page_size : keys), 1, 1, 1};
  return make_map_nd(m, d.dtype == CLLM_BF16, pool, 5, dims, strides, box);
}

bool paged_query_map(CUtensorMap* m, const PagedAttnArgs& a, int dtype, int hd, int rows) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(hd), static_cast<cuuint64_t>(a.H), static_cast<cuuint64_t>(a.rows)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(a.q_head) * 2, static_cast<cuuint64_t>(a.q_row) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(a.group), static_cast<cuuint32_t>(rows / a.group)};
  return make_map_nd(m, dtype == CLLM_BF16, a.q, 3, dims, strides, box);
}

cudaError_t launch_paged_attention_tc(const PagedAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int dtype,
                                      int hd, int hold, int grid, cudaStream_t s) {
  PagedMaps m;
  m.k = k;
  m.v = v;
  // rows of one key/value head in an average request
  const long long rows = (static_cast<long long>(a.rows) + a.batch - 1) / a.batch * a.group;
  // (measured with more bands and with one: 8 requests of 32 tokens and 600 keys, 32 heads,
  // 20.0 and 22.8 us; 16 of 6 tokens and 1000 keys, 32 heads on 8, 14.7 and 16.7 us; 4 of 64
  // tokens and 500 keys, 32 heads, 2 bands, 12.8 and 13.8 us)
  const int bands = rows <= 32 && a.group <= 32 ? 4 : rows <= 64 ? 2 : 1;
  if (!paged_query_map(&m.q, a, dtype, hd, kTcRows / bands)) return cudaErrorInvalidValue;
  if (dtype == CLLM_BF16)
    return hd == 64 ? launch_bands<__nv_bfloat16, 64>(m, a, bands, hold, grid, s)
                    : launch_bands<__nv_bfloat16, 128>(m, a, bands, hold, grid, s);
  return hd == 64 ? launch_bands<__half, 64>(m, a, bands, hold, grid, s)
                  : launch_bands<__half, 128>(m, a, bands, hold, grid, s);
}

}  // namespace cllm
