// What the paged attention kernels of 16-bit pools share: the loading warp, which walks the
// CTA's run of work and streams queries, keys and values by TMA, the bounded waits,
// and a tile's end: results, parts of cut tiles and their merging.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"
#include "paged_walk.cuh"
#include "ptx.cuh"

namespace cllm {

// A row's running maximum follows only growth of more than this (in log2): P may
// then reach 2^8, and O is rarely rescaled.
constexpr float kPageSlack = 8.f;

// The chunks of a piece that a slot works on (relative to the piece): first .. end - 1 without [hole,
// resume), which first keys have before them (hole 0: none left out), or every other one (hole -1).
struct SlotChunks {
  int first, end, hole, resume;
  __device__ bool any() const { return first < end; }
  __device__ bool has(int i) const {
    return i >= first && i < end && (hole < 0 ? ((i - first) & 1) == 0 : i < hole || i >= resume);
  }
  __device__ int next(int i) const { return hole < 0 ? i + 2 : i + 1 == hole ? resume : i + 1; }
};

// A piece as the loading warp hands it to the others.
struct PagePiece {
  int b, h, t0, n, len, row0;              // as in Piece
  TileKeys keys;
  int near, gap;
  int ca, chunks;                          // first chunk and number of chunks (0: no keys)
  short nt, two, whole, end;               // tokens; 128 rows in each slot; the whole tile; no piece: the run is over
  int slot, cta0, cta1, first_slot;        // of a cut tile: this part's slot, the CTAs of its parts, the first's slot
  SlotChunks c[2];
  __device__ int chunk(int i) const { return ca + i - (ca + i < near ? gap : 0); }  // where in the request its i-th is
  __device__ int part(int cta) const { return cta == cta0 ? first_slot : 2 * cta; }
};
constexpr int kPagePieces = 4;

struct PagedMaps {
  CUtensorMap q, k, v;
};

// mbar_wait, but time in which a warp redoes rows (busy) does not count, and once
// a wait has run out the others end at once.
static __device__ __noinline__ bool page_wait_on(uint64_t* bar, uint32_t parity, volatile int* abort,
                                                 volatile int* busy) {
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
__device__ __forceinline__ bool page_wait(uint64_t* bar, uint32_t parity, volatile int* abort, volatile int* busy) {
  return mbar_try_wait(bar, parity) || page_wait_on(bar, parity, abort, busy);
}

// A row warp's wait for its next piece.  The loading warp always brings one (an end,
// after a wait of its own has run out), and the row warps have to agree on it: they take no
// notice of the other roles' failures here, and the limit is past all of theirs.
__device__ __forceinline__ bool piece_wait(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t it = 0; !mbar_try_wait(bar, parity); ++it)
    if ((it & 63u) == 63u && globaltimer_ns() - t0 > 8 * kWaitBudgetNs) return false;
  return true;
}

// A position of a ring and the phase of its barriers.
template <int N>
struct RingAt {
  uint32_t i = 0, phase = 0;
  __device__ void operator++() {
    if (++i == N) i = 0, phase ^= 1;
  }
};

// Two fp32 values to 16 bits each.  kTop: log2 of P at its row's running maximum.  A row's l
// and O hold 2^kTop times their values, in every share of its keys, and the quotient does not.
// fp16 has room above (P reaches 2^(7 + 8) at most) and little below: P is a normal number from
// 2^-21 of the largest on, and lost below 2^-32 of it, which a context of 2^17 equally small
// probabilities feels as 2^-15 of V's size (with kTop 0: 2^-8).
template <class T> struct Pack16;
template <> struct Pack16<__half> {
  static constexpr float kTop = 7.f;
  static __device__ uint32_t pack(float a, float b) { return pack_f16x2(a, b); }
};
template <> struct Pack16<__nv_bfloat16> {
  static constexpr float kTop = 0.f;
  static __device__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
};

// Walk the CTA's run, hand each piece to the other warps, and load its queries, keys and
// values.
// S::kShift: log2 of the keys of a tile; S::kAhead: K one tile ahead of V (K0 K1 V0 K2 V1
// ..), else K0 V0 K1 V1 ..; S::kIssuer: a warp beside the row warps takes the pieces too;
// S::kBands: copies of a tile's queries.  Of K the pages that hold keys of the tile are loaded; V's other
// places get zeros (a page outside the map), since p = 0 times what was there may not be 0.  Keys
// in the loaded pages that no row sees, before hi, are the request's own: where one of them is not
// finite, the row is done again.  hold: test hook, 1 + the chunk of a
// piece at which this warp gives up (0: none).
template <int HD, class S>
__device__ __forceinline__ void issue_loads(S& s, const PagedAttnArgs& a, const PagedGeom& g, const PagedMaps& m,
                                            int hold) {
  constexpr int NH = HD / 64, NR = S::kRing, kChunk = 1 << S::kShift;
  const int lane = threadIdx.x & 31, tt = g.slot_tok, P = 1 << a.page_shift;
  const int box_shift = min(a.page_shift, S::kShift), box = 1 << box_shift;
  const int j = lane / NH, half = lane % NH;  // this lane's box of a tile and its 64 columns (at most 16 boxes)
  RingAt<NR> at;
  RingAt<kPagePieces> pat;
  uint32_t r = 0, pieces = 0, with_keys = 0;  // loads, pieces, pieces with keys so far
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    ok = ok && page_wait(bar, parity, &s.abort, &s.busy);
    ok = __all_sync(0xffffffffu, ok);
  };
  if (a.batch <= kWarpRequests) run_start_warp(a, g, &s.run);
  PagedWalk w;
  w.begin(s.run);
  for (;;) {
    Piece p;
    const bool more = w.next(a, g, p);
    if (pieces >= kPagePieces) {
      wait(&s.pempty[pat.i], pat.phase ^ 1);
      if constexpr (S::kIssuer) wait(&s.pfree[pat.i], pat.phase ^ 1);
    }
    if (!ok) break;
    ++pieces;
    auto hand_out = [&] {
      if (lane == 0) {
        PagePiece& o = s.piece[pat.i];
        o.end = !more;
        if (more) {
          o.b = p.b, o.h = p.h, o.t0 = p.t0, o.nt = p.nt, o.n = p.n, o.len = p.len, o.row0 = p.row0;
          o.keys = p.keys;
          o.near = p.near, o.gap = p.gap;
          o.ca = p.ca, o.chunks = p.cb - p.ca;
          o.two = p.nt > tt, o.whole = p.whole();
          if (!p.whole()) {
            o.slot = w.slot(p, blockIdx.x);
            o.cta0 = w.first_cta(p), o.cta1 = w.last_cta(p);
            o.first_slot = w.slot(p, o.cta0);
          }
          for (int t = 0; t < 2; ++t) {
            if (!o.two) {
              o.c[t] = {t, o.chunks, -1, 0};
              continue;
            }
            const int t0 = p.t0 + t * tt;
            const TileKeys k = tile_keys(a, p.n, p.len, t0, min(p.t0 + p.nt, t0 + tt));
            // the piece's chunks of first keys, and where the slot's window begins after them
            const int sinks = min(max(p.tca + (k.sink + kChunk - 1) / kChunk - p.ca, 0), o.chunks);
            const int from = max(k.lo / kChunk - p.ca, sinks);
            int end = min(o.chunks, (k.hi + kChunk - 1) / kChunk - p.ca);
            const bool hole = sinks > 0 && from > sinks && from < end;
            if (sinks > 0 && from >= end) end = min(end, sinks);
            o.c[t] = {sinks > 0 ? 0 : from, end, hole ? sinks : 0, hole ? from : 0};
          }
        }
        mbar_arrive(&s.pfull[pat.i]);
      }
      __syncwarp();
      ++pat;
    };
    if (!more || p.empty()) {
      hand_out();
      if (!more) break;
      continue;
    }
    const int n = p.cb - p.ca;
    // this lane's page of a chunk (its box's; the pages that hold keys of the tile are loaded)
    auto page_of = [&](int c) {
      const int pos = p.chunk(c) * kChunk + (j << box_shift);
      return pos < p.keys.hi ? a.table[static_cast<size_t>(p.b) * a.table_width + (pos >> a.page_shift)] : 0;
    };
    auto tile = [&](const CUtensorMap* map, int c, int page) {
      const int kb = p.chunk(c) * kChunk, pos = kb + (j << box_shift);
      if (r >= NR) wait(&s.empty[at.i], at.phase ^ 1);
      if (!ok) return;
      const bool seen = p.keys.some(pos, pos + box), mine = pos < kb + kChunk && (seen || map == &m.v);
      const int boxes = __popc(__ballot_sync(0xffffffffu, mine));  // (of 64 columns)
      if (lane == 0) mbar_arrive_expect_tx(&s.full[at.i], boxes * box * 128);
      __syncwarp();
      if (mine) {
        if (!seen) page = a.n_pages;
        else if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.n_pages)) {
          atomicOr(a.err, DERR_CAPACITY);
          page = a.n_pages;  // outside the map: reads as zeros
        }
        tma_load_5d(s.ring[at.i] + half * kChunk * 128 + (j << box_shift) * 128, map, &s.full[at.i], half * 64,
                    pos & (P - 1), p.h, page, a.layer);
      }
      ++r;
      ++at;
    };
    int page = page_of(p.ca);
    if (with_keys > 0) wait(&s.qempty, (with_keys - 1) & 1);
    if (!ok) break;
    // the queries: 128 rows to each slot, or in each of the bands
    const int copies = p.nt > tt ? 2 : S::kBands;
    if (lane == 0) mbar_arrive_expect_tx(&s.qfull, copies * NH * tt * a.group * 128);
    __syncwarp();
    if (lane < copies * NH) {
      const int c = lane / NH;
      uint8_t* to = S::kBands > 1 ? s.q[0] + c * (S::kRows / S::kBands) * 128 : s.q[c];
      tma_load_3d(to + lane % NH * S::kRows * 128, &m.q, &s.qfull, lane % NH * 64, p.h * a.group,
                  p.row0 + p.t0 + (S::kBands > 1 ? 0 : c * tt));
    }
    ++with_keys;
    tile(&m.k, p.ca, page);
    hand_out();  // (the first keys are on their way)
    for (int i = 0; ok && i < n; ++i) {
      if (hold > 0 && i + 1 >= hold) ok = false;
      const int next = ok && i + 1 < n ? page_of(p.ca + i + 1) : 0;
      if (ok && S::kAhead && i + 1 < n) tile(&m.k, p.ca + i + 1, next);
      if (ok) tile(&m.v, p.ca + i, page);
      if (ok && !S::kAhead && i + 1 < n) tile(&m.k, p.ca + i + 1, next);
      page = next;
    }
    if (!ok) break;
  }
  if (lane == 0) {
    if (!ok) {
      // the rows get their end (they go on past every wait now)
      *const_cast<volatile int*>(&s.abort) = 1;
      if (pieces >= kPagePieces) mbar_wait(&s.pempty[pat.i], pat.phase ^ 1, nullptr);
      s.piece[pat.i].end = 1;
      mbar_arrive(&s.pfull[pat.i]);
    }
    // Loads in flight land before the CTA leaves, also when it is another role that gave up
    // after the last one was issued here.
    for (uint32_t i = r > NR ? r - NR : 0; i < r; ++i) mbar_wait(&s.full[i % NR], (i / NR) & 1, nullptr);
    if (with_keys > 0) mbar_wait(&s.qfull, (with_keys - 1) & 1, nullptr);
  }
}

// ---- a tile's end --------------------------------------------------------------------

// The row warps (S::kRowWarps of them).
template <class S>
__device__ __forceinline__ void all_rows() {
  named_bar_sync(1, 32 * S::kRowWarps);
}

// 16 columns of a result (scale: 1 over the row's sum); whether one is not finite though the sum is.
template <class T>
__device__ __forceinline__ bool write16(T* out, const float (&o)[16], float scale) {
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 16; j += 8) {
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = scale != 0.f ? o[j + 2 * e] * scale : 0.f, y = scale != 0.f ? o[j + 2 * e + 1] * scale : 0.f;
      bad |= !isfinite(x) || !isfinite(y);
      u[e] = Pack16<T>::pack(x, y);
    }
    *reinterpret_cast<uint4*>(out + j) = make_uint4(u[0], u[1], u[2], u[3]);
  }
  return bad && scale == scale;
}

template <class T>
__device__ __forceinline__ void store_lse(const PagedAttnArgs& a, const PagePiece& p, int tok, int head, float m,
                                          float l) {
  if (a.lse == nullptr) return;
  a.lse[static_cast<size_t>(p.row0 + tok) * a.H + head] =
      l != 0.f ? (m + log2f(l * (1.f / (1 << static_cast<int>(Pack16<T>::kTop))))) * 0.69314718055994530942f : -INFINITY;
}

// Row rr of a tile from the definition (the whole warp).
template <class T, int HD, class S>
__device__ __forceinline__ void redo(S& s, const PagedAttnArgs& a, const PagePiece& p, int tt, int rr) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  if (lane == 0) atomicAdd(&s.busy, 1);
  exact_row<T, HD>(a, p.b, p.h, p.n, p.len, p.row0, p.t0 + (p.two ? rr / 128 * tt : 0) + (rr % 128) / a.group,
                   p.h * a.group + (rr % 128) % a.group);
  if (lane == 0) atomicAdd(&s.busy, -1);
}

// Rows marked in s.bad (marked by any warp, so after a barrier of all; the next mark comes after another).
template <class T, int HD, class S>
__device__ __forceinline__ void redo_bad(S& s, const PagedAttnArgs& a, const PagePiece& p, int tt) {
  const int tid = threadIdx.x, warp = tid >> 5;
  unsigned any = 0;
  for (int i = 0; i < 8; ++i) any |= s.bad[i];
  if (!any) return;
  for (int rr = warp; rr < 256; rr += S::kRowWarps)
    if (s.bad[rr >> 5] >> (rr & 31) & 1) redo<T, HD>(s, a, p, tt, rr);
  all_rows<S>();
  if (tid < 8) s.bad[tid] = 0;
  all_rows<S>();
}

// A part of a tile that is cut: [HD / 4][rows][4] floats and a row's (maximum, sum), in
// slots of S::kPartRows rows; the rows' threads write and read side by side.
template <class S>
__device__ __forceinline__ int rows_of_part(const PagedAttnArgs& a, const PagePiece& p) {
  return p.two ? S::kPartRows : (p.nt * a.group + 31) & ~31;
}
template <class S, int HD>
__device__ __forceinline__ float4* part_of(const PagedAttnArgs& a, int slot) {
  return reinterpret_cast<float4*>(a.part_o) + static_cast<size_t>(slot) * (S::kPartRows * HD / 4);
}
template <class S>
__device__ __forceinline__ float2* part_ml_of(const PagedAttnArgs& a, int slot) {
  return a.part_ml + static_cast<size_t>(slot) * S::kPartRows;
}

// Merge group `group` of a tile's rows from its parts, in order: 16 columns of a row to a
// thread, or to `ways` neighbouring lanes that share the parts; the loads of 4 parts are
// under way together.
__device__ __forceinline__ int merge_ways(int parts) { return parts >= 8 ? 4 : 1; }
template <class S, int HD>
__device__ __forceinline__ int merge_rows(int ways) {  // rows of a group
  return 32 * S::kRowWarps / (HD / 16) / ways;
}
template <class T, int HD, class S>
__device__ __forceinline__ void merge_group(S& s, const PagedAttnArgs& a, const PagePiece& p, int tt, int group,
                                            int ways) {
  const int rows = merge_rows<S, HD>(ways), tid = threadIdx.x, sub = tid & (ways - 1), it = tid / ways;
  const int k = group * rows + (it & (rows - 1)), d = it / rows * 16, live = p.nt * a.group;
  const int part_rows = rows_of_part<S>(a, p);
  const int kk = min(k, live - 1), rr = p.two && kk >= tt * a.group ? 128 + kk - tt * a.group : kk;
  float mm = -INFINITY, ll = 0.f, o[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) o[j] = 0.f;
#pragma unroll 1
  for (int c = p.cta0 + sub; c <= p.cta1; c += 4 * ways) {
    float4 y[4][4];
    float2 ml[4];
    float nm = mm;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      ml[u] = make_float2(-INFINITY, 0.f);
      if (c + u * ways > p.cta1) continue;
      const int part = p.part(c + u * ways);
      ml[u] = __ldcg(part_ml_of<S>(a, part) + rr);
      const float4* from = part_of<S, HD>(a, part) + d / 4 * part_rows + rr;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[u][j] = __ldcg(from + j * part_rows);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) nm = fmaxf(nm, ml[u].x);
    const float f = mm != -INFINITY ? ex2_ftz(mm - nm) : 0.f;
    mm = nm;
    ll *= f;
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] *= f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (ml[u].x == -INFINITY) continue;  // (none of its keys is seen)
      const float w = ex2_ftz(ml[u].x - mm);
      ll = fmaf(ml[u].y, w, ll);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o[4 * j] = fmaf(y[u][j].x, w, o[4 * j]);
        o[4 * j + 1] = fmaf(y[u][j].y, w, o[4 * j + 1]);
        o[4 * j + 2] = fmaf(y[u][j].z, w, o[4 * j + 2]);
        o[4 * j + 3] = fmaf(y[u][j].w, w, o[4 * j + 3]);
      }
    }
  }
  for (int w = 1; w < ways; w <<= 1) {
    const float m1 = __shfl_xor_sync(0xffffffffu, mm, w), l1 = __shfl_xor_sync(0xffffffffu, ll, w), nm = fmaxf(mm, m1);
    const float f0 = mm != -INFINITY ? ex2_ftz(mm - nm) : 0.f, f1 = m1 != -INFINITY ? ex2_ftz(m1 - nm) : 0.f;
    mm = nm;
    ll = ll * f0 + l1 * f1;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float o1 = __shfl_xor_sync(0xffffffffu, o[j], w);
      o[j] = (f0 != 0.f ? o[j] * f0 : 0.f) + (f1 != 0.f ? o1 * f1 : 0.f);
    }
  }
  if (sub == 0 && k < live) {
    const int kt = k * a.group_inv >> 16, head = p.h * a.group + k - kt * a.group;
    T* out = static_cast<T*>(a.out) + static_cast<long long>(p.row0 + p.t0 + kt) * a.out_row +
             static_cast<long long>(head) * a.out_head + d;
    if (write16(out, o, ll != 0.f ? 1.f / ll : 0.f)) atomicOr(&s.bad[rr >> 5], 1u << (rr & 31));
    if (d == 0) store_lse<T>(a, p, p.t0 + kt, head, mm, ll);
  }
}

// A part of a tile has been written (all row warps call; what its counter said goes to
// thread 0): the parts that were there before.
template <class S>
__device__ __forceinline__ int arrive_part(const PagedAttnArgs& a, const PagePiece& p) {
  all_rows<S>();
  int before = 0;
  if (threadIdx.x == 0) {
    __threadfence();
    before = atomicAdd(&a.tickets[p.cta0].arrived, 1);
  }
  return before;
}

// See to a cut tile after the run: its last part's CTA merges it.  Where that is much (a
// block of 64 rows in 19 parts: 0.6 MB, which one SM takes in in 9 us), the CTAs of the
// other parts stay for a while and take groups of its rows too; none is waited for.  (Without
// and with it: 16 tokens at 131072, 8 tiles of 19 parts, 97 and 91 us; 61 tokens at 1000, 32
// heads on 8, 16 tiles of 5, 31 and 18; 300 tokens at 2000, 8 heads, 26 and 20.)
constexpr uint64_t kMergeLingerNs = 20000;
template <class T, int HD, class S>
__device__ __forceinline__ void finish_cut(S& s, const PagedAttnArgs& a, const PagePiece& p, int tt, int before) {
  // (the piece was copied by other threads, and s.last of the tile before has been read)
  all_rows<S>();
  const int tid = threadIdx.x, parts = p.cta1 - p.cta0 + 1, live = p.nt * a.group, ways = merge_ways(parts);
  const int groups = (live + merge_rows<S, HD>(ways) - 1) / merge_rows<S, HD>(ways);
  const bool share = parts >= 4 && groups > 1;  // (of two or three parts each CTA has one to merge anyway)
  PageTicket* t = a.tickets + p.cta0;
  if (tid == 0) {
    bool there = before == parts - 1;
    if (!there && share) {
      const uint64_t t0 = globaltimer_ns();
      while (!there && globaltimer_ns() - t0 < kMergeLingerNs) {
        there = *const_cast<volatile int*>(&t->arrived) == parts;
        if (!there) __nanosleep(200);
      }
    }
    s.last = there;
    __threadfence();
  }
  all_rows<S>();
  if (s.last) {
    int g = 0;
    for (int k = 0;; ++k) {
      if (share) {
        all_rows<S>();
        if (tid == 0) s.claim = atomicAdd(&t->claimed, 1);
        all_rows<S>();
        g = s.claim;
      } else {
        g = k;
      }
      if (g >= groups) break;
      merge_group<T, HD>(s, a, p, tt, g, ways);
    }
    all_rows<S>();
    redo_bad<T, HD>(s, a, p, tt);
  }
  if (tid == 0 && atomicAdd(&t->left, 1) == parts - 1) t->arrived = t->claimed = t->left = 0;
}

}  // namespace cllm
