// The work of a paged attention launch and its division among CTAs, and what
// the attention kernels share at a row's end.
//
// A tile is a run of tokens of one request times the query heads of one key/value
// head; its units are the chunks of keys that any of its rows may see (one unit,
// if there are none: its rows are written as zeros).  Lengths live on the device, so
// the division is made there: all units in order (request, head, tile, chunk)
// are cut into equal runs, one per CTA.  A run's ends may cut a tile; the pieces
// leave partial results, and the CTA that finishes a tile last merges them in
// order of their CTAs, so sums do not depend on who that is.  Where the tiles are
// short, whole tiles are dealt out instead: cutting one costs more than it saves.
#pragma once
#include "act.cuh"
#include "internal.cuh"
#include "paged.cuh"

namespace cllm {

struct PagedGeom {
  int tile_tok;     // tokens of a tile
  int slot_tok;     // tokens of 128 rows (tensor-memory kernel: a tile has one or two times that)
  int chunk_shift;  // log2 of the keys of a unit
  int min_units;    // fewest units of a CTA's run
  int piece_cost;   // what a piece costs beside its units, and merging a cut tile, in units' time
  int merge_cost;
};
// (A CTA's first loads wait for what follows, in one thread: units are counted in 32
// bits, which the host sees to, and nothing is divided that a shift or a compare decides.)

// Request b's rows and length as the device has them.  Rows outside the arrays
// or a length past the block table make it a request without rows, or without keys.  Of a
// request without tokens, as a plan leaves one that it refuses, the rows past the arrays are
// left out without a word: want of rows may be why it was refused.
struct Request {
  int row0, n, len;
};
// Positions are held in 32 bits, a loading lane's too (32 boxes of up to 128 keys from a chunk's first).
constexpr int kLongest = 0x7fffffff - 8191;
__device__ __forceinline__ Request request(const PagedAttnArgs& a, int b) {
  Request r{a.row_start[b], a.row_start[b + 1], a.seq_len[b]};
  r.n -= r.row0;
  if (r.len == 0 && r.row0 >= 0 && r.n >= 0) {
    r.row0 = min(r.row0, a.rows);
    r.n = min(r.n, a.rows - r.row0);
  }
  const bool rows = r.row0 >= 0 && r.n >= 0 && r.row0 <= a.rows && r.n <= a.rows - r.row0;
  const bool fits = r.len <= kLongest && r.len <= static_cast<long long>(a.table_width) << a.page_shift;
  if (!rows) r.n = 0;
  if (!fits) r.len = 0;
  if (!rows || !fits) atomicOr(a.err, DERR_CAPACITY);
  return r;
}

struct TileKeys {
  int lo, hi, sink;  // keys [0, sink) and [lo, hi) that some row may see (hi <= lo: none; sink < lo, or 0)
  __device__ bool has(int key) const { return (key >= lo && key < hi) || key < sink; }
  __device__ bool some(int a, int b) const { return (a < hi && b > lo) || a < sink; }  // of keys [a, b)
};
// Keys seen by tokens [t0, t1) of a request of n new tokens and `len` in all.
__device__ __forceinline__ TileKeys tile_keys(const PagedAttnArgs& a, int n, int len, int t0, int t1) {
  TileKeys k;
  const int ctx = len - n;
  k.hi = ctx < 0 ? 0 : (a.mask != nullptr ? len : ctx + t1);
  k.lo = a.window > 0 ? max(0, ctx + t0 - a.window + 1) : 0;
  k.sink = a.sinks < k.lo ? min(a.sinks, k.hi) : 0;
  if (a.sinks >= k.lo) k.lo = 0;
  return k;
}
// The chunks of a tile: those of its first keys and those from `near` on, which come after them
// in the order of the work; a tile's chunks are counted so that the near ones have
// their own numbers, and the others the `gap` numbers before.
struct TileChunks {
  int near, gap, units;
};
__device__ __forceinline__ TileChunks tile_chunks(const PagedGeom& g, const TileKeys& k) {
  const int first = k.sink > 0 ? ((k.sink - 1) >> g.chunk_shift) + 1 : 0, near = max(k.lo >> g.chunk_shift, first);
  TileChunks c{near, near - first, 1};
  if (k.hi > k.lo) c.units = ((k.hi - 1) >> g.chunk_shift) + 1 - c.gap;
  return c;
}
__device__ __forceinline__ int tile_units(const PagedGeom& g, const TileKeys& k) { return tile_chunks(g, k).units; }
// Of one head of each lane's request (the whole warp calls; n = 0: none): all units, tiles, and
// the units of the longest tile.  A request of many tiles is summed by all lanes.
struct HeadWork {
  unsigned units, tiles, longest;
};
__device__ __forceinline__ HeadWork head_work(const PagedAttnArgs& a, const PagedGeom& g, int n, int len) {
  HeadWork w{0, 0, 0};
  const bool many = n > 2 * g.tile_tok;
  if (!many && n > 0) {
    w.units = w.longest = tile_units(g, tile_keys(a, n, len, 0, min(n, g.tile_tok)));
    w.tiles = 1;
    if (n > g.tile_tok) {
      const unsigned u = tile_units(g, tile_keys(a, n, len, g.tile_tok, n));
      w = {w.units + u, 2, max(w.longest, u)};
    }
  }
  for (unsigned rest = __ballot_sync(0xffffffffu, many); rest; rest &= rest - 1) {
    const int src = __ffs(rest) - 1, lane = threadIdx.x & 31;
    const int bn = __shfl_sync(0xffffffffu, n, src), bl = __shfl_sync(0xffffffffu, len, src);
    HeadWork v{0, 0, 0};
    for (int t0 = lane * g.tile_tok; t0 < bn; t0 += 32 * g.tile_tok) {
      const unsigned u = tile_units(g, tile_keys(a, bn, bl, t0, min(bn, t0 + g.tile_tok)));
      v = {v.units + u, v.tiles + 1, max(v.longest, u)};
    }
    v = {__reduce_add_sync(0xffffffffu, v.units), __reduce_add_sync(0xffffffffu, v.tiles),
         __reduce_max_sync(0xffffffffu, v.longest)};
    if (lane == src) w = v;
  }
  return w;
}

// Whether whole tiles are dealt out: rounds of whole tiles against equal runs of units, whose
// ends are pieces of their own and merged.  (Costs fitted to both sides' times: whole and
// cut, a block of 16 tokens, 32 heads, 144 keys 7.8 and 9.8 us; 8 requests of 32 tokens, 256
// to 1024 keys 26.5 and 35 us; 4 of 61 tokens, 32 heads on 8, 700 to 1100 keys 17.6 and
// 23.8 us; 6 of 32 tokens at 1000 keys, 32 heads 26.8 and 28.6 us.  Long tiles are always cut.)
__device__ __forceinline__ bool deal_tiles(const PagedGeom& g, unsigned units, unsigned tiles, unsigned longest) {
  if (longest > 64) return false;
  const unsigned per = max((units + gridDim.x - 1) / gridDim.x, static_cast<unsigned>(g.min_units));
  const unsigned rounds = (tiles + gridDim.x - 1) / gridDim.x;
  return rounds * (longest + g.piece_cost) <=
         per + g.piece_cost + g.piece_cost * per * tiles / max(units, 1u) + g.merge_cost;
}

// Where a CTA's run begins (shared memory).  (`whole`: a unit is a tile.)
struct RunStart {
  unsigned u0, u1, per;  // the run, and the units of every run
  unsigned begin, head;  // first unit of request b, and the units of one of its heads
  int b, row0, n, len, whole;
};

// A piece: the chunks [ca, cb) of a tile that belong to this CTA's run.
struct Piece {
  int b, h, t0, nt;        // request, key/value head, first token and tokens of the tile
  int n, len, row0;        // the request's new tokens, all tokens, first row
  TileKeys keys;           // of the tile
  int near, gap;           // as in TileChunks
  int ca, cb;              // this piece's chunks
  int tca, tcb;            // the tile's
  unsigned tile_u;         // the tile's first unit
  __device__ bool whole() const { return ca == tca && cb == tcb; }
  __device__ bool empty() const { return tca == tcb; }
  __device__ int chunk(int c) const { return c < near ? c - gap : c; }  // where in the request chunk c is
};

// The run of this CTA among `total` units, and where it begins if that is in one of the
// lanes' (threads') requests, each with `units` units after `before`.
__device__ __forceinline__ void set_run(RunStart* rs, unsigned total, int min_units, bool whole, bool writer) {
  const unsigned per = max((total + gridDim.x - 1) / gridDim.x, static_cast<unsigned>(min_units));
  const unsigned u0 = min(blockIdx.x * per, total);
  if (writer) rs->u0 = u0, rs->u1 = min(u0 + per, total), rs->per = per, rs->whole = whole;
}
__device__ __forceinline__ void set_begin(RunStart* rs, unsigned u0, unsigned before, unsigned units, unsigned head, int b,
                                          const Request& r) {
  if (u0 >= before && u0 < before + units) {  // one thread at most
    rs->b = b;
    rs->begin = before;
    rs->head = head;
    rs->row0 = r.row0, rs->n = r.n, rs->len = r.len;
  }
}

// Up to 32 requests: the block's run, by one warp.
constexpr int kWarpRequests = 32;
__device__ __forceinline__ void run_start_warp(const PagedAttnArgs& a, const PagedGeom& g, RunStart* rs) {
  const int lane = threadIdx.x & 31;
  const Request r = lane < a.batch ? request(a, lane) : Request{0, 0, 0};
  const HeadWork w = head_work(a, g, r.n, r.len);
  const unsigned units = __reduce_add_sync(0xffffffffu, w.units) * a.Hkv;
  const unsigned tiles = __reduce_add_sync(0xffffffffu, w.tiles) * a.Hkv;
  const bool whole = deal_tiles(g, units, tiles, __reduce_max_sync(0xffffffffu, w.longest));
  const unsigned head = whole ? w.tiles : w.units, mine = head * a.Hkv;
  unsigned v = mine;
  if (a.batch > 1) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v += o;
    }
  }
  set_run(rs, whole ? tiles : units, whole ? 1 : g.min_units, whole, lane == 0);
  __syncwarp();
  set_begin(rs, rs->u0, v - mine, mine, head, lane, r);
  __syncwarp();
}

// Any number: all threads of the block (a multiple of 32, at most 1024) call.  `sm` holds 32 values.
__device__ __forceinline__ void run_start_block(const PagedAttnArgs& a, const PagedGeom& g, RunStart* rs, unsigned* sm) {
  const int tid = threadIdx.x, nthr = blockDim.x, lane = tid & 31, warp = tid >> 5;
  HeadWork w{0, 0, 0};
  Request r{0, 0, 0};
  // a thread per request and round
  auto load = [&](int b) {
    r = b < a.batch ? request(a, b) : Request{0, 0, 0};
    w = head_work(a, g, r.n, r.len);
  };
  auto all = [&](unsigned x, bool largest) {
    x = largest ? __reduce_max_sync(0xffffffffu, x) : __reduce_add_sync(0xffffffffu, x);
    __syncthreads();
    if (lane == 0) sm[warp] = x;
    __syncthreads();
    unsigned sum = 0;
    for (int i = 0; i < nthr / 32; ++i) sum = largest ? max(sum, sm[i]) : sum + sm[i];
    return sum;
  };
  unsigned units = 0, tiles = 0, longest = 0;
  for (int b0 = 0; b0 < a.batch; b0 += nthr) {
    load(b0 + tid);
    units += w.units, tiles += w.tiles, longest = max(longest, w.longest);
  }
  units = all(units, false) * a.Hkv, tiles = all(tiles, false) * a.Hkv, longest = all(longest, true);
  const bool whole = deal_tiles(g, units, tiles, longest);
  set_run(rs, whole ? tiles : units, whole ? 1 : g.min_units, whole, tid == 0);
  unsigned base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += nthr) {
    if (a.batch > nthr) load(b0 + tid);
    const unsigned head = whole ? w.tiles : w.units, mine = head * a.Hkv;
    unsigned v = mine, before = 0, sum = 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned o = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) v += o;
    }
    __syncthreads();
    if (lane == 31) sm[warp] = v;
    __syncthreads();
    for (int i = 0; i < nthr / 32; ++i) {
      if (i < warp) before += sm[i];
      sum += sm[i];
    }
    set_begin(rs, rs->u0, base + before + v - mine, mine, head, b0 + tid, r);
    base += sum;
  }
  __syncthreads();
}

// The pieces of the block's run, in order (the whole warp calls).
struct PagedWalk {
  unsigned u, u1, per, tu;  // next unit, end of the run, units of a run, first unit of the tile
  int b, h, t0, n, len, row0, whole;

  __device__ void load(const PagedAttnArgs& a) {
    const Request q = request(a, b);
    row0 = q.row0, n = q.n, len = q.len;
    t0 = 0;
    h = 0;
  }
  __device__ void begin(const RunStart& rs) {
    u = rs.u0;
    u1 = rs.u1;
    per = rs.per;
    whole = rs.whole;
    if (u >= u1) return;
    b = rs.b, row0 = rs.row0, n = rs.n, len = rs.len;
    t0 = 0;
    const unsigned in = u - rs.begin;
    h = in < rs.head ? 0 : in / rs.head;
    tu = rs.begin + h * rs.head;
  }
  __device__ bool next(const PagedAttnArgs& a, const PagedGeom& g, Piece& p) {
    if (u >= u1) return false;
    for (;;) {
      const int t1 = min(n, t0 + g.tile_tok);
      const TileKeys k = tile_keys(a, n, len, t0, t1);
      const TileChunks ch = tile_chunks(g, k);
      const int chunks = ch.units, units = whole ? 1 : chunks;
      if (u < tu + units) {
        p.b = b, p.h = h, p.t0 = t0, p.nt = t1 - t0, p.n = n, p.len = len, p.row0 = row0;
        p.keys = k;
        p.near = ch.near, p.gap = ch.gap;
        p.tile_u = tu;
        p.tca = ch.gap;
        p.tcb = k.hi > k.lo ? p.tca + chunks : p.tca;
        const unsigned e = min(u1, tu + units);
        p.ca = p.tca, p.cb = p.tcb;
        if (!whole && p.tcb > p.tca) p.ca += u - tu, p.cb = p.tca + static_cast<int>(e - tu);
        u = e;
        return true;
      }
      tu += units;
      t0 = t1;
      if (t0 < n) continue;
      t0 = 0;
      if (++h < a.Hkv) continue;
      // the next request with rows, 32 at a time
      const int lane = threadIdx.x & 31;
      for (;;) {
        const int c = b + 1 + lane;
        const bool some = c < a.batch && request(a, c).n > 0;
        const unsigned any = __ballot_sync(0xffffffffu, some);
        if (any) {
          b += __ffs(any);
          break;
        }
        b += 32;
        if (b + 1 >= a.batch) return false;  // (the lengths changed under the launch)
      }
      load(a);
    }
  }
  // contributors of a cut tile: CTAs [first, last]; CTA c's partial slot
  __device__ int first_cta(const Piece& p) const { return p.ca == p.tca ? blockIdx.x : p.tile_u / per; }
  __device__ int last_cta(const Piece& p) const {
    return p.cb == p.tcb ? blockIdx.x : (p.tile_u + (p.tcb - p.tca) - 1) / per;
  }
  __device__ int slot(const Piece& p, int c) const { return 2 * c + (c * per < p.tile_u ? 1 : 0); }
};

// ---- a row's keys ------------------------------------------------------------------

// Keys [lo, hi), and of those before lo the first `sink`, that token i of a request may see; with a
// mask, those from ctx on only where their bit is set.
struct RowKeys {
  int lo, hi, sink, ctx;
  const uint32_t* bits;  // the row's mask words, or null
  int words;
};
__device__ __forceinline__ RowKeys row_keys(const PagedAttnArgs& a, int n, int len, int row0, int i) {
  RowKeys r;
  r.ctx = len - n;
  const int idx = r.ctx + i;
  r.hi = r.ctx < 0 ? 0 : (a.mask != nullptr ? len : idx + 1);
  r.lo = a.window > 0 ? max(0, idx - a.window + 1) : 0;
  r.sink = a.sinks;
  r.bits = a.mask != nullptr ? a.mask + static_cast<size_t>(row0 + i) * a.mask_words : nullptr;
  r.words = a.mask_words;
  return r;
}
// Bit j: whether the row sees key kb + j, j < 32.
__device__ __forceinline__ uint32_t key_bits(const RowKeys& r, int kb) {
  const int below = r.lo - kb, above = r.hi - kb, first = r.sink - kb;
  uint32_t m = below <= 0 ? ~0u : below >= 32 ? 0u : ~0u << below;
  if (first > 0) m |= first >= 32 ? ~0u : ~(~0u << first);
  m &= above >= 32 ? ~0u : above <= 0 ? 0u : ~(~0u << above);
  if (r.bits != nullptr && m != 0) {
    const int j = kb - r.ctx;  // new token of bit 0
    if (j >= 0) {
      const int w = j >> 5;
      const uint32_t w0 = w < r.words ? r.bits[w] : 0u, w1 = w + 1 < r.words ? r.bits[w + 1] : 0u;
      m &= __funnelshift_r(w0, w1, j & 31);
    } else if (j > -32) {
      m &= (r.bits[0] << -j) | ~(~0u << -j);
    }
  }
  return m;
}

// A row's maximum m and sum l over some of its keys, for merging: m -inf means that none of
// them has weight.  Maxima pass NaN over, sums do not, so a sum that is no number takes the
// maximum with it.  (The sum is NaN only where a score that the row sees is NaN or +inf: all
// of the row is NaN then, and needs no second look by exact_row.)
__device__ __forceinline__ float share_max(float m, float l) { return l == l ? m : l; }

// Address of (page of position pos) in a pool; null when the table's entry is
// outside the pool (noted in the status word).
template <class T>
__device__ __forceinline__ const T* pool_row(const PagedAttnArgs& a, const void* pool, int b, int h, int pos) {
  const int j = pos >> a.page_shift;
  const int page = j < a.table_width ? a.table[static_cast<size_t>(b) * a.table_width + j] : -1;
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.n_pages)) {
    atomicOr(a.err, DERR_CAPACITY);
    return nullptr;
  }
  return static_cast<const T*>(pool) + page * a.s_page + h * a.s_head + (pos & ((1 << a.page_shift) - 1)) * a.s_pos;
}

// One row (token tok of a request, query head `head` of key/value head h) from the
// definition, by a warp: a key that the row does not see is not touched.  Called where a
// row's tile gave something other than a finite number, which a value of a key that only
// other rows see can cause (0 * inf).
template <class T, int HD>
__device__ __noinline__ void exact_row(const PagedAttnArgs& a, int b, int h, int n, int len, int row0, int tok, int head) {
  const int lane = threadIdx.x & 31;
  constexpr int E = HD / 32;
  const RowKeys r = row_keys(a, n, len, row0, tok);
  const size_t row = static_cast<size_t>(row0 + tok);
  const T* q = static_cast<const T*>(a.q) + row * a.q_row + head * a.q_head;
  float qv[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) qv[e] = ld_act(q, lane * E + e), o[e] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int from = r.lo & ~31;
  for (int kb = r.sink > 0 ? 0 : from; kb < r.hi; kb = kb + 32 >= r.sink ? max(kb + 32, from) : kb + 32) {
    for (uint32_t bits = key_bits(r, kb); bits; bits &= bits - 1) {
      const int k = kb + __ffs(bits) - 1;
      const T* kp = pool_row<T>(a, a.k, b, h, k);
      const T* vp = pool_row<T>(a, a.v, b, h, k);
      float s = 0.f;
      if (kp != nullptr) {
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(qv[e], ld_act(kp, lane * E + e), s);
      }
      s = warp_sum(s) * a.scale_log2;
      const float nm = s > m ? s : m;
      const float f = m == -INFINITY ? 0.f : exp2f(m - nm), w = s == -INFINITY ? 0.f : exp2f(s - nm);
      m = nm;
      l = l * f + w;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = o[e] * f + (vp != nullptr ? w * ld_act(vp, lane * E + e) : 0.f);
    }
  }
  const bool any = l != 0.f;  // (NaN counts)
  T* out = static_cast<T*>(a.out) + row * a.out_row + head * a.out_head;
#pragma unroll
  for (int e = 0; e < E; ++e) st_act(out, lane * E + e, any ? o[e] / l : 0.f);
  if (lane == 0 && a.lse != nullptr) a.lse[row * a.H + head] = any ? (m + log2f(l)) * 0.69314718055994530942f : -INFINITY;
}

}  // namespace cllm
