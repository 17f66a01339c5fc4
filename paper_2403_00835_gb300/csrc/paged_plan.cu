// Block tables and slot maps of a step (cllm_page_plan): every request's pages
// and every new row's slot from the requests' lengths, in one launch.
//
//   need = ceil((ctx + new) / P), grow = max(need - held, 0), and a request gets
//   its pages when the inclusive sum of grow over the requests before it fits the
//   free ring: two prefix sums (rows; pages taken and given back) over B numbers.
//
// Bound: latency.  The bytes are small (a table of 512 x 265 entries and 65536
// row slots: 2 MB, 0.3 us), so what counts is the number of dependent steps and launches.
// Every CTA computes the whole scan for itself from L2 (B <= 4096 triples)
// instead of waiting for one that does: no grid-wide step, one launch, and
// tables and slots are then written by all CTAs at once.  Slots come from the
// input table and the ring, never from the table being written.  Measured: one request
// 4.1 us, 512 with 16384 rows 7.9 us.
//
// In-place updates: a CTA's table rows are read and written by one warp, the ring's
// new entries lie behind its live ones, and what every CTA reads (ctx, new_rows,
// held, state) is only written by the CTA that arrives last, after its scan.
#include "paged.cuh"
#include "ptx.cuh"

namespace cllm {

namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanWords = 5;       // shared memory of a request, in words
constexpr int kPlanStatic = 1024;   // at least the kernel's other shared memory

struct PlanArgs {
  cllm_page_tables in, out;
  cllm_page_rows rows;
  const int* ctx;
  const int* new_rows;
  int B, page_shift;
};

// Inclusive sum over the block's threads (T: long long or int2); every thread
// gets its own, `total` the whole.  `sm` holds a value per warp.
__device__ __forceinline__ long long plus(long long a, long long b) { return a + b; }
__device__ __forceinline__ int2 plus(int2 a, int2 b) { return make_int2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ long long shfl_up(long long v, int d) { return __shfl_up_sync(~0u, v, d); }
__device__ __forceinline__ int2 shfl_up(int2 v, int d) {
  return make_int2(__shfl_up_sync(~0u, v.x, d), __shfl_up_sync(~0u, v.y, d));
}
template <class T>
__device__ T block_scan(T v, T* sm, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int d = 1; d < 32; d <<= 1) {
    const T o = shfl_up(v, d);
    if (lane >= d) v = plus(v, o);
  }
  __syncthreads();
  if (lane == 31) sm[warp] = v;
  __syncthreads();
  T before{};
  total = T{};
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w < warp) before = plus(before, sm[w]);
    total = plus(total, sm[w]);
  }
  return plus(before, v);
}

// Index `k` places after `first` in the ring (both below n, unless the caller's numbers are
// not a ring's: the result is inside it in any case).
__device__ __forceinline__ unsigned ring_at(unsigned first, unsigned k, unsigned n) {
  const unsigned x = first + k;
  return x < n ? x : x - n < n ? x - n : x % n;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const PlanArgs a) {
  extern __shared__ int sm_req[];
  __shared__ long long sm_scan[kPlanThreads / 32];
  __shared__ int sm_taken, sm_last;
  static_assert(sizeof(sm_scan) + sizeof(sm_taken) + sizeof(sm_last) <= kPlanStatic, "shared memory without asking");
  const int tid = threadIdx.x, B = a.B, W = a.in.width, N = a.in.n_pages, P = a.in.page_size;
  int* row_end = sm_req;       // rows of the requests up to this one
  int* held = sm_req + B;      // pages before
  int* after = sm_req + 2 * B; // pages after the step; -1 - pages: refused
  int* first = sm_req + 3 * B; // ring index of the first page taken or given back
  int* start = sm_req + 4 * B; // position of the first new row
  if (tid == 0) sm_taken = 0;
  pdl_launch_dependents();
  pdl_wait();

  // the ring's words are the caller's: whatever they hold, indices stay inside it
  const int head = static_cast<int>(static_cast<unsigned>(__ldcg(a.in.state)) % static_cast<unsigned>(N));
  const int count = min(max(__ldcg(a.in.state + 1), 0), N);
  const int per = (B + kPlanThreads - 1) / kPlanThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);

  // (a thread's first request is loaded at once: most batches have no second)
  int c0 = 0, n0 = 0, h0 = 0;
  if (b0 < b1) c0 = __ldcg(a.ctx + b0), n0 = __ldcg(a.new_rows + b0), h0 = __ldcg(a.in.held + b0);
  long long rows = max(n0, 0), total_rows;
  for (int b = b0 + 1; b < b1; ++b) rows += max(__ldcg(a.new_rows + b), 0);
  long long end = block_scan(rows, sm_scan, total_rows) - rows;
  int2 pages = make_int2(0, 0), total;  // taken if granted, given back
  for (int b = b0; b < b1; ++b) {
    const long long c = b == b0 ? c0 : __ldcg(a.ctx + b), n = b == b0 ? n0 : __ldcg(a.new_rows + b);
    const int h = min(max(b == b0 ? h0 : __ldcg(a.in.held + b), 0), W);
    end += max(n, 0ll);
    const bool valid = c >= 0 && n >= 0 && c + n <= static_cast<long long>(W) * P && end <= a.rows.max_rows;
    const int need = valid ? static_cast<int>((c + n + P - 1) >> a.page_shift) : h;
    row_end[b] = static_cast<int>(min(end, 0x7fffffffll));
    held[b] = h;
    start[b] = static_cast<int>(c);
    after[b] = valid ? need : -1 - h;
    pages = plus(pages, make_int2(max(need - h, 0), max(h - need, 0)));
  }
  int2 at = block_scan(pages, reinterpret_cast<int2*>(sm_scan), total);
  at = make_int2(at.x - pages.x, at.y - pages.y);
  int taken = 0;
  for (int b = b0; b < b1; ++b) {
    const int h = held[b], need = after[b] >= 0 ? after[b] : h;
    const int grow = max(need - h, 0);
    first[b] = static_cast<int>((static_cast<long long>(head) + (grow > 0 ? at.x : count + at.y)) % N);
    at = plus(at, make_int2(grow, max(h - need, 0)));
    if (grow > 0) {
      if (at.x <= count) taken = at.x;  // (those granted come before those refused)
      else after[b] = -1 - h;
    }
  }
  if (taken > 0) atomicMax(&sm_taken, taken);
  __syncthreads();

  // Every input that may be updated in place has been read: the last CTA to get here
  // writes the requests' results, at its end (the counter's answer takes a while).
  int arrived = 0;
  if (tid == 0 && gridDim.x > 1) {
    __threadfence();
    arrived = atomicAdd(a.out.state + 2, 1);
  }

  // block tables, a warp per request
  const int lane = tid & 31, warps = gridDim.x * (kPlanThreads / 32);
  for (int b = blockIdx.x * (kPlanThreads / 32) + (tid >> 5); b < B; b += warps) {
    const unsigned h = held[b], h2 = after[b] >= 0 ? after[b] : h, keep = min(h, h2);
    const int* in = a.in.table + static_cast<size_t>(b) * W;
    int* out = a.out.table + static_cast<size_t>(b) * W;
    // (8 loads under way before the first store; a table may be 2^31 - 1 wide: steps pass that)
    for (unsigned j0 = (in == out ? keep : 0) + lane; j0 < static_cast<unsigned>(W); j0 += 256) {
      int page[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const unsigned j = j0 + 32 * u;
        page[u] = -1;
        if (j < h) page[u] = in[j];
        else if (j < h2) page[u] = __ldcg(a.in.ring + ring_at(first[b], j - h, N));
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const unsigned j = j0 + 32 * u;
        if (j >= static_cast<unsigned>(W)) break;
        if (j >= h2 && j < h) a.in.ring[ring_at(first[b], j - h2, N)] = page[u], page[u] = -1;
        out[j] = page[u];
      }
    }
  }

  // slots, a thread per row
  for (unsigned t = blockIdx.x * kPlanThreads + tid; t < static_cast<unsigned>(a.rows.max_rows);
       t += gridDim.x * kPlanThreads) {
    long long slot = -1;
    int pos = 0;
    if (t < total_rows) {
      int lo = 0, hi = B - 1;  // the request: the first whose rows end past t
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (static_cast<unsigned>(row_end[mid]) > t) hi = mid;
        else lo = mid + 1;
      }
      if (after[lo] >= 0) {
        pos = start[lo] + static_cast<int>(t - (lo > 0 ? row_end[lo - 1] : 0));
        const int j = pos >> a.page_shift, h = held[lo];
        const int page = j < h ? a.in.table[static_cast<size_t>(lo) * W + j]
                               : __ldcg(a.in.ring + ring_at(first[lo], j - h, N));
        slot = (static_cast<long long>(page) << a.page_shift) + (pos & (P - 1));
      }
    }
    a.rows.slots[t] = slot;
    a.rows.positions[t] = pos;
  }

  if (tid == 0) {
    sm_last = arrived == static_cast<int>(gridDim.x) - 1;
    __threadfence();
  }
  __syncthreads();
  if (sm_last) {
    for (int b = tid; b < B; b += kPlanThreads) {
      const bool ok = after[b] >= 0;
      const int len = ok ? start[b] + row_end[b] - (b > 0 ? row_end[b - 1] : 0) : 0;
      a.out.held[b] = ok ? after[b] : held[b];
      a.rows.granted[b] = ok;
      a.rows.seq_len[b] = len;
      a.rows.row_start[b + 1] = row_end[b];
    }
    if (tid == 0) {
      a.rows.row_start[0] = 0;
      a.out.state[0] = static_cast<int>((static_cast<long long>(head) + sm_taken) % N);
      a.out.state[1] = min(count - sm_taken + total.y, N);
      a.out.state[2] = 0;
    }
  }
}

}  // namespace

cudaError_t launch_page_plan(const cllm_page_tables& in, const cllm_page_tables& out, const cllm_page_rows& rows,
                             int B, const int* ctx, const int* new_rows, cudaStream_t s) {
  PlanArgs a{in, out, rows, ctx, new_rows, B, 0};
  while ((1 << a.page_shift) < in.page_size) ++a.page_shift;
  const int smem = kPlanWords * 4 * B;
  // 48 KB without asking, of which the kernel's own variables are a part.  The limit is raised to
  // the largest batch's need, and never lowered: calls of several threads do not take it
  // from each other.
  if (smem > 48 * 1024 - kPlanStatic) {
    const cudaError_t e = cudaFuncSetAttribute(page_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               kPlanWords * 4 * kPlanBatch);
    if (e != cudaSuccess) return e;
  }
  const int want = max((rows.max_rows + kPlanThreads - 1) / kPlanThreads,
                       (B + kPlanThreads / 32 - 1) / (kPlanThreads / 32));
  return launch_after(page_plan_kernel, dim3(min(max(want, 1), 152)), kPlanThreads, smem, s, a);
}

}  // namespace cllm
