// Internal declarations of the paged cache (include/cllm_paged.h).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/cllm_paged.h"

namespace cllm {

// A cut tile's counters: parts written, groups of its rows taken for merging, parts' CTAs
// that are done with it (the last of them clears the counters).
struct PageTicket {
  int arrived, claimed, left;
};

// Arguments of an attention launch (device pointers; strides in elements).
struct PagedAttnArgs {
  const void* q;
  void* out;
  float* lse;
  long long q_row, q_head, out_row, out_head;
  const int* row_start;
  const int* seq_len;
  const int* table;
  int table_width, batch, rows;
  int H, Hkv, group;       // group = H / Hkv query heads share a key/value head
  int group_inv;           // x / group = x * group_inv >> 16 for x < 256 (ceil(2^16 / group), group <= 64)
  float scale_log2;        // scale * log2(e)
  int window, sinks;       // sinks: first keys seen beside the window (0 without one)
  const uint32_t* mask;
  int mask_words;
  // this layer's pools
  const void* k;
  const void* v;
  long long s_page, s_head, s_pos;
  int layer, n_pages, page_shift;
  // work that is cut over several CTAs: two partial tiles per CTA, and the
  // counters of the tile that begins in it and goes on (zero between launches)
  float* part_o;
  float2* part_ml;
  PageTicket* tickets;
  int* err;
};

// Launch a kernel that may start while the one before it in the stream ends; it
// waits (griddepcontrol.wait) before it touches memory.  What it reads may be written by that
// one, so none of it is read by non-coherent loads, which ask for memory that nobody writes while the
// kernel lives (and may be moved to before the wait).
template <class... P, class... A>
inline cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s,
                                const A&... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Partials: CTA c's slot 2c is a tile that began in an earlier CTA, slot 2c + 1
// one that it begins and does not end.  The tensor-memory kernel has a CTA and slots of
// 256 rows per SM, the others two CTAs at most and fewer rows.
constexpr int kPagedPartRows = 256;
constexpr int kPagedCtas = 2;  // CTAs per SM, at most

constexpr int kPlanBatch = 4096;  // requests of a plan, at most
cudaError_t launch_page_plan(const cllm_page_tables& in, const cllm_page_tables& out, const cllm_page_rows& rows,
                             int B, const int* ctx, const int* new_rows, cudaStream_t s);

struct PagedAppendArgs {
  const void *k, *v, *q;
  void *kp, *vp, *q_out;  // this layer's pools
  long long k_row, v_row, q_row, qo_row, s_page, s_head, s_pos;
  const long long* slots;
  const float2* rope;
  const int* positions;
  const void *q_gain, *k_gain;  // of the heads' norms, or null
  float eps;
  int dims, interleaved;        // rotated values of a head; neighbours in pairs
  int max_pos, T, H, Hkv, hd, n_pages, page_shift;  // H = 0: no queries
  int* err;
};
cudaError_t launch_paged_append(const PagedAppendArgs& a, int dtype, cudaStream_t s);

constexpr int kRopeDims = 256;  // rotated values of a head, at most
// turns: a position's fraction of a turn, in 2^-64
cudaError_t launch_rope_table(float* table, int first, int positions, int dims, const unsigned long long* turns,
                              float amplitude, cudaStream_t s);

// fp32 pools (paged_attn.cu)
cudaError_t launch_paged_attention_f32(const PagedAttnArgs& a, int hd, int grid, cudaStream_t s);
cudaError_t paged_attention_f32_set_attributes();
// 16-bit pools (paged_attn_tc.cu); k, v: the pools' maps; hold: test hook, 1 + the chunk
// of a piece at which the MMA issuer gives up (0: none)
cudaError_t launch_paged_attention_tc(const PagedAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int dtype,
                                      int hd, int hold, int grid, cudaStream_t s);
cudaError_t paged_attention_tc_set_attributes();
// a pool in boxes of 64 columns and `keys` positions, or a page's if that is less
bool paged_pool_map(CUtensorMap* m, const void* pool, const cllm_paged_desc& d, int keys);
// queries of a tile of `rows` rows: group heads of rows / group tokens, row = token * group + head
bool paged_query_map(CUtensorMap* m, const PagedAttnArgs& a, int dtype, int hd, int rows);
// 16-bit pools, few rows (paged_attn_few.cu): tiles of 16 rows, group at most 16; k, v:
// maps of 64 positions; sms: SMs of the device; hold: 1 + the chunk of a piece at which
// the loading warp gives up
constexpr int kFewRows = 16, kFewKeys = 64;
cudaError_t launch_paged_attention_few(const PagedAttnArgs& a, const CUtensorMap& k, const CUtensorMap& v, int dtype,
                                       int hd, int hold, int sms, cudaStream_t s);
cudaError_t paged_attention_few_set_attributes();

}  // namespace cllm
