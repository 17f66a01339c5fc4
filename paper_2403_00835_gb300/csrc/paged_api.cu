// Host side of include/cllm_paged.h: argument checks, the cache's tensor maps and
// scratch, and the launches.
#include <math.h>

#include <new>

#include "../../include/cllm_testing.h"
#include "internal.cuh"
#include "on_device.cuh"
#include "paged.cuh"

using namespace cllm;

struct cllm_paged {
  cllm_paged_desc d;
  int dev = 0, sms = 0, page_shift = 0, es = 0;
  float* part_o = nullptr;
  float2* part_ml = nullptr;
  PageTicket* tickets = nullptr;  // one per CTA, then the status word (all in part_o's allocation)
  size_t ticket_bytes = 0;        // with the status word
  int* err = nullptr;
  CUtensorMap mk, mv, mk_few, mv_few;  // the pools (16-bit types) in boxes of 128 and 64 positions
  int hold = 0;            // test hook
};

namespace {

constexpr float kLog2e = 1.4426950408889634f;

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2i(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

bool tables_ok(const cllm_page_tables* t) {
  return t && t->table && t->held && t->ring && t->state && aligned(t->table, 4) && aligned(t->held, 4) &&
         aligned(t->ring, 4) && aligned(t->state, 4) && t->max_batch >= 1 && t->max_batch <= kPlanBatch && t->width >= 1 &&
         t->n_pages >= 1 && pow2(t->page_size) &&
         static_cast<int64_t>(t->width) * t->page_size <= 0x7fffffff &&
         static_cast<int64_t>(t->max_batch) * t->width <= 0x7fffffff;
}

}  // namespace

extern "C" int cllm_page_plan(const cllm_page_tables* in, const cllm_page_tables* out, const cllm_page_rows* rows,
                              int B, const int32_t* ctx, const int32_t* new_rows, void* cuda_stream) {
  if (!tables_ok(in) || !tables_ok(out) || !rows || !rows->row_start || !rows->seq_len || !rows->granted ||
      !rows->slots || !rows->positions || rows->max_rows < 1 || !aligned(rows->slots, 8) ||
      !aligned(rows->row_start, 4) || !aligned(rows->seq_len, 4) || !aligned(rows->granted, 4) ||
      !aligned(rows->positions, 4) || B < 0 || B > in->max_batch || in->max_batch != out->max_batch ||
      in->width != out->width || in->n_pages != out->n_pages || in->page_size != out->page_size ||
      in->ring != out->ring)
    return CLLM_EINVAL;
  if (B > 0 && (!ctx || !new_rows || !aligned(ctx, 4) || !aligned(new_rows, 4))) return CLLM_EINVAL;
  const cudaError_t e = launch_page_plan(*in, *out, *rows, B, ctx, new_rows, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? CLLM_OK : cuda_fail(e, "page_plan");
}

extern "C" void cllm_paged_destroy(cllm_paged* c) {
  if (!c) return;
  {
    const OnDevice on(c->dev);
    cudaDeviceSynchronize();
    cudaFree(c->part_o);
  }
  delete c;
}

extern "C" int cllm_paged_create(const cllm_paged_desc* desc, cllm_paged** out) {
  if (!desc || !out) return CLLM_EINVAL;
  *out = nullptr;
  const cllm_paged_desc& d = *desc;
  if (!d.k || !d.v || (d.dtype != CLLM_F32 && d.dtype != CLLM_BF16 && d.dtype != CLLM_F16) || d.layers < 1 ||
      d.n_pages < 1 || d.page_size < 1 || d.n_kv_heads < 1 || d.head_dim < 1 || d.n_heads < 1)
    return CLLM_EINVAL;
  if ((d.head_dim != 64 && d.head_dim != 128) || !pow2(d.page_size) || d.page_size < 8 || d.page_size > 256 ||
      d.n_heads % d.n_kv_heads || d.n_heads / d.n_kv_heads > 64)
    return CLLM_EUNSUPPORTED;
  const int es = d.dtype == CLLM_F32 ? 4 : 2;
  const int64_t strides[4] = {d.stride_layer, d.stride_page, d.stride_head, d.stride_pos};
  const int64_t counts[4] = {d.layers, d.n_pages, d.n_kv_heads, d.page_size};
  for (int i = 0; i < 4; ++i)
    if (counts[i] > 1 && (strides[i] < d.head_dim || strides[i] * es % 16 || strides[i] > (int64_t(1) << 38)))
      return CLLM_EINVAL;
  if (!aligned(d.k, 16) || !aligned(d.v, 16)) return CLLM_EINVAL;

  int dev = 0, major = 0, minor = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_fail(e, "paged_create");
  if (major != 10 || minor != 3) return CLLM_EUNSUPPORTED;

  cllm_paged* c = new (std::nothrow) cllm_paged;
  if (!c) return CLLM_ENOMEM;
  c->d = d;
  // a dimension of one needs no stride
  if (d.layers == 1) c->d.stride_layer = d.head_dim;
  if (d.n_pages == 1) c->d.stride_page = d.head_dim;
  if (d.n_kv_heads == 1) c->d.stride_head = d.head_dim;
  c->dev = dev;
  c->sms = sms;
  c->es = es;
  c->page_shift = log2i(d.page_size);
  int rc = CLLM_OK;
  do {
    e = es == 4 ? paged_attention_f32_set_attributes() : paged_attention_tc_set_attributes();
    if (e == cudaSuccess && es == 2) e = paged_attention_few_set_attributes();
    if (e != cudaSuccess) {
      rc = cuda_fail(e, "paged_create");
      break;
    }
    if (es == 2 && (!paged_pool_map(&c->mk, d.k, c->d, 128) || !paged_pool_map(&c->mv, d.v, c->d, 128) ||
                    !paged_pool_map(&c->mk_few, d.k, c->d, kFewKeys) ||
                    !paged_pool_map(&c->mv_few, d.v, c->d, kFewKeys))) {
      rc = CLLM_EINVAL;
      break;
    }
    // (one allocation: it takes as long as the rest of the call)
    const size_t rows = 2 * static_cast<size_t>(sms) * kPagedPartRows;
    const size_t tickets = static_cast<size_t>(sms) * kPagedCtas;
    const size_t st = tickets * sizeof(PageTicket) + 4, so = rows * d.head_dim * 4, sm = rows * 8;
    static_assert(kPagedPartRows >= 64 * kPagedCtas, "slots of the kernels with several CTAs per SM");
    void* base = nullptr;
    if (lib_malloc(&base, so + sm + st) != cudaSuccess) {
      rc = CLLM_ENOMEM;
      break;
    }
    c->part_o = static_cast<float*>(base);
    c->part_ml = reinterpret_cast<float2*>(static_cast<char*>(base) + so);
    c->tickets = reinterpret_cast<PageTicket*>(static_cast<char*>(base) + so + sm);
    c->ticket_bytes = st;
    c->err = reinterpret_cast<int*>(c->tickets + tickets);
    // (the default stream orders the clearing before any later work)
    e = cudaMemset(c->tickets, 0, st);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) rc = cuda_fail(e, "paged_create");
  } while (false);
  if (rc != CLLM_OK) {
    cllm_paged_destroy(c);
    return rc;
  }
  *out = c;
  return CLLM_OK;
}

extern "C" int cllm_paged_status(cllm_paged* c, void* cuda_stream) {
  if (!c) return CLLM_EINVAL;
  const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int err = 0;
  const OnDevice on(c->dev);
  cudaError_t e = on.error;
  if (e == cudaSuccess) e = cudaMemcpyAsync(&err, c->err, 4, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && err != 0) {
    // (a timed-out launch may leave arrival counters behind)
    e = cudaMemsetAsync(c->tickets, 0, c->ticket_bytes, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  }
  if (e != cudaSuccess) return cuda_fail(e, "paged_status");
  return err == 0 ? CLLM_OK : err & DERR_TIMEOUT ? CLLM_ETIMEOUT : CLLM_EDEVICE;
}

// heads: null for a rotation of whole heads in halves, no norms.
static int append(cllm_paged* c, const cllm_paged_rows* r, const cllm_paged_heads* heads, void* cuda_stream) {
  if (!c || !r || r->layer < 0 || r->layer >= c->d.layers || r->rows < 0) return CLLM_EINVAL;
  if (r->rows == 0) return CLLM_OK;
  const cllm_paged_desc& d = c->d;
  auto rows_ok = [&](const void* p, int64_t stride, int heads) {
    return p && aligned(p, 16) &&
           (r->rows == 1 || (stride * c->es % 16 == 0 && stride >= static_cast<int64_t>(heads) * d.head_dim));
  };
  if (!rows_ok(r->k, r->k_stride, d.n_kv_heads) || !rows_ok(r->v, r->v_stride, d.n_kv_heads) || !r->slots ||
      !aligned(r->slots, 8))
    return CLLM_EINVAL;
  if (r->rope && (!aligned(r->rope, 16) || r->max_pos < 1 || !r->positions || !aligned(r->positions, 4)))
    return CLLM_EINVAL;
  if (r->q && ((!r->rope && !heads) || !rows_ok(r->q, r->q_stride, d.n_heads) ||
               !rows_ok(r->q_out, r->q_out_stride, d.n_heads)))
    return CLLM_EINVAL;
  PagedAppendArgs a{};
  a.dims = r->rope ? d.head_dim : 0;
  if (heads) {
    if (!aligned(heads->q_norm, 16) || !aligned(heads->k_norm, 16) || (heads->q_norm && !r->q) ||
        ((heads->q_norm || heads->k_norm) && !(heads->eps >= 0.f && isfinite(heads->eps))) ||
        (!r->rope && !heads->q_norm && !heads->k_norm))
      return CLLM_EINVAL;
    if (r->rope) {
      if (heads->rotary_dims < 1 || heads->rotary_dims > d.head_dim) return CLLM_EINVAL;
      if (heads->rotary_dims % 16) return CLLM_EUNSUPPORTED;
      a.dims = heads->rotary_dims;
      a.interleaved = heads->interleaved != 0;
    }
    a.q_gain = heads->q_norm, a.k_gain = heads->k_norm, a.eps = heads->eps;
  }
  const int64_t at = r->layer * d.stride_layer * c->es;
  a.k = r->k, a.v = r->v, a.q = r->q, a.q_out = r->q_out;
  a.kp = static_cast<char*>(d.k) + at, a.vp = static_cast<char*>(d.v) + at;
  a.k_row = r->k_stride, a.v_row = r->v_stride, a.q_row = r->q_stride, a.qo_row = r->q_out_stride;
  a.s_page = d.stride_page, a.s_head = d.stride_head, a.s_pos = d.stride_pos;
  a.slots = reinterpret_cast<const long long*>(r->slots);
  a.rope = reinterpret_cast<const float2*>(r->rope);
  a.positions = r->positions;
  a.max_pos = r->max_pos, a.T = r->rows, a.H = r->q ? d.n_heads : 0, a.Hkv = d.n_kv_heads, a.hd = d.head_dim;
  a.n_pages = d.n_pages, a.page_shift = c->page_shift;
  a.err = c->err;
  const OnDevice on(c->dev);
  cudaError_t e = on.error;
  if (e == cudaSuccess) e = launch_paged_append(a, d.dtype, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? CLLM_OK : cuda_fail(e, "paged_append");
}

extern "C" int cllm_paged_append(cllm_paged* c, const cllm_paged_rows* r, void* cuda_stream) {
  return append(c, r, nullptr, cuda_stream);
}

extern "C" int cllm_paged_append_heads(cllm_paged* c, const cllm_paged_rows* r, const cllm_paged_heads* heads,
                                       void* cuda_stream) {
  return heads ? append(c, r, heads, cuda_stream) : CLLM_EINVAL;
}

// f / 2 pi modulo 1, in 2^-64: the quotient in two doubles (1 / 2 pi to 2^-109), whole turns taken off
// the first exactly.
static unsigned long long turns_of(double f) {
  constexpr double hi = 0.15915494309189534561, lo = -9.839338337591243e-18;  // 1 / 2 pi
  double t = f * hi;
  const double rest = fma(f, hi, -t) + f * lo;
  t -= nearbyint(t);
  if (t >= 0.5) t -= 1.0;
  return static_cast<unsigned long long>(static_cast<long long>(ldexp(t, 64))) +
         static_cast<unsigned long long>(llrint(ldexp(rest, 64)));
}

extern "C" int cllm_rope_table(float* table, int first, int positions, int dims, const double* frequencies,
                               float amplitude, void* cuda_stream) {
  if ((positions != 0 && !table) || !aligned(table, 16) || first < 0 || positions < 0 || first > 0x7fffffff - positions || dims < 2 ||
      dims > kRopeDims || dims % 2 || !frequencies || !isfinite(amplitude))
    return CLLM_EINVAL;
  unsigned long long turns[kRopeDims / 2];
  for (int i = 0; i < dims / 2; ++i) {
    if (!(fabs(frequencies[i]) <= 1048576.0)) return CLLM_EINVAL;
    turns[i] = turns_of(frequencies[i]);
  }
  if (positions == 0) return CLLM_OK;
  const cudaError_t e =
      launch_rope_table(table, first, positions, dims, turns, amplitude, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? CLLM_OK : cuda_fail(e, "rope_table");
}

extern "C" int cllm_paged_attention(cllm_paged* c, const cllm_paged_attn* p, void* cuda_stream) {
  return cllm_paged_attention_sinks(c, p, 0, cuda_stream);
}

extern "C" int cllm_paged_attention_sinks(cllm_paged* c, const cllm_paged_attn* p, int sinks, void* cuda_stream) {
  if (!c || !p || sinks < 0 || p->layer < 0 || p->layer >= c->d.layers || p->batch < 0 || p->rows < 0) return CLLM_EINVAL;
  if (p->batch == 0 || p->rows == 0) return CLLM_OK;
  const cllm_paged_desc& d = c->d;
  auto strides_ok = [&](const void* x, int64_t row, int64_t head) {
    auto ok = [&](int64_t stride) {
      return stride >= d.head_dim && stride * c->es % 16 == 0 && stride < (int64_t(1) << 37);
    };
    return x && aligned(x, 16) && (p->rows == 1 || ok(row)) && (d.n_heads == 1 || ok(head));
  };
  if (!strides_ok(p->q, p->q_stride, p->q_head_stride) || !strides_ok(p->out, p->out_stride, p->out_head_stride) ||
      p->q == p->out || !p->row_start || !p->seq_len || !p->table || !aligned(p->row_start, 4) || !aligned(p->seq_len, 4) ||
      !aligned(p->table, 4) || !aligned(p->lse, 4) || p->table_width < 1 || p->window < 0 ||
      !(p->scale > 0.f) || !isfinite(p->scale * kLog2e) ||
      static_cast<int64_t>(p->table_width) * d.page_size > 0x7fffffff ||
      (p->mask && (p->mask_words < 1 || !aligned(p->mask, 4))))
    return CLLM_EINVAL;
  // the kernels count (tile, 64 or 128 keys) units in 32 bits; tiles have at least 16 / group tokens
  const int group = d.n_heads / d.n_kv_heads;
  const int64_t tiles = p->rows / (group < 16 ? 16 / group : 1) + p->batch;
  const int64_t chunks = (static_cast<int64_t>(p->table_width) * d.page_size >> 6) + 1;
  if (tiles > 0x7fffffff / (chunks * d.n_kv_heads)) return CLLM_EUNSUPPORTED;
  PagedAttnArgs a{};
  const int64_t at = p->layer * d.stride_layer * c->es;
  a.q = p->q, a.out = p->out, a.lse = p->lse;
  // (one row, or one head, needs no stride)
  a.q_row = p->rows == 1 ? d.head_dim : p->q_stride, a.q_head = d.n_heads == 1 ? d.head_dim : p->q_head_stride;
  a.out_row = p->rows == 1 ? d.head_dim : p->out_stride, a.out_head = d.n_heads == 1 ? d.head_dim : p->out_head_stride;
  a.row_start = p->row_start, a.seq_len = p->seq_len, a.table = p->table;
  a.table_width = p->table_width, a.batch = p->batch, a.rows = p->rows;
  a.H = d.n_heads, a.Hkv = d.n_kv_heads, a.group = group;
  a.scale_log2 = p->scale * kLog2e;
  a.group_inv = (65536 + group - 1) / group;
  a.window = p->window, a.sinks = p->window > 0 ? sinks : 0, a.mask = p->mask, a.mask_words = p->mask_words;
  a.k = static_cast<const char*>(d.k) + at, a.v = static_cast<const char*>(d.v) + at;
  a.s_page = d.stride_page, a.s_head = d.stride_head, a.s_pos = d.stride_pos;
  a.layer = p->layer, a.n_pages = d.n_pages, a.page_shift = c->page_shift;
  a.part_o = c->part_o, a.part_ml = c->part_ml, a.tickets = c->tickets, a.err = c->err;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const OnDevice on(c->dev);
  if (on.error != cudaSuccess) return cuda_fail(on.error, "paged_attention");
  // rows of one key/value head in an average request
  const int64_t rows = (static_cast<int64_t>(p->rows) + p->batch - 1) / p->batch * a.group;
  cudaError_t e;
  if (c->es == 4) {
    e = launch_paged_attention_f32(a, d.head_dim, c->sms, st);
  } else if (group <= kFewRows && (rows <= kFewRows || (rows <= 2 * kFewRows && 2 * p->batch * d.n_kv_heads <= c->sms))) {
    // (a second tile of 16 rows reads its keys again: worth it while SMs are idle.  A block of
    // 32 tokens, 32 heads, 1000 keys 16.1 us against the tensor-memory kernel's 19.6; with
    // 6 requests, SMs busy, 35 and 28)
    e = launch_paged_attention_few(a, c->mk_few, c->mv_few, d.dtype, d.head_dim, c->hold, c->sms, st);
  } else {
    e = launch_paged_attention_tc(a, c->mk, c->mv, d.dtype, d.head_dim, c->hold, c->sms, st);
  }
  return e == cudaSuccess ? CLLM_OK : cuda_fail(e, "paged_attention");
}

extern "C" int cllm_test_paged_device(cllm_paged* c, int dev) {
  if (!c || dev < 0) return CLLM_EINVAL;
  const int before = c->dev;
  c->dev = dev;
  return before;
}

extern "C" int cllm_test_hold_paged(cllm_paged* c, int chunk) {
  if (!c || chunk < -1) return CLLM_EINVAL;
  c->hold = chunk + 1;
  return CLLM_OK;
}
