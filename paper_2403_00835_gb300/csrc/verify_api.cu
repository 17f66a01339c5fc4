// Host side of include/cllm_verify.h: argument checks, the verifier's scratch, and the launch.
#include <new>

#include "internal.cuh"
#include "on_device.cuh"
#include "paged.cuh"
#include "verify.cuh"

using namespace cllm;

struct cllm_verifier {
  int max_rows = 0, max_batch = 0, dev = 0, sms = 0;
  void* scratch = nullptr;
  unsigned long long *shares = nullptr, *best = nullptr;
  int *row_tickets = nullptr, *request_tickets = nullptr;
  VerifyRow* found = nullptr;
};

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
constexpr int kMostRows = 1 << 30;  // (and values of a vocabulary: steps past the last stay in 31 bits)

}  // namespace

extern "C" void cllm_verifier_destroy(cllm_verifier* v) {
  if (!v) return;
  {
    const OnDevice on(v->dev);
    cudaDeviceSynchronize();
    cudaFree(v->scratch);
  }
  delete v;
}

extern "C" int cllm_verifier_create(int max_rows, int max_batch, cllm_verifier** out) {
  if (!out) return CLLM_EINVAL;
  *out = nullptr;
  if (max_rows < 1 || max_rows > kMostRows || max_batch < 1 || max_batch > kPlanBatch) return CLLM_EINVAL;
  int dev = 0, major = 0, minor = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_fail(e, "verifier_create");
  if (major != 10 || minor != 3) return CLLM_EUNSUPPORTED;
  cllm_verifier* v = new (std::nothrow) cllm_verifier;
  if (!v) return CLLM_ENOMEM;
  v->max_rows = max_rows, v->max_batch = max_batch, v->dev = dev, v->sms = sms;
  const size_t rows = max_rows, batch = max_batch;
  const size_t found = rows * sizeof(VerifyRow), shares = (rows + static_cast<size_t>(kVerifyWarps) * sms) * 8, best = batch * 8;
  const size_t counters = (rows + batch) * 4;
  if (lib_malloc(&v->scratch, found + shares + best + counters) != cudaSuccess) {
    v->scratch = nullptr;
    cllm_verifier_destroy(v);
    return CLLM_ENOMEM;
  }
  char* p = static_cast<char*>(v->scratch);
  v->found = reinterpret_cast<VerifyRow*>(p);
  v->shares = reinterpret_cast<unsigned long long*>(p + found);
  v->best = reinterpret_cast<unsigned long long*>(p + found + shares);
  v->row_tickets = reinterpret_cast<int*>(p + found + shares + best);
  v->request_tickets = v->row_tickets + rows;
  // (the default stream orders the clearing before any later work)
  e = cudaMemset(v->best, 0, best + counters);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    cllm_verifier_destroy(v);
    return cuda_fail(e, "verifier_create");
  }
  *out = v;
  return CLLM_OK;
}

extern "C" int cllm_verify(cllm_verifier* v, const cllm_verify_args* p, void* cuda_stream) {
  if (!v || !p || p->batch < 0 || p->batch > v->max_batch || p->rows < 0 || p->rows > v->max_rows || p->vocab < 1 ||
      p->vocab > kMostRows || (p->dtype != CLLM_F32 && p->dtype != CLLM_BF16 && p->dtype != CLLM_F16))
    return CLLM_EINVAL;
  if (p->batch == 0) return CLLM_OK;
  const size_t es = p->dtype == CLLM_F32 ? 4 : 2;
  auto stride_ok = [&](int rows, int64_t stride) { return rows <= 1 || (stride >= p->vocab && stride < (int64_t(1) << 40)); };
  auto given = [](const void* x, size_t n) { return x && aligned(x, n); };
  if (!given(p->row_start, 4) || !given(p->seq_len, 4) || !given(p->accepted, 4) || !given(p->next, 4) ||
      !aligned(p->target_probs, 4) || (p->rows > 0 && (p->race != nullptr) != (p->uniforms != nullptr)) || !aligned(p->race, 4) ||
      !aligned(p->uniforms, 4) || !aligned(p->temperature, 4) || !aligned(p->draft_probs, 4) ||
      (!p->race && (p->temperature || p->draft_probs)) || (p->race && !stride_ok(p->batch, p->race_stride)) ||
      (p->draft_probs && !stride_ok(p->rows, p->probs_stride)))
    return CLLM_EINVAL;
  if (p->rows > 0 && (!given(p->logits, es) || !given(p->tokens, 4) || !stride_ok(p->rows, p->logits_stride)))
    return CLLM_EINVAL;
  VerifyArgs a{};
  a.logits = p->logits, a.tokens = p->tokens, a.row_start = p->row_start, a.seq_len = p->seq_len;
  a.temperature = p->temperature, a.uniforms = p->uniforms, a.race = p->race, a.draft_probs = p->draft_probs;
  a.accepted = p->accepted, a.next = p->next, a.target_probs = p->target_probs;
  // (one row needs no stride)
  a.logits_row = p->rows <= 1 ? 0 : p->logits_stride, a.race_row = p->batch <= 1 ? 0 : p->race_stride;
  a.probs_row = p->rows <= 1 ? 0 : p->probs_stride;
  a.batch = p->batch, a.rows = p->rows, a.vocab = p->vocab;
  a.shares = v->shares, a.row_tickets = v->row_tickets, a.found = v->found, a.best = v->best;
  a.request_tickets = v->request_tickets;
  const OnDevice on(v->dev);
  cudaError_t e = on.error;
  if (e == cudaSuccess) e = launch_verify(a, p->dtype, v->sms, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? CLLM_OK : cuda_fail(e, "verify");
}
