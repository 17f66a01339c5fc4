// Arguments of PagedCache.append and attention, rope_table and DraftVerifier.verify from torch tensors
// to include/cllm_paged.h and cllm_verify.h, for calls whose GPU time is shorter than Python's look at nine
// tensors (append of 16 rows: 2.2 us on the GPU, a call 8.2 us in Python, 2.6 here; verify of 4 rows 8.2 and 4).
//
// The functions answer with the library's status, or with None where an argument is not what the
// call takes: the caller then looks at them in Python, whose errors say what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/cllm_paged.h"
#include "../../include/cllm_verify.h"

namespace {

struct Cache {  // as the caller packs it: "@4P6i"
  int (*plain)(cllm_paged*, const cllm_paged_rows*, void*);
  int (*with_heads)(cllm_paged*, const cllm_paged_rows*, const cllm_paged_heads*, void*);
  int (*attention)(cllm_paged*, const cllm_paged_attn*, int, void*);
  cllm_paged* handle;
  int dtype, device, head_dim, n_kv_heads, n_heads, unused;
};
at::ScalarType type_of(const Cache& c) {
  return c.dtype == CLLM_F32 ? at::kFloat : c.dtype == CLLM_BF16 ? at::kBFloat16 : at::kHalf;
}

const at::Tensor* tensor(PyObject* o, at::ScalarType type, int device) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.scalar_type() == type && t.is_cuda() && t.get_device() == device ? &t : nullptr;
}
// rows of heads side by side
bool heads(PyObject* o, const Cache& c, at::ScalarType type, int64_t rows, int n, const void** p, int64_t* stride) {
  const at::Tensor* t = tensor(o, type, c.device);
  if (!t || t->dim() != 3) return false;
  const auto size = t->sizes(), step = t->strides();
  if (size[0] != rows || size[1] != n || size[2] != c.head_dim || step[2] != 1 || (step[1] != c.head_dim && n != 1))
    return false;
  *p = t->data_ptr();
  *stride = step[0];
  return true;
}
bool vector(PyObject* o, at::ScalarType type, int device, int64_t least, const void** p) {
  const at::Tensor* t = tensor(o, type, device);
  if (!t || !t->is_contiguous() || t->numel() < least) return false;
  *p = t->data_ptr();
  return true;
}
bool gain(PyObject* o, const Cache& c, at::ScalarType type, const void** p) {
  return o == Py_None ||
         (vector(o, type, c.device, c.head_dim, p) && THPVariable_Unpack(o).dim() == 1 && THPVariable_Unpack(o).size(0) == c.head_dim);
}

// The library's call, without the interpreter's lock (a launch may wait for room in the stream).
template <class F>
PyObject* called(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call();
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

// append(cache, layer, k, v, slots, q, q_out, rope, positions, q_norm, k_norm, eps, interleaved, stream)
PyObject* append_checked(PyObject* const* a) {
  if (!PyBytes_CheckExact(a[0]) || PyBytes_GET_SIZE(a[0]) != sizeof(Cache)) Py_RETURN_NONE;
  Cache c;
  memcpy(&c, PyBytes_AS_STRING(a[0]), sizeof c);
  const at::ScalarType type = type_of(c);
  if (!PyLong_CheckExact(a[1]) || !PyFloat_CheckExact(a[11]) || !PyBool_Check(a[12]) || !PyLong_CheckExact(a[13])) Py_RETURN_NONE;
  int far = 0;
  const long layer = PyLong_AsLongAndOverflow(a[1], &far);
  if (far || layer < 0 || layer > 0x7fffffff) Py_RETURN_NONE;
  void* stream = PyLong_AsVoidPtr(a[13]);
  if (stream == nullptr && PyErr_Occurred()) return nullptr;

  const at::Tensor* k = tensor(a[2], type, c.device);
  if (!k || k->dim() != 3 || k->size(0) > 0x7fffffff) Py_RETURN_NONE;
  const int64_t t = k->size(0);
  cllm_paged_rows r{};
  r.layer = static_cast<int>(layer);
  r.rows = static_cast<int>(t);
  const void* p = nullptr;
  if (!heads(a[2], c, type, t, c.n_kv_heads, &r.k, &r.k_stride) || !heads(a[3], c, type, t, c.n_kv_heads, &r.v, &r.v_stride) ||
      !vector(a[4], at::kLong, c.device, t, &p))
    Py_RETURN_NONE;
  r.slots = static_cast<const int64_t*>(p);
  cllm_paged_heads h{};
  if (!gain(a[9], c, type, &h.q_norm) || !gain(a[10], c, type, &h.k_norm)) Py_RETURN_NONE;
  const bool normed = h.q_norm || h.k_norm, rotated = a[7] != Py_None;
  h.eps = static_cast<float>(PyFloat_AS_DOUBLE(a[11]));
  h.interleaved = a[12] == Py_True;
  if (rotated) {
    const at::Tensor* table = tensor(a[7], at::kFloat, c.device);
    if (!table || table->dim() != 3 || !table->is_contiguous() || table->size(2) != 2 || table->size(1) < 1 ||
        2 * table->size(1) > c.head_dim || table->size(0) > 0x7fffffff || !vector(a[8], at::kInt, c.device, t, &p))
      Py_RETURN_NONE;
    r.rope = static_cast<const float*>(table->data_ptr());
    r.positions = static_cast<const int32_t*>(p);
    r.max_pos = static_cast<int>(table->size(0));
    h.rotary_dims = static_cast<int>(2 * table->size(1));
  }
  if (a[5] != Py_None) {
    if ((!normed && !rotated) || !heads(a[5], c, type, t, c.n_heads, &r.q, &r.q_stride)) Py_RETURN_NONE;
    const void* to = r.q;
    r.q_out_stride = r.q_stride;
    if (a[6] != Py_None && !heads(a[6], c, type, t, c.n_heads, &to, &r.q_out_stride)) Py_RETURN_NONE;
    r.q_out = const_cast<void*>(to);
  } else if (h.q_norm) {
    Py_RETURN_NONE;
  }
  const bool whole = !rotated || (h.rotary_dims == c.head_dim && !h.interleaved);
  return called([&] { return !normed && whole ? c.plain(c.handle, &r, stream) : c.with_heads(c.handle, &r, &h, stream); });
}

PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) Py_RETURN_NONE;
  try {
    return append_checked(a);
  } catch (...) {  // (a tensor without memory of its own, for one)
    Py_RETURN_NONE;
  }
}

// rope_table(call, positions, frequencies, amplitude, first, out, device, stream); device: the current one
PyObject* rope_checked(PyObject* const* a) {
  if (!PyLong_CheckExact(a[0]) || !PyLong_CheckExact(a[1]) || !PyFloat_CheckExact(a[3]) || !PyLong_CheckExact(a[4]) ||
      !PyLong_CheckExact(a[6]) || !PyLong_CheckExact(a[7]))
    Py_RETURN_NONE;
  using Call = int (*)(float*, int, int, int, const double*, float, void*);
  const Call call = reinterpret_cast<Call>(PyLong_AsVoidPtr(a[0]));
  int far1 = 0, far2 = 0, far3 = 0;
  const long positions = PyLong_AsLongAndOverflow(a[1], &far1), first = PyLong_AsLongAndOverflow(a[4], &far2);
  const long device = PyLong_AsLongAndOverflow(a[6], &far3);
  void* stream = PyLong_AsVoidPtr(a[7]);
  if ((call == nullptr || stream == nullptr) && PyErr_Occurred()) return nullptr;
  if (far1 || far2 || far3 || positions < 0 || first < 0 || positions > 0x7fffffff || first > 0x7fffffff - positions || device < 0 ||
      device > 0x7fffffff)
    Py_RETURN_NONE;
  const at::Tensor* out = tensor(a[5], at::kFloat, static_cast<int>(device));
  if (!out || out->dim() != 3 || !out->is_contiguous() || out->size(0) != positions || out->size(2) != 2) Py_RETURN_NONE;
  double f[128];
  const int64_t pairs = out->size(1);
  if (pairs < 1 || pairs > 128) Py_RETURN_NONE;
  if (PyList_CheckExact(a[2])) {
    if (PyList_GET_SIZE(a[2]) != pairs) Py_RETURN_NONE;
    for (int64_t i = 0; i < pairs; ++i) {
      PyObject* x = PyList_GET_ITEM(a[2], i);
      if (!PyFloat_CheckExact(x)) Py_RETURN_NONE;
      f[i] = PyFloat_AS_DOUBLE(x);
    }
  } else {  // array("d")
    Py_buffer b;
    if (PyObject_GetBuffer(a[2], &b, PyBUF_FORMAT | PyBUF_ND) != 0) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    const bool ok = b.ndim == 1 && b.format && strcmp(b.format, "d") == 0 && b.len == pairs * 8;
    if (ok) memcpy(f, b.buf, b.len);
    PyBuffer_Release(&b);
    if (!ok) Py_RETURN_NONE;
  }
  float* to = static_cast<float*>(out->data_ptr());
  const float amplitude = static_cast<float>(PyFloat_AS_DOUBLE(a[3]));
  return called([&] {
    return call(to, static_cast<int>(first), static_cast<int>(positions), static_cast<int>(2 * pairs), f, amplitude, stream);
  });
}

PyObject* rope_table(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8) Py_RETURN_NONE;
  try {
    return rope_checked(a);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// attention(cache, layer, q, out, lse, row_start, seq_len, batch, table, width, scale, window, sinks, mask, stream)
PyObject* attention_checked(PyObject* const* a) {
  if (!PyBytes_CheckExact(a[0]) || PyBytes_GET_SIZE(a[0]) != sizeof(Cache) || !PyFloat_CheckExact(a[10])) Py_RETURN_NONE;
  Cache c;
  memcpy(&c, PyBytes_AS_STRING(a[0]), sizeof c);
  long n[15] = {};
  for (int i : {1, 7, 9, 11, 12}) {
    int far = 0;
    if (!PyLong_CheckExact(a[i])) Py_RETURN_NONE;
    n[i] = PyLong_AsLongAndOverflow(a[i], &far);
    if (far || n[i] < 0 || n[i] > 0x7fffffff) Py_RETURN_NONE;
  }
  for (int i : {5, 6, 8, 14})
    if (!PyLong_CheckExact(a[i])) Py_RETURN_NONE;
  cllm_paged_attn p{};
  p.row_start = static_cast<const int32_t*>(PyLong_AsVoidPtr(a[5]));
  p.seq_len = static_cast<const int32_t*>(PyLong_AsVoidPtr(a[6]));
  p.table = static_cast<const int32_t*>(PyLong_AsVoidPtr(a[8]));
  void* stream = PyLong_AsVoidPtr(a[14]);
  if (PyErr_Occurred()) return nullptr;
  const at::ScalarType type = type_of(c);
  const at::Tensor *q = tensor(a[2], type, c.device), *out = tensor(a[3], type, c.device);
  if (!q || !out || q->dim() != 3 || q->size(0) > 0x7fffffff || q->size(1) != c.n_heads || q->size(2) != c.head_dim ||
      q->stride(2) != 1 || out->sizes() != q->sizes() || out->stride(2) != 1)
    Py_RETURN_NONE;
  const int64_t t = q->size(0);
  p.layer = static_cast<int>(n[1]), p.batch = static_cast<int>(n[7]), p.rows = static_cast<int>(t);
  p.q = q->data_ptr(), p.out = out->data_ptr();
  p.q_stride = q->stride(0), p.q_head_stride = q->stride(1), p.out_stride = out->stride(0), p.out_head_stride = out->stride(1);
  if (a[4] != Py_None) {
    const at::Tensor* lse = tensor(a[4], at::kFloat, c.device);
    if (!lse || lse->dim() != 2 || lse->size(0) != t || lse->size(1) != c.n_heads || !lse->is_contiguous()) Py_RETURN_NONE;
    p.lse = static_cast<float*>(lse->data_ptr());
  }
  if (a[13] != Py_None) {
    const at::Tensor* mask = tensor(a[13], at::kInt, c.device);
    if (!mask || mask->dim() != 2 || mask->size(0) != t || mask->size(1) < 1 || mask->size(1) > 0x7fffffff || !mask->is_contiguous())
      Py_RETURN_NONE;
    p.mask = static_cast<const uint32_t*>(mask->data_ptr());
    p.mask_words = static_cast<int>(mask->size(1));
  }
  p.table_width = static_cast<int>(n[9]);
  p.scale = static_cast<float>(PyFloat_AS_DOUBLE(a[10]));
  p.window = static_cast<int>(n[11]);
  const int sinks = static_cast<int>(n[12]);
  return called([&] { return c.attention(c.handle, &p, sinks, stream); });
}

PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 15) Py_RETURN_NONE;
  try {
    return attention_checked(a);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

struct Verifier {  // as the caller packs it: "@2P2i"
  int (*call)(cllm_verifier*, const cllm_verify_args*, void*);
  cllm_verifier* handle;
  int device, unused;
};

// [rows][vocab] or more rows, contiguous each
bool rows_of(PyObject* o, at::ScalarType type, int device, int64_t rows, int64_t vocab, const void** p, int64_t* stride) {
  const at::Tensor* t = tensor(o, type, device);
  if (!t || t->dim() != 2 || t->size(0) < rows || t->size(1) != vocab || (t->stride(1) != 1 && vocab != 1)) return false;
  *p = t->data_ptr();
  *stride = t->stride(0);
  return true;
}
template <class T>
bool values(PyObject* o, at::ScalarType type, int device, int64_t least, T** p) {
  const void* q = nullptr;
  if (!vector(o, type, device, least, &q)) return false;
  *p = static_cast<T*>(const_cast<void*>(q));
  return true;
}

// verify(verifier, batch, row_start, seq_len, logits, tokens, uniforms, race, temperature, draft_probs, accepted, next,
//        target_probs, stream)
PyObject* verify_checked(PyObject* const* a) {
  if (!PyBytes_CheckExact(a[0]) || PyBytes_GET_SIZE(a[0]) != sizeof(Verifier)) Py_RETURN_NONE;
  Verifier v;
  memcpy(&v, PyBytes_AS_STRING(a[0]), sizeof v);
  for (int i : {1, 2, 3, 13})
    if (!PyLong_CheckExact(a[i])) Py_RETURN_NONE;
  int far = 0;
  const long batch = PyLong_AsLongAndOverflow(a[1], &far);
  const void *start = PyLong_AsVoidPtr(a[2]), *len = PyLong_AsVoidPtr(a[3]);
  void* stream = PyLong_AsVoidPtr(a[13]);
  if (PyErr_Occurred()) return nullptr;
  if (far || batch < 0 || batch > 0x7fffffff || !THPVariable_Check(a[4])) Py_RETURN_NONE;
  const at::ScalarType type = THPVariable_Unpack(a[4]).scalar_type();
  const at::Tensor* z = tensor(a[4], type, v.device);
  if (!z || z->dim() != 2 || z->size(0) > 0x7fffffff || z->size(1) > 0x7fffffff ||
      (type != at::kFloat && type != at::kBFloat16 && type != at::kHalf))
    Py_RETURN_NONE;
  const int64_t t = z->size(0), vocab = z->size(1);
  cllm_verify_args p{};
  p.batch = static_cast<int>(batch), p.rows = static_cast<int>(t), p.vocab = static_cast<int>(vocab);
  p.dtype = type == at::kFloat ? CLLM_F32 : type == at::kBFloat16 ? CLLM_BF16 : CLLM_F16;
  p.row_start = static_cast<const int32_t*>(start), p.seq_len = static_cast<const int32_t*>(len);
  const void *race = nullptr, *probs = nullptr;
  auto given = [](PyObject* o) { return o != Py_None; };
  if (!rows_of(a[4], type, v.device, t, vocab, &p.logits, &p.logits_stride) || !values(a[5], at::kInt, v.device, t, &p.tokens) ||
      (given(a[6]) && !values(a[6], at::kFloat, v.device, t, &p.uniforms)) ||
      (given(a[7]) && !rows_of(a[7], at::kFloat, v.device, batch, vocab, &race, &p.race_stride)) ||
      (given(a[8]) && !values(a[8], at::kFloat, v.device, batch, &p.temperature)) ||
      (given(a[9]) && !rows_of(a[9], at::kFloat, v.device, t, vocab, &probs, &p.probs_stride)) ||
      !values(a[10], at::kInt, v.device, batch, &p.accepted) || !values(a[11], at::kInt, v.device, batch, &p.next) ||
      (given(a[12]) && !values(a[12], at::kFloat, v.device, t, &p.target_probs)))
    Py_RETURN_NONE;
  p.race = static_cast<const float*>(race), p.draft_probs = static_cast<const float*>(probs);
  return called([&] { return v.call(v.handle, &p, stream); });
}

PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) Py_RETURN_NONE;
  try {
    return verify_checked(a);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {{"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attention)), METH_FASTCALL, nullptr},
                         {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, nullptr},
                         {"rope_table", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rope_table)), METH_FASTCALL, nullptr},
                         {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
