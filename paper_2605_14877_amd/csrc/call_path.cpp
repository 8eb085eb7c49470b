// Python module _heatkv_call: the per-layer calls of binding.py without the interpreter in between.
//
// A generation pass makes one or two library calls per layer and scale, and below about 300 tokens the kernels are
// shorter than the 10 us that operand checks, stream lookup and argument conversion took in Python and ctypes (2.1, 2.9
// and 2.0 us, next to 3.7 us for the library call itself, 3.2 of them the launch).  The functions here do the same
// checks on the tensors and call the library.  They return its error code, or None for anything that is not plainly
// in order: the caller then takes the Python path, which names the mistake.  A tensor may answer a question about itself with
// an exception (one without sizes, a subclass with a sizes policy of its own): that is not plainly in order either.
#include "python_calls.h"

#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <new>
#include <vector>

#include "heatkv.h"

namespace {

constexpr const char* kPlanName = "heatkv_plan_info";

// What the operands of a plan's calls must look like.
struct PlanInfo {
  heatkv_plan* plan;
  int64_t L, H, d, batch, dtype;
  std::vector<int64_t> t;
  int64_t arena_bytes;
};

void free_plan_info(PyObject* capsule) {
  delete static_cast<PlanInfo*>(PyCapsule_GetPointer(capsule, kPlanName));
}

// plan_info(handle, L, H, d, batch, dtype, t, arena_bytes) -> capsule
PyObject* plan_info(PyObject*, PyObject* args) try {
  unsigned long long handle;
  long long L, H, d, batch, dtype, arena_bytes;
  PyObject* t;
  if (!PyArg_ParseTuple(args, "KLLLLLO!L", &handle, &L, &H, &d, &batch, &dtype, &PyTuple_Type, &t, &arena_bytes))
    return nullptr;
  std::vector<int64_t> tokens;
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(t); ++i) {
    const long long n = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    if (n == -1 && PyErr_Occurred()) return nullptr;
    tokens.push_back(n);
  }
  auto* info = new PlanInfo{reinterpret_cast<heatkv_plan*>(handle), L, H, d, batch, dtype, std::move(tokens), arena_bytes};
  PyObject* capsule = PyCapsule_New(info, kPlanName, free_plan_info);
  if (!capsule) delete info;
  return capsule;
} catch (const std::bad_alloc&) {
  return PyErr_NoMemory();
}

// Address and size of a contiguous device tensor; None is a null pointer.
bool device_tensor(PyObject* o, const at::Tensor** tensor, void** ptr) {
  *tensor = nullptr;
  *ptr = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& x = THPVariable_Unpack(o);
  if (!x.is_cuda() || !x.is_contiguous()) return false;
  *tensor = &x;
  *ptr = x.data_ptr();
  return true;
}

bool operand(PyObject* o, at::IntArrayRef shape, int64_t dtype, void** ptr) {
  const at::Tensor* x;
  if (!device_tensor(o, &x, ptr)) return false;
  return !x || (x->scalar_type() == (dtype == HEATKV_BF16 ? at::kBFloat16 : at::kFloat) && x->sizes() == shape);
}

bool buffer(PyObject* o, int64_t min_bytes, void** ptr, size_t* bytes) {
  const at::Tensor* x;
  if (!device_tensor(o, &x, ptr)) return false;
  const int64_t n = x ? x->numel() * static_cast<int64_t>(x->element_size()) : 0;
  if (bytes) *bytes = static_cast<size_t>(n);
  return !x || n >= min_bytes;
}

bool integer(PyObject* o, long* v) {
  *v = PyLong_AsLong(o);
  return !(*v == -1 && PyErr_Occurred());
}

bool number(PyObject* o, float* v) {
  *v = static_cast<float>(PyFloat_AsDouble(o));
  return !PyErr_Occurred();
}

bool stream_of(PyObject* o, void** stream) {
  if (o == Py_None) {
    *stream = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA().stream();
    return true;
  }
  if (!PyLong_Check(o)) return false;
  *stream = PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}

PyObject* not_plain() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// scale_call(plan_info, which, layer, k, q, k_cur, v_cur, k_arena, v_arena, sm_scale, out, ws, stream)
// which: 0 append_scale (q, sm_scale, out and ws unused), 1 attend_scale, 2 attend_append_scale
PyObject* scale_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 13) return not_plain();
  auto* info = static_cast<PlanInfo*>(PyCapsule_GetPointer(a[0], kPlanName));
  long which, layer, k;
  if (!info || !integer(a[1], &which) || !integer(a[2], &layer) || !integer(a[3], &k)) return not_plain();
  if (layer < 0 || layer >= info->L || k < 0 || k >= static_cast<long>(info->t.size())) return not_plain();
  const int64_t shape[4] = {info->batch, info->H, info->t[k], info->d};
  void *q = nullptr, *kc, *vc, *ka, *va, *out = nullptr, *ws = nullptr, *stream;
  size_t ws_bytes = 0;
  float sm = 0.f;
  if (!operand(a[5], shape, info->dtype, &kc) || !operand(a[6], shape, info->dtype, &vc) ||
      !buffer(a[7], info->arena_bytes, &ka, nullptr) || !buffer(a[8], info->arena_bytes, &va, nullptr) ||
      !stream_of(a[12], &stream))
    return not_plain();
  if (which != 0 && (!operand(a[4], shape, info->dtype, &q) || !number(a[9], &sm) ||
                     !operand(a[10], shape, info->dtype, &out) || !buffer(a[11], 0, &ws, &ws_bytes)))
    return not_plain();
  return PyLong_FromLong(heatkv::without_lock([&] {
    if (which == 0) return heatkv_append_scale(info->plan, layer, k, kc, vc, ka, va, stream);
    if (which == 1) return heatkv_attend_scale(info->plan, layer, k, q, kc, vc, ka, va, sm, out, ws, ws_bytes, stream);
    return heatkv_attend_append_scale(info->plan, layer, k, q, kc, vc, ka, va, sm, out, ws, ws_bytes, stream);
  }));
}

const heatkv_shape* shape_at(PyObject* o) {
  const auto* s = static_cast<const heatkv_shape*>(PyLong_AsVoidPtr(o));
  return s && s->t && s->K >= 1 && s->K <= HEATKV_MAX_SCALES ? s : nullptr;
}

bool calibrate_operands(const heatkv_shape* s, long k1, PyObject* q, PyObject* k_all, PyObject* mass, void** qp, void** kp,
                        void** mp) {
  if (k1 < 0 || k1 >= s->K) return false;
  int64_t c = 0;
  for (long k = 0; k <= k1; ++k) c += s->t[k];
  const int64_t q_shape[4] = {s->batch, s->H, s->t[k1], s->d}, k_shape[4] = {s->batch, s->H, c, s->d};
  const int64_t m_shape[3] = {s->batch, s->H, s->K};
  return operand(q, q_shape, s->dtype, qp) && operand(k_all, k_shape, s->dtype, kp) &&
         operand(mass, m_shape, HEATKV_F32, mp);
}

bool beta_operand(const heatkv_shape* s, PyObject* beta, void** ptr) {
  const int64_t shape[4] = {s->L, s->H, s->K, s->K};
  return operand(beta, shape, HEATKV_F32, ptr);
}

// calibrate_call(address of the heatkv_shape, which, layer, k1, q, k_all, sm_scale, weight, beta, mass, ws, stream)
// which: 0 calibrate, 1 calibrate_static (ws unused), 2 calibrate_accumulate
PyObject* calibrate_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 12) return not_plain();
  const heatkv_shape* s = shape_at(a[0]);
  long which, layer, k1;
  float sm, weight;
  void *q, *k_all, *beta, *mass, *ws, *stream;
  size_t ws_bytes;
  if (!s || !integer(a[1], &which) || !integer(a[2], &layer) || !integer(a[3], &k1) || !number(a[6], &sm) ||
      !number(a[7], &weight) || !calibrate_operands(s, k1, a[4], a[5], a[9], &q, &k_all, &mass) ||
      !beta_operand(s, a[8], &beta) || !buffer(a[10], 0, &ws, &ws_bytes) || !stream_of(a[11], &stream))
    return not_plain();
  return PyLong_FromLong(heatkv::without_lock([&] {
    float* const m = static_cast<float*>(mass);
    if (which == 0) return heatkv_calibrate(s, layer, k1, q, k_all, sm, m, ws, ws_bytes, stream);
    if (which == 1) return heatkv_calibrate_static(s, layer, k1, q, k_all, sm, m, stream);
    return heatkv_calibrate_accumulate(s, layer, k1, q, k_all, sm, weight, static_cast<float*>(beta), m, ws, ws_bytes,
                                       stream);
  }));
}

// calibrate_scales_call(address of the heatkv_shape, layer, k1 list, q list, k_all list, sm_scale, weight, beta,
//                       mass list or None, ws, stream); the lists have one length
PyObject* calibrate_scales_call(PyObject* const* a, Py_ssize_t n) {
  if (n != 11) return not_plain();
  const heatkv_shape* s = shape_at(a[0]);
  long layer;
  float sm, weight;
  void *beta, *ws, *stream;
  size_t ws_bytes;
  if (!s || !integer(a[1], &layer) || !PyList_Check(a[2]) || !PyList_Check(a[3]) || !PyList_Check(a[4]) ||
      !(a[8] == Py_None || PyList_Check(a[8])) || !number(a[5], &sm) || !number(a[6], &weight) ||
      !beta_operand(s, a[7], &beta) || !buffer(a[9], 0, &ws, &ws_bytes) || !stream_of(a[10], &stream))
    return not_plain();
  const Py_ssize_t scales = PyList_GET_SIZE(a[2]);
  if (scales < 1 || scales > s->K || PyList_GET_SIZE(a[3]) != scales || PyList_GET_SIZE(a[4]) != scales ||
      (a[8] != Py_None && PyList_GET_SIZE(a[8]) != scales))
    return not_plain();
  int32_t k1[HEATKV_MAX_SCALES];
  void *q[HEATKV_MAX_SCALES], *k_all[HEATKV_MAX_SCALES], *mass[HEATKV_MAX_SCALES];
  for (Py_ssize_t i = 0; i < scales; ++i) {
    long k;
    PyObject* m = a[8] == Py_None ? Py_None : PyList_GET_ITEM(a[8], i);
    if (!integer(PyList_GET_ITEM(a[2], i), &k) ||
        !calibrate_operands(s, k, PyList_GET_ITEM(a[3], i), PyList_GET_ITEM(a[4], i), m, &q[i], &k_all[i], &mass[i]))
      return not_plain();
    k1[i] = static_cast<int32_t>(k);
  }
  return PyLong_FromLong(heatkv::without_lock([&] {
    return heatkv_calibrate_scales_accumulate(s, layer, static_cast<int>(scales), k1, q, k_all, sm, weight,
                                              static_cast<float*>(beta),
                                              a[8] == Py_None ? nullptr : reinterpret_cast<float* const*>(mass), ws, ws_bytes,
                                              stream);
  }));
}

// ---- paged cache: shapes are the address of a heatkv_paged_shape ----

// The tensors of one call: all on the current device, else nothing here is plainly in order.
class PagedCall {
 public:
  PagedCall(PyObject* shape, PyObject* stream) {
    s_ = static_cast<const heatkv_paged_shape*>(PyLong_AsVoidPtr(shape));
    const auto current = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA();
    device_ = current.device_index();
    if (stream == Py_None)
      stream_ = current.stream();
    else
      ok_ = PyLong_Check(stream) && ((stream_ = PyLong_AsVoidPtr(stream)), !PyErr_Occurred());
    ok_ = ok_ && s_;
  }
  bool ok() const { return ok_; }
  const heatkv_paged_shape* shape() const { return s_; }
  void* stream() const { return stream_; }

  const at::Tensor* tensor(PyObject* o) {
    if (!THPVariable_Check(o)) return fail();
    const at::Tensor& x = THPVariable_Unpack(o);
    if (!x.is_cuda() || x.get_device() != device_) return fail();
    return &x;
  }
  // Contiguous, of the type and sizes given.
  void* dense(PyObject* o, at::ScalarType type, at::IntArrayRef sizes) {
    const at::Tensor* x = tensor(o);
    if (!x || x->scalar_type() != type || !x->is_contiguous() || x->sizes() != sizes) return fail_ptr();
    return x->data_ptr();
  }
  int32_t* ints(PyObject* o, at::IntArrayRef sizes) { return static_cast<int32_t*>(dense(o, at::kInt, sizes)); }
  // A one-dimensional int32 tensor of any length.
  int32_t* vector(PyObject* o, int64_t* n) {
    const at::Tensor* x = tensor(o);
    if (!x || x->scalar_type() != at::kInt || x->dim() != 1 || !x->is_contiguous()) return static_cast<int32_t*>(fail_ptr());
    *n = x->size(0);
    return static_cast<int32_t*>(x->data_ptr());
  }
  heatkv_rows rows(PyObject* o, int64_t heads, int64_t* tokens) {  // *tokens < 0: any number
    const at::Tensor* x = tensor(o);
    if (!x || x->scalar_type() != (s_->dtype == HEATKV_BF16 ? at::kBFloat16 : at::kFloat) || x->dim() != 3 ||
        x->size(1) != heads || x->size(2) != s_->d || x->stride(2) != 1 || (*tokens >= 0 && x->size(0) != *tokens)) {
      ok_ = false;
      return heatkv_rows{};
    }
    *tokens = x->size(0);
    return heatkv_rows{x->data_ptr(), x->stride(0), x->stride(1)};
  }
  void* pages(PyObject* o) {
    const at::Tensor* x = tensor(o);
    const int64_t sizes[4] = {s_->num_pages, s_->kv_heads, s_->page_size, s_->d};
    if (!x || !x->is_contiguous() || x->sizes() != at::IntArrayRef(sizes)) return fail_ptr();
    const at::ScalarType t = x->scalar_type();
    const bool fits = s_->kv_format == HEATKV_KV_FP8_E4M3 ? t == at::kFloat8_e4m3fn || t == at::kByte
                                                           : t == (s_->dtype == HEATKV_BF16 ? at::kBFloat16 : at::kFloat);
    return fits ? x->data_ptr() : fail_ptr();
  }

 private:
  const at::Tensor* fail() {
    ok_ = false;
    return nullptr;
  }
  void* fail_ptr() {
    ok_ = false;
    return nullptr;
  }
  const heatkv_paged_shape* s_;
  void* stream_ = nullptr;
  int64_t device_;
  bool ok_ = true;
};

bool boolean(PyObject* o, int* v) {
  *v = o == Py_True;
  return PyBool_Check(o);
}

// paged_assign(shape, keep, new_tokens, lens, ring, span, table, q_start, slots, status, lens_out, span_out, stream)
PyObject* paged_assign(PyObject* const* a, Py_ssize_t n) {
  if (n != 13) return not_plain();
  PagedCall c(a[0], a[12]);
  if (!c.ok()) return not_plain();
  const heatkv_paged_shape* s = c.shape();
  int64_t tokens = 0;
  const int64_t table_size[2] = {s->batch, s->max_pages};
  int32_t *keep = c.ints(a[1], {s->batch}), *come = c.ints(a[2], {s->batch}), *lens = c.ints(a[3], {s->batch});
  int32_t *ring = c.ints(a[4], {s->num_pages}), *span = c.ints(a[5], {2}), *table = c.ints(a[6], table_size);
  int32_t *q_start = c.ints(a[7], {int64_t(s->batch) + 1}), *slots = c.vector(a[8], &tokens), *status = c.ints(a[9], {1});
  int32_t* lens_out = a[10] == Py_None ? lens : c.ints(a[10], {s->batch});
  int32_t* span_out = a[11] == Py_None ? span : c.ints(a[11], {2});
  if (!c.ok()) return not_plain();
  return PyLong_FromLong(heatkv::without_lock([&] {
    return heatkv_paged_assign(s, keep, come, lens, lens_out, ring, span, span_out, table, q_start, slots, tokens, status,
                               c.stream());
  }));
}

// paged_append(shape, slots, k_new, v_new, k_pages, v_pages, bounds, scales, stream)
PyObject* paged_append(PyObject* const* a, Py_ssize_t n) {
  if (n != 9) return not_plain();
  PagedCall c(a[0], a[8]);
  if (!c.ok()) return not_plain();
  const heatkv_paged_shape* s = c.shape();
  int64_t tokens = 0;
  const int32_t* slots = c.vector(a[1], &tokens);
  const heatkv_rows k = c.rows(a[2], s->kv_heads, &tokens), v = c.rows(a[3], s->kv_heads, &tokens);
  void *kp = c.pages(a[4]), *vp = c.pages(a[5]);
  void* bounds = a[6] == Py_None ? nullptr : c.dense(a[6], at::kChar, {s->num_pages, s->kv_heads, 2, s->d});
  void* scales = a[7] == Py_None ? nullptr : c.dense(a[7], at::kFloat, {s->num_pages, s->kv_heads});
  if (!c.ok()) return not_plain();
  return PyLong_FromLong(heatkv::without_lock([&] {
    return heatkv_paged_append(s, slots, tokens, k, v, kp, vp, static_cast<int8_t*>(bounds), static_cast<float*>(scales),
                               c.stream());
  }));
}

// paged_attend(shape, q, k_pages, v_pages, table, q_start, lens, selected, sm_scale, out, ws, causal, lse, stream)
PyObject* paged_attend(PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return not_plain();
  PagedCall c(a[0], a[13]);
  if (!c.ok()) return not_plain();
  const heatkv_paged_shape* s = c.shape();
  int64_t tokens = -1, top = 0;
  float sm;
  int causal;
  const heatkv_rows q = c.rows(a[1], s->q_heads, &tokens);
  void *kp = c.pages(a[2]), *vp = c.pages(a[3]);
  const int32_t *table = c.ints(a[4], {s->batch, s->max_pages}), *q_start = c.ints(a[5], {int64_t(s->batch) + 1}),
                *lens = c.ints(a[6], {s->batch});
  const heatkv_rows out = c.rows(a[9], s->q_heads, &tokens);
  void* lse = a[12] == Py_None ? nullptr : c.dense(a[12], at::kFloat, {tokens, s->q_heads});
  const int32_t* selected = nullptr;
  const bool chosen = a[7] != Py_None;  // a tensor without elements has a null address
  if (chosen) {
    const at::Tensor* x = c.tensor(a[7]);
    if (!x || x->dim() != 3) return not_plain();
    top = x->size(2);
    selected = c.ints(a[7], {tokens, s->kv_heads, top});
  }
  void* ws;
  size_t ws_bytes;
  if (!number(a[8], &sm) || !boolean(a[11], &causal) || !buffer(a[10], 0, &ws, &ws_bytes) || !c.ok()) return not_plain();
  if (a[10] != Py_None && !c.tensor(a[10])) return not_plain();
  return PyLong_FromLong(heatkv::without_lock([&] {
    if (chosen)
      return heatkv_paged_attend_selected(s, tokens, q, kp, vp, table, q_start, lens, selected, static_cast<int>(top), sm, causal,
                                          out, static_cast<float*>(lse), ws, ws_bytes, c.stream());
    return heatkv_paged_attend(s, tokens, q, kp, vp, table, q_start, lens, sm, causal, out, static_cast<float*>(lse), ws, ws_bytes,
                               c.stream());
  }));
}

// paged_select(shape, q, bounds, scales, table, q_start, lens, first, last, selected, causal, stream)
PyObject* paged_select(PyObject* const* a, Py_ssize_t n) {
  if (n != 12) return not_plain();
  PagedCall c(a[0], a[11]);
  if (!c.ok()) return not_plain();
  const heatkv_paged_shape* s = c.shape();
  int64_t tokens = -1;
  long first, last;
  int causal;
  const heatkv_rows q = c.rows(a[1], s->q_heads, &tokens);
  const void* bounds = c.dense(a[2], at::kChar, {s->num_pages, s->kv_heads, 2, s->d});
  const void* scales = c.dense(a[3], at::kFloat, {s->num_pages, s->kv_heads});
  const int32_t *table = c.ints(a[4], {s->batch, s->max_pages}), *q_start = c.ints(a[5], {int64_t(s->batch) + 1}),
                *lens = c.ints(a[6], {s->batch});
  const at::Tensor* x = c.tensor(a[9]);
  if (!x || x->dim() != 3) return not_plain();
  const int64_t top = x->size(2);
  int32_t* selected = c.ints(a[9], {tokens, s->kv_heads, top});
  if (!integer(a[7], &first) || !integer(a[8], &last) || !boolean(a[10], &causal) || !c.ok() || top > INT32_MAX ||
      first != static_cast<int>(first) || last != static_cast<int>(last))
    return not_plain();
  return PyLong_FromLong(heatkv::without_lock([&] {
    return heatkv_paged_select(s, tokens, q, static_cast<const int8_t*>(bounds), static_cast<const float*>(scales), table, q_start,
                               lens, static_cast<int>(first), static_cast<int>(last), static_cast<int>(top), causal, selected,
                               c.stream());
  }));
}

PyMethodDef methods[] = {{"plan_info", plan_info, METH_VARARGS, nullptr},
                         {"scale_call", heatkv::fastcall<scale_call>(), METH_FASTCALL, nullptr},
                         {"calibrate_call", heatkv::fastcall<calibrate_call>(), METH_FASTCALL, nullptr},
                         {"calibrate_scales_call", heatkv::fastcall<calibrate_scales_call>(), METH_FASTCALL, nullptr},
                         {"paged_assign", heatkv::fastcall<paged_assign>(), METH_FASTCALL, nullptr},
                         {"paged_append", heatkv::fastcall<paged_append>(), METH_FASTCALL, nullptr},
                         {"paged_attend", heatkv::fastcall<paged_attend>(), METH_FASTCALL, nullptr},
                         {"paged_select", heatkv::fastcall<paged_select>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_heatkv_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__heatkv_call() { return PyModule_Create(&module); }
