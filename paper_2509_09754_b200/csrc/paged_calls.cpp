// The paged cache's calls from Python: looks into the tensors, refuses those that do not fit, and calls the C functions of
// lava.h, on the current stream unless another one is given.  It exists for the host's time: a decode step is two short
// calls per layer, and of 9 us that one took from Python through ctypes 5 went into the tensors' attributes and the
// arguments' conversion; the rest is the launch.  The functions here take plain positional arguments from paged.py.
#include <Python.h>

#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "lava.h"

namespace {

PyObject* g_error = nullptr;  // LavaError(status, message)

PyObject* raise_error(int status, const std::string& message) {
  PyObject* e = PyObject_CallFunction(g_error, "is", status, message.c_str());
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}

std::string shape_text(at::IntArrayRef shape) {
  std::string s = "(";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + ")";
}

at::ScalarType type_of(int dtype) {
  return dtype == LAVA_F32 ? at::kFloat : dtype == LAVA_BF16 ? at::kBFloat16 : at::ScalarType::Undefined;
}

// One call: its arguments one after the other.  After a refusal an exception is set and the call is dead.
class Call {
 public:
  Call(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected) : args_(args) {
    if (n != expected) {
      PyErr_Format(PyExc_TypeError, "%zd arguments were given, %zd are taken", n, expected);
      ok_ = false;
    }
  }
  bool ok() const { return ok_; }
  PyObject* peek() const { return args_[at_]; }
  bool none() {  // skips an argument that is None
    if (!ok_ || args_[at_] != Py_None) return false;
    ++at_;
    return true;
  }
  template <class T>
  const T* desc() {  // the address of a descriptor
    void* p = ok_ ? PyLong_AsVoidPtr(args_[at_++]) : nullptr;
    if (ok_ && !p) {
      if (!PyErr_Occurred()) raise_error(LAVA_ERR_INVALID_ARG, "a descriptor is NULL");
      ok_ = false;
    }
    return static_cast<const T*>(p);
  }
  long long integer(const char* name, long long most) {  // |x| <= most
    if (!ok_) return 0;
    int over = 0;
    const long long x = PyLong_AsLongLongAndOverflow(args_[at_++], &over);
    if (x == -1 && !over && PyErr_Occurred()) ok_ = false;
    else if (over || x > most || x < -most - 1) refuse(std::string(name) + " is out of range");
    return ok_ ? x : 0;
  }
  int int32(const char* name) { return (int)integer(name, 0x7fffffffLL); }
  // the next argument as a tensor, nullptr after a refusal
  const at::Tensor* tensor(const char* name) {
    if (!ok_) return nullptr;
    PyObject* o = args_[at_++];
    if (!THPVariable_Check(o)) {
      refuse(std::string(name) + " must be a tensor");
      return nullptr;
    }
    return &THPVariable_Unpack(o);
  }
  bool here(const at::Tensor& t) {  // on the current device
    if (!t.is_cuda()) return false;
    if (device_ < 0) device_ = c10::cuda::current_device();
    return t.get_device() == device_;
  }
  // the next argument, which the call writes to
  const at::Tensor* output(const char* name) {
    const at::Tensor* t = tensor(name);
    if (t && without_gradient(name, *t)) written_[n_written_++] = t;
    return ok_ ? t : nullptr;
  }
  // The calls write through addresses, which autograd does not see: a tensor that it follows is refused.
  bool without_gradient(const char* name, const at::Tensor& t) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
      refuse(std::string(name) + " requires a gradient, which this call does not follow: torch.no_grad(), or its own backward");
    return ok_;
  }
  // After the call: autograd asks whether what it saved was written to since.
  void bump_versions() const {
    for (int i = 0; i < n_written_; ++i)
      if (!written_[i]->is_inference()) written_[i]->unsafeGetTensorImpl()->bump_version();
  }
  // the address of a contiguous tensor of this type and shape on the current device
  void* buffer(const char* name, at::ScalarType type, std::initializer_list<int64_t> shape) {
    return buffer(name, tensor(name), type, shape);
  }
  void* written(const char* name, at::ScalarType type, std::initializer_list<int64_t> shape) {
    return buffer(name, output(name), type, shape);
  }
  void* buffer(const char* name, const at::Tensor* t, at::ScalarType type, std::initializer_list<int64_t> shape) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != at::IntArrayRef(shape) || !here(*t) || !t->is_contiguous()) {
      refuse(std::string(name) + " must be a " + c10::toString(type) + " tensor of shape " + shape_text(shape) +
             ", contiguous, on the current device (got " + c10::toString(t->scalar_type()) + " " + shape_text(t->sizes()) + ")");
      return nullptr;
    }
    return t->data_ptr();
  }
  // [tokens, heads, dim] vectors with contiguous elements
  struct Vectors {
    void* at;
    int64_t tok, head;
  };
  Vectors vectors(const char* name, at::ScalarType type, int64_t tokens, int64_t heads, int64_t dim) {
    return vectors(name, tensor(name), type, tokens, heads, dim);
  }
  Vectors vectors(const char* name, const at::Tensor* t, at::ScalarType type, int64_t tokens, int64_t heads, int64_t dim) {
    if (!t) return {};
    if (t->scalar_type() != type || t->sizes() != at::IntArrayRef({tokens, heads, dim}) || t->stride(2) != 1 || !here(*t)) {
      refuse(std::string(name) + " must be a " + c10::toString(type) + " tensor of shape " + shape_text({tokens, heads, dim}) +
             " with contiguous vectors, on the current device (got " + c10::toString(t->scalar_type()) + " " +
             shape_text(t->sizes()) + ")");
      return {};
    }
    return {t->data_ptr(), t->stride(0), t->stride(1)};
  }
  void* status_word() {  // the first bytes of a workspace, an int32, or None
    if (none()) return nullptr;
    const at::Tensor* t = tensor("status_word");
    if (!t) return nullptr;
    if ((int64_t)t->nbytes() < 4 || !here(*t) || !t->is_contiguous()) {
      refuse("status_word must have 4 bytes on the current device");
      return nullptr;
    }
    return t->data_ptr();
  }
  void* stream() {  // a stream's handle, or None for the current stream
    if (!ok_) return nullptr;
    PyObject* o = args_[at_++];
    if (o != Py_None) {
      void* p = PyLong_AsVoidPtr(o);
      if (!p && PyErr_Occurred()) ok_ = false;
      return p;
    }
    if (device_ < 0) device_ = c10::cuda::current_device();
    return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device_).stream();
  }
  void refuse(const std::string& message) {
    if (ok_) raise_error(LAVA_ERR_INVALID_ARG, message);
    ok_ = false;
  }

 private:
  PyObject* const* args_;
  Py_ssize_t at_ = 0;
  bool ok_ = true;
  int device_ = -1;
  const at::Tensor* written_[4] = {};
  int n_written_ = 0;
};

// Runs the C function without the interpreter's lock.
template <class F>
PyObject* finish(const Call& c, const F& f, bool writes = true) {
  lava_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  if (st != LAVA_OK) return raise_error(st, lava_last_error());
  if (writes) c.bump_versions();
  Py_RETURN_NONE;
}

// torch's own complaints become exceptions of Python.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(args, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyObject* page_admit(PyObject* const* args, Py_ssize_t n) {
  Call c(args, n, 12);
  const auto* d = c.desc<lava_cache_desc>();
  const int first_seq = c.int32("first_seq");
  if (!c.ok()) return nullptr;
  const int64_t L = d->n_layers, B = d->batch, H = d->n_kv_heads;
  int64_t n_seqs = 0;
  if (THPVariable_Check(c.peek())) {
    const at::Tensor& t = THPVariable_Unpack(c.peek());
    n_seqs = t.dim() == 3 ? t.size(1) : 0;
  }
  if (n_seqs > 0x7fffffff) c.refuse("head_offsets has too many sequences");
  const auto* hoff = (const int32_t*)c.buffer("head_offsets", at::kInt, {L, n_seqs, H + 1});
  auto* rows = (int32_t*)c.buffer("head_rows", at::kInt, {L, B, H});
  auto* table = (int32_t*)c.buffer("page_table", at::kInt, {L, B, H, d->max_pages});
  auto* ring = (int32_t*)c.buffer("free_pages", at::kInt, {d->n_pages});
  auto* counters = (int64_t*)c.buffer("counters", at::kLong, {2});
  auto* first_row = (int32_t*)c.buffer("first_row", at::kInt, {L, n_seqs, H});
  auto* status = (uint32_t*)c.status_word();
  auto* rows_out = c.none() ? rows : (int32_t*)c.buffer("head_rows_out", at::kInt, {L, B, H});
  auto* counters_out = c.none() ? counters : (int64_t*)c.buffer("counters_out", at::kLong, {2});
  void* stream = c.stream();
  if (!c.ok()) return nullptr;
  return finish(c, [&] {
    return lava_page_admit(d, first_seq, (int32_t)n_seqs, hoff, rows, rows_out, table, ring, counters, counters_out,
                           first_row, status, stream);
  });
}

PyObject* page_extend(PyObject* const* args, Py_ssize_t n) {
  Call c(args, n, 11);
  const auto* d = c.desc<lava_cache_desc>();
  if (!c.ok()) return nullptr;
  const int64_t L = d->n_layers, B = d->batch, H = d->n_kv_heads;
  const auto* add = (const int32_t*)c.buffer("add", at::kInt, {B});
  auto* rows = (int32_t*)c.buffer("head_rows", at::kInt, {L, B, H});
  auto* table = (int32_t*)c.buffer("page_table", at::kInt, {L, B, H, d->max_pages});
  auto* ring = (int32_t*)c.buffer("free_pages", at::kInt, {d->n_pages});
  auto* counters = (int64_t*)c.buffer("counters", at::kLong, {2});
  int64_t max_add = 0;
  if (c.ok() && THPVariable_Check(c.peek())) {
    const at::Tensor& t = THPVariable_Unpack(c.peek());
    max_add = t.dim() == 4 ? t.size(2) : 0;
  }
  if (max_add > 0x7fffffff) c.refuse("slots has too many rows");
  auto* slots = (int32_t*)c.buffer("slots", at::kInt, {L, B, max_add, H});
  auto* status = (uint32_t*)c.status_word();
  auto* rows_out = c.none() ? rows : (int32_t*)c.buffer("head_rows_out", at::kInt, {L, B, H});
  auto* counters_out = c.none() ? counters : (int64_t*)c.buffer("counters_out", at::kLong, {2});
  void* stream = c.stream();
  if (!c.ok()) return nullptr;
  return finish(c, [&] {
    return lava_page_extend(d, add, (int32_t)max_add, rows, rows_out, table, ring, counters, counters_out, slots, status,
                            stream);
  });
}

// The compaction, or what it refuses alone.
template <bool CHECK>
PyObject* compact_pages(PyObject* const* args, Py_ssize_t n) {
  Call c(args, n, 14);
  const auto* layer = c.desc<lava_layer_desc>();
  const auto* d = c.desc<lava_cache_desc>();
  const int first_seq = c.int32("first_seq");
  if (!c.ok()) return nullptr;
  const int64_t L = d->n_layers, H = d->n_kv_heads, D = d->head_dim, T = layer->total_tokens, S = layer->batch;
  const at::ScalarType type = type_of(d->dtype);
  const char* names[2] = {"k", "v"};
  const int64_t by_head[2] = {layer->k_stride_head, layer->v_stride_head}, by_tok[2] = {layer->k_stride_tok, layer->v_stride_tok};
  const at::Tensor* kv[2] = {};
  for (int i = 0; i < 2; ++i) {
    const at::Tensor* t = kv[i] = c.tensor(names[i]);
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != at::IntArrayRef({L, H, T, D}) || t->stride(3) != 1 || !c.here(*t))
      c.refuse(std::string(names[i]) + " must be a " + c10::toString(type) + " tensor of shape " + shape_text({L, H, T, D}) +
               " with contiguous rows, on the current device");
    else if ((H > 1 && t->stride(1) != by_head[i]) || (T > 1 && t->stride(2) != by_tok[i]))
      c.refuse(std::string(names[i]) + " does not have the strides that desc names");
  }
  const long long k_ls = c.integer("k_layer_stride", INT64_MAX), v_ls = c.integer("v_layer_stride", INT64_MAX);
  if (!c.ok()) return nullptr;
  if (L > 1 && (kv[0]->stride(0) != k_ls || kv[1]->stride(0) != v_ls)) c.refuse("the layer strides are not those of k and v");
  const auto* keep = (const int32_t*)c.buffer("keep_idx", at::kInt, {L, layer->n_kv_heads * (T - S * layer->window)});
  const auto* hoff = (const int32_t*)c.buffer("head_offsets", at::kInt, {L, S, H + 1});
  const auto* first_row = (const int32_t*)c.buffer("first_row", at::kInt, {L, S, H});
  const auto* table = (const int32_t*)c.buffer("page_table", at::kInt, {L, d->batch, H, d->max_pages});
  void* k_pages = c.written("k_pages", type, {d->n_pages, d->page_rows, D});
  void* v_pages = c.written("v_pages", type, {d->n_pages, d->page_rows, D});
  void* stream = c.stream();
  if (!c.ok()) return nullptr;
  const void *k = kv[0]->data_ptr(), *v = kv[1]->data_ptr();
  return finish(c, [&] {
    return CHECK ? lava_check_compact_kv_pages(layer, d, first_seq, k, v, k_ls, v_ls, keep, hoff, first_row, table, k_pages,
                                               v_pages)
                 : lava_compact_kv_pages(layer, d, first_seq, k, v, k_ls, v_ls, keep, hoff, first_row, table, k_pages,
                                         v_pages, stream);
  }, !CHECK);
}
PyObject* compact_kv_pages(PyObject* const* args, Py_ssize_t n) { return compact_pages<false>(args, n); }
PyObject* check_compact_kv_pages(PyObject* const* args, Py_ssize_t n) { return compact_pages<true>(args, n); }

const double* frequencies(Call& c, const lava_rotary_desc* r) {
  if (r->rotary_dim == 0 && c.none()) return nullptr;
  return (const double*)c.buffer("freqs", at::kDouble, {r->rotary_dim / 2});
}

PyObject* rotary(PyObject* const* args, Py_ssize_t n) {
  Call c(args, n, 8);
  const auto* r = c.desc<lava_rotary_desc>();
  if (!c.ok()) return nullptr;
  const double* freqs = frequencies(c, r);
  if (!c.ok()) return nullptr;
  int64_t tokens = 0;
  if (THPVariable_Check(c.peek())) tokens = THPVariable_Unpack(c.peek()).numel();
  const auto* positions = (const int32_t*)c.buffer("positions", at::kInt, {tokens});
  struct {
    const char *in_name, *out_name;
    int64_t heads;
    Call::Vectors in, out;
  } x[2] = {{"q", "q_out", 0, {}, {}}, {"k", "k_out", 0, {}, {}}};
  const at::ScalarType type = type_of(r->dtype);
  // q, q_out, k, k_out
  for (auto& a : x) {
    if (!c.ok()) return nullptr;
    const bool no_in = c.none();
    if (no_in) {
      if (!c.none()) c.refuse(std::string(a.in_name) + " and " + a.out_name + " are both given or both None");
      continue;
    }
    if (THPVariable_Check(c.peek())) {
      const at::Tensor& t = THPVariable_Unpack(c.peek());
      a.heads = t.dim() == 3 ? t.size(1) : 0;
    }
    if (a.heads > 0x7fffffff) c.refuse(std::string(a.in_name) + " has too many heads");
    const at::Tensor* in = c.tensor(a.in_name);
    if (!in || !c.without_gradient(a.in_name, *in)) return nullptr;
    a.in = c.vectors(a.in_name, in, type, tokens, a.heads, r->head_dim);
    if (c.ok() && c.peek() == Py_None) c.refuse(std::string(a.in_name) + " and " + a.out_name + " are both given or both None");
    a.out = c.vectors(a.out_name, c.output(a.out_name), type, tokens, a.heads, r->head_dim);
  }
  void* stream = c.stream();
  if (!c.ok()) return nullptr;
  return finish(c, [&] {
    return lava_rotary(r, freqs, tokens, positions, x[0].in.at, (int32_t)x[0].heads, x[0].in.tok, x[0].in.head, x[0].out.at,
                       x[0].out.tok, x[0].out.head, x[1].in.at, (int32_t)x[1].heads, x[1].in.tok, x[1].in.head, x[1].out.at,
                       x[1].out.tok, x[1].out.head, stream);
  });
}

PyObject* rotary_append(PyObject* const* args, Py_ssize_t n) {
  Call c(args, n, 13);
  const auto* r = c.desc<lava_rotary_desc>();
  if (!c.ok()) return nullptr;
  const double* freqs = frequencies(c, r);
  const auto* d = c.desc<lava_cache_desc>();
  const int layer = c.int32("layer");
  if (!c.ok()) return nullptr;
  const int64_t L = d->n_layers, B = d->batch, H = d->n_kv_heads, Hq = d->n_q_heads, D = d->head_dim;
  if (layer < 0 || layer >= L) {
    c.refuse("layer " + std::to_string(layer) + " is not in a cache of " + std::to_string(L));
    return nullptr;
  }
  int64_t max_add = 0;
  if (THPVariable_Check(c.peek())) {
    const at::Tensor& t = THPVariable_Unpack(c.peek());
    max_add = t.dim() == 4 ? t.size(2) : 0;
  }
  const auto* slots = (const int32_t*)c.buffer("slots", at::kInt, {L, B, max_add, H});
  const int64_t tokens = B * max_add;
  const at::ScalarType type = type_of(d->dtype);
  const auto* positions = (const int32_t*)c.buffer("positions", at::kInt, {tokens});
  const auto q = c.vectors("q", type, tokens, Hq, D), k = c.vectors("k", type, tokens, H, D),
             v = c.vectors("v", type, tokens, H, D);
  void* q_out = c.written("q_out", type, {tokens, Hq, D});
  void* k_pages = c.written("k_pages", type, {d->n_pages, d->page_rows, D});
  void* v_pages = c.written("v_pages", type, {d->n_pages, d->page_rows, D});
  void* stream = c.stream();
  if (!c.ok()) return nullptr;
  return finish(c, [&] {
    return lava_rotary_append(r, freqs, d, tokens, positions, q.at, q.tok, q.head, q_out, k.at, k.tok, k.head, v.at, v.tok,
                              v.head, slots + layer * tokens * H, k_pages, v_pages, stream);
  });
}

PyObject* decode_attention_pages(PyObject* const* args, Py_ssize_t n) {
  Call c(args, n, 11);
  const auto* d = c.desc<lava_cache_desc>();
  const int first_layer = c.int32("first_layer");
  if (!c.ok()) return nullptr;
  const int64_t L = d->n_layers, B = d->batch, H = d->n_kv_heads, Hq = d->n_q_heads, D = d->head_dim;
  const at::ScalarType type = type_of(d->dtype);
  int64_t layers = 0;
  if (THPVariable_Check(c.peek())) {
    const at::Tensor& t = THPVariable_Unpack(c.peek());
    layers = t.dim() == 4 ? t.size(0) : 0;
  }
  if (layers > 0x7fffffff) c.refuse("q has too many layers");
  const void* q = c.buffer("q", type, {layers, B, Hq, D});
  const void* k_pages = c.buffer("k_pages", type, {d->n_pages, d->page_rows, D});
  const void* v_pages = c.buffer("v_pages", type, {d->n_pages, d->page_rows, D});
  const auto* table = (const int32_t*)c.buffer("page_table", at::kInt, {L, B, H, d->max_pages});
  const auto* rows = (const int32_t*)c.buffer("head_rows", at::kInt, {L, B, H});
  void* out = c.written("out", type, {layers, B, Hq, D});
  auto* lse = c.none() ? nullptr : (float*)c.written("lse", at::kFloat, {layers, B, Hq});
  const at::Tensor* ws = c.tensor("workspace");
  if (ws && (!c.here(*ws) || !ws->is_contiguous())) c.refuse("workspace must be contiguous and on the current device");
  void* stream = c.stream();
  if (!c.ok()) return nullptr;
  void* ws_at = ws->data_ptr();
  const size_t ws_bytes = ws->nbytes();
  return finish(c, [&] {
    return lava_decode_attention_pages(d, first_layer, (int32_t)layers, q, k_pages, v_pages, table, rows, out, lse, ws_at,
                                       ws_bytes, stream);
  });
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XSETREF(g_error, type);
  Py_RETURN_NONE;
}

#define LAVA_METHOD(name) {#name, (PyCFunction)(void*)guarded<name>, METH_FASTCALL, ""}
PyMethodDef g_methods[] = {LAVA_METHOD(page_admit),     LAVA_METHOD(page_extend), LAVA_METHOD(compact_kv_pages),
                           LAVA_METHOD(check_compact_kv_pages),
                           LAVA_METHOD(rotary),         LAVA_METHOD(rotary_append), LAVA_METHOD(decode_attention_pages),
                           {"set_error", set_error, METH_O, "the class that refusals raise"},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_paged_calls", nullptr, -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__paged_calls() {
  PyObject* m = PyModule_Create(&g_module);
  // tensors are looked into as this torch lays them out: the loader compares
  if (m && PyModule_AddStringConstant(m, "torch_version", LAVA_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
