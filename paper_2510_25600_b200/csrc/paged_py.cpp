// The paged calls for Python (the module `_paged`): tensors in, the C entry point called on the current stream of their device with
// the GIL released, its status out.  Shapes, types and devices, which the C entry points cannot see, are checked here (ValueError);
// no step of the method runs here.  The tensors are read through torch's C++ interface: their forty sizes, strides, types and
// addresses cost 10-15 us a call read from Python, more than most of these kernels take, and 0.5 us this way.  The module belongs to the
// torch it was built with; `build.py` puts the version into its name.
#define PY_SSIZE_T_CLEAN
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <string>

#include "purekv.h"

namespace {

struct Refused {
  PyObject* kind;
  std::string why;
};
[[noreturn]] void refuse(const char* fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof(text), fmt, ap);
  va_end(ap);
  throw Refused{PyExc_ValueError, text};
}
struct PythonError {};  // one is set

// The positional arguments of one call, read in order.
class Args {
 public:
  Args(const char* name, PyObject* const* v, Py_ssize_t n, Py_ssize_t want) : v_(v) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "%s: %zd arguments, got %zd", name, want, n);
      throw PythonError{};
    }
  }
  PyObject* object() { return v_[at_++]; }
  const at::Tensor* tensor(const char* name) {  // or None
    PyObject* o = object();
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, std::string(name) + ": not a tensor"};
    const at::Tensor* t = &THPVariable_Unpack(o);
    if (t->layout() != at::kStrided) refuse("%s: not a strided tensor", name);
    return t;
  }
  const at::Tensor* some(const char* name) {
    const at::Tensor* t = tensor(name);
    if (!t) refuse("%s is missing", name);
    return t;
  }
  int64_t integer() {
    const long long x = PyLong_AsLongLong(object());
    if (x == -1 && PyErr_Occurred()) throw PythonError{};
    return x;
  }
  int32_t i32(const char* name) {
    const int64_t x = integer();
    if (x < INT32_MIN || x > INT32_MAX) refuse("%s does not fit 32 bits", name);
    return (int32_t)x;
  }
  float f32() {
    const double x = PyFloat_AsDouble(object());
    if (x == -1.0 && PyErr_Occurred()) throw PythonError{};
    return (float)x;
  }
  bool truth() {
    const int x = PyObject_IsTrue(object());
    if (x < 0) throw PythonError{};
    return x != 0;
  }

 private:
  PyObject* const* v_;
  Py_ssize_t at_ = 0;
};

std::string shape_of(const at::Tensor& t) {
  std::string s = c10::toString(t.scalar_type());
  s += " [";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + "]";
}
int32_t small(int64_t n, const char* name) {
  if (n > INT32_MAX) refuse("%s: a size of %lld does not fit 32 bits", name, (long long)n);
  return (int32_t)n;
}
template <typename T = void>
T* at_of(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

void same(const at::Tensor* t, const char* name, at::ScalarType type, at::IntArrayRef shape) {
  if (t && (t->scalar_type() != type || t->sizes() != shape)) {
    std::string want = std::string(c10::toString(type)) + " [";
    for (size_t i = 0; i < shape.size(); ++i) want += (i ? ", " : "") + std::to_string(shape[i]);
    refuse("%s: %s] is wanted, got %s", name, want.c_str(), shape_of(*t).c_str());
  }
}
void contiguous(const at::Tensor* t, const char* name, at::ScalarType type, at::IntArrayRef shape) {
  same(t, name, type, shape);
  if (t && !t->is_contiguous()) refuse("%s: not contiguous", name);
}
// All tensors on one GPU; returns its index.
int device_of(std::initializer_list<const at::Tensor*> all) {
  const at::Tensor* first = nullptr;
  for (const at::Tensor* t : all) {
    if (!t) continue;
    if (!first) first = t;
    if (!t->device().is_cuda()) refuse("the paged calls take tensors on a GPU");
    if (t->device() != first->device()) refuse("the tensors of a paged call lie on one device");
  }
  return first->device().index();
}
purekv_dtype type_of(const at::Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kBFloat16: return PUREKV_BF16;
    case at::kFloat: return PUREKV_FP32;
    case at::kFloat8_e4m3fn: return PUREKV_E4M3;
    default: refuse("%s: bfloat16, float32 or, for pools, float8_e4m3fn is wanted, got %s", name, c10::toString(t.scalar_type()));
  }
}

struct Rows {  // [n, heads, d], rows contiguous
  const void* p = nullptr;
  int64_t token = 0, head = 0;
  int32_t heads = 0;
};
Rows rows_of(const at::Tensor* t, const char* name, int64_t n, int64_t d, at::ScalarType type) {
  if (!t) return {};
  if (t->dim() != 3 || t->size(0) != n || t->size(2) != d || t->scalar_type() != type || (t->stride(2) != 1 && d > 1))
    refuse("%s: %s [%lld, heads, %lld] with contiguous rows is wanted, got %s", name, c10::toString(type), (long long)n, (long long)d, shape_of(*t).c_str());
  return {t->data_ptr(), t->stride(0), t->stride(1), small(t->size(1), name)};
}

// n_layers > 0: the pools of so many layers.
purekv_pages pages_of(const at::Tensor& k, const at::Tensor& v, const at::Tensor& table, const at::Tensor& lens, const at::Tensor* ks,
                      const at::Tensor* vs, int64_t n_layers) {
  const int64_t lead = n_layers ? 1 : 0;
  if (k.dim() != 4 + lead || (lead && k.size(0) != n_layers) || (k.stride(3 + lead) != 1 && k.size(3 + lead) > 1))
    refuse("pools are %sn_pages, page_size, H_kv, d] with contiguous rows, got %s", lead ? "[n_layers, " : "[", shape_of(k).c_str());
  if (v.sizes() != k.sizes() || v.strides() != k.strides() || v.scalar_type() != k.scalar_type())
    refuse("k_pages and v_pages have one shape, one layout and one dtype");
  purekv_pages p = {};
  p.k = k.data_ptr();
  p.v = v.data_ptr();
  p.layer_stride = lead ? k.stride(0) : 0;
  p.page_stride = k.stride(lead);
  p.token_stride = k.stride(lead + 1);
  p.head_stride = k.stride(lead + 2);
  p.n_pages = small(k.size(lead), "k_pages");
  p.page_size = small(k.size(lead + 1), "k_pages");
  p.n_kv_heads = small(k.size(lead + 2), "k_pages");
  p.head_dim = small(k.size(lead + 3), "k_pages");
  p.dtype = type_of(k, "k_pages");
  if (lens.dim() != 1) refuse("seq_lens: Int [n_req] is wanted, got %s", shape_of(lens).c_str());
  contiguous(&lens, "seq_lens", at::kInt, {lens.size(0)});
  if (table.dim() != 2) refuse("block_table: Int [n_req, max_pages] is wanted, got %s", shape_of(table).c_str());
  same(&table, "block_table", at::kInt, {lens.size(0), table.size(1)});
  if (table.stride(1) != 1 && table.size(1) > 1) refuse("block_table: its rows are not contiguous");
  const int64_t heads = p.n_kv_heads;
  for (const auto& s : {std::pair<const at::Tensor*, const char*>{ks, "k_scale"}, {vs, "v_scale"}}) {
    if (lead) contiguous(s.first, s.second, at::kFloat, {n_layers, heads});
    else contiguous(s.first, s.second, at::kFloat, {heads});
  }
  p.k_scale = at_of<const float>(ks);
  p.v_scale = at_of<const float>(vs);
  p.n_req = small(lens.size(0), "seq_lens");
  p.max_pages = small(table.size(1), "block_table");
  p.table_stride = table.stride(0);
  p.block_table = at_of<const int32_t>(&table);
  p.seq_lens = at_of<const int32_t>(&lens);
  return p;
}

int32_t* status_of(const at::Tensor* t) {
  if (t) contiguous(t, "status", at::kInt, {1});
  return at_of<int32_t>(t);
}

// The call on the current stream of `device`, which becomes the current device for as long.
template <typename F>
PyObject* launch(int device, F f) {
  purekv_status st;
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
  void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  Py_BEGIN_ALLOW_THREADS;
  st = f(stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong((long)st);
}

PyObject* append(PyObject* const* v, Py_ssize_t n) {
  Args a("append_paged", v, n, 17);
  const at::Tensor *k = a.tensor("k"), *val = a.tensor("v"), *kp = a.tensor("k_pages"), *vp = a.tensor("v_pages");
  const at::Tensor *table = a.tensor("block_table"), *lens = a.tensor("seq_lens"), *cu = a.tensor("cu_new");
  const at::Tensor *q = a.tensor("q"), *q_out = a.tensor("q_out"), *k_out = a.tensor("k_out");
  const at::Tensor *pos = a.tensor("positions"), *freq = a.tensor("inv_freq");
  PyObject* sections = a.object();
  const bool interleaved = a.truth();
  const at::Tensor *ks = a.tensor("k_scale"), *vs = a.tensor("v_scale"), *status = a.tensor("status");

  const at::Tensor* lead = k ? k : q;
  if (!lead) refuse("neither k nor q");
  if (lead->dim() != 3) refuse("%s: [T, heads, d] is wanted, got %s", k ? "k" : "q", shape_of(*lead).c_str());
  const int64_t t = lead->size(0), d = lead->size(2);
  const purekv_dtype type = type_of(*lead, k ? "k" : "q");
  const Rows kr = rows_of(k, "k", t, d, lead->scalar_type()), qr = rows_of(q, "q", t, d, lead->scalar_type());
  Rows vr;
  if ((q != nullptr) != (q_out != nullptr)) refuse("q_out goes with q");
  contiguous(q_out, "q_out", lead->scalar_type(), {t, qr.heads, d});
  if (k_out && !k) refuse("k_out goes with k");
  contiguous(k_out, "k_out", lead->scalar_type(), {t, kr.heads, d});
  purekv_pages pages;
  if (kp) {
    if (!k || !val || val->sizes() != k->sizes()) refuse("v goes with k into the pages");
    if (!vp || !table || !lens) refuse("v_pages, block_table and seq_lens go with k_pages");
    vr = rows_of(val, "v", t, d, lead->scalar_type());
    pages = pages_of(*kp, *vp, *table, *lens, ks, vs, 0);
    if (cu) contiguous(cu, "cu_new", at::kInt, {lens->size(0) + 1});
  } else {
    val = nullptr;
  }
  purekv_rope rope = {};
  if (pos) {
    if (!freq || freq->dim() != 1) refuse("inv_freq: Double [rotary_dim / 2] goes with positions");
    contiguous(freq, "inv_freq", at::kDouble, {freq->size(0)});
    rope.rotary_dim = small(2 * freq->size(0), "inv_freq");
    rope.n_axes = 1;
    rope.sections[0] = rope.rotary_dim / 2;
    if (sections != Py_None) {
      PyObject* list = PySequence_Fast(sections, "sections: not a sequence");
      if (!list) throw PythonError{};
      const Py_ssize_t axes = PySequence_Fast_GET_SIZE(list);
      bool fits = axes >= 1 && axes <= 4;
      for (Py_ssize_t i = 0; fits && i < axes; ++i) {
        const long x = PyLong_AsLong(PySequence_Fast_GET_ITEM(list, i));
        if (x == -1 && PyErr_Occurred()) {
          Py_DECREF(list);
          throw PythonError{};
        }
        fits = x >= 0 && x <= rope.rotary_dim;
        rope.sections[i] = (int32_t)x;
      }
      Py_DECREF(list);
      if (!fits) refuse("sections: 1 to 4 numbers that sum to rotary_dim / 2");
      rope.n_axes = (int32_t)axes;
    }
    if (rope.n_axes == 1 && pos->dim() == 1) {
      contiguous(pos, "positions", at::kInt, {t});
    } else {
      same(pos, "positions", at::kInt, {rope.n_axes, t});
      if (pos->stride(1) != 1 && t > 1) refuse("positions: an axis is not contiguous");
      rope.axis_stride = pos->stride(0);
    }
    rope.positions = at_of<const int32_t>(pos);
    rope.inv_freq = at_of<const double>(freq);
    rope.interleaved = interleaved;
  }
  int32_t* word = status_of(status);
  const int device = device_of({lead, q, val, kp, vp, table, lens, cu, q_out, k_out, pos, freq, ks, vs, status});
  const int32_t tokens = small(t, "k"), hkv = kr.heads, dim = small(d, "k");
  return launch(device, [&](void* stream) {
    return purekv_append_paged(qr.p, qr.token, qr.head, kr.p, kr.token, kr.head, vr.p, vr.token, vr.head, at_of(q_out), at_of(k_out), kp ? &pages : nullptr,
                               pos ? &rope : nullptr, at_of<const int32_t>(cu), tokens, qr.heads, hkv, dim, type, word, stream);
  });
}

PyObject* compact(PyObject* const* v, Py_ssize_t n) {
  Args a("compact_paged", v, n, 12);
  const at::Tensor *k = a.some("k"), *val = a.some("v"), *idx = a.some("idx"), *cu = a.some("cu_seqlens"), *ck = a.some("cu_kept");
  const at::Tensor *kp = a.some("k_pages"), *vp = a.some("v_pages"), *table = a.some("block_table"), *lens = a.some("seq_lens");
  const at::Tensor *ks = a.tensor("k_scale"), *vs = a.tensor("v_scale"), *status = a.tensor("status");
  if (k->dim() != 4) refuse("k: [n_layers, T, H_kv, d] is wanted, got %s", shape_of(*k).c_str());
  const int64_t layers = k->size(0), t = k->size(1), heads = k->size(2), d = k->size(3);
  auto packed = [&](const at::Tensor* x) { return x->stride(3) == 1 && (heads == 1 || x->stride(2) == d) && (t == 1 || x->stride(1) == heads * d); };
  if (val->sizes() != k->sizes() || val->scalar_type() != k->scalar_type() || (k->numel() && (!packed(k) || !packed(val))) || (layers > 1 && val->stride(0) != k->stride(0)))
    refuse("k and v are [n_layers, T, H_kv, d] of one dtype, each layer contiguous, layers as far apart");
  const purekv_dtype type = type_of(*k, "k");
  if (layers == 0) return PyLong_FromLong(PUREKV_OK);
  const purekv_pages pages = pages_of(*kp, *vp, *table, *lens, ks, vs, layers);
  if (pages.n_kv_heads != heads || pages.head_dim != d) refuse("the pages have other heads than k and v");
  if (idx->dim() != 3) refuse("idx: [n_layers, H_kv, K_tot] is wanted, got %s", shape_of(*idx).c_str());
  contiguous(idx, "idx", at::kInt, {layers, heads, idx->size(2)});
  contiguous(cu, "cu_seqlens", at::kInt, {lens->size(0) + 1});
  contiguous(ck, "cu_kept", at::kInt, {lens->size(0) + 1});
  int32_t* word = status_of(status);
  const int device = device_of({k, val, idx, cu, ck, kp, vp, table, lens, ks, vs, status});
  const int32_t n_layers = small(layers, "k"), k_tot = small(idx->size(2), "idx");
  return launch(device, [&](void* stream) {
    return purekv_compact_paged(k->data_ptr(), val->data_ptr(), k->stride(0), n_layers, at_of<const int32_t>(idx), at_of<const int32_t>(cu), t,
                                at_of<const int32_t>(ck), k_tot, type, &pages, word, stream);
  });
}

PyObject* decode(PyObject* const* v, Py_ssize_t n) {
  Args a("decode_paged", v, n, 13);
  const at::Tensor *q = a.some("q"), *kp = a.some("k_pages"), *vp = a.some("v_pages"), *table = a.some("block_table"), *lens = a.some("seq_lens");
  const int32_t max_len = a.i32("max_len");
  const at::Tensor *out = a.some("out"), *lse = a.tensor("lse");
  const float scale = a.f32();
  const at::Tensor *ks = a.tensor("k_scale"), *vs = a.tensor("v_scale"), *ws = a.tensor("ws"), *status = a.tensor("status");
  if (q->dim() != 3) refuse("q: [n_req, H, d] is wanted, got %s", shape_of(*q).c_str());
  const purekv_pages pages = pages_of(*kp, *vp, *table, *lens, ks, vs, 0);
  const Rows r = rows_of(q, "q", pages.n_req, pages.head_dim, q->scalar_type());
  const purekv_dtype type = type_of(*q, "q");
  contiguous(out, "out", q->scalar_type(), q->sizes());
  if (lse) contiguous(lse, "lse", at::kFloat, {q->size(0), q->size(1)});
  if (ws && !ws->is_contiguous()) refuse("ws: not contiguous");
  int32_t* word = status_of(status);
  const int device = device_of({q, kp, vp, table, lens, out, lse, ks, vs, ws, status});
  return launch(device, [&](void* stream) {
    return purekv_decode_paged(r.p, r.token, r.head, out->data_ptr(), at_of<float>(lse), &pages, max_len, r.heads, type, scale, at_of(ws),
                               ws ? ws->nbytes() : 0, word, stream);
  });
}

// C++ exceptions end here.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* v, Py_ssize_t n) {
  try {
    return F(v, n);
  } catch (const PythonError&) {
  } catch (const Refused& e) {
    PyErr_SetString(e.kind, e.why.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define PK_METHOD(name, f) {name, (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PK_METHOD("purekv_append_paged", append), PK_METHOD("purekv_compact_paged", compact),
                         PK_METHOD("purekv_decode_paged", decode), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged(void) { return PyModule_Create(&module); }
