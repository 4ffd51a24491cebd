// Python calls of the decoding operators: checks of tensors and marshalling of their addresses,
// sizes and strides to the C entry points.  Compiled because a call of these operators takes the GPU 2 us
// upwards, and the same checks took the interpreter 8 us and more; nothing is computed here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <optional>
#include <stdexcept>
#include <string>

#include "../../include/gar.h"

namespace {

using at::Tensor;

// Carries a Python exception that is already set.
struct python_error {};

[[noreturn]] void bad(const std::string &why) { throw std::invalid_argument(why); }

// The arguments of a call, by the names of its parameters; the first `needed` must be there.
template <int N> struct Arguments {
  PyObject *at[N] = {};
  Arguments(const char *call, const char *const (&names)[N], int needed, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
    const auto type_error = [&](const std::string &why) {
      PyErr_SetString(PyExc_TypeError, (std::string(call) + "() " + why).c_str());
      throw python_error();
    };
    if (n > N) type_error("takes at most " + std::to_string(N) + " arguments");
    for (Py_ssize_t i = 0; i < n; ++i) at[i] = args[i];
    const Py_ssize_t k = kw ? PyTuple_GET_SIZE(kw) : 0;
    for (Py_ssize_t j = 0; j < k; ++j) {
      PyObject *key = PyTuple_GET_ITEM(kw, j);
      int i = 0;
      while (i < N && PyUnicode_CompareWithASCIIString(key, names[i]) != 0) ++i;
      const char *name = PyUnicode_AsUTF8(key);
      if (i == N) type_error(std::string("got an unexpected argument '") + (name ? name : "?") + "'");
      if (at[i]) type_error(std::string("got two values for '") + names[i] + "'");
      at[i] = args[n + j];
    }
    for (int i = 0; i < needed; ++i)
      if (!at[i]) type_error(std::string("needs '") + names[i] + "'");
    for (int i = 0; i < N; ++i)
      if (at[i] == Py_None) at[i] = nullptr;
    for (int i = 0; i < needed; ++i)
      if (!at[i]) type_error(std::string("needs '") + names[i] + "', not None");
  }
};

const Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, (std::string(what) + " must be a tensor").c_str());
    throw python_error();
  }
  return THPVariable_Unpack(o);
}

int64_t integer(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}

// A number that the C entry points take as an int.
int narrow(int64_t v, const char *what) {
  if (v < INT_MIN || v > INT_MAX) bad(std::string(what) + " is out of range: " + std::to_string(v));
  return (int)v;
}

double number(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}

bool truth(PyObject *o) {
  const int v = o ? PyObject_IsTrue(o) : 0;
  if (v < 0) throw python_error();
  return v;
}

// Names of attributes, made once.
struct Names {
  PyObject *address = PyUnicode_InternFromString("address"), *device_index = PyUnicode_InternFromString("device_index"),
           *stream = PyUnicode_InternFromString("stream"), *tensors = PyUnicode_InternFromString("tensors");
};
const Names &names_of() {
  static const Names n;
  return n;
}

// The Python classes that keep the C objects.
PyObject *class_of(const char *name) {
  PyObject *m = PyImport_ImportModule("paper_2004_09362_gb300.gar");
  PyObject *c = m ? PyObject_GetAttrString(m, name) : nullptr;
  Py_XDECREF(m);
  if (!c) throw python_error();
  if (!PyType_Check(c)) bad(std::string(name) + " is no class");
  return c;
}
template <typename T> PyTypeObject *owner();
template <> PyTypeObject *owner<gar_kv_cache>() {
  static PyObject *const c = class_of("KVCache");
  return reinterpret_cast<PyTypeObject *>(c);
}
template <> PyTypeObject *owner<gar_attn_plan>() {
  static PyObject *const c = class_of("AttnPlan");
  return reinterpret_cast<PyTypeObject *>(c);
}

// The C object of a Python object of its class.
template <typename T> T *handle(PyObject *o, const char *what) {
  if (!PyObject_TypeCheck(o, owner<T>())) {
    PyErr_Format(PyExc_TypeError, "needs a %s, not a %s", owner<T>()->tp_name, Py_TYPE(o)->tp_name);
    throw python_error();
  }
  PyObject *v = PyObject_GetAttr(o, names_of().address);
  if (!v) throw python_error();
  void *p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) throw python_error();
  if (!p) bad(what);
  return static_cast<T *>(p);
}

int dtype_of(const Tensor &t, const char *what) {
  switch (t.scalar_type()) {
    case at::kFloat: return GAR_F32;
    case at::kBFloat16: return GAR_BF16;
    case at::kHalf: return GAR_F16;
    case at::kChar: return GAR_I8;
    case at::kFloat8_e4m3fn: return GAR_E4M3;
    default: bad(std::string(what) + ": this dtype is not supported");
  }
}

// [tokens, heads, dim] on the GPU, the channels of a head contiguous.
const Tensor &rows(PyObject *o, const char *what) {
  const Tensor &t = tensor(o, what);
  if (t.dim() != 3) bad(std::string(what) + " must be [tokens, heads, dim]");
  if (t.stride(2) != 1 && t.size(2) > 1) bad(std::string(what) + ": the channels of a head must be contiguous");
  if (!t.is_cuda()) bad(std::string(what) + " must be a CUDA tensor");
  narrow(t.size(1), "the number of heads"), narrow(t.size(2), "the number of channels");
  return t;
}

// n contiguous integers on the GPU, 8 bytes wide or (`narrow`) 4.
const Tensor &integers(PyObject *o, int64_t n, bool narrow, bool wide, const char *what) {
  const Tensor &t = tensor(o, what);
  if (t.dim() != 1 || (n >= 0 && t.size(0) != n) || !t.is_cuda() || (t.size(0) > 1 && t.stride(0) != 1))
    bad(std::string(what) + " must be contiguous integers on the GPU, one for each token or sequence");
  const auto type = t.scalar_type();
  if (!(wide && type == at::kLong) && !(narrow && type == at::kInt)) bad(std::string(what) + ": this dtype is not supported");
  return t;
}

const Tensor &rotations(PyObject *o, int64_t dim) {
  const Tensor &t = tensor(o, "table");
  if (t.dim() != 3 || t.size(2) != 2 || t.scalar_type() != at::kFloat || !t.is_cuda() || !t.is_contiguous())
    bad("the table must be a contiguous float32 CUDA tensor [positions, rot / 2, 2]");
  if (t.size(1) < 1 || 2 * t.size(1) > dim)
    bad("the table rotates " + std::to_string(2 * t.size(1)) + " channels, the heads have " + std::to_string(dim));
  return t;
}

// The GPU that a call's tensors are on: one for all, and the current one.
class Device {
  int at = -1;

 public:
  void add(int device, const char *what) {
    if (at < 0) at = device;
    if (device != at)
      bad(std::string(what) + " is on GPU " + std::to_string(device) + ", what comes before it on GPU " + std::to_string(at));
  }
  void add(const Tensor &t, const char *what) { add(t.get_device(), what); }
  int check() const {
    const int current = c10::cuda::current_device();
    if (at != current)
      bad("the tensors are on GPU " + std::to_string(at) + ", the current device is GPU " + std::to_string(current));
    return current;
  }
};

// The GPU of a cache.
int device_of(PyObject *cache) {
  PyObject *v = PyObject_GetAttr(cache, names_of().device_index);
  if (!v) throw python_error();
  const long d = PyLong_AsLong(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) throw python_error();
  return (int)d;
}

int layout_of(PyObject *o) {
  if (!o) return GAR_ROPE_HALF;
  if (PyUnicode_Check(o)) {
    if (PyUnicode_CompareWithASCIIString(o, "half") == 0) return GAR_ROPE_HALF;
    if (PyUnicode_CompareWithASCIIString(o, "interleaved") == 0) return GAR_ROPE_INTERLEAVED;
    bad("unknown layout");
  }
  return narrow(integer(o), "layout");
}

// The stream of a call: torch's current one, a torch stream, or a raw handle.
struct Stream {
  gar_stream_t raw;
  bool other;  // not torch's current stream
  explicit Stream(gar_stream_t raw) : raw(raw), other(raw != c10::cuda::getCurrentCUDAStream().stream()) {}
  Stream(PyObject *o, int device) {
    const cudaStream_t current = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    raw = current;
    if (o) {
      PyObject *v = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, "cuda_stream");
      if (!v) throw python_error();
      raw = static_cast<gar_stream_t>(PyLong_AsVoidPtr(v));
      Py_DECREF(v);
      if (PyErr_Occurred()) throw python_error();
    }
    other = raw != current;
  }
  // An output that the call fills: allocated under its stream, so that its memory is not given away
  // while that stream uses it.
  Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor &like) const {
    if (!other) return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
    c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(raw, like.get_device()));
    return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
  }
};

// Whether a gradient is asked of any of the tensors (null and undefined ones aside).
bool graded_any(std::initializer_list<const Tensor *> tensors) {
  if (!at::GradMode::is_enabled()) return false;
  for (const Tensor *t : tensors)
    if (t && t->defined() && t->requires_grad()) return true;
  return false;
}

// Counts a tensor's memory as changed, so that autograd sees it where it has kept the tensor.  (Tensors of inference mode
// are not counted.)
void changed(const Tensor &t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The same of a cache's.
void changed_cache(PyObject *cache) {
  PyObject *tensors = PyObject_GetAttr(cache, names_of().tensors);
  if (!tensors) throw python_error();
  const Py_ssize_t n = PyTuple_Check(tensors) ? PyTuple_GET_SIZE(tensors) : 0;
  for (Py_ssize_t i = 0; i < n; ++i)
    if (THPVariable_Check(PyTuple_GET_ITEM(tensors, i))) changed(THPVariable_Unpack(PyTuple_GET_ITEM(tensors, i)));
  Py_DECREF(tensors);
}

// For calls that no gradient goes through.
void refuse_graded(std::initializer_list<const Tensor *> tensors) {
  if (graded_any(tensors)) bad("this call has no gradient: detach its tensors, or call it under torch.no_grad()");
}

void check(int rc, const char *where) {
  if (rc == GAR_OK) return;
  PyObject *m = PyImport_ImportModule("paper_2004_09362_gb300.gar");
  PyObject *r = m ? PyObject_CallMethod(m, "_check", "is", rc, where) : nullptr;
  Py_XDECREF(r);
  Py_XDECREF(m);
  throw python_error();
}

// A refused call where there may be no Python.
struct call_failed : std::runtime_error {
  int rc;
  const char *where;
  call_failed(int rc, const char *where) : std::runtime_error(std::string(where) + ": " + gar_last_error()), rc(rc), where(where) {}
};

template <typename F> PyObject *guarded(F f) noexcept {
  try {
    try {
      return f();
    } catch (const call_failed &e) {
      check(e.rc, e.where);
    }
  } catch (const python_error &) {
  } catch (const std::invalid_argument &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

int rope_into(const Tensor &x, const Tensor &positions, const Tensor &table, int layout, bool inverse, const Tensor &out,
              gar_stream_t stream) {
  return gar_rope(x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0), out.stride(1), dtype_of(x, "x"),
                  x.size(0), (int)x.size(1), (int)x.size(2), 2 * (int)table.size(1), positions.data_ptr(),
                  (int)positions.element_size(), static_cast<const float *>(table.data_ptr()), table.size(0), layout, inverse,
                  stream);
}

// The rotation as a step that gradients go through: theirs is the rotation back.  (Without Python: gradients are computed
// on threads of autograd's, under the stream that was torch's current one.)
struct RopeStep : torch::autograd::Function<RopeStep> {
  static Tensor forward(torch::autograd::AutogradContext *ctx, const Tensor &x, const Tensor &positions, const Tensor &table,
                        int64_t layout, bool inverse, int64_t raw) {
    ctx->save_for_backward({positions, table});
    ctx->saved_data["layout"] = layout;
    ctx->saved_data["inverse"] = inverse;
    const Stream stream(reinterpret_cast<gar_stream_t>(raw));
    const Tensor out = stream.empty(x.sizes(), x.scalar_type(), x);
    if (const int rc = rope_into(x, positions, table, (int)layout, inverse, out, stream.raw)) throw call_failed(rc, "gar_rope");
    return out;
  }
  static torch::autograd::variable_list backward(torch::autograd::AutogradContext *ctx, torch::autograd::variable_list grads) {
    const auto saved = ctx->get_saved_variables();
    Tensor grad = grads[0];
    if (!grad.defined()) return {Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
    if (grad.size(2) > 1 && grad.stride(2) != 1) grad = grad.contiguous();
    const c10::cuda::CUDAGuard guard(grad.device());
    const Tensor out = apply(grad, saved[0], saved[1], ctx->saved_data["layout"].toInt(), !ctx->saved_data["inverse"].toBool(),
                             (int64_t)(intptr_t)c10::cuda::getCurrentCUDAStream().stream());
    return {out, Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
  }
};

PyObject *rope(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"x", "positions", "table", "layout", "inverse", "out", "stream"};
    const Arguments<7> a("gar_rope", names, 3, args, n, kw);
    const Tensor &x = rows(a.at[0], "x"), &table = rotations(a.at[2], x.size(2));
    const Tensor &positions = integers(a.at[1], x.size(0), true, true, "positions");
    Tensor out;
    Device device;
    device.add(x, "x"), device.add(positions, "positions"), device.add(table, "table");
    if (a.at[5]) {
      out = rows(a.at[5], "out");
      if (out.scalar_type() != x.scalar_type() || out.sizes() != x.sizes()) bad("out must have x's shape and dtype");
      device.add(out, "out");
    }
    const bool graded = graded_any({&x, &table, &out});
    if (graded && (a.at[5] || table.requires_grad()))
      bad(a.at[5] ? "out= goes with tensors that need no gradient" : "the table gets no gradient: detach it");
    const int layout = layout_of(a.at[3]), inverse = truth(a.at[4]);
    const Stream stream(a.at[6], device.check());
    if (graded) return THPVariable_Wrap(RopeStep::apply(x, positions, table, (int64_t)layout, (bool)inverse, (int64_t)(intptr_t)stream.raw));
    if (!a.at[5]) out = stream.empty(x.sizes(), x.scalar_type(), x);
    check(rope_into(x, positions, table, layout, inverse, out, stream.raw), "gar_rope");
    if (!a.at[5]) return THPVariable_Wrap(std::move(out));
    changed(out);
    return Py_NewRef(a.at[5]);
  });
}

PyObject *kv_write(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"cache", "k", "v", "slots", "positions", "table", "layout", "stream"};
    const Arguments<8> a("gar_kv_write", names, 4, args, n, kw);
    const gar_kv_cache *cache = handle<gar_kv_cache>(a.at[0], "the cache has no address");
    const Tensor &k = rows(a.at[1], "k"), &v = rows(a.at[2], "v");
    if (k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type() || k.size(1) != cache->heads || k.size(2) != cache->dim)
      bad("k and v must be [tokens, heads, dim] of the cache's heads and dim, alike in dtype");
    const Tensor &slots = integers(a.at[3], k.size(0), false, true, "slots");
    refuse_graded({&k, &v});
    const int layout = layout_of(a.at[6]);
    if (!a.at[4] != !a.at[5]) bad("positions and table go together");
    const void *positions = nullptr;
    const float *table = nullptr;
    int width = 8, rot = 0;
    int64_t table_rows = 0;
    Device device;
    device.add(device_of(a.at[0]), "cache"), device.add(k, "k"), device.add(v, "v"), device.add(slots, "slots");
    if (a.at[4]) {
      const Tensor &t = rotations(a.at[5], k.size(2)), &p = integers(a.at[4], k.size(0), true, true, "positions");
      positions = p.data_ptr(), width = (int)p.element_size(), table = static_cast<const float *>(t.data_ptr());
      table_rows = t.size(0), rot = 2 * (int)t.size(1);
      device.add(p, "positions"), device.add(t, "table");
      refuse_graded({&t});
    }
    const Stream stream(a.at[7], device.check());
    check(gar_kv_write(cache, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1),
                       dtype_of(k, "k"), k.size(0), static_cast<const int64_t *>(slots.data_ptr()), positions, width, table,
                       table_rows, rot, layout, stream.raw),
          "gar_kv_write");
    changed_cache(a.at[0]);
    return Py_NewRef(Py_None);
  });
}

PyObject *kv_read(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"cache", "slots", "dtype", "out", "stream"};
    const Arguments<5> a("gar_kv_read", names, 2, args, n, kw);
    const gar_kv_cache *cache = handle<gar_kv_cache>(a.at[0], "the cache has no address");
    const Tensor &slots = integers(a.at[1], -1, false, true, "slots");
    Tensor k, v;
    Device device;
    device.add(device_of(a.at[0]), "cache"), device.add(slots, "slots");
    const int64_t shape[3] = {slots.size(0), cache->heads, cache->dim};
    if (a.at[3]) {
      if (!PyTuple_Check(a.at[3]) || PyTuple_GET_SIZE(a.at[3]) != 2) bad("out must be a pair of tensors");
      k = tensor(PyTuple_GET_ITEM(a.at[3], 0), "out"), v = tensor(PyTuple_GET_ITEM(a.at[3], 1), "out");
      for (const Tensor &t : {k, v})
        if (t.sizes() != at::IntArrayRef(shape) || t.scalar_type() != k.scalar_type() || !t.is_cuda() || !t.is_contiguous())
          bad("out must be two contiguous CUDA tensors [tokens, heads, dim] of one dtype");
      device.add(k, "out"), device.add(v, "out");
      refuse_graded({&k, &v});
    }
    const Stream stream(a.at[4], device.check());
    if (!a.at[3]) {
      at::ScalarType type = cache->dtype == GAR_F32 ? at::kFloat : cache->dtype == GAR_F16 ? at::kHalf : at::kBFloat16;
      if (a.at[2]) {
        const char *s = PyUnicode_Check(a.at[2]) ? PyUnicode_AsUTF8(a.at[2]) : nullptr;
        const std::string name = s ? s : "?";
        if (name == "f32")
          type = at::kFloat;
        else if (name == "bf16")
          type = at::kBFloat16;
        else if (name == "f16")
          type = at::kHalf;
        else
          bad("unknown dtype '" + name + "'");
      }
      k = stream.empty(shape, type, slots), v = stream.empty(shape, type, slots);
    }
    check(gar_kv_read(cache, static_cast<const int64_t *>(slots.data_ptr()), slots.size(0), k.data_ptr(), v.data_ptr(),
                      dtype_of(k, "out"), stream.raw),
          "gar_kv_read");
    if (a.at[3]) {
      changed(k), changed(v);
      return Py_NewRef(a.at[3]);
    }
    PyObject *pair = PyTuple_New(2);
    if (!pair) throw python_error();
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(std::move(k)));
    PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(std::move(v)));
    return pair;
  });
}

// The plan's workspace comes with the first call; that the stream of a call uses it is known to its allocator.
void use_workspace(PyObject *plan, PyObject *like, const Stream &stream) {
  PyObject *last = PyObject_GetAttr(plan, names_of().stream);
  if (!last) throw python_error();
  const bool known = last != Py_None && PyLong_AsVoidPtr(last) == static_cast<void *>(stream.raw);
  Py_DECREF(last);
  if (PyErr_Occurred()) throw python_error();
  if (known) return;
  PyObject *m = PyImport_ImportModule("paper_2004_09362_gb300.gar");
  PyObject *r = m ? PyObject_CallMethod(m, "_use_workspace", "OOK", plan, like, (unsigned long long)(uintptr_t)stream.raw) : nullptr;
  Py_XDECREF(m);
  if (!r) throw python_error();
  Py_DECREF(r);
}

PyObject *decode_attention(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"plan",  "q",      "cache", "page_table", "lengths",
                                        "scale", "window", "out",   "lse",        "stream"};
    const Arguments<10> a("gar_decode_attention", names, 5, args, n, kw);
    gar_attn_plan *plan = handle<gar_attn_plan>(a.at[0], "plan destroyed");
    const gar_kv_cache *cache = handle<gar_kv_cache>(a.at[2], "the cache has no address");
    const Tensor &q = rows(a.at[1], "q"), &lengths = integers(a.at[4], q.size(0), true, false, "lengths");
    const Tensor &table = tensor(a.at[3], "page_table");
    if (table.dim() != 2 || table.size(0) != q.size(0) || table.scalar_type() != at::kInt || !table.is_cuda() ||
        (table.stride(1) != 1 && table.size(1) > 1))
      bad("page_table must be int32 [batch, width] on the GPU with contiguous rows");
    const int batch = narrow(q.size(0), "the batch"), width = narrow(table.size(1), "the page table's width");
    const int window = a.at[6] ? narrow(integer(a.at[6]), "window") : 0;
    int shape[3];
    check(gar_attn_plan_shape(plan, &shape[0], &shape[1], &shape[2]), "gar_attn_plan_shape");
    if (q.size(1) != shape[0] || q.size(2) != shape[2])
      bad("q must be [batch, " + std::to_string(shape[0]) + ", " + std::to_string(shape[2]) + "]");
    Tensor out, lse;
    Device device;
    device.add(device_of(a.at[2]), "cache"), device.add(q, "q"), device.add(table, "page_table"), device.add(lengths, "lengths");
    if (a.at[7]) {
      out = rows(a.at[7], "out");
      if (out.sizes() != q.sizes()) bad("out must have q's shape");
      device.add(out, "out");
    }
    const bool given = a.at[8] && !PyBool_Check(a.at[8]), wanted = given || truth(a.at[8]);
    if (given) {
      lse = tensor(a.at[8], "lse");
      if (lse.scalar_type() != at::kFloat || lse.sizes() != q.sizes().slice(0, 2) || !lse.is_contiguous() || !lse.is_cuda())
        bad("lse must be a contiguous float32 CUDA tensor [batch, q_heads]");
      device.add(lse, "lse");
    }
    refuse_graded({&q, &out, &lse});
    const Stream stream(a.at[9], device.check());
    use_workspace(a.at[0], a.at[1], stream);
    if (!a.at[7]) out = stream.empty(q.sizes(), q.scalar_type(), q);
    if (wanted && !given) lse = stream.empty(q.sizes().slice(0, 2), at::kFloat, q);
    const double scale = a.at[5] ? number(a.at[5]) : 1.0 / std::sqrt((double)shape[2]);
    check(gar_decode_attention(plan, cache, q.data_ptr(), q.stride(0), q.stride(1), dtype_of(q, "q"), out.data_ptr(),
                               out.stride(0), out.stride(1), dtype_of(out, "out"),
                               wanted ? static_cast<float *>(lse.data_ptr()) : nullptr,
                               static_cast<const int32_t *>(table.data_ptr()), table.stride(0), width,
                               static_cast<const int32_t *>(lengths.data_ptr()), batch, (float)scale, window, stream.raw),
          "gar_decode_attention");
    if (a.at[7]) changed(out);
    if (given) changed(lse);
    PyObject *first = a.at[7] ? Py_NewRef(a.at[7]) : THPVariable_Wrap(std::move(out));
    if (!wanted) return first;
    PyObject *pair = first ? PyTuple_New(2) : nullptr;
    if (!pair) throw python_error();
    PyTuple_SET_ITEM(pair, 0, first);
    PyTuple_SET_ITEM(pair, 1, given ? Py_NewRef(a.at[8]) : THPVariable_Wrap(std::move(lse)));
    return pair;
  });
}

// int32 [batch, width] on the GPU, each row contiguous.
const Tensor &pages_of(PyObject *o, int64_t batch, const char *what) {
  const Tensor &t = tensor(o, what);
  if (t.dim() != 2 || (batch >= 0 && t.size(0) != batch) || t.scalar_type() != at::kInt || !t.is_cuda() ||
      (t.stride(1) != 1 && t.size(1) > 1))
    bad(std::string(what) + " must be int32 [batch, width] on the GPU with contiguous rows");
  narrow(t.size(1), "the page table's width");
  return t;
}

// No element twice (an expanded tensor's are): for outputs.
void refuse_expanded(const Tensor &t, const char *what) {
  for (int64_t i = 0; i < t.dim(); ++i)
    if (t.size(i) > 1 && t.stride(i) == 0) bad(std::string(what) + " has elements that share memory");
}

// A contiguous tensor of a shape and a type on the GPU.
const Tensor &exactly(PyObject *o, at::IntArrayRef shape, at::ScalarType type, const char *what) {
  const Tensor &t = tensor(o, what);
  if (t.sizes() != shape || t.scalar_type() != type || !t.is_cuda() || !t.is_contiguous()) {
    std::string n;
    for (int64_t x : shape) n += (n.empty() ? "" : ", ") + std::to_string(x);
    bad(std::string(what) + " must be a contiguous " + (type == at::kFloat ? "float32" : type == at::kInt ? "int32" : "int64") +
        " CUDA tensor [" + n + "]");
  }
  return t;
}

PyObject *tuple_of(std::initializer_list<PyObject *> items) {
  PyObject *t = PyTuple_New((Py_ssize_t)items.size());
  Py_ssize_t i = 0;
  for (PyObject *x : items) {
    if (t)
      PyTuple_SET_ITEM(t, i++, x);
    else
      Py_XDECREF(x);
  }
  if (!t) throw python_error();
  return t;
}

PyObject *prefix_attention(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"plan",       "q",       "cache", "prefix_table", "prefix_lengths",
                                        "page_table", "lengths", "scale", "out",          "lse", "stream"};
    const Arguments<11> a("gar_prefix_attention", names, 7, args, n, kw);
    gar_attn_plan *plan = handle<gar_attn_plan>(a.at[0], "plan destroyed");
    const gar_kv_cache *cache = handle<gar_kv_cache>(a.at[2], "the cache has no address");
    const Tensor &q = rows(a.at[1], "q"), &lengths = integers(a.at[6], q.size(0), true, false, "lengths");
    const Tensor &table = pages_of(a.at[5], q.size(0), "page_table"), &prefix = pages_of(a.at[3], -1, "prefix_table");
    const Tensor &prefix_lengths = integers(a.at[4], prefix.size(0), true, false, "prefix_lengths");
    const int batch = narrow(q.size(0), "the batch"), groups = narrow(prefix.size(0), "the number of prefixes");
    if (batch > 0 && (groups == 0 || batch % groups)) bad("the batch must be a multiple of the prefixes");
    int shape[3];
    check(gar_attn_plan_shape(plan, &shape[0], &shape[1], &shape[2]), "gar_attn_plan_shape");
    if (q.size(1) != shape[0] || q.size(2) != shape[2])
      bad("q must be [batch, " + std::to_string(shape[0]) + ", " + std::to_string(shape[2]) + "]");
    Tensor out, lse;
    Device device;
    device.add(device_of(a.at[2]), "cache"), device.add(q, "q"), device.add(prefix, "prefix_table");
    device.add(prefix_lengths, "prefix_lengths"), device.add(table, "page_table"), device.add(lengths, "lengths");
    if (a.at[8]) {
      out = rows(a.at[8], "out");
      if (out.sizes() != q.sizes()) bad("out must have q's shape");
      refuse_expanded(out, "out");
      device.add(out, "out");
    }
    const bool given = a.at[9] && !PyBool_Check(a.at[9]), wanted = given || truth(a.at[9]);
    if (given) {
      lse = exactly(a.at[9], q.sizes().slice(0, 2), at::kFloat, "lse");
      device.add(lse, "lse");
    }
    refuse_graded({&q, &out, &lse});
    const Stream stream(a.at[10], device.check());
    size_t bytes = 0;
    check(gar_prefix_attention_call_bytes(plan, cache, batch, groups, (int)prefix.size(1), (int)table.size(1), &bytes),
          "gar_prefix_attention_call_bytes");
    use_workspace(a.at[0], a.at[1], stream);
    // (freed at the end: for what comes next on the stream)
    Tensor workspace;
    if (bytes > 0) workspace = stream.empty({(int64_t)bytes}, at::kByte, q);
    if (!a.at[8]) out = stream.empty(q.sizes(), q.scalar_type(), q);
    if (wanted && !given) lse = stream.empty(q.sizes().slice(0, 2), at::kFloat, q);
    const double scale = a.at[7] ? number(a.at[7]) : 1.0 / std::sqrt((double)shape[2]);
    check(gar_prefix_attention(plan, cache, q.data_ptr(), q.stride(0), q.stride(1), dtype_of(q, "q"), out.data_ptr(),
                               out.stride(0), out.stride(1), dtype_of(out, "out"),
                               wanted ? static_cast<float *>(lse.data_ptr()) : nullptr,
                               static_cast<const int32_t *>(prefix.data_ptr()), prefix.stride(0), (int)prefix.size(1),
                               static_cast<const int32_t *>(prefix_lengths.data_ptr()), groups,
                               static_cast<const int32_t *>(table.data_ptr()), table.stride(0), (int)table.size(1),
                               static_cast<const int32_t *>(lengths.data_ptr()), batch, (float)scale,
                               bytes > 0 ? workspace.data_ptr() : nullptr, bytes,
                               stream.raw),
          "gar_prefix_attention");
    if (a.at[8]) changed(out);
    if (given) changed(lse);
    PyObject *first = a.at[8] ? Py_NewRef(a.at[8]) : THPVariable_Wrap(std::move(out));
    if (!wanted) return first;
    return tuple_of({first, given ? Py_NewRef(a.at[9]) : THPVariable_Wrap(std::move(lse))});
  });
}

PyObject *kv_weigh(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"q", "cache", "page_table", "lengths", "lse", "weights", "scale", "window", "out", "stream"};
    const Arguments<10> a("gar_kv_weigh", names, 6, args, n, kw);
    const gar_kv_cache *cache = handle<gar_kv_cache>(a.at[1], "the cache has no address");
    const Tensor &q = rows(a.at[0], "q"), &lengths = integers(a.at[3], q.size(0), true, false, "lengths");
    const Tensor &table = pages_of(a.at[2], q.size(0), "page_table"), &lse = exactly(a.at[4], q.sizes().slice(0, 2), at::kFloat, "lse");
    if (q.size(2) != cache->dim) bad("q must have the cache's channels");
    const auto check_weights = [&](const Tensor &t, const char *what) {
      if (t.dim() != 3 || t.size(0) != q.size(0) || t.size(1) != cache->heads || t.scalar_type() != at::kFloat || !t.is_cuda() ||
          (t.stride(2) != 1 && t.size(2) > 1))
        bad(std::string(what) + " must be float32 [batch, the cache's heads, rows] on the GPU with contiguous rows");
    };
    const Tensor &weights = tensor(a.at[5], "weights");
    check_weights(weights, "weights");
    Tensor out;
    Device device;
    device.add(device_of(a.at[1]), "cache"), device.add(q, "q"), device.add(table, "page_table"), device.add(lengths, "lengths");
    device.add(lse, "lse"), device.add(weights, "weights");
    if (a.at[8]) {
      out = tensor(a.at[8], "out");
      check_weights(out, "out");
      if (out.sizes() != weights.sizes()) bad("out must have weights' shape");
      refuse_expanded(out, "out");
      device.add(out, "out");
    }
    refuse_graded({&q, &lse, &weights, &out});
    const int batch = narrow(q.size(0), "the batch"), window = a.at[7] ? narrow(integer(a.at[7]), "window") : 0;
    const Stream stream(a.at[9], device.check());
    if (!a.at[8]) out = stream.empty(weights.sizes(), at::kFloat, q);
    const double scale = a.at[6] ? number(a.at[6]) : 1.0 / std::sqrt((double)cache->dim);
    check(gar_kv_weigh(cache, q.data_ptr(), q.stride(0), q.stride(1), dtype_of(q, "q"), (int)q.size(1),
                       static_cast<const float *>(lse.data_ptr()), static_cast<const float *>(weights.data_ptr()), weights.stride(0),
                       weights.stride(1), static_cast<float *>(out.data_ptr()), out.stride(0), out.stride(1), weights.size(2),
                       static_cast<const int32_t *>(table.data_ptr()), table.stride(0), (int)table.size(1),
                       static_cast<const int32_t *>(lengths.data_ptr()), batch, (float)scale, window, stream.raw),
          "gar_kv_weigh");
    if (!a.at[8]) return THPVariable_Wrap(std::move(out));
    changed(out);
    return Py_NewRef(a.at[8]);
  });
}

PyObject *kv_evict(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"cache", "weights", "positions", "page_table", "lengths", "keep", "first", "recent", "out", "stream"};
    const Arguments<10> a("gar_kv_evict", names, 6, args, n, kw);
    const gar_kv_cache *cache = handle<gar_kv_cache>(a.at[0], "the cache has no address");
    const Tensor &any = tensor(a.at[1], "weights");
    if (any.dim() != 3 || any.size(1) != cache->heads) bad("weights must be [batch, the cache's heads, rows]");
    const Tensor &weights = exactly(a.at[1], any.sizes(), at::kFloat, "weights");
    const Tensor &positions = exactly(a.at[2], weights.sizes(), at::kInt, "positions");
    const int64_t count = weights.size(0);
    const Tensor &table = pages_of(a.at[3], count, "page_table"), &lengths = integers(a.at[4], count, true, false, "lengths");
    const int batch = narrow(count, "the batch"), keep = narrow(integer(a.at[5]), "keep"),
              first = a.at[6] ? narrow(integer(a.at[6]), "first") : 0, recent = a.at[7] ? narrow(integer(a.at[7]), "recent") : 0;
    Tensor out[3];
    Device device;
    device.add(device_of(a.at[0]), "cache"), device.add(weights, "weights"), device.add(positions, "positions");
    device.add(table, "page_table"), device.add(lengths, "lengths");
    if (a.at[8]) {
      if (!PyTuple_Check(a.at[8]) || PyTuple_GET_SIZE(a.at[8]) != 3) bad("out must be three tensors: weights, positions, lengths");
      out[0] = exactly(PyTuple_GET_ITEM(a.at[8], 0), weights.sizes(), at::kFloat, "out's weights");
      out[1] = exactly(PyTuple_GET_ITEM(a.at[8], 1), weights.sizes(), at::kInt, "out's positions");
      out[2] = exactly(PyTuple_GET_ITEM(a.at[8], 2), {count}, at::kInt, "out's lengths");
      for (const Tensor &t : out) device.add(t, "out");
    }
    refuse_graded({&weights, &out[0]});
    const Stream stream(a.at[9], device.check());
    if (!a.at[8]) {
      out[0] = stream.empty(weights.sizes(), at::kFloat, weights), out[1] = stream.empty(weights.sizes(), at::kInt, weights);
      out[2] = stream.empty({count}, at::kInt, weights);
    }
    check(gar_kv_evict(cache, static_cast<const float *>(weights.data_ptr()), static_cast<const int32_t *>(positions.data_ptr()),
                       weights.size(2), static_cast<const int32_t *>(table.data_ptr()), table.stride(0), (int)table.size(1),
                       static_cast<const int32_t *>(lengths.data_ptr()), batch, keep, first, recent,
                       static_cast<float *>(out[0].data_ptr()), static_cast<int32_t *>(out[1].data_ptr()),
                       static_cast<int32_t *>(out[2].data_ptr()), stream.raw),
          "gar_kv_evict");
    changed_cache(a.at[0]);
    if (a.at[8]) {
      for (const Tensor &t : out) changed(t);
      return Py_NewRef(a.at[8]);
    }
    return tuple_of({THPVariable_Wrap(std::move(out[0])), THPVariable_Wrap(std::move(out[1])), THPVariable_Wrap(std::move(out[2]))});
  });
}

PyObject *verify_drafts(PyObject *, PyObject *const *args, Py_ssize_t n, PyObject *kw) {
  return guarded([&] {
    static const char *const names[] = {"target", "draft", "tokens", "uniform", "out", "stream"};
    const Arguments<6> a("gar_verify_drafts", names, 4, args, n, kw);
    const auto table = [&](PyObject *o, const char *what) -> const Tensor & {
      const Tensor &t = tensor(o, what);
      if (t.dim() != 3 || !t.is_cuda() || (t.stride(2) != 1 && t.size(2) > 1))
        bad(std::string(what) + " must be [batch, drafts, vocab] on the GPU with contiguous rows");
      return t;
    };
    const Tensor &target = table(a.at[0], "target"), &draft = table(a.at[1], "draft"), &given = tensor(a.at[2], "tokens");
    const int64_t batch = target.size(0), drafts = draft.size(1), vocab = target.size(2);
    if (draft.size(0) != batch || draft.size(2) != vocab || target.size(1) != drafts + 1 || target.scalar_type() != draft.scalar_type())
      bad("target must be [batch, drafts + 1, vocab] and draft [batch, drafts, vocab], alike in dtype");
    const auto type = given.scalar_type();
    if (type != at::kLong && type != at::kInt) bad("tokens: this dtype is not supported");
    const int64_t shape[2] = {batch, drafts}, longer[2] = {batch, drafts + 1};
    const Tensor &tokens = exactly(a.at[2], shape, type, "tokens"), &uniform = exactly(a.at[3], longer, at::kFloat, "uniform");
    Tensor out[2];
    Device device;
    device.add(target, "target"), device.add(draft, "draft"), device.add(tokens, "tokens"), device.add(uniform, "uniform");
    if (a.at[4]) {
      if (!PyTuple_Check(a.at[4]) || PyTuple_GET_SIZE(a.at[4]) != 2) bad("out must be two tensors: tokens, accepted");
      out[0] = exactly(PyTuple_GET_ITEM(a.at[4], 0), longer, type, "out's tokens");
      out[1] = exactly(PyTuple_GET_ITEM(a.at[4], 1), {batch}, at::kInt, "out's accepted");
      device.add(out[0], "out"), device.add(out[1], "out");
    }
    refuse_graded({&target, &draft, &uniform});
    const Stream stream(a.at[5], device.check());
    if (!a.at[4]) out[0] = stream.empty(longer, type, target), out[1] = stream.empty({batch}, at::kInt, target);
    check(gar_verify_drafts(target.data_ptr(), target.stride(0), target.stride(1), draft.data_ptr(), draft.stride(0), draft.stride(1),
                            dtype_of(target, "target"), vocab, tokens.data_ptr(), (int)tokens.element_size(),
                            static_cast<const float *>(uniform.data_ptr()), narrow(batch, "the batch"),
                            narrow(drafts, "the number of drafts"), out[0].data_ptr(), static_cast<int32_t *>(out[1].data_ptr()),
                            stream.raw),
          "gar_verify_drafts");
    if (a.at[4]) {
      changed(out[0]), changed(out[1]);
      return Py_NewRef(a.at[4]);
    }
    return tuple_of({THPVariable_Wrap(std::move(out[0])), THPVariable_Wrap(std::move(out[1]))});
  });
}


PyMethodDef methods[] = {
    {"gar_rope", (PyCFunction)(void (*)())rope, METH_FASTCALL | METH_KEYWORDS,
     "gar_rope(x, positions, table, layout='half', inverse=False, out=None, stream=None)\n--\n\n"
     "x [tokens, heads, dim] with its first rot channels rotated by the table's rows at\n"
     "`positions` (int32 or int64); out may be x.  With inverse, the gradient: x is grad_out, the result\n"
     "grad_x.  layout: 'half' or 'interleaved'.  Gradients flow through a call without out, but not to the table."},
    {"gar_kv_write", (PyCFunction)(void (*)())kv_write, METH_FASTCALL | METH_KEYWORDS,
     "gar_kv_write(cache, k, v, slots, positions=None, table=None, layout='half', stream=None)\n--\n\n"
     "Writes k, v [tokens, heads, dim] to the cache's slots (int64; negative: skipped),\n"
     "quantised where the cache is; with positions and table, the keys rotated first.  Has no gradient, nor have\n"
     "the calls that read the cache: tensors that ask for one are refused."},
    {"gar_kv_read", (PyCFunction)(void (*)())kv_read, METH_FASTCALL | METH_KEYWORDS,
     "gar_kv_read(cache, slots, dtype=None, out=None, stream=None)\n--\n\n"
     "(k, v), each [tokens, heads, dim], of the cache's slots; rows of negative slots are 0.\n"
     "dtype: 'f32', 'bf16' or 'f16' (default: the cache's, bf16 for an 8-bit one); out: a pair of\n"
     "contiguous tensors to fill instead."},
    {"gar_decode_attention", (PyCFunction)(void (*)())decode_attention, METH_FASTCALL | METH_KEYWORDS,
     "gar_decode_attention(plan, q, cache, page_table, lengths, scale=None, window=0, out=None,\n"
     "                     lse=None, stream=None)\n--\n\n"
     "Attention of q [batch, q_heads, dim] over each sequence's cached rows.\n\n"
     "page_table: int32 [batch, width]; lengths: int32 [batch], the new token's row included.\n"
     "scale: dim**-0.5 by default.  window: only the last `window` rows (0: all).  out: q's shape, of\n"
     "q's dtype or float32.  lse: True, or a contiguous float32 [batch, q_heads] tensor, returns\n"
     "(out, log of the sum of weights); else returns out.  The plan's workspace is allocated on its\n"
     "first call; make one before capturing calls into a CUDA graph."},
    {"gar_prefix_attention", (PyCFunction)(void (*)())prefix_attention, METH_FASTCALL | METH_KEYWORDS,
     "gar_prefix_attention(plan, q, cache, prefix_table, prefix_lengths, page_table, lengths,\n"
     "                     scale=None, out=None, lse=None, stream=None)\n--\n\n"
     "Attention of q [batch, q_heads, dim] over a prefix that sequences share, then each one's own rows.\n\n"
     "prefix_table: int32 [groups, width]; prefix_lengths: int32 [groups].  Each batch / groups neighbouring sequences\n"
     "share a prefix, which is read once for them.  The rest is as in gar_decode_attention; drafted tokens of a\n"
     "context are such sequences, whose own rows are the drafts before them and themselves."},
    {"gar_kv_weigh", (PyCFunction)(void (*)())kv_weigh, METH_FASTCALL | METH_KEYWORDS,
     "gar_kv_weigh(q, cache, page_table, lengths, lse, weights, scale=None, window=0, out=None, stream=None)\n--\n\n"
     "weights float32 [batch, cached heads, rows] plus what each row gets in the attention of q [batch, q_heads, dim]:\n"
     "the sum of exp(scale q.k - lse) over its head's queries.  lse: float32 [batch, q_heads], as the attention gave it.  out may be\n"
     "weights.  Has no gradient."},
    {"gar_kv_evict", (PyCFunction)(void (*)())kv_evict, METH_FASTCALL | METH_KEYWORDS,
     "gar_kv_evict(cache, weights, positions, page_table, lengths, keep, first=0, recent=0, out=None, stream=None)\n--\n\n"
     "Cuts each sequence of more than `keep` rows down to that many, in each head those of most weight, moving kept rows of\n"
     "the cache to the places of rows that go.  The `first` rows and those of the `recent` last positions are kept whatever\n"
     "they weigh.  weights: float32, positions: int32, both contiguous [batch, cached heads, rows].  Returns the weights and positions of what is left\n"
     "(0 and -1 past it) and the lengths; out: three tensors to fill instead."},
    {"gar_verify_drafts", (PyCFunction)(void (*)())verify_drafts, METH_FASTCALL | METH_KEYWORDS,
     "gar_verify_drafts(target, draft, tokens, uniform, out=None, stream=None)\n--\n\n"
     "Which drafted tokens stand, and the token after them.  target [batch, drafts + 1, vocab] and draft [batch, drafts, vocab]:\n"
     "probabilities; tokens: int32 or int64 [batch, drafts], negative from where a sequence has no more; uniform:\n"
     "float32 [batch, drafts + 1] in [0, 1).  Returns tokens [batch, drafts + 1] (those that stand, the next one, then -1) and\n"
     "int32 [batch], how many stand; out: two tensors to fill instead."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Compiled calls of the decoding operators.", -1, methods,
                      nullptr,               nullptr,    nullptr,                                     nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
