// Argument marshalling of the operators around a bounded KV cache, for binding.py: checks type, shape, packing and device of the
// tensors and makes the C call.  In Python the checks (0.5 us a tensor) and a ctypes call of 26 arguments (2.7 us) took three
// quarters of a small call; the kernels of one take 2 to 5 us.  No arithmetic of any operator happens here.
//
// Every entry returns None, or (code, text) which binding.py raises.  The C functions' addresses come from binding.py (attach), so
// that there is one libmlora.so in the process.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "../../include/mlora.h"

namespace {

decltype(&mlora_rope_append) f_rope = nullptr;
decltype(&mlora_attention_scored) f_scored = nullptr;
decltype(&mlora_kv_evict) f_evict = nullptr;
decltype(&mlora_last_error) f_error = nullptr;

struct Refused { std::string text; };

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refused{std::string(what) + ": expected a tensor"};
  return THPVariable_Unpack(o);
}

std::string describe(const at::Tensor& t) {
  std::string s = c10::toString(t.scalar_type());
  s += " (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  s += ") with strides (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
  return s + ") on " + t.device().str();
}

// the device of a call: that of its first tensor, which must be the current one
int device_of(const at::Tensor& t, const char* what) {
  if (!t.is_cuda()) throw Refused{std::string(what) + ": expected a CUDA tensor, got " + describe(t)};
  const int dev = t.get_device();
  if (dev != c10::cuda::current_device()) throw Refused{std::string(what) + ": lies on CUDA device " + std::to_string(dev) + ", which is not the current device"};
  return dev;
}

// the address of a packed tensor of this type and shape on this device; None: null
void* packed(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, int dev, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type || t.sizes() != at::IntArrayRef(shape) || !t.is_contiguous() || !t.is_cuda() || t.get_device() != dev) {
    std::string s = std::string(what) + ": expected a packed " + c10::toString(type) + " (";
    bool first = true;
    for (int64_t x : shape) { s += (first ? "" : ", ") + std::to_string(x); first = false; }
    throw Refused{s + ") on CUDA device " + std::to_string(dev) + ", got " + describe(t)};
  }
  return t.data_ptr();
}

// rows of `width` packed features, [rows][width] or [rows][heads][head_dim], with any stride between rows
void* row_tensor(PyObject* o, int64_t rows, int64_t width, at::ScalarType type, int dev, const char* what, int64_t& stride) {
  stride = 0;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  bool ok = t.scalar_type() == type && t.is_cuda() && t.get_device() == dev && (t.dim() == 2 || t.dim() == 3) && t.size(0) == rows;
  if (ok && t.dim() == 2) ok = t.size(1) == width && t.stride(1) == 1;
  else if (ok) ok = t.size(1) * t.size(2) == width && t.stride(2) == 1 && (t.size(1) == 1 || t.stride(1) == t.size(2));
  if (!ok)
    throw Refused{std::string(what) + ": expected " + std::to_string(rows) + " rows of " + std::to_string(width) + " packed " + c10::toString(type) +
                  " features on CUDA device " + std::to_string(dev) + ", got " + describe(t)};
  stride = rows > 1 ? t.stride(0) : width;
  return t.data_ptr();
}

int32_t whole(PyObject* o, const char* what) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); throw Refused{std::string(what) + ": expected a whole number"}; }
  if (v < INT32_MIN || v > INT32_MAX) throw Refused{std::string(what) + ": out of range"};
  return (int32_t)v;
}
double number(PyObject* o, const char* what) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw Refused{std::string(what) + ": expected a number"}; }
  return v;
}
int32_t size32(int64_t v, const char* what) {
  if (v > INT32_MAX) throw Refused{std::string(what) + ": too large"};
  return (int32_t)v;
}

PyObject* refused(int code, const std::string& text) { return Py_BuildValue("(is)", code, text.c_str()); }

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F&& f) {
  if (n != want || f_error == nullptr) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or attach() was not called");
    return nullptr;
  }
  try {
    const int code = f();
    if (code != MLORA_OK) return refused(code, f_error(nullptr));
    Py_RETURN_NONE;
  } catch (const Refused& r) {
    return refused(MLORA_ERR_ARG, r.text);
  } catch (const std::exception& e) {
    return refused(MLORA_ERR_CUDA, e.what());
  }
}

constexpr at::ScalarType F16 = at::kHalf, F32 = at::kFloat, F64 = at::kDouble, I32 = at::kInt;

// q, k, v, positions, freq, q_out, own_k, own_v, suffix_len, status, gain, interleaved, own_weight, own_position
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 14, [&] {
    const bool has_q = a[0] != Py_None, app = a[6] != Py_None;
    if (has_q != (a[5] != Py_None)) throw Refused{"rope_append: q and q_out go together"};
    if (app != (a[1] != Py_None) || app != (a[2] != Py_None) || app != (a[7] != Py_None)) throw Refused{"rope_append: k, v, own_k and own_v go together"};
    if (!has_q && !app) throw Refused{"rope_append: nothing to do"};
    const at::Tensor &pos = tensor(a[3], "positions"), &freq = tensor(a[4], "freq");
    const int dev = device_of(pos, "positions");
    const int64_t rows = pos.numel();
    const at::ScalarType type = tensor(has_q ? a[0] : a[1], "q or k").scalar_type();
    if (type != F16 && type != F32) throw Refused{std::string("rope_append: rows of ") + c10::toString(type)};
    int64_t n = rows, Hq = 0, Hkv = 0, cap = 0, hd = 0, qs, ks, vs;
    if (has_q) {
      const at::Tensor& t = tensor(a[5], "q_out");
      if (t.dim() != 3) throw Refused{"q_out: expected [rows][Hq][hd], got " + describe(t)};
      Hq = t.size(1); hd = t.size(2);
    }
    if (app) {
      const at::Tensor& t = tensor(a[6], "own_k");
      if (t.dim() != 4 || (has_q && t.size(3) != hd)) throw Refused{"own_k: expected [n][Hkv][capacity][hd], got " + describe(t)};
      n = t.size(0); Hkv = t.size(1); cap = t.size(2); hd = t.size(3);
    }
    if (n == 0 || rows == 0 || rows % n) throw Refused{"rope_append: no rows, or not the same number for every stream"};
    void* q = row_tensor(a[0], rows, Hq * hd, type, dev, "q", qs);
    void* k = row_tensor(a[1], rows, Hkv * hd, type, dev, "k", ks);
    void* v = row_tensor(a[2], rows, Hkv * hd, type, dev, "v", vs);
    if (!pos.is_contiguous() || pos.scalar_type() != I32) throw Refused{"positions: expected packed int32, got " + describe(pos)};
    const int interleaved = PyObject_IsTrue(a[11]);
    if (interleaved < 0) { PyErr_Clear(); throw Refused{"interleaved: expected a truth value"}; }
    return f_rope(q, k, v, type == F32, qs, ks, vs, pos.data_ptr<int32_t>(), (const double*)packed(a[4], F64, {freq.numel()}, dev, "freq"),
                  (float)number(a[10], "gain"), size32(2 * freq.numel(), "freq"), interleaved, size32(n, "streams"), size32(rows / n, "rows"),
                  size32(Hq, "heads"), size32(Hkv, "heads"), size32(hd, "head_dim"), packed(a[5], F16, {rows, Hq, hd}, dev, "q_out"),
                  packed(a[6], F16, {n, Hkv, cap, hd}, dev, "own_k"), packed(a[7], F16, {n, Hkv, cap, hd}, dev, "own_v"), size32(cap, "own_capacity"),
                  (const int32_t*)(app ? packed(a[8], I32, {n}, dev, "suffix_len") : nullptr), (float*)packed(a[12], F32, {n, Hkv, cap}, dev, "own_weight"),
                  (int32_t*)packed(a[13], I32, {n, Hkv, cap}, dev, "own_position"), (int32_t*)(app ? packed(a[9], I32, {1}, dev, "status") : nullptr),
                  c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream());
  });
}

void* scratch(PyObject* o, int dev, size_t& bytes) {
  const at::Tensor& t = tensor(o, "workspace");
  if (!t.is_cuda() || t.get_device() != dev || !t.is_contiguous()) throw Refused{"workspace: expected a packed tensor on the call's device, got " + describe(t)};
  bytes = t.nbytes();
  return t.data_ptr();
}

// q, prefix_k, prefix_v, own_k, own_v, suffix_len, suffix_bound, tree_parent, out, own_weight, prefix_weight, workspace, status
PyObject* attention_scored(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 13, [&] {
    const at::Tensor &q = tensor(a[0], "q"), &ok = tensor(a[3], "own_k");
    if (q.dim() != 3) throw Refused{"q: expected [rows][Hq][hd], got " + describe(q)};
    if (ok.dim() != 4) throw Refused{"own_k: expected [n][Hkv][capacity][hd], got " + describe(ok)};
    const int dev = device_of(q, "q");
    const int64_t rows = q.size(0), Hq = q.size(1), hd = q.size(2), n = ok.size(0), Hkv = ok.size(1), cap = ok.size(2);
    if (n == 0 || rows % n) throw Refused{"attention_scored: rows that are no multiple of the streams"};
    const int64_t T = rows / n;
    int64_t P = 0;
    if (a[1] != Py_None) {
      const at::Tensor& t = tensor(a[1], "prefix_k");
      if (t.dim() != 3) throw Refused{"prefix_k: expected [Hkv][P][hd], got " + describe(t)};
      P = t.size(1);
    }
    size_t bytes;
    void* ws = scratch(a[11], dev, bytes);
    return f_scored(packed(a[0], F16, {rows, Hq, hd}, dev, "q"), packed(a[1], F16, {Hkv, P, hd}, dev, "prefix_k"),
                    packed(a[2], F16, {Hkv, P, hd}, dev, "prefix_v"), size32(P, "prefix"), packed(a[3], F16, {n, Hkv, cap, hd}, dev, "own_k"),
                    packed(a[4], F16, {n, Hkv, cap, hd}, dev, "own_v"), size32(cap, "own_capacity"), (const int32_t*)packed(a[5], I32, {n}, dev, "suffix_len"),
                    whole(a[6], "suffix_bound"), (const int32_t*)packed(a[7], I32, {n, T}, dev, "tree_parent"), size32(n, "streams"), size32(T, "rows"),
                    size32(Hq, "heads"), size32(Hkv, "heads"), size32(hd, "head_dim"), packed(a[8], F16, {rows, Hq, hd}, dev, "out"),
                    (float*)packed(a[9], F32, {n, Hkv, cap}, dev, "own_weight"), (float*)packed(a[10], F32, {Hkv, P}, dev, "prefix_weight"), ws, bytes,
                    (int32_t*)packed(a[12], I32, {1}, dev, "status"), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream());
  });
}

// own_k, own_v, own_weight, own_position, suffix_len, suffix_bound, newest, budget, recent, out_weight, out_position, out_len, workspace,
// status, out_source
PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 15, [&] {
    const at::Tensor& ok = tensor(a[0], "own_k");
    if (ok.dim() != 4) throw Refused{"own_k: expected [n][Hkv][capacity][hd], got " + describe(ok)};
    const int dev = device_of(ok, "own_k");
    const int64_t n = ok.size(0), Hkv = ok.size(1), cap = ok.size(2), hd = ok.size(3);
    const int32_t budget = whole(a[7], "budget");
    size_t bytes;
    void* ws = scratch(a[12], dev, bytes);
    return f_evict(packed(a[0], F16, {n, Hkv, cap, hd}, dev, "own_k"), packed(a[1], F16, {n, Hkv, cap, hd}, dev, "own_v"),
                   (const float*)packed(a[2], F32, {n, Hkv, cap}, dev, "own_weight"), (const int32_t*)packed(a[3], I32, {n, Hkv, cap}, dev, "own_position"),
                   size32(cap, "own_capacity"), (const int32_t*)packed(a[4], I32, {n}, dev, "suffix_len"), whole(a[5], "suffix_bound"),
                   (const int32_t*)packed(a[6], I32, {n}, dev, "newest"), budget, whole(a[8], "recent"), size32(n, "streams"), size32(Hkv, "heads"),
                   size32(hd, "head_dim"), (float*)packed(a[9], F32, {n, Hkv, cap}, dev, "out_weight"), (int32_t*)packed(a[10], I32, {n, Hkv, cap}, dev, "out_position"),
                   (int32_t*)packed(a[11], I32, {n}, dev, "out_len"), (int32_t*)packed(a[14], I32, {n, Hkv, budget}, dev, "out_source"), ws, bytes,
                   (int32_t*)packed(a[13], I32, {1}, dev, "status"), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream());
  });
}

// the addresses of mlora_rope_append, mlora_attention_scored, mlora_kv_evict, mlora_last_error
PyObject* attach(PyObject*, PyObject* args) {
  unsigned long long r, s, e, l;
  if (!PyArg_ParseTuple(args, "KKKK", &r, &s, &e, &l)) return nullptr;
  f_rope = (decltype(f_rope))r; f_scored = (decltype(f_scored))s; f_evict = (decltype(f_evict))e; f_error = (decltype(f_error))l;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"rope_append", (PyCFunction)(void*)rope_append, METH_FASTCALL, nullptr},
    {"attention_scored", (PyCFunction)(void*)attention_scored, METH_FASTCALL, nullptr},
    {"kv_evict", (PyCFunction)(void*)kv_evict, METH_FASTCALL, nullptr},
    {"attach", attach, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
