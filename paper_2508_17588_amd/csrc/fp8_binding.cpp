// The calls of the 8-bit building blocks from Python: takes tensors apart, checks them and makes the call of include/hero.h whose
// address it was given.  Host code only, a module of its own (_fp8_binding): on a few rows these calls are as short as their
// launch, some 3 us, and checking seven tensors from Python took as long again (one row of 1920 channels, hero_gather_rms_fp8).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/hero.h"

namespace {

struct {
  decltype(&hero_quantize_fp8) quantize;
  decltype(&hero_gather_rms_fp8) rms;
  decltype(&hero_linear_fp8) linear;
  decltype(&hero_linear_fp8_quantized) linear_quantized;
  PyObject* device;                    // () -> the current device
  PyObject* stream;                    // device -> the handle of its current stream
} calls = {};

struct Refused {};                     // a Python exception is set
[[noreturn]] void refuse(PyObject* type, const char* format, const char* name = "") {
  PyErr_Format(type, format, name);
  throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor", name);
  return THPVariable_Unpack(o);
}
const at::Tensor* optional(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int32_t int32(int64_t v) {
  if (v >= (int64_t)1 << 31 || v < -((int64_t)1 << 31)) refuse(PyExc_ValueError, "sizes must stay below 2^31");
  return (int32_t)v;
}

// The current device, on which all tensors of a call lie, and its current stream
struct Place {
  int64_t device;
  void* stream;
};
Place place(const at::Tensor& first) {
  if (!first.is_cuda()) refuse(PyExc_TypeError, "not a device tensor");
  PyObject* d = PyObject_CallNoArgs(calls.device);
  if (d == nullptr) throw Refused();
  PyObject* s = PyObject_CallOneArg(calls.stream, d);
  const int64_t device = PyLong_AsLongLong(d);
  Py_DECREF(d);
  if (s == nullptr) throw Refused();
  void* stream = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  if (PyErr_Occurred()) throw Refused();
  return {device, stream};
}

// Address of a contiguous tensor of that type on the device that has room for `least` elements
void* address(const at::Tensor& t, at::ScalarType type, const Place& at, int64_t least, const char* name) {
  if (t.scalar_type() != type || !t.is_contiguous() || !t.is_cuda())
    refuse(PyExc_TypeError, (std::string("%s must be a contiguous device tensor of type ") + c10::toString(type)).c_str(), name);
  if (t.get_device() != at.device) refuse(PyExc_ValueError, "%s does not lie on the current device", name);
  if (t.numel() < least) refuse(PyExc_ValueError, "%s is too small", name);
  return t.data_ptr();
}
void* address(const at::Tensor* t, at::ScalarType type, const Place& at, int64_t least, const char* name) {
  return t == nullptr ? nullptr : address(*t, type, at, least, name);
}

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  return a != nullptr && b != nullptr && a_bytes > 0 && b_bytes > 0 && (uintptr_t)a < (uintptr_t)b + (uint64_t)b_bytes &&
         (uintptr_t)b < (uintptr_t)a + (uint64_t)a_bytes;
}

int32_t activation(const at::Tensor& x) {
  if (x.scalar_type() == at::kFloat) return HERO_DTYPE_FP32;
  if (x.scalar_type() != at::kBFloat16) refuse(PyExc_TypeError, "unsupported activation dtype %s", c10::toString(x.scalar_type()));
  return HERO_DTYPE_BF16;
}

template <typename Body>
PyObject* entry(Py_ssize_t given, Py_ssize_t wanted, Body body) {
  try {
    if (given != wanted) refuse(PyExc_TypeError, "wrong number of arguments%s");
    return PyLong_FromLong(body());
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
// the call itself, without the interpreter's lock: a launch may wait for room in its queue
template <typename Call>
int unlocked(Call call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}

// (addresses of the four calls, current device, stream of a device)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&] {
    calls.quantize = (decltype(calls.quantize))integer(a[0]);
    calls.rms = (decltype(calls.rms))integer(a[1]);
    calls.linear = (decltype(calls.linear))integer(a[2]);
    calls.linear_quantized = (decltype(calls.linear_quantized))integer(a[3]);
    Py_INCREF(a[4]);
    Py_INCREF(a[5]);
    calls.device = a[4];
    calls.stream = a[5];
    return 0;
  });
}

// (x, q, scales, block_rows)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 4, [&] {
    const at::Tensor &x = tensor(a[0], "x"), &q = tensor(a[1], "q"), &scales = tensor(a[2], "scales");
    const Place p = place(x);
    if (x.dim() != 2) refuse(PyExc_ValueError, "x must be [rows, columns]%s");
    const int64_t block_rows = integer(a[3]);
    if (block_rows != 1 && block_rows != HERO_FP8_BLOCK) refuse(PyExc_ValueError, "block_rows must be 1 or 128%s");
    const int32_t rows = int32(x.size(0)), columns = int32(x.size(1)), type = activation(x);
    const int64_t blocks = (rows + block_rows - 1) / block_rows, pitch = HERO_FP8_SCALE_PITCH((int64_t)columns);
    const void* from = address(x, x.scalar_type(), p, 0, "x");
    void* to = address(q, at::kFloat8_e4m3fn, p, (int64_t)rows * columns, "q");
    void* to_scales = address(scales, at::kFloat8_e8m0fnu, p, blocks * pitch, "scales");
    return unlocked([&] { return calls.quantize(from, type, rows, columns, (int32_t)block_rows, to, to_scales, p.stream); });
  });
}

// (x, add, rows, n_rows, gain, eps, q, scales, sum)
PyObject* rms(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 9, [&] {
    const at::Tensor &x = tensor(a[0], "x"), &gain = tensor(a[4], "gain"), &q = tensor(a[6], "q"), &scales = tensor(a[7], "scales");
    const at::Tensor *add = optional(a[1], "add"), *rows = optional(a[2], "rows"), *sum = optional(a[8], "sum");
    const Place p = place(x);
    if (x.dim() < 1) refuse(PyExc_ValueError, "x must be [rows, hidden]%s");
    const int64_t size = x.numel(), listed = integer(a[3]);
    const int32_t hidden = int32(x.size(-1)), n_rows = int32(listed);
    const double eps = PyFloat_AsDouble(a[5]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused();
    const int64_t elements = (int64_t)n_rows * hidden;
    if (gain.numel() != hidden || (add && add->numel() != size) || (!rows && size < elements))
      refuse(PyExc_ValueError, "shape mismatch%s");
    const int32_t type = activation(x);
    const void* from = address(x, x.scalar_type(), p, 0, "x");
    const void* branch = address(add, at::kBFloat16, p, 0, "add");
    const int32_t* list = (const int32_t*)address(rows, at::kInt, p, n_rows, "rows");
    const void* gains = address(gain, at::kBFloat16, p, hidden, "gain");
    void* total = address(sum, x.scalar_type(), p, elements, "sum");
    void* to = address(q, at::kFloat8_e4m3fn, p, elements, "q");
    const int64_t scale_bytes = (int64_t)n_rows * HERO_FP8_SCALE_PITCH(hidden);
    void* to_scales = address(scales, at::kFloat8_e8m0fnu, p, scale_bytes, "scales");
    // (the library does not know how many rows there are to be listed)
    auto reads = [&](const void* out, int64_t bytes) {
      return overlap(out, bytes, from, x.nbytes()) || overlap(out, bytes, branch, add ? add->nbytes() : 0);
    };
    if (rows && (reads(total, elements * x.element_size()) || reads(to, elements) || reads(to_scales, scale_bytes)))
      refuse(PyExc_ValueError, "sum, q and scales cannot share memory with x or add where rows are listed: other rows may still be read%s");
    return unlocked([&] { return calls.rms(from, type, branch, list, n_rows, hidden, gains, (float)eps, total, to, to_scales, p.stream); });
  });
}

// What both products are given: (a, a_scales, w, w_scales, bias), ..., act, scratch
struct Operands {
  Place p;
  int32_t m, n, k, act;
  const void *a, *a_scales, *w, *w_scales, *bias;
  void* scratch;
  size_t scratch_bytes;

  Operands(PyObject* const* o, PyObject* act_, PyObject* scratch_) {
    const at::Tensor &ta = tensor(o[0], "a"), &tw = tensor(o[2], "w");
    const at::Tensor *tb = optional(o[4], "bias"), *ts = optional(scratch_, "scratch");
    p = place(ta);
    if (ta.dim() != 2 || tw.dim() != 2) refuse(PyExc_ValueError, "a and w must be [rows, k]%s");
    if (tw.size(1) != ta.size(1) || (tb && tb->numel() != tw.size(0))) refuse(PyExc_ValueError, "shape mismatch%s");
    m = int32(ta.size(0));
    n = int32(tw.size(0));
    k = int32(ta.size(1));
    act = int32(integer(act_));
    const int64_t pitch = HERO_FP8_SCALE_PITCH((int64_t)k);
    a = address(ta, at::kFloat8_e4m3fn, p, 0, "a");
    a_scales = address(tensor(o[1], "a_scales"), at::kFloat8_e8m0fnu, p, m * pitch, "a_scales");
    w = address(tw, at::kFloat8_e4m3fn, p, 0, "w");
    w_scales = address(tensor(o[3], "w_scales"), at::kFloat8_e8m0fnu, p, ((int64_t)n + HERO_FP8_BLOCK - 1) / HERO_FP8_BLOCK * pitch, "w_scales");
    bias = address(tb, at::kBFloat16, p, n, "bias");
    scratch = ts ? address(*ts, ts->scalar_type(), p, 0, "scratch") : nullptr;
    scratch_bytes = ts ? ts->nbytes() : 0;
  }
};

// (a, a_scales, w, w_scales, bias, c, act, scratch)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 8, [&] {
    const Operands o(a, a[6], a[7]);
    void* c = address(tensor(a[5], "c"), at::kBFloat16, o.p, (int64_t)o.m * o.n, "c");
    return unlocked([&] {
      return calls.linear(o.a, o.a_scales, o.w, o.w_scales, o.bias, c, o.m, o.n, o.k, o.act, o.scratch, o.scratch_bytes, o.p.stream);
    });
  });
}

// (a, a_scales, w, w_scales, bias, q, scales, act, scratch)
PyObject* linear_quantized(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 9, [&] {
    const Operands o(a, a[7], a[8]);
    void* q = address(tensor(a[5], "q"), at::kFloat8_e4m3fn, o.p, (int64_t)o.m * o.n, "q");
    void* scales = address(tensor(a[6], "scales"), at::kFloat8_e8m0fnu, o.p, (int64_t)o.m * HERO_FP8_SCALE_PITCH((int64_t)o.n), "scales");
    return unlocked([&] {
      return calls.linear_quantized(o.a, o.a_scales, o.w, o.w_scales, o.bias, q, scales, o.m, o.n, o.k, o.act, o.scratch, o.scratch_bytes, o.p.stream);
    });
  });
}

#define CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(init), CALL(quantize), CALL(rms), CALL(linear), CALL(linear_quantized), {nullptr, nullptr, 0, nullptr}};
#undef CALL
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fp8_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fp8_binding(void) { return PyModule_Create(&module); }
