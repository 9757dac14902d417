// bind.cpp -- the execute calls and the layer operators of the Python binding
// (ar.py) in native code.
//
// A call passes up to 128 rank tensors.  Checking each of them and reading
// its address in Python cost 0.14 us per rank and 4 us per call, most of the
// time of a small Allreduce; here it is 0.02 us per rank.  The checks are
// those of ar._ptr_table, made anew on every call (nothing is kept from one
// call to the next).  Whatever fails one, or is no plain torch tensor in a
// list or tuple -- raw addresses, subclasses, other sequences -- is answered
// with None, and the caller takes the Python path, which names the fault.
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <string>

#include "../../include/ar.h"

namespace {

using ExecuteFn = ar_status (*)(ar_plan*, void* const*, int64_t, int64_t, hipStream_t);
ExecuteFn g_execute[2] = {nullptr, nullptr};  // ar_execute_batched, ar_execute_noalloc; set once, at import

constexpr Py_ssize_t kMaxRanks = 128;
constexpr int64_t kMaxExtent = int64_t(1) << 46;

// Reads an int argument; false (no error set) if it is none or does not fit.
bool as_int(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow != 0 || (x == -1 && PyErr_Occurred())) {
    PyErr_Clear();
    return false;
  }
  *v = x;
  return true;
}

// Whether tensor t can serve as a rank buffer of `extent` elements of the
// plan's dtype (0 int32, 1 float32, < 0 any of 4 bytes) on GPU `device`.
bool rank_buffer(const at::Tensor& t, int64_t extent, int64_t dtype, int64_t device) {
  if (extent == 0) return true;
  if (!t.is_cuda() || t.get_device() != device) return false;
  const auto st = t.scalar_type();
  if (dtype == 0 ? st != at::kInt : dtype == 1 ? st != at::kFloat : t.element_size() != 4) return false;
  if (t.layout() != at::kStrided || !t.is_contiguous() || !t.has_storage()) return false;
  const int64_t have = int64_t(t.storage().nbytes() / 4) - t.storage_offset();
  return have >= extent;
}

// execute(handle, (P, n, dtype), buffers, batch, stride, device, stream, which)
// -> status, or None where the Python path has to look.
PyObject* execute(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 8 || !PyTuple_CheckExact(args[1]) || PyTuple_GET_SIZE(args[1]) != 3) Py_RETURN_NONE;
  int64_t handle, P, n, dtype = -1, batch, stride, device, stream, which;
  PyObject* dt = PyTuple_GET_ITEM(args[1], 2);
  if (!as_int(args[0], &handle) || !as_int(PyTuple_GET_ITEM(args[1], 0), &P) ||
      !as_int(PyTuple_GET_ITEM(args[1], 1), &n) || (dt != Py_None && !as_int(dt, &dtype)) ||
      !as_int(args[3], &batch) || !as_int(args[4], &stride) || !as_int(args[5], &device) ||
      !as_int(args[6], &stream) || !as_int(args[7], &which) || which < 0 || which > 1 || g_execute[which] == nullptr)
    Py_RETURN_NONE;
  PyObject* seq = args[2];
  const bool list = PyList_CheckExact(seq);
  if (!list && !PyTuple_CheckExact(seq)) Py_RETURN_NONE;
  if (P < 1 || P > kMaxRanks || Py_SIZE(seq) != P || n < 0 || batch < 1 || stride < 0) Py_RETURN_NONE;
  const int64_t step = batch == 1 && stride < n ? n : stride;
  if (n > kMaxExtent || (step > 0 && batch - 1 > (kMaxExtent - n) / step)) Py_RETURN_NONE;
  const int64_t extent = n > 0 ? (batch - 1) * step + n : 0;
  void* table[kMaxRanks];
  try {
    for (Py_ssize_t x = 0; x < P; ++x) {
      PyObject* o = list ? PyList_GET_ITEM(seq, x) : PyTuple_GET_ITEM(seq, x);
      if (!THPVariable_CheckExact(o)) Py_RETURN_NONE;
      const at::Tensor& t = THPVariable_Unpack(o);
      if (!rank_buffer(t, extent, dtype, device)) Py_RETURN_NONE;
      table[x] = t.data_ptr();
    }
  } catch (...) {  // a tensor without an address of its own: the Python path raises
    Py_RETURN_NONE;
  }
  ar_status st;
  Py_BEGIN_ALLOW_THREADS
  st = g_execute[which](reinterpret_cast<ar_plan*>(handle), table, batch, stride, reinterpret_cast<hipStream_t>(stream));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(long(st));
}

// bind(address of ar_execute_batched, address of ar_execute_noalloc): the
// functions of the library that ar.py loaded.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  int64_t a, b;
  if (nargs != 2 || !as_int(args[0], &a) || !as_int(args[1], &b)) {
    PyErr_SetString(PyExc_TypeError, "bind takes two addresses");
    return nullptr;
  }
  g_execute[0] = reinterpret_cast<ExecuteFn>(a);
  g_execute[1] = reinterpret_cast<ExecuteFn>(b);
  Py_RETURN_NONE;
}

// ---- layer operators ----
//
// The layer calls read their tensors, allocate what they return and the
// workspace, and call the library, all on the current device and stream (the
// Python side makes a given stream current).  A failed check is a Fault: its
// text is returned, and ar.py raises it; the library's own status is returned
// as a number.

ar_status (*g_linear_forward)(int64_t, int64_t, int64_t, const ar_matrix*, const ar_matrix*, const ar_matrix*,
                              const ar_matrix*, ar_activation, const ar_dropout*, const ar_matrix*, const ar_matrix*,
                              void*, int64_t, hipStream_t) = nullptr;
ar_status (*g_linear_forward_workspace)(int64_t, int64_t, int64_t, const ar_matrix*, const ar_matrix*,
                                        int64_t*) = nullptr;
ar_status (*g_linear_backward)(int64_t, int64_t, int64_t, const ar_matrix*, const ar_matrix*, const ar_matrix*,
                               const ar_matrix*, ar_activation, const ar_dropout*, const ar_matrix*, const ar_matrix*,
                               const ar_matrix*, int32_t, void*, int64_t, hipStream_t) = nullptr;
ar_status (*g_linear_backward_workspace)(int64_t, int64_t, int64_t, const ar_matrix*, const ar_matrix*,
                                         const ar_matrix*, const ar_matrix*, ar_activation, const ar_dropout*,
                                         const ar_matrix*, const ar_matrix*, const ar_matrix*, int64_t*) = nullptr;
ar_status (*g_dropout_forward)(int64_t, int64_t, const ar_matrix*, const ar_matrix*, const ar_dropout*,
                               const ar_matrix*, hipStream_t) = nullptr;

struct Fault {
  std::string text;
};

// What a call needs to know of where it runs.
struct Place {
  int64_t device, stream;
  hipStream_t hip() const { return reinterpret_cast<hipStream_t>(stream); }
};

int64_t number(PyObject* o, const char* name) {
  int64_t v;
  if (!as_int(o, &v)) throw Fault{std::string(name) + " must be an integer"};
  return v;
}

ar_dtype dtype_of(const at::Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kFloat: return AR_FLOAT32;
    case at::kHalf: return AR_FLOAT16;
    case at::kBFloat16: return AR_BFLOAT16;
    default: throw Fault{std::string(name) + " must be float32, float16 or bfloat16"};
  }
}
at::ScalarType scalar_of(int64_t code, at::ScalarType otherwise) {
  switch (code) {
    case -1: return otherwise;
    case AR_FLOAT32: return at::kFloat;
    case AR_FLOAT16: return at::kHalf;
    case AR_BFLOAT16: return at::kBFloat16;
    default: throw Fault{"results are float32, float16 or bfloat16"};
  }
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Fault{std::string(name) + " must be a tensor"};
  return THPVariable_Unpack(o);
}

// The same of a forward call, which torch would not know to have happened: a
// gradient that it is to record is not lost silently.
const at::Tensor& unrecorded(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (at::GradMode::is_enabled() && t.requires_grad())
    throw Fault{std::string(name) + " requires a gradient, which this call does not record: call it under torch.no_grad() (the "
                "_backward calls compute the gradient)"};
  return t;
}

// A given tensor was written: torch's check of what a backward pass still needs.
void written(PyObject* given, const at::Tensor& t) {
  if (THPVariable_Check(given) && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A tensor of `dims` dimensions (2, or 1: a vector) with consecutive elements
// in a row, on the call's device; rows and cols < 0 are not checked.
ar_matrix view(const at::Tensor& t, const char* name, int dims, int64_t rows, int64_t cols, const Place& at_) {
  const std::string n(name);
  if (t.layout() != at::kStrided) throw Fault{n + " must be a dense tensor"};
  if (t.is_neg()) throw Fault{n + " is a negated view, whose memory holds other values"};
  if (!t.is_cuda()) throw Fault{n + " is not on a GPU"};
  if (t.get_device() != at_.device)
    throw Fault{n + " is on cuda:" + std::to_string(t.get_device()) + ", the current device is cuda:" +
                std::to_string(at_.device)};
  if (t.dim() != dims) throw Fault{n + " must have " + std::to_string(dims) + " dimension" + (dims > 1 ? "s" : "")};
  ar_matrix m;
  m.dtype = dtype_of(t, name);
  const int64_t r = dims == 2 ? t.size(0) : 1, c = t.size(dims - 1);
  if ((rows >= 0 && r != rows) || (cols >= 0 && c != cols))
    throw Fault{n + " is " + std::to_string(r) + " x " + std::to_string(c) + ", the call needs " +
                (rows >= 0 ? std::to_string(rows) : std::string("any")) + " x " +
                (cols >= 0 ? std::to_string(cols) : std::string("any"))};
  if (c > 1 && t.stride(dims - 1) != 1) throw Fault{n + "'s rows must have consecutive elements"};
  if (r > 1 && t.stride(0) < c) throw Fault{n + "'s rows overlap"};
  m.ld = r > 1 ? t.stride(0) : c;
  m.data = t.numel() > 0 ? t.data_ptr() : nullptr;
  return m;
}

// None or (p, seed, site, row0).
const ar_dropout* dropout_of(PyObject* o, ar_dropout* d) {
  if (o == Py_None) return nullptr;
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) throw Fault{"dropout must be a Dropout"};
  d->p = PyFloat_AsDouble(PyTuple_GET_ITEM(o, 0));
  const bool bad_p = PyErr_Occurred() != nullptr;
  PyErr_Clear();
  if (bad_p) throw Fault{"dropout's p must be a number"};
  uint64_t v[3];
  for (int i = 0; i < 3; ++i) {
    PyObject* x = PyTuple_GET_ITEM(o, i + 1);
    v[i] = PyLong_Check(x) ? PyLong_AsUnsignedLongLong(x) : 0;
    const bool bad = !PyLong_Check(x) || PyErr_Occurred() != nullptr;
    PyErr_Clear();
    if (bad) throw Fault{"dropout's seed, site and row0 must be integers from 0 to 2^64 - 1"};
  }
  if (v[1] >> 32) throw Fault{"dropout's site must be below 2^32"};
  d->seed = v[0];
  d->site = uint32_t(v[1]);
  d->row0 = v[2];
  return d;
}

at::Tensor workspace(int64_t bytes, const at::Tensor& like) {
  return bytes > 0 ? at::empty({bytes}, like.options().dtype(at::kByte)) : at::Tensor();
}
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// Runs a call's body; what it throws becomes the text that ar.py raises.
template <typename F>
PyObject* answer(F&& body) {
  try {
    return body();
  } catch (const Fault& f) {
    return PyUnicode_FromString(f.text.c_str());
  } catch (const std::bad_alloc&) {
    return PyErr_NoMemory();
  } catch (...) {  // torch's own, of an allocation: as the error that torch raises for it
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

// linear_forward(x, w, bias, residual, out, preact, activation, out dtype, dropout, device, stream)
// -> y, (y, z) where preact is a tensor or True, a status, or a text.
PyObject* linear_forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return answer([&]() -> PyObject* {
    if (nargs != 11 || !g_linear_forward) throw Fault{"linear_forward takes 11 arguments"};
    const Place at_{number(args[9], "device"), number(args[10], "stream")};
    const at::Tensor& x = unrecorded(args[0], "x");
    const at::Tensor& w = unrecorded(args[1], "w");
    const ar_matrix mx = view(x, "x", 2, -1, -1, at_);
    const int64_t M = x.size(0), K = x.size(1);
    const ar_matrix mw = view(w, "w", 2, -1, K, at_);
    const int64_t N = w.size(0);
    ar_matrix mb, mr, mz;
    if (args[2] != Py_None) mb = view(unrecorded(args[2], "bias"), "bias", 1, 1, N, at_);
    if (args[3] != Py_None) mr = view(unrecorded(args[3], "residual"), "residual", 2, M, N, at_);
    const int64_t act = number(args[6], "activation"), code = number(args[7], "out dtype");
    ar_dropout d;
    const ar_dropout* drop = dropout_of(args[8], &d);
    at::Tensor y, z;
    if (args[4] != Py_None) y = unrecorded(args[4], "out");
    else y = at::empty({M, N}, x.options().dtype(scalar_of(code, x.scalar_type())));
    if (args[5] == Py_True) z = at::empty({M, N}, x.options());
    else if (args[5] != Py_None && args[5] != Py_False) z = unrecorded(args[5], "preact");
    const ar_matrix my = view(y, "out", 2, M, N, at_);
    if (z.defined()) mz = view(z, "preact", 2, M, N, at_);
    int64_t bytes = 0;
    ar_status st = g_linear_forward_workspace(M, N, K, &mx, &mw, &bytes);
    if (st == AR_OK) {
      const at::Tensor ws = workspace(bytes, x);
      Py_BEGIN_ALLOW_THREADS
      st = g_linear_forward(M, N, K, &mx, &mw, args[2] != Py_None ? &mb : nullptr, args[3] != Py_None ? &mr : nullptr,
                            ar_activation(act), drop, &my, z.defined() ? &mz : nullptr, address(ws), bytes, at_.hip());
      Py_END_ALLOW_THREADS
    }
    if (st != AR_OK) return PyLong_FromLong(long(st));
    written(args[4], y);
    if (z.defined()) written(args[5], z);
    PyObject* py = THPVariable_Wrap(y);
    if (!z.defined() || !py) return py;
    PyObject* pz = THPVariable_Wrap(z);
    PyObject* both = pz ? PyTuple_Pack(2, py, pz) : nullptr;
    Py_DECREF(py);
    Py_XDECREF(pz);
    return both;
  });
}

// None and False: not wanted; True: a new tensor; else the tensor given.
at::Tensor wanted(PyObject* o, const char* name, at::IntArrayRef shape, const at::TensorOptions& options) {
  if (o == Py_None || o == Py_False) return at::Tensor();
  if (o == Py_True) return at::empty(shape, options);
  return tensor(o, name);
}

// linear_backward(dy, x, w, preact, activation, dropout, dx, dw, db, dx dtype, dw dtype, accumulate, device, stream)
// -> (dx, dw, db) with None for what was not wanted, a status, or a text.
PyObject* linear_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return answer([&]() -> PyObject* {
    if (nargs != 14 || !g_linear_backward) throw Fault{"linear_backward takes 14 arguments"};
    const Place at_{number(args[12], "device"), number(args[13], "stream")};
    const at::Tensor& dy = tensor(args[0], "dy");
    const at::Tensor& x = tensor(args[1], "x");
    const at::Tensor& w = tensor(args[2], "w");
    const ar_matrix mdy = view(dy, "dy", 2, -1, -1, at_);
    const int64_t M = dy.size(0), N = dy.size(1);
    const ar_matrix mx = view(x, "x", 2, M, -1, at_);
    const int64_t K = x.size(1);
    const ar_matrix mw = view(w, "w", 2, N, K, at_);
    ar_matrix mz, mdx, mdw, mdb;
    const bool has_z = args[3] != Py_None;
    if (has_z) mz = view(tensor(args[3], "preact"), "preact", 2, M, N, at_);
    const int64_t act = number(args[4], "activation");
    ar_dropout d;
    const ar_dropout* drop = dropout_of(args[5], &d);
    const auto same = x.options();
    const auto other = same.dtype(scalar_of(number(args[10], "dw dtype"), x.scalar_type()));
    const bool accumulate = args[11] == Py_True;
    if (accumulate && (args[7] == Py_True || args[8] == Py_True))
      throw Fault{"accumulate adds to the dw and db that are given: they must be tensors"};
    const at::Tensor dx =
        wanted(args[6], "dx", {M, K}, same.dtype(scalar_of(number(args[9], "dx dtype"), x.scalar_type())));
    const at::Tensor dw = wanted(args[7], "dw", {N, K}, other), db = wanted(args[8], "db", {N}, other);
    if (dx.defined()) mdx = view(dx, "dx", 2, M, K, at_);
    if (dw.defined()) mdw = view(dw, "dw", 2, N, K, at_);
    if (db.defined()) mdb = view(db, "db", 1, 1, N, at_);
    const ar_matrix* pz = has_z ? &mz : nullptr;
    const ar_matrix* pdx = dx.defined() ? &mdx : nullptr;
    const ar_matrix* pdw = dw.defined() ? &mdw : nullptr;
    const ar_matrix* pdb = db.defined() ? &mdb : nullptr;
    int64_t bytes = 0;
    ar_status st = g_linear_backward_workspace(M, N, K, &mdy, &mx, &mw, pz, ar_activation(act), drop, pdx, pdw, pdb,
                                               &bytes);
    if (st == AR_OK) {
      const at::Tensor ws = workspace(bytes, dy);
      Py_BEGIN_ALLOW_THREADS
      st = g_linear_backward(M, N, K, &mdy, &mx, &mw, pz, ar_activation(act), drop, pdx, pdw, pdb, accumulate,
                             address(ws), bytes, at_.hip());
      Py_END_ALLOW_THREADS
    }
    if (st != AR_OK) return PyLong_FromLong(long(st));
    PyObject* got = PyTuple_New(3);
    const at::Tensor* const parts[] = {&dx, &dw, &db};
    for (int i = 0; got && i < 3; ++i) {
      PyObject* o = Py_None;
      if (parts[i]->defined()) {
        written(args[6 + i], *parts[i]);
        o = THPVariable_Wrap(*parts[i]);
      } else {
        Py_INCREF(o);
      }
      if (!o) {
        Py_DECREF(got);
        return nullptr;
      }
      PyTuple_SET_ITEM(got, i, o);
    }
    return got;
  });
}

// dropout(x, residual, out, out dtype, dropout, backward, device, stream) -> y, a status, or a text.
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return answer([&]() -> PyObject* {
    if (nargs != 8 || !g_dropout_forward) throw Fault{"dropout takes 8 arguments"};
    const Place at_{number(args[6], "device"), number(args[7], "stream")};
    auto* const operand = args[5] == Py_True ? tensor : unrecorded;
    const at::Tensor& x = operand(args[0], "x");
    const ar_matrix mx = view(x, "x", 2, -1, -1, at_);
    const int64_t rows = x.size(0), cols = x.size(1);
    ar_matrix mr;
    if (args[1] != Py_None) mr = view(operand(args[1], "residual"), "residual", 2, rows, cols, at_);
    const int64_t code = number(args[3], "out dtype");
    at::Tensor y;
    if (args[2] != Py_None) y = operand(args[2], "out");
    else y = at::empty({rows, cols}, x.options().dtype(scalar_of(code, x.scalar_type())));
    const ar_matrix my = view(y, "out", 2, rows, cols, at_);
    ar_dropout d;
    const ar_dropout* drop = dropout_of(args[4], &d);
    ar_status st;
    Py_BEGIN_ALLOW_THREADS
    st = g_dropout_forward(rows, cols, &mx, args[1] != Py_None ? &mr : nullptr, drop, &my, at_.hip());
    Py_END_ALLOW_THREADS
    if (st != AR_OK) return PyLong_FromLong(long(st));
    written(args[2], y);
    return THPVariable_Wrap(y);
  });
}

// bind_layers(addresses of the five functions above, in their order)
PyObject* bind_layers(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  int64_t a[5];
  for (int i = 0; i < 5; ++i) {
    if (nargs != 5 || !as_int(args[i], &a[i])) {
      PyErr_SetString(PyExc_TypeError, "bind_layers takes five addresses");
      return nullptr;
    }
  }
  g_linear_forward = reinterpret_cast<decltype(g_linear_forward)>(a[0]);
  g_linear_forward_workspace = reinterpret_cast<decltype(g_linear_forward_workspace)>(a[1]);
  g_linear_backward = reinterpret_cast<decltype(g_linear_backward)>(a[2]);
  g_linear_backward_workspace = reinterpret_cast<decltype(g_linear_backward_workspace)>(a[3]);
  g_dropout_forward = reinterpret_cast<decltype(g_dropout_forward)>(a[4]);
  Py_RETURN_NONE;
}

template <typename F>
PyCFunction fastcall(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)); }

PyMethodDef kMethods[] = {
    {"linear_forward", fastcall(linear_forward), METH_FASTCALL, nullptr},
    {"linear_backward", fastcall(linear_backward), METH_FASTCALL, nullptr},
    {"dropout", fastcall(dropout), METH_FASTCALL, nullptr},
    {"bind_layers", fastcall(bind_layers), METH_FASTCALL, nullptr},
    {"execute", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(execute)), METH_FASTCALL, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(bind)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_arbind", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__arbind(void) { return PyModule_Create(&kModule); }
