// What a call from Python costs besides its launch: the arguments of a C entry point taken from Python objects, tensors as their
// addresses on the current stream.  Every conversion goes by the entry point's own parameter types (capmoe.h).  With ctypes the
// same takes about 3 us of a call, as much as a launch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <ATen/Functions.h>
#include <ATen/cuda/EmptyTensor.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <string_view>
#include <unordered_map>
#include <utility>
#include <vector>

#include "capmoe.h"

namespace {

struct Slot { int64_t i; double f; };            // an argument as an integer or address, and as a number
constexpr int MAX_ARGS = 32;

enum Kind : uint8_t { ADDRESS, WIDE, INT, REAL };            // pointer, 64-bit integer, int, number
template <class T>
constexpr Kind kind_of() {
  return std::is_pointer_v<T> ? ADDRESS : std::is_floating_point_v<T> ? REAL : sizeof(T) == 8 ? WIDE : INT;
}
template <class T>
T as(const Slot& s) {
  if constexpr (std::is_pointer_v<T>) return reinterpret_cast<T>(s.i);
  else if constexpr (std::is_floating_point_v<T>) return static_cast<T>(s.f);
  else return static_cast<T>(s.i);
}
template <auto Fn> struct Entry;
template <class... P, int (*Fn)(P...)>
struct Entry<Fn> {
  static constexpr int params = sizeof...(P);
  static constexpr Kind kinds[] = {kind_of<P>()...};
  template <size_t... I>
  static int call(const Slot* s, std::index_sequence<I...>) { return Fn(as<P>(s[I])...); }
  static int run(const Slot* s) { return call(s, std::make_index_sequence<sizeof...(P)>{}); }
};
struct Call { int (*run)(const Slot*); int params; const Kind* kinds; };
template <auto Fn> constexpr Call entry() { return {&Entry<Fn>::run, Entry<Fn>::params, Entry<Fn>::kinds}; }

const std::unordered_map<std::string_view, Call>& entries() {
  static const std::unordered_map<std::string_view, Call> table = {
#define CAPMOE_ENTRY(name) {#name, entry<&name>()}
      CAPMOE_ENTRY(capmoe_grouped_mm), CAPMOE_ENTRY(capmoe_grouped_mm_dx), CAPMOE_ENTRY(capmoe_grouped_mm_dw),
      CAPMOE_ENTRY(capmoe_grouped_ffn_backward), CAPMOE_ENTRY(capmoe_quantize_rows), CAPMOE_ENTRY(capmoe_quantize_weights),
      CAPMOE_ENTRY(capmoe_grouped_mm_fp8), CAPMOE_ENTRY(capmoe_grouped_ffn_fp8), CAPMOE_ENTRY(capmoe_grouped_ffn_fp8_codes),
      CAPMOE_ENTRY(capmoe_rms_norm), CAPMOE_ENTRY(capmoe_rms_norm_backward), CAPMOE_ENTRY(capmoe_permute_fp8),
      CAPMOE_ENTRY(capmoe_combine_backward), CAPMOE_ENTRY(capmoe_permute_backward), CAPMOE_ENTRY(capmoe_route_backward),
#undef CAPMOE_ENTRY
  };
  return table;
}

// run(name, like, *args): the entry point's status, the current stream as its last argument, CAPMOE_EUNSUPPORTED for a size that
// does not fit the int it is passed as; None where a tensor may not be passed (it is not on like's device or not contiguous, or
// like's device is not the current one), which the caller turns into its message.  Other types than the entry point's are a
// TypeError.
PyObject* run(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n < 2 || !PyUnicode_Check(args[0]) || !THPVariable_Check(args[1])) {
    PyErr_SetString(PyExc_TypeError, "run(name, like, *args)");
    return nullptr;
  }
  Py_ssize_t length = 0;
  const char* name = PyUnicode_AsUTF8AndSize(args[0], &length);
  if (!name) return nullptr;
  const auto it = entries().find(std::string_view(name, (size_t)length));
  if (it == entries().end() || n - 1 != it->second.params || n - 1 > MAX_ARGS) {
    PyErr_Format(PyExc_TypeError, "%s: no such entry point, or %zd arguments are not what it takes", name, n - 2);
    return nullptr;
  }
  const at::Tensor& like = THPVariable_Unpack(args[1]);
  if (!like.is_cuda()) Py_RETURN_NONE;
  const auto here = like.get_device();
  Slot slots[MAX_ARGS];
  int k = 0;
  for (Py_ssize_t i = 2; i < n; ++i, ++k) {
    PyObject* o = args[i];
    Slot& s = slots[k];
    const Kind kind = it->second.kinds[k];
    if (kind == REAL) {
      const double v = PyFloat_AsDouble(o);
      if (v == -1.0 && PyErr_Occurred()) return nullptr;
      s = {0, v};
    } else if (o == Py_None && kind == ADDRESS) {
      s = {0, 0.0};
    } else if (kind == ADDRESS && THPVariable_Check(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      if (!t.is_cuda() || t.get_device() != here || !t.is_contiguous()) Py_RETURN_NONE;
      s = {reinterpret_cast<int64_t>(t.data_ptr()), 0.0};
    } else {
      if (!PyLong_Check(o) && (!PyIndex_Check(o) || THPVariable_Check(o))) {
        PyErr_Format(PyExc_TypeError, "%s: argument %d is a %s", name, k, Py_TYPE(o)->tp_name);
        return nullptr;
      }
      PyObject* index = PyLong_Check(o) ? Py_NewRef(o) : PyNumber_Index(o);      // (a NumPy integer)
      if (!index) return nullptr;
      const long long v = PyLong_AsLongLong(index);
      Py_DECREF(index);
      if (v == -1 && PyErr_Occurred()) return nullptr;
      if (kind == INT && v != (int)v) return PyLong_FromLong(CAPMOE_EUNSUPPORTED);
      s = {(int64_t)v, 0.0};
    }
  }
  if (c10::cuda::current_device() != here) Py_RETURN_NONE;
  slots[k] = {reinterpret_cast<int64_t>(c10::cuda::getCurrentCUDAStream(here).stream()), 0.0};
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = it->second.run(slots);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// new(like, dtype, *sizes): an uninitialised tensor on like's device, of like's type where dtype is None, and its sizes where there
// are none: torch.empty without the parsing of its arguments, half of its time.
PyObject* make(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS                               // torch's exceptions as their Python types, out of memory among them
  if (n < 2 || n > 6 || !THPVariable_Check(args[0]) || !(args[1] == Py_None || THPDtype_Check(args[1]))) {
    PyErr_SetString(PyExc_TypeError, "new(like, dtype, *sizes)");
    return nullptr;
  }
  const at::Tensor& like = THPVariable_Unpack(args[0]);
  int64_t sizes[4];
  for (Py_ssize_t i = 2; i < n; ++i) {
    sizes[i - 2] = PyLong_AsLongLong(args[i]);
    if (sizes[i - 2] == -1 && PyErr_Occurred()) return nullptr;
  }
  const auto shape = n == 2 ? like.sizes() : at::IntArrayRef(sizes, (size_t)(n - 2));
  const auto dtype = args[1] == Py_None ? like.scalar_type() : reinterpret_cast<THPDtype*>(args[1])->scalar_type;
  if (!like.is_cuda()) return THPVariable_Wrap(at::empty(shape, at::TensorOptions().device(like.device()).dtype(dtype)));   // (run refuses it)
  return THPVariable_Wrap(at::detail::empty_cuda(shape, dtype, like.device(), c10::nullopt));
  END_HANDLE_TH_ERRORS
}

// What match() knows of an argument: its type (T: float32 or bfloat16, one type for all T; f float32, i int32, q and s the 8-bit codes
// and their scales), whether it may be None, and its sizes, letters that mean the same number wherever they stand (B: blocks of 128 of d).
struct Shape {
  char type;
  bool optional;
  int dims;
  char size[4];
};
struct Pattern {
  std::vector<Shape> args;
  std::string letters;                           // in the order of their first place
};
// "T[N,d] T?[d]": a shape per argument
Pattern parse(const char* p) {
  Pattern out;
  while (*p) {
    Shape a = {*p++, false, 0, {}};
    if (*p == '?') { a.optional = true; ++p; }
    for (++p; *p && *p != ']'; ++p)
      if (*p != ',' && a.dims < 4) {
        a.size[a.dims++] = *p;
        if (*p != 'B' && out.letters.find(*p) == std::string::npos) out.letters += *p;
      }
    if (*p) ++p;
    if (*p) ++p;
    out.args.push_back(a);
  }
  return out;
}
bool is_type(char type, at::ScalarType t, at::ScalarType& bound) {
  switch (type) {
    case 'f': return t == at::kFloat;
    case 'i': return t == at::kInt;
    case 'q': return t == at::kFloat8_e4m3fn;
    case 's': return t == at::kFloat8_e8m0fnu;
    default:
      if (bound == at::ScalarType::Undefined && (t == at::kFloat || t == at::kBFloat16)) bound = t;
      return t == bound;
  }
}

// match(pattern, *tensors): (dtype code of the T's, or -1, and the letters' numbers), None where an argument does not fit; the caller
// then finds out why.  One call for what takes 2 to 4 us of attribute look-ups.
PyObject* match(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  static std::unordered_map<std::string, Pattern> known;
  Py_ssize_t length = 0;
  const char* text = n > 0 && PyUnicode_Check(args[0]) ? PyUnicode_AsUTF8AndSize(args[0], &length) : nullptr;
  if (!text) {
    PyErr_SetString(PyExc_TypeError, "match(pattern, *tensors)");
    return nullptr;
  }
  std::string key(text, (size_t)length);
  auto it = known.find(key);
  if (it == known.end()) it = known.emplace(key, parse(text)).first;
  const Pattern& pattern = it->second;
  if ((size_t)(n - 1) != pattern.args.size()) {
    PyErr_Format(PyExc_TypeError, "match: %zd tensors expected", (Py_ssize_t)pattern.args.size());
    return nullptr;
  }
  int64_t size[128];
  for (char c : pattern.letters) size[(int)c] = -1;
  at::ScalarType bound = at::ScalarType::Undefined;
  for (Py_ssize_t i = 1; i < n; ++i) {
    const Shape& a = pattern.args[(size_t)i - 1];
    if (args[i] == Py_None && a.optional) continue;
    if (!THPVariable_Check(args[i])) Py_RETURN_NONE;
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (t.dim() != a.dims || !is_type(a.type, t.scalar_type(), bound)) Py_RETURN_NONE;
    for (int j = 0; j < a.dims; ++j) {
      const int64_t have = t.size(j);
      const char c = a.size[j];
      if (c == 'B') {
        if (have != (size['d'] + 127) / 128) Py_RETURN_NONE;
      } else {
        int64_t& want = size[(int)c];
        if (want < 0) want = have;
        if (want != have) Py_RETURN_NONE;
      }
    }
  }
  PyObject* out = PyTuple_New(1 + (Py_ssize_t)pattern.letters.size());
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, PyLong_FromLong(bound == at::kFloat ? CAPMOE_F32 : bound == at::kBFloat16 ? CAPMOE_BF16 : -1));
  for (size_t i = 0; i < pattern.letters.size(); ++i) PyTuple_SET_ITEM(out, (Py_ssize_t)i + 1, PyLong_FromLongLong(size[(int)pattern.letters[i]]));
  return out;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"match", (PyCFunction)(void (*)(void))match, METH_FASTCALL, "Types and sizes of arguments."},
                         {"run", (PyCFunction)(void (*)(void))run, METH_FASTCALL, "Calls an entry point of libcapmoe.so."},
                         {"new", (PyCFunction)(void (*)(void))make, METH_FASTCALL, "An uninitialised tensor."}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind() { return PyModule_Create(&module); }
