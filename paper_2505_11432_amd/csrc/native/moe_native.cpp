// Python entry points of the C ABI: one function per call of include/moe.h, its arguments converted from Python objects by
// the types of the C declaration, the current stream added as the last one, the status returned as an int.
//
// A step of a small layer is a sequence of some twenty calls whose kernels run for a few microseconds each, so the caller's
// own time per call is what bounds it.  In Python and through ctypes every tensor costs three attribute or method calls
// (device, contiguity, pointer); here the same checks are made on the tensor object.  moe_route + moe_route_bwd of 4096
// tokens 20.4 -> 13.0 us, the twenty launches of a small fp32 training step (T = 256, d = 128, f = 256) 120 -> 87 us.
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <tuple>
#include <type_traits>
#include <utility>
#include <vector>

#include "../../../include/moe.h"

namespace {

bool refuse_tensor() {
  PyErr_SetString(PyExc_AssertionError, "tensors must be contiguous and on the GPU");
  return false;
}

// Device pointer of a tensor (None -> NULL).  A plain tensor or parameter is read directly; anything else (subclasses with
// their own behaviour, objects that quack like a tensor) is asked through Python.
bool to_pointer(PyObject* o, void** out) {
  if (o == Py_None) { *out = nullptr; return true; }
  if (THPVariable_CheckExact(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) return refuse_tensor();
    *out = t.data_ptr();
    return true;
  }
  PyObject* cuda = PyObject_GetAttrString(o, "is_cuda");
  if (!cuda) return false;
  const int is_cuda = PyObject_IsTrue(cuda);
  Py_DECREF(cuda);
  if (is_cuda < 0) return false;
  PyObject* cont = PyObject_CallMethod(o, "is_contiguous", nullptr);
  if (!cont) return false;
  const int is_contiguous = PyObject_IsTrue(cont);
  Py_DECREF(cont);
  if (is_contiguous < 0) return false;
  if (!is_cuda || !is_contiguous) return refuse_tensor();
  PyObject* ptr = PyObject_CallMethod(o, "data_ptr", nullptr);
  if (!ptr) return false;
  *out = PyLong_AsVoidPtr(ptr);
  Py_DECREF(ptr);
  return !PyErr_Occurred();
}

template <typename A> bool convert(PyObject* o, A* out) {
  if constexpr (std::is_pointer_v<A>) {
    void* p = nullptr;
    if (!to_pointer(o, &p)) return false;
    *out = static_cast<A>(p);
    return true;
  } else if constexpr (std::is_floating_point_v<A>) {
    const double v = PyFloat_AsDouble(o);
    *out = static_cast<A>(v);
    return !(v == -1.0 && PyErr_Occurred());
  } else {                                        // integers and the enums, wrapped to the C type as ctypes does
    *out = static_cast<A>(static_cast<long long>(PyLong_AsUnsignedLongLongMask(o)));
    return !PyErr_Occurred();
  }
}

template <auto FN> struct Bound;
template <typename... A, int (*FN)(A...)> struct Bound<FN> {
  static constexpr size_t kArgs = sizeof...(A) - 1;                 // the last parameter is the stream

  template <size_t... I> static bool parse(PyObject* const* args, std::tuple<A...>& v, std::index_sequence<I...>) {
    return (convert(args[I], &std::get<I>(v)) && ...);
  }

  static PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != static_cast<Py_ssize_t>(kArgs)) {
      PyErr_Format(PyExc_TypeError, "takes %zu arguments (%zd given)", kArgs, n);
      return nullptr;
    }
    try {
      std::tuple<A...> v{};
      if (!parse(args, v, std::make_index_sequence<kArgs>())) return nullptr;
      std::get<kArgs>(v) = static_cast<void*>(c10::hip::getCurrentHIPStream().stream());
      int rc;
      Py_BEGIN_ALLOW_THREADS
      rc = std::apply(FN, v);
      Py_END_ALLOW_THREADS
      return PyLong_FromLong(rc);
    } catch (const std::exception& e) {
      PyErr_SetString(PyExc_RuntimeError, e.what());
      return nullptr;
    }
  }
};

// tensor_list(tensors) -> (pointers, element counts, types) of a list of tensors as three bytes objects of int64, int64 and int32: what the tables of
// tensors are made from.  None gives (0, -1, -1), an empty tensor the pointer 0.  The checks are those of a call's arguments; the types are MOE_F32
// and MOE_BF16.  (Asked through Python, 300 tensors in five lists take 0.5 ms.)
PyObject* tensor_list(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 1) {
    PyErr_SetString(PyExc_TypeError, "takes a list of tensors");
    return nullptr;
  }
  PyObject* seq = PySequence_Fast(args[0], "takes a list of tensors");
  if (!seq) return nullptr;
  PyObject* result = nullptr;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject* bytes[3] = {PyBytes_FromStringAndSize(nullptr, n * 8), PyBytes_FromStringAndSize(nullptr, n * 8), PyBytes_FromStringAndSize(nullptr, n * 4)};
  bool ok = bytes[0] && bytes[1] && bytes[2];
  try {
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
      PyObject* o = PySequence_Fast_GET_ITEM(seq, i);
      int64_t pointer = 0, numel = -1;
      int32_t type = -1;
      if (o != Py_None) {
        if (!THPVariable_Check(o)) {
          PyErr_SetString(PyExc_TypeError, "takes a list of tensors");
          ok = false;
          break;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        const auto dt = t.scalar_type();
        if (!t.is_cuda() || !t.is_contiguous()) {
          ok = refuse_tensor();
          break;
        }
        if (dt != at::kFloat && dt != at::kBFloat16) {
          PyErr_SetString(PyExc_TypeError, "unsupported dtype: tensors are float32 or bfloat16");
          ok = false;
          break;
        }
        numel = t.numel();
        pointer = numel ? reinterpret_cast<int64_t>(t.data_ptr()) : 0;
        type = dt == at::kFloat ? MOE_F32 : MOE_BF16;
      }
      reinterpret_cast<int64_t*>(PyBytes_AS_STRING(bytes[0]))[i] = pointer;
      reinterpret_cast<int64_t*>(PyBytes_AS_STRING(bytes[1]))[i] = numel;
      reinterpret_cast<int32_t*>(PyBytes_AS_STRING(bytes[2]))[i] = type;
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    ok = false;
  }
  if (ok) result = PyTuple_Pack(3, bytes[0], bytes[1], bytes[2]);
  for (PyObject* b : bytes) Py_XDECREF(b);
  Py_DECREF(seq);
  return result;
}

// lists_apart(written, read, in_place) -> whether no byte of a list that is written belongs to another tensor of any of them: a launch over the lists writes
// and reads them in no order.  written, read: sequences of what tensor_list gives; in_place: a tensor of read[0] may be the one of written[0] at its place.
PyObject* lists_apart(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 3) {
    PyErr_SetString(PyExc_TypeError, "takes two sequences of lists and a truth value");
    return nullptr;
  }
  struct Range { uintptr_t begin, end; bool written; };
  struct List { const int64_t* pointers; const int64_t* numel; const int32_t* types; Py_ssize_t n; };
  const int in_place = PyObject_IsTrue(args[2]);
  if (in_place < 0) return nullptr;
  PyObject* seq[2] = {PySequence_Fast(args[0], "takes sequences of lists"), nullptr};
  if (seq[0]) seq[1] = PySequence_Fast(args[1], "takes sequences of lists");
  bool ok = seq[1] != nullptr, apart = true;
  try {
    std::vector<List> lists[2];
    for (int k = 0; ok && k < 2; ++k)
      for (Py_ssize_t i = 0; ok && i < PySequence_Fast_GET_SIZE(seq[k]); ++i) {
        PyObject* bytes[3];
        PyObject* list = PySequence_Fast_GET_ITEM(seq[k], i);
        if (!PyTuple_Check(list)) PyErr_SetString(PyExc_TypeError, "a list is what tensor_list gives");
        ok = PyTuple_Check(list) && PyArg_ParseTuple(list, "SSS", &bytes[0], &bytes[1], &bytes[2]);
        if (!ok) break;
        const Py_ssize_t n = PyBytes_GET_SIZE(bytes[2]) / 4;
        if (PyBytes_GET_SIZE(bytes[0]) != n * 8 || PyBytes_GET_SIZE(bytes[1]) != n * 8) {
          PyErr_SetString(PyExc_ValueError, "lists of one length");
          ok = false;
          break;
        }
        lists[k].push_back({reinterpret_cast<const int64_t*>(PyBytes_AS_STRING(bytes[0])), reinterpret_cast<const int64_t*>(PyBytes_AS_STRING(bytes[1])),
                            reinterpret_cast<const int32_t*>(PyBytes_AS_STRING(bytes[2])), n});
      }
    std::vector<Range> all;
    for (int k = 0; ok && k < 2; ++k)
      for (size_t j = 0; j < lists[k].size(); ++j) {
        const List& l = lists[k][j];
        for (Py_ssize_t i = 0; i < l.n; ++i) {
          if (l.numel[i] <= 0 || !l.pointers[i]) continue;
          if (k == 1 && j == 0 && in_place && !lists[0].empty() && i < lists[0][0].n && lists[0][0].pointers[i] == l.pointers[i]) continue;
          const uintptr_t begin = static_cast<uintptr_t>(l.pointers[i]);
          all.push_back({begin, begin + static_cast<uintptr_t>(l.numel[i]) * (l.types[i] == MOE_F32 ? 4 : 2), k == 0});
        }
      }
    std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t any = 0, written = 0;          // ends of what begins in front
    for (const Range& r : all) {
      apart = apart && r.begin >= (r.written ? any : written);
      any = std::max(any, r.end);
      if (r.written) written = std::max(written, r.end);
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    ok = false;
  }
  for (PyObject* s : seq) Py_XDECREF(s);
  return ok ? PyBool_FromLong(apart) : nullptr;
}

#define MOE_BOUND(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&Bound<&name>::call)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    MOE_BOUND(moe_router_fwd), MOE_BOUND(moe_router_bwd), MOE_BOUND(moe_route), MOE_BOUND(moe_route_noalloc),
    MOE_BOUND(moe_route_range), MOE_BOUND(moe_route_capacity), MOE_BOUND(moe_balance_loss), MOE_BOUND(moe_balance_loss_bwd),
    MOE_BOUND(moe_route_bwd), MOE_BOUND(moe_dispatch), MOE_BOUND(moe_combine), MOE_BOUND(moe_gate_grad),
    MOE_BOUND(moe_expert_ffn_fwd), MOE_BOUND(moe_expert_ffn_bwd), MOE_BOUND(moe_row_map), MOE_BOUND(moe_expert_ffn_fused_fwd),
    MOE_BOUND(moe_expert_ffn_fused_bwd), MOE_BOUND(moe_quant_fp8), MOE_BOUND(moe_dequant_fp8), MOE_BOUND(moe_quant_fp8_tgroup),
    MOE_BOUND(moe_transpose), MOE_BOUND(moe_vocab_score), MOE_BOUND(moe_vocab_loss), MOE_BOUND(moe_grad_clip), MOE_BOUND(moe_adamw),
    {"tensor_list", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&tensor_list)), METH_FASTCALL, nullptr},
    {"lists_apart", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&lists_apart)), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_moe_native", "Calls of the MoE library on torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__moe_native(void) { return PyModule_Create(&module); }
