// Python module _tensors: looks over the lists of tensors of an AdamW step and writes down where they are, for osscar_adamw.  A step over hundreds of small tensors takes tens of
// microseconds on the GPU; a property of a tensor read in Python takes 35 to 70 ns and a step needs about 20 of each parameter and its states.  Here a call over 192 parameters takes 12 us of the host,
// under the 28 that its kernels take, with the gradients of the step before or new ones: so every step can look again, and nothing is kept by address from one to the next.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <algorithm>
#include <string>
#include <vector>
#include "../../include/osscar.h"

namespace {

struct Refused { std::string why; };
struct Range { uintptr_t begin, end; Py_ssize_t k; };      // what a step writes
const at::ScalarType F32 = at::kFloat, BF16 = at::kBFloat16;

const at::Tensor& tensor(PyObject* x, const char* what, Py_ssize_t k) {
  if (!x || !THPVariable_Check(x)) throw Refused{std::string(what) + " " + std::to_string(k) + " is not a tensor"};
  const at::Tensor& t = THPVariable_Unpack(x);
  if (t.layout() != at::kStrided) throw Refused{std::string(what) + " " + std::to_string(k) + " is not a dense tensor"};
  return t;
}
// Shape, and strides where they say something.
bool alike(const at::Tensor& a, const at::Tensor& b) {
  if (!a.sizes().equals(b.sizes())) return false;
  for (int64_t d = 0; d < a.dim(); d++)
    if (a.size(d) > 1 && a.stride(d) != b.stride(d)) return false;
  return true;
}
std::string at_place(const char* what, Py_ssize_t k, const std::string& more) { return std::string(what) + " " + std::to_string(k) + more; }

PyObject* numbers(at::IntArrayRef v) {
  PyObject* t = PyTuple_New((Py_ssize_t)v.size());
  for (size_t k = 0; t && k < v.size(); k++) PyTuple_SET_ITEM(t, (Py_ssize_t)k, PyLong_FromLongLong(v[k]));
  return t;
}
// An AdamWState's `place`: shape and strides of the parameter that it goes with, for its values.
void set_place(PyObject* state, const at::Tensor& p) {
  static PyObject* const name = PyUnicode_InternFromString("place");
  PyObject* place = PyTuple_New(2);
  if (place) {
    PyTuple_SET_ITEM(place, 0, numbers(p.sizes()));
    PyTuple_SET_ITEM(place, 1, numbers(p.strides()));
  }
  if (!place || PyObject_SetAttr(state, name, place) != 0) PyErr_Clear();      // (a tuple of another kind has none)
  Py_XDECREF(place);
}

PyObject* item(PyObject* list, Py_ssize_t k) { return list == Py_None ? Py_None : PyList_GET_ITEM(list, k); }

void look(osscar_adamw_tensor* rows, PyObject* params, PyObject* grads, PyObject* masters, PyObject* states, int bits, int device) {
  const Py_ssize_t count = PyList_GET_SIZE(states);
  for (PyObject* list : {params, grads, masters})
    if (list != Py_None && (!PyList_Check(list) || PyList_GET_SIZE(list) != count)) throw Refused{"gradients, masters and states have one entry per parameter"};
  std::vector<Range> written;
  written.reserve(6 * count);
  auto write = [&](const at::Tensor& t, Py_ssize_t k) -> void* {
    if (t.get_device() != device) throw Refused{at_place("parameter", k, ", its master or its state is on " + t.device().str() + ", expected cuda:" + std::to_string(device))};
    void* p = t.data_ptr();
    if (t.numel() > 0) written.push_back(Range{(uintptr_t)p, (uintptr_t)p + t.nbytes(), k});
    return p;
  };
  for (Py_ssize_t k = 0; k < count; k++) {
    osscar_adamw_tensor& r = rows[k] = osscar_adamw_tensor{};
    const bool has = params != Py_None;
    const at::Tensor none;
    const at::Tensor& p = has ? tensor(item(params, k), "parameter", k) : none;
    if (has) {
      if (p.scalar_type() != F32 && p.scalar_type() != BF16) throw Refused{at_place("parameter", k, " is neither float32 nor bfloat16")};
      if (!p.is_contiguous() && !p.is_non_overlapping_and_dense()) throw Refused{at_place("the elements of parameter", k, " are not side by side")};
      r.n = p.numel();
      r.p = write(p, k);
      r.p_dtype = p.scalar_type() == F32 ? OSSCAR_F32 : OSSCAR_BF16;
      if (item(masters, k) != Py_None) {
        const at::Tensor& m = tensor(item(masters, k), "master", k);
        if (p.scalar_type() != BF16 || m.scalar_type() != F32 || !alike(m, p)) throw Refused{at_place("master", k, " must be float32, of the shape and layout of a bfloat16 parameter")};
        r.master = reinterpret_cast<float*>(write(m, k));
      }
      if (grads != Py_None) {
        const at::Tensor& g = tensor(item(grads, k), "gradient", k);
        if (g.scalar_type() != F32 && g.scalar_type() != BF16) throw Refused{at_place("gradient", k, " is neither float32 nor bfloat16")};
        if (!alike(g, p)) throw Refused{at_place("gradient", k, " has another shape or layout than its parameter")};
        if (g.get_device() != device) throw Refused{at_place("gradient", k, " is on " + g.device().str() + ", expected cuda:" + std::to_string(device))};
        r.g = g.data_ptr();
        r.g_dtype = g.scalar_type() == F32 ? OSSCAR_F32 : OSSCAR_BF16;
      }
    }
    PyObject* s = PyList_GET_ITEM(states, k);
    if (!PyTuple_Check(s) || PyTuple_GET_SIZE(s) != 4) throw Refused{at_place("state", k, " is not an AdamWState")};
    if (!has) r.n = tensor(PyTuple_GET_ITEM(s, 0), "state", k).numel();
    const int64_t blocks = (r.n + OSSCAR_ADAMW_BLOCK - 1) / OSSCAR_ADAMW_BLOCK;
    void* at[4] = {};
    for (int c = 0; c < (bits == 8 ? 4 : 2); c++) {
      PyObject* x = PyTuple_GET_ITEM(s, c);
      bool good = x != Py_None;
      if (good) {
        const at::Tensor& t = tensor(x, "state", k);
        const at::ScalarType d = t.scalar_type();
        good = t.numel() == (c < 2 ? r.n : blocks) && t.is_contiguous() && (bits == 32 || c >= 2 ? d == F32 : d == at::kByte || (c == 0 && d == at::kFloat8_e4m3fn));
        if (good) at[c] = write(t, k);
      }
      if (!good) throw Refused{at_place("state", k, " is not of " + std::to_string(bits) + " bits and parameter " + std::to_string(k) + "'s size, side by side")};
    }
    r.m = at[0];
    r.v = at[1];
    r.m_scale = reinterpret_cast<float*>(at[2]);
    r.v_scale = reinterpret_cast<float*>(at[3]);
  }
  std::sort(written.begin(), written.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  for (size_t k = 1; k < written.size(); k++)
    if (written[k].begin < written[k - 1].end)
      throw Refused{"parameters " + std::to_string(written[k - 1].k) + " and " + std::to_string(written[k].k) + " or their states share memory"};
  if (bits == 8 && params != Py_None)
    for (Py_ssize_t k = 0; k < count; k++)
      if (!PyTuple_CheckExact(PyList_GET_ITEM(states, k))) set_place(PyList_GET_ITEM(states, k), THPVariable_Unpack(PyList_GET_ITEM(params, k)));
}

// adamw_rows(address of the rows, params or None, grads or None, masters or None, states, bits, device): fills one osscar_adamw_tensor per state, and gives 8-bit states of parameters their place.  Returns None, or why it refuses.
PyObject* adamw_rows(PyObject*, PyObject* args) {
  unsigned long long rows;
  PyObject *params, *grads, *masters, *states;
  int bits, device;
  if (!PyArg_ParseTuple(args, "KOOOO!ii", &rows, &params, &grads, &masters, &PyList_Type, &states, &bits, &device)) return nullptr;
  try {
    look(reinterpret_cast<osscar_adamw_tensor*>(rows), params, grads, masters, states, bits, device);
  } catch (const Refused& e) {
    return PyUnicode_FromString(e.why.c_str());
  } catch (const std::exception& e) {      // (a tensor without memory, as of torch's tracers)
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"adamw_rows", adamw_rows, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
