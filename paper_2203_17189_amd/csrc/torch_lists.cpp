// Reads the tensors of a list of Python dicts into the entries of adamw_step_multi.  An optimizer's step has hundreds of
// tensors; asked for one property at a time from Python, each costs 2 us, more than its share of the kernel.
#include <torch/csrc/autograd/python_variable.h>
#include <cstring>
#include "../../include/t5mi.h"

namespace {

PyObject* names[8];  // of an entry's fields, made once
enum { PARAM, GRAD, M, V, M_SCALE, V_SCALE, COPY, DECAY };

// The tensor under a name: contiguous, of n elements (n < 0: any number) on CUDA device `index`; nullptr if it is not.
const at::Tensor* field(PyObject* entry, int name, int64_t n, int index) {
  PyObject* o = PyDict_GetItem(entry, names[name]);  // (borrowed)
  if (!o || o == Py_None || !THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.get_device() != index || !t.is_contiguous() || (n >= 0 && t.numel() != n)) return nullptr;
  return &t;
}
bool absent(PyObject* entry, int name) {
  PyObject* o = PyDict_GetItem(entry, names[name]);
  return !o || o == Py_None;
}

bool read_entry(PyObject* entry, int index, adamw_tensor* out) {
  std::memset(out, 0, sizeof(*out));
  const at::Tensor* p = field(entry, PARAM, -1, index);
  if (!p || p->scalar_type() != at::kFloat) return false;
  const int64_t n = p->numel();
  const at::Tensor *g = field(entry, GRAD, n, index), *m = field(entry, M, n, index), *v = field(entry, V, n, index);
  if (!g || !m || !v || m->scalar_type() != v->scalar_type()) return false;
  if (g->scalar_type() != at::kFloat && g->scalar_type() != at::kBFloat16) return false;
  out->param = static_cast<float*>(p->data_ptr());
  out->grad = g->data_ptr();
  out->m = m->data_ptr();
  out->v = v->data_ptr();
  out->n = n;
  out->grad_dtype = g->scalar_type() == at::kFloat ? T5_F32 : T5_BF16;
  if (m->scalar_type() == at::kFloat) {
    out->state_bits = 32;
  } else {
    if (m->scalar_type() != at::kFloat8_e4m3fn) return false;
    const at::Tensor *ms = field(entry, M_SCALE, (n + 127) / 128, index), *vs = field(entry, V_SCALE, (n + 127) / 128, index);
    if (!ms || !vs || ms->scalar_type() != at::kFloat8_e8m0fnu || vs->scalar_type() != at::kFloat8_e8m0fnu) return false;
    out->state_bits = 8;
    out->m_scale = static_cast<uint8_t*>(ms->data_ptr());
    out->v_scale = static_cast<uint8_t*>(vs->data_ptr());
  }
  if (!absent(entry, COPY)) {
    const at::Tensor* c = field(entry, COPY, n, index);
    if (!c || c->scalar_type() != at::kBFloat16) return false;
    out->bf16_copy_out = c->data_ptr();
  }
  PyObject* decay = PyDict_GetItem(entry, names[DECAY]);
  if (decay) {
    out->weight_decay = PyFloat_AsDouble(decay);
    if (PyErr_Occurred()) return false;
  }
  return true;
}

// adamw_entries(list, device index, writable buffer) -> the number of entries read before the first that is not in order
PyObject* adamw_entries(PyObject*, PyObject* args) {
  PyObject* list;
  int index;
  Py_buffer to;
  if (!PyArg_ParseTuple(args, "O!iw*", &PyList_Type, &list, &index, &to)) return nullptr;
  Py_ssize_t i = 0;
  const Py_ssize_t n = PyList_GET_SIZE(list);
  PyObject* result = nullptr;
  try {
    if (to.len == n * (Py_ssize_t)sizeof(adamw_tensor))
      for (; i < n; ++i) {
        PyObject* entry = PyList_GET_ITEM(list, i);
        if (!PyDict_Check(entry) || !read_entry(entry, index, static_cast<adamw_tensor*>(to.buf) + i)) break;
      }
    PyErr_Clear();
    result = PyLong_FromSsize_t(i);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  PyBuffer_Release(&to);
  return result;
}

PyMethodDef methods[] = {{"adamw_entries", adamw_entries, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_lists", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_lists() {
  const char* all[8] = {"param", "grad", "m", "v", "m_scale", "v_scale", "bf16_copy_out", "weight_decay"};
  for (int i = 0; i < 8; ++i) {
    names[i] = PyUnicode_InternFromString(all[i]);
    if (!names[i]) return nullptr;
  }
  return PyModule_Create(&module);
}
