// Arguments of the 8-bit operators, read from torch's tensors by native code: the list of adamw_step_multi, whose tensors cost
// 2 us each when asked for one property at a time from Python, more than their share of the kernel; and the ordinary calls of
// t5_quantize_fp8 and t5_gemm_fp8, of which the checks were half (9.3 us and 8.1, of a launch of 3.5).  Whatever is not in
// order is left to binding.py, which says what it is.
#include <ATen/Functions.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <climits>
#include <cstdint>
#include <cstring>
#include "../../include/t5mi.h"

namespace {

PyObject* names[8];  // of an entry's fields, made once
enum { PARAM, GRAD, M, V, M_SCALE, V_SCALE, COPY, DECAY };

// Whether a tensor is rows of memory on CUDA device `index`: sparse and nested ones have no strides, and say so by a C++ exception.
bool plain_on(const at::Tensor& t, int index) {
  return t.defined() && t.is_cuda() && t.get_device() == index && t.layout() == at::kStrided && !t.is_nested();
}

// The tensor under a name: contiguous, of n elements (n < 0: any number) on CUDA device `index`; nullptr if it is not.
const at::Tensor* field(PyObject* entry, int name, int64_t n, int index) {
  PyObject* o = PyDict_GetItem(entry, names[name]);  // (borrowed)
  if (!o || o == Py_None || !THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!plain_on(t, index) || !t.is_contiguous() || (n >= 0 && t.numel() != n)) return nullptr;
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
  struct Release {  // however the function is left
    Py_buffer* b;
    ~Release() { PyBuffer_Release(b); }
  } release{&to};
  HANDLE_TH_ERRORS
  Py_ssize_t i = 0;
  const Py_ssize_t n = PyList_GET_SIZE(list);
  if (to.len == n * (Py_ssize_t)sizeof(adamw_tensor))
    for (; i < n; ++i) {
      PyObject* entry = PyList_GET_ITEM(list, i);
      if (!PyDict_Check(entry) || !read_entry(entry, index, static_cast<adamw_tensor*>(to.buf) + i)) break;
    }
  PyErr_Clear();
  return PyLong_FromSsize_t(i);
  END_HANDLE_TH_ERRORS
}

typedef int (*QuantizeFn)(const t5_quantize_cfg*, const void*, void*, uint8_t*, void*, uint8_t*, void*);
typedef int (*GemmFn)(const t5_gemm_fp8_cfg*, const void*, const uint8_t*, const void*, const uint8_t*, void*, void*, size_t, void*);
typedef size_t (*GemmBytesFn)(const t5_gemm_fp8_cfg*);

const at::Tensor* tensor_on(PyObject* o, int index) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return plain_on(t, index) ? &t : nullptr;
}

struct Rows { int64_t n, cols, ld; };
// Rows of a matrix whose elements are contiguous and that do not overlap.
bool rows_of(const at::Tensor& t, Rows* r) {
  if (t.dim() != 2) return false;
  r->n = t.size(0);
  r->cols = t.size(1);
  r->ld = r->n > 1 && !t.is_contiguous() ? t.stride(0) : r->cols;
  return (r->cols <= 1 || t.stride(1) == 1) && r->ld >= r->cols;
}
// The same of bytes that are read in whole pieces of `step`: the last row's has to be in memory; one row is of any length.
bool pieces_of(const at::Tensor& t, int step, Rows* r) {
  if (!rows_of(t, r)) return false;
  if (r->cols % step == 0) return true;
  const int64_t whole = (r->cols + step - 1) / step * step;
  if (r->n > 0 && (int64_t)t.storage().nbytes() - t.storage_offset() < (r->n - 1) * r->ld + whole) return false;
  if (r->n <= 1) r->ld = whole;
  return true;
}
bool fp8_code(at::ScalarType t, int32_t* code) {
  *code = t == at::kFloat8_e5m2 ? T5_E5M2 : T5_E4M3;
  return t == at::kFloat8_e4m3fn || t == at::kFloat8_e5m2;
}
struct Operand { Rows q, s; int32_t type, block_rows; };
bool operand_of(const at::Tensor& q, const at::Tensor& s, Operand* o) {
  if (!fp8_code(q.scalar_type(), &o->type) || s.scalar_type() != at::kFloat8_e8m0fnu || !pieces_of(q, 16, &o->q) || !pieces_of(s, 4, &o->s)) return false;
  const int64_t squares = (o->q.n + 127) / 128;
  o->block_rows = o->s.n == o->q.n ? 1 : 128;
  return o->s.cols == (o->q.cols + 127) / 128 && (o->s.n == o->q.n || o->s.n == squares);
}
// A flag; an object that is neither true nor false (a tensor of several elements, say) leaves its error in *wrong.
bool flag(PyObject* o, bool* wrong) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) {
    PyErr_Clear();
    *wrong = true;
  }
  return v == 1;
}
bool fits32(int64_t v) { return v <= INT32_MAX; }

// quantize_fp8(entry point, x, e5m2, block_rows, rows, transposed, stream, device) -> (q, scale, qt, scale_t), a status, or None
PyObject* quantize_fp8(PyObject*, PyObject* const* args, Py_ssize_t count) {
  HANDLE_TH_ERRORS  // (around everything that asks torch for something: an exception that left a C function would end the process)
  if (count != 8) Py_RETURN_NONE;
  const int index = (int)PyLong_AsLong(args[7]);
  const at::Tensor* x = tensor_on(args[1], index);
  Rows r;
  if (!x || !rows_of(*x, &r) || (x->scalar_type() != at::kFloat && x->scalar_type() != at::kBFloat16)) Py_RETURN_NONE;
  const long e5m2 = PyLong_AsLong(args[2]), block_rows = PyLong_AsLong(args[3]);
  if (PyErr_Occurred() || (block_rows != 1 && block_rows != 128)) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  bool wrong = false;
  const bool straight = flag(args[4], &wrong), turned = flag(args[5], &wrong);
  if (wrong) Py_RETURN_NONE;
  const at::ScalarType type = e5m2 ? at::kFloat8_e5m2 : at::kFloat8_e4m3fn;
  at::Tensor out[4];
  auto make = [&](int64_t n, int64_t cols, at::Tensor* q, at::Tensor* s) {
    const int64_t blocks = (cols + 127) / 128, ld = (cols + 15) / 16 * 16, lds = (blocks + 3) / 4 * 4;
    *q = at::empty({n, ld}, x->options().dtype(type));
    *s = at::empty({(n + block_rows - 1) / block_rows, lds}, x->options().dtype(at::kFloat8_e8m0fnu));
  };
  if (straight) make(r.n, r.cols, &out[0], &out[1]);
  if (turned) make(r.cols, r.n, &out[2], &out[3]);
  const t5_quantize_cfg cfg = {r.n, r.cols, r.ld, x->scalar_type() == at::kFloat ? T5_F32 : T5_BF16, e5m2 ? T5_E5M2 : T5_E4M3, (int32_t)block_rows};
  const int rc = ((QuantizeFn)PyLong_AsVoidPtr(args[0]))(&cfg, x->data_ptr(), straight ? out[0].data_ptr() : nullptr, straight ? (uint8_t*)out[1].data_ptr() : nullptr,
                                                         turned ? out[2].data_ptr() : nullptr, turned ? (uint8_t*)out[3].data_ptr() : nullptr, PyLong_AsVoidPtr(args[6]));
  if (rc != T5_OK) return PyLong_FromLong(rc);
  PyObject* result = PyTuple_New(4);
  if (!result) return nullptr;
  const int64_t cols[4] = {r.cols, (r.cols + 127) / 128, r.n, (r.n + 127) / 128};
  for (int i = 0; i < 4; ++i) {
    PyObject* o = Py_None;
    if (out[i].defined()) o = THPVariable_Wrap(out[i].size(1) == cols[i] ? out[i] : out[i].narrow(1, 0, cols[i]));
    else Py_INCREF(o);
    PyTuple_SET_ITEM(result, i, o);
  }
  return result;
  END_HANDLE_TH_ERRORS
}

// gemm_fp8(entry point, its size query, a, a_scale, b, b_scale, out or None, float32, accumulate, stream, device) -> out, a status, or None
PyObject* gemm_fp8(PyObject*, PyObject* const* args, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  if (count != 11) Py_RETURN_NONE;
  const int index = (int)PyLong_AsLong(args[10]);
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i)
    if (!(t[i] = tensor_on(args[2 + i], index))) Py_RETURN_NONE;
  Operand a, b;
  if (!operand_of(*t[0], *t[1], &a) || !operand_of(*t[2], *t[3], &b) || a.q.cols != b.q.cols || !fits32(a.q.n) || !fits32(b.q.n) || !fits32(a.q.cols))
    Py_RETURN_NONE;
  bool wrong = false, f32 = flag(args[7], &wrong);
  const bool add = flag(args[8], &wrong);
  if (wrong) Py_RETURN_NONE;
  at::Tensor out;
  Rows c = {a.q.n, b.q.n, b.q.n};
  if (args[6] == Py_None) {
    if (add) Py_RETURN_NONE;
    out = at::empty({a.q.n, b.q.n}, t[0]->options().dtype(f32 ? at::kFloat : at::kBFloat16));
  } else {
    const at::Tensor* given = tensor_on(args[6], index);
    if (!given || !rows_of(*given, &c) || c.n != a.q.n || c.cols != b.q.n || (given->scalar_type() != at::kFloat && given->scalar_type() != at::kBFloat16))
      Py_RETURN_NONE;
    out = *given;
    f32 = out.scalar_type() == at::kFloat;
  }
  const t5_gemm_fp8_cfg cfg = {(int32_t)a.q.n, (int32_t)b.q.n, (int32_t)a.q.cols, a.q.ld, b.q.ld, c.ld, a.s.ld, b.s.ld, a.type, b.type,
                               a.block_rows, b.block_rows, f32 ? T5_F32 : T5_BF16, add ? 1 : 0};
  const size_t bytes = ((GemmBytesFn)PyLong_AsVoidPtr(args[1]))(&cfg);
  at::Tensor workspace;
  if (bytes) workspace = at::empty({(int64_t)bytes}, t[0]->options().dtype(at::kByte));
  const int rc = ((GemmFn)PyLong_AsVoidPtr(args[0]))(&cfg, t[0]->data_ptr(), (const uint8_t*)t[1]->data_ptr(), t[2]->data_ptr(), (const uint8_t*)t[3]->data_ptr(),
                                                     out.data_ptr(), bytes ? workspace.data_ptr() : nullptr, bytes, PyLong_AsVoidPtr(args[9]));
  if (rc != T5_OK) return PyLong_FromLong(rc);
  if (args[6] != Py_None) {
    Py_INCREF(args[6]);
    return args[6];
  }
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"adamw_entries", adamw_entries, METH_VARARGS, nullptr},
                         {"quantize_fp8", (PyCFunction)(void*)quantize_fp8, METH_FASTCALL, nullptr},
                         {"gemm_fp8", (PyCFunction)(void*)gemm_fp8, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
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
