// Argument marshalling of the calls that a serving loop makes: pointers of torch tensors, the cache struct, the
// current stream, and the C entry point, in one C function per call.  A generation step of a few heads takes
// the GPU 7 us and a launch takes the host 2.8, so what the interpreter spends around it counts: 32 heads x 205 slots,
// binding.py's call through ctypes 5.9 us, here 4.1.
//
// Only the plain case is taken: torch.Tensor itself or None for a pointer, int and float themselves for numbers,
// binding.Cache itself for the cache.  Anything else (subclasses, addresses, structs, numpy numbers, values that do not fit)
// returns -1 before anything is done, and binding.py goes through ctypes, whose conversions and errors then apply.
#include <Python.h>

#include <exception>

#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include "../../include/a2sf.h"

namespace {

PyObject *g_cache_type, *g_f32, *g_bf16, *g_raw_stream, *g_get_device;  // set once, by init
PyObject *n_k, *n_v, *n_scores, *n_pos, *n_len, *n_G, *n_capacity, *n_d, *n_dtype;

// Each reader: true if `x` is of the plain kind.
bool tensor(PyObject* x, const at::Tensor** t) {
  if (!THPVariable_CheckExact(x)) return false;
  *t = &THPVariable_Unpack(x);
  return true;
}
bool pointer(PyObject* x, void** p) {
  const at::Tensor* t;
  if (x == Py_None) { *p = nullptr; return true; }
  if (!tensor(x, &t)) return false;
  *p = t->data_ptr();  // (throws for a tensor without storage)
  return true;
}
bool number(PyObject* x, int32_t* v) {
  if (!PyLong_CheckExact(x)) return false;
  int over = 0;
  const long long l = PyLong_AsLongLongAndOverflow(x, &over);
  *v = (int32_t)l;
  return !over && l == *v;
}
bool number(PyObject* x, float* v) {
  if (!PyFloat_CheckExact(x)) return false;
  *v = (float)PyFloat_AS_DOUBLE(x);
  return true;
}
struct Owned {  // a new reference, given back
  PyObject* p;
  ~Owned() { Py_XDECREF(p); }
};
template <typename F>
bool attribute(PyObject* x, PyObject* name, F read) {
  const Owned a{PyObject_GetAttr(x, name)};
  if (!a.p) { PyErr_Clear(); return false; }
  return read(a.p);
}
bool cache_struct(PyObject* x, a2sf_cache* c) {
  if ((PyObject*)Py_TYPE(x) != g_cache_type) return false;
  const auto data = [&](PyObject* name, void** p) {
    return attribute(x, name, [&](PyObject* a) { return a != Py_None && pointer(a, p); });
  };
  const auto field = [&](PyObject* name, int32_t* v) { return attribute(x, name, [&](PyObject* a) { return number(a, v); }); };
  return data(n_k, &c->k) && data(n_v, &c->v) && data(n_scores, (void**)&c->scores) && data(n_pos, (void**)&c->pos) &&
         data(n_len, (void**)&c->len) && field(n_G, &c->G) && field(n_capacity, &c->capacity) && field(n_d, &c->d) &&
         attribute(x, n_dtype, [&](PyObject* a) {
           c->dtype = a == g_f32 ? A2SF_F32 : A2SF_BF16;
           return a == g_f32 || a == g_bf16;
         });
}
bool workspace(PyObject* x, PyObject* bytes, void** p, size_t* n) {
  const at::Tensor* t = nullptr;
  if (x != Py_None && !tensor(x, &t)) return false;
  *p = t ? t->data_ptr() : nullptr;
  if (bytes == Py_None) {
    *n = t ? t->nbytes() : 0;
    return true;
  }
  if (!PyLong_CheckExact(bytes)) return false;
  int over = 0;
  const long long l = PyLong_AsLongLongAndOverflow(bytes, &over);
  *n = (size_t)l;
  return !over && l >= 0;
}
// torch's current stream of the current device; `any` is an argument of the call: with a tensor on the GPU torch is initialised
bool stream(PyObject* x, PyObject* any, void** st) {
  const at::Tensor* t;
  if (x != Py_None || !g_raw_stream || !tensor(any, &t) || !t->is_cuda()) return false;
  const Owned dev{PyObject_CallNoArgs(g_get_device)};
  const Owned raw{dev.p ? PyObject_CallOneArg(g_raw_stream, dev.p) : nullptr};
  if (!raw.p) { PyErr_Clear(); return false; }
  *st = PyLong_AsVoidPtr(raw.p);
  return true;
}

// Runs the body of a call; C++ exceptions (a tensor without storage) become Python's.
template <typename F>
PyObject* guarded(F body) {
  try {
    const int status = body();
    return PyErr_Occurred() ? nullptr : PyLong_FromLong(status);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
template <typename F>
int without_gil(F call) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return status;
}
bool expects(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, got);
  return got == want;
}

// (entry point, q, k_new, v_new, t_pos, cache, group or None, alpha, select, recent, o, mode, workspace, workspace_bytes, stream)
PyObject* decode_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 15)) return nullptr;
  return guarded([&] {
    void *q, *k, *v, *o, *ws, *st, *fn = PyLong_AsVoidPtr(a[0]);
    int32_t t_pos, group = 1, mode;
    a2sf_budget b;
    float alpha;
    size_t bytes;
    a2sf_cache c;
    if (!(fn && pointer(a[1], &q) && pointer(a[2], &k) && pointer(a[3], &v) && number(a[4], &t_pos) && cache_struct(a[5], &c) &&
          (a[6] == Py_None || number(a[6], &group)) && number(a[7], &alpha) && number(a[8], &b.select) &&
          number(a[9], &b.recent) && pointer(a[10], &o) && number(a[11], &mode) && workspace(a[12], a[13], &ws, &bytes) &&
          stream(a[14], a[1], &st)))
      return -1;
    return without_gil([&]() -> int {
      if (a[6] == Py_None) return ((decltype(&a2sf_decode_step))fn)(q, k, v, t_pos, &c, alpha, b, mode, o, ws, bytes, st);
      return ((decltype(&a2sf_decode_step_gqa))fn)(q, k, v, t_pos, &c, group, alpha, b, mode, o, ws, bytes, st);
    });
  });
}

// (entry point, q, k, v, n, group or None, alpha, select, recent, cache, o, scores_full, workspace, workspace_bytes, stream)
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 15)) return nullptr;
  return guarded([&] {
    void *q, *k, *v, *o, *full, *ws, *st, *fn = PyLong_AsVoidPtr(a[0]);
    int32_t rows, group = 1;
    a2sf_budget b;
    float alpha;
    size_t bytes;
    a2sf_cache c;
    if (!(fn && pointer(a[1], &q) && pointer(a[2], &k) && pointer(a[3], &v) && number(a[4], &rows) &&
          (a[5] == Py_None || number(a[5], &group)) && number(a[6], &alpha) && number(a[7], &b.select) &&
          number(a[8], &b.recent) && cache_struct(a[9], &c) && pointer(a[10], &o) && pointer(a[11], &full) &&
          workspace(a[12], a[13], &ws, &bytes) && stream(a[14], a[1], &st)))
      return -1;
    return without_gil([&]() -> int {
      if (a[5] == Py_None) return ((decltype(&a2sf_prefill))fn)(q, k, v, rows, alpha, b, &c, o, (float*)full, ws, bytes, st);
      return ((decltype(&a2sf_prefill_gqa))fn)(q, k, v, rows, group, alpha, b, &c, o, (float*)full, ws, bytes, st);
    });
  });
}

// (entry point, q, k, v, m, pos0, group or None, alpha, select, recent, cache, o, workspace, workspace_bytes, stream)
PyObject* prefill_chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 15)) return nullptr;
  return guarded([&] {
    void *q, *k, *v, *o, *ws, *st, *fn = PyLong_AsVoidPtr(a[0]);
    int32_t m, pos0, group = 1;
    a2sf_budget b;
    float alpha;
    size_t bytes;
    a2sf_cache c;
    if (!(fn && pointer(a[1], &q) && pointer(a[2], &k) && pointer(a[3], &v) && number(a[4], &m) && number(a[5], &pos0) &&
          (a[6] == Py_None || number(a[6], &group)) && number(a[7], &alpha) && number(a[8], &b.select) &&
          number(a[9], &b.recent) && cache_struct(a[10], &c) && pointer(a[11], &o) && workspace(a[12], a[13], &ws, &bytes) &&
          stream(a[14], a[1], &st)))
      return -1;
    return without_gil([&]() -> int {
      if (a[6] == Py_None) return ((decltype(&a2sf_prefill_chunk))fn)(q, k, v, m, pos0, alpha, b, &c, o, ws, bytes, st);
      return ((decltype(&a2sf_prefill_chunk_gqa))fn)(q, k, v, m, pos0, group, alpha, b, &c, o, ws, bytes, st);
    });
  });
}

// ---- the operators around the attention: [rows, n] tensors, whose sizes, strides and types the C arguments come from.  What
// does not fit together, lies on another device (or is no plain tensor) is left to binding.py, which names the error.
bool type_of(const at::Tensor& t, int32_t* dtype) {
  const auto k = t.scalar_type();
  *dtype = k == at::kFloat ? A2SF_F32 : A2SF_BF16;
  return k == at::kFloat || k == at::kBFloat16;
}
bool matrix(const at::Tensor& t, int64_t rows, int64_t n) {
  return t.dim() == 2 && t.size(0) == rows && t.size(1) == n && (n == 1 || t.stride(1) == 1);
}
// `to` is null after an absent tensor
bool rows_like(PyObject* x, const at::Tensor& like, at::ScalarType type, a2sf_rows* s, const a2sf_rows** to) {
  const at::Tensor* t;
  *to = nullptr;
  if (x == Py_None) return true;
  if (!tensor(x, &t) || t->scalar_type() != type || !matrix(*t, like.size(0), like.size(1)) || t->device() != like.device()) return false;
  *s = {t->data_ptr(), t->stride(0)};
  *to = s;
  return true;
}
bool rows8(PyObject* q, PyObject* scales, const at::Tensor& like, int64_t rows, int64_t scale_rows, int64_t n, a2sf_rows8* s,
           const a2sf_rows8** to) {
  const at::Tensor *t, *u;
  *to = nullptr;
  if (q == Py_None && scales == Py_None) return true;
  if (!tensor(q, &t) || !tensor(scales, &u) || u->scalar_type() != at::kByte || t->device() != like.device() || u->device() != like.device())
    return false;
  if (t->scalar_type() != at::kFloat8_e4m3fn && t->scalar_type() != at::kByte) return false;
  const int64_t nb = n / 128 + (n % 128 != 0);
  if (!matrix(*t, rows, n) || !matrix(*u, scale_rows, nb)) return false;
  *s = {t->data_ptr(), (uint8_t*)u->data_ptr(), t->stride(0), u->stride(0)};
  *to = s;
  return true;
}
bool column(PyObject* x, const at::Tensor& like, int64_t rows, at::ScalarType type, const void** p) {
  const at::Tensor* t;
  *p = nullptr;
  if (x == Py_None) return true;
  if (!tensor(x, &t) || t->scalar_type() != type || t->dim() != 1 || t->size(0) != rows || (rows != 1 && t->stride(0) != 1) ||
      t->device() != like.device())
    return false;
  *p = t->data_ptr();
  return true;
}
bool first(PyObject* x, const at::Tensor** t, int32_t* dtype) {  // the tensor that gives a call its sizes
  return tensor(x, t) && (*t)->dim() == 2 && type_of(**t, dtype) && (*t)->size(0) <= INT32_MAX && (*t)->size(1) <= INT32_MAX;
}

// (entry point, x, weight, eps, residual, total, out, q, scales, stream)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 10)) return nullptr;
  return guarded([&] {
    void *st, *fn = PyLong_AsVoidPtr(a[0]);
    const at::Tensor* x;
    const void* w;
    a2sf_rows s[4];
    a2sf_rows8 s8;
    const a2sf_rows *rx, *residual, *total, *out;
    const a2sf_rows8* out8;
    int32_t dtype;
    float eps;
    if (!(fn && first(a[1], &x, &dtype) && rows_like(a[1], *x, x->scalar_type(), s, &rx) &&
          column(a[2], *x, x->size(1), x->scalar_type(), &w) && number(a[3], &eps) &&
          rows_like(a[4], *x, x->scalar_type(), s + 1, &residual) && rows_like(a[5], *x, x->scalar_type(), s + 2, &total) &&
          rows_like(a[6], *x, x->scalar_type(), s + 3, &out) && rows8(a[7], a[8], *x, x->size(0), x->size(0), x->size(1), &s8, &out8) &&
          stream(a[9], a[1], &st)))
      return -1;
    return without_gil([&]() -> int {
      return ((decltype(&a2sf_rms_norm))fn)(rx, residual, w, eps, (int32_t)x->size(0), (int32_t)x->size(1), dtype, total, out,
                                            out8, st);
    });
  });
}

// (entry point, x, q, scales, gate, out, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 7)) return nullptr;
  return guarded([&] {
    void *st, *fn = PyLong_AsVoidPtr(a[0]);
    const at::Tensor* x;
    a2sf_rows s[3];
    a2sf_rows8 s8;
    const a2sf_rows *rx, *gate, *out;
    const a2sf_rows8* out8;
    int32_t dtype;
    if (!(fn && first(a[1], &x, &dtype) && rows_like(a[1], *x, x->scalar_type(), s, &rx) &&
          rows8(a[2], a[3], *x, x->size(0), x->size(0), x->size(1), &s8, &out8) &&
          rows_like(a[4], *x, x->scalar_type(), s + 1, &gate) && rows_like(a[5], *x, x->scalar_type(), s + 2, &out) &&
          stream(a[6], a[1], &st)))
      return -1;
    return without_gil([&]() -> int {
      return ((decltype(&a2sf_quantize))fn)(rx, gate, (int32_t)x->size(0), (int32_t)x->size(1), dtype, out, out8, st);
    });
  });
}

// (entry point, a, a_scales, b, b_scales, c, workspace, workspace_bytes, stream[, wide_sums])
PyObject* matmul_scaled(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 10 && !expects(n, 9)) return nullptr;
  return guarded([&] {
    void *ws, *st, *fn = PyLong_AsVoidPtr(a[0]);
    const at::Tensor *c, *b;
    a2sf_rows s;
    a2sf_rows8 s8[2];
    const a2sf_rows* rc;
    const a2sf_rows8 *ra, *rb;
    const at::Tensor *ta, *room;
    size_t bytes;
    int32_t dtype;
    if (!(fn && first(a[5], &c, &dtype) && rows_like(a[5], *c, c->scalar_type(), &s, &rc) && tensor(a[1], &ta) && ta->dim() == 2 &&
          tensor(a[3], &b) && ta->size(1) <= INT32_MAX &&
          rows8(a[1], a[2], *c, c->size(0), c->size(0), ta->size(1), s8, &ra) &&
          rows8(a[3], a[4], *c, c->size(1), c->size(1) / 128 + (c->size(1) % 128 != 0), ta->size(1), s8 + 1, &rb) &&
          workspace(a[6], a[7], &ws, &bytes) && (!tensor(a[6], &room) || room->device() == c->device()) && stream(a[8], a[1], &st) && (n == 9 || PyBool_Check(a[9]))))
      return -1;
    if (n == 10 && a[9] == Py_True) dtype |= A2SF_WIDE_SUMS;
    return without_gil([&]() -> int {
      return ((decltype(&a2sf_matmul_scaled))fn)(ra, rb, (int32_t)c->size(0), (int32_t)c->size(1), (int32_t)ta->size(1), rc, dtype,
                                                 ws, bytes, st);
    });
  });
}

// (entry point, list of (x, y[, rotate]), pos, table, interleaved, inverse, stream)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 7)) return nullptr;
  return guarded([&] {
    void *st, *fn = PyLong_AsVoidPtr(a[0]);
    const at::Tensor *x, *y, *head = nullptr, *pos, *table;
    a2sf_rotary_part parts[A2SF_MAX_ROTARY_PARTS];
    int32_t dtype = 0;
    if (!fn || !PyList_CheckExact(a[1]) || PyList_GET_SIZE(a[1]) < 1 || PyList_GET_SIZE(a[1]) > A2SF_MAX_ROTARY_PARTS) return -1;
    const int count = (int)PyList_GET_SIZE(a[1]);
    for (int i = 0; i < count; ++i) {
      PyObject* p = PyList_GET_ITEM(a[1], i);
      if (!PyTuple_CheckExact(p) || PyTuple_GET_SIZE(p) < 2 || PyTuple_GET_SIZE(p) > 3) return -1;
      if (!tensor(PyTuple_GET_ITEM(p, 0), &x) || !tensor(PyTuple_GET_ITEM(p, 1), &y) || x->dim() != 4 || x->sizes() != y->sizes()) return -1;
      PyObject* turn = PyTuple_GET_SIZE(p) == 3 ? PyTuple_GET_ITEM(p, 2) : Py_True;
      if (!PyBool_Check(turn)) return -1;
      if (i == 0) {
        head = x;
        if (!type_of(*x, &dtype)) return -1;
        for (int j = 0; j < 4; ++j)
          if (x->size(j) > INT32_MAX) return -1;
      }
      if (x->size(0) != head->size(0) || x->size(1) != head->size(1) || x->size(3) != head->size(3) || x->size(2) > INT32_MAX ||
          x->scalar_type() != head->scalar_type() || y->scalar_type() != head->scalar_type() || x->device() != head->device() ||
          y->device() != head->device() ||
          (x->size(3) != 1 && (x->stride(3) != 1 || y->stride(3) != 1)))
        return -1;
      parts[i].x = x->data_ptr();
      parts[i].y = y->data_ptr();
      for (int j = 0; j < 3; ++j) {
        parts[i].x_stride[j] = x->stride(j);
        parts[i].y_stride[j] = y->stride(j);
      }
      parts[i].heads = (int32_t)x->size(2);
      parts[i].rotate = turn == Py_True;
    }
    if (!tensor(a[2], &pos) || pos->scalar_type() != at::kInt || !matrix(*pos, head->size(0), head->size(1)) || !tensor(a[3], &table) ||
        table->scalar_type() != at::kFloat || table->dim() != 2 || !table->is_contiguous() || table->size(0) > INT32_MAX ||
        table->size(1) > INT32_MAX || pos->device() != head->device() || table->device() != head->device() || !PyBool_Check(a[4]) || !PyBool_Check(a[5]) || !stream(a[6], a[2], &st))
      return -1;
    return without_gil([&]() -> int {
      return ((decltype(&a2sf_rotary))fn)(parts, count, (int32_t)head->size(0), (int32_t)head->size(1), (int32_t)head->size(3), dtype,
                                          (const int32_t*)pos->data_ptr(), pos->stride(0), (const float*)table->data_ptr(),
                                          (int32_t)table->size(0), (int32_t)table->size(1), a[4] == Py_True, a[5] == Py_True, st);
    });
  });
}

// (entry point, logits, noise, token, temperature, top_k, top_p, min_p, prob, stream)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 10)) return nullptr;
  return guarded([&] {
    void *st, *fn = PyLong_AsVoidPtr(a[0]);
    const at::Tensor* x;
    a2sf_rows s[2];
    const a2sf_rows *logits, *noise;
    const void *token, *temperature, *top_k, *top_p, *min_p, *prob;
    int32_t dtype;
    if (!(fn && first(a[1], &x, &dtype) && rows_like(a[1], *x, x->scalar_type(), s, &logits) &&
          rows_like(a[2], *x, at::kFloat, s + 1, &noise) && column(a[3], *x, x->size(0), at::kInt, &token) &&
          column(a[4], *x, x->size(0), at::kFloat, &temperature) && column(a[5], *x, x->size(0), at::kInt, &top_k) &&
          column(a[6], *x, x->size(0), at::kFloat, &top_p) && column(a[7], *x, x->size(0), at::kFloat, &min_p) &&
          column(a[8], *x, x->size(0), at::kFloat, &prob) && stream(a[9], a[1], &st)))
      return -1;
    return without_gil([&]() -> int {
      return ((decltype(&a2sf_sample))fn)(logits, noise, (int32_t)x->size(0), (int32_t)x->size(1), dtype, (const float*)temperature,
                                          (const int32_t*)top_k, (const float*)top_p, (const float*)min_p, (int32_t*)token,
                                          (float*)prob, st);
    });
  });
}

// (binding.Cache, torch.float32, torch.bfloat16, function device -> current raw stream or None, function -> current device)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!expects(n, 5)) return nullptr;
  PyObject** const to[] = {&g_cache_type, &g_f32, &g_bf16, &g_raw_stream, &g_get_device};
  for (int i = 0; i < 5; ++i) {
    Py_XDECREF(*to[i]);
    *to[i] = a[i] == Py_None ? nullptr : a[i];
    Py_XINCREF(*to[i]);
  }
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", (PyCFunction)(void (*)())init, METH_FASTCALL, nullptr},
                         {"decode_step", (PyCFunction)(void (*)())decode_step, METH_FASTCALL, nullptr},
                         {"prefill", (PyCFunction)(void (*)())prefill, METH_FASTCALL, nullptr},
                         {"prefill_chunk", (PyCFunction)(void (*)())prefill_chunk, METH_FASTCALL, nullptr},
                         {"rms_norm", (PyCFunction)(void (*)())rms_norm, METH_FASTCALL, nullptr},
                         {"quantize", (PyCFunction)(void (*)())quantize, METH_FASTCALL, nullptr},
                         {"matmul_scaled", (PyCFunction)(void (*)())matmul_scaled, METH_FASTCALL, nullptr},
                         {"rotary", (PyCFunction)(void (*)())rotary, METH_FASTCALL, nullptr},
                         {"sample", (PyCFunction)(void (*)())sample, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#define A2SF_STR_(x) #x
#define A2SF_STR(x) A2SF_STR_(x)
PyMODINIT_FUNC PyInit__call() {
  PyObject** const names[] = {&n_k, &n_v, &n_scores, &n_pos, &n_len, &n_G, &n_capacity, &n_d, &n_dtype};
  const char* const text[] = {"k", "v", "scores", "pos", "len", "G", "capacity", "d", "dtype"};
  for (int i = 0; i < 9; ++i)
    if (!*names[i] && !(*names[i] = PyUnicode_InternFromString(text[i]))) return nullptr;
  PyObject* m = PyModule_Create(&module);
  // (binding.py does without the extension where these are not the ones that run)
  const char* const built_for = "torch " TORCH_VERSION ", Python " A2SF_STR(PY_MAJOR_VERSION) "." A2SF_STR(PY_MINOR_VERSION);
  if (m && PyModule_AddStringConstant(m, "built_for", built_for) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
