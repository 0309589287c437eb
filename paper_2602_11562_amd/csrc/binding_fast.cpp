// The marshalling of laser_forward and of attention among a history's items in native code, for calls of the ordinary form: plain device
// tensors, contiguous (rows of heads: apart by token), outputs given. Anything else returns None, and the caller (binding.py) goes its
// own way, with its own checks and errors. A small request is 8 us of kernels; attribute by attribute in Python, with ctypes, its host
// part took 10.5 us a call. Torch's accessors are inlined here, so the module names the torch that it was built against (`stamp`), and the
// caller leaves it alone in any other.
#include <torch/csrc/autograd/python_variable.h>

typedef int (*Forward)(const void*, const void*, const void*, const void*, const void*, const void*, const void*, const int32_t*, int, int,
                       int, int, int, int, float, int, int, void*, int32_t*, float*, void*);

// a tensor's data where it is a plain contiguous device tensor of the type, else null
static void* data_of(PyObject* o, at::ScalarType type) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || !t.has_storage() || !t.is_contiguous())
    return nullptr;
  return t.data_ptr();
}

// whether the number just read was no address: then nothing may be called with it, and nothing returned beside its error
static bool no_address() {
  const bool bad = PyErr_Occurred() != nullptr;
  if (bad) PyErr_Clear();
  return bad;
}

// forward(address of laser_forward, q, k, v, t0, wq, wk, wv, lens, w, gamma, seg_out, seg_cnt, z_out, stream) -> status, or None:
// not a call of this form, nothing done
static PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    if (n != 15 || !PyLong_CheckExact(a[0]) || !PyLong_CheckExact(a[9]) || !PyFloat_CheckExact(a[10])) Py_RETURN_NONE;
    const auto fn = reinterpret_cast<Forward>(PyLong_AsVoidPtr(a[0]));
    int overflow = 0;
    const long w = PyLong_AsLongAndOverflow(a[9], &overflow);
    if (no_address()) Py_RETURN_NONE;
    if (!fn || overflow || w != (int)w || w == 0 || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
    const at::Tensor& q = THPVariable_Unpack(a[1]);
    const at::ScalarType type = q.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) Py_RETURN_NONE;
    void* p[7];
    for (int i = 0; i < 7; ++i)
      if (!(p[i] = data_of(a[1 + i], type))) Py_RETURN_NONE;
    const at::Tensor &v = THPVariable_Unpack(a[3]), &wq = THPVariable_Unpack(a[5]);
    if (q.dim() != 3 || v.dim() < 3 || wq.dim() < 1) Py_RETURN_NONE;
    void *lens = nullptr, *cnt = nullptr, *stream = nullptr;
    if (a[8] != Py_None && !(lens = data_of(a[8], at::kInt))) Py_RETURN_NONE;
    if (a[12] != Py_None && !(cnt = data_of(a[12], at::kInt))) Py_RETURN_NONE;
    void *seg = data_of(a[11], type), *z = data_of(a[13], at::kFloat);
    if (!seg || !z) Py_RETURN_NONE;
    if (a[14] != Py_None) {
      if (!PyLong_CheckExact(a[14])) Py_RETURN_NONE;
      stream = PyLong_AsVoidPtr(a[14]);
      if (no_address()) Py_RETURN_NONE;
    }
    const int64_t sizes[6] = {q.size(0), q.size(1), v.size(1), q.size(2), v.size(2), wq.size(0)};
    for (const int64_t s : sizes)
      if (s != (int)s) Py_RETURN_NONE;
    const float gamma = (float)PyFloat_AS_DOUBLE(a[10]);
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = fn(p[0], p[1], p[2], p[3], p[4], p[5], p[6], static_cast<int32_t*>(lens), (int)sizes[0], (int)sizes[1], (int)sizes[2],
              (int)sizes[3], (int)sizes[4], (int)w, gamma, (int)sizes[5], type == at::kFloat ? 0 : 1, seg, static_cast<int32_t*>(cnt),
              static_cast<float*>(z), stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(code);
  } catch (...) {   // (a tensor without data of its own: as any other form)
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// ---------------------------------------------------------------- attention among a history's items
// What a call of the ordinary form hands over, argument by argument; `ok` falls with the first that is of another form. All tensors are
// on device `device`, the current one.
struct Args {
  PyObject* const* a;
  int device = -1;
  bool ok = true;
  const void* address(int i) {
    const void* p = PyLong_CheckExact(a[i]) ? PyLong_AsVoidPtr(a[i]) : nullptr;
    if (no_address() || !p) ok = false;
    return p;
  }
  int number(int i) {
    int overflow = 0;
    const long x = PyLong_CheckExact(a[i]) || PyBool_Check(a[i]) ? PyLong_AsLongAndOverflow(a[i], &overflow) : 0;
    if ((!PyLong_CheckExact(a[i]) && !PyBool_Check(a[i])) || overflow || x != (int)x || no_address()) ok = false;
    return (int)x;
  }
  float real(int i) {
    if (!PyFloat_CheckExact(a[i])) ok = false;
    return ok ? (float)PyFloat_AS_DOUBLE(a[i]) : 0.0f;
  }
  void* stream(int i) {
    if (a[i] == Py_None) return nullptr;
    void* p = PyLong_CheckExact(a[i]) ? PyLong_AsVoidPtr(a[i]) : nullptr;
    if (no_address() || !PyLong_CheckExact(a[i])) ok = false;
    return p;
  }
  const at::Tensor* tensor(int i, at::ScalarType type) {
    if (!ok || !THPVariable_CheckExact(a[i])) return ok = false, nullptr;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (!t.defined() || !t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.layout() != at::kStrided ||
        !t.has_storage())
      return ok = false, nullptr;
    return &t;
  }
  // a contiguous tensor of these sizes (-1: any, and told)
  void* flat(int i, at::ScalarType type, std::initializer_list<int64_t> sizes, int64_t* told = nullptr) {
    const at::Tensor* t = tensor(i, type);
    if (!t || t->dim() != (int64_t)sizes.size() || !t->is_contiguous()) return ok = false, nullptr;
    int d = 0;
    for (const int64_t s : sizes) {
      if (s >= 0 ? t->size(d) != s : t->size(d) != (int)t->size(d)) return ok = false, nullptr;
      if (s < 0) *told++ = t->size(d);
      ++d;
    }
    return t->data_ptr();
  }
  // [tokens, heads, D], heads side by side
  void* rows(int i, at::ScalarType type, int64_t tokens, int64_t heads, int64_t D, int64_t* pitch) {
    const at::Tensor* t = tensor(i, type);
    if (!t || t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != D || (t->stride(2) != 1 && D > 1) ||
        (t->stride(1) != D && heads > 1))
      return ok = false, nullptr;
    *pitch = tokens > 1 ? t->stride(0) : heads * D;
    return t->data_ptr();
  }
  // the sizes of [a, b, c] of either storage type
  bool sizes3(int i, int64_t* x, at::ScalarType* type) {
    if (!ok || !THPVariable_CheckExact(a[i])) return ok = false;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (!t.defined() || t.dim() != 3 || (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16)) return ok = false;
    *type = t.scalar_type();
    for (int d = 0; d < 3; ++d)
      if ((x[d] = t.size(d)) != (int)x[d]) return ok = false;
    return true;
  }
};

static int dtype_of(at::ScalarType type) { return type == at::kFloat ? 0 : 1; }

template <typename F>
static PyObject* guarded(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F&& f) {
  if (n != want) Py_RETURN_NONE;
  try {
    Args x{a};
    x.device = x.number(1);
    int code = 0;
    if (x.ok) f(x, &code);
    if (!x.ok) Py_RETURN_NONE;
    return PyLong_FromLong(code);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

#define LASER_UNLOCKED(call)  \
  do {                        \
    Py_BEGIN_ALLOW_THREADS    \
    *code = call;             \
    Py_END_ALLOW_THREADS      \
  } while (0)

// (address, device, q, k, v, off, L_max, gamma, o_out, lse_out, stream)
static PyObject* history_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 11, [](Args& x, int* code) {
    typedef int (*Fn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, const void*, int, int, int, int, int, int, float, int,
                      void*, void*, void*);
    const auto fn = reinterpret_cast<Fn>(x.address(0));
    int64_t s[3], kv[3], parts, qp, kp, vp;
    at::ScalarType type, type_k;
    if (!x.sizes3(2, s, &type) || !x.sizes3(3, kv, &type_k)) return;
    const void *q = x.rows(2, type, s[0], s[1], s[2], &qp), *k = x.rows(3, type, s[0], kv[1], s[2], &kp),
               *v = x.rows(4, type, s[0], kv[1], s[2], &vp);
    const void* off = x.flat(5, at::kInt, {-1}, &parts);
    const int L = x.number(6);
    const float gamma = x.real(7);
    void *o = x.flat(8, type, {s[0], s[1], s[2]}), *lse = x.flat(9, at::kFloat, {s[0], s[1]}), *stream = x.stream(10);
    if (!x.ok || parts < 2) return x.ok = false, void();
    LASER_UNLOCKED(fn(q, qp, k, kp, v, vp, off, (int)parts - 1, (int)s[0], L, (int)s[1], (int)kv[1], (int)s[2], gamma, dtype_of(type), o, lse,
                      stream));
  });
}

// (address, device, q, k, v, o, lse, d_o, off, L_max, gamma, dq, dk, dv, work, stream)
static PyObject* history_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 16, [](Args& x, int* code) {
    typedef int (*Fn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, const void*, const void*, const void*, const void*, int,
                      int, int, int, int, int, float, int, void*, int64_t, void*, int64_t, void*, int64_t, void*, size_t, void*);
    const auto fn = reinterpret_cast<Fn>(x.address(0));
    int64_t s[3], kv[3], parts, room, qp, kp, vp, dqp, dkp, dvp;
    at::ScalarType type, type_k;
    if (!x.sizes3(2, s, &type) || !x.sizes3(3, kv, &type_k)) return;
    const void *q = x.rows(2, type, s[0], s[1], s[2], &qp), *k = x.rows(3, type, s[0], kv[1], s[2], &kp),
               *v = x.rows(4, type, s[0], kv[1], s[2], &vp);
    const void *o = x.flat(5, type, {s[0], s[1], s[2]}), *lse = x.flat(6, at::kFloat, {s[0], s[1]}),
               *go = x.flat(7, type, {s[0], s[1], s[2]});
    const void* off = x.flat(8, at::kInt, {-1}, &parts);
    const int L = x.number(9);
    const float gamma = x.real(10);
    void *dq = x.rows(11, type, s[0], s[1], s[2], &dqp), *dk = x.rows(12, type, s[0], kv[1], s[2], &dkp),
         *dv = x.rows(13, type, s[0], kv[1], s[2], &dvp);
    void *work = x.flat(14, at::kByte, {-1}, &room), *stream = x.stream(15);
    if (!x.ok || parts < 2) return x.ok = false, void();
    LASER_UNLOCKED(fn(q, qp, k, kp, v, vp, o, lse, go, off, (int)parts - 1, (int)s[0], L, (int)s[1], (int)kv[1], (int)s[2], gamma, dtype_of(type),
                      dq, dqp, dk, dkp, dv, dvp, work, (size_t)room, stream));
  });
}

// k_cache, v_cache, pages, lens
struct Cache {
  void *k = nullptr, *v = nullptr, *pages = nullptr, *lens = nullptr;
  int64_t P = 0, Hkv = 0, page = 0, D = 0, U = 0, most = 0;
  at::ScalarType type = at::kFloat;
  Cache(Args& x, int k_at, int v_at, int pages_at, int lens_at) {
    int64_t s[4], t[2];
    if (!x.ok || !THPVariable_CheckExact(x.a[k_at])) {
      x.ok = false;
      return;
    }
    type = THPVariable_Unpack(x.a[k_at]).scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) x.ok = false;
    k = x.flat(k_at, type, {-1, -1, -1, -1}, s);
    pages = x.flat(pages_at, at::kInt, {-1, -1}, t);
    if (!x.ok) return;
    P = s[0], Hkv = s[1], page = s[2], D = s[3], U = t[0], most = t[1];
    v = v_at < 0 ? k : x.flat(v_at, type, {P, Hkv, page, D});
    lens = x.flat(lens_at, at::kInt, {U});
  }
};

// (address, device, k, v, k_cache, v_cache, off, pages, lens, C_max, L_max, weight or None, stream)
static PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 13, [](Args& x, int* code) {
    typedef int (*Fn)(const void*, int64_t, const void*, int64_t, void*, void*, const void*, const void*, const void*, int, int, int, int, int, int,
                      int, int, int, int, void*, void*);
    const auto fn = reinterpret_cast<Fn>(x.address(0));
    const Cache c(x, 4, 5, 7, 8);
    int64_t s[3], kp, vp;
    at::ScalarType type;
    if (!x.sizes3(2, s, &type)) return;
    const void *k = x.rows(2, c.type, s[0], c.Hkv, c.D, &kp), *v = x.rows(3, c.type, s[0], c.Hkv, c.D, &vp),
               *off = x.flat(6, at::kInt, {c.U + 1});
    const int C = x.number(9), L = x.number(10);
    void *weight = x.a[11] == Py_None ? nullptr : x.flat(11, at::kFloat, {c.P, c.page}), *stream = x.stream(12);
    if (!x.ok) return;
    LASER_UNLOCKED(fn(k, kp, v, vp, c.k, c.v, off, c.pages, c.lens, (int)c.U, (int)s[0], C, (int)c.P, (int)c.page, (int)c.most, L, (int)c.Hkv,
                      (int)c.D, dtype_of(c.type), weight, stream));
  });
}

// (address, device, q, k_cache, v_cache, off, pages, lens, C_max, L_max, gamma, causal, o_out, lse_out, work, stream)
static PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 16, [](Args& x, int* code) {
    typedef int (*Fn)(const void*, int64_t, const void*, const void*, const void*, const void*, const void*, int, int, int, int, int, int, int, int,
                      int, int, float, int, int, void*, void*, void*, size_t, void*);
    const auto fn = reinterpret_cast<Fn>(x.address(0));
    const Cache c(x, 3, 4, 6, 7);
    int64_t s[3], qp, room;
    at::ScalarType type;
    if (!x.sizes3(2, s, &type)) return;
    const void *q = x.rows(2, c.type, s[0], s[1], c.D, &qp), *off = x.flat(5, at::kInt, {c.U + 1});
    const int C = x.number(8), L = x.number(9), causal = x.number(11);
    const float gamma = x.real(10);
    void *o = x.flat(12, c.type, {s[0], s[1], c.D}), *lse = x.flat(13, at::kFloat, {s[0], s[1]}),
         *work = x.flat(14, at::kByte, {-1}, &room);
    void* stream = x.stream(15);
    if (!x.ok) return;
    LASER_UNLOCKED(fn(q, qp, c.k, c.v, off, c.pages, c.lens, (int)c.U, (int)s[0], C, (int)c.P, (int)c.page, (int)c.most, L, (int)s[1], (int)c.Hkv,
                      (int)c.D, gamma, causal != 0, dtype_of(c.type), o, lse, work, (size_t)room, stream));
  });
}

// (address, device, q, lse, k_cache, off, pages, lens, C_max, L_max, gamma, weight, causal, add, stream)
static PyObject* cache_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 15, [](Args& x, int* code) {
    typedef int (*Fn)(const void*, int64_t, const void*, const void*, const void*, const void*, const void*, int, int, int, int, int, int, int, int,
                      int, int, float, int, int, int, void*, void*);
    const auto fn = reinterpret_cast<Fn>(x.address(0));
    const Cache c(x, 4, -1, 6, 7);
    int64_t s[3], qp;
    at::ScalarType type;
    if (!x.sizes3(2, s, &type)) return;
    const void *q = x.rows(2, c.type, s[0], s[1], c.D, &qp), *lse = x.flat(3, at::kFloat, {s[0], s[1]}), *off = x.flat(5, at::kInt, {c.U + 1});
    const int C = x.number(8), L = x.number(9), causal = x.number(12), add = x.number(13);
    const float gamma = x.real(10);
    void *weight = x.flat(11, at::kFloat, {c.P, c.page}), *stream = x.stream(14);
    if (!x.ok) return;
    LASER_UNLOCKED(fn(q, qp, lse, c.k, off, c.pages, c.lens, (int)c.U, (int)s[0], C, (int)c.P, (int)c.page, (int)c.most, L, (int)s[1], (int)c.Hkv,
                      (int)c.D, gamma, causal != 0, add != 0, dtype_of(c.type), weight, stream));
  });
}

// (address, device, k_cache, v_cache, weight, pages, lens, pages_out, budget, recent, L_max, lens_out, kept_out, stream)
static PyObject* cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 14, [](Args& x, int* code) {
    typedef int (*Fn)(void*, void*, void*, const void*, const void*, const void*, int, int, int, int, int, int, int, int, int, int, int, void*, void*,
                      void*);
    const auto fn = reinterpret_cast<Fn>(x.address(0));
    const Cache c(x, 2, 3, 5, 6);
    if (!x.ok) return;
    int64_t out;
    void* weight = x.flat(4, at::kFloat, {c.P, c.page});
    const void* pages_out = x.flat(7, at::kInt, {c.U, -1}, &out);
    const int budget = x.number(8), recent = x.number(9), L = x.number(10);
    if (budget < 0) x.ok = false;
    void *lens_out = x.flat(11, at::kInt, {c.U}), *kept = x.ok ? x.flat(12, at::kInt, {c.U, budget}) : nullptr, *stream = x.stream(13);
    if (!x.ok) return;
    LASER_UNLOCKED(fn(c.k, c.v, weight, c.pages, c.lens, pages_out, (int)c.U, (int)c.P, (int)c.page, (int)c.most, (int)out, L, budget, recent,
                      (int)c.Hkv, (int)c.D, dtype_of(c.type), lens_out, kept, stream));
  });
}

#define LASER_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
static PyMethodDef methods[] = {LASER_METHOD(forward),      LASER_METHOD(history_forward), LASER_METHOD(history_backward),
                                LASER_METHOD(cache_append), LASER_METHOD(cache_attention), LASER_METHOD(cache_weights),
                                LASER_METHOD(cache_evict),  {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "laser_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
PyMODINIT_FUNC PyInit_laser_fast() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "stamp", LASER_TORCH_STAMP) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
