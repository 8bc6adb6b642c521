// Native marshalling of the rotary, page-table and 4-bit-cache entry points for
// Python: checks of placement, dtype, shape and contiguity, then the C call on
// torch's current stream of the tensors' GPU, with that GPU current.  A step of one
// sequence is as short as these checks, which cost microseconds in Python.
//
// The functions take every argument by position (None where there is none) and return
// the C status; __init__.py holds the public signatures, defaults and allocations.
// bind() gives the addresses of the C entry points in the loaded libsfa.so.
#include <torch/csrc/autograd/python_variable.h>

#include <hip/hip_runtime_api.h>

#include <initializer_list>
#include <string>

#include "../../include/sfa.h"

namespace {

struct Refused {
  PyObject* type;
  std::string what;
};
[[noreturn]] void refuse(PyObject* type, const std::string& what) { throw Refused{type, what}; }

typedef std::initializer_list<int64_t> Shape;

std::string list(Shape s) {
  std::string r = "[";
  for (int64_t v : s) r += (r.size() > 1 ? ", " : "") + std::to_string(v);
  return r + "]";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + " must be a torch.Tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse(PyExc_ValueError, std::string(name) + " must be a GPU tensor (got " + t.device().str() + ")");
  return t;
}

const at::Tensor& on(PyObject* o, const char* name, int dev) {
  const at::Tensor& t = tensor(o, name);
  if (t.get_device() != dev)
    refuse(PyExc_ValueError, std::string(name) + " is on " + t.device().str() + ", not on GPU " + std::to_string(dev));
  return t;
}

bool is_shape(const at::Tensor& t, Shape s) {
  return t.sizes() == at::IntArrayRef(s.begin(), s.size());
}

[[noreturn]] void bad_dtype(const at::Tensor& t, const char* name) {
  refuse(PyExc_TypeError, std::string(name) + ": unsupported dtype " + c10::toString(t.scalar_type()));
}

void* contiguous(const at::Tensor& t, const char* name) {
  if (!t.is_contiguous()) refuse(PyExc_ValueError, std::string(name) + " must be contiguous");
  return t.data_ptr();
}

// A contiguous tensor of that dtype on GPU dev, of that shape where one is given.
void* array(PyObject* o, const char* name, at::ScalarType type, int dev) {
  const at::Tensor& t = on(o, name, dev);
  if (t.scalar_type() != type) bad_dtype(t, name);
  return contiguous(t, name);
}
void* array(PyObject* o, const char* name, at::ScalarType type, int dev, Shape s) {
  void* p = array(o, name, type, dev);
  if (!is_shape(THPVariable_Unpack(o), s)) refuse(PyExc_ValueError, std::string(name) + " must be " + list(s));
  return p;
}
// int32 with n entries, any shape
int32_t* ints(PyObject* o, const char* name, int64_t n, int dev) {
  void* p = array(o, name, at::kInt, dev);
  if (THPVariable_Unpack(o).numel() != n)
    refuse(PyExc_ValueError, std::string(name) + " must hold " + std::to_string(n) + " entries");
  return (int32_t*)p;
}

int idx_code(const at::Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kInt: return SFA_I32;
    case at::kShort: return SFA_I16;
    case at::kByte: return SFA_U8;
    default: bad_dtype(t, name);
  }
}
int val_code(const at::Tensor& t, const char* name, bool half) {
  switch (t.scalar_type()) {
    case at::kFloat: return SFA_F32;
    case at::kBFloat16: return SFA_BF16;
    case at::kHalf: if (half) return SFA_F16;  // codes only
    default: bad_dtype(t, name);
  }
}

bool none(PyObject* o) { return o == Py_None; }

int64_t integer(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse(PyExc_TypeError, std::string(name) + " must be an integer");
  }
  return v;
}
int small(PyObject* o, const char* name) {
  const int64_t v = integer(o, name);
  if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, std::string(name) + " is out of range");
  return (int)v;
}
int size(int64_t v, const char* name) {
  if (v > INT32_MAX) refuse(PyExc_ValueError, std::string(name) + " is out of range");
  return (int)v;
}

// Rows [B, H, n, d] of float32 or bf16, coordinates contiguous.
struct Rows {
  void* p;
  int code;
  int64_t st[3];
  Rows(PyObject* o, const char* name, int dev, Shape s) {
    const at::Tensor& t = on(o, name, dev);
    code = val_code(t, name, false);
    if (!is_shape(t, s)) refuse(PyExc_ValueError, std::string(name) + " must be " + list(s));
    if (t.stride(3) != 1 && t.size(3) != 1)
      refuse(PyExc_ValueError, std::string(name) + ": a row's coordinates must be contiguous");
    for (int i = 0; i < 3; ++i) st[i] = t.stride(i);
    p = t.data_ptr();
  }
};
// The shape of a [B, H, n, d] tensor.
at::IntArrayRef heads(const at::Tensor& t, const char* name) {
  if (t.dim() != 4) refuse(PyExc_ValueError, std::string(name) + " must be [B, H, n, d]");
  return t.sizes();
}

// Positions [naxes, B, n], [B, n] or [n]; entries of size 1 are shared.
struct Positions {
  const int32_t* p;
  int64_t axis = 0, batch = 0;
  Positions(PyObject* o, int naxes, int64_t B, int64_t n, int dev) {
    const at::Tensor& t = on(o, "pos", dev);
    if (t.scalar_type() != at::kInt) refuse(PyExc_TypeError, "pos must be an int32 tensor");
    const int k = (int)t.dim();
    bool ok = k >= 1 && k <= 3 && t.size(k - 1) == n;
    if (ok && k >= 2 && t.size(k - 2) != 1) { ok = t.size(k - 2) == B; batch = t.stride(k - 2); }
    if (ok && k == 3 && t.size(0) != 1) { ok = t.size(0) == naxes; axis = t.stride(0); }
    if (!ok) refuse(PyExc_ValueError, "pos must be [naxes, B, n], [B, n] or [n]");
    if (n > 1 && t.stride(k - 1) != 1) refuse(PyExc_ValueError, "pos: tokens must be contiguous");
    p = (const int32_t*)t.data_ptr();
  }
};

// The C entry points, and torch's current stream.
decltype(&sfa_rope) c_rope;
decltype(&sfa_rope_encode) c_rope_encode;
decltype(&sfa_rope_encode_bwd) c_rope_encode_bwd;
decltype(&sfa_page_tables) c_page_tables;
decltype(&sfa_kv_append_q4) c_kv_append_q4;
decltype(&sfa_attn_decode_q4) c_attn_decode_q4;
PyObject* raw_stream;

void* stream_of(int dev) {
  PyObject* i = PyLong_FromLong(dev);
  PyObject* r = i ? PyObject_CallOneArg(raw_stream, i) : nullptr;
  Py_XDECREF(i);
  if (!r) {
    PyErr_Clear();
    refuse(PyExc_RuntimeError, "torch gave no current stream");
  }
  void* s = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return s;
}

// GPU dev current for the call.
struct Current {
  int before = -1;
  explicit Current(int dev) {
    int now = dev;
    if (hipGetDevice(&now) != hipSuccess) refuse(PyExc_RuntimeError, "no current GPU");
    if (now != dev) {
      if (hipSetDevice(dev) != hipSuccess) refuse(PyExc_RuntimeError, "GPU cannot be made current");
      before = now;
    }
  }
  ~Current() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F f) {
  try {
    if (given != wanted) refuse(PyExc_TypeError, "wrong number of arguments");
    return PyLong_FromLong(f());
  } catch (const Refused& r) {
    PyErr_SetString(r.type, r.what.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

const sfa_rope_plan* plan_of(PyObject* o) { return (const sfa_rope_plan*)PyLong_AsVoidPtr(o); }
void plan_d(const sfa_rope_plan* plan, int64_t d) {
  if (d != plan->d)
    refuse(PyExc_ValueError, "x has " + std::to_string(d) + " coordinates, the plan " + std::to_string(plan->d));
}

// rope(x, pos, plan address, inverse, y)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> long {
    const at::Tensor& x = tensor(a[0], "x");
    const int dev = x.get_device();
    const auto s = heads(x, "x");
    const sfa_rope_plan* plan = plan_of(a[2]);
    plan_d(plan, s[3]);
    const Positions pos(a[1], plan->naxes, s[0], s[2], dev);
    const Rows rx(a[0], "x", dev, {s[0], s[1], s[2], s[3]}), ry(a[4], "y", dev, {s[0], s[1], s[2], s[3]});
    if (s[0] == 0 || s[1] == 0 || s[2] == 0) return SFA_OK;
    const Current cur(dev);
    return c_rope(rx.p, rx.st, pos.p, pos.axis, pos.batch, plan, size(s[0], "B"), size(s[1], "H"), size(s[2], "n"),
                  a[3] == Py_True, rx.code, ry.code, ry.p, ry.st, stream_of(dev));
  });
}

// rope_encode(x, pos, plan address, k, idx, val)
PyObject* rope_encode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> long {
    const at::Tensor& x = tensor(a[0], "x");
    const int dev = x.get_device();
    const auto s = heads(x, "x");
    const sfa_rope_plan* plan = plan_of(a[2]);
    plan_d(plan, s[3]);
    const Positions pos(a[1], plan->naxes, s[0], s[2], dev);
    const Rows rx(a[0], "x", dev, {s[0], s[1], s[2], s[3]});
    const int k = small(a[3], "k");
    const at::Tensor &idx = on(a[4], "idx", dev), &val = on(a[5], "val", dev);
    const int it = idx_code(idx, "idx"), vt = val_code(val, "val", true);
    if (!is_shape(idx, {s[0], s[1], s[2], k}) || !is_shape(val, {s[0], s[1], s[2], k}))
      refuse(PyExc_ValueError, "idx and val must be [B, H, n, k]");
    void *ip = contiguous(idx, "idx"), *vp = contiguous(val, "val");
    if (s[0] == 0 || s[1] == 0 || s[2] == 0) return SFA_OK;
    const Current cur(dev);
    return c_rope_encode(rx.p, rx.st, pos.p, pos.axis, pos.batch, plan, size(s[0], "B"), size(s[1], "H"),
                         size(s[2], "n"), k, rx.code, ip, it, vp, vt, stream_of(dev));
  });
}

// rope_encode_bwd(idx, dval, pos, plan address, dx)
PyObject* rope_encode_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> long {
    const at::Tensor& idx = tensor(a[0], "idx");
    const int dev = idx.get_device();
    if (idx.dim() != 4) refuse(PyExc_ValueError, "idx must be [B, H, n, k]");
    const auto s = idx.sizes();
    const int it = idx_code(idx, "idx");
    void* ip = contiguous(idx, "idx");
    const sfa_rope_plan* plan = plan_of(a[3]);
    const float* g = (const float*)array(a[1], "dval", at::kFloat, dev, {s[0], s[1], s[2], s[3]});
    const Positions pos(a[2], plan->naxes, s[0], s[2], dev);
    const Rows dx(a[4], "dx", dev, {s[0], s[1], s[2], plan->d});
    if (s[0] == 0 || s[1] == 0 || s[2] == 0) return SFA_OK;
    const Current cur(dev);
    return c_rope_encode_bwd(ip, it, g, pos.p, pos.axis, pos.batch, plan, size(s[0], "B"), size(s[1], "H"),
                             size(s[2], "n"), size(s[3], "k"), dx.code, dx.p, dx.st, stream_of(dev));
  });
}

const int32_t* table_of(PyObject* o, int64_t B, int dev, int& max_pages) {
  const at::Tensor& t = on(o, "block_table", dev);
  if (t.dim() != 2 || t.size(0) != B) refuse(PyExc_ValueError, "block_table must be [B, max_pages]");
  max_pages = size(t.size(1), "max_pages");
  return (const int32_t*)array(o, "block_table", at::kInt, dev);
}

// page_tables(old_len, new_len, block_table, free_pages, free_in, page_size, free_out,
//             got, starts, slots, positions, ws)
PyObject* page_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> long {
    const at::Tensor& len = tensor(a[1], "new_len");
    const int dev = len.get_device();
    const int64_t B = len.numel();
    int max_pages = 0;
    int32_t* table = const_cast<int32_t*>(table_of(a[2], B, dev, max_pages));
    int32_t* free_pages = (int32_t*)array(a[3], "free_pages", at::kInt, dev);
    const int64_t rows = !none(a[9]) ? tensor(a[9], "slots").numel() : !none(a[10]) ? tensor(a[10], "pos").numel() : 0;
    const at::Tensor& ws = on(a[11], "ws", dev);
    void* wp = contiguous(ws, "ws");
    const int32_t* old_len = none(a[0]) ? nullptr : ints(a[0], "old_len", B, dev);
    const int32_t* new_len = ints(a[1], "new_len", B, dev);
    const int32_t* in = ints(a[4], "free_in", 1, dev);
    int32_t* out = ints(a[6], "free_out", 1, dev);
    int32_t* got = ints(a[7], "got", B, dev);
    int32_t* starts = ints(a[8], "starts", B + 1, dev);
    int32_t* slots = none(a[9]) ? nullptr : ints(a[9], "slots", rows, dev);
    int32_t* pos = none(a[10]) ? nullptr : ints(a[10], "pos", rows, dev);
    const Current cur(dev);
    return c_page_tables(old_len, new_len, size(B, "B"), table, max_pages, small(a[5], "page_size"), free_pages,
                         size(THPVariable_Unpack(a[3]).numel(), "free_pages"), in, out, got, starts, slots, pos,
                         size(rows, "slots"), wp, ws.nbytes(), stream_of(dev));
  });
}

// The five arrays of a 4-bit cache.
struct Cache {
  int dev;
  int64_t N, H, P, k, d;
  uint8_t *ci, *cv, *vc;
  float* cs;
  uint16_t* vs;
  explicit Cache(PyObject* const* a) {
    const at::Tensor& i = tensor(a[0], "kc_idx");
    dev = i.get_device();
    const at::Tensor& v = on(a[3], "v_cache", dev);
    if (i.dim() != 4 || v.dim() != 4)
      refuse(PyExc_ValueError, "kc_idx must be [pages, Hkv, page_size, k], v_cache [pages, Hkv, page_size, d / 2]");
    N = i.size(0); H = i.size(1); P = i.size(2); k = i.size(3); d = 2 * v.size(3);
    ci = (uint8_t*)array(a[0], "kc_idx", at::kByte, dev);
    cv = (uint8_t*)array(a[1], "kc_val", at::kByte, dev, {N, H, P, k / 2});
    cs = (float*)array(a[2], "kc_scale", at::kFloat, dev, {N, H, P});
    vc = (uint8_t*)array(a[3], "v_cache", at::kByte, dev, {N, H, P, d / 2});
    vs = (uint16_t*)array(a[4], "v_scale", at::kBFloat16, dev, {N, H, P, d / 32});
  }
};

// kv_append_q4(5 cache arrays, k_new, v_new, k, seq_len, n_new, block_table, slots,
//              k_idx, k_val, v_out)
PyObject* kv_append_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> long {
    const Cache c(a);
    const at::Tensor& kn = tensor(a[5], "k_new");
    const auto s = heads(kn, "k_new");
    const Rows kr(a[5], "k_new", c.dev, {s[0], s[1], s[2], s[3]}), vr(a[6], "v_new", c.dev, {s[0], s[1], s[2], s[3]});
    const int64_t B = s[0], H = s[1], T = s[2], d = s[3];
    if (c.H != H || c.k != integer(a[7], "k") || c.d != d)
      refuse(PyExc_ValueError, "the cache's heads, k or d are not those of k_new");
    const int32_t *slots = nullptr, *n_new = nullptr, *table = nullptr;
    int32_t* len = nullptr;
    int max_pages = 0;
    if (!none(a[11])) {
      if (!none(a[8]) || !none(a[9]) || !none(a[10]))
        refuse(PyExc_ValueError, "slots say where every token goes: give no seq_len, n_new or block_table");
      slots = ints(a[11], "slots", B * T, c.dev);
    } else {
      len = ints(a[8], "seq_len", B, c.dev);
      if (!none(a[9])) n_new = ints(a[9], "n_new", B, c.dev);
      if (!none(a[10])) table = table_of(a[10], B, c.dev, max_pages);
      else if (c.N != B) refuse(PyExc_ValueError, "a contiguous cache holds B sequences");
    }
    int16_t* ki = none(a[12]) ? nullptr : (int16_t*)array(a[12], "k_idx", at::kShort, c.dev, {B, H, T, c.k});
    float* kv = none(a[13]) ? nullptr : (float*)array(a[13], "k_val", at::kFloat, c.dev, {B, H, T, c.k});
    uint16_t* vo = none(a[14]) ? nullptr : (uint16_t*)array(a[14], "v_out", at::kBFloat16, c.dev, {B, H, T, d});
    const int64_t st[6] = {kr.st[0], kr.st[1], kr.st[2], vr.st[0], vr.st[1], vr.st[2]};
    const Current cur(c.dev);
    return c_kv_append_q4(kr.p, vr.p, st, slots, n_new, len, size(B, "B"), size(H, "Hkv"), size(T, "T"), size(d, "d"),
                          size(c.k, "k"), table, max_pages, size(c.P, "page_size"), size(c.N, "pages"), c.ci, c.cv,
                          c.cs, c.vc, c.vs, ki, kv, vo, kr.code, vr.code, stream_of(c.dev));
  });
}

// attn_decode_q4(5 cache arrays, block_table, seq_len, q, q_idx, q_val, scale or None, o,
//                lse, ws, window, n_global)
PyObject* attn_decode_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&]() -> long {
    const Cache c(a);
    const float* q = nullptr;
    void *qi = nullptr, *qv = nullptr;
    int qit = 0, qvt = 0;
    int64_t B, Hq;
    if (!none(a[7])) {
      if (!none(a[8]) || !none(a[9])) refuse(PyExc_ValueError, "give either q or (q_idx, q_val)");
      q = (const float*)array(a[7], "q", at::kFloat, c.dev);
      const at::Tensor& t = THPVariable_Unpack(a[7]);
      if (t.dim() != 3 || t.size(2) != c.d) refuse(PyExc_ValueError, "q must be [B, Hq, d]");
      B = t.size(0); Hq = t.size(1);
    } else {
      const at::Tensor &ti = on(a[8], "q_idx", c.dev), &tv = on(a[9], "q_val", c.dev);
      qit = idx_code(ti, "q_idx");
      qvt = val_code(tv, "q_val", true);
      if (ti.dim() != 3 || ti.size(2) != c.k || ti.sizes() != tv.sizes())
        refuse(PyExc_ValueError, "q codes must be [B, Hq, k]");
      B = ti.size(0); Hq = ti.size(1);
      qi = contiguous(ti, "q_idx");
      qv = contiguous(tv, "q_val");
    }
    const int32_t* table = nullptr;
    int max_pages = 0;
    if (!none(a[5])) table = table_of(a[5], B, c.dev, max_pages);
    else if (c.N != B) refuse(PyExc_ValueError, "a contiguous cache holds B sequences");
    const int32_t* len = none(a[6]) ? nullptr : ints(a[6], "seq_len", B, c.dev);
    double scale = none(a[10]) ? 1.0 / std::sqrt((double)c.d) : PyFloat_AsDouble(a[10]);
    if (scale == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      refuse(PyExc_TypeError, "scale must be a number");
    }
    const at::Tensor& o = on(a[11], "o", c.dev);
    const int ot = val_code(o, "o", false);
    if (!is_shape(o, {B, Hq, c.d})) refuse(PyExc_ValueError, "o must be [B, Hq, d]");
    void* op = contiguous(o, "o");
    float* lse = nullptr;
    if (!none(a[12])) {
      lse = (float*)array(a[12], "lse", at::kFloat, c.dev);
      if (THPVariable_Unpack(a[12]).numel() != B * Hq) refuse(PyExc_ValueError, "lse must hold B * Hq entries");
    }
    const at::Tensor& ws = on(a[13], "ws", c.dev);
    void* wp = contiguous(ws, "ws");
    const Current cur(c.dev);
    return c_attn_decode_q4(q, qi, qv, c.ci, c.cv, c.cs, c.vc, c.vs, table, max_pages, size(c.P, "page_size"),
                            size(c.N, "pages"), len, size(B, "B"), size(Hq, "Hq"), size(c.H, "Hkv"), size(c.d, "d"),
                            size(c.k, "k"), (float)scale, small(a[14], "window"), small(a[15], "n_global"), qit, qvt,
                            ot, op, lse, wp, ws.nbytes(), stream_of(c.dev));
  });
}

// bind(addresses of the six entry points, in the order below; torch's stream function)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  c_rope = (decltype(c_rope))PyLong_AsVoidPtr(a[0]);
  c_rope_encode = (decltype(c_rope_encode))PyLong_AsVoidPtr(a[1]);
  c_rope_encode_bwd = (decltype(c_rope_encode_bwd))PyLong_AsVoidPtr(a[2]);
  c_page_tables = (decltype(c_page_tables))PyLong_AsVoidPtr(a[3]);
  c_kv_append_q4 = (decltype(c_kv_append_q4))PyLong_AsVoidPtr(a[4]);
  c_attn_decode_q4 = (decltype(c_attn_decode_q4))PyLong_AsVoidPtr(a[5]);
  if (PyErr_Occurred()) return nullptr;
  Py_INCREF(a[6]);
  Py_XSETREF(raw_stream, a[6]);
  Py_RETURN_NONE;
}

#define SFA_METHOD(f) {#f, (PyCFunction)(void*)f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SFA_METHOD(bind), SFA_METHOD(rope), SFA_METHOD(rope_encode), SFA_METHOD(rope_encode_bwd),
                         SFA_METHOD(page_tables), SFA_METHOD(kv_append_q4), SFA_METHOD(attn_decode_q4),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
