// Python entry of the decoding-step calls: argument checks and marshalling only, in C++.  A decoding
// step calls them once a layer and token; the same checks in Python took longer than the kernels of
// a small step (22 us around a kernel of 3.5).  Every function takes the context's capsule first, raises ValueError
// where a tensor does not fit the context, and returns the status of the C call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <cstring>
#include <new>
#include <string>

#include "../../include/gto.h"

namespace {

struct Raised {};  // a Python exception is set

struct Ctx {
  gto_decode_ctx* handle;
  gto_decode_config cfg;
  int device;
  at::ScalarType kv, logit;
};

at::ScalarType scalar(int code) {
  return code == GTO_F32 ? at::kFloat : code == GTO_BF16 ? at::kBFloat16 : at::kHalf;
}

constexpr const char* kCapsule = "gto_decode_ctx";

const Ctx& context(PyObject* o) {
  Ctx* c = static_cast<Ctx*>(PyCapsule_GetPointer(o, kCapsule));
  if (!c) throw Raised{};
  return *c;
}

template <typename S>
std::string text(const S& sizes) {
  std::string s = "[";
  for (size_t i = 0; i < sizes.size(); ++i) s += (i ? ", " : "") + std::to_string(sizes[i]);
  return s + "]";
}

[[noreturn]] void refuse(const Ctx& c, const char* name, at::ScalarType dtype, const std::string& shape, const at::Tensor& t) {
  PyErr_Format(PyExc_ValueError, "%s: expected %s %s on cuda:%d, got %s %s strides %s on %s", name, c10::toString(dtype),
               shape.c_str(), c.device, c10::toString(t.scalar_type()), text(t.sizes()).c_str(), text(t.strides()).c_str(),
               t.device().str().c_str());
  throw Raised{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor, got %s", name, Py_TYPE(o)->tp_name);
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}

bool here(const Ctx& c, const at::Tensor& t, at::ScalarType dtype) {
  return t.scalar_type() == dtype && t.is_cuda() && t.get_device() == c.device;
}

// Pointer of a dense tensor of that type and shape.
template <size_t N>
void* dense(const Ctx& c, PyObject* o, const char* name, at::ScalarType dtype, const std::array<int64_t, N>& shape) {
  const at::Tensor& t = tensor(o, name);
  if (!here(c, t, dtype) || t.sizes() != at::IntArrayRef(shape) || !t.is_contiguous())
    refuse(c, name, dtype, "contiguous " + text(shape), t);
  return t.data_ptr();
}

template <size_t N>
void* maybe(const Ctx& c, PyObject* o, const char* name, at::ScalarType dtype, const std::array<int64_t, N>& shape) {
  return !o || o == Py_None ? nullptr : dense(c, o, name, dtype, shape);
}

struct Rows {
  void* p = nullptr;
  int64_t stride = 0, T = 0;
};
// [T, heads, head_dim] with dense heads.
Rows rows(const Ctx& c, PyObject* o, const char* name, int64_t heads) {
  const at::Tensor& t = tensor(o, name);
  const int64_t dh = c.cfg.head_dim;
  if (!here(c, t, c.kv) || t.dim() != 3 || t.size(1) != heads || t.size(2) != dh ||
      (t.size(0) > 0 && (t.stride(2) != 1 || (heads > 1 && t.stride(1) != dh))))
    refuse(c, name, c.kv, "[T, " + std::to_string(heads) + ", " + std::to_string(dh) + "] with dense heads", t);
  return Rows{t.data_ptr(), t.size(0) > 1 ? t.stride(0) : heads * dh, t.size(0)};
}

PyObject* key(const char* name) { return PyUnicode_InternFromString(name); }

// Entry of a dict; null where there is none.
PyObject* get(PyObject* dict, PyObject* name) {
  PyObject* o = PyDict_GetItemWithError(dict, name);
  if (!o && PyErr_Occurred()) throw Raised{};
  return o;
}
PyObject* need(PyObject* dict, PyObject* name) {
  PyObject* o = get(dict, name);
  if (!o) {
    PyErr_SetObject(PyExc_KeyError, name);
    throw Raised{};
  }
  return o;
}

int64_t first_size(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() < 1) {
    PyErr_Format(PyExc_ValueError, "%s: expected a vector", name);
    throw Raised{};
  }
  return t.size(0);
}

int32_t small(int64_t n, const char* name) {
  if (n > INT32_MAX || n < 0) {
    PyErr_Format(PyExc_ValueError, "%s: %lld rows", name, static_cast<long long>(n));
    throw Raised{};
  }
  return static_cast<int32_t>(n);
}

using I1 = std::array<int64_t, 1>;
using I2 = std::array<int64_t, 2>;
using I3 = std::array<int64_t, 3>;

gto_batch batch_of(const Ctx& c, PyObject* dict, int64_t T) {
  static PyObject *q_start = key("q_start"), *kv_len = key("kv_len"), *page_table = key("page_table"),
                  *n_nodes = key("n_nodes"), *node_mask = key("node_mask"), *node_depth = key("node_depth");
  if (!PyDict_Check(dict)) {
    PyErr_SetString(PyExc_ValueError, "batch: expected a dict");
    throw Raised{};
  }
  const int64_t S = first_size(need(dict, kv_len), "kv_len"), g = c.cfg.g;
  gto_batch b{};
  b.S = small(S, "kv_len");
  b.T = small(T, "tokens");
  b.q_start = static_cast<const int32_t*>(dense(c, need(dict, q_start), "q_start", at::kInt, I1{S + 1}));
  b.kv_len = static_cast<const int32_t*>(dense(c, need(dict, kv_len), "kv_len", at::kInt, I1{S}));
  b.page_table = static_cast<const int32_t*>(dense(c, need(dict, page_table), "page_table", at::kInt, I2{S, c.cfg.max_pages}));
  b.n_nodes = static_cast<const int32_t*>(maybe(c, get(dict, n_nodes), "n_nodes", at::kInt, I1{S}));
  b.node_mask = static_cast<const uint64_t*>(maybe(c, get(dict, node_mask), "node_mask", at::kLong, I3{S, g, (g + 63) / 64}));
  b.node_depth = static_cast<const int32_t*>(maybe(c, get(dict, node_depth), "node_depth", at::kInt, I2{S, g}));
  return b;
}

// [n_pages, page_size, n_kv_heads, head_dim] with dense heads, with `layers` also [n_layers, ...].
gto_kv_cache cache_of(const Ctx& c, PyObject* ko, PyObject* vo, bool layers) {
  const at::Tensor &k = tensor(ko, "k_cache"), &v = tensor(vo, "v_cache");
  const std::array<int64_t, 4> pool{c.cfg.n_pages, c.cfg.page_size, c.cfg.n_kv_heads, c.cfg.head_dim};
  const std::string want = std::string(layers ? "[n_layers, ]" : "") + text(pool) + " with dense heads";
  const bool deep = layers && k.dim() == 5;
  if (!here(c, k, c.kv) || (deep ? k.sizes().slice(1) : k.sizes()) != at::IntArrayRef(pool) || k.stride(-1) != 1)
    refuse(c, "k_cache", c.kv, want, k);
  if (!here(c, v, c.kv) || v.sizes() != k.sizes() || v.stride(-1) != 1) refuse(c, "v_cache", c.kv, want, v);
  const int o = deep ? 1 : 0;
  return gto_kv_cache{k.data_ptr(), v.data_ptr(), k.stride(o), k.stride(o + 1), k.stride(o + 2), deep ? k.stride(0) : 0,
                      v.stride(o), v.stride(o + 1), v.stride(o + 2), deep ? v.stride(0) : 0,
                      deep ? small(k.size(0), "k_cache") : 1};
}

gto_verdict verdict_of(const Ctx& c, PyObject* dict, int64_t S) {
  static PyObject *accept_len = key("accept_len"), *path_node = key("path_node"), *token = key("token");
  if (!PyDict_Check(dict)) {
    PyErr_SetString(PyExc_ValueError, "verdict: expected a dict");
    throw Raised{};
  }
  return gto_verdict{static_cast<int32_t*>(dense(c, need(dict, accept_len), "accept_len", at::kInt, I1{S})),
                     static_cast<int32_t*>(dense(c, need(dict, path_node), "path_node", at::kInt, I2{S, c.cfg.D})),
                     static_cast<int32_t*>(dense(c, need(dict, token), "token", at::kInt, I2{S, c.cfg.D + 1}))};
}

void* stream_of(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Raised{};
  return p;
}

// Runs a call; a Python error or a C++ exception becomes a Python exception.
template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return nullptr;
  }
  try {
    return PyLong_FromLong(f());
  } catch (const Raised&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
    return nullptr;
  }
}

// (ctx, batch, q, k, v, q_out, k_cache, v_cache, inv_freq, q_norm, k_norm, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> long {
    const Ctx& c = context(a[0]);
    const int64_t hq = c.cfg.n_q_heads, hkv = c.cfg.n_kv_heads, dh = c.cfg.head_dim;
    const Rows k = rows(c, a[3], "k", hkv), v = rows(c, a[4], "v", hkv);
    Rows q;
    q.T = k.T;
    if (a[2] != Py_None) q = rows(c, a[2], "q", hq);
    if (v.T != k.T || q.T != k.T) {
      PyErr_SetString(PyExc_ValueError, "q, k and v must have the same number of tokens");
      throw Raised{};
    }
    void* q_out = maybe(c, a[5], "q_out", c.kv, I3{k.T, hq, dh});
    const gto_kv_cache cache = cache_of(c, a[6], a[7], false);
    const void* f = maybe(c, a[8], "inv_freq", at::kDouble, I1{c.cfg.rope_dims / 2});
    const void* qn = maybe(c, a[9], "q_norm", c.kv, I1{dh});
    const void* kn = maybe(c, a[10], "k_norm", c.kv, I1{dh});
    const gto_batch b = batch_of(c, a[1], k.T);
    return gto_kv_append(c.handle, &b, &cache, q.p, q.stride, k.p, k.stride, v.p, v.stride, q_out,
                         static_cast<const double*>(f), qn, kn, stream_of(a[11]));
  });
}

// (ctx, batch, q, k_cache, v_cache, out, lse, stream)
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> long {
    const Ctx& c = context(a[0]);
    const Rows q = rows(c, a[2], "q", c.cfg.n_q_heads);
    void* out = dense(c, a[5], "out", c.kv, I3{q.T, c.cfg.n_q_heads, c.cfg.head_dim});
    void* lse = maybe(c, a[6], "lse", at::kFloat, I2{q.T, c.cfg.n_q_heads});
    const gto_kv_cache cache = cache_of(c, a[3], a[4], false);
    const gto_batch b = batch_of(c, a[1], q.T);
    return gto_tree_attention(c.handle, &b, &cache, q.p, q.stride, out, static_cast<float*>(lse), stream_of(a[7]));
  });
}

// (ctx, tree, target, d2t, temperature, u_node, u_bonus, verdict, stream)
PyObject* verify_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> long {
    static PyObject *node_token = key("node_token"), *node_parent = key("node_parent"), *node_depth = key("node_depth"),
                    *node_slot = key("node_slot"), *n_nodes = key("n_nodes");
    const Ctx& c = context(a[0]);
    const int64_t S = first_size(a[4], "temperature"), g = c.cfg.g;
    const bool ctx_rows = (c.cfg.flags & GTO_DECODE_CONTEXT_ROWS) != 0;
    gto_draft_tree t{};
    t.S = small(S, "temperature");
    if (g > 0) {
      if (!PyDict_Check(a[1])) {
        PyErr_SetString(PyExc_ValueError, "tree: expected a dict");
        throw Raised{};
      }
      const auto node = [&](PyObject* name, const char* s) {
        return static_cast<const int32_t*>(dense(c, need(a[1], name), s, at::kInt, I2{S, g}));
      };
      t.node_token = node(node_token, "node_token");
      t.node_parent = node(node_parent, "node_parent");
      if (ctx_rows) {
        t.node_depth = node(node_depth, "node_depth");
        t.node_slot = node(node_slot, "node_slot");
      }
      t.n_nodes = static_cast<const int32_t*>(maybe(c, get(a[1], n_nodes), "n_nodes", at::kInt, I1{S}));
    }
    const int64_t R = ctx_rows ? 1 + static_cast<int64_t>(c.cfg.D - 1) * c.cfg.k : 1 + g;
    const void* target = dense(c, a[2], "target", c.logit, I3{S, R, c.cfg.V_target});
    const void* d2t = maybe(c, a[3], "d2t", at::kInt, I1{c.cfg.V_draft});
    const void* temperature = dense(c, a[4], "temperature", at::kFloat, I1{S});
    const void* u_node = maybe(c, a[5], "u_node", at::kFloat, I2{S, g});
    const void* u_bonus = dense(c, a[6], "u_bonus", at::kFloat, I1{S});
    const gto_verdict out = verdict_of(c, a[7], S);
    return gto_verify_tree(c.handle, &t, target, static_cast<const int32_t*>(d2t), static_cast<const float*>(temperature),
                           static_cast<const float*>(u_node), static_cast<const float*>(u_bonus), &out, stream_of(a[8]));
  });
}

// (ctx, batch, verdict, k_cache, v_cache, kv_len_out, tokens, stream); tokens None: as many as the context takes
PyObject* kv_commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> long {
    const Ctx& c = context(a[0]);
    int64_t T = c.cfg.T;
    if (a[6] != Py_None) {
      T = PyLong_AsLongLong(a[6]);
      if (T == -1 && PyErr_Occurred()) throw Raised{};
    }
    const gto_batch b = batch_of(c, a[1], T);
    const gto_verdict v = verdict_of(c, a[2], b.S);
    const gto_kv_cache cache = cache_of(c, a[3], a[4], true);
    void* out = dense(c, a[5], "kv_len_out", at::kInt, I1{b.S});
    return gto_kv_commit(c.handle, &b, &v, &cache, static_cast<int32_t*>(out), stream_of(a[7]));
  });
}

// (handle, bytes of gto_decode_config, device) -> capsule; it does not own the handle
PyObject* make(PyObject*, PyObject* const* a, Py_ssize_t n) {
  char* bytes = nullptr;
  Py_ssize_t size = 0;
  if (n != 3 || PyBytes_AsStringAndSize(a[1], &bytes, &size) != 0 || size != sizeof(gto_decode_config)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "expected a handle, a configuration and a device");
    return nullptr;
  }
  void* handle = PyLong_AsVoidPtr(a[0]);
  const long device = PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  Ctx* c = new (std::nothrow) Ctx();
  if (!c) return PyErr_NoMemory();
  c->handle = static_cast<gto_decode_ctx*>(handle);
  std::memcpy(&c->cfg, bytes, sizeof(c->cfg));
  c->device = static_cast<int>(device);
  c->kv = scalar(c->cfg.kv_dtype);
  c->logit = scalar(c->cfg.logit_dtype);
  PyObject* o = PyCapsule_New(c, kCapsule, [](PyObject* p) {
    delete static_cast<Ctx*>(PyCapsule_GetPointer(p, kCapsule));
  });
  if (!o) delete c;
  return o;
}

#define GTO_FN(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {GTO_FN(make),        GTO_FN(kv_append), GTO_FN(tree_attention),
                          GTO_FN(verify_tree), GTO_FN(kv_commit), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_gto_decode", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gto_decode() {
  PyObject* m = PyModule_Create(&kModule);
  if (m && PyModule_AddStringConstant(m, "built_for", GTO_BUILT_FOR) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
