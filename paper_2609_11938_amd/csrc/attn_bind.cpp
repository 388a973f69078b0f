// Python binding of the attention operators: checks torch tensors, writes the C
// ABI's structs and calls it. Only marshalling, as in the ctypes binding of the
// join, but here a call is a few microseconds and reading a dozen tensors'
// types, shapes, strides and addresses from Python would be most of it (8.6 us
// an append against 3.8 us for the launch alone).
//
// Every function takes its arguments by position, checked by attn.py's
// signatures, and goes to the current stream of its tensors' device. A function
// with a workspace returns the bytes it needs, having done nothing,
// when `ws` is None or smaller; otherwise None.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/opattr_attn.h"

namespace {

struct TypeError : std::runtime_error {
  using runtime_error::runtime_error;
};
struct ValueError : std::runtime_error {
  using runtime_error::runtime_error;
};

std::string shape_of(c10::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) throw TypeError(std::string(name) + ": a tensor is wanted");
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.is_cuda()) throw TypeError(std::string(name) + ": device tensors are taken");
  return t;
}

// Autograd does not see the calls: with it on, inputs that require a gradient would
// lose it without a word.
void no_gradient(std::initializer_list<PyObject *> inputs, const char *name) {
  if (!c10::GradMode::is_enabled()) return;
  for (PyObject *o : inputs)
    if (tensor(o, name).requires_grad())
      throw std::runtime_error(std::string(name) +
                               ": an input requires a gradient, which the call does not record; "
                               "detach it or call under torch.no_grad()");
}

int dtype_of(const at::Tensor &t) {
  if (t.scalar_type() == at::kBFloat16) return OPATTR_BF16;
  if (t.scalar_type() == at::kHalf) return OPATTR_F16;
  throw TypeError("bfloat16 or float16 tensors are taken");
}

void alike(const at::Tensor &t, const at::Tensor &like, const char *name) {
  if (t.scalar_type() != like.scalar_type() || t.get_device() != like.get_device())
    throw TypeError(std::string(name) + ": not of the type and device of the others");
}

void want_shape(const at::Tensor &t, c10::IntArrayRef shape, const char *name) {
  if (t.sizes() != shape)
    throw ValueError(std::string(name) + ": shape " + shape_of(t.sizes()) + ", expected " +
                     shape_of(shape));
}

// A [tokens, heads, head_dim] tensor of like's type. The stride of a single row
// or head says nothing.
opattr_rows rows(PyObject *o, const at::Tensor &like, int64_t n, int64_t heads, int64_t d,
                 const char *name) {
  const at::Tensor &t = tensor(o, name);
  alike(t, like, name);
  want_shape(t, {n, heads, d}, name);
  if (t.stride(2) != 1 && d > 1)
    throw ValueError(std::string(name) + ": the last dimension's values must lie side by side");
  return {t.data_ptr(), n > 1 ? t.stride(0) : d, heads > 1 ? t.stride(1) : 0};
}

// The address of a contiguous array.
void *array(PyObject *o, at::ScalarType type, const at::Tensor &like, c10::IntArrayRef shape,
            const char *name) {
  const at::Tensor &t = tensor(o, name);
  if (t.scalar_type() != type || t.get_device() != like.get_device() || !t.is_contiguous())
    throw TypeError(std::string(name) + ": a contiguous " +
                    (type == at::kInt ? "int32" : "float32") +
                    " tensor on the others' device is wanted");
  want_shape(t, shape, name);
  return t.data_ptr();
}
int32_t *ints(PyObject *o, const at::Tensor &like, c10::IntArrayRef shape, const char *name) {
  return static_cast<int32_t *>(array(o, at::kInt, like, shape, name));
}
float *floats(PyObject *o, const at::Tensor &like, c10::IntArrayRef shape, const char *name) {
  return static_cast<float *>(array(o, at::kFloat, like, shape, name));
}

opattr_diag *diag_of(PyObject *o, const at::Tensor &like) {
  if (o == Py_None) return nullptr;
  const at::Tensor &t = tensor(o, "diag");
  if (t.get_device() != like.get_device()) throw TypeError("diag: not on the others' device");
  if (t.nbytes() < sizeof(opattr_diag)) throw ValueError("diag: not a diag record");
  return static_cast<opattr_diag *>(t.data_ptr());
}

int64_t integer(PyObject *o) {
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw std::exception();
  return x;
}

// The current stream of the tensor's device.
void *stream_of(const at::Tensor &on) {
  return c10::hip::getCurrentHIPStream(on.get_device()).stream();
}

int32_t small(int64_t x) {
  if (x > INT32_MAX) throw ValueError("a size past 2^31");
  return static_cast<int32_t>(x);
}

// None, or the bytes wanted, or the call's error.
PyObject *done(int rc, const char *name) {
  if (rc == OPATTR_OK) Py_RETURN_NONE;
  throw std::runtime_error(std::string(name) + ": " + opattr_strerror(rc) + " (" +
                           std::to_string(rc) + ")");
}

// A workspace. One that a call on another stream allocated is that stream's memory:
// let go, it stays until the current stream has passed this call too (on its own
// stream the allocator notes nothing).
struct Work {
  void *p = nullptr;
  size_t bytes = 0;
  Work(PyObject *o, const at::Tensor &like) {
    if (o == Py_None) return;
    const at::Tensor &t = tensor(o, "ws");
    if (t.get_device() != like.get_device() || !t.is_contiguous())
      throw TypeError("ws: a contiguous tensor on the others' device is wanted");
    p = t.data_ptr();
    bytes = t.nbytes();
    c10::hip::HIPCachingAllocator::recordStream(
        t.storage().data_ptr(), c10::hip::getCurrentHIPStream(like.get_device()));
  }
};

float scale_of(PyObject *o, int64_t d) {
  if (o == Py_None) return static_cast<float>(1.0 / std::sqrt(static_cast<double>(d)));
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw std::exception();
  return static_cast<float>(x);
}

opattr_attn_shape shape(const at::Tensor &q, PyObject *ko, PyObject *cu_q, PyObject *cu_k,
                        PyObject *causal, PyObject *scale) {
  const at::Tensor &k = tensor(ko, "k"), &cu = tensor(cu_q, "cu_q");
  if (q.dim() != 3 || k.dim() != 3 || cu.dim() != 1 || cu.size(0) < 1)
    throw ValueError("queries and keys are [tokens, heads, head_dim], offsets one more than "
                     "sequences");
  const int64_t n = cu.size(0);
  opattr_attn_shape a{};
  a.n_q = q.size(0);
  a.n_k = k.size(0);
  a.cu_q = ints(cu_q, q, {n}, "cu_q");
  a.cu_k = cu_k == Py_None ? a.cu_q : ints(cu_k, q, {n}, "cu_k");
  a.n_seqs = small(n - 1);
  a.n_heads = small(q.size(1));
  a.n_kv_heads = small(k.size(1));
  a.head_dim = small(q.size(2));
  a.dtype = dtype_of(q);
  const int c = PyObject_IsTrue(causal);
  if (c < 0) throw std::exception();
  a.causal = c;
  a.scale = scale_of(scale, a.head_dim);
  return a;
}

// q k v cu_q cu_k causal scale out lse diag
PyObject *attn_prompt(PyObject *const *o) {
  const at::Tensor &q = tensor(o[0], "q");
  const c10::DeviceGuard on(q.device());
  const opattr_attn_shape a = shape(q, o[1], o[3], o[4], o[5], o[6]);
  const int64_t h = a.n_heads, g = a.n_kv_heads, d = a.head_dim;
  const opattr_rows rq = rows(o[0], q, a.n_q, h, d, "q"), rk = rows(o[1], q, a.n_k, g, d, "k"),
                    rv = rows(o[2], q, a.n_k, g, d, "v"),
                    ro = rows(o[7], q, a.n_q, h, d, "out");
  no_gradient({o[0], o[1], o[2]}, "opattr_attn_prompt");
  return done(opattr_attn_prompt(&a, &rq, &rk, &rv, &ro, floats(o[8], q, {h, a.n_q}, "lse"),
                                 diag_of(o[9], q), stream_of(q)),
              "opattr_attn_prompt");
}

// dout q k v out lse cu_q cu_k causal scale dq dk dv ws diag
PyObject *attn_prompt_grad(PyObject *const *o) {
  const at::Tensor &q = tensor(o[1], "q");
  const c10::DeviceGuard on(q.device());
  const opattr_attn_shape a = shape(q, o[2], o[6], o[7], o[8], o[9]);
  const int64_t h = a.n_heads, g = a.n_kv_heads, d = a.head_dim;
  const opattr_rows rd = rows(o[0], q, a.n_q, h, d, "dout"), rq = rows(o[1], q, a.n_q, h, d, "q"),
                    rk = rows(o[2], q, a.n_k, g, d, "k"), rv = rows(o[3], q, a.n_k, g, d, "v"),
                    ro = rows(o[4], q, a.n_q, h, d, "out"),
                    sq = rows(o[10], q, a.n_q, h, d, "dq"),
                    sk = rows(o[11], q, a.n_k, g, d, "dk"),
                    sv = rows(o[12], q, a.n_k, g, d, "dv");
  const float *lse = floats(o[5], q, {h, a.n_q}, "lse");
  const Work ws(o[13], q);
  const size_t need = opattr_attn_prompt_grad_workspace_bytes(&a);
  if (need > ws.bytes) return PyLong_FromSize_t(need);
  return done(opattr_attn_prompt_grad(&a, &rd, &rq, &rk, &rv, &ro, lse, &sq, &sk, &sv,
                                      diag_of(o[14], q), ws.p, ws.bytes, stream_of(q)),
              "opattr_attn_prompt_grad");
}

opattr_kv_pages kv_pages(PyObject *ko, PyObject *vo, PyObject *to) {
  const at::Tensor &k = tensor(ko, "k_pages"), &v = tensor(vo, "v_pages"),
                   &t = tensor(to, "table");
  if (k.dim() != 4 || k.sizes() != v.sizes() || k.strides() != v.strides())
    throw ValueError("k_pages and v_pages are [pages, page_size, kv_heads, head_dim], alike in "
                     "shape and strides");
  alike(v, k, "v_pages");
  if (k.stride(3) != 1 && k.size(3) > 1)
    throw ValueError("k_pages: the last dimension's values must lie side by side");
  if (t.dim() != 2) throw ValueError("table is [sequences, entries]");
  opattr_kv_pages c{};
  c.k = k.data_ptr();
  c.v = v.data_ptr();
  c.page_stride = k.size(0) > 1 ? k.stride(0) : 0;
  c.token_stride = k.size(1) > 1 ? k.stride(1) : 0;
  c.head_stride = k.size(2) > 1 ? k.stride(2) : 0;
  c.n_pages = small(k.size(0));
  c.page_size = small(k.size(1));
  c.table = ints(to, k, {t.size(0), t.size(1)}, "table");
  c.n_seqs = small(t.size(0));
  c.table_stride = small(t.size(1));
  c.n_kv_heads = small(k.size(2));
  c.head_dim = small(k.size(3));
  c.dtype = dtype_of(k);
  return c;
}

// q k_pages v_pages table lens scale out lse ws diag
PyObject *attn_paged(PyObject *const *o) {
  const at::Tensor &q = tensor(o[0], "q");
  const c10::DeviceGuard on(q.device());
  const opattr_kv_pages c = kv_pages(o[1], o[2], o[3]);
  if (q.dim() != 3) throw ValueError("q is [sequences, heads, head_dim]");
  alike(q, THPVariable_Unpack(o[1]), "q");
  const int64_t b = c.n_seqs, h = q.size(1), d = c.head_dim;
  const opattr_rows rq = rows(o[0], q, b, h, d, "q"), ro = rows(o[6], q, b, h, d, "out");
  no_gradient({o[0], o[1], o[2]}, "opattr_attn_paged");
  const int32_t *lens = ints(o[4], q, {b}, "lens");
  float *lse = floats(o[7], q, {h, b}, "lse");
  const Work ws(o[8], q);
  const size_t need = opattr_attn_paged_workspace_bytes(&c, small(h));
  if (need > ws.bytes) return PyLong_FromSize_t(need);
  return done(opattr_attn_paged(&c, small(h), &rq, lens, scale_of(o[5], d), &ro, lse,
                                diag_of(o[9], q), ws.p, ws.bytes, stream_of(q)),
              "opattr_attn_paged");
}

// k_new v_new cu k_pages v_pages table lens lens_out diag
PyObject *kv_append(PyObject *const *o) {
  const at::Tensor &k = tensor(o[0], "k_new"), &cache = tensor(o[3], "k_pages");
  const c10::DeviceGuard on(cache.device());
  const opattr_kv_pages c = kv_pages(o[3], o[4], o[5]);
  const int64_t b = c.n_seqs, n = k.dim() ? k.size(0) : 0;
  const opattr_rows rk = rows(o[0], cache, n, c.n_kv_heads, c.head_dim, "k_new"),
                    rv = rows(o[1], cache, n, c.n_kv_heads, c.head_dim, "v_new");
  no_gradient({o[0], o[1]}, "opattr_kv_append");
  return done(opattr_kv_append(&c, n, ints(o[2], cache, {b + 1}, "cu"), &rk, &rv,
                               ints(o[6], cache, {b}, "lens"),
                               ints(o[7], cache, {b}, "lens_out"), diag_of(o[8], cache),
                               stream_of(cache)),
              "opattr_kv_append");
}

// A [planes, pages, ...] tensor whose pages lie in one piece each.
opattr_page_pool page_pool(const at::Tensor &t, int64_t page_size, PyObject *held) {
  if (t.dim() < 3) throw ValueError("pool is [planes, pages, ...]");
  int64_t each = 1;
  for (int64_t i = t.dim() - 1; i >= 2; --i) {
    if (t.size(i) > 1 && t.stride(i) != each)
      throw ValueError("pool: a page's values must lie side by side");
    each *= t.size(i);
  }
  const int64_t size = t.element_size();
  opattr_page_pool p{};
  p.data = t.data_ptr();
  p.plane_stride = t.size(0) > 1 ? t.stride(0) * size : 0;
  p.page_stride = (t.size(1) > 1 ? t.stride(1) : each) * size;
  p.n_planes = small(t.size(0));
  p.n_pages = small(t.size(1));
  p.page_bytes = small(each * size);
  p.page_size = small(page_size);
  p.held = held == Py_None ? nullptr : ints(held, t, {t.size(1)}, "held");
  return p;
}

// pool page_size table lens parent room held table_out lens_out refs ws diag
PyObject *pages_fork(PyObject *const *o) {
  const at::Tensor &pool = tensor(o[0], "pool"), &table = tensor(o[2], "table"),
                   &parent = tensor(o[4], "parent");
  if (table.dim() != 2 || parent.dim() != 1)
    throw ValueError("table is [rows, entries], parent [rows of the next table]");
  const c10::DeviceGuard on(pool.device());
  const opattr_page_pool p = page_pool(pool, integer(o[1]), o[6]);
  const int64_t rows = table.size(0), width = table.size(1), n = parent.size(0);
  const Work ws(o[10], pool);
  const size_t need =
      opattr_pages_fork_workspace_bytes(small(rows), small(n), small(width), p.n_pages);
  if (need > ws.bytes) return PyLong_FromSize_t(need);
  return done(
      opattr_pages_fork(&p, ints(o[2], pool, {rows, width}, "table"),
                        ints(o[3], pool, {rows}, "lens"), small(rows), small(width),
                        ints(o[4], pool, {n}, "parent"),
                        o[5] == Py_None ? nullptr : ints(o[5], pool, {n}, "room"), small(n),
                        ints(o[7], pool, {n, width}, "table_out"),
                        ints(o[8], pool, {n}, "lens_out"), ints(o[9], pool, {p.n_pages}, "refs"),
                        diag_of(o[11], pool), ws.p, ws.bytes, stream_of(pool)),
      "opattr_pages_fork");
}

// pool table held table_out moved live ws diag
PyObject *pages_compact(PyObject *const *o) {
  const at::Tensor &pool = tensor(o[0], "pool"), &table = tensor(o[1], "table");
  if (table.dim() != 2) throw ValueError("table is [rows, entries]");
  const c10::DeviceGuard on(pool.device());
  const opattr_page_pool p = page_pool(pool, 1, o[2]);
  const int64_t rows = table.size(0), width = table.size(1);
  const Work ws(o[6], pool);
  const size_t need = opattr_pages_compact_workspace_bytes(p.n_pages);
  if (need > ws.bytes) return PyLong_FromSize_t(need);
  return done(opattr_pages_compact(&p, ints(o[1], pool, {rows, width}, "table"), small(rows),
                                   small(width), ints(o[3], pool, {rows, width}, "table_out"),
                                   ints(o[4], pool, {p.n_pages}, "moved"),
                                   ints(o[5], pool, {1}, "live"), diag_of(o[7], pool), ws.p, ws.bytes,
                                   stream_of(pool)),
              "opattr_pages_compact");
}

// No C++ exception leaves a call.
template <PyObject *(*f)(PyObject *const *), int kArgs>
PyObject *guarded(PyObject *, PyObject *const *o, Py_ssize_t n) {
  if (n != kArgs) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return f(o);
  } catch (const TypeError &e) {
    PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const ValueError &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

template <PyObject *(*f)(PyObject *const *), int kArgs>
PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&guarded<f, kArgs>)),
          METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<attn_prompt, 10>("attn_prompt"),
                         method<attn_prompt_grad, 15>("attn_prompt_grad"),
                         method<attn_paged, 10>("attn_paged"),
                         method<kv_append, 9>("kv_append"),
                         method<pages_fork, 12>("pages_fork"),
                         method<pages_compact, 8>("pages_compact"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "attn_bind", nullptr, -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_attn_bind() { return PyModule_Create(&module_def); }
