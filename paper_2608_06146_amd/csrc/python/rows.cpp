// Python's calls of the rotary entry points and padoc_cache_copy_blocks, for
// layers of a decode step whose kernels are shorter than the call: the checks
// and the packing of a call take some 4 us more in Python than here (forward of 81
// rows 13.1 and 9.9 us a call, of which its launch 4.3; append 14.0 and 9.1,
// backward 22.0 and 15.1, block copy 6.0 and 3.2).
//
// Each function makes the call where its arguments are in order and the stream
// is the tensors' device's current one, and otherwise returns None: the Python
// function then checks them one by one and says what is wrong.  A status other
// than 0 comes back as an int.  The library is not linked: ctypes, which loads it
// on first use, hands over the addresses.
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "padoc_attn.h"

namespace {

using Fwd = padoc_status (*)(const padoc_rotary*, const padoc_rotary_fwd_args*, hipStream_t);
using Bwd = padoc_status (*)(const padoc_rotary*, const padoc_rotary_bwd_args*, void*, size_t, hipStream_t);
using BwdBytes = padoc_status (*)(const padoc_rotary*, int64_t, int32_t, int32_t, size_t*);
using Append = padoc_status (*)(const padoc_rotary*, const padoc_rotary_append_args*, hipStream_t);
using Copy = padoc_status (*)(const void*, const void*, int64_t, void*, void*, int64_t, const int32_t*, int64_t,
                              const int32_t*, int32_t, int32_t, padoc_dtype, hipStream_t);

struct Rows {
  PyObject_HEAD
  const padoc_rotary* handle;
  Fwd fwd;
  Bwd bwd;
  BwdBytes bwd_bytes;
  Append append;
  int64_t d, axes;
  at::ScalarType dtype;
};

struct Unfit {};  // the Python function's turn

void need(bool ok) {
  if (!ok) throw Unfit{};
}

const at::Tensor* tensor(PyObject* o) {
  if (o == Py_None) return nullptr;
  need(THPVariable_Check(o));
  return &THPVariable_Unpack(o);
}

// A call's device and stream: the current ones, of its first tensor.
struct Where {
  c10::Device device;
  hipStream_t stream;
  explicit Where(const at::Tensor& t) : device(t.device()) {
    need(t.is_cuda() && c10::hip::current_device() == device.index());
    stream = c10::hip::getCurrentHIPStream(device.index()).stream();
  }
};

// (What is written is no longer shared with a lazy clone: data_ptr.)
padoc_heads heads(const at::Tensor& t, const Rows* r, const Where& w, int64_t n, int64_t h, bool written = false) {
  need(t.device() == w.device && t.scalar_type() == r->dtype && t.dim() == 3 && t.size(0) == n && t.size(1) == h &&
       t.size(2) == r->d && t.stride(2) == 1);
  void* data = written ? t.data_ptr() : const_cast<void*>(t.const_data_ptr());
  return padoc_heads{data, t.stride(0), t.stride(1)};
}

const void* weight(const at::Tensor* t, const Rows* r, const Where& w) {
  if (!t) return nullptr;
  need(t->device() == w.device && t->scalar_type() == r->dtype && t->dim() == 1 && t->size(0) == r->d &&
       t->stride(0) == 1);
  return t->const_data_ptr();
}

const int32_t* positions(const at::Tensor* t, const Rows* r, const Where& w, int64_t n, int64_t* stride) {
  need(t && t->device() == w.device && t->scalar_type() == at::kInt);
  *stride = 0;
  if (t->dim() == 1) {
    need(r->axes == 1 && t->size(0) == n && (n <= 1 || t->stride(0) == 1));
  } else {
    need(t->dim() == 2 && t->size(0) == r->axes && t->size(1) == n && (n <= 1 || t->stride(1) == 1));
    if (r->axes > 1) *stride = t->stride(0);
  }
  return static_cast<const int32_t*>(t->const_data_ptr());
}

struct Caches {
  int64_t blocks, heads, d;
};
Caches caches(const at::Tensor& k, const at::Tensor& v, const Where& w) {
  need(k.device() == w.device && v.device() == w.device && k.scalar_type() == v.scalar_type() && k.is_contiguous() &&
       v.is_contiguous() && v.dim() == 4 && k.dim() == 5);
  const Caches c{v.size(0), v.size(1), v.size(2)};
  need(v.size(3) == 16 && k.size(0) == c.blocks && k.size(1) == c.heads && k.size(2) == c.d / 8 && k.size(3) == 16 &&
       k.size(4) == 8);
  return c;
}

const int32_t* pairs(const at::Tensor* t, const Where& w, int64_t n) {
  need(t && t->device() == w.device && t->scalar_type() == at::kInt && t->dim() == 2 && t->size(1) == 2 &&
       t->is_contiguous() && (n < 0 || t->size(0) == n));
  return static_cast<const int32_t*>(t->const_data_ptr());
}

// A new tensor, or the one given.
struct Out {
  at::Tensor made;
  PyObject* given = nullptr;
  padoc_heads at{};
  PyObject* take() {
    if (given) return Py_NewRef(given);
    return THPVariable_Wrap(std::move(made));
  }
};
Out out_rows(PyObject* given, const at::Tensor& like, const Rows* r, const Where& w, int64_t n, int64_t h) {
  Out o;
  if (given != Py_None) {
    o.given = given;
    o.at = heads(*tensor(given), r, w, n, h, /*written=*/true);
  } else {
    o.made = at::empty({n, h, r->d}, like.options());
    o.at = padoc_heads{o.made.data_ptr(), h * r->d, r->d};
  }
  return o;
}

template <class F>
PyObject* call(F f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const Unfit&) {
    Py_RETURN_NONE;
  }
  END_HANDLE_TH_ERRORS
}

template <class F>
padoc_status unlocked(F f) {
  Py_BEGIN_ALLOW_THREADS
  const padoc_status st = f();
  Py_BLOCK_THREADS
  return st;
  Py_UNBLOCK_THREADS
  Py_END_ALLOW_THREADS
}

int64_t heads_of(const at::Tensor* t) {
  need(t->dim() == 3);
  return t->size(1);
}

// fwd(q, k, positions, q_weight, k_weight, q_out, k_out) -> (q_out, k_out)
PyObject* rows_fwd(PyObject* self, PyObject* const* a, Py_ssize_t count) {
  return call([&]() -> PyObject* {
    need(count == 7);
    const Rows* r = reinterpret_cast<Rows*>(self);
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]);
    need(q || k);
    need((q ? *q : *k).dim() == 3);
    const Where w(q ? *q : *k);
    padoc_rotary_fwd_args p{};
    p.n_rows = (q ? *q : *k).size(0);
    Out qo, ko;
    if (q) {
      p.num_heads_q = (int32_t)heads_of(q);
      p.q = heads(*q, r, w, p.n_rows, p.num_heads_q);
    }
    if (k) {
      p.num_heads_kv = (int32_t)heads_of(k);
      p.k = heads(*k, r, w, p.n_rows, p.num_heads_kv);
    }
    p.pos = positions(tensor(a[2]), r, w, p.n_rows, &p.pos_stride);
    p.q_weight = weight(tensor(a[3]), r, w);
    p.k_weight = weight(tensor(a[4]), r, w);
    if (q) p.q_out = (qo = out_rows(a[5], *q, r, w, p.n_rows, p.num_heads_q)).at;
    if (k) p.k_out = (ko = out_rows(a[6], *k, r, w, p.n_rows, p.num_heads_kv)).at;
    const padoc_status st = unlocked([&] { return r->fwd(r->handle, &p, w.stream); });
    if (st != PADOC_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", q ? qo.take() : Py_NewRef(Py_None), k ? ko.take() : Py_NewRef(Py_None));
  });
}

// bwd(dq_out, dk_out, positions, q, k, q_weight, k_weight, dq, dk, weight_grads)
// -> (dq, dk, dq_weight, dk_weight)
PyObject* rows_bwd(PyObject* self, PyObject* const* a, Py_ssize_t count) {
  return call([&]() -> PyObject* {
    need(count == 10);
    const Rows* r = reinterpret_cast<Rows*>(self);
    const at::Tensor* g[2] = {tensor(a[0]), tensor(a[1])};
    need(g[0] || g[1]);
    const at::Tensor& like = g[0] ? *g[0] : *g[1];
    need(like.dim() == 3);
    const Where w(like);
    const int grads = PyObject_IsTrue(a[9]);
    if (grads < 0) return nullptr;
    const int64_t n = like.size(0);
    int64_t h[2] = {0, 0};
    padoc_heads in[2]{}, x[2]{}, to[2]{};
    const void* wt[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
      if (!g[i]) continue;
      h[i] = heads_of(g[i]);
      in[i] = heads(*g[i], r, w, n, h[i]);
      wt[i] = weight(tensor(a[5 + i]), r, w);
      if (wt[i]) {
        const at::Tensor* xi = tensor(a[3 + i]);
        need(xi);
        x[i] = heads(*xi, r, w, n, h[i]);
      }
    }
    padoc_rotary_bwd_args p{};
    p.n_rows = n;
    p.num_heads_q = (int32_t)h[0];
    p.num_heads_kv = (int32_t)h[1];
    p.pos = positions(tensor(a[2]), r, w, n, &p.pos_stride);
    Out out[2];
    at::Tensor dw[2], work;
    float* dwp[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
      if (!g[i]) continue;
      to[i] = (out[i] = out_rows(a[7 + i], *g[i], r, w, n, h[i])).at;
      if (wt[i] && grads) {
        dw[i] = at::empty({r->d}, like.options().dtype(at::kFloat));
        dwp[i] = dw[i].data_ptr<float>();
      }
    }
    p.q = x[0];
    p.k = x[1];
    p.dq_out = in[0];
    p.dk_out = in[1];
    p.dq = to[0];
    p.dk = to[1];
    p.q_weight = wt[0];
    p.k_weight = wt[1];
    p.dq_weight = dwp[0];
    p.dk_weight = dwp[1];
    size_t bytes = 0;
    if (dwp[0] || dwp[1]) {
      const padoc_status st = r->bwd_bytes(r->handle, n, p.num_heads_q, p.num_heads_kv, &bytes);
      if (st != PADOC_OK) return PyLong_FromLong(st);
      work = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));  // (512-byte aligned)
    }
    void* ws = bytes ? work.data_ptr() : nullptr;
    const padoc_status st = unlocked([&] { return r->bwd(r->handle, &p, ws, bytes, w.stream); });
    if (st != PADOC_OK) return PyLong_FromLong(st);
    PyObject* res[4];
    for (int i = 0; i < 2; ++i) {
      res[i] = g[i] ? out[i].take() : Py_NewRef(Py_None);
      res[2 + i] = dwp[i] ? THPVariable_Wrap(std::move(dw[i])) : Py_NewRef(Py_None);
    }
    return Py_BuildValue("(NNNN)", res[0], res[1], res[2], res[3]);
  });
}

// append(q, k, v, positions, slots, k_cache, v_cache, q_weight, k_weight,
// q_positions, q_out) -> (q_out,)
PyObject* rows_append(PyObject* self, PyObject* const* a, Py_ssize_t count) {
  return call([&]() -> PyObject* {
    need(count == 11);
    const Rows* r = reinterpret_cast<Rows*>(self);
    const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]);
    const at::Tensor *kc = tensor(a[5]), *vc = tensor(a[6]);
    need(k && v && kc && vc);
    const Where w(*k);
    padoc_rotary_append_args p{};
    p.n_new = k->size(0);
    p.num_heads_kv = (int32_t)heads_of(k);
    p.k = heads(*k, r, w, p.n_new, p.num_heads_kv);
    p.v = heads(*v, r, w, p.n_new, p.num_heads_kv);
    p.pos = positions(tensor(a[3]), r, w, p.n_new, &p.pos_stride);
    p.slots = pairs(tensor(a[4]), w, p.n_new);
    const Caches c = caches(*kc, *vc, w);
    need(kc->scalar_type() == r->dtype && c.heads == p.num_heads_kv && c.d == r->d);
    p.k_cache = kc->data_ptr();
    p.v_cache = vc->data_ptr();
    p.num_blocks = c.blocks;
    p.q_weight = weight(tensor(a[7]), r, w);
    p.k_weight = weight(tensor(a[8]), r, w);
    Out qo;
    if (q) {
      need(q->dim() == 3);
      p.n_q = q->size(0);
      p.num_heads_q = (int32_t)q->size(1);
      p.q = heads(*q, r, w, p.n_q, p.num_heads_q);
      if (a[9] != Py_None) p.q_pos = positions(tensor(a[9]), r, w, p.n_q, &p.q_pos_stride);
      p.q_out = (qo = out_rows(a[10], *q, r, w, p.n_q, p.num_heads_q)).at;
    }
    const padoc_status st = unlocked([&] { return r->append(r->handle, &p, w.stream); });
    if (st != PADOC_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(N)", q ? qo.take() : Py_NewRef(Py_None));
  });
}

// copy_blocks(function, k_cache, v_cache, pairs) -> 0
PyObject* rows_copy(PyObject*, PyObject* const* a, Py_ssize_t count) {
  return call([&]() -> PyObject* {
    need(count == 4);
    const Copy copy = reinterpret_cast<Copy>(PyLong_AsVoidPtr(a[0]));
    const at::Tensor *k = tensor(a[1]), *v = tensor(a[2]), *t = tensor(a[3]);
    need(copy && k && v && t);
    const Where w(*k);
    const Caches c = caches(*k, *v, w);
    need(k->scalar_type() == at::kBFloat16 || k->scalar_type() == at::kFloat);
    const int32_t* p = pairs(t, w, -1);
    const padoc_dtype dt = k->scalar_type() == at::kBFloat16 ? PADOC_BF16 : PADOC_F32;
    void *kp = k->data_ptr(), *vp = v->data_ptr();
    return PyLong_FromLong(unlocked([&] {
      return copy(kp, vp, c.blocks, kp, vp, c.blocks, p, t->size(0), nullptr, (int32_t)c.heads, (int32_t)c.d, dt,
                  w.stream);
    }));
  });
}

// Rows(handle, fwd, bwd, bwd_workspace_bytes, append, head_dim, n_axes, bf16)
PyObject* rows_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long handle, fwd, bwd, bytes, append;
  long long d, axes;
  int bf16;
  if (!PyArg_ParseTuple(args, "KKKKKLLp", &handle, &fwd, &bwd, &bytes, &append, &d, &axes, &bf16)) return nullptr;
  Rows* r = reinterpret_cast<Rows*>(type->tp_alloc(type, 0));
  if (!r) return nullptr;
  r->handle = reinterpret_cast<const padoc_rotary*>((uintptr_t)handle);
  r->fwd = reinterpret_cast<Fwd>((uintptr_t)fwd);
  r->bwd = reinterpret_cast<Bwd>((uintptr_t)bwd);
  r->bwd_bytes = reinterpret_cast<BwdBytes>((uintptr_t)bytes);
  r->append = reinterpret_cast<Append>((uintptr_t)append);
  r->d = d;
  r->axes = axes;
  r->dtype = bf16 ? at::kBFloat16 : at::kFloat;
  return reinterpret_cast<PyObject*>(r);
}

void rows_dealloc(PyObject* self) {
  PyTypeObject* type = Py_TYPE(self);
  type->tp_free(self);
  Py_DECREF(type);
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef kMethods[] = {{"fwd", fast(rows_fwd), METH_FASTCALL, nullptr},
                          {"bwd", fast(rows_bwd), METH_FASTCALL, nullptr},
                          {"append", fast(rows_append), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};

PyType_Slot kSlots[] = {{Py_tp_new, reinterpret_cast<void*>(rows_new)},
                        {Py_tp_dealloc, reinterpret_cast<void*>(rows_dealloc)},
                        {Py_tp_methods, kMethods},
                        {0, nullptr}};

PyType_Spec kSpec = {"paper_2608_06146_amd._rows.Rows", sizeof(Rows), 0, Py_TPFLAGS_DEFAULT, kSlots};

PyMethodDef kFunctions[] = {{"copy_blocks", fast(rows_copy), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, kFunctions, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows() {
  PyObject* m = PyModule_Create(&kModule);
  if (!m) return nullptr;
  PyObject* t = PyType_FromSpec(&kSpec);
  if (!t || PyModule_AddObject(m, "Rows", t) < 0) {
    Py_XDECREF(t);
    Py_DECREF(m);
    return nullptr;
  }
  if (PyModule_AddStringConstant(m, "torch_version", PADOC_TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
