// The short way into the library for calls whose work on the GPU takes a few
// microseconds: argument checks, the current stream and the C entry point in one native
// call.  binding.py asks here first; every function returns its result, or None where a
// check fails or anything is out of the ordinary, and binding.py then goes its own way,
// which does the same work and raises what is to be raised.  Nothing is computed, kept or
// decided here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/torch.h>

#include <initializer_list>

namespace {

using at::ScalarType;
constexpr int TV_OK = 0, TV_ERR_LAUNCH = -6;  // as in treeverify.h
constexpr ScalarType kF8 = ScalarType::Float8_e4m3fn, kBF16 = ScalarType::BFloat16,
                     kI32 = ScalarType::Int, kU8 = ScalarType::Byte;

// binding.py's: the current stream of a device, the current device, a stream's workspace
// for the attention, a capture's
PyObject *raw_stream, *current_device, *workspace, *capture_workspace;

struct Library {
  unsigned long long (*capture_id)(void*);
  size_t (*attention_ws)(int, int, int, int, int, int);
  int (*attention)(const void*, const void*, const void*, const void*, const void*, const void*, int, int,
                   int, const void*, const void*, const void*, const void*, void*, int, int, int, int, int,
                   float, void*, size_t, void*);
  int (*append)(const void*, const void*, const void*, void*, void*, void*, void*, const void*, int, int,
                int, void*, int, int, int, int, void*);
  int (*commit)(const void*, const void*, const void*, const void*, void*, void*, void*, void*, const void*,
                int, int, int, void*, int, int, int, int, int, void*);
  int (*reserve)(const void*, void*, const void*, void*, void*, int, int, int, int, void*);
  int (*fork)(const void*, const void*, int, void*, void*, void*, int, int, int, int, void* const*,
              const int64_t*, int, void*, void*, void*, void*);
  int (*free_)(const void*, int, void*, void*, void*, int, int, int, void*);
} lib;

// A call's tensors: all on one device, contiguous, of the type and shape asked for.
struct Tensors {
  int64_t device = -1;
  bool good = true;

  const at::Tensor* any(PyObject* o) {
    if (!THPVariable_Check(o)) {
      good = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous() || (device >= 0 && t.get_device() != device)) {
      good = false;
      return nullptr;
    }
    device = t.get_device();
    return &t;
  }
  // of `rank` axes, any sizes
  const at::Tensor* ranked(PyObject* o, ScalarType type, int64_t rank) {
    const at::Tensor* t = any(o);
    if (t && (t->scalar_type() != type || t->dim() != rank)) good = false;
    return good ? t : nullptr;
  }
  void* at(PyObject* o, ScalarType type, std::initializer_list<int64_t> sizes) {
    const at::Tensor* t = any(o);
    if (!t || t->scalar_type() != type || t->sizes() != c10::IntArrayRef(sizes)) {
      good = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  void* maybe(PyObject* o, ScalarType type, std::initializer_list<int64_t> sizes) {
    return o == Py_None ? nullptr : at(o, type, sizes);
  }
};

// The device's current stream; false if it is not the current device.
bool stream_of(int64_t device, void** stream) {
  PyObject* now = PyObject_CallNoArgs(current_device);
  if (!now) return false;
  const int64_t on = PyLong_AsLongLong(now);
  Py_DECREF(now);
  if (on != device) return false;
  PyObject* number = PyLong_FromLongLong(device);
  PyObject* s = PyObject_CallFunctionObjArgs(raw_stream, number, nullptr);
  Py_DECREF(number);
  if (!s) return false;
  *stream = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

// What binding.py will meet and raise again is cleared; an interrupt or exit that came in
// while a Python function was asked is not an error of the call, and goes on.
PyObject* none() {
  if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return nullptr;
  PyErr_Clear();
  Py_RETURN_NONE;
}

// A refused call is left to binding.py; one that the runtime rejected may have begun, and
// is not made again.
PyObject* refused(int rc) {
  if (rc != TV_ERR_LAUNCH) return none();
  PyErr_SetString(PyExc_RuntimeError, "TV_ERR_LAUNCH: the HIP runtime rejected a launch");
  return nullptr;
}

PyObject* done(int rc, PyObject* result) {
  if (rc != TV_OK) return refused(rc);
  Py_INCREF(result);
  return result;
}

// An 8-bit paged cache: pools, exponents and table, with num_blocks, block_size, max_blocks.
struct Cache {
  void *k, *v, *ke, *ve, *table;
  int64_t nb, bs, mb;
  Cache(Tensors& t, PyObject* const* a, PyObject* bt, int64_t B, int64_t Hkv, int64_t D) {
    const at::Tensor *p = t.ranked(a[0], kF8, 4), *b = t.ranked(bt, kI32, 2);
    if (!p || !b) return;
    nb = p->size(0);
    bs = p->size(2);
    mb = b->size(1);
    k = t.at(a[0], kF8, {nb, Hkv, bs, D});
    v = t.at(a[1], kF8, {nb, Hkv, bs, D});
    ke = t.at(a[2], kU8, {nb, Hkv, bs / 32});
    ve = t.at(a[3], kU8, {nb, Hkv, bs / 32});
    table = t.at(bt, kI32, {B, mb});
    t.good = t.good && nb < (1ll << 31) && bs < (1ll << 31) && mb < (1ll << 31) && mb * bs < (1ll << 31);
  }
};

bool small(std::initializer_list<int64_t> sizes) {
  for (const int64_t s : sizes)
    if (s >= (1ll << 31)) return false;
  return true;
}

// Runs f, which may throw what torch throws.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (...) {
    return none();
  }
}

// q, k_pool, v_pool, k_exp, v_exp, block_table, k_tree, v_tree, parent, out, kv_len, scale,
// workspace_tensor
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 13) return none();
    Tensors t;
    const at::Tensor *q = t.ranked(a[0], kBF16, 4), *kt = t.ranked(a[6], kBF16, 4);
    if (!q || !kt) return none();
    const int64_t B = q->size(0), N = q->size(1), Hq = q->size(2), D = q->size(3), Hkv = kt->size(2);
    const Cache c(t, a + 1, a[5], B, Hkv, D);
    void* ktp = t.at(a[6], kBF16, {B, N, Hkv, D});
    void* vtp = t.at(a[7], kBF16, {B, N, Hkv, D});
    void* parent = t.maybe(a[8], kI32, {B, N});
    void* out = t.at(a[9], kBF16, {B, N, Hq, D});
    void* len = t.maybe(a[10], kI32, {B});
    double scale = 0;
    if (a[11] != Py_None) scale = PyFloat_AsDouble(a[11]);
    void* stream;
    if (!t.good || PyErr_Occurred() || !small({B, N, Hq, D, Hkv}) || !stream_of(t.device, &stream))
      return none();
    const size_t need = lib.attention_ws((int)B, (int)N, (int)Hq, (int)Hkv, (int)D, (int)(c.mb * c.bs));
    if (need == 0) return none();
    PyObject* ws = a[12];
    PyObject* own = nullptr;
    if (ws == Py_None) {
      const unsigned long long capture = lib.capture_id(stream);
      PyObject* args[4] = {capture ? PyLong_FromUnsignedLongLong(capture) : PyUnicode_FromString("attn_fp8"),
                           PyLong_FromSize_t(need), PyObject_GetAttrString(a[0], "device"),
                           PyLong_FromVoidPtr(stream)};
      ws = own = PyObject_Vectorcall(capture ? capture_workspace : workspace, args, 4, nullptr);
      for (PyObject* o : args) Py_XDECREF(o);
    }
    if (!ws || !t.any(ws)) {
      Py_XDECREF(own);
      return none();
    }
    const at::Tensor& w = THPVariable_Unpack(ws);
    const size_t bytes = (size_t)w.nbytes();
    const int rc = lib.attention(q->data_ptr(), c.k, c.v, c.ke, c.ve, c.table, (int)c.bs, (int)c.mb,
                                 (int)c.nb, ktp, vtp, parent, len, out, (int)B, (int)N, (int)Hq, (int)Hkv,
                                 (int)D, (float)scale, w.data_ptr(), bytes, stream);
    Py_XDECREF(own);
    return done(rc, a[9]);
  });
}

// k_new, v_new, k_pool, v_pool, k_exp, v_exp, block_table, kv_len, n_new
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9) return none();
    Tensors t;
    const at::Tensor* k = t.ranked(a[0], kBF16, 4);
    if (!k) return none();
    const int64_t B = k->size(0), T = k->size(1), Hkv = k->size(2), D = k->size(3);
    void* v = t.at(a[1], kBF16, {B, T, Hkv, D});
    const Cache c(t, a + 2, a[6], B, Hkv, D);
    void* len = t.at(a[7], kI32, {B});
    void* rows = t.maybe(a[8], kI32, {B});
    void* stream;
    if (!t.good || !small({B, T, Hkv, D}) || !stream_of(t.device, &stream)) return none();
    return done(lib.append(k->data_ptr(), v, rows, c.k, c.v, c.ke, c.ve, c.table, (int)c.bs, (int)c.mb,
                           (int)c.nb, len, (int)B, (int)T, (int)Hkv, (int)D, stream),
                Py_True);
  });
}

// k_tree, v_tree, path, accept_len, k_pool, v_pool, k_exp, v_exp, block_table, kv_len
PyObject* commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10) return none();
    Tensors t;
    const at::Tensor *k = t.ranked(a[0], kBF16, 4), *path = t.ranked(a[2], kI32, 2);
    if (!k || !path) return none();
    const int64_t B = k->size(0), N = k->size(1), Hkv = k->size(2), D = k->size(3), P = path->size(1);
    void* v = t.at(a[1], kBF16, {B, N, Hkv, D});
    void* pp = t.at(a[2], kI32, {B, P});
    void* rows = t.at(a[3], kI32, {B});
    const Cache c(t, a + 4, a[8], B, Hkv, D);
    void* len = t.at(a[9], kI32, {B});
    void* stream;
    if (!t.good || !small({B, N, Hkv, D, P}) || !stream_of(t.device, &stream)) return none();
    return done(lib.commit(k->data_ptr(), v, pp, rows, c.k, c.v, c.ke, c.ve, c.table, (int)c.bs, (int)c.mb,
                           (int)c.nb, len, (int)B, (int)N, (int)Hkv, (int)D, (int)P, stream),
                Py_True);
  });
}

// Table, lengths and counts of the page calls.
struct Pages {
  void *table, *len, *ref;
  int64_t B, mb, nb;
  Pages(Tensors& t, PyObject* bt, PyObject* kv, PyObject* counts) {
    const at::Tensor *b = t.ranked(bt, kI32, 2), *r = t.ranked(counts, kI32, 1);
    if (!b || !r) return;
    B = b->size(0);
    mb = b->size(1);
    nb = r->size(0);
    table = b->data_ptr();
    ref = r->data_ptr();
    len = t.at(kv, kI32, {B});
    t.good = t.good && small({B, mb, nb});
  }
};

// n_rows, block_table, kv_len, ref_count, block_size
PyObject* reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5) return none();
    Tensors t;
    const Pages p(t, a[1], a[2], a[3]);
    if (!t.good) return none();
    void* rows = t.at(a[0], kI32, {p.B});
    const long bs = PyLong_AsLong(a[4]);
    void* stream;
    if (!t.good || PyErr_Occurred() || !small({bs}) || !stream_of(t.device, &stream)) return none();
    at::Tensor ok = at::empty({p.B}, THPVariable_Unpack(a[1]).options());
    const int rc = lib.reserve(rows, p.table, p.len, p.ref, ok.data_ptr(), (int)p.B, (int)p.mb, (int)bs,
                               (int)p.nb, stream);
    return rc == TV_OK ? THPVariable_Wrap(std::move(ok)) : refused(rc);
  });
}

// src, dst, block_table, kv_len, ref_count, block_size, pools
PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 7 || !PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) > 64) return none();
    Tensors t;
    const Pages p(t, a[2], a[3], a[4]);
    const at::Tensor* src = t.ranked(a[0], kI32, 1);
    if (!t.good) return none();
    const int64_t forks = src->size(0);
    void* dst = t.at(a[1], kI32, {forks});
    const long bs = PyLong_AsLong(a[5]);
    void* base[64];
    int64_t bytes[64];
    const int pools = (int)PyTuple_GET_SIZE(a[6]);
    for (int k = 0; k < pools; ++k) {
      const at::Tensor* x = t.any(PyTuple_GET_ITEM(a[6], k));
      if (!x || x->dim() < 1 || x->size(0) != p.nb || p.nb < 1) return none();
      base[k] = x->data_ptr();
      bytes[k] = (int64_t)x->nbytes() / p.nb;
    }
    void* stream;
    if (!t.good || PyErr_Occurred() || !small({bs, forks}) || !stream_of(t.device, &stream)) return none();
    const at::Tensor said = at::empty({3, forks}, src->options());
    int32_t* o = said.data_ptr<int32_t>();
    const int rc = lib.fork(src->data_ptr(), dst, (int)forks, p.table, p.len, p.ref, (int)p.B, (int)p.mb,
                            (int)bs, (int)p.nb, base, bytes, pools, o, o + forks, o + 2 * forks, stream);
    if (rc != TV_OK) return refused(rc);
    PyObject* result = PyTuple_New(3);
    for (int k = 0; result && k < 3; ++k) PyTuple_SET_ITEM(result, k, THPVariable_Wrap(said.select(0, k)));
    return result;
  });
}

// seqs, block_table, kv_len, ref_count
PyObject* free_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 4) return none();
    Tensors t;
    const Pages p(t, a[1], a[2], a[3]);
    const at::Tensor* seqs = t.ranked(a[0], kI32, 1);
    void* stream;
    if (!t.good || !small({seqs->size(0)}) || !stream_of(t.device, &stream)) return none();
    return done(lib.free_(seqs->data_ptr(), (int)seqs->size(0), p.table, p.len, p.ref, (int)p.B, (int)p.mb,
                          (int)p.nb, stream),
                Py_True);
  });
}

// handle of the loaded library, raw_stream, current_device, workspace, capture_workspace
PyObject* connect(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "connect takes five arguments");
    return nullptr;
  }
  void* handle = PyLong_AsVoidPtr(a[0]);
  if (PyErr_Occurred()) return nullptr;
  const auto find = [&](auto& f, const char* name) {
    f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(handle, name));
    return f != nullptr;
  };
  if (!find(lib.capture_id, "tv_capture_id") ||
      !find(lib.attention_ws, "tv_tree_verify_attention_paged_fp8_workspace") ||
      !find(lib.attention, "tv_tree_verify_attention_paged_fp8") || !find(lib.append, "tv_append_paged_fp8") ||
      !find(lib.commit, "tv_commit_path_paged_fp8") || !find(lib.reserve, "tv_reserve_pages") ||
      !find(lib.fork, "tv_fork_pages") || !find(lib.free_, "tv_free_pages")) {
    PyErr_SetString(PyExc_RuntimeError, "libtreeverify.so lacks an entry point");
    return nullptr;
  }
  PyObject** kept[4] = {&raw_stream, &current_device, &workspace, &capture_workspace};
  for (int k = 0; k < 4; ++k) {
    Py_INCREF(a[k + 1]);
    Py_XDECREF(*kept[k]);
    *kept[k] = a[k + 1];
  }
  Py_RETURN_NONE;
}

#define TV_METHOD(name, f) {name, (PyCFunction)(void (*)())f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TV_METHOD("connect", connect),
                         TV_METHOD("attention", attention),
                         TV_METHOD("append", append),
                         TV_METHOD("commit", commit),
                         TV_METHOD("reserve", reserve),
                         TV_METHOD("fork", fork),
                         TV_METHOD("free", free_pages),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_direct", nullptr, -1, methods, nullptr, nullptr, nullptr,
                      nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__direct() { return PyModule_Create(&module); }
