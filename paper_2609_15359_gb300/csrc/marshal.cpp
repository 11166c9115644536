// marshal.cpp -- what maps.py does before a call of the KV memory that a decode step makes, in native code: tensors to
// pointers, sizes and strides, checked.  In Python that takes 5 to 9 us a call, more than the call's launch and, for a small
// batch, its kernel.
//
// Every function here takes the Python function's arguments, then the workspace's address and bytes and the stream's handle.  It
// returns the call's status, or None where an argument is not as expected (another type, shape, device or layout, a tensor
// subclass, a workspace too small): maps.py then goes its own way, which finds out what is wrong and says so.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "maps.h"

namespace {

// The library's functions, as maps.py has loaded them.
decltype(&maps_kv4_record_bytes) record_bytes;
decltype(&maps_kv4_append) append;
decltype(&maps_kv4_read) read;
decltype(&maps_kv4_append_rotated) append_rotated;
decltype(&maps_kv4_block_ranges) block_ranges;
decltype(&maps_kv4_select_blocks_workspace_size) select_workspace;
decltype(&maps_kv4_select_blocks) select_blocks;
decltype(&maps_kv4_attention_blocks) attention_blocks;

// A dense tensor, asked for everything at once: what has no memory throws when it is asked for it, which has to be while the
// interpreter is held.  None where that may be: p is NULL, and so it is for an empty tensor.
struct Dense {
  void *p = nullptr;
  bool given = false;
  int64_t n = 0, dims = 0, size[4] = {};
};

// Arguments one after the other; `ok` falls at the first that is not as expected.
struct Args {
  PyObject *const *at;
  Py_ssize_t left;
  bool ok = true;

  PyObject *next() {
    if (left == 0) ok = false;
    if (!ok) return nullptr;
    --left;
    return *at++;
  }
  void want(bool x) { ok = ok && x; }
  int64_t integer() {
    PyObject *o = next();
    if (o == nullptr) return 0;
    if (PyBool_Check(o)) return o == Py_True;
    if (!PyLong_CheckExact(o)) return ok = false, 0;
    int overflow = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
    want(overflow == 0);
    return x;
  }
  int32_t integer32() {
    const int64_t x = integer();
    want(x >= INT32_MIN && x <= INT32_MAX);
    return static_cast<int32_t>(x);
  }
  void *address() { return reinterpret_cast<void *>(static_cast<intptr_t>(integer())); }
  float number() {
    PyObject *o = next();
    if (o == nullptr || !PyFloat_CheckExact(o)) return ok = false, 0.0f;
    return static_cast<float>(PyFloat_AS_DOUBLE(o));
  }
  // A tensor on the GPU, or (may_be_none) NULL.
  const at::Tensor *tensor(bool may_be_none = false) {
    PyObject *o = next();
    if (o == nullptr) return nullptr;
    if (o == Py_None) return want(may_be_none), nullptr;
    if (!THPVariable_CheckExact(o)) return ok = false, nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    want(t.is_cuda());
    return ok ? &t : nullptr;
  }
  // The same, dense; of any number of dimensions where that is -1.
  Dense dense(at::ScalarType type, int64_t dims, bool may_be_none = false) {
    Dense d;
    const at::Tensor *t = tensor(may_be_none);
    if (t == nullptr) return d;
    want(t->scalar_type() == type && (dims < 0 || t->dim() == dims) && t->is_contiguous());
    if (!ok) return d;
    d.p = t->data_ptr(), d.given = true, d.n = t->numel(), d.dims = t->dim();
    for (int64_t i = 0; i < d.dims && i < 4; ++i) d.size[i] = t->size(i);
    return d;
  }
};

template <class T>
T *data(const Dense &d) {
  return static_cast<T *>(d.p);
}

// Rows of heads whose channels lie side by side: [rows, heads, channels].
struct Rows {
  void *p = nullptr;
  int64_t n = 0, heads = 0, D = 0, row = 0, head = 0;
  at::ScalarType type = at::kBFloat16;
  Rows() = default;
  Rows(Args &a, bool may_be_none = false) {
    const at::Tensor *t = a.tensor(may_be_none);
    if (t == nullptr) return;
    a.want(t->dim() == 3 && t->numel() > 0);
    if (!a.ok) return;
    type = t->scalar_type();
    n = t->size(0), heads = t->size(1), D = t->size(2), row = t->stride(0), head = t->stride(1);
    a.want(t->stride(2) == 1 && (type == at::kBFloat16 || type == at::kHalf) && heads <= INT32_MAX);
    p = t->data_ptr();
  }
  bool like(const Rows &x) const { return n == x.n && heads == x.heads && D == x.D && type == x.type; }
  int32_t dtype() const { return type == at::kBFloat16 ? MAPS_BF16 : MAPS_F16; }
};

// A cache of H heads, blocks of S tokens and D channels.
struct Cache {
  void *p = nullptr;
  int64_t n = 0, H = 0, bytes = 0;
  explicit Cache(Args &a) {
    const Dense t = a.dense(at::kByte, 3);
    p = t.p, n = t.size[0], H = t.size[1], bytes = t.size[2];
  }
  bool holds(int64_t heads, int32_t S, int64_t D) const {
    return H == heads && bytes > 0 && D <= INT32_MAX && bytes == static_cast<int64_t>(record_bytes(S, static_cast<int32_t>(D)));
  }
};

struct Last {  // workspace and stream, which end every call's arguments
  void *ws;
  size_t bytes;
  void *stream;
  explicit Last(Args &a) : ws(a.address()), bytes(static_cast<size_t>(a.integer())), stream(a.address()) { a.want(a.left == 0); }
};

// `call` works on plain values alone: it runs without the interpreter, and may not throw.
template <class Call>
PyObject *status(const Args &a, Call call) {
  if (!a.ok) Py_RETURN_NONE;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

PyObject *py_append(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  const Rows k(a), v(a);
  const Dense slots = a.dense(at::kLong, -1);
  const Cache cache(a);
  const int32_t S = a.integer32();
  const Last l(a);
  if (a.ok) a.want(v.like(k) && slots.n == k.n && cache.holds(k.heads, S, k.D));
  return status(a, [&] {
    return append(k.dtype(), k.n, static_cast<int32_t>(k.heads), static_cast<int32_t>(k.D), S, k.p, k.row, k.head, v.p, v.row, v.head, data<int64_t>(slots), cache.p,
                  cache.n, l.ws, l.bytes, l.stream);
  });
}

PyObject *py_read(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  const Dense slots = a.dense(at::kLong, -1);
  const Cache cache(a);
  const int32_t S = a.integer32();
  const Rows k(a), v(a);
  const Last l(a);
  if (a.ok) a.want(v.like(k) && slots.n == k.n && cache.holds(k.heads, S, k.D));
  return status(a, [&] {
    return read(k.dtype(), k.n, static_cast<int32_t>(k.heads), static_cast<int32_t>(k.D), S, data<int64_t>(slots), cache.p, cache.n, k.p, k.row, k.head, v.p, v.row,
                v.head, l.ws, l.bytes, l.stream);
  });
}

PyObject *py_append_rotated(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  const Rows q(a, true), k(a), v(a);
  const Dense pos = a.dense(at::kInt, -1), cos_sin = a.dense(at::kFloat, 2), slots = a.dense(at::kLong, -1);
  const Cache cache(a);
  const int32_t S = a.integer32();
  const Rows out(a, true);
  const Dense axis = a.dense(at::kInt, -1, true);
  const int32_t interleaved = a.integer() != 0;
  const Last l(a);
  int64_t axes = 1, rot = 0;
  if (a.ok) {
    axes = pos.dims == 2 ? pos.size[0] : 1;
    rot = cos_sin.size[1];
    a.want(v.like(k) && slots.n == k.n && cache.holds(k.heads, S, k.D) && (q.p == nullptr) == (out.p == nullptr) && axes <= INT32_MAX &&
           pos.n == axes * k.n && rot <= INT32_MAX && (!axis.given || axis.n == rot / 2));
    if (q.p != nullptr) a.want(out.like(q) && q.n == k.n && q.D == k.D && q.type == k.type);
  }
  return status(a, [&] {
    return append_rotated(k.dtype(), k.n, static_cast<int32_t>(q.heads), static_cast<int32_t>(k.heads), static_cast<int32_t>(k.D), S, q.p, q.row, q.head, k.p, k.row,
                          k.head, v.p, v.row, v.head, static_cast<int32_t>(axes), data<int32_t>(pos), data<int32_t>(axis), static_cast<int32_t>(rot), interleaved,
                          data<float>(cos_sin), cos_sin.size[0], data<int64_t>(slots), cache.p, cache.n, out.p, out.row, out.head, l.ws, l.bytes, l.stream);
  });
}

// Ranges of blocks of the cache: codes [blocks, H, 2, D], scale [blocks, H].
struct Ranges {
  Dense codes, scale;
  int64_t n = 0, H = 0, D = 0;
  explicit Ranges(Args &a) : codes(a.dense(at::kChar, 4)), scale(a.dense(at::kFloat, 2)) {
    if (!a.ok) return;
    n = codes.size[0], H = codes.size[1], D = codes.size[3];
    a.want(codes.size[2] == 2 && scale.size[0] == n && scale.size[1] == H && H <= INT32_MAX && D <= INT32_MAX);
  }
};

PyObject *py_block_ranges(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  const Dense held = a.dense(at::kInt, -1, true), len = a.dense(at::kInt, -1), table = a.dense(at::kInt, 2);
  const Cache cache(a);
  const int32_t S = a.integer32();
  const Ranges r(a);
  const Last l(a);
  if (a.ok) {
    const int64_t B = len.n;
    a.want(B <= INT32_MAX && (!held.given || held.n == B) && table.size[0] == B && cache.n == r.n && cache.holds(r.H, S, r.D));
  }
  return status(a, [&] {
    return block_ranges(static_cast<int32_t>(len.n), static_cast<int32_t>(r.H), static_cast<int32_t>(r.D), S, data<int32_t>(held), data<int32_t>(len),
                        data<int32_t>(table), table.size[1], cache.p, cache.n, data<int8_t>(r.codes), data<float>(r.scale), l.ws, l.bytes, l.stream);
  });
}

PyObject *py_select_blocks(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  const Rows q(a);
  const Dense off = a.dense(at::kLong, -1), len = a.dense(at::kInt, -1), table = a.dense(at::kInt, 2);
  const Ranges r(a);
  const int32_t S = a.integer32(), first = a.integer32(), last = a.integer32();
  const Dense blocks = a.dense(at::kInt, 3), tokens = a.dense(at::kInt, 2);
  const Last l(a);
  if (a.ok) {
    const int64_t B = len.n;
    a.want(B <= INT32_MAX && q.D == r.D && off.n == B + 1 && table.size[0] == B && blocks.size[0] == q.n && blocks.size[1] == r.H &&
           blocks.size[2] <= INT32_MAX && tokens.size[0] == q.n && tokens.size[1] == r.H &&
           l.bytes >= select_workspace(q.n, static_cast<int32_t>(r.H), table.size[1]));
  }
  return status(a, [&] {
    return select_blocks(q.dtype(), static_cast<int32_t>(len.n), q.n, static_cast<int32_t>(q.heads), static_cast<int32_t>(r.H), static_cast<int32_t>(q.D), S, q.p,
                         q.row, q.head, data<int64_t>(off), data<int32_t>(len), data<int32_t>(table), table.size[1], data<int8_t>(r.codes), data<float>(r.scale), r.n,
                         first, last, static_cast<int32_t>(blocks.size[2]), data<int32_t>(blocks), data<int32_t>(tokens), l.ws, l.bytes, l.stream);
  });
}

PyObject *py_attention_blocks(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  const Rows q(a);
  const Dense blocks = a.dense(at::kInt, 3), tokens = a.dense(at::kInt, 2);
  const Cache cache(a);
  const int32_t S = a.integer32();
  const float scale = a.number();
  const Rows out(a);
  const Dense lse = a.dense(at::kFloat, 2, true);
  const Last l(a);
  if (a.ok)
    a.want(out.like(q) && cache.holds(cache.H, S, q.D) && cache.H <= INT32_MAX && blocks.size[0] == q.n && blocks.size[1] == cache.H &&
           tokens.size[0] == q.n && tokens.size[1] == cache.H && (!lse.given || (lse.size[0] == q.n && lse.size[1] == q.heads)));
  return status(a, [&] {
    return attention_blocks(q.dtype(), q.n, static_cast<int32_t>(q.heads), static_cast<int32_t>(cache.H), static_cast<int32_t>(q.D), S, q.p, q.row, q.head,
                            data<int32_t>(blocks), data<int32_t>(tokens), blocks.size[2], cache.p, cache.n, scale, out.p, out.row, out.head, data<float>(lse), l.ws,
                            l.bytes, l.stream);
  });
}

// The addresses of the library's functions, in the order above.
PyObject *py_bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
  Args a{args, n};
  auto take = [&](auto &f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(a.address()); };
  take(record_bytes), take(append), take(read), take(append_rotated), take(block_ranges), take(select_workspace), take(select_blocks), take(attention_blocks);
  if (!a.ok || a.left != 0) {
    PyErr_SetString(PyExc_TypeError, "expected the addresses of the library's functions");
    return nullptr;
  }
  Py_RETURN_NONE;
}

// A tensor that has no memory or no plain sizes throws where it is asked for them: not as expected either.
template <PyObject *(*kCall)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *self, PyObject *const *args, Py_ssize_t n) {
  try {
    return kCall(self, args, n);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<py_##name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind),          FAST(append),        FAST(read),
                         FAST(append_rotated), FAST(block_ranges), FAST(select_blocks),
                         FAST(attention_blocks), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  PyObject *m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", MAPS_TORCH_VERSION) != 0) Py_CLEAR(m);  // whose tensors it knows
  return m;
}
