// Python side of the calls around a decode step (rotary positions, appends, the 8-bit cache): tensors are checked and handed to the
// C ABI here, natively, because a serving loop makes these calls once per layer and step and the kernels of small steps take 3 us (the same
// checks through ctypes: 20 us a call).  binding.py has the methods and their documentation; liblocks.so's functions come as
// addresses from there.  Nothing is computed here, and calls only enqueue, so the interpreter's lock is kept.
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "locks.h"

// what this module was compiled for: binding.py looks for it in the file before it loads it
extern "C" __attribute__((used, visibility("default"))) const char locks_calls_stamp[] = LOCKS_CALLS_STAMP;

namespace {

struct Context {
  locks_ctx *h;
  int Hq, Hkv, max_batch, pages, B, k, dev;
  bool per_head;
  int64_t summary_bytes;
  at::ScalarType dt;
};

struct Api {
  decltype(&locks_rope) rope;
  decltype(&locks_append_rows) append_rows;
  decltype(&locks_kvq_append) kvq_append;
  decltype(&locks_kvq_attend) kvq_attend;
  decltype(&locks_kvq_build_summaries) kvq_build;
  decltype(&locks_strerror) strerror_;
} api;
PyObject *error_type = nullptr;

struct Refused {
  std::string what;
};
struct Raised {};   // a Python error is set already

[[noreturn]] void refuse(const char *call, const std::string &what) { throw Refused{std::string(call) + ": " + what}; }
void need(bool ok, const char *call, const char *what) {
  if (!ok) refuse(call, what);
}

const at::Tensor &tensor(PyObject *o, const char *call, const char *name) {
  if (!THPVariable_Check(o)) refuse(call, std::string(name) + " is no tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor &on(const Context &c, PyObject *o, const char *call, const char *name) {
  const at::Tensor &t = tensor(o, call, name);
  if (!t.is_cuda() || t.get_device() != c.dev) refuse(call, std::string(name) + " has to be on cuda:" + std::to_string(c.dev));
  return t;
}

struct Owned {   // a reference that ends with its scope
  PyObject *o;
  explicit Owned(PyObject *p) : o(p) {
    if (!p) throw Raised{};
  }
  Owned(const Owned &) = delete;
  ~Owned() { Py_XDECREF(o); }
};

locks_rows rows(const Context &c, PyObject *o, int heads, int64_t n, const char *call, const char *name) {
  const at::Tensor &t = on(c, o, call, name);
  if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != 128 || t.stride(2) != 1 || t.scalar_type() != c.dt)
    refuse(call, std::string(name) + " has to be [" + std::to_string(n) + ", " + std::to_string(heads) + ", 128], dims contiguous, of the configuration's type");
  return locks_rows{t.data_ptr(), t.stride(0), t.stride(1)};
}
// contiguous int32 of these sizes, or nullptr for None
const int32_t *ints(const Context &c, PyObject *o, std::initializer_list<int64_t> sizes, const char *call, const char *name) {
  if (o == Py_None) return nullptr;
  const at::Tensor &t = on(c, o, call, name);
  if (t.scalar_type() != at::kInt || t.sizes() != at::IntArrayRef(sizes) || !t.is_contiguous()) {
    std::string want;
    for (int64_t s : sizes) want += (want.empty() ? "" : ", ") + std::to_string(s);
    refuse(call, std::string(name) + " has to be contiguous int32 [" + want + "]");
  }
  return t.data_ptr<int32_t>();
}

struct RotaryArg {
  Py_buffer b{};
  const locks_rotary *r = nullptr;
  RotaryArg(PyObject *o, const char *call) {
    if (o == Py_None) return;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Raised{};
    if (b.len != (Py_ssize_t)sizeof(locks_rotary)) {
      PyBuffer_Release(&b);
      refuse(call, "rotary has to come from make_rotary");
    }
    r = reinterpret_cast<const locks_rotary *>(b.buf);
  }
  ~RotaryArg() {
    if (r) PyBuffer_Release(&b);
  }
};
const int32_t *positions(const Context &c, PyObject *o, const RotaryArg &rot, int64_t n, const char *call) {
  if (o == Py_None) return nullptr;
  need(rot.r != nullptr, call, "positions go with a rotary description");
  if (THPVariable_Check(o) && rot.r->num_axes == 1 && THPVariable_Unpack(o).dim() == 1) return ints(c, o, {n}, call, "positions");
  return ints(c, o, {rot.r->num_axes, n}, call, "positions");
}

locks_stream stream_of(const Context &c, PyObject *o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream(c.dev).stream();
  if (PyLong_Check(o)) return PyLong_AsVoidPtr(o);
  Owned s(PyObject_GetAttrString(o, "cuda_stream"));
  return PyLong_AsVoidPtr(s.o);
}

int64_t integer(PyObject *o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
int batch_of(const Context &c, PyObject *o, const char *call) {
  const int64_t b = integer(o);
  need(b >= 1 && b <= c.max_batch, call, "batch is outside the configuration's");
  return (int)b;
}
void table_ok(const Context &c, const at::Tensor &table, const at::Tensor &lens, int batch, const char *call) {
  need(table.scalar_type() == at::kInt && table.dim() == 2 && table.is_contiguous() && table.size(0) >= batch && table.size(1) == c.pages, call,
       "block_table has to be contiguous int32 [max_batch, max_pages_per_seq] of the configuration");
  need(lens.scalar_type() == at::kInt && lens.dim() == 1 && lens.is_contiguous() && lens.size(0) >= batch, call, "seq_lens has to be contiguous int32 [max_batch]");
}

locks_kv kv_view(const Context &c, PyObject *o, int batch, const char *call) {
  Owned k(PyObject_GetAttrString(o, "k")), v(PyObject_GetAttrString(o, "v")), st(PyObject_GetAttrString(o, "strides"));
  Owned nb(PyObject_GetAttrString(o, "num_blocks")), tb(PyObject_GetAttrString(o, "block_table")), sl(PyObject_GetAttrString(o, "seq_lens"));
  const at::Tensor &kt = on(c, k.o, call, "k"), &vt = on(c, v.o, call, "v"), &table = on(c, tb.o, call, "block_table"), &lens = on(c, sl.o, call, "seq_lens");
  need(kt.scalar_type() == c.dt && vt.scalar_type() == c.dt, call, "the cache has to be of the configuration's type");
  table_ok(c, table, lens, batch, call);
  Owned seq(PySequence_Fast(st.o, "strides"));
  need(PySequence_Fast_GET_SIZE(seq.o) == 3, call, "strides are those of block, head and token");
  PyObject **s = PySequence_Fast_ITEMS(seq.o);
  return locks_kv{kt.data_ptr(), vt.data_ptr(), integer(s[0]), integer(s[1]), integer(s[2]), (int32_t)integer(nb.o), table.data_ptr<int32_t>(), lens.data_ptr<int32_t>()};
}

locks_kvq kvq_view(const Context &c, PyObject *o, int batch, const char *call) {
  Owned k(PyObject_GetAttrString(o, "k")), v(PyObject_GetAttrString(o, "v")), ks(PyObject_GetAttrString(o, "k_scale")), vs(PyObject_GetAttrString(o, "v_scale"));
  Owned kt(PyObject_GetAttrString(o, "k_tail")), vt(PyObject_GetAttrString(o, "v_tail")), tb(PyObject_GetAttrString(o, "block_table")), sl(PyObject_GetAttrString(o, "seq_lens"));
  const at::Tensor &kc = on(c, k.o, call, "k"), &vc = on(c, v.o, call, "v");
  need(kc.dim() == 4 && kc.sizes() == vc.sizes() && kc.strides() == vc.strides() && kc.size(1) == c.Hkv && kc.size(2) == c.B && kc.size(3) == 128 && kc.stride(3) == 1, call,
       "codes have to be [block, head, token, 128] of the configuration's heads and page size, dims contiguous, keys and values laid out alike");
  need(kc.scalar_type() == vc.scalar_type() && (kc.scalar_type() == at::kChar || kc.scalar_type() == at::kFloat8_e4m3fn), call, "codes have to be int8 or float8_e4m3fn");
  float *scale[2], *tail[2];
  int64_t tail_rows = 0;
  PyObject *so[2] = {ks.o, vs.o}, *to[2] = {kt.o, vt.o};
  for (int i = 0; i < 2; ++i) {
    const at::Tensor &s = on(c, so[i], call, "scales"), &t = on(c, to[i], call, "tails");
    need(s.scalar_type() == at::kFloat && s.dim() == 2 && s.size(0) == kc.size(0) && s.size(1) == c.Hkv && s.is_contiguous(), call, "scales have to be contiguous fp32 [block, head]");
    need(t.scalar_type() == at::kFloat && t.dim() == 4 && t.size(0) >= batch && t.size(1) == c.Hkv && (t.size(2) == c.B || t.size(2) == 2 * c.B) && t.size(3) == 128 && t.is_contiguous(), call,
         "tails have to be contiguous fp32 [max_batch, head, page_size or twice that, 128]");
    need(i == 0 || t.size(2) == tail_rows, call, "tails of keys and values have to be of one size");
    tail_rows = t.size(2);
    scale[i] = s.data_ptr<float>();
    tail[i] = t.data_ptr<float>();
  }
  const at::Tensor &table = on(c, tb.o, call, "block_table"), &lens = on(c, sl.o, call, "seq_lens");
  table_ok(c, table, lens, batch, call);
  return locks_kvq{kc.data_ptr(), vc.data_ptr(), kc.stride(0), kc.stride(1), kc.stride(2), (int32_t)kc.size(0), kc.scalar_type() == at::kChar ? LOCKS_KVQ_INT : LOCKS_KVQ_FLOAT,
                   scale[0], scale[1], tail[0], tail[1], table.data_ptr<int32_t>(), lens.data_ptr<int32_t>(), (int32_t)(tail_rows / c.B)};
}

void check(int rc, const char *call) {
  if (rc != LOCKS_OK) throw Refused{std::string(call) + " failed: " + api.strerror_(rc) + " (" + std::to_string(rc) + ")"};
}

const Context &context_of(PyObject *o) {
  void *p = PyCapsule_GetPointer(o, "locks.context");
  if (!p) throw Raised{};
  const Context *c = reinterpret_cast<Context *>(p);
  if (!c->h) throw Refused{"the context is closed"};
  return *c;
}

// a call's body, its errors as Python's
template <typename F> PyObject *guarded(F &&body) {
  try {
    body();
  } catch (const Refused &r) {
    PyErr_SetString(error_type ? error_type : PyExc_RuntimeError, r.what.c_str());
    return nullptr;
  } catch (const Raised &) {
    return nullptr;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  Py_RETURN_NONE;
}
bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}

// (context, rotary, positions, q, q_out, k, k_out, stream)
PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&] {
    const char *call = "locks_rope";
    const Context &c = context_of(a[0]);
    RotaryArg rot(a[1], call);
    need(rot.r && a[2] != Py_None, call, "rotary and positions are needed");
    need((a[3] == Py_None) == (a[4] == Py_None) && (a[5] == Py_None) == (a[6] == Py_None) && (a[3] != Py_None || a[5] != Py_None), call, "q goes with q_out, k with k_out");
    const at::Tensor &first = tensor(a[3] != Py_None ? a[3] : a[5], call, "rows");
    need(first.dim() == 3, call, "rows are [tokens, heads, 128]");
    const int64_t tokens = first.size(0);
    const int heads[4] = {c.Hq, c.Hq, c.Hkv, c.Hkv};
    const char *names[4] = {"q", "q_out", "k", "k_out"};
    locks_rows r[4];
    const locks_rows *p[4];
    for (int i = 0; i < 4; ++i) {
      p[i] = a[3 + i] == Py_None ? nullptr : &r[i];
      if (p[i]) r[i] = rows(c, a[3 + i], heads[i], tokens, call, names[i]);
    }
    need(tokens <= INT32_MAX, call, "too many tokens");
    const int32_t *pos = positions(c, a[2], rot, tokens, call);
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    check(api.rope(c.h, rot.r, pos, (int)tokens, p[0], p[1], p[2], p[3], stream_of(c, a[7])), call);
  });
}

// (context, k_new, v_new, view, batch, rotary, positions, q, q_out, cu_tokens, stream)
template <bool KVQ> PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 11)) return nullptr;
  return guarded([&] {
    const char *call = KVQ ? "locks_kvq_append" : "locks_append_rows";
    const Context &c = context_of(a[0]);
    const int batch = batch_of(c, a[4], call);
    RotaryArg rot(a[5], call);
    need((a[7] == Py_None) == (a[8] == Py_None) && (a[7] == Py_None || rot.r), call, "q goes with q_out and a rotary description");
    const at::Tensor &first = tensor(a[1], call, "k_new");
    need(first.dim() == 3 && first.size(0) <= INT32_MAX, call, "rows are [tokens, heads, 128]");
    const int64_t tokens = first.size(0);
    const locks_rows kn = rows(c, a[1], c.Hkv, tokens, call, "k_new"), vn = rows(c, a[2], c.Hkv, tokens, call, "v_new");
    locks_rows q, qo;
    const bool has_q = a[7] != Py_None;
    if (has_q) {
      q = rows(c, a[7], c.Hq, tokens, call, "q");
      qo = rows(c, a[8], c.Hq, tokens, call, "q_out");
    }
    const int32_t *pos = positions(c, a[6], rot, tokens, call), *cu = ints(c, a[9], {batch + 1}, call, "cu_tokens");
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    if (KVQ) {
      const locks_kvq kv = kvq_view(c, a[3], batch, call);
      check(api.kvq_append(c.h, rot.r, pos, cu, (int)tokens, has_q ? &q : nullptr, has_q ? &qo : nullptr, &kn, &vn, &kv, batch, stream_of(c, a[10])), call);
    } else {
      const locks_kv kv = kv_view(c, a[3], batch, call);
      check(api.append_rows(c.h, rot.r, pos, cu, (int)tokens, has_q ? &q : nullptr, has_q ? &qo : nullptr, &kn, &vn, &kv, batch, stream_of(c, a[10])), call);
    }
  });
}

// (context, q, view, batch, out, lse, page_ids, page_count, cu_tokens, stream)
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 10)) return nullptr;
  return guarded([&] {
    const char *call = "locks_kvq_attend";
    const Context &c = context_of(a[0]);
    const int batch = batch_of(c, a[3], call);
    const locks_kvq kv = kvq_view(c, a[2], batch, call);
    const at::Tensor &q = on(c, a[1], call, "q"), &out = on(c, a[4], call, "out");
    const int64_t tokens = q.dim() == 3 ? q.size(0) : 0;
    for (const at::Tensor *t : {&q, &out})
      need(t->dim() == 3 && t->size(0) == tokens && t->size(1) == c.Hq && t->size(2) == 128 && t->is_contiguous() && t->scalar_type() == c.dt && tokens <= INT32_MAX, call,
           "q and out have to be contiguous [tokens, heads, 128] of the configuration's type");
    float *lse = nullptr;
    if (a[5] != Py_None) {
      const at::Tensor &t = on(c, a[5], call, "lse");
      need(t.dim() == 2 && t.size(0) == tokens && t.size(1) == c.Hq && t.is_contiguous() && t.scalar_type() == at::kFloat, call, "lse has to be contiguous fp32 [tokens, heads]");
      lse = t.data_ptr<float>();
    }
    const int heads = c.per_head ? c.Hq : c.Hkv;
    const int32_t *ids = ints(c, a[6], {batch, heads, c.k}, call, "page_ids"), *cnt = ints(c, a[7], {batch, heads}, call, "page_count"),
                  *cu = ints(c, a[8], {batch + 1}, call, "cu_tokens");
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    check(api.kvq_attend(c.h, q.data_ptr(), cu, (int)tokens, &kv, batch, ids, cnt, out.data_ptr(), lse, stream_of(c, a[9])), call);
  });
}

// (context, view, batch, summaries, page_begin, page_end, stream)
PyObject *build(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 7)) return nullptr;
  return guarded([&] {
    const char *call = "locks_kvq_build_summaries";
    const Context &c = context_of(a[0]);
    const int batch = batch_of(c, a[2], call);
    const locks_kvq kv = kvq_view(c, a[1], batch, call);
    const at::Tensor &s = on(c, a[3], call, "summaries");
    need(s.scalar_type() == at::kByte && s.is_contiguous() && s.numel() >= kv.num_blocks * c.Hkv * c.summary_bytes, call, "summaries have to be those of Context.new_summaries");
    const int32_t *pb = ints(c, a[4], {batch}, call, "page_begin"), *pe = ints(c, a[5], {batch}, call, "page_end");
    c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.dev);
    check(api.kvq_build(c.h, &kv, batch, pb, pe, s.data_ptr(), stream_of(c, a[6])), call);
  });
}

// (error type, addresses of the six functions in Api's order)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 7)) return nullptr;
  void *p[6];
  for (int i = 0; i < 6; ++i)
    if (!(p[i] = PyLong_AsVoidPtr(a[1 + i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "no address");
  Py_INCREF(a[0]);
  error_type = a[0];
  api = Api{(decltype(api.rope))p[0], (decltype(api.append_rows))p[1], (decltype(api.kvq_append))p[2], (decltype(api.kvq_attend))p[3], (decltype(api.kvq_build))p[4], (decltype(api.strerror_))p[5]};
  Py_RETURN_NONE;
}

// (handle, Hq, Hkv, max_batch, pages, page size, k, device, per head, summary bytes, bf16) -> capsule; close(capsule)
PyObject *context(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 11)) return nullptr;
  long long v[11];
  for (int i = 0; i < 11; ++i)
    if ((v[i] = PyLong_AsLongLong(a[i])) == -1 && PyErr_Occurred()) return nullptr;
  Context *c = new Context{reinterpret_cast<locks_ctx *>(v[0]), (int)v[1], (int)v[2], (int)v[3], (int)v[4], (int)v[5], (int)v[6], (int)v[7], v[8] != 0, v[9], v[10] ? at::kBFloat16 : at::kFloat};
  return PyCapsule_New(c, "locks.context", [](PyObject *o) { delete reinterpret_cast<Context *>(PyCapsule_GetPointer(o, "locks.context")); });
}
PyObject *close(PyObject *, PyObject *o) {
  Context *c = reinterpret_cast<Context *>(PyCapsule_GetPointer(o, "locks.context"));
  if (!c) return nullptr;
  c->h = nullptr;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void *)bind, METH_FASTCALL, nullptr},
                         {"context", (PyCFunction)(void *)context, METH_FASTCALL, nullptr},
                         {"close", (PyCFunction)close, METH_O, nullptr},
                         {"rope", (PyCFunction)(void *)rope, METH_FASTCALL, nullptr},
                         {"append_rows", (PyCFunction)(void *)append<false>, METH_FASTCALL, nullptr},
                         {"kvq_append", (PyCFunction)(void *)append<true>, METH_FASTCALL, nullptr},
                         {"kvq_attend", (PyCFunction)(void *)attend, METH_FASTCALL, nullptr},
                         {"kvq_build_summaries", (PyCFunction)(void *)build, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "native marshalling of binding.py", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
