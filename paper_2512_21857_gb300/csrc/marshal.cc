// Marshalling of the calls that are made from Python one at a time: the same checks
// as binding.py makes for the others, of tensors as C++ sees them.  (A decoded
// token's calls take less than their marshalling: looking at 9 to 18 tensors
// attribute by attribute from Python takes 10 to 17 us of the host, this 1 to 2.)
//
// Every function takes its arguments by position, as binding.py passes them,
// raises TypeError or ValueError for tensors that do not fit, and returns the
// status of the C entry point.
#include <Python.h>

#include <dlfcn.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "adt.h"

namespace {

using at::ScalarType;
using at::Tensor;

// The library's entry points, looked up by load().
struct Library {
  decltype(&adt_norm_rope_qkv) norm_rope_qkv;
  decltype(&adt_kv_compact_q8) kv_compact_q8;
  decltype(&adt_kv_read_q8) kv_read_q8;
  decltype(&adt_tree_attn_q8) tree_attn_q8;
} g_lib;

struct TypeProblem : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct ValueProblem : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct PythonProblem {};  // already set

[[noreturn]] void bad_value(const std::string& s) { throw ValueProblem(s); }

// Positional arguments in turn.
struct Args {
  PyObject* const* a;
  Py_ssize_t n, at = 0;
  PyObject* next() {
    if (at >= n) throw TypeProblem("too few arguments");
    return a[at++];
  }
  // NULL for None.
  const Tensor* tensor(const char* name) {
    PyObject* o = next();
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw TypeProblem(std::string(name) + ": expected a tensor");
    return &THPVariable_Unpack(o);
  }
  const Tensor& some(const char* name) {
    const Tensor* t = tensor(name);
    if (!t) throw TypeProblem(std::string(name) + ": expected a tensor");
    return *t;
  }
  int64_t integer() {
    const int64_t v = PyLong_AsLongLong(next());
    if (v == -1 && PyErr_Occurred()) throw PythonProblem();
    return v;
  }
  int32_t i32(const char* name) {
    const int64_t v = integer();
    if (v != static_cast<int32_t>(v)) bad_value(std::string(name) + ": does not fit 32 bits");
    return static_cast<int32_t>(v);
  }
  float real() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw PythonProblem();
    return static_cast<float>(v);
  }
  void done() const {
    if (at != n) throw TypeProblem("too many arguments");
  }
};

std::string type_name(ScalarType t) { return c10::toString(t); }

// The current CUDA device, which the launch goes to, and the stream: `stream`, a
// torch.cuda.Stream, or that device's current one.
struct Place {
  int dev;
  void* stream;
};

void on_device(const Tensor& t, int dev, const char* name) {
  if (!t.is_cuda() || t.get_device() != dev)
    bad_value(std::string(name) + ": expected a tensor on the current CUDA device, got one on " + t.device().str());
}

Place place_of(const Tensor& t, PyObject* stream, const char* name) {
  if (!t.is_cuda()) bad_value(std::string(name) + ": expected a tensor on the current CUDA device, got one on " + t.device().str());
  Place p;
  p.dev = c10::cuda::current_device();
  on_device(t, p.dev, name);
  if (stream == Py_None) {
    p.stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(p.dev)).stream();
    return p;
  }
  PyObject* h = PyObject_GetAttrString(stream, "cuda_stream");
  if (!h) throw PythonProblem();
  p.stream = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (PyErr_Occurred()) throw PythonProblem();
  return p;
}

// The address of a tensor of that type on device dev; NULL for None.
void* addr(const Tensor* t, ScalarType type, int dev, const char* name) {
  if (!t) return nullptr;
  on_device(*t, dev, name);
  if (t->scalar_type() != type)
    throw TypeProblem(std::string(name) + ": expected " + type_name(type) + ", got " + type_name(t->scalar_type()));
  return t->data_ptr();
}

// ... and of a contiguous one of at least `count` elements.
void* vec(const Tensor* t, ScalarType type, int dev, int64_t count, const char* name) {
  void* p = addr(t, type, dev, name);
  if (t && (t->numel() < count || !t->is_contiguous()))
    bad_value(std::string(name) + ": expected " + std::to_string(count) + " elements, contiguous");
  return p;
}

// A call of the library, without the interpreter's lock: a launch waits where the
// device's queue is full, which may be for another thread's sake.
template <class F, class... A>
adt_status unlocked(F f, A... a) {
  PyThreadState* state = PyEval_SaveThread();
  const adt_status st = f(a...);
  PyEval_RestoreThread(state);
  return st;
}

template <class T>
T* as(void* p) {
  return static_cast<T*>(p);
}

int32_t rows_type(ScalarType t, const char* what) {
  if (t == at::kBFloat16) return ADT_TYPE_BF16;
  if (t == at::kFloat) return ADT_TYPE_F32;
  throw TypeProblem(std::string(what) + ": bf16 or fp32, all the same");
}

// Rows [N, heads * D] or heads [N, heads, D], contiguous within a row, with their output.
struct Rows {
  const void* in = nullptr;
  int64_t ld = 0;
  void* out = nullptr;
};

Rows rows_of(const Tensor* t, const Tensor* out, ScalarType type, int dev, int64_t heads, int64_t D, int64_t N, const char* name) {
  const std::string who(name);
  if (!t || !out) {
    if (t || out) bad_value(who + " and " + who + "_out: both or neither");
    return {};
  }
  const int64_t width = heads * D;
  const auto s = t->sizes(), st = t->strides();
  const bool flat = s.size() == 2 && s[0] == N && s[1] == width && st[1] == 1;
  const bool split = s.size() == 3 && s[0] == N && s[1] == heads && s[2] == D && st[2] == 1 && (st[1] == D || heads == 1);
  if (!flat && !split)
    bad_value(who + ": expected rows [" + std::to_string(N) + ", " + std::to_string(width) + "] or [" + std::to_string(N) + ", " +
              std::to_string(heads) + ", " + std::to_string(D) + "], contiguous within a row");
  if (out->numel() != N * width)
    bad_value(who + "_out: expected [" + std::to_string(N) + ", " + std::to_string(heads) + ", " + std::to_string(D) + "]");
  Rows r;
  r.in = addr(t, type, dev, name);
  r.ld = N > 1 ? st[0] : width;
  r.out = vec(out, at::kBFloat16, dev, 0, (who + "_out").c_str());
  return r;
}

// A weight and its bias, [D] or [heads, D] each; the stride from head to head.
struct Affine {
  const void *weight, *bias;
  int32_t stride;
};

Affine affine_of(const Tensor* w, const Tensor* b, ScalarType type, int dev, int64_t heads, int64_t D, const char* name) {
  const std::string who(name);
  if (w && b && w->dim() != b->dim())
    bad_value(who + "_weight and " + who + "_bias: both [" + std::to_string(D) + "] or both [" + std::to_string(heads) + ", " +
              std::to_string(D) + "]");
  for (const Tensor* t : {w, b}) {
    if (!t) continue;
    const auto s = t->sizes();
    if (!(s.size() == 1 && s[0] == D) && !(s.size() == 2 && s[0] == heads && s[1] == D))
      bad_value(who + "_weight, " + who + "_bias: expected [" + std::to_string(D) + "] or [" + std::to_string(heads) + ", " +
                std::to_string(D) + "]");
  }
  const Tensor* any = w ? w : b;
  return {vec(w, type, dev, 0, (who + "_weight").c_str()), vec(b, type, dev, 0, (who + "_bias").c_str()),
          any && any->dim() == 2 ? static_cast<int32_t>(D) : 0};
}

// Strides of [layers, B, Hkv, rows or more, D] (D = 0: without D; one_layer: without
// layers), those of a dimension of one as 0: they say nothing; the rows are packed.
struct Strides {
  int64_t s[3];
  bool operator==(const Strides& o) const { return s[0] == o.s[0] && s[1] == o.s[1] && s[2] == o.s[2]; }
};

Strides strides_of(const Tensor& t, int64_t layers, int64_t B, int64_t Hkv, int64_t rows, int64_t D, bool one_layer,
                   const char* name) {
  const auto s = t.sizes(), st = t.strides();
  const size_t off = one_layer ? 0 : 1, want = (D ? 4 : 3) + off;
  const bool fits = s.size() == want && (one_layer || s[0] == layers) && s[off] == B && s[off + 1] == Hkv && s[off + 2] >= rows &&
                    (!D || s[off + 3] == D);
  if (!fits)
    bad_value(std::string(name) + ": expected [" + (one_layer ? "" : std::to_string(layers) + ", ") + std::to_string(B) + ", " +
              std::to_string(Hkv) + ", " + std::to_string(rows) + (D ? ", " + std::to_string(D) : "") + "] or more rows");
  if ((st[off + 2] != (D ? D : 1) && s[off + 2] > 1) || (D && st[off + 3] != 1)) bad_value(std::string(name) + ": expected packed rows");
  return {{layers > 1 ? st[0] : 0, B > 1 ? st[off] : 0, Hkv > 1 ? st[off + 1] : 0}};
}

struct Cache {
  uint8_t *k, *v, *ks, *vs;
  Strides cs, ss;
};

Cache cache_of(const Tensor& k, const Tensor& v, const Tensor& ks, const Tensor& vs, int64_t layers, int64_t B, int64_t Hkv,
               int64_t rows, int64_t D, bool one_layer, int dev) {
  Cache c;
  c.cs = strides_of(k, layers, B, Hkv, rows, D, one_layer, "k_cache");
  c.ss = strides_of(ks, layers, B, Hkv, rows, 0, one_layer, "k_scale");
  if (!(strides_of(v, layers, B, Hkv, rows, D, one_layer, "v_cache") == c.cs) ||
      !(strides_of(vs, layers, B, Hkv, rows, 0, one_layer, "v_scale") == c.ss))
    bad_value("K and V must share strides");
  c.k = as<uint8_t>(addr(&k, at::kFloat8_e4m3fn, dev, "k_cache"));
  c.v = as<uint8_t>(addr(&v, at::kFloat8_e4m3fn, dev, "v_cache"));
  c.ks = as<uint8_t>(addr(&ks, at::kByte, dev, "k_scale"));
  c.vs = as<uint8_t>(addr(&vs, at::kByte, dev, "v_scale"));
  return c;
}

adt_status norm_rope_qkv(Args& a) {
  const Tensor *q = a.tensor("q"), *k = a.tensor("k"), *v = a.tensor("v");
  const Tensor &pos = a.some("positions"), &inv = a.some("inv_freq");
  const int32_t H = a.i32("H"), Hkv = a.i32("Hkv"), D = a.i32("D"), norm = a.i32("norm");
  const float eps = a.real();
  const Tensor *qw = a.tensor("q_weight"), *qb = a.tensor("q_bias"), *kw = a.tensor("k_weight"), *kb = a.tensor("k_bias");
  const int32_t layout = a.i32("layout");
  const float magnitude = a.real();
  const Tensor *qo = a.tensor("q_out"), *ko = a.tensor("k_out"), *vo = a.tensor("v_out");
  const Place p = place_of(pos, a.next(), "positions");
  a.done();
  const int64_t N = pos.numel();
  if (N > INT32_MAX) bad_value("positions: too many");
  const Tensor* first = q ? q : k ? k : v;
  if (!first) throw TypeProblem("q, k, v: bf16 or fp32, all the same");
  const ScalarType type = first->scalar_type();
  const int32_t in_type = rows_type(type, "q, k, v");
  ScalarType wtype = at::kFloat;
  for (const Tensor* t : {kb, kw, qb, qw})
    if (t) wtype = t->scalar_type();
  const int32_t weight_type = rows_type(wtype, "weights and biases");
  const Rows rq = rows_of(q, qo, type, p.dev, H, D, N, "q"), rk = rows_of(k, ko, type, p.dev, Hkv, D, N, "k"),
             rv = rows_of(v, vo, type, p.dev, Hkv, D, N, "v");
  const Affine aq = affine_of(qw, qb, wtype, p.dev, H, D, "q"), ak = affine_of(kw, kb, wtype, p.dev, Hkv, D, "k");
  const int32_t* positions = as<int32_t>(vec(&pos, at::kInt, p.dev, N, "positions"));
  const double* freq = as<double>(vec(&inv, at::kDouble, p.dev, 0, "inv_freq"));
  if (inv.numel() > (1 << 20)) bad_value("inv_freq: too many");
  return unlocked(
      g_lib.norm_rope_qkv, rq.in, rq.ld, rk.in, rk.ld, rv.in, rv.ld, static_cast<adt_dtype>(in_type), static_cast<adt_norm>(norm),
                           eps, aq.weight, aq.bias, aq.stride, ak.weight, ak.bias, ak.stride,
                           static_cast<adt_dtype>(weight_type), positions, freq, magnitude, static_cast<adt_rope_layout>(layout),
                           static_cast<int32_t>(N), H, Hkv, D, static_cast<int32_t>(2 * inv.numel()), as<adt_bf16>(rq.out),
                           as<adt_bf16>(rk.out), as<adt_bf16>(rv.out), p.stream);
}

// k_tree, v_tree [layers, nodes, Hkv, D], each layer contiguous; the layer stride.
int64_t tree_stride(const Tensor& k, const Tensor& v, int64_t layers, int64_t Hkv, int64_t D) {
  for (const Tensor* t : {&k, &v}) {
    const auto s = t->sizes(), st = t->strides();
    const bool fits = s.size() == 4 && s[0] >= layers && s[2] == Hkv && s[3] == D && (st[3] == 1 || D == 1) &&
                      (st[2] == D || Hkv == 1) && (st[1] == Hkv * D || s[1] <= 1);
    if (!fits)
      bad_value(std::string(t == &k ? "k_tree" : "v_tree") + ": expected [" + std::to_string(layers) + ", nodes, " +
                std::to_string(Hkv) + ", " + std::to_string(D) + "], each layer contiguous");
  }
  if (k.size(1) != v.size(1) || (layers > 1 && k.stride(0) != v.stride(0)))
    bad_value("k_tree and v_tree must share their shape and strides");
  return layers > 1 ? k.stride(0) : 0;
}

adt_status kv_compact_q8(Args& a) {
  const Tensor &kc = a.some("k_cache"), &vc = a.some("v_cache"), &ks = a.some("k_scale"), &vs = a.some("v_scale"),
               &kv = a.some("kv_len");
  const Tensor* kvo = a.tensor("kv_len_out");
  const Tensor &kt = a.some("k_tree"), &vt = a.some("v_tree"), &offs = a.some("node_offsets"), &path = a.some("path");
  const int32_t max_path = a.i32("max_path");
  const Tensor& alen = a.some("accept_len");
  const int32_t B = a.i32("B"), Hkv = a.i32("Hkv"), D = a.i32("D"), layers = a.i32("num_layers"), max_kv = a.i32("max_kv");
  const Place p = place_of(kc, a.next(), "k_cache");
  a.done();
  const Cache c = cache_of(kc, vc, ks, vs, layers, B, Hkv, max_kv, D, false, p.dev);
  const int64_t tls = tree_stride(kt, vt, layers, Hkv, D);
  return unlocked(
      g_lib.kv_compact_q8,
      c.k, c.v, c.ks, c.vs, as<int32_t>(vec(&kv, at::kInt, p.dev, B, "kv_len")), as<int32_t>(vec(kvo, at::kInt, p.dev, B, "kv_len_out")),
      as<adt_bf16>(addr(&kt, at::kBFloat16, p.dev, "k_tree")), as<adt_bf16>(addr(&vt, at::kBFloat16, p.dev, "v_tree")),
      as<int32_t>(vec(&offs, at::kInt, p.dev, B + int64_t{1}, "node_offsets")),
      as<int32_t>(vec(&path, at::kInt, p.dev, static_cast<int64_t>(B) * max_path, "path")), max_path,
      as<int32_t>(vec(&alen, at::kInt, p.dev, B, "accept_len")), B, Hkv, D, layers, max_kv, c.cs.s[0], c.cs.s[1], c.cs.s[2],
      c.ss.s[0], c.ss.s[1], c.ss.s[2], tls, p.stream);
}

adt_status kv_read_q8(Args& a) {
  const Tensor &kc = a.some("k_cache"), &vc = a.some("v_cache"), &ks = a.some("k_scale"), &vs = a.some("v_scale"),
               &kv = a.some("kv_len"), &ko = a.some("k_out"), &vo = a.some("v_out");
  const int32_t B = a.i32("B"), Hkv = a.i32("Hkv"), D = a.i32("D"), layers = a.i32("num_layers"), max_kv = a.i32("max_kv");
  const Place p = place_of(kc, a.next(), "k_cache");
  a.done();
  const Cache c = cache_of(kc, vc, ks, vs, layers, B, Hkv, max_kv, D, false, p.dev);
  const Strides os = strides_of(ko, layers, B, Hkv, max_kv, D, false, "k_out");
  if (!(strides_of(vo, layers, B, Hkv, max_kv, D, false, "v_out") == os)) bad_value("k_out and v_out must share strides");
  return unlocked(
      g_lib.kv_read_q8, c.k, c.v, c.ks, c.vs, as<int32_t>(vec(&kv, at::kInt, p.dev, B, "kv_len")),
                        as<adt_bf16>(addr(&ko, at::kBFloat16, p.dev, "k_out")), as<adt_bf16>(addr(&vo, at::kBFloat16, p.dev, "v_out")),
                        B, Hkv, D, layers, max_kv, c.cs.s[0], c.cs.s[1], c.cs.s[2], c.ss.s[0], c.ss.s[1], c.ss.s[2], os.s[0],
                        os.s[1], os.s[2], p.stream);
}

adt_status tree_attn_q8(Args& a) {
  const Tensor &q = a.some("q"), &kc = a.some("k_cache"), &vc = a.some("v_cache"), &ks = a.some("k_scale"), &vs = a.some("v_scale"),
               &kv = a.some("kv_len"), &kt = a.some("k_tree"), &vt = a.some("v_tree"), &par = a.some("parents"),
               &offs = a.some("node_offsets");
  const int32_t B = a.i32("B"), H = a.i32("H"), Hkv = a.i32("Hkv"), D = a.i32("D"), max_nodes = a.i32("max_nodes"),
                max_kv = a.i32("max_kv");
  const float scale = a.real();
  const Tensor& out = a.some("out");
  const Tensor* lse = a.tensor("lse");
  const Tensor& ws = a.some("workspace");
  const Place p = place_of(q, a.next(), "q");
  a.done();
  if (q.dim() < 1) bad_value("q: expected [Ntot, H, D]");
  const int64_t N = q.size(0), qn = N * H * D, tn = N * Hkv * D;
  const Cache c = cache_of(kc, vc, ks, vs, 1, B, Hkv, max_kv, D, true, p.dev);
  return unlocked(
      g_lib.tree_attn_q8,
      as<adt_bf16>(vec(&q, at::kBFloat16, p.dev, qn, "q")), c.k, c.v, c.ks, c.vs, as<int32_t>(vec(&kv, at::kInt, p.dev, B, "kv_len")),
      c.cs.s[1], c.cs.s[2], c.ss.s[1], c.ss.s[2], as<adt_bf16>(vec(&kt, at::kBFloat16, p.dev, tn, "k_tree")),
      as<adt_bf16>(vec(&vt, at::kBFloat16, p.dev, tn, "v_tree")), as<int32_t>(vec(&par, at::kInt, p.dev, N, "parents")),
      as<int32_t>(vec(&offs, at::kInt, p.dev, B + int64_t{1}, "node_offsets")), B, H, Hkv, D, max_nodes, max_kv, scale,
      as<adt_bf16>(vec(&out, at::kBFloat16, p.dev, qn, "out")), as<float>(vec(lse, at::kFloat, p.dev, N * H, "lse")),
      vec(&ws, at::kByte, p.dev, 0, "workspace"), ws.nbytes(), p.stream);
}

template <adt_status (*F)(Args&)>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    Args a{args, n};
    return PyLong_FromLong(F(a));
  } catch (const PythonProblem&) {
  } catch (const TypeProblem& e) {
    PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const ValueProblem& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

template <adt_status (*F)(Args&)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<F>)), METH_FASTCALL, nullptr};
}

// load(path): the library that the calls go to.
PyObject* load(PyObject*, PyObject* path) {
  const char* name = PyUnicode_AsUTF8(path);
  if (!name) return nullptr;
  void* so = dlopen(name, RTLD_NOW);
  Library lib{};
  if (so) {
    lib.norm_rope_qkv = reinterpret_cast<decltype(lib.norm_rope_qkv)>(dlsym(so, "adt_norm_rope_qkv"));
    lib.kv_compact_q8 = reinterpret_cast<decltype(lib.kv_compact_q8)>(dlsym(so, "adt_kv_compact_q8"));
    lib.kv_read_q8 = reinterpret_cast<decltype(lib.kv_read_q8)>(dlsym(so, "adt_kv_read_q8"));
    lib.tree_attn_q8 = reinterpret_cast<decltype(lib.tree_attn_q8)>(dlsym(so, "adt_tree_attn_q8"));
  }
  if (!lib.norm_rope_qkv || !lib.kv_compact_q8 || !lib.kv_read_q8 || !lib.tree_attn_q8) {
    PyErr_Format(PyExc_RuntimeError, "%s: not the library", name);
    return nullptr;
  }
  g_lib = lib;
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {{"load", load, METH_O, nullptr},
                          method<norm_rope_qkv>("norm_rope_qkv"), method<kv_compact_q8>("kv_compact_q8"),
                          method<kv_read_q8>("kv_read_q8"), method<tree_attn_q8>("tree_attn_q8"),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }
