// Argument marshalling of the cache and attention calls in native code: what binding.py does for the other entry
// points through ctypes, for the calls that a decode step makes once per layer.  Checking some ten tensors
// and converting thirty arguments in Python takes longer than the kernels of a small step run (17 us
// a call measured, 4.3 here).  Same checks, same exceptions; a call returns the library's status.
//
// The module holds no pointer into the library of its own: binding.py hands over the entry points' addresses.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <stdexcept>
#include <string>

namespace {

struct TypeMismatch : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct BadValue : std::runtime_error {
  using std::runtime_error::runtime_error;
};

typedef int (*AppendFn)(const void*, int64_t, const void*, int64_t, const void*, int64_t, int64_t, int64_t, int64_t, int64_t,
                        const int32_t*, const float*, int64_t, int, int, void*, int64_t, void*, int64_t, const int64_t*, int,
                        int64_t, int64_t, void*, void*, float*, float*, float, void*);
typedef int (*GatherFn)(const int64_t*, int64_t, int64_t, int64_t, int, int64_t, int64_t, const void*, const void*,
                        const float*, const float*, void*, int64_t, void*, int64_t, void*);
typedef int (*DecodeFn)(const void*, int64_t, int64_t, int64_t, int64_t, int64_t, int, int64_t, int64_t, const void*,
                        const void*, const float*, const float*, const int32_t*, int64_t, const int32_t*, float, void*,
                        int64_t, void*, size_t, void*);
typedef int (*PrefillFn)(const void*, int64_t, int64_t, const void*, int64_t, const void*, int64_t, int64_t, int64_t, int64_t,
                         int64_t, const int32_t*, const int32_t*, int64_t, int, float, void*, int64_t, void*);

AppendFn g_append = nullptr;
GatherFn g_gather = nullptr;
DecodeFn g_decode = nullptr;
PrefillFn g_prefill = nullptr;

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw TypeMismatch(std::string(name) + " must be a CUDA tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) throw TypeMismatch(std::string(name) + " must be a CUDA tensor");
  return t;
}
const at::Tensor& typed(PyObject* o, at::ScalarType type, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type)
    throw TypeMismatch(std::string(name) + " must be " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  return t;
}
void* address(const at::Tensor& t) { return t.numel() > 0 ? t.data_ptr() : nullptr; }

struct Rows {
  void* p = nullptr;
  int64_t rows = 0, cols = 0, ld = 0;
};
// fp16 rows with unit inner stride, of a single row too: the library takes a row's values as neighbours
Rows rows_of(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 2 || (t.size(0) > 0 && t.size(1) > 1 && t.stride(1) != 1))
    throw BadValue(std::string(name) + " must be 2-D with unit inner stride");
  typed(o, at::kHalf, name);
  Rows r;
  r.p = address(t);
  r.rows = t.size(0);
  r.cols = t.size(1);
  r.ld = r.rows > 1 ? t.stride(0) : std::max<int64_t>(r.cols, 1);
  return r;
}
Rows rows_of(PyObject* o, int64_t rows, int64_t cols, const char* name) {
  const Rows r = rows_of(o, name);
  if (r.rows != rows || r.cols != cols)
    throw BadValue(std::string(name) + " must be [" + std::to_string(rows) + ", " + std::to_string(cols) + "]");
  return r;
}
void* vector_of(PyObject* o, int64_t n, at::ScalarType type, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
    throw BadValue(std::string(name) + " must be a contiguous vector of length " + std::to_string(n));
  return address(typed(o, type, name));
}

struct Cache {
  int bits = 0;
  int64_t pages = 0, heads = 0, page = 0, dim = 0;
  void *k = nullptr, *v = nullptr;
  float *kp = nullptr, *vp = nullptr;
};
float* params_of(PyObject* o, const Cache& c, const char* name) {
  const int64_t groups = c.heads * c.dim / 128;
  const std::string what = std::string(name) + " must be a contiguous float32 [" + std::to_string(c.pages) + ", " +
                           std::to_string(groups) + ", " + std::to_string(c.page) + ", 2] tensor";
  if (o == Py_None) throw BadValue(what);
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != at::kFloat || t.dim() != 4 || t.size(0) != c.pages || t.size(1) != groups || t.size(2) != c.page ||
      t.size(3) != 2 || !t.is_contiguous())
    throw BadValue(what);
  return static_cast<float*>(address(t));
}
Cache cache_of(PyObject* ko, PyObject* vo, PyObject* kpo, PyObject* vpo) {
  const at::Tensor& k = tensor(ko, "k_cache");
  const at::Tensor& v = tensor(vo, "v_cache");
  if (k.dim() != 4 || k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type())
    throw BadValue("k_cache and v_cache must be 4-D tensors of one shape and type");
  if (!k.is_contiguous() || !v.is_contiguous()) throw BadValue("k_cache and v_cache must be contiguous");
  Cache c;
  c.pages = k.size(0);
  c.heads = k.size(1);
  c.page = k.size(2);
  c.k = address(k);
  c.v = address(v);
  if (k.scalar_type() == at::kHalf) {
    c.bits = 16;
    c.dim = k.size(3);
  } else if (k.scalar_type() == at::kByte) {
    c.bits = 4;
    c.dim = 2 * k.size(3);
    c.kp = params_of(kpo, c, "k_params");
    c.vp = params_of(vpo, c, "v_params");
  } else {
    throw TypeMismatch(std::string("k_cache must be float16 or uint8 (4-bit codes), got ") + c10::toString(k.scalar_type()));
  }
  return c;
}

double number(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw TypeMismatch("a number is wanted");
  return x;
}
bool truth(PyObject* o) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw TypeMismatch("a truth value is wanted");
  return x != 0;
}
float scale_of(PyObject* o, int64_t dim) {
  return o == Py_None ? float(1.0 / std::sqrt(double(dim))) : float(number(o));
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Runs a call, with what it throws turned into a Python exception.
template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F call) {
  try {
    if (got != want) throw TypeMismatch("wrong number of arguments");
    return PyLong_FromLong(call());
  } catch (const TypeMismatch& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const BadValue& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

// q, k, v, positions, rotary, slots, k_cache, v_cache, k_params, v_params, q_out, k_out, clip, walsh, interleaved
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> int {
    const Cache c = cache_of(a[6], a[7], a[8], a[9]);
    const at::Tensor& kt = tensor(a[1], "k");
    const int64_t T = kt.dim() > 0 ? kt.size(0) : 0, width = c.heads * c.dim;
    const Rows k = rows_of(a[1], T, width, "k"), v = rows_of(a[2], T, width, "v");
    Rows q, qo, ko;
    int64_t heads = 0;
    if (a[0] != Py_None) {
      if (a[10] == Py_None) throw BadValue("q_out is required with q");
      q = rows_of(a[0], "q");
      heads = c.dim > 0 ? q.cols / c.dim : 0;
      if (q.rows != T || q.cols != heads * c.dim) throw BadValue("q must be [" + std::to_string(T) + ", whole heads]");
      qo = rows_of(a[10], T, q.cols, "q_out");
    }
    if (a[11] != Py_None) ko = rows_of(a[11], T, width, "k_out");
    const at::Tensor& rotary = tensor(a[4], "rotary");
    if (rotary.dim() != 2 || rotary.size(1) != c.dim || !rotary.is_contiguous())
      throw BadValue("rotary must be a contiguous [rows, " + std::to_string(c.dim) + "] tensor");
    typed(a[4], at::kFloat, "rotary");
    const void* positions = vector_of(a[3], T, at::kInt, "positions");
    const void* slots = vector_of(a[5], T, at::kLong, "slots");
    return g_append(q.p, q.ld, k.p, k.ld, v.p, v.ld, T, heads, c.heads, c.dim, static_cast<const int32_t*>(positions),
                    static_cast<const float*>(address(rotary)), rotary.size(0), truth(a[14]), truth(a[13]), qo.p, qo.ld, ko.p,
                    ko.ld, static_cast<const int64_t*>(slots), c.bits, c.pages, c.page, c.k, c.v, c.kp, c.vp,
                    float(number(a[12])), stream());
  });
}

// slots, k_cache, v_cache, k_out, v_out, k_params, v_params
PyObject* kv_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> int {
    const Cache c = cache_of(a[1], a[2], a[5], a[6]);
    const at::Tensor& st = tensor(a[0], "slots");
    const int64_t T = st.dim() > 0 ? st.size(0) : 0;
    const Rows k = rows_of(a[3], T, c.heads * c.dim, "k_out"), v = rows_of(a[4], T, c.heads * c.dim, "v_out");
    const void* slots = vector_of(a[0], T, at::kLong, "slots");
    return g_gather(static_cast<const int64_t*>(slots), T, c.heads, c.dim, c.bits, c.pages, c.page, c.k, c.v, c.kp, c.vp, k.p,
                    k.ld, v.p, v.ld, stream());
  });
}

// q, k_cache, v_cache, block_table, lengths, Y, k_params, v_params, scale, workspace
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> int {
    const Cache c = cache_of(a[1], a[2], a[6], a[7]);
    const Rows q = rows_of(a[0], "q");
    if (q.cols == 0 || c.dim == 0 || q.cols % c.dim != 0)
      throw BadValue("the rows of q must hold whole heads of " + std::to_string(c.dim));
    const Rows y = rows_of(a[5], q.rows, q.cols, "Y");
    const at::Tensor& table = tensor(a[3], "block_table");
    if (table.dim() != 2 || table.size(0) != q.rows || !table.is_contiguous())
      throw BadValue("block_table must be a contiguous [" + std::to_string(q.rows) + ", max_pages] tensor");
    typed(a[3], at::kInt, "block_table");
    const void* lengths = vector_of(a[4], q.rows, at::kInt, "lengths");
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[9] != Py_None) {
      const at::Tensor& w = tensor(a[9], "workspace");
      if (!w.is_contiguous()) throw BadValue("workspace must be contiguous");
      ws = address(w);
      bytes = size_t(w.numel()) * w.element_size();
    }
    return g_decode(q.p, q.ld, q.rows, q.cols / c.dim, c.heads, c.dim, c.bits, c.pages, c.page, c.k, c.v, c.kp, c.vp,
                    static_cast<const int32_t*>(address(table)), table.size(1), static_cast<const int32_t*>(lengths),
                    scale_of(a[8], c.dim), y.p, y.ld, ws, bytes, stream());
  });
}

// q, k, v, cu_q, cu_k, Y, head_dim, causal, scale
PyObject* attn_prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> int {
    const Rows q = rows_of(a[0], "q"), k = rows_of(a[1], "k");
    const Rows v = rows_of(a[2], k.rows, k.cols, "v"), y = rows_of(a[5], q.rows, q.cols, "Y");
    const int64_t dim = PyLong_AsLongLong(a[6]);
    if (dim == -1 && PyErr_Occurred()) throw TypeMismatch("head_dim must be a whole number");
    if (dim <= 0 || q.cols % dim != 0 || k.cols % dim != 0)
      throw BadValue("the rows of q and k must hold whole heads of " + std::to_string(dim));
    const at::Tensor& cq = tensor(a[3], "cu_q");
    const int64_t ends = cq.dim() > 0 ? cq.size(0) : 0;
    if (ends == 0) throw BadValue("cu_q must have at least one entry");
    const void* cu_q = vector_of(a[3], ends, at::kInt, "cu_q");
    const void* cu_k = vector_of(a[4], ends, at::kInt, "cu_k");
    return g_prefill(q.p, q.ld, q.rows, k.p, k.ld, v.p, v.ld, k.rows, q.cols / dim, k.cols / dim, dim,
                     static_cast<const int32_t*>(cu_q), static_cast<const int32_t*>(cu_k), ends - 1, truth(a[7]),
                     scale_of(a[8], dim), y.p, y.ld, stream());
  });
}

// The addresses of the library's four entry points.
PyObject* connect(PyObject*, PyObject* args) {
  unsigned long long append, gather, decode, prefill;
  if (!PyArg_ParseTuple(args, "KKKK", &append, &gather, &decode, &prefill)) return nullptr;
  g_append = reinterpret_cast<AppendFn>(append);
  g_gather = reinterpret_cast<GatherFn>(gather);
  g_decode = reinterpret_cast<DecodeFn>(decode);
  g_prefill = reinterpret_cast<PrefillFn>(prefill);
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"connect", connect, METH_VARARGS, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_append)), METH_FASTCALL, nullptr},
    {"kv_gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(kv_gather)), METH_FASTCALL, nullptr},
    {"attn_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attn_decode)), METH_FASTCALL, nullptr},
    {"attn_prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attn_prefill)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }
