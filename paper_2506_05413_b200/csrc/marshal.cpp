// Argument marshalling of the cache, attention, microscaled and norm calls in native code: what binding.py does for the other entry
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

typedef int (*MxQuantFn)(const void*, int64_t, int64_t, int64_t, int64_t, const float*, int, uint8_t*, uint8_t*, float*, void*);
typedef int (*MxDequantFn)(const uint8_t*, const uint8_t*, const float*, int64_t, int64_t, int64_t, void*, int64_t, void*);
typedef int (*MxLinearFn)(const uint8_t*, const uint8_t*, const float*, int64_t, const uint8_t*, const uint8_t*, const float*,
                          int64_t, int64_t, int64_t, void*, int64_t, void*);
typedef int (*MxGluFn)(const uint8_t*, const uint8_t*, const float*, int64_t, const uint8_t*, const uint8_t*, const float*,
                       const uint8_t*, const uint8_t*, const float*, int64_t, int64_t, int64_t, int, void*, int64_t, uint8_t*,
                       uint8_t*, const float*, void*);
typedef int (*AddNormFn)(const void*, int64_t, const void*, int64_t, int64_t, int64_t, int, const float*, const float*, float,
                         float, const float*, float, void*, int64_t, void*, int64_t, int, float, uint8_t*, uint8_t*, float*, void*);
typedef size_t (*MxScaleBytesFn)(int64_t, int64_t, int64_t);

AppendFn g_append = nullptr;
GatherFn g_gather = nullptr;
DecodeFn g_decode = nullptr;
PrefillFn g_prefill = nullptr;
MxQuantFn g_mx_quant = nullptr;
MxDequantFn g_mx_dequant = nullptr;
MxLinearFn g_mx_linear = nullptr;
MxGluFn g_mx_glu = nullptr;
AddNormFn g_add_norm = nullptr;
MxScaleBytesFn g_mx_scale_bytes = nullptr;

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

// ---- microscaled codes and norms ----

// The work goes to the current device's current stream: its tensors have to be there too.
thread_local int g_device = -1;        // asked for once a call, when a CUDA tensor has been seen
void here(const at::Tensor& t, const char* name) {
  if (g_device < 0) g_device = c10::cuda::current_device();
  if (t.device().index() != g_device)
    throw BadValue(std::string(name) + " is not on the current CUDA device");
}
float* step_of(PyObject* o, int64_t n, const char* name) {
  if (o == Py_None) return nullptr;
  float* p = static_cast<float*>(vector_of(o, n, at::kFloat, name));
  here(THPVariable_Unpack(o), name);
  return p;
}
Rows half_rows(PyObject* o, const char* name) {
  const Rows r = rows_of(o, name);
  here(THPVariable_Unpack(o), name);
  return r;
}
Rows half_rows(PyObject* o, int64_t rows, int64_t cols, const char* name) {
  const Rows r = rows_of(o, rows, cols, name);
  here(THPVariable_Unpack(o), name);
  return r;
}
int64_t whole(PyObject* o, const char* name) {
  const int64_t x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw TypeMismatch(std::string(name) + " must be a whole number");
  if (x != int(x)) throw BadValue(std::string(name) + " is out of range");
  return x;
}

struct Coded {
  uint8_t *q = nullptr, *scale = nullptr;
  int64_t rows = 0, K = 0;
};
uint8_t* codes_of(PyObject* o, int64_t rows, int64_t bytes, const char* name) {
  const at::Tensor& t = typed(o, at::kByte, name);
  here(t, name);
  if (t.dim() != 2 || !t.is_contiguous()) throw BadValue(std::string(name) + " must be a contiguous 2-D uint8 tensor");
  if (bytes >= 0 && (t.size(0) != rows || t.size(1) != bytes))
    throw BadValue(std::string(name) + " must be [" + std::to_string(rows) + ", " + std::to_string(bytes) + "]");
  return static_cast<uint8_t*>(address(t));
}
uint8_t* scales_of(PyObject* o, int64_t rows, int64_t K, int64_t group, const char* name) {
  const at::Tensor& t = typed(o, at::kByte, name);
  here(t, name);
  const int64_t need = int64_t(g_mx_scale_bytes(rows, K, group));
  if (!t.is_contiguous() || t.numel() < need)
    throw BadValue(std::string(name) + " must be a contiguous uint8 tensor of at least " + std::to_string(need) + " bytes");
  return static_cast<uint8_t*>(address(t));
}
Coded coded(PyObject* q, PyObject* scale, int64_t group, const char* q_name, const char* scale_name) {
  Coded c;
  c.q = codes_of(q, 0, -1, q_name);
  const at::Tensor& t = THPVariable_Unpack(q);
  c.rows = t.size(0);
  c.K = 2 * t.size(1);
  c.scale = scales_of(scale, c.rows, c.K, group, scale_name);
  return c;
}

// X, q_out, scale_out, step_out, group, pre, walsh
PyObject* mx_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> int {
    g_device = -1;
    const Rows x = half_rows(a[0], "X");
    const int64_t group = whole(a[4], "group");
    uint8_t* q = codes_of(a[1], x.rows, x.cols / 2, "q_out");
    uint8_t* scale = scales_of(a[2], x.rows, x.cols, group, "scale_out");
    return g_mx_quant(x.p, x.rows, x.cols, x.ld, group, step_of(a[5], x.cols, "pre"), int(whole(a[6], "walsh")), q, scale,
                      step_of(a[3], x.rows, "step_out"), stream());
  });
}

// q, scale, step, Y, group
PyObject* mx_dequant(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> int {
    g_device = -1;
    const int64_t group = whole(a[4], "group");
    const Coded c = coded(a[0], a[1], group, "q", "scale");
    const Rows y = half_rows(a[3], c.rows, c.K, "Y");
    return g_mx_dequant(c.q, c.scale, step_of(a[2], c.rows, "step"), c.rows, c.K, group, y.p, y.ld, stream());
  });
}

// Xq, x_scale, x_step, Wq, w_scale, w_step, Y, group
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> int {
    g_device = -1;
    const int64_t group = whole(a[7], "group");
    const Coded x = coded(a[0], a[1], group, "Xq", "x_scale"), w = coded(a[3], a[4], group, "Wq", "w_scale");
    if (x.K != w.K) throw BadValue("Xq and Wq disagree on K");
    const Rows y = half_rows(a[6], x.rows, w.rows, "Y");
    return g_mx_linear(x.q, x.scale, step_of(a[2], x.rows, "x_step"), x.rows, w.q, w.scale, step_of(a[5], w.rows, "w_step"), w.rows,
                       x.K, group, y.p, y.ld, stream());
  });
}

// Xq, x_scale, x_step, gate_q, gate_scale, gate_step, up_q, up_scale, up_step, h_out, q_out, scale_out, h_step, group, walsh
PyObject* mx_glu(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> int {
    g_device = -1;
    const int64_t group = whole(a[13], "group");
    const Coded x = coded(a[0], a[1], group, "Xq", "x_scale");
    const Coded g = coded(a[3], a[4], group, "gate_q", "gate_scale"), u = coded(a[6], a[7], group, "up_q", "up_scale");
    if (x.K != g.K || x.K != u.K) throw BadValue("Xq, gate_q and up_q disagree on K");
    if (g.rows != u.rows) throw BadValue("gate_q and up_q must have the same shape");
    Rows h;
    uint8_t *q = nullptr, *scale = nullptr;
    if ((a[9] == Py_None) == (a[10] == Py_None)) throw BadValue("one of h_out and q_out is wanted");
    if (a[9] != Py_None) {
      h = half_rows(a[9], x.rows, g.rows, "h_out");
      if (a[11] != Py_None || a[12] != Py_None) throw BadValue("scale_out and h_step go with q_out");
    } else {
      if (a[11] == Py_None) throw BadValue("scale_out is required with q_out");
      if (g.rows % 128 != 0) throw BadValue("codes need a multiple of 128 features");
      q = codes_of(a[10], x.rows, g.rows / 2, "q_out");
      scale = scales_of(a[11], x.rows, g.rows, group, "scale_out");
    }
    return g_mx_glu(x.q, x.scale, step_of(a[2], x.rows, "x_step"), x.rows, g.q, g.scale, step_of(a[5], g.rows, "gate_step"), u.q,
                    u.scale, step_of(a[8], u.rows, "up_step"), g.rows, x.K, group, int(whole(a[14], "walsh")), h.p, h.ld, q, scale,
                    step_of(a[12], x.rows, "h_step"), stream());
  });
}

// y, h, pre_weight, h_out, x_out, q_out, scale_out, step_out, codes, post_norm, post_weight, gate, block_scale,
// residual_scale, eps, clip
PyObject* add_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&]() -> int {
    g_device = -1;
    if (a[0] == Py_None && a[1] == Py_None) throw BadValue("one of y and h is required");
    Rows y, h, ho, xo;
    if (a[0] != Py_None) y = half_rows(a[0], "y");
    if (a[1] != Py_None) h = a[0] != Py_None ? half_rows(a[1], y.rows, y.cols, "h") : half_rows(a[1], "h");
    const int64_t rows = a[0] != Py_None ? y.rows : h.rows, K = a[0] != Py_None ? y.cols : h.cols;
    if (a[3] != Py_None) ho = half_rows(a[3], rows, K, "h_out");
    if (a[4] != Py_None) xo = half_rows(a[4], rows, K, "x_out");
    const int64_t codes = whole(a[8], "codes");
    uint8_t *q = nullptr, *scale = nullptr;
    float* step = nullptr;
    if ((codes == 0 && (a[5] != Py_None || a[7] != Py_None)) || (codes < 16 && a[6] != Py_None))
      throw BadValue("q_out and step_out go with codes, scale_out with microscaled ones");
    if (codes != 0) {
      if (a[5] == Py_None || (codes >= 16 && a[6] == Py_None)) throw BadValue("codes need q_out, and scale_out where they are microscaled");
      q = codes_of(a[5], rows, K / 2, "q_out");
      if (codes >= 16) scale = scales_of(a[6], rows, K, codes, "scale_out");
      step = step_of(a[7], rows, "step_out");
    }
    return g_add_norm(y.p, y.ld, h.p, h.ld, rows, K, truth(a[9]), step_of(a[10], K, "post_weight"), step_of(a[11], K, "gate"),
                      float(number(a[12])), float(number(a[13])), step_of(a[2], K, "pre_weight"), float(number(a[14])), ho.p,
                      ho.ld, xo.p, xo.ld, int(codes), float(number(a[15])), q, scale, step, stream());
  });
}

// The addresses of the entry points for microscaled codes and norms.
PyObject* connect_mx(PyObject*, PyObject* args) {
  unsigned long long quant, dequant, linear, glu, norm, bytes;
  if (!PyArg_ParseTuple(args, "KKKKKK", &quant, &dequant, &linear, &glu, &norm, &bytes)) return nullptr;
  g_mx_quant = reinterpret_cast<MxQuantFn>(quant);
  g_mx_dequant = reinterpret_cast<MxDequantFn>(dequant);
  g_mx_linear = reinterpret_cast<MxLinearFn>(linear);
  g_mx_glu = reinterpret_cast<MxGluFn>(glu);
  g_add_norm = reinterpret_cast<AddNormFn>(norm);
  g_mx_scale_bytes = reinterpret_cast<MxScaleBytesFn>(bytes);
  Py_RETURN_NONE;
}

// The addresses of the cache's and the attention's entry points.
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
    {"connect_mx", connect_mx, METH_VARARGS, nullptr},
    {"mx_quant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx_quant)), METH_FASTCALL, nullptr},
    {"mx_dequant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx_dequant)), METH_FASTCALL, nullptr},
    {"mx_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx_linear)), METH_FASTCALL, nullptr},
    {"mx_glu", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(mx_glu)), METH_FASTCALL, nullptr},
    {"add_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(add_norm)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }
