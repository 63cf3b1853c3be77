// Argument marshalling of the 8-bit layers' and cache's operators for Python: the checks of the
// binding and the call into libfeatfix.so, without building a Python object for each
// size, stride and pointer.  Through ctypes a call of six tensors took 9 us of host time
// on a Grace core; it takes 3, of which the launch is 2 (the kernels of one token take
// 1.5 to 6).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "featfix_ops.h"

namespace {

PyObject* g_error = nullptr;   // featfix.FeatFixError

enum Type { F32, BF16, Q8, I32 };   // element types: those of the C ABI, then 8-bit values and positions

bool is_type(at::ScalarType t, int want) {
  switch (want) {
    case F32: return t == at::kFloat;
    case BF16: return t == at::kBFloat16;
    case Q8: return t == at::kFloat8_e4m3fn || t == at::kByte;
    default: return t == at::kInt;
  }
}

struct Refused {
  int status;
  std::string what;
};
[[noreturn]] void refuse(const std::string& what) { throw Refused{FEATFIX_ERR_INVALID_ARG, what}; }

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is expected");
  return THPVariable_Unpack(o);
}

// The device that this call's launches go to, and its stream for calls that give none:
// asked for once a call (for each tensor it would cost a call of five 0.25 us).
// Guarded by the interpreter's lock.
struct Current {
  int device = -1;
  cudaStream_t stream = nullptr;
  void ask() {
    if (device >= 0) return;
    const c10::cuda::CUDAStream s = c10::cuda::getCurrentCUDAStream();
    device = s.device_index();
    stream = s.stream();
  }
} g_current;

void check(const at::Tensor& t, const char* name, int type) {
  if (!t.is_cuda()) refuse(std::string(name) + " is not on the GPU");
  g_current.ask();
  if (t.get_device() != g_current.device) refuse(std::string(name) + " is on another GPU than the current one");
  if (!is_type(t.scalar_type(), type)) refuse(std::string(name) + ": element type " + c10::toString(t.scalar_type()));
}

// address and row stride of a 2-D tensor of the given size; None is NULL
struct Mat {
  void* p = nullptr;
  long long ld = 0;
};
Mat mat(PyObject* o, const char* name, int type, int64_t rows, int64_t cols) {
  if (o == Py_None) return {};
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols)
    refuse(std::string(name) + ": expected [" + std::to_string(rows) + ", " + std::to_string(cols) + "]");
  check(t, name, type);
  if (cols > 1 && t.stride(1) != 1) refuse(std::string(name) + ": columns must be adjacent");
  // (the stride of a single row says nothing)
  return {t.data_ptr(), rows != 1 ? t.stride(0) : type == Q8 ? (cols + 15) / 16 * 16 : cols};
}

// address of n adjacent elements; None is NULL
void* vec(PyObject* o, const char* name, int type, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, name);
  if (t.numel() != n || !t.is_contiguous()) refuse(std::string(name) + ": expected " + std::to_string(n) + " adjacent elements");
  check(t, name, type);
  return t.data_ptr();
}

struct Dims {
  int64_t rows, cols;
};
Dims dims(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 2) refuse(std::string(name) + ": expected two dimensions");
  return {t.size(0), t.size(1)};
}

// an 8-bit tensor and its scales, in the layout of activations (tile 1) or weights
struct Eight {
  Mat q, scale;
};
Eight eight(PyObject* q, PyObject* scale, int64_t rows, int64_t cols, int tile) {
  if ((q == Py_None) != (scale == Py_None)) refuse("8-bit values and their scales come together");
  const int64_t nb = (cols + 127) / 128;
  return {mat(q, "8-bit values", Q8, rows, cols),
          tile == 1 ? mat(scale, "scales", F32, nb, rows) : mat(scale, "scales", F32, (rows + 127) / 128, nb)};
}

long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw 0;
  return v;
}
int int32(PyObject* o, const char* name) {
  const long long v = integer(o);
  if (v != (int)v) refuse(std::string(name) + " is out of range");
  return (int)v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw 0;
  return v;
}
int dtype(PyObject* o) {
  const int d = int32(o, "dtype");
  if (d != F32 && d != BF16) refuse("dtype is f32 or bf16");
  return d;
}
int size32(int64_t n, const char* name) {
  if (n > 0x7fffffff) refuse(std::string(name) + " is out of range");
  return (int)n;
}
// a stream handle, or PyTorch's current stream for None
void* stream(PyObject* o) {
  if (o == Py_None) {
    g_current.ask();
    return g_current.stream;
  }
  return reinterpret_cast<void*>(integer(o));
}

// An operator without the interpreter's lock: its launch may have to wait for room in the
// stream's queue, and other threads go on meanwhile.
template <class F, class... A> featfix_status run(F op, A... args) {
  struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
  } unlocked;
  return op(args...);
}

// The call, its status and every refusal as a Python exception.
template <class F> PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments are expected, not %zd", want, n);
    return nullptr;
  }
  Refused r = {0, ""};
  g_current.device = -1;
  try {
    const featfix_status s = f();
    if (s == FEATFIX_OK) Py_RETURN_NONE;
    r = {(int)s, featfix_status_string(s)};
  } catch (const Refused& e) {
    r = e;
  } catch (int) {   // a Python exception is set
    return nullptr;
  } catch (const std::exception& e) {
    r = {FEATFIX_ERR_CUDA, e.what()};
  }
  PyObject* v = PyObject_CallFunction(g_error, "is", r.status, r.what.c_str());
  if (v) {
    PyErr_SetObject(g_error, v);
    Py_DECREF(v);
  }
  return nullptr;
}

PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {   // dtype x weight eps resid sum out q scale stream
    const int dt = dtype(a[0]);
    const Dims d = dims(a[1], "x");
    const Mat x = mat(a[1], "x", dt, d.rows, d.cols), r = mat(a[4], "resid", dt, d.rows, d.cols);
    const Mat s = mat(a[5], "sum_out", dt, d.rows, d.cols), o = mat(a[6], "out", dt, d.rows, d.cols);
    const Eight e = eight(a[7], a[8], d.rows, d.cols, 1);
    return run(featfix_op_rms_norm, dt, d.rows, size32(d.cols, "C"), x.p, x.ld, r.p, r.ld, s.p, s.ld,
                               vec(a[2], "weight", dt, d.cols), (float)real(a[3]), o.p, o.ld, e.q.p, e.q.ld,
                               (float*)e.scale.p, e.scale.ld, stream(a[9]));
  });
}

PyObject* quant8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&] {   // dtype x q scale tile stream
    const int dt = dtype(a[0]), tile = int32(a[4], "tile");
    const Dims d = dims(a[1], "x");
    const Mat x = mat(a[1], "x", dt, d.rows, d.cols);
    const Eight e = eight(a[2], a[3], d.rows, d.cols, tile);
    return run(featfix_op_quant8, dt, tile, d.rows, size32(d.cols, "cols"), x.p, x.ld, e.q.p, e.q.ld, (float*)e.scale.p,
                             e.scale.ld, stream(a[5]));
  });
}

PyObject* gemm8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&] {   // dtype a a_scale w w_scale out bias act gate rows_per_batch resid q q_scale stream
    const int dt = dtype(a[0]), rpb = int32(a[9], "rows_per_batch");
    const Dims da = dims(a[1], "a");
    const int64_t M = da.rows, K = da.cols, N = dims(a[3], "w").rows;
    const Eight x = eight(a[1], a[2], M, K, 1), w = eight(a[3], a[4], N, K, 128), q = eight(a[11], a[12], M, N, 1);
    const Mat o = mat(a[5], "out", dt, M, N), r = mat(a[10], "resid", dt, M, N);
    const Mat gate = mat(a[8], "gate", F32, rpb > 0 ? (M + rpb - 1) / rpb : M, N);
    return run(featfix_op_gemm8, dt, size32(M, "M"), size32(N, "N"), size32(K, "K"), x.q.p, x.q.ld, (float*)x.scale.p, x.scale.ld,
                            w.q.p, w.q.ld, (float*)w.scale.p, w.scale.ld, vec(a[6], "bias", dt, N), int32(a[7], "act"),
                            (float*)gate.p, gate.ld, rpb, r.p, r.ld, o.p, o.ld, q.q.p, q.q.ld, (float*)q.scale.p,
                            q.scale.ld, stream(a[13]));
  });
}

PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&] {   // dtype pos axes head_dim q q_out k k_out theta flags q_weight k_weight eps stream
    const int dt = dtype(a[0]), hd = int32(a[3], "head_dim");
    if (hd <= 0) refuse("head_dim is positive");
    int axes[8];
    const Py_ssize_t na = PySequence_Size(a[2]);
    if (na < 0) throw 0;
    if (na < 1 || na > 8) refuse("one to eight axes");
    for (Py_ssize_t i = 0; i < na; ++i) {
      PyObject* v = PySequence_GetItem(a[2], i);
      if (!v) throw 0;
      const long long w = PyLong_AsLongLong(v);
      Py_DECREF(v);
      if (w == -1 && PyErr_Occurred()) throw 0;
      if (w != (int)w) refuse("an axis' width is out of range");
      axes[i] = (int)w;
    }
    const int64_t rows = dims(a[1], "pos").cols;
    const Mat pos = mat(a[1], "pos", I32, na, rows);
    struct Side {
      Mat x, out;
      int heads;
    } s[2] = {};
    const char* names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
    for (int i = 0; i < 2; ++i) {
      if (a[4 + 2 * i] == Py_None) continue;
      const int64_t width = dims(a[4 + 2 * i], names[i][0]).cols;
      if (width % hd) refuse(std::string(names[i][0]) + ": its columns are no whole number of heads");
      s[i] = {mat(a[4 + 2 * i], names[i][0], dt, rows, width), mat(a[5 + 2 * i], names[i][1], dt, rows, width),
              size32(width / hd, "heads")};
    }
    return run(featfix_op_rope, dt, rows, hd, (int)na, axes, (const int*)pos.p, pos.ld, real(a[8]), (unsigned)int32(a[9], "flags"),
                           s[0].x.p, s[0].x.ld, s[0].heads, vec(a[10], "q_weight", dt, hd), s[0].out.p, s[0].out.ld, s[1].x.p,
                           s[1].x.ld, s[1].heads, vec(a[11], "k_weight", dt, hd), s[1].out.p, s[1].out.ld,
                           (float)real(a[12]), stream(a[13]));
  });
}

// The cache's values or scales: base address and the strides of page, slot and head, of
// sizes that the first tensor of a cache sets.
struct Pool {
  void* p = nullptr;
  long long stride[3] = {0, 0, 0};
};
Pool pool(PyObject* o, const char* name, int type, const int64_t (&size)[4]) {
  const at::Tensor& t = tensor(o, name);
  const int64_t dims = type == Q8 ? 4 : 3;
  bool same = t.dim() == dims;
  for (int64_t i = 0; same && i < dims; ++i) same = t.size(i) == size[i];
  if (!same) {
    std::string want;
    for (int64_t i = 0; i < dims; ++i) want += (i ? ", " : "") + std::to_string(size[i]);
    refuse(std::string(name) + ": expected [" + want + "]");
  }
  check(t, name, type);
  if (type == Q8 && size[3] > 1 && t.stride(3) != 1) refuse(std::string(name) + ": a head's columns must be adjacent");
  Pool p;
  p.p = t.data_ptr();
  for (int i = 0; i < 3; ++i) p.stride[i] = t.stride(i);
  return p;
}

// (k8, k_scale, v8, v_scale), the page table and the lengths
featfix_kv_cache kv_cache(PyObject* cache, PyObject* table, PyObject* lens) {
  if (!PyTuple_Check(cache) || PyTuple_GET_SIZE(cache) != 4) refuse("cache: expected (k8, k_scale, v8, v_scale)");
  const at::Tensor& k8 = tensor(PyTuple_GET_ITEM(cache, 0), "k8");
  if (k8.dim() != 4) refuse("k8: expected [pages, page size, heads, head_dim]");
  const int64_t size[4] = {k8.size(0), k8.size(1), k8.size(2), k8.size(3)};
  static const char* names[4] = {"k8", "k_scale", "v8", "v_scale"};
  Pool p[4];
  for (int i = 0; i < 4; ++i) p[i] = pool(PyTuple_GET_ITEM(cache, i), names[i], i & 1 ? F32 : Q8, size);
  featfix_kv_cache c = {};
  c.k = p[0].p, c.k_scale = (float*)p[1].p, c.v = p[2].p, c.v_scale = (float*)p[3].p;
  for (int i = 0; i < 3; ++i) {
    c.k_stride[i] = p[0].stride[i], c.k_scale_stride[i] = p[1].stride[i];
    c.v_stride[i] = p[2].stride[i], c.v_scale_stride[i] = p[3].stride[i];
  }
  c.pages = size32(size[0], "pages"), c.page_size = size32(size[1], "page size");
  c.heads = size32(size[2], "heads"), c.head_dim = size32(size[3], "head_dim");
  const Dims d = dims(table, "table");
  const Mat t = mat(table, "table", I32, d.rows, d.cols);
  c.table = (const int*)t.p, c.ld_table = t.ld;
  c.seqs = size32(d.rows, "sequences"), c.table_pages = size32(d.cols, "pages of the table");
  c.lens = (const int*)vec(lens, "lens", I32, d.rows);
  return c;
}

template <class F> PyObject* kv_rows(PyObject* const* a, Py_ssize_t n, F op) {
  return guarded(n, 8, [&] {   // dtype cache table lens k v row_start stream
    const int dt = dtype(a[0]);
    const featfix_kv_cache c = kv_cache(a[1], a[2], a[3]);
    const int64_t rows = dims(a[4], "k").rows, width = (int64_t)c.heads * c.head_dim;
    const Mat k = mat(a[4], "k", dt, rows, width), v = mat(a[5], "v", dt, rows, width);
    return run(op, dt, &c, (long long)rows, (const int*)vec(a[6], "row_start", I32, c.seqs + 1ll), k.p, k.ld, v.p, v.ld,
               stream(a[7]));
  });
}
PyObject* kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) { return kv_rows(a, n, featfix_op_kv_write); }
PyObject* kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) { return kv_rows(a, n, featfix_op_kv_read); }

PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {   // dtype cache table lens q out workspace scale window lse stream
    const int dt = dtype(a[0]);
    const featfix_kv_cache c = kv_cache(a[1], a[2], a[3]);
    const int64_t width = dims(a[4], "q").cols;
    if (c.head_dim == 0 || width % c.head_dim) refuse("q: its columns are no whole number of heads");
    const int heads = size32(width / c.head_dim, "heads");
    const Mat q = mat(a[4], "q", dt, c.seqs, width), o = mat(a[5], "out", dt, c.seqs, width);
    const Mat lse = mat(a[9], "lse", F32, c.seqs, heads);
    if (c.seqs > 1 && lse.p && lse.ld != heads) refuse("lse: rows must be adjacent");
    void* ws = nullptr;
    size_t bytes = 0;
    if (a[6] != Py_None) {
      const at::Tensor& t = tensor(a[6], "workspace");
      if (!t.is_contiguous()) refuse("workspace: expected adjacent elements");
      if (!t.is_cuda()) refuse("workspace is not on the GPU");
      g_current.ask();
      if (t.get_device() != g_current.device) refuse("workspace is on another GPU than the current one");
      ws = t.data_ptr();
      bytes = t.nbytes();
    }
    return run(featfix_op_kv_attention, dt, &c, q.p, q.ld, heads, (float)real(a[7]), int32(a[8], "window"), o.p, o.ld,
               (float*)lse.p, ws, bytes, stream(a[10]));
  });
}

PyObject* block_norms(PyObject*, PyObject* const* a, Py_ssize_t n) {
  // dtype y x eps flags weight_after resid_scale gate sum weight shift scale rows_per_batch out q q_scale stream
  return guarded(n, 17, [&] {
    const int dt = dtype(a[0]), rpb = int32(a[12], "rows_per_batch");
    const Dims d = dims(a[1], "y");
    const Mat y = mat(a[1], "y", dt, d.rows, d.cols), x = mat(a[2], "x", dt, d.rows, d.cols);
    const Mat sum = mat(a[8], "sum_out", dt, d.rows, d.cols), o = mat(a[13], "out", dt, d.rows, d.cols);
    const Eight e = eight(a[14], a[15], d.rows, d.cols, 1);
    const int64_t samples = rpb > 0 ? (d.rows + rpb - 1) / rpb : d.rows;
    const Mat gate = mat(a[7], "gate", F32, samples, d.cols), shift = mat(a[10], "shift", F32, samples, d.cols);
    const Mat scale = mat(a[11], "scale", F32, samples, d.cols);
    return run(featfix_op_block_norms, dt, d.rows, size32(d.cols, "C"), (unsigned)int32(a[4], "flags"), (float)real(a[3]),
               y.p, y.ld, vec(a[5], "weight_after", dt, d.cols), (const float*)gate.p, gate.ld, x.p, x.ld, (float)real(a[6]),
               sum.p, sum.ld, vec(a[9], "weight", dt, d.cols), (const float*)scale.p, scale.ld, (const float*)shift.p,
               shift.ld, rpb, o.p, o.ld, e.q.p, e.q.ld, (float*)e.scale.p, e.scale.ld, stream(a[16]));
  });
}

PyObject* set_error(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XDECREF(g_error);
  g_error = type;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"rms_norm", (PyCFunction)(void (*)())rms_norm, METH_FASTCALL, nullptr},
    {"quant8", (PyCFunction)(void (*)())quant8, METH_FASTCALL, nullptr},
    {"gemm8", (PyCFunction)(void (*)())gemm8, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)())rope, METH_FASTCALL, nullptr},
    {"kv_write", (PyCFunction)(void (*)())kv_write, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void (*)())kv_read, METH_FASTCALL, nullptr},
    {"kv_attention", (PyCFunction)(void (*)())kv_attention, METH_FASTCALL, nullptr},
    {"block_norms", (PyCFunction)(void (*)())block_norms, METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops8", "Marshalling of the 8-bit layer operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops8(void) { return PyModule_Create(&module); }
