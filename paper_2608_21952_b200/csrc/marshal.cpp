// Argument marshalling of the Python binding (paper_2608_21952_b200/binding.py): torch tensors and ctypes structures
// to the pointers the C entry points take, the current stream, the call with the interpreter lock released.  No
// arithmetic and no checks beyond the ones a pointer needs (a contiguous CUDA tensor, the right ctypes structure; for the operators
// around the layer, which take their sizes from the tensors and the cache, those too).
// Why native: through ctypes a call with a dozen tensors took 9 to 13 us of host time (0.25 us per tensor for
// its type checks and address, 3.4 us for the stream object) ahead of a launch of 3 us, more than the device time of
// a decode step of one sequence (7 us for its three calls); from here a call takes 3.5 to 4 us, launch included, and
// that decode step 8.1 to 9.3 us, by the machine, instead of 29.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/cuda/CUDAStream.h>

#include <limits>

#include "../../include/ssdi8.h"

namespace {

struct BadArgument {};   // a Python exception is set

// device address of a tensor, 0 for None, or an address given as an integer
void* ptr(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
      PyErr_SetString(PyExc_AssertionError, "tensors must be contiguous CUDA tensors");
      throw BadArgument{};
    }
    return t.data_ptr();
  }
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw BadArgument{};
  return p;
}
template <typename T>
T* ptr_as(PyObject* o) { return static_cast<T*>(ptr(o)); }

size_t nbytes(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a workspace is a tensor");
    throw BadArgument{};
  }
  return THPVariable_Unpack(o).nbytes();
}

long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw BadArgument{};
  return v;
}
// a count or a set of flags of 32 bits: what is beyond them is not cut off
template <typename T>
T integer32(PyObject* o) {
  const long long v = integer(o);
  if (v < (long long)std::numeric_limits<T>::min() || v > (long long)std::numeric_limits<T>::max()) {
    PyErr_SetString(PyExc_OverflowError, "a number of 32 bits is expected");
    throw BadArgument{};
  }
  return (T)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw BadArgument{};
  return (float)v;
}

// The binding's ctypes types, given once at its import (init): a structure of another type, or any other object with a
// buffer, would be read as pointers and sizes that it does not hold.  The errors are those of ctypes' byref and argtypes.
struct Types {
  PyObject *dims = nullptr, *fwd = nullptr, *layer = nullptr, *cache = nullptr, *fp4 = nullptr, *ctypes_base = nullptr, *argument_error = nullptr;
} g_types;

// the memory of a ctypes structure
struct Struct {
  Py_buffer b{};
  Struct(PyObject* o, PyObject* type, size_t bytes) {
    const auto is_a = [o](PyObject* t) { return t != nullptr && PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject*>(t)); };
    if (!is_a(type)) {
      if (is_a(g_types.ctypes_base))
        PyErr_Format(g_types.argument_error, "expected %R instead of %R", type, reinterpret_cast<PyObject*>(Py_TYPE(o)));
      else
        PyErr_Format(PyExc_TypeError, "a ctypes structure is expected, not '%s'", Py_TYPE(o)->tp_name);
      throw BadArgument{};
    }
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw BadArgument{};
    if ((size_t)b.len < bytes) {
      PyBuffer_Release(&b);
      PyErr_SetString(PyExc_TypeError, "wrong argument structure");
      throw BadArgument{};
    }
  }
  ~Struct() { PyBuffer_Release(&b); }
  Struct(const Struct&) = delete;
  Struct& operator=(const Struct&) = delete;
};
struct DimsArg : Struct {
  explicit DimsArg(PyObject* o) : Struct(o, g_types.dims, sizeof(ssdi8_dims_t)) {}
  const ssdi8_dims_t* get() const { return static_cast<const ssdi8_dims_t*>(b.buf); }
};
struct FwdArg : Struct {
  explicit FwdArg(PyObject* o) : Struct(o, g_types.fwd, sizeof(ssdi8_fwd_args_t)) {}
  const ssdi8_fwd_args_t* get() const { return static_cast<const ssdi8_fwd_args_t*>(b.buf); }
};
struct LayerArg : Struct {
  explicit LayerArg(PyObject* o) : Struct(o, g_types.layer, sizeof(ssdi8_layer_args_t)) {}
  const ssdi8_layer_args_t* get() const { return static_cast<const ssdi8_layer_args_t*>(b.buf); }
};

// A cache as cache_of leaves it says what its arrays were laid out for (`heads`: H, P, N, G) and where they live (`device`); a structure
// filled by hand says neither, and its caller answers for both.  A call with other dims would read and write past the arrays: it is
// refused as a tensor of another shape is.
struct BadShape {};
PyObject* const kHeads = PyUnicode_InternFromString("heads");
PyObject* const kDevice = PyUnicode_InternFromString("device");
void on_current_device(PyObject* o, const char* what) {
  PyObject* v = PyObject_GetAttr(o, kDevice);
  if (!v) {
    PyErr_Clear();
    return;
  }
  const long index = PyLong_AsLong(v);
  Py_DECREF(v);
  if (index == -1 && PyErr_Occurred()) throw BadArgument{};
  if (index != c10::cuda::current_device()) {
    PyErr_Format(PyExc_ValueError, "%s lives on another device than the current one", what);
    throw BadArgument{};
  }
}
struct CacheArg : Struct {
  CacheArg(PyObject* o, const ssdi8_dims_t& d) : Struct(o, g_types.cache, sizeof(ssdi8_cache_t)) {
    if (PyObject* h = PyObject_GetAttr(o, kHeads)) {
      const int32_t want[4] = {d.nheads, d.headdim, d.dstate, d.ngroups};
      bool same = PyTuple_Check(h) && PyTuple_GET_SIZE(h) == 4;
      for (int i = 0; same && i < 4; ++i) same = PyLong_AsLong(PyTuple_GET_ITEM(h, i)) == want[i];
      Py_DECREF(h);
      if (PyErr_Occurred()) throw BadArgument{};
      if (!same) throw BadShape{};
    } else {
      PyErr_Clear();
    }
    on_current_device(o, "the cache");
  }
  const ssdi8_cache_t* get() const { return static_cast<const ssdi8_cache_t*>(b.buf); }
};

// a matrix in four bits as fp4_of leaves it, or filled by hand
struct Fp4Arg : Struct {
  Fp4Arg(PyObject* o, const char* what) : Struct(o, g_types.fp4, sizeof(ssdi8_fp4_t)) { on_current_device(o, what); }
  const ssdi8_fp4_t* get() const { return static_cast<const ssdi8_fp4_t*>(b.buf); }
};

// the stream of a call: the current one of the current device for None, else a torch stream object's
void* stream(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
  if (!h) throw BadArgument{};
  void* p = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (p == nullptr && PyErr_Occurred()) throw BadArgument{};
  return p;
}

// Tensors of the operators around the layer.  These take their sizes and strides from the tensors, so the shapes are checked here:
// a wrong one is SSDI8_ERR_SHAPE, as from the library; a wrong element type a TypeError, a tensor of another device than the
// current one (the stream's) a ValueError.
constexpr int kInt8 = -1, kInt32 = -2;   // beside the library's 0 = fp32, 1 = fp16, 2 = bf16
constexpr int kAnyFloat = -3;
struct Tensor {
  const at::Tensor* t = nullptr;
  int dtype = 0;
  explicit operator bool() const { return t != nullptr; }
  void* data() const { return t ? t->data_ptr() : nullptr; }
  template <typename E>
  E* as() const { return static_cast<E*>(data()); }
  int64_t size(int i) const { return t->size(i); }
  int64_t stride(int i) const { return t->stride(i); }
};
// strided: the last axis contiguous, the others free (as the caller reads the strides)
Tensor tensor(PyObject* o, const char* name, int dtype, std::initializer_list<int64_t> shape, bool optional = false, bool strided = false) {
  Tensor r;
  if (o == Py_None && optional) return r;
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: a tensor is expected", name);
    throw BadArgument{};
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || !(strided ? t.dim() > 0 && (t.size(-1) <= 1 || t.stride(-1) == 1) : t.is_contiguous())) {
    PyErr_Format(PyExc_AssertionError, "%s must be a CUDA tensor with %s", name, strided ? "a contiguous last axis" : "contiguous elements");
    throw BadArgument{};
  }
  if (t.device().index() != c10::cuda::current_device()) {
    PyErr_Format(PyExc_ValueError, "%s lives on another device than the current one", name);
    throw BadArgument{};
  }
  const auto st = t.scalar_type();
  r.dtype = st == at::kFloat ? 0 : st == at::kHalf ? 1 : st == at::kBFloat16 ? 2 : st == at::kChar ? kInt8 : st == at::kInt ? kInt32 : -4;
  if (dtype == kAnyFloat ? r.dtype < 0 : r.dtype != dtype) {
    PyErr_Format(PyExc_TypeError, "%s has the wrong element type", name);
    throw BadArgument{};
  }
  if ((size_t)t.dim() != shape.size()) throw BadShape{};
  int i = 0;
  for (int64_t n : shape) {
    if (n >= 0 && t.size(i) != n) throw BadShape{};   // (-1: any)
    ++i;
  }
  r.t = &t;
  return r;
}

// the library call with the interpreter lock released; the status code as a Python integer
template <typename F>
PyObject* call(F f) {
  ssdi8_status_t s;
  Py_BEGIN_ALLOW_THREADS
  s = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(s);
}

// wraps a body that throws BadArgument (exception set) or a C++ exception of torch
template <int N, typename F>
PyObject* entry(Py_ssize_t n, F f) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, n);
    return nullptr;
  }
  try {
    return f();
  } catch (const BadArgument&) {
    return nullptr;
  } catch (const BadShape&) {
    return PyLong_FromLong(SSDI8_ERR_SHAPE);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define ENTRY(NAME, N) PyObject* NAME(PyObject*, PyObject* const* a, Py_ssize_t n) { return entry<N>(n, [&]() -> PyObject*
#define END ); }

ENTRY(init, 7) {   // Dims, FwdArgs, LayerArgs, Cache, Fp4, the base type of ctypes objects, ctypes.ArgumentError
  for (int i = 0; i < 7; ++i) {
    if (!PyType_Check(a[i])) {
      PyErr_SetString(PyExc_TypeError, "a type is expected");
      throw BadArgument{};
    }
    Py_INCREF(a[i]);   // (kept for the life of the process, like the module)
  }
  g_types = {a[0], a[1], a[2], a[3], a[4], a[5], a[6]};
  Py_RETURN_NONE;
} END

ENTRY(quantize_act, 8) {   // inp, R, Ch, I, scale, mode, out, stream
  const float* in = ptr_as<const float>(a[0]);
  const long long R = integer(a[1]), Ch = integer(a[2]), I = integer(a[3]);
  float* scale = ptr_as<float>(a[4]);
  const int mode = (int)integer(a[5]);
  int8_t* out = ptr_as<int8_t>(a[6]);
  void* st = stream(a[7]);
  return call([=] { return ssdi8_quantize_act(in, R, Ch, I, scale, mode, out, st); });
} END

ENTRY(quantize_entry, 13) {   // xBC, dtype, T, D, G, N, s_x, s_B, s_C, xq, Bq, Cq, stream
  const void* in = ptr(a[0]);
  const int dtype = (int)integer(a[1]);
  const long long T = integer(a[2]);
  const int D = (int)integer(a[3]), G = (int)integer(a[4]), N = (int)integer(a[5]);
  const float *sx = ptr_as<const float>(a[6]), *sB = ptr_as<const float>(a[7]), *sC = ptr_as<const float>(a[8]);
  int8_t *xq = ptr_as<int8_t>(a[9]), *Bq = ptr_as<int8_t>(a[10]), *Cq = ptr_as<int8_t>(a[11]);
  void* st = stream(a[12]);
  return call([=] { return ssdi8_quantize_entry(in, dtype, T, D, G, N, sx, sB, sC, xq, Bq, Cq, st); });
} END

ENTRY(chunk_scan_fwd, 5) {   // dims, args, workspace, flags, stream
  DimsArg d(a[0]);
  FwdArg f(a[1]);
  void* ws = ptr(a[2]);
  const size_t nb = nbytes(a[2]);
  const uint32_t flags = (uint32_t)integer(a[3]);
  void* st = stream(a[4]);
  return call([&] { return ssdi8_chunk_scan_fwd(d.get(), f.get(), flags, ws, nb, st); });
} END

ENTRY(chunk_scan_fwd_static, 4) {   // dims, args, flags, stream
  DimsArg d(a[0]);
  FwdArg f(a[1]);
  const uint32_t flags = (uint32_t)integer(a[2]);
  void* st = stream(a[3]);
  return call([&] { return ssdi8_chunk_scan_fwd_static(d.get(), f.get(), flags, st); });
} END

ENTRY(layer_fwd, 5) {   // dims, args, workspace, flags, stream
  DimsArg d(a[0]);
  LayerArg f(a[1]);
  void* ws = ptr(a[2]);
  const size_t nb = nbytes(a[2]);
  const uint32_t flags = (uint32_t)integer(a[3]);
  void* st = stream(a[4]);
  return call([&] { return ssdi8_layer_fwd(d.get(), f.get(), ws, nb, flags, st); });
} END

ENTRY(layer_fwd_host, 5) {   // dims, args, scratch, flags, stream
  DimsArg d(a[0]);
  LayerArg f(a[1]);
  void* ws = ptr(a[2]);
  const size_t nb = nbytes(a[2]);
  const uint32_t flags = (uint32_t)integer(a[3]);
  void* st = stream(a[4]);
  return call([&] { return ssdi8_layer_fwd_host(d.get(), f.get(), ws, nb, flags, st); });
} END

ENTRY(calibrate, 7) {   // dims, args, s_xs, s_cb, s_h, workspace, stream
  DimsArg d(a[0]);
  FwdArg f(a[1]);
  float *sxs = ptr_as<float>(a[2]), *scb = ptr_as<float>(a[3]), *sh = ptr_as<float>(a[4]);
  void* ws = ptr(a[5]);
  const size_t nb = nbytes(a[5]);
  void* st = stream(a[6]);
  return call([&] { return ssdi8_calibrate(d.get(), f.get(), sxs, scb, sh, ws, nb, st); });
} END

ENTRY(mean_correction, 8) {   // y_ref, y_q, R, Ch, eta, corr, workspace, stream
  const float *y = ptr_as<const float>(a[0]), *yq = ptr_as<const float>(a[1]);
  const long long R = integer(a[2]), Ch = integer(a[3]);
  const float eta = real(a[4]);
  float* corr = ptr_as<float>(a[5]);
  void* ws = ptr(a[6]);
  const size_t nb = nbytes(a[6]);
  void* st = stream(a[7]);
  return call([=] { return ssdi8_mean_correction(y, yq, R, Ch, eta, corr, ws, nb, st); });
} END

ENTRY(state_passing, 9) {   // dims, loc, gamma, init_state, prev, final_state, hq, s_h, stream
  DimsArg d(a[0]);
  const float *loc = ptr_as<const float>(a[1]), *gamma = ptr_as<const float>(a[2]), *init = ptr_as<const float>(a[3]);
  float *prev = ptr_as<float>(a[4]), *fin = ptr_as<float>(a[5]);
  int8_t* hq = ptr_as<int8_t>(a[6]);
  const float* sh = ptr_as<const float>(a[7]);
  void* st = stream(a[8]);
  return call([&] { return ssdi8_state_passing(d.get(), loc, gamma, init, prev, fin, hq, sh, st); });
} END

ENTRY(ssd_step, 14) {   // dims, xq, s_x, Bq, s_B, Cq, s_C, dt, A, D, corr, state, y, stream
  DimsArg d(a[0]);
  const int8_t* xq = ptr_as<const int8_t>(a[1]);
  const float* sx = ptr_as<const float>(a[2]);
  const int8_t* Bq = ptr_as<const int8_t>(a[3]);
  const float* sB = ptr_as<const float>(a[4]);
  const int8_t* Cq = ptr_as<const int8_t>(a[5]);
  const float* sC = ptr_as<const float>(a[6]);
  const float *dt = ptr_as<const float>(a[7]), *A = ptr_as<const float>(a[8]), *D = ptr_as<const float>(a[9]),
              *corr = ptr_as<const float>(a[10]);
  float *state = ptr_as<float>(a[11]), *y = ptr_as<float>(a[12]);
  void* st = stream(a[13]);
  return call([&] { return ssdi8_ssd_step(d.get(), xq, sx, Bq, sB, Cq, sC, dt, A, D, corr, state, y, st); });
} END

ENTRY(softplus_dt, 6) {   // dt_raw, dt_bias, rows, H, dt, stream
  const float *raw = ptr_as<const float>(a[0]), *bias = ptr_as<const float>(a[1]);
  const long long rows = integer(a[2]);
  const int H = (int)integer(a[3]);
  float* dt = ptr_as<float>(a[4]);
  void* st = stream(a[5]);
  return call([=] { return ssdi8_softplus_dt(raw, bias, rows, H, dt, st); });
} END

// dims, xBC, weight, bias, s_x, s_B, s_C, xq, Bq, Cq, out, dt_raw, dt_bias, dt, lens, ring, slots, pos, status, flags, stream
ENTRY(conv_fwd, 21) {
  DimsArg d(a[0]);
  const int64_t B = d.get()->batch, L = d.get()->seqlen, H = d.get()->nheads, HP = H * d.get()->headdim,
                GN = (int64_t)d.get()->ngroups * d.get()->dstate, Ch = HP + 2 * GN;
  ssdi8_conv_args_t c = {};
  const Tensor x = tensor(a[1], "xBC", kAnyFloat, {B, L, Ch}, false, true);
  const Tensor w = tensor(a[2], "weight", 0, {Ch, -1});
  const int width = (int)w.size(1);
  c.xBC = x.data(); c.stride_b = x.stride(0); c.stride_t = x.stride(1);
  c.weight = w.as<float>();
  c.bias = tensor(a[3], "bias", 0, {Ch}, true).as<float>();
  c.s_x = tensor(a[4], "s_x", 0, {HP}, true).as<float>();
  c.s_B = tensor(a[5], "s_B", 0, {d.get()->ngroups}, true).as<float>();
  c.s_C = tensor(a[6], "s_C", 0, {d.get()->ngroups}, true).as<float>();
  c.xq = tensor(a[7], "xq", kInt8, {B, L, HP}, true).as<int8_t>();
  c.Bq = tensor(a[8], "Bq", kInt8, {B, L, GN}, true).as<int8_t>();
  c.Cq = tensor(a[9], "Cq", kInt8, {B, L, GN}, true).as<int8_t>();
  c.out = tensor(a[10], "out", x.dtype, {B, L, Ch}, true).data();
  const Tensor raw = tensor(a[11], "dt_raw", x.dtype, {B, L, H}, true, true);
  if (raw) { c.dt_raw = raw.data(); c.dt_stride_b = raw.stride(0); c.dt_stride_t = raw.stride(1); }
  c.dt_bias = tensor(a[12], "dt_bias", 0, {H}, true).as<float>();
  c.dt = tensor(a[13], "dt", 0, {B, L, H}, true).as<float>();
  c.lens = tensor(a[14], "lens", kInt32, {B}, true).as<int32_t>();
  const Tensor ring = tensor(a[15], "ring", x.dtype, {-1, width, Ch}, true);
  if (ring) { c.ring = ring.data(); c.nslots = (int32_t)ring.size(0); }
  c.slots = tensor(a[16], "slots", kInt32, {B}, true).as<int32_t>();
  c.pos = tensor(a[17], "pos", kInt32, {B}, true).as<int32_t>();
  c.status = tensor(a[18], "status", kInt32, {1}, true).as<int32_t>();
  const uint32_t flags = integer32<uint32_t>(a[19]);
  void* st = stream(a[20]);
  return call([&] { return ssdi8_conv_fwd(d.get(), &c, x.dtype, width, flags, st); });
} END

ENTRY(cache_write, 7) {   // dims, cache, slots, pos, state, status, stream
  DimsArg d(a[0]);
  CacheArg c(a[1], *d.get());
  const int64_t B = d.get()->batch;
  const int32_t* slots = tensor(a[2], "slots", kInt32, {B}, true).as<int32_t>();
  const int32_t* pos = tensor(a[3], "pos", kInt32, {B}, true).as<int32_t>();
  const float* state = tensor(a[4], "state", 0, {B, d.get()->nheads, d.get()->headdim, d.get()->dstate}, true).as<float>();
  int32_t* status = tensor(a[5], "status", kInt32, {1}, true).as<int32_t>();
  void* st = stream(a[6]);
  return call([&] { return ssdi8_cache_write(d.get(), c.get(), slots, pos, state, status, st); });
} END

ENTRY(cache_read, 11) {   // dims, cache, slots, first, pos, A, s_x, s_B, state, status, stream
  DimsArg d(a[0]);
  CacheArg c(a[1], *d.get());
  const int64_t B = d.get()->batch, H = d.get()->nheads, P = d.get()->headdim;
  const int32_t* slots = tensor(a[2], "slots", kInt32, {B}, true).as<int32_t>();
  const int32_t* first = tensor(a[3], "first", kInt32, {B}, true).as<int32_t>();
  const int32_t* pos = tensor(a[4], "pos", kInt32, {B}).as<int32_t>();
  const float* A = tensor(a[5], "A", 0, {H}).as<float>();
  const float* s_x = tensor(a[6], "s_x", 0, {H * P}).as<float>();
  const float* s_B = tensor(a[7], "s_B", 0, {d.get()->ngroups}).as<float>();
  float* state = tensor(a[8], "state", 0, {B, H, P, d.get()->dstate}).as<float>();
  int32_t* status = tensor(a[9], "status", kInt32, {1}, true).as<int32_t>();
  void* st = stream(a[10]);
  return call([&] { return ssdi8_cache_read(d.get(), c.get(), slots, first, pos, A, s_x, s_B, state, status, st); });
} END

// dims, cache, xBC, weight, bias, dt_raw, dt_bias, A, D, corr, s_x, s_B, s_C, slots, pos, y, status, flags, stream
ENTRY(token_step, 19) {
  DimsArg d(a[0]);
  CacheArg c(a[1], *d.get());
  const int64_t B = d.get()->batch, H = d.get()->nheads, G = d.get()->ngroups, HP = H * d.get()->headdim,
                Ch = HP + 2 * G * d.get()->dstate;
  const int dtype = c.get()->dtype;
  const uint32_t flags = integer32<uint32_t>(a[17]);
  ssdi8_token_args_t t = {};
  const Tensor x = tensor(a[2], "xBC", dtype, {B, Ch}, false, true), raw = tensor(a[5], "dt_raw", dtype, {B, H}, false, true);
  t.xBC = x.data(); t.stride_b = x.stride(0);
  t.weight = tensor(a[3], "weight", 0, {Ch, c.get()->width}).as<float>();
  t.bias = tensor(a[4], "bias", 0, {Ch}, true).as<float>();
  t.dt_raw = raw.data(); t.dt_stride_b = raw.stride(0);
  t.dt_bias = tensor(a[6], "dt_bias", 0, {H}, true).as<float>();
  t.A = tensor(a[7], "A", 0, {H}).as<float>();
  t.D = tensor(a[8], "D", 0, {H}, true).as<float>();
  t.corr = tensor(a[9], "corr", 0, {HP}, true).as<float>();
  t.s_x = tensor(a[10], "s_x", 0, {HP}).as<float>();
  t.s_B = tensor(a[11], "s_B", 0, {G}).as<float>();
  t.s_C = tensor(a[12], "s_C", 0, {G}).as<float>();
  t.slots = tensor(a[13], "slots", kInt32, {B}, true).as<int32_t>();
  t.pos = tensor(a[14], "pos", kInt32, {B}).as<int32_t>();
  const Tensor y = tensor(a[15], "y", kAnyFloat, {B, HP});
  t.y = y.data();
  t.status = tensor(a[16], "status", kInt32, {1}, true).as<int32_t>();
  // (y's type comes from the tensor: a flag that says another one is refused, with two of them by the library)
  const uint32_t own = y.dtype == 1 ? SSDI8_FLAG_Y_FP16 : y.dtype == 2 ? SSDI8_FLAG_Y_BF16 : 0, fl = flags | own;
  void* st = stream(a[18]);
  if (!own && (flags & (SSDI8_FLAG_Y_FP16 | SSDI8_FLAG_Y_BF16))) return PyLong_FromLong(SSDI8_ERR_UNSUPPORTED);
  return call([&] { return ssdi8_token_step(d.get(), c.get(), &t, fl, st); });
} END

ENTRY(norm_quantize, 9) {   // x, xq, weight, z, groups, eps, scale, static_scale, stream
  const Tensor x = tensor(a[0], "x", kAnyFloat, {-1, -1}, false, true);
  const int64_t T = x.size(0), D = x.size(1);
  if (D > 0x7fffffff) throw BadShape{};
  ssdi8_norm_args_t n = {};
  n.x = x.data(); n.stride_x = x.stride(0);
  n.xq = tensor(a[1], "xq", kInt8, {T, D}).as<int8_t>();
  n.weight = tensor(a[2], "weight", 0, {D}, true).as<float>();
  const Tensor z = tensor(a[3], "z", kAnyFloat, {T, D}, true, true);
  if (z) { n.z = z.data(); n.stride_z = z.stride(0); }
  n.groups = integer32<int32_t>(a[4]);
  n.eps = real(a[5]);
  n.scale = tensor(a[6], "scale", 0, {T}, true).as<float>();
  n.static_scale = tensor(a[7], "static_scale", 0, {1}, true).as<float>();
  n.rows = T; n.width = (int32_t)D;
  void* st = stream(a[8]);
  return call([&] { return ssdi8_norm_quantize(&n, x.dtype, z.dtype, st); });
} END

ENTRY(linear, 10) {   // xq, wq, s_w, out, s_row, bias, residual, act, status, stream
  const Tensor x = tensor(a[0], "xq", kInt8, {-1, -1});
  const int64_t T = x.size(0), K = x.size(1);
  const Tensor w = tensor(a[1], "wq", kInt8, {-1, K});
  const int64_t O = w.size(0);
  if (T > 0x7fffffff || O > 0x7fffffff || K > 0x7fffffff) throw BadShape{};
  ssdi8_linear_args_t l = {};
  l.xq = x.as<int8_t>(); l.wq = w.as<int8_t>();
  l.s_w = tensor(a[2], "s_w", 0, {O}).as<float>();
  const Tensor out = tensor(a[3], "out", kAnyFloat, {T, O}, false, true);
  l.out = out.data(); l.stride_out = out.stride(0);
  l.s_row = tensor(a[4], "s_row", 0, {T}, true).as<float>();
  l.bias = tensor(a[5], "bias", 0, {O}, true).as<float>();
  const Tensor r = tensor(a[6], "residual", out.dtype, {T, O}, true, true);
  if (r) { l.residual = r.data(); l.stride_residual = r.stride(0); }
  l.rows = (int32_t)T; l.outs = (int32_t)O; l.inner = (int32_t)K;
  l.act = integer32<int32_t>(a[7]);
  l.status = tensor(a[8], "status", kInt32, {1}, true).as<int32_t>();
  void* st = stream(a[9]);
  return call([&] { return ssdi8_linear(&l, out.dtype, st); });
} END

ENTRY(fp4_quantize, 4) {   // x, q, status, stream
  Fp4Arg q(a[1], "q");
  const Tensor x = tensor(a[0], "x", kAnyFloat, {q.get()->rows, q.get()->width}, false, true);
  int32_t* status = tensor(a[2], "status", kInt32, {1}, true).as<int32_t>();
  void* st = stream(a[3]);
  return call([&] { return ssdi8_fp4_quantize(x.data(), x.stride(0), x.dtype, q.get(), status, st); });
} END

ENTRY(fp4_dequantize, 3) {   // q, out, stream
  Fp4Arg q(a[0], "q");
  const Tensor out = tensor(a[1], "out", kAnyFloat, {q.get()->rows, q.get()->width}, false, true);
  void* st = stream(a[2]);
  return call([&] { return ssdi8_fp4_dequantize(q.get(), out.data(), out.stride(0), out.dtype, st); });
} END

ENTRY(add_norm_quantize, 11) {   // x, residual, residual_out, weight, eps, xq, scale, static_scale, fp4, status, stream
  const Tensor x = tensor(a[0], "x", kAnyFloat, {-1, -1}, false, true);
  const int64_t T = x.size(0), D = x.size(1);
  if (D > 0x7fffffff) throw BadShape{};
  ssdi8_add_norm_args_t n = {};
  n.x = x.data(); n.stride_x = x.stride(0);
  const Tensor r = tensor(a[1], "residual", kAnyFloat, {T, D}, true, true);
  const Tensor o = tensor(a[2], "residual_out", r ? r.dtype : kAnyFloat, {T, D}, true, true);
  if (r) { n.residual = r.data(); n.stride_residual = r.stride(0); }
  if (o) { n.residual_out = o.data(); n.stride_out = o.stride(0); }
  n.weight = tensor(a[3], "weight", 0, {D}, true).as<float>();
  n.eps = real(a[4]);
  n.xq = tensor(a[5], "xq", kInt8, {T, D}, true).as<int8_t>();
  n.scale = tensor(a[6], "scale", 0, {T}, true).as<float>();
  n.static_scale = tensor(a[7], "static_scale", 0, {1}, true).as<float>();
  n.rows = T; n.width = (int32_t)D;
  n.status = tensor(a[9], "status", kInt32, {1}, true).as<int32_t>();
  const int rdtype = r ? r.dtype : o ? o.dtype : 0;
  void* st = stream(a[10]);
  if (a[8] == Py_None) return call([&] { return ssdi8_add_norm_quantize(&n, x.dtype, rdtype, st); });
  Fp4Arg q(a[8], "fp4");
  n.fp4 = q.get();
  return call([&] { return ssdi8_add_norm_quantize(&n, x.dtype, rdtype, st); });
} END

ENTRY(fp4_linear, 8) {   // x, w, out, bias, residual, act, status, stream
  Fp4Arg x(a[0], "x"), w(a[1], "w");
  const int64_t T = x.get()->rows, O = w.get()->rows;
  ssdi8_fp4_linear_args_t l = {};
  l.x = x.get(); l.w = w.get();
  const Tensor out = tensor(a[2], "out", kAnyFloat, {T, O}, false, true);
  l.out = out.data(); l.stride_out = out.stride(0);
  l.bias = tensor(a[3], "bias", 0, {O}, true).as<float>();
  const Tensor r = tensor(a[4], "residual", out.dtype, {T, O}, true, true);
  if (r) { l.residual = r.data(); l.stride_residual = r.stride(0); }
  l.act = integer32<int32_t>(a[5]);
  l.status = tensor(a[6], "status", kInt32, {1}, true).as<int32_t>();
  void* st = stream(a[7]);
  return call([&] { return ssdi8_fp4_linear(&l, out.dtype, st); });
} END

#undef ENTRY
#undef END

#define METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(init), METHOD(quantize_act), METHOD(quantize_entry), METHOD(chunk_scan_fwd), METHOD(chunk_scan_fwd_static),
                          METHOD(layer_fwd), METHOD(layer_fwd_host), METHOD(calibrate), METHOD(mean_correction),
                          METHOD(state_passing), METHOD(ssd_step), METHOD(softplus_dt), METHOD(conv_fwd), METHOD(cache_write),
                          METHOD(cache_read), METHOD(token_step), METHOD(norm_quantize), METHOD(linear),
                          METHOD(fp4_quantize), METHOD(fp4_dequantize), METHOD(add_norm_quantize), METHOD(fp4_linear), {nullptr, nullptr, 0, nullptr}};
#undef METHOD

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&kModule);
  // the torch whose C++ classes this was compiled against: the binding compares it with the torch that is loaded
  if (m && PyModule_AddStringConstant(m, "TORCH_VERSION", SSDI8_TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
