// Python side of the block operators (include/compact_block.h): takes torch tensors, checks them, allocates what the caller did
// not bring, and calls the C ABI on the tensors' device and torch's current stream.  The calls of a decoding step take a
// few microseconds on the GPU; marshalled by ctypes they took 20 to 28 in Python, here they take 4 to 8, the longest a norm whose four
// outputs are allocated (a torch addition takes 4 to 6, an allocation of a tensor 0.7).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/compact_block.h"

namespace {

// The library is opened by path, the same file that the ctypes binding has loaded.
struct Api {
  decltype(&compact_quantize_rows) quantize_rows;
  decltype(&compact_quantize_blocks) quantize_blocks;
  decltype(&compact_rms_norm_fwd) rms_norm_fwd;
  decltype(&compact_rms_norm_bwd_workspace_bytes) rms_norm_bwd_workspace_bytes;
  decltype(&compact_rms_norm_bwd) rms_norm_bwd;
  decltype(&compact_rotary_apply) rotary_apply;
  decltype(&compact_fp8_product_run) fp8_product_run;
} api;
PyObject* error_class = nullptr;      // binding.CompactError

struct Refused {
  int code;
  const char* where;
};

void must(bool ok, int code, const char* where) {
  if (!ok) throw Refused{code, where};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) throw torch::TypeError("expected a torch tensor");
  return THPVariable_Unpack(o);
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
template <class T>
T* address(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw python_error();
  return static_cast<T*>(p);
}

int float_code(const at::Tensor& t, const char* where) {
  if (t.scalar_type() == at::kBFloat16) return COMPACT_BF16;
  if (t.scalar_type() == at::kFloat) return COMPACT_F32;
  throw Refused{COMPACT_ERR_DTYPE, where};
}
at::ScalarType float_type(int64_t code) { return code == COMPACT_BF16 ? at::kBFloat16 : at::kFloat; }
int fp8_code(const at::Tensor& t, const char* where) {
  if (t.scalar_type() == at::kFloat8_e4m3fn) return COMPACT_E4M3;
  if (t.scalar_type() == at::kFloat8_e5m2) return COMPACT_E5M2;
  throw Refused{COMPACT_ERR_DTYPE, where};
}
at::ScalarType fp8_type(int64_t code) { return code == COMPACT_E4M3 ? at::kFloat8_e4m3fn : at::kFloat8_e5m2; }

// One call: its name, the device of its first tensor (made current), that device's current stream.
struct Call {
  const char* where;
  c10::Device device;
  c10::cuda::CUDAGuard guard;
  Call(const at::Tensor& first, const char* name) : where(name), device(checked(first, name)), guard(device) {}
  static c10::Device checked(const at::Tensor& t, const char* name) {
    must(t.is_cuda(), COMPACT_ERR_INVALID_ARG, name);
    return t.device();
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(device.index()).stream(); }
  void here(const at::Tensor& t, at::ScalarType type) const {
    must(t.is_cuda() && t.device() == device, COMPACT_ERR_INVALID_ARG, where);
    must(t.scalar_type() == type, COMPACT_ERR_DTYPE, where);
  }
  // rows x cols with neighbouring columns: its pitch (of a single row any legal number, since it is never used)
  int64_t matrix(const at::Tensor& t, int64_t rows, int64_t cols, at::ScalarType type) const {
    here(t, type);
    must(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols, COMPACT_ERR_SHAPE, where);
    must(cols <= 1 || t.stride(1) == 1, COMPACT_ERR_INVALID_ARG, where);
    return rows > 1 ? t.stride(0) : (cols + 15) / 16 * 16;
  }
  void* vector(const at::Tensor& t, int64_t n, at::ScalarType type) const {
    here(t, type);
    must(t.dim() == 1 && t.size(0) == n, COMPACT_ERR_SHAPE, where);
    must(n <= 1 || t.stride(0) == 1, COMPACT_ERR_INVALID_ARG, where);
    return t.data_ptr();
  }
  // scales of a rows x cols matrix: their pitch in rows
  int64_t scales(const at::Tensor& s, int64_t rows, int64_t cols) const {
    here(s, at::kFloat8_e8m0fnu);
    const int64_t groups = (cols + 511) / 512;
    must(s.dim() == 3 && s.size(0) == groups && s.size(1) == rows && s.size(2) == 4, COMPACT_ERR_SHAPE, where);
    must(s.stride(2) == 1 && (rows <= 1 || s.stride(1) == 4) && (groups <= 1 || s.stride(0) % 4 == 0), COMPACT_ERR_INVALID_ARG, where);
    return groups > 1 ? s.stride(0) / 4 : (rows > 1 ? rows : 1);
  }
  at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type) const {
    return at::Tensor(at::detail::empty_cuda(sizes, type, device, c10::nullopt));
  }
  // a matrix whose rows start on 16-byte boundaries; of 8 bits on 128, the span of a copied tile's row, which otherwise straddles two
  // (2359 x 4248 x 3760: 33 us against 42; 77 tokens 8.5 against 14)
  at::Tensor new_matrix(int64_t rows, int64_t cols, at::ScalarType type) const {
    const int64_t size = (int64_t)c10::elementSize(type), unit = size == 1 && cols > 128 ? 128 : 16 / size, pitch = (cols + unit - 1) / unit * unit;
    at::Tensor t = empty({rows, pitch}, type);
    return pitch == cols ? t : t.narrow(1, 0, cols);
  }
  at::Tensor new_scales(int64_t rows, int64_t cols) const { return empty({(cols + 511) / 512, rows, 4}, at::kFloat8_e8m0fnu); }
};

// The tensor passed in, or a new one.
template <class Make>
at::Tensor given_or(PyObject* o, Make make) {
  return o == Py_None ? make() : tensor(o);
}

// Tensors that the caller brought and the call has written: autograd must not take what it saved of them for what they are now.
template <class... P>
void written(P*... o) {
  const auto one = [](PyObject* p) {
    if (p == Py_None) return;
    const at::Tensor& t = tensor(p);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  };
  (one(o), ...);
}

// Without the interpreter's lock: a launch may wait for room in the stream.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class F>
void run(const char* where, F f) {
  int code;
  {
    const Unlocked unlocked;
    code = f();
  }
  must(code == COMPACT_OK, code, where);
}

PyObject* refuse(const Refused& r) {
  PyObject* e = PyObject_CallFunction(error_class, "is", r.code, r.where);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  return nullptr;
}

#define ENTRY(name, count)                                                          \
  PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n) {                     \
    HANDLE_TH_ERRORS                                                                \
    if (n != count || !error_class) throw torch::TypeError(#name ": wrong number of arguments, or no open library"); \
    try {                                                                           \
      return name##_impl(a);                                                        \
    } catch (const Refused& r) {                                                    \
      return refuse(r);                                                             \
    }                                                                               \
    END_HANDLE_TH_ERRORS                                                            \
  }

PyObject* wrap(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }
template <class... T>
PyObject* tuple(const T&... t) {
  PyObject* out = PyTuple_New(sizeof...(t));
  if (!out) throw python_error();
  Py_ssize_t i = 0;
  (PyTuple_SET_ITEM(out, i++, wrap(t)), ...);
  return out;
}

// (x, fp8, data or None, scales or None) -> (data, scales)
PyObject* quantize_rows_impl(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  const Call c(x, "compact_quantize_rows");
  must(x.dim() == 2, COMPACT_ERR_SHAPE, c.where);
  const int64_t rows = x.size(0), cols = x.size(1);
  const int code = float_code(x, c.where);
  const int64_t fp8 = integer(a[1]);
  const at::ScalarType type = fp8_type(fp8);
  const int64_t ldx = c.matrix(x, rows, cols, x.scalar_type());
  const at::Tensor q = given_or(a[2], [&] { return c.new_matrix(rows, cols, type); });
  const at::Tensor s = given_or(a[3], [&] { return c.new_scales(rows, cols); });
  const int64_t ldq = c.matrix(q, rows, cols, type), lds = c.scales(s, rows, cols);
  run(c.where, [&] {
    return api.quantize_rows(code, rows, cols, x.data_ptr(), ldx, (int)fp8, q.data_ptr(), ldq, s.data_ptr(), lds, c.stream());
  });
  written(a[2], a[3]);
  return tuple(q, s);
}
ENTRY(quantize_rows, 4)

// (x, fp8, data, scales, transpose, data_t, scales_t) -> (data, scales, data_t, scales_t)
PyObject* quantize_blocks_impl(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  const Call c(x, "compact_quantize_blocks");
  must(x.dim() == 2, COMPACT_ERR_SHAPE, c.where);
  const int64_t rows = x.size(0), cols = x.size(1);
  const int code = float_code(x, c.where);
  const int64_t fp8 = integer(a[1]);
  const at::ScalarType type = fp8_type(fp8);
  const int64_t ldx = c.matrix(x, rows, cols, x.scalar_type());
  const at::Tensor q = given_or(a[2], [&] { return c.new_matrix(rows, cols, type); });
  const at::Tensor s = given_or(a[3], [&] { return c.new_scales(rows, cols); });
  const int64_t ldq = c.matrix(q, rows, cols, type), lds = c.scales(s, rows, cols);
  at::Tensor qt, st;
  int64_t ldqt = 0, ldst = 0;
  if (integer(a[4]) != 0 || a[5] != Py_None) {
    qt = given_or(a[5], [&] { return c.new_matrix(cols, rows, type); });
    st = given_or(a[6], [&] { return c.new_scales(cols, rows); });
    if (rows > 0) ldqt = c.matrix(qt, cols, rows, type), ldst = c.scales(st, cols, rows);
  }
  const bool both = qt.defined() && rows > 0;
  run(c.where, [&] {
    return api.quantize_blocks(code, rows, cols, x.data_ptr(), ldx, (int)fp8, q.data_ptr(), ldq, s.data_ptr(), lds, both ? qt.data_ptr() : nullptr, ldqt,
                               both ? st.data_ptr() : nullptr, ldst, c.stream());
  });
  written(a[2], a[3], a[5], a[6]);
  return tuple(q, s, qt, st);
}
ENTRY(quantize_blocks, 7)

// (dtype code, n, eps, x, weight, residual, h, want_y, y, want_fp8, fp8, data, scales) -> (h, y, rstd, data, scales)
PyObject* rms_norm_fwd_impl(PyObject* const* a) {
  const int64_t code = integer(a[0]), n = integer(a[1]);
  const double eps = PyFloat_AsDouble(a[2]);
  const at::Tensor& x = tensor(a[3]);
  const Call c(x, "compact_rms_norm_fwd");
  const at::ScalarType type = float_type(code);
  must(x.dim() == 2, COMPACT_ERR_SHAPE, c.where);
  const int64_t tokens = x.size(0), ldx = c.matrix(x, tokens, n, type);
  const void* w = c.vector(tensor(a[4]), n, type);
  at::Tensor h = x, y, q, s;
  const void* res = nullptr;
  void *hp = nullptr, *yp = nullptr, *qp = nullptr, *sp = nullptr;
  int64_t ldr = 0, ldh = 0, ldy = 0, ldq = 0, lds = 0;
  if (a[5] != Py_None) {
    const at::Tensor& r = tensor(a[5]);
    ldr = c.matrix(r, tokens, n, type);
    res = r.data_ptr();
    h = given_or(a[6], [&] { return c.new_matrix(tokens, n, type); });
    ldh = c.matrix(h, tokens, n, type);
    hp = h.data_ptr();
  } else {
    must(a[6] == Py_None, COMPACT_ERR_INVALID_ARG, c.where);      // without a residual h is x itself
  }
  if (a[8] != Py_None || integer(a[7])) {
    y = given_or(a[8], [&] { return c.new_matrix(tokens, n, type); });
    ldy = c.matrix(y, tokens, n, type);
    yp = y.data_ptr();
  }
  int fp8 = COMPACT_E4M3;
  if (a[11] != Py_None || integer(a[9])) {
    const int64_t wanted = integer(a[10]);
    q = given_or(a[11], [&] { return c.new_matrix(tokens, n, fp8_type(wanted)); });
    s = given_or(a[12], [&] { return c.new_scales(tokens, n); });
    fp8 = fp8_code(q, c.where);
    ldq = c.matrix(q, tokens, n, q.scalar_type());
    lds = c.scales(s, tokens, n);
    qp = q.data_ptr();
    sp = s.data_ptr();
  }
  const at::Tensor rstd = c.empty({tokens}, at::kFloat);
  run(c.where, [&] {
    return api.rms_norm_fwd((int)code, tokens, (int32_t)n, (float)eps, x.data_ptr(), ldx, res, ldr, w, hp, ldh, yp, ldy, (float*)rstd.data_ptr(), fp8, qp,
                            ldq, sp, lds, c.stream());
  });
  written(a[6], a[8], a[11], a[12]);
  return tuple(h, y, rstd, q, s);
}
ENTRY(rms_norm_fwd, 13)

// (dtype code, n, dy, h, weight, rstd, residual_grad, need_dx, dx, need_dweight, dweight, accumulate) -> (dx, dweight)
PyObject* rms_norm_bwd_impl(PyObject* const* a) {
  const int64_t code = integer(a[0]), n = integer(a[1]);
  const at::Tensor &dy = tensor(a[2]), &h = tensor(a[3]);
  const Call c(dy, "compact_rms_norm_bwd");
  const at::ScalarType type = float_type(code);
  must(dy.dim() == 2, COMPACT_ERR_SHAPE, c.where);
  const int64_t tokens = dy.size(0), lddy = c.matrix(dy, tokens, n, type), ldh = c.matrix(h, tokens, n, type);
  const void *w = c.vector(tensor(a[4]), n, type), *rstd = c.vector(tensor(a[5]), tokens, at::kFloat);
  const void* res = nullptr;
  void *dxp = nullptr, *wsp = nullptr;
  float* dwp = nullptr;
  int64_t ldr = 0, lddx = 0;
  size_t ws_bytes = 0;
  at::Tensor dx, dw, ws;
  if (a[6] != Py_None) {
    const at::Tensor& r = tensor(a[6]);
    ldr = c.matrix(r, tokens, n, type);
    res = r.data_ptr();
  }
  if (a[8] != Py_None || integer(a[7])) {
    dx = given_or(a[8], [&] { return c.new_matrix(tokens, n, type); });
    lddx = c.matrix(dx, tokens, n, type);
    dxp = dx.data_ptr();
  }
  const bool accumulate = integer(a[11]) != 0;
  if (a[10] != Py_None || integer(a[9])) {
    must(a[10] != Py_None || !accumulate, COMPACT_ERR_INVALID_ARG, c.where);      // nothing to accumulate to
    dw = given_or(a[10], [&] { return c.empty({n}, at::kFloat); });
    dwp = (float*)c.vector(dw, n, at::kFloat);
    ws_bytes = api.rms_norm_bwd_workspace_bytes((int)code, tokens, (int32_t)n);
    if (ws_bytes) {
      ws = c.empty({(int64_t)ws_bytes}, at::kByte);
      wsp = ws.data_ptr();
    }
  }
  run(c.where, [&] {
    return api.rms_norm_bwd((int)code, tokens, (int32_t)n, dy.data_ptr(), lddy, h.data_ptr(), ldh, w, (const float*)rstd, res, ldr, dxp, lddx, dwp, accumulate,
                            wsp, ws_bytes, c.stream());
  });
  written(a[8], a[10]);
  return tuple(dx, dw);
}
ENTRY(rms_norm_bwd, 12)

// (handle, head_dim, q, k, positions, first_position, back, q_out, k_out) -> (q_out, k_out)
PyObject* rotary_apply_impl(PyObject* const* a) {
  const auto* handle = address<const compact_rotary_t>(a[0]);
  const int64_t d = integer(a[1]);
  const at::Tensor& q = tensor(a[2]);
  const Call c(q, "compact_rotary_apply");
  must(q.dim() == 3, COMPACT_ERR_SHAPE, c.where);
  const int code = float_code(q, c.where);
  const at::ScalarType type = q.scalar_type();
  const int64_t tokens = q.size(0), heads = q.size(1);
  struct Strides {
    int64_t token, head;
  };
  const auto strides = [&](const at::Tensor& t, int64_t h) {
    c.here(t, type);
    must(t.dim() == 3 && t.size(0) == tokens && t.size(1) == h && t.size(2) == d, COMPACT_ERR_SHAPE, c.where);
    must(t.stride(2) == 1, COMPACT_ERR_INVALID_ARG, c.where);
    // a stride that is never used must not cost the wide loads
    return Strides{tokens > 1 ? t.stride(0) : 0, h > 1 ? t.stride(1) : 0};
  };
  const Strides qs = strides(q, heads);
  const at::Tensor qo = given_or(a[7], [&] { return c.empty(q.sizes(), type); });
  const Strides qos = strides(qo, heads);
  at::Tensor k, ko;
  Strides ks{0, 0}, kos{0, 0};
  int64_t kv = 0;
  if (a[3] != Py_None) {
    k = tensor(a[3]);
    must(k.dim() == 3, COMPACT_ERR_SHAPE, c.where);
    kv = k.size(1);
    ks = strides(k, kv);
    ko = given_or(a[8], [&] { return c.empty(k.sizes(), type); });
    kos = strides(ko, kv);
  }
  const void* pos = nullptr;
  int bits = 64;
  if (a[4] != Py_None) {
    const at::Tensor& p = tensor(a[4]);
    must(p.scalar_type() == at::kLong || p.scalar_type() == at::kInt, COMPACT_ERR_DTYPE, c.where);
    pos = c.vector(p, tokens, p.scalar_type());
    bits = p.scalar_type() == at::kLong ? 64 : 32;
  }
  const int64_t first = integer(a[5]);
  const int back = (int)integer(a[6]);
  run(c.where, [&] {
    return api.rotary_apply(handle, code, tokens, (int32_t)heads, (int32_t)kv, q.data_ptr(), qs.token, qs.head, kv ? k.data_ptr() : nullptr, ks.token,
                            ks.head, pos, bits, first, back, qo.data_ptr(), qos.token, qos.head, kv ? ko.data_ptr() : nullptr, kos.token, kos.head,
                            c.stream());
  });
  written(a[7], a[8]);
  return tuple(qo, ko);
}
ENTRY(rotary_apply, 9)

// (handle, A, A's scales, B, B's scales, out or None, dtype code) -> out
PyObject* fp8_product_impl(PyObject* const* a) {
  auto* handle = address<compact_fp8_product_t>(a[0]);
  const at::Tensor &A = tensor(a[1]), &sa = tensor(a[2]), &B = tensor(a[3]), &sb = tensor(a[4]);
  const Call c(A, "compact_fp8_product_run");
  must(A.dim() == 2 && B.dim() == 2 && A.size(1) == B.size(1), COMPACT_ERR_SHAPE, c.where);
  const int64_t M = A.size(0), K = A.size(1), N = B.size(0);
  const at::Tensor out = given_or(a[5], [&] { return c.new_matrix(M, N, float_type(integer(a[6]))); });
  const int at_ = fp8_code(A, c.where), bt = fp8_code(B, c.where), ct = float_code(out, c.where);
  const int64_t lda = c.matrix(A, M, K, A.scalar_type()), ldb = c.matrix(B, N, K, B.scalar_type()), ldc = c.matrix(out, M, N, out.scalar_type());
  const int64_t la = c.scales(sa, M, K), lb = c.scales(sb, N, K);
  run(c.where, [&] {
    return api.fp8_product_run(handle, M, N, K, at_, A.data_ptr(), lda, sa.data_ptr(), la, bt, B.data_ptr(), ldb, sb.data_ptr(), lb, ct, out.data_ptr(), ldc,
                               c.stream());
  });
  written(a[5]);
  return wrap(out);
}
ENTRY(fp8_product, 7)

// (path of the library, error class): opens the library, once
PyObject* open_library(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 2) return PyErr_Format(PyExc_TypeError, "open_library: 2 arguments");
  const char* path = PyUnicode_AsUTF8(a[0]);
  if (!path) return nullptr;
  void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
  if (!lib) return PyErr_Format(PyExc_RuntimeError, "%s", dlerror());
#define FIND(name)                                                                          \
  api.name = reinterpret_cast<decltype(api.name)>(dlsym(lib, "compact_" #name));            \
  if (!api.name) return PyErr_Format(PyExc_RuntimeError, "%s has no compact_" #name, path);
  FIND(quantize_rows) FIND(quantize_blocks) FIND(rms_norm_fwd) FIND(rms_norm_bwd_workspace_bytes) FIND(rms_norm_bwd) FIND(rotary_apply)
  FIND(fp8_product_run)
#undef FIND
  Py_XSETREF(error_class, Py_NewRef(a[1]));
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(open_library), METHOD(quantize_rows), METHOD(quantize_blocks), METHOD(rms_norm_fwd), METHOD(rms_norm_bwd),
                         METHOD(rotary_apply), METHOD(fp8_product), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The Python and torch that the module was built for, found in its file by build.module_fits before it is loaded
extern "C" __attribute__((visibility("default"), used)) const char compact_block_py_tag[] = "built for [" BUILT_FOR "]";

PyMODINIT_FUNC PyInit__block_py() { return PyModule_Create(&module); }
