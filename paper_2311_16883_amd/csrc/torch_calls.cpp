// The single-tensor calls of libbsr_actprune, the token operators among them, with torch tensors as arguments: what binding.py's
// functions do between Python and the C ABI, in native code.  Argument checks, output and workspace
// tensors (torch's caching allocator), device pointers, the current stream, then one C call with the GIL
// released.  No step of the pruning path is computed here.
//
// Why native: a layer of a training step is three calls of a few microseconds of GPU time each, and
// marshalling in Python took 8 to 10 us a call (torch.cuda.current_stream() 2.9 us, torch.empty 1.4 us
// per output, ctypes 0.6 us and more); here it is about 2 us.
//
// Every function takes positional arguments only (binding.py has the keyword forms and turns a negative
// return value, a BSR_ERR_* code, into an exception).
#include <Python.h>

#include <climits>
#include <cmath>
#include <optional>
#include <string>

#include <ATen/ops/empty.h>
#include <ATen/ops/fill.h>
#include <ATen/ops/select.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bsr_actprune.h"
#include "bsr_token_step.h"
#include "bsr_layer_ops.h"

namespace {

// A Python exception is set already.
struct PythonError {};

[[noreturn]] void value_error(const std::string &what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw PythonError();
}

const at::Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor, not %s", what, Py_TYPE(o)->tp_name);
    throw PythonError();
  }
  return THPVariable_Unpack(o);
}

int64_t integer(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  return v;
}

// A block extent or a kind of something: beyond the range of int it becomes a value that the library refuses.
int extent(PyObject *o) {
  const int64_t v = integer(o);
  return v > INT_MAX ? INT_MAX : v < 0 ? -1 : (int)v;
}

// int(o)
int64_t converted_integer(PyObject *o) {
  if (PyLong_Check(o)) return integer(o);
  PyObject *n = PyNumber_Long(o);
  if (n == nullptr) throw PythonError();
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  return v;
}

// float(o)
double real(PyObject *o) {
  if (PyFloat_Check(o)) return PyFloat_AS_DOUBLE(o);
  PyObject *f = PyNumber_Float(o);
  if (f == nullptr) throw PythonError();
  const double v = PyFloat_AS_DOUBLE(f);
  Py_DECREF(f);
  return v;
}

bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PythonError();
  return v != 0;
}

void *pointer(const at::Tensor &t) { return t.data_ptr(); }

// Address of an optional tensor (None: null).
void *optional_pointer(PyObject *o, const char *what) { return o == Py_None ? nullptr : pointer(tensor(o, what)); }

// Extent and leading dimension of a row-major matrix on the device.
struct Dense {
  int64_t rows, cols, ld;
};
Dense dense2d(const at::Tensor &x, const char *what) {
  if (x.dim() != 2 || !x.is_cuda()) value_error(std::string(what) + " must be a 2-D device tensor");
  Dense d{x.size(0), x.size(1), 0};
  if (d.cols > 1 && x.stride(1) != 1) value_error(std::string(what) + " must be row-major (unit stride along columns)");
  d.ld = d.rows > 1 ? x.stride(0) : d.cols;
  if (d.ld < d.cols) value_error(std::string(what) + " has overlapping rows");
  return d;
}

// BSR_F32 / BSR_BF16, or BSR_ERR_DTYPE.
int dtype_code(const at::Tensor &t) {
  const auto s = t.scalar_type();
  return s == at::kFloat ? BSR_F32 : s == at::kBFloat16 ? BSR_BF16 : BSR_ERR_DTYPE;
}

// The stream's handle: `o` a torch stream or an integer, None for the current stream.
void *stream_handle(PyObject *o) {
  if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
  PyObject *h = PyObject_GetAttrString(o, "cuda_stream");
  if (h == nullptr) {
    PyErr_Clear();
    h = PyNumber_Long(o);
    if (h == nullptr) throw PythonError();
  }
  void *p = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (p == nullptr && PyErr_Occurred()) throw PythonError();
  return p;
}

at::Tensor new_tensor(at::IntArrayRef size, at::ScalarType type, const at::Tensor &like) {
  return at::empty(size, at::TensorOptions().dtype(type).device(like.device()));
}

// The workspace of a call: the caller's, or one of `need` bytes (none when need == 0).
struct Workspace {
  at::Tensor own;
  void *p = nullptr;
  size_t bytes = 0;
  Workspace(PyObject *given, size_t need, const at::Tensor &like) {
    if (given != Py_None) {
      const at::Tensor &t = tensor(given, "ws");
      p = pointer(t);
      bytes = (size_t)t.numel();
    } else if (need > 0) {
      own = new_tensor({(int64_t)need}, at::kByte, like);
      p = pointer(own);
      bytes = need;
    }
  }
};

// A tensor that the caller gave, or a new one: what goes back to Python, and its address.
struct Output {
  at::Tensor own;
  PyObject *given = Py_None;
  const at::Tensor &get() const { return given != Py_None ? THPVariable_Unpack(given) : own; }
  PyObject *result() const {
    if (given == Py_None) return THPVariable_Wrap(own);
    Py_INCREF(given);
    return given;
  }
};
Output output(PyObject *given, const char *what, at::IntArrayRef size, at::ScalarType type, const at::Tensor &like) {
  Output o;
  o.given = given;
  if (given == Py_None) o.own = new_tensor(size, type, like);
  else (void)tensor(given, what);
  return o;
}

int64_t blocks(int64_t n, int64_t b) { return b > 0 ? (n + b - 1) / b : 0; }

PyObject *code_result(int rc) { return PyLong_FromLong(rc); }

// Parts of one allocation: each a contiguous tensor of its own from element `offset` on.  (Several small outputs cost one allocation
// this way, and a view made by torch's operators costs as much as an allocation.)
at::Tensor part_of(const at::Tensor &whole, int64_t offset, at::IntArrayRef size) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(offset);
  t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
  return t;
}

// Runs f, which calls the C library, without the GIL; it is held again however f ends.
struct GilReleased {
  PyThreadState *const save = PyEval_SaveThread();
  ~GilReleased() { PyEval_RestoreThread(save); }
};
template <typename F>
int released(F f) {
  const GilReleased guard;
  return f();
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  return false;
}

template <typename F>
PyObject *guarded(F f) {
  HANDLE_TH_ERRORS
  try {
    return f();
  } catch (const PythonError &) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (X, br, bc, group_rows or None, keep, scores, want_scores, keep_mask, ws, stream) -> mask or (mask, scores)
PyObject *score_select(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 10)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &X = tensor(a[0], "X");
    const Dense x = dense2d(X, "X");
    const int br = extent(a[1]), bc = extent(a[2]);
    const int64_t nblocks = br > 0 && bc > 0 ? blocks(x.rows, br) * blocks(x.cols, bc) : 0;
    const bool with_scores = a[5] != Py_None || truth(a[6]);
    Output scores;
    if (with_scores) scores = output(a[5], "scores", {nblocks}, at::kDouble, X);
    const Output mask = output(a[7], "keep_mask", {nblocks}, at::kByte, X);
    const int code = dtype_code(X);
    if (code < 0) return code_result(code);
    const size_t need = a[8] == Py_None ? bsr_workspace_bytes(BSR_OP_SCORE_SELECT, x.rows, x.cols, 0, br, bc, code) : 0;
    const Workspace ws(a[8], need, X);
    const double keep = real(a[4]);
    const int64_t group_rows = a[3] == Py_None ? 0 : converted_integer(a[3]);
    void *stream = stream_handle(a[9]);
    void *px = pointer(X), *pm = pointer(mask.get());
    double *ps = with_scores ? static_cast<double *>(pointer(scores.get())) : nullptr;
    const bool grouped = a[3] != Py_None;
    const int rc = released([&] {
      return grouped ? bsr_score_select_grouped(px, code, x.rows, x.cols, x.ld, br, bc, group_rows, keep, ps,
                                                static_cast<uint8_t *>(pm), ws.p, ws.bytes, stream)
                     : bsr_score_select(px, code, x.rows, x.cols, x.ld, br, bc, keep, ps, static_cast<uint8_t *>(pm),
                                        ws.p, ws.bytes, stream);
    });
    if (rc != BSR_OK) return code_result(rc);
    if (!with_scores) return mask.result();
    return Py_BuildValue("(NN)", mask.result(), scores.result());
  });
}

// (X, br, bc, keep_mask, n_keep, row_ptr, col_idx, values, ws, stream) -> (row_ptr, col_idx, values)
PyObject *compress(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 10)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &X = tensor(a[0], "X");
    const Dense x = dense2d(X, "X");
    const int br = extent(a[1]), bc = extent(a[2]);
    // (a count that sizes an output has to be a whole number; one that does not is converted as by int())
    const int64_t n_keep = a[6] == Py_None || a[7] == Py_None ? integer(a[4]) : converted_integer(a[4]);
    const int64_t places = n_keep > 0 ? n_keep : 0;
    const Output row_ptr = output(a[5], "row_ptr", {blocks(x.rows, br) + 1}, at::kInt, X);
    const Output col_idx = output(a[6], "col_idx", {places}, at::kInt, X);
    const Output values = output(a[7], "values", {places, br, bc}, X.scalar_type(), X);
    const int code = dtype_code(X);
    if (code < 0) return code_result(code);
    const size_t need = a[8] == Py_None ? bsr_workspace_bytes(BSR_OP_COMPRESS, x.rows, x.cols, 0, br, bc, code) : 0;
    const Workspace ws(a[8], need, X);
    void *stream = stream_handle(a[9]);
    void *px = pointer(X), *pm = optional_pointer(a[3], "keep_mask"), *pv = pointer(values.get());
    int32_t *pr = static_cast<int32_t *>(pointer(row_ptr.get())), *pc = static_cast<int32_t *>(pointer(col_idx.get()));
    const int rc = released([&] {
      return bsr_compress(px, code, x.rows, x.cols, x.ld, br, bc, static_cast<const uint8_t *>(pm), n_keep, pr, pc, pv,
                          ws.p, ws.bytes, stream);
    });
    if (rc != BSR_OK) return code_result(rc);
    return Py_BuildValue("(NNN)", row_ptr.result(), col_idx.result(), values.result());
  });
}

// (row_ptr, col_idx, values, M, K, br, bc, out, stream) -> out
PyObject *decompress(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 9)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &values = tensor(a[2], "values");
    const int64_t M = integer(a[3]), K = integer(a[4]);
    const int br = extent(a[5]), bc = extent(a[6]);
    const Output out = output(a[7], "out", {M, K}, values.scalar_type(), values);
    const Dense o = dense2d(out.get(), "out");
    const int code = dtype_code(values);
    if (code < 0) return code_result(code);
    void *stream = stream_handle(a[8]);
    void *pr = optional_pointer(a[0], "row_ptr"), *pc = optional_pointer(a[1], "col_idx"), *pv = pointer(values);
    void *po = pointer(out.get());
    const int rc = released([&] {
      return bsr_decompress(static_cast<const int32_t *>(pr), static_cast<const int32_t *>(pc), pv, code, M, K, o.ld, br,
                            bc, po, stream);
    });
    return rc != BSR_OK ? code_result(rc) : out.result();
  });
}

// (row_ptr, col_idx, values, M, K, br, bc, dY, dW, accumulate, ws, stream) -> dW
PyObject *t_dense_matmul(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 12)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &dY = tensor(a[7], "dY"), &values = tensor(a[2], "values");
    const Dense y = dense2d(dY, "dY");
    const int64_t M = integer(a[3]), K = integer(a[4]);
    const int br = extent(a[5]), bc = extent(a[6]);
    if (y.rows != M) value_error("dY must have M rows");
    const bool accumulate = truth(a[9]);
    if (a[8] == Py_None && accumulate) value_error("accumulate needs an existing dW");
    const Output dW = output(a[8], "dW", {K, y.cols}, at::kFloat, dY);
    const Dense w = dense2d(dW.get(), "dW");
    const int code = dtype_code(dY);
    if (code < 0 || values.scalar_type() != dY.scalar_type()) return code_result(BSR_ERR_DTYPE);
    const size_t need =
        a[10] == Py_None ? bsr_workspace_bytes(BSR_OP_T_DENSE_MATMUL, M, K, y.cols, br, bc, code) : 0;
    const Workspace ws(a[10], need, dY);
    void *stream = stream_handle(a[11]);
    void *pr = optional_pointer(a[0], "row_ptr"), *pc = optional_pointer(a[1], "col_idx"), *pv = pointer(values);
    void *py = pointer(dY);
    float *pw = static_cast<float *>(pointer(dW.get()));
    const int rc = released([&] {
      return bsr_t_dense_matmul(static_cast<const int32_t *>(pr), static_cast<const int32_t *>(pc), pv, code, M, K, br,
                                bc, py, y.cols, y.ld, pw, w.ld, accumulate ? 1 : 0, ws.p, ws.bytes, stream);
    });
    return rc != BSR_OK ? code_result(rc) : dW.result();
  });
}

// (row_ptr, col_idx, values, M, K, br, bc, dY, dalpha, accumulate, ws, stream) -> dalpha
PyObject *affine_scale_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 12)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &dY = tensor(a[7], "dY"), &values = tensor(a[2], "values");
    const Dense y = dense2d(dY, "dY");
    const int64_t M = integer(a[3]), K = integer(a[4]);
    const int br = extent(a[5]), bc = extent(a[6]);
    if (y.rows != M || y.cols != K) value_error("dY must be [M x K]");
    const bool accumulate = truth(a[9]);
    if (a[8] == Py_None && accumulate) value_error("accumulate needs an existing dalpha");
    const Output dalpha = output(a[8], "dalpha", {K}, at::kFloat, dY);
    const int code = dtype_code(dY);
    if (code < 0 || values.scalar_type() != dY.scalar_type()) return code_result(BSR_ERR_DTYPE);
    const size_t need = a[10] == Py_None ? bsr_workspace_bytes(BSR_OP_AFFINE_SCALE_GRAD, M, K, 0, br, bc, code) : 0;
    const Workspace ws(a[10], need, dY);
    void *stream = stream_handle(a[11]);
    void *pr = optional_pointer(a[0], "row_ptr"), *pc = optional_pointer(a[1], "col_idx"), *pv = pointer(values);
    void *py = pointer(dY);
    float *pa = static_cast<float *>(pointer(dalpha.get()));
    const int rc = released([&] {
      return bsr_affine_scale_grad(static_cast<const int32_t *>(pr), static_cast<const int32_t *>(pc), pv, code, M, K, br,
                                   bc, py, y.ld, pa, accumulate ? 1 : 0, ws.p, ws.bytes, stream);
    });
    return rc != BSR_OK ? code_result(rc) : dalpha.result();
  });
}

// ---- token operators ----
// Their index arrays, weights and statistics are packed arrays, which are checked for type, place and extent here.

// The stream of a call on tensors of like's device: `o` as for stream_handle.  While it lives that stream is the current one, so
// that outputs and workspaces made here belong to it, and its device is the current device.
class CallStream {
 public:
  CallStream(PyObject *o, const at::Tensor &like) : device_(like.device().index()), before_(c10::hip::current_device()) {
    if (device_ != before_) c10::hip::set_device(device_);
    current_ = c10::hip::getCurrentHIPStream(device_);
    handle_ = current_->stream();
    if (o == Py_None) return;
    void *h = nullptr;
    try {
      h = stream_handle(o);
    } catch (...) {
      restore();
      throw;
    }
    if (h == handle_) return;
    handle_ = h;
    changed_ = true;
    c10::hip::setCurrentHIPStream(h == nullptr ? c10::hip::getDefaultHIPStream(device_)
                                               : c10::hip::getStreamFromExternal(static_cast<hipStream_t>(h), device_));
  }
  ~CallStream() { restore(); }
  CallStream(const CallStream &) = delete;
  CallStream &operator=(const CallStream &) = delete;
  void *handle() const { return handle_; }

 private:
  void restore() {
    if (changed_) c10::hip::setCurrentHIPStream(*current_);
    if (device_ != before_) c10::hip::set_device(before_);
  }
  c10::DeviceIndex device_, before_;
  std::optional<c10::hip::HIPStream> current_;
  void *handle_ = nullptr;
  bool changed_ = false;
};

// A packed array on the device of `like`.
const at::Tensor &packed(PyObject *o, const char *what, const at::Tensor &like) {
  const at::Tensor &t = tensor(o, what);
  if (!t.is_cuda() || t.device() != like.device()) value_error(std::string(what) + " must be on the device of the other tensors");
  if (!t.is_contiguous()) value_error(std::string(what) + " must be contiguous");
  return t;
}
const at::Tensor &packed(PyObject *o, const char *what, const at::Tensor &like, at::ScalarType type, at::IntArrayRef size) {
  const at::Tensor &t = packed(o, what, like);
  if (t.scalar_type() != type) value_error(std::string(what) + " must be " + c10::toString(type));
  if (t.sizes() != size) value_error(std::string(what) + " has the wrong shape");
  return t;
}
// ... that is an output: the caller's or a new one.
Output packed_output(PyObject *given, const char *what, at::IntArrayRef size, at::ScalarType type, const at::Tensor &like) {
  if (given != Py_None) (void)packed(given, what, like, type, size);
  return output(given, what, size, type, like);
}
// A matrix that is an output: the caller's, of this extent and type, or a new one.
Output matrix_output(PyObject *given, const char *what, int64_t rows, int64_t cols, at::ScalarType type, const at::Tensor &like,
                     int64_t *ld) {
  Output o = output(given, what, {rows, cols}, type, like);
  const Dense d = dense2d(o.get(), what);
  if (d.rows != rows || d.cols != cols) value_error(std::string(what) + " has the wrong shape");
  if (o.get().scalar_type() != type) value_error(std::string(what) + " must be " + c10::toString(type));
  if (o.get().device() != like.device()) value_error(std::string(what) + " must be on the device of the other tensors");
  *ld = d.ld;
  return o;
}
// A matrix of the type and on the device of `like`.
Dense matrix_like(const at::Tensor &x, const char *what, const at::Tensor &like) {
  const Dense d = dense2d(x, what);
  if (x.scalar_type() != like.scalar_type()) value_error(std::string(what) + " has another dtype");
  if (x.device() != like.device()) value_error(std::string(what) + " must be on the device of the other tensors");
  return d;
}

// The workspace of a token operator: the caller's, whose extent the library takes at its word, or a new one.
template <typename F>
Workspace token_workspace(PyObject *given, F need, const at::Tensor &like) {
  if (given != Py_None && packed(given, "ws", like).scalar_type() != at::kByte) value_error("ws must be uint8");
  return Workspace(given, given == Py_None ? need() : 0, like);
}

// BSR_I32 / BSR_I64, or BSR_ERR_DTYPE.
int index_code(const at::Tensor &t) {
  const auto s = t.scalar_type();
  return s == at::kInt ? BSR_I32 : s == at::kLong ? BSR_I64 : BSR_ERR_DTYPE;
}

template <typename P>
P *typed(const at::Tensor &t) { return static_cast<P *>(pointer(t)); }

// (table, tokens, scale, out, stream) -> out
PyObject *embedding_lookup(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &table = tensor(a[0], "table");
    const Dense e = dense2d(table, "table");
    const at::Tensor &tokens = packed(a[1], "tokens", table);
    if (tokens.dim() != 1) value_error("tokens must be 1-D");
    const double scale = real(a[2]);
    const int code = dtype_code(table), index = index_code(tokens);
    if (code < 0 || index < 0) return code_result(BSR_ERR_DTYPE);
    const CallStream stream(a[4], table);
    int64_t ldo;
    const Output out = matrix_output(a[3], "out", tokens.size(0), e.cols, table.scalar_type(), table, &ldo);
    const int rc = released([&] {
      return bsr_embedding_lookup(pointer(table), code, e.rows, e.cols, e.ld, pointer(tokens), index, tokens.size(0), (float)scale,
                                  pointer(out.get()), ldo, stream.handle());
    });
    return rc != BSR_OK ? code_result(rc) : out.result();
  });
}

// (tokens, dY, vocab, scale, dE, accumulate, ws, stream) -> dE
PyObject *embedding_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &dY = tensor(a[1], "dY");
    const Dense y = dense2d(dY, "dY");
    const at::Tensor &tokens = packed(a[0], "tokens", dY);
    if (tokens.dim() != 1 || tokens.size(0) != y.rows) value_error("tokens must be 1-D, one for each row of dY");
    const int64_t V = integer(a[2]);
    if (V < 0) value_error("vocab must not be negative");
    const double scale = real(a[3]);
    const bool accumulate = truth(a[5]);
    if (a[4] == Py_None && accumulate) value_error("accumulate needs an existing dE");
    const int code = dtype_code(dY), index = index_code(tokens);
    if (code < 0 || index < 0) return code_result(BSR_ERR_DTYPE);
    if (V > BSR_MAX_VOCAB) return code_result(BSR_ERR_SHAPE);      // (and in expert_sort: before outputs of that size are made)
    const CallStream stream(a[7], dY);
    int64_t ldde;
    const Output dE = matrix_output(a[4], "dE", V, y.cols, at::kFloat, dY, &ldde);
    const Workspace ws = token_workspace(a[6], [&] { return bsr_embedding_grad_workspace_bytes(y.rows, V, y.cols); }, dY);
    const int rc = released([&] {
      return bsr_embedding_grad(pointer(tokens), index, y.rows, pointer(dY), code, y.cols, y.ld, (float)scale, V,
                                typed<float>(dE.get()), ldde, accumulate ? 1 : 0, ws.p, ws.bytes, stream.handle());
    });
    return rc != BSR_OK ? code_result(rc) : dE.result();
  });
}

// (expert_ids, experts, align, offsets, counts, order, slots, ws, stream) -> (offsets, counts, order, slots)
PyObject *expert_sort(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 9)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &ids = tensor(a[0], "expert_ids");
    (void)packed(a[0], "expert_ids", ids);
    const int64_t E = integer(a[1]), align = integer(a[2]), entries = ids.numel();
    const int index = index_code(ids);
    if (index < 0) return code_result(BSR_ERR_DTYPE);
    const int64_t rows = bsr_expert_capacity(entries, E, align);
    if (rows < 0) return code_result(BSR_ERR_SHAPE);
    if (E > BSR_MAX_EXPERTS) return code_result(BSR_ERR_LIMIT);
    const CallStream stream(a[8], ids);
    Output offsets, counts, order, slots;
    if (a[3] == Py_None && a[4] == Py_None && a[5] == Py_None && a[6] == Py_None) {
      const at::Tensor all = new_tensor({2 * E + 1 + rows + entries}, at::kInt, ids);
      offsets.own = part_of(all, rows + entries, {E + 1});
      counts.own = part_of(all, rows + entries + E + 1, {E});
      order.own = part_of(all, 0, {rows});
      slots.own = part_of(all, rows, ids.sizes());
    } else {
      offsets = packed_output(a[3], "offsets", {E + 1}, at::kInt, ids);
      counts = packed_output(a[4], "counts", {E}, at::kInt, ids);
      order = packed_output(a[5], "order", {rows}, at::kInt, ids);
      slots = packed_output(a[6], "slots", ids.sizes(), at::kInt, ids);
    }
    const Workspace ws = token_workspace(a[7], [&] { return bsr_expert_sort_workspace_bytes(entries, E); }, ids);
    const int rc = released([&] {
      return bsr_expert_sort(pointer(ids), index, entries, E, align, typed<int32_t>(offsets.get()), typed<int32_t>(counts.get()),
                             typed<int32_t>(order.get()), typed<int32_t>(slots.get()), ws.p, ws.bytes, stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return Py_BuildValue("(NNNN)", offsets.result(), counts.result(), order.result(), slots.result());
  });
}

// The [T x k] slots of a call.
const at::Tensor &routing(PyObject *o, const at::Tensor &like) {
  const at::Tensor &slots = packed(o, "slots", like);
  if (slots.dim() != 2 || slots.scalar_type() != at::kInt) value_error("slots must be a 2-D int32 tensor [tokens, choices]");
  return slots;
}

// (X, slots, order, out, stream) -> Xs
PyObject *expert_gather(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &X = tensor(a[0], "X");
    const Dense x = dense2d(X, "X");
    const at::Tensor &slots = routing(a[1], X);
    if (slots.size(0) != x.rows) value_error("slots must have a row for each row of X");
    const int64_t rows = tensor(a[2], "order").numel();
    const at::Tensor &order = packed(a[2], "order", X, at::kInt, {rows});
    const int code = dtype_code(X);
    if (code < 0) return code_result(code);
    const CallStream stream(a[4], X);
    int64_t ldo;
    const Output out = matrix_output(a[3], "out", rows, x.cols, X.scalar_type(), X, &ldo);
    const int rc = released([&] {
      return bsr_expert_gather(pointer(X), code, x.rows, x.cols, x.ld, typed<int32_t>(slots), slots.size(1), typed<int32_t>(order),
                               rows, pointer(out.get()), ldo, stream.handle());
    });
    return rc != BSR_OK ? code_result(rc) : out.result();
  });
}

// (Ys, slots, weights or None, out, stream) -> out
PyObject *expert_combine(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &Ys = tensor(a[0], "Ys");
    const Dense y = dense2d(Ys, "Ys");
    const at::Tensor &slots = routing(a[1], Ys);
    const float *weights = a[2] == Py_None ? nullptr : typed<float>(packed(a[2], "weights", Ys, at::kFloat, slots.sizes()));
    const int code = dtype_code(Ys);
    if (code < 0) return code_result(code);
    const CallStream stream(a[4], Ys);
    int64_t ldo;
    const Output out = matrix_output(a[3], "out", slots.size(0), y.cols, Ys.scalar_type(), Ys, &ldo);
    const int rc = released([&] {
      return bsr_expert_combine(pointer(Ys), code, y.rows, y.cols, y.ld, typed<int32_t>(slots), slots.size(0), slots.size(1),
                                weights, pointer(out.get()), ldo, stream.handle());
    });
    return rc != BSR_OK ? code_result(rc) : out.result();
  });
}

// (Ys, slots, order, weights, dOut, dYs, dweights, stream) -> (dYs, dweights)
PyObject *expert_combine_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &Ys = tensor(a[0], "Ys"), &dOut = tensor(a[4], "dOut");
    const Dense y = dense2d(Ys, "Ys"), g = matrix_like(dOut, "dOut", Ys);
    const at::Tensor &slots = routing(a[1], Ys);
    if (g.rows != slots.size(0) || g.cols != y.cols) value_error("dOut must have a row for each row of slots, as wide as Ys");
    const at::Tensor &order = packed(a[2], "order", Ys, at::kInt, {y.rows});
    const at::Tensor &weights = packed(a[3], "weights", Ys, at::kFloat, slots.sizes());
    const int code = dtype_code(Ys);
    if (code < 0) return code_result(code);
    const CallStream stream(a[7], Ys);
    int64_t ldd;
    const Output dYs = matrix_output(a[5], "dYs", y.rows, y.cols, Ys.scalar_type(), Ys, &ldd);
    const Output dweights = packed_output(a[6], "dweights", slots.sizes(), at::kFloat, Ys);
    const int rc = released([&] {
      return bsr_expert_combine_grad(pointer(Ys), code, y.rows, y.cols, y.ld, typed<int32_t>(slots), typed<int32_t>(order),
                                     slots.size(0), slots.size(1), typed<float>(weights), pointer(dOut), g.ld, pointer(dYs.get()),
                                     ldd, typed<float>(dweights.get()), stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return Py_BuildValue("(NN)", dYs.result(), dweights.result());
  });
}

// The tensors that every distillation call starts with: (logits, ids, teacher, temperature).
struct DistillCall {
  const at::Tensor &logits, &ids, &teacher;
  Dense z;
  int64_t K = 0;
  int code, index, teacher_code;
  float temperature;
  DistillCall(PyObject *const *a)
      : logits(tensor(a[0], "logits")), ids(tensor(a[1], "ids")), teacher(tensor(a[2], "teacher")), z(dense2d(logits, "logits")) {
    (void)packed(a[1], "ids", logits);
    (void)packed(a[2], "teacher", logits);
    if (ids.dim() != 2 || ids.size(0) != z.rows || teacher.sizes() != ids.sizes())
      value_error("ids and teacher must be [rows of logits, entries]");
    K = ids.size(1);
    code = dtype_code(logits);
    index = index_code(ids);
    teacher_code = dtype_code(teacher);
    temperature = (float)real(a[3]);
  }
  bool types() const { return code >= 0 && index >= 0 && teacher_code >= 0; }
  size_t workspace() const { return bsr_distill_workspace_bytes(z.rows, z.cols, K); }
};

// (logits, ids, teacher, temperature, loss, stats, ws, stream) -> (loss, stats)
PyObject *distill_loss(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject * {
    const DistillCall c(a);
    if (!c.types()) return code_result(BSR_ERR_DTYPE);
    const CallStream stream(a[7], c.logits);
    Output loss, stats;
    if (a[4] == Py_None && a[5] == Py_None) {
      const at::Tensor all = new_tensor({3 * c.z.rows}, at::kFloat, c.logits);
      stats.own = part_of(all, 0, {c.z.rows, 2});
      loss.own = part_of(all, 2 * c.z.rows, {c.z.rows});
    } else {
      loss = packed_output(a[4], "loss", {c.z.rows}, at::kFloat, c.logits);
      stats = packed_output(a[5], "stats", {c.z.rows, 2}, at::kFloat, c.logits);
    }
    const Workspace ws = token_workspace(a[6], [&] { return c.workspace(); }, c.logits);
    const int rc = released([&] {
      return bsr_distill_loss(pointer(c.logits), c.code, c.z.rows, c.z.cols, c.z.ld, pointer(c.ids), c.index, pointer(c.teacher),
                              c.teacher_code, c.K, c.temperature, typed<float>(loss.get()), typed<float>(stats.get()), ws.p,
                              ws.bytes, stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return Py_BuildValue("(NN)", loss.result(), stats.result());
  });
}

// (logits, ids, teacher, temperature, stats, dloss, dlogits, stream) -> dlogits
PyObject *distill_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject * {
    const DistillCall c(a);
    if (!c.types()) return code_result(BSR_ERR_DTYPE);
    const at::Tensor &stats = packed(a[4], "stats", c.logits, at::kFloat, {c.z.rows, 2});
    const at::Tensor &dloss = packed(a[5], "dloss", c.logits, at::kFloat, {c.z.rows});
    const CallStream stream(a[7], c.logits);
    int64_t ldd;
    const Output dlogits = matrix_output(a[6], "dlogits", c.z.rows, c.z.cols, c.logits.scalar_type(), c.logits, &ldd);
    const int rc = released([&] {
      return bsr_distill_grad(pointer(c.logits), c.code, c.z.rows, c.z.cols, c.z.ld, pointer(c.ids), c.index, pointer(c.teacher),
                              c.teacher_code, c.K, c.temperature, typed<float>(stats), typed<float>(dloss), pointer(dlogits.get()),
                              ldd, stream.handle());
    });
    return rc != BSR_OK ? code_result(rc) : dlogits.result();
  });
}

// (logits, ids, teacher, temperature, dloss, loss, dlogits, ws, stream) -> (loss, dlogits)
PyObject *distill_loss_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 9)) return nullptr;
  return guarded([&]() -> PyObject * {
    const DistillCall c(a);
    if (!c.types()) return code_result(BSR_ERR_DTYPE);
    const at::Tensor &dloss = packed(a[4], "dloss", c.logits, at::kFloat, {c.z.rows});
    const CallStream stream(a[8], c.logits);
    const Output loss = packed_output(a[5], "loss", {c.z.rows}, at::kFloat, c.logits);
    int64_t ldd;
    const Output dlogits = matrix_output(a[6], "dlogits", c.z.rows, c.z.cols, c.logits.scalar_type(), c.logits, &ldd);
    const Workspace ws = token_workspace(a[7], [&] { return c.workspace(); }, c.logits);
    const int rc = released([&] {
      return bsr_distill_loss_grad(pointer(c.logits), c.code, c.z.rows, c.z.cols, c.z.ld, pointer(c.ids), c.index,
                                   pointer(c.teacher), c.teacher_code, c.K, c.temperature, typed<float>(dloss),
                                   typed<float>(loss.get()), pointer(dlogits.get()), ldd, ws.p, ws.bytes, stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return Py_BuildValue("(NN)", loss.result(), dlogits.result());
  });
}

// ---- layer operators ----

// gamma or beta of a norm over D columns: null for None.
const at::Tensor *norm_param(PyObject *o, const char *what, const at::Tensor &like, int64_t D) {
  if (o == Py_None) return nullptr;
  const at::Tensor &t = packed(o, what, like);
  if (t.dim() != 1 || t.size(0) != D) value_error(std::string(what) + " must be 1-D, a number for each column");
  return &t;
}

// (X, gamma or None, beta or None, eps, Y, stats, want_stats, stream) -> Y or (Y, stats)
PyObject *layer_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &X = tensor(a[0], "X");
    const Dense x = dense2d(X, "X");
    const at::Tensor *gamma = norm_param(a[1], "gamma", X, x.cols), *beta = norm_param(a[2], "beta", X, x.cols);
    if (gamma != nullptr && beta != nullptr && gamma->scalar_type() != beta->scalar_type()) value_error("gamma and beta differ in dtype");
    const double eps = real(a[3]);
    const bool with_stats = a[5] != Py_None || truth(a[6]);
    const at::Tensor *param = gamma != nullptr ? gamma : beta;
    const int code = dtype_code(X), pcode = param != nullptr ? dtype_code(*param) : BSR_F32;
    if (code < 0 || pcode < 0) return code_result(BSR_ERR_DTYPE);
    const CallStream stream(a[7], X);
    int64_t ldy;
    const Output Y = matrix_output(a[4], "Y", x.rows, x.cols, X.scalar_type(), X, &ldy);
    Output stats;
    if (with_stats) stats = packed_output(a[5], "stats", {x.rows, 2}, at::kFloat, X);
    const int rc = released([&] {
      return bsr_layer_norm(pointer(X), code, x.rows, x.cols, x.ld, gamma != nullptr ? pointer(*gamma) : nullptr,
                            beta != nullptr ? pointer(*beta) : nullptr, pcode, (float)eps, pointer(Y.get()), ldy,
                            with_stats ? typed<float>(stats.get()) : nullptr, stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    if (with_stats && x.cols == 0 && x.rows > 0) {          // (the library writes nothing then)
      const at::AutoDispatchBelowAutograd plain;
      at::Tensor mean = at::select(stats.get(), 1, 0), rstd = at::select(stats.get(), 1, 1);
      at::fill_(mean, 0.0);
      at::fill_(rstd, 1.0 / std::sqrt((double)(float)eps));
    }
    return with_stats ? Py_BuildValue("(NN)", Y.result(), stats.result()) : Y.result();
  });
}

// (X, gamma or None, stats, dY, dX, dgamma, dbeta, want_params, accumulate, ws, stream) -> (dX, dgamma, dbeta) or dX
PyObject *layer_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 11)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &X = tensor(a[0], "X"), &dY = tensor(a[3], "dY");
    const Dense x = dense2d(X, "X"), y = matrix_like(dY, "dY", X);
    if (y.rows != x.rows || y.cols != x.cols) value_error("dY must have the shape of X");
    const at::Tensor *gamma = norm_param(a[1], "gamma", X, x.cols);
    const at::Tensor &stats = packed(a[2], "stats", X, at::kFloat, {x.rows, 2});
    const bool params = truth(a[7]), accumulate = truth(a[8]);
    if (!params && (a[5] != Py_None || a[6] != Py_None)) value_error("dgamma and dbeta are not wanted");
    if (accumulate && params && (a[5] == Py_None || a[6] == Py_None)) value_error("accumulate needs existing dgamma and dbeta");
    const int code = dtype_code(X), pcode = gamma != nullptr ? dtype_code(*gamma) : BSR_F32;
    if (code < 0 || pcode < 0) return code_result(BSR_ERR_DTYPE);
    const CallStream stream(a[10], X);
    int64_t ldx;
    const Output dX = matrix_output(a[4], "dX", x.rows, x.cols, X.scalar_type(), X, &ldx);
    Output dgamma, dbeta;
    if (params && a[5] == Py_None && a[6] == Py_None) {
      const at::Tensor both = new_tensor({2 * x.cols}, at::kFloat, X);
      dgamma.own = part_of(both, 0, {x.cols});
      dbeta.own = part_of(both, x.cols, {x.cols});
    } else if (params) {
      dgamma = packed_output(a[5], "dgamma", {x.cols}, at::kFloat, X);
      dbeta = packed_output(a[6], "dbeta", {x.cols}, at::kFloat, X);
    }
    const Workspace ws = token_workspace(a[9], [&] { return params ? bsr_layer_norm_grad_workspace_bytes(x.rows, x.cols) : 0; }, X);
    const int rc = released([&] {
      return bsr_layer_norm_grad(pointer(X), code, x.rows, x.cols, x.ld, gamma != nullptr ? pointer(*gamma) : nullptr, pcode,
                                 typed<float>(stats), pointer(dY), y.ld, pointer(dX.get()), ldx,
                                 params ? typed<float>(dgamma.get()) : nullptr, params ? typed<float>(dbeta.get()) : nullptr,
                                 accumulate ? 1 : 0, ws.p, ws.bytes, stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return params ? Py_BuildValue("(NNN)", dX.result(), dgamma.result(), dbeta.result()) : dX.result();
  });
}

// The weights of a gated block: [D x 2F].
Dense gated_weights(const at::Tensor &W, const at::Tensor &like) {
  const Dense w = matrix_like(W, "W", like);
  if (w.cols % 2 != 0) value_error("W must have two columns for each of H: the gate's, then the other projection's");
  return w;
}

// (X, W, act, H, GU, want_GU, ws, stream) -> H or (H, GU)
PyObject *gated_ff(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &X = tensor(a[0], "X"), &W = tensor(a[1], "W");
    const Dense x = dense2d(X, "X"), w = gated_weights(W, X);
    if (w.rows != x.cols) value_error("W must have a row for each column of X");
    const int act = extent(a[2]);
    const int64_t F = w.cols / 2;
    const bool save = a[4] != Py_None || truth(a[5]);
    const int code = dtype_code(X);
    if (code < 0) return code_result(code);
    const CallStream stream(a[7], X);
    int64_t ldh, ldgu = 0;
    const Output H = matrix_output(a[3], "H", x.rows, F, X.scalar_type(), X, &ldh);
    Output GU;
    if (save) GU = matrix_output(a[4], "GU", x.rows, 2 * F, X.scalar_type(), X, &ldgu);
    const Workspace ws = token_workspace(
        a[6], [&] { return bsr_gated_ff_workspace_bytes(pointer(X), code, x.rows, x.cols, x.ld, pointer(W), F, w.ld); }, X);
    const int rc = released([&] {
      return bsr_gated_ff(pointer(X), code, x.rows, x.cols, x.ld, pointer(W), F, w.ld, act, pointer(H.get()), ldh,
                          save ? pointer(GU.get()) : nullptr, ldgu, ws.p, ws.bytes, stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return save ? Py_BuildValue("(NN)", H.result(), GU.result()) : H.result();
  });
}

// (GU, dH, W, act, dGU, dX, want_dX, ws, stream) -> (dX, dGU) or dGU
PyObject *gated_ff_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 9)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &GU = tensor(a[0], "GU"), &dH = tensor(a[1], "dH");
    const Dense gu = dense2d(GU, "GU"), h = matrix_like(dH, "dH", GU);
    if (gu.cols != 2 * h.cols || gu.rows != h.rows) value_error("GU must have the rows of dH and twice its columns");
    const int act = extent(a[3]);
    const bool with_x = truth(a[6]);
    if (!with_x && a[5] != Py_None) value_error("dX is not wanted");
    const at::Tensor *W = with_x ? &tensor(a[2], "W") : nullptr;
    Dense w{0, gu.cols, gu.cols};
    if (with_x) {
      w = gated_weights(*W, GU);
      if (w.cols != gu.cols) value_error("W must have the columns of GU");
    }
    const int code = dtype_code(GU);
    if (code < 0) return code_result(code);
    const CallStream stream(a[8], GU);
    int64_t ldd, ldx = 0;
    const Output dGU = matrix_output(a[4], "dGU", gu.rows, gu.cols, GU.scalar_type(), GU, &ldd);
    Output dX;
    if (with_x) dX = matrix_output(a[5], "dX", gu.rows, w.rows, GU.scalar_type(), GU, &ldx);
    const Workspace ws = token_workspace(
        a[7],
        [&] {
          return with_x ? bsr_gated_ff_grad_workspace_bytes(pointer(dGU.get()), code, gu.rows, h.cols, ldd, pointer(*W), w.rows, w.ld) : 0;
        },
        GU);
    const int rc = released([&] {
      return bsr_gated_ff_grad(pointer(GU), code, gu.rows, h.cols, gu.ld, pointer(dH), h.ld, act, with_x ? pointer(*W) : nullptr, w.rows,
                               w.ld, pointer(dGU.get()), ldd, with_x && w.rows > 0 ? pointer(dX.get()) : nullptr, ldx, ws.p, ws.bytes,
                               stream.handle());
    });
    if (rc != BSR_OK) return code_result(rc);
    return with_x ? Py_BuildValue("(NN)", dX.result(), dGU.result()) : dGU.result();
  });
}

// A number of an optimizer step: a Python number, or one element on the device.
template <typename T>
const T *device_number(PyObject *o, const char *what, const at::Tensor &like, at::ScalarType type) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor &t = packed(o, what, like);
  if (t.scalar_type() != type || t.numel() != 1) value_error(std::string(what) + " on the device must be one number of type " + c10::toString(type));
  return typed<T>(t);
}

// (like, address of the items, items, param code, grad code, moments, lr, step, beta1, beta2, eps, grad_scale, seed, stream) -> code
PyObject *adamw_batched(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 14)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &like = tensor(a[0], "params");
    const auto *items = static_cast<const bsr_adamw_item *>(PyLong_AsVoidPtr(a[1]));
    bsr_adamw_options o = {};
    o.lr_device = device_number<float>(a[6], "lr", like, at::kFloat);
    o.step_device = device_number<int64_t>(a[7], "step", like, at::kLong);
    o.grad_scale_device = device_number<float>(a[11], "grad_scale", like, at::kFloat);
    o.lr = o.lr_device != nullptr ? 0.0 : real(a[6]);
    o.step = o.step_device != nullptr ? 1 : integer(a[7]);
    o.beta1 = real(a[8]);
    o.beta2 = real(a[9]);
    o.eps = real(a[10]);
    o.grad_scale = o.grad_scale_device != nullptr ? 1.0 : real(a[11]);
    o.seed = PyLong_AsUnsignedLongLong(a[12]);
    if (PyErr_Occurred()) throw PythonError();
    const int count = (int)integer(a[2]), param = (int)integer(a[3]), grad = (int)integer(a[4]), moments = (int)integer(a[5]);
    const CallStream stream(a[13], like);
    return code_result(released([&] { return bsr_adamw_batched(items, count, param, grad, moments, &o, stream.handle()); }));
  });
}

// (codes, scales, which, out, dtype, stream) -> out
PyObject *adamw_state_values(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (!arity(n, 6)) return nullptr;
  return guarded([&]() -> PyObject * {
    const at::Tensor &codes = tensor(a[0], "codes");
    if (!codes.is_cuda() || codes.scalar_type() != at::kByte || !codes.is_contiguous()) value_error("codes must be a contiguous uint8 tensor on the device");
    const int64_t count = codes.numel();
    const at::Tensor &scales = packed(a[1], "scales", codes, at::kByte, {bsr_adamw_blocks(count)});
    const int which = (int)integer(a[2]), code = (int)integer(a[4]);
    if (code != BSR_F32 && code != BSR_BF16) return code_result(BSR_ERR_DTYPE);
    const CallStream stream(a[5], codes);
    const Output out = packed_output(a[3], "out", codes.sizes(), code == BSR_F32 ? at::kFloat : at::kBFloat16, codes);
    const int rc = released([&] {
      return bsr_adamw_state_values(typed<uint8_t>(codes), typed<uint8_t>(scales), count, which, pointer(out.get()), code, stream.handle());
    });
    return rc != BSR_OK ? code_result(rc) : out.result();
  });
}

// () -> handle of the current stream of the current device
PyObject *current_stream(PyObject *, PyObject *) {
  return guarded([&]() -> PyObject * { return PyLong_FromVoidPtr(c10::hip::getCurrentHIPStream().stream()); });
}

PyMethodDef methods[] = {
    {"score_select", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(score_select)), METH_FASTCALL, nullptr},
    {"compress", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(compress)), METH_FASTCALL, nullptr},
    {"decompress", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(decompress)), METH_FASTCALL, nullptr},
    {"t_dense_matmul", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(t_dense_matmul)), METH_FASTCALL, nullptr},
    {"affine_scale_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(affine_scale_grad)), METH_FASTCALL, nullptr},
    {"embedding_lookup", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(embedding_lookup)), METH_FASTCALL, nullptr},
    {"embedding_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(embedding_grad)), METH_FASTCALL, nullptr},
    {"expert_sort", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(expert_sort)), METH_FASTCALL, nullptr},
    {"expert_gather", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(expert_gather)), METH_FASTCALL, nullptr},
    {"expert_combine", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(expert_combine)), METH_FASTCALL, nullptr},
    {"expert_combine_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(expert_combine_grad)), METH_FASTCALL, nullptr},
    {"distill_loss", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(distill_loss)), METH_FASTCALL, nullptr},
    {"distill_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(distill_grad)), METH_FASTCALL, nullptr},
    {"distill_loss_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(distill_loss_grad)), METH_FASTCALL, nullptr},
    {"layer_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(layer_norm)), METH_FASTCALL, nullptr},
    {"layer_norm_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(layer_norm_grad)), METH_FASTCALL, nullptr},
    {"gated_ff", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(gated_ff)), METH_FASTCALL, nullptr},
    {"gated_ff_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(gated_ff_grad)), METH_FASTCALL, nullptr},
    {"adamw_batched", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(adamw_batched)), METH_FASTCALL, nullptr},
    {"adamw_state_values", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(adamw_state_values)), METH_FASTCALL, nullptr},
    {"current_stream", current_stream, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit__torch_calls() { return PyModule_Create(&module); }
