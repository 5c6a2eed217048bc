// The calls of binding.py in native code: reads the tensors, allocates the results and calls the C ABI of
// include/cnn.h on the current stream.
//
// A call of the library with small tensors is over in about 5 us on the GPU, less than Python needed to make it: 10.5 us
// for a convolution, of which 3.4 are the launch itself, 2.9 the lookup of the current stream, 1.7 each allocation and
// the rest the conversion of a dozen arguments by ctypes.  Here the same call takes 4.2 us, or 5 to 6 where the host's
// processor runs slower (both occur on one machine).  A network made of single operations at batch 100 (18 calls, 21
// launches, 67 us of kernels) is still limited by the host: 98 to 107 us a pass, 211 before.
// Arguments arrive positionally from the wrappers in binding.py, which hold the names, the defaults and the
// descriptions.  The interpreter lock is released around each call of the library, as ctypes does.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>

#include <climits>
#include <vector>

#include "cnn.h"

namespace {

struct Raised {};  // a Python exception is set

PyObject* check = nullptr;  // binding._check: raises CnnError for a code other than 0

template <class FN>
PyObject* guarded(FN fn) {
  try {
    return fn();
  } catch (const Raised&) {
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Raised();
}

const at::Tensor& tensor(PyObject* o, at::ScalarType type = at::kFloat) {
  if (!THPVariable_Check(o)) {
    if (PyObject* a = PyObject_GetAttrString(o, "is_cuda")) {  // None and other objects: AttributeError
      Py_DECREF(a);
      raise(PyExc_TypeError, "expected a tensor");
    }
    throw Raised();
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous())
    raise(PyExc_ValueError, type == at::kInt ? "expected a contiguous torch.int32 tensor on the GPU"
                                             : "expected a contiguous torch.float32 tensor on the GPU");
  return t;
}

const at::Tensor& tensor(PyObject* o, int dims) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != dims) {
    PyErr_Format(PyExc_ValueError, "expected %d dimensions, got %d", dims, (int)t.dim());
    throw Raised();
  }
  return t;
}

template <class T = float>
T* data(const at::Tensor& t) {
  return static_cast<T*>(t.data_ptr());
}

template <class T = float>
T* data_or_null(PyObject* o, at::ScalarType type = at::kFloat) {
  return o == Py_None ? nullptr : data<T>(tensor(o, type));
}

int size(const at::Tensor& t, int i) { return (int)t.sizes()[i]; }

int first_size(const at::Tensor& t) {
  if (t.dim() < 1) raise(PyExc_IndexError, "tuple index out of range");
  return size(t, 0);
}

long integer(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}

at::Tensor empty(at::IntArrayRef sizes, at::Device device, at::ScalarType type = at::kFloat) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(device));
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

template <class FN>
void call(const char* name, FN fn) {
  int code;
  Py_BEGIN_ALLOW_THREADS;
  code = fn();
  Py_END_ALLOW_THREADS;
  if (code == 0) return;
  if (PyObject* r = PyObject_CallFunction(check, "is", code, name)) Py_DECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
  throw Raised();
}

PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

PyObject* pair(PyObject* a, PyObject* b) {
  PyObject* r = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  return r;
}

void* context(PyObject* o) {
  if (o == Py_None) return nullptr;  // closed: the library refuses it
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Raised();
  return p;
}

at::Device device_at(PyObject* index) { return at::Device(at::kCUDA, (c10::DeviceIndex)integer(index)); }

#define CALL(name, count)                                                                      \
  PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n) {                                \
    if (n != count) return PyErr_Format(PyExc_TypeError, #name " takes %d arguments", count);  \
    return guarded([&]() -> PyObject* {
#define END \
  });       \
  }

// ---- the network: ctx, ..., device index -------------------------------------------------------------------
CALL(forward, 4)  // ctx, images, yhat or None, device
  const at::Tensor& x = tensor(a[1]);
  const int B = first_size(x);
  at::Tensor made;
  if (a[2] == Py_None) made = empty({B, 10}, device_at(a[3]));
  float* y = a[2] == Py_None ? data(made) : data(tensor(a[2]));
  void* ctx = context(a[0]);
  call("cnn_forward", [&] { return cnn_forward(static_cast<cnn_ctx*>(ctx), data(x), B, y); });
  if (a[2] == Py_None) return wrap(std::move(made));
  Py_INCREF(a[2]);
  return a[2];
END

CALL(gradient, 4)  // ctx, images, labels, device
  const at::Tensor& x = tensor(a[1]);
  const int32_t* labels = data_or_null<int32_t>(a[2], at::kInt);
  const int B = first_size(x);
  at::Tensor grad = empty({CNN_NPARAM}, device_at(a[3])), loss = empty({1}, device_at(a[3]));
  void* ctx = context(a[0]);
  call("cnn_gradient", [&] { return cnn_gradient(static_cast<cnn_ctx*>(ctx), data(x), labels, B, data(grad), data(loss)); });
  return pair(wrap(std::move(grad)), wrap(std::move(loss)));
END

CALL(train_batch, 5)  // ctx, images, labels, rate, loss or None
  const at::Tensor& x = tensor(a[1]);
  const int32_t* labels = data_or_null<int32_t>(a[2], at::kInt);
  const int B = first_size(x);
  const float rate = (float)number(a[3]);
  float* loss = data_or_null(a[4]);
  void* ctx = context(a[0]);
  call("cnn_train_batch", [&] { return cnn_train_batch(static_cast<cnn_ctx*>(ctx), data(x), labels, B, rate, loss); });
  Py_INCREF(a[4]);
  return a[4];
END

CALL(evaluate, 4)  // ctx, images, labels, device
  const at::Tensor& x = tensor(a[1]);
  const int32_t* labels = data_or_null<int32_t>(a[2], at::kInt);
  const int B = first_size(x);
  at::Tensor right = empty({1}, device_at(a[3]), at::kLong), loss = empty({1}, device_at(a[3]));
  void* ctx = context(a[0]);
  call("cnn_evaluate", [&] {
    return cnn_evaluate(static_cast<cnn_ctx*>(ctx), data(x), labels, B, data<int64_t>(right), data(loss));
  });
  return pair(wrap(std::move(right)), wrap(std::move(loss)));
END

// ---- single operations -------------------------------------------------------------------------------------
CALL(conv_fwd, 4)  // in, k, bias or None, form: 0 fp32, 1 bf16, 2 plain
  const at::Tensor &x = tensor(a[0], 4), &k = tensor(a[1], 4);
  const float* bias = data_or_null(a[2]);
  const int B = size(x, 0), Cin = size(x, 1), H = size(x, 2), W = size(x, 3), Cout = size(k, 0), KH = size(k, 2), KW = size(k, 3);
  at::Tensor out = empty({B, Cout, H - KH + 1, W - KW + 1}, x.device());
  const long form = integer(a[3]);
  const auto fn = form == 1 ? cnn_conv_fwd_bf16 : form == 2 ? cnn_conv_fwd_valu : cnn_conv_fwd;
  call(form == 1 ? "cnn_conv_fwd_bf16" : form == 2 ? "cnn_conv_fwd_valu" : "cnn_conv_fwd",
       [&] { return fn(data(x), data(k), bias, data(out), B, Cin, H, W, Cout, KH, KW, stream()); });
  return wrap(std::move(out));
END

CALL(conv_bwd_input, 5)  // d_out, k, H, W, form
  const at::Tensor &d = tensor(a[0]), &k = tensor(a[1], 4);
  const int B = first_size(d), Cout = size(k, 0), Cin = size(k, 1), KH = size(k, 2), KW = size(k, 3);
  const long H = integer(a[2]), W = integer(a[3]), form = integer(a[4]);
  at::Tensor out = empty({B, Cin, H, W}, d.device());
  const auto fn = form == 1 ? cnn_conv_bwd_input_bf16 : form == 2 ? cnn_conv_bwd_input_valu : cnn_conv_bwd_input;
  call(form == 1 ? "cnn_conv_bwd_input_bf16" : form == 2 ? "cnn_conv_bwd_input_valu" : "cnn_conv_bwd_input",
       [&] { return fn(data(d), data(k), data(out), B, Cin, (int)H, (int)W, Cout, KH, KW, stream()); });
  return wrap(std::move(out));
END

CALL(conv_bwd_weight, 5)  // in, d_out, want_bias, workspace, bf16
  const at::Tensor &x = tensor(a[0], 4), &d = tensor(a[1], 4);
  const int B = size(x, 0), Cin = size(x, 1), H = size(x, 2), W = size(x, 3), Cout = size(d, 1);
  const int KH = H - size(d, 2) + 1, KW = W - size(d, 3) + 1;
  const bool bf16 = integer(a[4]);
  at::Tensor d_k = empty({Cout, Cin, KH, KW}, x.device()), d_b, ws;
  if (integer(a[2])) d_b = empty({Cout}, x.device());
  size_t bytes = 0;
  if (integer(a[3])) {
    bytes = (bf16 ? cnn_conv_bwd_weight_bf16_workspace_bytes : cnn_conv_bwd_weight_workspace_bytes)(B, Cin, H, W, Cout, KH, KW);
    if (bytes) ws = empty({(int64_t)bytes}, x.device(), at::kByte);
  }
  const auto fn = bf16 ? cnn_conv_bwd_weight_bf16 : cnn_conv_bwd_weight;
  call(bf16 ? "cnn_conv_bwd_weight_bf16" : "cnn_conv_bwd_weight", [&] {
    return fn(data(x), data(d), data(d_k), d_b.defined() ? data(d_b) : nullptr, B, Cin, H, W, Cout, KH, KW,
              bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(wrap(std::move(d_k)), d_b.defined() ? wrap(std::move(d_b)) : (Py_INCREF(Py_None), Py_None));
END

CALL(avgpool_fwd, 1)
  const at::Tensor& x = tensor(a[0], 4);
  const int B = size(x, 0), C = size(x, 1), H = size(x, 2), W = size(x, 3);
  at::Tensor out = empty({B, C, H / 2, W / 2}, x.device());
  call("cnn_avgpool_fwd", [&] { return cnn_avgpool_fwd(data(x), data(out), B, C, H, W, stream()); });
  return wrap(std::move(out));
END

CALL(avgpool_bwd, 1)
  const at::Tensor& d = tensor(a[0], 4);
  const int B = size(d, 0), C = size(d, 1), Ho = size(d, 2), Wo = size(d, 3);
  at::Tensor out = empty({B, C, 2 * Ho, 2 * Wo}, d.device());
  call("cnn_avgpool_bwd", [&] { return cnn_avgpool_bwd(data(d), data(out), B, C, Ho, Wo, stream()); });
  return wrap(std::move(out));
END

CALL(fc_fwd, 3)  // in, w, bias or None
  const at::Tensor &x = tensor(a[0], 2), &w = tensor(a[1]);
  const float* bias = data_or_null(a[2]);
  const int B = size(x, 0), I = size(x, 1), O = first_size(w);
  at::Tensor out = empty({B, O}, x.device());
  call("cnn_fc_fwd", [&] { return cnn_fc_fwd(data(x), data(w), bias, data(out), B, I, O, stream()); });
  return wrap(std::move(out));
END

CALL(fc_bwd_input, 2)  // d_out, w
  const at::Tensor &d = tensor(a[0], 2), &w = tensor(a[1]);
  if (w.dim() < 2) raise(PyExc_IndexError, "tuple index out of range");
  const int B = size(d, 0), O = size(d, 1), I = size(w, 1);
  at::Tensor out = empty({B, I}, d.device());
  call("cnn_fc_bwd_input", [&] { return cnn_fc_bwd_input(data(d), data(w), data(out), B, I, O, stream()); });
  return wrap(std::move(out));
END

CALL(fc_bwd_weight, 4)  // in, d_out, want_bias, workspace
  const at::Tensor &x = tensor(a[0], 2), &d = tensor(a[1]);
  if (d.dim() < 2) raise(PyExc_IndexError, "tuple index out of range");
  const int B = size(x, 0), I = size(x, 1), O = size(d, 1);
  at::Tensor d_w = empty({O, I}, x.device()), d_b, ws;
  if (integer(a[2])) d_b = empty({O}, x.device());
  size_t bytes = 0;
  if (integer(a[3])) {
    bytes = cnn_fc_bwd_weight_workspace_bytes(B, I, O);
    if (bytes) ws = empty({(int64_t)bytes}, x.device(), at::kByte);
  }
  call("cnn_fc_bwd_weight", [&] {
    return cnn_fc_bwd_weight(data(x), data(d), data(d_w), d_b.defined() ? data(d_b) : nullptr, B, I, O,
                             bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(wrap(std::move(d_w)), d_b.defined() ? wrap(std::move(d_b)) : (Py_INCREF(Py_None), Py_None));
END

CALL(logistic_fwd, 1)
  const at::Tensor& x = tensor(a[0]);
  at::Tensor y = empty(x.sizes(), x.device());
  call("cnn_logistic_fwd", [&] { return cnn_logistic_fwd(data(x), data(y), (size_t)x.numel(), stream()); });
  return wrap(std::move(y));
END

CALL(logistic_bwd, 2)  // y, d_y
  const at::Tensor& y = tensor(a[0]);
  const float* d_y = data_or_null(a[1]);
  at::Tensor d_x = empty(y.sizes(), y.device());
  call("cnn_logistic_bwd", [&] { return cnn_logistic_bwd(data(y), d_y, data(d_x), (size_t)y.numel(), stream()); });
  return wrap(std::move(d_x));
END

// ---- operators on sequences ----------------------------------------------------------------------------------
// Element type of a tensor on the GPU (contiguous unless `strided`), as the library counts them.
int element_type(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return CNN_F32;
    case at::kBFloat16: return CNN_BF16;
    case at::kHalf: return CNN_F16;
    default: raise(PyExc_ValueError, "expected a torch.float32, torch.bfloat16 or torch.float16 tensor on the GPU");
  }
}

const at::Tensor& any_tensor(PyObject* o, bool strided = false) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) raise(PyExc_ValueError, "expected a tensor on the GPU");
  if (!strided && !t.is_contiguous()) raise(PyExc_ValueError, "expected a contiguous tensor on the GPU");
  return t;
}

const at::Tensor& like(PyObject* o, const at::Tensor& x) {
  const at::Tensor& t = any_tensor(o);
  if (t.scalar_type() != x.scalar_type() || t.sizes() != x.sizes()) raise(PyExc_ValueError, "expected a tensor of the same shape and type");
  return t;
}

const at::Tensor& token_tensor(PyObject* o) {
  const at::Tensor& t = any_tensor(o);
  if (t.scalar_type() != at::kInt && t.scalar_type() != at::kLong) raise(PyExc_ValueError, "expected a torch.int32 or torch.int64 tensor of tokens");
  return t;
}

uint64_t word64(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Raised();
  return v;
}

CALL(embedding_fwd, 3)  // table, tokens, scale
  const at::Tensor &table = any_tensor(a[0]), &tokens = token_tensor(a[1]);
  if (table.dim() != 2) raise(PyExc_ValueError, "expected a table of 2 dimensions");
  if (table.size(1) > INT_MAX) raise(PyExc_ValueError, "a dimension is too large");
  const int type = element_type(table);
  const float scale = (float)number(a[2]);
  std::vector<int64_t> sizes = tokens.sizes().vec();
  sizes.push_back(table.size(1));
  at::Tensor out = empty(sizes, table.device(), table.scalar_type());
  call("cnn_embedding_fwd", [&] {
    return cnn_embedding_fwd(table.data_ptr(), tokens.data_ptr(), out.data_ptr(), tokens.numel(), table.size(0), (int)table.size(1), type,
                             tokens.scalar_type() == at::kLong, scale, stream());
  });
  return wrap(std::move(out));
END

CALL(embedding_bwd, 4)  // d_out, tokens, vocab, scale
  const at::Tensor &d = any_tensor(a[0]), &tokens = token_tensor(a[1]);
  const int type = element_type(d);
  const int64_t V = integer(a[2]), N = tokens.numel();
  const float scale = (float)number(a[3]);
  if (d.dim() != tokens.dim() + 1 || d.sizes().slice(0, tokens.dim()) != tokens.sizes())
    raise(PyExc_ValueError, "expected an output error with one row per token");
  const int64_t D = d.size(-1);
  const size_t bytes = D > INT_MAX ? 0 : cnn_embedding_bwd_workspace_bytes(N, V, (int)D, type);
  at::Tensor table, ws;
  if (bytes) table = empty({V, D}, d.device(), d.scalar_type()), ws = empty({(int64_t)bytes}, d.device(), at::kByte);
  call("cnn_embedding_bwd", [&] {
    return bytes ? cnn_embedding_bwd(d.data_ptr(), tokens.data_ptr(), table.data_ptr(), N, V, (int)D, type, tokens.scalar_type() == at::kLong,
                                     scale, ws.data_ptr(), bytes, stream())
                 : CNN_EINVAL;
  });
  return wrap(std::move(table));
END

const int64_t* step_or_null(PyObject* o) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = any_tensor(o);
  if (t.scalar_type() != at::kLong || t.numel() != 1) raise(PyExc_ValueError, "expected a torch.int64 tensor of one element");
  return data<int64_t>(t);
}

CALL(dropout_fwd, 6)  // x, p, seed, offset, residual or None, step or None
  const at::Tensor& x = any_tensor(a[0]);
  const int type = element_type(x);
  const double p = number(a[1]);
  const uint64_t seed = word64(a[2]), offset = word64(a[3]);
  const void* residual = a[4] == Py_None ? nullptr : like(a[4], x).data_ptr();
  const int64_t* step = step_or_null(a[5]);
  at::Tensor y = empty(x.sizes(), x.device(), x.scalar_type());
  call("cnn_dropout_fwd", [&] {
    return cnn_dropout_fwd(x.data_ptr(), residual, y.data_ptr(), (size_t)x.numel(), type, p, seed, offset, step, stream());
  });
  return wrap(std::move(y));
END

CALL(dropout_bwd, 5)  // d_y, p, seed, offset, step or None
  const at::Tensor& d = any_tensor(a[0]);
  const int type = element_type(d);
  const double p = number(a[1]);
  const uint64_t seed = word64(a[2]), offset = word64(a[3]);
  const int64_t* step = step_or_null(a[4]);
  at::Tensor d_x = empty(d.sizes(), d.device(), d.scalar_type());
  call("cnn_dropout_bwd", [&] {
    return cnn_dropout_bwd(d.data_ptr(), d_x.data_ptr(), (size_t)d.numel(), type, p, seed, offset, step, stream());
  });
  return wrap(std::move(d_x));
END

// A [batch, token, head, width] tensor with whatever strides (the step's has no tokens), its last dimension without gaps.
cnn_heads heads_of(const at::Tensor& t) {
  const bool tokens = t.dim() == 4;
  return {t.data_ptr(), t.stride(0), tokens ? t.stride(1) : 0, t.stride(tokens ? 2 : 1)};
}

const at::Tensor& heads_tensor(PyObject* o, int dims, at::ScalarType type) {
  const at::Tensor& t = any_tensor(o, true);
  if (t.dim() != dims) {
    PyErr_Format(PyExc_ValueError, "expected %d dimensions, got %d", dims, (int)t.dim());
    throw Raised();
  }
  if (t.scalar_type() != type) raise(PyExc_ValueError, "expected tensors of one type");
  if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) raise(PyExc_ValueError, "expected a last dimension without gaps");
  return t;
}

const float* optional(PyObject* o, at::IntArrayRef sizes, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.sizes() != sizes) {
    PyErr_Format(PyExc_ValueError, "expected %s of another shape", what);
    throw Raised();
  }
  return data(t);
}

struct Linear {
  cnn_linear_shape shape;
  cnn_heads q, k, v;
  const float* decay;
  float scale;
  at::Device device;
  at::ScalarType type;
  int64_t B, T, H, Hk, Dk, Dv;
};

Linear linear_of(PyObject* const* a, int dims) {  // q, k, v, decay, scale
  if (!THPVariable_Check(a[0])) raise(PyExc_TypeError, "expected a tensor");
  const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
  const at::Tensor &q = heads_tensor(a[0], dims, type), &k = heads_tensor(a[1], dims, type), &v = heads_tensor(a[2], dims, type);
  const int code = element_type(q), h = dims - 2, d = dims - 1;
  const int64_t B = q.size(0), T = dims == 4 ? q.size(1) : 1;
  bool fits = k.size(0) == B && v.size(0) == B && k.size(h) == v.size(h) && k.size(d) == q.size(d);
  if (dims == 4) fits = fits && k.size(1) == T && v.size(1) == T;
  if (!fits) raise(PyExc_ValueError, "expected q, k and v of one batch and length, k and v of as many heads, q and k of one width");
  for (const int64_t n : {B, T, q.size(h), k.size(h), q.size(d), v.size(d)})
    if (n > INT_MAX) raise(PyExc_ValueError, "a dimension is too large");
  const int64_t H = q.size(h), Hk = k.size(h), Dk = q.size(d), Dv = v.size(d);
  const float* decay = a[3] == Py_None ? (raise(PyExc_TypeError, "expected a tensor of decays"), nullptr) : optional(a[3], {H}, "decays");
  return {{(int)B, (int)T, (int)H, (int)Hk, (int)Dk, (int)Dv, code}, heads_of(q), heads_of(k), heads_of(v), decay, (float)number(a[4]), q.device(), type,
          B, T, H, Hk, Dk, Dv};
}

const int32_t* whole_numbers(PyObject* o, int64_t count, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, at::kInt);
  if (t.dim() != 1 || t.size(0) != count) {
    PyErr_Format(PyExc_ValueError, "expected one of %s per sequence", what);
    throw Raised();
  }
  return data<int32_t>(t);
}

PyObject* or_none(at::Tensor t) {
  if (t.defined()) return wrap(std::move(t));
  Py_RETURN_NONE;
}

CALL(linear_attention_fwd, 8)  // q, k, v, decay, scale, lengths or None, initial state or None, want_state
  const Linear x = linear_of(a, 4);
  const int32_t* lengths = whole_numbers(a[5], x.B, "the lengths");
  const float* initial = optional(a[6], {x.B, x.H, x.Dk, x.Dv}, "a state");
  const size_t bytes = cnn_linear_attention_fwd_workspace_bytes(&x.shape);
  at::Tensor o = empty({x.B, x.T, x.H, x.Dv}, x.device, x.type), state, ws;
  if (integer(a[7])) state = empty({x.B, x.H, x.Dk, x.Dv}, x.device);
  if (bytes) ws = empty({(int64_t)bytes}, x.device, at::kByte);
  call("cnn_linear_attention_fwd", [&] {
    return cnn_linear_attention_fwd(&x.shape, &x.q, &x.k, &x.v, x.decay, x.scale, lengths, initial, o.data_ptr(),
                                    state.defined() ? data(state) : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(wrap(std::move(o)), or_none(std::move(state)));
END

CALL(linear_attention_bwd, 10)  // q, k, v, decay, scale, d_o, lengths, initial state, error of the final state, want_d_state
  const Linear x = linear_of(a, 4);
  const at::Tensor& d = heads_tensor(a[5], 4, x.type);
  if (d.sizes() != at::IntArrayRef({x.B, x.T, x.H, x.Dv})) raise(PyExc_ValueError, "expected an output error of the output's shape");
  const cnn_heads d_o = heads_of(d);
  const int32_t* lengths = whole_numbers(a[6], x.B, "the lengths");
  const float* initial = optional(a[7], {x.B, x.H, x.Dk, x.Dv}, "a state");
  const float* d_final = optional(a[8], {x.B, x.H, x.Dk, x.Dv}, "a state's error");
  const size_t bytes = cnn_linear_attention_bwd_workspace_bytes(&x.shape);
  at::Tensor d_q = empty({x.B, x.T, x.H, x.Dk}, x.device, x.type), d_k = empty({x.B, x.T, x.Hk, x.Dk}, x.device, x.type);
  at::Tensor d_v = empty({x.B, x.T, x.Hk, x.Dv}, x.device, x.type), d_state, ws;
  if (integer(a[9])) d_state = empty({x.B, x.H, x.Dk, x.Dv}, x.device);
  if (bytes) ws = empty({(int64_t)bytes}, x.device, at::kByte);
  call("cnn_linear_attention_bwd", [&] {
    return cnn_linear_attention_bwd(&x.shape, &x.q, &x.k, &x.v, x.decay, &d_o, x.scale, lengths, initial, d_final, d_q.data_ptr(), d_k.data_ptr(),
                                    d_v.data_ptr(), d_state.defined() ? data(d_state) : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(pair(wrap(std::move(d_q)), wrap(std::move(d_k))), pair(wrap(std::move(d_v)), or_none(std::move(d_state))));
END

CALL(linear_attention_step, 7)  // q, k, v, decay, scale, state, slots or None
  const Linear x = linear_of(a, 3);
  const at::Tensor& state = tensor(a[5], 4);
  if (state.size(1) != x.H || state.size(2) != x.Dk || state.size(3) != x.Dv) raise(PyExc_ValueError, "expected a pool of states of another shape");
  const int32_t* slots = whole_numbers(a[6], x.B, "the slots");
  at::Tensor o = empty({x.B, x.H, x.Dv}, x.device, x.type);
  call("cnn_linear_attention_step", [&] {
    return cnn_linear_attention_step(&x.shape, &x.q, &x.k, &x.v, x.decay, x.scale, data(state), state.size(0), slots, o.data_ptr(), stream());
  });
  return wrap(std::move(o));
END

// ---- around a block, and the loss ------------------------------------------------------------------------------
// These calls run on the device of their first tensor, whatever the current one is, and want all tensors there.
const at::Tensor& on(const at::Tensor& t, at::Device device) {
  if (t.device() != device) raise(PyExc_ValueError, "expected all tensors on one GPU");
  return t;
}

// Rows of the last dimension, which has no gaps, at one distance.
const at::Tensor& rows_tensor(PyObject* o, cnn_rows* rows) {
  const at::Tensor& t = any_tensor(o, true);
  if (t.dim() < 1) raise(PyExc_ValueError, "expected a tensor of at least 1 dimension");
  const int last = (int)t.dim() - 1;
  if (t.size(last) > 1 && t.stride(last) != 1) raise(PyExc_ValueError, "expected a last dimension without gaps");
  int64_t row = t.size(last), next = -1;  // what the dimension in front would have for a stride
  for (int i = last - 1; i >= 0; --i) {
    if (t.size(i) == 1) continue;
    if (next < 0) row = t.stride(i);
    else if (t.stride(i) != next) raise(PyExc_ValueError, "expected rows at one distance");
    next = t.stride(i) * t.size(i);
  }
  *rows = {t.data_ptr(), row};
  return t;
}

const cnn_rows* rows_or_null(PyObject* o, cnn_rows* rows, const at::Tensor& x, at::ScalarType type, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = on(rows_tensor(o, rows), x.device());
  if (t.scalar_type() != type || t.sizes() != x.sizes()) {
    PyErr_Format(PyExc_ValueError, "expected %s of the same shape and a fitting type", what);
    throw Raised();
  }
  return rows;
}

at::ScalarType type_or(PyObject* o, at::ScalarType type) {
  return THPVariable_Check(o) ? THPVariable_Unpack(o).scalar_type() : type;
}

// x or r [..., groups * width], its weight, scale, eps, groups.
cnn_norm_shape norm_shape(const at::Tensor& x, at::ScalarType type, at::ScalarType stream_type, PyObject* scale, PyObject* eps, PyObject* groups) {
  const auto code = [](at::ScalarType t) {
    return t == at::kFloat ? CNN_F32 : t == at::kBFloat16 ? CNN_BF16 : t == at::kHalf ? CNN_F16 : -1;
  };
  const int64_t D = x.size(-1), G = integer(groups);
  if (G < 1 || G > INT_MAX || D < 1 || D > INT_MAX || D % G) raise(PyExc_ValueError, "expected groups that divide the last dimension");
  if (code(type) < 0 || code(stream_type) < 0 || (stream_type != type && stream_type != at::kFloat))
    raise(PyExc_ValueError, "expected torch.float32, torch.bfloat16 or torch.float16 tensors, of one type or with a residual stream of torch.float32");
  return {x.numel() / D, (int)G, (int)(D / G), code(type), code(stream_type), (float)number(scale), (float)number(eps)};
}

const float* weight_of(PyObject* o, const at::Tensor& x) {
  const at::Tensor& w = on(tensor(o), x.device());
  if (w.dim() != 1 || w.size(0) != x.size(-1)) raise(PyExc_ValueError, "expected one weight for each element of a row");
  return data(w);
}

PyObject* object(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : (Py_INCREF(Py_None), Py_None); }

CALL(add_norm_fwd, 6)  // x, weight, residual or None, scale, eps, groups
  cnn_rows rx, rr;
  const at::Tensor& x = rows_tensor(a[0], &rx);
  const at::ScalarType stream_type = type_or(a[2], x.scalar_type());
  const cnn_norm_shape shape = norm_shape(x, x.scalar_type(), stream_type, a[3], a[4], a[5]);
  const float* weight = weight_of(a[1], x);
  const cnn_rows* residual = rows_or_null(a[2], &rr, x, stream_type, "a residual");
  const c10::DeviceGuard guard(x.device());
  at::Tensor y = empty(x.sizes(), x.device(), x.scalar_type()), r;
  if (residual) r = empty(x.sizes(), x.device(), stream_type);
  call("cnn_add_norm_fwd", [&] { return cnn_add_norm_fwd(&shape, &rx, residual, weight, y.data_ptr(), residual ? r.data_ptr() : nullptr, stream()); });
  return pair(wrap(std::move(y)), residual ? wrap(std::move(r)) : (Py_INCREF(a[0]), a[0]));
END

at::Tensor bytes_on(size_t bytes, at::Device device) { return bytes ? empty({(int64_t)bytes}, device, at::kByte) : at::Tensor(); }

CALL(add_norm_bwd, 7)  // d_y, r, weight, d_r or None, scale, eps, groups
  cnn_rows ry, rr, rd;
  const at::Tensor& r = rows_tensor(a[1], &rr);
  const at::ScalarType type = type_or(a[0], r.scalar_type()), stream_type = r.scalar_type();
  const cnn_norm_shape shape = norm_shape(r, type, stream_type, a[4], a[5], a[6]);
  if (!rows_or_null(a[0], &ry, r, type, "an output error")) raise(PyExc_TypeError, "expected a tensor");
  const float* weight = weight_of(a[2], r);
  const cnn_rows* d_r = rows_or_null(a[3], &rd, r, stream_type, "a residual stream's error");
  const c10::DeviceGuard guard(r.device());
  const bool two = type != stream_type || shape.scale != 1.0f;
  at::Tensor d_residual = empty(r.sizes(), r.device(), stream_type), d_x, d_weight = empty({r.size(-1)}, r.device());
  if (two) d_x = empty(r.sizes(), r.device(), type);
  const size_t bytes = cnn_norm_bwd_workspace_bytes(&shape);
  const at::Tensor ws = bytes_on(bytes, r.device());
  call("cnn_add_norm_bwd", [&] {
    return cnn_add_norm_bwd(&shape, &ry, &rr, d_r, weight, two ? d_x.data_ptr() : nullptr, d_residual.data_ptr(), data(d_weight),
                            bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  PyObject* residual = object(d_residual);
  return pair(pair(two ? object(d_x) : (Py_XINCREF(residual), residual), residual), object(d_weight));
END

CALL(norm_gate_fwd, 7)  // x, weight, gate or None, residual or None, scale, eps, groups
  cnn_rows rx, rg, rr;
  const at::Tensor& x = rows_tensor(a[0], &rx);
  const at::ScalarType stream_type = type_or(a[3], x.scalar_type());
  const cnn_norm_shape shape = norm_shape(x, x.scalar_type(), stream_type, a[4], a[5], a[6]);
  const float* weight = weight_of(a[1], x);
  const cnn_rows *gate = rows_or_null(a[2], &rg, x, x.scalar_type(), "a gate"), *residual = rows_or_null(a[3], &rr, x, stream_type, "a residual");
  const c10::DeviceGuard guard(x.device());
  at::Tensor y = empty(x.sizes(), x.device(), stream_type);
  call("cnn_norm_gate_fwd", [&] { return cnn_norm_gate_fwd(&shape, &rx, gate, residual, weight, y.data_ptr(), stream()); });
  return wrap(std::move(y));
END

CALL(norm_gate_bwd, 7)  // d_y, x, weight, gate or None, scale, eps, groups
  cnn_rows ry, rx, rg;
  const at::Tensor& x = rows_tensor(a[1], &rx);
  const at::ScalarType type = x.scalar_type(), stream_type = type_or(a[0], type);
  const cnn_norm_shape shape = norm_shape(x, type, stream_type, a[4], a[5], a[6]);
  if (!rows_or_null(a[0], &ry, x, stream_type, "an output error")) raise(PyExc_TypeError, "expected a tensor");
  const float* weight = weight_of(a[2], x);
  const cnn_rows* gate = rows_or_null(a[3], &rg, x, type, "a gate");
  const c10::DeviceGuard guard(x.device());
  at::Tensor d_x = empty(x.sizes(), x.device(), type), d_gate, d_weight = empty({x.size(-1)}, x.device());
  if (gate) d_gate = empty(x.sizes(), x.device(), type);
  const size_t bytes = cnn_norm_bwd_workspace_bytes(&shape);
  const at::Tensor ws = bytes_on(bytes, x.device());
  call("cnn_norm_gate_bwd", [&] {
    return cnn_norm_gate_bwd(&shape, &ry, &rx, gate, weight, d_x.data_ptr(), gate ? d_gate.data_ptr() : nullptr, data(d_weight),
                             bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(pair(object(d_x), object(d_gate)), object(d_weight));
END

// logits [..., V] and tokens [...] or [..., M]
struct LogProbs {
  cnn_log_probs_shape shape;
  cnn_rows logits;
  const at::Tensor &x, &tokens;
};

LogProbs log_probs_of(PyObject* logits, PyObject* tokens, PyObject* scale, PyObject* top) {
  cnn_rows rows;
  const at::Tensor& x = rows_tensor(logits, &rows);
  const at::Tensor& t = on(token_tensor(tokens), x.device());
  const int type = element_type(x);
  const int64_t lead = x.dim() - 1, V = x.size(-1), M = t.dim() == lead ? 1 : t.size(-1), k = top ? integer(top) : 0;
  if ((t.dim() != lead && t.dim() != lead + 1) || t.sizes().slice(0, lead) != x.sizes().slice(0, lead))
    raise(PyExc_ValueError, "expected one token, or as many as the last dimension of tokens says, for each row of logits");
  if (V < 1) raise(PyExc_ValueError, "expected logits");
  if (M > INT_MAX) raise(PyExc_ValueError, "a dimension is too large");
  if (k < 0 || k > V || k > INT_MAX) raise(PyExc_ValueError, "expected no more top tokens than a row has");
  return {{x.numel() / V, V, (int)M, (int)k, type, t.scalar_type() == at::kLong, (float)number(scale)}, rows, x, t};
}

CALL(log_probs_fwd, 4)  // logits, tokens, scale, top
  const LogProbs l = log_probs_of(a[0], a[1], a[2], a[3]);
  const at::Device device = l.x.device();
  const c10::DeviceGuard guard(device);
  const std::vector<int64_t> lead(l.x.sizes().begin(), l.x.sizes().end() - 1);
  const auto with = [&](int64_t n) {
    std::vector<int64_t> sizes = lead;
    sizes.push_back(n);
    return sizes;
  };
  const int top = l.shape.top;
  at::Tensor log_probs = empty(l.tokens.sizes(), device), entropy = empty(lead, device), stats = empty(with(3), device), top_log_probs, top_tokens;
  if (top) top_log_probs = empty(with(top), device), top_tokens = empty(with(top), device, at::kInt);
  const size_t bytes = cnn_log_probs_fwd_workspace_bytes(&l.shape);
  const at::Tensor ws = bytes_on(bytes, device);
  call("cnn_log_probs_fwd", [&] {
    return cnn_log_probs_fwd(&l.shape, &l.logits, l.tokens.data_ptr(), data(log_probs), data(entropy), data(stats), top ? data(top_log_probs) : nullptr,
                             top ? data<int32_t>(top_tokens) : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(pair(object(log_probs), object(entropy)), pair(object(stats), pair(object(top_log_probs), object(top_tokens))));
END

CALL(log_probs_bwd, 6)  // logits, tokens, stats, d_log_probs, d_entropy or None, scale
  const LogProbs l = log_probs_of(a[0], a[1], a[5], nullptr);
  const at::Device device = l.x.device();
  const at::Tensor &stats = on(tensor(a[2]), device), &d = on(tensor(a[3]), device);
  const at::IntArrayRef lead = l.x.sizes().slice(0, l.x.dim() - 1);
  if (stats.dim() != l.x.dim() || stats.sizes().slice(0, lead.size()) != lead || stats.size(-1) != 3) raise(PyExc_ValueError, "expected the stats of the forward call");
  if (d.sizes() != l.tokens.sizes()) raise(PyExc_ValueError, "expected an error for each given token");
  const float* d_entropy = optional(a[4], lead, "an entropy's error");
  if (d_entropy) on(THPVariable_Unpack(a[4]), device);
  const c10::DeviceGuard guard(device);
  at::Tensor d_logits = empty(l.x.sizes(), device, l.x.scalar_type());
  call("cnn_log_probs_bwd", [&] {
    return cnn_log_probs_bwd(&l.shape, &l.logits, l.tokens.data_ptr(), data(stats), data(d), d_entropy, d_logits.data_ptr(), stream());
  });
  return wrap(std::move(d_logits));
END

// A [batch, token, width] (the step's: [batch, width]) tensor with whatever strides, its last dimension without gaps.
const at::Tensor& tokens_tensor(PyObject* o, int dims, cnn_tokens* tokens) {
  const at::Tensor& t = any_tensor(o, true);
  if (t.dim() != dims) {
    PyErr_Format(PyExc_ValueError, "expected %d dimensions, got %d", dims, (int)t.dim());
    throw Raised();
  }
  for (int i = 0; i < dims; ++i)
    if (t.size(i) > INT_MAX) raise(PyExc_ValueError, "a dimension is too large");
  if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) raise(PyExc_ValueError, "expected a last dimension without gaps");
  *tokens = {t.data_ptr(), t.stride(0), dims == 3 && t.size(1) > 1 ? t.stride(1) : 0};  // (a single token's stride may be anything)
  return t;
}

const cnn_tokens& same_tokens(PyObject* o, cnn_tokens* tokens, const at::Tensor& x) {
  const at::Tensor& t = on(tokens_tensor(o, (int)x.dim(), tokens), x.device());
  if (t.scalar_type() != x.scalar_type() || t.sizes() != x.sizes()) raise(PyExc_ValueError, "expected tensors of one shape and type");
  return *tokens;
}

// A contiguous tensor of a type and shape, on a device.
void* optional_on(PyObject* o, at::IntArrayRef sizes, at::ScalarType type, at::Device device, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = on(any_tensor(o), device);
  if (t.scalar_type() != type || t.sizes() != sizes) {
    PyErr_Format(PyExc_ValueError, "expected %s of another shape or type", what);
    throw Raised();
  }
  return t.data_ptr();
}

struct Conv {
  cnn_causal_conv_shape shape;
  cnn_tokens tokens;
  const at::Tensor& x;
  const float *weight, *bias;
  int64_t B, T, D, K;
};

Conv conv_of(PyObject* const* a, int dims) {  // x, weight, bias or None, silu
  cnn_tokens tokens;
  const at::Tensor &x = tokens_tensor(a[0], dims, &tokens), &w = on(tensor(a[1]), x.device());
  const int type = element_type(x);
  const int64_t B = x.size(0), T = dims == 3 ? x.size(1) : 1, D = x.size(dims - 1);
  if (w.dim() != 2 || w.size(0) != D || w.size(1) > INT_MAX) raise(PyExc_ValueError, "expected a weight of a few taps for each channel");
  const int64_t K = w.size(1);
  const float* bias = static_cast<const float*>(optional_on(a[2], {D}, at::kFloat, x.device(), "a bias"));
  return {{(int)B, (int)T, (int)D, (int)K, type, integer(a[3]) != 0}, tokens, x, data(w), bias, B, T, D, K};
}

const int32_t* lengths_on(PyObject* o, int64_t count, at::Device device, const char* what) {
  return static_cast<const int32_t*>(optional_on(o, {count}, at::kInt, device, what));
}

CALL(causal_conv_fwd, 7)  // x, weight, bias or None, silu, lengths or None, initial state or None, want_state
  const Conv c = conv_of(a, 3);
  const at::Device device = c.x.device();
  const at::ScalarType type = c.x.scalar_type();
  const int32_t* lengths = lengths_on(a[4], c.B, device, "one length per sequence (torch.int32)");
  const void* initial = optional_on(a[5], {c.B, c.K - 1, c.D}, type, device, "a state");
  const c10::DeviceGuard guard(device);
  at::Tensor y = empty({c.B, c.T, c.D}, device, type), state;
  if (integer(a[6]) && c.K > 1) state = empty({c.B, c.K - 1, c.D}, device, type);
  call("cnn_causal_conv_fwd", [&] {
    return cnn_causal_conv_fwd(&c.shape, &c.tokens, c.weight, c.bias, lengths, initial, y.data_ptr(), state.defined() ? state.data_ptr() : nullptr, stream());
  });
  return pair(wrap(std::move(y)), or_none(std::move(state)));
END

CALL(causal_conv_bwd, 9)  // x, weight, bias or None, silu, d_y, lengths, initial state, error of the final state, want_d_state
  const Conv c = conv_of(a, 3);
  const at::Device device = c.x.device();
  const at::ScalarType type = c.x.scalar_type();
  cnn_tokens d_tokens;
  const cnn_tokens& d_y = same_tokens(a[4], &d_tokens, c.x);
  const int32_t* lengths = lengths_on(a[5], c.B, device, "one length per sequence (torch.int32)");
  const void* initial = optional_on(a[6], {c.B, c.K - 1, c.D}, type, device, "a state");
  const void* d_final = optional_on(a[7], {c.B, c.K - 1, c.D}, type, device, "a state's error");
  const c10::DeviceGuard guard(device);
  const size_t bytes = cnn_causal_conv_bwd_workspace_bytes(&c.shape);
  at::Tensor d_x = empty({c.B, c.T, c.D}, device, type), d_weight = empty({c.D, c.K}, device), d_bias, d_state;
  if (c.bias) d_bias = empty({c.D}, device);
  if (integer(a[8]) && c.K > 1) d_state = empty({c.B, c.K - 1, c.D}, device, type);
  const at::Tensor ws = bytes_on(bytes, device);
  call("cnn_causal_conv_bwd", [&] {
    return cnn_causal_conv_bwd(&c.shape, &c.tokens, &d_y, c.weight, c.bias, lengths, initial, d_final, d_x.data_ptr(), data(d_weight),
                               c.bias ? data(d_bias) : nullptr, d_state.defined() ? d_state.data_ptr() : nullptr, bytes ? ws.data_ptr() : nullptr, bytes,
                               stream());
  });
  return pair(pair(object(d_x), object(d_weight)), pair(object(d_bias), object(d_state)));
END

CALL(causal_conv_step, 6)  // x, weight, bias or None, silu, state, slots or None
  const Conv c = conv_of(a, 2);
  const at::Device device = c.x.device();
  const at::Tensor& state = on(any_tensor(a[4]), device);
  if (state.dim() != 3 || state.size(1) != c.K - 1 || state.size(2) != c.D || state.scalar_type() != c.x.scalar_type())
    raise(PyExc_ValueError, "expected a pool of states of another shape or type");
  const int32_t* slots = lengths_on(a[5], c.B, device, "one slot per sequence (torch.int32)");
  const c10::DeviceGuard guard(device);
  at::Tensor y = empty({c.B, c.D}, device, c.x.scalar_type());
  call("cnn_causal_conv_step", [&] {
    return cnn_causal_conv_step(&c.shape, &c.tokens, c.weight, c.bias, state.data_ptr(), state.size(0), slots, y.data_ptr(), stream());
  });
  return wrap(std::move(y));
END

struct Scan {
  cnn_selective_scan_shape shape;
  cnn_tokens x, dt;
  cnn_heads b, c;
  const float *a, *skip, *dt_bias;
  const at::Tensor& first;  // x
  at::Device device;
  at::ScalarType type;
  int64_t B, T, D, N, G;
};

Scan scan_of(PyObject* const* a, int dims) {  // x, dt, a, b, c, skip or None, dt_bias or None, softplus
  cnn_tokens x, dt;
  const at::Tensor& t = tokens_tensor(a[0], dims, &x);
  const at::Device device = t.device();
  const at::ScalarType type = t.scalar_type();
  const int code = element_type(t);
  same_tokens(a[1], &dt, t);
  const at::Tensor &b = on(heads_tensor(a[3], dims + 1, type), device), &c = on(heads_tensor(a[4], dims + 1, type), device), &w = on(tensor(a[2]), device);
  const int64_t B = t.size(0), T = dims == 3 ? t.size(1) : 1, D = t.size(dims - 1), G = b.size(dims - 1), N = b.size(dims);
  if (b.sizes() != c.sizes() || b.size(0) != B || (dims == 3 && b.size(1) != T)) raise(PyExc_ValueError, "expected b and c of one shape, of x's batch and length");
  for (const int64_t n : {G, N})
    if (n > INT_MAX) raise(PyExc_ValueError, "a dimension is too large");
  if (w.sizes() != at::IntArrayRef({D, N})) raise(PyExc_ValueError, "expected a of as many rows as channels and as many columns as b and c");
  const float* skip = static_cast<const float*>(optional_on(a[5], {D}, at::kFloat, device, "a skip"));
  const float* bias = static_cast<const float*>(optional_on(a[6], {D}, at::kFloat, device, "a bias"));
  const auto bc = [&](const at::Tensor& h) {
    cnn_heads v = heads_of(h);
    if (T == 1) v.token = 0;
    return v;
  };
  return {{(int)B, (int)T, (int)D, (int)N, (int)G, code, integer(a[7]) != 0}, x, dt, bc(b), bc(c), data(w), skip, bias, t, device, type, B, T, D, N, G};
}

CALL(selective_scan_fwd, 11)  // as scan_of, lengths or None, initial state or None, want_state
  const Scan s = scan_of(a, 3);
  const int32_t* lengths = lengths_on(a[8], s.B, s.device, "one length per sequence (torch.int32)");
  const float* initial = static_cast<const float*>(optional_on(a[9], {s.B, s.D, s.N}, at::kFloat, s.device, "a state"));
  const c10::DeviceGuard guard(s.device);
  const size_t bytes = cnn_selective_scan_fwd_workspace_bytes(&s.shape);
  at::Tensor y = empty({s.B, s.T, s.D}, s.device, s.type), state;
  if (integer(a[10])) state = empty({s.B, s.D, s.N}, s.device);
  const at::Tensor ws = bytes_on(bytes, s.device);
  call("cnn_selective_scan_fwd", [&] {
    return cnn_selective_scan_fwd(&s.shape, &s.x, &s.dt, s.a, &s.b, &s.c, s.skip, s.dt_bias, lengths, initial, y.data_ptr(),
                                  state.defined() ? data(state) : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  return pair(wrap(std::move(y)), or_none(std::move(state)));
END

CALL(selective_scan_bwd, 13)  // as scan_of, d_y, lengths, initial state, error of the final state, want_d_state
  const Scan s = scan_of(a, 3);
  cnn_tokens d_y;
  same_tokens(a[8], &d_y, s.first);
  const int32_t* lengths = lengths_on(a[9], s.B, s.device, "one length per sequence (torch.int32)");
  const float* initial = static_cast<const float*>(optional_on(a[10], {s.B, s.D, s.N}, at::kFloat, s.device, "a state"));
  const float* d_final = static_cast<const float*>(optional_on(a[11], {s.B, s.D, s.N}, at::kFloat, s.device, "a state's error"));
  const c10::DeviceGuard guard(s.device);
  const size_t bytes = cnn_selective_scan_bwd_workspace_bytes(&s.shape);
  at::Tensor d_x = empty({s.B, s.T, s.D}, s.device, s.type), d_dt = empty({s.B, s.T, s.D}, s.device, s.type), d_a = empty({s.D, s.N}, s.device);
  at::Tensor d_b = empty({s.B, s.T, s.G, s.N}, s.device, s.type), d_c = empty({s.B, s.T, s.G, s.N}, s.device, s.type), d_skip, d_bias, d_state;
  if (s.skip) d_skip = empty({s.D}, s.device);
  if (s.dt_bias) d_bias = empty({s.D}, s.device);
  if (integer(a[12])) d_state = empty({s.B, s.D, s.N}, s.device);
  const at::Tensor ws = bytes_on(bytes, s.device);
  const auto or_null = [](const at::Tensor& t) { return t.defined() ? data(t) : nullptr; };
  call("cnn_selective_scan_bwd", [&] {
    return cnn_selective_scan_bwd(&s.shape, &s.x, &s.dt, s.a, &s.b, &s.c, &d_y, s.skip, s.dt_bias, lengths, initial, d_final, d_x.data_ptr(), d_dt.data_ptr(),
                                  data(d_a), d_b.data_ptr(), d_c.data_ptr(), or_null(d_skip), or_null(d_bias), or_null(d_state),
                                  bytes ? ws.data_ptr() : nullptr, bytes, stream());
  });
  PyObject* all = PyTuple_New(8);
  if (!all) throw Raised();
  int i = 0;
  for (const at::Tensor* t : {&d_x, &d_dt, &d_a, &d_b, &d_c, &d_skip, &d_bias, &d_state}) PyTuple_SET_ITEM(all, i++, object(*t));
  return all;
END

CALL(selective_scan_step, 10)  // as scan_of, state, slots or None
  const Scan s = scan_of(a, 2);
  const at::Tensor& state = on(tensor(a[8], 3), s.device);
  if (state.size(1) != s.D || state.size(2) != s.N) raise(PyExc_ValueError, "expected a pool of states of another shape");
  const int32_t* slots = lengths_on(a[9], s.B, s.device, "one slot per sequence (torch.int32)");
  const c10::DeviceGuard guard(s.device);
  at::Tensor y = empty({s.B, s.D}, s.device, s.type);
  call("cnn_selective_scan_step", [&] {
    return cnn_selective_scan_step(&s.shape, &s.x, &s.dt, s.a, &s.b, &s.c, s.skip, s.dt_bias, data(state), state.size(0), slots, y.data_ptr(), stream());
  });
  return wrap(std::move(y));
END

PyObject* raise_through(PyObject*, PyObject* fn) {  // binding._check
  Py_INCREF(fn);
  Py_XSETREF(check, fn);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(forward), FAST(gradient), FAST(train_batch), FAST(evaluate), FAST(conv_fwd), FAST(conv_bwd_input),
                         FAST(conv_bwd_weight), FAST(avgpool_fwd), FAST(avgpool_bwd), FAST(fc_fwd), FAST(fc_bwd_input),
                         FAST(fc_bwd_weight), FAST(logistic_fwd), FAST(logistic_bwd), FAST(embedding_fwd), FAST(embedding_bwd), FAST(dropout_fwd),
                         FAST(dropout_bwd), FAST(linear_attention_fwd), FAST(linear_attention_bwd), FAST(linear_attention_step),
                         FAST(add_norm_fwd), FAST(add_norm_bwd), FAST(norm_gate_fwd), FAST(norm_gate_bwd), FAST(log_probs_fwd), FAST(log_probs_bwd),
                         FAST(causal_conv_fwd), FAST(causal_conv_bwd), FAST(causal_conv_step),
                         FAST(selective_scan_fwd), FAST(selective_scan_bwd), FAST(selective_scan_step),
                         {"raise_through", raise_through, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
