// Python binding of the encoder-block, attention and rotary entry points, as a CPython extension.
//
// It checks and marshals torch tensors and allocates outputs, as mpm.py does
// for the merge through ctypes; every step of the computation is the C ABI's,
// whose addresses blocks.py hands over at start.  Small calls are bound by the
// host, and these take up to thirty arguments: one row through block_norm took
// 19 us a call through ctypes (14 with every check in one expression), 4.4 here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <utility>

#include "mpm.h"

namespace {

struct EntryPoints {
  decltype(&mpm_block_norm) block_norm;
  decltype(&mpm_block_norm_workspace_size) block_norm_workspace_size;
  decltype(&mpm_block_norm_backward) block_norm_backward;
  decltype(&mpm_mxfp4_quantize) mxfp4_quantize;
  decltype(&mpm_mxfp4_dequantize) mxfp4_dequantize;
  decltype(&mpm_mxfp4_matmul) mxfp4_matmul;
  decltype(&mpm_cross_attention) cross_attention;
  decltype(&mpm_cross_attention_workspace_size) cross_attention_workspace_size;
  decltype(&mpm_cross_attention_backward) cross_attention_backward;
  decltype(&mpm_cross_attention_backward_workspace_size) cross_attention_backward_workspace_size;
  decltype(&mpm_rotary) rotary;
};
EntryPoints entry = {};
PyObject* raise_status = nullptr;  // Python callable (name, code) that raises the library's error

// A Python exception that has been set; unwinds to the entry point.
struct Raised {};

[[noreturn]] void value_error(const char* name, const char* what) {
  PyErr_Format(PyExc_ValueError, "%s %s", name, what);
  throw Raised{};
}
[[noreturn]] void type_error(const char* name, const char* what) {
  PyErr_Format(PyExc_TypeError, "%s %s", name, what);
  throw Raised{};
}

void check(const char* name, int code) {
  if (code == MPM_OK) return;
  PyObject* r = PyObject_CallFunction(raise_status, "si", name, code);
  Py_XDECREF(r);
  if (r != nullptr) PyErr_SetString(PyExc_RuntimeError, "an error was not raised");
  throw Raised{};
}

// A CUDA tensor, or null where None is allowed.
const at::Tensor* tensor(PyObject* o, const char* name, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) value_error(name, "must be a CUDA tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) value_error(name, "must be a CUDA tensor");
  // Outputs belong to no graph: a gradient would be lost without a word.
  if (t.requires_grad() && c10::GradMode::is_enabled())
    value_error(name, "must not require grad outside torch.no_grad(): the block operators record nothing for autograd");
  return &t;
}

mpm_dtype dtype_of(const at::Tensor& t, const char* name) {
  if (t.scalar_type() == at::kBFloat16) return MPM_BF16;
  if (t.scalar_type() == at::kFloat) return MPM_F32;
  type_error(name, "must be bfloat16 or float32");
}

// A matrix of bf16 or fp32 rows, each contiguous, any distance apart; of the
// shape and on the device of `like` if that is given.
const at::Tensor* rows_of(PyObject* o, const char* name, const at::Tensor* like = nullptr, bool optional = false) {
  const at::Tensor* t = tensor(o, name, optional);
  if (t == nullptr) return nullptr;
  if (t->dim() != 2) value_error(name, "must have 2 dimensions");
  if (like != nullptr) {
    if (t->get_device() != like->get_device()) value_error(name, "must be on the other tensors' device");
    if (t->sizes() != like->sizes()) value_error(name, "must have the tokens' shape");
  }
  dtype_of(*t, name);
  if ((t->size(1) > 1 && t->stride(1) != 1) || (t->size(0) > 1 && t->stride(0) < t->size(1)))
    value_error(name, "must have contiguous rows that do not overlap");
  return t;
}

// The address of a contiguous tensor of the given type and shape (null for none, or an empty one).
void* buffer(PyObject* o, const char* name, at::ScalarType type, int64_t device, at::IntArrayRef shape, bool optional = true) {
  const at::Tensor* t = tensor(o, name, optional);
  if (t == nullptr) return nullptr;
  if (t->scalar_type() != type) type_error(name, type == at::kFloat ? "must be float32" : "has the wrong type");
  if (t->get_device() != device) value_error(name, "must be on the other tensors' device");
  if (!t->is_contiguous()) value_error(name, "must be contiguous");
  if (shape.data() != nullptr && t->sizes() != shape) value_error(name, "has the wrong shape");
  return t->data_ptr();
}
float* parameter(PyObject* o, const char* name, int64_t device, at::IntArrayRef shape) {
  return static_cast<float*>(buffer(o, name, at::kFloat, device, shape));
}
int32_t* status_word(PyObject* o, int64_t device) {
  const at::Tensor* t = tensor(o, "device_status", true);
  if (t == nullptr) return nullptr;
  if (t->scalar_type() != at::kInt) type_error("device_status", "must be int32");
  if (t->get_device() != device || t->numel() < 2 || !t->is_contiguous())
    value_error("device_status", "must be an int32 [2] tensor on the other tensors' device");
  return static_cast<int32_t*>(t->data_ptr());
}

// A new contiguous tensor on t's device, without the dispatcher on the way
// (a backward pass makes up to eight: 13.4 us of host time with it, 10.3 without).
at::Tensor new_like(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type) {
  return at::Tensor(at::detail::empty_cuda(shape, type, t.device(), at::MemoryFormat::Contiguous));
}

// A tensor of the caller's has been written: autograd's check of saved tensors goes by the version.
void written(PyObject* o) {
  if (o == Py_None) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();  // (those have none)
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}
int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
at::ScalarType token_type(PyObject* o, const char* name) {
  if (THPDtype_Check(o)) {
    const at::ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
    if (t == at::kBFloat16 || t == at::kFloat) return t;
  }
  type_error(name, "must be torch.bfloat16 or torch.float32");
}

// A new tuple of references that it takes over; null entries are None.
PyObject* tuple_of(std::initializer_list<PyObject*> items) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(items.size()));
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (o == nullptr) {
      Py_INCREF(Py_None);
      o = Py_None;
    }
    if (r != nullptr) PyTuple_SET_ITEM(r, i++, o);
    else Py_DECREF(o);
  }
  return r;
}
PyObject* wrapped(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : nullptr; }
PyObject* again(PyObject* o) {
  Py_INCREF(o);
  return o;
}

// Sets the device that a call's tensors are on, and has its current stream.
struct OnDevice {
  c10::cuda::CUDAGuard guard;
  void* stream;
  explicit OnDevice(int64_t device)
      : guard(static_cast<c10::DeviceIndex>(device)),
        stream(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream()) {}
};

// The arguments that both directions of block_norm share.
struct NormArgs {
  const at::Tensor *y, *residual;
  int64_t device, rows, dim;
  mpm_dtype dtype, stream_dtype;
  mpm_norm_kind norm;
  const int64_t* offsets = nullptr;
  int64_t batch = 1;
  float *pre_weight, *pre_bias, *post_weight, *post_bias, *gate = nullptr;
  int32_t per_image = 0;
  float scale, eps;

  // y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets, residual_scale, eps
  explicit NormArgs(PyObject* const* p) {
    y = rows_of(p[0], "y");
    residual = rows_of(p[1], "residual", y);
    device = y->get_device();
    rows = y->size(0);
    dim = y->size(1);
    if (dim > INT32_MAX) value_error("y", "has too many features");
    dtype = dtype_of(*y, "y");
    stream_dtype = dtype_of(*residual, "residual");
    if (!PyUnicode_Check(p[2])) type_error("norm", "must be a string");
    if (PyUnicode_CompareWithASCIIString(p[2], "layer") == 0) norm = MPM_NORM_LAYER;
    else if (PyUnicode_CompareWithASCIIString(p[2], "rms") == 0) norm = MPM_NORM_RMS;
    else value_error("norm", "must be 'layer' or 'rms'");
    const int64_t vector[1] = {dim};
    pre_weight = parameter(p[3], "pre_weight", device, vector);
    pre_bias = parameter(p[4], "pre_bias", device, vector);
    post_weight = parameter(p[5], "post_weight", device, vector);
    post_bias = parameter(p[6], "post_bias", device, vector);
    if (pre_bias != nullptr && p[3] == Py_None) value_error("pre_bias", "needs pre_weight");
    if (post_bias != nullptr && p[5] == Py_None) value_error("post_bias", "needs post_weight");
    if (const at::Tensor* o = tensor(p[8], "offsets", true)) {
      if (o->scalar_type() != at::kLong) type_error("offsets", "must be int64");
      if (o->dim() != 1 || o->numel() < 2 || o->get_device() != device || !o->is_contiguous())
        value_error("offsets", "must be a contiguous [B+1] tensor on the other tensors' device");
      offsets = static_cast<const int64_t*>(o->data_ptr());
      batch = o->numel() - 1;
      if (batch > INT32_MAX) value_error("offsets", "has too many images");
    }
    if (const at::Tensor* g = tensor(p[7], "gate", true)) {
      per_image = g->dim() == 2;
      if (per_image && offsets == nullptr) value_error("gate", "per image needs offsets");
      const int64_t matrix[2] = {batch, dim};
      gate = parameter(p[7], "gate", device, per_image ? at::IntArrayRef(matrix, 2) : at::IntArrayRef(vector, 1));
    }
    scale = static_cast<float>(number(p[9]));
    eps = static_cast<float>(number(p[10]));
  }
};

// block_norm(<NormArgs>, residual_out, h, with_stats, device_status)
PyObject* block_norm(PyObject* const* p) {
  const NormArgs a(p);
  const OnDevice on(a.device);
  at::Tensor out, h, stats;
  void *pout, *ph = nullptr;
  if (p[11] == Py_None) {
    out = new_like(*a.residual, a.y->sizes(), a.residual->scalar_type());
    pout = out.data_ptr();
  } else {
    pout = buffer(p[11], "residual_out", a.residual->scalar_type(), a.device, a.y->sizes());
  }
  const bool pre = p[3] != Py_None;
  if (!pre) {
    if (p[12] != Py_None) value_error("h", "needs pre_weight");
  } else if (p[12] == Py_None) {
    h = new_like(*a.y, a.y->sizes(), a.y->scalar_type());
    ph = h.data_ptr();
  } else {
    ph = buffer(p[12], "h", a.y->scalar_type(), a.device, a.y->sizes());
  }
  if (truth(p[13])) stats = new_like(*a.y, {a.rows, 4}, at::kFloat);
  check("mpm_block_norm",
        entry.block_norm(a.y->data_ptr(), a.y->stride(0), a.residual->data_ptr(), a.residual->stride(0), a.offsets,
                         static_cast<int32_t>(a.batch), a.rows, static_cast<int32_t>(a.dim), a.dtype, a.stream_dtype, a.norm,
                         a.eps, a.scale, a.post_weight, a.post_bias, a.gate, a.per_image, a.pre_weight, a.pre_bias, pout, ph,
                         stats.defined() ? static_cast<float*>(stats.data_ptr()) : nullptr, status_word(p[14], a.device),
                         on.stream));
  written(p[11]);
  written(p[12]);
  return tuple_of({out.defined() ? wrapped(out) : again(p[11]), h.defined() ? wrapped(h) : pre ? again(p[12]) : nullptr,
                   wrapped(stats)});
}

// block_norm_backward(<NormArgs>, d_residual_out, d_h, stats, workspace, device_status)
PyObject* block_norm_backward(PyObject* const* p) {
  const NormArgs a(p);
  const OnDevice on(a.device);
  const at::Tensor* dxo = rows_of(p[11], "d_residual_out", a.y, true);
  const at::Tensor* dh = rows_of(p[12], "d_h", a.y, true);
  if (dh != nullptr && p[3] == Py_None) value_error("d_h", "needs pre_weight");
  if (dh != nullptr && dh->scalar_type() != a.y->scalar_type()) type_error("d_h", "must have y's type");
  if (dxo != nullptr && dxo->scalar_type() != a.residual->scalar_type())
    type_error("d_residual_out", "must have the residual's type");
  const int64_t four[2] = {a.rows, 4};
  const float* stats = static_cast<float*>(buffer(p[13], "stats", at::kFloat, a.device, four, false));
  at::Tensor workspace;
  void* pws;
  int64_t ws_bytes;
  if (p[14] == Py_None) {
    ws_bytes = static_cast<int64_t>(entry.block_norm_workspace_size(static_cast<int32_t>(a.dim)));
    workspace = new_like(*a.y, {ws_bytes}, at::kByte);
    pws = workspace.data_ptr();
  } else {
    pws = buffer(p[14], "workspace", at::kByte, a.device, at::IntArrayRef());
    ws_bytes = THPVariable_Unpack(p[14]).numel();
  }
  at::Tensor dy = new_like(*a.y, a.y->sizes(), a.y->scalar_type());
  at::Tensor dx = new_like(*a.residual, a.y->sizes(), a.residual->scalar_type());
  const int64_t vector[1] = {a.dim}, matrix[2] = {a.batch, a.dim};
  auto gradient = [&](PyObject* parameter, at::IntArrayRef shape) {
    return parameter == Py_None ? at::Tensor() : new_like(*a.y, shape, at::kFloat);
  };
  at::Tensor d_gate = gradient(p[7], a.per_image ? at::IntArrayRef(matrix, 2) : at::IntArrayRef(vector, 1));
  at::Tensor d_wpost = gradient(p[5], vector), d_bpost = gradient(p[6], vector);
  at::Tensor d_wpre = gradient(p[3], vector), d_bpre = gradient(p[4], vector);
  auto address = [](at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
  check("mpm_block_norm_backward",
        entry.block_norm_backward(
            dxo == nullptr ? nullptr : dxo->data_ptr(), dxo == nullptr ? 0 : dxo->stride(0),
            dh == nullptr ? nullptr : dh->data_ptr(), dh == nullptr ? 0 : dh->stride(0), a.y->data_ptr(), a.y->stride(0),
            a.residual->data_ptr(), a.residual->stride(0), stats, a.offsets, static_cast<int32_t>(a.batch), a.rows,
            static_cast<int32_t>(a.dim), a.dtype, a.stream_dtype, a.norm, a.scale, a.post_weight, a.post_bias, a.gate,
            a.per_image, a.pre_weight, dy.data_ptr(), dx.data_ptr(), address(d_wpost), address(d_bpost), address(d_gate),
            address(d_wpre), address(d_bpre), pws, static_cast<size_t>(ws_bytes), status_word(p[15], a.device), on.stream));
  return tuple_of({wrapped(dy), wrapped(dx), wrapped(d_gate), wrapped(d_wpost), wrapped(d_bpost), wrapped(d_wpre),
                   wrapped(d_bpre)});
}

// Codes and scales of an MXFP4 matrix.
struct Mx {
  const at::Tensor* codes;
  int64_t device, rows, dim;
  uint8_t *pcodes, *pscales;
  Mx(PyObject* c, PyObject* s, PyObject* d, const char* name, int64_t on = -1) {
    codes = tensor(c, name);
    dim = whole(d);
    device = on < 0 ? codes->get_device() : on;
    if (codes->dim() != 2 || dim < 1 || dim > MPM_MXFP4_MAX_DIM) value_error(name, "must be codes [rows, ..] of dim values a row");
    rows = codes->size(0);
    const int64_t code_shape[2] = {rows, (dim + 63) / 64 * 32};
    const int64_t scale_shape[3] = {(rows + 127) / 128, (dim + 127) / 128, 512};
    pcodes = static_cast<uint8_t*>(buffer(c, name, at::kByte, device, code_shape, false));
    pscales = static_cast<uint8_t*>(buffer(s, name, at::kByte, device, scale_shape, false));
  }
};

// quantize(tokens, codes, scales): new codes and scales where None
PyObject* quantize(PyObject* const* p) {
  const at::Tensor* x = rows_of(p[0], "tokens");
  const int64_t rows = x->size(0), dim = x->size(1);
  const OnDevice on(x->get_device());
  at::Tensor codes, scales;
  uint8_t *pc, *ps;
  if (p[1] == Py_None) {
    codes = new_like(*x, {rows, (dim + 63) / 64 * 32}, at::kByte);
    scales = new_like(*x, {(rows + 127) / 128, (dim + 127) / 128, 512}, at::kByte);
    pc = static_cast<uint8_t*>(codes.data_ptr());
    ps = static_cast<uint8_t*>(scales.data_ptr());
  } else {
    const int64_t code_shape[2] = {rows, (dim + 63) / 64 * 32};
    const int64_t scale_shape[3] = {(rows + 127) / 128, (dim + 127) / 128, 512};
    pc = static_cast<uint8_t*>(buffer(p[1], "out.codes", at::kByte, x->get_device(), code_shape, false));
    ps = static_cast<uint8_t*>(buffer(p[2], "out.scales", at::kByte, x->get_device(), scale_shape, false));
  }
  check("mpm_mxfp4_quantize", entry.mxfp4_quantize(x->data_ptr(), x->stride(0), rows,
                                                   static_cast<int32_t>(dim > INT32_MAX ? INT32_MAX : dim),
                                                   dtype_of(*x, "tokens"), pc, ps, on.stream));
  written(p[1]);
  written(p[2]);
  return tuple_of({codes.defined() ? wrapped(codes) : again(p[1]), scales.defined() ? wrapped(scales) : again(p[2])});
}

// A matrix to write into: `out`, or a new one of the given type.
at::Tensor output(PyObject* out, PyObject* dtype, const at::Tensor& on, int64_t rows, int64_t cols) {
  if (out == Py_None) return new_like(on, {rows, cols}, token_type(dtype, "the output's type"));
  const at::Tensor* t = rows_of(out, "out");
  if (t->get_device() != on.get_device()) value_error("out", "must be on the other tensors' device");
  if (t->size(0) != rows || t->size(1) != cols) value_error("out", "has the wrong shape");
  return *t;
}

// dequantize(codes, scales, dim, dtype, out)
PyObject* dequantize(PyObject* const* p) {
  const Mx x(p[0], p[1], p[2], "x");
  const OnDevice on(x.device);
  const at::Tensor out = output(p[4], p[3], *x.codes, x.rows, x.dim);
  check("mpm_mxfp4_dequantize", entry.mxfp4_dequantize(x.pcodes, x.pscales, x.rows, static_cast<int32_t>(x.dim),
                                                       dtype_of(out, "out"), out.data_ptr(), out.stride(0), on.stream));
  written(p[4]);
  return p[4] == Py_None ? THPVariable_Wrap(out) : again(p[4]);
}

// matmul(a.codes, a.scales, a.dim, b.codes, b.scales, b.dim, bias, dtype, out, device_status)
PyObject* matmul(PyObject* const* p) {
  const Mx a(p[0], p[1], p[2], "a");
  const Mx b(p[3], p[4], p[5], "b", a.device);
  if (a.dim != b.dim) value_error("a and b", "must have as many features");
  const OnDevice on(a.device);
  const int64_t vector[1] = {b.rows};
  const float* bias = parameter(p[6], "bias", a.device, vector);
  const at::Tensor out = output(p[8], p[7], *a.codes, a.rows, b.rows);
  check("mpm_mxfp4_matmul",
        entry.mxfp4_matmul(a.pcodes, a.pscales, a.rows, b.pcodes, b.pscales,
                           static_cast<int32_t>(b.rows > INT32_MAX ? INT32_MAX : b.rows), static_cast<int32_t>(a.dim), bias,
                           dtype_of(out, "out"), out.data_ptr(), out.stride(0), status_word(p[9], a.device), on.stream));
  written(p[8]);
  return p[8] == Py_None ? THPVariable_Wrap(out) : again(p[8]);
}

// [rows, heads, head_dim] bf16 or fp32 values with contiguous heads, any distance apart.
const at::Tensor* heads_of(PyObject* o, const char* name) {
  const at::Tensor* t = tensor(o, name);
  if (t->dim() != 3) value_error(name, "must be [rows, heads, head_dim]");
  dtype_of(*t, name);
  if (t->size(0) > INT32_MAX || t->size(1) > INT32_MAX || t->size(2) > INT32_MAX) value_error(name, "is too large");
  if (t->size(1) < 1 || t->size(2) < 1) value_error(name, "must have heads and features");
  if (t->size(2) > 1 && t->stride(2) != 1) value_error(name, "must have contiguous heads");
  const int64_t rows = t->size(0), heads = t->size(1), dim = t->size(2), row = t->stride(0), head = t->stride(1);
  if ((rows > 1 && row < dim) || (heads > 1 && head < dim) ||
      (rows > 1 && heads > 1 && row < (heads - 1) * head + dim && head < (rows - 1) * row + dim))
    value_error(name, "must have rows and heads that do not overlap");
  return t;
}
void same_kind(const at::Tensor& t, const char* name, const at::Tensor& like) {
  if (t.get_device() != like.get_device()) value_error(name, "must be on the other tensors' device");
  if (t.scalar_type() != like.scalar_type()) type_error(name, "must have the other tensors' type");
}
// int64 offsets of sequences, and how many those are (null and 1 for None).
const int64_t* offsets_of(PyObject* o, const char* name, int64_t device, int64_t* batch) {
  *batch = 1;
  const at::Tensor* t = tensor(o, name, true);
  if (t == nullptr) return nullptr;
  if (t->scalar_type() != at::kLong) type_error(name, "must be int64");
  if (t->dim() != 1 || t->numel() < 2 || t->get_device() != device || !t->is_contiguous())
    value_error(name, "must be a contiguous [B+1] tensor on the other tensors' device");
  *batch = t->numel() - 1;
  if (*batch > INT32_MAX) value_error(name, "has too many sequences");
  return static_cast<const int64_t*>(t->data_ptr());
}

// The arguments that both directions of cross_attention share.
struct AttentionInputs {
  const at::Tensor *q, *k, *v;
  int64_t device, batch;
  const int64_t *q_offsets, *k_offsets;
  const uint8_t* mask = nullptr;
  int32_t q_heads, kv_heads, dim;
  mpm_dtype dtype;
  float scale;

  // q, k, v, q_offsets, k_offsets, key_mask, scale
  explicit AttentionInputs(PyObject* const* p) {
    q = heads_of(p[0], "q");
    k = heads_of(p[1], "k");
    v = heads_of(p[2], "v");
    device = q->get_device();
    dtype = dtype_of(*q, "q");
    same_kind(*k, "k", *q);
    same_kind(*v, "v", *q);
    if (k->sizes() != v->sizes()) value_error("v", "must have k's shape");
    if (k->size(2) != q->size(2)) value_error("k", "must have heads as wide as q's");
    if (q->size(1) % k->size(1) != 0) value_error("q", "must have a multiple of k's heads");
    q_heads = static_cast<int32_t>(q->size(1));
    kv_heads = static_cast<int32_t>(k->size(1));
    dim = static_cast<int32_t>(q->size(2));
    int64_t k_batch;
    q_offsets = offsets_of(p[3], "q_offsets", device, &batch);
    k_offsets = offsets_of(p[4], "k_offsets", device, &k_batch);
    if (batch != k_batch || (q_offsets == nullptr) != (k_offsets == nullptr))
      value_error("q_offsets and k_offsets", "must be of as many sequences");
    if (const at::Tensor* m = tensor(p[5], "key_mask", true)) {
      if (m->scalar_type() != at::kByte && m->scalar_type() != at::kBool) type_error("key_mask", "must be bool or uint8");
      if (m->get_device() != device || !m->is_contiguous() || m->numel() != k->size(0))
        value_error("key_mask", "must be contiguous, a value per row of k, on the other tensors' device");
      mask = static_cast<const uint8_t*>(m->data_ptr());
    }
    scale = p[6] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(dim))) : static_cast<float>(number(p[6]));
  }
};
// Scratch of `need` bytes: the caller's, or new.
struct Scratch {
  at::Tensor made;
  void* p = nullptr;
  size_t bytes = 0;
  Scratch(PyObject* given, size_t need, const at::Tensor& like) {
    if (given != Py_None) {
      p = buffer(given, "workspace", at::kByte, like.get_device(), at::IntArrayRef());
      bytes = static_cast<size_t>(THPVariable_Unpack(given).numel());
    } else if (need > 0) {
      made = new_like(like, {static_cast<int64_t>(need)}, at::kByte);
      p = made.data_ptr();
      bytes = need;
    }
  }
};

// cross_attention(<AttentionInputs>, out, with_lse, workspace, device_status)
PyObject* cross_attention(PyObject* const* p) {
  const AttentionInputs a(p);
  const OnDevice on(a.device);
  at::Tensor out, lse, rest;
  void* pout;
  if (p[7] == Py_None) {
    out = new_like(*a.q, a.q->sizes(), a.q->scalar_type());
    pout = out.data_ptr();
  } else {
    pout = buffer(p[7], "out", a.q->scalar_type(), a.device, a.q->sizes());
  }
  if (truth(p[8])) {
    lse = new_like(*a.q, {a.q->size(0), a.q->size(1)}, at::kFloat);
    if (a.dtype == MPM_BF16) rest = new_like(*a.q, a.q->sizes(), at::kBFloat16);
  }
  const Scratch scratch(p[9],
                        entry.cross_attention_workspace_size(static_cast<int32_t>(a.batch), a.q->size(0), a.k->size(0),
                                                             a.q_heads, a.kv_heads, a.dim, a.dtype),
                        *a.q);
  check("mpm_cross_attention",
        entry.cross_attention(a.q->data_ptr(), a.q->stride(0), a.q->stride(1), a.k->data_ptr(), a.k->stride(0),
                              a.k->stride(1), a.v->data_ptr(), a.v->stride(0), a.v->stride(1), a.q_offsets, a.k_offsets,
                              static_cast<int32_t>(a.batch), a.q->size(0), a.k->size(0), a.q_heads, a.kv_heads, a.dim,
                              a.dtype, a.scale, a.mask, pout, rest.defined() ? rest.data_ptr() : nullptr,
                              lse.defined() ? static_cast<float*>(lse.data_ptr()) : nullptr,
                              scratch.p, scratch.bytes, status_word(p[10], a.device), on.stream));
  written(p[7]);
  return tuple_of({out.defined() ? wrapped(out) : again(p[7]), wrapped(lse), wrapped(rest)});
}

// cross_attention_backward(<AttentionInputs>, d_out, out, lse, rest, workspace, device_status)
PyObject* cross_attention_backward(PyObject* const* p) {
  const AttentionInputs a(p);
  const OnDevice on(a.device);
  const at::Tensor* g = heads_of(p[7], "d_out");
  same_kind(*g, "d_out", *a.q);
  if (g->sizes() != a.q->sizes()) value_error("d_out", "must have q's shape");
  const void* out = buffer(p[8], "out", a.q->scalar_type(), a.device, a.q->sizes(), false);
  const void* rest = buffer(p[10], "stats.rest", at::kBFloat16, a.device, a.q->sizes());
  const int64_t rows_heads[2] = {a.q->size(0), a.q->size(1)};
  const float* lse = static_cast<float*>(buffer(p[9], "stats.lse", at::kFloat, a.device, rows_heads, false));
  at::Tensor d_q = new_like(*a.q, a.q->sizes(), a.q->scalar_type());
  at::Tensor d_k = new_like(*a.k, a.k->sizes(), a.k->scalar_type()), d_v = new_like(*a.k, a.k->sizes(), a.k->scalar_type());
  const Scratch scratch(p[11],
                        entry.cross_attention_backward_workspace_size(static_cast<int32_t>(a.batch), a.q->size(0),
                                                                      a.k->size(0), a.q_heads, a.kv_heads, a.dim, a.dtype),
                        *a.q);
  check("mpm_cross_attention_backward",
        entry.cross_attention_backward(
            g->data_ptr(), g->stride(0), g->stride(1), a.q->data_ptr(), a.q->stride(0), a.q->stride(1), a.k->data_ptr(),
            a.k->stride(0), a.k->stride(1), a.v->data_ptr(), a.v->stride(0), a.v->stride(1), out, rest, lse, a.q_offsets,
            a.k_offsets, static_cast<int32_t>(a.batch), a.q->size(0), a.k->size(0), a.q_heads, a.kv_heads, a.dim, a.dtype,
            a.scale, a.mask, d_q.data_ptr(), d_k.data_ptr(), d_v.data_ptr(), scratch.p, scratch.bytes,
            status_word(p[12], a.device), on.stream));
  return tuple_of({wrapped(d_q), wrapped(d_k), wrapped(d_v)});
}

// rotary(x, positions, frequencies, sections, layout, inverse, offsets, out, device_status)
PyObject* rotary(PyObject* const* p) {
  const at::Tensor* x = heads_of(p[0], "x");
  const int64_t device = x->get_device(), rows = x->size(0);
  if (!PyTuple_Check(p[3]) && !PyList_Check(p[3])) type_error("sections", "must be a tuple or a list");
  int32_t sections[MPM_ROTARY_MAX_AXES];
  const Py_ssize_t axes = PySequence_Size(p[3]);
  if (axes < 1 || axes > MPM_ROTARY_MAX_AXES) value_error("sections", "must be of 1 to 8 axes");
  int64_t pairs = 0;
  for (Py_ssize_t i = 0; i < axes; ++i) {
    PyObject* item = PySequence_GetItem(p[3], i);
    const long long n = item == nullptr ? -1 : PyLong_AsLongLong(item);
    Py_XDECREF(item);
    if (n == -1 && PyErr_Occurred()) throw Raised{};
    if (n < 1 || n > x->size(2)) value_error("sections", "must be positive, and no more than a head's pairs in all");
    sections[i] = static_cast<int32_t>(n);
    pairs += n;
  }
  if (2 * pairs > x->size(2)) value_error("sections", "must be positive, and no more than a head's pairs in all");
  const at::Tensor* at = tensor(p[1], "positions");
  if (at->scalar_type() != at::kFloat) type_error("positions", "must be float32");
  if (at->get_device() != device || !at->is_contiguous() || at->numel() != rows * axes || at->dim() < 1 || at->size(0) != rows)
    value_error("positions", "must be a contiguous [rows, axes] tensor on x's device");
  const int64_t vector[1] = {pairs};
  const double* frequencies = static_cast<double*>(buffer(p[2], "frequencies", at::kDouble, device, vector, false));
  if (!PyUnicode_Check(p[4])) type_error("layout", "must be a string");
  mpm_rotary_layout layout;
  if (PyUnicode_CompareWithASCIIString(p[4], "halves") == 0) layout = MPM_ROTARY_HALVES;
  else if (PyUnicode_CompareWithASCIIString(p[4], "interleaved") == 0) layout = MPM_ROTARY_INTERLEAVED;
  else value_error("layout", "must be 'halves' or 'interleaved'");
  int64_t batch;
  const int64_t* offsets = offsets_of(p[6], "offsets", device, &batch);
  const OnDevice on(device);
  at::Tensor out;
  if (p[7] == Py_None) {
    out = new_like(*x, x->sizes(), x->scalar_type());
  } else {
    const at::Tensor* t = heads_of(p[7], "out");
    same_kind(*t, "out", *x);
    if (t->sizes() != x->sizes()) value_error("out", "must have x's shape");
    out = *t;
  }
  check("mpm_rotary",
        entry.rotary(x->data_ptr(), x->stride(0), x->stride(1), static_cast<const float*>(at->data_ptr()), frequencies,
                     sections, static_cast<int32_t>(axes), layout, truth(p[5]), offsets, static_cast<int32_t>(batch), rows,
                     static_cast<int32_t>(x->size(1)), static_cast<int32_t>(x->size(2)), dtype_of(*x, "x"), out.data_ptr(),
                     out.stride(0), out.stride(1), status_word(p[8], device), on.stream));
  written(p[7]);
  return p[7] == Py_None ? THPVariable_Wrap(out) : again(p[7]);
}

// Calls F with its arguments, of which there are N; no C++ exception leaves.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N || entry.block_norm == nullptr) {
    PyErr_SetString(PyExc_TypeError, n != N ? "wrong number of arguments" : "the library's entry points are not set");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  try {
    return F(args);
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// bind(addresses of the entry points in EntryPoints' order, callable that raises a status)
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *addresses, *raise;
  if (!PyArg_ParseTuple(args, "O!O", &PyTuple_Type, &addresses, &raise)) return nullptr;
  constexpr Py_ssize_t kEntries = sizeof(EntryPoints) / sizeof(void*);
  if (PyTuple_GET_SIZE(addresses) != kEntries) {
    PyErr_SetString(PyExc_TypeError, "wrong number of entry points");
    return nullptr;
  }
  void* found[kEntries];
  for (Py_ssize_t i = 0; i < kEntries; ++i) {
    found[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (found[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an entry point has no address");
      return nullptr;
    }
  }
  memcpy(&entry, found, sizeof(entry));
  Py_INCREF(raise);
  Py_XDECREF(std::exchange(raise_status, raise));
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F, N>));
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"block_norm", fast<block_norm, 15>(), METH_FASTCALL, nullptr},
                         {"block_norm_backward", fast<block_norm_backward, 16>(), METH_FASTCALL, nullptr},
                         {"quantize", fast<quantize, 3>(), METH_FASTCALL, nullptr},
                         {"dequantize", fast<dequantize, 5>(), METH_FASTCALL, nullptr},
                         {"matmul", fast<matmul, 10>(), METH_FASTCALL, nullptr},
                         {"cross_attention", fast<cross_attention, 11>(), METH_FASTCALL, nullptr},
                         {"cross_attention_backward", fast<cross_attention_backward, 13>(), METH_FASTCALL, nullptr},
                         {"rotary", fast<rotary, 9>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_blocks", "Binding of the encoder-block, attention and rotary entry points of libmpm.so.", -1,
                      methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__blocks() { return PyModule_Create(&module); }
