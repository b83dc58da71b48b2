// Python helper: the per-token outputs of a call as views of one allocation, and the marshalling of dvp_forward and of the
// rollout's calls.
//
// A call has up to twenty output vectors.  Sliced from three allocations through Python they took more than half of
// the 33 us that a call of dvp_forward on a few tokens spends on the host; as tensors laid directly over one
// storage they cost 5 us (16 tokens x 151 936 bf16 logits: 32.6 -> 18.3 us a call).

#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include "dvp.h"

namespace {

// T elements of `type` over `storage`, starting at byte row * stride.
at::Tensor row_view(const c10::Storage &storage, c10::DispatchKeySet keys, at::ScalarType type, int64_t row,
                    int64_t stride, int64_t T) {
  auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(storage), keys, c10::scalarTypeToTypeMeta(type));
  impl->set_sizes_contiguous({T});
  impl->set_storage_offset(row * stride / static_cast<int64_t>(c10::elementSize(type)));
  return at::Tensor(std::move(impl));
}

// outputs(like, T, floats, counts) -> (tensors, address, stride): `floats` float32 vectors, `counts` int32 vectors
// and one uint8 vector of T elements on the device of `like`, in this order; vector i starts at address + i * stride.
PyObject *outputs(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  if (n_args != 4 || !THPVariable_Check(args[0])) {
    PyErr_SetString(PyExc_TypeError, "outputs(like, T, floats, counts)");
    return nullptr;
  }
  const int64_t T = PyLong_AsLongLong(args[1]), floats = PyLong_AsLongLong(args[2]), counts = PyLong_AsLongLong(args[3]);
  if (PyErr_Occurred()) return nullptr;
  if (T < 0 || T >= (int64_t(1) << 56)) {
    PyErr_Format(PyExc_RuntimeError, "outputs: there are no vectors of %lld elements", static_cast<long long>(T));
    return nullptr;
  }
  // torch's own exception types reach Python, out-of-memory errors among them
  HANDLE_TH_ERRORS
  const int64_t rows = floats + counts + 1, stride = (T + 3) / 4 * 16;
  const at::Tensor buf =
      at::empty({rows * stride}, THPVariable_Unpack(args[0]).options().dtype(at::kByte).requires_grad(false));
  const c10::Storage &storage = buf.storage();
  const c10::DispatchKeySet keys = buf.key_set();
  THPObjectPtr tensors(PyTuple_New(rows));
  if (!tensors) return nullptr;
  for (int64_t i = 0; i < rows; ++i) {
    const at::ScalarType type = i < floats ? at::kFloat : i < floats + counts ? at::kInt : at::kByte;
    PyObject *t = THPVariable_Wrap(row_view(storage, keys, type, i, stride, T));
    if (!t) return nullptr;
    PyTuple_SET_ITEM(tensors.get(), i, t);
  }
  return Py_BuildValue("(NLL)", tensors.release(), static_cast<long long>(reinterpret_cast<uintptr_t>(buf.data_ptr())),
                       static_cast<long long>(stride));
  END_HANDLE_TH_ERRORS
}

// ---- dvp_forward ------------------------------------------------------------------------------------------------------
// What binding.dvp_forward does beside the library's call, for results that it makes itself.  In Python its checks, packing
// and namespaces took half of a small call: 64 x 4,096 float32 with the gradient 20.7 -> 12.3 us, 16 x 151,936 bfloat16
// forward 17.3 -> 14.3 (then the device's).

// The error that Python code gets for what it passes; thrown inside HANDLE_TH_ERRORS blocks.
[[noreturn]] void refuse(PyObject *type, const char *format, const char *name = "") {
  PyErr_Format(type, format, name);
  throw python_error();
}

const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor", name);
  return THPVariable_Unpack(o);
}

const at::Tensor &matrix(PyObject *o, const char *name) {
  const at::Tensor &x = tensor(o, name);
  if (x.dim() != 2 || x.stride(1) != 1) refuse(PyExc_ValueError, "%s must be 2-D with unit inner stride", name);
  if (!x.is_cuda()) refuse(PyExc_ValueError, "%s must live on a CUDA device", name);
  return x;
}

int32_t dtype_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return DVP_F32;
    case at::kBFloat16: return DVP_BF16;
    case at::kHalf: return DVP_F16;
    default: break;
  }
  PyErr_SetObject(PyExc_KeyError, reinterpret_cast<PyObject *>(torch::getTHPDtype(t)));
  throw python_error();
}

// Names that results have, and the type of results; made once.
struct Names {
  PyObject *max, *lse, *lse_safe, *logp, *logp_mp, *comp_mp, *log_cov, *count, *mask, *train, *infer, *log_ratio, *flags,
      *grad_train, *weight, *ns;
} g_names;

struct MoreNames {
  PyObject *y, *scale, *rstd, *residual, *d_x, *d_weight, *ids;
} g_more;

bool make_names() {
  const char *more[] = {"y", "scale", "rstd", "residual", "d_x", "d_weight", "ids"};
  PyObject **to = &g_more.y;
  for (const char *t : more)
    if (!(*to++ = PyUnicode_InternFromString(t))) return false;
  const char *text[] = {"max", "lse", "lse_safe", "logp", "logp_mp", "comp_mp", "log_cov", "count", "mask", "train",
                        "infer", "log_ratio", "flags", "grad_train", "weight"};
  PyObject **at = &g_names.max;
  for (const char *t : text)
    if (!(*at++ = PyUnicode_InternFromString(t))) return false;
  PyObject *types = PyImport_ImportModule("types");
  g_names.ns = types ? PyObject_GetAttrString(types, "SimpleNamespace") : nullptr;
  Py_XDECREF(types);
  return g_names.ns != nullptr;
}

void put(PyObject *dict, PyObject *name, PyObject *value) {  // takes `value`
  THPObjectPtr v(value);
  if (!v || PyDict_SetItem(dict, name, v.get()) != 0) throw python_error();
}
PyObject *none() {
  Py_INCREF(Py_None);
  return Py_None;
}
PyObject *namespace_of(PyObject *dict) {
  static PyObject *empty = PyTuple_New(0);
  PyObject *r = PyObject_Call(g_names.ns, empty, dict);
  if (!r) throw python_error();
  return r;
}

// Vectors over one storage, vector i at `base` + i * `stride`.
struct Vectors {
  at::Tensor buf;
  c10::DispatchKeySet keys;
  int64_t T, stride;
  char *base;

  Vectors(const at::Tensor &like, int64_t T_, int64_t rows) : T(T_), stride((T_ + 3) / 4 * 16) {
    buf = at::empty({rows * stride}, like.options().dtype(at::kByte).requires_grad(false));
    keys = buf.key_set();
    base = static_cast<char *>(buf.data_ptr());
  }
  template <typename P>
  PyObject *make(int64_t i, at::ScalarType type, P **address) {
    *address = reinterpret_cast<P *>(base + i * stride);
    return THPVariable_Wrap(row_view(buf.storage(), keys, type, i, stride, T));
  }
};

PyObject *side(Vectors &v, int64_t first, int64_t count_row, dvp_side_out &o) {
  THPObjectPtr d(PyDict_New());
  if (!d) throw python_error();
  const Names &n = g_names;
  put(d.get(), n.max, v.make(first, at::kFloat, &o.max));
  put(d.get(), n.lse, v.make(first + 1, at::kFloat, &o.lse));
  put(d.get(), n.lse_safe, v.make(first + 2, at::kFloat, &o.lse_safe));
  put(d.get(), n.logp, v.make(first + 3, at::kFloat, &o.logp));
  put(d.get(), n.logp_mp, v.make(first + 4, at::kFloat, &o.logp_mp));
  put(d.get(), n.comp_mp, v.make(first + 5, at::kFloat, &o.comp_mp));
  put(d.get(), n.log_cov, v.make(first + 6, at::kFloat, &o.log_cov));
  put(d.get(), n.count, v.make(count_row, at::kInt, &o.count));
  put(d.get(), n.mask, none());
  return namespace_of(d.get());
}

// forward(entry, train, ids, rho, infer, upstream, grad, grad_dtype, stream, hint, mode, mask_value, weight_kind,
// weight_lo, weight_hi) -> the result, or the library's status where that is not DVP_OK.  `entry`: the address of the
// library's dvp_forward; None for tensors and the gradient's type that are not given, and for the current stream.
PyObject *forward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  if (n_args != 15) {
    PyErr_SetString(PyExc_TypeError, "forward takes 15 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  const Names &n = g_names;
  const auto entry = reinterpret_cast<int (*)(const dvp_forward_args *)>(PyLong_AsVoidPtr(args[0]));
  const at::Tensor &train = matrix(args[1], "train_logits");
  const bool has_infer = args[4] != Py_None, has_grad = args[5] != Py_None;
  dvp_forward_args a = {};
  a.struct_size = sizeof(a);
  a.rho = PyFloat_AsDouble(args[3]);
  a.stream = args[8] == Py_None ? c10::cuda::getCurrentCUDAStream().stream() : PyLong_AsVoidPtr(args[8]);
  a.launch_hint = static_cast<uint32_t>(PyLong_AsUnsignedLong(args[9]));
  a.mode = static_cast<uint32_t>(PyLong_AsUnsignedLong(args[10]));
  a.mask_value = static_cast<float>(PyFloat_AsDouble(args[11]));
  a.weight_kind = static_cast<uint32_t>(PyLong_AsUnsignedLong(args[12]));
  a.weight_lo = static_cast<float>(PyFloat_AsDouble(args[13]));
  a.weight_hi = static_cast<float>(PyFloat_AsDouble(args[14]));
  if (PyErr_Occurred()) throw python_error();
  const bool weighted = a.weight_kind != DVP_WEIGHT_NONE;
  const int64_t T = a.T = train.size(0), V = a.V = train.size(1);
  a.ld_train = train.stride(0);
  a.train_logits = train.data_ptr();
  if (has_infer) {
    const at::Tensor &infer = matrix(args[4], "infer_logits");
    if (infer.scalar_type() != train.scalar_type() || infer.size(0) != T || infer.size(1) != V)
      refuse(PyExc_ValueError, "infer_logits must match train_logits in dtype and shape");
    a.ld_infer = infer.stride(0);
    a.infer_logits = infer.data_ptr();
  }
  const int sides = has_infer ? 2 : 1, floats = 7 * sides + has_infer + weighted;
  Vectors v(train, T, floats + sides + 1);
  THPObjectPtr d(PyDict_New());
  if (!d) throw python_error();
  put(d.get(), n.train, side(v, 0, floats, a.train));
  put(d.get(), n.infer, has_infer ? side(v, 7, floats + 1, a.infer) : none());
  put(d.get(), n.log_ratio, has_infer ? v.make(14, at::kFloat, &a.log_ratio) : none());
  put(d.get(), n.flags, v.make(floats + sides, at::kByte, &a.flags));
  at::Tensor made;
  if (has_grad) {
    const at::Tensor &upstream = tensor(args[5], "upstream");
    if (upstream.scalar_type() != at::kFloat) refuse(PyExc_TypeError, "upstream must be float32");
    a.upstream = static_cast<const float *>(upstream.data_ptr());
    PyObject *grad = args[6];
    if (grad == Py_None) {
      at::ScalarType type = train.scalar_type();
      if (args[7] != Py_None) {
        if (!THPDtype_Check(args[7])) refuse(PyExc_TypeError, "grad_dtype must be a torch.dtype");
        type = reinterpret_cast<THPDtype *>(args[7])->scalar_type;
      }
      made = at::empty({T, V}, train.options().dtype(type).requires_grad(false));
      put(d.get(), n.grad_train, THPVariable_Wrap(made));
    } else {
      made = matrix(grad, "grad_train");
      Py_INCREF(grad);
      put(d.get(), n.grad_train, grad);
    }
    a.grad_dtype = dtype_code(made.scalar_type());
    a.ld_grad = made.stride(0);
    a.grad_train = made.data_ptr();
  } else {
    put(d.get(), n.grad_train, none());
  }
  if (weighted) put(d.get(), n.weight, v.make(floats - 1, at::kFloat, &a.weight_out));
  a.logits_dtype = dtype_code(train.scalar_type());
  const at::Tensor &ids = tensor(args[2], "ids");
  if (ids.scalar_type() == at::kLong)
    a.id_dtype = DVP_ID_I64;
  else if (ids.scalar_type() == at::kInt)
    a.id_dtype = DVP_ID_I32;
  else
    refuse(PyExc_TypeError, "ids must be int64 or int32");
  a.ids = ids.data_ptr();
  THPObjectPtr result(namespace_of(d.get()));
  int status;
  Py_BEGIN_ALLOW_THREADS status = entry(&a);
  Py_END_ALLOW_THREADS if (status != DVP_OK) return PyLong_FromLong(status);
  return result.release();
  END_HANDLE_TH_ERRORS
}

// ---- the rollout's last stage -------------------------------------------------------------------------------------------
// What binding's functions of these names do beside the library's call.  A decoding step's calls are a few microseconds of
// the device's each.

bool given(PyObject *o) { return o != Py_None; }
void *stream_of(PyObject *o, int device) {
  return given(o) ? PyLong_AsVoidPtr(o) : static_cast<void *>(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream());
}
// What the call makes for itself stays put until the stream that the caller has named is through with it, whoever lets go of it before.
void keep_for(const at::Tensor &t, PyObject *stream) {
  if (given(stream) && t.numel() > 0)
    c10::cuda::CUDACachingAllocator::recordStream(
        t.storage().data_ptr(), c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(PyLong_AsVoidPtr(stream)),
                                                                 static_cast<c10::DeviceIndex>(t.get_device())));
}
void same_device(const at::Tensor &like, const at::Tensor &x, const char *name) {
  if (x.device() != like.device()) refuse(PyExc_ValueError, "%s must live on the device of the others", name);
}
// A vector of n elements side by side, of one of two types.
const at::Tensor &vector(PyObject *o, const char *name, int64_t n, at::ScalarType a, at::ScalarType b, const at::Tensor &like) {
  const at::Tensor &x = tensor(o, name);
  if (x.dim() != 1 || x.size(0) != n || (n > 1 && x.stride(0) != 1)) refuse(PyExc_ValueError, "%s must be a contiguous vector of the right length", name);
  if (x.scalar_type() != a && x.scalar_type() != b) refuse(PyExc_TypeError, "%s has a type that is not taken here", name);
  same_device(like, x, name);
  return x;
}
const at::Tensor &like_matrix(PyObject *o, const char *name, const at::Tensor &like) {
  const at::Tensor &x = matrix(o, name);
  if (x.sizes() != like.sizes() || x.scalar_type() != like.scalar_type()) refuse(PyExc_ValueError, "%s must match in shape and type", name);
  same_device(like, x, name);
  return x;
}
// The code of one of the three types that matrices have here.
int32_t code_of(at::ScalarType t, const char *name) {
  if (t != at::kFloat && t != at::kBFloat16 && t != at::kHalf) refuse(PyExc_TypeError, "%s must be float32, bfloat16 or float16", name);
  return dtype_code(t);
}
int32_t out_code(at::ScalarType t) { return t == at::kFloat8_e4m3fn ? DVP_E4M3 : code_of(t, "out_dtype"); }
at::ScalarType type_of(PyObject *o) {
  if (!THPDtype_Check(o)) refuse(PyExc_TypeError, "%s must be a torch.dtype", "out_dtype");
  return reinterpret_cast<THPDtype *>(o)->scalar_type;
}
at::Tensor make(const at::Tensor &like, at::IntArrayRef sizes, at::ScalarType type) {
  return at::empty(sizes, like.options().dtype(type).requires_grad(false));
}
// Tensors that a call makes: of a small call all over one storage, since an allocation takes longer than its part of the kernel; of
// larger ones each by itself, so that keeping one keeps nothing else.
struct Outputs {
  static constexpr int64_t kSmall = 1 << 20;
  const at::Tensor &like;
  at::Tensor buf;
  int64_t at = 0;
  Outputs(const at::Tensor &like_, int64_t bytes) : like(like_) {
    if (bytes <= kSmall) buf = ::make(like, {bytes}, at::kByte);
  }
  static int64_t room(int64_t rows, int64_t cols, at::ScalarType type) {
    return (rows * cols * static_cast<int64_t>(c10::elementSize(type)) + 255) / 256 * 256;
  }
  // [rows, cols] of rows of `ld` elements; cols < 0: a vector
  at::Tensor take(int64_t rows, int64_t cols, int64_t ld, at::ScalarType type) {
    if (!buf.defined()) {
      at::Tensor t = cols < 0 ? ::make(like, {rows}, type) : ::make(like, {rows, ld}, type);
      return cols >= 0 && cols != ld ? t.narrow(1, 0, cols) : t;
    }
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(buf.storage()), buf.key_set(), c10::scalarTypeToTypeMeta(type));
    impl->set_storage_offset(at / static_cast<int64_t>(c10::elementSize(type)));
    if (cols < 0)
      impl->set_sizes_contiguous({rows});
    else
      impl->set_sizes_and_strides(at::IntArrayRef({rows, cols}), at::IntArrayRef({ld, int64_t(1)}));
    at += room(rows, cols < 0 ? 1 : ld, type);
    return at::Tensor(std::move(impl));
  }
};
PyObject *finish(int status, THPObjectPtr &result) { return status == DVP_OK ? result.release() : PyLong_FromLong(status); }

// rms_norm(entry, x, weight, residual, eps, out_dtype, residual_out, stream)
PyObject *rms_norm(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  if (n_args != 8) {
    PyErr_SetString(PyExc_TypeError, "rms_norm takes 8 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  const auto entry = reinterpret_cast<int (*)(const dvp_rms_norm_args *)>(PyLong_AsVoidPtr(args[0]));
  const at::Tensor &x = matrix(args[1], "x");
  const c10::cuda::CUDAGuard guard(x.device());
  const int64_t T = x.size(0), H = x.size(1);
  dvp_rms_norm_args a = {};
  a.struct_size = sizeof(a);
  a.x_dtype = code_of(x.scalar_type(), "x");
  a.T = T, a.H = H;
  a.ld_x = x.stride(0), a.x = x.data_ptr();
  const at::Tensor &w = vector(args[2], "weight", H, x.scalar_type(), at::kFloat, x);
  a.weight_dtype = dtype_code(w.scalar_type()), a.weight = w.data_ptr();
  a.eps = PyFloat_AsDouble(args[4]);
  if (PyErr_Occurred()) throw python_error();
  const at::ScalarType out = given(args[5]) ? type_of(args[5]) : x.scalar_type();
  a.out_dtype = out_code(out);
  a.stream = stream_of(args[7], x.get_device());
  THPObjectPtr d(PyDict_New());
  if (!d) throw python_error();
  at::Tensor h;
  if (given(args[3])) {
    const at::Tensor &r = like_matrix(args[3], "residual", x);
    a.residual = r.data_ptr(), a.ld_residual = r.stride(0);
  }
  if (given(args[6])) h = like_matrix(args[6], "residual_out", x);
  const bool fp8 = a.out_dtype == DVP_E4M3;
  // 8-bit rows start on 16-byte boundaries, where the tensor cores' loads want them
  const int64_t ld = fp8 ? (H + 15) / 16 * 16 : H, blocks = (H + 127) / 128;
  const bool make_h = !h.defined() && given(args[3]);
  Outputs made(x, Outputs::room(T, ld, out) + Outputs::room(T, 1, at::kFloat) + (fp8 ? Outputs::room(T, blocks, at::kFloat) : 0) +
                      (make_h ? Outputs::room(T, H, x.scalar_type()) : 0));
  if (make_h) {
    h = made.take(T, H, H, x.scalar_type());
    keep_for(h, args[7]);
  }
  if (h.defined()) a.residual_out = h.data_ptr(), a.ld_residual_out = h.stride(0);
  const at::Tensor y = made.take(T, H, ld, out), rstd = made.take(T, -1, 0, at::kFloat);
  a.out = y.data_ptr(), a.ld_out = ld;
  a.rstd = static_cast<float *>(rstd.data_ptr());
  if (fp8) {
    const at::Tensor scale = made.take(T, blocks, blocks, at::kFloat);
    a.scale = static_cast<float *>(scale.data_ptr()), a.ld_scale = blocks;
    keep_for(scale, args[7]);
    put(d.get(), g_more.scale, THPVariable_Wrap(scale));
  } else {
    put(d.get(), g_more.scale, none());
  }
  keep_for(y, args[7]);
  keep_for(rstd, args[7]);
  put(d.get(), g_more.y, THPVariable_Wrap(y));
  put(d.get(), g_more.rstd, THPVariable_Wrap(rstd));
  put(d.get(), g_more.residual, h.defined() ? THPVariable_Wrap(h) : none());
  THPObjectPtr result(namespace_of(d.get()));
  int status;
  Py_BEGIN_ALLOW_THREADS status = entry(&a);
  Py_END_ALLOW_THREADS return finish(status, result);
  END_HANDLE_TH_ERRORS
}

// rms_norm_backward(entry, workspace_bytes, dy, h, weight, rstd, d_residual, d_weight, accumulate, workspace, stream)
PyObject *rms_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  if (n_args != 11) {
    PyErr_SetString(PyExc_TypeError, "rms_norm_backward takes 11 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  const auto entry = reinterpret_cast<int (*)(const dvp_rms_norm_backward_args *)>(PyLong_AsVoidPtr(args[0]));
  const auto bytes = reinterpret_cast<size_t (*)(int, const void *)>(PyLong_AsVoidPtr(args[1]));
  const at::Tensor &dy = matrix(args[2], "dy"), &h = matrix(args[3], "h");
  if (dy.sizes() != h.sizes()) refuse(PyExc_ValueError, "%s must match h in shape", "dy");
  same_device(h, dy, "dy");
  const c10::cuda::CUDAGuard guard(h.device());
  const int64_t T = h.size(0), H = h.size(1);
  dvp_rms_norm_backward_args a = {};
  a.struct_size = sizeof(a);
  a.h_dtype = code_of(h.scalar_type(), "h"), a.dy_dtype = code_of(dy.scalar_type(), "dy");
  a.T = T, a.H = H;
  a.dy = dy.data_ptr(), a.ld_dy = dy.stride(0);
  a.h = h.data_ptr(), a.ld_h = h.stride(0);
  const at::Tensor &w = vector(args[4], "weight", H, h.scalar_type(), at::kFloat, h);
  a.weight_dtype = dtype_code(w.scalar_type()), a.weight = w.data_ptr();
  a.rstd = static_cast<const float *>(vector(args[5], "rstd", T, at::kFloat, at::kFloat, h).data_ptr());
  if (given(args[6])) {
    const at::Tensor &r = like_matrix(args[6], "d_residual", h);
    a.d_residual = r.data_ptr(), a.ld_d_residual = r.stride(0);
  }
  a.accumulate_dw = PyObject_IsTrue(args[8]);
  if (a.accumulate_dw && !given(args[7])) refuse(PyExc_ValueError, "%s needs d_weight", "accumulate_dw");
  Outputs made(h, Outputs::room(T, H, h.scalar_type()) + Outputs::room(H, 1, at::kFloat));
  const at::Tensor d_x = made.take(T, H, H, h.scalar_type());
  a.d_x = d_x.data_ptr(), a.ld_d_x = H;
  const at::Tensor d_weight = given(args[7]) ? vector(args[7], "d_weight", H, at::kFloat, at::kFloat, h) : made.take(H, -1, 0, at::kFloat);
  a.d_weight = static_cast<float *>(d_weight.data_ptr());
  keep_for(d_x, args[10]);
  if (!given(args[7])) keep_for(d_weight, args[10]);
  at::Tensor workspace;
  if (given(args[9])) {
    workspace = tensor(args[9], "workspace");
    same_device(h, workspace, "workspace");
  } else {
    workspace = make(h, {static_cast<int64_t>(std::max<size_t>(bytes(DVP_ENTRY_RMS_NORM_BACKWARD, &a), 256))}, at::kByte);
  }
  a.workspace = workspace.data_ptr();
  if (!given(args[9])) keep_for(workspace, args[10]);
  a.workspace_bytes = static_cast<size_t>(workspace.numel() * workspace.element_size());
  a.stream = stream_of(args[10], h.get_device());
  THPObjectPtr d(PyDict_New());
  if (!d) throw python_error();
  put(d.get(), g_more.d_x, THPVariable_Wrap(d_x));
  put(d.get(), g_more.d_weight, THPVariable_Wrap(d_weight));
  THPObjectPtr result(namespace_of(d.get()));
  int status;
  Py_BEGIN_ALLOW_THREADS status = entry(&a);
  Py_END_ALLOW_THREADS return finish(status, result);
  END_HANDLE_TH_ERRORS
}

// gemm_fp8(entry, a, a_scale, b, b_scale, out_dtype, out, stream, hint) -> (out, status tensor)
PyObject *gemm_fp8(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  if (n_args != 9) {
    PyErr_SetString(PyExc_TypeError, "gemm_fp8 takes 9 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  const auto entry = reinterpret_cast<int (*)(const dvp_gemm_fp8_args *)>(PyLong_AsVoidPtr(args[0]));
  const char *names[] = {"a", "a_scale", "b", "b_scale"};
  const at::Tensor *in[4];
  for (int i = 0; i < 4; ++i) {
    in[i] = &matrix(args[1 + i], names[i]);
    if (in[i]->scalar_type() != (i % 2 ? at::kFloat : at::kFloat8_e4m3fn))
      refuse(PyExc_TypeError, i % 2 ? "%s must be float32" : "%s must be float8_e4m3fn", names[i]);
    same_device(*in[0], *in[i], names[i]);
  }
  const at::Tensor &x = *in[0], &b = *in[2];
  const c10::cuda::CUDAGuard guard(x.device());
  const int64_t M = x.size(0), K = x.size(1), N = b.size(0), blocks = (K + 127) / 128;
  if (b.size(1) != K) refuse(PyExc_ValueError, "%s and b must have the same number of columns", "a");
  if (in[1]->size(0) != M || in[1]->size(1) != blocks || in[3]->size(0) != (N + 127) / 128 || in[3]->size(1) != blocks)
    refuse(PyExc_ValueError, "%s must be [M, ceil(K / 128)] and b_scale [ceil(N / 128), ceil(K / 128)]", "a_scale");
  at::Tensor out;
  if (given(args[6])) {
    out = matrix(args[6], "out");
    if (out.size(0) != M || out.size(1) != N) refuse(PyExc_ValueError, "%s must be [M, N]", "out");
    same_device(x, out, "out");
  }
  const at::ScalarType type = given(args[6]) ? out.scalar_type() : type_of(args[5]);
  const int32_t code = code_of(type, "out");
  if (!out.defined()) {
    out = make(x, {M, N}, type);
    keep_for(out, args[7]);
  }
  const at::Tensor status = make(x, {1}, at::kInt);
  keep_for(status, args[7]);  // callers let go of it at once
  if (M == 0 || N == 0) {  // no kernel runs that would say that none has given up
    c10::cuda::OptionalCUDAStreamGuard on;
    if (given(args[7]))
      on.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(PyLong_AsVoidPtr(args[7])),
                                                       static_cast<c10::DeviceIndex>(x.get_device())));
    status.zero_();
  }
  dvp_gemm_fp8_args a = {};
  a.struct_size = sizeof(a);
  a.c_dtype = code;
  a.M = M, a.N = N, a.K = K;
  a.lda = x.stride(0), a.ldb = b.stride(0), a.ldc = out.stride(0);
  a.ld_a_scale = in[1]->stride(0), a.ld_b_scale = in[3]->stride(0);
  a.a = x.data_ptr(), a.b = b.data_ptr();
  a.a_scale = static_cast<const float *>(in[1]->data_ptr()), a.b_scale = static_cast<const float *>(in[3]->data_ptr());
  a.c = out.data_ptr();
  a.status = static_cast<int32_t *>(status.data_ptr());
  a.stream = stream_of(args[7], x.get_device());
  a.launch_hint = static_cast<uint32_t>(PyLong_AsUnsignedLong(args[8]));
  if (PyErr_Occurred()) throw python_error();
  THPObjectPtr result(PyTuple_New(2));
  if (!result) throw python_error();
  PyTuple_SET_ITEM(result.get(), 0, THPVariable_Wrap(out));
  PyTuple_SET_ITEM(result.get(), 1, THPVariable_Wrap(status));
  int st;
  Py_BEGIN_ALLOW_THREADS st = entry(&a);
  Py_END_ALLOW_THREADS return finish(st, result);
  END_HANDLE_TH_ERRORS
}

// sample(entry, logits, uniform, temperature, top_k, top_p, rho, id32, stream, hint)
PyObject *sample(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
  if (n_args != 10) {
    PyErr_SetString(PyExc_TypeError, "sample takes 10 arguments");
    return nullptr;
  }
  HANDLE_TH_ERRORS
  const auto entry = reinterpret_cast<int (*)(const dvp_sample_args *)>(PyLong_AsVoidPtr(args[0]));
  const at::Tensor &z = matrix(args[1], "logits");
  const c10::cuda::CUDAGuard guard(z.device());
  const int64_t T = z.size(0);
  dvp_sample_args a = {};
  a.struct_size = sizeof(a);
  a.logits_dtype = code_of(z.scalar_type(), "logits");
  a.T = T, a.V = z.size(1), a.ld = z.stride(0);
  a.logits = z.data_ptr();
  a.uniform = static_cast<const float *>(vector(args[2], "uniform", T, at::kFloat, at::kFloat, z).data_ptr());
  // a number for all rows, or one a row; of no rows, no address is looked at, but whose it is
  const auto setting = [&](PyObject *o, const char *name, at::ScalarType type, const void **rows) {
    if (!THPVariable_Check(o)) return false;
    *rows = vector(o, name, T, type, type, z).data_ptr();
    if (!*rows) *rows = a.logits ? a.logits : &a;
    return true;
  };
  const void *rows = nullptr;
  a.temperature = a.top_p = 1.0;
  if (setting(args[3], "temperature", at::kFloat, &rows)) a.temperature_rows = static_cast<const float *>(rows);
  else a.temperature = PyFloat_AsDouble(args[3]);
  if (setting(args[4], "top_k", at::kInt, &rows)) a.top_k_rows = static_cast<const int32_t *>(rows);
  else a.top_k = PyLong_AsLongLong(args[4]);
  if (setting(args[5], "top_p", at::kFloat, &rows)) a.top_p_rows = static_cast<const float *>(rows);
  else a.top_p = PyFloat_AsDouble(args[5]);
  if (setting(args[6], "rho", at::kFloat, &rows)) a.rho_rows = static_cast<const float *>(rows);
  else a.rho = PyFloat_AsDouble(args[6]);
  const bool id32 = PyObject_IsTrue(args[7]);
  a.id_dtype = id32 ? DVP_ID_I32 : DVP_ID_I64;
  a.stream = stream_of(args[8], z.get_device());
  a.launch_hint = static_cast<uint32_t>(PyLong_AsUnsignedLong(args[9]));
  if (PyErr_Occurred()) throw python_error();
  // rows 0 to 3 of the storage: three vectors of 4 bytes a token; behind them the ids
  Vectors v(z, T, 5);
  keep_for(v.buf, args[8]);
  THPObjectPtr d(PyDict_New());
  if (!d) throw python_error();
  put(d.get(), g_names.logp, v.make(0, at::kFloat, &a.logp));
  put(d.get(), g_names.logp_mp, v.make(1, at::kFloat, &a.logp_mp));
  put(d.get(), g_names.count, v.make(2, at::kInt, &a.count));
  a.ids = v.base + 3 * v.stride;
  put(d.get(), g_more.ids, THPVariable_Wrap(row_view(v.buf.storage(), v.keys, id32 ? at::kInt : at::kLong, 3, v.stride, T)));
  THPObjectPtr result(namespace_of(d.get()));
  int status;
  Py_BEGIN_ALLOW_THREADS status = entry(&a);
  Py_END_ALLOW_THREADS return finish(status, result);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"outputs", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(outputs)), METH_FASTCALL,
                          "outputs(like, T, floats, counts) -> (tensors, address, stride)"},
                         {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward)), METH_FASTCALL,
                          "dvp_forward's arguments in, its result or the library's status out"},
                         {"rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rms_norm)), METH_FASTCALL,
                          "dvp_rms_norm's arguments in, its result or the library's status out"},
                         {"rms_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rms_norm_backward)),
                          METH_FASTCALL, "dvp_rms_norm_backward's arguments in, its result or the library's status out"},
                         {"gemm_fp8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gemm_fp8)), METH_FASTCALL,
                          "dvp_gemm_fp8's arguments in, its result or the library's status out"},
                         {"sample", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(sample)), METH_FASTCALL,
                          "dvp_sample's arguments in, its result or the library's status out"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// PyInit__host: the module says what it was built for (build.py looks for the text in the file, binding.py asks the module)
extern "C" __attribute__((visibility("default"))) PyObject *PyInit__host() {
  static const char text[] = "[built for " DVP_HOST_TARGET "]";
  if (!make_names()) return nullptr;
  PyObject *m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", text) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
