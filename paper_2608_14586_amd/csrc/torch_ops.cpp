// The 4-bit operators' Python calls: sizes and strides read off torch tensors,
// checked, and handed to the C ABI of include/vla_ops.h.
//
// A decode step's kernels take two to five microseconds.  Reading one tensor's
// type, shape, strides, device and address through Python attributes takes
// half a microsecond, and a call has up to nine tensors; here it takes
// nanoseconds.  Each function returns the vla_status, after raising ValueError
// for a tensor whose type, shape, device or size does not fit.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>

#include "../../include/vla_ops.h"

namespace {

// what is wrong, as the ValueError to raise
struct Misfit {
  const char *name, *need;
};

const at::Tensor& tensor_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Misfit{name, "a torch tensor"};
  return THPVariable_Unpack(o);
}
// on a GPU, and the current one: kernels run there
int device_of(const at::Tensor& t, const char* name) {
  if (!t.is_cuda()) throw Misfit{name, "a tensor on the GPU"};
  int current = -1;
  if (hipGetDevice(&current) != hipSuccess || current != t.get_device())
    throw Misfit{name, "a tensor on the current GPU"};
  return current;
}
void on(const at::Tensor& t, int device, const char* name) {
  if (!t.is_cuda() || t.get_device() != device) throw Misfit{name, "a tensor on the same GPU"};
}

// a dense tensor of that type and shape; NULL for None
void* dense(PyObject* o, at::ScalarType type, at::IntArrayRef shape, int device, const char* name) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor_of(o, name);
  on(t, device, name);
  if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
    throw Misfit{name, "a contiguous tensor of the type and shape that the call's other sizes give"};
  return t.data_ptr();
}
// dense memory of at least `need` bytes
void* memory(PyObject* o, size_t need, int device, const char* name, size_t* bytes = nullptr) {
  const at::Tensor& t = tensor_of(o, name);
  on(t, device, name);
  if (t.nbytes() < need || !t.is_contiguous()) throw Misfit{name, "as many contiguous bytes as the sizes need"};
  if (bytes) *bytes = t.nbytes();
  return t.data_ptr();
}
// [B, tokens, heads, dh], any outer strides; the stride of a dimension of one is never used
vla_heads heads(const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape, int device, const char* name) {
  on(t, device, name);
  if (t.scalar_type() != type || t.sizes() != shape || (t.stride(3) != 1 && t.size(3) != 1))
    throw Misfit{name, "a tensor of the type and shape that the call's other sizes give, its last dimension dense"};
  auto stride = [&](int d) { return t.size(d) == 1 ? 0 : t.stride(d); };
  return vla_heads{t.data_ptr(), stride(0), stride(1), stride(2)};
}
int int_of(PyObject* o, const char* name) {
  const long v = PyLong_AsLong(o);
  if ((v == -1 && PyErr_Occurred()) || v != (int)v) {
    PyErr_Clear();
    throw Misfit{name, "an integer of 32 bits"};
  }
  return (int)v;
}
// None: torch's current stream of the current device, where its tensors' work is
void* stream_of(PyObject* o) {
  if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
  void* s = PyLong_AsVoidPtr(o);
  if (!s && PyErr_Occurred()) {
    PyErr_Clear();
    throw Misfit{"stream", "None or a stream's address"};
  }
  return s;
}
int dim(const at::Tensor& t, int d, const char* name) {
  if (t.size(d) != (int)t.size(d)) throw Misfit{name, "sizes of 32 bits"};
  return (int)t.size(d);
}
void four(const at::Tensor& t, const char* name) {
  if (t.dim() != 4) throw Misfit{name, "four dimensions"};
}

constexpr auto BF16 = at::kBFloat16, F32 = at::kFloat, I32 = at::kInt;

// args: codes, scales, zeros, Wp, group, stream
vla_status w4_pack(PyObject* const* a) {
  const at::Tensor& codes = tensor_of(a[0], "codes");
  const int dev = device_of(codes, "codes"), group = int_of(a[4], "group");
  if (codes.dim() != 2 || codes.scalar_type() != at::kByte || !codes.is_contiguous())
    throw Misfit{"codes", "contiguous uint8 [N, K]"};
  if (group <= 0) return VLA_ERR_INVALID_ARG;
  const int N = dim(codes, 0, "codes"), K = dim(codes, 1, "codes");
  const int64_t per[2] = {N, (K + (int64_t)group - 1) / group};
  void* s = dense(a[1], BF16, per, dev, "scales");
  void* z = dense(a[2], BF16, per, dev, "zeros");
  return vla_op_w4_pack(codes.data_ptr(), s, z, memory(a[3], vla_op_w4_packed_bytes(N, K, group), dev, "Wp"), N, K,
                        group, stream_of(a[5]));
}

// args: x, Wp, residual, out, N, group, swiglu, stream
vla_status gemv_w4(PyObject* const* a) {
  const at::Tensor &x = tensor_of(a[0], "x"), &out = tensor_of(a[3], "out");
  const int dev = device_of(x, "x"), N = int_of(a[4], "N"), group = int_of(a[5], "group");
  const int swiglu = PyObject_IsTrue(a[6]);
  if (swiglu < 0) {
    PyErr_Clear();
    throw Misfit{"swiglu", "True or False"};
  }
  if (x.scalar_type() != BF16 || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) != 1))
    throw Misfit{"x", "bfloat16 [M, K] with dense rows"};
  const int M = dim(x, 0, "x"), K = dim(x, 1, "x");
  const int64_t wide[2] = {M, swiglu ? N / 2 : N};
  const bool f32 = out.scalar_type() == F32;
  on(out, dev, "out");
  if ((!f32 && out.scalar_type() != BF16) || out.sizes() != at::IntArrayRef(wide) ||
      (out.stride(1) != 1 && out.size(1) != 1))
    throw Misfit{"out", "float32 or bfloat16 [M, N] ([M, N / 2] with swiglu) with dense rows"};
  const int64_t ldx = M > 1 ? x.stride(0) : 0, ldo = M > 1 ? out.stride(0) : 0;
  const float* res = nullptr;
  if (a[2] != Py_None) {
    const at::Tensor& r = tensor_of(a[2], "residual");
    on(r, dev, "residual");
    if (r.scalar_type() != F32 || r.sizes() != at::IntArrayRef(wide) || (r.stride(1) != 1 && r.size(1) != 1) ||
        (M > 1 && r.stride(0) != ldo))
      throw Misfit{"residual", "float32 of out's shape and row stride"};
    res = (const float*)r.data_ptr();
  }
  return vla_op_gemv_w4(x.data_ptr(), ldx, memory(a[1], vla_op_w4_packed_bytes(N, K, group), dev, "Wp"), res,
                        out.data_ptr(), ldo, f32 ? VLA_F32 : VLA_BF16, swiglu, M, N, K, group, stream_of(a[7]));
}

// args: q, k, gq, gk, eps, cos, sin, pos, q_out, k_out, stream
vla_status qk_norm_rope(PyObject* const* a) {
  const at::Tensor &q = tensor_of(a[0], "q"), &k = tensor_of(a[1], "k");
  const int dev = device_of(q, "q");
  four(q, "q");
  four(k, "k");
  const at::ScalarType type = q.scalar_type();
  if (type != BF16 && type != F32) throw Misfit{"q", "float32 or bfloat16"};
  const int B = dim(q, 0, "q"), L = dim(q, 1, "q"), H = dim(q, 2, "q"), dh = dim(q, 3, "q"), Hkv = dim(k, 2, "k");
  const int64_t ks[4] = {B, L, Hkv, dh}, gs[1] = {dh}, ps[2] = {B, L};
  const vla_heads qh = heads(q, type, q.sizes(), dev, "q"), kh = heads(k, type, ks, dev, "k");
  const vla_heads qo = heads(tensor_of(a[8], "q_out"), BF16, q.sizes(), dev, "q_out");
  const vla_heads ko = heads(tensor_of(a[9], "k_out"), BF16, ks, dev, "k_out");
  int n_pos = 0;
  if (a[5] != Py_None) {
    const at::Tensor& c = tensor_of(a[5], "cos");
    if (c.dim() != 2) throw Misfit{"cos", "[n_pos, dh / 2]"};
    n_pos = dim(c, 0, "cos");
  }
  const int64_t ts[2] = {n_pos, dh / 2};
  // a table without rows has no address, and none at all means no rotation: any address, never read, stands for it
  auto table = [&](PyObject* o, const char* name) {
    void* p = dense(o, F32, ts, dev, name);
    return (const float*)(o != Py_None && n_pos == 0 ? qh.p : p);
  };
  const double eps = PyFloat_AsDouble(a[4]);
  if (eps == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Misfit{"eps", "a number"};
  }
  return vla_op_qk_norm_rope(&qh, &kh, type == F32 ? VLA_F32 : VLA_BF16, (float*)dense(a[2], F32, gs, dev, "gq"),
                             (float*)dense(a[3], F32, gs, dev, "gk"), (float)eps,
                             table(a[5], "cos"), table(a[6], "sin"), n_pos,
                             (int32_t*)dense(a[7], I32, ps, dev, "pos"), &qo, &ko, B, L, H, Hkv, dh, stream_of(a[10]));
}

// args: k, v, start, count, cache, L_cap, stream
vla_status kv4_rows(PyObject* const* a, bool load) {
  const at::Tensor &k = tensor_of(a[0], "k"), &v = tensor_of(a[1], "v");
  const int dev = device_of(k, "k"), cap = int_of(a[5], "L_cap");
  four(k, "k");
  const int B = dim(k, 0, "k"), L = dim(k, 1, "k"), Hkv = dim(k, 2, "k"), dh = dim(k, 3, "k");
  const vla_heads kh = heads(k, BF16, k.sizes(), dev, "k"), vh = heads(v, BF16, k.sizes(), dev, "v");
  const int64_t bs[1] = {B};
  const int32_t *start = (int32_t*)dense(a[2], I32, bs, dev, "start"), *count = (int32_t*)dense(a[3], I32, bs, dev, "count");
  void* cache = memory(a[4], vla_op_kv4_bytes(B, Hkv, cap, dh), dev, "cache");
  return load ? vla_op_kv4_load(cache, start, count, &kh, &vh, B, L, Hkv, cap, dh, stream_of(a[6]))
              : vla_op_kv4_store(&kh, &vh, start, count, cache, B, L, Hkv, cap, dh, stream_of(a[6]));
}
vla_status kv4_store(PyObject* const* a) { return kv4_rows(a, false); }
vla_status kv4_load(PyObject* const* a) { return kv4_rows(a, true); }

// args: q, cache, L_cap, Hkv, lens, o, max_len, window, sinks, scratch, stream
vla_status attention_kv4(PyObject* const* a) {
  const at::Tensor& q = tensor_of(a[0], "q");
  const int dev = device_of(q, "q"), cap = int_of(a[2], "L_cap"), Hkv = int_of(a[3], "Hkv");
  four(q, "q");
  const int B = dim(q, 0, "q"), Lq = dim(q, 1, "q"), H = dim(q, 2, "q"), dh = dim(q, 3, "q");
  const vla_heads qh = heads(q, BF16, q.sizes(), dev, "q");
  const vla_heads oh = heads(tensor_of(a[5], "o"), BF16, q.sizes(), dev, "o");
  const int64_t bs[1] = {B};
  if (a[4] == Py_None) throw Misfit{"lens", "int32 [B]"};
  size_t bytes = 0;
  void* scratch = a[9] == Py_None ? nullptr : memory(a[9], 0, dev, "scratch", &bytes);
  return vla_op_attention_kv4(&qh, memory(a[1], vla_op_kv4_bytes(B, Hkv, cap, dh), dev, "cache"),
                              (int32_t*)dense(a[4], I32, bs, dev, "lens"), &oh, B, Lq, H, Hkv, cap, dh,
                              int_of(a[6], "max_len"), int_of(a[7], "window"), int_of(a[8], "sinks"),
                              bytes ? scratch : nullptr, bytes, stream_of(a[10]));
}

// no exception leaves a call: a misfit becomes ValueError, anything else RuntimeError
template <vla_status (*F)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments are needed, %zd given", N, n);
    return nullptr;
  }
  try {
    const vla_status s = F(args);
    return PyErr_Occurred() ? nullptr : PyLong_FromLong(s);
  } catch (const Misfit& m) {
    PyErr_Format(PyExc_ValueError, "%s: %s is needed", m.name, m.need);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}
template <vla_status (*F)(PyObject* const*), int N>
constexpr PyMethodDef method(const char* name) {
  return {name, (PyCFunction)(void (*)(void))call<F, N>, METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<w4_pack, 6>("w4_pack"),
                         method<gemv_w4, 8>("gemv_w4"),
                         method<qk_norm_rope, 11>("qk_norm_rope"),
                         method<kv4_store, 7>("kv4_store"),
                         method<kv4_load, 7>("kv4_load"),
                         method<attention_kv4, 11>("attention_kv4"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_ops() { return PyModule_Create(&module); }
