// Python binding of the hosted-model operators, in C++: a single-token call takes a few microseconds on the GPU, and
// marshalling its two dozen numbers in Python would take longer.  Marshalling only, as in binding.py: tensors become device
// pointers and strides in the C structs of approxifer.h, outputs that are not given are allocated, and the C entry point --
// handed over by address from the loaded library -- is called.  Nothing is computed here and there is no fallback.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <sstream>
#include <stdexcept>

#include "../../include/approxifer.h"

namespace {

struct Entry {
  int (*linear)(const approxifer_linear_args*, void*) = nullptr;
  int (*norm_rope)(const approxifer_norm_rope_args*, void*) = nullptr;
  int (*attention)(const approxifer_attention_args*, void*) = nullptr;
  int64_t (*attention_workspace)(const approxifer_attention_args*) = nullptr;
  PyObject* error = nullptr;  // ApproxiferError(code, where)
} entry;

struct Refusal : std::runtime_error {  // becomes a ValueError
  using std::runtime_error::runtime_error;
};
struct Raised {};  // a Python exception is set already

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refusal(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}

std::string describe(at::IntArrayRef shape) {
  std::ostringstream s;
  s << shape;
  return s.str();
}

// A CUDA tensor on this device, of this type and shape, innermost dimension contiguous.
void check(const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape, int device, const char* name) {
  const int64_t n = t.dim();
  if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.sizes() != shape || (n > 0 && shape[n - 1] > 1 && t.stride(n - 1) != 1)) {
    std::ostringstream s;
    s << name << " must be " << c10::toString(type) << " " << shape << " on CUDA device " << device << " with a contiguous innermost dimension, got "
      << c10::toString(t.scalar_type()) << " " << t.sizes() << " on " << t.device() << " with strides " << t.strides();
    throw Refusal(s.str());
  }
}

int device_of(const at::Tensor& t, const char* name) {
  if (!t.is_cuda()) throw Refusal(std::string(name) + " must be a CUDA tensor (the library has no CPU path)");
  const int device = t.get_device();
  if (device != c10::cuda::current_device()) throw Refusal(std::string(name) + " must be on the current CUDA device");
  return device;
}

void* stream_of(PyObject* handle, int device) {
  if (handle == Py_None) return c10::cuda::getCurrentCUDAStream(device).stream();
  void* p = PyLong_AsVoidPtr(handle);
  if (p == nullptr && PyErr_Occurred()) throw Raised();
  return p;
}

at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) { return at::empty(shape, like.options().dtype(type)); }

PyObject* finish(int rc, const char* where, const at::Tensor& out, PyObject* given) {
  if (rc != APPROXIFER_OK) {
    PyObject* args = Py_BuildValue("(is)", rc, where);
    PyObject* e = args ? PyObject_CallObject(entry.error, args) : nullptr;
    Py_XDECREF(args);
    if (e) PyErr_SetObject(entry.error, e);
    Py_XDECREF(e);
    return nullptr;
  }
  if (given != Py_None) return Py_NewRef(given);
  return THPVariable_Wrap(out);
}

template <typename F>
PyObject* guarded(F&& body) {
  try {
    return body();
  } catch (const Raised&) {
  } catch (const Refusal& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

int64_t number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
int32_t number32(PyObject* o, const char* name) {
  const int64_t v = number(o);
  if (v != (int32_t)v) throw Refusal(std::string(name) + " is out of range");
  return (int32_t)v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v != 0;
}

int32_t type_code(at::ScalarType t, const char* name) {
  if (t == at::kBFloat16) return APPROXIFER_TYPE_BF16;
  if (t == at::kFloat) return APPROXIFER_TYPE_F32;
  throw Refusal(std::string(name) + " must be torch.bfloat16 or torch.float32");
}

void need(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) throw Refusal("wrong number of arguments");
}

template <typename T>
T* data(const at::Tensor& t) {
  return static_cast<T*>(t.data_ptr());
}

// (X, weight, bias, activation code, residual, out_dtype, Y, stream)
PyObject* linear(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 8);
    const at::Tensor &x = tensor(arg[0], "X"), &w = tensor(arg[1], "weight");
    const int device = device_of(x, "X");
    if (x.dim() != 2 || w.dim() != 2) throw Refusal("X must be [M][K] and weight [N][K]");
    approxifer_linear_args a{};
    a.M = x.size(0), a.K = x.size(1), a.N = w.size(0);
    at::ScalarType out = at::kBFloat16;
    if (arg[5] != Py_None) {
      if (!THPDtype_Check(arg[5])) throw Refusal("out_dtype must be a torch.dtype");
      out = reinterpret_cast<THPDtype*>(arg[5])->scalar_type;
    } else if (arg[6] != Py_None) {
      out = tensor(arg[6], "Y").scalar_type();
    }
    a.out_type = type_code(out, "out_dtype");
    a.activation = number32(arg[3], "activation");
    check(x, at::kBFloat16, {a.M, a.K}, device, "X");
    check(w, at::kBFloat16, {a.N, a.K}, device, "weight");
    a.X = data<uint16_t>(x), a.x_rstride = x.stride(0);
    a.Wt = data<uint16_t>(w), a.w_rstride = w.stride(0);
    if (arg[2] != Py_None) {
      const at::Tensor& b = tensor(arg[2], "bias");
      check(b, at::kBFloat16, {a.N}, device, "bias");
      a.bias = data<uint16_t>(b);
    }
    if (arg[4] != Py_None) {
      const at::Tensor& r = tensor(arg[4], "residual");
      check(r, out, {a.M, a.N}, device, "residual");
      a.R = r.data_ptr(), a.r_rstride = r.stride(0);
    }
    at::Tensor y;
    if (arg[6] == Py_None) {
      y = fresh({a.M, a.N}, out, x);
    } else {
      y = tensor(arg[6], "Y");
      check(y, out, {a.M, a.N}, device, "Y");
    }
    a.Y = y.data_ptr(), a.y_rstride = y.stride(0);
    if (a.M == 1) {  // (the row stride of a single row says nothing)
      a.x_rstride = std::max(a.x_rstride, a.K), a.y_rstride = std::max(a.y_rstride, a.N);
      if (a.R) a.r_rstride = std::max(a.r_rstride, a.N);
    }
    if (a.N == 1) a.w_rstride = std::max(a.w_rstride, a.K);
    return finish(entry.linear(&a, stream_of(arg[7], device)), "approxifer_linear", y, arg[6]);
  });
}

// (q, k, v, q_weight, k_weight, cos_sin, positions, k_cache, v_cache, slots, q_out, eps, interleaved, status, stream)
PyObject* norm_rope(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 15);
    const at::Tensor &q = tensor(arg[0], "q"), &cs = tensor(arg[5], "cos_sin"), &pos = tensor(arg[6], "positions");
    const int device = device_of(q, "q");
    const at::ScalarType type = q.scalar_type();
    const bool has_k = arg[1] != Py_None, has_v = arg[2] != Py_None;
    if (q.dim() != 3 || cs.dim() != 2 || !cs.is_contiguous()) throw Refusal("q must be [T][Hq][D] and cos_sin a contiguous [positions][rot]");
    if (has_k != (arg[7] != Py_None) || has_v != (arg[8] != Py_None)) throw Refusal("k comes with k_cache and v with v_cache");
    approxifer_norm_rope_args a{};
    a.type = type_code(type, "q");
    a.T = q.size(0), a.Hq = (int32_t)q.size(1), a.D = (int32_t)q.size(2);
    a.Hkv = 1, a.page_size = 1;
    int64_t kv_heads = 1, page = 1;
    if (has_k || has_v) {
      const at::Tensor& c = tensor(arg[has_k ? 7 : 8], has_k ? "k_cache" : "v_cache");
      if (c.dim() != 4 || arg[9] == Py_None) throw Refusal("the caches must be [pages][Hkv][page][D], with slots");
      a.num_pages = c.size(0), kv_heads = c.size(1), page = c.size(2);
      a.Hkv = (int32_t)kv_heads, a.page_size = (int32_t)page;
      if (a.Hkv != kv_heads || a.page_size != page) throw Refusal("the caches' heads or pages are out of range");
    }
    if (a.Hq != q.size(1) || a.D != q.size(2)) throw Refusal("q's heads are out of range");
    check(q, type, {a.T, q.size(1), q.size(2)}, device, "q");
    a.q = q.data_ptr(), a.q_tstride = q.stride(0), a.q_hstride = q.stride(1);
    auto rows = [&](PyObject* o, const char* name, const void*& p, int64_t& ts, int64_t& hs) {
      const at::Tensor& t = tensor(o, name);
      check(t, type, {a.T, kv_heads, q.size(2)}, device, name);
      p = t.data_ptr(), ts = t.stride(0), hs = t.stride(1);
    };
    auto cache = [&](PyObject* o, const char* name, void*& p, int64_t& ps, int64_t& hs, int64_t& rs) {
      const at::Tensor& t = tensor(o, name);
      check(t, type, {a.num_pages, kv_heads, page, q.size(2)}, device, name);
      p = t.data_ptr(), ps = t.stride(0), hs = t.stride(1), rs = t.stride(2);
    };
    if (has_k) rows(arg[1], "k", a.k, a.k_tstride, a.k_hstride), cache(arg[7], "k_cache", a.k_cache, a.kc_pstride, a.kc_hstride, a.kc_rstride);
    if (has_v) rows(arg[2], "v", a.v, a.v_tstride, a.v_hstride), cache(arg[8], "v_cache", a.v_cache, a.vc_pstride, a.vc_hstride, a.vc_rstride);
    auto vec = [&](PyObject* o, at::ScalarType t, int64_t len, const char* name) -> const at::Tensor& {
      const at::Tensor& v = tensor(o, name);
      check(v, t, {len}, device, name);
      return v;
    };
    if (arg[3] != Py_None) a.q_weight = vec(arg[3], type, q.size(2), "q_weight").data_ptr();
    if (arg[4] != Py_None) a.k_weight = vec(arg[4], type, q.size(2), "k_weight").data_ptr();
    check(cs, at::kFloat, {cs.size(0), cs.size(1)}, device, "cos_sin");
    a.positions_max = cs.size(0), a.rot = (int32_t)cs.size(1);
    if (a.rot != cs.size(1)) throw Refusal("cos_sin is out of range");
    a.cos_sin = data<float>(cs);
    a.positions = data<int32_t>(vec(arg[6], at::kInt, a.T, "positions"));
    (void)pos;
    if (arg[9] != Py_None) a.slots = data<int64_t>(vec(arg[9], at::kLong, a.T, "slots"));
    at::Tensor out;
    if (arg[10] == Py_None) {
      out = fresh(q.sizes(), type, q);
    } else {
      out = tensor(arg[10], "q_out");
      check(out, type, q.sizes(), device, "q_out");
    }
    a.q_out = out.data_ptr(), a.qo_tstride = out.stride(0), a.qo_hstride = out.stride(1);
    a.eps = (float)real(arg[11]);
    a.interleaved = truth(arg[12]);
    if (arg[13] != Py_None) a.status = reinterpret_cast<uint32_t*>(data<int32_t>(vec(arg[13], at::kInt, a.T, "status")));
    return finish(entry.norm_rope(&a, stream_of(arg[14], device)), "approxifer_qk_norm_rope", out, arg[10]);
  });
}

// (q, k_cache, v_cache, block_table, q_start, kv_len, max_q, window, sinks, scale or None, out, workspace or None, stream)
PyObject* attention(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 13);
    const at::Tensor &q = tensor(arg[0], "q"), &k = tensor(arg[1], "k_cache"), &v = tensor(arg[2], "v_cache"), &table = tensor(arg[3], "block_table"),
                     &start = tensor(arg[4], "q_start"), &len = tensor(arg[5], "kv_len");
    const int device = device_of(q, "q");
    if (q.dim() != 3 || k.dim() != 4 || table.dim() != 2) throw Refusal("q must be [T][Hq][D], the caches [pages][Hkv][page][D], block_table [batch][pages]");
    approxifer_attention_args a{};
    a.T = q.size(0), a.Hq = (int32_t)q.size(1), a.D = (int32_t)q.size(2);
    a.num_pages = k.size(0), a.Hkv = (int32_t)k.size(1), a.page_size = (int32_t)k.size(2);
    a.batch = (int32_t)table.size(0), a.table_pages = table.size(1);
    if (a.Hq != q.size(1) || a.D != q.size(2) || a.Hkv != k.size(1) || a.page_size != k.size(2) || a.batch != table.size(0)) throw Refusal("a size is out of range");
    a.max_q = number32(arg[6], "max_q"), a.window = number32(arg[7], "window"), a.sinks = number32(arg[8], "sinks");
    a.scale = arg[9] == Py_None ? 1.f / std::sqrt((float)a.D) : (float)real(arg[9]);
    check(q, at::kBFloat16, q.sizes(), device, "q");
    check(k, at::kBFloat16, {k.size(0), k.size(1), k.size(2), q.size(2)}, device, "k_cache");
    check(v, at::kBFloat16, k.sizes(), device, "v_cache");
    check(table, at::kInt, table.sizes(), device, "block_table");
    check(start, at::kInt, {table.size(0) + 1}, device, "q_start");
    check(len, at::kInt, {table.size(0)}, device, "kv_len");
    a.q = data<uint16_t>(q), a.q_tstride = q.stride(0), a.q_hstride = q.stride(1);
    a.k_cache = data<uint16_t>(k), a.kc_pstride = k.stride(0), a.kc_hstride = k.stride(1), a.kc_rstride = k.stride(2);
    a.v_cache = data<uint16_t>(v), a.vc_pstride = v.stride(0), a.vc_hstride = v.stride(1), a.vc_rstride = v.stride(2);
    a.block_table = data<int32_t>(table), a.table_stride = table.stride(0);
    a.q_start = data<int32_t>(start), a.kv_len = data<int32_t>(len);
    at::Tensor out, room;
    if (arg[10] == Py_None) {
      out = fresh(q.sizes(), at::kBFloat16, q);
    } else {
      out = tensor(arg[10], "out");
      check(out, at::kBFloat16, q.sizes(), device, "out");
    }
    a.out = data<uint16_t>(out), a.o_tstride = out.stride(0), a.o_hstride = out.stride(1);
    if (arg[11] != Py_None) {
      room = tensor(arg[11], "workspace");
      if (!room.is_cuda() || room.get_device() != device || !room.is_contiguous()) throw Refusal("workspace must be a contiguous CUDA tensor on q's device");
    } else if (arg[12] == Py_None) {  // (on the current stream the allocator's order makes a temporary safe)
      const int64_t bytes = entry.attention_workspace(&a);
      if (bytes > 0) room = fresh({bytes}, at::kByte, q);
    }
    if (room.defined()) a.workspace = room.data_ptr(), a.workspace_bytes = room.numel() * (int64_t)room.element_size();
    return finish(entry.attention(&a, stream_of(arg[12], device)), "approxifer_attention", out, arg[10]);
  });
}

// (addresses of approxifer_linear, _qk_norm_rope, _attention, _attention_workspace, the error class)
PyObject* bind(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 5);
    entry.linear = reinterpret_cast<decltype(entry.linear)>(PyLong_AsVoidPtr(arg[0]));
    entry.norm_rope = reinterpret_cast<decltype(entry.norm_rope)>(PyLong_AsVoidPtr(arg[1]));
    entry.attention = reinterpret_cast<decltype(entry.attention)>(PyLong_AsVoidPtr(arg[2]));
    entry.attention_workspace = reinterpret_cast<decltype(entry.attention_workspace)>(PyLong_AsVoidPtr(arg[3]));
    if (PyErr_Occurred()) throw Raised();
    entry.error = Py_NewRef(arg[4]);
    return Py_NewRef(Py_None);
  });
}

PyMethodDef methods[] = {{"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear)), METH_FASTCALL, nullptr},
                         {"norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_rope)), METH_FASTCALL, nullptr},
                         {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attention)), METH_FASTCALL, nullptr},
                         {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hosted", "Marshalling of the hosted-model operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__hosted(void) { return PyModule_Create(&module); }
