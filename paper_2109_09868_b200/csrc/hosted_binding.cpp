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
  int (*block_norm)(const approxifer_block_norm_args*, void*) = nullptr;
  int (*mx_quantize)(const approxifer_mx_array_args*, void*) = nullptr;
  int (*mx_dequantize)(const approxifer_mx_array_args*, void*) = nullptr;
  int (*mx_linear)(const approxifer_mx_linear_args*, void*) = nullptr;
  int64_t (*mx_linear_workspace)(const approxifer_mx_linear_args*) = nullptr;
  int (*prefix_attention)(const approxifer_prefix_attention_args*, void*) = nullptr;
  int64_t (*prefix_attention_workspace)(const approxifer_prefix_attention_args*) = nullptr;
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

// Whether the call went well; sets the Python exception where not.
bool succeeded(int rc, const char* where) {
  if (rc == APPROXIFER_OK) return true;
  PyObject* args = Py_BuildValue("(is)", rc, where);
  PyObject* e = args ? PyObject_CallObject(entry.error, args) : nullptr;
  Py_XDECREF(args);
  if (e) PyErr_SetObject(entry.error, e);
  Py_XDECREF(e);
  return false;
}

PyObject* output(const at::Tensor& out, PyObject* given) { return given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(out); }

PyObject* finish(int rc, const char* where, const at::Tensor& out, PyObject* given) { return succeeded(rc, where) ? output(out, given) : nullptr; }

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

// What both attentions take: queries, caches, table, starts, lengths, bound, scale, output.
void fill_attention(approxifer_attention_args& a, PyObject* qo, PyObject* ko, PyObject* vo, PyObject* to, PyObject* so, PyObject* lo, PyObject* max_q, PyObject* scale,
                    PyObject* given, at::Tensor& out, int device) {
  const at::Tensor &q = tensor(qo, "q"), &k = tensor(ko, "k_cache"), &v = tensor(vo, "v_cache"), &table = tensor(to, "block_table"), &start = tensor(so, "q_start"),
                   &len = tensor(lo, "kv_len");
  if (q.dim() != 3 || k.dim() != 4 || table.dim() != 2) throw Refusal("q must be [T][Hq][D], the caches [pages][Hkv][page][D], block_table [batch][pages]");
  a.T = q.size(0), a.Hq = (int32_t)q.size(1), a.D = (int32_t)q.size(2);
  a.num_pages = k.size(0), a.Hkv = (int32_t)k.size(1), a.page_size = (int32_t)k.size(2);
  a.batch = (int32_t)table.size(0), a.table_pages = table.size(1);
  if (a.Hq != q.size(1) || a.D != q.size(2) || a.Hkv != k.size(1) || a.page_size != k.size(2) || a.batch != table.size(0)) throw Refusal("a size is out of range");
  a.max_q = number32(max_q, "max_q");
  a.scale = scale == Py_None ? 1.f / std::sqrt((float)a.D) : (float)real(scale);
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
  if (given == Py_None) {
    out = fresh(q.sizes(), at::kBFloat16, q);
  } else {
    out = tensor(given, "out");
    check(out, at::kBFloat16, q.sizes(), device, "out");
  }
  a.out = data<uint16_t>(out), a.o_tstride = out.stride(0), a.o_hstride = out.stride(1);
}

// A workspace: the one given, or a new one of `bytes`.
at::Tensor workspace_of(PyObject* given, int64_t bytes, const at::Tensor& like, int device) {
  at::Tensor room;
  if (given != Py_None) {
    room = tensor(given, "workspace");
    if (!room.is_cuda() || room.get_device() != device || !room.is_contiguous()) throw Refusal("workspace must be a contiguous CUDA tensor on the operands' device");
  } else if (bytes > 0) {
    room = fresh({bytes}, at::kByte, like);
  }
  return room;
}

// (q, k_cache, v_cache, block_table, q_start, kv_len, max_q, window, sinks, scale or None, out, workspace or None, stream)
PyObject* attention(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 13);
    const at::Tensor& q = tensor(arg[0], "q");
    const int device = device_of(q, "q");
    approxifer_attention_args a{};
    at::Tensor out;
    a.window = number32(arg[7], "window"), a.sinks = number32(arg[8], "sinks");
    fill_attention(a, arg[0], arg[1], arg[2], arg[3], arg[4], arg[5], arg[6], arg[9], arg[10], out, device);
    // (on the current stream the allocator's order makes a temporary safe; with another stream the call does without)
    const at::Tensor room = workspace_of(arg[11], arg[11] == Py_None && arg[12] == Py_None ? entry.attention_workspace(&a) : 0, q, device);
    if (room.defined()) a.workspace = room.data_ptr(), a.workspace_bytes = room.numel() * (int64_t)room.element_size();
    return finish(entry.attention(&a, stream_of(arg[12], device)), "approxifer_attention", out, arg[10]);
  });
}

// (q, k_cache, v_cache, prefix_table, prefix_len, block_table, q_start, kv_len, max_q, scale or None, out, workspace or None, stream)
PyObject* prefix_attention(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 13);
    const at::Tensor &q = tensor(arg[0], "q"), &prefix = tensor(arg[3], "prefix_table");
    const int device = device_of(q, "q");
    approxifer_prefix_attention_args g{};
    at::Tensor out;
    fill_attention(g.own, arg[0], arg[1], arg[2], arg[5], arg[6], arg[7], arg[8], arg[9], arg[10], out, device);
    if (prefix.dim() != 1) throw Refusal("prefix_table must be [pages]");
    check(prefix, at::kInt, prefix.sizes(), device, "prefix_table");
    g.prefix_table = data<int32_t>(prefix), g.prefix_pages = prefix.size(0), g.prefix_len = number(arg[4]);
    const at::Tensor room = workspace_of(arg[11], arg[11] == Py_None ? entry.prefix_attention_workspace(&g) : 0, q, device);
    if (room.defined()) g.own.workspace = room.data_ptr(), g.own.workspace_bytes = room.numel() * (int64_t)room.element_size();
    return finish(entry.prefix_attention(&g, stream_of(arg[12], device)), "approxifer_prefix_attention", out, arg[10]);
  });
}

// (residual, block, gate, block_weight, block_bias, next_weight, next_bias, after, before, gate activation (codes), residual_scale,
//  block_scale, eps, residual_out, next_out, stream) -> (residual_out, next or None)
PyObject* block_norm(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 16);
    const at::Tensor& r = tensor(arg[0], "residual");
    const int device = device_of(r, "residual");
    if (r.dim() != 2) throw Refusal("residual must be [T][N]");
    const bool has_block = arg[1] != Py_None;
    approxifer_block_norm_args a{};
    a.T = r.size(0), a.N = (int32_t)r.size(1);
    if (a.N != r.size(1)) throw Refusal("residual's rows are out of range");
    a.stream_type = type_code(r.scalar_type(), "residual");
    // the type of all but the residuals: the block's; without one that of the first weight, or of the output, else the residuals'
    at::ScalarType type = r.scalar_type();
    for (int i : {14, 6, 5, 1})
      if (arg[i] != Py_None) type = tensor(arg[i], i == 14 ? "next_out" : i == 6 ? "next_bias" : i == 5 ? "next_weight" : "block").scalar_type();
    a.type = type_code(type, "block");
    a.after = number32(arg[7], "after"), a.before = number32(arg[8], "before"), a.gate_activation = number32(arg[9], "gate_activation");
    a.residual_scale = (float)real(arg[10]), a.block_scale = (float)real(arg[11]), a.eps = (float)real(arg[12]);
    const int64_t width = r.size(1);
    auto rows = [&](PyObject* o, at::ScalarType t, const char* name, int64_t& stride) -> const at::Tensor& {
      const at::Tensor& v = tensor(o, name);
      check(v, t, {a.T, width}, device, name);
      stride = a.T == 1 ? width : v.stride(0);  // (of a single row the stride says nothing)
      return v;
    };
    auto vec = [&](PyObject* o, const char* name) -> const void* {
      if (o == Py_None) return nullptr;
      const at::Tensor& v = tensor(o, name);
      check(v, type, {width}, device, name);
      return v.data_ptr();
    };
    a.R = rows(arg[0], r.scalar_type(), "residual", a.r_rstride).data_ptr();
    if (has_block) a.Y = rows(arg[1], type, "block", a.y_rstride).data_ptr();
    if (arg[2] != Py_None) {
      const at::Tensor& g = tensor(arg[2], "gate");
      const bool columns = g.dim() == 1, tokens = g.dim() == 2 && g.size(1) == 1 && width != 1;
      if (columns) check(g, type, {width}, device, "gate");
      else if (tokens) check(g, type, {a.T, 1}, device, "gate");
      else check(g, type, {a.T, width}, device, "gate");
      a.gate = g.data_ptr(), a.g_cstride = tokens ? 0 : 1, a.g_rstride = columns || a.T == 1 ? 0 : g.stride(0);
    }
    a.after_weight = vec(arg[3], "block_weight"), a.after_bias = vec(arg[4], "block_bias");
    a.before_weight = vec(arg[5], "next_weight"), a.before_bias = vec(arg[6], "next_bias");
    if ((a.after_weight || a.after_bias) && a.after == APPROXIFER_NORM_NONE) throw Refusal("block_weight and block_bias come with after");
    if ((a.before_weight || a.before_bias || arg[14] != Py_None) && a.before == APPROXIFER_NORM_NONE) throw Refusal("next_weight, next_bias and next_out come with before");
    if (!has_block && arg[13] != Py_None) throw Refusal("residual_out comes with block");
    at::Tensor r_out, x;
    if (has_block) {
      r_out = arg[13] == Py_None ? fresh({a.T, width}, r.scalar_type(), r) : rows(arg[13], r.scalar_type(), "residual_out", a.ro_rstride);
      a.R_out = r_out.data_ptr(), a.ro_rstride = a.T == 1 ? width : r_out.stride(0);
    }
    if (a.before != APPROXIFER_NORM_NONE) {
      x = arg[14] == Py_None ? fresh({a.T, width}, type, r) : rows(arg[14], type, "next_out", a.x_rstride);
      a.X = x.data_ptr(), a.x_rstride = a.T == 1 ? width : x.stride(0);
    }
    if (!succeeded(entry.block_norm(&a, stream_of(arg[15], device)), "approxifer_block_norm")) return nullptr;
    PyObject* first = has_block ? output(r_out, arg[13]) : Py_NewRef(arg[0]);
    PyObject* second = x.defined() ? output(x, arg[14]) : Py_NewRef(Py_None);
    return Py_BuildValue("(NN)", first, second);
  });
}

// Codes [M][K/2] and scales [ceil(M/128)][ceil(K/128)][512] of an array; returns K.
int64_t check_mx(const at::Tensor& codes, const at::Tensor& scales, int device, const char* codes_name, const char* scales_name) {
  if (codes.dim() != 2) throw Refusal(std::string(codes_name) + " must be [rows][K/2]");
  check(codes, at::kByte, codes.sizes(), device, codes_name);
  const int64_t m = codes.size(0), k = 2 * codes.size(1);
  check(scales, at::kByte, {(m + 127) / 128, (k + 127) / 128, 512}, device, scales_name);
  if (!scales.is_contiguous()) throw Refusal(std::string(scales_name) + " must be contiguous");
  return k;
}
// (of a single row the stride says nothing)
int64_t code_stride(const at::Tensor& codes) { return codes.size(0) <= 1 ? (codes.size(1) + 15) / 16 * 16 : codes.stride(0); }

// (X, codes, scales, stream) -> (codes, scales)
PyObject* mx_quantize(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 4);
    const at::Tensor& x = tensor(arg[0], "X");
    const int device = device_of(x, "X");
    if (x.dim() != 2) throw Refusal("X must be [M][K]");
    const int64_t m = x.size(0), k = x.size(1);
    if (k % 32 != 0) throw Refusal("X's rows must be whole groups of 32");
    check(x, x.scalar_type(), x.sizes(), device, "X");
    approxifer_mx_array_args a{};
    a.M = m, a.K = k, a.type = type_code(x.scalar_type(), "X");
    a.X = x.data_ptr(), a.x_rstride = m == 1 ? k : x.stride(0);
    const at::Tensor codes = arg[1] == Py_None ? fresh({m, k / 2}, at::kByte, x) : tensor(arg[1], "codes");
    const at::Tensor scales = arg[2] == Py_None ? fresh({(m + 127) / 128, (k + 127) / 128, 512}, at::kByte, x) : tensor(arg[2], "scales");
    if (codes.dim() != 2 || codes.size(0) != m || check_mx(codes, scales, device, "codes", "scales") != k) throw Refusal("codes must be [M][K/2]");
    a.codes = data<uint8_t>(codes), a.c_rstride = code_stride(codes), a.scales = data<uint8_t>(scales);
    if (!succeeded(entry.mx_quantize(&a, stream_of(arg[3], device)), "approxifer_mx_quantize")) return nullptr;
    PyObject* first = output(codes, arg[1]);
    return Py_BuildValue("(NN)", first, output(scales, arg[2]));
  });
}

// (codes, scales, out_dtype, X, stream)
PyObject* mx_dequantize(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 5);
    const at::Tensor &codes = tensor(arg[0], "codes"), &scales = tensor(arg[1], "scales");
    const int device = device_of(codes, "codes");
    const int64_t k = check_mx(codes, scales, device, "codes", "scales"), m = codes.size(0);
    at::ScalarType type = at::kBFloat16;
    if (arg[2] != Py_None) {
      if (!THPDtype_Check(arg[2])) throw Refusal("out_dtype must be a torch.dtype");
      type = reinterpret_cast<THPDtype*>(arg[2])->scalar_type;
    } else if (arg[3] != Py_None) {
      type = tensor(arg[3], "X").scalar_type();
    }
    approxifer_mx_array_args a{};
    a.M = m, a.K = k, a.type = type_code(type, "out_dtype");
    const at::Tensor x = arg[3] == Py_None ? fresh({m, k}, type, codes) : tensor(arg[3], "X");
    check(x, type, {m, k}, device, "X");
    a.X = x.data_ptr(), a.x_rstride = m == 1 ? k : x.stride(0);
    a.codes = data<uint8_t>(codes), a.c_rstride = code_stride(codes), a.scales = data<uint8_t>(scales);
    return finish(entry.mx_dequantize(&a, stream_of(arg[4], device)), "approxifer_mx_dequantize", x, arg[3]);
  });
}

// (X, weight codes, weight scales, x_scales or None, bias, activation code, residual, out_dtype, Y, workspace or None, stream)
PyObject* mx_linear(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 11);
    const at::Tensor &x = tensor(arg[0], "X"), &w = tensor(arg[1], "weight"), &ws = tensor(arg[2], "weight_scales");
    const int device = device_of(x, "X");
    if (x.dim() != 2) throw Refusal("X must be [M][K], or [M][K/2] codes");
    approxifer_mx_linear_args a{};
    a.M = x.size(0), a.N = w.dim() > 0 ? w.size(0) : 0, a.K = check_mx(w, ws, device, "weight", "weight_scales");
    a.Wt = data<uint8_t>(w), a.w_rstride = code_stride(w), a.w_scales = data<uint8_t>(ws);
    if (arg[3] != Py_None) {
      const at::Tensor& xs = tensor(arg[3], "x_scales");
      if (check_mx(x, xs, device, "X", "x_scales") != a.K) throw Refusal("X and weight must have rows of the same length");
      a.x_rstride = code_stride(x), a.x_scales = data<uint8_t>(xs);
      if (a.x_scales == nullptr) a.x_scales = a.w_scales;  // (no rows: nothing is read)
    } else {
      check(x, at::kBFloat16, {a.M, a.K}, device, "X");
      a.x_rstride = a.M == 1 ? a.K : x.stride(0);
    }
    a.X = x.data_ptr();
    at::ScalarType out = at::kBFloat16;
    if (arg[7] != Py_None) {
      if (!THPDtype_Check(arg[7])) throw Refusal("out_dtype must be a torch.dtype");
      out = reinterpret_cast<THPDtype*>(arg[7])->scalar_type;
    } else if (arg[8] != Py_None) {
      out = tensor(arg[8], "Y").scalar_type();
    }
    a.out_type = type_code(out, "out_dtype");
    a.activation = number32(arg[5], "activation");
    if (arg[4] != Py_None) {
      const at::Tensor& b = tensor(arg[4], "bias");
      check(b, at::kBFloat16, {a.N}, device, "bias");
      a.bias = data<uint16_t>(b);
    }
    if (arg[6] != Py_None) {
      const at::Tensor& r = tensor(arg[6], "residual");
      check(r, out, {a.M, a.N}, device, "residual");
      a.R = r.data_ptr(), a.r_rstride = a.M == 1 ? a.N : r.stride(0);
    }
    at::Tensor y;
    if (arg[8] == Py_None) {
      y = fresh({a.M, a.N}, out, x);
    } else {
      y = tensor(arg[8], "Y");
      check(y, out, {a.M, a.N}, device, "Y");
    }
    a.Y = y.data_ptr(), a.y_rstride = a.M == 1 ? a.N : y.stride(0);
    const at::Tensor room = workspace_of(arg[9], arg[9] == Py_None ? entry.mx_linear_workspace(&a) : 0, x, device);
    if (room.defined()) a.workspace = room.data_ptr(), a.workspace_bytes = room.numel() * (int64_t)room.element_size();
    return finish(entry.mx_linear(&a, stream_of(arg[10], device)), "approxifer_mx_linear", y, arg[8]);
  });
}

// (the error class, then the addresses of the C entry points, in this order)
PyObject* bind(PyObject*, PyObject* const* arg, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n, 12);
    Py_ssize_t at = 1;
    auto take = [&](auto& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(PyLong_AsVoidPtr(arg[at++])); };
    take(entry.linear), take(entry.norm_rope), take(entry.attention), take(entry.attention_workspace), take(entry.block_norm), take(entry.mx_quantize),
        take(entry.mx_dequantize), take(entry.mx_linear), take(entry.mx_linear_workspace), take(entry.prefix_attention), take(entry.prefix_attention_workspace);
    if (PyErr_Occurred()) throw Raised();
    entry.error = Py_NewRef(arg[0]);
    return Py_NewRef(Py_None);
  });
}

PyMethodDef methods[] = {{"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear)), METH_FASTCALL, nullptr},
                         {"norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_rope)), METH_FASTCALL, nullptr},
                         {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attention)), METH_FASTCALL, nullptr},
                         {"block_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(block_norm)), METH_FASTCALL, nullptr},
                         {"mx_quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_quantize)), METH_FASTCALL, nullptr},
                         {"mx_dequantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_dequantize)), METH_FASTCALL, nullptr},
                         {"mx_linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_linear)), METH_FASTCALL, nullptr},
                         {"prefix_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(prefix_attention)), METH_FASTCALL, nullptr},
                         {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hosted", "Marshalling of the hosted-model operators.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject* PyInit__hosted(void) { return PyModule_Create(&module); }
