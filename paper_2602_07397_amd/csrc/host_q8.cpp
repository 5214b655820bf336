// Argument marshalling of the 8-bit cache's per-layer calls: checks tensors,
// allocates outputs that were not passed and calls the C ABI, as binding.py does
// for the other calls. The calls of a decode step take 4 to 10 us on the GPU; the
// same in Python and ctypes takes longer than that on the host (decode attention
// 13.2 us, of which the launches are 6).
//
// A CPython module. The library's entry points come from binding.py, which has
// loaded it (setup); no computation and no state beyond their addresses.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <stdexcept>
#include <string>

#include "../../include/sketchwalk.h"

namespace {

PyObject* g_error = nullptr;                       // SketchWalkError
decltype(&sw_last_error) p_last_error;
decltype(&sw_block_tables) p_block_tables;
decltype(&sw_block_tables_workspace_bytes) p_block_tables_ws;
decltype(&sw_kv_append_q8) p_append;
decltype(&sw_kv_fetch_q8) p_fetch;
decltype(&sw_sparse_attn_decode_q8) p_attn;
decltype(&sw_decode_attn_q8_workspace_bytes) p_attn_ws;

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};

std::string shape_of(const at::Tensor& t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a CUDA (HIP) tensor");
  return THPVariable_Unpack(o);
}

// Address of a contiguous tensor of a type on the call's device.
void* address(const at::Tensor& t, at::ScalarType type, int64_t di, const char* name) {
  if (!t.is_cuda()) throw Refused(std::string(name) + " must be a CUDA (HIP) tensor");
  if (t.get_device() != di)
    throw Refused(std::string(name) + " is on " + t.device().str() + ", the call on cuda:" + std::to_string(di));
  if (t.scalar_type() != type)
    throw Refused(std::string(name) + " must have dtype " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
  if (!t.is_contiguous()) throw Refused(std::string(name) + " must be contiguous");
  return t.data_ptr();
}

int32_t* ints(const at::Tensor& t, int64_t n, int64_t di, const char* name) {
  if (t.numel() != n)
    throw Refused(std::string(name) + " has " + std::to_string(t.numel()) + " entries, " + std::to_string(n) + " needed");
  return static_cast<int32_t*>(address(t, at::kInt, di, name));
}

int32_t* ints(PyObject* o, int64_t n, int64_t di, const char* name) { return ints(tensor(o, name), n, di, name); }

// A size that the C ABI takes as int.
int fits(int64_t n, const char* what) {
  if (n > INT32_MAX) throw Refused(std::string(what) + ": " + std::to_string(n) + " does not fit in 32 bits");
  return (int)n;
}

void shaped(const at::Tensor& t, at::IntArrayRef want, const char* name) {
  if (t.sizes() == want) return;
  std::string s = std::string(name) + " of shape " + shape_of(t) + ", (";
  for (size_t i = 0; i < want.size(); ++i) s += (i ? ", " : "") + std::to_string(want[i]);
  throw Refused(s + ") needed");
}

int type_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return SW_BF16;
  if (t.scalar_type() == at::kFloat) return SW_F32;
  throw Refused(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
}

int64_t integer(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refused(std::string(name) + " must be an integer");
  }
  return v;
}

int small(PyObject* o, const char* name) {
  const int64_t v = integer(o, name);
  if (v < INT32_MIN || v > INT32_MAX) throw Refused(std::string(name) + " does not fit in 32 bits");
  return (int)v;
}

void* stream_of(PyObject* o) { return reinterpret_cast<void*>(PyLong_AsUnsignedLongLong(o)); }

void check(int rc, const char* what) {
  if (rc != SW_OK)
    throw Refused(std::string(what) + " failed with code " + std::to_string(rc) + ": " + p_last_error());
}

// A tensor that the caller passed, or a new one.
at::Tensor out_or(PyObject* o, const at::Tensor& like, int64_t n, at::ScalarType type, const char* name) {
  if (o != nullptr && o != Py_None) return tensor(o, name);
  return at::empty({n}, like.options().dtype(type));
}

// A vector of n entries of t's memory from entry `from` on.
at::Tensor piece(const at::Tensor& t, int64_t from, int64_t n) {
  at::Tensor x = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(t.storage()), t.key_set(), t.dtype());
  x.unsafeGetTensorImpl()->set_storage_offset(from);
  x.unsafeGetTensorImpl()->set_sizes_contiguous(n);
  return x;
}

struct Pool {
  int n_pages, h_kv, B, d;
  void *k, *v;
  uint8_t *ks, *vs;
};

// a[0..3]: keys, values and their scales.
Pool pool_of(PyObject* const* a, int64_t di) {
  const at::Tensor &k = tensor(a[0], "cache k"), &v = tensor(a[1], "cache v"), &ks = tensor(a[2], "cache k_scale"),
                   &vs = tensor(a[3], "cache v_scale");
  const bool same = k.dim() == 4 && v.dim() == 4 && ks.dim() == 2 && v.size(0) == k.size(0) && v.size(1) == k.size(1) &&
                    v.size(2) == k.size(3) && v.size(3) == k.size(2) && ks.size(0) == k.size(0) &&
                    ks.size(1) == k.size(1) && vs.sizes() == ks.sizes();
  if (!same)
    throw Refused("cache of shapes k " + shape_of(k) + ", v " + shape_of(v) + ", k_scale " + shape_of(ks) + ", v_scale " +
                  shape_of(vs) + ": (n_pages, h_kv, B, d), (n_pages, h_kv, d, B) and twice (n_pages, h_kv) needed");
  return {fits(k.size(0), "pages"), fits(k.size(1), "h_kv"), fits(k.size(2), "B"), fits(k.size(3), "d"),
          address(k, at::kFloat8_e4m3fn, di, "cache k"), address(v, at::kFloat8_e4m3fn, di, "cache v"),
          static_cast<uint8_t*>(address(ks, at::kByte, di, "cache k_scale")),
          static_cast<uint8_t*>(address(vs, at::kByte, di, "cache v_scale"))};
}

void count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) throw Refused("wrong number of arguments");
}

// (device, stream, old_len, new_len, B, tables, free_pages, n_free, n_slots, rows,
//  slots, cu, pos, status, workspace) -> (slots, cu, pos, status)
PyObject* block_tables(PyObject* const* a, Py_ssize_t n_args) {
  count(n_args, 15);
  const int64_t di = integer(a[0], "device");
  const at::Tensor &old = tensor(a[2], "old_len"), &tables = tensor(a[5], "tables"), &pages = tensor(a[6], "free_pages");
  if (tables.dim() != 2) throw Refused("tables of shape " + shape_of(tables) + ", (n, b_max) needed");
  const int64_t n_slots = integer(a[8], "n_slots");
  const int n = fits(tables.size(0), "requests"), b_max = fits(tables.size(1), "b_max"),
            n_pages = fits(pages.numel(), "free_pages");
  void* p_old = ints(old, n, di, "old_len");
  const int64_t wsb = p_block_tables_ws(n, n_slots);
  if (wsb < 0) check(SW_ERR_INVALID_ARG, "sw_block_tables_workspace_bytes");
  const at::Tensor slots = out_or(a[10], old, n_slots, at::kInt, "slots");
  at::Tensor cu, pos, status, ws;
  if (a[11] == Py_None && a[12] == Py_None && a[13] == Py_None) {
    // the small outputs together, in 64-byte pieces: an allocation takes 0.7 us on the host
    const int64_t c = (n + 16ll) & ~15ll, p = (n + 15ll) & ~15ll;
    const at::Tensor all = at::empty({c + p + 1}, old.options().dtype(at::kInt));
    cu = piece(all, 0, n + 1ll);
    pos = piece(all, c, n);
    status = piece(all, c + p, 1);
  } else {
    cu = out_or(a[11], old, n + 1ll, at::kInt, "cu");
    pos = out_or(a[12], old, n, at::kInt, "pos");
    status = out_or(a[13], old, 1, at::kInt, "status");
  }
  if (a[14] != Py_None) ws = tensor(a[14], "workspace");
  if (wsb > 0 && (!ws.defined() || ws.numel() < wsb)) ws = at::empty({wsb}, old.options().dtype(at::kByte));
  check(p_block_tables(n, small(a[4], "B"), b_max, static_cast<int32_t*>(p_old),
                       ints(a[3], n, di, "new_len"), static_cast<int32_t*>(address(tables, at::kInt, di, "tables")),
                       static_cast<int32_t*>(address(pages, at::kInt, di, "free_pages")), ints(a[7], 1, di, "n_free"),
                       n_pages, small(a[9], "rows"), n_slots, ints(slots, n_slots, di, "slots"),
                       ints(cu, n + 1ll, di, "cu"), ints(pos, n, di, "pos"), ints(status, 1, di, "status"),
                       ws.defined() ? address(ws, at::kByte, di, "workspace") : nullptr,
                       ws.defined() ? ws.numel() : 0, stream_of(a[1])),
        "sw_block_tables");
  return Py_BuildValue("(NNNN)", THPVariable_Wrap(slots), THPVariable_Wrap(cu), THPVariable_Wrap(pos),
                       THPVariable_Wrap(status));
}

// (device, stream, k, v, slots, cache k, v, k_scale, v_scale, cu)
PyObject* kv_append_q8(PyObject* const* a, Py_ssize_t n_args) {
  count(n_args, 10);
  const int64_t di = integer(a[0], "device");
  const Pool c = pool_of(a + 5, di);
  const at::Tensor &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &slots = tensor(a[4], "slots");
  const int64_t N = slots.numel();
  shaped(k, {c.h_kv, N, c.d}, "k");
  shaped(v, {c.h_kv, N, c.d}, "v");
  if (!k.is_cuda() || !v.is_cuda() || k.get_device() != di || v.get_device() != di)
    throw Refused("k, v on " + k.device().str() + ", " + v.device().str() + ", the cache on cuda:" + std::to_string(di));
  if (k.scalar_type() != v.scalar_type()) throw Refused("k and v must share a dtype");
  if (k.stride(2) != 1 || v.stride(2) != 1) throw Refused("k and v must be contiguous in their last dimension");
  // of a dimension of one entry the stride means nothing
  auto stride = [](const at::Tensor& x, int64_t dim) { return x.size(dim) > 1 ? x.stride(dim) : 0; };
  const int32_t* p_cu = nullptr;
  int n = 0;
  if (a[9] != Py_None) {
    const at::Tensor& cu = tensor(a[9], "cu");
    if (cu.numel() < 1 || cu.numel() > INT32_MAX) throw Refused("cu has " + std::to_string(cu.numel()) + " entries");
    n = (int)cu.numel() - 1;
    p_cu = ints(cu, cu.numel(), di, "cu");
  }
  check(p_append(type_code(k), k.data_ptr(), v.data_ptr(), stride(k, 0), stride(k, 1), stride(v, 0), stride(v, 1), N,
                 n, p_cu, ints(slots, N, di, "slots"), c.n_pages, c.h_kv, c.d, c.B, c.k, c.v, c.ks, c.vs, stream_of(a[1])),
        "sw_kv_append_q8");
  Py_RETURN_NONE;
}

// (device, stream, cache k, v, k_scale, v_scale, tables, first, cu, N, type code, K, V) -> (K, V)
PyObject* kv_fetch_q8(PyObject* const* a, Py_ssize_t n_args) {
  count(n_args, 13);
  const int64_t di = integer(a[0], "device"), N = integer(a[9], "N");
  const at::Tensor& tables = tensor(a[6], "tables");
  if (tables.dim() != 2) throw Refused("tables of shape " + shape_of(tables) + ", (n, b_max) needed");
  const int n = fits(tables.size(0), "sequences"), b_max = fits(tables.size(1), "b_max");
  const Pool c = pool_of(a + 2, di);
  if (N < 0) throw Refused("N=" + std::to_string(N) + " < 0");
  void* p_tables = address(tables, at::kInt, di, "tables");
  const int32_t* p_first = a[7] == Py_None ? nullptr : ints(a[7], n, di, "first");
  const int32_t* p_cu = ints(a[8], n + 1ll, di, "cu");
  at::Tensor K, V;
  if (a[11] == Py_None) {
    const auto type = integer(a[10], "dtype") == SW_BF16 ? at::kBFloat16 : at::kFloat;
    K = at::empty({c.h_kv, N, c.d}, tables.options().dtype(type));
    V = at::empty_like(K);
  } else {
    K = tensor(a[11], "K");
    V = tensor(a[12], "V");
    shaped(K, {c.h_kv, N, c.d}, "K");
    shaped(V, {c.h_kv, N, c.d}, "V");
  }
  const auto type = K.scalar_type();
  check(p_fetch(type_code(K), c.k, c.v, c.ks, c.vs, c.n_pages, c.h_kv, c.d, c.B, n, b_max,
                static_cast<int32_t*>(p_tables), p_first, p_cu, N, address(K, type, di, "K"), address(V, type, di, "V"),
                stream_of(a[1])),
        "sw_kv_fetch_q8");
  return Py_BuildValue("(NN)", THPVariable_Wrap(K), THPVariable_Wrap(V));
}

// (device, stream, q, cache k, v, k_scale, v_scale, tables, pos, idx, cnt, kmax,
//  scale, O, workspace) -> O
PyObject* sparse_attn_decode_q8(PyObject* const* a, Py_ssize_t n_args) {
  count(n_args, 15);
  const int64_t di = integer(a[0], "device");
  const at::Tensor &q = tensor(a[2], "q"), &tables = tensor(a[7], "tables"), &idx = tensor(a[9], "idx");
  const int b_max = tables.dim() == 2 ? fits(tables.size(1), "b_max") : 0;
  const Pool c = pool_of(a + 3, di);
  if (q.dim() != 3 || q.size(2) != c.d)
    throw Refused("q of shape " + shape_of(q) + ", (batch, h_q, " + std::to_string(c.d) + ") needed");
  const int batch = fits(q.size(0), "batch"), h_q = fits(q.size(1), "h_q");
  if (tables.dim() != 2 || tables.size(0) != batch)
    throw Refused("tables of shape " + shape_of(tables) + ", (" + std::to_string(batch) + ", b_max) needed");
  const int kmax = small(a[11], "kmax");
  shaped(idx, {batch, kmax}, "idx");
  const auto type = q.scalar_type();
  const int code = type_code(q);
  void* p_q = address(q, type, di, "q");
  const double scale = PyFloat_AsDouble(a[12]);
  if (scale == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refused("scale must be a number");
  }
  const int64_t wsb = p_attn_ws(batch, h_q, c.h_kv, c.d);
  if (wsb < 0) check(SW_ERR_INVALID_ARG, "sw_decode_attn_q8_workspace_bytes");
  at::Tensor O, ws;
  if (a[13] == Py_None) {
    O = at::empty_like(q);
  } else {
    O = tensor(a[13], "O");
    shaped(O, q.sizes(), "O");
  }
  if (a[14] != Py_None) ws = tensor(a[14], "workspace");
  if (wsb > 0 && (!ws.defined() || ws.numel() < wsb)) ws = at::empty({wsb}, q.options().dtype(at::kByte));
  check(p_attn(code, p_q, c.k, c.v, c.ks, c.vs, batch, h_q, c.h_kv, c.d, c.n_pages,
               static_cast<int32_t*>(address(tables, at::kInt, di, "tables")), b_max, c.B,
               ints(a[8], batch, di, "pos"), static_cast<int32_t*>(address(idx, at::kInt, di, "idx")),
               ints(a[10], batch, di, "cnt"), kmax, (float)scale, address(O, type, di, "O"),
               ws.defined() ? address(ws, at::kByte, di, "workspace") : nullptr, ws.defined() ? ws.numel() : 0,
               stream_of(a[1])),
        "sw_sparse_attn_decode_q8");
  return THPVariable_Wrap(O);
}

// Entry points by name -> address, and the exception that refusals raise.
PyObject* setup(PyObject* const* a, Py_ssize_t n_args) {
  count(n_args, 2);
  auto find = [&](const char* name) {
    PyObject* v = PyDict_GetItemString(a[1], name);
    if (v == nullptr) throw Refused(std::string("no entry point ") + name);
    return PyLong_AsVoidPtr(v);
  };
  Py_INCREF(a[0]);
  Py_XSETREF(g_error, a[0]);
  p_last_error = reinterpret_cast<decltype(p_last_error)>(find("sw_last_error"));
  p_block_tables = reinterpret_cast<decltype(p_block_tables)>(find("sw_block_tables"));
  p_block_tables_ws = reinterpret_cast<decltype(p_block_tables_ws)>(find("sw_block_tables_workspace_bytes"));
  p_append = reinterpret_cast<decltype(p_append)>(find("sw_kv_append_q8"));
  p_fetch = reinterpret_cast<decltype(p_fetch)>(find("sw_kv_fetch_q8"));
  p_attn = reinterpret_cast<decltype(p_attn)>(find("sw_sparse_attn_decode_q8"));
  p_attn_ws = reinterpret_cast<decltype(p_attn_ws)>(find("sw_decode_attn_q8_workspace_bytes"));
  Py_RETURN_NONE;
}

// A refusal raises SketchWalkError; other exceptions (memory) as torch raises them.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    return F(a, n);
  } catch (const Refused& e) {
    PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, e.what());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

#define SW_METHOD(F) {#F, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<F>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {SW_METHOD(setup), SW_METHOD(block_tables), SW_METHOD(kv_append_q8), SW_METHOD(kv_fetch_q8),
                           SW_METHOD(sparse_attn_decode_q8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_host_q8", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_q8(void) { return PyModule_Create(&g_module); }
