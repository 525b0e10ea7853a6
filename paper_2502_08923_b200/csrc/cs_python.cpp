// The short calls for Python, in native code: marshalling of cs_find_match, cs_qk_norm_rope, cs_paged_append and cs_paged_attention with
// their outputs made by the allocator directly.
//
// The search takes 2.3 to 5.1 us on the device, a call through ctypes 10.7: three tensors made from Python, eleven
// arguments converted, two tensors looked at, the launch.  Here 5.0 - 5.3 for one history of 4,097 tokens, and 5.3 - 5.5 for 64 of 32,768, where the
// device sets the pace.  The calls around the paged cache, whose smallest take 2.4 to 9 us on the device, through ctypes / here (a call among others, us): norms of
// 21 rows 23.8 / 5.6, an append of 11 rows 20.3 / 5.4, attention of the small model 12.7 / 8.3 (an elementwise call of torch takes 4.5).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "copyspec.h"

namespace {

// (what vmap and other transforms hand in looks like a tensor, but has no memory of its own)
bool plain(const at::Tensor& t, int64_t dim) {
  return t.has_storage() && t.is_cuda() && t.scalar_type() == at::kInt && t.layout() == at::kStrided && t.dim() == dim && t.is_contiguous();
}

// find_match(hist, hist_len, gamma, k, policy) -> (match_pos [B], draft [B][k], draft_len [B]), or the call's status where that
// is an error, or None where the arguments are not plain ones: the caller's general path takes those.
PyObject* find_match(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 5 || !THPVariable_CheckExact(args[0]) || !THPVariable_CheckExact(args[1]) || !PyLong_CheckExact(args[2]) ||
      !PyLong_CheckExact(args[3]) || !PyLong_CheckExact(args[4]) || c10::impl::TorchDispatchModeTLS::any_modes_set())
    Py_RETURN_NONE;
  const at::Tensor& hist = THPVariable_Unpack(args[0]);
  const at::Tensor& len = THPVariable_Unpack(args[1]);
  int overflow[3];
  const long gamma = PyLong_AsLongAndOverflow(args[2], &overflow[0]), k = PyLong_AsLongAndOverflow(args[3], &overflow[1]),
             policy = PyLong_AsLongAndOverflow(args[4], &overflow[2]);
  constexpr int64_t kMost = 1 << 30;
  if (overflow[0] || overflow[1] || overflow[2] || gamma < 0 || gamma > kMost || k < 0 || k > kMost || policy < 0 || policy > kMost ||
      !plain(hist, 2) || !plain(len, 1))
    Py_RETURN_NONE;
  const int64_t B = hist.size(0), stride = hist.size(1);
  if (B < 1 || B > kMost || stride > kMost || len.size(0) != B || len.device() != hist.device()) Py_RETURN_NONE;
  const at::Tensor pos = at::detail::empty_cuda({B}, at::kInt, hist.device(), std::nullopt);
  const at::Tensor draft = at::detail::empty_cuda({B, k}, at::kInt, hist.device(), std::nullopt);
  const at::Tensor draft_len = at::detail::empty_cuda({B}, at::kInt, hist.device(), std::nullopt);
  // (everything that may throw comes before the interpreter's lock is given up: the handler below needs it)
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  const int32_t* const h = static_cast<const int32_t*>(hist.const_data_ptr());
  const int32_t* const n = static_cast<const int32_t*>(len.const_data_ptr());
  int32_t* const out_pos = static_cast<int32_t*>(pos.mutable_data_ptr());
  int32_t* const out_draft = k > 0 ? static_cast<int32_t*>(draft.mutable_data_ptr()) : nullptr;
  int32_t* const out_len = static_cast<int32_t*>(draft_len.mutable_data_ptr());
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_find_match(h, n, (int)B, (int)stride, (int)gamma, (int)k, (cs_match_policy)policy, out_pos, out_draft, out_len, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  PyObject* out = PyTuple_New(3);
  if (out == nullptr) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(pos));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(draft));
  PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(draft_len));
  return out;
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ operators around the paged cache
// All of these return None where an argument is not a plain one (the caller's general path takes those and says what is wrong), the call's
// status as an int where that is an error, and otherwise the outputs.
bool tensor_of(PyObject* o, const at::Tensor*& t) {
  if (!THPVariable_CheckExact(o)) return false;
  t = &THPVariable_Unpack(o);
  return t->has_storage() && t->is_cuda() && t->layout() == at::kStrided && t->device().index() == c10::cuda::current_device() && !t->is_conj() && !t->is_neg();
}
bool optional_of(PyObject* o, const at::Tensor*& t) {
  t = nullptr;
  return o == Py_None || tensor_of(o, t);
}
int code_of(at::ScalarType s) { return s == at::kBFloat16 ? CS_BF16 : s == at::kHalf ? CS_F16 : s == at::kFloat ? CS_F32 : -1; }
at::ScalarType type_of(int code) { return code == CS_BF16 ? at::kBFloat16 : code == CS_F16 ? at::kHalf : at::kFloat; }
bool small_int(PyObject* o, long& v) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow;
  v = PyLong_AsLongAndOverflow(o, &overflow);
  return !overflow && v >= -(1l << 30) && v <= 1l << 30;
}
bool ints(PyObject* o, int64_t dim, int64_t n, const at::Tensor*& t) {
  return tensor_of(o, t) && plain(*t, dim) && (n < 0 || t->size(0) == n);
}
// [rows][heads][head_dim] with contiguous heads; sizes the calls' ints can hold
bool rows_of(const at::Tensor& t, cs_heads& h) {
  if (t.dim() != 3 || code_of(t.scalar_type()) < 0 || (t.size(2) > 1 && t.stride(2) != 1) || t.size(0) > (1 << 30) || t.size(1) > (1 << 20) || t.numel() == 0) return false;
  h.x = t.const_data_ptr();
  h.row_stride = t.size(0) > 1 ? t.stride(0) : 0;
  h.head_stride = t.size(1) > 1 ? t.stride(1) : 0;
  h.n_heads = (int32_t)t.size(1);
  return true;
}
bool gain_of(const at::Tensor* g, int64_t d, at::ScalarType type, cs_heads& h) {
  if (g == nullptr) return true;
  if (!g->is_contiguous() || g->scalar_type() != type || g->dim() != 1 || g->size(0) != d) return false;
  h.gain = g->const_data_ptr();
  return true;
}
bool table_of(const at::Tensor* rope, const float*& p, int& n, int& rot) {
  p = nullptr; n = rot = 0;
  if (rope == nullptr) return true;
  if (rope->dim() != 2 || !rope->is_contiguous() || rope->scalar_type() != at::kFloat || rope->size(0) > (1 << 30) || rope->size(1) > 4096) return false;
  p = static_cast<const float*>(rope->const_data_ptr());
  n = (int)rope->size(0); rot = (int)rope->size(1);
  return true;
}
// a new [rows][heads][head_dim] tensor, as h's destination
at::Tensor output_for(const at::Tensor& x, at::ScalarType type, cs_heads& h) {
  at::Tensor y = at::detail::empty_cuda(x.sizes(), type, x.device(), std::nullopt);
  h.y = y.mutable_data_ptr();
  h.y_row_stride = x.size(1) * x.size(2);
  h.y_head_stride = x.size(2);
  return y;
}
bool blocks_of(PyObject* const* args, int64_t rows, cs_blocks& b) {
  const at::Tensor *start, *len, *kv, *table;
  if (!ints(args[0], 1, -1, start) || !ints(args[1], 1, start->size(0), len) || !ints(args[2], 1, start->size(0), kv) || !ints(args[3], 2, start->size(0), table) ||
      start->size(0) > (1 << 30) || table->size(1) > (1 << 30))
    return false;
  auto at = [](const at::Tensor* t) { return static_cast<const int32_t*>(t->const_data_ptr()); };
  b = cs_blocks{at(start), at(len), at(kv), at(table), (int32_t)start->size(0), (int32_t)table->size(1), (int32_t)rows};
  return true;
}
PyObject* pair_of(const at::Tensor& x, const at::Tensor& y) {
  PyObject* out = PyTuple_New(2);
  if (out == nullptr) return nullptr;
  PyTuple_SET_ITEM(out, 0, x.defined() ? THPVariable_Wrap(x) : Py_NewRef(Py_None));
  PyTuple_SET_ITEM(out, 1, y.defined() ? THPVariable_Wrap(y) : Py_NewRef(Py_None));
  return out;
}

// qk_norm_rope(q, k, pos, rope, q_gain, k_gain, eps, dtype code) -> (q, k)
PyObject* qk_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor *q, *k, *pos, *rope, *qg, *kg;
  long code;
  if (n_args != 8 || c10::impl::TorchDispatchModeTLS::any_modes_set() || !optional_of(args[0], q) || !optional_of(args[1], k) || !optional_of(args[2], pos) ||
      !optional_of(args[3], rope) || !optional_of(args[4], qg) || !optional_of(args[5], kg) || !PyFloat_CheckExact(args[6]) || !small_int(args[7], code) || (q == nullptr && k == nullptr) ||
      code < 0 || code > 2)
    Py_RETURN_NONE;
  const at::Tensor& some = q != nullptr ? *q : *k;
  cs_heads hq = {}, hk = {};
  const float* table;
  int n, rot;
  const at::ScalarType type = type_of((int)code);
  if ((q != nullptr && (!rows_of(*q, hq) || !gain_of(qg, q->size(2), type, hq))) || (k != nullptr && (!rows_of(*k, hk) || !gain_of(kg, k->size(2), type, hk))) || !table_of(rope, table, n, rot) ||
      (q != nullptr && k != nullptr && (q->scalar_type() != k->scalar_type() || q->size(0) != k->size(0) || q->size(2) != k->size(2))) ||
      (rope != nullptr && (pos == nullptr || !plain(*pos, 1) || pos->size(0) != some.size(0))))
    Py_RETURN_NONE;
  const at::Tensor yq = q != nullptr ? output_for(*q, type, hq) : at::Tensor(), yk = k != nullptr ? output_for(*k, type, hk) : at::Tensor();
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  const int32_t* const p = rope != nullptr ? static_cast<const int32_t*>(pos->const_data_ptr()) : nullptr;
  const float eps = (float)PyFloat_AS_DOUBLE(args[6]);
  const int rows = (int)some.size(0), dim = (int)some.size(2), in = code_of(some.scalar_type());
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_qk_norm_rope(&hq, &hk, rows, dim, (cs_dtype)in, (cs_dtype)code, p, table, n, rot, eps, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  return pair_of(yq, yk);
  END_HANDLE_TH_ERRORS
}

// the handle of a cache on the current device (the other tensors are), nullptr if it is not one
cs_paged_cache* cache_of(PyObject* handle, PyObject* device, int64_t head_dim) {
  long d;
  if (!PyLong_CheckExact(handle) || !small_int(device, d) || d != c10::cuda::current_device()) return nullptr;
  cs_paged_cache* const cache = static_cast<cs_paged_cache*>(PyLong_AsVoidPtr(handle));
  return cache != nullptr && cs_paged_head_dim(cache) == (int)head_dim ? cache : nullptr;
}

// paged_append(handle, dtype code, device, k, v, block_start, block_len, kv_len, page_table, rope, k_gain, q, q_gain, eps) -> (q,)
PyObject* paged_append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor *q, *k, *v, *rope, *qg, *kg;
  long code;
  if (n_args != 14 || c10::impl::TorchDispatchModeTLS::any_modes_set() || !small_int(args[1], code) || !tensor_of(args[3], k) || !tensor_of(args[4], v) ||
      !optional_of(args[9], rope) || !optional_of(args[10], kg) || !optional_of(args[11], q) || !optional_of(args[12], qg) || !PyFloat_CheckExact(args[13]))
    Py_RETURN_NONE;
  cs_heads hq = {}, hk = {}, hv = {};
  cs_blocks blocks;
  const float* table;
  int n, rot;
  const at::ScalarType type = type_of((int)code);
  if (!rows_of(*k, hk) || !rows_of(*v, hv) || k->scalar_type() != v->scalar_type() || k->sizes() != v->sizes() || !gain_of(kg, k->size(2), type, hk) || !table_of(rope, table, n, rot) ||
      !blocks_of(args + 5, k->size(0), blocks) ||
      (q != nullptr && (!rows_of(*q, hq) || q->scalar_type() != k->scalar_type() || q->size(0) != k->size(0) || q->size(2) != k->size(2) || !gain_of(qg, k->size(2), type, hq))))
    Py_RETURN_NONE;
  cs_paged_cache* const cache = cache_of(args[0], args[2], k->size(2));
  if (cache == nullptr) Py_RETURN_NONE;
  const at::Tensor yq = q != nullptr ? output_for(*q, type, hq) : at::Tensor();
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  const float eps = (float)PyFloat_AS_DOUBLE(args[13]);
  const int in = code_of(k->scalar_type());
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_paged_append(cache, &blocks, &hk, &hv, &hq, (cs_dtype)in, table, n, rot, eps, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  PyObject* out = PyTuple_New(1);
  if (out == nullptr) return nullptr;
  PyTuple_SET_ITEM(out, 0, yq.defined() ? THPVariable_Wrap(yq) : Py_NewRef(Py_None));
  return out;
  END_HANDLE_TH_ERRORS
}

// paged_attention(handle, dtype code, device, q, block_start, block_len, kv_len, page_table, mask, window, scale, with_lse) -> (out, lse or None)
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor* q;
  long code, mask, window;
  if (n_args != 12 || c10::impl::TorchDispatchModeTLS::any_modes_set() || !small_int(args[1], code) || !tensor_of(args[3], q) || !small_int(args[8], mask) ||
      !small_int(args[9], window) || !PyFloat_CheckExact(args[10]) || !PyBool_Check(args[11]))
    Py_RETURN_NONE;
  cs_heads hq = {};
  cs_blocks blocks;
  if (!rows_of(*q, hq) || code_of(q->scalar_type()) != code || !blocks_of(args + 4, q->size(0), blocks)) Py_RETURN_NONE;
  cs_paged_cache* const cache = cache_of(args[0], args[2], q->size(2));
  if (cache == nullptr) Py_RETURN_NONE;
  const bool with_lse = args[11] == Py_True;
  const at::Tensor out = output_for(*q, q->scalar_type(), hq);
  const at::Tensor lse = with_lse ? at::detail::empty_cuda({q->size(0), q->size(1)}, at::kFloat, q->device(), std::nullopt) : at::Tensor();
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  float* const lse_p = with_lse ? static_cast<float*>(lse.mutable_data_ptr()) : nullptr;
  const float scale = (float)PyFloat_AS_DOUBLE(args[10]);
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_paged_attention(cache, &blocks, hq.x, hq.row_stride, hq.head_stride, hq.n_heads, (cs_mask)mask, (int)window, scale, hq.y, lse_p, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  return pair_of(out, lse);
  END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ and around the cache held in 4 bits
cs_quant_cache* quant_of(PyObject* handle, PyObject* device, int64_t head_dim) {
  long d;
  if (!PyLong_CheckExact(handle) || !small_int(device, d) || d != c10::cuda::current_device()) return nullptr;
  cs_quant_cache* const cache = static_cast<cs_quant_cache*>(PyLong_AsVoidPtr(handle));
  return cache != nullptr && cs_quant_head_dim(cache) == (int)head_dim ? cache : nullptr;
}

// quant_append(handle, device, k, v, block_start, block_len, kv_len, page_table, rope, k_gain, q, q_gain, eps, dtype code) -> (q,)
PyObject* quant_append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor *q, *k, *v, *rope, *qg, *kg;
  long code;
  if (n_args != 14 || c10::impl::TorchDispatchModeTLS::any_modes_set() || !tensor_of(args[2], k) || !tensor_of(args[3], v) || !optional_of(args[8], rope) || !optional_of(args[9], kg) ||
      !optional_of(args[10], q) || !optional_of(args[11], qg) || !PyFloat_CheckExact(args[12]) || !small_int(args[13], code) || (code != CS_BF16 && code != CS_F16))
    Py_RETURN_NONE;
  cs_heads hq = {}, hk = {}, hv = {};
  cs_blocks blocks;
  const float* table;
  int n, rot;
  const at::ScalarType type = type_of((int)code);
  if (!rows_of(*k, hk) || !rows_of(*v, hv) || k->scalar_type() != v->scalar_type() || k->sizes() != v->sizes() || !gain_of(kg, k->size(2), type, hk) || !table_of(rope, table, n, rot) ||
      !blocks_of(args + 4, k->size(0), blocks) ||
      (q != nullptr && (!rows_of(*q, hq) || q->scalar_type() != k->scalar_type() || q->size(0) != k->size(0) || q->size(2) != k->size(2) || !gain_of(qg, k->size(2), type, hq))))
    Py_RETURN_NONE;
  cs_quant_cache* const cache = quant_of(args[0], args[1], k->size(2));
  if (cache == nullptr) Py_RETURN_NONE;
  const at::Tensor yq = q != nullptr ? output_for(*q, type, hq) : at::Tensor();
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  const float eps = (float)PyFloat_AS_DOUBLE(args[12]);
  const int in = code_of(k->scalar_type());
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_quant_append(cache, &blocks, &hk, &hv, &hq, (cs_dtype)in, (cs_dtype)code, table, n, rot, eps, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  PyObject* out = PyTuple_New(1);
  if (out == nullptr) return nullptr;
  PyTuple_SET_ITEM(out, 0, yq.defined() ? THPVariable_Wrap(yq) : Py_NewRef(Py_None));
  return out;
  END_HANDLE_TH_ERRORS
}

// quant_read(handle, device, KV heads, head_dim, block_start, block_len, kv_len, page_table, rows, dtype code) -> (keys, values)
PyObject* quant_read(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  long heads, dim, rows, code;
  cs_blocks blocks;
  if (n_args != 10 || c10::impl::TorchDispatchModeTLS::any_modes_set() || !small_int(args[2], heads) || !small_int(args[3], dim) || !small_int(args[8], rows) || !small_int(args[9], code) ||
      rows < 1 || heads < 1 || code < 0 || code > 2 || !blocks_of(args + 4, rows, blocks))
    Py_RETURN_NONE;
  cs_quant_cache* const cache = quant_of(args[0], args[1], dim);
  if (cache == nullptr) Py_RETURN_NONE;
  const at::Device device = THPVariable_Unpack(args[4]).device();
  const at::Tensor k = at::detail::empty_cuda({rows, heads, dim}, type_of((int)code), device, std::nullopt), v = at::detail::empty_cuda({rows, heads, dim}, type_of((int)code), device, std::nullopt);
  cs_heads hk = {}, hv = {};
  hk.y = k.mutable_data_ptr(); hv.y = v.mutable_data_ptr();
  hk.y_row_stride = hv.y_row_stride = heads * dim;
  hk.y_head_stride = hv.y_head_stride = dim;
  hk.n_heads = hv.n_heads = (int32_t)heads;
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_quant_read(cache, &blocks, &hk, &hv, (cs_dtype)code, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  return pair_of(k, v);
  END_HANDLE_TH_ERRORS
}

// quant_attention(handle, device, q, block_start, block_len, kv_len, page_table, mask, window, scale, with_lse) -> (out, lse or None)
PyObject* quant_attention(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const at::Tensor* q;
  long mask, window;
  if (n_args != 11 || c10::impl::TorchDispatchModeTLS::any_modes_set() || !tensor_of(args[2], q) || !small_int(args[7], mask) || !small_int(args[8], window) || !PyFloat_CheckExact(args[9]) ||
      !PyBool_Check(args[10]))
    Py_RETURN_NONE;
  cs_heads hq = {};
  cs_blocks blocks;
  if (!rows_of(*q, hq) || q->scalar_type() == at::kFloat || !blocks_of(args + 3, q->size(0), blocks)) Py_RETURN_NONE;
  cs_quant_cache* const cache = quant_of(args[0], args[1], q->size(2));
  if (cache == nullptr) Py_RETURN_NONE;
  const bool with_lse = args[10] == Py_True;
  const at::Tensor out = output_for(*q, q->scalar_type(), hq);
  const at::Tensor lse = with_lse ? at::detail::empty_cuda({q->size(0), q->size(1)}, at::kFloat, q->device(), std::nullopt) : at::Tensor();
  void* const stream = c10::cuda::getCurrentCUDAStream().stream();
  float* const lse_p = with_lse ? static_cast<float*>(lse.mutable_data_ptr()) : nullptr;
  const float scale = (float)PyFloat_AS_DOUBLE(args[9]);
  const int type = code_of(q->scalar_type());
  cs_status s;
  Py_BEGIN_ALLOW_THREADS
  s = cs_quant_attention(cache, &blocks, hq.x, hq.row_stride, hq.head_stride, hq.n_heads, (cs_dtype)type, (cs_mask)mask, (int)window, scale, hq.y, lse_p, stream);
  Py_END_ALLOW_THREADS
  if (s != CS_OK) return PyLong_FromLong(s);
  return pair_of(out, lse);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"find_match", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(find_match)), METH_FASTCALL, nullptr},
                         {"qk_norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(qk_norm_rope)), METH_FASTCALL, nullptr},
                         {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(paged_append)), METH_FASTCALL, nullptr},
                         {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(paged_attention)), METH_FASTCALL, nullptr},
                         {"quant_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quant_append)), METH_FASTCALL, nullptr},
                         {"quant_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quant_read)), METH_FASTCALL, nullptr},
                         {"quant_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quant_attention)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
