// Marshalling of the attention calls (fikit_cache_*, fikit_prompt_attention) for Python, compiled: checks of tensors, output
// tensors, and the C calls, whose addresses binding.py passes in.  A call on the GPU may take 4 us; the same checks and
// allocations as Python statements take 9.
//
// Every function takes its arguments by place, returns the outputs, or the status if the C call refused, and raises ValueError
// for what a pointer cannot describe.
#include <torch/csrc/python_headers.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/python_numbers.h>

#include "fikit.h"

namespace {

decltype(&fikit_cache_pieces) cache_pieces;
decltype(&fikit_cache_plan_workspace_bytes) cache_plan_workspace_bytes;
decltype(&fikit_cache_plan) cache_plan;
decltype(&fikit_cache_append) cache_append;
decltype(&fikit_cache_attention_workspace_bytes) cache_attention_workspace_bytes;
decltype(&fikit_cache_attention) cache_attention;
decltype(&fikit_prompt_attention) prompt_attention;

const at::Tensor& tensor(PyObject* o, const char* what) {
  TORCH_CHECK_VALUE(THPVariable_Check(o), what, ": a tensor");
  return THPVariable_Unpack(o);
}

// The address of a dense tensor of a type and device.
template <typename T>
T* dense(const at::Tensor& t, at::ScalarType type, const at::Device& device, const char* what) {
  TORCH_CHECK_VALUE(t.scalar_type() == type && t.device() == device && t.is_contiguous(), what, ": a dense ", type, " tensor on ", device);
  return static_cast<T*>(t.data_ptr());
}

uint32_t count(int64_t n, const char* what) {
  TORCH_CHECK_VALUE(n >= 0 && n <= UINT32_MAX, what, ": from 0 to 2^32 - 1");
  return static_cast<uint32_t>(n);
}
uint32_t count(PyObject* o, const char* what) { return count(THPUtils_unpackLong(o), what); }

bool truth(PyObject* o) {
  const int is = PyObject_IsTrue(o);
  if (is < 0) throw python_error();
  return is;
}

int32_t value_type(const at::Tensor& t, const char* what) {
  TORCH_CHECK_VALUE(t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf, what, ": bfloat16 or float16");
  return t.scalar_type() == at::kBFloat16 ? FIKIT_BF16 : FIKIT_F16;
}

// [tokens, heads, head_dim] with the last dimension dense.  (For inference only: an output that silently had no gradient would be wrong.)
fikit_vectors vectors(const at::Tensor& t, at::ScalarType type, const at::Device& device, const char* what) {
  TORCH_CHECK_VALUE(t.dim() == 3 && (t.stride(2) == 1 || t.size(2) <= 1) && t.stride(0) >= 0 && t.stride(1) >= 0 && t.scalar_type() == type &&
                        t.device() == device,
                    what, ": [tokens, heads, head_dim] ", type, " on ", device, ", the last dimension dense");
  TORCH_CHECK_VALUE(!(t.requires_grad() && at::GradMode::is_enabled()), what, ": requires a gradient, and there is no backward pass; detach it or use no_grad()");
  // (the stride of a dimension of size one may be anything, and is not used)
  return fikit_vectors{t.data_ptr(), t.size(0) > 1 ? static_cast<uint64_t>(t.stride(0)) : 0, t.size(1) > 1 ? static_cast<uint64_t>(t.stride(1)) : 0};
}

fikit_cache cache_of(PyObject* const* a, const at::Device& device) {
  const at::Tensor &k = tensor(a[0], "k_cache"), &v = tensor(a[1], "v_cache"), &k_exp = tensor(a[2], "k_exp"), &v_exp = tensor(a[3], "v_exp");
  TORCH_CHECK_VALUE(k.dim() == 4 && v.sizes() == k.sizes(), "k_cache, v_cache: [blocks, kv heads, block tokens, head_dim]");
  TORCH_CHECK_VALUE(k.scalar_type() == at::kFloat8_e4m3fn || k.scalar_type() == at::kByte, "k_cache, v_cache: float8_e4m3fn or uint8");
  TORCH_CHECK_VALUE(k_exp.dim() == 2 && k_exp.size(0) == k.size(0) && k_exp.size(1) == k.size(1) && v_exp.sizes() == k_exp.sizes(),
                    "k_exp, v_exp: [blocks, kv heads]");
  return fikit_cache{dense<uint8_t>(k, k.scalar_type(), device, "k_cache"), dense<uint8_t>(v, k.scalar_type(), device, "v_cache"),
                     dense<uint8_t>(k_exp, at::kByte, device, "k_exp"), dense<uint8_t>(v_exp, at::kByte, device, "v_exp"),
                     count(k.size(0), "blocks"), count(k.size(1), "kv heads"), count(k.size(2), "block tokens"), count(k.size(3), "head_dim")};
}

// Other Python threads run while this lives: an allocation may wait for memory, and a launch for room in a queue.  What is taken from
// Python objects is taken before.
class Unlocked {
  PyThreadState* state = PyEval_SaveThread();

 public:
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// A tensor, or one that is not defined.
at::Tensor given_or_none(PyObject* o, const char* what) { return o == Py_None ? at::Tensor() : tensor(o, what); }

at::Tensor workspace_of(const at::Tensor& given, size_t bytes, const at::Device& device) {
  if (given.defined()) {
    dense<uint8_t>(given, at::kByte, device, "workspace_buf");
    return given;
  }
  return bytes ? at::empty({static_cast<int64_t>(bytes < 256 ? 256 : bytes)}, at::TensorOptions().dtype(at::kByte).device(device)) : at::Tensor();
}

void* stream_of(PyObject* o) { return reinterpret_cast<void*>(THPUtils_unpackLong(o)); }

// A tensor in the memory of another one, from place `from` (in its own type) on.
at::Tensor part_of(const at::Tensor& all, at::ScalarType type, int64_t from, at::IntArrayRef sizes) {
  at::Tensor t = at::detail::make_tensor<at::TensorImpl>(at::TensorImpl::VIEW, at::Storage(all.storage()), all.key_set(), at::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
  t.unsafeGetTensorImpl()->set_storage_offset(from);
  return t;
}

PyObject* wrapped(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}

void need_arguments(Py_ssize_t n, Py_ssize_t want) { TORCH_CHECK_VALUE(n == want, "takes ", want, " arguments"); }

// cached, added, n_tokens, block_tokens, block_table, free_blocks, status, want_slots, out, workspace_buf, stream
PyObject* py_cache_plan(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 11);
  const at::Tensor &cached = tensor(a[0], "cached"), &added = tensor(a[1], "added"), &table = tensor(a[4], "block_table"), &free = tensor(a[5], "free_blocks"),
                   &status = tensor(a[6], "status");
  const at::Device device = cached.device();
  const uint32_t n = count(cached.numel(), "cached"), n_tokens = count(a[2], "n_tokens"), block_tokens = count(a[3], "block_tokens");
  TORCH_CHECK_VALUE(added.numel() == n && table.dim() == 2 && table.size(0) == n, "cached, added: [R]; block_table: [R, width]");
  TORCH_CHECK_VALUE(status.numel() == 1, "status: [1]");
  const bool want_slots = truth(a[7]);
  const int64_t room = static_cast<int64_t>(cache_pieces(n_tokens, n, block_tokens));
  at::Tensor lengths, offsets, slots, pieces, counts;
  const bool allocate = a[8] == Py_None;
  if (!allocate) {
    TORCH_CHECK_VALUE(PyTuple_Check(a[8]) && PyTuple_GET_SIZE(a[8]) == 5, "out: a CachePlan");
    lengths = tensor(PyTuple_GET_ITEM(a[8], 0), "lengths");
    offsets = tensor(PyTuple_GET_ITEM(a[8], 1), "token_offsets");
    slots = given_or_none(PyTuple_GET_ITEM(a[8], 2), "slots");
    pieces = tensor(PyTuple_GET_ITEM(a[8], 3), "pieces");
    counts = tensor(PyTuple_GET_ITEM(a[8], 4), "counts");
    TORCH_CHECK_VALUE(lengths.numel() == n && offsets.numel() == static_cast<int64_t>(n) + 1 && counts.numel() == 2 && pieces.numel() == 4 * room &&
                          (!slots.defined() || slots.numel() == n_tokens),
                      "out: tensors of the plan's sizes");
  }
  const at::Tensor workspace = given_or_none(a[9], "workspace_buf");
  void* const stream = stream_of(a[10]);
  int rc;
  {
    const Unlocked unlocked;
    if (allocate) {
      // one allocation: slots (two words each), pieces, lengths, places, counts
      const int64_t of_pieces = want_slots ? (2 * static_cast<int64_t>(n_tokens) + 3) / 4 * 4 : 0, of_lengths = of_pieces + 4 * room;
      const at::Tensor all = at::empty({of_lengths + 2 * static_cast<int64_t>(n) + 3}, at::TensorOptions().dtype(at::kInt).device(device));
      if (want_slots) slots = part_of(all, at::kLong, 0, {n_tokens});
      pieces = part_of(all, at::kInt, of_pieces, {room, 4});
      lengths = part_of(all, at::kInt, of_lengths, {n});
      offsets = part_of(all, at::kInt, of_lengths + n, {static_cast<int64_t>(n) + 1});
      counts = part_of(all, at::kInt, of_lengths + 2 * static_cast<int64_t>(n) + 1, {2});
    }
    const at::Tensor ws = workspace_of(workspace, cache_plan_workspace_bytes(n), device);
    rc = cache_plan(dense<int32_t>(cached, at::kInt, device, "cached"), dense<int32_t>(added, at::kInt, device, "added"), n, n_tokens, block_tokens,
                    dense<int32_t>(table, at::kInt, device, "block_table"), count(table.size(1), "block_table"),
                    dense<int32_t>(free, at::kInt, device, "free_blocks"), count(free.numel(), "free_blocks"),
                    dense<int32_t>(lengths, at::kInt, device, "lengths"), dense<int32_t>(offsets, at::kInt, device, "token_offsets"),
                    slots.defined() ? dense<int64_t>(slots, at::kLong, device, "slots") : nullptr,
                    dense<fikit_piece>(pieces, at::kInt, device, "pieces"), dense<int32_t>(counts, at::kInt, device, "counts"),
                    dense<int32_t>(status, at::kInt, device, "status"), ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0,
                    stream);
  }
  if (rc != FIKIT_OK) return PyLong_FromLong(rc);
  if (!allocate) {
    Py_INCREF(a[8]);
    return a[8];
  }
  return Py_BuildValue("(NNNNN)", wrapped(lengths), wrapped(offsets), wrapped(slots), wrapped(pieces), wrapped(counts));
  END_HANDLE_TH_ERRORS
}

// k_cache, v_cache, k_exp, v_exp, k, v, pieces, status, stream
PyObject* py_cache_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 9);
  const at::Tensor &k = tensor(a[4], "k"), &v = tensor(a[5], "v"), &pieces = tensor(a[6], "pieces"), &status = tensor(a[7], "status");
  const at::Device device = k.device();
  const fikit_cache cache = cache_of(a, device);
  const int32_t type = value_type(k, "k");
  const fikit_vectors kv = vectors(k, k.scalar_type(), device, "k"), vv = vectors(v, k.scalar_type(), device, "v");
  TORCH_CHECK_VALUE(k.sizes() == v.sizes() && k.size(1) == cache.kv_heads && k.size(2) == cache.head_dim, "k, v: [n_tokens, kv heads, head_dim] of the cache");
  TORCH_CHECK_VALUE(pieces.dim() == 2 && pieces.size(1) == 4 && status.numel() == 1, "pieces: [n, 4]; status: [1]");
  void* const stream = stream_of(a[8]);
  int rc;
  {
    const Unlocked unlocked;
    rc = cache_append(&cache, &kv, &vv, count(k.size(0), "tokens"), type, dense<fikit_piece>(pieces, at::kInt, device, "pieces"),
                      static_cast<uint64_t>(pieces.size(0)), dense<int32_t>(status, at::kInt, device, "status"), stream);
  }
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// The outputs of an attention call that are given.
void given_out(const at::Tensor& q, PyObject* given, at::Tensor* out, at::Tensor* lse) {
  if (given == Py_None) return;
  TORCH_CHECK_VALUE(PyTuple_Check(given) && PyTuple_GET_SIZE(given) == 2, "out: an Attention");
  *out = tensor(PyTuple_GET_ITEM(given, 0), "out");
  *lse = given_or_none(PyTuple_GET_ITEM(given, 1), "lse");
  TORCH_CHECK_VALUE(out->sizes() == q.sizes(), "out: the shape of q");
  TORCH_CHECK_VALUE(!lse->defined() || (lse->dim() == 2 && lse->size(0) == q.size(0) && lse->size(1) == q.size(1)), "lse: [rows, q heads]");
}

// New ones, if none are.
void new_out(const at::Tensor& q, bool want_lse, at::Tensor* out, at::Tensor* lse) {
  if (out->defined()) return;
  *out = at::empty(q.sizes(), at::TensorOptions().dtype(q.scalar_type()).device(q.device()));
  if (want_lse) *lse = at::empty({q.size(0), q.size(1)}, at::TensorOptions().dtype(at::kFloat).device(q.device()));
}

PyObject* attention_result(int rc, PyObject* given, const at::Tensor& out, const at::Tensor& lse) {
  if (rc != FIKIT_OK) return PyLong_FromLong(rc);
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return Py_BuildValue("(NN)", wrapped(out), wrapped(lse));
}

// k_cache, v_cache, k_exp, v_exp, q, block_table, lengths, scale, status, max_length or None, want_lse, out, workspace_buf, stream
PyObject* py_cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 14);
  const at::Tensor &q = tensor(a[4], "q"), &table = tensor(a[5], "block_table"), &lengths = tensor(a[6], "lengths"), &status = tensor(a[8], "status");
  const at::Device device = q.device();
  const fikit_cache cache = cache_of(a, device);
  const int32_t type = value_type(q, "q");
  const fikit_vectors qv = vectors(q, q.scalar_type(), device, "q");
  const uint32_t n = count(q.size(0), "requests"), heads = count(q.size(1), "q heads");
  TORCH_CHECK_VALUE(q.size(2) == cache.head_dim && table.dim() == 2 && table.size(0) == n && lengths.numel() == n && status.numel() == 1,
                    "q: [R, q heads, head_dim]; block_table: [R, width]; lengths: [R]; status: [1]");
  const uint32_t width = count(table.size(1), "block_table");
  const uint32_t longest = a[9] == Py_None ? count(static_cast<int64_t>(width) * cache.block_tokens, "max_length") : count(a[9], "max_length");
  at::Tensor out, lse;
  given_out(q, a[11], &out, &lse);
  const bool want_lse = truth(a[10]);
  const float scale = static_cast<float>(THPUtils_unpackDouble(a[7]));
  const at::Tensor workspace = given_or_none(a[12], "workspace_buf");
  void* const stream = stream_of(a[13]);
  int rc;
  {
    const Unlocked unlocked;
    new_out(q, want_lse, &out, &lse);
    const at::Tensor ws = workspace_of(workspace, cache_attention_workspace_bytes(n, heads, cache.kv_heads, cache.head_dim, longest), device);
    rc = cache_attention(&cache, &qv, heads, type, scale, dense<int32_t>(table, at::kInt, device, "block_table"), width,
                         dense<int32_t>(lengths, at::kInt, device, "lengths"), n, longest, dense<void>(out, q.scalar_type(), device, "out"),
                         lse.defined() ? dense<float>(lse, at::kFloat, device, "lse") : nullptr, dense<int32_t>(status, at::kInt, device, "status"),
                         ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, stream);
  }
  return attention_result(rc, a[11], out, lse);
  END_HANDLE_TH_ERRORS
}

// q, k, v, offsets, scale, status, want_lse, out, stream
PyObject* py_prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 9);
  const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &offsets = tensor(a[3], "offsets"), &status = tensor(a[5], "status");
  const at::Device device = q.device();
  const int32_t type = value_type(q, "q");
  const fikit_vectors qv = vectors(q, q.scalar_type(), device, "q"), kv = vectors(k, q.scalar_type(), device, "k"), vv = vectors(v, q.scalar_type(), device, "v");
  TORCH_CHECK_VALUE(k.sizes() == v.sizes() && k.size(0) == q.size(0) && k.size(2) == q.size(2), "k, v: [n_tokens, kv heads, head_dim]");
  TORCH_CHECK_VALUE(offsets.numel() >= 1 && status.numel() == 1, "offsets: [prompts + 1]; status: [1]");
  at::Tensor out, lse;
  given_out(q, a[7], &out, &lse);
  const bool want_lse = truth(a[6]);
  const float scale = static_cast<float>(THPUtils_unpackDouble(a[4]));
  void* const stream = stream_of(a[8]);
  int rc;
  {
    const Unlocked unlocked;
    new_out(q, want_lse, &out, &lse);
    rc = prompt_attention(&qv, &kv, &vv, count(q.size(1), "q heads"), count(k.size(1), "kv heads"), count(q.size(2), "head_dim"), type, scale,
                          dense<int32_t>(offsets, at::kInt, device, "offsets"), count(offsets.numel() - 1, "offsets"), count(q.size(0), "tokens"),
                          dense<void>(out, q.scalar_type(), device, "out"), lse.defined() ? dense<float>(lse, at::kFloat, device, "lse") : nullptr,
                          dense<int32_t>(status, at::kInt, device, "status"), stream);
  }
  return attention_result(rc, a[7], out, lse);
  END_HANDLE_TH_ERRORS
}

// The addresses of the C calls, in the order of the variables above.
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 7);
  const auto set = [&](auto& f, int i) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(PyLong_AsVoidPtr(a[i])); };
  set(cache_pieces, 0);
  set(cache_plan_workspace_bytes, 1);
  set(cache_plan, 2);
  set(cache_append, 3);
  set(cache_attention_workspace_bytes, 4);
  set(cache_attention, 5);
  set(prompt_attention, 6);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(cache_plan), METHOD(cache_append), METHOD(cache_attention), METHOD(prompt_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serve_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serve_marshal() { return PyModule_Create(&module); }
