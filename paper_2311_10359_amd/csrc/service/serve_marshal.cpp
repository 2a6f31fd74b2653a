// Marshalling of the calls of a language model service (fikit_cache_*, fikit_prompt_attention, fikit_rotate_heads,
// fikit_token_scores) for Python, compiled: checks of tensors, output
// tensors, and the C calls, whose addresses binding.py passes in.  A call on the GPU may take 4 us; the same checks and
// allocations as Python statements take 9.
//
// Every function takes its arguments by place, returns the outputs, or the status if the C call refused, and raises ValueError
// for what a pointer cannot describe.
#include <torch/csrc/python_headers.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/AutogradState.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/python_numbers.h>

#include <initializer_list>
#include <vector>

#include "fikit.h"

namespace {

decltype(&fikit_cache_pieces) cache_pieces;
decltype(&fikit_cache_plan_workspace_bytes) cache_plan_workspace_bytes;
decltype(&fikit_cache_plan) cache_plan;
decltype(&fikit_cache_append) cache_append;
decltype(&fikit_cache_attention_workspace_bytes) cache_attention_workspace_bytes;
decltype(&fikit_cache_attention) cache_attention;
decltype(&fikit_prompt_attention) prompt_attention;
decltype(&fikit_rotate_heads) rotate_heads;
decltype(&fikit_cache_fork_workspace_bytes) cache_fork_workspace_bytes;
decltype(&fikit_cache_fork) cache_fork;
decltype(&fikit_cache_compact_workspace_bytes) cache_compact_workspace_bytes;
decltype(&fikit_cache_compact) cache_compact;
decltype(&fikit_cache_copy) cache_copy;
decltype(&fikit_token_scores_workspace_bytes) token_scores_workspace_bytes;
decltype(&fikit_token_scores) token_scores;

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

// (For inference only: an output that silently had no gradient, or no tangent in forward mode, would be wrong.)
void without_gradient(const at::Tensor& t, const char* what) {
  TORCH_CHECK_VALUE(!(t.requires_grad() && at::GradMode::is_enabled()), what, ": requires a gradient, and there is no backward pass; detach it or use no_grad()");
  TORCH_CHECK_VALUE(!(t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode()), what,
                    ": has a tangent, and there is no forward mode; unpack it");
}

// [tokens, heads, head_dim] with the last dimension dense.
fikit_vectors vectors(const at::Tensor& t, at::ScalarType type, const at::Device& device, const char* what) {
  TORCH_CHECK_VALUE(t.dim() == 3 && (t.stride(2) == 1 || t.size(2) <= 1) && t.stride(0) >= 0 && t.stride(1) >= 0 && t.scalar_type() == type &&
                        t.device() == device,
                    what, ": [tokens, heads, head_dim] ", type, " on ", device, ", the last dimension dense");
  without_gradient(t, what);
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

// What a call has written in place: autograd, if it has saved one of these tensors, has to know.  (An inference tensor has no version; the status word and
// the workspace are the calls' own.)
void written(int rc, std::initializer_list<const at::Tensor*> tensors) {
  if (rc != FIKIT_OK && rc != FIKIT_HIP_ERROR) return;         // refused
  for (const at::Tensor* t : tensors)
    if (t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
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
  written(rc, {&table});
  if (!allocate) written(rc, {&lengths, &offsets, &slots, &pieces, &counts});
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
  for (int i = 0; i < 4; ++i) written(rc, {&THPVariable_Unpack(a[i])});
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
  without_gradient(*out, "out");
  TORCH_CHECK_VALUE(!lse->defined() || (lse->dim() == 2 && lse->size(0) == q.size(0) && lse->size(1) == q.size(1)), "lse: [rows, q heads]");
  if (lse->defined()) without_gradient(*lse, "lse");
}

// New ones, if none are.
void new_out(const at::Tensor& q, bool want_lse, at::Tensor* out, at::Tensor* lse) {
  if (out->defined()) return;
  *out = at::empty(q.sizes(), at::TensorOptions().dtype(q.scalar_type()).device(q.device()));
  if (want_lse) *lse = at::empty({q.size(0), q.size(1)}, at::TensorOptions().dtype(at::kFloat).device(q.device()));
}

PyObject* attention_result(int rc, PyObject* given, const at::Tensor& out, const at::Tensor& lse) {
  if (given != Py_None) written(rc, {&out, &lse});
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

// q or None, k or None, positions, frequencies or None, status, q_weight or None, k_weight or None, epsilon, neighbours, out, stream
PyObject* py_rotate_heads(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 11);
  const at::Tensor q = given_or_none(a[0], "q"), k = given_or_none(a[1], "k");
  TORCH_CHECK_VALUE(q.defined() || k.defined(), "q or k: a tensor");
  const at::Tensor &any = q.defined() ? q : k, &positions = tensor(a[2], "positions"), frequencies = given_or_none(a[3], "frequencies"),
                   &status = tensor(a[4], "status"), q_weight = given_or_none(a[5], "q_weight"), k_weight = given_or_none(a[6], "k_weight");
  const at::Device device = any.device();
  const at::ScalarType type = any.scalar_type();
  const int32_t of_values = value_type(any, "q, k");
  const float epsilon = static_cast<float>(THPUtils_unpackDouble(a[7]));
  const bool neighbours = truth(a[8]);
  void* const stream = stream_of(a[10]);
  at::Tensor q_out, k_out;
  if (a[9] != Py_None) {
    TORCH_CHECK_VALUE(PyTuple_Check(a[9]) && PyTuple_GET_SIZE(a[9]) == 2, "out: a RotatedHeads");
    q_out = given_or_none(PyTuple_GET_ITEM(a[9], 0), "out.q");
    k_out = given_or_none(PyTuple_GET_ITEM(a[9], 1), "out.k");
    TORCH_CHECK_VALUE(q_out.defined() == q.defined() && k_out.defined() == k.defined(), "out: a tensor for each one that is given");
  }
  fikit_vectors in[2] = {}, out[2] = {};
  uint32_t heads[2] = {};
  const at::Tensor* const sides[2][3] = {{&q, &q_out, &q_weight}, {&k, &k_out, &k_weight}};
  const char* const names[2][3] = {{"q", "out.q", "q_weight"}, {"k", "out.k", "k_weight"}};
  const void* weights[2] = {};
  for (int i = 0; i < 2; ++i) {
    const at::Tensor &x = *sides[i][0], &y = *sides[i][1], &w = *sides[i][2];
    TORCH_CHECK_VALUE(x.defined() || !w.defined(), names[i][2], ": without heads");
    if (!x.defined()) continue;
    in[i] = vectors(x, type, device, names[i][0]);
    TORCH_CHECK_VALUE(x.size(0) == any.size(0) && x.size(2) == any.size(2), "q, k: [n_tokens, heads, head_dim]");
    heads[i] = count(x.size(1), names[i][0]);
    if (y.defined()) {
      TORCH_CHECK_VALUE(y.sizes() == x.sizes(), names[i][1], ": the shape of its input");
      out[i] = vectors(y, type, device, names[i][1]);
    }
    if (w.defined()) {
      TORCH_CHECK_VALUE(w.numel() == x.size(2), names[i][2], ": [head_dim]");
      without_gradient(w, names[i][2]);
      weights[i] = dense<void>(w, type, device, names[i][2]);
    }
  }
  TORCH_CHECK_VALUE(positions.numel() == any.size(0) && status.numel() == 1, "positions: [n_tokens]; status: [1]");
  if (frequencies.defined()) without_gradient(frequencies, "frequencies");
  int rc;
  {
    const Unlocked unlocked;
    if (a[9] == Py_None) {      // one allocation
      const int64_t of_q = q.defined() ? q.numel() : 0;
      const at::Tensor all = at::empty({of_q + (k.defined() ? k.numel() : 0)}, at::TensorOptions().dtype(type).device(device));
      if (q.defined()) q_out = part_of(all, type, 0, q.sizes());
      if (k.defined()) k_out = part_of(all, type, of_q, k.sizes());
      if (q.defined()) out[0] = vectors(q_out, type, device, "out.q");
      if (k.defined()) out[1] = vectors(k_out, type, device, "out.k");
    }
    rc = rotate_heads(&in[0], &in[1], heads[0], heads[1], count(any.size(2), "head_dim"), of_values, weights[0], weights[1], epsilon,
                      dense<int32_t>(positions, at::kInt, device, "positions"),
                      frequencies.defined() ? dense<float>(frequencies, at::kFloat, device, "frequencies") : nullptr,
                      frequencies.defined() ? count(2 * frequencies.numel(), "frequencies") : 0, neighbours ? FIKIT_PAIRS_NEIGHBOURS : FIKIT_PAIRS_HALVES,
                      count(any.size(0), "tokens"), &out[0], &out[1], dense<int32_t>(status, at::kInt, device, "status"), stream);
  }
  if (a[9] != Py_None) written(rc, {&q_out, &k_out});
  if (rc != FIKIT_OK) return PyLong_FromLong(rc);
  if (a[9] != Py_None) {
    Py_INCREF(a[9]);
    return a[9];
  }
  return Py_BuildValue("(NN)", wrapped(q_out), wrapped(k_out));
  END_HANDLE_TH_ERRORS
}

// The tensors of a tuple that is given for a call's outputs.
template <int N>
void given_tuple(PyObject* given, at::Tensor* const (&parts)[N], const char* what) {
  TORCH_CHECK_VALUE(PyTuple_Check(given) && PyTuple_GET_SIZE(given) == N, "out: a ", what);
  for (int i = 0; i < N; ++i) *parts[i] = tensor(PyTuple_GET_ITEM(given, i), "out");
}

// Dense tensors of 32-bit integers in one allocation; pairs come first, which are 8-byte aligned.
struct Ints {
  at::Tensor all;
  int64_t at = 0;
  Ints(int64_t n, const at::Device& device) : all(at::empty({n}, at::TensorOptions().dtype(at::kInt).device(device))) {}
  at::Tensor take(at::IntArrayRef sizes) {
    const at::Tensor t = part_of(all, at::kInt, at, sizes);
    at += t.numel();
    return t;
  }
};

// block_table, lengths, parents, block_tokens, n_blocks, free_blocks, status, out, workspace_buf, stream
PyObject* py_cache_fork(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 10);
  const at::Tensor &table = tensor(a[0], "block_table"), &lengths = tensor(a[1], "lengths"), &parents = tensor(a[2], "parents"),
                   &free = tensor(a[5], "free_blocks"), &status = tensor(a[6], "status");
  const at::Device device = table.device();
  const uint32_t block_tokens = count(a[3], "block_tokens"), n_blocks = count(a[4], "n_blocks");
  TORCH_CHECK_VALUE(table.dim() == 2 && lengths.numel() == table.size(0) && status.numel() == 1, "block_table: [R, width]; lengths: [R]; status: [1]");
  const uint32_t n = count(table.size(0), "block_table"), width = count(table.size(1), "block_table"), children = count(parents.numel(), "parents");
  at::Tensor new_table, new_lengths, copies, new_free, counts;
  const bool allocate = a[7] == Py_None;
  if (!allocate) {
    given_tuple(a[7], {&new_table, &new_lengths, &copies, &new_free, &counts}, "CacheFork");
    TORCH_CHECK_VALUE(new_table.dim() == 2 && new_table.size(0) == children && new_table.size(1) == width && new_lengths.numel() == children &&
                          copies.numel() == 2 * static_cast<int64_t>(children) && new_free.numel() == n_blocks && counts.numel() == 3,
                      "out: tensors of the fork's sizes");
  }
  const at::Tensor workspace = given_or_none(a[8], "workspace_buf");
  void* const stream = stream_of(a[9]);
  int rc;
  {
    const Unlocked unlocked;
    if (allocate) {
      const int64_t c = children;
      Ints ints(2 * c + c * width + c + n_blocks + 3, device);
      copies = ints.take({c, 2});
      new_table = ints.take({c, width});
      new_lengths = ints.take({c});
      new_free = ints.take({n_blocks});
      counts = ints.take({3});
    }
    const at::Tensor ws = workspace_of(workspace, cache_fork_workspace_bytes(n, children, width, n_blocks), device);
    rc = cache_fork(dense<int32_t>(table, at::kInt, device, "block_table"), width, dense<int32_t>(lengths, at::kInt, device, "lengths"), n,
                    dense<int32_t>(parents, at::kInt, device, "parents"), children, block_tokens, n_blocks,
                    dense<int32_t>(free, at::kInt, device, "free_blocks"), count(free.numel(), "free_blocks"),
                    dense<int32_t>(new_table, at::kInt, device, "out"), dense<int32_t>(new_lengths, at::kInt, device, "out"),
                    dense<fikit_block_copy>(copies, at::kInt, device, "out"), dense<int32_t>(new_free, at::kInt, device, "out"),
                    dense<int32_t>(counts, at::kInt, device, "out"), dense<int32_t>(status, at::kInt, device, "status"),
                    ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, stream);
  }
  if (!allocate) written(rc, {&new_table, &new_lengths, &copies, &new_free, &counts});
  if (rc != FIKIT_OK) return PyLong_FromLong(rc);
  if (!allocate) {
    Py_INCREF(a[7]);
    return a[7];
  }
  return Py_BuildValue("(NNNNN)", wrapped(new_table), wrapped(new_lengths), wrapped(copies), wrapped(new_free), wrapped(counts));
  END_HANDLE_TH_ERRORS
}

// block_table, lengths, block_tokens, n_blocks, free_blocks, status, out, workspace_buf, stream
PyObject* py_cache_compact(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 9);
  const at::Tensor &table = tensor(a[0], "block_table"), &lengths = tensor(a[1], "lengths"), &free = tensor(a[4], "free_blocks"), &status = tensor(a[5], "status");
  const at::Device device = table.device();
  const uint32_t block_tokens = count(a[2], "block_tokens"), n_blocks = count(a[3], "n_blocks"), n_free = count(free.numel(), "free_blocks");
  TORCH_CHECK_VALUE(table.dim() == 2 && lengths.numel() == table.size(0) && status.numel() == 1, "block_table: [R, width]; lengths: [R]; status: [1]");
  const uint32_t n = count(table.size(0), "block_table"), width = count(table.size(1), "block_table");
  const int64_t room = n_free < n_blocks / 2 ? n_free : n_blocks / 2;
  at::Tensor new_table, copies, new_free, counts;
  const bool allocate = a[6] == Py_None;
  if (!allocate) {
    given_tuple(a[6], {&new_table, &copies, &new_free, &counts}, "CacheCompaction");
    TORCH_CHECK_VALUE(new_table.sizes() == table.sizes() && copies.numel() == 2 * room && new_free.numel() == n_free && counts.numel() == 2,
                      "out: tensors of the compaction's sizes");
  }
  const at::Tensor workspace = given_or_none(a[7], "workspace_buf");
  void* const stream = stream_of(a[8]);
  int rc;
  {
    const Unlocked unlocked;
    if (allocate) {
      Ints ints(2 * room + table.numel() + n_free + 2, device);
      copies = ints.take({room, 2});
      new_table = ints.take(table.sizes());
      new_free = ints.take({n_free});
      counts = ints.take({2});
    }
    const at::Tensor ws = workspace_of(workspace, cache_compact_workspace_bytes(n, width, n_blocks), device);
    rc = cache_compact(dense<int32_t>(table, at::kInt, device, "block_table"), width, dense<int32_t>(lengths, at::kInt, device, "lengths"), n, block_tokens,
                       n_blocks, dense<int32_t>(free, at::kInt, device, "free_blocks"), n_free, dense<int32_t>(new_table, at::kInt, device, "out"),
                       dense<fikit_block_copy>(copies, at::kInt, device, "out"), dense<int32_t>(new_free, at::kInt, device, "out"),
                       dense<int32_t>(counts, at::kInt, device, "out"), dense<int32_t>(status, at::kInt, device, "status"),
                       ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, stream);
  }
  if (!allocate) written(rc, {&new_table, &copies, &new_free, &counts});
  if (rc != FIKIT_OK) return PyLong_FromLong(rc);
  if (!allocate) {
    Py_INCREF(a[6]);
    return a[6];
  }
  return Py_BuildValue("(NNNN)", wrapped(new_table), wrapped(copies), wrapped(new_free), wrapped(counts));
  END_HANDLE_TH_ERRORS
}

// A reference of one's own.
struct Owned {
  PyObject* o;
  explicit Owned(PyObject* given) : o(given) { if (!o) throw python_error(); }
  Owned(Owned&& other) noexcept : o(other.o) { other.o = nullptr; }
  ~Owned() { Py_XDECREF(o); }
};

// caches (a sequence of sequences k_cache, v_cache, k_exp, v_exp), copies, status, stream
PyObject* py_cache_copy(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 4);
  const at::Tensor &copies = tensor(a[1], "copies"), &status = tensor(a[2], "status");
  const at::Device device = copies.device();
  TORCH_CHECK_VALUE(copies.dim() == 2 && copies.size(1) == 2 && status.numel() == 1, "copies: [n, 2]; status: [1]");
  const Owned all(PySequence_Tuple(a[0]));
  std::vector<fikit_cache> caches;
  std::vector<Owned> held;                     // (other threads may change the sequences while the call enqueues)
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(all.o); ++i) {
    held.emplace_back(PySequence_Tuple(PyTuple_GET_ITEM(all.o, i)));
    const Owned& one = held.back();
    TORCH_CHECK_VALUE(PyTuple_GET_SIZE(one.o) == 4, "caches: of k_cache, v_cache, k_exp, v_exp each");
    PyObject* const parts[] = {PyTuple_GET_ITEM(one.o, 0), PyTuple_GET_ITEM(one.o, 1), PyTuple_GET_ITEM(one.o, 2), PyTuple_GET_ITEM(one.o, 3)};
    caches.push_back(cache_of(parts, device));
  }
  void* const stream = stream_of(a[3]);
  int rc;
  {
    const Unlocked unlocked;
    rc = cache_copy(caches.data(), count(static_cast<int64_t>(caches.size()), "caches"), dense<fikit_block_copy>(copies, at::kInt, device, "copies"),
                    count(copies.size(0), "copies"), dense<int32_t>(status, at::kInt, device, "status"), stream);
  }
  for (const Owned& one : held)
    for (int i = 0; i < 4; ++i) written(rc, {&THPVariable_Unpack(PyTuple_GET_ITEM(one.o, i))});
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// logits, tokens or None, status, scale, n_top, out, workspace_buf, stream
PyObject* py_token_scores(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 8);
  const at::Tensor &logits = tensor(a[0], "logits"), tokens = given_or_none(a[1], "tokens"), &status = tensor(a[2], "status");
  const at::Device device = logits.device();
  TORCH_CHECK_VALUE(logits.dim() == 2 && (logits.stride(1) == 1 || logits.size(1) <= 1) && logits.stride(0) >= 0, "logits: [rows, vocabulary], the last dimension dense");
  without_gradient(logits, "logits");
  const at::ScalarType type = logits.scalar_type();
  TORCH_CHECK_VALUE(type == at::kFloat || type == at::kBFloat16 || type == at::kHalf, "logits: bfloat16, float16 or float32");
  const int32_t of_values = type == at::kFloat ? FIKIT_F32 : value_type(logits, "logits");
  const float scale = static_cast<float>(THPUtils_unpackDouble(a[3]));
  const uint32_t n_top = count(a[4], "n_top"), rows = count(logits.size(0), "rows"), vocabulary = count(logits.size(1), "vocabulary");
  TORCH_CHECK_VALUE((!tokens.defined() || tokens.numel() == rows) && status.numel() == 1, "tokens: [rows]; status: [1]");
  at::Tensor logprob, entropy, lse, top_tokens, top_logprob;
  const bool allocate = a[5] == Py_None;
  if (!allocate) {
    TORCH_CHECK_VALUE(PyTuple_Check(a[5]) && PyTuple_GET_SIZE(a[5]) == 5, "out: a TokenScores");
    logprob = given_or_none(PyTuple_GET_ITEM(a[5], 0), "logprob");
    entropy = given_or_none(PyTuple_GET_ITEM(a[5], 1), "entropy");
    lse = given_or_none(PyTuple_GET_ITEM(a[5], 2), "lse");
    top_tokens = given_or_none(PyTuple_GET_ITEM(a[5], 3), "top_tokens");
    top_logprob = given_or_none(PyTuple_GET_ITEM(a[5], 4), "top_logprob");
    for (const at::Tensor* t : {&logprob, &entropy, &lse}) TORCH_CHECK_VALUE(!t->defined() || t->numel() == rows, "out: [rows]");
    const int64_t tops = static_cast<int64_t>(rows) * n_top;
    for (const at::Tensor* t : {&logprob, &entropy, &lse, &top_logprob})
      if (t->defined()) without_gradient(*t, "out");
    for (const at::Tensor* t : {&top_tokens, &top_logprob}) TORCH_CHECK_VALUE(t->defined() ? t->numel() == tops : n_top == 0, "out: [rows, n_top]");
  }
  const at::Tensor workspace = given_or_none(a[6], "workspace_buf");
  void* const stream = stream_of(a[7]);
  int rc;
  {
    const Unlocked unlocked;
    if (allocate && n_top <= 32) {      // one allocation
      const int64_t n = rows, k = n_top;
      const at::Tensor all = at::empty({n * (3 + 2 * k)}, at::TensorOptions().dtype(at::kFloat).device(device));
      if (tokens.defined()) logprob = part_of(all, at::kFloat, 0, {n});
      entropy = part_of(all, at::kFloat, n, {n});
      lse = part_of(all, at::kFloat, 2 * n, {n});
      top_logprob = part_of(all, at::kFloat, 3 * n, {n, k});
      top_tokens = part_of(all, at::kInt, 3 * n + n * k, {n, k});
    }
    const auto floats = [&](const at::Tensor& t) { return t.defined() ? dense<float>(t, at::kFloat, device, "out") : nullptr; };
    const at::Tensor ws = workspace_of(workspace, token_scores_workspace_bytes(rows, vocabulary, of_values, n_top), device);
    rc = token_scores(logits.data_ptr(), of_values, rows > 1 ? static_cast<uint64_t>(logits.stride(0)) : 0, rows, vocabulary, scale,
                      tokens.defined() ? dense<int32_t>(tokens, at::kInt, device, "tokens") : nullptr, n_top, floats(logprob), floats(entropy), floats(lse),
                      top_tokens.defined() ? dense<int32_t>(top_tokens, at::kInt, device, "out") : nullptr, floats(top_logprob),
                      dense<int32_t>(status, at::kInt, device, "status"), ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.numel() : 0, stream);
  }
  if (!allocate) written(rc, {&logprob, &entropy, &lse, &top_tokens, &top_logprob});
  if (rc != FIKIT_OK) return PyLong_FromLong(rc);
  if (!allocate) {
    Py_INCREF(a[5]);
    return a[5];
  }
  return Py_BuildValue("(NNNNN)", wrapped(logprob), wrapped(entropy), wrapped(lse), wrapped(top_tokens), wrapped(top_logprob));
  END_HANDLE_TH_ERRORS
}

template <typename F>
void set_address(F& f, PyObject* o) { f = reinterpret_cast<F>(PyLong_AsVoidPtr(o)); }

// The addresses of the C calls around the attention, in the order of the variables above.
PyObject* py_bind_around(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 8);
  set_address(rotate_heads, a[0]);
  set_address(cache_fork_workspace_bytes, a[1]);
  set_address(cache_fork, a[2]);
  set_address(cache_compact_workspace_bytes, a[3]);
  set_address(cache_compact, a[4]);
  set_address(cache_copy, a[5]);
  set_address(token_scores_workspace_bytes, a[6]);
  set_address(token_scores, a[7]);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// The addresses of the attention calls, in the order of the variables above.
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  need_arguments(n_args, 7);
  set_address(cache_pieces, a[0]);
  set_address(cache_plan_workspace_bytes, a[1]);
  set_address(cache_plan, a[2]);
  set_address(cache_append, a[3]);
  set_address(cache_attention_workspace_bytes, a[4]);
  set_address(cache_attention, a[5]);
  set_address(prompt_attention, a[6]);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(cache_plan), METHOD(cache_append), METHOD(cache_attention), METHOD(prompt_attention),
                         METHOD(bind_around), METHOD(rotate_heads), METHOD(cache_fork), METHOD(cache_compact), METHOD(cache_copy),
                         METHOD(token_scores), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serve_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serve_marshal() { return PyModule_Create(&module); }
