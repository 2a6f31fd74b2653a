// C ABI of the calls around the attention: argument checks, how the work is cut up, kernel sequencing.
#include "fikit.h"

#include <hip/hip_runtime.h>

#include "rotate_kernels.hip.h"
#include "serve_host.h"

namespace {

using namespace fikit;

constexpr uint32_t ROTATE_MOST_GROUPS = 1u << 16;
constexpr uint32_t ROTATE_SPREAD = 2048;          // waves: eight for each CU

struct RotateCall {
  const RotateArgs& a;
  bool neighbours;
  hipStream_t st;
  template <typename T, int D>
  int run() {
    const uint32_t groups = (a.units + ROTATE_WAVES - 1) / ROTATE_WAVES;
    const dim3 grid(groups < ROTATE_MOST_GROUPS ? groups : ROTATE_MOST_GROUPS), block(ROTATE_WAVES * WAVE);
    return neighbours ? enqueue(k_rotate<T, D, true>, grid, block, st, a) : enqueue(k_rotate<T, D, false>, grid, block, st, a);
  }
  template <typename T>
  int with_dim(uint32_t head_dim) { return head_dim == 64 ? run<T, 64>() : head_dim == 128 ? run<T, 128>() : run<T, 256>(); }
};

// Outputs of `heads` heads whose vectors do not lie over each other.
bool apart(const fikit_vectors* v, uint32_t heads, uint32_t n_tokens, uint32_t head_dim) {
  return (heads <= 1 || v->head_stride >= head_dim) && (n_tokens <= 1 || v->token_stride >= head_dim);
}

bool rotates_in_place_or_elsewhere(const fikit_vectors* in, const fikit_vectors* out, uint32_t heads, uint32_t n_tokens) {
  return in->d_data != out->d_data || ((heads <= 1 || in->head_stride == out->head_stride) && (n_tokens <= 1 || in->token_stride == out->token_stride));
}

}  // namespace

extern "C" {

int fikit_rotate_heads(const fikit_vectors* h_q, const fikit_vectors* h_k, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim,
                       int32_t value_type, const void* d_q_weight, const void* d_k_weight, float epsilon, const int32_t* d_positions,
                       const float* d_frequencies, uint32_t rotary_dim, int32_t pairs, uint32_t n_tokens, const fikit_vectors* h_q_out,
                       const fikit_vectors* h_k_out, int32_t* d_status, void* hip_stream) {
  if (!type_ok(value_type) || !d_status || !aligned(d_status, 4) || n_tokens > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (pairs != FIKIT_PAIRS_HALVES && pairs != FIKIT_PAIRS_NEIGHBOURS) return FIKIT_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return FIKIT_UNSUPPORTED;
  if (rotary_dim % 16 || rotary_dim > head_dim || q_heads > 65535 || kv_heads > 65535) return FIKIT_UNSUPPORTED;
  if (!aligned(d_q_weight, 16) || !aligned(d_k_weight, 16)) return FIKIT_INVALID_ARG;
  if ((d_q_weight || d_k_weight) && !(epsilon >= 0x1p-126f && epsilon <= 3.4028234663852886e38f)) return FIKIT_INVALID_ARG;
  if (n_tokens == 0 || (q_heads == 0 && kv_heads == 0)) return FIKIT_OK;
  if (!d_positions || !aligned(d_positions, 4) || !aligned(d_frequencies, 4) || (rotary_dim > 0 && !d_frequencies)) return FIKIT_INVALID_ARG;
  struct { const fikit_vectors *in, *out; uint32_t heads; } sides[] = {{h_q, h_q_out, q_heads}, {h_k, h_k_out, kv_heads}};
  for (const auto& s : sides)
    if (s.heads > 0 && (!vectors_ok(s.in) || !vectors_ok(s.out) || !apart(s.out, s.heads, n_tokens, head_dim) ||
                        !rotates_in_place_or_elsewhere(s.in, s.out, s.heads, n_tokens)))
      return FIKIT_INVALID_ARG;
  if (q_heads > 0 && kv_heads > 0 && (h_q_out->d_data == h_k_out->d_data || h_q_out->d_data == h_k->d_data || h_k_out->d_data == h_q->d_data))
    return FIKIT_INVALID_ARG;
  RotateArgs a{};
  if (q_heads > 0) { a.q = *h_q; a.q_out = *h_q_out; }
  if (kv_heads > 0) { a.k = *h_k; a.k_out = *h_k_out; }
  a.q_weight = d_q_weight;
  a.k_weight = d_k_weight;
  a.positions = d_positions;
  a.frequencies = d_frequencies;
  a.status = d_status;
  a.q_heads = q_heads;
  a.kv_heads = kv_heads;
  a.half = rotary_dim / 2;
  const uint32_t heads = static_cast<uint32_t>(rotate_heads(static_cast<int>(head_dim)));
  a.q_passes = (q_heads + heads - 1) / heads;
  a.passes = a.q_passes + (kv_heads + heads - 1) / heads;
  // a wave for each pass as long as that does not fill the chip, else for each token, whose angles then are computed once
  a.per = static_cast<uint64_t>(n_tokens) * a.passes <= ROTATE_SPREAD ? 1 : a.passes;
  a.parts = (a.passes + a.per - 1) / a.per;
  a.units = n_tokens * a.parts;
  a.epsilon = epsilon;
  RotateCall call{a, pairs == FIKIT_PAIRS_NEIGHBOURS, static_cast<hipStream_t>(hip_stream)};
  return value_type == FIKIT_BF16 ? call.with_dim<Bf16>(head_dim) : call.with_dim<F16>(head_dim);
}

}  // extern "C"
