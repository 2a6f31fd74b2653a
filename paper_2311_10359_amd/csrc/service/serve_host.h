// What the entry points of the service's calls share on the host: checks of arguments, launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fikit.h"
#include "launches.h"

namespace fikit {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

constexpr uint64_t MOST_GROUPS = 0xffffffull;     // workgroups of 256 threads of a launch, whose threads number less than 2^32

template <typename... P, typename... A>
int enqueue(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t st, A... args) {
  count_launch();
  hipLaunchKernelGGL(kernel, grid, block, 0, st, args...);
  return hipGetLastError() == hipSuccess ? FIKIT_OK : FIKIT_HIP_ERROR;
}

struct Extent {
  const void* begin;
  uint64_t bytes;
};
inline bool overlap(const Extent& a, const Extent& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.begin), y = reinterpret_cast<uintptr_t>(b.begin);
  return a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

inline bool vectors_ok(const fikit_vectors* v) {
  return v && v->d_data && aligned(v->d_data, 16) && v->token_stride % 8 == 0 && v->head_stride % 8 == 0;
}

// FIKIT_OK, or what is wrong with a cache.
inline int cache_status(const fikit_cache* c) {
  if (!c || !c->d_k || !c->d_v || !c->d_k_exp || !c->d_v_exp || !aligned(c->d_k, 16) || !aligned(c->d_v, 16) || c->n_blocks == 0 ||
      c->n_blocks > 0x7fffffffu || c->kv_heads == 0)
    return FIKIT_INVALID_ARG;
  const uint32_t b = c->block_tokens;
  if (b < 16 || b > 256 || (b & (b - 1)) || (c->head_dim != 64 && c->head_dim != 128) || c->kv_heads > 65535) return FIKIT_UNSUPPORTED;
  return FIKIT_OK;
}

inline bool type_ok(int32_t value_type) { return value_type == FIKIT_BF16 || value_type == FIKIT_F16; }

}  // namespace fikit
