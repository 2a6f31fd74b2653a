// Causal attention of packed prompts.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// A workgroup takes 32 query rows per wave of one prompt and head and passes once over the keys and values up to its last row,
// 64 tokens at a time through LDS (two buffers, filled by loads that go there directly):
//
//   scores   S^T[token][row] = K Q^T by 32x32 tiles, so a lane has the scores of one row, and the running maximum and sum
//            of the softmax need one exchange, between the halves of the wave;
//   outputs  O^T[dim][row] += V^T P^T: the weights are an operand as they stand in the registers, their tokens in the order
//            that the score tiles left them in; values are read from LDS transposed, in the same order.
//
// The maximum is raised, and what has been summed rescaled, only when a score passes it by 2^8.  Rows of LDS are stored with
// their 16-byte pieces permuted, by the row's number, so that neither read meets a bank twice.

struct PromptArgs {
  fikit_vectors q, k, v;
  const int32_t* offsets;
  void* out;
  float* lse;
  int32_t* status;
  uint32_t q_heads, kv_heads, n_prompts, n_tokens, slots;
  float scale;
};

constexpr int PROMPT_KEYS = 64, PROMPT_WAVE_ROWS = 32;
constexpr float PROMPT_SLACK = 8.f;

typedef __attribute__((address_space(3))) uint16_t lds_u16;
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void load_to_lds(const uint16_t* from, uint16_t* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

__device__ __forceinline__ u32x2 read_transposed(const uint16_t* at) {
  return bits_as<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
}

template <int D>
__device__ __forceinline__ uint32_t key_swizzle(uint32_t row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ uint32_t value_swizzle(uint32_t row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; }

// The two halves of a word that are not finite, as a mask.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  constexpr uint32_t LO = T::EXP_MASK & 0xffffu, HI = T::EXP_MASK & 0xffff0000u;
  return ((w & LO) == LO ? 0xffffu : 0u) | ((w & HI) == HI ? 0xffff0000u : 0u);
}

template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * WAVE) void k_prompt(PromptArgs a) {
  constexpr int ROWS = WAVES * PROMPT_WAVE_ROWS, PIECES = D / 8, TILE = PROMPT_KEYS * D;
  constexpr int LOADS = PROMPT_KEYS * PIECES / (WAVES * WAVE);
  __shared__ __align__(16) uint16_t keys[2][TILE];
  __shared__ __align__(16) uint16_t vals[2][TILE];
  if (stopped(a.status)) return;
  const uint32_t lane = lane_id(), wave = threadIdx.x / WAVE, col = lane % 32, half = lane / 32;
  const uint32_t head = blockIdx.x % a.q_heads, slot = a.slots - 1 - blockIdx.x / a.q_heads;
  if (blockIdx.x == 0) {
    bool bad = a.offsets[0] != 0 || static_cast<uint32_t>(a.offsets[a.n_prompts]) != a.n_tokens;
    for (uint32_t p = threadIdx.x; p < a.n_prompts; p += WAVES * WAVE) bad |= a.offsets[p] > a.offsets[p + 1];
    if (bad) *a.status = FIKIT_INVALID_ARG;
  }
  // prompt p owns the slots from offsets[p] / ROWS + p on: enough for its rows, and found without a list
  uint32_t prompt = 0;
  for (uint32_t hi = a.n_prompts; hi - prompt > 1;) {
    const uint32_t mid = prompt + (hi - prompt) / 2;
    if (static_cast<uint32_t>(a.offsets[mid]) / ROWS + mid <= slot) prompt = mid; else hi = mid;
  }
  const uint32_t start = static_cast<uint32_t>(a.offsets[prompt]), stop = static_cast<uint32_t>(a.offsets[prompt + 1]);
  if (start > stop || stop > a.n_tokens) {
    if (threadIdx.x == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  const uint32_t length = stop - start, first = (slot - (start / ROWS + prompt)) * ROWS;
  if (first >= length) return;
  const uint32_t row0 = first + wave * PROMPT_WAVE_ROWS, row = row0 + col;      // in the prompt
  const uint32_t kv_head = head / (a.q_heads / a.kv_heads);
  const uint32_t tiles = (min_u32(first + ROWS, length) + PROMPT_KEYS - 1) / PROMPT_KEYS;

  const uint16_t* k = static_cast<const uint16_t*>(a.k.d_data) + start * a.k.token_stride + kv_head * a.k.head_stride;
  const uint16_t* v = static_cast<const uint16_t*>(a.v.d_data) + start * a.v.token_stride + kv_head * a.v.head_stride;
  auto fill = [&](uint32_t tile, int to) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t base = (i * WAVES + wave) * WAVE, c = base + lane, r = c / PIECES, piece = c % PIECES;
      const uint64_t token = min_u32(tile * PROMPT_KEYS + r, length - 1);       // (behind the end: the last token, masked)
      load_to_lds(k + token * a.k.token_stride + (piece ^ key_swizzle<D>(r)) * 8, keys[to] + base * 8);
      load_to_lds(v + token * a.v.token_stride + (piece ^ value_swizzle<D>(r)) * 8, vals[to] + base * 8);
    }
  };
  fill(0, 0);

  typename T::x8 q[D / 16];
  {
    const uint16_t* src = static_cast<const uint16_t*>(a.q.d_data) + (start + static_cast<uint64_t>(min_u32(row, length - 1))) * a.q.token_stride +
                          head * a.q.head_stride + half * 8;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) q[j] = bits_as<typename T::x8>(*reinterpret_cast<const u32x4*>(src + j * 16));
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  float m = -__builtin_huge_valf(), l = 0.f;
  const float scale = a.scale * LOG2E;
  const uint32_t l16 = lane % 16, pair16 = (lane / 16) % 2;

  for (uint32_t tile = 0; tile < tiles; ++tile) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tile + 1 < tiles) fill(tile + 1, (tile + 1) & 1);
    const uint32_t token0 = tile * PROMPT_KEYS;
    if (token0 > row0 + PROMPT_WAVE_ROWS - 1) continue;        // (nothing of it is seen by this wave's rows)
    const uint16_t* kt = keys[tile & 1];
    const uint16_t* vt = vals[tile & 1];
    const bool masked = token0 + PROMPT_KEYS - 1 > row0;
    f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
      const uint32_t r = t * 32 + col;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(kt + r * D + ((2 * j + half) ^ key_swizzle<D>(r)) * 8);
        s[t] = T::mfma32(bits_as<typename T::x8>(w), q[j], s[t]);
      }
    }
    float most = -__builtin_huge_valf();
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[t][r] *= scale;
        if (masked && token0 + t * 32 + r / 4 * 8 + half * 4 + r % 4 > row) s[t][r] = -__builtin_huge_valf();
        most = fmaxf(most, s[t][r]);
      }
    if (ballot(most > m + (PROMPT_SLACK + T::WEIGHT_BIAS))) {
      most = fmaxf(most, __shfl_xor(most, 32, WAVE));
      const float raised = fmaxf(m, most - T::WEIGHT_BIAS);
      const float down = raised > -__builtin_huge_valf() ? exp2_fast(m - raised) : 1.f;
      m = raised;
      l *= down;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) acc[d] *= down;
    }
    const float origin = m > -__builtin_huge_valf() ? m : 0.f;
    typename T::x8 weights[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(s[t][8 * u + 2 * i] - origin), r = exp2_fast(s[t][8 * u + 2 * i + 1] - origin);
          l += p + r;
          w[i] = T::pair(p, r);
        }
        weights[2 * t + u] = bits_as<typename T::x8>(w);
      }
    auto value = [&](int step, int d) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t r = step * 16 + e * 8 + half * 4 + l16 / 4, piece = 4 * d + 2 * pair16 + l16 % 4 / 2;
        const u32x2 x = read_transposed(vt + r * D + (piece ^ value_swizzle<D>(r)) * 8 + l16 % 2 * 4);
        w[2 * e] = x[0];
        w[2 * e + 1] = x[1];
      }
      return w;
    };
    uint32_t dirty = 0;
#pragma unroll
    for (int step = 0; step < 4; ++step)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        u32x4 w = value(step, d);
        if (masked) {      // a weight of zero must not meet what is not finite
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = not_finite<T>(w[i]);
            dirty |= x;
            w[i] &= ~x;
          }
        }
        acc[d] = T::mfma32(bits_as<typename T::x8>(w), weights[step], acc[d]);
      }
    if (masked && ballot(dirty != 0)) {      // rows that do see it: found with products of ones
      for (int step = 0; step < 4; ++step) {
        u32x4 seen;
        for (int i = 0; i < 4; ++i) {
          uint32_t bits = 0;
          for (int b = 0; b < 2; ++b) {
            const uint32_t j = 2 * i + b, token = token0 + step * 16 + j / 4 * 8 + half * 4 + j % 4;
            if (token <= row) bits |= T::pair(1.f, 0.f) << (16 * b);
          }
          seen[i] = bits;
        }
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const u32x4 w = value(step, d);
          for (uint32_t kind = 0; kind < 3; ++kind) {      // infinity, -infinity, NaN
            u32x4 ones;
            for (int i = 0; i < 4; ++i) {
              uint32_t bits = 0;
              for (int b = 0; b < 2; ++b) {
                const uint32_t x = w[i] >> (16 * b) & 0xffffu;
                const uint32_t is = x == T::INF ? 0 : x == (T::INF | 0x8000u) ? 1 : (x & T::INF) == T::INF ? 2 : 3;
                if (is == kind) bits |= T::pair(1.f, 0.f) << (16 * b);
              }
              ones[i] = bits;
            }
            f32x16 c;
            for (int r = 0; r < 16; ++r) c[r] = 0.f;
            c = T::mfma32(bits_as<typename T::x8>(ones), bits_as<typename T::x8>(seen), c);
            const float add = kind == 0 ? __builtin_huge_valf() : kind == 1 ? -__builtin_huge_valf() : __builtin_nanf("");
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (c[r] > 0.f) acc[d][r] += add;
          }
        }
      }
    }
  }
  l += __shfl_xor(l, 32, WAVE);
  if (row >= length) return;
  const float f = l > 0.f ? 1.f / l : l == 0.f ? 1.f : l;
  const uint64_t at = (start + static_cast<uint64_t>(row)) * a.q_heads + head;
  uint16_t* out = static_cast<uint16_t*>(a.out) + at * D + half * 4;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const u32x2 w = {T::pair(acc[d][4 * r] * f, acc[d][4 * r + 1] * f), T::pair(acc[d][4 * r + 2] * f, acc[d][4 * r + 3] * f)};
      *reinterpret_cast<u32x2*>(out + d * 32 + r * 8) = w;
    }
  if (a.lse && half == 0) a.lse[at] = (m + log2f(l)) * LN2;
}

}  // namespace fikit
