// Attention of one query per request over the paged 8-bit cache.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// One pass over the keys and values with the running maximum and sum of the softmax.  A workgroup takes a part of one request's
// context for one key head and up to 16 of its query heads; its waves take a quarter of the part each, in steps of 32 tokens:
//
//   scores   S^T[token][query] = K Q^T, two 16x16 tiles: lane l holds the key codes of token l % 16, a quarter (l / 16) of the
//            dimensions, and the query's same quarter.  It receives the scores of query l % 16 at tokens 4 (l / 16) + 0..3.
//   weights  p = 2^(s - m), in the lane that has the score; m is raised, and what has been summed rescaled, only when a score
//            passes it by 2^8 (32 bits have room), so most steps exchange nothing between lanes.
//   outputs  O^T[dim][query] += V^T P^T: the order of the tokens within the product is free, so lane l takes as its eight
//            those whose weights it has, and reads their value codes at D / 16 consecutive dimensions.
//
// Codes become 16-bit values, scale included, in one instruction for two; nothing goes through LDS but the joining of
// the waves' results.  Parts of one request are joined by k_decode_join.

struct DecodeArgs {
  fikit_cache cache;
  fikit_vectors q;
  const int32_t* table;
  const int32_t* lengths;
  void* out;
  float* lse;
  int32_t* status;
  float* part_out;         // [request][part][q head][D]
  float2* part_sums;       // [request][part][q head]: maximum (of scores times log2 e), sum
  uint32_t q_heads, table_width, max_length, parts, part_tokens, head_tiles, n_requests;
  float scale;
};

constexpr int DECODE_WAVES = 4, DECODE_ROWS = 16, DECODE_STEP = 32;
constexpr float DECODE_SLACK = 8.f;   // log2 of how far a weight may pass 1 before the maximum is raised

template <int D>
struct DecodeStep {
  u32x4 k[2][D / 64];        // D / 4 codes of a key, two tiles of tokens
  uint32_t v[8][D / 64];     // D / 16 codes of each of eight values
};

template <typename T, int D>
__global__ __launch_bounds__(DECODE_WAVES * WAVE) void k_decode(DecodeArgs a) {
  constexpr int KV_WORDS = D / 64;
  __shared__ float joined[DECODE_WAVES][DECODE_ROWS][D + 4];
  __shared__ float2 sums[DECODE_WAVES][DECODE_ROWS];
  if (stopped(a.status)) return;
  const uint32_t head_units = a.cache.kv_heads * a.head_tiles;
  const uint32_t unit = blockIdx.x % head_units, rest = blockIdx.x / head_units;
  const uint32_t part = rest % a.parts, request = rest / a.parts;
  const uint32_t kv_head = unit / a.head_tiles, tile = unit % a.head_tiles;
  const uint32_t group = a.q_heads / a.cache.kv_heads;
  const uint32_t rows = min_u32(group - tile * DECODE_ROWS, DECODE_ROWS), first_head = kv_head * group + tile * DECODE_ROWS;
  const uint32_t shift = __builtin_ctz(a.cache.block_tokens);
  const int32_t signed_length = a.lengths[request];
  const uint32_t length = static_cast<uint32_t>(signed_length);
  if (signed_length < 0 || length > a.max_length) {
    if (threadIdx.x == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  const uint32_t lane = lane_id(), wave = threadIdx.x / WAVE, col = lane % 16, quarter = lane / 16;
  const bool alone = length <= a.part_tokens;       // no other part: the outputs are written here
  const uint32_t from = part * a.part_tokens;
  if (from >= length) {
    if (length == 0 && part == 0)
      for (uint32_t i = threadIdx.x; i < rows * D; i += DECODE_WAVES * WAVE) {
        const uint64_t row = static_cast<uint64_t>(request) * a.q_heads + first_head + i / D;
        static_cast<uint16_t*>(a.out)[row * D + i % D] = 0;
        if (a.lse && i % D == 0) a.lse[row] = -__builtin_huge_valf();
      }
    return;
  }
  const uint32_t until = min_u32(length, from + a.part_tokens);
  // this wave's quarter, in whole steps
  const uint32_t per_wave = ((until - from + DECODE_WAVES - 1) / DECODE_WAVES + DECODE_STEP - 1) / DECODE_STEP * DECODE_STEP;
  const uint32_t begin = from + wave * per_wave, end = min_u32(begin + per_wave, until);

  f32x4 acc[D / 16];
#pragma unroll
  for (int t = 0; t < D / 16; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_huge_valf(), l = 0.f;        // of query col; l over this lane's tokens

  if (begin < end) {
    // the queries: this lane's quarter of the dimensions of query col
    typename T::x8 q[D / 32];
    {
      const uint16_t* src = static_cast<const uint16_t*>(a.q.d_data) + request * a.q.token_stride +
                            static_cast<uint64_t>(first_head + min_u32(col, rows - 1)) * a.q.head_stride + quarter * (D / 4);
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        u32x4 w = *reinterpret_cast<const u32x4*>(src + j * 8);
        if (col >= rows) w = u32x4{0, 0, 0, 0};
        q[j] = bits_as<typename T::x8>(w);
      }
    }
    // lane i holds block and exponents of the i-th page of the wave's tokens (at most 64, see the host)
    const uint32_t first_page = begin >> shift, last_page = (end - 1) >> shift;
    const uint32_t my_page = min_u32(first_page + lane, last_page);
    const int32_t my_block = a.table[static_cast<uint64_t>(request) * a.table_width + my_page];
    const bool bad = static_cast<uint32_t>(my_block) >= a.cache.n_blocks;
    if (ballot(bad)) {
      if (lane == 0) *a.status = FIKIT_INVALID_ARG;
    } else {
      const uint64_t my_unit = static_cast<uint64_t>(my_block) * a.cache.kv_heads + kv_head;
      const uint32_t my_exps = a.cache.d_k_exp[my_unit] | static_cast<uint32_t>(a.cache.d_v_exp[my_unit]) << 8;
      const uint64_t unit_bytes = static_cast<uint64_t>(a.cache.block_tokens) * D;
      const float scale = a.scale * LOG2E;

      // tiles of 16 tokens lie in one page; a tile behind the last token is read from the last page
      auto tile_at = [&](uint32_t token, uint32_t* exps) {
        const uint32_t page = min_u32(token >> shift, last_page) - first_page;
        const uint32_t block = read_lane_u32(static_cast<uint32_t>(my_block), page);
        *exps = read_lane_u32(my_exps, page);
        return (static_cast<uint64_t>(block) * a.cache.kv_heads + kv_head) * unit_bytes + static_cast<uint64_t>(token & (a.cache.block_tokens - 1)) * D;
      };
      auto load = [&](uint32_t token, DecodeStep<D>* s, uint32_t* exps) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint64_t at = tile_at(token + 16 * h, exps + h);
          const uint8_t* k = a.cache.d_k + at + (col * D + quarter * (D / 4));
          const uint8_t* v = a.cache.d_v + at + (quarter * 4 * D + col * (D / 16));
#pragma unroll
          for (int j = 0; j < KV_WORDS; ++j) s->k[h][j] = *reinterpret_cast<const u32x4*>(k + j * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (KV_WORDS == 2) {
              const u32x2 w = *reinterpret_cast<const u32x2*>(v + i * D);
              s->v[4 * h + i][0] = w[0];
              s->v[4 * h + i][1] = w[1];
            } else {
              s->v[4 * h + i][0] = *reinterpret_cast<const uint32_t*>(v + i * D);
            }
          }
        }
      };
      DecodeStep<D> now, next;
      uint32_t exps[2], next_exps[2];
      load(begin, &now, exps);
      for (uint32_t token = begin; token < end; token += DECODE_STEP) {
        if (token + DECODE_STEP < end) load(token + DECODE_STEP, &next, next_exps);
        float s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 c = {0.f, 0.f, 0.f, 0.f};
          const float up = power_of(exps[h] & 255u);
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t codes = now.k[h][j / 2][(j & 1) * 2 + i];
              w[2 * i] = T::template codes<false>(codes, up);
              w[2 * i + 1] = T::template codes<true>(codes, up);
            }
            c = T::mfma16(bits_as<typename T::x8>(w), q[j], c);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) s[4 * h + i] = c[i] * scale;
        }
        if (token + DECODE_STEP > end) {     // what lies behind the last token counts for nothing, whatever it is
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (token + (i / 4) * 16 + quarter * 4 + i % 4 >= end) {
              s[i] = -__builtin_huge_valf();
#pragma unroll
              for (int j = 0; j < KV_WORDS; ++j) now.v[i][j] = 0;
            }
        }
        float most = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        if (ballot(most > m + (DECODE_SLACK + T::WEIGHT_BIAS))) {
          most = fmaxf(most, __shfl_xor(most, 16, WAVE));
          most = fmaxf(most, __shfl_xor(most, 32, WAVE));
          const float raised = fmaxf(m, most - T::WEIGHT_BIAS);
          const float down = raised > -__builtin_huge_valf() ? exp2_fast(m - raised) : 1.f;
          m = raised;
          l *= down;
#pragma unroll
          for (int t = 0; t < D / 16; ++t) acc[t] *= down;
        }
        const float origin = m > -__builtin_huge_valf() ? m : 0.f;
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(s[2 * i] - origin), r = exp2_fast(s[2 * i + 1] - origin);
          l += p + r;
          w[i] = T::pair(p, r);
        }
        const typename T::x8 weights = bits_as<typename T::x8>(w);
        const float up[2] = {power_of(exps[0] >> 8), power_of(exps[1] >> 8)};
#pragma unroll
        for (int j = 0; j < KV_WORDS; ++j) {
          u32x4 v[4];       // operands of four tiles of dimensions
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // bytes of two tokens side by side: dimensions 0 and 1, 2 and 3
            const uint32_t lo = __builtin_amdgcn_perm(now.v[2 * i + 1][j], now.v[2 * i][j], 0x05010400u);
            const uint32_t hi = __builtin_amdgcn_perm(now.v[2 * i + 1][j], now.v[2 * i][j], 0x07030602u);
            v[0][i] = T::template codes<false>(lo, up[i / 2]);
            v[1][i] = T::template codes<true>(lo, up[i / 2]);
            v[2][i] = T::template codes<false>(hi, up[i / 2]);
            v[3][i] = T::template codes<true>(hi, up[i / 2]);
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) acc[4 * j + t] = T::mfma16(bits_as<typename T::x8>(v[t]), weights, acc[4 * j + t]);
        }
        now = next;
        exps[0] = next_exps[0];
        exps[1] = next_exps[1];
      }
      l += __shfl_xor(l, 16, WAVE);
      l += __shfl_xor(l, 32, WAVE);
    }
  }
  // join the waves: lane l holds of query col the dimensions (D / 16) * (4 * quarter + i) + t
  if (quarter == 0) sums[wave][col] = make_float2(m, l);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int t = 0; t < D / 16; t += 4) {
      const f32x4 x = {acc[t][i], acc[t + 1][i], acc[t + 2][i], acc[t + 3][i]};
      *reinterpret_cast<f32x4*>(&joined[wave][col][D / 16 * (4 * quarter + i) + t]) = x;
    }
  __syncthreads();
  for (uint32_t at = threadIdx.x * 4; at < rows * D; at += DECODE_WAVES * WAVE * 4) {
    const uint32_t row = at / D, dim = at % D;
    float most = -__builtin_huge_valf(), total = 0.f;
#pragma unroll
    for (int w = 0; w < DECODE_WAVES; ++w) most = fmaxf(most, sums[w][row].x);
    const float origin = most > -__builtin_huge_valf() ? most : 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < DECODE_WAVES; ++w) {
      const float f = exp2_fast(sums[w][row].x - origin);
      total += sums[w][row].y * f;
      x += *reinterpret_cast<const f32x4*>(&joined[w][row][dim]) * f;
    }
    const uint64_t head = static_cast<uint64_t>(request) * a.q_heads + first_head + row;
    if (alone) {
      const float f = total > 0.f ? 1.f / total : total == 0.f ? 1.f : total;
      const u32x2 w = {T::pair(x[0] * f, x[1] * f), T::pair(x[2] * f, x[3] * f)};
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + head * D + dim) = w;
      if (dim == 0 && a.lse) a.lse[head] = (most + log2f(total)) * LN2;
    } else {
      const uint64_t slot = (static_cast<uint64_t>(request) * a.parts + part) * a.q_heads + first_head + row;
      *reinterpret_cast<f32x4*>(a.part_out + slot * D + dim) = x;
      if (dim == 0) a.part_sums[slot] = make_float2(most, total);
    }
  }
}

// Joins the parts of one request and query head, always in the same order; a wave each.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_decode_join(DecodeArgs a) {
  if (stopped(a.status)) return;
  const uint64_t head = static_cast<uint64_t>(blockIdx.x) * 4 + threadIdx.x / WAVE;
  if (head >= static_cast<uint64_t>(a.n_requests) * a.q_heads) return;
  const uint64_t request = head / a.q_heads, q_head = head % a.q_heads;
  const uint32_t length = static_cast<uint32_t>(a.lengths[request]);
  if (length <= a.part_tokens || length > a.max_length) return;
  const uint32_t parts = (length + a.part_tokens - 1) / a.part_tokens;
  const uint32_t lane = lane_id();
  constexpr int PER = D / WAVE;
  const float2* sums = a.part_sums + request * a.parts * a.q_heads + q_head;
  const float* part = a.part_out + (request * a.parts * a.q_heads + q_head) * D + lane * PER;
  float most = -__builtin_huge_valf();
  for (uint32_t p = lane; p < parts; p += WAVE) most = fmaxf(most, sums[static_cast<uint64_t>(p) * a.q_heads].x);
  for (int d = 1; d < WAVE; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, WAVE));
  const float origin = most > -__builtin_huge_valf() ? most : 0.f;
  float total = 0.f, x[PER];
  for (int i = 0; i < PER; ++i) x[i] = 0.f;
  for (uint32_t p = 0; p < parts; ++p) {
    const float2 s = sums[static_cast<uint64_t>(p) * a.q_heads];
    const float f = exp2_fast(s.x - origin);
    total += s.y * f;
    for (int i = 0; i < PER; ++i) x[i] += part[static_cast<uint64_t>(p) * a.q_heads * D + i] * f;
  }
  const float f = total > 0.f ? 1.f / total : total == 0.f ? 1.f : total;
  uint16_t* out = static_cast<uint16_t*>(a.out) + head * D + lane * PER;
  if constexpr (PER == 2) *reinterpret_cast<uint32_t*>(out) = T::pair(x[0] * f, x[1] * f);
  else *out = static_cast<uint16_t>(T::pair(x[0] * f, 0.f));
  if (lane == 0 && a.lse) a.lse[head] = (most + log2f(total)) * LN2;
}

}  // namespace fikit
