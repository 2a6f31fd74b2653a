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
  uint2* spans;            // [request]: first part, number of parts
  float2* part_sums;       // [part][q head]: maximum (of scores times log2 e), sum
  float* part_out;         // [part][q head][D]
  uint32_t q_heads, table_width, max_length, head_tiles, n_requests;
  uint32_t parts;          // most parts of all requests together
  uint32_t per_request;    // 0: see k_decode; else so many parts for each request, of part_tokens
  uint32_t part_tokens;
  float scale;
};

// How contexts are cut into parts.  A part is a workgroup's for each key head and tile of query heads; many parts fill the chip
// and end together, few need less joining: a part's result is 4 G bytes a dimension (G query heads to a key head), written and
// read, for 2 part_tokens bytes of keys and values.  So with `units` key heads and tiles:
//   DECODE_GROUPS workgroups, of at least 64 G tokens each, but DECODE_FEW workgroups before that counts;
//   DECODE_LEAST to DECODE_MOST tokens (a wave's quarter holds at most 64 blocks).
constexpr uint32_t DECODE_GROUPS = 4096, DECODE_FEW = 512, DECODE_LEAST = 128, DECODE_MOST = 4096;
// Up to so many requests each workgroup looks at all lengths; for more, every request is cut alike, into parts of DECODE_MOST.
constexpr uint32_t DECODE_LOOK = 1024;

__host__ __device__ inline uint32_t decode_part_tokens(uint64_t tokens, uint32_t units, uint32_t rows) {
  uint64_t least = 64ull * rows;
  if (least > tokens * units / DECODE_FEW) least = tokens * units / DECODE_FEW;
  uint64_t part = (tokens * units + DECODE_GROUPS - 1) / DECODE_GROUPS;
  if (part < least) part = least;
  part = (part + DECODE_LEAST - 1) / DECODE_LEAST * DECODE_LEAST;
  return static_cast<uint32_t>(part < DECODE_LEAST ? DECODE_LEAST : part > DECODE_MOST ? DECODE_MOST : part);
}

constexpr int DECODE_WAVES = 4, DECODE_ROWS = 16, DECODE_STEP = 32;
constexpr float DECODE_SLACK = 8.f;   // log2 of how far a weight may pass 1 before the maximum is raised

template <int D>
struct DecodeStep {
  u32x4 k[2][D / 64];        // D / 4 codes of a key, two tiles of tokens
  uint32_t v[8][D / 64];     // D / 16 codes of each of eight values
};

// The item-th part, counting through the requests: every workgroup adds up all lengths for itself, which fixes the parts' size,
// and then the requests' parts.  False if there are fewer parts or the call has failed.
struct DecodeLook {
  uint64_t tokens[DECODE_WAVES];
  uint32_t parts[DECODE_WAVES];
  uint32_t request, part, n_parts, length;
};

__device__ __forceinline__ bool decode_find(const DecodeArgs& a, uint32_t item, uint32_t units, uint32_t rows, DecodeLook* lds, uint32_t* request,
                                            uint32_t* part, uint32_t* part_tokens, uint32_t* n_parts, uint32_t* length) {
  constexpr uint32_t PER = DECODE_LOOK / (DECODE_WAVES * WAVE);
  const uint32_t per = (a.n_requests + DECODE_WAVES * WAVE - 1) / (DECODE_WAVES * WAVE), first = threadIdx.x * per;
  const bool stop = stopped(a.status);
  uint32_t lengths[PER];
  uint64_t tokens = 0;
  bool ok = !stop;
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const bool there = i < per && first + i < a.n_requests;
    const int32_t n = there ? a.lengths[first + i] : 0;
    lengths[i] = static_cast<uint32_t>(n);
    if (n < 0 || lengths[i] > a.max_length) ok = false; else tokens += lengths[i];
  }
  const uint32_t wave = threadIdx.x / WAVE;
  for (int d = 1; d < WAVE; d <<= 1) tokens += shfl_xor_u64(tokens, d);
  if (lane_id() == 0) lds->tokens[wave] = tokens;
  if (threadIdx.x == 0) lds->request = 0xffffffffu;
  if (!__syncthreads_and(ok)) {
    if (threadIdx.x == 0 && !stop) *a.status = FIKIT_INVALID_ARG;
    return false;
  }
  tokens = 0;
  for (int w = 0; w < DECODE_WAVES; ++w) tokens += lds->tokens[w];
  const uint32_t size = decode_part_tokens(tokens, units, min_u32(rows, DECODE_ROWS));
  uint32_t count[PER], mine = 0;
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const bool there = i < per && first + i < a.n_requests;
    count[i] = !there ? 0 : lengths[i] == 0 ? 1 : (lengths[i] + size - 1) / size;
    mine += count[i];
  }
  uint32_t before = mine;
  for (int d = 1; d < WAVE; d <<= 1) {
    const uint32_t x = __shfl_up(before, d, WAVE);
    if (lane_id() >= static_cast<uint32_t>(d)) before += x;
  }
  if (lane_id() == WAVE - 1) lds->parts[wave] = before;
  __syncthreads();
  before -= mine;
  for (uint32_t w = 0; w < wave; ++w) before += lds->parts[w];
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    if (item >= before && item - before < count[i]) {
      lds->request = first + i;
      lds->part = item - before;
      lds->n_parts = count[i];
      lds->length = lengths[i];
    }
    before += count[i];
  }
  __syncthreads();
  *request = uniform(lds->request);
  *part = uniform(lds->part);
  *part_tokens = uniform(size);
  *n_parts = uniform(lds->n_parts);
  *length = uniform(lds->length);
  return *request != 0xffffffffu;
}

template <typename T, int D>
__global__ __launch_bounds__(DECODE_WAVES * WAVE) void k_decode(DecodeArgs a) {
  constexpr int KV_WORDS = D / 64;
  __shared__ float joined[DECODE_WAVES][DECODE_ROWS][D + 4];
  __shared__ float2 sums[DECODE_WAVES][DECODE_ROWS];
  __shared__ DecodeLook look;
  const uint32_t head_units = a.cache.kv_heads * a.head_tiles;
  const uint32_t unit = blockIdx.x % head_units, item = blockIdx.x / head_units;
  const uint32_t kv_head = unit / a.head_tiles, tile = unit % a.head_tiles;
  const uint32_t group = a.q_heads / a.cache.kv_heads;
  const uint32_t rows = min_u32(group - tile * DECODE_ROWS, DECODE_ROWS), first_head = kv_head * group + tile * DECODE_ROWS;
  const uint32_t shift = __builtin_ctz(a.cache.block_tokens);
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE), col = lane % 16, quarter = lane / 16;
  // which part of which request
  uint32_t request, part, part_tokens, n_parts, length;
  if (a.per_request) {
    if (stopped(a.status)) return;
    request = item / a.per_request;
    part = item % a.per_request;
    part_tokens = a.part_tokens;
    const int32_t signed_length = a.lengths[request];
    length = static_cast<uint32_t>(signed_length);
    if (signed_length < 0 || length > a.max_length) {
      if (threadIdx.x == 0) *a.status = FIKIT_INVALID_ARG;
      return;
    }
    n_parts = length == 0 ? 1 : (length + part_tokens - 1) / part_tokens;
    if (part >= n_parts) return;
    if (part == 0 && unit == 0 && threadIdx.x == 0) a.spans[request] = make_uint2(item, n_parts);
  } else {
    if (!decode_find(a, item, head_units, group, &look, &request, &part, &part_tokens, &n_parts, &length)) return;
    if (part == 0 && unit == 0 && threadIdx.x == 0) a.spans[request] = make_uint2(item, n_parts);
  }
  const uint32_t from = part * part_tokens;
  if (length == 0) {
    for (uint32_t i = threadIdx.x; i < rows * D; i += DECODE_WAVES * WAVE) {
      const uint64_t row = static_cast<uint64_t>(request) * a.q_heads + first_head + i / D;
      static_cast<uint16_t*>(a.out)[row * D + i % D] = 0;
      if (a.lse && i % D == 0) a.lse[row] = -__builtin_huge_valf();
    }
    return;
  }
  const uint32_t until = min_u32(length, from + part_tokens);
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
    if (n_parts == 1) {
      const float f = total > 0.f ? 1.f / total : total == 0.f ? 1.f : total;
      const u32x2 w = {T::pair(x[0] * f, x[1] * f), T::pair(x[2] * f, x[3] * f)};
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + head * D + dim) = w;
      if (dim == 0 && a.lse) a.lse[head] = (most + log2f(total)) * LN2;
    } else {
      const uint64_t slot = static_cast<uint64_t>(item) * a.q_heads + first_head + row;
      *reinterpret_cast<f32x4*>(a.part_out + slot * D + dim) = x;
      if (dim == 0) a.part_sums[slot] = make_float2(most, total);
    }
  }
}

// Joins the parts of one request and query head, always in the same order: each wave every fourth part, then the waves.
template <typename T, int D>
__global__ __launch_bounds__(DECODE_WAVES * WAVE) void k_decode_join(DecodeArgs a) {
  __shared__ float2 sums[DECODE_WAVES];
  __shared__ float outs[DECODE_WAVES][D];
  if (stopped(a.status)) return;
  const uint64_t head = blockIdx.x;
  const uint32_t request = blockIdx.x / a.q_heads, q_head = blockIdx.x % a.q_heads;
  const uint2 span = a.spans[request];
  if (span.y <= 1 || span.y > a.parts || span.x > a.parts - span.y) return;
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE);
  constexpr int PER = D / WAVE, MANY = 8;
  const uint64_t at = static_cast<uint64_t>(span.x) * a.q_heads + q_head;
  const float2* from = a.part_sums + at;
  const float* part = a.part_out + at * D + lane * PER;
  float most = -__builtin_huge_valf(), total = 0.f, x[PER];
  for (int i = 0; i < PER; ++i) x[i] = 0.f;
  for (uint32_t p = wave; p < span.y; p += DECODE_WAVES * MANY) {
    float2 s[MANY];
    float y[MANY][PER];
#pragma unroll
    for (int j = 0; j < MANY; ++j) {
      const uint64_t q = min_u32(p + j * DECODE_WAVES, span.y - 1);
      s[j] = from[q * a.q_heads];
      for (int i = 0; i < PER; ++i) y[j][i] = part[q * a.q_heads * D + i];
    }
    float top = most;
#pragma unroll
    for (int j = 0; j < MANY; ++j) top = fmaxf(top, s[j].x);
    const float origin = top > -__builtin_huge_valf() ? top : 0.f, down = exp2_fast(most - origin);
    total *= down;
    for (int i = 0; i < PER; ++i) x[i] *= down;
#pragma unroll
    for (int j = 0; j < MANY; ++j) {
      if (p + j * DECODE_WAVES >= span.y) continue;
      const float f = exp2_fast(s[j].x - origin);
      total += s[j].y * f;
      for (int i = 0; i < PER; ++i) x[i] += y[j][i] * f;
    }
    most = top;
  }
  if (lane == 0) sums[wave] = make_float2(most, total);
  for (int i = 0; i < PER; ++i) outs[wave][lane * PER + i] = x[i];
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  float top = -__builtin_huge_valf();
  for (int w = 0; w < DECODE_WAVES; ++w) top = fmaxf(top, sums[w].x);
  const float origin = top > -__builtin_huge_valf() ? top : 0.f;
  float sum = 0.f, lo = 0.f, hi = 0.f;
  for (int w = 0; w < DECODE_WAVES; ++w) {
    const float f = exp2_fast(sums[w].x - origin);
    sum += sums[w].y * f;
    lo += outs[w][2 * threadIdx.x] * f;
    hi += outs[w][2 * threadIdx.x + 1] * f;
  }
  const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 1.f : sum;
  reinterpret_cast<uint32_t*>(a.out)[head * (D / 2) + threadIdx.x] = T::pair(lo * f, hi * f);
  if (threadIdx.x == 0 && a.lse) a.lse[head] = (top + log2f(sum)) * LN2;
}

}  // namespace fikit
