// Attention of one query per request over the paged 8-bit cache.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// One pass over the keys and values with the running maximum and sum of the softmax.  A workgroup takes a stretch of one request's
// context for one key head and up to 16 of its query heads; its waves take a quarter of it each, in steps of 32 tokens:
//
//   scores   S^T[token][query] = K Q^T, two 16x16 tiles: lane l holds key codes of token l % 16, a quarter of the dimensions (by
//            l / 16), and the same of query l % 16.  It receives the scores of that query at tokens 4 (l / 16) + 0..3.
//   weights  p = 2^(s - m), in the lane that has the score; m is raised, and what has been summed rescaled, only when a score
//            passes it by 2^8 (32 bits have room), so most steps exchange nothing between lanes.
//   outputs  O^T[dim][query] += V^T P^T: the order of the tokens within the product is free, so lane l takes as its eight
//            those whose weights it has, and reads their value codes at D / 16 consecutive dimensions.  Rounding a weight to 16
//            bits would cost as much as rounding the output; what it leaves is a second operand, which costs nothing here: the
//            matrix unit is busy for an eighth of the time.
//
// Codes become 16-bit values in one instruction for two; nothing goes through LDS but the joining of the waves' results.  No 16-bit type
// may cut the cache's range: codes without their scale are exact in either type, so keys become values of the queries' type and the
// scale meets the score, in 32 bits; values become bfloat16, which holds them with their scale, whatever the queries' type (in
// float16 the largest float16 values, 65,536 in the cache, would be infinite), and so do the weights, 16 bits of them in two operands.
//
// Bound by memory: a token costs 2 D bytes a key head and no more than 4 D operations for each of its query heads.  Two steps of codes are
// in flight per wave, in registers, which is what 8 waves (16 with heads of 64) on a compute unit leave room for.  128 requests of 4096 to
// 16,384 tokens, 8 heads of 128 (2.2 GB): 340 to 350 us, 6.4 to 6.5 TB/s, of the 7.2 that a kernel reaches which only reads past the caches; 64 requests
// of 1 to 13,517 tokens, 16 heads of 64, blocks of 16 (145 MB): 31 us, 4.6 TB/s; 2 of 76,687 and 127,690, 4 heads of 128 (209 MB): 38, 5.4
// TB/s; one of 4097 (8 MB): 6.8, latency.
//
// The work is cut evenly: with 128 tokens of a request, for one unit (key head and tile of query heads), as a chunk, and chunks in
// the order of requests, units, tokens, workgroup b of W takes chunks b T / W .. (b + 1) T / W - 1 of all T, whatever requests they
// belong to.  W is what the chip holds at once, so nothing is left over at the end, and what a workgroup begins with (adding up all
// lengths, first loads) is paid once.  Beginning and ending a stretch takes as long as DECODE_FIXED chunks, so a request's chunks
// are followed by so many empty ones (the 64 ragged requests with the joining: one 36.8 us, none 43.1, two 38.3, four 40.6).  Only the first and
// the last of a workgroup's stretches can be parts of longer ones; these are joined by k_decode_join.  (One workgroup for each part of equal
// length, as many as the longest request takes of all, was 41 us for the ragged requests, most of it for workgroups that found nothing to do.)

struct DecodeArgs {
  fikit_cache cache;
  fikit_vectors q;
  const int32_t* table;
  const int32_t* lengths;
  void* out;
  float* lse;
  int32_t* status;
  uint4* cuts;             // [W]: request, unit, chunk and chunks (with the empty ones) where a workgroup begins
  uint32_t* per_unit;      // chunks of one unit of all requests
  float2* part_sums;       // [2 W][rows]: maximum (of scores times log2 e), sum
  float* part_out;         // [2 W][rows][D]
  uint32_t q_heads, table_width, max_length, head_tiles, n_requests, groups;
  float scale;
};

constexpr int DECODE_WAVES = 4, DECODE_ROWS = 16, DECODE_STEP = 32;
constexpr uint32_t DECODE_CHUNK = DECODE_WAVES * DECODE_STEP;
constexpr float DECODE_SLACK = 8.f;   // log2 of how far a weight may pass 1 before the maximum is raised

// (a request without tokens has one chunk too, in which its outputs are written)
__host__ __device__ inline uint32_t decode_chunks(uint32_t length) { return length == 0 ? 1 : (length + DECODE_CHUNK - 1) / DECODE_CHUNK; }

constexpr uint32_t DECODE_FIXED = 1;
__host__ __device__ inline uint32_t decode_weight(uint32_t length) { return decode_chunks(length) + DECODE_FIXED; }

struct DecodeLook {
  uint32_t sums[DECODE_WAVES];
  uint32_t request, first;
};

// Adds up the chunks of all requests in every workgroup, a run of consecutive requests per thread; false if the call has failed.
__device__ __forceinline__ bool decode_look(const DecodeArgs& a, DecodeLook* lds, uint32_t* before, uint32_t* mine, uint32_t* total) {
  const uint32_t per = (a.n_requests + DECODE_WAVES * WAVE - 1) / (DECODE_WAVES * WAVE), first = threadIdx.x * per;
  const bool stop = stopped(a.status);
  bool ok = true;
  uint32_t sum = 0;
#pragma unroll 4
  for (uint32_t r = first; r < min_u32(first + per, a.n_requests); ++r) {
    const int32_t n = a.lengths[r];
    ok &= n >= 0 && static_cast<uint32_t>(n) <= a.max_length;
    sum += decode_weight(static_cast<uint32_t>(n));
  }
  const uint32_t run = wave_incl_scan_u32(sum);
  const uint32_t wave = threadIdx.x / WAVE;
  if (lane_id() == WAVE - 1) lds->sums[wave] = run;
  if (!__syncthreads_and(ok & !stop)) {
    if (threadIdx.x == 0 && !stop) *a.status = FIKIT_INVALID_ARG;
    return false;
  }
  uint32_t all = 0, earlier = 0;
  for (uint32_t w = 0; w < DECODE_WAVES; ++w) {
    if (w < wave) earlier += lds->sums[w];
    all += lds->sums[w];
  }
  *before = earlier + run - sum;
  *mine = sum;
  *total = uniform(all);
  return true;
}

// (Numbers of chunks fit 32 bits nearly always, and dividing 64 takes half a microsecond.)
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) {
  return (a | b) >> 32 ? a / b : static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
}
// Of all chunks workgroup b takes first(b) = b * total / groups and those up to first(b + 1), so the larger shares are spread evenly.
struct DecodeShares {
  uint32_t groups, more;
  uint64_t total, each;
  __device__ __forceinline__ DecodeShares(uint64_t total_, uint32_t most_groups) : total(total_) {
    groups = total < most_groups ? static_cast<uint32_t>(total) : most_groups;
    each = quotient(total, groups);
    more = static_cast<uint32_t>(total - each * groups);
  }
  __device__ __forceinline__ uint64_t first(uint32_t group) const { return group * each + group * more / groups; }      // (2^10 groups at most)
  __device__ __forceinline__ uint32_t owner(uint64_t chunk) const { return static_cast<uint32_t>(quotient((chunk + 1) * groups - 1, total)); }
};

// ONCE: no other workgroup reads these keys and values, so they are read past the caches: 5 to 10 % of the time of large
// calls.  That is the case for up to 16 query heads to a key head; for 32 the second reader finds them in a cache (64 requests of 8192
// tokens, 2 heads of 128: 94 us through the caches, 119 past them).
template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(DECODE_WAVES * WAVE, D == 128 ? 2 : 4) void k_decode(DecodeArgs a) {
  constexpr int KV_WORDS = D / 64;
  const auto read = [](const auto* p) { return ONCE ? __builtin_nontemporal_load(p) : *p; };
  __shared__ float joined[DECODE_WAVES][DECODE_ROWS][D + 4];
  __shared__ float2 sums[DECODE_WAVES][DECODE_ROWS];
  __shared__ DecodeLook look;
  const uint32_t units = a.cache.kv_heads * a.head_tiles, group = a.q_heads / a.cache.kv_heads, most_rows = min_u32(group, DECODE_ROWS);
  const uint32_t shift = __builtin_ctz(a.cache.block_tokens);
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE), col = lane % 16, quarter = lane / 16;
  const uint64_t unit_bytes = static_cast<uint64_t>(a.cache.block_tokens) * D;
  const float scale = a.scale * LOG2E;

  // where this workgroup's chunks begin: request, its length, its weight, the weights of the requests before
  uint32_t request, length, weight, first, per_unit, groups;
  uint64_t lo, left;
  auto cut = [&] {
    const DecodeShares shares(static_cast<uint64_t>(per_unit) * units, a.groups);
    groups = shares.groups;
    lo = shares.first(blockIdx.x);
    left = shares.first(blockIdx.x + 1) - lo;
    return static_cast<uint32_t>(quotient(lo, units));
  };
  auto pick = [&](uint32_t n, uint32_t w, uint32_t upto, uint32_t target) {      // the lane's request whose weight reaches past the target
    const uint64_t beyond = ballot(upto > target);
    if (!beyond) return false;
    const uint32_t owner = uniform(static_cast<uint32_t>(__builtin_ctzll(beyond)));
    length = read_lane_u32(n, owner);
    weight = read_lane_u32(w, owner);
    first = read_lane_u32(upto, owner) - weight;
    request += owner;
    return true;
  };
  if (a.n_requests <= WAVE) {      // each wave by itself, nothing is exchanged
    const bool stop = stopped(a.status), there = lane < a.n_requests;
    const int32_t n = there ? a.lengths[lane] : 0;
    if (ballot(n < 0 || static_cast<uint32_t>(n) > a.max_length) || stop) {
      if (threadIdx.x == 0 && !stop) *a.status = FIKIT_INVALID_ARG;
      return;
    }
    const uint32_t w = there ? decode_weight(static_cast<uint32_t>(n)) : 0, upto = wave_incl_scan_u32(w);
    per_unit = read_lane_u32(upto, WAVE - 1);
    const uint32_t target = cut();
    if (blockIdx.x >= groups) return;
    request = 0;
    pick(static_cast<uint32_t>(n), w, upto, target);
  } else {
    uint32_t before, mine;
    if (!decode_look(a, &look, &before, &mine, &per_unit)) return;
    const uint32_t target = cut();
    if (blockIdx.x >= groups) return;
    if (target >= before && target - before < mine) {
      look.request = threadIdx.x * ((a.n_requests + DECODE_WAVES * WAVE - 1) / (DECODE_WAVES * WAVE));
      look.first = before;
    }
    __syncthreads();
    request = uniform(look.request);
    uint32_t upto = uniform(look.first);
    for (;;) {               // of the requests that a thread has added up, 64 at a time
      const uint32_t r = request + lane;
      const uint32_t n = r < a.n_requests ? static_cast<uint32_t>(a.lengths[r]) : 0, w = decode_weight(n), run = wave_incl_scan_u32(w);
      if (pick(n, w, upto + run, target)) break;
      upto += read_lane_u32(run, WAVE - 1);
      request += WAVE;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.per_unit = per_unit;
  const uint64_t inside = lo - static_cast<uint64_t>(first) * units;
  uint32_t unit = static_cast<uint32_t>(quotient(inside, weight)), chunk = static_cast<uint32_t>(inside - static_cast<uint64_t>(unit) * weight);

  if (threadIdx.x == 0) a.cuts[blockIdx.x] = make_uint4(request, unit, chunk, weight);

  // The stretch that is next to be read: chunks chunk .. last_chunk - 1 of a request and unit, this wave's quarter of its tokens.
  uint32_t next_length = 0, last_chunk, kv_head, first_head, rows, begin, end;
  bool first_stretch = true;
  auto derive = [&] {
    const uint32_t take = left < weight - chunk ? static_cast<uint32_t>(left) : weight - chunk, tile = unit % a.head_tiles;
    left -= take;
    last_chunk = min_u32(chunk + take, weight - DECODE_FIXED);
    kv_head = unit / a.head_tiles;
    first_head = kv_head * group + tile * DECODE_ROWS;
    rows = min_u32(group - tile * DECODE_ROWS, DECODE_ROWS);
    const uint32_t from = chunk * DECODE_CHUNK, until = min_u32(length, last_chunk * DECODE_CHUNK);
    const uint32_t per_wave = (((until - from) + DECODE_WAVES - 1) / DECODE_WAVES + DECODE_STEP - 1) / DECODE_STEP * DECODE_STEP;
    begin = from + wave * per_wave;
    end = min_u32(begin + per_wave, until);
  };
  auto ask_length = [&] { next_length = static_cast<uint32_t>(a.lengths[min_u32(request + 1, a.n_requests - 1)]); };
  auto advance = [&] {
    if (left == 0) return false;
    first_stretch = false;
    chunk = 0;
    if (++unit == units) {
      unit = 0;
      ++request;
      length = uniform(next_length);
      weight = decode_weight(length);
      ask_length();
    }
    derive();
    return true;
  };

  // Lane i holds block and exponents of the i-th page of a window of 64; of the next window the blocks are read when a window
  // begins, and the exponents a step later.
  uint32_t window = 0, last_page = 0, my_block = 0, my_exps = 0, next_block = 0, next_exps = 0;
  bool asked = false;
  const int32_t* table = a.table;
  auto checked = [&](uint32_t block) {      // (a block outside the cache: the call has failed, block 0 is read instead)
    const bool bad = block >= a.cache.n_blocks;
    if (ballot(bad)) *a.status = FIKIT_INVALID_ARG;
    return bad ? 0u : block;
  };
  auto exponents = [&](uint32_t block) {
    const uint64_t at = static_cast<uint64_t>(block) * a.cache.kv_heads + kv_head;
    return a.cache.d_k_exp[at] | static_cast<uint32_t>(a.cache.d_v_exp[at]) << 8;
  };
  auto ask_blocks = [&] {
    if (begin >= end) return;
    window = begin >> shift;
    last_page = (end - 1) >> shift;
    table = a.table + static_cast<uint64_t>(request) * a.table_width;
    my_block = static_cast<uint32_t>(table[min_u32(window + lane, last_page)]);
  };
  auto ask_next_blocks = [&] {
    asked = window + WAVE <= last_page;
    if (asked) next_block = static_cast<uint32_t>(table[min_u32(window + WAVE + lane, last_page)]);
  };
  // Two steps are on their way: a step's keys and values are read into the registers of the step two before as soon as these have
  // been used.
  struct Step {
    u32x4 k[2][D / 64];        // 16 of every 64 codes of a key, of two tiles of tokens
    uint32_t v[8][KV_WORDS];   // D / 16 codes of each of eight values
    uint32_t exps[2];
    uint64_t at[2];
  };
  // (tiles of 16 tokens lie in one page; a tile behind the last token is read from the last page)
  auto page_of = [&](uint32_t token) { return min_u32(token >> shift, last_page) - window; };
  auto load_keys = [&](uint32_t token, Step& x) {
    if ((token >> shift) - window >= WAVE) {
      window += WAVE;
      my_block = next_block;
      my_exps = next_exps;
      ask_next_blocks();
    } else if (asked) {
      asked = false;
      next_block = checked(next_block);
      next_exps = exponents(next_block);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t block = read_lane_u32(my_block, page_of(token + 16 * h));
      x.at[h] = (static_cast<uint64_t>(block) * a.cache.kv_heads + kv_head) * unit_bytes + static_cast<uint64_t>((token + 16 * h) & (a.cache.block_tokens - 1)) * D;
      const uint8_t* from = a.cache.d_k + x.at[h] + (col * D + quarter * 16);
#pragma unroll
      for (int j = 0; j < KV_WORDS; ++j) x.k[h][j] = read(reinterpret_cast<const u32x4*>(from + j * 64));
    }
  };
  auto load_values = [&](uint32_t token, Step& x) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* from = a.cache.d_v + x.at[h] + (quarter * 4 * D + col * (D / 16));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (KV_WORDS == 2) {
          const u32x2 w = read(reinterpret_cast<const u32x2*>(from + i * D));
          x.v[4 * h + i][0] = w[0];
          x.v[4 * h + i][1] = w[1];
        } else {
          x.v[4 * h + i][0] = read(reinterpret_cast<const uint32_t*>(from + i * D));
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) x.exps[h] = read_lane_u32(my_exps, page_of(token + 16 * h));
  };
  Step even, odd;
  typename T::x8 q[D / 32];      // of query col the dimensions of which this lane reads the keys, 16 of every 64
  auto begin_reading = [&] {     // (ask_blocks before)
    if (begin >= end) return;
    const uint16_t* src = static_cast<const uint16_t*>(a.q.d_data) + request * a.q.token_stride +
                          static_cast<uint64_t>(first_head + min_u32(col, rows - 1)) * a.q.head_stride + quarter * 16;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      u32x4 w = *reinterpret_cast<const u32x4*>(src + j / 2 * 64 + j % 2 * 8);
      if (col >= rows) w = u32x4{0, 0, 0, 0};
      q[j] = bits_as<typename T::x8>(w);
    }
    my_block = checked(my_block);
    my_exps = exponents(my_block);
    asked = false;
    load_keys(begin, even);
    const bool two = begin + DECODE_STEP < end;
    if (two) load_keys(begin + DECODE_STEP, odd);
    load_values(begin, even);
    if (two) load_values(begin + DECODE_STEP, odd);
    ask_next_blocks();
  };

  ask_length();
  derive();
  if (chunk >= last_chunk && !advance()) return;
  ask_blocks();
  begin_reading();
  for (;;) {
    f32x4 acc[D / 16];
#pragma unroll
    for (int t = 0; t < D / 16; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_huge_valf(), l = 0.f;        // of query col; l over this lane's tokens
    auto step = [&](uint32_t token, Step& x) {
      const uint32_t ahead = token + 2 * DECODE_STEP;
      const float up[2] = {power_of(x.exps[0] >> 8), power_of(x.exps[1] >> 8)};
      float s[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
        const float k_up = power_of(x.exps[h] & 255u);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t codes = x.k[h][j / 2][(j & 1) * 2 + i];
            w[2 * i] = T::template codes<false>(codes, 1.f);
            w[2 * i + 1] = T::template codes<true>(codes, 1.f);
          }
          c = T::mfma16(bits_as<typename T::x8>(w), q[j], c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * h + i] = c[i] * k_up * scale;
      }
      if (ahead < end) load_keys(ahead, x);
      if (token + DECODE_STEP > end) {     // what lies behind the last token counts for nothing, whatever it is
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (token + (i / 4) * 16 + quarter * 4 + i % 4 >= end) {
            s[i] = -__builtin_huge_valf();
#pragma unroll
            for (int j = 0; j < KV_WORDS; ++j) x.v[i][j] = 0;
          }
      }
      float most = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
      if (ballot(most > m + DECODE_SLACK)) {
        most = fmaxf(most, __shfl_xor(most, 16, WAVE));
        most = fmaxf(most, __shfl_xor(most, 32, WAVE));
        const float raised = fmaxf(m, most);
        const float down = raised > -__builtin_huge_valf() ? exp2_fast(m - raised) : 1.f;
        m = raised;
        l *= down;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) acc[t] *= down;
      }
      const float origin = m > -__builtin_huge_valf() ? m : 0.f;
      u32x4 w, rest;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = exp2_fast(s[2 * i] - origin), r = exp2_fast(s[2 * i + 1] - origin);
        l += p + r;
        w[i] = Bf16::pair(p, r);
        rest[i] = Bf16::pair(p - Bf16::low(w[i]), r - Bf16::high(w[i]));
      }
      const Bf16::x8 weights = bits_as<Bf16::x8>(w);
#pragma unroll
      for (int j = 0; j < KV_WORDS; ++j) {
        u32x4 y[4];       // operands of four tiles of dimensions
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // bytes of two tokens side by side: dimensions 0 and 1, 2 and 3
          const uint32_t lo = __builtin_amdgcn_perm(x.v[2 * i + 1][j], x.v[2 * i][j], 0x05010400u);
          const uint32_t hi = __builtin_amdgcn_perm(x.v[2 * i + 1][j], x.v[2 * i][j], 0x07030602u);
          y[0][i] = Bf16::codes<false>(lo, up[i / 2]);
          y[1][i] = Bf16::codes<true>(lo, up[i / 2]);
          y[2][i] = Bf16::codes<false>(hi, up[i / 2]);
          y[3][i] = Bf16::codes<true>(hi, up[i / 2]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          acc[4 * j + t] = Bf16::mfma16(bits_as<Bf16::x8>(y[t]), weights, acc[4 * j + t]);
          acc[4 * j + t] = Bf16::mfma16(bits_as<Bf16::x8>(y[t]), bits_as<Bf16::x8>(rest), acc[4 * j + t]);
        }
      }
      if (ahead < end) load_values(ahead, x);
    };
    for (uint32_t token = begin; token < end; token += 2 * DECODE_STEP) {
      step(token, even);
      if (token + DECODE_STEP < end) step(token + DECODE_STEP, odd);
    }
    l += __shfl_xor(l, 16, WAVE);
    l += __shfl_xor(l, 32, WAVE);
    // where the results go; then the next stretch's blocks are asked for, while the waves write what they have, and its keys and
    // values, while that is joined (for another key head of a request the blocks are mostly the same)
    const uint64_t out_head = static_cast<uint64_t>(request) * a.q_heads + first_head;
    const uint32_t out_rows = rows, slot = 2 * blockIdx.x + (first_stretch ? 0 : 1);
    const bool whole = chunk == 0 && last_chunk == weight - DECODE_FIXED;
    const uint32_t old_request = request, old_begin = begin, old_end = end;
    const bool more = advance();
    if (more && (request != old_request || begin != old_begin || end != old_end || ((end - 1) >> shift) - (begin >> shift) >= WAVE)) ask_blocks();

    __syncthreads();          // (the stretch before has been read)
    // lane l holds of query col the dimensions (D / 16) * (4 * quarter + i) + t
    if (quarter == 0) sums[wave][col] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < D / 16; t += 4) {
        const f32x4 x = {acc[t][i], acc[t + 1][i], acc[t + 2][i], acc[t + 3][i]};
        *reinterpret_cast<f32x4*>(&joined[wave][col][D / 16 * (4 * quarter + i) + t]) = x;
      }
    __syncthreads();
    if (more) begin_reading();
    for (uint32_t at = threadIdx.x * 4; at < out_rows * D; at += DECODE_WAVES * WAVE * 4) {
      const uint32_t row = at / D, dim = at % D;
      float most = -__builtin_huge_valf(), sum = 0.f;
#pragma unroll
      for (int w = 0; w < DECODE_WAVES; ++w) most = fmaxf(most, sums[w][row].x);
      const float origin = most > -__builtin_huge_valf() ? most : 0.f;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < DECODE_WAVES; ++w) {
        const float f = exp2_fast(sums[w][row].x - origin);
        sum += sums[w][row].y * f;
        x += *reinterpret_cast<const f32x4*>(&joined[w][row][dim]) * f;
      }
      if (whole) {
        const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 1.f : sum;
        const u32x2 w = {T::pair(x[0] * f, x[1] * f), T::pair(x[2] * f, x[3] * f)};
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + (out_head + row) * D + dim) = w;
        if (dim == 0 && a.lse) a.lse[out_head + row] = (most + log2f(sum)) * LN2;
      } else {
        const uint64_t to = static_cast<uint64_t>(slot) * most_rows + row;
        *reinterpret_cast<f32x4*>(a.part_out + to * D + dim) = x;
        if (dim == 0) a.part_sums[to] = make_float2(most, sum);
      }
    }
    if (!more) return;
  }
}

// Joins the parts of a request and unit that was cut.  A workgroup for each place where one of k_decode's workgroups began: the n
// parts of a unit have n - 1 such places, whose workgroups share its query heads.  The parts of a head are added up in the same order
// always: by one wave, or, if a workgroup has a single head, by each wave every fourth part and then the waves.  Latency of two dependent
// loads and a launch: 4.9 us for up to 512 cuts, 6.8 where two requests of 76,687 and 127,690 tokens left up to 80 parts to a unit.  (A workgroup for each
// request and head took 30 us for 4000 requests, of which few were cut.)
template <typename T, int D>
__global__ __launch_bounds__(DECODE_WAVES * WAVE) void k_decode_join(DecodeArgs a) {
  __shared__ float2 sums[DECODE_WAVES];
  __shared__ float outs[DECODE_WAVES][D];
  const bool stop = stopped(a.status);        // (of the three loads none waits for another)
  const uint32_t per_unit = uniform(*a.per_unit);
  uint4 cut = a.cuts[blockIdx.x];
  asm volatile("" : "+v"(cut.x), "+v"(cut.y), "+v"(cut.z), "+v"(cut.w));      // (or it is read behind the branch)
  if (stop) return;
  const uint32_t units = a.cache.kv_heads * a.head_tiles, group = a.q_heads / a.cache.kv_heads, most_rows = min_u32(group, DECODE_ROWS);
  const DecodeShares shares(static_cast<uint64_t>(per_unit) * units, a.groups);
  if (blockIdx.x >= shares.groups) return;
  cut = make_uint4(uniform(cut.x), uniform(cut.y), uniform(cut.z), uniform(cut.w));
  const uint32_t request = cut.x, unit = cut.y, chunks = cut.w - DECODE_FIXED;
  if (cut.z == 0 || cut.z >= chunks) return;                  // (begins with the unit, or behind its last chunk)
  const uint64_t begin = shares.first(blockIdx.x) - cut.z;
  const uint32_t from = shares.owner(begin), parts = shares.owner(begin + chunks - 1) - from + 1;
  const uint32_t mine = blockIdx.x - from - 1, sharers = parts - 1;
  const uint32_t tile = unit % a.head_tiles, rows = min_u32(group - tile * DECODE_ROWS, DECODE_ROWS);
  if (mine >= sharers || mine >= rows) return;
  const uint64_t head0 = static_cast<uint64_t>(request) * a.q_heads + unit / a.head_tiles * group + tile * DECODE_ROWS;
  // the first part is its workgroup's last stretch, and its first one too if the workgroup begins here
  const uint32_t from_slot = 2 * from + (shares.first(from) >= begin ? 0 : 1);
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE);
  const bool shared = rows <= mine + sharers;                 // one head, all waves
  const uint32_t stride = shared ? DECODE_WAVES : 1;
  constexpr int PER = D / WAVE, MANY = 8;
  for (uint32_t row = mine + (shared ? 0 : wave * sharers); row < rows; row += sharers * DECODE_WAVES) {
    float most = -__builtin_huge_valf(), sum = 0.f, x[PER];
    for (int i = 0; i < PER; ++i) x[i] = 0.f;
    for (uint32_t p = shared ? wave : 0; p < parts; p += stride * MANY) {
      float2 s[MANY];
      float y[MANY][PER];
#pragma unroll
      for (int j = 0; j < MANY; ++j) {
        const uint32_t part = min_u32(p + j * stride, parts - 1);
        const uint64_t at = static_cast<uint64_t>(part == 0 ? from_slot : 2 * (from + part)) * most_rows + row;
        s[j] = a.part_sums[at];
        for (int i = 0; i < PER; ++i) y[j][i] = a.part_out[at * D + lane * PER + i];
      }
      float top = most;
#pragma unroll
      for (int j = 0; j < MANY; ++j) top = fmaxf(top, s[j].x);
      const float origin = top > -__builtin_huge_valf() ? top : 0.f, down = exp2_fast(most - origin);
      sum *= down;
      for (int i = 0; i < PER; ++i) x[i] *= down;
#pragma unroll
      for (int j = 0; j < MANY; ++j) {
        if (p + j * stride >= parts) continue;
        const float f = exp2_fast(s[j].x - origin);
        sum += s[j].y * f;
        for (int i = 0; i < PER; ++i) x[i] += y[j][i] * f;
      }
      most = top;
    }
    if (shared) {
      if (lane == 0) sums[wave] = make_float2(most, sum);
      for (int i = 0; i < PER; ++i) outs[wave][lane * PER + i] = x[i];
      __syncthreads();
      if (wave != 0) return;
      most = -__builtin_huge_valf();
      for (int w = 0; w < DECODE_WAVES; ++w) most = fmaxf(most, sums[w].x);
      const float origin = most > -__builtin_huge_valf() ? most : 0.f;
      sum = 0.f;
      for (int i = 0; i < PER; ++i) x[i] = 0.f;
      for (int w = 0; w < DECODE_WAVES; ++w) {
        const float f = exp2_fast(sums[w].x - origin);
        sum += sums[w].y * f;
        for (int i = 0; i < PER; ++i) x[i] += outs[w][lane * PER + i] * f;
      }
    }
    const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 1.f : sum;
    uint16_t* out = static_cast<uint16_t*>(a.out) + (head0 + row) * D + lane * PER;
    if constexpr (PER == 2) *reinterpret_cast<uint32_t*>(out) = T::pair(x[0] * f, x[1] * f);
    else *out = static_cast<uint16_t>(T::pair(x[0] * f, 0.f));
    if (lane == 0 && a.lse) a.lse[head0 + row] = (most + log2f(sum)) * LN2;
  }
}

}  // namespace fikit
