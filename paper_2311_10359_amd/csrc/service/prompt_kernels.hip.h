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
//
// Bound by the rate of matrix instructions together with the vector instructions of the softmax, five for each score: heads of 128 take
// 32 products of 32 clocks for a wave's 64 tokens, and 130 vector instructions, 32 of them exponentials at twice the time.  So both are made at
// once, the scores of a tile while the one before is weighed, in an order that is written down (weigh_and_go_on); one after the other took
// 778 us where this takes 500.  One prompt of 8192 tokens, 32 query and 8 key heads of 128: 485 to 530 us from card to card, 1.04 to 1.13
// PFLOP/s of the 1.6 that a large product reaches; the matrix unit is busy for 65 % of the time, at the clock of 1.7 GHz that the power
// allows.  (That is in a row, from the 60th call on; of calls that begin on an idle card the first three take 510, the next ones up to 670
// while the clock settles, the 20th 540.)  Heads of 64 have half the products for as many vector instructions, about 660 clocks of these
// for 512 of those, so the vector unit binds: 4 prompts of 4096 tokens, 16 heads: 155 to 162 us, 0.85 to 0.89 PFLOP/s.  24 prompts of 1 to
// 1788 tokens: 83 to 90 us, 0.68 to 0.73 PFLOP/s, with tiles that are seen in part and, for each 128 rows, 5 us before and behind the
// tiles, mostly latency.  5 of 3 to 49 tokens: 5.4 us, a launch and four loads that depend on each other.

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

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// 16 bytes per lane, to `to` and behind it in the order of the lanes; zeros for what lies behind the end of `from`.
__device__ __forceinline__ void load_to_lds(bounded from, uint32_t at, lds_char* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, static_cast<int>(at), 0, 0, 0);
}
__device__ __forceinline__ u32x4 read_row(const lds_char* at) { return *(const __attribute__((address_space(3))) u32x4*)at; }
// Of 16 lanes each that point at four rows of 16 values, lane l receives value l of the four rows.
__device__ __forceinline__ u32x2 read_transposed(lds_char* at) {
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

template <typename T, int D>
struct PromptWave {              // what a wave holds of its 32 rows; a lane of row lane % 32
  static constexpr uint32_t ROW = D * 2, TILE = PROMPT_KEYS * ROW;
  typename T::x8 q[D / 16];
  f32x16 s[2];                   // scores of the next tile, before scaling
  f32x16 acc[D / 32];
  float m, l;                    // reference of the weights (of scores times log2 e), sum over this lane's tokens
  float most;                    // largest of this lane's scores, scaled
  float scale;
  uint32_t row;
  uint32_t key_at, val_at;       // where this lane reads in a tile: the first place, from which the others differ in single bits

  __device__ __forceinline__ void set_up(const PromptArgs& a, uint32_t start, uint32_t length, uint32_t row0, uint32_t head) {
    const uint32_t lane = lane_id(), col = lane % 32, half = lane / 32;
    // The largest score is found, and what is not seen masked, before scaling: that takes a scale above zero.
    const bool flip = a.scale < 0.f, none = a.scale == 0.f;
    scale = none ? LOG2E : fabsf(a.scale) * LOG2E;
    row = row0 + col;
    const uint16_t* src = static_cast<const uint16_t*>(a.q.d_data) + (start + static_cast<uint64_t>(min_u32(row, length - 1))) * a.q.token_stride +
                          head * a.q.head_stride + half * 8;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      u32x4 x = *reinterpret_cast<const u32x4*>(src + j * 16);
      if (flip) x ^= 0x80008000u;
      if (none) x = u32x4{0, 0, 0, 0};
      q[j] = bits_as<typename T::x8>(x);
    }
    // (a row's piece 2 j + half is stored at (2 j + half) ^ swizzle, value piece 4 d + .. likewise)
    const uint32_t l16 = lane % 16, r = half * 4 + l16 / 4;
    key_at = col * ROW + (half ^ key_swizzle<D>(col)) * 16;
    val_at = r * ROW + ((2 * (lane / 16 % 2) + l16 % 4 / 2) ^ value_swizzle<D>(r)) * 16 + l16 % 2 * 8;
  }
  __device__ __forceinline__ void start() {
    m = -__builtin_huge_valf();
    l = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  }
  __device__ __forceinline__ u32x4 key(const lds_char* keys, int j, int t) const { return read_row(keys + (key_at ^ j * 32) + t * 32 * ROW); }
  // The first operands of a tile's scores, read before what stands between them and the products.
  u32x4 first_keys[4];
  __device__ __forceinline__ void read_ahead(const lds_char* keys) {
#pragma unroll
    for (int i = 0; i < 4; ++i) first_keys[i] = key(keys, i / 2, i % 2);
  }
  __device__ __forceinline__ void scores(const lds_char* keys, bool ahead) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (j == 0)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
        s[t] = T::mfma32(bits_as<typename T::x8>(ahead && j < 2 ? first_keys[2 * j + t] : key(keys, j, t)), q[j], s[t]);
      }
  }
  __device__ __forceinline__ void mask(uint32_t token0) {
    const uint32_t half = lane_id() / 32;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (token0 + t * 32 + r / 4 * 8 + half * 4 + r % 4 > row) s[t][r] = -__builtin_huge_valf();
  }
  __device__ __forceinline__ void find_most() {
    float x = s[0][0];
#pragma unroll
    for (int i = 1; i < 31; i += 2) x = fmaxf(fmaxf(x, s[i / 16][i % 16]), s[(i + 1) / 16][(i + 1) % 16]);
    most = fmaxf(x, s[1][15]) * scale;
  }
  __device__ __forceinline__ void raise() {
    if (ballot(most > m + (PROMPT_SLACK + T::WEIGHT_BIAS))) {
      const float both = fmaxf(most, __shfl_xor(most, 32, WAVE));
      const float raised = fmaxf(m, both - T::WEIGHT_BIAS);
      const float down = raised > -__builtin_huge_valf() ? exp2_fast(m - raised) : 1.f;
      m = raised;
      l *= down;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) acc[d] *= down;
    }
  }
  // Weights are rounded to 16 bits, as an operand of the matrix instruction has to be, and summed before that: error against 64 bits
  // 0.0019 to 0.0021 (bfloat16) and 0.00021 (float16); the rounding of the output is 0.0015 and 0.00018.  What rounding leaves as a second
  // operand, as in a decode step, brings it down to the output's and is half more products of the kernel that products bind: 8192 tokens
  // 514 -> 712 us, 4 prompts of 4096 with heads of 64 162 -> 223, 24 ragged ones 88 -> 109, 64 of 500 142 -> 165.
  __device__ __forceinline__ void weigh(typename T::x8 (&weights)[4]) {
    const float origin = m > -__builtin_huge_valf() ? m : 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = exp2_fast(__builtin_fmaf(s[t][8 * u + 2 * i], scale, -origin)), y = exp2_fast(__builtin_fmaf(s[t][8 * u + 2 * i + 1], scale, -origin));
          l += x;
          l += y;
          p[i] = T::pair(x, y);
        }
        weights[2 * t + u] = bits_as<typename T::x8>(p);
      }
  }
  __device__ __forceinline__ u32x4 value(lds_char* vals, int step, int d) const {
    const u32x2 x = read_transposed(vals + (val_at ^ d * 64) + step * 16 * ROW), y = read_transposed(vals + (val_at ^ d * 64) + (step * 16 + 8) * ROW);
    return u32x4{x[0], x[1], y[0], y[1]};
  }
  __device__ __forceinline__ void sum(lds_char* vals, const typename T::x8 (&weights)[4]) {
#pragma unroll
    for (int step = 0; step < 4; ++step)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) acc[d] = T::mfma32(bits_as<typename T::x8>(value(vals, step, d)), weights[step], acc[d]);
  }
  // The same where a weight of zero may meet what is not finite: such values are left out of the product, and the rows that do
  // see them are found with products of ones.
  __device__ __forceinline__ void sum_with_care(lds_char* vals, const typename T::x8 (&weights)[4], uint32_t token0) {
    const uint32_t half = lane_id() / 32;
    for (int step = 0; step < 4; ++step) {
      u32x4 seen;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t bits = 0;
        for (int b = 0; b < 2; ++b) {
          const uint32_t j = 2 * i + b, token = token0 + step * 16 + j / 4 * 8 + half * 4 + j % 4;
          if (token <= row) bits |= T::ONE << (16 * b);
        }
        seen[i] = bits;
      }
      const typename T::x8 weight = step == 0 ? weights[0] : step == 1 ? weights[1] : step == 2 ? weights[2] : weights[3];
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        const u32x4 v = value(vals, step, d);
        u32x4 clean;
#pragma unroll
        for (int i = 0; i < 4; ++i) clean[i] = v[i] & ~not_finite<T>(v[i]);
        acc[d] = T::mfma32(bits_as<typename T::x8>(clean), weight, acc[d]);
        for (uint32_t kind = 0; kind < 3; ++kind) {      // infinity, -infinity, NaN
          u32x4 ones;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t bits = 0;
            for (int b = 0; b < 2; ++b) {
              const uint32_t x = v[i] >> (16 * b) & 0xffffu;
              const uint32_t is = x == T::INF ? 0 : x == (T::INF | 0x8000u) ? 1 : (x & T::INF) == T::INF ? 2 : 3;
              if (is == kind) bits |= T::ONE << (16 * b);
            }
            ones[i] = bits;
          }
          f32x16 c;
#pragma unroll
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
  // Weighs and sums one tile and makes the scores of the next, matrix instructions and others in turn: the matrix unit is busy for
  // 32 clocks with one, of which the wave needs 16, and the weights of a tile take as long as its products.
  __device__ __forceinline__ void weigh_and_go_on(const lds_char* next_keys, lds_char* vals) {
    __builtin_amdgcn_sched_barrier(0);
    typename T::x8 weights[4];
    weigh(weights);
    scores(next_keys, true);
    sum(vals, weights);
    find_most();
    asm volatile("" : "+v"(l), "+v"(most));      // (made here and not where they are next needed)
    constexpr int MFMA = 0x8, READ = 0x100, OTHER = 0x2, HALF = D / 16;
    __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
    __builtin_amdgcn_sched_group_barrier(OTHER, 8, 0);
#pragma unroll
    for (int i = 0; i < 2 * HALF - 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
      __builtin_amdgcn_sched_group_barrier(OTHER, 64 / (2 * HALF), 0);
      __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
      __builtin_amdgcn_sched_group_barrier(OTHER, 64 / (2 * HALF), 0);
      __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
    }
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
      __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
      __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
      __builtin_amdgcn_sched_group_barrier(OTHER, 48 / HALF, 0);
    }
#pragma unroll
    for (int i = 0; i < HALF; ++i) {
      __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
      __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
      __builtin_amdgcn_sched_group_barrier(OTHER, 16 / HALF, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // A lane has four values of its row here and there, so rows go through LDS, half of each through `to0` and `to1` (32 * D bytes that only
  // this wave uses), and leave 16 bytes a lane, 128 or 64 of a row together.  (Straight from the registers, 8 bytes a lane: 166 us
  // instead of 150 for 64 prompts of 500 tokens.)
  __device__ __forceinline__ void write(const PromptArgs& a, uint32_t start, uint32_t length, uint32_t head, lds_char* to0, lds_char* to1) const {
    const float sum = l + __shfl_xor(l, 32, WAVE);
    const float f = sum > 0.f ? 1.f / sum : sum == 0.f ? 1.f : sum;
    const uint32_t lane = lane_id(), half = lane / 32, col = lane % 32, row0 = row - col;
    if (a.lse && half == 0 && row < length) a.lse[(start + static_cast<uint64_t>(row)) * a.q_heads + head] = (m + log2f(sum)) * LN2;
    constexpr uint32_t PIECES = D / 16, ROWS = WAVE / PIECES;       // (of half a row)
    const auto place = [](uint32_t r, uint32_t piece) { return r * D + (piece ^ (D == 128 ? (r >> 1) & 7 : (r >> 2) & 3)) * 16; };
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32x2 x = {T::pair(acc[d][4 * r] * f, acc[d][4 * r + 1] * f), T::pair(acc[d][4 * r + 2] * f, acc[d][4 * r + 3] * f)};
        *(__attribute__((address_space(3))) u32x2*)((d < D / 64 ? to0 : to1) + place(col, d % (D / 64) * 4 + r) + half * 8) = x;
      }
    const uint32_t piece = lane % PIECES, r0 = lane / PIECES;
    uint16_t* out = static_cast<uint16_t*>(a.out) + ((start + static_cast<uint64_t>(row0 + r0)) * a.q_heads + head) * D + piece * 8;
    const uint64_t stride = static_cast<uint64_t>(a.q_heads) * D * ROWS;
#pragma unroll
    for (uint32_t i = 0; i < 32 / ROWS; ++i) {
      const u32x4 x = read_row(to0 + place(i * ROWS + r0, piece)), y = read_row(to1 + place(i * ROWS + r0, piece));
      if (row0 + i * ROWS + r0 < length) {
        *reinterpret_cast<u32x4*>(out + i * stride) = x;
        *reinterpret_cast<u32x4*>(out + i * stride + D / 2) = y;
      }
    }
  }
  __device__ __forceinline__ bool finite() const {
    float z = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) z = __builtin_fmaf(acc[d][r], 0.f, z);
    return z == 0.f;
  }
};

// Which rows a workgroup takes.  Later rows see more, so up to PROMPT_ORDERED prompts the work is handed out by the rows'
// place in their prompt, the last ones first: item i is in level L (rows L * rows .. of a prompt) if C(L + 1) <= i < C(L), C(L) =
// sum over prompts of max(0, slots - L).  For more prompts, which fill the chip many times over, slot by slot from the back; prompt
// p owns the slots from offsets[p] / rows + p on, enough for its rows and found without a list.
constexpr uint32_t PROMPT_ORDERED = 64;
// False if the offsets cannot be; `stop`: an earlier call has failed (asked here, so that it is on its way together with the offsets).
__device__ __forceinline__ bool prompt_find(const PromptArgs& a, uint32_t rows, uint32_t item, uint32_t* start, uint32_t* length, uint32_t* first, bool* stop) {
  if (a.n_prompts <= PROMPT_ORDERED) {
    const uint32_t lane = lane_id(), p = min_u32(lane, a.n_prompts - 1);
    const uint32_t from = static_cast<uint32_t>(a.offsets[p]), to = static_cast<uint32_t>(a.offsets[p + 1]);
    *stop = stopped(a.status);
    const bool good = from <= to && to <= a.n_tokens;
    if (ballot(!good)) return false;
    const uint32_t slots = lane < a.n_prompts ? (to - from + rows - 1) / rows : 0;
    // From below: C is convex, so the line through C(level) and C(level + 1) = C(level) - here never leads too far.
    uint32_t level = 0, left = sum_over_wave(slots), here;
    if (left <= item) { *length = *first = *start = 0; return true; }
    uint64_t these;
    for (;;) {
      these = ballot(slots > level);
      here = static_cast<uint32_t>(__builtin_popcountll(these));
      if (left - here <= item) break;
      const float step = (static_cast<float>(left - item - 1) + 0.5f) * (0.999999f * __builtin_amdgcn_rcpf(static_cast<float>(here)));
      level += max_u32(uniform(static_cast<uint32_t>(step)), 1);
      left = sum_over_wave(slots > level ? slots - level : 0);
    }
    for (uint32_t skip = item - (left - here); skip > 0; --skip) these &= these - 1;
    const uint32_t owner = uniform(static_cast<uint32_t>(__builtin_ctzll(these)));
    *start = read_lane_u32(from, owner);
    *length = read_lane_u32(to - from, owner);
    *first = level * rows;
    return true;
  }
  *stop = stopped(a.status);
  const uint32_t slot = a.slots - 1 - item;
  uint32_t prompt = 0;
  for (uint32_t hi = a.n_prompts; hi - prompt > 1;) {
    const uint32_t mid = prompt + (hi - prompt) / 2;
    if (static_cast<uint32_t>(a.offsets[mid]) / rows + mid <= slot) prompt = mid; else hi = mid;
  }
  const uint32_t from = static_cast<uint32_t>(a.offsets[prompt]), to = static_cast<uint32_t>(a.offsets[prompt + 1]);
  if (from > to || to > a.n_tokens) return false;
  *start = uniform(from);
  *length = uniform(to - from);
  *first = uniform((slot - (from / rows + prompt)) * rows);
  return true;
}

// This thread's 16-byte pieces of a tile of keys or of values, which go from global memory straight to LDS.
template <int D, int WAVES>
struct PromptFill {
  static constexpr uint32_t PIECES = D / 8, ROW = D * 2;
  static constexpr int LOADS = PROMPT_KEYS * PIECES / (WAVES * WAVE);
  const char* from;
  uint64_t stride;               // of a token, in bytes
  uint32_t off[LOADS];
  uint32_t wave;

  __device__ __forceinline__ void set_up(const fikit_vectors& x, uint32_t start, uint32_t head, uint32_t wave_, bool values) {
    wave = wave_;
    from = reinterpret_cast<const char*>(static_cast<const uint16_t*>(x.d_data) + start * x.token_stride + head * x.head_stride);
    stride = x.token_stride * 2;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t c = (i * WAVES + wave) * WAVE + lane_id(), r = c / PIECES, piece = c % PIECES;
      off[i] = r * static_cast<uint32_t>(stride) + (piece ^ (values ? value_swizzle<D>(r) : key_swizzle<D>(r))) * 16;
    }
  }
  // (rows behind the prompt's end become zeros)
  __device__ __forceinline__ void load(uint32_t tile, uint32_t length, lds_char* to) const {
    const uint32_t rows = min_u32(length - tile * PROMPT_KEYS, PROMPT_KEYS);
    const bounded at = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from + tile * (PROMPT_KEYS * stride)), 0,
                                                         static_cast<int>((rows - 1) * static_cast<uint32_t>(stride) + ROW), 0x00027000);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_to_lds(at, off[i], to + (i * WAVES + wave) * WAVE * 16);
  }
};

// What this wave has asked for is in LDS, and so is what the others have.
__device__ __forceinline__ void prompt_arrive() {
  __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
  __syncthreads();
}

// A workgroup's rows where values that are not finite follow tokens: one tile after the other, nothing ahead of time.
template <typename T, int D, int WAVES>
__device__ __attribute__((noinline)) void prompt_with_care(PromptArgs a, uint32_t start, uint32_t length, uint32_t first, uint32_t head, uint32_t kv_head,
                                                           lds_char* keys, lds_char* vals) {
  constexpr uint32_t ROWS = WAVES * PROMPT_WAVE_ROWS;
  const uint32_t wave = uniform(threadIdx.x / WAVE), row0 = first + wave * PROMPT_WAVE_ROWS;
  const uint32_t tiles = (min_u32(first + ROWS, length) + PROMPT_KEYS - 1) / PROMPT_KEYS;
  PromptFill<D, WAVES> k, v;
  k.set_up(a.k, start, kv_head, wave, false);
  v.set_up(a.v, start, kv_head, wave, true);
  PromptWave<T, D> w;
  w.set_up(a, start, length, row0, head);
  w.start();
  for (uint32_t tile = 0; tile < tiles; ++tile) {
    __syncthreads();
    k.load(tile, length, keys);
    v.load(tile, length, vals);
    prompt_arrive();
    const uint32_t token0 = tile * PROMPT_KEYS;
    if (token0 > row0 + PROMPT_WAVE_ROWS - 1) continue;
    typename T::x8 weights[4];
    w.scores(keys, false);
    w.mask(token0);
    w.find_most();
    w.raise();
    w.weigh(weights);
    w.sum_with_care(vals, weights, token0);
  }
  __syncthreads();
  w.write(a, start, length, head, keys + wave * (32 * D), vals + wave * (32 * D));
}

// Heads of 64 leave room for a third workgroup on a compute unit (4 prompts of 4096 tokens: 155 to 162 us; with two 168, with four, which spill, 171).
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * WAVE, D == 64 ? 3 : 2) void k_prompt(PromptArgs a) {
  constexpr uint32_t ROWS = WAVES * PROMPT_WAVE_ROWS, TILE = PROMPT_KEYS * D * 2;
  // Keys and values of two tiles.  (Arrays of their own: the compiler sees that a tile that is read is not one that is being filled,
  // and does not wait for the latter.)
  __shared__ __align__(1024) char lds_k0[TILE], lds_k1[TILE], lds_v0[TILE], lds_v1[TILE];
  lds_char *const k0 = (lds_char*)lds_k0, *const k1 = (lds_char*)lds_k1, *const v0 = (lds_char*)lds_v0, *const v1 = (lds_char*)lds_v1;
  const uint32_t wave = uniform(threadIdx.x / WAVE);
  // neighbours in the grid go to different dies: those of one key head are kept on few of them
  const uint32_t place = blockIdx.x % a.q_heads;
  const uint32_t kv_head = place % a.kv_heads, head = kv_head * (a.q_heads / a.kv_heads) + place / a.kv_heads;
  uint32_t start, length, first;
  bool stop;
  if (!prompt_find(a, ROWS, blockIdx.x / a.q_heads, &start, &length, &first, &stop)) {
    if (threadIdx.x == 0 && !stop) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  if (blockIdx.x == 0 && !stop) {
    bool bad = a.offsets[0] != 0 || static_cast<uint32_t>(a.offsets[a.n_prompts]) != a.n_tokens;
    for (uint32_t p = threadIdx.x; p < a.n_prompts; p += WAVES * WAVE) bad |= a.offsets[p] > a.offsets[p + 1];
    if (bad) *a.status = FIKIT_INVALID_ARG;
  }
  if (stop || first >= length) return;
  const uint32_t row0 = first + wave * PROMPT_WAVE_ROWS;
  const uint32_t tiles = (min_u32(first + ROWS, length) + PROMPT_KEYS - 1) / PROMPT_KEYS;

  PromptFill<D, WAVES> k, v;
  k.set_up(a.k, start, kv_head, wave, false);
  v.set_up(a.v, start, kv_head, wave, true);
  k.load(0, length, k0);
  if (tiles > 1) k.load(1, length, k1);
  v.load(0, length, v0);

  PromptWave<T, D> w;
  w.set_up(a, start, length, row0, head);
  // Tile i's scores are made while tile i - 1 is weighed and summed.  Before each tile: its values and the next one's keys have
  // arrived, and what their successors replace is no longer read.
  static_assert(ROWS == 2 * PROMPT_KEYS, "tiles that some rows see in part: the last two");
  const uint32_t full = first / PROMPT_KEYS;      // tiles that all rows of the workgroup see whole, an even number
  if (row0 >= length) {      // a wave without rows fills LDS for the others
    prompt_arrive();
    for (uint32_t tile = 0; tile < full; tile += 2) {
      prompt_arrive();
      k.load(tile + 2, length, k0);
      v.load(tile + 1, length, v1);
      prompt_arrive();
      if (tile + 3 < tiles) k.load(tile + 3, length, k1);
      v.load(tile + 2, length, v0);
    }
    prompt_arrive();
    if (full + 1 < tiles) {
      v.load(full + 1, length, v1);
      prompt_arrive();
    }
    if (uniform(__syncthreads_or(false)) != 0) prompt_with_care<T, D, WAVES>(a, start, length, first, head, kv_head, k0, v0);
    return;
  }
  w.start();
  prompt_arrive();
  w.scores(k0, false);
  w.find_most();
  for (uint32_t tile = 0; tile < full; tile += 2) {
    prompt_arrive();
    w.read_ahead(k1);
    k.load(tile + 2, length, k0);
    v.load(tile + 1, length, v1);
    w.raise();
    w.weigh_and_go_on(k1, v0);
    prompt_arrive();
    w.read_ahead(k0);
    if (tile + 3 < tiles) k.load(tile + 3, length, k1);
    v.load(tile + 2, length, v0);
    w.raise();
    w.weigh_and_go_on(k0, v1);
  }
  prompt_arrive();
  if (full + 1 < tiles) v.load(full + 1, length, v1);
  {
    typename T::x8 weights[4];
    w.mask(full * PROMPT_KEYS);
    w.find_most();
    w.raise();
    w.weigh(weights);
    w.sum(v0, weights);
  }
  if (full + 1 < tiles) {
    if (row0 >= (full + 1) * PROMPT_KEYS) {
      w.read_ahead(k1);
      w.scores(k1, true);
      w.mask((full + 1) * PROMPT_KEYS);
      w.find_most();
      w.raise();
    }
    prompt_arrive();
    if (row0 >= (full + 1) * PROMPT_KEYS) {
      typename T::x8 weights[4];
      w.weigh(weights);
      w.sum(v1, weights);
    }
  }
  // Weights of zero have met whatever values follow a row's token.  If that has left anything that is not finite, which only values
  // that are not finite can, all of it is done again with care.  (Written first all the same: results that live across a call are spilled.)
  const uint32_t again = uniform(__syncthreads_or(!w.finite()));
  w.write(a, start, length, head, k0 + wave * (32 * D), k1 + wave * (32 * D));
  if (again) prompt_with_care<T, D, WAVES>(a, start, length, first, head, kv_head, k0, v0);
}

}  // namespace fikit
