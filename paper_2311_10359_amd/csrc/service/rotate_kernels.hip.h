// Norm and rotation of query and key heads.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// A head x of D values: y = x w / sqrt(mean(x^2) + epsilon) if it has a weight, then the pairs (a, b) of the first `rotary` values become
// (a cos t - b sin t, b cos t + a sin t), t = position * frequency of the pair.  Held in 32 bits between one reading and one writing.
//
// Two bytes read and two written for a value, ten instructions: bound by memory.  23,171 tokens of 40 heads of 128, 474 MB: 86 us, 5.5 TB/s, past the
// caches, 97 through them (only read past them 94, only written 90); workgroups of 8 waves 6 more.  What a product before has left in the caches, and what
// append and attention behind read there, is worth more up to 128 MB: rotation, append and attention of 8192 tokens take 118 us through the caches
// and 126 past them, of 24,000 tokens 363 and 354.  One token 2.7 us, a launch.  D / 16 lanes hold a head, 16 values each in two chunks of
// eight: those of a pair's two sides are in one lane, so that only the sum of squares crosses lanes.  A wave takes 64 / (D / 16) heads
// of one token at a time, a pass.  An angle counts for all heads of a token and takes 50 instructions, so each lane computes one, or two, and
// reads back those of its pairs from LDS.
//
// An angle is taken in turns: position * frequency / 2 pi in 64 bits, of which the fraction is left; in 32 bits the angle of a position
// of 2^17 would be off by 2^-8.

struct RotateArgs {
  fikit_vectors q, k, q_out, k_out;
  const void* q_weight;
  const void* k_weight;
  const int32_t* positions;
  const float* frequencies;
  const int32_t* status;
  uint32_t q_heads, kv_heads, half;            // half: pairs that are turned
  uint32_t q_passes, passes, per, parts;       // a token's passes, how many a wave takes, and how many waves that is
  uint32_t units;                              // tokens times parts
  float epsilon;
};

constexpr int ROTATE_WAVES = 4;
constexpr int rotate_heads(int d) { return WAVE / (d / 16); }        // of a pass

// cos and sin of so many turns.  The nearest quarter turn is taken off; the rest, up to pi / 4, by the series of sine and cosine, whose
// first terms left out are below 2^-25 there.
__device__ __forceinline__ float2 cos_sin_of_turns(double turns) {
  const float u = static_cast<float>(turns - __builtin_rint(turns));          // -1/2 .. 1/2
  const float quarter = __builtin_rintf(u * 4.f);
  const float x = (u - quarter * 0.25f) * 6.28318530717958648f, z = x * x;
  const float s = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320))));
  const int q = static_cast<int>(quarter) & 3;
  const float cc = q & 1 ? s : c, ss = q & 1 ? c : s;
  return make_float2(q == 1 || q == 2 ? -cc : cc, q >= 2 ? -ss : ss);
}

// The sum over N neighbouring lanes, in each of them.
template <int N>
__device__ __forceinline__ float sum_of_lanes(float v) {
  v += __uint_as_float(dpp_move<0xB1>(__float_as_uint(v)));        // pairs
  v += __uint_as_float(dpp_move<0x4E>(__float_as_uint(v)));        // fours
  if (N >= 8) v += __uint_as_float(dpp_move<0x141>(__float_as_uint(v)));       // mirrored in eight lanes
  if (N >= 16) v += __uint_as_float(dpp_move<0x140>(__float_as_uint(v)));      // mirrored in sixteen
  return v;
}

template <typename T>
__device__ __forceinline__ void rotate_unpack(const u32x4& w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = T::low(w[i]); x[2 * i + 1] = T::high(w[i]); }
}

// PAST: the caches, both ways.
template <typename T, int D, bool NEIGHBOURS, bool PAST>
__global__ __launch_bounds__(ROTATE_WAVES * WAVE) void k_rotate(RotateArgs a) {
  constexpr uint32_t LANES = D / 16, HEADS = WAVE / LANES;
  __shared__ float2 lds[ROTATE_WAVES][D / 2];
  const bool stop = stopped(a.status);         // (the first position is on its way meanwhile)
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE), j = lane % LANES;
  const bool turned = 8 * j < a.half;
  // where the lane's chunks begin in a head
  const uint32_t at_a = NEIGHBOURS || !turned ? 16 * j : 8 * j, at_b = NEIGHBOURS || !turned ? 16 * j + 8 : a.half + 8 * j;
  float2* angles = lds[wave];
  for (uint64_t at = static_cast<uint64_t>(blockIdx.x) * ROTATE_WAVES + wave; at < a.units; at += static_cast<uint64_t>(gridDim.x) * ROTATE_WAVES) {
    const uint32_t unit = static_cast<uint32_t>(at), token = unit / a.parts, part = unit % a.parts;
    const int32_t position = static_cast<int32_t>(uniform(static_cast<uint32_t>(a.positions[token])));
    if (stop) return;
    if (position < 0) continue;
    for (uint32_t p = lane; p < a.half; p += WAVE)
      angles[p] = cos_sin_of_turns(static_cast<double>(position) * static_cast<double>(a.frequencies[p]) * 0.15915494309189533577);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float2 turn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = turned ? angles[8 * j + i] : make_float2(1.f, 0.f);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const uint32_t last = min_u32(part * a.per + a.per, a.passes);
    for (uint32_t pass = part * a.per; pass < last; ++pass) {
      const bool is_q = pass < a.q_passes;
      const uint32_t head = (is_q ? pass : pass - a.q_passes) * HEADS + lane / LANES;
      const fikit_vectors in = is_q ? a.q : a.k, out = is_q ? a.q_out : a.k_out;
      const bool there = head < (is_q ? a.q_heads : a.kv_heads);
      const uint16_t* x_at = static_cast<const uint16_t*>(in.d_data) + token * in.token_stride + head * in.head_stride;
      u32x4 wa = {0, 0, 0, 0}, wb = {0, 0, 0, 0};
      if (there) {
        if constexpr (PAST) {
          wa = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x_at + at_a));
          wb = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x_at + at_b));
        } else {
          wa = *reinterpret_cast<const u32x4*>(x_at + at_a);
          wb = *reinterpret_cast<const u32x4*>(x_at + at_b);
        }
      }
      float x[16];
      rotate_unpack<T>(wa, x);
      rotate_unpack<T>(wb, x + 8);
      const uint16_t* weight = static_cast<const uint16_t*>(is_q ? a.q_weight : a.k_weight);
      if (weight) {
        float w[16];
        rotate_unpack<T>(*reinterpret_cast<const u32x4*>(weight + at_a), w);
        rotate_unpack<T>(*reinterpret_cast<const u32x4*>(weight + at_b), w + 8);
        float sum = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(x[i], x[i], sum);
        sum = sum_of_lanes<LANES>(sum);
        float mean = sum * (1.f / D) + a.epsilon;
        if (!(mean <= 3e38f)) {        // squares of bfloat16 values may pass the largest float: of 2^-72 of them
          sum = 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            x[i] *= 0x1p-72f;
            sum = __builtin_fmaf(x[i], x[i], sum);
          }
          mean = sum_of_lanes<LANES>(sum) * (1.f / D) + a.epsilon * 0x1p-144f;
        }
        const float r = __builtin_amdgcn_rsqf(mean);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
      }
      float y[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int ia = NEIGHBOURS ? 2 * i : i, ib = NEIGHBOURS ? 2 * i + 1 : i + 8;
        y[ia] = __builtin_fmaf(x[ia], turn[i].x, -(x[ib] * turn[i].y));
        y[ib] = __builtin_fmaf(x[ib], turn[i].x, x[ia] * turn[i].y);
      }
      if (!turned)                     // (an infinity times a sine of zero would be none)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = x[i];
      if (there) {
        uint16_t* y_at = static_cast<uint16_t*>(const_cast<void*>(out.d_data)) + token * out.token_stride + head * out.head_stride;
        u32x4 va, vb;
#pragma unroll
        for (int i = 0; i < 4; ++i) { va[i] = T::pair(y[2 * i], y[2 * i + 1]); vb[i] = T::pair(y[8 + 2 * i], y[9 + 2 * i]); }
        if constexpr (PAST) {
          __builtin_nontemporal_store(va, reinterpret_cast<u32x4*>(y_at + at_a));
          __builtin_nontemporal_store(vb, reinterpret_cast<u32x4*>(y_at + at_b));
        } else {
          *reinterpret_cast<u32x4*>(y_at + at_a) = va;
          *reinterpret_cast<u32x4*>(y_at + at_b) = vb;
        }
      }
    }
  }
}

}  // namespace fikit
