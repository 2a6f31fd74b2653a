// What the attention kernels share: value types, conversions, matrix instructions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hip.h"
#include "fikit.h"

namespace fikit {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename To, typename From>
__device__ __forceinline__ To bits_as(From v) {
  static_assert(sizeof(To) == sizeof(From), "same bits");
  return __builtin_bit_cast(To, v);
}

// A 16-bit value type.  `x8`: eight values, an operand of a matrix instruction.  `pair`: two 32-bit values rounded to nearest
// even.  `codes<hi>`: two E4M3 codes, the low or the high ones of a word, times a power of two (exact in the type's range).
// `codes_of_pairs`: the codes of four finite values divided by a power of two, at most 448 then.
struct Bf16 {
  typedef bf16x8 x8;
  static constexpr uint32_t EXP_MASK = 0x7f807f80u, INF = 0x7f80u, ONE = 0x3f80u;
  static constexpr float WEIGHT_BIAS = 0.f;
  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    const bf16x2 v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return bits_as<uint32_t>(v);
  }
  static __device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
  static __device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
  template <bool hi>
  static __device__ __forceinline__ uint32_t codes(uint32_t word, float scale) {
    return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(word), scale, hi));
  }
  static __device__ __forceinline__ uint32_t codes_of_pairs(uint32_t a, uint32_t b, float scale) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, bits_as<bf16x2>(a), scale, false);
    return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, bits_as<bf16x2>(b), scale, true));
  }
  static __device__ __forceinline__ f32x4 mfma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mfma32(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

struct F16 {
  typedef f16x8 x8;
  static constexpr uint32_t EXP_MASK = 0x7c007c00u, INF = 0x7c00u, ONE = 0x3c00u;
  // Weights are held relative to the largest score seen, times 2^7: what is far below it keeps its bits longer.
  static constexpr float WEIGHT_BIAS = 7.f;
  static __device__ __forceinline__ uint32_t pair(float a, float b) {
    const f16x2 v = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
    return bits_as<uint32_t>(v);
  }
  static __device__ __forceinline__ float low(uint32_t v) { return static_cast<float>(bits_as<f16x2>(v)[0]); }
  static __device__ __forceinline__ float high(uint32_t v) { return static_cast<float>(bits_as<f16x2>(v)[1]); }
  template <bool hi>
  static __device__ __forceinline__ uint32_t codes(uint32_t word, float scale) {
    return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(word), scale, hi));
  }
  static __device__ __forceinline__ uint32_t codes_of_pairs(uint32_t a, uint32_t b, float scale) {
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, bits_as<f16x2>(a), scale, false);
    return bits_as<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, bits_as<f16x2>(b), scale, true));
  }
  static __device__ __forceinline__ f32x4 mfma16(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ f32x16 mfma32(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// A value that is the same in the whole wave, where the compiler cannot know it.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(v))); }

// 2^(x - 127), x = 1 .. 254.
__device__ __forceinline__ float power_of(uint32_t x) { return __uint_as_float(x << 23); }

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The sum and the maximum over the wave, by data-parallel-primitive moves (see wave_incl_scan_u32).
__device__ __forceinline__ uint32_t sum_over_wave(uint32_t v) { return read_lane_u32(wave_incl_scan_u32(v), WAVE - 1); }
__device__ __forceinline__ uint32_t max_over_wave(uint32_t v) {
  v = max_u32(v, dpp_or_zero<0x111, 0xf>(v));
  v = max_u32(v, dpp_or_zero<0x112, 0xf>(v));
  v = max_u32(v, dpp_or_zero<0x114, 0xf>(v));
  v = max_u32(v, dpp_or_zero<0x118, 0xf>(v));
  v = max_u32(v, dpp_or_zero<0x142, 0xa>(v));
  v = max_u32(v, dpp_or_zero<0x143, 0xc>(v));
  return read_lane_u32(v, WAVE - 1);
}

// Errors are written, success is not: see fikit.h.
// (Read once and through the caches: what this kernel's other workgroups write there may be seen or not.)
__device__ __forceinline__ bool stopped(const int32_t* status) {
  return __hip_atomic_load(status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT) != FIKIT_OK;
}

}  // namespace fikit
