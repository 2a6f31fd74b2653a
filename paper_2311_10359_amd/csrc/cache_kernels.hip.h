// The paged 8-bit cache: the plan of a step and the append of new keys and values.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// ---- plan -------------------------------------------------------------------------------------------------------
//
// With B = tokens per block, c cached and a added tokens of a request: it holds ceil(c / B) blocks, needs ceil((c + a) / B), and
// its new tokens are cut into floor((c + a - 1) / B) - floor(c / B) + 1 pieces (none if a = 0).  Three prefix sums over the
// requests (tokens, new blocks, pieces) say where everything of a request begins; then each new token finds its request by
// a search in the token sums and writes its slot, and those that open a block or a piece write these, with no word from one to
// another.

struct PlanArgs {
  const int32_t* cached;
  const int32_t* added;
  int32_t* table;
  const int32_t* free_blocks;
  int32_t* lengths;
  int32_t* token_offsets;
  int64_t* slots;
  int4* pieces;
  int32_t* counts;
  int32_t* status;
  int2* bases;              // per request: new blocks and pieces of those before it
  uint32_t n_requests, n_tokens, table_width, n_free, room;
  uint32_t shift;           // of the block length
};

struct PlanSums {
  uint64_t tokens;
  uint32_t blocks, pieces;  // (at most as many as tokens that fit 31 bits, or the call has failed)
};

constexpr int PLAN_THREADS = 1024;

// What request r adds to the sums; false if its lengths cannot be.
__device__ __forceinline__ bool plan_request(const PlanArgs& a, int64_t cached, int64_t added, PlanSums* s) {
  const int64_t length = cached + added;
  if (cached < 0 || added < 0 || length > INT32_MAX || length > static_cast<int64_t>(a.table_width) << a.shift) return false;
  const int64_t block = int64_t{1} << a.shift;
  s->tokens += static_cast<uint64_t>(added);
  s->blocks += static_cast<uint32_t>(((length + block - 1) >> a.shift) - ((cached + block - 1) >> a.shift));
  if (added > 0) s->pieces += static_cast<uint32_t>(((length - 1) >> a.shift) - (cached >> a.shift) + 1);
  return true;
}

// Prefix sums over all requests by one workgroup, a run of consecutive requests per thread.
__global__ __launch_bounds__(PLAN_THREADS) void k_plan_sums(PlanArgs a) {
  __shared__ uint64_t wave_tokens[PLAN_THREADS / WAVE];
  __shared__ uint32_t wave_blocks[PLAN_THREADS / WAVE], wave_pieces[PLAN_THREADS / WAVE];
  __shared__ int32_t bad;
  if (stopped(a.status)) return;
  const uint32_t per = (a.n_requests + PLAN_THREADS - 1) / PLAN_THREADS;
  const uint32_t first = min_u32(threadIdx.x * per, a.n_requests), last = min_u32(first + per, a.n_requests);
  if (threadIdx.x == 0) bad = 0;
  PlanSums mine{0, 0, 0};
  bool ok = true;
  for (uint32_t r = first; r < last; ++r) ok &= plan_request(a, a.cached[r], a.added[r], &mine);
  // inclusive sums over the wave, then over the waves
  PlanSums run = mine;
  for (int d = 1; d < WAVE; d <<= 1) {
    const uint64_t t = shfl_up_u64(run.tokens, d);
    const uint32_t b = __shfl_up(run.blocks, d, WAVE), p = __shfl_up(run.pieces, d, WAVE);
    if (lane_id() >= static_cast<uint32_t>(d)) { run.tokens += t; run.blocks += b; run.pieces += p; }
  }
  const uint32_t wave = threadIdx.x / WAVE;
  if (lane_id() == WAVE - 1) { wave_tokens[wave] = run.tokens; wave_blocks[wave] = run.blocks; wave_pieces[wave] = run.pieces; }
  __syncthreads();
  if (!ok) bad = 1;
  PlanSums before{0, 0, 0}, total{0, 0, 0};
  for (uint32_t w = 0; w < PLAN_THREADS / WAVE; ++w) {
    if (w < wave) { before.tokens += wave_tokens[w]; before.blocks += wave_blocks[w]; before.pieces += wave_pieces[w]; }
    total.tokens += wave_tokens[w]; total.blocks += wave_blocks[w]; total.pieces += wave_pieces[w];
  }
  __syncthreads();
  const int32_t error = bad || total.tokens != a.n_tokens ? FIKIT_INVALID_ARG : total.blocks > a.n_free ? FIKIT_CACHE_FULL : FIKIT_OK;
  if (error != FIKIT_OK) {
    if (threadIdx.x == 0) *a.status = error;
    return;
  }
  PlanSums at{before.tokens + run.tokens - mine.tokens, before.blocks + run.blocks - mine.blocks, before.pieces + run.pieces - mine.pieces};
  for (uint32_t r = first; r < last; ++r) {
    const int32_t cached = a.cached[r], added = a.added[r];
    a.lengths[r] = cached + added;
    a.token_offsets[r] = static_cast<int32_t>(at.tokens);
    a.bases[r] = make_int2(static_cast<int32_t>(at.blocks), static_cast<int32_t>(at.pieces));
    plan_request(a, cached, added, &at);
  }
  if (threadIdx.x == 0) {
    a.token_offsets[a.n_requests] = static_cast<int32_t>(a.n_tokens);
    a.counts[0] = static_cast<int32_t>(total.blocks);
    a.counts[1] = static_cast<int32_t>(total.pieces);
  }
}

// The last request that begins at token t or before; lo begins so, hi does not.
__device__ __forceinline__ uint32_t plan_find(const int32_t* offsets, uint32_t lo, uint32_t hi, uint32_t t) {
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (static_cast<uint32_t>(offsets[mid]) <= t) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ void plan_token(const PlanArgs& a, uint32_t t, uint32_t r) {
  const uint32_t block_tokens = 1u << a.shift;
  const uint32_t cached = static_cast<uint32_t>(a.cached[r]), length = cached + static_cast<uint32_t>(a.added[r]);
  const uint32_t index = t - static_cast<uint32_t>(a.token_offsets[r]);
  const uint32_t place = cached + index, page = place >> a.shift, at = place & (block_tokens - 1);
  const uint32_t held = (cached + block_tokens - 1) >> a.shift;
  const int2 base = a.bases[r];
  int32_t* entry = a.table + static_cast<uint64_t>(r) * a.table_width + page;
  const int32_t block = page >= held ? a.free_blocks[base.x + (page - held)] : *entry;
  if (at == 0) *entry = block;      // (a block that begins at a new token is a new one)
  if (a.slots) a.slots[t] = static_cast<int64_t>(block) * block_tokens + at;
  if (at == 0 || index == 0)
    a.pieces[base.y + (page - (cached >> a.shift))] = make_int4(block, static_cast<int32_t>(t), static_cast<int32_t>(at),
                                                               static_cast<int32_t>(min_u32(block_tokens - at, length - place)));
}

__global__ __launch_bounds__(256) void k_plan_tokens(PlanArgs a) {
  if (stopped(a.status)) return;
  const uint32_t t = blockIdx.x * 256 + threadIdx.x;
  if (t < a.n_tokens) plan_token(a, t, plan_find(a.token_offsets, 0, a.n_requests, t));
  const uint32_t n_pieces = static_cast<uint32_t>(a.counts[1]);
  for (uint64_t i = static_cast<uint64_t>(n_pieces) + t; i < a.room; i += static_cast<uint64_t>(gridDim.x) * 256)
    a.pieces[i] = make_int4(-1, -1, -1, -1);
}

// ---- append -----------------------------------------------------------------------------------------------------
//
// A piece lies in one block, so the largest magnitude of its values, the block's exponent and the codes belong to one
// workgroup per piece, head, and keys or values.  Memory bound: 2 bytes read and 1 written per value.

struct AppendArgs {
  fikit_cache cache;
  fikit_vectors k, v;
  const int4* pieces;
  int32_t* status;
  uint32_t n_tokens;
};

constexpr int APPEND_THREADS = 256;

// Two values as codes, in the low 16 bits.
__device__ __forceinline__ uint32_t codes_of(float a, float b) {
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}

// What is not finite becomes NaN, whose code is 0x7f with either sign.
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) < __builtin_huge_valf() ? x : __builtin_nanf(""); }

// The smallest exponent byte x >= 1 with most <= 448 * 2^(x - 127); 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t exponent_for(float most) {
  const uint32_t bits = __float_as_uint(most);
  const int32_t x = static_cast<int32_t>(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return x < 1 ? 1u : static_cast<uint32_t>(x);
}

template <typename T, int D, int CHUNKS>   // CHUNKS: eight values each that a thread holds
__global__ __launch_bounds__(APPEND_THREADS) void k_cache_append(AppendArgs a) {
  __shared__ float wave_most[APPEND_THREADS / WAVE];
  if (stopped(a.status)) return;
  const int4 piece = a.pieces[blockIdx.x];
  if (piece.x == -1) return;
  const uint32_t head = blockIdx.y, block_tokens = a.cache.block_tokens;
  const uint32_t block = static_cast<uint32_t>(piece.x), first = static_cast<uint32_t>(piece.y), at = static_cast<uint32_t>(piece.z),
                 count = static_cast<uint32_t>(piece.w);
  if (block >= a.cache.n_blocks || at >= block_tokens || count == 0 || count > block_tokens - at || first >= a.n_tokens ||
      count > a.n_tokens - first) {
    if (threadIdx.x == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  const bool values = blockIdx.z != 0;
  const fikit_vectors in = values ? a.v : a.k;
  const uint16_t* x = static_cast<const uint16_t*>(in.d_data) + first * in.token_stride + head * in.head_stride;
  const uint64_t unit = static_cast<uint64_t>(block) * a.cache.kv_heads + head;
  uint8_t* codes = (values ? a.cache.d_v : a.cache.d_k) + unit * block_tokens * D;
  uint8_t* exponent = (values ? a.cache.d_v_exp : a.cache.d_k_exp) + unit;
  const uint32_t old = at > 0 ? min_u32(*exponent, 254u) : 0;

  constexpr uint32_t PER_TOKEN = D / 8;
  u32x4 held[CHUNKS];
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const uint32_t c = i * APPEND_THREADS + threadIdx.x, token = c / PER_TOKEN;
    held[i] = u32x4{0, 0, 0, 0};
    if (token < count) held[i] = *reinterpret_cast<const u32x4*>(x + token * in.token_stride + c % PER_TOKEN * 8);
  }
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
    for (int j = 0; j < 4; ++j) {
      const float lo = fabsf(T::low(held[i][j])), hi = fabsf(T::high(held[i][j]));
      most = fmaxf(most, lo < __builtin_huge_valf() ? lo : 0.f);
      most = fmaxf(most, hi < __builtin_huge_valf() ? hi : 0.f);
    }
  for (int d = 1; d < WAVE; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, WAVE));
  if (lane_id() == 0) wave_most[threadIdx.x / WAVE] = most;
  __syncthreads();
  most = fmaxf(fmaxf(wave_most[0], wave_most[1]), fmaxf(wave_most[2], wave_most[3]));
  uint32_t chosen = exponent_for(most);
  if (old > chosen) chosen = old;
  const float inverse = power_of(254 - chosen);

#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const uint32_t c = i * APPEND_THREADS + threadIdx.x, token = c / PER_TOKEN;
    u32x2 out;
    for (int j = 0; j < 2; ++j) {
      const uint32_t p = held[i][2 * j], q = held[i][2 * j + 1];
      out[j] = codes_of(finite_or_nan(T::low(p)) * inverse, finite_or_nan(T::high(p)) * inverse) |
               codes_of(finite_or_nan(T::low(q)) * inverse, finite_or_nan(T::high(q)) * inverse) << 16;
    }
    if (token < count) *reinterpret_cast<u32x2*>(codes + (at + token) * D + c % PER_TOKEN * 8) = out;
  }
  // earlier tokens of the block: the same values to a larger scale (old 0: a block that nothing has been put into)
  if (at > 0 && chosen != old) {
    const float down = old + 126 < chosen ? 0.f : power_of(127 + old - chosen);
    for (uint32_t c = threadIdx.x; c < at * D / 16; c += APPEND_THREADS) {
      u32x4 w = *reinterpret_cast<const u32x4*>(codes + c * 16);
      for (int j = 0; j < 4; ++j) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[j]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[j]), true);
        w[j] = codes_of(lo[0] * down, lo[1] * down) | codes_of(hi[0] * down, hi[1] * down) << 16;
      }
      *reinterpret_cast<u32x4*>(codes + c * 16) = w;
    }
  }
  if (threadIdx.x == 0) *exponent = static_cast<uint8_t>(chosen);
}

}  // namespace fikit
