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
  uint2* bases;             // per request: new blocks and pieces of those before it
  uint32_t n_requests, n_tokens, table_width, n_free, room;
  uint32_t shift;           // of the block length
};

constexpr int PLAN_THREADS = 1024;

struct PlanSums {
  uint32_t tokens, blocks, pieces;
};

// What a request of c cached and a added tokens adds to the sums; false if these cannot be, or a sum does not fit.  (Blocks and
// pieces are at most as many as tokens.)
__device__ __forceinline__ bool plan_request(const PlanArgs& a, int32_t c, int32_t d, PlanSums* s) {
  const uint32_t cached = static_cast<uint32_t>(c), added = static_cast<uint32_t>(d), length = cached + added, last = (1u << a.shift) - 1;
  const bool ok = c >= 0 && d >= 0 && length <= INT32_MAX && ((static_cast<uint64_t>(length) + last) >> a.shift) <= a.table_width;
  s->blocks += ((length + last) >> a.shift) - ((cached + last) >> a.shift);
  s->pieces += d > 0 ? ((length - 1) >> a.shift) - (cached >> a.shift) + 1 : 0;
  s->tokens += added;
  return ok && s->tokens >= added;
}

struct PlanScan {
  uint32_t blocks[PLAN_THREADS / WAVE], pieces[PLAN_THREADS / WAVE];
  uint64_t tokens[PLAN_THREADS / WAVE];
};

// The sums of the threads before, and of all of them, in a workgroup of PLAN_THREADS; whether `ok` holds in all and all sums fit.
__device__ __forceinline__ bool plan_scan(const PlanSums& mine, bool ok, PlanScan* lds, PlanSums* before, PlanSums* total) {
  constexpr uint32_t WAVES = PLAN_THREADS / WAVE;
  const uint64_t run_tokens = wave_incl_scan_u64(mine.tokens);
  const uint32_t run_blocks = wave_incl_scan_u32(mine.blocks), run_pieces = wave_incl_scan_u32(mine.pieces);
  const uint32_t wave = uniform(threadIdx.x / WAVE), lane = lane_id();
  if (lane == WAVE - 1) { lds->tokens[wave] = run_tokens; lds->blocks[wave] = run_blocks; lds->pieces[wave] = run_pieces; }
  const bool all = __syncthreads_and(ok);
  // each wave scans the waves' sums
  const bool there = lane < WAVES;
  const uint64_t tokens = there ? lds->tokens[lane % WAVES] : 0;
  const uint32_t blocks = there ? lds->blocks[lane % WAVES] : 0, pieces = there ? lds->pieces[lane % WAVES] : 0;
  const uint64_t upto = wave_incl_scan_u64(tokens);
  const uint32_t upto_blocks = wave_incl_scan_u32(blocks), upto_pieces = wave_incl_scan_u32(pieces);
  *total = PlanSums{read_lane_u32(static_cast<uint32_t>(upto), WAVES - 1), read_lane_u32(upto_blocks, WAVES - 1), read_lane_u32(upto_pieces, WAVES - 1)};
  *before = PlanSums{read_lane_u32(static_cast<uint32_t>(upto - tokens), wave) + static_cast<uint32_t>(run_tokens) - mine.tokens,
                     read_lane_u32(upto_blocks - blocks, wave) + run_blocks - mine.blocks,
                     read_lane_u32(upto_pieces - pieces, wave) + run_pieces - mine.pieces};
  return all && read_lane_u64(upto, WAVES - 1) <= INT32_MAX;
}

__device__ __forceinline__ int32_t plan_error(const PlanArgs& a, const PlanSums& total, bool ok) {
  return !ok || total.tokens != a.n_tokens ? FIKIT_INVALID_ARG : total.blocks > a.n_free ? FIKIT_CACHE_FULL : FIKIT_OK;
}

// The last of the requests lo .. hi - 1 that begins at token t or before; lo begins so.
__device__ __forceinline__ uint32_t plan_find(const int32_t* offsets, uint32_t lo, uint32_t hi, uint32_t t) {
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (static_cast<uint32_t>(offsets[mid]) <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// What new token t, of request r that begins at token `first`, writes; `blocks`, `pieces`: those of the requests before.
__device__ __forceinline__ void plan_token(const PlanArgs& a, uint32_t t, uint32_t r, uint32_t first, uint32_t blocks, uint32_t pieces) {
  const uint32_t block_tokens = 1u << a.shift;
  const uint32_t cached = static_cast<uint32_t>(a.cached[r]), length = cached + static_cast<uint32_t>(a.added[r]);
  const uint32_t index = t - first;
  const uint32_t place = cached + index, page = place >> a.shift, at = place & (block_tokens - 1);
  const uint32_t held = (cached + block_tokens - 1) >> a.shift;
  int32_t* entry = a.table + static_cast<uint64_t>(r) * a.table_width + page;
  const int32_t block = page >= held ? a.free_blocks[blocks + (page - held)] : *entry;
  if (at == 0) *entry = block;      // (a block that begins at a new token is a new one)
  if (a.slots) a.slots[t] = static_cast<int64_t>(block) * block_tokens + at;
  if (at == 0 || index == 0)
    a.pieces[pieces + (page - (cached >> a.shift))] = make_int4(block, static_cast<int32_t>(t), static_cast<int32_t>(at),
                                                               static_cast<int32_t>(min_u32(block_tokens - at, length - place)));
}

// Eight or sixteen consecutive requests are read as vectors of words; the arrays need no more alignment than that.
typedef int32_t i32x4_by_words __attribute__((ext_vector_type(4), aligned(4)));
template <uint32_t PER>
__device__ __forceinline__ void plan_read(const int32_t* from, uint64_t first, uint32_t n, int32_t (&to)[PER]) {
  if (PER % 4 == 0 && first + PER <= n) {
#pragma unroll
    for (uint32_t i = 0; i < PER; i += 4) {
      const i32x4_by_words x = *reinterpret_cast<const i32x4_by_words*>(from + first + i);
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) to[i + j] = x[j];
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < PER; ++i) to[i] = first + i < n ? from[first + i] : 0;
  }
}

// The whole plan in one launch: every workgroup sums all requests for itself, a run of PER consecutive ones per thread, and takes
// 1024 tokens at a time.  Where each request begins is kept in LDS; its blocks and pieces too for runs of up to four, else they
// are added up again from where its run begins.
constexpr uint32_t PLAN_ONE_REQUESTS = 16 * PLAN_THREADS;
template <uint32_t PER>
__global__ __launch_bounds__(PLAN_THREADS) void k_plan_one(PlanArgs a) {
  constexpr bool ALL = PER <= 4;
  constexpr uint32_t GAP = ALL ? 0 : 1;       // (a word behind every run, so that threads write to different banks)
  __shared__ int32_t offsets[(PER + GAP) * PLAN_THREADS];
  __shared__ uint2 bases[(ALL ? PER : 1) * PLAN_THREADS];
  __shared__ PlanScan scan;
  const bool stop = stopped(a.status);
  const uint32_t first = threadIdx.x * PER;
  int32_t cached[PER], added[PER];
  plan_read<PER>(a.cached, first, a.n_requests, cached);
  plan_read<PER>(a.added, first, a.n_requests, added);
  if (stop) return;
  PlanSums mine{0, 0, 0}, at, total;
  bool ok = true;
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) ok &= plan_request(a, cached[i], added[i], &mine);
  ok = plan_scan(mine, ok, &scan, &at, &total);
  if (const int32_t error = plan_error(a, total, ok)) {
    if (threadIdx.x == 0) *a.status = error;
    return;
  }
  const bool writes = blockIdx.x == 0;
  if (!ALL) bases[threadIdx.x] = make_uint2(at.blocks, at.pieces);
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const uint32_t r = first + i;
    offsets[r + GAP * threadIdx.x] = static_cast<int32_t>(at.tokens);
    if (ALL) bases[r] = make_uint2(at.blocks, at.pieces);
    if (writes && r < a.n_requests) {
      a.lengths[r] = cached[i] + added[i];
      a.token_offsets[r] = static_cast<int32_t>(at.tokens);
    }
    if (ALL) plan_request(a, cached[i], added[i], &at);
    else at.tokens += static_cast<uint32_t>(added[i]);
  }
  if (writes && threadIdx.x == 0) {
    a.token_offsets[a.n_requests] = static_cast<int32_t>(a.n_tokens);
    a.counts[0] = static_cast<int32_t>(total.blocks);
    a.counts[1] = static_cast<int32_t>(total.pieces);
  }
  __syncthreads();
  const uint32_t from = blockIdx.x * PLAN_THREADS + threadIdx.x, stride = gridDim.x * PLAN_THREADS;
  for (uint64_t t = from; t < a.n_tokens; t += stride) {
    const uint32_t token = static_cast<uint32_t>(t);
    if constexpr (ALL) {
      const uint32_t r = plan_find(offsets, 0, a.n_requests, token);
      plan_token(a, token, r, static_cast<uint32_t>(offsets[r]), bases[r].x, bases[r].y);
    } else {
      // the run, then the request in it
      uint32_t run = 0;
      for (uint32_t hi = (a.n_requests + PER - 1) / PER; hi - run > 1;) {
        const uint32_t mid = run + (hi - run) / 2;
        if (static_cast<uint32_t>(offsets[mid * (PER + GAP)]) <= token) run = mid; else hi = mid;
      }
      plan_read<PER>(a.cached, run * PER, a.n_requests, cached);
      plan_read<PER>(a.added, run * PER, a.n_requests, added);
      PlanSums s{static_cast<uint32_t>(offsets[run * (PER + GAP)]), bases[run].x, bases[run].y};
      uint32_t r = run * PER;
#pragma unroll
      for (uint32_t i = 0; i + 1 < PER; ++i) {        // past the requests that end at the token or before
        const bool past = r == run * PER + i && r + 1 < a.n_requests && s.tokens + static_cast<uint32_t>(added[i]) <= token;
        if (past) {
          plan_request(a, cached[i], added[i], &s);
          ++r;
        }
      }
      plan_token(a, token, r, s.tokens, s.blocks, s.pieces);
    }
  }
  for (uint64_t i = static_cast<uint64_t>(total.pieces) + from; i < a.room; i += stride) a.pieces[i] = make_int4(-1, -1, -1, -1);
}

// For more requests the sums are one workgroup's, 8 consecutive requests per thread and round, and the tokens a launch behind it.
constexpr uint32_t PLAN_PER = 8;
__global__ __launch_bounds__(PLAN_THREADS) void k_plan_sums(PlanArgs a) {
  __shared__ PlanScan scan[2];
  if (stopped(a.status)) return;
  PlanSums carry{0, 0, 0};
  bool ok = true;
  uint32_t turn = 0;
  for (uint64_t round = 0; round < a.n_requests; round += PLAN_THREADS * PLAN_PER, turn ^= 1) {
    const uint64_t first = round + threadIdx.x * PLAN_PER;
    const bool whole = first + PLAN_PER <= a.n_requests;
    int32_t cached[PLAN_PER], added[PLAN_PER];
    plan_read<PLAN_PER>(a.cached, first, a.n_requests, cached);
    plan_read<PLAN_PER>(a.added, first, a.n_requests, added);
    PlanSums mine{0, 0, 0}, at, total;
#pragma unroll
    for (uint32_t i = 0; i < PLAN_PER; ++i) ok &= plan_request(a, cached[i], added[i], &mine);
    ok = plan_scan(mine, ok, &scan[turn], &at, &total);
    at.tokens += carry.tokens; at.blocks += carry.blocks; at.pieces += carry.pieces;
    carry.tokens += total.tokens; carry.blocks += total.blocks; carry.pieces += total.pieces;
    ok &= carry.tokens >= total.tokens;
#pragma unroll
    for (uint32_t i = 0; i < PLAN_PER; i += 4) {
      i32x4_by_words length, offset;
      uint2 base[4];
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        length[j] = static_cast<int32_t>(static_cast<uint32_t>(cached[i + j]) + static_cast<uint32_t>(added[i + j]));
        offset[j] = static_cast<int32_t>(at.tokens);
        base[j] = make_uint2(at.blocks, at.pieces);
        plan_request(a, cached[i + j], added[i + j], &at);
      }
      if (whole) {
        *reinterpret_cast<i32x4_by_words*>(a.lengths + first + i) = length;
        *reinterpret_cast<i32x4_by_words*>(a.token_offsets + first + i) = offset;
        uint4* to = reinterpret_cast<uint4*>(a.bases + first + i);
        to[0] = make_uint4(base[0].x, base[0].y, base[1].x, base[1].y);
        to[1] = make_uint4(base[2].x, base[2].y, base[3].x, base[3].y);
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
          if (first + i + j < a.n_requests) {
            a.lengths[first + i + j] = length[j];
            a.token_offsets[first + i + j] = offset[j];
            a.bases[first + i + j] = base[j];
          }
      }
    }
  }
  if (threadIdx.x == 0) {
    if (const int32_t error = plan_error(a, carry, ok)) *a.status = error;
    a.token_offsets[a.n_requests] = static_cast<int32_t>(a.n_tokens);
    a.counts[0] = static_cast<int32_t>(carry.blocks);
    a.counts[1] = static_cast<int32_t>(carry.pieces);
  }
}

__global__ __launch_bounds__(256) void k_plan_tokens(PlanArgs a) {
  if (stopped(a.status)) return;
  const uint32_t t = blockIdx.x * 256 + threadIdx.x;
  if (t < a.n_tokens) {
    const uint32_t r = plan_find(a.token_offsets, 0, a.n_requests, t);
    plan_token(a, t, r, static_cast<uint32_t>(a.token_offsets[r]), a.bases[r].x, a.bases[r].y);
  }
  for (uint64_t i = static_cast<uint64_t>(static_cast<uint32_t>(a.counts[1])) + t; i < a.room; i += static_cast<uint64_t>(gridDim.x) * 256)
    a.pieces[i] = make_int4(-1, -1, -1, -1);
}

// ---- append -----------------------------------------------------------------------------------------------------
//
// A piece lies in one block, so the largest magnitude of its values, the block's exponent and the codes belong to one wave
// per piece, head, and keys or values.  It reads the values once and holds up to 8192 of them (64 tokens of 128) in registers
// between the maximum and the rounding; of longer pieces it reads them again, from the cache.  Memory bound: 2 bytes read and 1
// written per value, and half an instruction each for the maximum (of pairs, as integers) and for the rounding of a pair.

struct AppendArgs {
  fikit_cache cache;
  fikit_vectors k, v;
  const int4* pieces;
  int32_t* status;
  uint32_t n_tokens;
};

constexpr int APPEND_WAVES = 4, APPEND_HOLD = 16;   // (pieces of eight values per lane)

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

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t most_of_pairs(uint32_t a, uint32_t b) {
  return bits_as<uint32_t>(__builtin_elementwise_max(bits_as<u16x2>(a), bits_as<u16x2>(b)));
}

template <typename T, int D>
__global__ __launch_bounds__(APPEND_WAVES * WAVE) void k_cache_append(AppendArgs a) {
  const int4 piece = a.pieces[blockIdx.x];
  const bool stop = stopped(a.status);
  if (piece.x == -1 || stop) return;
  const uint32_t lane = lane_id(), unit = blockIdx.y * APPEND_WAVES + uniform(threadIdx.x / WAVE), block_tokens = a.cache.block_tokens;
  const uint32_t block = static_cast<uint32_t>(piece.x), first = static_cast<uint32_t>(piece.y), at = static_cast<uint32_t>(piece.z),
                 count = static_cast<uint32_t>(piece.w);
  if (block >= a.cache.n_blocks || at >= block_tokens || count == 0 || count > block_tokens - at || first >= a.n_tokens ||
      count > a.n_tokens - first) {
    if (threadIdx.x == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  if (unit >= 2 * a.cache.kv_heads) return;
  const bool values = unit >= a.cache.kv_heads;
  const uint32_t head = values ? unit - a.cache.kv_heads : unit;
  const fikit_vectors in = values ? a.v : a.k;
  const uint16_t* x = static_cast<const uint16_t*>(in.d_data) + first * in.token_stride + head * in.head_stride;
  const uint64_t place = static_cast<uint64_t>(block) * a.cache.kv_heads + head;
  uint8_t* codes = (values ? a.cache.d_v : a.cache.d_k) + place * block_tokens * D;
  uint8_t* exponent = (values ? a.cache.d_v_exp : a.cache.d_k_exp) + place;
  const uint32_t old = at > 0 ? min_u32(*exponent, 254u) : 0;

  constexpr uint32_t PER_TOKEN = D / 8, ROUND = APPEND_HOLD * WAVE;
  const uint32_t chunks = count * PER_TOKEN;
  u32x4 held[APPEND_HOLD];
  auto read = [&](uint32_t round) {
#pragma unroll
    for (uint32_t i = 0; i < APPEND_HOLD; ++i) {
      held[i] = u32x4{0, 0, 0, 0};
      if (round + i * WAVE < chunks) {
        const uint32_t c = round + i * WAVE + lane;
        if (c < chunks) held[i] = *reinterpret_cast<const u32x4*>(x + c / PER_TOKEN * in.token_stride + c % PER_TOKEN * 8);
      }
    }
  };
  uint32_t pairs = 0;               // largest magnitudes of even and of odd values, as the bits of their type
  for (uint32_t round = 0; round < chunks; round += ROUND) {
    read(round);
#pragma unroll
    for (uint32_t i = 0; i < APPEND_HOLD; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) pairs = most_of_pairs(pairs, held[i][j] & 0x7fff7fffu);
  }
  uint32_t bits = max_u32(pairs & 0xffffu, pairs >> 16);
  bits = max_over_wave(bits);
  const bool odd = bits >= T::INF;  // something is not finite: look again, without it
  if (odd) {
    bits = 0;
    for (uint32_t round = 0; round < chunks; round += ROUND) {
      if (chunks > ROUND) read(round);
#pragma unroll
      for (uint32_t i = 0; i < APPEND_HOLD; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = held[i][j] & 0x7fffu, hi = held[i][j] >> 16 & 0x7fffu;
          bits = max_u32(bits, max_u32(lo < T::INF ? lo : 0, hi < T::INF ? hi : 0));
        }
    }
    bits = max_over_wave(bits);
  }
  const uint32_t chosen = max_u32(exponent_for(T::low(bits)), old);
  const float scale = power_of(chosen), inverse = power_of(254 - chosen);

  for (uint32_t round = 0; round < chunks; round += ROUND) {
    if (chunks > ROUND) read(round);
#pragma unroll
    for (uint32_t i = 0; i < APPEND_HOLD; ++i) {
      if (round + i * WAVE >= chunks) break;
      const uint32_t c = round + i * WAVE + lane;
      u32x2 out;
      if (odd) {
        for (int j = 0; j < 2; ++j) {
          const uint32_t p = held[i][2 * j], q = held[i][2 * j + 1];
          out[j] = codes_of(finite_or_nan(T::low(p)) * inverse, finite_or_nan(T::high(p)) * inverse) |
                   codes_of(finite_or_nan(T::low(q)) * inverse, finite_or_nan(T::high(q)) * inverse) << 16;
        }
      } else {
        for (int j = 0; j < 2; ++j) out[j] = T::codes_of_pairs(held[i][2 * j], held[i][2 * j + 1], scale);
      }
      if (c < chunks) *reinterpret_cast<u32x2*>(codes + at * D + c * 8) = out;
    }
  }
  // earlier tokens of the block: the same values to a larger scale (old 0: a block that nothing has been put into)
  if (at > 0 && chosen != old) {
    const float down = old + 126 < chosen ? 0.f : power_of(127 + old - chosen);
    for (uint32_t c = lane; c < at * D / 16; c += WAVE) {
      u32x4 w = *reinterpret_cast<const u32x4*>(codes + c * 16);
      for (int j = 0; j < 4; ++j) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[j]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[j]), true);
        w[j] = codes_of(lo[0] * down, lo[1] * down) | codes_of(hi[0] * down, hi[1] * down) << 16;
      }
      *reinterpret_cast<u32x4*>(codes + c * 16) = w;
    }
  }
  if (lane == 0) *exponent = static_cast<uint8_t>(chosen);
}

}  // namespace fikit
