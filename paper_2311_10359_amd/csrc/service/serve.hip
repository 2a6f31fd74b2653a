// C ABI of the attention calls: argument checks, how the work is cut up, kernel sequencing.
#include "fikit.h"

#include <hip/hip_runtime.h>

#include "cache_kernels.hip.h"
#include "decode_kernels.hip.h"
#include "prompt_kernels.hip.h"
#include "serve_host.h"

namespace {

using namespace fikit;

constexpr uint32_t PLAN_GROUPS = 512;             // two for each CU

constexpr uint64_t MOST_STRIDE = 1ull << 24;      // of a token, in values: places within a tile are 32-bit numbers of bytes

// Calls f<T, D>() for a value type and head size that have been checked.
template <typename F>
int with_types(int32_t value_type, uint32_t head_dim, F f) {
  if (value_type == FIKIT_BF16) return head_dim == 128 ? f.template operator()<Bf16, 128>() : f.template operator()<Bf16, 64>();
  return head_dim == 128 ? f.template operator()<F16, 128>() : f.template operator()<F16, 64>();
}

static_assert(APPEND_WAVES * WAVE == 256, "threads of MOST_GROUPS");
struct AppendCall {
  const AppendArgs& a;
  uint32_t n_pieces;
  hipStream_t st;
  template <typename T, int D>
  int operator()() {
    return enqueue(k_cache_append<T, D>, dim3(n_pieces, (2 * a.cache.kv_heads + APPEND_WAVES - 1) / APPEND_WAVES), dim3(APPEND_WAVES * WAVE), st, a);
  }
};

// How many workgroups a decode step takes, and its workspace.
struct DecodeCut {
  uint32_t head_tiles, groups;
  uint64_t cuts_bytes, sums_bytes, bytes;
  bool fits;
};
// What the chip holds at once of k_decode, by the head's size: registers allow 2 and 4 workgroups on each of 256 compute units.
constexpr uint64_t DECODE_CHIP_128 = 512, DECODE_CHIP_64 = 1024;

DecodeCut decode_cut(uint32_t n_requests, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, uint32_t max_length) {
  DecodeCut c{};
  const auto whole = [](uint64_t v) { return (v + 255) / 256 * 256; };
  const uint64_t group = q_heads / kv_heads, rows = group < DECODE_ROWS ? group : DECODE_ROWS;
  c.head_tiles = static_cast<uint32_t>((group + DECODE_ROWS - 1) / DECODE_ROWS);
  const uint64_t chunks = static_cast<uint64_t>(n_requests) * decode_chunks(max_length), all = chunks * kv_heads * c.head_tiles;
  c.fits = chunks + n_requests * DECODE_FIXED < (1ull << 32);
  const uint64_t chip = head_dim == 128 ? DECODE_CHIP_128 : DECODE_CHIP_64;
  c.groups = static_cast<uint32_t>(all < chip ? all : chip);
  c.cuts_bytes = whole(c.groups * sizeof(uint4) + sizeof(uint32_t));
  c.sums_bytes = whole(2 * c.groups * rows * sizeof(float2));
  c.bytes = c.cuts_bytes + c.sums_bytes + 2 * c.groups * rows * head_dim * sizeof(float);
  return c;
}

struct DecodeCall {
  const DecodeArgs& a;
  const DecodeCut& c;
  hipStream_t st;
  template <typename T, int D>
  int operator()() {
    const dim3 grid(c.groups), block(DECODE_WAVES * WAVE);
    if (int rc = c.head_tiles == 1 ? enqueue(k_decode<T, D, true>, grid, block, st, a) : enqueue(k_decode<T, D, false>, grid, block, st, a)) return rc;
    if (a.max_length <= DECODE_CHUNK) return FIKIT_OK;      // (no request has several chunks)
    return enqueue(k_decode_join<T, D>, grid, block, st, a);
  }
};

// Rows per workgroup, 32 a wave: 128 rows and two workgroups on a compute unit, so that one computes while the other waits.  256 rows read keys and
// values half as often, and lose that again by waiting together (24 prompts of up to 2048 tokens: 113 us against 95 at the time; 64 of 500: 197 against 156;
// one of 8192: 491 against 493).
constexpr int PROMPT_WAVES = 4;
static_assert(PROMPT_WAVES * WAVE == 256, "threads of MOST_GROUPS");
struct PromptCall {
  const PromptArgs& a;
  uint32_t groups;
  hipStream_t st;
  template <typename T, int D>
  int operator()() { return enqueue(k_prompt<T, D, PROMPT_WAVES>, dim3(groups), dim3(PROMPT_WAVES * WAVE), st, a); }
};

}  // namespace

extern "C" {

uint64_t fikit_cache_pieces(uint32_t n_tokens, uint32_t n_requests, uint32_t block_tokens) {
  if (block_tokens == 0) return 0;
  const uint64_t cut = n_tokens / block_tokens + 2ull * n_requests;
  return cut < n_tokens ? cut : n_tokens;
}

// (Asked for from 1025 requests on, read and written beyond 4096: which kernels take how many is no part of the interface.)
size_t fikit_cache_plan_workspace_bytes(uint32_t n_requests) {
  return n_requests <= PLAN_THREADS ? 0 : ((static_cast<size_t>(n_requests) + PLAN_THREADS - 1) / PLAN_THREADS * sizeof(PlanTile) + 255) / 256 * 256;
}

int fikit_cache_plan(const int32_t* d_cached, const int32_t* d_added, uint32_t n_requests, uint32_t n_tokens,
                     uint32_t block_tokens, int32_t* d_block_table, uint32_t table_width, const int32_t* d_free,
                     uint32_t n_free, int32_t* d_lengths, int32_t* d_token_offsets, int64_t* d_slots,
                     fikit_piece* d_pieces, int32_t* d_counts, int32_t* d_status, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream) {
  if (!d_token_offsets || !d_counts || !d_status || !aligned(d_token_offsets, 4) || !aligned(d_counts, 4) || !aligned(d_status, 4))
    return FIKIT_INVALID_ARG;
  if (n_requests > 0 && (!d_cached || !d_added || !d_lengths || !aligned(d_cached, 4) || !aligned(d_added, 4) || !aligned(d_lengths, 4)))
    return FIKIT_INVALID_ARG;
  if (n_tokens > 0x7fffffffu || n_requests > 0x7fffffffu || n_free > 0x7fffffffu || table_width > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (n_tokens > 0 && (n_requests == 0 || table_width == 0 || !d_block_table || !d_pieces)) return FIKIT_INVALID_ARG;
  if (n_free > 0 && !d_free) return FIKIT_INVALID_ARG;
  if (!aligned(d_block_table, 4) || !aligned(d_free, 4) || !aligned(d_slots, 8) || !aligned(d_pieces, 16)) return FIKIT_INVALID_ARG;
  if (block_tokens < 16 || block_tokens > 256 || (block_tokens & (block_tokens - 1))) return FIKIT_UNSUPPORTED;
  if (n_requests > PLAN_MOST_REQUESTS) return FIKIT_UNSUPPORTED;
  if (const size_t need = fikit_cache_plan_workspace_bytes(n_requests)) {
    if (!d_workspace || !aligned(d_workspace, 256)) return FIKIT_INVALID_ARG;
    if (workspace_bytes < need) return FIKIT_WORKSPACE_TOO_SMALL;
  }
  const uint64_t room = fikit_cache_pieces(n_tokens, n_requests, block_tokens);
  // (outputs, then what every workgroup reads while others write)
  const Extent extents[] = {{d_lengths, 4ull * n_requests}, {d_token_offsets, 4ull * n_requests + 4}, {d_slots, d_slots ? 8ull * n_tokens : 0},
                            {d_pieces, sizeof(fikit_piece) * room}, {d_counts, 8}, {d_cached, 4ull * n_requests}, {d_added, 4ull * n_requests},
                            {d_free, 4ull * n_free}};
  for (int out = 0; out < 5; ++out)
    for (int other = out + 1; other < 8; ++other)
      if (overlap(extents[out], extents[other])) return FIKIT_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  PlanArgs a{};
  a.cached = d_cached;
  a.added = d_added;
  a.table = d_block_table;
  a.free_blocks = d_free;
  a.lengths = d_lengths;
  a.token_offsets = d_token_offsets;
  a.slots = d_slots;
  a.pieces = reinterpret_cast<int4*>(d_pieces);
  a.counts = d_counts;
  a.status = d_status;
  a.tiles = static_cast<PlanTile*>(d_workspace);
  a.n_requests = n_requests;
  a.n_tokens = n_tokens;
  a.table_width = table_width;
  a.n_free = n_free;
  a.room = static_cast<uint32_t>(room);
  a.shift = static_cast<uint32_t>(__builtin_ctz(block_tokens));
  const dim3 block(PLAN_THREADS);
  const uint32_t of_tokens = (n_tokens + PLAN_THREADS - 1) / PLAN_THREADS, tiles = (n_requests + PLAN_THREADS - 1) / PLAN_THREADS;
  const uint32_t groups = of_tokens < PLAN_GROUPS ? of_tokens : PLAN_GROUPS;
  const dim3 one(groups < 1 ? 1 : groups);
  if (n_requests <= PLAN_THREADS) return enqueue(k_plan_one<1>, one, block, st, a);
  if (n_requests <= PLAN_THREADS * PLAN_PER) return enqueue(k_plan_one<PLAN_PER>, one, block, st, a);
  if (int rc = enqueue(k_plan_tiles, dim3(tiles), block, st, a)) return rc;
  return enqueue(k_plan_tokens, dim3(tiles + groups), block, st, a);
}

int fikit_cache_append(const fikit_cache* h_cache, const fikit_vectors* h_k, const fikit_vectors* h_v, uint32_t n_tokens,
                       int32_t value_type, const fikit_piece* d_pieces, uint64_t n_pieces, int32_t* d_status,
                       void* hip_stream) {
  if (int rc = cache_status(h_cache)) return rc;
  if (!type_ok(value_type) || !d_status || !aligned(d_status, 4) || !aligned(d_pieces, 16)) return FIKIT_INVALID_ARG;
  if (n_tokens > 0x7fffffffu || n_pieces > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (n_pieces == 0) return FIKIT_OK;
  if (!d_pieces || !vectors_ok(h_k) || !vectors_ok(h_v)) return FIKIT_INVALID_ARG;
  if (n_pieces > MOST_GROUPS) return FIKIT_UNSUPPORTED;
  AppendArgs a{};
  a.cache = *h_cache;
  a.k = *h_k;
  a.v = *h_v;
  a.pieces = reinterpret_cast<const int4*>(d_pieces);
  a.status = d_status;
  a.n_tokens = n_tokens;
  return with_types(value_type, h_cache->head_dim, AppendCall{a, static_cast<uint32_t>(n_pieces), static_cast<hipStream_t>(hip_stream)});
}

size_t fikit_cache_attention_workspace_bytes(uint32_t n_requests, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim,
                                             uint32_t max_length) {
  if (kv_heads == 0 || q_heads == 0 || q_heads % kv_heads || q_heads > 65535 || max_length > 0x7fffffffu || n_requests > 0x7fffffffu) return 0;
  if (head_dim != 64 && head_dim != 128) return 0;
  const DecodeCut c = decode_cut(n_requests, q_heads, kv_heads, head_dim, max_length);
  return c.fits ? static_cast<size_t>(c.bytes) : 0;
}

int fikit_cache_attention(const fikit_cache* h_cache, const fikit_vectors* h_q, uint32_t q_heads, int32_t value_type, float scale,
                          const int32_t* d_block_table, uint32_t table_width, const int32_t* d_lengths, uint32_t n_requests,
                          uint32_t max_length, void* d_out, float* d_lse, int32_t* d_status, void* d_workspace,
                          size_t workspace_bytes, void* hip_stream) {
  if (int rc = cache_status(h_cache)) return rc;
  if (!type_ok(value_type) || !d_status || !aligned(d_status, 4) || q_heads == 0 || q_heads % h_cache->kv_heads) return FIKIT_INVALID_ARG;
  if (max_length > 0x7fffffffu || n_requests > 0x7fffffffu || table_width > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (max_length > static_cast<uint64_t>(table_width) * h_cache->block_tokens) return FIKIT_INVALID_ARG;
  if (q_heads > 65535) return FIKIT_UNSUPPORTED;
  if (n_requests == 0) return FIKIT_OK;
  if (!vectors_ok(h_q) || !d_lengths || !d_out || !aligned(d_block_table, 4) || !aligned(d_lengths, 4) || !aligned(d_out, 16) ||
      !aligned(d_lse, 4) || (max_length > 0 && !d_block_table))
    return FIKIT_INVALID_ARG;
  const DecodeCut c = decode_cut(n_requests, q_heads, h_cache->kv_heads, h_cache->head_dim, max_length);
  if (!c.fits) return FIKIT_UNSUPPORTED;
  if (!d_workspace || !aligned(d_workspace, 256)) return FIKIT_INVALID_ARG;
  if (workspace_bytes < c.bytes) return FIKIT_WORKSPACE_TOO_SMALL;
  DecodeArgs a{};
  a.cache = *h_cache;
  a.q = *h_q;
  a.table = d_block_table;
  a.lengths = d_lengths;
  a.out = d_out;
  a.lse = d_lse;
  a.status = d_status;
  unsigned char* ws = static_cast<unsigned char*>(d_workspace);
  a.cuts = reinterpret_cast<uint4*>(ws);
  a.per_unit = reinterpret_cast<uint32_t*>(ws + c.groups * sizeof(uint4));
  a.part_sums = reinterpret_cast<float2*>(ws + c.cuts_bytes);
  a.part_out = reinterpret_cast<float*>(ws + c.cuts_bytes + c.sums_bytes);
  a.q_heads = q_heads;
  a.table_width = table_width;
  a.max_length = max_length;
  a.groups = c.groups;
  a.head_tiles = c.head_tiles;
  a.n_requests = n_requests;
  a.scale = scale;
  return with_types(value_type, h_cache->head_dim, DecodeCall{a, c, static_cast<hipStream_t>(hip_stream)});
}

int fikit_prompt_attention(const fikit_vectors* h_q, const fikit_vectors* h_k, const fikit_vectors* h_v, uint32_t q_heads,
                           uint32_t kv_heads, uint32_t head_dim, int32_t value_type, float scale, const int32_t* d_offsets,
                           uint32_t n_prompts, uint32_t n_tokens, void* d_out, float* d_lse, int32_t* d_status,
                           void* hip_stream) {
  if (!type_ok(value_type) || !d_status || !aligned(d_status, 4) || kv_heads == 0 || q_heads == 0 || q_heads % kv_heads) return FIKIT_INVALID_ARG;
  if (n_tokens > 0x7fffffffu || n_prompts > 0x7fffffffu || (n_tokens > 0 && n_prompts == 0)) return FIKIT_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return FIKIT_UNSUPPORTED;
  if (n_tokens == 0) return FIKIT_OK;
  if (!vectors_ok(h_q) || !vectors_ok(h_k) || !vectors_ok(h_v) || !d_offsets || !d_out || !aligned(d_offsets, 4) || !aligned(d_out, 16) ||
      !aligned(d_lse, 4))
    return FIKIT_INVALID_ARG;
  if (h_k->token_stride > MOST_STRIDE || h_v->token_stride > MOST_STRIDE) return FIKIT_UNSUPPORTED;
  // (rows are read again where values are not finite, after they have been written)
  if (d_out == h_q->d_data || d_out == h_k->d_data || d_out == h_v->d_data) return FIKIT_INVALID_ARG;
  const uint64_t slots = n_tokens / (PROMPT_WAVES * PROMPT_WAVE_ROWS) + static_cast<uint64_t>(n_prompts);
  if (slots * q_heads > MOST_GROUPS) return FIKIT_UNSUPPORTED;
  PromptArgs a{};
  a.q = *h_q;
  a.k = *h_k;
  a.v = *h_v;
  a.offsets = d_offsets;
  a.out = d_out;
  a.lse = d_lse;
  a.status = d_status;
  a.q_heads = q_heads;
  a.kv_heads = kv_heads;
  a.n_prompts = n_prompts;
  a.n_tokens = n_tokens;
  a.slots = static_cast<uint32_t>(slots);
  a.scale = scale;
  return with_types(value_type, head_dim, PromptCall{a, static_cast<uint32_t>(slots * q_heads), static_cast<hipStream_t>(hip_stream)});
}

}  // extern "C"
