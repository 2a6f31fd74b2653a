// C ABI of the calls around the attention: argument checks, how the work is cut up, kernel sequencing.
#include "fikit.h"

#include <hip/hip_runtime.h>

#include "blocks_kernels.hip.h"
#include "rotate_kernels.hip.h"
#include "scores_kernels.hip.h"
#include "serve_host.h"

namespace {

using namespace fikit;

constexpr uint32_t ROTATE_MOST_GROUPS = 1u << 16;
constexpr uint32_t ROTATE_SPREAD = 2048;          // waves: eight for each CU
constexpr uint64_t ROTATE_PAST = 1ull << 27;      // bytes from which on the caches are passed by: half of the last one's

struct RotateCall {
  const RotateArgs& a;
  bool neighbours, past;
  hipStream_t st;
  template <typename T, int D, bool NEIGHBOURS>
  int run() {
    const uint32_t groups = (a.units + ROTATE_WAVES - 1) / ROTATE_WAVES;
    const dim3 grid(groups < ROTATE_MOST_GROUPS ? groups : ROTATE_MOST_GROUPS), block(ROTATE_WAVES * WAVE);
    return past ? enqueue(k_rotate<T, D, NEIGHBOURS, true>, grid, block, st, a) : enqueue(k_rotate<T, D, NEIGHBOURS, false>, grid, block, st, a);
  }
  template <typename T, int D>
  int with_pairs() { return neighbours ? run<T, D, true>() : run<T, D, false>(); }
  template <typename T>
  int with_dim(uint32_t head_dim) { return head_dim == 64 ? with_pairs<T, 64>() : head_dim == 128 ? with_pairs<T, 128>() : with_pairs<T, 256>(); }
};

// Do the vectors lie apart?  Those of the smaller stride beside each other, and the larger stride beyond all of them.
bool apart(const fikit_vectors* v, uint32_t heads, uint32_t n_tokens, uint32_t head_dim) {
  struct { uint64_t stride, n; } inner{v->head_stride, heads}, outer{v->token_stride, n_tokens};
  if (inner.n <= 1 || (outer.n > 1 && outer.stride < inner.stride)) {
    const auto other = inner;
    inner = outer;
    outer = other;
  }
  if (inner.n > 1 && inner.stride < head_dim) return false;
  return outer.n <= 1 || (outer.stride >= head_dim && (outer.stride - head_dim) / (inner.n > 1 ? inner.stride : 1) >= (inner.n > 1 ? inner.n - 1 : 0));
}

// Does no vector of a lie over one of b?  They may share a product's rows, beside each other or head by head.
bool apart(const fikit_vectors* a, uint32_t heads_a, const fikit_vectors* b, uint32_t heads_b, uint32_t n_tokens, uint32_t head_dim) {
  const auto row = [&](const fikit_vectors* v, uint32_t heads) { return (heads - 1) * v->head_stride + head_dim; };        // values from a token's first to its last
  const auto all = [&](const fikit_vectors* v, uint32_t heads) { return Extent{v->d_data, 2 * ((n_tokens - 1) * v->token_stride + row(v, heads))}; };
  if (!overlap(all(a, heads_a), all(b, heads_b))) return true;
  // how far the first value of b's is behind one of a's, in steps of that many values
  const auto behind = [&](uint64_t step) {
    const int64_t d = (reinterpret_cast<intptr_t>(b->d_data) - reinterpret_cast<intptr_t>(a->d_data)) / 2 % static_cast<int64_t>(step);
    return static_cast<uint64_t>(d < 0 ? d + static_cast<int64_t>(step) : d);
  };
  const uint64_t step = n_tokens > 1 ? a->token_stride : 0;
  if (n_tokens > 1 && (b->token_stride != step || step == 0 || step > 1ull << 60)) return false;
  if (step > 0 && behind(step) >= row(a, heads_a) && behind(step) + row(b, heads_b) <= step) return true;
  const uint64_t heads = a->head_stride;
  if (heads == 0 || heads_a <= 1 || heads_b <= 1 || b->head_stride != heads || (step > 0 && step % heads) || heads > 1ull << 60) return false;
  return behind(heads) >= head_dim && behind(heads) + head_dim <= heads;
}

// Are an output's places its input's?
bool in_place(const fikit_vectors* in, const fikit_vectors* out, uint32_t heads, uint32_t n_tokens) {
  return in->d_data == out->d_data && (heads <= 1 || in->head_stride == out->head_stride) && (n_tokens <= 1 || in->token_stride == out->token_stride);
}

uint64_t slices_of(uint32_t n_blocks) { return ((n_blocks + 31ull) / 32 + SLICE - 1) / SLICE; }

// Parts of the workspace of a fork or a compaction, one behind the other, in words.
struct Parts {
  uint64_t bytes = 0;
  uint64_t take(uint64_t count) {
    const uint64_t at = bytes;
    bytes += (4 * count + 255) / 256 * 256;
    return at;
  }
};
struct ForkParts : Parts {
  uint64_t words, flags, flags_too, flags_free, marks, sums, sums_too, first, rank, wants;
  ForkParts(uint32_t n_requests, uint32_t n_children, uint32_t n_blocks) : words((n_blocks + 31) / 32) {
    take(1);
    flags = take(8 * words);
    flags_too = take(8 * words);
    flags_free = take(8 * words);
    marks = take(SLICE * slices_of(n_blocks));
    sums = take(slices_of(n_blocks));
    sums_too = take(slices_of(n_blocks));
    first = take(n_requests);
    rank = take(n_children);
    wants = take(n_children);
  }
};
struct CompactParts : Parts {
  uint64_t words, flags, flags_too, marks, marks_too, sums, sums_too, before;
  explicit CompactParts(uint32_t n_blocks) : words((n_blocks + 31) / 32) {
    take(2);
    flags = take(8 * words);
    flags_too = take(8 * words);
    marks = take(SLICE * slices_of(n_blocks));
    marks_too = take(SLICE * slices_of(n_blocks));
    sums = take(slices_of(n_blocks));
    sums_too = take(slices_of(n_blocks));
    before = take(SLICE * slices_of(n_blocks));
  }
};

// Workgroups of the kernels that do all in one launch, or 0 for sizes that they do not take.
uint32_t one_launch(uint32_t n_requests, uint32_t rows, uint32_t table_width, uint32_t n_blocks, uint32_t most_cells) {
  if (n_requests > ONE_REQUESTS || rows > ONE_REQUESTS || n_blocks > ONE_BLOCKS || static_cast<uint64_t>(n_requests) * table_width > most_cells) return 0;
  const uint32_t groups = (rows + BLOCKS_THREADS / WAVE - 1) / (BLOCKS_THREADS / WAVE);
  return groups < 1 ? 1 : groups < ONE_MOST_GROUPS ? groups : ONE_MOST_GROUPS;
}

bool blocks_fit(uint32_t n_requests, uint32_t n_children, uint32_t n_blocks) {
  return n_requests <= BLOCKS_MOST_REQUESTS && n_children <= BLOCKS_MOST_REQUESTS && n_blocks <= BLOCKS_MOST_BLOCKS;
}

// FIKIT_OK, or what is wrong with the inputs that fork and compaction share.
int blocks_status(const int32_t* d_block_table, uint32_t table_width, const int32_t* d_lengths, uint32_t n_requests, uint32_t n_children,
                  uint32_t block_tokens, uint32_t n_blocks, const int32_t* d_free, uint32_t n_free, const int32_t* d_status) {
  if (!d_status || !aligned(d_status, 4) || n_blocks == 0 || n_free > n_blocks || table_width > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (n_requests > 0 && (!d_lengths || (table_width > 0 && !d_block_table))) return FIKIT_INVALID_ARG;
  if (n_free > 0 && !d_free) return FIKIT_INVALID_ARG;
  if (!aligned(d_block_table, 4) || !aligned(d_lengths, 4) || !aligned(d_free, 4)) return FIKIT_INVALID_ARG;
  if (block_tokens < 16 || block_tokens > 256 || (block_tokens & (block_tokens - 1))) return FIKIT_UNSUPPORTED;
  return blocks_fit(n_requests, n_children, n_blocks) ? FIKIT_OK : FIKIT_UNSUPPORTED;
}

// The first `outputs` of n extents overlap neither each other nor those behind them.
bool outputs_apart(const Extent* extents, int outputs, int n) {
  for (int out = 0; out < outputs; ++out)
    for (int other = out + 1; other < n; ++other)
      if (overlap(extents[out], extents[other])) return false;
  return true;
}

BlocksArgs blocks_args(const int32_t* d_block_table, uint32_t table_width, const int32_t* d_lengths, uint32_t n_requests, uint32_t block_tokens,
                       uint32_t n_blocks, const int32_t* d_free, uint32_t n_free, int32_t* d_status) {
  BlocksArgs a{};
  a.table = d_block_table;
  a.lengths = d_lengths;
  a.free_blocks = d_free;
  a.status = d_status;
  a.n_requests = n_requests;
  a.width = table_width;
  a.n_blocks = n_blocks;
  a.n_free = n_free;
  a.words = (n_blocks + 31) / 32;
  a.shift = static_cast<uint32_t>(__builtin_ctz(block_tokens));
  return a;
}

// How rows of logits are cut up, and the workspace.
struct ScoresCut {
  uint32_t parts, per_part, waves;
  uint64_t sums_bytes, bytes;
};
// A row is one wave's where that takes it in a turn, or in four and there are many (20,000 rows of 1000 bfloat16 logits 40 us, 4 waves 67; 8000 rows of
// 8192 37 and 42).  It is one workgroup's where that takes it in one turn, of 4 waves or of 16 (one row of 32,000 bfloat16 logits 9.3 us; 10.9 in parts that
// a second launch joins), and from 128 rows on, of as many waves as the chip holds for so many rows: 16 up to 511 (256 rows of 50,001 float32 15 us, 4 waves
// 21; 300 rows of 131,072 bfloat16 32, 8 waves 34), 8 up to 1023 (700 such rows 43, 16 waves 48, 4 waves 46), 4 beyond (1100 rows 60, 8 waves 65, 16 waves 72).
// Else rows are cut into parts of 4 waves, for two workgroups on a compute unit: one compute unit takes 2 us to read what 16 waves want first (one row of
// 131,072 logits 15.9 us, in parts of 16 waves 17.1, when that was measured; 64 such rows 19.5 and 20.5).
constexpr uint32_t SCORES_CHIP = 256, SCORES_MORE = 512, SCORES_MANY = 1024;

ScoresCut scores_cut(uint32_t n_rows, uint32_t vocabulary, int32_t value_type, uint32_t n_top) {
  ScoresCut c{};
  const uint32_t groups = vocabulary / (value_type == FIKIT_F32 ? LogitsF32::VEC : LogitsBf16::VEC), turn = SCORES_BATCH * WAVE;
  const bool few = n_rows < SCORES_CHIP / 2;
  const bool one_wave = groups <= turn || (n_rows >= 2 * SCORES_MANY && groups <= 4 * turn);
  c.waves = one_wave ? 1 : groups <= 4 * turn || n_rows >= SCORES_MANY || (few && groups > 16 * turn) ? 4 : n_rows >= SCORES_MORE ? 8 : 16;
  const uint32_t most = (groups + c.waves * turn - 1) / (c.waves * turn), want = n_rows > 0 && few && c.waves == 4 ? 2 * SCORES_CHIP / n_rows : 1;
  c.parts = want < most ? want : most;
  if (c.parts < 1) c.parts = 1;
  const uint32_t each = (groups + c.parts - 1) / c.parts;
  c.per_part = (each + WAVE - 1) / WAVE * WAVE;
  if (groups > 0) c.parts = (groups + c.per_part - 1) / c.per_part;
  if (c.parts == 1) return c;
  const uint64_t lists = static_cast<uint64_t>(n_rows) * c.parts;
  c.sums_bytes = (lists * sizeof(float4) + 255) / 256 * 256;
  c.bytes = c.sums_bytes + (n_top > 0 ? lists * SCORES_MOST * sizeof(float2) : 0);
  return c;
}

struct ScoresCall {
  const ScoresArgs& a;
  uint32_t waves;
  hipStream_t st;
  template <typename L>
  int run() {
    const dim3 grid(a.rows * a.parts), block(waves * WAVE), join(JOIN_WAVES * WAVE);
    if (int rc = waves == 16  ? enqueue(k_scores<L, 16>, grid, block, st, a)
                 : waves == 8 ? enqueue(k_scores<L, 8>, grid, block, st, a)
                 : waves == 4 ? enqueue(k_scores<L, 4>, grid, block, st, a)
                              : enqueue(k_scores<L, 1>, grid, block, st, a))
      return rc;
    return a.parts == 1 ? FIKIT_OK : enqueue(k_scores_join<L>, dim3((a.rows + JOIN_WAVES - 1) / JOIN_WAVES), join, st, a);
  }
};

bool logits_ok(int32_t value_type) { return type_ok(value_type) || value_type == FIKIT_F32; }

dim3 clear_groups(uint32_t words) { return dim3((2 * words + BLOCKS_THREADS - 1) / BLOCKS_THREADS); }        // 16 flags of both kinds to a thread
constexpr uint32_t COPY_GROUPS = 16384;

}  // namespace

extern "C" {

size_t fikit_cache_fork_workspace_bytes(uint32_t n_requests, uint32_t n_children, uint32_t table_width, uint32_t n_blocks) {
  if (!blocks_fit(n_requests, n_children, n_blocks) || one_launch(n_requests, n_children, table_width, n_blocks, FORK_CELLS)) return 0;
  return static_cast<size_t>(ForkParts(n_requests, n_children, n_blocks).bytes);
}

int fikit_cache_fork(const int32_t* d_block_table, uint32_t table_width, const int32_t* d_lengths, uint32_t n_requests,
                     const int32_t* d_parents, uint32_t n_children, uint32_t block_tokens, uint32_t n_blocks, const int32_t* d_free,
                     uint32_t n_free, int32_t* d_new_table, int32_t* d_new_lengths, fikit_block_copy* d_copies, int32_t* d_new_free,
                     int32_t* d_counts, int32_t* d_status, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = blocks_status(d_block_table, table_width, d_lengths, n_requests, n_children, block_tokens, n_blocks, d_free, n_free, d_status)) return rc;
  if (n_children > 0 && (!d_parents || !d_new_lengths || !d_copies || (table_width > 0 && !d_new_table))) return FIKIT_INVALID_ARG;
  if (!d_new_free || !d_counts || !aligned(d_parents, 4) || !aligned(d_new_table, 4) || !aligned(d_new_lengths, 4) || !aligned(d_copies, 8) ||
      !aligned(d_new_free, 4) || !aligned(d_counts, 4))
    return FIKIT_INVALID_ARG;
  const uint64_t row = 4ull * table_width;
  const Extent extents[] = {{d_new_table, row * n_children}, {d_new_lengths, 4ull * n_children}, {d_copies, sizeof(fikit_block_copy) * n_children},
                            {d_new_free, 4ull * n_blocks}, {d_counts, 12}, {d_block_table, row * n_requests}, {d_lengths, 4ull * n_requests},
                            {d_parents, 4ull * n_children}, {d_free, 4ull * n_free}};
  if (!outputs_apart(extents, 5, 9)) return FIKIT_INVALID_ARG;
  BlocksArgs a = blocks_args(d_block_table, table_width, d_lengths, n_requests, block_tokens, n_blocks, d_free, n_free, d_status);
  a.parents = d_parents;
  a.new_table = d_new_table;
  a.new_lengths = d_new_lengths;
  a.copies = reinterpret_cast<int2*>(d_copies);
  a.new_free = d_new_free;
  a.counts = d_counts;
  a.n_children = n_children;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const uint32_t groups = one_launch(n_requests, n_children, table_width, n_blocks, FORK_CELLS))
    return enqueue(k_fork_one, dim3(groups + 1), dim3(BLOCKS_THREADS), st, a);
  const ForkParts parts(n_requests, n_children, n_blocks);
  if (!d_workspace || !aligned(d_workspace, 256)) return FIKIT_INVALID_ARG;
  if (workspace_bytes < parts.bytes) return FIKIT_WORKSPACE_TOO_SMALL;
  const auto part = [&](uint64_t at) { return reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(d_workspace) + at); };
  a.words_of_call = part(0);
  a.flags = reinterpret_cast<uint8_t*>(part(parts.flags));
  a.flags_too = reinterpret_cast<uint8_t*>(part(parts.flags_too));
  a.flags_free = reinterpret_cast<uint8_t*>(part(parts.flags_free));
  a.marks = part(parts.marks);
  a.sums = part(parts.sums);
  a.sums_too = part(parts.sums_too);
  a.first = part(parts.first);
  a.rank = reinterpret_cast<int32_t*>(part(parts.rank));
  a.wants = part(parts.wants);
  const dim3 clear(1 + clear_groups(a.words).x), threads(BLOCKS_THREADS);
  const uint32_t most = n_requests > n_children ? n_requests : n_children;
  if (int rc = most <= 4 * BLOCKS_THREADS ? enqueue(k_fork_begin<4>, clear, threads, st, a) : most <= 8 * BLOCKS_THREADS ? enqueue(k_fork_begin<8>, clear, threads, st, a)
                                                                                             : enqueue(k_fork_begin<16>, clear, threads, st, a))
    return rc;
  if (const uint32_t rows = n_requests + n_children + (n_free + WAVE - 1) / WAVE)
    if (int rc = enqueue(k_fork_rows, dim3((rows + ROW_WAVES - 1) / ROW_WAVES), dim3(ROW_WAVES * WAVE), st, a)) return rc;
  const uint32_t slices = static_cast<uint32_t>(slices_of(n_blocks));
  if (int rc = enqueue(k_blocks_pack<true>, dim3(slices), dim3(SLICE), st, a)) return rc;
  return enqueue(k_fork_end, dim3(slices * SLICE_WAVES / ROW_WAVES), dim3(ROW_WAVES * WAVE), st, a);
}

size_t fikit_cache_compact_workspace_bytes(uint32_t n_requests, uint32_t table_width, uint32_t n_blocks) {
  if (!blocks_fit(n_requests, 0, n_blocks) || one_launch(n_requests, n_requests, table_width, n_blocks, COMPACT_CELLS)) return 0;
  return static_cast<size_t>(CompactParts(n_blocks).bytes);
}

int fikit_cache_compact(const int32_t* d_block_table, uint32_t table_width, const int32_t* d_lengths, uint32_t n_requests,
                        uint32_t block_tokens, uint32_t n_blocks, const int32_t* d_free, uint32_t n_free, int32_t* d_new_table,
                        fikit_block_copy* d_copies, int32_t* d_new_free, int32_t* d_counts, int32_t* d_status, void* d_workspace,
                        size_t workspace_bytes, void* hip_stream) {
  if (int rc = blocks_status(d_block_table, table_width, d_lengths, n_requests, 0, block_tokens, n_blocks, d_free, n_free, d_status)) return rc;
  const uint32_t room = n_free < n_blocks / 2 ? n_free : n_blocks / 2;
  if ((n_requests > 0 && table_width > 0 && !d_new_table) || (room > 0 && !d_copies) || (n_free > 0 && !d_new_free)) return FIKIT_INVALID_ARG;
  if (!d_counts || !aligned(d_new_table, 4) || !aligned(d_copies, 8) || !aligned(d_new_free, 4) || !aligned(d_counts, 4)) return FIKIT_INVALID_ARG;
  const uint64_t table = 4ull * table_width * n_requests;
  const Extent extents[] = {{d_new_table, table}, {d_copies, sizeof(fikit_block_copy) * room}, {d_new_free, 4ull * n_free}, {d_counts, 8},
                            {d_block_table, table}, {d_lengths, 4ull * n_requests}, {d_free, 4ull * n_free}};
  if (!outputs_apart(extents, 4, 7)) return FIKIT_INVALID_ARG;
  BlocksArgs a = blocks_args(d_block_table, table_width, d_lengths, n_requests, block_tokens, n_blocks, d_free, n_free, d_status);
  a.new_table = d_new_table;
  a.copies = reinterpret_cast<int2*>(d_copies);
  a.new_free = d_new_free;
  a.counts = d_counts;
  a.room = room;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (const uint32_t groups = one_launch(n_requests, n_requests, table_width, n_blocks, COMPACT_CELLS))
    return enqueue(k_compact_one, dim3(groups), dim3(BLOCKS_THREADS), st, a);
  const CompactParts parts(n_blocks);
  if (!d_workspace || !aligned(d_workspace, 256)) return FIKIT_INVALID_ARG;
  if (workspace_bytes < parts.bytes) return FIKIT_WORKSPACE_TOO_SMALL;
  const auto part = [&](uint64_t at) { return reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(d_workspace) + at); };
  a.words_of_call = part(0);
  a.flags = reinterpret_cast<uint8_t*>(part(parts.flags));
  a.flags_too = reinterpret_cast<uint8_t*>(part(parts.flags_too));
  a.marks = part(parts.marks);
  a.marks_too = part(parts.marks_too);
  a.sums = part(parts.sums);
  a.sums_too = part(parts.sums_too);
  a.before = part(parts.before);
  const dim3 rows(ROW_WAVES * WAVE);
  const uint32_t slices = static_cast<uint32_t>(slices_of(n_blocks));
  const uint32_t waves = n_requests + (n_free + WAVE - 1) / WAVE;
  if (int rc = enqueue(k_compact_begin, clear_groups(a.words), dim3(BLOCKS_THREADS), st, a)) return rc;
  if (waves > 0)
    if (int rc = enqueue(k_compact_mark, dim3((waves + ROW_WAVES - 1) / ROW_WAVES), rows, st, a)) return rc;
  if (int rc = enqueue(k_blocks_pack<false>, dim3(slices), dim3(SLICE), st, a)) return rc;
  if (int rc = enqueue(k_compact_lists, dim3(slices * SLICE_WAVES / ROW_WAVES), rows, st, a)) return rc;
  return n_requests > 0 ? enqueue(k_compact_rows, dim3((n_requests + ROW_WAVES - 1) / ROW_WAVES), rows, st, a) : FIKIT_OK;
}

int fikit_cache_copy(const fikit_cache* h_caches, uint32_t n_caches, const fikit_block_copy* d_copies, uint32_t n_copies,
                     int32_t* d_status, void* hip_stream) {
  if (!d_status || !aligned(d_status, 4) || !aligned(d_copies, 8) || n_copies > 0x7fffffffu || (n_caches > 0 && !h_caches)) return FIKIT_INVALID_ARG;
  for (uint32_t i = 0; i < n_caches; ++i) {
    if (int rc = cache_status(h_caches + i)) return rc;
    const fikit_cache &c = h_caches[i], &one = h_caches[0];
    if (c.n_blocks != one.n_blocks || c.kv_heads != one.kv_heads || c.block_tokens != one.block_tokens || c.head_dim != one.head_dim) return FIKIT_INVALID_ARG;
  }
  if (n_caches == 0 || n_copies == 0) return FIKIT_OK;
  if (!d_copies) return FIKIT_INVALID_ARG;
  CopyArgs a{};
  a.copies = reinterpret_cast<const int2*>(d_copies);
  a.status = d_status;
  a.n_blocks = h_caches->n_blocks;
  a.heads = h_caches->kv_heads;
  a.block_bytes = a.heads * h_caches->block_tokens * h_caches->head_dim;      // (below 2^31)
  a.chunks = (a.block_bytes + COPY_CHUNK - 1) / COPY_CHUNK;
  a.n_copies = n_copies;
  for (uint32_t from = 0; from < n_caches; from += COPY_CACHES) {
    const uint32_t n = n_caches - from < COPY_CACHES ? n_caches - from : COPY_CACHES;
    for (uint32_t i = 0; i < n; ++i) a.caches[i] = {h_caches[from + i].d_k, h_caches[from + i].d_v, h_caches[from + i].d_k_exp, h_caches[from + i].d_v_exp};
    a.per_copy = 2 * n * a.chunks;                   // (at most 64 * 2^17)
    const uint32_t most = COPY_GROUPS / a.per_copy;
    a.step = most < 1 ? 1 : most < n_copies ? most : n_copies;
    if (int rc = enqueue(k_cache_copy, dim3(a.per_copy * a.step), dim3(COPY_THREADS), static_cast<hipStream_t>(hip_stream), a)) return rc;
  }
  return FIKIT_OK;
}

int fikit_rotate_heads(const fikit_vectors* h_q, const fikit_vectors* h_k, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim,
                       int32_t value_type, const void* d_q_weight, const void* d_k_weight, float epsilon, const int32_t* d_positions,
                       const float* d_frequencies, uint32_t rotary_dim, int32_t pairs, uint32_t n_tokens, const fikit_vectors* h_q_out,
                       const fikit_vectors* h_k_out, int32_t* d_status, void* hip_stream) {
  if (!type_ok(value_type) || !d_status || !aligned(d_status, 4) || n_tokens > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (pairs != FIKIT_PAIRS_HALVES && pairs != FIKIT_PAIRS_NEIGHBOURS) return FIKIT_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return FIKIT_UNSUPPORTED;
  if (rotary_dim % 16 || rotary_dim > head_dim || q_heads > 65535 || kv_heads > 65535) return FIKIT_UNSUPPORTED;
  if (!aligned(d_q_weight, 16) || !aligned(d_k_weight, 16)) return FIKIT_INVALID_ARG;
  if ((d_q_weight || d_k_weight) && !(epsilon >= 0x1p-126f && epsilon <= 3.4028234663852886e38f)) return FIKIT_INVALID_ARG;
  if (n_tokens == 0 || (q_heads == 0 && kv_heads == 0)) return FIKIT_OK;
  if (!d_positions || !aligned(d_positions, 4) || !aligned(d_frequencies, 4) || (rotary_dim > 0 && !d_frequencies)) return FIKIT_INVALID_ARG;
  struct { const fikit_vectors *in, *out; uint32_t heads; } sides[] = {{h_q, h_q_out, q_heads}, {h_k, h_k_out, kv_heads}};
  for (const auto& s : sides)
    if (s.heads > 0 && (!vectors_ok(s.in) || !vectors_ok(s.out) || !apart(s.out, s.heads, n_tokens, head_dim) ||
                        !(in_place(s.in, s.out, s.heads, n_tokens) || apart(s.out, s.heads, s.in, s.heads, n_tokens, head_dim))))
      return FIKIT_INVALID_ARG;
  if (q_heads > 0 && kv_heads > 0 &&
      (!apart(h_q_out, q_heads, h_k_out, kv_heads, n_tokens, head_dim) || !apart(h_q_out, q_heads, h_k, kv_heads, n_tokens, head_dim) ||
       !apart(h_k_out, kv_heads, h_q, q_heads, n_tokens, head_dim)))
    return FIKIT_INVALID_ARG;
  RotateArgs a{};
  if (q_heads > 0) { a.q = *h_q; a.q_out = *h_q_out; }
  if (kv_heads > 0) { a.k = *h_k; a.k_out = *h_k_out; }
  a.q_weight = d_q_weight;
  a.k_weight = d_k_weight;
  a.positions = d_positions;
  a.frequencies = d_frequencies;
  a.status = d_status;
  a.q_heads = q_heads;
  a.kv_heads = kv_heads;
  a.half = rotary_dim / 2;
  const uint32_t heads = static_cast<uint32_t>(rotate_heads(static_cast<int>(head_dim)));
  a.q_passes = (q_heads + heads - 1) / heads;
  a.passes = a.q_passes + (kv_heads + heads - 1) / heads;
  // a wave for each pass as long as that does not fill the chip, else for each token, whose angles then are computed once
  a.per = static_cast<uint64_t>(n_tokens) * a.passes <= ROTATE_SPREAD ? 1 : a.passes;
  a.parts = (a.passes + a.per - 1) / a.per;
  a.units = n_tokens * a.parts;
  a.epsilon = epsilon;
  const bool past = 2ull * n_tokens * (q_heads + kv_heads) * head_dim >= ROTATE_PAST;
  RotateCall call{a, pairs == FIKIT_PAIRS_NEIGHBOURS, past, static_cast<hipStream_t>(hip_stream)};
  return value_type == FIKIT_BF16 ? call.with_dim<Bf16>(head_dim) : call.with_dim<F16>(head_dim);
}

size_t fikit_token_scores_workspace_bytes(uint32_t n_rows, uint32_t vocabulary, int32_t value_type, uint32_t n_top) {
  if (!logits_ok(value_type) || n_rows > MOST_GROUPS || vocabulary > 0x7fffffffu || n_top > SCORES_MOST) return 0;
  return static_cast<size_t>(scores_cut(n_rows, vocabulary, value_type, n_top).bytes);
}

int fikit_token_scores(const void* d_logits, int32_t value_type, uint64_t row_stride, uint32_t n_rows, uint32_t vocabulary, float scale,
                       const int32_t* d_tokens, uint32_t n_top, float* d_logprob, float* d_entropy, float* d_lse, int32_t* d_top_tokens,
                       float* d_top_logprob, int32_t* d_status, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!logits_ok(value_type) || !d_status || !aligned(d_status, 4) || n_rows > 0x7fffffffu || vocabulary > 0x7fffffffu) return FIKIT_INVALID_ARG;
  if (!(scale >= 0x1p-100f && scale <= 0x1p100f)) return FIKIT_INVALID_ARG;
  if (n_top > SCORES_MOST || n_rows > MOST_GROUPS) return FIKIT_UNSUPPORTED;
  if (n_rows == 0) return FIKIT_OK;
  if ((vocabulary > 0 && !d_logits) || !aligned(d_logits, value_type == FIKIT_F32 ? 4 : 2) || !aligned(d_tokens, 4) || !aligned(d_logprob, 4) ||
      !aligned(d_entropy, 4) || !aligned(d_lse, 4) || !aligned(d_top_tokens, 4) || !aligned(d_top_logprob, 4))
    return FIKIT_INVALID_ARG;
  if (n_top > 0 && (!d_top_tokens || !d_top_logprob)) return FIKIT_INVALID_ARG;
  const uint64_t tops = 4ull * n_rows * n_top, row = 4ull * n_rows;
  const Extent extents[] = {{d_logprob, d_logprob ? row : 0}, {d_entropy, d_entropy ? row : 0}, {d_lse, d_lse ? row : 0}, {d_top_tokens, tops}, {d_top_logprob, tops},
                            {d_logits, ((n_rows - 1) * row_stride + vocabulary) * (value_type == FIKIT_F32 ? 4 : 2)}, {d_tokens, d_tokens ? row : 0}};
  if (!outputs_apart(extents, 5, 7)) return FIKIT_INVALID_ARG;
  const ScoresCut c = scores_cut(n_rows, vocabulary, value_type, n_top);
  if (c.bytes > 0) {
    if (!d_workspace || !aligned(d_workspace, 256)) return FIKIT_INVALID_ARG;
    if (workspace_bytes < c.bytes) return FIKIT_WORKSPACE_TOO_SMALL;
  }
  ScoresArgs a{};
  a.logits = d_logits;
  a.row_stride = row_stride;
  a.tokens = d_tokens;
  a.logprob = d_logprob;
  a.entropy = d_entropy;
  a.lse = d_lse;
  a.top_tokens = d_top_tokens;
  a.top_logprob = d_top_logprob;
  a.status = d_status;
  a.sums = static_cast<float4*>(d_workspace);
  a.lists = reinterpret_cast<float2*>(static_cast<unsigned char*>(d_workspace) + c.sums_bytes);
  a.rows = n_rows;
  a.vocabulary = vocabulary;
  a.n_top = n_top;
  a.parts = c.parts;
  a.per_part = c.per_part;
  a.scale = scale;
  a.c = scale * LOG2E;
  ScoresCall call{a, c.waves, static_cast<hipStream_t>(hip_stream)};
  return value_type == FIKIT_BF16 ? call.run<LogitsBf16>() : value_type == FIKIT_F16 ? call.run<LogitsF16>() : call.run<LogitsF32>();
}

}  // extern "C"
