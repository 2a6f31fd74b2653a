// Blocks of the paged cache: requests that fork and end, compaction, copies.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// Nobody counts who holds a block: what is held follows from the table and the lengths, so a call marks blocks in bitmaps of its own and the
// order of its marks changes nothing.  With L = a request's length and B = tokens per block it holds the first ceil(L / B) entries of
// its row.
//
// Four bytes are read for an entry and four written for an entry of the new table: bound by the latency of launches and of loads one
// behind the other.

struct BlocksArgs {
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* parents;
  const int32_t* free_blocks;
  int32_t* new_table;
  int32_t* new_lengths;
  int2* copies;
  int32_t* new_free;
  int32_t* counts;
  int32_t* status;
  uint8_t* flags;           // a byte for each block, in whole words of the bitmaps; fork: blocks of requests that nobody continues; compaction: used blocks
  uint8_t* flags_too;       // fork: blocks of the others; compaction: free ones
  uint8_t* flags_free;      // fork: free ones
  uint32_t* marks;          // bitmaps, in whole slices; fork: blocks given back; compaction: used blocks
  uint32_t* marks_too;      // compaction: free blocks
  uint32_t* sums;           // [slices]: how many of them are marked in a slice
  uint32_t* sums_too;       // how many are free
  uint32_t* first;          // fork, [n_requests]: a request's first child, or NO_CHILD
  int32_t* rank;            // fork, [n_children]: a child's place among those that need a block for a copy, or -1
  uint32_t* wants;          // fork, [n_children]: the child of a place
  uint32_t* before;         // compaction, [words]: used blocks before a word's
  uint32_t* words_of_call;  // fork: blocks taken; compaction: the border, used blocks before it
  uint32_t n_requests, n_children, width, n_blocks, n_free, room, words;
  uint32_t shift;           // of the block length
};

constexpr int BLOCKS_THREADS = 1024, ROW_WAVES = 4;
constexpr uint32_t BLOCKS_MOST_REQUESTS = 16384, BLOCKS_MOST_BLOCKS = 1u << 20;
constexpr uint32_t SLICE = 256;                // words of the bitmaps that are counted together
constexpr uint32_t SLICE_WAVES = 64;           // waves that list a slice's blocks (16: 4.1 us for a fork and 5.2 for a compaction, 64: 3.3 and 4.2)
constexpr uint32_t NO_CHILD = 0xffffffffu;

__device__ __forceinline__ uint32_t pages_of(const BlocksArgs& a, uint32_t length) { return (length + (1u << a.shift) - 1) >> a.shift; }

// Can a request be that long?  (no more entries than its row of the table has)
__device__ __forceinline__ bool length_ok(const BlocksArgs& a, int32_t length) {
  return length >= 0 && (static_cast<uint64_t>(length) + (1u << a.shift) - 1) >> a.shift <= a.width;
}

// Whole sets of flags as words of 16 bytes.
template <bool FORK>
__device__ __forceinline__ void clear_flags(const BlocksArgs& a, uint32_t from, uint32_t stride) {
  for (uint32_t i = from; i < 2 * a.words; i += stride) {
    reinterpret_cast<u32x4*>(a.flags)[i] = reinterpret_cast<u32x4*>(a.flags_too)[i] = u32x4{0, 0, 0, 0};
    if constexpr (FORK) reinterpret_cast<u32x4*>(a.flags_free)[i] = u32x4{0, 0, 0, 0};
  }
}

// 64 entries of the free list in a wave, from the first-th on.  (The status is looked at behind the load.)
__device__ __forceinline__ void mark_free(const BlocksArgs& a, uint32_t first, bool stop, uint8_t* flags) {
  const uint32_t i = first + lane_id();
  if (i >= a.n_free) return;
  const uint32_t block = static_cast<uint32_t>(a.free_blocks[i]);
  if (stop) return;
  if (block < a.n_blocks) flags[block] = 1;
  else *a.status = FIKIT_INVALID_ARG;
}

// The bitmaps from the flags.  (Many workgroups mark at once.  Or-ing bits into words in memory took 12.2 us for 176,000 marks; stores of a byte, of which none
// waits for another, and this take 4.0 and 2.7.)
__device__ __forceinline__ uint32_t packed(const uint8_t* flags, uint32_t word) {
  uint32_t bits = 0;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const u32x4 w = reinterpret_cast<const u32x4*>(flags)[2 * word + half];
#pragma unroll
    for (int i = 0; i < 4; ++i)       // four bytes of 0 or 1
      bits |= (w[i] * 0x01020408u >> 24 & 15u) << (16 * half + 4 * i);
  }
  return bits;
}
// A slice in a workgroup, with how many are marked in it, so that who lists them reads a number for each slice and the words of its own.  (Lists for which each
// workgroup added up all words took 7.7 us for a fork and 9.3 for a compaction, these take 3.3 and 4.2.)
template <bool FORK>
__global__ __launch_bounds__(SLICE) void k_blocks_pack(BlocksArgs a) {
  __shared__ uint32_t waves[SLICE / WAVE];
  const uint32_t w = blockIdx.x * SLICE + threadIdx.x;
  uint32_t marks = 0, marks_too = 0, spare = 0;
  if (w < a.words) {
    marks = packed(a.flags, w);
    marks_too = packed(a.flags_too, w);
    spare = FORK ? packed(a.flags_free, w) : marks_too;
  }
  if (((FORK ? marks | marks_too : marks) & spare) && !stopped(a.status)) *a.status = FIKIT_INVALID_ARG;        // used and free
  if constexpr (FORK) marks &= ~marks_too;
  else a.marks_too[w] = marks_too;
  a.marks[w] = marks;
  const uint32_t sum = sum_over_wave(__popc(marks) << 16 | __popc(spare));       // (up to 8192 each)
  if (lane_id() == 0) waves[threadIdx.x / WAVE] = sum;
  __syncthreads();
  if (threadIdx.x > 0) return;
  uint32_t all = 0;
  for (uint32_t i = 0; i < SLICE / WAVE; ++i) all += waves[i];
  a.sums[blockIdx.x] = all >> 16;
  a.sums_too[blockIdx.x] = all & 0xffffu;
}

// The counts of all slices in a wave, two neighbours to a lane.
struct SliceSums {
  static_assert(BLOCKS_MOST_BLOCKS / 32 / SLICE <= 2 * WAVE, "two slices to a lane");
  uint32_t first, both, total, before;                // of the lane's slices, of all, of those before the lane's

  __device__ __forceinline__ SliceSums(const BlocksArgs& a, const uint32_t* sums) {
    const uint32_t at = 2 * lane_id(), slices = (a.words + SLICE - 1) / SLICE;
    first = at < slices ? sums[at] : 0;
    both = first + (at + 1 < slices ? sums[at + 1] : 0);
  }
  __device__ __forceinline__ void add_up() {
    const uint32_t upto = wave_incl_scan_u32(both);
    before = upto - both;
    total = read_lane_u32(upto, WAVE - 1);
  }
  __device__ __forceinline__ uint32_t before_slice(uint32_t slice) const {
    return read_lane_u32(slice & 1 ? before + first : before, slice / 2);
  }
};

// A slice's words in a wave, four neighbours to a lane.
struct SliceWords {
  u32x4 marks;
  uint32_t before;                                    // marked ones before the lane's

  __device__ __forceinline__ SliceWords(const uint32_t* words, uint32_t slice) : marks(reinterpret_cast<const u32x4*>(words)[slice * WAVE + lane_id()]) {}
  __device__ __forceinline__ void add_up(uint32_t before_slice) {
    const uint32_t mine = __popc(marks[0]) + __popc(marks[1]) + __popc(marks[2]) + __popc(marks[3]);
    before = before_slice + wave_incl_scan_u32(mine) - mine;
  }
};

// The words that each wave lists, two at a time: a lane's word of both, and the marked ones before the lane's block.
constexpr uint32_t WAVE_WORDS = SLICE / SLICE_WAVES;
__device__ __forceinline__ uint32_t word_of(const SliceWords& s, uint32_t first, uint32_t pair, uint32_t& before) {
  const uint32_t e = 2 * pair % 4, from = first / 4 + pair / 2, lane = lane_id();
  uint32_t until = s.before;
  if (e == 2) until += __popc(s.marks[0]) + __popc(s.marks[1]);
  const uint32_t low = read_lane_u32(s.marks[e], from), high = read_lane_u32(s.marks[e + 1], from), at = read_lane_u32(until, from);
  const uint32_t word = lane < 32 ? low : high;
  before = at + (lane < 32 ? 0 : __popc(low)) + __popc(word & ((1u << lane % 32) - 1));
  return word;
}

// f(page, entry) for the first `pages` entries of a row, by a wave, several loads on their way; from page `first` on.
template <typename F>
__device__ __forceinline__ void each_page(const int32_t* entries, uint32_t pages, F f, uint32_t first = 0) {
  constexpr int AHEAD = 4;
  for (uint32_t from = first + lane_id(); from < pages; from += AHEAD * WAVE) {
    int32_t held[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (from + i * WAVE < pages) held[i] = entries[from + i * WAVE];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (from + i * WAVE < pages) f(from + i * WAVE, held[i]);
  }
}

// ---- fork -------------------------------------------------------------------------------------------------------
//
// Child i continues request parents[i].  The first child keeps the parent's last block if that is not full, each later one needs a block:
// its place among those is a prefix sum over the children.  Blocks to take come from the front of (free blocks, blocks given back in
// ascending order); what is left of the two is the new list.  The kernels of both calls load what they may before they look at the status.
//
// 8192 children of 4096 requests over 107,000 blocks: 17 to 19 us in four launches, of which marks of the free blocks, to refuse those in use, take 0.4.

// The children, in one workgroup, PER requests and children to a thread, whose loads are on their way at once; the others clear the bitmaps.  (8192 children
// 6.0 us, 1500 4.0; with code for 16,384, which is fetched although no thread has work in it, 7.8 and 6.9.)
template <uint32_t PER>
__global__ __launch_bounds__(BLOCKS_THREADS) void k_fork_begin(BlocksArgs a) {
  __shared__ uint32_t first[PER * BLOCKS_THREADS], sums[PER * BLOCKS_THREADS / WAVE], scan[BLOCKS_THREADS / WAVE];
  if (blockIdx.x > 0) {
    clear_flags<true>(a, (blockIdx.x - 1) * BLOCKS_THREADS + threadIdx.x, (gridDim.x - 1) * BLOCKS_THREADS);
    return;
  }
  const bool stop = stopped(a.status);         // (nobody else writes it in this launch)
  constexpr uint32_t WAVES = BLOCKS_THREADS / WAVE;
  bool bad = false;
  const uint32_t wave = uniform(threadIdx.x / WAVE);
  int32_t lengths[PER], parents[PER];
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const uint32_t at = i * BLOCKS_THREADS + threadIdx.x;
    lengths[i] = at < a.n_requests ? a.lengths[at] : 0;
    parents[i] = at < a.n_children ? a.parents[at] : -1;
  }
  if (stop) return;
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const uint32_t at = i * BLOCKS_THREADS + threadIdx.x;
    if (at < a.n_requests) first[at] = NO_CHILD;
    bad |= !length_ok(a, lengths[i]) || parents[i] < -1 || (parents[i] >= 0 && static_cast<uint32_t>(parents[i]) >= a.n_requests);
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    if (parents[i] >= 0) atomicMin(&first[parents[i]], i * BLOCKS_THREADS + threadIdx.x);
    lengths[i] = parents[i] >= 0 ? a.lengths[parents[i]] : 0;
  }
  __syncthreads();
  for (uint32_t r = threadIdx.x; r < a.n_requests; r += BLOCKS_THREADS) a.first[r] = first[r];
  // how many of each 64 children need a block, then the sums of the 64s before: a child's place
  uint64_t needs[PER];
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const bool need = parents[i] >= 0 && (static_cast<uint32_t>(lengths[i]) & ((1u << a.shift) - 1)) && first[parents[i]] != i * BLOCKS_THREADS + threadIdx.x;
    needs[i] = ballot(need);
    if (lane_id() == 0) sums[i * WAVES + wave] = popc64(needs[i]);
  }
  __syncthreads();
  uint32_t taken;
  const uint32_t before = block_excl_scan_1024(threadIdx.x < PER * WAVES ? sums[threadIdx.x] : 0, scan, taken);
  if (threadIdx.x < PER * WAVES) sums[threadIdx.x] = before;
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < PER; ++i) {
    const uint32_t c = i * BLOCKS_THREADS + threadIdx.x, place = sums[i * WAVES + wave] + popc_below(needs[i]);
    if (c < a.n_children) {
      const bool need = needs[i] >> lane_id() & 1;
      a.rank[c] = need ? static_cast<int32_t>(place) : -1;
      if (need) a.wants[place] = c;
    }
  }
  if (threadIdx.x == 0) a.words_of_call[0] = taken;
}

// A wave for each request, which marks its blocks, for each child, which writes its row, and for 64 free blocks, which marks them: one that is in use, or
// there twice, would be handed out while somebody holds it.
__global__ __launch_bounds__(ROW_WAVES * WAVE) void k_fork_rows(BlocksArgs a) {
  const bool stop = stopped(a.status);
  const uint32_t lane = lane_id(), row = blockIdx.x * ROW_WAVES + uniform(threadIdx.x / WAVE);
  if (row < a.n_requests) {
    const uint32_t pages = pages_of(a, static_cast<uint32_t>(a.lengths[row])), first = a.first[row];
    if (stop) return;
    uint8_t* flags = first == NO_CHILD ? a.flags : a.flags_too;
    const int32_t* entries = a.table + static_cast<uint64_t>(row) * a.width;
    each_page(entries, pages, [&](uint32_t, int32_t entry) {
      const uint32_t block = static_cast<uint32_t>(entry);
      if (block < a.n_blocks) flags[block] = 1;
      else *a.status = FIKIT_INVALID_ARG;
    });
    return;
  }
  const uint32_t c = row - a.n_requests;
  if (c >= a.n_children) return mark_free(a, (c - a.n_children) * WAVE, stop, a.flags_free);
  const int32_t p = a.parents[c], rank = a.rank[c];
  if (stop) return;
  const int32_t length = p >= 0 ? a.lengths[p] : 0;
  if (lane == 0) a.new_lengths[c] = length;
  const uint32_t pages = pages_of(a, static_cast<uint32_t>(length));
  const int32_t* entries = a.table + static_cast<uint64_t>(p >= 0 ? p : 0) * a.width;
  int32_t* out = a.new_table + static_cast<uint64_t>(c) * a.width;
  each_page(entries, pages, [&](uint32_t page, int32_t block) {
    if (page + 1 == pages && rank >= 0) {
      a.copies[rank].x = block;
      if (static_cast<uint32_t>(rank) < a.n_free) {
        block = a.free_blocks[rank];
        a.copies[rank].y = block;
      }                                          // (else what is given back says which: k_fork_end)
    }
    out[page] = block;
  });
  for (uint32_t page = pages + lane; page < a.width; page += WAVE) out[page] = -1;
}

// The lists, in waves that do not wait for one another.
__global__ __launch_bounds__(ROW_WAVES * WAVE) void k_fork_end(BlocksArgs a) {
  const bool stop = stopped(a.status);
  const uint32_t row = blockIdx.x * ROW_WAVES + uniform(threadIdx.x / WAVE), slice = row / SLICE_WAVES, word = row % SLICE_WAVES * WAVE_WORDS;
  const uint32_t lane = lane_id(), taken = a.words_of_call[0];
  SliceSums sums(a, a.sums), spare(a, a.sums_too);
  SliceWords words(a.marks, slice);
  if (stop) return;
  sums.add_up();
  spare.add_up();
  words.add_up(sums.before_slice(slice));
  const uint32_t given = sums.total, total = a.n_free + given;          // (as free blocks are not in use, nor there twice, at most n_blocks)
  if (spare.total != a.n_free || taken > total) {                       // free twice; too few
    if (lane == 0) *a.status = spare.total != a.n_free ? FIKIT_INVALID_ARG : FIKIT_CACHE_FULL;
    return;
  }
#pragma unroll
  for (uint32_t pair = 0; pair < WAVE_WORDS / 2; ++pair) {
    uint32_t place;
    const bool is_given = word_of(words, word, pair, place) >> lane % 32 & 1;
    const uint32_t block = (slice * SLICE + word + 2 * pair) * 32 + lane;
    place += a.n_free;
    if (is_given && place >= taken) {
      a.new_free[place - taken] = static_cast<int32_t>(block);
    } else if (is_given) {
      const uint32_t c = a.wants[place];
      a.copies[place].y = static_cast<int32_t>(block);
      a.new_table[static_cast<uint64_t>(c) * a.width + pages_of(a, static_cast<uint32_t>(a.new_lengths[c])) - 1] = static_cast<int32_t>(block);
    }
  }
  const uint32_t from = blockIdx.x * ROW_WAVES * WAVE + threadIdx.x, stride = gridDim.x * ROW_WAVES * WAVE;
  for (uint32_t i = taken + from; i < a.n_free; i += stride) a.new_free[i - taken] = a.free_blocks[i];
  for (uint32_t i = total - taken + from; i < a.n_blocks; i += stride) a.new_free[i] = -1;
  for (uint32_t i = taken + from; i < a.n_children; i += stride) a.copies[i] = make_int2(-1, -1);
  if (from == 0) {
    a.counts[0] = static_cast<int32_t>(taken);
    a.counts[1] = static_cast<int32_t>(given);
    a.counts[2] = static_cast<int32_t>(total - taken);
  }
}

// ---- one launch -------------------------------------------------------------------------------------------------
//
// Up to ONE_REQUESTS requests and children, ONE_BLOCKS blocks and FORK_CELLS or COMPACT_CELLS entries of the table, with bitmaps in LDS: every workgroup marks all
// blocks for itself and writes its share of the outputs, so that none waits for another.  A fork has one more, which marks the free blocks too and alone says
// what is wrong, so that the others neither read all of that list nor find different errors.  128 beams of 32 prompts 6.1 us, their compaction 5.9; in the launches
// that larger sizes take, 13 and 16.
//
// The marks that every workgroup makes bound it, and with them the entries that are read.  Calls of 128 requests whose rows are full, of scattered blocks and of
// neighbouring ones, whose bits lie in one word; compactions of 16 requests, in several launches, come to 17 to 25 us for scattered blocks:
//
//                        fork                                compaction
//   entries              scattered   neighbours   several    scattered   neighbours   several
//   8192                   6.9          13          12          8.9          15        17
//   16,384                 9.0          21          12         11            23        14-17
//   32,768                12.6          34          12         14            35        14-18
//   65,536                20            52          12         20            53        16-19
//
// The new table's entries cost the same either way: 1024 children of one request, 16.8 million of them, 25 us and 28.

constexpr uint32_t ONE_REQUESTS = BLOCKS_THREADS, ONE_BLOCKS = 32 * BLOCKS_THREADS, ONE_MOST_GROUPS = 64, FORK_CELLS = 16384, COMPACT_CELLS = 32768;

struct OneLds {
  uint32_t marks[BLOCKS_THREADS], marks_too[BLOCKS_THREADS], pages[ONE_REQUESTS], scan[BLOCKS_THREADS / WAVE];
};

// f(row, entry) for the entries of all requests, by a workgroup, several loads on their way.
template <typename F>
__device__ __forceinline__ void each_entry(const BlocksArgs& a, const uint32_t* pages, F f) {
  constexpr int AHEAD = 8;
  const uint32_t rows = BLOCKS_THREADS / a.width, rest = BLOCKS_THREADS % a.width;
  uint32_t row = threadIdx.x / a.width, page = threadIdx.x % a.width;
  while (row < a.n_requests) {
    int32_t held[AHEAD];
    uint32_t of[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const bool there = row < a.n_requests && page < pages[row < a.n_requests ? row : 0];
      of[i] = there ? row : ~0u;
      if (there) held[i] = a.table[row * a.width + page];
      row += rows;
      page += rest;
      if (page >= a.width) { page -= a.width; ++row; }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (of[i] != ~0u) f(of[i], static_cast<uint32_t>(held[i]));
  }
}

// The k-th marked block: word(w) are the marks, before[w] those before them, ascending.
template <typename F>
__device__ __forceinline__ uint32_t marked_block(const uint32_t* before, uint32_t k, F word) {
  uint32_t lo = 0, hi = BLOCKS_THREADS;
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (before[mid] <= k) lo = mid; else hi = mid;
  }
  uint32_t left = word(lo);
  for (uint32_t skip = k - before[lo]; skip > 0; --skip) left &= left - 1;
  return lo * 32 + __ffs(static_cast<int>(left)) - 1;
}

__global__ __launch_bounds__(BLOCKS_THREADS) void k_fork_one(BlocksArgs a) {
  __shared__ OneLds lds;
  __shared__ uint32_t before[BLOCKS_THREADS], spare[BLOCKS_THREADS], first[ONE_REQUESTS], ranks[ONE_REQUESTS];
  __shared__ int32_t lengths[ONE_REQUESTS], parents[ONE_REQUESTS], fresh[ONE_REQUESTS];
  const uint32_t t = threadIdx.x, lane = lane_id(), waves = BLOCKS_THREADS / WAVE, groups = gridDim.x - 1, mine = blockIdx.x * waves + uniform(t / WAVE);
  const bool checks = blockIdx.x == groups, stop = stopped(a.status);
  const int32_t length = t < a.n_requests ? a.lengths[t] : 0, parent = t < a.n_children ? a.parents[t] : -1;
  const bool fits = length_ok(a, length) && parent >= -1 && (parent < 0 || static_cast<uint32_t>(parent) < a.n_requests);
  lds.marks[t] = lds.marks_too[t] = spare[t] = 0;
  first[t] = NO_CHILD;
  lengths[t] = length;
  parents[t] = parent;
  lds.pages[t] = fits ? pages_of(a, static_cast<uint32_t>(length)) : 0;
  if (__syncthreads_or(stop || !fits)) {
    if (!__syncthreads_or(stop) && checks && t == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  if (parent >= 0) atomicMin(&first[parent], t);
  // what the wave's first row begins with is on its way from here on
  const int32_t my_parent = !checks && mine < a.n_children ? parents[mine] : -1;
  const uint32_t my_pages = my_parent >= 0 ? lds.pages[my_parent] : 0;
  const int32_t early = lane < my_pages ? a.table[static_cast<uint64_t>(my_parent) * a.width + lane] : 0;
  constexpr uint32_t AHEAD = 8;
  int32_t held[AHEAD];                                           // (so are the first free blocks)
  const auto load_free = [&](uint32_t from) {
#pragma unroll
    for (uint32_t j = 0; j < AHEAD; ++j)
      if (from + j * BLOCKS_THREADS < a.n_free) held[j] = a.free_blocks[from + j * BLOCKS_THREADS];
  };
  if (checks) load_free(t);
  __syncthreads();
  bool bad = false;
  if (a.width > 0)
    each_entry(a, lds.pages, [&](uint32_t row, uint32_t block) {
      if (block < a.n_blocks) atomicOr(&(first[row] == NO_CHILD ? lds.marks : lds.marks_too)[block / 32], 1u << block % 32);
      else bad = true;
    });
  const int32_t child_length = parent >= 0 ? lengths[parent] : 0;
  const bool need = (static_cast<uint32_t>(child_length) & ((1u << a.shift) - 1)) && first[parent] != t;
  bad = __syncthreads_or(bad);
  if (checks && !bad) {
    // A block's bit in the word of its number, so that neighbours, as lists hold them, lie in different words: 29,696 of those 12.0 us a call, with their bits in
    // one word 31.  (Scattered ones 11; in several launches 15.)
    for (uint32_t from = t; from < a.n_free;) {
#pragma unroll
      for (uint32_t j = 0; j < AHEAD; ++j)
        if (from + j * BLOCKS_THREADS < a.n_free) {
          const uint32_t block = static_cast<uint32_t>(held[j]), bit = 1u << block / BLOCKS_THREADS % 32;
          if (block >= a.n_blocks) bad = true;
          else bad |= (atomicOr(&spare[block % BLOCKS_THREADS], bit) & bit) || ((lds.marks[block / 32] | lds.marks_too[block / 32]) >> block % 32 & 1);       // there twice, or in use
        }
      from += AHEAD * BLOCKS_THREADS;
      load_free(from);
    }
    bad = __syncthreads_or(bad);
  }
  if (bad) {
    if (checks && t == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  // two sums in one: children that need a block, and blocks given back, up to 32,768
  uint32_t both;
  const uint32_t upto = block_excl_scan_1024(__popc(lds.marks[t] & ~lds.marks_too[t]) | (need ? 1u << 16 : 0), lds.scan, both);
  const uint32_t rank = upto >> 16, taken = both >> 16, given = both & 0xffffu, total = a.n_free + given;
  ranks[t] = need ? rank : ~0u;
  before[t] = upto & 0xffffu;
  if (checks && taken > total && t == 0) *a.status = FIKIT_CACHE_FULL;
  if (checks || taken > total || total - taken > a.n_blocks) return;           // (more than n_blocks: of a list that the one which checks refuses)
  fresh[t] = need && rank < a.n_free ? a.free_blocks[rank] : 0;
  const uint32_t from = blockIdx.x * BLOCKS_THREADS + t, stride = groups * BLOCKS_THREADS;
  const int32_t left = taken + from < a.n_free ? a.free_blocks[taken + from] : 0;
  __syncthreads();
  const auto given_word = [&](uint32_t w) { return lds.marks[w] & ~lds.marks_too[w]; };
  // rows, a wave each
  for (uint32_t c = mine; c < a.n_children; c += groups * waves) {
    const int32_t p = parents[c];
    const uint32_t pages = p >= 0 ? lds.pages[p] : 0, place = ranks[c];
    int32_t* out = a.new_table + static_cast<uint64_t>(c) * a.width;
    const auto put = [&](uint32_t page, int32_t block) {
      if (page + 1 == pages && place != ~0u) {
        const uint32_t one = place < a.n_free ? static_cast<uint32_t>(fresh[c]) : marked_block(before, place - a.n_free, given_word);
        a.copies[place] = make_int2(block, static_cast<int32_t>(one));
        block = static_cast<int32_t>(one);
      }
      out[page] = block;
    };
    if (c == mine && lane < pages) put(lane, early);
    each_page(a.table + static_cast<uint64_t>(p >= 0 ? p : 0) * a.width, pages, put, c == mine ? WAVE : 0);
    for (uint32_t page = pages + lane; page < a.width; page += WAVE) out[page] = -1;
  }
  for (uint32_t block = from; block < a.n_blocks; block += stride) {
    const uint32_t marks = given_word(block / 32), bit = 1u << block % 32, place = a.n_free + before[block / 32] + __popc(marks & (bit - 1));
    if ((marks & bit) && place >= taken) a.new_free[place - taken] = static_cast<int32_t>(block);
  }
  if (taken + from < a.n_free) a.new_free[from] = left;
  for (uint32_t i = taken + from + stride; i < a.n_free; i += stride) a.new_free[i - taken] = a.free_blocks[i];
  for (uint32_t i = total - taken + from; i < a.n_blocks; i += stride) a.new_free[i] = -1;
  for (uint32_t i = taken + from; i < a.n_children; i += stride) a.copies[i] = make_int2(-1, -1);
  if (blockIdx.x > 0) return;
  if (t < a.n_children) a.new_lengths[t] = child_length;
  if (t == 0) {
    a.counts[0] = static_cast<int32_t>(taken);
    a.counts[1] = static_cast<int32_t>(given);
    a.counts[2] = static_cast<int32_t>(total - taken);
  }
}

// ---- compaction -------------------------------------------------------------------------------------------------
//
// Used and free blocks together, ascending: behind the first n_used of them lies the border.  The k-th used block behind the border goes
// to the k-th free one before it, and what lies behind it is the new free list.  3001 requests over 177,000 blocks: 20 us in five launches.

__global__ __launch_bounds__(BLOCKS_THREADS) void k_compact_begin(BlocksArgs a) {
  clear_flags<false>(a, blockIdx.x * BLOCKS_THREADS + threadIdx.x, gridDim.x * BLOCKS_THREADS);
}

// A wave for each request marks its blocks; the waves behind them the free ones, 64 each.
__global__ __launch_bounds__(ROW_WAVES * WAVE) void k_compact_mark(BlocksArgs a) {
  const bool stop = stopped(a.status);
  const uint32_t row = blockIdx.x * ROW_WAVES + uniform(threadIdx.x / WAVE);
  if (row < a.n_requests) {
    const int32_t length = a.lengths[row];
    if (stop) return;
    if (!length_ok(a, length)) {
      *a.status = FIKIT_INVALID_ARG;
      return;
    }
    const uint32_t pages = pages_of(a, static_cast<uint32_t>(length));
    const int32_t* entries = a.table + static_cast<uint64_t>(row) * a.width;
    each_page(entries, pages, [&](uint32_t, int32_t entry) {
      const uint32_t block = static_cast<uint32_t>(entry);
      if (block < a.n_blocks) a.flags[block] = 1;
      else *a.status = FIKIT_INVALID_ARG;
    });
    return;
  }
  mark_free(a, (row - a.n_requests) * WAVE, stop, a.flags_too);
}

struct Border {
  uint32_t block, used;          // the border, and the used blocks before it
};

// The border, if the last of the first `total` used and free blocks is one of a word's; used, all: those before the word.
__device__ __forceinline__ void find_border(uint32_t w, uint32_t marks, uint32_t marks_too, uint32_t used, uint32_t all, uint32_t total, Border* lds) {
  uint32_t of = marks | marks_too;
  if (all >= total || all + __popc(of) < total) return;
  for (uint32_t skip = total - all - 1; skip > 0; --skip) of &= of - 1;
  const uint32_t bit = __ffs(static_cast<int>(of)) - 1, below = bit == 31 ? ~0u : (2u << bit) - 1;
  lds->block = w * 32 + bit + 1;
  lds->used = used + __popc(marks & below);
}

// The border, in a wave: in the slice, the lane's four words and the word in which used and free blocks come to `total`.
__device__ __forceinline__ Border border_of(const BlocksArgs& a, const SliceSums& used, const SliceSums& spare, uint32_t total) {
  if (total == 0) return Border{0, 0};
  const uint32_t lane = lane_id(), upto = used.before + spare.before;
  const uint32_t at = static_cast<uint32_t>(__builtin_ctzll(ballot(upto < total && upto + used.both + spare.both >= total)));
  const uint32_t slice = 2 * at + (read_lane_u32(upto + used.first + spare.first, at) < total ? 1 : 0);
  SliceWords marks(a.marks, slice), marks_too(a.marks_too, slice);
  marks.add_up(used.before_slice(slice));
  marks_too.add_up(spare.before_slice(slice));
  const u32x4 of = marks.marks | marks_too.marks;
  const uint32_t all = marks.before + marks_too.before;
  const uint32_t in = static_cast<uint32_t>(__builtin_ctzll(ballot(all < total && all + __popc(of[0]) + __popc(of[1]) + __popc(of[2]) + __popc(of[3]) >= total)));
  uint32_t left = total - read_lane_u32(all, in), before = read_lane_u32(marks.before, in);
  Border border{0, 0};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t word = read_lane_u32(of[e], in), mine = read_lane_u32(marks.marks[e], in), here = __popc(word);
    if (left > 0 && left <= here) {
      const uint32_t bit = static_cast<uint32_t>(__builtin_ctzll(ballot(lane < 32 && (word >> lane % 32 & 1) && __popc(word & ((1u << lane % 32) - 1)) == left - 1)));
      border.block = (slice * SLICE + 4 * in + e) * 32 + bit + 1;
      border.used = before + __popc(mine & (bit == 31 ? ~0u : (2u << bit) - 1));
    }
    left = left > here ? left - here : 0;
    before += __popc(mine);
  }
  return border;
}

__global__ __launch_bounds__(ROW_WAVES * WAVE) void k_compact_lists(BlocksArgs a) {
  const bool stop = stopped(a.status);
  const uint32_t row = blockIdx.x * ROW_WAVES + uniform(threadIdx.x / WAVE), slice = row / SLICE_WAVES, word = row % SLICE_WAVES * WAVE_WORDS;
  const uint32_t lane = lane_id();
  SliceSums used(a, a.sums), spare(a, a.sums_too);
  SliceWords marks(a.marks, slice), marks_too(a.marks_too, slice);
  if (stop) return;
  used.add_up();
  spare.add_up();
  if (spare.total != a.n_free) {                     // free twice
    if (lane == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  const Border border = border_of(a, used, spare, used.total);
  marks.add_up(used.before_slice(slice));
  marks_too.add_up(spare.before_slice(slice));
#pragma unroll
  for (uint32_t pair = 0; pair < WAVE_WORDS / 2; ++pair) {
    uint32_t used_before, spare_before;
    const uint32_t w = slice * SLICE + word + 2 * pair, block = w * 32 + lane;
    const bool is_used = word_of(marks, word, pair, used_before) >> lane % 32 & 1, is_spare = word_of(marks_too, word, pair, spare_before) >> lane % 32 & 1;
    if (lane % 32 == 0) a.before[w + lane / 32] = used_before;
    if (block >= border.block) {
      if (is_used) a.copies[used_before - border.used].x = static_cast<int32_t>(block);
      if (is_used || is_spare) a.new_free[used_before + spare_before - used.total] = static_cast<int32_t>(block);
    } else if (is_spare) {
      a.copies[spare_before].y = static_cast<int32_t>(block);
    }
  }
  const uint32_t moved = used.total - border.used, from = blockIdx.x * ROW_WAVES * WAVE + threadIdx.x, stride = gridDim.x * ROW_WAVES * WAVE;
  for (uint32_t i = moved + from; i < a.room; i += stride) a.copies[i] = make_int2(-1, -1);
  if (from == 0) {
    a.counts[0] = static_cast<int32_t>(moved);
    a.counts[1] = static_cast<int32_t>(used.total);
    a.words_of_call[0] = border.block;
    a.words_of_call[1] = border.used;
  }
}

// A wave for each request writes its row.
__global__ __launch_bounds__(ROW_WAVES * WAVE) void k_compact_rows(BlocksArgs a) {
  const bool stop = stopped(a.status);
  const uint32_t lane = lane_id(), row = blockIdx.x * ROW_WAVES + uniform(threadIdx.x / WAVE);
  if (row >= a.n_requests) return;
  const uint32_t border = a.words_of_call[0], used = a.words_of_call[1], pages = pages_of(a, static_cast<uint32_t>(a.lengths[row]));
  if (stop) return;
  const int32_t* entries = a.table + static_cast<uint64_t>(row) * a.width;
  int32_t* out = a.new_table + static_cast<uint64_t>(row) * a.width;
  each_page(entries, pages, [&](uint32_t page, int32_t entry) {
    const uint32_t block = static_cast<uint32_t>(entry), w = block / 32, bit = 1u << block % 32;
    out[page] = block >= border ? a.copies[a.before[w] + __popc(a.marks[w] & (bit - 1)) - used].y : entry;
  });
  for (uint32_t page = pages + lane; page < a.width; page += WAVE) out[page] = -1;
}

// In one launch, as a fork.
__global__ __launch_bounds__(BLOCKS_THREADS) void k_compact_one(BlocksArgs a) {
  __shared__ OneLds lds;
  __shared__ uint32_t used_before[BLOCKS_THREADS], spare_before[BLOCKS_THREADS];
  __shared__ uint16_t holes[ONE_BLOCKS / 2];
  __shared__ Border border;
  const uint32_t t = threadIdx.x;
  const bool stop = stopped(a.status);
  const int32_t length = t < a.n_requests ? a.lengths[t] : 0;
  lds.marks[t] = lds.marks_too[t] = 0;
  bool bad = !length_ok(a, length);
  lds.pages[t] = bad ? 0 : pages_of(a, static_cast<uint32_t>(length));
  if (__syncthreads_or(stop)) return;
  const auto put = [&](uint32_t* marks, uint32_t block) {
    if (block < a.n_blocks) atomicOr(&marks[block / 32], 1u << block % 32);
    else bad = true;
  };
  // what the wave's first row begins with, and the first free blocks, are on their way from here on
  const uint32_t lane = lane_id(), waves = BLOCKS_THREADS / WAVE, mine = blockIdx.x * waves + uniform(t / WAVE);
  const int32_t early = mine < a.n_requests && lane < lds.pages[mine] ? a.table[static_cast<uint64_t>(mine) * a.width + lane] : 0;
  constexpr int AHEAD = 4;
  int32_t held[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    if (t + j * BLOCKS_THREADS < a.n_free) held[j] = a.free_blocks[t + j * BLOCKS_THREADS];
  if (a.width > 0) each_entry(a, lds.pages, [&](uint32_t, uint32_t block) { put(lds.marks, block); });
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    if (t + j * BLOCKS_THREADS < a.n_free) put(lds.marks_too, static_cast<uint32_t>(held[j]));
  for (uint32_t i = t + AHEAD * BLOCKS_THREADS; i < a.n_free; i += BLOCKS_THREADS) put(lds.marks_too, static_cast<uint32_t>(a.free_blocks[i]));
  __syncthreads();
  const uint32_t used = lds.marks[t], spare = lds.marks_too[t];
  bad |= (used & spare) != 0;
  uint32_t both;                               // two sums in one, of up to 32,768 each
  const uint32_t upto = block_excl_scan_1024(__popc(used) << 16 | __popc(spare), lds.scan, both);
  const uint32_t sums[2] = {upto >> 16, upto & 0xffffu}, total[2] = {both >> 16, both & 0xffffu};
  used_before[t] = sums[0];
  spare_before[t] = sums[1];
  if (t == 0 && total[0] == 0) border = Border{0, 0};
  find_border(t, used, spare, sums[0], sums[0] + sums[1], total[0], &border);
  if (__syncthreads_or(bad) || total[1] != a.n_free) {             // also: a block that is used and free, or free twice
    if (blockIdx.x == 0 && t == 0) *a.status = FIKIT_INVALID_ARG;
    return;
  }
  // the free blocks before the border, to which used ones go
  for (uint32_t block = t; block < border.block; block += BLOCKS_THREADS) {
    const uint32_t w = block / 32, bit = 1u << block % 32, marks = lds.marks_too[w];
    if (marks & bit) holes[spare_before[w] + __popc(marks & (bit - 1))] = static_cast<uint16_t>(block);
  }
  __syncthreads();
  const auto goes = [&](uint32_t block) {
    const uint32_t w = block / 32;
    return static_cast<int32_t>(holes[used_before[w] + __popc(lds.marks[w] & ((1u << block % 32) - 1)) - border.used]);
  };
  for (uint32_t r = mine; r < a.n_requests; r += gridDim.x * waves) {
    const uint32_t pages = lds.pages[r];
    int32_t* out = a.new_table + static_cast<uint64_t>(r) * a.width;
    const auto write = [&](uint32_t page, int32_t entry) {
      out[page] = static_cast<uint32_t>(entry) >= border.block ? goes(static_cast<uint32_t>(entry)) : entry;
    };
    if (r == mine && lane < pages) write(lane, early);
    each_page(a.table + static_cast<uint64_t>(r) * a.width, pages, write, r == mine ? WAVE : 0);
    for (uint32_t page = pages + lane; page < a.width; page += WAVE) out[page] = -1;
  }
  const uint32_t moved = total[0] - border.used, from = blockIdx.x * BLOCKS_THREADS + t, stride = gridDim.x * BLOCKS_THREADS;
  for (uint32_t block = border.block + from; block < a.n_blocks; block += stride) {
    const uint32_t w = block / 32, bit = 1u << block % 32, in_use = lds.marks[w], both = in_use | lds.marks_too[w];
    if (in_use & bit) a.copies[used_before[w] + __popc(in_use & (bit - 1)) - border.used] = make_int2(static_cast<int32_t>(block), goes(block));
    if (both & bit) a.new_free[used_before[w] + spare_before[w] + __popc(both & (bit - 1)) - total[0]] = static_cast<int32_t>(block);
  }
  for (uint32_t i = moved + from; i < a.room; i += stride) a.copies[i] = make_int2(-1, -1);
  if (from == 0) {
    a.counts[0] = static_cast<int32_t>(moved);
    a.counts[1] = static_cast<int32_t>(total[0]);
  }
}

// ---- copies -----------------------------------------------------------------------------------------------------
//
// A block's codes of one cache lie in one piece, so a workgroup moves 16 KiB of it, four 16-byte loads a thread on their way; memory bound.  5000 blocks
// of 32 KiB in 3 layers, 983 MB read and written: 199 us, 4.9 TB/s, a large copy's rate; with stores through the caches 202, with 4096 workgroups 205.
// 61 blocks of 128 KiB in 4 layers 11.5 us; with loads past the caches 12.7, as the last step's tokens still lie there.
// Workgroups are a piece of a block, of keys or values, in a cache, for every `step`-th entry of the list; a wave looks at 64 of its entries at
// once, so that a long list of which little is used costs little.

constexpr int COPY_CACHES = 32, COPY_THREADS = 256, COPY_LOADS = 4;
constexpr uint32_t COPY_CHUNK = COPY_THREADS * COPY_LOADS * 16;
struct CopyArgs {
  struct { uint8_t *k, *v, *k_exp, *v_exp; } caches[COPY_CACHES];
  const int2* copies;
  int32_t* status;
  uint32_t n_copies, n_blocks, heads, block_bytes, chunks, per_copy, step;      // per_copy: pieces of a copy, in all caches
};

__global__ __launch_bounds__(COPY_THREADS) void k_cache_copy(CopyArgs a) {
  const bool stop = stopped(a.status);
  const uint32_t rest = blockIdx.x % a.per_copy, side = rest / a.chunks, chunk = rest % a.chunks, lane = lane_id();
  const auto& cache = a.caches[side / 2];
  uint8_t* codes = side % 2 ? cache.v : cache.k;
  uint8_t* exps = side % 2 ? cache.v_exp : cache.k_exp;
  const uint32_t begin = chunk * COPY_CHUNK + threadIdx.x * 16;
  for (uint64_t first = blockIdx.x / a.per_copy; first < a.n_copies; first += static_cast<uint64_t>(WAVE) * a.step) {
    const uint64_t mine = first + static_cast<uint64_t>(lane) * a.step;
    const int2 copy = mine < a.n_copies ? a.copies[mine] : make_int2(-1, -1);
    if (stop) return;
    const bool used = (copy.x & copy.y) != -1;
    const bool bad = used && (static_cast<uint32_t>(copy.x) >= a.n_blocks || static_cast<uint32_t>(copy.y) >= a.n_blocks);
    if (bad) *a.status = FIKIT_INVALID_ARG;
    for (uint64_t left = ballot(used && !bad && copy.x != copy.y); left; left &= left - 1) {
      const uint32_t which = static_cast<uint32_t>(__builtin_ctzll(left));
      const uint64_t from = read_lane_u32(static_cast<uint32_t>(copy.x), which), to = read_lane_u32(static_cast<uint32_t>(copy.y), which);
      const uint8_t* x = codes + from * a.block_bytes;
      uint8_t* y = codes + to * a.block_bytes;
      u32x4 held[COPY_LOADS];
#pragma unroll
      for (int i = 0; i < COPY_LOADS; ++i)
        if (begin + i * COPY_THREADS * 16 < a.block_bytes) held[i] = *reinterpret_cast<const u32x4*>(x + begin + i * COPY_THREADS * 16);
#pragma unroll
      for (int i = 0; i < COPY_LOADS; ++i)
        if (begin + i * COPY_THREADS * 16 < a.block_bytes) __builtin_nontemporal_store(held[i], reinterpret_cast<u32x4*>(y + begin + i * COPY_THREADS * 16));
      if (chunk == 0)
        for (uint32_t h = threadIdx.x; h < a.heads; h += COPY_THREADS) exps[to * a.heads + h] = exps[from * a.heads + h];
    }
  }
}

}  // namespace fikit
