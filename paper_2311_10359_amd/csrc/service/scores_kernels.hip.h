// What rows of logits say about tokens: log probabilities, entropy, alternatives.
#pragma once

#include "serve_common.hip.h"

namespace fikit {

// A row x of V logits and a scale s.  In units of log 2, with c = s log2(e), m the largest logit and d = c (x - m):
//
//   S = sum 2^d,  T = sum 2^d d      log(sum exp(s x)) = s m + ln 2 log2 S      entropy = ln 2 (log2 S - T / S)
//   log probability of a token = ln 2 (d - log2 S)
//
// in one pass: every lane keeps m, S and T of what it has seen, and moves the sums to another m where a larger logit comes.  d of the largest is 0 whatever
// its size, so that one token that holds all has entropy and log probability 0, and the type's lowest value, a mask in many programs, is a number as others.
// (c x - c m in one instruction would leave the rounding of c m in d, and the pass is no faster with it.)
//
// The k alternatives lie in k groups of neighbouring logits (16 bytes, as one load brings them): those with the largest maxima, among equal ones
// the first, since of any other group k groups before it in this order hold a value that comes before all of its own.  So the pass looks
// at one maximum for a group, and at the end the k groups are read again and k of their values taken.  A wave takes groups in ascending order,
// so a later group that is only as large as the k-th so far is none of them, and few pass: about k (1 + log(groups / k)).
//
// V * bytes are read: bound by memory, if a logit takes few instructions: one to unpack, one for maximum and minimum, four for d, S and T, and the
// exponential.  2999 rows of 100,003 bfloat16 logits, 600 MB: 98 us without alternatives, 6.1 TB/s, 108 to 113 with 20, the vector unit busy for 84 % of
// it.  A workgroup's waves take batches in turn, past the caches (without alternatives 100 us when that was tried, a stretch for each wave 113, through the caches 111), and
// 4 groups a lane in a batch (8 are 6 us more: half the waves).

struct ScoresArgs {
  const void* logits;
  uint64_t row_stride;
  const int32_t* tokens;
  float* logprob;
  float* entropy;
  float* lse;
  int32_t* top_tokens;
  float* top_logprob;
  int32_t* status;
  float4* sums;             // workspace: [rows][parts] m, S, T and the border
  float2* lists;            // [rows][parts][SCORES_MOST] maxima and groups, minus infinity where there is none
  uint32_t rows, vocabulary, n_top, parts, per_part;      // per_part: groups
  float scale, c;           // c = scale log2(e)
};

constexpr int SCORES_BATCH = 4, SCORES_MOST = 32, SCORES_ROOM = 128, JOIN_WAVES = 4, JOIN_ROOM = 512;
constexpr float LOWEST = -3.4028234663852886e38f;       // m where nothing has been seen

struct LogitsBf16 {
  typedef uint16_t raw;
  static constexpr int VEC = 8, KEY_BITS = 16;            // KEY_BITS: what differs between values
  static __device__ __forceinline__ float value(raw v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
  static __device__ __forceinline__ void unpack(const u32x4& w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = Bf16::low(w[i]); x[2 * i + 1] = Bf16::high(w[i]); }
  }
  static constexpr uint32_t NOTHING = 0xff80ff80u;        // minus infinity
};
struct LogitsF16 {
  typedef uint16_t raw;
  static constexpr int VEC = 8, KEY_BITS = 19;
  static __device__ __forceinline__ float value(raw v) { return static_cast<float>(bits_as<_Float16>(v)); }
  static __device__ __forceinline__ void unpack(const u32x4& w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = F16::low(w[i]); x[2 * i + 1] = F16::high(w[i]); }
  }
  static constexpr uint32_t NOTHING = 0xfc00fc00u;
};
struct LogitsF32 {
  typedef float raw;
  static constexpr int VEC = 4, KEY_BITS = 32;
  static __device__ __forceinline__ float value(raw v) { return v; }
  static __device__ __forceinline__ void unpack(const u32x4& w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  static constexpr uint32_t NOTHING = 0xff800000u;
};

// Whole numbers in the order of the values; zeros of both signs are equal.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t bits = __float_as_uint(v + 0.f);
  return bits >> 31 ? ~bits : bits | 0x80000000u;
}
constexpr uint32_t LOWEST_KEY = 0x00800000u;             // of the lowest finite value
__device__ __forceinline__ float value_of_key(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); }

// A key that k of the wave's keys reach (N to a lane; 0: none) and no more, or the largest one that k or more reach, if some are equal.  More than k
// keys are given, of which the upper BITS differ; the k-th largest is `least` or more.  (Two bits at a time from the first one in which `least` and
// the largest key differ: a step is one trip from the comparisons to the counts and back, however many comparisons it makes.)
template <int BITS, int N>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&keys)[N], uint32_t k, uint32_t least) {
  uint32_t most = keys[0];
#pragma unroll
  for (int i = 1; i < N; ++i) most = max_u32(most, keys[i]);
  most = max_over_wave(most);
  const int from = (31 - __builtin_clz((most ^ least) | 1)) | 1;             // bits 2 i + 1 and 2 i
  uint32_t found = most >> from >> 1 << from << 1;
#pragma unroll 1
  for (int b = from - 1; b >= (32 - BITS) / 2 * 2; b -= 2) {
    uint32_t n[3] = {};
#pragma unroll
    for (uint32_t j = 0; j < 3; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) n[j] += popc64(ballot(keys[i] >= (found | (j + 1) << b)));
    const uint32_t passed = n[2] >= k ? 3 : n[1] >= k ? 2 : n[0] >= k ? 1 : 0;
    const uint32_t reached = n[2] >= k ? n[2] : n[1] >= k ? n[1] : n[0];
    found |= passed << b;
    if (reached == k) break;
  }
  return found;
}

// Which of the keys are the first k: the larger ones, and of those equal to the k-th largest the ones of the lowest `order`, which is different for
// each.  Their places in turn.  Returns a key that all of them reach; of those equal to it none of an order of `limit` or more is one of the k.
template <int BITS, int N>
__device__ __forceinline__ uint32_t first_of(const uint32_t (&keys)[N], const uint32_t (&order)[N], uint32_t k, uint32_t least, bool (&keep)[N],
                                             uint32_t (&place)[N], uint32_t* limit) {
  const uint32_t border = reached_by<BITS, N>(keys, k, least);
  uint32_t reached = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    keep[i] = keys[i] >= border;
    reached += popc64(ballot(keep[i]));
  }
  *limit = ~0u;
  if (reached > k) {                           // some are equal to the k-th
    const uint32_t largest_equal = border | (BITS < 32 ? (1u << (32 - BITS) % 32) - 1 : 0);
    if (reached > k + 16) {                    // many: the order of those that stay, from the largest ~order on
      uint32_t equal[N], larger = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        equal[i] = keep[i] && keys[i] <= largest_equal ? ~order[i] : 0;
        larger += popc64(ballot(keys[i] > largest_equal));
      }
      const uint32_t last = reached_by<32, N>(equal, k - larger, 0);
#pragma unroll
      for (int i = 0; i < N; ++i) keep[i] = keep[i] && (keys[i] > largest_equal || ~order[i] >= last);
      reached = k;
      *limit = ~last;
    }
#pragma unroll 1
    for (; reached > k; --reached) {           // few: one after the other, of the highest order first, goes
      uint32_t last = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) last = max_u32(last, keep[i] && keys[i] <= largest_equal ? order[i] + 1 : 0);
      last = max_over_wave(last);
      *limit = last - 1;
#pragma unroll
      for (int i = 0; i < N; ++i) keep[i] = keep[i] && (keys[i] > largest_equal || order[i] + 1 != last);
    }
  }
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint64_t kept = ballot(keep[i]);
    place[i] = n + popc_below(kept);
    n += popc64(kept);
  }
  return border;
}

struct ScoresLds {          // of a wave: its groups
  float most[SCORES_ROOM];
  uint32_t group[SCORES_ROOM];
};

__device__ __forceinline__ void lds_in_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// m, S and T of some logits.
struct Sums {
  float m = LOWEST, s = 0, t = 0;

  // The same relative to another m that is no smaller; far below it nothing is left.
  __device__ __forceinline__ void move_to(float next, float c) {
    const float move = (m - next) * c, f = exp2_fast(move);
    t = f == 0.f ? 0.f : (t + move * s) * f;
    s *= f;
    m = next;
  }
  __device__ __forceinline__ void add(Sums other, float c) {
    const float next = fmaxf(m, other.m);
    move_to(next, c);
    other.move_to(next, c);
    s += other.s;
    t += other.t;
  }
};

__device__ __forceinline__ float sum_over_wave(float v) {
  const auto from = [](float x, auto dpp) { return __uint_as_float(dpp(__float_as_uint(x))); };
  v += from(v, dpp_or_zero<0x111, 0xf>);
  v += from(v, dpp_or_zero<0x112, 0xf>);
  v += from(v, dpp_or_zero<0x114, 0xf>);
  v += from(v, dpp_or_zero<0x118, 0xf>);
  v += from(v, dpp_or_zero<0x142, 0xa>);
  v += from(v, dpp_or_zero<0x143, 0xc>);
  return __uint_as_float(read_lane_u32(__float_as_uint(v), WAVE - 1));
}

// What a wave has seen of a row.
template <typename L>
struct Seen {
  Sums sums;                               // of each lane
  uint32_t n = 0, k;                       // groups in the list; how many are wanted
  float border;                            // only groups that reach it are; none reaches NaN
  uint32_t limit = ~0u;                    // ... and if they are only as large, come before this

  __device__ __forceinline__ explicit Seen(uint32_t n_top) : k(n_top), border(n_top ? -INFINITY : NAN) {}

  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], float most, float least, float c) {
    sums.move_to(fmaxf(sums.m, most), c);
    float s = 0, t = 0;
    if (ballot((least - sums.m) * c == -INFINITY)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = (x[i] - sums.m) * c, e = exp2_fast(d);
        s += e;
        t = __builtin_fmaf(e, d == -INFINITY ? 0.f : d, t);       // (nothing times minus infinity)
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = (x[i] - sums.m) * c, e = exp2_fast(d);
        s += e;
        t = __builtin_fmaf(e, d, t);
      }
    }
    sums.s += s;
    sums.t += t;
  }

  __device__ __forceinline__ bool may_be(float most, uint32_t group) const { return most > border || (most == border && group < limit); }

  // Groups, one to a lane, of which some join the list.  (It has room for 64 more.)
  __device__ __forceinline__ void append(bool hit, float most, uint32_t group, ScoresLds* lds) {
    const uint64_t hits = ballot(hit);
    if (!hits) return;
    if (hit) {
      const uint32_t at = n + popc_below(hits);
      lds->most[at] = most;
      lds->group[at] = group;
    }
    n += popc64(hits);
    lds_in_order();
  }

  // Takes from a list of up to JOIN_ROOM in LDS what can be of the first k, and no more than `room`.  (In loops, as elsewhere here: code that a wave
  // runs once costs it more to fetch than to run.)
  __device__ __forceinline__ void take(const float2* from, uint32_t count, bool look, uint32_t room, ScoresLds* lds) {
    constexpr uint32_t N = JOIN_ROOM / WAVE;
    const uint32_t lane = lane_id();
    float of[N], all = -INFINITY;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) {
      of[i] = i * WAVE + lane < count ? from[i * WAVE + lane].x : -INFINITY;
      all = fmaxf(all, of[i]);
    }
    if (look) begin(all);
    uint32_t hits = 0;
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) hits |= of[i] >= border && of[i] > -INFINITY ? 1u << i : 0;
#pragma unroll 1
    while (ballot(hits)) {
      const float2 one = hits ? from[(__ffs(static_cast<int>(hits)) - 1) * WAVE + lane] : make_float2(-INFINITY, 0.f);
      append(hits && may_be(one.x, __float_as_uint(one.y)), one.x, __float_as_uint(one.y), lds);
      hits &= hits - 1;
      if (n > WAVE) shorten(lds);
    }
    if (n > room) shorten(lds);
  }

  // The first k stay, of more.  (n is up to SCORES_ROOM)
  __device__ __forceinline__ void shorten(ScoresLds* lds) {
    constexpr int N = SCORES_ROOM / WAVE;
    const uint32_t lane = lane_id();
    uint32_t keys[N], groups[N], place[N];
    bool keep[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool there = lane + i * WAVE < n;
      keys[i] = there ? key_of(lds->most[lane + i * WAVE]) : 0;
      groups[i] = lds->group[lane + i * WAVE];
    }
    lds_in_order();
    const uint32_t reached = first_of<L::KEY_BITS, N>(keys, groups, k, key_of(border), keep, place, &limit);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (keep[i]) {
        lds->most[place[i]] = value_of_key(keys[i]);
        lds->group[place[i]] = groups[i];
      }
    lds_in_order();
    n = k;
    // (of negative values the bits that do not differ are ones)
    constexpr uint32_t LOW = L::KEY_BITS < 32 ? (1u << (32 - L::KEY_BITS) % 32) - 1 : 0;
    border = value_of_key(reached >> 31 ? reached : max_u32(reached | LOW, LOWEST_KEY));
  }

  // The k-th largest of the lanes' maxima is a border for what they have, of which not much more than k is left then.
  __device__ __forceinline__ void begin(float most) {
    const uint32_t keys[1] = {most > -INFINITY ? key_of(most) : 0};
    if (popc64(ballot(keys[0] != 0)) <= k) return;
    const uint32_t least = ~max_over_wave(keys[0] ? ~keys[0] : 0);
    const uint32_t reached = reached_by<L::KEY_BITS, 1>(keys, k, least);
    if (reached <= LOWEST_KEY) return;
    const float below = value_of_key(reached - (reached == 0x80000000u ? 2 : 1));         // (there is no key of -0)
    if (below > border) {
      border = below;
      limit = ~0u;
    }
  }

  // Lists of others: k groups of each reach its border.
  __device__ __forceinline__ void begin_at(float theirs) {
    if (k > 0) border = value_of_key(max_over_wave(key_of(theirs)));
  }

  // The lanes' sums become one, in all lanes.
  __device__ __forceinline__ void sum_over_lanes(float c) {
    sums.move_to(value_of_key(max_over_wave(key_of(sums.m))), c);
    sums.s = sum_over_wave(sums.s);
    sums.t = sum_over_wave(sums.t);
  }
};

// A row: `head` logits in front of the first 16-byte border, whole groups, and the rest.  Group 0 is the head, 1 .. whole the groups, then the rest.
template <typename L>
struct Row {
  const typename L::raw* x;
  uint32_t head, whole, vocabulary;
  __device__ __forceinline__ Row(const ScoresArgs& a, uint32_t row) {
    x = static_cast<const typename L::raw*>(a.logits) + row * a.row_stride;
    vocabulary = a.vocabulary;
    const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(x) % 16) / sizeof(typename L::raw);
    head = min_u32(off ? L::VEC - off : 0, vocabulary);
    whole = (vocabulary - head) / L::VEC;
  }
  __device__ __forceinline__ uint32_t rest() const { return vocabulary - head - whole * L::VEC; }
  // the i-th logit of a group, and whether there is one
  __device__ __forceinline__ bool place(uint32_t group, uint32_t i, uint32_t* at) const {
    *at = group == 0 ? i : head + (group - 1) * L::VEC + i;
    return group == 0 ? i < head : *at < vocabulary;
  }
};

// A row's given token; its logit is asked for early.
struct Given {
  int32_t token;
  float x;
};
template <typename L>
__device__ __forceinline__ float given_logit(const ScoresArgs& a, const Row<L>& row, int32_t token) {
  return token >= 0 && static_cast<uint32_t>(token) < a.vocabulary ? L::value(row.x[token]) : 0.f;
}

// The first k groups of the `count` in `from`, and, if this is all of the row, its outputs, by one wave that knows its sums.  `from` has room for the
// groups' logits.
template <typename L>
__device__ __forceinline__ void finish_row(const ScoresArgs& a, const Row<L>& row, uint32_t r, const Given& given, Seen<L>& seen, float2* from, uint32_t count,
                                           bool all, ScoresLds* lds) {
  const uint32_t lane = lane_id(), k = a.n_top;
  const Sums& sums = seen.sums;
  const bool nothing = sums.s == 0.f, odd = sums.s != sums.s;
  const float log_s = __builtin_amdgcn_logf(sums.s), lse = __builtin_fmaf(a.scale, sums.m, LN2 * log_s);
  auto logprob = [&](float v) {
    if (nothing || v == -INFINITY) return -INFINITY;
    const float d = (v - sums.m) * a.c;
    return d > -0x1p22f ? fminf(LN2 * (d - log_s), 0.f) : v * a.scale - lse;
  };
  if (lane == 0 && all) {
    if (given.token >= 0 && static_cast<uint32_t>(given.token) >= a.vocabulary) *a.status = FIKIT_INVALID_ARG;
    if (a.logprob) a.logprob[r] = given.token < 0 ? 0.f : odd ? NAN : logprob(given.x);
    if (a.lse) a.lse[r] = nothing ? -INFINITY : odd ? NAN : lse;
    if (a.entropy) a.entropy[r] = nothing ? 0.f : odd ? NAN : fmaxf(LN2 * (log_s - sums.t / sums.s), 0.f);
  }
  if (k == 0) return;
#pragma unroll 1
  for (bool logits = false;; logits = true) {
    seen.take(from, count, !logits, logits ? WAVE : SCORES_MOST, lds);
    if (logits || !all) break;
    // the groups' logits, of which those that reach the groups' border can be of the k
    constexpr int N = SCORES_MOST * L::VEC / WAVE;
    float x[N];
    uint32_t at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t e = lane + i * WAVE;
      x[i] = -INFINITY;
      at[i] = 0;
      if (e / L::VEC < seen.n && row.place(lds->group[e / L::VEC], e % L::VEC, &at[i])) x[i] = L::value(row.x[at[i]]);
    }
    count = seen.n * L::VEC;
#pragma unroll
    for (int i = 0; i < N; ++i) from[lane + i * WAVE] = make_float2(x[i], __uint_as_float(at[i]));
    seen.n = 0;
    seen.limit = ~0u;                          // (of groups)
    lds_in_order();
  }
  const uint32_t n = seen.n;
  const float mine = lane < n ? lds->most[lane] : -INFINITY;
  const uint32_t which = lane < n ? lds->group[lane] : 0;
  if (!all) {
    if (lane < SCORES_MOST) a.lists[static_cast<uint64_t>(blockIdx.x) * SCORES_MOST + lane] = make_float2(mine, __uint_as_float(which));
    return;
  }
  uint32_t rank = 0;                           // of up to 64
  for (uint32_t i = 0; i < n; ++i) {
    const float other = __uint_as_float(read_lane_u32(__float_as_uint(mine), i));
    rank += other > mine || (other == mine && read_lane_u32(which, i) < which);
  }
  const uint64_t out = static_cast<uint64_t>(r) * k;
  if (lane < k && (lane >= n || odd)) {
    a.top_tokens[out + lane] = -1;
    a.top_logprob[out + lane] = odd ? NAN : -INFINITY;
  }
  if (lane >= n || rank >= k || odd) return;
  a.top_tokens[out + rank] = static_cast<int32_t>(which);
  a.top_logprob[out + rank] = logprob(mine);
}

// A workgroup of W waves takes a part of a row, a batch of each wave's behind the other's.
template <typename L, int W>
__global__ __launch_bounds__(W * WAVE) void k_scores(ScoresArgs a) {
  __shared__ ScoresLds lists[W];
  __shared__ float2 firsts[JOIN_ROOM];
  __shared__ float4 sums[W];
  static_assert(W * SCORES_MOST <= JOIN_ROOM && SCORES_MOST * L::VEC <= JOIN_ROOM, "room for the waves' lists, and for their groups' logits");
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE), r = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  const Row<L> row(a, r);
  ScoresLds* lds = &lists[wave];
  Seen<L> seen(a.n_top);
  Given given{a.tokens ? a.tokens[r] : -1, 0.f};
  const uint32_t begin = part * a.per_part, end = row.whole - begin < a.per_part ? row.whole : begin + a.per_part;       // (parts begin within the row)
  const u32x4* groups = reinterpret_cast<const u32x4*>(row.x + row.head);
#pragma unroll 1
  for (uint64_t from = begin + wave * SCORES_BATCH * WAVE; from < end; from += W * SCORES_BATCH * WAVE) {
    u32x4 w[SCORES_BATCH];
    const uint32_t mine = static_cast<uint32_t>(from) + lane;
#pragma unroll
    for (int i = 0; i < SCORES_BATCH; ++i) {
      w[i] = u32x4{L::NOTHING, L::NOTHING, L::NOTHING, L::NOTHING};
      if (mine + i * WAVE < end) w[i] = __builtin_nontemporal_load(groups + mine + i * WAVE);
    }
    float x[SCORES_BATCH * L::VEC], most[SCORES_BATCH], all = -INFINITY, least = INFINITY;
#pragma unroll
    for (int i = 0; i < SCORES_BATCH; ++i) {
      L::unpack(w[i], x + i * L::VEC);
      most[i] = -INFINITY;
#pragma unroll
      for (int j = 0; j < L::VEC; j += 2) {
        most[i] = fmaxf(fmaxf(most[i], x[i * L::VEC + j]), x[i * L::VEC + j + 1]);
        least = fminf(fminf(least, x[i * L::VEC + j]), x[i * L::VEC + j + 1]);
      }
      all = fmaxf(all, most[i]);
    }
    seen.add(x, all, least, a.c);
    if (seen.border == -INFINITY) seen.begin(all);
    if (!ballot(all > seen.border)) continue;
    // (Groups before these are all that the list holds: one that is only as large as the k-th is none of the k.)
    uint32_t hits = 0;
#pragma unroll
    for (uint32_t i = 0; i < SCORES_BATCH; ++i) hits |= most[i] > seen.border ? 1u << i : 0;
#pragma unroll 1
    while (ballot(hits)) {                       // a lane's first one, and mostly its only one
      const uint32_t i = __ffs(static_cast<int>(hits)) - 1;
      float of = most[0];
#pragma unroll
      for (uint32_t j = 1; j < SCORES_BATCH; ++j) of = i == j ? most[j] : of;
      seen.append(hits && seen.may_be(of, 1 + mine + i * WAVE), of, 1 + mine + i * WAVE, lds);
      hits &= hits - 1;
      if (seen.n > WAVE) seen.shorten(lds);
    }
  }
  const bool stop = stopped(a.status);         // (nothing is written before; asked for at the start it costs 0.5 us, and registers if not waited for)
  if (wave == 0) given.x = given_logit(a, row, given.token);
  if (wave == W - 1 && (part == 0 || part == a.parts - 1)) {
    // what is less than a group, a logit to a lane: the head in the first eight lanes, the rest in the next
    const uint32_t i = lane % 8;
    const bool head = lane < 8 && part == 0 && i < row.head, rest = lane >= 8 && lane < 16 && part == a.parts - 1 && i < row.rest();
    const float x[1] = {head || rest ? L::value(row.x[head ? i : row.vocabulary - row.rest() + i]) : -INFINITY};
    seen.add(x, x[0], x[0], a.c);
    uint32_t most = key_of(x[0]);
    most = max_u32(most, dpp_move<0xB1>(most));
    most = max_u32(most, dpp_move<0x4E>(most));
    most = max_u32(most, dpp_move<0x141>(most));
    const float of = value_of_key(most);
    const uint32_t group = lane < 8 ? 0 : row.whole + 1;
    seen.append(i == 0 && seen.may_be(of, group) && of > -INFINITY, of, group, lds);
  }
  if (seen.n > SCORES_MOST) seen.shorten(lds);
  seen.sum_over_lanes(a.c);
  if (lane == 0) sums[wave] = make_float4(seen.sums.m, seen.sums.s, seen.sums.t, seen.border);
  if (lane < SCORES_MOST) firsts[wave * SCORES_MOST + lane] = lane < seen.n ? make_float2(lds->most[lane], __uint_as_float(lds->group[lane])) : make_float2(-INFINITY, 0.f);
  if (__syncthreads_or(stop) || wave > 0) return;
  // the first wave joins the sums and the lists
  Seen<L> joined(a.n_top);
  const float4 of_wave = lane < W ? sums[lane] : make_float4(LOWEST, 0.f, 0.f, -INFINITY);
  joined.sums = Sums{of_wave.x, of_wave.y, of_wave.z};
  joined.sum_over_lanes(a.c);
  joined.begin_at(of_wave.w);
  if (a.parts > 1 && lane == 0) a.sums[blockIdx.x] = make_float4(joined.sums.m, joined.sums.s, joined.sums.t, joined.border);
  finish_row<L>(a, row, r, given, joined, firsts, W * SCORES_MOST, a.parts == 1, lds);
}

// Joins a row's parts: a wave each.
template <typename L>
__global__ __launch_bounds__(JOIN_WAVES * WAVE) void k_scores_join(ScoresArgs a) {
  __shared__ ScoresLds lists[JOIN_WAVES];
  __shared__ float2 firsts[JOIN_WAVES][JOIN_ROOM];
  const uint32_t lane = lane_id(), wave = uniform(threadIdx.x / WAVE), r = blockIdx.x * JOIN_WAVES + wave;
  if (r >= a.rows) return;
  const bool stop = stopped(a.status);
  const uint64_t first = static_cast<uint64_t>(r) * a.parts;
  const uint32_t n = a.n_top ? a.parts * SCORES_MOST : 0;
  const float2* entries = a.lists + first * SCORES_MOST;
  constexpr uint32_t AHEAD = JOIN_ROOM / WAVE;  // loads that wait for nothing
  float2 of[AHEAD];
#pragma unroll
  for (uint32_t i = 0; i < AHEAD; ++i) of[i] = i * WAVE + lane < n ? entries[i * WAVE + lane] : make_float2(-INFINITY, 0.f);
  Given given{a.tokens ? a.tokens[r] : -1, 0.f};
  Seen<L> seen(a.n_top);
  float border = -INFINITY;
  for (uint32_t p = lane; p < a.parts; p += WAVE) {
    const float4 theirs = a.sums[first + p];
    seen.sums.add(Sums{theirs.x, theirs.y, theirs.z}, a.c);
    border = fmaxf(border, theirs.w);
  }
  if (stop) return;
  const Row<L> row(a, r);
  given.x = given_logit(a, row, given.token);
  seen.sum_over_lanes(a.c);
  seen.begin_at(border);
  ScoresLds* lds = &lists[wave];
#pragma unroll
  for (uint32_t i = 0; i < AHEAD; ++i) firsts[wave][i * WAVE + lane] = of[i];
  uint32_t at = 0, count = min_u32(n, JOIN_ROOM);
  lds_in_order();
  while (at + count < n) {                     // more lists than there is room for: those so far become one, which stays
    seen.take(firsts[wave], count, true, SCORES_MOST, lds);
    at += count;
    count = min_u32(n - at, JOIN_ROOM);
    for (uint32_t e = lane; e < count; e += WAVE) firsts[wave][e] = entries[at + e];
    lds_in_order();
  }
  finish_row<L>(a, row, r, given, seen, firsts[wave], count, true, lds);
}

}  // namespace fikit
