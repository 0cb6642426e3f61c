// Eviction from a paged cache: which tokens stay under a budget (pkv_cache_keep)
// and their rows moved to the front of their sequence (pkv_cache_evict).
//
// The choice reads little and is bound by its steps, one behind the other: a workgroup a row takes 21 us for 32 rows of up to
// 16384 tokens (of which the instructions of its four passes over the keys are some 7), four launches take 28 us for 16 rows
// of up to 131072.  Moving rows is bound by memory: 32 ragged sequences cut to 2048 tokens of 4 bits, 8 heads of 128,
// 104 MB, 39 us (2.7 TB/s; every workgroup reads before it writes, and they all begin together), 85547 tokens of 16-bit rows
// cut to 14000, 137 MB, 38 us (3.6 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pkv.h"
#include "pkv_internal.h"
#include "serve.h"

namespace pkv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---- Which tokens stay ----
//
// The weights' bits as whole numbers in their order (keys).  The key of the last token kept is found by its digits from the top:
// how many tokens have each value of the first 11 bits; the ones that share the last one's are copied to LDS, and their next
// bits are counted there (all tokens again, where they are too many).  Then the tokens above it and the first ones
// equal to it are written in order.  A workgroup takes one row of weights, each wave a run of it, whose keys it keeps
// in registers as far as they go.

constexpr int kKeepThreads = 1024;
constexpr int kKeepWaves = kKeepThreads / 64;
constexpr int kDigits = 2048;       // of 11 bits
constexpr int kCopies = 4;          // of their counts, so that lanes seldom meet in one
constexpr int kListed = 20480;      // keys in LDS
constexpr int kHeldKeys = 32;       // a lane's keys in registers
constexpr int kLoadsAhead = 8;      // of the others, a lane's on their way at once

// Larger weights have larger keys; +0 and -0 are one, NaN is below everything.
__device__ __forceinline__ uint32_t key_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  if (w != w) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Lanes of a mask before this one.
__device__ __forceinline__ int32_t before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

struct KeepShared {
  uint32_t count[kDigits * kCopies];
  uint32_t list[kListed];
  uint32_t sums[kKeepWaves];
  int32_t above[kKeepWaves], equal[kKeepWaves];
  uint32_t digit, left, among, listed;
};

// Adds a lane's digit to the counts, all lanes of a wave at once where they agree.
__device__ __forceinline__ void count_digit(KeepShared& lds, bool on, uint32_t digit, int lane) {
  if (!on) return;
  const uint64_t who = __ballot(1);
  if (__ballot(digit == uint32_t(__builtin_amdgcn_readfirstlane(int(digit)))) == who) {
    if (before(who) == 0) atomicAdd(&lds.count[digit * kCopies], uint32_t(__builtin_popcountll(who)));
  } else {
    atomicAdd(&lds.count[digit * kCopies + (lane & (kCopies - 1))], 1u);
  }
}

// The digit of the `need`-th largest key among those counted: lds.digit; lds.left of them are to be kept among the lds.among
// that have it.  The counts are cleared for the next digit.
__device__ __forceinline__ void take_counts(KeepShared& lds, uint32_t (&mine)[2]) {
  static_assert(kDigits == 2 * kKeepThreads && kCopies == 4, "two digits to a thread");
#pragma unroll
  for (int d = 0; d < 2; ++d) {  // digits from the top
    u32x4& c = *reinterpret_cast<u32x4*>(&lds.count[(kDigits - 1 - 2 * int(threadIdx.x) - d) * kCopies]);
    mine[d] = c[0] + c[1] + c[2] + c[3];
    c = u32x4{};
  }
}
__device__ __forceinline__ void find_digit(KeepShared& lds, const uint32_t (&mine)[2], uint32_t need) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t upto = mine[0] + mine[1];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t other = __shfl_up(upto, off);
    upto += lane >= off ? other : 0;
  }
  if (lane == 63) lds.sums[wave] = upto;
  __syncthreads();
  uint32_t upper = upto - mine[0] - mine[1];  // keys of larger digits
#pragma unroll
  for (int i = 0; i < kKeepWaves; ++i) upper += i < wave ? lds.sums[i] : 0;  // (all read at once)
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    if (upper < need && need <= upper + mine[d]) {
      lds.digit = uint32_t(kDigits - 1 - 2 * tid - d);
      lds.left = need - upper;
      lds.among = mine[d];
    }
    upper += mine[d];
  }
  __syncthreads();
}

// One row of weights and what is to be chosen of it.
struct Choice {
  const float* w;      // of the tokens between the first and the last ones,
  int32_t middle;      // so many,
  uint32_t need;       // of which so many stay
  int32_t n, m, first, last;
  int32_t* kept;
  bool choose;
};
__device__ __forceinline__ Choice choice_of(const ServeArgs& s, const KeepArgs& a, int32_t row) {
  const int32_t seq = int32_t(uint32_t(row) / uint32_t(a.heads)), head = int32_t(uint32_t(row) % uint32_t(a.heads));
  Choice c;
  c.n = kept_len(s, s.kv_lens[seq]);
  c.m = kept_budget(a, c.n, a.budgets ? a.budgets[seq] : a.budget);
  c.first = a.sinks < c.m ? a.sinks : c.m;
  c.last = a.recent < c.m - c.first ? a.recent : c.m - c.first;
  c.middle = c.n - c.first - c.last;
  c.need = uint32_t(c.m - c.first - c.last);
  c.kept = a.kept + int64_t(row) * a.budget;
  c.w = a.weights + int64_t(seq) * a.seq_stride + int64_t(head) * a.head_stride + c.first;
  c.choose = c.need != 0 && c.need != uint32_t(c.middle);
  if (head == 0 && threadIdx.x == 0) a.kept_lens[seq] = c.m;
  return c;
}
// What of a row is known without its weights.
__device__ __forceinline__ void keep_ends(const KeepArgs& a, const Choice& c) {
  const int tid = threadIdx.x;
  for (int32_t j = tid; j < c.first; j += kKeepThreads) c.kept[j] = j;
  for (int32_t j = tid; j < c.last; j += kKeepThreads) c.kept[c.m - c.last + j] = c.n - c.last + j;
  for (int32_t j = c.m + tid; j < a.budget; j += kKeepThreads) c.kept[j] = -1;
  if (!c.choose && c.need)
    for (int32_t j = tid; j < c.middle; j += kKeepThreads) c.kept[c.first + j] = c.first + j;
}

// Writes a wave's tokens that stay: those of larger keys than `found` and the first `most` equal to it, after `higher` and
// `ties` of such tokens before the wave's.
template <typename Each>
__device__ __forceinline__ void keep_in_order(const Choice& c, uint32_t found, int32_t most, int32_t higher, int32_t ties,
                                              Each each) {
  each([&](int32_t at, bool is, uint32_t key) {
    const uint64_t gt = __ballot(is && key > found), eq = __ballot(is && key == found);
    const int32_t tie = ties + before(eq);
    const int32_t place = higher + before(gt) + (tie < most ? tie : most);
    if (is && (key > found || (key == found && tie < most))) c.kept[c.first + place] = c.first + at;
    higher += __builtin_popcountll(gt);
    ties += __builtin_popcountll(eq);
  });
}

__global__ __launch_bounds__(kKeepThreads) void keep_kernel(ServeArgs s, KeepArgs a) {
  __shared__ KeepShared lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Choice c = choice_of(s, a, int32_t(blockIdx.x));
  const int32_t first = c.first, middle = c.middle;
  const bool choose = c.choose;
  uint32_t need = c.need;
  const float* w = c.w;
  int32_t* kept = c.kept;

  // The wave's run of the middle.
  const int32_t run = ((middle + kKeepThreads - 1) / kKeepThreads) * 64;
  const int32_t from = wave * run < middle ? wave * run : middle, upto = from + run < middle ? from + run : middle;
  uint32_t held[kHeldKeys];
  if (choose) {
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) {
      const int32_t at = from + 64 * i + lane;
      held[i] = at < upto ? __float_as_uint(w[at]) : 0;
    }
  }
  keep_ends(a, c);
  if (!choose) return;
  for (int i = tid; i < kDigits * kCopies; i += kKeepThreads) lds.count[i] = 0;
  if (tid == 0) lds.listed = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kHeldKeys; ++i) held[i] = key_of(__uint_as_float(held[i]));

  // f(place in the middle, whether there is such a token, its key) for the wave's run in order, all lanes at once.
  auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i)
      if (from + 64 * i < upto) f(from + 64 * i + lane, from + 64 * i + lane < upto, held[i]);
    for (int32_t i = from + 64 * kHeldKeys; i < upto; i += 64 * kLoadsAhead) {
      float v[kLoadsAhead];
#pragma unroll
      for (int e = 0; e < kLoadsAhead; ++e) v[e] = i + 64 * e + lane < upto ? w[i + 64 * e + lane] : 0.0f;
#pragma unroll
      for (int e = 0; e < kLoadsAhead; ++e)
        if (i + 64 * e < upto) f(i + 64 * e + lane, i + 64 * e + lane < upto, key_of(v[e]));
    }
  };

  each([&](int32_t, bool is, uint32_t key) { count_digit(lds, is, key >> 21, lane); });
  __syncthreads();
  uint32_t mine[2];
  take_counts(lds, mine);
  find_digit(lds, mine, need);
  uint32_t found = lds.digit;  // the digits found so far
  need = lds.left;
  const uint32_t among = lds.among;
  const bool few = among <= kListed;
  if (few) {
    each([&](int32_t, bool is, uint32_t key) {
      const bool on = is && key >> 21 == found;
      const uint64_t who = __ballot(on);
      if (!who) return;
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&lds.listed, uint32_t(__builtin_popcountll(who)));
      at = uint32_t(__shfl(int(at), 0));
      if (on) lds.list[at + before(who)] = key;
    });
    __syncthreads();
  }
  constexpr int kAt[2] = {10, 0}, kBits[2] = {11, 10};
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const int shift = kAt[d], bits = kBits[d];
    const uint32_t mask = (1u << bits) - 1;
    if (few) {
      for (uint32_t i = tid - lane; i < among; i += kKeepThreads) {
        const bool is = i + lane < among;
        const uint32_t key = is ? lds.list[i + lane] : 0;
        count_digit(lds, is && key >> (shift + bits) == found, key >> shift & mask, lane);
      }
    } else {
      each([&](int32_t, bool is, uint32_t key) {
        count_digit(lds, is && key >> (shift + bits) == found, key >> shift & mask, lane);
      });
    }
    __syncthreads();
    take_counts(lds, mine);
    find_digit(lds, mine, need);
    found = found << bits | lds.digit;
    need = lds.left;
  }

  // `found` is the last key kept, `need` of its tokens stay.
  int32_t more = 0, same = 0;
  each([&](int32_t, bool is, uint32_t key) {
    more += __builtin_popcountll(__ballot(is && key > found));
    same += __builtin_popcountll(__ballot(is && key == found));
  });
  if (lane == 0) {
    lds.above[wave] = more;
    lds.equal[wave] = same;
  }
  __syncthreads();
  int32_t higher = 0, ties = 0;  // in the runs before
#pragma unroll
  for (int i = 0; i < kKeepWaves; ++i) {
    higher += i < wave ? lds.above[i] : 0;
    ties += i < wave ? lds.equal[i] : 0;
  }
  keep_in_order(c, found, int32_t(need), higher, ties, each);
}

// The same of long rows that are few, by many workgroups: a segment of a row is one's, in four launches.  The first digits are
// counted; with the row's counts together every workgroup knows the last one kept and lists its keys that have it; one
// workgroup a row finds the last key among them, and how many tokens of each segment are above it and equal to it; and the
// segments write their tokens.
constexpr int kSegmentKeys = kKeepSegment / kKeepThreads;  // of a lane

// A lane's keys of a segment, each wave a run of it: f(place in the middle, whether there is such a token, its key).
struct Segment {
  int32_t from, upto;
  uint32_t key[kSegmentKeys];
  template <typename F>
  __device__ __forceinline__ void each(int lane, F f) const {
#pragma unroll
    for (int i = 0; i < kSegmentKeys; ++i)
      if (from + 64 * i < upto) f(from + 64 * i + lane, from + 64 * i + lane < upto, key[i]);
  }
};
__device__ __forceinline__ Segment segment_of(const Choice& c, int32_t segment, int lane, int wave) {
  Segment g;
  const int64_t begin = int64_t(segment) * kKeepSegment + wave * (64 * kSegmentKeys);
  g.from = int32_t(begin < c.middle ? begin : c.middle);
  g.upto = int32_t(begin + 64 * kSegmentKeys < c.middle ? begin + 64 * kSegmentKeys : c.middle);
  float w[kSegmentKeys];
#pragma unroll
  for (int i = 0; i < kSegmentKeys; ++i) w[i] = g.from + 64 * i + lane < g.upto ? c.w[g.from + 64 * i + lane] : 0.0f;
#pragma unroll
  for (int i = 0; i < kSegmentKeys; ++i) g.key[i] = key_of(w[i]);
  return g;
}
__device__ __forceinline__ int32_t segments_of(const Choice& c) { return (c.middle + kKeepSegment - 1) / kKeepSegment; }

__global__ __launch_bounds__(kKeepThreads) void keep_count_kernel(ServeArgs s, KeepArgs a) {
  __shared__ KeepShared lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t row = int32_t(blockIdx.x / uint32_t(a.segments)), segment = int32_t(blockIdx.x % uint32_t(a.segments));
  const Choice c = choice_of(s, a, row);
  if (segment == 0) keep_ends(a, c);
  if (!c.choose || segment >= segments_of(c)) return;
  const Segment g = segment_of(c, segment, lane, wave);
  for (int i = tid; i < kDigits * kCopies; i += kKeepThreads) lds.count[i] = 0;
  __syncthreads();
  g.each(lane, [&](int32_t, bool is, uint32_t key) { count_digit(lds, is, key >> 21, lane); });
  __syncthreads();
  uint32_t mine[2];
  take_counts(lds, mine);
  reinterpret_cast<u32x2*>(a.counts)[int64_t(blockIdx.x) * kKeepThreads + tid] = u32x2{mine[0], mine[1]};
}

__global__ __launch_bounds__(kKeepThreads) void keep_list_kernel(ServeArgs s, KeepArgs a) {
  __shared__ KeepShared lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t row = int32_t(blockIdx.x / uint32_t(a.segments)), segment = int32_t(blockIdx.x % uint32_t(a.segments));
  const Choice c = choice_of(s, a, row);
  const int32_t segments = segments_of(c);
  if (!c.choose || segment >= segments) return;
  const Segment g = segment_of(c, segment, lane, wave);
  const u32x2* counts = reinterpret_cast<const u32x2*>(a.counts) + int64_t(row) * a.segments * kKeepThreads + tid;
  uint32_t mine[2] = {};
  for (int32_t i = 0; i < segments; i += 8) {
    u32x2 v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e < segments ? counts[int64_t(i + e) * kKeepThreads] : u32x2{};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mine[0] += v[e][0];
      mine[1] += v[e][1];
    }
  }
  if (tid == 0) {
    lds.listed = 0;
    lds.above[0] = 0;
  }
  find_digit(lds, mine, c.need);
  const uint32_t found = lds.digit;
  uint32_t* list = a.lists + int64_t(blockIdx.x) * kKeepSegment;
  int32_t more = 0;
  g.each(lane, [&](int32_t, bool is, uint32_t key) {
    more += __builtin_popcountll(__ballot(is && key >> 21 > found));
    const bool on = is && key >> 21 == found;
    const uint64_t who = __ballot(on);
    if (!who) return;
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(&lds.listed, uint32_t(__builtin_popcountll(who)));
    at = uint32_t(__builtin_amdgcn_readfirstlane(int(at)));
    if (on) list[at + before(who)] = key;
  });
  if (lane == 0) atomicAdd(&lds.above[0], more);
  __syncthreads();
  if (tid == 0) {
    a.segment[blockIdx.x] = KeepSegment{int32_t(lds.listed), lds.above[0]};
    if (segment == 0) a.row[row] = KeepRow{found, lds.left};
  }
}

__global__ __launch_bounds__(kKeepThreads) void keep_find_kernel(ServeArgs s, KeepArgs a) {
  __shared__ KeepShared lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t row = int32_t(blockIdx.x);
  const Choice c = choice_of(s, a, row);
  if (!c.choose) return;
  const int32_t segments = segments_of(c);
  KeepSegment* segment = a.segment + int64_t(row) * a.segments;
  const uint32_t* lists = a.lists + int64_t(row) * a.segments * kKeepSegment;
  uint32_t found = a.row[row].last, need = a.row[row].need;
  for (int i = tid; i < kDigits * kCopies; i += kKeepThreads) lds.count[i] = 0;
  __syncthreads();
  // The listed keys of each segment, a wave to a segment.
  auto each = [&](int32_t which, auto f) {
    const int32_t many = segment[which].listed;
    const uint32_t* list = lists + int64_t(which) * kKeepSegment;
    for (int32_t i = 0; i < many; i += 64 * kLoadsAhead) {
      uint32_t v[kLoadsAhead];
#pragma unroll
      for (int e = 0; e < kLoadsAhead; ++e) v[e] = i + 64 * e + lane < many ? list[i + 64 * e + lane] : 0;
#pragma unroll
      for (int e = 0; e < kLoadsAhead; ++e)
        if (i + 64 * e < many) f(i + 64 * e + lane < many, v[e]);
    }
  };
  constexpr int kAt[2] = {10, 0}, kBits[2] = {11, 10};
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const int shift = kAt[d], bits = kBits[d];
    for (int32_t i = wave; i < segments; i += kKeepWaves)
      each(i, [&](bool is, uint32_t key) {
        count_digit(lds, is && key >> (shift + bits) == found, key >> shift & ((1u << bits) - 1), lane);
      });
    __syncthreads();
    uint32_t mine[2];
    take_counts(lds, mine);
    find_digit(lds, mine, need);
    found = found << bits | lds.digit;
    need = lds.left;
  }
  if (tid == 0) a.row[row] = KeepRow{found, need};
  // Tokens of each segment above the last key and equal to it, then those of the segments before.
  for (int32_t i = wave; i < segments; i += kKeepWaves) {
    int32_t more = segment[i].above, same = 0;
    each(i, [&](bool is, uint32_t key) {
      more += __builtin_popcountll(__ballot(is && key > found));
      same += __builtin_popcountll(__ballot(is && key == found));
    });
    if (lane == 0) segment[i] = KeepSegment{same, more};
  }
  __syncthreads();
  if (wave != 0) return;
  int32_t higher = 0, ties = 0;
  for (int32_t i0 = 0; i0 < segments; i0 += 64) {
    const KeepSegment mine = i0 + lane < segments ? segment[i0 + lane] : KeepSegment{0, 0};
    int32_t more = mine.above, same = mine.listed;
    for (int off = 1; off < 64; off <<= 1) {
      const int32_t m = __shfl_up(more, off), e = __shfl_up(same, off);
      more += lane >= off ? m : 0;
      same += lane >= off ? e : 0;
    }
    if (i0 + lane < segments) segment[i0 + lane] = KeepSegment{ties + same - mine.listed, higher + more - mine.above};
    higher += __shfl(more, 63);
    ties += __shfl(same, 63);
  }
}

__global__ __launch_bounds__(kKeepThreads) void keep_write_kernel(ServeArgs s, KeepArgs a) {
  __shared__ int32_t above[kKeepWaves], equal[kKeepWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t row = int32_t(blockIdx.x / uint32_t(a.segments)), segment = int32_t(blockIdx.x % uint32_t(a.segments));
  const Choice c = choice_of(s, a, row);
  if (!c.choose || segment >= segments_of(c)) return;
  const Segment g = segment_of(c, segment, lane, wave);
  const KeepRow last = a.row[row];
  const KeepSegment begin = a.segment[blockIdx.x];
  const uint32_t found = last.last;
  int32_t more = 0, same = 0;
  g.each(lane, [&](int32_t, bool is, uint32_t key) {
    more += __builtin_popcountll(__ballot(is && key > found));
    same += __builtin_popcountll(__ballot(is && key == found));
  });
  if (lane == 0) {
    above[wave] = more;
    equal[wave] = same;
  }
  __syncthreads();
  int32_t higher = begin.above, ties = begin.listed;
#pragma unroll
  for (int i = 0; i < kKeepWaves; ++i) {
    higher += i < wave ? above[i] : 0;
    ties += i < wave ? equal[i] : 0;
  }
  keep_in_order(c, found, int32_t(last.need), higher, ties, [&](auto f) { g.each(lane, f); });
}

// ---- Their rows to the front ----
//
// Row j of a sequence becomes its row kept[j] >= j.  In place that is one chain: a workgroup goes over one slice of the rows'
// bytes (of one head's K or V) in order, reads a chunk of rows, and writes it once all its threads have read theirs; what later
// chunks read lies behind what it writes.  Chains are many because every head, K and V, and every slice of a row are one
// of their own, and a chunk is as much as 1024 threads hold.  To other pages there is no order to keep, and chunks are workgroups.

template <int BYTES>
struct Piece;
template <>
struct Piece<16> { typedef u32x4 type; };
template <>
struct Piece<8> { typedef u32x2 type; };

constexpr int kPart = 2;  // rows of a thread, of the kRowsAhead of a chunk, that are written while as many are read

// Where a row goes from and to: page and slot, page -1 for none.
struct Move {
  int32_t from_page, from_slot, to_page, to_slot;
};

__device__ __forceinline__ int32_t page_at(const int32_t* table, int32_t width, int64_t pool, int32_t at) {
  if (at >= width) return -1;
  const int32_t p = table[at];
  return p >= 0 && p < pool ? p : -1;
}

template <int BYTES, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS > 256 ? 8 : 4) void evict_kernel(ServeArgs s, EvictArgs a) {
  typedef typename Piece<BYTES>::type Word;
  __shared__ Move moves[move_rows(THREADS, 2)];
  const int tid = threadIdx.x;
  const int32_t seq = int32_t(blockIdx.x / uint32_t(a.units));
  int32_t unit = int32_t(blockIdx.x % uint32_t(a.units));
  const int32_t n = kept_len(s, s.kv_lens[seq]);
  int32_t m = a.kept_lens[seq];
  m = m < 0 ? 0 : m < n ? m : n;
  m = m < a.budget ? m : a.budget;
  const bool in_place = a.table == nullptr;

  if (unit < a.weight_units) {  // a row of weights, always in place
    float* w = a.weights + int64_t(seq) * a.seq_stride + int64_t(unit) * a.weight_stride;
    const int32_t* kept = a.kept + (int64_t(seq) * a.heads + unit) * a.budget;
    if (m >= n) return;
    for (int32_t c0 = 0; c0 < m; c0 += THREADS * kRowsAhead) {
      int32_t from[kRowsAhead];
      float v[kRowsAhead];
#pragma unroll
      for (int i = 0; i < kRowsAhead; ++i) {
        const int32_t j = c0 + i * THREADS + tid;
        from[i] = j < m ? kept[j] : -1;
        if (from[i] >= n) from[i] = -1;
      }
#pragma unroll
      for (int i = 0; i < kRowsAhead; ++i) v[i] = from[i] >= 0 ? w[from[i]] : 0.0f;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRowsAhead; ++i)
        if (from[i] >= 0) w[c0 + i * THREADS + tid] = v[i];
    }
    __syncthreads();
    for (int64_t j = m + tid; j < n; j += THREADS) w[j] = 0.0f;
    return;
  }
  unit -= a.weight_units;
  const int32_t split = unit % a.splits;
  unit /= a.splits;
  const int32_t slice = unit % a.slices;
  unit /= a.slices;
  const int32_t which = unit % 2, head = unit / 2;
  if (which ? slice >= a.v_slices : slice >= a.k_slices) return;
  if (in_place && m >= n) return;
  const int32_t* kept = a.kept + (int64_t(seq) * a.heads + (a.heads > 1 ? head : 0)) * a.budget;
  const int32_t* source_table = s.page_table + int64_t(seq) * s.pages_per_seq;
  const int32_t* target_table = in_place ? source_table : a.table + int64_t(seq) * a.table_pages;
  const int32_t target_pages = in_place ? s.pages_per_seq : a.table_pages;

  // A row's slice is 1 << log2_lanes pieces, one to a lane.
  const int32_t lane = tid & ((1 << a.log2_lanes) - 1), row0 = tid >> a.log2_lanes;
  const int32_t piece = (slice << a.log2_lanes) + lane;
  const int32_t per = THREADS >> a.log2_lanes, chunk = move_rows(THREADS, a.log2_lanes);
  const int32_t row_bytes = which ? a.v_bytes : a.k_bytes;
  const bool mine = piece * BYTES < row_bytes;
  const bool scaled = s.tag != PKV_TAG_FP16 && piece == 0;  // the lane with a row's scale and zero
  char* base;
  int64_t page_bytes, slot_bytes;
  if (s.tag == PKV_TAG_FP16) {
    base = reinterpret_cast<char*>((which ? s.v_cache : s.k_cache) + int64_t(head) * s.D) + piece * BYTES;
    page_bytes = 2 * s.page_stride;
    slot_bytes = int64_t(s.H) * s.D * 2;
  } else {
    base = reinterpret_cast<char*>(s.codes) + head * s.head_stride + (which ? s.v_offset : 0) + piece * BYTES;
    page_bytes = s.page_stride;
    slot_bytes = row_bytes;
  }
  uint32_t* scales = s.scales + ((int64_t(head) * 2 + which) << s.log2P);
  const int32_t slots = (1 << s.log2P) - 1;
  for (int64_t c0 = int64_t(split) * chunk; c0 < m; c0 += int64_t(a.splits) * chunk) {
    // The chunk's moves, a row to a thread.
    for (int32_t r = tid; r < chunk; r += THREADS) {
      const int64_t j = c0 + r;
      Move v{-1, 0, -1, int32_t(j) & slots};
      const int32_t at = j < m ? kept[j] : -1;
      if (at >= 0 && at < n && (!in_place || at != j)) {
        v.from_page = page_at(source_table, s.pages_per_seq, s.pool_pages, at >> s.log2P);
        v.from_slot = at & slots;
        v.to_page = page_at(target_table, target_pages, s.pool_pages, int32_t(j >> s.log2P));
        if (v.to_page < 0) v.from_page = -1;
      }
      moves[r] = v;
    }
    __syncthreads();
    // In place a part of the chunk is written while the next one is read: a barrier between a part's loads and its stores.
    Word v[2][kPart];
    uint32_t sz[2][kPart];
    auto each = [&](int p, auto f) {
#pragma unroll
      for (int e = 0; e < kPart; ++e) {
        const int32_t r = (p * kPart + e) * per + row0;
        if (r >= chunk) break;
        const Move at = moves[r];
        if (mine && at.from_page >= 0) f(e, at);
      }
    };
    auto load = [&](int p) {
      each(p, [&](int e, const Move& at) {
        v[p & 1][e] = *reinterpret_cast<const Word*>(base + at.from_page * page_bytes + at.from_slot * slot_bytes);
        if (scaled) sz[p & 1][e] = scales[at.from_page * s.scale_stride + at.from_slot];
      });
    };
    load(0);
#pragma unroll
    for (int p = 0; p < kRowsAhead / kPart; ++p) {
      if (p + 1 < kRowsAhead / kPart) load(p + 1);
      if (in_place) __syncthreads();
      each(p, [&](int e, const Move& at) {
        *reinterpret_cast<Word*>(base + at.to_page * page_bytes + at.to_slot * slot_bytes) = v[p & 1][e];
        if (scaled) scales[at.to_page * s.scale_stride + at.to_slot] = sz[p & 1][e];
      });
    }
    __syncthreads();
  }
}

}  // namespace

pkv_status_t launch_keep(const ServeArgs& s, const KeepArgs& a, hipStream_t stream) {
  const uint32_t rows = uint32_t(s.num_seqs) * uint32_t(a.heads);
  auto go = [&](auto kernel, uint32_t groups) {
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(kKeepThreads), 0, stream, s, a);
  };
  if (a.segments) {
    go(keep_count_kernel, rows * uint32_t(a.segments));
    go(keep_list_kernel, rows * uint32_t(a.segments));
    go(keep_find_kernel, rows);
    go(keep_write_kernel, rows * uint32_t(a.segments));
  } else {
    go(keep_kernel, rows);
  }
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_DEVICE;
}

pkv_status_t launch_evict(const ServeArgs& s, const EvictArgs& a, hipStream_t stream) {
  const dim3 grid(uint32_t(s.num_seqs) * uint32_t(a.units));
  auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, s, a); };
  if (a.table) {
    if (a.piece_bytes == 16) go(evict_kernel<16, kMoveThreads>, kMoveThreads);
    else go(evict_kernel<8, kMoveThreads>, kMoveThreads);
  } else {
    if (a.piece_bytes == 16) go(evict_kernel<16, kChainThreads>, kChainThreads);
    else go(evict_kernel<8, kChainThreads>, kChainThreads);
  }
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_DEVICE;
}

}  // namespace pkv
