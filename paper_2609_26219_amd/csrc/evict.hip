// Eviction from a paged cache: which tokens stay under a budget (pkv_cache_keep)
// and their rows moved to the front of their sequence (pkv_cache_evict).
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
// The weights' bits as whole numbers in their order; the number of the last one kept is found a digit of 8 bits at a time
// from the top (a count of each digit among those that share the digits found, in LDS), and then the tokens above it and the
// first ones equal to it are written in order.  A workgroup takes one row of weights, each wave a run of it.

constexpr int kKeepThreads = 1024;
constexpr int kKeepWaves = kKeepThreads / 64;
constexpr int kCopies = 16;      // of a digit's count, so that lanes seldom meet in one
constexpr int kHeldKeys = 32;    // a lane's keys that stay in registers

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

template <bool HELD>
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(ServeArgs s, KeepArgs a) {
  __shared__ uint32_t count[256 * kCopies];
  __shared__ uint32_t digit, left;
  __shared__ int32_t above[kKeepWaves], equal[kKeepWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t seq = int32_t(blockIdx.x / uint32_t(a.heads)), head = int32_t(blockIdx.x % uint32_t(a.heads));
  const float* w = a.weights + int64_t(seq) * a.seq_stride + int64_t(head) * a.head_stride;
  int32_t* kept = a.kept + (int64_t(seq) * a.heads + head) * a.budget;
  const int32_t n = kept_len(s, s.kv_lens[seq]);
  const int32_t m = kept_budget(a, n, a.budgets ? a.budgets[seq] : a.budget);
  const int32_t first = a.sinks < m ? a.sinks : m, last = a.recent < m - first ? a.recent : m - first;
  if (head == 0 && tid == 0) a.kept_lens[seq] = m;
  const int32_t middle = n - first - last;  // tokens to choose from,
  uint32_t need = uint32_t(m - first - last);  // and how many of them stay
  for (int32_t j = tid; j < first; j += kKeepThreads) kept[j] = j;
  for (int32_t j = tid; j < last; j += kKeepThreads) kept[m - last + j] = n - last + j;
  for (int32_t j = m + tid; j < a.budget; j += kKeepThreads) kept[j] = -1;
  if (need == 0) return;
  if (need == uint32_t(middle)) {
    for (int32_t j = tid; j < middle; j += kKeepThreads) kept[first + j] = first + j;
    return;
  }

  // The wave's run of the middle.
  const int32_t run = ((middle + kKeepThreads - 1) / kKeepThreads) * 64;
  const int32_t from = wave * run, upto = from + run < middle ? from + run : middle;
  w += first;
  uint32_t held[HELD ? kHeldKeys : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i) {
      const int32_t at = from + 64 * i + lane;
      held[i] = at < upto ? key_of(w[at]) : 0;
    }
  }
  auto each = [&](auto f) {
    if constexpr (HELD) {
#pragma unroll
      for (int i = 0; i < kHeldKeys; ++i)
        if (from + 64 * i < upto) f(from + 64 * i + lane, held[i]);
    } else {
      for (int32_t i = from; i < upto; i += 64) f(i + lane, i + lane < upto ? key_of(w[i + lane]) : 0);
    }
  };

  uint32_t found = 0;  // digits found so far
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256 * kCopies; i += kKeepThreads) count[i] = 0;
    __syncthreads();
    each([&](int32_t at, uint32_t key) {
      if (at < upto && uint64_t(key) >> (shift + 8) == found)
        atomicAdd(&count[((key >> shift) & 255) * kCopies + (lane & (kCopies - 1))], 1u);
    });
    __syncthreads();
    if (tid < 64) {  // digits 255 - 4 tid .. downwards
      uint32_t mine[4], sum = 0;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint32_t c = 0;
        for (int i = 0; i < kCopies; ++i) c += count[(255 - 4 * lane - d) * kCopies + ((i + lane) & (kCopies - 1))];
        mine[d] = c;
        sum += c;
      }
      uint32_t upper = sum;
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t other = __shfl_up(upper, off);
        upper += lane >= off ? other : 0;
      }
      upper -= sum;  // of larger digits
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        if (upper < need && need <= upper + mine[d]) {
          digit = uint32_t(255 - 4 * lane - d);
          left = need - upper;
        }
        upper += mine[d];
      }
    }
    __syncthreads();
    found = found << 8 | digit;
    need = left;
  }

  // `found` is the last key kept, `need` of its tokens stay.
  int32_t more = 0, same = 0;
  each([&](int32_t at, uint32_t key) {
    more += __builtin_popcountll(__ballot(at < upto && key > found));
    same += __builtin_popcountll(__ballot(at < upto && key == found));
  });
  if (lane == 0) {
    above[wave] = more;
    equal[wave] = same;
  }
  __syncthreads();
  int32_t higher = 0, ties = 0;  // in the runs before
  for (int i = 0; i < wave; ++i) {
    higher += above[i];
    ties += equal[i];
  }
  const int32_t most = int32_t(need);
  each([&](int32_t at, uint32_t key) {
    const bool is = at < upto;
    const uint64_t gt = __ballot(is && key > found), eq = __ballot(is && key == found);
    const int32_t tie = ties + before(eq);
    const int32_t place = higher + before(gt) + (tie < most ? tie : most);
    if (is && (key > found || (key == found && tie < most))) kept[first + place] = first + at;
    higher += __builtin_popcountll(gt);
    ties += __builtin_popcountll(eq);
  });
}

// ---- Their rows to the front ----
//
// Row j of a sequence becomes its row kept[j] >= j.  In place that is one chain: a workgroup goes over one slice of the rows'
// bytes (of one head's K or V) in order, reads a chunk of rows, and writes it once all its threads have read theirs; what later
// chunks read lies behind what it writes.  Chains are many because every head, K and V, and every 64 bytes of a row are one
// of their own.  To other pages there is no order to keep, and chunks are workgroups too.

constexpr int kThreads = 256;
constexpr int kRowsAhead = 8;  // rows of a thread in a chunk

template <int BYTES>
struct Piece;
template <>
struct Piece<16> { typedef u32x4 type; };
template <>
struct Piece<8> { typedef u32x2 type; };

// Rows that are not there.
constexpr int32_t kNone = -1;

__device__ __forceinline__ int32_t page_at(const int32_t* table, int32_t width, int64_t pool, int32_t at) {
  if (at >= width) return kNone;
  const int32_t p = table[at];
  return p >= 0 && p < pool ? p : kNone;
}

template <int BYTES>
__global__ __launch_bounds__(kThreads) void evict_kernel(ServeArgs s, EvictArgs a) {
  typedef typename Piece<BYTES>::type Word;
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
    for (int32_t c0 = 0; c0 < m; c0 += kThreads * kRowsAhead) {
      float v[kRowsAhead];
#pragma unroll
      for (int i = 0; i < kRowsAhead; ++i) {
        const int32_t j = c0 + i * kThreads + tid;
        const int32_t from = j < m ? kept[j] : kNone;
        v[i] = from >= 0 && from < n ? w[from] : 0.0f;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRowsAhead; ++i) {
        const int32_t j = c0 + i * kThreads + tid;
        if (j < m) w[j] = v[i];
      }
    }
    __syncthreads();
    for (int64_t j = m + tid; j < n; j += kThreads) w[j] = 0.0f;
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
  const int32_t piece = (slice << a.log2_lanes) + (tid & ((1 << a.log2_lanes) - 1)), row_of = tid >> a.log2_lanes;
  const int32_t per = kThreads >> a.log2_lanes, chunk = per * kRowsAhead;
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
  for (int32_t c0 = split * chunk; c0 < m; c0 += a.splits * chunk) {
    Word v[kRowsAhead];
    uint32_t sz[kRowsAhead];
    int32_t from[kRowsAhead], to[kRowsAhead];
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int32_t j = c0 + i * per + row_of;
      from[i] = j < m ? kept[j] : kNone;
    }
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int32_t j = c0 + i * per + row_of, at = from[i];
      to[i] = kNone;
      if (mine && at >= 0 && at < n && (!in_place || at != j)) {
        const int32_t page = page_at(source_table, s.pages_per_seq, s.pool_pages, at >> s.log2P);
        if (page >= 0) {
          to[i] = page_at(target_table, target_pages, s.pool_pages, j >> s.log2P);
          v[i] = *reinterpret_cast<const Word*>(base + page * page_bytes + (at & slots) * slot_bytes);
          if (scaled) sz[i] = scales[page * s.scale_stride + (at & slots)];
        }
      }
    }
    if (in_place) __syncthreads();
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int32_t j = c0 + i * per + row_of;
      if (to[i] >= 0) {
        *reinterpret_cast<Word*>(base + to[i] * page_bytes + (j & slots) * slot_bytes) = v[i];
        if (scaled) scales[to[i] * s.scale_stride + (j & slots)] = sz[i];
      }
    }
  }
}

}  // namespace

pkv_status_t launch_keep(const ServeArgs& s, const KeepArgs& a, hipStream_t stream) {
  const dim3 grid(uint32_t(s.num_seqs) * uint32_t(a.heads));
  if (s.max_kv <= kHeldKeys * kKeepThreads) hipLaunchKernelGGL(keep_kernel<true>, grid, dim3(kKeepThreads), 0, stream, s, a);
  else hipLaunchKernelGGL(keep_kernel<false>, grid, dim3(kKeepThreads), 0, stream, s, a);
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_DEVICE;
}

pkv_status_t launch_evict(const ServeArgs& s, const EvictArgs& a, hipStream_t stream) {
  const dim3 grid(uint32_t(s.num_seqs) * uint32_t(a.units));
  if (a.piece_bytes == 16) hipLaunchKernelGGL(evict_kernel<16>, grid, dim3(kThreads), 0, stream, s, a);
  else hipLaunchKernelGGL(evict_kernel<8>, grid, dim3(kThreads), 0, stream, s, a);
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_DEVICE;
}

}  // namespace pkv
