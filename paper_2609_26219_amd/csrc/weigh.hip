// The attention weight that cached tokens receive (pkv_attention_weights), for one
// head_dim (PKV_HEAD_DIM; built once for each of 64, 128 and 256).
//
// A token's weight is the column sum of the softmax: with the rows' log-sum-exp from the attention call,
//   w_t = sum over rows i and query heads h of exp(scale q_ih . k_t - lse_ih),
// so no row needs another's result, nothing is rescaled, and V is not read.  Scores are matrix instructions with
// rows along M and tokens along N: a lane holds one token's scores of several rows, and the sum over rows is
// additions in its own registers but for one exchange at the end.  Every token is summed by one lane group in a
// fixed order, or in parts that are joined in a fixed order, so the result does not depend on how workgroups run.
//
// Codes go in as attention takes them (integers around mid-code, exact in binary16), a token's scale and zero
// act on its lane: q . k_t = s_t (q . codes_t) + z'_t sum(q).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pkv.h"
#include "paged_tiles.h"
#include "pkv_internal.h"
#include "serve.h"

namespace pkv {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// A sequence's rows, from what the device holds.
__device__ __forceinline__ SequenceRows sequence_rows(const ServeArgs& s, int32_t seq) {
  return rows_of_sequence(s, scalar_entry(s.token_start, seq), scalar_entry(s.token_start, seq + 1),
                          scalar_entry(s.kv_lens, seq));
}

// Position of a sequence's row `token`, and what it sees.
__device__ __forceinline__ Sight sight_of(const ServeArgs& s, const WeighArgs& a, const SequenceRows& g, int32_t token) {
  const int32_t pos = s.positions ? s.positions[g.start + token] : g.kv_len - g.trail + token;
  Sight see;
  see.hi = pos < g.kv_len ? pos : g.kv_len - 1;
  see.hi = see.hi < -1 ? -1 : see.hi;
  see.lo = a.window > 0 && pos >= a.window ? pos - a.window : -1;
  return see;
}

// What a row's scores are turned into probabilities by: exp2(f * (q . k) + less), the query's sum for the zeros of codes.
struct RowScale {
  float f, less, sum;
};

// -lse in base 2; a row that saw nothing has lse = -inf and gives nothing.
__device__ __forceinline__ float less_of(const WeighArgs& a, const SequenceRows& g, int32_t token, int32_t head) {
  const float lse = a.lse[int64_t(g.start + token) * a.Hq + head];
  return lse == -kInf ? -kInf : lse * -1.44269504088896340736f;
}

// What is put where: the sum itself if a call has no parts.
__device__ __forceinline__ void put(const WeighArgs& a, int64_t at, float sum) {
  a.out[at] = a.weights ? __builtin_fmaf(a.decay, a.weights[at], sum) : sum;
}

template <bool HALF>
__device__ __forceinline__ f32x4 mfma16(const u32x4& x, const u32x4& y, const f32x4& z) {
  if constexpr (HALF)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
}
template <bool HALF>
__device__ __forceinline__ f32x16 mfma32(const u32x4& x, const u32x4& y, const f32x16& z) {
  if constexpr (HALF)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
}

// 8 channels of a query as floats.
__device__ __forceinline__ void widen(bool bf16, const u32x4& w, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t bits = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFF;
    v[e] = bf16 ? bf16_float(bits) : f16_float(bits);
  }
}
// The power of two that brings a row's largest magnitude to 1..2, and its inverse (both normal numbers).
__device__ __forceinline__ void row_scale(uint32_t top, float& down, float& up) {
  int e = int(top >> 23) - 127;
  e = e < -60 ? -60 : e > 120 ? 120 : e;
  down = __uint_as_float(uint32_t(127 - e) << 23);
  up = __uint_as_float(uint32_t(127 + e) << 23);
}
// The channels in the operand's order for codes of so many bits.
template <int KB>
__device__ __forceinline__ u32x4 query_operand(const float (&v)[8], float down) {
  u32x4 q;
#pragma unroll
  for (int p = 0; p < 4; ++p) q[p] = pack_f16(v[k_channel<KB>(p, 0)] * down, v[k_channel<KB>(p, 1)] * down);
  return q;
}

// ---- Few rows ----
//
// The rows of a sequence and KV head fit RT tiles of 16, whose queries a wave keeps in registers while it goes over
// tokens: the call waits for the cache's bytes.  A workgroup takes `chunk` tokens of one sequence and all heads: wave w the
// w % subs-th part of them, of heads w / subs and on.  Where heads are joined, the waves' sums of a token meet in LDS.

constexpr int kFewWaves = 8;

template <bool BF16, int KB, bool WHOLE, int RT>
__global__ __launch_bounds__(64 * kFewWaves, KB * D * RT <= 512 ? 4 : 2) void few_kernel(ServeArgs s, WeighArgs a) {
  constexpr bool kCodes = KB != 16;
  constexpr bool kHalf = kCodes || !BF16;
  constexpr int kSteps = D / 32;
  __shared__ float sums[kFewWaves][kMostChunk];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4, x = lane & 15;
  const int32_t seq = int32_t(blockIdx.x / uint32_t(a.tiles)), tile0 = int32_t(blockIdx.x % uint32_t(a.tiles));
  const SequenceRows g = sequence_rows(s, seq);
  const int64_t begin = int64_t(tile0) * a.chunk;
  if (begin >= g.kv_len) return;
  const int32_t part = a.chunk / a.subs, sub = wave % a.subs, first_head = wave / a.subs, heads = kFewWaves / a.subs;
  const int32_t from = int32_t(begin) + sub * part;
  const int32_t upto = g.kv_len - from < part ? g.kv_len : from + part;
  const Magic m = magic();
  if (a.joint) {
    for (int32_t i = lane; i < part; i += 64) sums[wave][i] = 0.0f;
    __syncthreads();
  }

  // What the rows see between them; tiles of which none sees anything are not looked at.
  int32_t hi_most = -1, lo_least = 0x7FFFFFFF;
  if (g.count > 0 && !s.positions) {
    hi_most = g.kv_len - g.trail + g.count - 1;
    lo_least = sight_of(s, a, g, 0).lo;
  } else if (s.positions) {
    for (int32_t i = lane; i < g.count; i += 64) {
      const Sight see = sight_of(s, a, g, i);
      hi_most = max(hi_most, see.hi);
      if (see.hi >= 0) lo_least = min(lo_least, see.lo);
    }
    for (int off = 1; off < 64; off <<= 1) {
      hi_most = max(hi_most, __shfl_xor(hi_most, off));
      lo_least = min(lo_least, __shfl_xor(lo_least, off));
    }
  }
  hi_most = __builtin_amdgcn_readfirstlane(hi_most);
  lo_least = __builtin_amdgcn_readfirstlane(lo_least);
  auto seen = [&](int32_t t0) { return t0 <= hi_most && (t0 + kTokenTile - 1 > lo_least || t0 < a.sinks); };

  for (int32_t head = first_head; head < s.H && from < upto; head += heads) {
    const Source src = source_of<KB>(s, seq, head);
    Keys<KB> keys[2];  // of two tiles: one is used while the other is on its way
    uint32_t words[2][2];
    bool there[2][2];
    auto load = [&](int b, int32_t t0) {
      if (t0 >= upto || !seen(t0)) return;
      Tile tile{t0, {-1, -1}};
      if constexpr (WHOLE) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int32_t at = (t0 + 16 * u) >> s.log2P;
          if (at < s.pages_per_seq) {
            const int32_t p = scalar_entry(src.table, at);
            tile.page[u] = p >= 0 && p < s.pool_pages ? p : -1;
          }
        }
      }
      load_keys<KB, WHOLE>(s, src, tile, c, x, keys[b]);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int32_t t = t0 + 16 * u + x;
        const int32_t page = WHOLE ? tile.page[u] : page_of(s, src.table, t >> s.log2P);
        there[b][u] = page >= 0 && t < g.kv_len;
        if constexpr (kCodes)
          words[b][u] = src.scales[uint64_t(uint32_t(page < 0 ? 0 : page)) * uint32_t(s.scale_stride) +
                                uint32_t(t & ((1 << s.log2P) - 1))];
      }
    };
    load(0, from);
    load(1, from + kTokenTile);

    // Row x of each row tile: its queries, and what it is scaled by.
    u32x4 q[RT][kSteps];
    f32x4 f[RT], less[RT], sum[RT];
    int32_t hi[RT][4], lo[RT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int32_t row = 16 * r + x, token = row / a.group, qhead = head * a.group + row % a.group;
      const bool on = token < g.count;
      Sight see{-1, -1};
      RowScale rs{a.scale, -kInf, 0.0f};
      if (on) {
        rs.less = less_of(a, g, token, qhead);
        if (rs.less != -kInf) see = sight_of(s, a, g, token);
      }
      const uint16_t* rowq = a.q + int64_t(g.start + (on ? token : 0)) * a.q_token_stride + int64_t(qhead) * a.q_head_stride;
      float v[kSteps][8];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        u32x4 w{};
        if (on) w = *reinterpret_cast<const u32x4*>(rowq + k_first<KB>(i, c));
        if constexpr (kCodes) {
          widen(s.bf16, w, v[i]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t mag = __float_as_uint(v[i][e]) & 0x7FFFFFFF;
            top = top > mag ? top : mag;
          }
        } else {
          q[r][i] = w;
        }
      }
      if constexpr (kCodes) {
        top = max(top, uint32_t(__shfl_xor(int(top), 16)));
        top = max(top, uint32_t(__shfl_xor(int(top), 32)));
        float down, up;
        row_scale(top, down, up);
        rs.f *= up;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          q[r][i] = query_operand<KB>(v[i], down);
#pragma unroll
          for (int e = 0; e < 8; ++e) rs.sum += v[i][e] * down;
        }
        rs.sum = over_c_sum(rs.sum);
      }
      // The lane's rows of the scores are 4c + 0..3.
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[r][i] = __shfl(rs.f, 4 * c + i);
        less[r][i] = __shfl(rs.less, 4 * c + i);
        sum[r][i] = __shfl(rs.sum, 4 * c + i);
        hi[r][i] = __shfl(see.hi, 4 * c + i);
        lo[r][i] = __shfl(see.lo, 4 * c + i);
      }
    }

    auto weigh = [&](int b, int32_t t0) {
      float w[2] = {0.0f, 0.0f};
      if (seen(t0)) {
        f32x4 score[RT][2];
        float ks[2], kz[2];
        bool is[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          is[u] = there[b][u];
          if constexpr (kCodes) {
            ks[u] = f16_float(words[b][u]);
            kz[u] = __builtin_fmaf(ks[u], float(1 << (KB - 1)), f16_float(words[b][u] >> 16));
          }
#pragma unroll
          for (int r = 0; r < RT; ++r) score[r][u] = f32x4{};
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            const u32x4 k = k_operand<KB>(m, keys[b].w[u], i);
#pragma unroll
            for (int r = 0; r < RT; ++r) score[r][u] = mfma16<kHalf>(q[r][i], k, score[r][u]);
          }
        }
        load(b, t0 + 2 * kTokenTile);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int32_t tok = t0 + 16 * u + x;
          const bool sink = tok < a.sinks;
          float total = 0.0f;
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float t = score[r][u][i];
              if constexpr (kCodes) t = __builtin_fmaf(ks[u], t, kz[u] * sum[r][i]);
              const float p = exp2_of(__builtin_fmaf(t, f[r][i], less[r][i]));
              total += tok <= hi[r][i] && (tok > lo[r][i] || sink) ? p : 0.0f;
            }
          w[u] = over_c_sum(total);
          if (!is[u]) w[u] = 0.0f;
        }
      } else {
        load(b, t0 + 2 * kTokenTile);
      }
      const int32_t tok = t0 + (lane & 31);
      if (lane < 32 && tok < upto) {
        const float mine = lane & 16 ? w[1] : w[0];
        if (a.joint) sums[wave][tok - from] += mine;
        else put(a, int64_t(seq) * a.seq_stride + int64_t(head) * a.head_stride + tok, mine);
      }
    };
    for (int32_t t0 = from; t0 < upto; t0 += 2 * kTokenTile) {
      weigh(0, t0);
      if (t0 + kTokenTile < upto) weigh(1, t0 + kTokenTile);
    }
  }
  if (!a.joint) return;
  __syncthreads();
  for (int32_t i = threadIdx.x; i < a.chunk; i += 64 * kFewWaves) {
    const int32_t tok = int32_t(begin) + i;
    if (tok >= g.kv_len) break;
    float total = 0.0f;
    for (int32_t w = i / part; w < kFewWaves; w += a.subs) total += sums[w][i % part];
    put(a, int64_t(seq) * a.seq_stride + tok, total);
  }
}

// ---- Many rows ----
//
// A workgroup keeps the keys of 4 * kTokens tokens of one sequence and KV head in registers (each wave its own) and goes
// over the rows that see them, 32 at a time, which its threads bring to LDS in the operands' order, the next ones on
// their way while these are used.

constexpr int kThreads = 256;
constexpr int kNT = D > 128 ? 1 : 2;  // token tiles of 32 of a wave
constexpr int kRows = 32;
constexpr int kRowPieces = D / 8;

// First channel of the 8 that lane half k has in instruction `step`, from pieces of up to 16 bytes; and the other way round.
template <int BITS>
struct Halves {
  static constexpr int kBytes = D / 2 * BITS / 8 < 16 ? D / 2 * BITS / 8 : 16, kPer = kBytes * 8 / BITS, kOps = kPer / 8;
  static constexpr int kPieces = D / 2 * BITS / 8 / kBytes;
  static __device__ constexpr int slot(int channel) {  // 2 * step + half
    const int piece = channel / kPer, step = piece / 2 * kOps + channel % kPer / 8;
    return 2 * step + (piece & 1);
  }
};

struct RowTile {
  u32x4 q[2 * D / 16][kRows + 1];  // [step][half][row], 4 banks on from one to the next
  float f[kRows], less[kRows], sum[kRows];
  int32_t hi[kRows], lo[kRows];
  int32_t off;                             // whether some row gives nothing
  int32_t all_hi, any_hi, all_lo, any_lo;  // rows at positions of their own: least and most of hi, most and least of lo
};

template <bool BF16, int KB>
__global__ __launch_bounds__(kThreads, 2) void many_kernel(ServeArgs s, WeighArgs a) {
  constexpr bool kCodes = KB != 16;
  constexpr bool kHalf = kCodes || !BF16;
  constexpr int kSteps = D / 16, kPasses = kRows * kRowPieces / kThreads;
  typedef Halves<KB> Order;
  __shared__ RowTile lds[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, half = lane >> 5;
  uint32_t b = blockIdx.x;
  const int32_t head = int32_t(b % uint32_t(s.H));
  b /= uint32_t(s.H);
  const int32_t tile = int32_t(b % uint32_t(a.tiles));
  b /= uint32_t(a.tiles);
  const int32_t split = int32_t(b % uint32_t(a.splits)), seq = int32_t(b / uint32_t(a.splits));
  const SequenceRows g = sequence_rows(s, seq);
  constexpr int32_t kTokens = 4 * 32 * kNT;
  const int64_t begin64 = int64_t(tile) * kTokens;
  if (begin64 >= g.kv_len) return;
  const int32_t begin = int32_t(begin64);
  const int32_t last = g.kv_len - begin < kTokens ? g.kv_len - 1 : begin + kTokens - 1;

  // The wave's keys, as operands.
  const Source src = source_of<KB>(s, seq, head);
  const Magic m = magic();
  u32x4 k[kNT][kSteps];
  float ks[kNT], kz[kNT];
  bool there[kNT];
  const int32_t mine = begin + 32 * kNT * wave;  // first token
#pragma unroll
  for (int t = 0; t < kNT; ++t) {
    const int32_t tok = mine + 32 * t + n;
    const int32_t page = tok < g.kv_len ? page_of(s, src.table, tok >> s.log2P) : -1;
    const uint32_t slot = uint32_t(tok & ((1 << s.log2P) - 1));
    there[t] = page >= 0;
    const uint32_t row = KB == 16 ? uint32_t(s.H) * D * 2 : D * KB / 8;
    const char* at = src.k + row_at<KB>(s, page, slot, row) + half * Order::kBytes;
    uint32_t w[D / 2 * KB / 32];
#pragma unroll
    for (int i = 0; i < Order::kPieces; ++i)
      load_bytes<Order::kBytes>(w + i * (Order::kBytes / 4), at + 2 * i * Order::kBytes);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k[t][i] = k_operand<KB>(m, w, i);
    if constexpr (kCodes) {
      const uint32_t word = src.scales[uint64_t(uint32_t(page < 0 ? 0 : page)) * uint32_t(s.scale_stride) + slot];
      ks[t] = f16_float(word);
      kz[t] = __builtin_fmaf(ks[t], float(1 << (KB - 1)), f16_float(word >> 16));
    }
  }

  // The row tiles that see one of the workgroup's tokens, and this split's of them.
  RowRange see_us{0, g.count > 0 ? g.count : 0};
  if (!s.positions) see_us = rows_that_see(g, begin, last, a.window, a.sinks);
  const int64_t first_row = int64_t(see_us.first) * a.group, rows = int64_t(see_us.end) * a.group;
  const int64_t tile0 = first_row / kRows, tiles = rows > first_row ? (rows + kRows - 1) / kRows - tile0 : 0;
  const int32_t from = int32_t(tile0 + tiles * split / a.splits), upto = int32_t(tile0 + tiles * (split + 1) / a.splits);
  const int32_t most = g.count * a.group;  // (below 2^31: num_tokens * Hq)

  // A thread's part of a row tile: a piece of 8 channels of some rows, and one row's numbers.  From one tile to the
  // next its rows are kRows on, so that their tokens and heads are stepped, not divided for.
  struct Cursor {
    int32_t row, token, sub;
  };
  const int32_t step_token = kRows / a.group, step_sub = kRows % a.group;
  auto cursor = [&](int64_t row) {
    return Cursor{int32_t(row), int32_t(row / a.group), int32_t(row % a.group)};
  };
  auto step = [&](Cursor& at) {
    at.row += kRows;
    at.token += step_token;
    at.sub += step_sub;
    if (at.sub >= a.group) {
      at.sub -= a.group;
      ++at.token;
    }
  };
  const int piece = tid % kRowPieces, row0 = tid / kRowPieces;
  const uint16_t* q_head = a.q + int64_t(g.start) * a.q_token_stride + int64_t(head * a.group) * a.q_head_stride + 8 * piece;
  const float* lse = a.lse + int64_t(g.start) * a.Hq + head * a.group;
  Cursor mine_rows[kPasses], my_row = cursor(int64_t(from) * kRows + (tid & (kRows - 1)));
#pragma unroll
  for (int i = 0; i < kPasses; ++i) mine_rows[i] = cursor(int64_t(from) * kRows + row0 + i * (kThreads / kRowPieces));
  u32x4 w[kPasses];
  float less = -kInf;
  Sight see{-1, -1};
  auto fetch = [&] {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      Cursor& at = mine_rows[i];
      w[i] = u32x4{};
      if (at.row < most)
        w[i] = *reinterpret_cast<const u32x4*>(q_head + int64_t(at.token) * a.q_token_stride + at.sub * a.q_head_stride);
      step(at);
    }
    if (tid < kRows) {
      less = -kInf;
      see = Sight{-1, -1};
      if (my_row.row < most) {
        less = lse[int64_t(my_row.token) * a.Hq + my_row.sub];
        see = sight_of(s, a, g, my_row.token);
      }
      step(my_row);
    }
  };
  auto leave = [&](RowTile& to) {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int row = row0 + i * (kThreads / kRowPieces);
      if constexpr (kCodes) {
        float v[8], down, up, sum = 0.0f;
        uint32_t top = 0;
        widen(s.bf16, w[i], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t mag = __float_as_uint(v[e]) & 0x7FFFFFFF;
          top = top > mag ? top : mag;
        }
        for (int off = 1; off < kRowPieces; off <<= 1) top = max(top, uint32_t(__shfl_xor(int(top), off)));
        row_scale(top, down, up);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e] * down;
        for (int off = 1; off < kRowPieces; off <<= 1) sum += __shfl_xor(sum, off);
        to.q[Order::slot(8 * piece)][row] = query_operand<KB>(v, down);
        if (piece == 0) {
          to.f[row] = a.scale * up;
          to.sum[row] = sum;
        }
      } else {
        to.q[Order::slot(8 * piece)][row] = w[i];
      }
    }
    if (tid < kRows) {
      if (less == -kInf) see = Sight{-1, -1};  // it saw nothing, and gives nothing
      to.less[tid] = less == -kInf ? -kInf : less * -1.44269504088896340736f;
      to.hi[tid] = see.hi;
      to.lo[tid] = see.lo;
      const bool off = __any(see.hi < 0);
      if (tid == 0) to.off = off;
      if (s.positions) {
        int32_t all_hi = see.hi, any_hi = see.hi, all_lo = see.lo, any_lo = see.hi < 0 ? 0x7FFFFFFF : see.lo;
        for (int by = 1; by < kRows; by <<= 1) {
          all_hi = min(all_hi, __shfl_xor(all_hi, by));
          any_hi = max(any_hi, __shfl_xor(any_hi, by));
          all_lo = max(all_lo, __shfl_xor(all_lo, by));
          any_lo = min(any_lo, __shfl_xor(any_lo, by));
        }
        if (tid == 0) {
          to.all_hi = all_hi;
          to.any_hi = any_hi;
          to.all_lo = all_lo;
          to.any_lo = any_lo;
        }
      }
    }
  };
  // First and last row of a tile, for rows in order.
  Cursor first_of = cursor(int64_t(from) * kRows), last_of = cursor(int64_t(from) * kRows + kRows - 1);

  float total[kNT] = {};
  if (from < upto) {
    fetch();
    leave(lds[0]);
  }
  __syncthreads();
  for (int32_t at = from; at < upto; ++at) {
    const RowTile& r = lds[(at - from) & 1];
    if (at + 1 < upto) fetch();
    const int32_t end = mine + 32 * kNT - 1;
    int32_t any_hi, any_lo, all_hi, all_lo;
    if (s.positions) {
      any_hi = __builtin_amdgcn_readfirstlane(r.any_hi), any_lo = __builtin_amdgcn_readfirstlane(r.any_lo);
      all_hi = __builtin_amdgcn_readfirstlane(r.all_hi), all_lo = __builtin_amdgcn_readfirstlane(r.all_lo);
    } else {
      const Sight begins = sight_of(s, a, g, first_of.token);
      const Sight ends = sight_of(s, a, g, last_of.token < g.count ? last_of.token : g.count - 1);
      all_hi = begins.hi, any_hi = ends.hi, any_lo = begins.lo, all_lo = ends.lo;
      step(first_of);
      step(last_of);
    }
    const bool off = __builtin_amdgcn_readfirstlane(r.off);
    const bool none = any_hi < mine || (any_lo >= end && mine >= a.sinks);
    if (!none) {
      f32x16 score[kNT];
#pragma unroll
      for (int t = 0; t < kNT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) score[t][e] = 0.0f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const u32x4 q = r.q[2 * i + half][n];
#pragma unroll
        for (int t = 0; t < kNT; ++t) score[t] = mfma32<kHalf>(q, k[t][i], score[t]);
      }
      const bool all = !off && all_hi >= end && (all_lo < mine || end < a.sinks);
      // Value e of a lane is row 8 (e / 4) + 4 half + e % 4.
#pragma unroll
      for (int t = 0; t < kNT; ++t) {
        const int32_t tok = mine + 32 * t + n;
        float part[4] = {};
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const int at_row = 8 * e4 + 4 * half;
          const f32x4 ls = *reinterpret_cast<const f32x4*>(&r.less[at_row]);
          f32x4 f, sum;
          if constexpr (kCodes) {
            f = *reinterpret_cast<const f32x4*>(&r.f[at_row]);
            sum = *reinterpret_cast<const f32x4*>(&r.sum[at_row]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = score[t][4 * e4 + e];
            if constexpr (kCodes) x = __builtin_fmaf(ks[t], x, kz[t] * sum[e]);
            float p = exp2_of(__builtin_fmaf(x, kCodes ? f[e] : a.scale, ls[e]));
            if (!all) {
              const int32_t hi = r.hi[at_row + e], lo = r.lo[at_row + e];
              p = tok <= hi && (tok > lo || tok < a.sinks) ? p : 0.0f;
            }
            part[e] += p;
          }
        }
        total[t] += (part[0] + part[1]) + (part[2] + part[3]);
      }
    }
    if (at + 1 < upto) leave(lds[(at + 1 - from) & 1]);
    __syncthreads();
  }

#pragma unroll
  for (int t = 0; t < kNT; ++t) {
    float sum = total[t] + __shfl_xor(total[t], 32);
    const int32_t tok = mine + 32 * t + n;
    if (!there[t]) sum = 0.0f;
    if (half == 0 && tok < g.kv_len) {
      if (a.part)
        a.part[((int64_t(split) * s.H + head) * s.num_seqs + seq) * s.max_kv + tok] = sum;
      else
        put(a, int64_t(seq) * a.seq_stride + int64_t(head) * a.head_stride + tok, sum);
    }
  }
}

// The parts of a token's weight together, in order.
__global__ __launch_bounds__(kThreads) void join_kernel(ServeArgs s, WeighArgs a, int32_t blocks) {
  const int32_t heads = a.joint ? 1 : s.H;
  uint32_t b = blockIdx.x;
  const int32_t block = int32_t(b % uint32_t(blocks));
  b /= uint32_t(blocks);
  const int32_t head = int32_t(b % uint32_t(heads)), seq = int32_t(b / uint32_t(heads));
  const int64_t tok = int64_t(block) * kThreads + threadIdx.x;
  const int32_t len = s.kv_lens[seq];
  if (tok >= (len < s.max_kv ? len : s.max_kv)) return;
  float sum = 0.0f;
  const int64_t step = int64_t(s.num_seqs) * s.max_kv;
  for (int32_t split = 0; split < a.splits; ++split)
    for (int32_t h = head; h < (a.joint ? s.H : head + 1); ++h)
      sum += a.part[(int64_t(split) * s.H + h) * step + int64_t(seq) * s.max_kv + tok];
  put(a, int64_t(seq) * a.seq_stride + int64_t(head) * a.head_stride + tok, sum);
}

template <bool BF16, int KB>
void launch(const ServeArgs& s, const WeighArgs& a, const WeighLaunch& l, hipStream_t stream) {
  auto few = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(uint32_t(l.groups)), dim3(64 * kFewWaves), 0, stream, s, a);
  };
  if (l.row_tiles) {
    const bool whole = s.log2P >= 4;
    if constexpr (D <= 128) {
      if (l.row_tiles > 1) {
        if (whole) few(few_kernel<BF16, KB, true, 2>);
        else few(few_kernel<BF16, KB, false, 2>);
        return;
      }
    }
    if (whole) few(few_kernel<BF16, KB, true, 1>);
    else few(few_kernel<BF16, KB, false, 1>);
    return;
  }
  hipLaunchKernelGGL((many_kernel<BF16, KB>), dim3(uint32_t(l.groups)), dim3(kThreads), 0, stream, s, a);
  if (l.join_groups)
    hipLaunchKernelGGL(join_kernel, dim3(uint32_t(l.join_groups)), dim3(kThreads), 0, stream, s, a,
                       int32_t(l.join_groups / ((a.joint ? 1 : s.H) * int64_t(s.num_seqs))));
}

}  // namespace

#define PKV_JOINED2(a, b) a##b
#define PKV_JOINED(a, b) PKV_JOINED2(a, b)

pkv_status_t PKV_JOINED(launch_weigh_, PKV_HEAD_DIM)(const ServeArgs& s, const WeighArgs& a, const WeighLaunch& l, hipStream_t stream) {
  switch (s.tag) {
    case PKV_TAG_FP16:
      if (s.bf16) launch<true, 16>(s, a, l, stream);
      else launch<false, 16>(s, a, l, stream);
      break;
    case PKV_TAG_K4V4: launch<false, 4>(s, a, l, stream); break;
    default: launch<false, 8>(s, a, l, stream); break;
  }
  return hipGetLastError() == hipSuccess ? PKV_OK : PKV_ERR_DEVICE;
}

}  // namespace pkv
