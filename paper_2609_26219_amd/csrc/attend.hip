// Attention over a paged cache (pkv_attention), for one head_dim
// (PKV_HEAD_DIM; built once for each of 64, 128 and 256).
//
// A row is a token of the call and one of the query heads that share a KV head, so
// that every cached row is loaded and decoded once for 16 of them or more.  A call of
// few rows a sequence (decode steps, drafts) cuts the tokens into pieces and each piece
// among a workgroup's waves; one of many (prompts, recomputed rows) gives
// every wave rows of its own and shares the tokens in LDS.  A wave keeps the running maximum and
// sum of the softmax, and what was cut is joined at the end: one pass over the cache.
//
// Few rows wait for the cache's bytes and, over codes, for their decoding as well: 32 ragged sequences (255 thousand tokens,
// 8 heads of 128, 4 query heads each) in 4 bits take 65 to 68 us, 4.1 to 4.3 TB/s where a large copy reaches 5.2, with the
// vector units busy 52% of it; over 16-bit pages 203 us, 5.1 TB/s, and with a window of 1024 21.4 us, 5.3 TB/s (its
// 113 MB partly in the 256 MB cache).
// Many rows over codes share their time between the vector units (the softmax, scales and zeros) and the matrix units, which
// two waves a SIMD seldom overlap: 2825 rows of 32 heads behind up to 10240 tokens in 8 and 4 bits run at 681 TFLOP/s,
// vector units busy 62%, matrix units 27%, LDS 32%.  Over 16 bits no unit is busy half of the time (1229 scattered rows
// over 32768 tokens: 675 to 689 TFLOP/s, 42%, 29%, 27%): two waves a SIMD do not cover each other's waits, and 250 of 256
// registers leave no room for a third or for work of the next tile.  A large library product in bfloat16 reaches 1235.
// At 256 channels the kernels over 16 bits spill registers (many rows 21, few rows 42,
// 74 with pages below 16 slots): 2825 rows 571 TFLOP/s against 770 at 128 channels, a decode step 4.5 TB/s.
//
// For its tile a wave computes S^T = K Q^T and then O^T += V^T P^T with
// 16x16x32 matrix instructions.  With lane l = (c = l / 16, x = l % 16):
//   K operand    row x = token, channels c*D/4 + 8i.. of instruction i: a lane
//                loads D/4 consecutive channels of one token;
//   Q operand    column x = row of the tile, the same channels, in the order
//                in which the decoder leaves a word's codes;
//   S^T          column x = row, tokens 4c + 0..3: every lane has its row's scores
//                for 4 tokens of each 16, so maxima, sums and rescaling are
//                the lane's own but for one exchange between the four c;
//   P^T operand  column x = row, the lane's 8 tokens of both halves of the tile:
//                the same registers, rounded and packed, with no exchange;
//   V^T operand  row x = channel x*D/16 + j of instruction j, the same 8 tokens: a
//                lane loads D/16 consecutive channels of 8 tokens and transposes
//                them in registers as it decodes them;
//   O^T          column x = row, channels (4c + 0..3)*D/16 + j.
//
// Codes go into the matrix instructions as the integers code - 2^(bits-1), exact in binary16, and a
// token's scale s and zero z act outside: with z' = z + 2^(bits-1) s,
//   q . k_t = s_t (q . codes_t) + z'_t sum(q),
//   sum_t p_t v_t = sum_t (p_t s_t) codes_t + sum_t p_t z'_t,
// so the one rounding on the way is p_t s_t to binary16 (scaled by a power of
// two that keeps the largest near 2^14, so that small scales lose nothing).  Where a row's outliers put mid-code far
// from its other channels, that rounding costs more than a binary16 result's own (4.5e-4 of a result in all, 2.0e-4
// without it) and is lost in a bfloat16 one's (1.6e-3): for binary16 results p_t s_t goes in as two binary16 numbers, the
// second what the first leaves.
// Queries go in as binary16 too, each row scaled by a power of two.  16-bit caches use the
// matrix instructions of their own type, p_t rounded to it: 2.2e-3 of a bfloat16 result in all, 1.5e-4 to 2.9e-4 of a
// binary16 one (1.65e-3, and 1.2e-4 to 2.1e-4, are the result's own rounding).  With two numbers there as well, 8192 rows
// with a window take 283 us instead of 240 and 1229 scattered rows 610 instead of 510, and an infinite value that a row
// sees becomes NaN, the sum of both numbers' products with it, where one number keeps it.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pkv.h"
#include "paged_tiles.h"
#include "pkv_internal.h"
#include "serve.h"

namespace pkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kQkSteps = D / 32;  // matrix instructions of one S^T

struct Span {  // of a row tile, over its rows
  int32_t hi_most, hi_least, lo_most, lo_least;
  int32_t sink_tiles, first, tiles;  // tiles of tokens to look at: the sinks', then those from token `first` on
};

// The running softmax of a wave over its rows (lane: row x of each of RT row tiles).
template <int RT>
struct Running {
  f32x4 o[RT][kChannels];
  float ref[RT];  // exponents (base 2) are taken relative to it; -inf at first
  float l[RT], o_zero[RT];
};

// The operand P (times the token's value scale, where the cache holds codes) has to fit
// binary16 with room below, so the reference is chosen that the largest p (times scale) so far is
// 2^kTop, and moved only when one passes that by kSlack (binary16 ends at 2^16): O is then rescaled once or
// twice a row and not at every new maximum, of which 32 rows have one in nearly every tile.  A
// scale counts as at least 2^-24, binary16's least.  bfloat16 needs no room: kTop = 0.  (The largest score and the largest
// scale of several tokens will not do: where a token of large scale is seen little of or not at all, the others'
// probabilities would lose their bits, 2% of a result with scales 2^24 apart and all of it with 2^30.)
constexpr float kSlack = 8.0f;
template <bool HALF>
constexpr float kTop = HALF ? 6.0f : 0.0f;

// What stands for a token beside its codes, for the lane's 4 tokens of each half of a tile: key scale and zero, value
// scale and zero at mid-code.  As the cache has it, or as numbers.
template <int VB>
struct WordScales {
  u32x4 k[2], v[2];
  __device__ float ks(int u, int i) const { return f16_float(k[u][i]); }
  __device__ float kz(int u, int i) const { return f16_float(k[u][i] >> 16); }
  __device__ float vs(int u, int i) const { return f16_float(v[u][i]); }
  __device__ float vz(int u, int i) const {
    return __builtin_fmaf(f16_float(v[u][i]), float(1 << (VB - 1)), f16_float(v[u][i] >> 16));
  }
  __device__ void hide(int u, int i) { v[u][i] = 0; }
};
struct FloatScales {
  f32x4 ks_[2], kz_[2], vs_[2], vz_[2];
  __device__ float ks(int u, int i) const { return ks_[u][i]; }
  __device__ float kz(int u, int i) const { return kz_[u][i]; }
  __device__ float vs(int u, int i) const { return vs_[u][i]; }
  __device__ float vz(int u, int i) const { return vz_[u][i]; }
  __device__ void hide(int u, int i) { vs_[u][i] = vz_[u][i] = 0.0f; }
};

// The first row x of each of a wave's RT row tiles: what it sees and its queries.
template <int RT>
struct Rows {
  Sight see[RT];
  u32x4 q[RT][kQkSteps];
  float q_sum[RT], f[RT];
};

// One tile of 32 tokens from t0 on, of which the lane's are `there` (bit 4u + i: t0 + 16u + 4c + i).
// key(u, i) and value(j) give the operands, after_keys() runs when the last key has been used, hide(keep) leaves of
// 16-bit values only the halves of operand words that `keep` has.
template <bool BF16, int KB, int VB, int RT, typename Scales, typename Key, typename Value, typename After, typename Hide>
__device__ __forceinline__ void attend_tile(const AttendArgs& a, const Span& span, const Rows<RT>& rows, int c,
                                            int32_t t0, uint32_t there, Scales& sc, Running<RT>& st, Key key,
                                            Value value, After after_keys, Hide hide) {
  constexpr bool kCodes = KB != 16;
  constexpr bool kHalf = kCodes || !BF16;  // operands in binary16
  constexpr bool kFine = kCodes && !BF16;
  const bool all = t0 + kTokenTile - 1 <= span.hi_least && (span.lo_most < t0 || t0 + kTokenTile <= a.sinks) &&
                   __all(there == 0xFFu);
  auto mfma = [](const u32x4& x, const u32x4& y, const f32x4& z) {
    if constexpr (kHalf)
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), z, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), z, 0, 0, 0);
  };
  // S^T, in units of 1 / f.  (Codes: their centre times sum(q) to begin with, so that it is of the codes themselves.)
  f32x4 t[RT][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float first = kCodes ? rows.q_sum[r] * float(1 << (KB - 1)) : 0.0f;
      t[r][u] = f32x4{first, first, first, first};
    }
#pragma unroll
    for (int i = 0; i < kQkSteps; ++i) {
      const u32x4 k = key(u, i);
#pragma unroll
      for (int r = 0; r < RT; ++r) t[r][u] = mfma(k, rows.q[r][i], t[r][u]);
    }
  }
  after_keys();
  if constexpr (kCodes) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          t[r][u][i] = __builtin_fmaf(sc.ks(u, i), t[r][u][i], sc.kz(u, i) * rows.q_sum[r]);
  }
  if (!all) {
    u32x4 keep{};
    // A row's score where it does not see; the values of tokens that no row of the wave sees, whatever lies there.
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t tok = t0 + 16 * u + 4 * c + i;
        const bool is = (there >> (4 * u + i)) & 1;
        bool any = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const bool sees = is && tok <= rows.see[r].hi && (tok > rows.see[r].lo || tok < a.sinks);
          t[r][u][i] = sees ? t[r][u][i] : -kInf;
          any |= sees;
        }
        any = (__ballot(any) >> (16 * c)) & 0xFFFF;
        if constexpr (kCodes) {
          if (!any) sc.hide(u, i);
        } else {
          keep[2 * u + i / 2] |= any ? 0xFFFFu << (16 * (i & 1)) : 0;
        }
      }
    if constexpr (!kCodes) hide(keep);
  }
  // The reference of the exponents.  Over codes it goes by score + log2(scale) of each token; that it stays is decided by
  // the lane's largest score and its largest scale, which are no less and take one logarithm.
  float above = -kTop<kHalf>;
  if constexpr (kCodes) {
    float most = 0x1p-24f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = __builtin_fmaxf(most, sc.vs(u, i));
    above += __builtin_amdgcn_logf(most);
  }
  float top[RT];
  bool move = false;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    top[r] = t[r][0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) top[r] = __builtin_fmaxf(top[r], t[r][u][i]);
    top[r] = __builtin_fmaf(top[r], rows.f[r], above);
    move |= top[r] > st.ref[r] + kSlack;
  }
  if (__any(move)) {
    if constexpr (kCodes) {
#pragma unroll
      for (int r = 0; r < RT; ++r) top[r] = -kInf;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float bits = __builtin_amdgcn_logf(__builtin_fmaxf(sc.vs(u, i), 0x1p-24f)) - kTop<kHalf>;
#pragma unroll
          for (int r = 0; r < RT; ++r) top[r] = __builtin_fmaxf(top[r], __builtin_fmaf(t[r][u][i], rows.f[r], bits));
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float next = over_c_max(top[r]);
      next = next > st.ref[r] ? next : st.ref[r];
      const float shrink = st.ref[r] == -kInf ? 0.0f : exp2_of(st.ref[r] - next);
      st.ref[r] = next;
      st.l[r] *= shrink;
      st.o_zero[r] *= shrink;
#pragma unroll
      for (int j = 0; j < kChannels; ++j) st.o[r][j] *= shrink;
    }
  }
  // The probabilities and their sum.
  u32x4 pt[RT], rest[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float base = st.ref[r] == -kInf ? 0.0f : -st.ref[r];
    float pr[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pr[u][i] = exp2_of(__builtin_fmaf(t[r][u][i], rows.f[r], base));
        st.l[r] += pr[u][i];
        if constexpr (kCodes) {
          st.o_zero[r] = __builtin_fmaf(pr[u][i], sc.vz(u, i), st.o_zero[r]);
          pr[u][i] *= sc.vs(u, i);
        }
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t w = kHalf ? pack_f16(pr[u][2 * i], pr[u][2 * i + 1]) : pack_bf16(pr[u][2 * i], pr[u][2 * i + 1]);
        pt[r][2 * u + i] = w;
        if constexpr (kFine) rest[r][2 * u + i] = pack_f16(pr[u][2 * i] - f16_float(w), pr[u][2 * i + 1] - f16_float(w >> 16));
      }
  }
#pragma unroll
  for (int j = 0; j < kChannels; ++j) {
    const u32x4 v = value(j);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      st.o[r][j] = mfma(v, pt[r], st.o[r][j]);
      if constexpr (kFine) st.o[r][j] = mfma(v, rest[r], st.o[r][j]);
    }
  }
}

// The rows of a call that a workgroup shares: one sequence's, of one KV head.
struct Group : SequenceRows {
  int32_t head, split, tile, seq;
};

__device__ __forceinline__ Group group_from(const ServeArgs& s, int32_t start, int32_t end, int32_t kv_len) {
  return Group{rows_of_sequence(s, start, end, kv_len), 0, 0, 0, 0};
}

__device__ __forceinline__ Group group_of_sequence(const ServeArgs& s, int32_t seq) {
  Group g = group_from(s, scalar_entry(s.token_start, seq), scalar_entry(s.token_start, seq + 1),
                       scalar_entry(s.kv_lens, seq));
  g.seq = seq;
  return g;
}

// Of a launch of splits x row tiles x heads for each sequence.
__device__ __forceinline__ Group group_of(const ServeArgs& s, const AttendArgs& a) {
  uint32_t b = blockIdx.x;
  const int32_t head = int32_t(b % uint32_t(s.H));
  b /= uint32_t(s.H);
  const int32_t split = int32_t(b % uint32_t(a.splits));
  b /= uint32_t(a.splits);
  Group g = group_of_sequence(s, int32_t(b / uint32_t(a.row_tiles)));
  g.head = head;
  g.split = split;
  g.tile = a.row_tiles - 1 - int32_t(b % uint32_t(a.row_tiles));  // the rows that see the most start first
  return g;
}

// Rows row0 + 16 r + x of the group: what they see (and the lane's part of the span) and their queries in the
// operands' order, 8 channels from first(i) on in instruction i.
template <int KB, int RT, typename First>
__device__ __forceinline__ void load_rows(const ServeArgs& s, const AttendArgs& a, const Group& g, uint32_t row0, int x,
                                          First first, Rows<RT>& rows, Span& span) {
  constexpr bool kCodes = KB != 16;
  span = Span{-1, 0x7FFFFFFF, -1, 0x7FFFFFFF, 0, 0, 0};
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const uint32_t row = row0 + kRowTile * r + x;
    const int32_t token = int32_t(row / uint32_t(a.group)), sub = int32_t(row % uint32_t(a.group));
    const bool on = token < g.count;
    Sight see{-1, -1};
    if (on) {
      const int32_t pos = s.positions ? s.positions[g.start + token] : g.kv_len - g.trail + token;
      see.hi = pos < g.kv_len ? pos : g.kv_len - 1;
      see.hi = see.hi < -1 ? -1 : see.hi;
      see.lo = a.window > 0 && pos >= a.window ? pos - a.window : -1;
      span.hi_least = span.hi_least < see.hi ? span.hi_least : see.hi;
      if (see.hi >= 0 && see.lo < span.lo_least) span.lo_least = see.lo;
    }
    span.hi_most = span.hi_most > see.hi ? span.hi_most : see.hi;
    span.lo_most = span.lo_most > see.lo ? span.lo_most : see.lo;
    rows.see[r] = see;

    rows.q_sum[r] = 0.0f;
    rows.f[r] = a.scale;
    const uint16_t* from = a.q + int64_t(g.start + token) * a.q_token_stride +
                           int64_t(g.head * a.group + sub) * a.q_head_stride;
    float v[kQkSteps][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kQkSteps; ++i) {
      u32x4 w{};
      if (on) w = *reinterpret_cast<const u32x4*>(from + first(i));
      if constexpr (!kCodes) {
        rows.q[r][i] = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t bits = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xFFFF;
          v[i][e] = s.bf16 ? bf16_float(bits) : f16_float(bits);
          const uint32_t mag = __float_as_uint(v[i][e]) & 0x7FFFFFFF;
          top = top > mag ? top : mag;
        }
      }
    }
    if constexpr (kCodes) {
      top = max(top, uint32_t(__shfl_xor(int(top), 16)));
      top = max(top, uint32_t(__shfl_xor(int(top), 32)));
      // 2^-e with 2^e <= |q| < 2^(e + 1): the largest becomes 1..2 and S is scaled back by 2^e in f.
      int e = int(top >> 23) - 127;
      e = e < -60 ? -60 : e > 120 ? 120 : e;  // f stays a normal number
      const float down = __uint_as_float(uint32_t(127 - e) << 23);
      rows.f[r] *= __uint_as_float(uint32_t(127 + e) << 23);
#pragma unroll
      for (int i = 0; i < kQkSteps; ++i) {
#pragma unroll
        for (int p = 0; p < 4; ++p)
          rows.q[r][i][p] = pack_f16(v[i][k_channel<KB>(p, 0)] * down, v[i][k_channel<KB>(p, 1)] * down);
#pragma unroll
        for (int e2 = 0; e2 < 8; ++e2) rows.q_sum[r] += v[i][e2] * down;
      }
      rows.q_sum[r] = over_c_sum(rows.q_sum[r]);
    }
  }
  span.hi_most = __builtin_amdgcn_readfirstlane(over_x_max(span.hi_most));
  span.hi_least = __builtin_amdgcn_readfirstlane(over_x_min(span.hi_least));
  span.lo_most = __builtin_amdgcn_readfirstlane(over_x_max(span.lo_most));
  span.lo_least = __builtin_amdgcn_readfirstlane(over_x_min(span.lo_least));
}

// The tiles of TOKENS tokens that some row of a span sees, and the first and the end of a split's share.
template <int TOKENS>
__device__ __forceinline__ void tiles_of(const AttendArgs& a, int32_t split, Span& span, int32_t& from, int32_t& upto) {
  span.first = span.sink_tiles = span.tiles = 0;
  if (span.hi_most >= 0) {
    span.first = (span.lo_least + 1) & ~(TOKENS - 1);
    const int32_t sinks = a.sinks < span.hi_most + 1 ? a.sinks : span.hi_most + 1;
    span.sink_tiles = (sinks + TOKENS - 1) / TOKENS;
    span.sink_tiles = span.sink_tiles < span.first / TOKENS ? span.sink_tiles : span.first / TOKENS;
    // (a position past kv_lens may leave a row its sinks alone)
    span.tiles = span.sink_tiles + (span.hi_most >= span.first ? (span.hi_most - span.first) / TOKENS + 1 : 0);
  }
  int32_t share = (span.tiles + a.splits - 1) / a.splits;
  share = share > a.chunk ? share : a.chunk;
  const int64_t begin = int64_t(split) * share;
  from = int32_t(begin < span.tiles ? begin : span.tiles);
  upto = int32_t(begin + share < span.tiles ? begin + share : span.tiles);
}

template <int TOKENS>
__device__ __forceinline__ int32_t tile_at(const Span& span, int32_t it) {
  return it < span.sink_tiles ? it * TOKENS : span.first + (it - span.sink_tiles) * TOKENS;
}

template <int RT>
__device__ __forceinline__ void begin(Running<RT>& st) {
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    st.ref[r] = -kInf;
    st.l[r] = st.o_zero[r] = 0.0f;
#pragma unroll
    for (int j = 0; j < kChannels; ++j) st.o[r][j] = f32x4{};
  }
}

__device__ __forceinline__ float inverse(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }
// Log-sum-exp from the reference (base 2) and the sum relative to it.
__device__ __forceinline__ float lse_of(float ref, float l) {
  return l == 0.0f ? -kInf : (ref + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// ---- Few rows ----
//
// A sequence's rows of one KV head fit one row tile or two.  Its tiles of tokens are cut into even pieces, one to a
// workgroup and head: as many pieces for each sequence as make the longest piece of all shortest, with as many workgroups
// as run at once, so that sequences of any lengths keep the whole GPU busy to the end.  Every workgroup
// works the pieces out from the lengths, which only the device knows.

// What a sequence's rows look at, without the queries: a span that bounds the rows' own.  (Positions are
// read only where there is a window: 32 sequences, a window of 1024 over 16 bits, a row anywhere in each 24 + 7 us instead
// of 203 + 8, two rows 97 + 10 instead of 210 + 9.)
__device__ __forceinline__ Span few_span(const ServeArgs& s, const AttendArgs& a, const Group& g) {
  Span span{-1, 0, -1, -1, 0, 0, 0};
  if (s.positions && a.window > 0) {
    span.lo_least = 0x7FFFFFFF;
    for (int32_t i = 0; i < g.count; ++i) {
      const int32_t pos = s.positions[g.start + i], hi = pos < g.kv_len ? pos : g.kv_len - 1;
      if (hi < 0) continue;
      const int32_t lo = pos >= a.window ? pos - a.window : -1;
      span.hi_most = span.hi_most > hi ? span.hi_most : hi;
      span.lo_least = span.lo_least < lo ? span.lo_least : lo;
    }
  } else if (s.positions) {
    span.hi_most = g.kv_len - 1;
  } else {
    const int32_t pos0 = g.kv_len - g.trail;
    span.hi_most = pos0 + g.count - 1;
    const int32_t first = pos0 > 0 ? pos0 : 0;
    span.lo_least = a.window > 0 && first >= a.window ? first - a.window : -1;
  }
  int32_t from, upto;
  tiles_of<kTokenTile>(a, 0, span, from, upto);
  return span;
}

// Tiles of a sequence, or -1 if it has no rows.
__device__ __forceinline__ int32_t tiles_of_sequence(const ServeArgs& s, const AttendArgs& a, int32_t seq) {
  if (seq >= s.num_seqs) return -1;
  const Group g = group_from(s, s.token_start[seq], s.token_start[seq + 1], s.kv_lens[seq]);
  return g.count > 0 ? few_span(s, a, g).tiles : -1;
}
__device__ __forceinline__ int32_t pieces_of(int32_t tiles, int32_t per) {
  return tiles < 0 ? 0 : tiles == 0 ? 1 : (tiles - 1) / per + 1;
}

// Inclusive sums over the lanes of a wave, and the sum of all.
template <typename T>
__device__ __forceinline__ T wave_sums(T v, int lane) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T other = __shfl_up(v, off);
    v += lane >= off ? other : 0;
  }
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) v += __shfl_xor(v, off);
  return v;
}

// Tiles of the longest piece, by every wave for itself.  `mine`: the tiles of sequence `lane`.  With p pieces wanted, total / p is
// the least that could do and total / (p - sequences) surely does; up to 64 sequences the least that does is found
// between them.
__device__ __forceinline__ int32_t piece_tiles(const ServeArgs& s, const AttendArgs& a, int lane, int32_t mine) {
  int64_t total = 0;
  int32_t rows = 0;
  for (int32_t first = 0; first < s.num_seqs; first += 64) {
    const int32_t tiles = first ? tiles_of_sequence(s, a, first + lane) : mine;
    total += tiles > 0 ? tiles : 0;
    rows += __popcll(__ballot(tiles >= 0));
  }
  total = wave_sum(total);
  int64_t low = (total + a.pieces - 1) / a.pieces, high = (total + a.pieces - rows - 1) / (a.pieces - rows);
  low = low > a.chunk ? low : a.chunk;
  high = high > a.chunk ? high : a.chunk;
  if (s.num_seqs <= 64) {
    for (int step = 0; step < 6 && low < high; ++step) {
      const int64_t middle = (low + high) / 2;
      if (wave_sum(pieces_of(mine, int32_t(middle))) <= a.pieces)
        high = middle;
      else
        low = middle + 1;
    }
  }
  return __builtin_amdgcn_readfirstlane(int32_t(high));
}

// The first sequence, with sequence `first` + lane's tiles, for which found(lanes' inclusive sums of pieces, tiles) holds in
// some lane: its number, the pieces before it and its tiles; -1 if there is none.
struct Found {
  int32_t seq, before, tiles;
};
template <typename Test>
__device__ __forceinline__ Found find_sequence(const ServeArgs& s, const AttendArgs& a, int lane, int32_t mine, int32_t per,
                                               Test test) {
  int32_t before = 0;
  for (int32_t first = 0; first < s.num_seqs; first += 64) {
    const int32_t tiles = first ? tiles_of_sequence(s, a, first + lane) : mine;
    const int32_t own = pieces_of(tiles, per), sums = before + wave_sums(own, lane);
    const uint64_t hit = __ballot(test(first + lane, sums, own));
    if (hit) {
      const int at = __builtin_ctzll(hit);
      return Found{first + at, __builtin_amdgcn_readlane(sums - own, at), __builtin_amdgcn_readlane(tiles, at)};
    }
    before = __builtin_amdgcn_readlane(sums, 63);
  }
  return Found{-1, 0, 0};
}

template <int RT>
struct FewLds {
  float join_ml[kWaves][kRowTile][2];
  float join[kWaves][kRowTile][D + 4];
  u32x4 words[kWaves][16];
};

// Tiles [from, upto) of a sequence and head, into `out` and `lse` if they are all of them, else as part `part_slot`.
template <bool BF16, int KB, int VB, bool WHOLE, int RT>
__device__ __forceinline__ void few_piece(const ServeArgs& s, const AttendArgs& a, const Group& g, int32_t from,
                                          int32_t upto, int64_t part_slot, const Magic& code, FewLds<RT>& m) {
  constexpr bool kCodes = KB != 16;
  const int lane = threadIdx.x & 63, c = lane >> 4, x = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t row0 = g.tile * (kRowTile * RT);
  if (row0 >= g.count * a.group) return;  // the whole workgroup
  const Span looks = few_span(s, a, g);
  const Source f = source_of<KB>(s, g.seq, g.head);
  // The wave's tiles are `from` + wave + kWaves n.  Their pages are looked up 32 tiles at a time, a half of a tile to
  // a lane, and read from there: a scalar load for each tile would have every wait for LDS wait for it too.
  const int32_t first = from + wave, count = first < upto ? (upto - first + kWaves - 1) / kWaves : 0;
  auto pages_from = [&](int32_t n) -> int32_t {
    if constexpr (!WHOLE) return -1;
    const int32_t it = first + (n + (lane >> 1)) * kWaves;
    return it < upto ? page_of(s, f.table, (tile_at<kTokenTile>(looks, it) + 16 * (lane & 1)) >> s.log2P) : -1;
  };
  auto tile_of = [&](int32_t n, int32_t pages) {
    const int at = (n & 31) * 2;
    return Tile{tile_at<kTokenTile>(looks, first + n * kWaves),
                {__builtin_amdgcn_readlane(pages, at), __builtin_amdgcn_readlane(pages, at + 1)}};
  };
  // The first tile is asked for before the queries are.
  Keys<KB> keys;
  Values<VB> values;
  uint32_t scale = 0;
  int32_t pages = -1;
  Tile tile{};
  if (count > 0) {
    pages = pages_from(0);
    tile = tile_of(0, pages);
    load_keys<KB, WHOLE>(s, f, tile, c, x, keys);
    load_values<VB, WHOLE>(s, f, tile, c, x, values);
    if constexpr (kCodes) scale = load_scale<WHOLE>(s, f, tile, lane);
  }
  Rows<RT> rows;
  Span span;
  load_rows<KB, RT>(s, a, g, uint32_t(row0), x, [&](int i) { return k_first<KB>(i, c); }, rows, span);
  Running<RT> st;
  begin(st);
  if (count > 0) {
    // A tile's registers are filled again, keys and then values, as soon as its own have been used.
    for (int32_t n = 0; n < count; ++n) {
      const bool more = n + 1 < count;
      if (((n + 1) & 31) == 0) pages = pages_from(n + 1);
      const Tile next = tile_of(n + 1, pages);
      const uint32_t there = tokens_there<WHOLE>(s, f, tile, c);
      // Through LDS, where each lane finds the words of its 4 tokens of each half (the wave's own: no barrier).
      WordScales<VB> sc;
      if constexpr (kCodes) {
        reinterpret_cast<uint32_t*>(m.words[wave])[lane] = scale;
        sc.k[0] = m.words[wave][c];
        sc.k[1] = m.words[wave][4 + c];
      }
      attend_tile<BF16, KB, VB, RT>(
          a, span, rows, c, tile.t0, there, sc, st, [&](int u, int i) { return k_operand<KB>(code, keys.w[u], i); },
          [&](int j) {
            u32x4 v;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 2; ++i)
                v[2 * u + i] = v_pair<VB>(code, values.w[u][2 * i], values.w[u][2 * i + 1], j);
            return v;
          },
          [&] {
            if (more) load_keys<KB, WHOLE>(s, f, next, c, x, keys);
            if constexpr (kCodes) {
              sc.v[0] = m.words[wave][8 + c];
              sc.v[1] = m.words[wave][12 + c];
              if (more) scale = load_scale<WHOLE>(s, f, next, lane);
            }
          },
          [&](const u32x4& keep) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < Values<VB>::kWords; ++w)
                  values.w[u][i][w] = (keep[2 * u + i / 2] >> (16 * (i & 1))) & 1 ? values.w[u][i][w] : 0;
          });
      if (more) load_values<VB, WHOLE>(s, f, next, c, x, values);
      tile = next;
    }
  }

  // Join the waves, a row tile at a time: every one's sums relative to the largest reference.  A wave whose tokens a row
  // does not see has l = 0; one that sees NaN alone keeps its reference at -inf, and its l is NaN.
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = over_c_sum(st.l[r]), ref = st.ref[r];
    const float o_zero = kCodes ? over_c_sum(st.o_zero[r]) : 0.0f;
    __syncthreads();
    if (c == 0) {
      m.join_ml[wave][x][0] = ref;
      m.join_ml[wave][x][1] = l;
    }
    __syncthreads();
    float all = -kInf;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all = __builtin_fmaxf(all, m.join_ml[w][x][0]);
    const float part = exp2_of(ref - all);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kChannels; ++j)
        m.join[wave][x][(4 * c + i) * kChannels + j] = l == 0.0f ? 0.0f : (st.o[r][j][i] + o_zero) * part;
    __syncthreads();
    constexpr int kPerRow = kThreads / kRowTile, kPer = D / kPerRow;  // 16 threads to a row
    const int y = threadIdx.x / kPerRow, at = (threadIdx.x % kPerRow) * kPer;
    const uint32_t row = row0 + kRowTile * r + y;
    const int32_t token = int32_t(row / uint32_t(a.group));
    if (token >= g.count) continue;
    const int32_t out_head = g.head * a.group + int32_t(row % uint32_t(a.group));
    float mm = -kInf, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mm = __builtin_fmaxf(mm, m.join_ml[w][y][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      ll += m.join_ml[w][y][1] == 0.0f ? 0.0f : m.join_ml[w][y][1] * exp2_of(m.join_ml[w][y][0] - mm);
    float sum[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      sum[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum[e] += m.join[w][y][at + e];
    }
    if (part_slot >= 0) {
      const int64_t slot = part_slot * a.part_rows + row;
#pragma unroll
      for (int e = 0; e < kPer; e += 4)
        *reinterpret_cast<f32x4*>(a.part + slot * D + at + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
      if (at == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * slot) = f32x2{mm, ll};
      continue;
    }
    const float inv = inverse(ll);
    uint32_t word[kPer / 2];
#pragma unroll
    for (int e = 0; e < kPer; e += 2)
      word[e / 2] = s.bf16 ? pack_bf16(sum[e] * inv, sum[e + 1] * inv) : pack_f16(sum[e] * inv, sum[e + 1] * inv);
    uint16_t* to = a.out + int64_t(g.start + token) * a.out_token_stride + int64_t(out_head) * a.out_head_stride + at;
#pragma unroll
    for (int e = 0; e < kPer / 2; e += 2) *reinterpret_cast<u32x2*>(to + 2 * e) = u32x2{word[e], word[e + 1]};
    if (a.lse && at == 0) a.lse[int64_t(g.start + token) * a.Hq + out_head] = lse_of(mm, ll);
  }
}

// The four waves of a workgroup share the rows and deal the piece's tiles among themselves.  Each lane's pieces of the cache
// go from memory to its registers and, decoded, straight into the matrix instructions.
template <bool BF16, int KB, int VB, bool WHOLE, int RT>
__global__ __launch_bounds__(kThreads, 2) void attend_few_kernel(ServeArgs s, AttendArgs a) {
  __shared__ __attribute__((aligned(16))) FewLds<RT> m;
  const int lane = threadIdx.x & 63;
  const Magic code = magic();
  uint32_t piece = blockIdx.x / uint32_t(s.H);
  const int32_t head = int32_t(blockIdx.x % uint32_t(s.H)), tile = int32_t(piece % uint32_t(a.row_tiles));
  piece /= uint32_t(a.row_tiles);
  if (a.pieces == 0) {  // a sequence to a workgroup, head and row tile
    Group g = group_of_sequence(s, int32_t(piece));
    g.head = head;
    g.tile = tile;
    if (g.count > 0) few_piece<BF16, KB, VB, WHOLE, RT>(s, a, g, 0, few_span(s, a, g).tiles, -1, code, m);
    return;
  }
  const int32_t mine = tiles_of_sequence(s, a, lane), per = piece_tiles(s, a, lane, mine);
  const Found at = find_sequence(s, a, lane, mine, per, [&](int32_t, int32_t sums, int32_t own) {
    return own > 0 && sums > int32_t(piece);
  });
  if (at.seq < 0) return;
  Group g = group_of_sequence(s, at.seq);
  g.head = head;
  g.tile = tile;
  const int32_t pieces = pieces_of(at.tiles, per), share = (at.tiles + pieces - 1) / pieces;
  const int32_t from = (int32_t(piece) - at.before) * share;
  few_piece<BF16, KB, VB, WHOLE, RT>(s, a, g, from, from + share < at.tiles ? from + share : at.tiles,
                                     pieces == 1 ? -1 : int64_t(piece) * s.H + head, code, m);
}

// Many rows: each wave has 32 of its own (16 at 256 channels), and the workgroup's four share the cache through LDS.  A tile of
// kManyTokens tokens (64 at 128 channels: 16 KiB of keys, 16 of values, in binary16 or the cache's type) is decoded
// once for all of them and lies in LDS as the matrix operands want it, 16 bytes to a lane; two tiles take
// turns, the next one's loads in flight while one is computed, with one barrier to a tile.  Eight waves of 16 rows
// read LDS twice as much: 975 us instead of 603 over codes, 628 instead of 582 over 16 bits.  The operands are read where
// they are used: held ahead they spill registers (661 us over codes).
constexpr int kManyTokens = kManyElems / D;
constexpr int kManyRows = kRowTile * many_tiles(D) / kWaves;  // of a wave
constexpr int kOperand = 64;  // 16-byte pieces of one operand of a wave

template <int KB, int VB>
struct ManyLds {
  u32x4 k[2][kManyElems / 8];
  u32x4 v[2][kManyElems / 8];
  f32x4 scale[2][4][KB != 16 ? kManyTokens / 4 : 1];  // ks, kz, vs, vz
  int64_t k_off[2][kManyTokens];                  // bytes from the layer's first key (code) to the token's row of this head
  int64_t v_off[2][KB != 16 ? kManyTokens : 1];
  int64_t s_off[2][KB != 16 ? kManyTokens : 1];   // words to its key scale
  uint64_t there[4][2];                           // (written two tiles ahead, while a tile's own is read)
  int32_t span[kWaves][4];
};

template <bool BF16, int KB, int VB>
__global__ __launch_bounds__(kThreads, 2) void attend_many_kernel(ServeArgs s, AttendArgs a) {
  constexpr bool kCodes = KB != 16;
  constexpr int RT = kManyRows / kRowTile;
  __shared__ __attribute__((aligned(16))) ManyLds<KB, VB> m;

  const Group g = group_of(s, a);
  const int tid = threadIdx.x, lane = tid & 63, c = lane >> 4, x = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t group_row0 = int64_t(g.tile) * (kManyRows * kWaves);
  if (group_row0 >= int64_t(g.count) * a.group) return;  // the whole workgroup
  const uint32_t row0 = uint32_t(group_row0) + wave * kManyRows;
  Rows<RT> rows;
  Span mine;
  load_rows<KB, RT>(s, a, g, row0, x, [&](int i) { return 32 * i + 8 * c; }, rows, mine);
  if (lane == 0) {
    m.span[wave][0] = mine.hi_most;
    m.span[wave][1] = mine.lo_least;
  }
  __syncthreads();
  Span span = mine;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    span.hi_most = span.hi_most > m.span[w][0] ? span.hi_most : m.span[w][0];
    span.lo_least = span.lo_least < m.span[w][1] ? span.lo_least : m.span[w][1];
  }
  int32_t from, upto;
  tiles_of<kManyTokens>(a, g.split, span, from, upto);
  from = __builtin_amdgcn_readfirstlane(from);
  upto = __builtin_amdgcn_readfirstlane(upto);

  const int32_t* table = s.page_table + int64_t(g.seq) * s.pages_per_seq;
  // Where the tokens of a tile lie; a token that is not there is read from page 0.  (More threads than tokens: the
  // others repeat them.)
  const int own = tid & (kManyTokens - 1);
  auto entry_of = [&](int32_t it) -> int32_t {
    const int32_t at = (tile_at<kManyTokens>(span, it) + own) >> s.log2P;
    return table[at < s.pages_per_seq ? at : s.pages_per_seq - 1];
  };
  auto put_places = [&](int32_t it, int32_t entry) {
    const int b = it & 1;
    const int32_t t = tile_at<kManyTokens>(span, it) + own;
    const bool is = entry >= 0 && entry < s.pool_pages && (t >> s.log2P) < s.pages_per_seq;
    const uint64_t there = __ballot(is);
    if (lane == 0) m.there[it & 3][wave & 1] = there;  // (one lane: 64 writes to one place take 64 turns)
    const int64_t slot = t & ((1 << s.log2P) - 1), page = is ? entry : 0;
    if constexpr (kCodes) {
      const int64_t at = page * s.page_stride + g.head * s.head_stride;
      m.k_off[b][own] = at + slot * (D * KB / 8);
      m.v_off[b][own] = at + s.v_offset + slot * (D * VB / 8);
      m.s_off[b][own] = page * s.scale_stride + ((int64_t(g.head) * 2) << s.log2P) + slot;
    } else {
      m.k_off[b][own] = 2 * (page * s.page_stride + slot * s.H * D + g.head * D);
    }
  };
  const Magic code = magic();
  // A thread's share of a tile: 32 values (8 tokens x 4 channels), 32 keys (32 channels of a token in codes, four times 8 in
  // 16 bits) and, in codes, the scales of a token.
  constexpr int kPairs = D / 32, kVPiece = VB / 2, kVWords = (kVPiece + 3) / 4;
  uint32_t raw_k[kCodes ? KB : 16], raw_v[8][kVWords], raw_scale[2];
  const int v_piece = tid % (D / 4), v_tokens = tid / (D / 4);  // tokens 32 (v_tokens / 4) + {0, 16} + 4 (v_tokens % 4) + 0..3
  const int k_token = tid / 16 / kPairs * 16 + tid % 16, k_step = tid / 16 % kPairs;  // of codes
  auto bring = [&](int32_t it) {
    const int b = it & 1;
    if constexpr (kCodes) {
      load_bytes<4 * KB>(raw_k, s.codes + m.k_off[b][k_token] + k_step * (4 * KB));
      raw_scale[0] = s.scales[m.s_off[b][own]];
      raw_scale[1] = s.scales[m.s_off[b][own] + (int64_t(1) << s.log2P)];
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int id = tid + kThreads * n, tok = id / (D / 8), piece = id % (D / 8);
        load_bytes<16>(raw_k + 4 * n, reinterpret_cast<const char*>(s.k_cache) + m.k_off[b][tok] + piece * 16);
      }
    }
    const char* values = kCodes ? reinterpret_cast<const char*>(s.codes) : reinterpret_cast<const char*>(s.v_cache);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const int tok = v_tokens / 4 * 32 + (n >> 2) * 16 + v_tokens % 4 * 4 + (n & 3);
      load_bytes<kVPiece>(raw_v[n], values + (kCodes ? m.v_off[b][tok] : m.k_off[b][tok]) + v_piece * kVPiece);
    }
  };
  // Into LDS.  The 16 tokens of a 16-bit key operand and the 16 rows of a value operand are permuted so that the threads
  // of a write, which hold one token's channels or neighbouring channels, reach all banks.
  auto k_place = [](int u, int i, int cc, int token) {
    return (u * kPairs + i) * kOperand + cc * 16 + (token ^ (kCodes ? 0 : (4 * i + cc) & 15));
  };
  auto v_place = [](int p, int j, int cc, int row) {
    return (p * kChannels + j) * kOperand + cc * 16 + (row ^ (j / 4 * (32 / kChannels)));
  };
  auto seen = [&](int32_t t, bool is) { return is && t <= span.hi_most && (t > span.lo_least || t < a.sinks); };
  auto put_tile = [&](int32_t it) {
    const int b = it & 1;
    // Values (scales) of tokens that no row of the workgroup sees are zero, whatever lies there.
    const int32_t t0 = tile_at<kManyTokens>(span, it);
    const uint64_t there[2] = {m.there[it & 3][0], m.there[it & 3][1]};
    if constexpr (kCodes) {
#pragma unroll
      for (int cc = 0; cc < 4; ++cc)
        m.k[b][k_place(k_token / 16, k_step, cc, k_token % 16)] = k_operand<KB>(code, raw_k, cc);
      if (!seen(t0 + own, (there[own >> 6] >> (own & 63)) & 1)) raw_scale[1] = 0;
      const float ks = f16_float(raw_scale[0]), vs = f16_float(raw_scale[1]);
      m.scale[b][0][own / 4][own % 4] = ks;
      m.scale[b][1][own / 4][own % 4] = f16_float(raw_scale[0] >> 16);
      m.scale[b][2][own / 4][own % 4] = vs;
      m.scale[b][3][own / 4][own % 4] = __builtin_fmaf(vs, float(1 << (VB - 1)), f16_float(raw_scale[1] >> 16));
    } else {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int id = tid + kThreads * n, tok = id / (D / 8), piece = id % (D / 8);
        m.k[b][k_place(tok / 16, piece / 4, piece % 4, tok % 16)] =
            u32x4{raw_k[4 * n], raw_k[4 * n + 1], raw_k[4 * n + 2], raw_k[4 * n + 3]};
      }
    }
    if constexpr (!kCodes) {
      constexpr uint64_t kAll = kManyTokens < 64 ? (uint64_t(1) << (kManyTokens & 63)) - 1 : ~uint64_t(0);
      const bool whole = t0 + kManyTokens - 1 <= span.hi_most && (t0 > span.lo_least || t0 + kManyTokens <= a.sinks) &&
                         (there[0] & there[1] & kAll) == kAll;
      if (!__builtin_amdgcn_readfirstlane(whole)) {
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const int tok = v_tokens / 4 * 32 + (n >> 2) * 16 + v_tokens % 4 * 4 + (n & 3);
          const bool keep = seen(t0 + tok, (there[tok >> 6] >> (tok & 63)) & 1);
#pragma unroll
          for (uint32_t& w : raw_v[n]) w = keep ? w : 0;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int channel = 4 * v_piece + e;
      u32x4 w;
#pragma unroll
      for (int n = 0; n < 4; ++n) w[n] = v_pair<VB>(code, raw_v[2 * n], raw_v[2 * n + 1], e);
      m.v[b][v_place(v_tokens / 4, channel % kChannels, v_tokens % 4, channel / kChannels)] = w;
    }
  };

  Running<RT> st;
  begin(st);
  if (from < upto) {
    put_places(from, entry_of(from));
    __syncthreads();
    bring(from);
    if (from + 1 < upto) put_places(from + 1, entry_of(from + 1));
    put_tile(from);
    __syncthreads();
    uint64_t there[2] = {m.there[from & 3][0], m.there[from & 3][1]};
    for (int32_t it = from; it < upto; ++it) {
      const int b = it & 1;
      const uint64_t there_next[2] = {m.there[(it + 1) & 3][0], m.there[(it + 1) & 3][1]};  // (of nothing behind the last)
      const bool more = it + 1 < upto, later = it + 2 < upto;
      if (more) bring(it + 1);
      int32_t entry = later ? entry_of(it + 2) : -1;
      const int32_t t0 = tile_at<kManyTokens>(span, it);
#pragma unroll
      for (int p = 0; p < kManyTokens / 32; ++p) {
        const int32_t t = t0 + 32 * p;
        if (t > mine.hi_most || (t + 31 <= mine.lo_least && t >= a.sinks)) continue;  // no row of this wave sees it
        const uint32_t word = uint32_t(there[p >> 1] >> (32 * (p & 1)));
        const uint32_t there = ((word >> (4 * c)) & 0xF) | (((word >> (16 + 4 * c)) & 0xF) << 4);
        FloatScales sc;
        if constexpr (kCodes) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int at = 8 * p + 4 * u + c;
            sc.ks_[u] = m.scale[b][0][at];
            sc.kz_[u] = m.scale[b][1][at];
          }
        }
        attend_tile<BF16, KB, VB, RT>(
            a, mine, rows, c, t, there, sc, st, [&](int u, int i) { return m.k[b][k_place(2 * p + u, i, c, x)]; },
            [&](int j) { return m.v[b][v_place(p, j, c, x)]; },
            [&] {
              if constexpr (kCodes) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                  sc.vs_[u] = m.scale[b][2][8 * p + 4 * u + c];
                  sc.vz_[u] = m.scale[b][3][8 * p + 4 * u + c];
                }
              }
            },
            [](const u32x4&) {});
      }
      // What was loaded is first looked at here, behind the whole tile's work.
#pragma unroll
      for (uint32_t& w : raw_k) asm volatile("" : "+v"(w));
#pragma unroll
      for (auto& row : raw_v)
#pragma unroll
        for (uint32_t& w : row) asm volatile("" : "+v"(w));
      if constexpr (kCodes) asm volatile("" : "+v"(raw_scale[0]), "+v"(raw_scale[1]));
      asm volatile("" : "+v"(entry));
      if (more) put_tile(it + 1);
      if (later) put_places(it + 2, entry);
      there[0] = there_next[0];
      there[1] = there_next[1];
      __syncthreads();
    }
  }

  // Every row's sums are one wave's.
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = over_c_sum(st.l[r]);
    const float o_zero = kCodes ? over_c_sum(st.o_zero[r]) : 0.0f;
    const uint32_t row = row0 + kRowTile * r + x;
    const int32_t token = int32_t(row / uint32_t(a.group)), out_head = g.head * a.group + int32_t(row % uint32_t(a.group));
    if (token >= g.count) continue;
    const int64_t flat = int64_t(g.start + token) * a.Hq + out_head;
    if (a.splits > 1) {
      const int64_t slot = flat * a.splits + g.split;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kChannels; j += 4) {
          f32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = st.o[r][j + e][i] + o_zero;
          *reinterpret_cast<f32x4*>(a.part + slot * D + (4 * c + i) * kChannels + j) = w;
        }
      if (c == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * slot) = f32x2{st.ref[r], l};
      continue;
    }
    // (A row that sees nothing has 0 times the values that others see, and those may be infinite.)
    const float inv = inverse(l);
    uint16_t* to = a.out + int64_t(g.start + token) * a.out_token_stride + int64_t(out_head) * a.out_head_stride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kChannels; j += 4) {
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = l == 0.0f ? 0.0f : (st.o[r][j + e][i] + o_zero) * inv;
        *reinterpret_cast<u32x2*>(to + (4 * c + i) * kChannels + j) =
            s.bf16 ? u32x2{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])} : u32x2{pack_f16(w[0], w[1]), pack_f16(w[2], w[3])};
      }
    if (a.lse && c == 0) a.lse[flat] = lse_of(st.ref[r], l);
  }
}

// Joins the parts of a row, by GROUPS groups of D / 4 threads, each with every GROUPS-th part; part i is at slot(i).
// (One group to a row needs no exchange; a workgroup of them takes as many rows as it has groups.)
template <int GROUPS, typename Slot>
__device__ __forceinline__ void join_parts(const ServeArgs& s, const AttendArgs& a, int32_t token, int32_t head,
                                           int32_t parts, Slot slot) {
  constexpr int kLanes = D / 4;
  static_assert(GROUPS == 1 || GROUPS * kLanes == kThreads, "a workgroup or a group");
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml);
  const f32x4* part = reinterpret_cast<const f32x4*>(a.part);
  const int group = GROUPS == 1 ? 0 : threadIdx.x / kLanes, at = threadIdx.x % kLanes;
  float m = -kInf;
  if constexpr (GROUPS == 1) {
#pragma unroll 4
    for (int i = 0; i < parts; ++i) m = __builtin_fmaxf(m, ml[slot(i)][0]);
  } else {
    __shared__ float wave_most[kWaves];
    for (int i = threadIdx.x; i < parts; i += kThreads) m = __builtin_fmaxf(m, ml[slot(i)][0]);
    for (int off = 1; off < 64; off <<= 1) m = __builtin_fmaxf(m, __shfl_xor(m, off));
    if ((threadIdx.x & 63) == 0) wave_most[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = __builtin_fmaxf(m, wave_most[w]);
  }
  float l = 0.0f;
  f32x4 sum{};
#pragma unroll 4
  for (int i = group; i < parts; i += GROUPS) {
    const int64_t from = slot(i);
    const f32x2 w = ml[from];
    const f32x4 p = part[from * kLanes + at];
    // A part that saw nothing has sums of nothing in particular.
    const float scale = w[1] == 0.0f ? 0.0f : exp2_of(w[0] - m);
    l += w[1] * scale;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += w[1] == 0.0f ? 0.0f : p[e] * scale;
  }
  if constexpr (GROUPS > 1) {
    __shared__ f32x4 sums[GROUPS][kLanes];
    __shared__ float totals[GROUPS];
    sums[group][at] = sum;
    if (at == 0) totals[group] = l;
    __syncthreads();
    if (group) return;
    l = 0.0f;
    sum = f32x4{};
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      l += totals[i];
      sum += sums[i][at];
    }
  }
  const float inv = inverse(l);
  uint16_t* to = a.out + token * a.out_token_stride + head * a.out_head_stride + 4 * at;
  sum *= inv;
  *reinterpret_cast<u32x2*>(to) = s.bf16 ? u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])}
                                         : u32x2{pack_f16(sum[0], sum[1]), pack_f16(sum[2], sum[3])};
  if (a.lse && at == 0) a.lse[int64_t(token) * a.Hq + head] = lse_of(m, l);
}

constexpr int kJoinGroups = kThreads / (D / 4);
constexpr int kFewSplits = 16;
constexpr int kManyJoins = 1024;

// The splits of each row of a call of many rows: a row to a workgroup, or, where there are few splits (a workgroup to a
// row then costs 1 ns of launching each and does little), to a group of its threads: 39328 rows of 4 splits 16 us instead
// of 40; 40 rows of 20 splits 5.7 instead of 4.6.
template <int GROUPS>
__global__ __launch_bounds__(kThreads) void join_splits_kernel(ServeArgs s, AttendArgs a) {
  const uint32_t row = GROUPS == 1 ? blockIdx.x * kJoinGroups + threadIdx.x / (D / 4) : blockIdx.x;
  const int32_t token = int32_t(row / uint32_t(a.Hq)), head = int32_t(row % uint32_t(a.Hq));
  // Rows of no sequence have no parts, and neither have a sequence's rows past max_tokens.
  if (token < scalar_entry(s.token_start, 0) || token >= scalar_entry(s.token_start, s.num_seqs)) return;
  if (token >= s.num_tokens) return;
  if (s.max_tokens < s.num_tokens) {
    int32_t seq = 0;
    for (int32_t end = s.num_seqs; end - seq > 1;) {
      const int32_t mid = seq + (end - seq) / 2;
      if (s.token_start[mid] <= token) seq = mid; else end = mid;
    }
    const Group g = group_from(s, s.token_start[seq], s.token_start[seq + 1], 0);
    if (token >= g.start + g.count) return;
  }
  const int64_t first = int64_t(row) * a.splits;
  join_parts<GROUPS>(s, a, token, head, a.splits, [&](int i) { return first + i; });
}

// The pieces of a sequence of few rows, a row to a workgroup or, where there are many rows, to a group of its threads (of
// one token's heads): 8192 rows 9.6 us instead of 33, 1024 rows 7.2 instead of 8.0, 256 rows either 4.6.  A
// sequence of one piece is done.
template <int GROUPS>
__global__ __launch_bounds__(kThreads) void join_pieces_kernel(ServeArgs s, AttendArgs a) {
  const int lane = threadIdx.x & 63;
  constexpr int kHeads = GROUPS == 1 ? kJoinGroups : 1;
  const uint32_t shares = (uint32_t(a.Hq) + kHeads - 1) / kHeads;
  const int32_t token = int32_t(blockIdx.x / shares);
  const int32_t head = int32_t(blockIdx.x % shares) * kHeads + (GROUPS == 1 ? threadIdx.x / (D / 4) : 0);
  const int32_t mine = tiles_of_sequence(s, a, lane), per = piece_tiles(s, a, lane, mine);
  const Found at = find_sequence(s, a, lane, mine, per, [&](int32_t seq, int32_t, int32_t own) {
    if (own == 0) return false;
    const Group g = group_from(s, s.token_start[seq], s.token_start[seq + 1], s.kv_lens[seq]);
    return token >= g.start && token < g.start + g.count;
  });
  if (at.seq < 0) return;
  const int32_t pieces = pieces_of(at.tiles, per);
  if (pieces == 1 || head >= a.Hq) return;
  const int32_t start = scalar_entry(s.token_start, at.seq);
  const int32_t row = (token - (start < 0 ? 0 : start)) * a.group + head % a.group;
  join_parts<GROUPS>(s, a, token, head, pieces, [&](int i) {
    return (int64_t(at.before + i) * s.H + head / a.group) * a.part_rows + row;
  });
}

}  // namespace

#define PKV_JOINED2(a, b) a##b
#define PKV_JOINED(a, b) PKV_JOINED2(a, b)

pkv_status_t PKV_JOINED(launch_attend_, PKV_HEAD_DIM)(const ServeArgs& s, const AttendArgs& a, int64_t groups,
                                                      hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(uint32_t(groups)), dim3(kThreads), 0, stream, s, a); };
  auto few = [&](auto whole, auto tiles) {
    constexpr bool kWhole = decltype(whole)::value;
    constexpr int kTiles = decltype(tiles)::value;
    switch (s.tag) {
      case PKV_TAG_FP16:
        s.bf16 ? go(attend_few_kernel<true, 16, 16, kWhole, kTiles>) : go(attend_few_kernel<false, 16, 16, kWhole, kTiles>);
        break;
      case PKV_TAG_K8V8:
        s.bf16 ? go(attend_few_kernel<true, 8, 8, kWhole, kTiles>)
               : go(attend_few_kernel<false, 8, 8, kWhole, kTiles>);
        break;
      case PKV_TAG_K8V4:
        s.bf16 ? go(attend_few_kernel<true, 8, 4, kWhole, kTiles>)
               : go(attend_few_kernel<false, 8, 4, kWhole, kTiles>);
        break;
      default: s.bf16 ? go(attend_few_kernel<true, 4, 4, kWhole, kTiles>) : go(attend_few_kernel<false, 4, 4, kWhole, kTiles>); break;
    }
  };
  auto few_of = [&](auto whole) {
    a.tiles == 1 ? few(whole, std::integral_constant<int, 1>{}) : few(whole, std::integral_constant<int, few_tiles(D)>{});
  };
  if (a.tiles > few_tiles(D)) {
    switch (s.tag) {
      case PKV_TAG_FP16: s.bf16 ? go(attend_many_kernel<true, 16, 16>) : go(attend_many_kernel<false, 16, 16>); break;
      case PKV_TAG_K8V8: s.bf16 ? go(attend_many_kernel<true, 8, 8>) : go(attend_many_kernel<false, 8, 8>); break;
      case PKV_TAG_K8V4: s.bf16 ? go(attend_many_kernel<true, 8, 4>) : go(attend_many_kernel<false, 8, 4>); break;
      default: s.bf16 ? go(attend_many_kernel<true, 4, 4>) : go(attend_many_kernel<false, 4, 4>); break;
    }
  } else {
    s.log2P >= 4 ? few_of(std::true_type{}) : few_of(std::false_type{});
  }
  if (hipGetLastError() != hipSuccess) return PKV_ERR_DEVICE;
  const dim3 rows(uint32_t(s.num_tokens) * uint32_t(a.Hq));
  if (a.pieces && int32_t(rows.x) >= kManyJoins && a.pieces <= int64_t(kFewSplits) * s.num_seqs)
    hipLaunchKernelGGL(join_pieces_kernel<1>, dim3(uint32_t(s.num_tokens) * ((uint32_t(a.Hq) + kJoinGroups - 1) / kJoinGroups)),
                       dim3(kThreads), 0, stream, s, a);
  else if (a.pieces)
    hipLaunchKernelGGL(join_pieces_kernel<kJoinGroups>, rows, dim3(kThreads), 0, stream, s, a);
  else if (a.splits > kFewSplits)
    hipLaunchKernelGGL(join_splits_kernel<kJoinGroups>, rows, dim3(kThreads), 0, stream, s, a);
  else if (a.splits > 1)
    hipLaunchKernelGGL(join_splits_kernel<1>, dim3((rows.x + kJoinGroups - 1) / kJoinGroups), dim3(kThreads), 0, stream, s,
                       a);
  if (hipGetLastError() != hipSuccess) return PKV_ERR_DEVICE;
  return PKV_OK;
}

}  // namespace pkv
