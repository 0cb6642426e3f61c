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
//
// Few rows wait for the cache's bytes, in 16 bits for nothing else (32 sequences of 8192 tokens, 8 heads of 128, 537 MB: 101 us,
// 5.3 TB/s, where a large copy reaches 5.3); over codes the vector units decode them as well (32 ragged sequences of 255 thousand
// tokens in 4 bits, 141 MB: 53 to 55 us, 2.6 TB/s, vector units busy 42% of the launch).  Many rows share
// their time between the matrix units and the exponentials: 8192 rows of 32 heads over 8192 tokens of 16 bits take 29 us to
// prepare and 335 to 345 to weigh (275 GFLOP that the mask leaves, 810 TFLOP/s; a large library product reaches 1218), vector units
// busy 51% and matrix units 37% of it, of which the last workgroups' end is a fifth.  A wave's own instructions of both kinds,
// taken in turn, run one behind the other (430 us with three waves a SIMD); through LDS with a barrier for each tile of rows 502.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pkv.h"
#include "paged_tiles.h"
#include "pkv_internal.h"
#include "serve.h"

namespace pkv {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// A sequence's rows, from what the device holds.
__device__ __forceinline__ SequenceRows sequence_rows(const ServeArgs& s, int32_t seq) {
  return rows_of_sequence(s, scalar_entry(s.token_start, seq), scalar_entry(s.token_start, seq + 1),
                          scalar_entry(s.kv_lens, seq));
}

// over_c_sum by lane swaps.
__device__ __forceinline__ float over_c_add(float v) {
  u32x2 w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}

// What a row at position `pos` sees.
__device__ __forceinline__ Sight sight_at(const WeighArgs& a, const SequenceRows& g, int32_t pos) {
  Sight see;
  see.hi = pos < g.kv_len ? pos : g.kv_len - 1;
  see.hi = see.hi < -1 ? -1 : see.hi;
  see.lo = a.window > 0 && pos >= a.window ? pos - a.window : -1;
  return see;
}

__device__ __forceinline__ Sight sight_of(const ServeArgs& s, const WeighArgs& a, const SequenceRows& g, int32_t token) {
  return sight_at(a, g, s.positions ? s.positions[g.start + token] : g.kv_len - g.trail + token);
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
// tokens.  A workgroup takes tokens of one sequence and all heads: wave w the w % subs-th part of them, of heads w / subs and
// on.  Where heads are joined, the waves' sums of a token meet in LDS.  All sequences' tokens are cut into even shares, one to a
// workgroup, so that the GPU is done at once whatever their lengths; with a window, of whose tokens most are not looked at, into
// chunks.

// Tokens [begin, end) of one sequence (end at most kv_len), by the whole workgroup.
template <bool BF16, int KB, bool WHOLE, int RT>
__device__ __forceinline__ void weigh_tokens(const ServeArgs& s, const WeighArgs& a, float (*sums)[kMostChunk],
                                             const SequenceRows& g, int32_t seq, int32_t begin, int32_t end) {
  constexpr bool kCodes = KB != 16;
  constexpr bool kHalf = kCodes || !BF16;
  constexpr int kSteps = D / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane >> 4, x = lane & 15;
  const int32_t each = kTokenTile * a.subs, part = (end - begin + each - 1) / each * kTokenTile;
  const int32_t sub = wave % a.subs, first_head = wave / a.subs, heads = kFewWaves / a.subs;
  const int32_t from = begin + sub * part;
  const int32_t upto = end - from < part ? end : from + part;
  const Magic m = magic();
  if (a.joint) {
    for (int32_t i = lane; i < part; i += 64) sums[wave][i] = 0.0f;
    __syncthreads();
  }

  // What the rows see between them: tiles of which none sees anything are not looked at, and of which all see everything need
  // no masks.
  int32_t hi_most = -1, lo_least = 0x7FFFFFFF, hi_least = 0x7FFFFFFF, lo_most = -1;
  if (g.count > 0 && !s.positions) {
    const Sight begins = sight_of(s, a, g, 0), ends = sight_of(s, a, g, g.count - 1);
    hi_least = begins.hi, lo_least = begins.lo, hi_most = ends.hi, lo_most = ends.lo;
  } else if (s.positions) {
    for (int32_t i = lane; i < g.count; i += 64) {
      const Sight see = sight_of(s, a, g, i);
      hi_most = max(hi_most, see.hi);
      hi_least = min(hi_least, see.hi);
      lo_most = max(lo_most, see.lo);
      if (see.hi >= 0) lo_least = min(lo_least, see.lo);
    }
    for (int off = 1; off < 64; off <<= 1) {
      hi_most = max(hi_most, __shfl_xor(hi_most, off));
      hi_least = min(hi_least, __shfl_xor(hi_least, off));
      lo_most = max(lo_most, __shfl_xor(lo_most, off));
      lo_least = min(lo_least, __shfl_xor(lo_least, off));
    }
  }
  hi_most = __builtin_amdgcn_readfirstlane(hi_most);
  hi_least = __builtin_amdgcn_readfirstlane(hi_least);
  lo_most = __builtin_amdgcn_readfirstlane(lo_most);
  lo_least = __builtin_amdgcn_readfirstlane(lo_least);
  auto seen = [&](int32_t t0) { return t0 <= hi_most && (t0 + kTokenTile - 1 > lo_least || t0 < a.sinks); };
  auto open = [&](int32_t t0) {
    const int32_t end = t0 + kTokenTile - 1;
    return end <= hi_least && (lo_most < t0 || end < a.sinks);
  };

  // The pages of the wave's part, a half of a tile to a lane, so that no load waits for its page.
  static_assert(kMostChunk <= 64 * 16, "a lane each");
  int32_t pages = -1;
  if constexpr (WHOLE) {
    if (from + 16 * lane < upto) pages = page_of(s, s.page_table + int64_t(seq) * s.pages_per_seq, (from + 16 * lane) >> s.log2P);
  }

  for (int32_t head = first_head; head < s.H && from < upto; head += heads) {
    const Source src = source_of<KB>(s, seq, head);
    constexpr int kTiles = KB * D > 2048 ? 1 : 2;  // on their way while one is used, as registers allow
    Keys<KB> keys[kTiles];
    uint32_t words[kTiles][2];
    bool there[kTiles][2];
    auto load = [&](int b, int32_t t0) {
      if (t0 >= upto || !seen(t0)) return;
      Tile tile{t0, {-1, -1}};
      if constexpr (WHOLE) {
#pragma unroll
        for (int u = 0; u < 2; ++u) tile.page[u] = __builtin_amdgcn_readlane(pages, (t0 - from) / 16 + u);
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
#pragma unroll
    for (int b = 0; b < kTiles; ++b) load(b, from + b * kTokenTile);

    // Row x of each row tile: its queries, and what it is scaled by.
    bool plain = true;  // no row with a mask of its own
    u32x4 q[RT][kSteps];
    f32x4 f[RT], less[RT], sum[RT];
    Sight see[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int32_t row = 16 * r + x, token = row / a.group, qhead = head * a.group + row % a.group;
      const bool on = token < g.count;
      see[r] = Sight{-1, -1};
      RowScale rs{a.scale, -kInf, 0.0f};
      if (on) {
        rs.less = less_of(a, g, token, qhead);
        if (rs.less != -kInf) see[r] = sight_of(s, a, g, token);
        else plain = false;
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
      }
    }

    plain = __all(plain);
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
        load(b, t0 + kTiles * kTokenTile);
        // (Rows past the last have less = -inf and queries of 0, and add nothing.)
        auto sums_of = [&](auto masked) {
          constexpr bool kMasked = decltype(masked)::value;
          int32_t hi[RT][4], lo[RT][4];
          if constexpr (kMasked) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                hi[r][i] = __shfl(see[r].hi, 4 * c + i);
                lo[r][i] = __shfl(see[r].lo, 4 * c + i);
              }
          }
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
                float p = exp2_of(__builtin_fmaf(t, f[r][i], less[r][i]));
                if constexpr (kMasked) p = (tok <= hi[r][i]) & ((tok > lo[r][i]) | sink) ? p : 0.0f;
                total += p;
              }
            w[u] = over_c_add(total);
            if (!is[u]) w[u] = 0.0f;
          }
        };
        bool sure = open(t0) && plain;
        if (sure) {
          sums_of(std::false_type{});
          // 0 times an infinite key is NaN: where there is one, the sums are worked out again without the rows past the last.
          // (Without a cost that shows; those rows left out by a select each took 1 us more of 51, 2.7 of 84 with two tiles.)
          sure = !__any(__builtin_isunordered(w[0], w[1]));
        }
        if (!sure) sums_of(std::true_type{});
      } else {
        load(b, t0 + kTiles * kTokenTile);
      }
      const int32_t tok = t0 + (lane & 31);
      if (lane < 32 && tok < upto) {
        const float mine = lane & 16 ? w[1] : w[0];
        if (a.joint) sums[wave][tok - from] += mine;
        else put(a, int64_t(seq) * a.seq_stride + int64_t(head) * a.head_stride + tok, mine);
      }
    };
    for (int32_t t0 = from; t0 < upto; t0 += kTiles * kTokenTile) {
#pragma unroll
      for (int b = 0; b < kTiles; ++b)
        if (t0 + b * kTokenTile < upto) weigh(b, t0 + b * kTokenTile);
    }
  }
  if (!a.joint) return;
  __syncthreads();
  for (int32_t i = threadIdx.x; i < end - begin; i += 64 * kFewWaves) {
    const int32_t tok = begin + i;
    float total = 0.0f;
    for (int32_t w = i / part; w < kFewWaves; w += a.subs) total += sums[w][i % part];
    put(a, int64_t(seq) * a.seq_stride + tok, total);
  }
  __syncthreads();
}

__device__ __forceinline__ int32_t token_tiles(const ServeArgs& s, int32_t seq) {
  if (seq >= s.num_seqs) return 0;
  const int32_t len = s.kv_lens[seq];
  return ((len < 0 ? 0 : len < s.max_kv ? len : s.max_kv) + kTokenTile - 1) / kTokenTile;
}

// Inclusive sums over the lanes of a wave.
__device__ __forceinline__ int64_t wave_sums(int64_t v, int lane) {
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t other = __shfl_up(v, off);
    v += lane >= off ? other : 0;
  }
  return v;
}

template <bool BF16, int KB, bool WHOLE, int RT>
__global__ __launch_bounds__(64 * kFewWaves, WHOLE && RT == 1 && KB * D <= 512 ? 3 : 2) void few_kernel(ServeArgs s, WeighArgs a) {
  __shared__ float sums[kFewWaves][kMostChunk];
  const int lane = threadIdx.x & 63;
  int32_t seq = 0, tile = 0, left = 0;  // the workgroup's first sequence, its first tile there, and its tiles
  if (a.chunk) {  // a chunk of one sequence
    seq = int32_t(blockIdx.x / uint32_t(a.tiles));
    tile = int32_t(blockIdx.x % uint32_t(a.tiles)) * (a.chunk / kTokenTile);
    const int32_t rest = token_tiles(s, seq) - tile;
    left = rest < a.chunk / kTokenTile ? rest : a.chunk / kTokenTile;
  } else {  // an even share of all sequences' tiles, whose number only the device knows
    int64_t all = 0;
    for (int32_t s0 = 0; s0 < s.num_seqs; s0 += 64) all += __shfl(wave_sums(token_tiles(s, s0 + lane), lane), 63);
    const int64_t step = int64_t(gridDim.x) * a.subs, share = (all + step - 1) / step * a.subs;
    int64_t at = share * blockIdx.x;
    for (int32_t s0 = 0; s0 < s.num_seqs; s0 += 64) {
      const int32_t mine = token_tiles(s, s0 + lane);
      const int64_t upto = wave_sums(mine, lane), here = __shfl(upto, 63);
      if (at < here) {
        const int which = __builtin_ctzll(__ballot(upto > at));
        seq = s0 + which;
        tile = int32_t(at - __shfl(upto - mine, which));
        left = int32_t(share < (int64_t(1) << 30) ? share : int64_t(1) << 30);
        break;
      }
      at -= here;
    }
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  tile = __builtin_amdgcn_readfirstlane(tile);
  left = __builtin_amdgcn_readfirstlane(left);
  for (; left > 0 && seq < s.num_seqs; ++seq, tile = 0) {
    const SequenceRows g = sequence_rows(s, seq);
    int32_t tiles = (g.kv_len + kTokenTile - 1) / kTokenTile - tile;
    tiles = tiles < left ? tiles : left;
    left -= tiles;
    while (tiles > 0) {
      const int32_t most = kMostChunk / kTokenTile * a.subs, now = tiles < most ? tiles : most;  // what the waves' parts hold
      const int32_t begin = tile * kTokenTile, end = begin + now * kTokenTile;
      weigh_tokens<BF16, KB, WHOLE, RT>(s, a, sums, g, seq, begin, end < g.kv_len ? end : g.kv_len);
      tile += now;
      tiles -= now;
    }
  }
}

// ---- Many rows ----
//
// Every row is used by all the tokens that it sees, so the rows are prepared once: their queries in the order of the matrix
// operands, 32 rows to a tile, what they are scaled by and what they see.  Then every wave keeps the keys of 32 * kNT tokens
// of one sequence and KV head in registers and goes over the tiles, a tile ahead of use loaded straight to registers as they
// lie (the four waves of a workgroup find them in L1 after the first of them; through LDS the barrier of every tile cost more
// than the loads).  While the exponentials of some scores are worked out the matrix units work on the next ones.

constexpr int kThreads = 256;
constexpr int kNT = D > 128 ? 1 : 2;  // token tiles of 32 of a wave
constexpr int kRows = kWeighRows;
constexpr int kRowPieces = D / 8;
constexpr int kQueries = 2 * D / 16 * kRows;  // pieces of 8 channels of a tile

// Which operand the 8 channels from `channel` on are part of (2 * step + lane half), with lanes that load pieces of up to 16
// bytes of keys.
template <int BITS>
struct Halves {
  static constexpr int kBytes = D / 2 * BITS / 8 < 16 ? D / 2 * BITS / 8 : 16, kPer = kBytes * 8 / BITS, kOps = kPer / 8;
  static constexpr int kPieces = D / 2 * BITS / 8 / kBytes;
  static __device__ constexpr int slot(int channel) {
    const int piece = channel / kPer, step = piece / 2 * kOps + channel % kPer / 8;
    return 2 * step + (piece & 1);
  }
};

struct RowNumbers {
  float less[kRows];
  // Whether some row gives nothing; least and most of hi, most and least of lo.
  int32_t off, all_hi, any_hi, all_lo, any_lo, unused[3];
  float f[kRows], sum[kRows];
  int32_t hi[kRows], lo[kRows];
};
struct RowTile {
  u32x4 q[kQueries];  // [step][half][row]
  RowNumbers row;
};
static_assert(sizeof(RowTile) == weigh_tile_bytes(D), "the workspace's tiles");

// The first tile of a sequence: sequences' tiles do not meet, since each has at most one that is not full.
__device__ __forceinline__ int64_t first_tile(const WeighArgs& a, const SequenceRows& g, int32_t seq) {
  return int64_t(g.start) * a.group / kRows + seq;
}

template <int KB>
__global__ __launch_bounds__(kThreads) void prepare_kernel(ServeArgs s, WeighArgs a) {
  constexpr bool kCodes = KB != 16;
  const int tid = threadIdx.x;
  uint32_t b = blockIdx.x;
  const int32_t head = int32_t(b % uint32_t(s.H));
  b /= uint32_t(s.H);
  const int32_t tile = int32_t(b % uint32_t(a.row_tiles)), seq = int32_t(b / uint32_t(a.row_tiles));
  const SequenceRows g = sequence_rows(s, seq);
  const int32_t row_first = tile * kRows, rows = g.count * a.group;  // (below 2^31: num_tokens * Hq)
  if (row_first >= rows) return;
  RowTile& to = static_cast<RowTile*>(a.rows)[head * a.all_tiles + first_tile(a, g, seq) + tile];
  const int piece = tid % kRowPieces;
  for (int row = tid / kRowPieces; row < kRows; row += kThreads / kRowPieces) {
    const uint32_t at = uint32_t(row_first + row), token = at / uint32_t(a.group), sub = at % uint32_t(a.group);
    u32x4 w{};
    if (int32_t(at) < rows)
      w = *reinterpret_cast<const u32x4*>(a.q + int64_t(g.start + token) * a.q_token_stride +
                                          int64_t(head * a.group + sub) * a.q_head_stride + 8 * piece);
    if constexpr (kCodes) {
      float v[8], down, up, sum = 0.0f;
      uint32_t top = 0;
      widen(s.bf16, w, v);
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
      w = query_operand<KB>(v, down);
      if (piece == 0) {
        to.row.f[row] = a.scale * up;
        to.row.sum[row] = sum;
      }
    }
    to.q[Halves<KB>::slot(8 * piece) * kRows + row] = w;
  }
  if (tid < kRows) {
    const uint32_t at = uint32_t(row_first + tid), token = at / uint32_t(a.group), sub = at % uint32_t(a.group);
    float less = -kInf;
    Sight see{-1, -1};
    if (int32_t(at) < rows) {
      less = less_of(a, g, int32_t(token), head * a.group + int32_t(sub));
      if constexpr (!kCodes) less /= a.scale;  // (in the scores' unit)
      if (less != -kInf) see = sight_of(s, a, g, int32_t(token));  // else it saw nothing, and gives nothing
    }
    to.row.less[tid] = less;
    to.row.hi[tid] = see.hi;
    to.row.lo[tid] = see.lo;
    int32_t all_hi = see.hi, any_hi = see.hi, all_lo = see.lo, any_lo = see.hi < 0 ? 0x7FFFFFFF : see.lo;
    for (int by = 1; by < kRows; by <<= 1) {
      all_hi = min(all_hi, __shfl_xor(all_hi, by));
      any_hi = max(any_hi, __shfl_xor(any_hi, by));
      all_lo = max(all_lo, __shfl_xor(all_lo, by));
      any_lo = min(any_lo, __shfl_xor(any_lo, by));
    }
    if (tid == 0) {
      to.row.off = all_hi < 0;
      to.row.all_hi = all_hi;
      to.row.any_hi = any_hi;
      to.row.all_lo = all_lo;
      to.row.any_lo = any_lo;
    }
  }
}

template <bool BF16, int KB>
__global__ __launch_bounds__(kThreads, 2) void many_kernel(ServeArgs s, WeighArgs a) {
  constexpr bool kCodes = KB != 16;
  constexpr bool kHalf = kCodes || !BF16;
  constexpr int kSteps = D / 16, kNumbers = kCodes ? 3 : 1;
  typedef Halves<KB> Order;
  __shared__ float lds[kThreads / 64][2][kNumbers][kRows];  // rows' numbers, each wave its own
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
  // A split is the same rows for all tiles of tokens, whose workgroups run side by side and find them in L2.
  const int64_t every = (int64_t(g.count > 0 ? g.count : 0) * a.group + kRows - 1) / kRows;
  const int64_t begin_split = every * split / a.splits, end_split = every * (split + 1) / a.splits;
  int32_t from = int32_t(tile0 > begin_split ? tile0 : begin_split);
  int32_t upto = int32_t(tile0 + tiles < end_split ? tile0 + tiles : end_split);

  // A tile in registers: its queries and row n's numbers (other half: of all rows).  Past the last tile it is that one again.
  struct Loaded {
    u32x4 q[kSteps];
    float number[kNumbers];
  };
  const RowTile* tiles_of = static_cast<const RowTile*>(a.rows) + head * a.all_tiles + first_tile(a, g, seq);
  if (s.positions) {  // from the first tile of rows that sees one of the wave's tokens to the last one
    int32_t first = upto, end = from;
    for (int32_t t0 = from; t0 < upto; t0 += 64) {
      bool sees = false;
      if (t0 + lane < upto) {
        const RowNumbers& row = tiles_of[t0 + lane].row;
        sees = row.any_hi >= mine && (row.any_lo < mine + 32 * kNT - 1 || mine < a.sinks);
      }
      const uint64_t who = __ballot(sees);
      if (!who) continue;
      first = first < upto ? first : t0 + __builtin_ctzll(who);
      end = t0 + 64 - __builtin_clzll(who);
    }
    from = __builtin_amdgcn_readfirstlane(first);
    upto = __builtin_amdgcn_readfirstlane(end);
  }
  auto fetch_query = [&](int32_t at, int i, Loaded& to) {
    to.q[i] = tiles_of[at < upto ? at : upto - 1].q[64 * i + lane];
  };
  auto fetch_numbers = [&](int32_t at, Loaded& to) {
    const float* from = tiles_of[at < upto ? at : upto - 1].row.less;
    to.number[0] = from[half && n >= 8 ? n : lane];
#pragma unroll
    for (int i = 1; i < kNumbers; ++i) to.number[i] = from[40 + kRows * (i - 1) + n];
  };
  auto fetch = [&](int32_t at, Loaded& to) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) fetch_query(at, i, to);
    fetch_numbers(at, to);
  };
  // The numbers where every lane finds those of its rows: value e of a lane's scores is row 8 (e / 4) + 4 half + e % 4.
  float(*numbers)[kNumbers][kRows] = lds[wave];
  auto leave = [&](const Loaded& in, int which) {
    if (half == 0) {
#pragma unroll
      for (int i = 0; i < kNumbers; ++i) numbers[which][i][n] = in.number[i];
    }
    __builtin_amdgcn_wave_barrier();
  };
  auto number = [&](int which, int i, int e4) {
    return *reinterpret_cast<const f32x4*>(&numbers[which][i][8 * e4 + 4 * half]);
  };

  float total[kNT] = {};
  // The scores of a tile and token tile t; `then(i)` after the i-th operand.  (16 bits: less the rows' lse in the scores' unit,
  // which the sums begin with.)
  auto begin_scores = [&](int which, f32x16& score) {
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      f32x4 v{};
      if constexpr (!kCodes) v = number(which, 0, e4);
#pragma unroll
      for (int e = 0; e < 4; ++e) score[4 * e4 + e] = v[e];
    }
  };
  auto scores = [&](const Loaded& r, auto t, f32x16& score, auto then) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      score = mfma32<kHalf>(r.q[i], k[t][i], score);
      then(i);
    }
  };
  auto nothing = [](int) {};
  // The sum of their exponentials.
  auto sum_of = [&](auto masked, int32_t at, int which, auto t, const f32x16& score) {
    constexpr bool kMasked = decltype(masked)::value;
    const int32_t tok = mine + 32 * t + n;
    const bool sink = tok < a.sinks;
    float part[4] = {};
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      f32x4 f, sum, ls;
      i32x4 hi, lo;
      if constexpr (kCodes) {
        ls = number(which, 0, e4);
        f = number(which, 1, e4);
        sum = number(which, 2, e4);
      }
      if constexpr (kMasked) {
        const RowNumbers& row = tiles_of[at].row;
        hi = *reinterpret_cast<const i32x4*>(&row.hi[8 * e4 + 4 * half]);
        lo = *reinterpret_cast<const i32x4*>(&row.lo[8 * e4 + 4 * half]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = score[4 * e4 + e];
        if constexpr (kCodes) x = __builtin_fmaf(__builtin_fmaf(ks[t], x, kz[t] * sum[e]), f[e], ls[e]);
        else x *= a.scale;
        float p = exp2_of(x);
        if constexpr (kMasked) p = (tok <= hi[e]) & ((tok > lo[e]) | sink) ? p : 0.0f;
        part[e] += p;
      }
    }
    return (part[0] + part[1]) + (part[2] + part[3]);
  };
  // The exponentials of one tile while the matrix units work on the next scores: a matrix instruction of 32 cycles, then the
  // vector instructions of as long.
  auto both = [&](bool all, bool none, int32_t at, int which, auto t, const f32x16& score, const Loaded& next, auto next_t,
                  f32x16& later, auto then) {
    scores(next, next_t, later, then);
    float sum = sum_of(std::false_type{}, at, which, t, score);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                 // matrix
      __builtin_amdgcn_sched_group_barrier(0x002, (kCodes ? 68 : 36) / kSteps + 1, 0);  // vector
    }
    asm("" : "+v"(sum));  // (here, beside the matrix instructions, not where it turns out to be of use)
    // (Masked they are worked out again: the matrix instructions stay in one place, where their results need no moves.)
    if (!all) sum = none ? 0.0f : sum_of(std::true_type{}, at, which, t, score);
    total[t] += sum;
  };
  constexpr std::integral_constant<int, 0> kFirst{};
  constexpr std::integral_constant<int, kNT - 1> kLast{};
  f32x16 score_a, score_b;
  // Tile `at` of parity `which`, in `r`, whose first scores are in `now`; the next one is in `next` (of 256 channels its queries
  // in `queries`).
  auto iterate = [&](int32_t at, int which, Loaded& r, Loaded& next, Loaded& queries, f32x16& now, f32x16& later) {
    const int32_t end = mine + 32 * kNT - 1;
    auto of_all = [&](int i) { return __builtin_amdgcn_readlane(__float_as_int(r.number[0]), 32 + i); };
    const int32_t off = of_all(0), all_hi = of_all(1), any_hi = of_all(2), all_lo = of_all(3), any_lo = of_all(4);
    const bool none = any_hi < mine || (any_lo >= end && mine >= a.sinks);
    const bool all = !off && all_hi >= end && (all_lo < mine || end < a.sinks);
    if constexpr (kNT == 2) {
      begin_scores(which, later);
      both(all, none, at, which, kFirst, now, r, kLast, later, nothing);
      fetch(at + 2, r);
      leave(next, which ^ 1);
      begin_scores(which ^ 1, now);
      both(all, none, at, which, kLast, later, next, kFirst, now, nothing);
    } else {
      leave(next, which ^ 1);
      begin_scores(which ^ 1, later);
      fetch_numbers(at + 2, r);
      both(all, none, at, which, kFirst, now, queries, kFirst, later, [&](int i) { fetch_query(at + 2, i, queries); });
    }
  };
  if (from < upto) {
    Loaded even, odd;
    fetch(from, even);
    leave(even, 0);
    begin_scores(0, score_a);
    if constexpr (kNT == 2) {
      fetch(from + 1, odd);
      scores(even, kFirst, score_a, nothing);
      // (After the last tile its scores are worked out again and not used.)
      for (int32_t at = from; at < upto; at += 2) {
        iterate(at, 0, even, odd, even, score_a, score_b);
        if (at + 1 < upto) iterate(at + 1, 1, odd, even, even, score_a, score_b);
      }
    } else {
      fetch_numbers(from + 1, odd);
      scores(even, kFirst, score_a, [&](int i) { fetch_query(from + 1, i, even); });
      for (int32_t at = from; at < upto; at += 2) {
        iterate(at, 0, even, odd, even, score_a, score_b);
        if (at + 1 < upto) iterate(at + 1, 1, odd, even, even, score_b, score_a);
      }
    }
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
  if (l.few_tiles) {
    const bool whole = s.log2P >= 4;
    if constexpr (D <= 128) {
      if (l.few_tiles > 1) {
        if (whole) few(few_kernel<BF16, KB, true, 2>);
        else few(few_kernel<BF16, KB, false, 2>);
        return;
      }
    }
    if (whole) few(few_kernel<BF16, KB, true, 1>);
    else few(few_kernel<BF16, KB, false, 1>);
    return;
  }
  if (l.prepare_groups)
    hipLaunchKernelGGL(prepare_kernel<KB>, dim3(uint32_t(l.prepare_groups)), dim3(kThreads), 0, stream, s, a);
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
